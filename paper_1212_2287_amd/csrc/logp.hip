// logp.hip -- log-probabilities of given tokens under the softmax of their logits, and the gradient
// with respect to the logits, on gfx950.
//
// With z = scale * (x - max x) and L = log sum exp z over a row: logp = z[target] - L and
// entropy = L - sum p z with p = exp(z - L). One pass over the row keeps a running maximum m with
// S = sum exp2(d) and W = sum exp2(d) d of d = log2(e) * scale * (x - m); when the maximum grows by
// delta (in units of d), S and W + delta S are scaled by exp2(delta).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "status.hpp"
#include "tree_ens.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;
constexpr int64_t kMaxBlocks = 1 << 20; // rows beyond this many are taken in turn
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// 16 bytes of logits. A row may start anywhere, so what it is read through claims no alignment.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef type unaligned __attribute__((aligned(sizeof(T))));
};

// Elements of `p` before the first 16-byte boundary.
template <typename T> __device__ __forceinline__ int lead_of(const T *p) {
    return int((16u - unsigned(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / int(sizeof(T));
}

// Running maximum m (of the logits as they are), S and W. NaN logits reach S and W, never m.
struct Running {
    float m, S, W;
};

// Scores below the maximum by more than this (in powers of two) are held here: exp2 is 0 there, and
// 0 times it is 0, where 0 times the -inf of a masked logit would be NaN. Its product with the sum of
// any row is a float.
constexpr float kFar = -1024.0f;

// log2(e) times the scale, for a scale of which it is no float the largest one: differences of logits, 0 among
// them, come out alike.
__device__ __forceinline__ float base2_of(float scale) { return fminf(scale * kLog2e, 3.402823466e38f); }

// m = -inf (nothing but masked logits so far) subtracts 0: their differences stay -inf.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

__device__ __forceinline__ void raise_to(Running &r, float m, float c) {
    const float delta = fmaxf((r.m - base_of(m)) * c, kFar);
    const float f = __builtin_amdgcn_exp2f(delta);
    r.W = f * fmaf(delta, r.S, r.W);
    r.S *= f;
    r.m = m;
}

__device__ __forceinline__ Running join(Running a, Running b, float c) {
    const float m = fmaxf(a.m, b.m);
    raise_to(a, m, c);
    raise_to(b, m, c);
    return {m, a.S + b.S, a.W + b.W};
}

// Adds N logits. Their own maximum comes first, so that S and W are rescaled once for all of them,
// and by the lanes whose maximum grows alone.
template <bool kEntropy, int N> __device__ __forceinline__ void add(Running &r, const float (&x)[N], float c) {
    float m = x[0];
#pragma unroll
    for (int i = 1; i < N; ++i)
        m = fmaxf(m, x[i]);
    if (m > r.m)
        raise_to(r, m, c);
    const float base = base_of(r.m);
    float s[2] = {0.0f, 0.0f}, w[2] = {0.0f, 0.0f};
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float d = (x[i] - base) * c, e = __builtin_amdgcn_exp2f(d);
        s[i & 1] += e;
        if (kEntropy)
            w[i & 1] = fmaf(e, fmaxf(d, kFar), w[i & 1]);
    }
    r.S += s[0] + s[1];
    r.W += w[0] + w[1];
}

template <bool kStream, typename V> __device__ __forceinline__ V load(const V *p) {
    if constexpr (kStream)
        return __builtin_nontemporal_load(p);
    return *p;
}

// What kGroup threads find in their share of `len` logits, a batch of kAhead vectors at a time. Small
// groups take rows of a few batches, where a shorter one leaves less of the last one empty: on 16,384
// rows of 2,000 (bf16, 16 threads) batches of 2, 3 and 4 take 17.3, 16.9 and 18.0 us.
template <typename T, bool kEntropy, bool kStream, int kGroup>
__device__ __forceinline__ Running scan(const T *x, int len, int tid, float c) {
    using V = Vec<T>;
    constexpr int kAhead = kGroup > kWave ? 4 : 3, kStep = kAhead * kGroup;
    Running r{-INFINITY, 0.0f, 0.0f};
    const int lead = min(lead_of(x), len), vecs = (len - lead) / V::N;
    const int rest = len - vecs * V::N; // elements before and after the whole vectors
    float last[1] = {-INFINITY};
    if (tid < rest)
        last[0] = float(x[tid < lead ? tid : tid + vecs * V::N]);
    const auto *v = reinterpret_cast<const typename V::type *>(x + lead);
    typename V::type q[kAhead];
    float y[kAhead * V::N];
    int i = tid;
    for (; i + kStep - kGroup < vecs; i += kStep) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            q[k] = load<kStream>(v + i + k * kGroup);
#pragma unroll
        for (int k = 0; k < kAhead * V::N; ++k)
            y[k] = float(q[k / V::N][k % V::N]);
        add<kEntropy>(r, y, c);
    }
    if (i < vecs) { // -inf where there is nothing left adds nothing
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            q[k] = i + k * kGroup < vecs ? load<kStream>(v + i + k * kGroup) : typename V::type(T(-INFINITY));
#pragma unroll
        for (int k = 0; k < kAhead * V::N; ++k)
            y[k] = float(q[k / V::N][k % V::N]);
        add<kEntropy>(r, y, c);
    }
    if (rest > 0)
        add<kEntropy>(r, last, c);
    return r;
}

template <int kGroup> __device__ __forceinline__ Running group_join(Running r, float c) {
    for (int off = kGroup / 2; off; off >>= 1)
        r = join(r, Running{__shfl_xor(r.m, off), __shfl_xor(r.S, off), __shfl_xor(r.W, off)}, c);
    return r;
}

struct RowOut {
    float *logp, *entropy, *stats;
};

__device__ __forceinline__ void store_row(RowOut out, int64_t row, float m, float log_sum, float logp, float entropy) {
    out.logp[row] = logp;
    if (out.entropy)
        out.entropy[row] = entropy;
    if (out.stats) {
        out.stats[2 * row] = m;
        out.stats[2 * row + 1] = log_sum;
    }
}

// `at`: the target's logit
__device__ __forceinline__ void finish_row(RowOut out, int64_t row, Running r, float at, float scale) {
    if (r.S == 0.0f) // every logit is -inf
        return store_row(out, row, -INFINITY, 0.0f, -INFINITY, 0.0f);
    const float log_sum = logf(r.S);
    store_row(out, row, r.m, log_sum, (at - base_of(r.m)) * scale - log_sum, log_sum - kLn2 * (r.W / r.S));
}

// The row's result from every thread's, in the row's first wave. kGroup threads, a workgroup where they
// are more than a wave.
template <int kGroup> __device__ __forceinline__ Running row_join(Running r, int tid, float c) {
    constexpr int kWaves = kGroup / kWave;
    r = group_join<kGroup < kWave ? kGroup : kWave>(r, c);
    if constexpr (kWaves > 1) {
        __shared__ Running part[kWaves];
        __syncthreads(); // part may still be read for the row before
        if (tid % kWave == 0)
            part[tid / kWave] = r;
        __syncthreads();
        if (tid < kWave)
            r = group_join<kWaves>(part[tid % kWaves], c);
    }
    return r;
}

// kGroup threads take a row, in workgroups of at least kThreads. Bound by memory: 16,384 rows of 131,072
// (bf16) with entropies go in 620 us, 6.9 TB/s (in a row of passes; 669 in a trace); their instructions (8.7 a
// logit, one of them exp2) come close behind.
template <typename T, bool kEntropy, bool kStream, int kGroup>
__global__ void __launch_bounds__(kGroup < kThreads ? kThreads : kGroup)
logp_kernel(const T *logits, int64_t n, int V, int64_t stride, const int64_t *targets, float scale, RowOut out) {
    constexpr int kRows = kGroup < kThreads ? kThreads / kGroup : 1;
    const float c = base2_of(scale);
    const int tid = threadIdx.x % kGroup;
    for (int64_t row = blockIdx.x * int64_t(kRows) + threadIdx.x / kGroup; row < n; row += int64_t(gridDim.x) * kRows) {
        const int64_t t = targets[row];
        if (t < 0 || t >= V) {
            if (tid == 0)
                store_row(out, row, 0.0f, 0.0f, 0.0f, 0.0f);
            continue;
        }
        const T *x = logits + row * stride;
        const float at = float(x[t]);
        const Running r = row_join<kGroup>(scan<T, kEntropy, kStream, kGroup>(x, V, tid, c), tid, c);
        if (tid == 0)
            finish_row(out, row, r, at, scale);
    }
}

// A workgroup takes one of `parts` shares of a row, for rows too few to fill the card: bound by the trip to
// memory, 3.9 us for one row of 128,000 and 2.0 for its join.
template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads)
logp_part_kernel(const T *logits, int V, int64_t stride, const int64_t *targets, float scale, int parts, int share,
                 float4 *partial) {
    const float c = base2_of(scale);
    const int row = blockIdx.x / parts, first = blockIdx.x % parts * share;
    const int64_t t = targets[row];
    if (t < 0 || t >= V)
        return;
    const T *x = logits + row * stride + first;
    const Running r = row_join<kThreads>(scan<T, kEntropy, false, kThreads>(x, min(share, V - first), threadIdx.x, c), threadIdx.x, c);
    if (threadIdx.x == 0)
        partial[blockIdx.x] = make_float4(r.m, r.S, r.W, 0.0f);
}

template <typename T>
__global__ void __launch_bounds__(kWave)
logp_join_kernel(const T *logits, int V, int64_t stride, const int64_t *targets, float scale, int parts,
                 const float4 *partial, RowOut out) {
    const float c = base2_of(scale);
    const int row = blockIdx.x;
    const int64_t t = targets[row];
    if (t < 0 || t >= V) {
        if (threadIdx.x == 0)
            store_row(out, row, 0.0f, 0.0f, 0.0f, 0.0f);
        return;
    }
    const float at = float(logits[row * stride + t]);
    Running r{-INFINITY, 0.0f, 0.0f};
    for (int k = threadIdx.x; k < parts; k += kWave) {
        const float4 q = partial[int64_t(row) * parts + k];
        r = join(r, Running{q.x, q.y, q.z}, c);
    }
    r = group_join<kWave>(r, c);
    if (threadIdx.x == 0)
        finish_row(out, row, r, at, scale);
}

// kGroup threads take one of `parts` shares of a row, of `share` vectors; the first takes the elements
// before and after the whole vectors too. Bound by memory: 2.1 GB read and written on 4,096 rows of
// 131,072 (bf16) go in 342 us, 6.3 TB/s. Shares of two vectors a thread keep the card's reads and
// writes close together: whole rows take 397 us. Stores past the caches leave those to the logits
// (347 us without, 8.7 for 6.9 us on 200 rows of 32,001); loads past them gain nothing (339 us, but
// 7.9 us there).
template <typename T, bool kEntropy, int kGroup>
__global__ void __launch_bounds__(kThreads)
logp_backward_kernel(const T *logits, int64_t n, int V, int64_t stride, const int64_t *targets, float scale,
                     const float *stats, const float *grad_logp, const float *entropy, const float *grad_entropy,
                     T *grad, int64_t grad_stride, int parts, int share) {
    using Vc = Vec<T>;
    constexpr int kItems = kThreads / kGroup, kAhead = 2;
    const float c = base2_of(scale);
    const int tid = threadIdx.x % kGroup;
    const int64_t items = n * parts;
    for (int64_t item = blockIdx.x * int64_t(kItems) + threadIdx.x / kGroup; item < items; item += int64_t(gridDim.x) * kItems) {
        const int64_t row = parts > 1 ? item / parts : item;
        const int part = parts > 1 ? int(item - row * parts) : 0;
        const int64_t t = targets[row];
        const float m = stats[2 * row], log_sum = stats[2 * row + 1];
        const float g = grad_logp[row], h = kEntropy ? grad_entropy[row] : 0.0f;
        T *dx = grad + row * grad_stride;
        const T *x = logits + row * stride;
        const int lead = min(lead_of(dx), V), vecs = (V - lead) / Vc::N, rest = part == 0 ? V - vecs * Vc::N : 0;
        const int end = min(vecs, (part + 1) * share);
        const int one = tid < lead ? tid : tid + vecs * Vc::N; // single elements
        auto *out = reinterpret_cast<typename Vc::type *>(dx + lead);
        int i = part * share + tid;
        if (t < 0 || t >= V || (g == 0.0f && h == 0.0f) || (m == -INFINITY && log_sum == 0.0f)) {
            for (; i < end; i += kGroup)
                __builtin_nontemporal_store(typename Vc::type(T(0.0f)), out + i);
            if (tid < rest)
                dx[one] = T(0.0f);
            continue;
        }
        const float base = base_of(m), low = log_sum * kLog2e;
        // p (A + B log2 p) with A = -scale (g + h entropy), B = -scale h ln 2. Where p is 0, log2 p may be -inf and its
        // product with B as well; adding (p log2 p) B instead took 420 for 396 us on 4,096 rows of 131,072 (bf16).
        const float A = -scale * fmaf(h, kEntropy ? entropy[row] : 0.0f, g), B = -scale * h * kLn2, at_target = scale * g;
        auto slope = [&](float y) {
            const float l = fmaf(y - base, c, -low), p = __builtin_amdgcn_exp2f(l);
            return !kEntropy ? p * A : p == 0.0f ? 0.0f : p * fmaf(B, l, A);
        };
        auto vec_slope = [&](typename Vc::type q, int at) {
            float d[Vc::N];
#pragma unroll
            for (int k = 0; k < Vc::N; ++k)
                d[k] = slope(float(q[k]));
            const int first = lead + at * Vc::N;
            if (int(t) >= first && int(t) < first + Vc::N)
#pragma unroll
                for (int k = 0; k < Vc::N; ++k)
                    d[k] += first + k == int(t) ? at_target : 0.0f;
            typename Vc::type o;
#pragma unroll
            for (int k = 0; k < Vc::N; ++k)
                o[k] = T(d[k]);
            __builtin_nontemporal_store(o, out + at);
        };
        const auto *in = reinterpret_cast<const typename Vc::unaligned *>(x + lead);
        for (; i + (kAhead - 1) * kGroup < end; i += kAhead * kGroup) {
            typename Vc::type q[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                q[k] = in[i + k * kGroup];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                vec_slope(q[k], i + k * kGroup);
        }
        for (; i < end; i += kGroup)
            vec_slope(in[i], i);
        if (tid < rest)
            dx[one] = T(slope(float(x[one])) + (one == int(t) ? at_target : 0.0f));
    }
}

int size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }

// How a forward pass is split: kGroup of logp_kernel, or shares of a row for logp_part_kernel.
struct Plan {
    int group, parts, share; // parts > 1: logp_part_kernel and logp_join_kernel
    bool stream;             // loads past the caches
};

// The fewest threads a row that still make 2,000 waves, 8 to a CU, and no more than its vectors can
// feed. Measured (us, bf16, with entropies, in graphs of 20 passes over one to 20 inputs; 16 / 64 / 256
// / 1,024 threads): 16,384 x 500: 8.6 / 13.3; 16,384 x 2,000: 16.9 / 19.9; 16,384 x 8,000: - / 49 / 66 /
// 133; 8,192 x 32,000: - / 93 / 93; 16,384 x 131,072: - / 680 / 649; 1,000 x 128,000: - / 74 / 54 / 53;
// 200 x 128,000: - / - / 28 / 17; 300 x 8,000: - / 7.9 / 6.8 / 6.4; 8,192 x 32,000 with 40% of the rows
// ignored: - / 69 / 57 (the others' waves are then too few). Few long rows are split: one of 128,000
// takes 12.7 us with 1,024 threads, 5.5 in 62 shares and their join, 64 of them 15.3 and 10.1; one of
// 32,000 6.3 and 5.2, where the second launch costs the host what it gains; 200 of 128,000 17.3 and
// 18.8.
// Loads past the caches: 16,384 x 131,072 731 -> 649, 16,384 x 8,000 54 -> 49. Below 64 MiB the pass
// that made the logits has left them in the caches, and the gradient wants them there: a copy, this
// pass, the gradient and a sum over 256 x 32,000 take 28.4 us with cached loads, 30.8 past the caches.
Plan plan_of(int32_t dtype, int64_t n, int64_t V) {
    const int64_t size = size_of(dtype), per = 16 / size, vecs = (V + per - 1) / per;
    Plan p{1024, 1, 0, n >= (int64_t(64) << 20) / (V * size)};
    const auto feeds = [&](int group) { return n * group >= 2000 * kWave; };
    if (n <= 128 && V * size > (64 << 10)) {
        const int64_t parts = std::min((511 + n) / n, (vecs + kThreads - 1) / kThreads);
        p.share = int(((vecs + parts - 1) / parts) * per);
        p.parts = int((V + p.share - 1) / p.share);
    }
    if (vecs <= 256 && feeds(16))
        p.group = 16;
    else if (vecs <= kWave || (vecs <= 2048 && feeds(64)))
        p.group = 64;
    else if (vecs <= 512 || feeds(256))
        p.group = 256;
    return p;
}

// Threads that share a row of the gradient: 16,384 x 500 takes 11.4 us with 16 and 12.1 with 64, 16,384
// x 1,000 23 with 16, 16.5 with 64 and 28 with 256, 16,384 x 4,000 50 with 64 and 46 with 256.
int backward_group(int64_t vecs) { return vecs <= 64 ? 16 : vecs <= 256 ? 64 : 256; }
constexpr int kBackwardShare = 512;

using treeens::set_error;

int check_rows(const void *logits, int32_t dtype, int64_t n, int64_t V, int64_t stride, const int64_t *targets,
               float scale) {
    if (dtype != TREE_ENS_F32 && dtype != TREE_ENS_BF16 && dtype != TREE_ENS_F16)
        return set_error(TREE_ENS_E_ARG, "dtype must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
    if (n < 0 || V < 1 || V > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and n_vocab in [1, INT32_MAX]");
    if (!std::isfinite(scale) || !(scale > 0.0f))
        return set_error(TREE_ENS_E_ARG, "scale must be finite and > 0");
    if (n == 0)
        return TREE_ENS_OK;
    if (stride < V || stride > INT64_MAX / 8 / n)
        return set_error(TREE_ENS_E_ARG, "row_stride must be at least n_vocab, and the rows within memory");
    if (!logits || !targets)
        return set_error(TREE_ENS_E_ARG, "logits or targets is NULL");
    if (reinterpret_cast<uintptr_t>(logits) % unsigned(size_of(dtype)) || reinterpret_cast<uintptr_t>(targets) % 8)
        return set_error(TREE_ENS_E_ARG, "logits or targets is misaligned for its type");
    return TREE_ENS_OK;
}

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(TREE_ENS_E_DEVICE, std::string(what) + " launch: " + hipGetErrorString(e));
    return TREE_ENS_OK;
}

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

// Calls f with a null pointer of the logits' type.
template <typename F> void with_type(int32_t dtype, F &&f) {
    if (dtype == TREE_ENS_F32)
        f(static_cast<const float *>(nullptr));
    else if (dtype == TREE_ENS_BF16)
        f(static_cast<const __bf16 *>(nullptr));
    else
        f(static_cast<const _Float16 *>(nullptr));
}

// Calls f with two std::bool_constant.
template <typename F> void with_flags(bool a, bool b, F &&f) {
    const auto second = [&](auto x) { b ? f(x, std::true_type()) : f(x, std::false_type()); };
    a ? second(std::true_type()) : second(std::false_type());
}

// Bytes of a forward pass's partial results.
int64_t partial_bytes(const Plan &p, int64_t n) { return p.parts > 1 ? n * p.parts * int64_t(sizeof(float4)) : 0; }

} // namespace

extern "C" {

int tree_ens_token_logp_workspace(int32_t dtype, int64_t n_tokens, int64_t n_vocab, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (dtype != TREE_ENS_F32 && dtype != TREE_ENS_BF16 && dtype != TREE_ENS_F16)
        return set_error(TREE_ENS_E_ARG, "dtype must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
    if (n_tokens < 0 || n_vocab < 1 || n_vocab > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and n_vocab in [1, INT32_MAX]");
    if (n_tokens > 0)
        *bytes = partial_bytes(plan_of(dtype, n_tokens, n_vocab), n_tokens);
    return TREE_ENS_OK;
}

int tree_ens_token_logp(void *stream, const void *logits, int32_t dtype, int64_t n_tokens, int64_t n_vocab,
                        int64_t row_stride, const int64_t *targets, float scale, float *logp, float *entropy,
                        float *stats, void *workspace, int64_t workspace_bytes) {
    treeens::clear_error();
    if (int rc = check_rows(logits, dtype, n_tokens, n_vocab, row_stride, targets, scale))
        return rc;
    if (n_tokens == 0)
        return TREE_ENS_OK;
    if (!logp)
        return set_error(TREE_ENS_E_ARG, "logp is NULL");
    if (misaligned(logp, 4) || misaligned(entropy, 4) || misaligned(stats, 8))
        return set_error(TREE_ENS_E_ARG, "logp, entropy or stats is misaligned");
    const Plan p = plan_of(dtype, n_tokens, n_vocab);
    if (const int64_t need = partial_bytes(p, n_tokens)) {
        if (!workspace || workspace_bytes < need)
            return set_error(TREE_ENS_E_ARG, "workspace is NULL or smaller than " + std::to_string(need) + " bytes");
        if (misaligned(workspace, 16))
            return set_error(TREE_ENS_E_ARG, "workspace must be 16-byte aligned");
    }
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const RowOut out{logp, entropy, stats};
    (void)hipGetLastError();
    with_type(dtype, [&](auto *type) {
        using T = std::decay_t<decltype(*type)>;
        const auto *x = static_cast<const T *>(logits);
        if (p.parts > 1) {
            hipLaunchKernelGGL((entropy ? logp_part_kernel<T, true> : logp_part_kernel<T, false>),
                               dim3(unsigned(n_tokens * p.parts)), dim3(kThreads), 0, s, x, int(n_vocab), row_stride, targets,
                               scale, p.parts, p.share, static_cast<float4 *>(workspace));
            hipLaunchKernelGGL(logp_join_kernel<T>, dim3(unsigned(n_tokens)), dim3(kWave), 0, s, x, int(n_vocab), row_stride,
                               targets, scale, p.parts, static_cast<const float4 *>(workspace), out);
            return;
        }
        const auto launch = [&](auto kernel) {
            const int rows = std::max(1, kThreads / p.group);
            hipLaunchKernelGGL(kernel, dim3(unsigned(std::min((n_tokens + rows - 1) / rows, kMaxBlocks))),
                               dim3(std::max(p.group, kThreads)), 0, s, x, n_tokens, int(n_vocab), row_stride, targets, scale, out);
        };
        with_flags(entropy != nullptr, p.stream, [&](auto e, auto stream_) {
            constexpr bool kE = decltype(e)::value, kS = decltype(stream_)::value;
            if (p.group == 16)
                launch(logp_kernel<T, kE, kS, 16>);
            else if (p.group == 64)
                launch(logp_kernel<T, kE, kS, 64>);
            else if (p.group == 256)
                launch(logp_kernel<T, kE, kS, 256>);
            else
                launch(logp_kernel<T, kE, kS, 1024>);
        });
    });
    return launched("token log-probability");
}

int tree_ens_token_logp_backward(void *stream, const void *logits, int32_t dtype, int64_t n_tokens, int64_t n_vocab,
                                 int64_t row_stride, const int64_t *targets, float scale, const float *stats,
                                 const float *grad_logp, const float *entropy, const float *grad_entropy,
                                 void *grad_logits, int64_t grad_stride) {
    treeens::clear_error();
    if (int rc = check_rows(logits, dtype, n_tokens, n_vocab, row_stride, targets, scale))
        return rc;
    if (n_tokens == 0)
        return TREE_ENS_OK;
    if (grad_stride < n_vocab || grad_stride > INT64_MAX / 8 / n_tokens)
        return set_error(TREE_ENS_E_ARG, "grad_stride must be at least n_vocab, and the rows within memory");
    if (!stats || !grad_logp || !grad_logits)
        return set_error(TREE_ENS_E_ARG, "stats, grad_logp or grad_logits is NULL");
    if (!entropy != !grad_entropy)
        return set_error(TREE_ENS_E_ARG, "entropy and grad_entropy must both be given or both be NULL");
    if (misaligned(stats, 8) || misaligned(grad_logp, 4) || misaligned(entropy, 4) || misaligned(grad_entropy, 4) ||
        misaligned(grad_logits, unsigned(size_of(dtype))))
        return set_error(TREE_ENS_E_ARG, "stats, entropy or a gradient is misaligned for its type");
    const uintptr_t in = reinterpret_cast<uintptr_t>(logits), out = reinterpret_cast<uintptr_t>(grad_logits);
    const uintptr_t size = uintptr_t(size_of(dtype));
    const uintptr_t in_bytes = size * uintptr_t((n_tokens - 1) * row_stride + n_vocab);
    const uintptr_t out_bytes = size * uintptr_t((n_tokens - 1) * grad_stride + n_vocab);
    const bool same = in == out && (row_stride == grad_stride || n_tokens == 1);
    if (!same && in < out + out_bytes && out < in + in_bytes)
        return set_error(TREE_ENS_E_ARG, "grad_logits overlaps the logits without being the same rows");
    (void)hipGetLastError();
    with_type(dtype, [&](auto *type) {
        using T = std::decay_t<decltype(*type)>;
        const int64_t vecs = n_vocab / Vec<T>::N; // of an aligned row; others have as many or one less
        const int group = backward_group(vecs);
        const int64_t parts = group == 256 ? (vecs + kBackwardShare - 1) / kBackwardShare : 1;
        const int64_t items = n_tokens * parts, per_block = kThreads / group;
        const auto launch = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3(unsigned(std::min((items + per_block - 1) / per_block, kMaxBlocks))), dim3(kThreads), 0,
                               reinterpret_cast<hipStream_t>(stream), static_cast<const T *>(logits), n_tokens, int(n_vocab),
                               row_stride, targets, scale, stats, grad_logp, entropy, grad_entropy,
                               static_cast<T *>(grad_logits), grad_stride, int(parts), kBackwardShare);
        };
        with_flags(grad_entropy != nullptr, false, [&](auto e, auto) {
            constexpr bool kE = decltype(e)::value;
            if (group == 16)
                launch(logp_backward_kernel<T, kE, 16>);
            else if (group == 64)
                launch(logp_backward_kernel<T, kE, 64>);
            else
                launch(logp_backward_kernel<T, kE, 256>);
        });
    });
    return launched("token log-probability gradient");
}

} // extern "C"
