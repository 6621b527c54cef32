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
// 0 times it is 0, where 0 times the -inf of a masked logit would be NaN.
constexpr float kFar = -1e30f;

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

// What kGroup threads find in their share of `len` logits.
template <typename T, bool kEntropy, int kGroup>
__device__ __forceinline__ Running scan(const T *x, int len, int tid, float c) {
    using V = Vec<T>;
    constexpr int kAhead = 4; // loads in flight
    Running r{-INFINITY, 0.0f, 0.0f};
    const int lead = min(lead_of(x), len), vecs = (len - lead) / V::N;
    const auto *v = reinterpret_cast<const typename V::type *>(x + lead);
    int i = tid;
    for (; i + (kAhead - 1) * kGroup < vecs; i += kAhead * kGroup) {
        typename V::type q[kAhead];
        float y[kAhead * V::N];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            q[k] = v[i + k * kGroup];
#pragma unroll
        for (int k = 0; k < kAhead * V::N; ++k)
            y[k] = float(q[k / V::N][k % V::N]);
        add<kEntropy>(r, y, c);
    }
    for (; i < vecs; i += kGroup) {
        float y[V::N];
#pragma unroll
        for (int k = 0; k < V::N; ++k)
            y[k] = float(v[i][k]);
        add<kEntropy>(r, y, c);
    }
    // what lies before and after the whole vectors
    const int rest = len - vecs * V::N;
    if (tid < rest) {
        const float y[1] = {float(x[tid < lead ? tid : tid + vecs * V::N])};
        add<kEntropy>(r, y, c);
    }
    return r;
}

__device__ __forceinline__ Running wave_join(Running r, float c) {
    for (int off = kWave / 2; off; off >>= 1)
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

template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads)
logp_kernel(const T *logits, int64_t n, int V, int64_t stride, const int64_t *targets, float scale, RowOut out) {
    __shared__ Running part[kThreads / kWave];
    const float c = scale * kLog2e;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const int64_t t = targets[row];
        if (t < 0 || t >= V) {
            if (threadIdx.x == 0)
                store_row(out, row, 0.0f, 0.0f, 0.0f, 0.0f);
            continue;
        }
        const T *x = logits + row * stride;
        Running r = wave_join(scan<T, kEntropy, kThreads>(x, V, threadIdx.x, c), c);
        if (threadIdx.x % kWave == 0)
            part[threadIdx.x / kWave] = r;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kThreads / kWave; ++w)
                r = join(r, part[w], c);
            finish_row(out, row, r, float(x[t]), scale);
        }
        __syncthreads();
    }
}

template <typename T, bool kEntropy>
__global__ void __launch_bounds__(kThreads)
logp_backward_kernel(const T *logits, int64_t n, int V, int64_t stride, const int64_t *targets, float scale,
                     const float *stats, const float *grad_logp, const float *entropy, const float *grad_entropy,
                     T *grad, int64_t grad_stride) {
    using Vc = Vec<T>;
    const float c = scale * kLog2e;
    for (int64_t row = blockIdx.x; row < n; row += gridDim.x) {
        const int64_t t = targets[row];
        const float m = stats[2 * row], log_sum = stats[2 * row + 1];
        const float g = grad_logp[row], h = kEntropy ? grad_entropy[row] : 0.0f;
        T *dx = grad + row * grad_stride;
        const T *x = logits + row * stride;
        const int lead = min(lead_of(dx), V), vecs = (V - lead) / Vc::N, rest = V - vecs * Vc::N;
        const int one = threadIdx.x < lead ? threadIdx.x : threadIdx.x + vecs * Vc::N; // single elements
        auto *out = reinterpret_cast<typename Vc::type *>(dx + lead);
        if (t < 0 || t >= V || (g == 0.0f && h == 0.0f) || (m == -INFINITY && log_sum == 0.0f)) {
            for (int i = threadIdx.x; i < vecs; i += kThreads)
                out[i] = typename Vc::type(0.0f);
            if (threadIdx.x < rest)
                dx[one] = T(0.0f);
            continue;
        }
        const float base = base_of(m), low = log_sum * kLog2e;
        // p (A + B log2 p) with A = -scale (g + h entropy), B = -scale h ln 2
        const float A = -scale * fmaf(h, kEntropy ? entropy[row] : 0.0f, g), B = -scale * h * kLn2, at_target = scale * g;
        auto slope = [&](float y) {
            const float l = fmaf(y - base, c, -low), p = __builtin_amdgcn_exp2f(l);
            return kEntropy ? p * fmaf(B, fmaxf(l, kFar), A) : p * A;
        };
        auto vec_slope = [&](typename Vc::type q, int i) {
            float d[Vc::N];
#pragma unroll
            for (int k = 0; k < Vc::N; ++k)
                d[k] = slope(float(q[k]));
            const int first = lead + i * Vc::N;
            if (int(t) >= first && int(t) < first + Vc::N)
#pragma unroll
                for (int k = 0; k < Vc::N; ++k)
                    d[k] += first + k == int(t) ? at_target : 0.0f;
            typename Vc::type o;
#pragma unroll
            for (int k = 0; k < Vc::N; ++k)
                o[k] = T(d[k]);
            out[i] = o;
        };
        constexpr int kAhead = 4;
        const auto *in = reinterpret_cast<const typename Vc::unaligned *>(x + lead);
        int i = threadIdx.x;
        for (; i + (kAhead - 1) * kThreads < vecs; i += kAhead * kThreads) {
            typename Vc::type q[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                q[k] = in[i + k * kThreads];
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                vec_slope(q[k], i + k * kThreads);
        }
        for (; i < vecs; i += kThreads)
            vec_slope(in[i], i);
        if (threadIdx.x < rest)
            dx[one] = T(slope(float(x[one])) + (one == int(t) ? at_target : 0.0f));
    }
}

int size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }

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
    (void)workspace;
    (void)workspace_bytes;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const RowOut out{logp, entropy, stats};
    (void)hipGetLastError();
    with_type(dtype, [&](auto *type) {
        using T = std::decay_t<decltype(*type)>;
        const auto kernel = entropy ? logp_kernel<T, true> : logp_kernel<T, false>;
        hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(n_tokens, kMaxBlocks))), dim3(kThreads), 0, s,
                           static_cast<const T *>(logits), n_tokens, int(n_vocab), row_stride, targets, scale, out);
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
        const auto kernel = grad_entropy ? logp_backward_kernel<T, true> : logp_backward_kernel<T, false>;
        hipLaunchKernelGGL(kernel, dim3(unsigned(std::min(n_tokens, kMaxBlocks))), dim3(kThreads), 0,
                           reinterpret_cast<hipStream_t>(stream), static_cast<const T *>(logits), n_tokens, int(n_vocab),
                           row_stride, targets, scale, stats, grad_logp, entropy, grad_entropy,
                           static_cast<T *>(grad_logits), grad_stride);
    });
    return launched("token log-probability gradient");
}

} // extern "C"
