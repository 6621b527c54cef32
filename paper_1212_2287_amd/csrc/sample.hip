// sample.hip -- one token for each row of logits from a given random number, under temperature, top-k,
// min-p and top-p, on gfx950.
//
// Weights w = exp(scale * (x - max x)) are whole numbers of 2^-shift, so that sums are exact in any order.
// Tokens are kept down to a last one in the order of the logits (the largest first, equal ones by index):
// top-k and top-p are both the search for the place in that order where a running count or a running sum of
// weights reaches a target. It goes by the bits of the logits, eight at a time, from histograms in LDS.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>
#include <type_traits>

#include "status.hpp"
#include "tree_ens.h"

namespace {

constexpr int kWave = 64;
constexpr int64_t kMaxBlocks = 1 << 20; // rows beyond this many are taken in turn

struct Args {
    int64_t n, stride;
    int V, shift;
    const double *uniform;
    float scale, top_p, min_p;
    int top_k;
    const float *row_scale, *row_top_p, *row_min_p;
    const int *row_top_k;
    int64_t *tokens;
    float *logp, *log_kept;
};

// The parameters of a row. Fractions are whole numbers of 2^-53.
struct Params {
    double scale;      // 0: the row has no distribution
    double least;      // log of min_p; -inf: all
    uint64_t fraction; // top_p; 2^53: all
    uint64_t at;       // the random number, below 2^53
    int top_k;         // at least 1
};

constexpr uint64_t kOne = uint64_t(1) << 53;

__device__ __forceinline__ Params params_of(const Args &a, int64_t row) {
    Params p;
    const float scale = a.row_scale ? a.row_scale[row] : a.scale;
    p.scale = scale > 0.0f && scale < INFINITY ? double(scale) : 0.0;
    const int k = a.row_top_k ? a.row_top_k[row] : a.top_k;
    p.top_k = k > 0 && k < a.V ? k : a.V;
    const float q = a.row_top_p ? a.row_top_p[row] : a.top_p;
    p.fraction = q < 1.0f ? uint64_t(double(fmaxf(q, 0.0f)) * 0x1p53) : kOne;
    const float m = a.row_min_p ? a.row_min_p[row] : a.min_p;
    p.least = m > 0.0f ? log(double(fminf(m, 1.0f))) : -INFINITY;
    const double u = a.uniform[row];
    p.at = u > 0.0 ? min(uint64_t(fmin(u, 1.0) * 0x1p53), kOne - 1) : 0;
    return p;
}

// Whole-number products of a sum below 2^63 and a fraction of 2^53, rounded down or up.
__device__ __forceinline__ uint64_t share_down(uint64_t sum, uint64_t fraction) {
    return __umul64hi(sum, fraction) << 11 | sum * fraction >> 53;
}
__device__ __forceinline__ uint64_t share_up(uint64_t sum, uint64_t fraction) {
    return share_down(sum, fraction) + ((sum * fraction & (kOne - 1)) != 0);
}

// exp(z) in whole numbers of 2^-shift for z <= 0: 2^y with y = log2(e) z taken apart into a whole number n and a
// rest r within a half, and 2^r by the polynomial of degree 8 whose largest relative error there, 1.1e-12, is the
// smallest with p(0) = 1 (found by exchange). Adding 2^52 rounds to a whole number, which the low bits then hold. The
// double-precision multiply-adds run at the rate of single ones on this card.
__device__ __forceinline__ uint64_t weight_of(double z, int shift) {
    constexpr double kLog2e = 1.4426950408889634, kRound = 0x1.8p52;
    z = fmax(z, -64.0); // 0 already; masked logits among them
    const double t = fma(z, kLog2e, kRound), r = fma(z, kLog2e, kRound - t);
    double p = 0x1.663487d8abc81p-20;
    p = fma(p, r, 0x1.00ee071c7c030p-16);
    p = fma(p, r, 0x1.4306c1165a375p-13);
    p = fma(p, r, 0x1.5d872975c4ed2p-10);
    p = fma(p, r, 0x1.3b2ab7f3b3217p-7);
    p = fma(p, r, 0x1.c6b08defc25fdp-5);
    p = fma(p, r, 0x1.ebfbdff7c5a79p-3);
    p = fma(p, r, 0x1.62e42fef7a78bp-1);
    p = fma(p, r, 1.0);
    const int n = int(__double2loint(t)) + shift;
    p = __hiloint2double(__double2hiint(p) + (n << 20), __double2loint(p));
    return uint64_t(__double_as_longlong(p + 0x1p52)) & ((uint64_t(1) << 52) - 1);
}

// Whole numbers in the order of the floats; -0 counts as 0.
__device__ __forceinline__ uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.0f);
    return b ^ (uint32_t(int32_t(b) >> 31) | 0x80000000u);
}
__device__ __forceinline__ float float_of(uint32_t key) {
    return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// The smallest key whose float has z >= least: a search of 64 places at a time, by the lanes of a wave.
__device__ __forceinline__ uint32_t floor_key(double m, double scale, double least, uint32_t top) {
    if (least == -INFINITY)
        return 0;
    uint32_t low = key_of(-INFINITY); // not enough (the difference from a float's is never 0), `top` is
    const int lane = threadIdx.x % kWave;
    while (top - low > 1) {
        const uint64_t span = top - low;
        const uint32_t k = low + uint32_t(span * uint64_t(lane + 1) / (kWave + 1));
        const uint64_t yes = __ballot((double(float_of(k)) - m) * scale >= least);
        const int first = yes ? __builtin_ctzll(yes) : kWave; // places from here on are enough
        const uint32_t old = low;
        if (first > 0)
            low = old + uint32_t(span * uint64_t(first) / (kWave + 1));
        if (first < kWave)
            top = old + uint32_t(span * uint64_t(first + 1) / (kWave + 1));
    }
    return top;
}

template <typename V> __device__ __forceinline__ V wave_sum(V v) {
    for (int off = kWave / 2; off; off >>= 1)
        v += __shfl_xor(v, off);
    return v;
}

// Sums over the lanes up to and with this one.
template <typename V> __device__ __forceinline__ V wave_scan(V v) {
    const int lane = threadIdx.x % kWave;
    for (int off = 1; off < kWave; off *= 2) {
        const V o = __shfl_up(v, off);
        v += lane >= off ? o : V(0);
    }
    return v;
}

__device__ __forceinline__ void store_row(const Args &a, int64_t row, int64_t token, float logp, float log_kept) {
    a.tokens[row] = token;
    if (a.logp)
        a.logp[row] = logp;
    if (a.log_kept)
        a.log_kept[row] = log_kept;
}

// log(kept / total), which is 0 exactly where they are equal
__device__ __forceinline__ float log_share(uint64_t kept, uint64_t total) {
    return float(log1p(-double(int64_t(total - kept)) / double(total)));
}

constexpr int kThreads = 1024, kWaves = kThreads / kWave, kBins = 256;

// A place in the order of the logits: keys above `key`, and the first `spare` ones of it.
struct Place {
    uint32_t key;
    uint64_t spare;
    uint64_t above; // their weights (of the keys above)
};

template <typename T> struct Row {
    const T *x;
    int V, shift;
    double m, scale;
    uint32_t floor; // keys below it are not there
    __device__ __forceinline__ uint64_t weight(float v) const { return weight_of((double(v) - m) * scale, shift); }
};

struct Shared {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t part[kWaves], sum;
    uint32_t ties[kWaves], digit;
    float max[kWaves];
    int bad;
};

// Where the count (kByMass: the weights) of the keys from the top reaches `target`, which it does.
template <bool kByMass, typename T>
__device__ Place place_of(const Row<T> &r, uint64_t target, Shared &s) {
    Place p{0, target, 0};
    for (int bit = 24; bit >= 0; bit -= 8) {
        __syncthreads();
        if (threadIdx.x < kBins)
            s.mass[threadIdx.x] = s.count[threadIdx.x] = 0;
        __syncthreads();
        for (int i = threadIdx.x; i < r.V; i += kThreads) {
            const float v = float(r.x[i]);
            const uint32_t k = key_of(v);
            if (k < r.floor || (bit < 24 && (k ^ p.key) >> (bit + 8)))
                continue;
            const int bin = k >> bit & (kBins - 1);
            atomicAdd(&s.count[bin], 1u);
            atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[bin]), (unsigned long long)r.weight(v));
        }
        __syncthreads();
        if (threadIdx.x == 0) {
            uint64_t left = p.spare, above = 0;
            int d = kBins - 1;
            for (;; --d) {
                const uint64_t here = kByMass ? s.mass[d] : s.count[d];
                if (left <= here || d == 0)
                    break;
                left -= here;
                above += s.mass[d];
            }
            s.digit = uint32_t(d);
            s.part[0] = left;
            s.part[1] = above;
        }
        __syncthreads();
        p.key |= s.digit << bit;
        p.spare = s.part[0];
        p.above += s.part[1];
    }
    if (kByMass) { // the weight that is left, in tokens of this one's
        const uint64_t w = r.weight(float_of(p.key));
        p.spare = w ? (p.spare + w - 1) / w : 1;
    }
    __syncthreads();
    return p;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) sample_kernel(const T *logits, Args a) {
    __shared__ Shared s;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        Row<T> r{logits + row * a.stride, a.V, a.shift, 0.0, 0.0, 0};
        const Params p = params_of(a, row);
        r.scale = p.scale;
        float m = -INFINITY;
        bool bad = p.scale == 0.0;
        for (int i = tid; i < a.V; i += kThreads) {
            const float v = float(r.x[i]);
            bad |= !(v < INFINITY);
            m = fmaxf(m, v);
        }
        for (int off = kWave / 2; off; off >>= 1)
            m = fmaxf(m, __shfl_xor(m, off));
        __syncthreads();
        if (tid == 0)
            s.bad = 0;
        if (lane == 0)
            s.max[wave] = m;
        __syncthreads();
        if (bad)
            s.bad = 1;
        for (int w = 0; w < kWaves; ++w)
            m = fmaxf(m, s.max[w]);
        __syncthreads();
        if (s.bad || m == -INFINITY) {
            if (tid == 0)
                store_row(a, row, -1, s.bad ? NAN : -INFINITY, s.bad ? NAN : 0.0f);
            continue;
        }
        r.m = double(m);
        r.floor = floor_key(r.m, p.scale, p.least, key_of(m));
        uint64_t total = 0, inside = 0, there = 0;
        for (int i = tid; i < a.V; i += kThreads) {
            const float v = float(r.x[i]);
            const uint64_t w = r.weight(v);
            const bool in = key_of(v) >= r.floor;
            total += w;
            inside += in ? w : 0;
            there += in;
        }
        auto block_sum = [&](uint64_t v) {
            v = wave_sum(v);
            __syncthreads();
            if (lane == 0)
                s.part[wave] = v;
            __syncthreads();
            v = 0;
            for (int w = 0; w < kWaves; ++w)
                v += s.part[w];
            return v;
        };
        total = block_sum(total);
        inside = block_sum(inside);
        there = block_sum(there);
        Place last{r.floor, there, 0};
        bool all = true;
        if (uint64_t(p.top_k) < there) {
            last = place_of<false>(r, uint64_t(p.top_k), s);
            inside = last.above + last.spare * r.weight(float_of(last.key));
            all = false;
        }
        if (p.fraction < kOne) {
            last = place_of<true>(r, max(share_up(inside, p.fraction), uint64_t(1)), s);
            all = false;
        }
        // waves take stretches of the vocabulary; each token's equals before it decide whether it is kept
        const int each = ((a.V + kThreads - 1) / kThreads) * kWave, from = min(wave * each, a.V), to = min(from + each, a.V);
        const uint64_t level = all ? 0 : r.weight(float_of(last.key));
        uint64_t mass = 0;
        uint32_t ties = 0;
        for (int i = from + lane; i < to; i += kWave) {
            const float v = float(r.x[i]);
            const uint32_t k = key_of(v);
            if (all ? k >= last.key : k > last.key)
                mass += r.weight(v);
            else if (k == last.key)
                ++ties;
        }
        mass = wave_sum(mass);
        ties = wave_sum(ties);
        __syncthreads();
        if (lane == 0) {
            s.part[wave] = mass;
            s.ties[wave] = ties;
        }
        __syncthreads();
        uint64_t kept = 0, before = 0, equal = 0, my_equal = 0;
        for (int w = 0; w < kWaves; ++w) {
            if (w == wave) {
                before = kept;
                my_equal = equal;
            }
            const uint64_t some = min(uint64_t(s.ties[w]), last.spare - min(equal, last.spare));
            kept += s.part[w] + (all ? 0 : some * level);
            equal += s.ties[w];
        }
        const uint64_t target = share_down(kept, p.at);
        uint64_t running = before;
        for (int i = from + lane; i - lane < to && running <= target; i += kWave) {
            const float v = i < to ? float(r.x[i]) : -INFINITY;
            const uint32_t k = i < to ? key_of(v) : 0;
            const bool tie = !all && i < to && k == last.key;
            const uint64_t tied = __ballot(tie);
            const uint64_t rank = my_equal + __builtin_popcountll(tied & ((uint64_t(1) << lane) - 1));
            const bool keep = i < to && (all ? k >= last.key : k > last.key || (tie && rank < last.spare));
            const uint64_t sum = running + wave_scan(keep ? r.weight(v) : 0);
            const uint64_t past = __ballot(sum > target);
            if (past && lane == __builtin_ctzll(past) && before <= target) {
                const double z = (double(v) - r.m) * p.scale;
                store_row(a, row, i, float(z - log(ldexp(double(total), -a.shift))), log_share(kept, total));
            }
            my_equal += __builtin_popcountll(tied);
            running = __shfl(sum, kWave - 1);
        }
        __syncthreads();
    }
}

int size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }

using treeens::set_error;

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

} // namespace

extern "C" {

int tree_ens_sample_workspace(int32_t dtype, int64_t n_tokens, int64_t n_vocab, int64_t *bytes) {
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

int tree_ens_sample(void *stream, const void *logits, int32_t dtype, int64_t n_tokens, int64_t n_vocab, int64_t row_stride,
                    const double *uniform, float scale, int32_t top_k, float top_p, float min_p, const float *row_scale,
                    const int32_t *row_top_k, const float *row_top_p, const float *row_min_p, int64_t *tokens, float *logp,
                    float *log_kept, void *workspace, int64_t workspace_bytes) {
    treeens::clear_error();
    if (dtype != TREE_ENS_F32 && dtype != TREE_ENS_BF16 && dtype != TREE_ENS_F16)
        return set_error(TREE_ENS_E_ARG, "dtype must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
    if (n_tokens < 0 || n_vocab < 1 || n_vocab > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and n_vocab in [1, INT32_MAX]");
    if (!row_scale && !(std::isfinite(scale) && scale > 0.0f))
        return set_error(TREE_ENS_E_ARG, "scale must be finite and > 0");
    if (!row_top_k && top_k < 0)
        return set_error(TREE_ENS_E_ARG, "top_k must be >= 0");
    if (!row_top_p && !(top_p > 0.0f && top_p <= 1.0f))
        return set_error(TREE_ENS_E_ARG, "top_p must be in (0, 1]");
    if (!row_min_p && !(min_p >= 0.0f && min_p <= 1.0f))
        return set_error(TREE_ENS_E_ARG, "min_p must be in [0, 1]");
    if (n_tokens == 0)
        return TREE_ENS_OK;
    if (row_stride < n_vocab || row_stride > INT64_MAX / 8 / n_tokens)
        return set_error(TREE_ENS_E_ARG, "row_stride must be at least n_vocab, and the rows within memory");
    if (!logits || !uniform || !tokens)
        return set_error(TREE_ENS_E_ARG, "logits, uniform or tokens is NULL");
    if (misaligned(logits, unsigned(size_of(dtype))) || misaligned(uniform, 8) || misaligned(tokens, 8))
        return set_error(TREE_ENS_E_ARG, "logits, uniform or tokens is misaligned for its type");
    if (misaligned(row_scale, 4) || misaligned(row_top_k, 4) || misaligned(row_top_p, 4) || misaligned(row_min_p, 4) ||
        misaligned(logp, 4) || misaligned(log_kept, 4))
        return set_error(TREE_ENS_E_ARG, "a row's parameters, logp or log_kept is misaligned");
    int shift = 44;
    while (n_vocab >> (63 - shift))
        --shift;
    const Args a{n_tokens, row_stride, int(n_vocab), shift, uniform, scale, top_p, min_p, top_k, row_scale, row_top_p,
                 row_min_p, row_top_k, tokens, logp, log_kept};
    (void)hipGetLastError();
    const auto launch = [&](auto *type) {
        using T = std::decay_t<decltype(*type)>;
        hipLaunchKernelGGL(sample_kernel<T>, dim3(unsigned(std::min(n_tokens, kMaxBlocks))), dim3(kThreads), 0,
                           reinterpret_cast<hipStream_t>(stream), static_cast<const T *>(logits), a);
    };
    if (dtype == TREE_ENS_F32)
        launch(static_cast<float *>(nullptr));
    else if (dtype == TREE_ENS_BF16)
        launch(static_cast<__bf16 *>(nullptr));
    else
        launch(static_cast<_Float16 *>(nullptr));
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(TREE_ENS_E_DEVICE, std::string("sample launch: ") + hipGetErrorString(e));
    return TREE_ENS_OK;
}

} // extern "C"
