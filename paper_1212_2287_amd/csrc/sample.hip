// sample.hip -- one token for each row of logits from a given random number, under temperature, top-k,
// min-p and top-p, on gfx950.
//
// Weights w = exp(scale * (x - max x)) are whole numbers of 2^-shift, so that sums are exact in any order.
// Tokens are kept down to a last one in the order of the logits (the largest first, equal ones by index):
// top-k and top-p are both the search for the place in that order where a running count or a running sum of
// weights reaches a target.
//
// Rows of up to 2,048 tokens go to one workgroup (small_kernel), which sorts them. Of longer rows scan_kernel
// reads every logit once and leaves a digest: the largest logit of every 128, and the largest and the weights of
// every 2,048. pick_kernel, a workgroup a row, finds from it the few segments that can hold a kept token, sorts
// their candidates and takes the token; where nothing is cut off, the digest's weights lead to the 2,048 logits that
// hold it. Rows whose kept tokens are more than its list holds are read again (wide_row).
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
constexpr double kLog2e = 1.4426950408889634;

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

// 2^(d c) in whole numbers of 2^-shift for -128 <= d c <= 0: the exponent taken apart into a whole number n and a rest
// r within a half, and 2^r by the polynomial of degree 8 whose largest relative error there, 1.1e-12, is the smallest
// with p(0) = 1 (found by exchange). Double-precision multiply-adds run at the rate of single ones on this card.
__device__ __forceinline__ double power_of(double d, double c, int shift) {
    constexpr double kRound = 0x1.8p52; // adding it leaves the whole number in the low bits
    const double t = fma(d, c, kRound), r = fma(d, c, kRound - t);
    double p = 0x1.663487d8abc81p-20;
    p = fma(p, r, 0x1.00ee071c7c030p-16);
    p = fma(p, r, 0x1.4306c1165a375p-13);
    p = fma(p, r, 0x1.5d872975c4ed2p-10);
    p = fma(p, r, 0x1.3b2ab7f3b3217p-7);
    p = fma(p, r, 0x1.c6b08defc25fdp-5);
    p = fma(p, r, 0x1.ebfbdff7c5a79p-3);
    p = fma(p, r, 0x1.62e42fef7a78bp-1);
    p = fma(p, r, 1.0);
    return __hiloint2double(__double2hiint(p) + ((__double2loint(t) + shift) << 20), __double2loint(p));
}

// The number that adding 2^52 leaves in the low bits, rounded to nearest, for 0 <= v < 2^52.
__device__ __forceinline__ uint64_t whole_of(double v) {
    return uint64_t(__double_as_longlong(v + 0x1p52)) & ((uint64_t(1) << 52) - 1);
}
__device__ __forceinline__ uint64_t weight_of(double d, double c, int shift) { return whole_of(power_of(d, c, shift)); }

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

// The larger one; NaN if either is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

__device__ __forceinline__ void store_row(const Args &a, int64_t row, int64_t token, float logp, float log_kept) {
    a.tokens[row] = token;
    if (a.logp)
        a.logp[row] = logp;
    if (a.log_kept)
        a.log_kept[row] = log_kept;
}

// A row: its largest logit m, and what turns a logit's distance from it into its weight.
struct Row {
    double m, scale, c, far;
    int shift;
    uint32_t floor; // keys below it are not kept (min_p)
    __device__ __forceinline__ Row(float top, const Params &p, int shift_)
        : m(double(top)), scale(p.scale), c(p.scale * kLog2e), far(-64.0 / p.scale), shift(shift_), floor(0) {}
    // masked logits are taken at `far`, where the weight is 0
    __device__ __forceinline__ uint64_t weight(float x) const { return weight_of(fmax(double(x) - m, far), c, shift); }
    __device__ __forceinline__ uint64_t key_weight(uint32_t k) const { return weight(float_of(k)); }
};

// The token's log-probability and the logarithm of the kept share, which is 0 exactly where everything is kept.
__device__ __forceinline__ void finish_row(const Args &a, int64_t row, const Row &r, int token, float x, uint64_t kept, uint64_t total) {
    if (!a.logp && !a.log_kept)
        return store_row(a, row, token, 0.0f, 0.0f);
    const double logp = (double(x) - r.m) * r.scale - log(ldexp(double(total), -r.shift));
    const double dropped = total > kept ? double(total - kept) / double(total) : 0.0;
    store_row(a, row, token, float(logp), float(log1p(-dropped)));
}
__device__ __forceinline__ void finish_without(const Args &a, int64_t row, bool bad) {
    if (threadIdx.x == 0)
        store_row(a, row, -1, bad ? NAN : -INFINITY, bad ? NAN : 0.0f);
}

// A place in the order of the logits: keys above `key` are kept, and the first `spare` ones of it.
struct Place {
    uint32_t key;
    uint64_t spare;
};

constexpr int kBins = 256;

// Sums over kT threads and the search for a place by all of them.
template <int kT> struct Block {
    static constexpr int kWaves = kT / kWave;
    struct Shared {
        uint64_t part[kWaves];
        float max[kWaves];
        uint64_t left;
        uint32_t digit;
    };

    // The sum over all threads.
    static __device__ uint64_t sum(uint64_t v, Shared &s) {
        v = wave_sum(v);
        if constexpr (kWaves == 1)
            return v;
        __syncthreads();
        if (threadIdx.x % kWave == 0)
            s.part[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0;
        for (int w = 0; w < kWaves; ++w)
            v += s.part[w];
        return v;
    }

    // The sum over the threads before this one; `total` receives that over all.
    static __device__ uint64_t before(uint64_t v, uint64_t &total, Shared &s) {
        const uint64_t with = wave_scan(v);
        if constexpr (kWaves == 1) {
            total = __shfl(with, kWave - 1);
            return with - v;
        }
        __syncthreads();
        if (threadIdx.x % kWave == kWave - 1)
            s.part[threadIdx.x / kWave] = with;
        __syncthreads();
        uint64_t sum = with - v;
        total = 0;
        for (int w = 0; w < kWaves; ++w) {
            sum += w < int(threadIdx.x / kWave) ? s.part[w] : 0;
            total += s.part[w];
        }
        return sum;
    }

    static __device__ float max(float v, Shared &s) {
        for (int off = kWave / 2; off; off >>= 1)
            v = larger(v, __shfl_xor(v, off));
        if constexpr (kWaves == 1)
            return v;
        __syncthreads();
        if (threadIdx.x % kWave == 0)
            s.max[threadIdx.x / kWave] = v;
        __syncthreads();
        for (int w = 0; w < kWaves; ++w)
            v = larger(v, s.max[w]);
        return v;
    }

    // Where the count (kByMass: the weights) of the keys from the top reaches `target`, which it does; `above` receives
    // the weights of the keys above the place's. Eight bits of the keys at a time, from histograms.
    template <bool kByMass, typename T>
    static __device__ Place place_of(const T *x, int V, const Row &r, uint64_t target, uint64_t &above, uint64_t *mass, uint32_t *count,
                                     Shared &s) {
        Place p{0, target};
        above = 0;
        for (int bit = 24; bit >= 0; bit -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kT)
                mass[i] = count[i] = 0;
            __syncthreads();
            for (int i = threadIdx.x; i < V; i += kT) {
                const float v = float(x[i]);
                const uint32_t k = key_of(v);
                if (k < r.floor || (bit < 24 && (k ^ p.key) >> (bit + 8)))
                    continue;
                const int bin = k >> bit & (kBins - 1);
                atomicAdd(&count[bin], 1u);
                atomicAdd(reinterpret_cast<unsigned long long *>(&mass[bin]), (unsigned long long)r.weight(v));
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint64_t left = p.spare, over = 0;
                int d = kBins - 1;
                for (;; --d) {
                    const uint64_t here = kByMass ? mass[d] : count[d];
                    if (left <= here || d == 0)
                        break;
                    left -= here;
                    over += mass[d];
                }
                s.digit = uint32_t(d);
                s.left = left;
                s.part[0] = over;
            }
            __syncthreads();
            p.key |= s.digit << bit;
            p.spare = s.left;
            above += s.part[0];
        }
        if (kByMass) { // the weight that is left, in tokens of this one's
            const uint64_t w = r.key_weight(p.key);
            p.spare = w ? (p.spare + w - 1) / w : 1;
        }
        __syncthreads();
        return p;
    }
};

// ------------------------------------------------------------------------------------------------
// sorting in LDS
// ------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int index) { return uint64_t(key) << 32 | uint32_t(~index); }
__device__ __forceinline__ int index_of(uint64_t entry) { return int(~uint32_t(entry)); }

// Waits for the other threads of what shares stretches of `stride` pairs: a wave's LDS accesses are in order.
template <int kT> __device__ __forceinline__ void sort_wait(int stride) {
    if (kT > kWave && stride > kWave)
        __syncthreads();
    else {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// Sorts n (a power of two) entries, the largest first. Pairs of a stride up to 64 lie in the 128 entries that one wave
// takes, and need no barrier between the steps.
template <int kT> __device__ void sort_down(uint64_t *v, int n) {
    __syncthreads();
    for (int k = 2; k <= n; k *= 2)
        for (int j = k / 2; j > 0; j /= 2) {
            for (int p = threadIdx.x; p < n / 2; p += kT) {
                const int i = 2 * p - (p & (j - 1));
                const uint64_t a = v[i], b = v[i + j];
                if ((a < b) == ((i & k) == 0)) {
                    v[i] = b;
                    v[i + j] = a;
                }
            }
            sort_wait<kT>(std::max(j, j > 1 ? j / 2 : k));
        }
    __syncthreads();
}

__device__ __forceinline__ int power_of_two(int n) { return n <= 2 ? 2 : 1 << (32 - __builtin_clz(unsigned(n - 1))); }

// ------------------------------------------------------------------------------------------------
// short rows
// ------------------------------------------------------------------------------------------------
constexpr int kOwn = 8; // logits of a thread

template <typename T, int kT>
__global__ void __launch_bounds__(kT) small_kernel(const T *logits, Args a) {
    using B = Block<kT>;
    __shared__ typename B::Shared s;
    __shared__ uint64_t list[kOwn * kT];
    __shared__ uint64_t last;
    const int tid = threadIdx.x, each = (a.V + kT - 1) / kT, from = tid * each;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        float v[kOwn], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            v[i] = i < each && from + i < a.V ? float(x[from + i]) : -INFINITY;
            m = larger(m, v[i]);
        }
        m = B::max(m, s);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        Row r(m, p, a.shift);
        r.floor = floor_key(r.m, p.scale, p.least, key_of(m));
        uint64_t w[kOwn], total = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            w[i] = i < each && from + i < a.V ? r.weight(v[i]) : 0;
            total += w[i];
        }
        total = B::sum(total, s);
        uint64_t lowest = entry_of(r.floor, -1); // entries from here on are kept
        if (p.top_k < a.V || p.fraction < kOne) {
            const int n = power_of_two(a.V);
            __syncthreads();
            if (tid == 0)
                last = 0;
            for (int i = tid; i < n; i += kT)
                if (i >= a.V)
                    list[i] = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                if (i < each && from + i < a.V) {
                    const uint32_t k = key_of(v[i]);
                    list[from + i] = k >= r.floor ? entry_of(k, from + i) : 0;
                }
            sort_down<kT>(list, n);
            const int share = std::max(n / kT, 1);
            uint64_t sorted[kOwn], mine = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                const int at = tid * share + i;
                const uint64_t e = i < share && at < std::min(n, p.top_k) ? list[at] : 0;
                sorted[i] = e ? r.key_weight(uint32_t(e >> 32)) : 0;
                mine += sorted[i];
            }
            uint64_t all;
            uint64_t sum = B::before(mine, all, s);
            if (p.fraction < kOne) {
                const uint64_t target = std::max(share_up(all, p.fraction), uint64_t(1));
                if (sum < target && target <= sum + mine)
#pragma unroll
                    for (int i = 0; i < kOwn; ++i) {
                        if (sum < target && target <= sum + sorted[i])
                            last = list[tid * share + i];
                        sum += sorted[i];
                    }
            } else if (tid == 0)
                last = list[p.top_k - 1]; // 0 where min_p keeps fewer
            __syncthreads();
            lowest = std::max(lowest, last);
        }
        uint64_t mine = 0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (entry_of(key_of(v[i]), from + i) < lowest)
                w[i] = 0;
            mine += w[i];
        }
        uint64_t kept;
        uint64_t sum = B::before(mine, kept, s);
        const uint64_t target = share_down(kept, p.at);
        if (sum <= target && target < sum + mine)
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (sum <= target && target < sum + w[i])
                    finish_row(a, row, r, from + i, v[i], kept, total);
                sum += w[i];
            }
    }
}

// ------------------------------------------------------------------------------------------------
// the digest of a row
// ------------------------------------------------------------------------------------------------
constexpr int kPart = 2048, kSeg = 128, kSegs = kPart / kSeg;
constexpr int kMostParts = (1 << 19) / kPart; // longer rows are read again and again by wide_row

// 16 bytes of logits. A row may start anywhere, so what it is read through claims no alignment.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef type unaligned __attribute__((aligned(sizeof(T))));
};

// A wave reads a part in kLoads loads of 64 vectors; the 16 lanes of a quarter hold a segment in 16 / kSegs * kLoads of
// them, which is one load of 2-byte logits and two of 4-byte ones.
template <typename T> struct Part {
    static constexpr int N = Vec<T>::N, kLoads = kPart / kWave / N, kSame = kLoads / 4;
    // the lane's first element of a load
    static __device__ __forceinline__ int at(int load, int lane) { return (load * kWave + lane) * N; }
    static __device__ __forceinline__ void read(const T *x, int len, int lane, float (&v)[kLoads * N]) {
        typename Vec<T>::type q[kLoads];
        if (len >= kPart) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                q[j] = *reinterpret_cast<const typename Vec<T>::unaligned *>(x + at(j, lane));
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j) {
                q[j] = typename Vec<T>::type(T(-INFINITY));
                if (at(j, lane) + N <= len)
                    q[j] = *reinterpret_cast<const typename Vec<T>::unaligned *>(x + at(j, lane));
                else
#pragma unroll
                    for (int i = 0; i < N; ++i)
                        if (at(j, lane) + i < len)
                            q[j][i] = x[at(j, lane) + i];
            }
        }
#pragma unroll
        for (int k = 0; k < kLoads * N; ++k)
            v[k] = float(q[k / N][k % N]);
    }
};

struct Digest {
    uint64_t *mass; // [n][parts]: weights relative to the part's own largest logit
    float *top;     // [n][parts]
    float *seg;     // [n][parts][kSegs]
    int parts;
};

// Whether the weights of a whole row are asked for: for its log-probabilities, or because nothing but top_p, or nothing
// at all, cuts it off.
__device__ __forceinline__ bool needs_mass(const Args &a, const Params &p) {
    return a.logp || a.log_kept || (p.top_k == a.V && p.least == -INFINITY);
}

template <int kCtrl> __device__ __forceinline__ float row_larger(float v) {
    return larger(v, __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), kCtrl, 0xf, 0xf, true)));
}

template <typename T>
__global__ void __launch_bounds__(256) scan_kernel(const T *logits, Args a, Digest g) {
    using P = Part<T>;
    constexpr int kN = P::kLoads * P::N;
    const int lane = threadIdx.x % kWave;
    const int64_t items = a.n * g.parts;
    for (int64_t item = blockIdx.x * int64_t(4) + threadIdx.x / kWave; item < items; item += gridDim.x * int64_t(4)) {
        const int64_t row = item / g.parts;
        const int part = int(item - row * g.parts);
        const Params p = params_of(a, row);
        float v[kN];
        P::read(logits + row * a.stride + part * kPart, a.V - part * kPart, lane, v);
        float m = -INFINITY, mine = -INFINITY;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float top = -INFINITY;
#pragma unroll
            for (int k = 0; k < P::kSame * P::N; ++k)
                top = larger(top, v[i * P::kSame * P::N + k]);
            top = row_larger<0x128>(top); // rotations by 8, 4, 2 and 1 among 16 lanes
            top = row_larger<0x124>(top);
            top = row_larger<0x122>(top);
            top = row_larger<0x121>(top);
            mine = lane % 16 == i ? top : mine;
            m = larger(m, top);
        }
        m = larger(m, __shfl_xor(m, 16));
        m = larger(m, __shfl_xor(m, 32));
        if (lane % 16 < 4)
            g.seg[item * kSegs + lane % 16 * 4 + lane / 16] = mine;
        uint64_t mass = 0;
        if (needs_mass(a, p) && p.scale != 0.0 && m < INFINITY && m > -INFINITY) {
            const Row r(m, p, a.shift);
#pragma unroll
            for (int k = 0; k < kN; ++k)
                mass += r.weight(v[k]);
            mass = wave_sum(mass);
        }
        if (lane == 0) {
            g.top[item] = m;
            g.mass[item] = mass;
        }
    }
}

// ------------------------------------------------------------------------------------------------
// the token of a row
// ------------------------------------------------------------------------------------------------
constexpr int kPick = 512;
constexpr int kList = 2048; // candidates
constexpr int kFine = 1024; // bins of wide_row
using PickBlock = Block<kPick>;

struct PickShared {
    uint64_t list[kList];
    union {
        struct {
            uint64_t mass[kFine];
            uint32_t count[kFine];
        };
        struct {
            uint64_t part_mass[kMostParts];
            uint32_t part_ties[kMostParts];
        };
        uint16_t segs[kMostParts * kSegs];
    };
    PickBlock::Shared block;
    uint64_t found_mass, found_left;
    uint32_t found_key;
    int found, n;
    bool spoiled;
    int ge[2][PickBlock::kWaves];
};

// The token among the logits of one part, at which the running sum of weights (relative to r.m) passes `target`. Keys above
// the place's count, and the first `spare` of its own.
template <typename T>
__device__ void pick_in_part(const Args &a, int64_t row, const T *x, int part, const Row &weights, const Row &r, Place place,
                             uint64_t target, uint64_t kept, uint64_t total, PickShared &s) {
    constexpr int kEach = kPart / kPick;
    const int from = part * kPart + threadIdx.x * kEach;
    float v[kEach];
    uint64_t ties = 0, unused;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        v[i] = from + i < a.V ? float(x[from + i]) : -INFINITY;
        ties += from + i < a.V && key_of(v[i]) == place.key;
    }
    uint64_t rank = PickBlock::before(ties, unused, s.block);
    uint64_t w[kEach], mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const uint32_t k = key_of(v[i]);
        const bool tie = k == place.key;
        w[i] = from + i < a.V && (k > place.key || (tie && rank < place.spare)) ? weights.weight(v[i]) : 0;
        rank += tie;
        mine += w[i];
    }
    uint64_t all;
    uint64_t sum = PickBlock::before(mine, all, s.block);
    if (sum <= target && target < sum + mine)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (sum <= target && target < sum + w[i])
                finish_row(a, row, r, from + i, v[i], kept, total);
            sum += w[i];
        }
}

// The bin of a logit by its distance from the largest, which never decreases as logits do; kFine: its weight is 0. Halves,
// because the distance itself may be no float.
struct Bins {
    float half, step;
    __device__ __forceinline__ Bins(const Row &r)
        : half(float(r.m) * 0.5f), step(fminf(float(r.scale) * (2.0f * kFine / 31.5f), 3.402823466e38f)) {}
    __device__ __forceinline__ int of(float x) const {
        const float d = (half - x * 0.5f) * step;
        return d < float(kFine) ? int(d) : kFine;
    }
};

// Where the count (kByMass: the weights) from the top reaches `target`, which it does within the bins; `above` receives the
// weights above the place's key.
template <bool kByMass, typename T>
__device__ Place place_in_bins(const Args &a, const T *x, const Row &r, const Bins &bins, uint64_t target, uint64_t &above, PickShared &s) {
    constexpr int kEach = kFine / kPick;
    uint64_t mine = 0, mine_mass = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = threadIdx.x * kEach + i;
        mine += kByMass ? s.mass[b] : s.count[b];
        mine_mass += s.mass[b];
    }
    uint64_t sum = PickBlock::before(mine, all, s.block);
    uint64_t sum_mass = kByMass ? sum : PickBlock::before(mine_mass, all, s.block);
    if (sum < target && target <= sum + mine)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int b = threadIdx.x * kEach + i;
            const uint64_t here = kByMass ? s.mass[b] : s.count[b];
            if (sum < target && target <= sum + here) {
                s.found = b;
                s.found_left = target - sum;
                s.found_mass = sum_mass;
            }
            sum += here;
            sum_mass += s.mass[b];
        }
    if (threadIdx.x == 0)
        s.n = 0;
    __syncthreads();
    const int bin = s.found;
    const uint64_t left = s.found_left;
    const uint32_t members = s.count[bin];
    above = s.found_mass;
    if (members > kList) { // a great many near equals: place_of overwrites the bins
        __syncthreads();
        s.spoiled = true;
        return PickBlock::place_of<kByMass>(x, a.V, r, target, above, s.mass, s.count, s.block);
    }
    for (int i = threadIdx.x; i < a.V; i += kPick) {
        const float v = float(x[i]);
        const uint32_t k = key_of(v);
        if (k >= r.floor && bins.of(v) == bin)
            s.list[atomicAdd(&s.n, 1)] = entry_of(k, i);
    }
    __syncthreads();
    const int n = power_of_two(int(members));
    for (int i = int(members) + threadIdx.x; i < n; i += kPick)
        s.list[i] = 0;
    sort_down<kPick>(s.list, n);
    // the place is that of an entry: its key, and how many entries of this key there are down to it
    constexpr int kSome = kList / kPick;
    const int share = std::max(n / kPick, 1);
    uint64_t w[kSome];
    mine = 0;
    mine_mass = 0;
#pragma unroll
    for (int i = 0; i < kSome; ++i) {
        const int at = threadIdx.x * share + i;
        const bool in = i < share && at < int(members);
        w[i] = in ? r.key_weight(uint32_t(s.list[at] >> 32)) : 0;
        mine += kByMass ? w[i] : in;
        mine_mass += w[i];
    }
    sum = PickBlock::before(mine, all, s.block);
    sum_mass = kByMass ? sum : PickBlock::before(mine_mass, all, s.block);
    if (sum < left && left <= sum + mine)
#pragma unroll
        for (int i = 0; i < kSome; ++i) {
            const int at = threadIdx.x * share + i;
            const uint64_t here = kByMass ? w[i] : uint64_t(i < share && at < int(members));
            if (sum < left && left <= sum + here)
                s.found = at;
            sum += here;
        }
    __syncthreads();
    const int at = s.found;
    Place p{uint32_t(s.list[at] >> 32), 0};
    // entries of the key before this one, and the weights before the first of them
    uint64_t same = 0, over = 0;
#pragma unroll
    for (int i = 0; i < kSome; ++i) {
        const int k = threadIdx.x * share + i;
        if (i < share && k <= at) {
            const bool tie = uint32_t(s.list[k] >> 32) == p.key;
            same += tie;
            over += tie ? 0 : w[i];
        }
    }
    p.spare = PickBlock::sum(same, s.block);
    above += PickBlock::sum(over, s.block);
    __syncthreads();
    return p;
}

// Counts and weights of the logits in each bin.
template <typename T>
__device__ void fill_bins(const Args &a, const T *x, const Row &r, const Bins &bins, PickShared &s) {
    __syncthreads();
    for (int i = threadIdx.x; i < kFine; i += kPick)
        s.mass[i] = s.count[i] = 0;
    s.spoiled = false;
    __syncthreads();
    for (int i = threadIdx.x; i < a.V; i += kPick) {
        const float v = float(x[i]);
        const int bin = bins.of(v);
        if (bin < kFine && key_of(v) >= r.floor) {
            atomicAdd(&s.count[bin], 1u);
            atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[bin]), (unsigned long long)r.weight(v));
        }
    }
    __syncthreads();
}

// A row whose kept tokens are too many for a list: weights and counts in bins of the distance from the largest logit, the
// bin of the last kept token looked through, and the kept weights of every part of the row.
template <typename T>
__device__ void wide_row(const Args &a, int64_t row, const T *x, const Row &r, const Params &p, uint64_t total, PickShared &s) {
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    Place place{r.floor ? r.floor - 1 : 0, 0};
    if (p.top_k < a.V || p.fraction < kOne) {
        const Bins bins(r);
        fill_bins(a, x, r, bins, s);
        uint64_t there = 0, inside = 0, above;
        for (int i = tid; i < kFine; i += kPick) {
            there += s.count[i];
            inside += s.mass[i];
        }
        there = PickBlock::sum(there, s.block);
        inside = PickBlock::sum(inside, s.block);
        if (uint64_t(p.top_k) < there) { // otherwise what it cuts off has no weight
            place = place_in_bins<false>(a, x, r, bins, uint64_t(p.top_k), above, s);
            inside = above + place.spare * r.key_weight(place.key);
            if (p.fraction < kOne && s.spoiled)
                fill_bins(a, x, r, bins, s);
        }
        if (p.fraction < kOne)
            place = place_in_bins<true>(a, x, r, bins, std::max(share_up(inside, p.fraction), uint64_t(1)), above, s);
    }
    // the kept weights of the parts, and how many of the place's own key each has
    __syncthreads();
    const int parts = (a.V + kPart - 1) / kPart;
    const uint64_t level = place.spare ? r.key_weight(place.key) : 0;
    for (int q = wave; q < parts; q += PickBlock::kWaves) {
        float v[kPart / kWave];
        Part<T>::read(x + q * kPart, a.V - q * kPart, lane, v);
        uint64_t mass = 0;
        uint32_t ties = 0;
#pragma unroll
        for (int k = 0; k < kPart / kWave; ++k) {
            const uint32_t key = key_of(v[k]);
            mass += key > place.key ? r.weight(v[k]) : 0;
            ties += key == place.key;
        }
        mass = wave_sum(mass);
        ties = wave_sum(ties);
        if (lane == 0) {
            s.part_mass[q] = mass;
            s.part_ties[q] = ties;
        }
    }
    __syncthreads();
    static_assert(kMostParts <= kPick, "a part a thread");
    uint64_t all_ties, kept;
    const uint64_t ties = tid < parts ? s.part_ties[tid] : 0;
    const uint64_t ties_before = PickBlock::before(ties, all_ties, s.block);
    const uint64_t spare = place.spare > ties_before ? place.spare - ties_before : 0;
    const uint64_t mine = tid < parts ? s.part_mass[tid] + std::min(ties, spare) * level : 0;
    const uint64_t sum = PickBlock::before(mine, kept, s.block);
    const uint64_t target = share_down(kept, p.at);
    if (sum <= target && target < sum + mine) {
        s.found = tid;
        s.found_left = target - sum;
        s.found_mass = spare;
    }
    __syncthreads();
    place.spare = s.found_mass;
    pick_in_part(a, row, x, s.found, r, r, place, s.found_left, kept, total, s);
}

// The number of segments whose largest logit has a key of at least k.
__device__ __forceinline__ int segments_from(const uint32_t (&keys)[kMostParts * kSegs / kPick], int segs, uint32_t k, int step, PickShared &s) {
    int n = 0;
#pragma unroll
    for (int i = 0; i < kMostParts * kSegs / kPick; ++i)
        if (i * kPick < segs)
            n += __builtin_popcountll(__ballot(keys[i] >= k));
    if (threadIdx.x % kWave == 0)
        s.ge[step & 1][threadIdx.x / kWave] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < PickBlock::kWaves; ++w)
        n += s.ge[step & 1][w];
    return n;
}

// The token from s.list[0, n), which holds every token down to some place of the order. `whole`: all that min_p and top_k
// leave is among them; otherwise `total` is the weight of all that top_p is a share of. False where the list ends before the
// last kept token does.
template <typename T>
__device__ bool pick_from_list(const Args &a, int64_t row, const Row &r, const Params &p, int n, bool whole, uint64_t total, PickShared &s) {
    constexpr int kEach = kList / kPick;
    const int padded = power_of_two(n), tid = threadIdx.x;
    __syncthreads();
    for (int i = n + tid; i < padded; i += kPick)
        s.list[i] = 0;
    sort_down<kPick>(s.list, padded);
    int many = std::min(n, p.top_k), share = std::max(padded / kPick, 1);
    uint64_t w[kEach], mine = 0, kept;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = tid * share + i;
        w[i] = i < share && at < many ? r.key_weight(uint32_t(s.list[at] >> 32)) : 0;
        mine += w[i];
    }
    uint64_t sum = PickBlock::before(mine, kept, s.block);
    if (p.fraction < kOne) {
        const uint64_t target = std::max(share_up(whole ? kept : total, p.fraction), uint64_t(1));
        if (kept < target)
            return false;
        if (sum < target && target <= sum + mine)
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                if (sum < target && target <= sum + w[i]) {
                    s.found = tid * share + i + 1;
                    s.found_mass = sum + w[i];
                }
                sum += w[i];
            }
        __syncthreads();
        many = s.found;
        kept = s.found_mass;
    }
    const uint64_t target = share_down(kept, p.at);
    // in the order of the vocabulary
    const int sorted = power_of_two(many);
    for (int i = tid; i < sorted; i += kPick) {
        const uint64_t e = s.list[i];
        s.list[i] = i < many ? ~(uint64_t(uint32_t(index_of(e))) << 32 | e >> 32) : 0;
    }
    sort_down<kPick>(s.list, sorted);
    share = std::max(sorted / kPick, 1);
    mine = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int at = tid * share + i;
        w[i] = i < share && at < many ? r.key_weight(uint32_t(~s.list[at])) : 0;
        mine += w[i];
    }
    uint64_t unused;
    sum = PickBlock::before(mine, unused, s.block);
    if (sum <= target && target < sum + mine)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (sum <= target && target < sum + w[i]) {
                const uint64_t e = ~s.list[tid * share + i];
                finish_row(a, row, r, int(e >> 32), float_of(uint32_t(e)), kept, total);
            }
            sum += w[i];
        }
    return true;
}

template <typename T>
__global__ void __launch_bounds__(kPick) pick_kernel(const T *logits, Args a, Digest g) {
    __shared__ PickShared s;
    constexpr int kKeys = kMostParts * kSegs / kPick;
    const int tid = threadIdx.x, segs = g.parts * kSegs;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        const float top = tid < g.parts ? g.top[row * g.parts + tid] : -INFINITY;
        const uint64_t part_mass = tid < g.parts ? g.mass[row * g.parts + tid] : 0;
        const float m = PickBlock::max(top, s.block);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        Row r(m, p, a.shift);
        // the parts' weights, relative to the row's largest logit
        const uint64_t mine = part_mass ? uint64_t(rint(double(part_mass) * power_of(fmax(double(top) - r.m, r.far), r.c, 0))) : 0;
        uint64_t total;
        const uint64_t sum = PickBlock::before(mine, total, s.block);
        if (p.top_k == a.V && p.fraction == kOne && p.least == -INFINITY) {
            const uint64_t target = share_down(total, p.at);
            if (sum <= target && target < sum + mine) {
                s.found = tid;
                s.found_key = key_of(top);
                // as far into the part's own sum
                s.found_left = mine == part_mass ? target - sum : std::min(uint64_t(double(target - sum) / double(mine) * double(part_mass)), part_mass - 1);
            }
            __syncthreads();
            const Row own(float_of(s.found_key), p, a.shift);
            pick_in_part(a, row, x, s.found, own, r, Place{0, 0}, s.found_left, total, total, s);
            __syncthreads();
            continue;
        }
        r.floor = floor_key(r.m, p.scale, p.least, key_of(m));
        int want = 0;
        if (p.top_k < a.V)
            want = p.top_k <= segs / 2 ? p.top_k : 0;
        else if (r.floor == 0)
            want = std::min(segs / 2, 128);
        bool wide = want == 0 && r.floor == 0, whole = true;
        uint32_t low = r.floor;
        uint32_t keys[kKeys];
#pragma unroll
        for (int i = 0; i < kKeys; ++i)
            keys[i] = i * kPick + tid < segs ? key_of(g.seg[row * segs + i * kPick + tid]) : 0;
        if (want) {
            // the largest key (or one not far below it) that the largest logits of `want` segments have
            uint32_t from = 0, to = key_of(m) + 1;
            for (int step = 0; to - from > 1; ++step) {
                const uint32_t k = from + (to - from) / 2;
                const int n = segments_from(keys, segs, k, step, s);
                if (n >= want)
                    from = k;
                else
                    to = k;
                if (n >= want && n <= want + want / 8 + 8)
                    break;
            }
            whole = p.top_k < a.V || from <= low;
            low = std::max(low, from);
        }
        if (!wide) {
            // segments that have a candidate, and their candidates
            __syncthreads();
            if (tid == 0)
                s.found = s.n = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < kKeys; ++i)
                if (i * kPick + tid < segs && keys[i] >= low)
                    s.segs[atomicAdd(&s.found, 1)] = uint16_t(i * kPick + tid);
            __syncthreads();
            const int many = s.found;
            for (int i = tid / 16; i < many; i += kPick / 16) {
                const int seg = s.segs[i], quarter = seg % 4, load = seg / 4 % 4 * Part<T>::kSame;
#pragma unroll
                for (int j = 0; j < Part<T>::kSame; ++j) {
                    const int at = seg / kSegs * kPart + Part<T>::at(load + j, quarter * 16 + tid % 16);
#pragma unroll
                    for (int k = 0; k < Part<T>::N; ++k)
                        if (at + k < a.V) {
                            const uint32_t key = key_of(float(x[at + k]));
                            if (key >= low) {
                                const int to = atomicAdd(&s.n, 1);
                                if (to < kList)
                                    s.list[to] = entry_of(key, at + k);
                            }
                        }
                }
            }
            __syncthreads();
            const int n = s.n;
            wide = n > kList || !pick_from_list<T>(a, row, r, p, n, whole, total, s);
        }
        if (wide)
            wide_row(a, row, x, r, p, total, s);
        __syncthreads();
    }
}

// Rows too long for a digest's sums: read once for the largest logit, once for the weights, and then by wide_row's means.
constexpr int kLong = 1024;
template <typename T>
__global__ void __launch_bounds__(kLong) long_kernel(const T *logits, Args a) {
    using B = Block<kLong>;
    __shared__ B::Shared s;
    __shared__ uint64_t mass[kBins];
    __shared__ uint32_t count[kBins];
    __shared__ uint64_t part[B::kWaves], ties[B::kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        float m = -INFINITY;
        for (int i = tid; i < a.V; i += kLong)
            m = larger(m, float(x[i]));
        m = B::max(m, s);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        Row r(m, p, a.shift);
        r.floor = floor_key(r.m, p.scale, p.least, key_of(m));
        uint64_t total = 0, inside = 0, there = 0, above;
        for (int i = tid; i < a.V; i += kLong) {
            const float v = float(x[i]);
            const uint64_t w = r.weight(v);
            const bool in = key_of(v) >= r.floor;
            total += w;
            inside += in ? w : 0;
            there += in;
        }
        total = B::sum(total, s);
        inside = B::sum(inside, s);
        there = B::sum(there, s);
        Place place{r.floor ? r.floor - 1 : 0, 0};
        if (uint64_t(p.top_k) < there) {
            place = B::template place_of<false>(x, a.V, r, uint64_t(p.top_k), above, mass, count, s);
            inside = above + place.spare * r.key_weight(place.key);
        }
        if (p.fraction < kOne)
            place = B::template place_of<true>(x, a.V, r, std::max(share_up(inside, p.fraction), uint64_t(1)), above, mass, count, s);
        // waves take stretches of the vocabulary; a token's equals before it decide whether it is kept
        const int each = (a.V + kLong - 1) / kLong * kWave;
        const int from = int(std::min(int64_t(wave) * each, int64_t(a.V))), to = int(std::min(int64_t(from) + each, int64_t(a.V)));
        const uint64_t level = place.spare ? r.key_weight(place.key) : 0;
        uint64_t my_mass = 0, my_ties = 0;
        for (int64_t i = int64_t(from) + lane; i < to; i += kWave) {
            const float v = float(x[i]);
            const uint32_t k = key_of(v);
            my_mass += k > place.key ? r.weight(v) : 0;
            my_ties += k == place.key;
        }
        my_mass = wave_sum(my_mass);
        my_ties = wave_sum(my_ties);
        __syncthreads();
        if (lane == 0) {
            part[wave] = my_mass;
            ties[wave] = my_ties;
        }
        __syncthreads();
        uint64_t kept = 0, sum = 0, equal = 0, rank = 0;
        for (int w = 0; w < B::kWaves; ++w) {
            if (w == wave) {
                sum = kept;
                rank = equal;
            }
            kept += part[w] + std::min(ties[w], place.spare - std::min(equal, place.spare)) * level;
            equal += ties[w];
        }
        const uint64_t target = share_down(kept, p.at);
        const bool mine = sum <= target;
        for (int64_t i = int64_t(from) + lane; i - lane < to && sum <= target; i += kWave) {
            const bool in = i < to;
            const float v = in ? float(x[i]) : -INFINITY;
            const uint32_t k = key_of(v);
            const uint64_t tied = __ballot(in && k == place.key);
            const uint64_t my_rank = rank + __builtin_popcountll(tied & ((uint64_t(1) << lane) - 1));
            const bool keep = in && (k > place.key || (k == place.key && my_rank < place.spare));
            const uint64_t with = sum + wave_scan(keep ? r.weight(v) : 0);
            const uint64_t past = __ballot(with > target);
            if (mine && past && lane == __builtin_ctzll(past))
                finish_row(a, row, r, int(i), v, kept, total);
            rank += __builtin_popcountll(tied);
            sum = __shfl(with, kWave - 1);
        }
        __syncthreads();
    }
}

// How rows of V tokens are taken.
struct Plan {
    int group; // of small_kernel; 0: a digest
    int parts; // 0 and no group: long_kernel
};

Plan plan_of(int64_t V) {
    if (V <= kOwn * kWave)
        return {kWave, 0};
    if (V <= kOwn * 256)
        return {256, 0};
    if (V < int64_t(kMostParts) * kPart)
        return {0, int((V + kPart - 1) / kPart)};
    return {0, 0};
}

constexpr int64_t kPartBytes = sizeof(uint64_t) + sizeof(float) * (1 + kSegs);

int size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }

using treeens::set_error;

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

int check_sizes(int32_t dtype, int64_t n, int64_t V) {
    if (dtype != TREE_ENS_F32 && dtype != TREE_ENS_BF16 && dtype != TREE_ENS_F16)
        return set_error(TREE_ENS_E_ARG, "dtype must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
    if (n < 0 || V < 1 || V > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and n_vocab in [1, INT32_MAX]");
    if (n > INT64_MAX / kPartBytes / kMostParts)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be within memory");
    return TREE_ENS_OK;
}

} // namespace

extern "C" {

int tree_ens_sample_workspace(int32_t dtype, int64_t n_tokens, int64_t n_vocab, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (int rc = check_sizes(dtype, n_tokens, n_vocab))
        return rc;
    *bytes = n_tokens * plan_of(n_vocab).parts * kPartBytes;
    return TREE_ENS_OK;
}

int tree_ens_sample(void *stream, const void *logits, int32_t dtype, int64_t n_tokens, int64_t n_vocab, int64_t row_stride,
                    const double *uniform, float scale, int32_t top_k, float top_p, float min_p, const float *row_scale,
                    const int32_t *row_top_k, const float *row_top_p, const float *row_min_p, int64_t *tokens, float *logp,
                    float *log_kept, void *workspace, int64_t workspace_bytes) {
    treeens::clear_error();
    if (int rc = check_sizes(dtype, n_tokens, n_vocab))
        return rc;
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
    const Plan plan = plan_of(n_vocab);
    if (const int64_t need = n_tokens * plan.parts * kPartBytes) {
        if (!workspace || workspace_bytes < need)
            return set_error(TREE_ENS_E_ARG, "workspace is NULL or smaller than " + std::to_string(need) + " bytes");
        if (misaligned(workspace, 16))
            return set_error(TREE_ENS_E_ARG, "workspace must be 16-byte aligned");
    }
    int shift = 44;
    while (n_vocab >> (63 - shift))
        --shift;
    const Args a{n_tokens, row_stride, int(n_vocab), shift, uniform, scale, top_p, min_p, top_k, row_scale, row_top_p,
                 row_min_p, row_top_k, tokens, logp, log_kept};
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const dim3 rows(unsigned(std::min(n_tokens, kMaxBlocks)));
    (void)hipGetLastError();
    const auto launch = [&](auto *type) {
        using T = std::decay_t<decltype(*type)>;
        const T *x = static_cast<const T *>(logits);
        if (plan.group == kWave)
            hipLaunchKernelGGL((small_kernel<T, kWave>), rows, dim3(kWave), 0, s, x, a);
        else if (plan.group)
            hipLaunchKernelGGL((small_kernel<T, 256>), rows, dim3(256), 0, s, x, a);
        else if (plan.parts) {
            Digest g;
            g.parts = plan.parts;
            g.mass = static_cast<uint64_t *>(workspace);
            g.top = reinterpret_cast<float *>(g.mass + n_tokens * plan.parts);
            g.seg = g.top + n_tokens * plan.parts;
            const int64_t blocks = (n_tokens * plan.parts + 3) / 4;
            hipLaunchKernelGGL(scan_kernel<T>, dim3(unsigned(std::min(blocks, kMaxBlocks))), dim3(256), 0, s, x, a, g);
            hipLaunchKernelGGL(pick_kernel<T>, rows, dim3(kPick), 0, s, x, a, g);
        } else
            hipLaunchKernelGGL(long_kernel<T>, rows, dim3(kLong), 0, s, x, a);
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
