// sample.hip -- one token for each row of logits from a given random number, under temperature, top-k,
// min-p and top-p, on gfx950.
//
// Weights w = exp(scale * (x - max x)) are taken in double and rounded to whole numbers of 2^-shift where tokens are decided
// on, so that sums are exact in any order. Tokens are kept down to a last one in the order of the logits (the largest first,
// equal ones by index): top-k and top-p are both the search for the place in that order where a running count or a running sum
// of weights reaches a target. Nothing is sorted.
//
// Rows of up to 2,048 tokens go to one workgroup (small_kernel). Of longer rows scan_kernel reads every logit once and
// leaves a digest: the largest logit of every 128, and the largest and the weights of every 2,048. pick_kernel, a
// workgroup a row, finds from it the few segments that can hold a kept token, lists their candidates and takes the
// token; where nothing is cut off, the digest's weights lead to the 2,048 logits that hold it. Rows whose kept tokens are
// more than its list holds are read twice more, by wide_place_kernel and wide_pick_kernel, up to 16 workgroups to a row. What
// a row's token and log-probabilities are depends on the row alone, since parts, sums and lists do.
//
// Times below are of kernels on one MI355X, in these cases: A 1 x 128,000 bf16, top-p 0.95; B 256 x 128,000 bf16, nothing cut
// off; C 512 x 131,072 fp16, parameters by row; D 2,048 x 32,001 bf16, min-p 0.05; E 64 x 128,000 fp32 at scale 0.75, top-p 0.98,
// which thousands of tokens make up.
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

// a / b to about 2^-50, in a third of an exact division's instructions.
__device__ __forceinline__ double ratio(double a, double b) {
    double r = __builtin_amdgcn_rcp(b);
    r = fma(fma(-b, r, 1.0), r, r);
    r = fma(fma(-b, r, 1.0), r, r);
    return a * r;
}

// The natural logarithm of a number of at least 2^-1000, to about 2^-45: of the exponent, and 2 atanh of (m - 1) / (m + 1) for
// the rest m, within sqrt(2) of 1, by its series. A few dozen instructions where the library's has hundreds, which a
// workgroup that comes by once has to fetch first.
__device__ __forceinline__ double log_of(double x) {
    const int high = __double2hiint(x), n = (high - 0x3fe6a09e) >> 20; // 0x3fe6a09e...: sqrt(1/2)
    const double m = __hiloint2double(high - (n << 20), __double2loint(x));
    const double q = ratio(m - 1.0, m + 1.0), y = q * q;
    double p = 1.0 / 15;
    p = fma(p, y, 1.0 / 13);
    p = fma(p, y, 1.0 / 11);
    p = fma(p, y, 1.0 / 9);
    p = fma(p, y, 1.0 / 7);
    p = fma(p, y, 1.0 / 5);
    p = fma(p, y, 1.0 / 3);
    return fma(double(n), 0.6931471805599453, 2.0 * fma(p * y, q, q));
}

__device__ __forceinline__ double scale_of(const Args &a, int64_t row) {
    const float scale = a.row_scale ? a.row_scale[row] : a.scale;
    return scale > 0.0f && scale < INFINITY ? double(scale) : 0.0;
}
__device__ __forceinline__ int top_k_of(const Args &a, int64_t row) {
    const int k = a.row_top_k ? a.row_top_k[row] : a.top_k;
    return k > 0 && k < a.V ? k : a.V;
}
__device__ __forceinline__ float min_p_of(const Args &a, int64_t row) { return a.row_min_p ? a.row_min_p[row] : a.min_p; }

__device__ __forceinline__ bool wants_logp(const Args &a) { return a.logp || a.log_kept; }

// What the weights of a whole row are for: they decide on tokens where nothing but top_p, or nothing at all, cuts it off, and are
// exact then; otherwise log-probabilities ask for what is not kept, for which single precision does.
enum class Mass { kNone, kExact, kQuick };
__device__ __forceinline__ Mass mass_of(const Args &a, int64_t row) {
    if (top_k_of(a, row) == a.V && !(min_p_of(a, row) > 0.0f))
        return Mass::kExact;
    // below the one scale a distance that is no float could have a weight, beyond the other the exponents' factor is none
    const unsigned exponent = __float_as_uint(float(scale_of(a, row))) >> 23;
    return !wants_logp(a) ? Mass::kNone : exponent < 127 - 100 || exponent >= 127 + 100 ? Mass::kExact : Mass::kQuick;
}

__device__ __forceinline__ Params params_of(const Args &a, int64_t row) {
    Params p;
    p.scale = scale_of(a, row);
    p.top_k = top_k_of(a, row);
    const float q = a.row_top_p ? a.row_top_p[row] : a.top_p;
    p.fraction = q < 1.0f ? uint64_t(double(fmaxf(q, 0.0f)) * 0x1p53) : kOne;
    const float m = min_p_of(a, row);
    p.least = m > 0.0f ? log_of(double(fminf(m, 1.0f))) : -INFINITY;
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

// 2^(d c + shift) for -1000 <= d c <= 0: the exponent taken apart into a whole number and a rest r within a half, and 2^r by
// the polynomial of degree 8 whose largest relative error there, 1.1e-12, is the smallest with p(0) = 1 (found by exchange).
// Double-precision multiply-adds run at the rate of single ones on this card.
__device__ __forceinline__ double power_of(double d, double c, int shift) {
    const double round = 0x1.8p52 + double(shift); // adding it leaves the whole number in the low bits
    const double t = fma(d, c, round), r = fma(d, c, round - t);
    double p = 0x1.663487d8abc81p-20;
    p = fma(p, r, 0x1.00ee071c7c030p-16);
    p = fma(p, r, 0x1.4306c1165a375p-13);
    p = fma(p, r, 0x1.5d872975c4ed2p-10);
    p = fma(p, r, 0x1.3b2ab7f3b3217p-7);
    p = fma(p, r, 0x1.c6b08defc25fdp-5);
    p = fma(p, r, 0x1.ebfbdff7c5a79p-3);
    p = fma(p, r, 0x1.62e42fef7a78bp-1);
    p = fma(p, r, 1.0);
    return __hiloint2double(__double2hiint(p) + (__double2loint(t) << 20), __double2loint(p));
}

// The whole number nearest to 0 <= v < 2^52, which adding 2^52 leaves in the low bits.
__device__ __forceinline__ uint64_t whole_of(double v) {
    return uint64_t(__double_as_longlong(v + 0x1p52)) & ((uint64_t(1) << 52) - 1);
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
    // within a few roundings of m + least / scale, as a rule
    const uint32_t near = key_of(fmaxf(float(m + least * __builtin_amdgcn_rcp(scale)), -3e38f));
    if (near - low > kWave && near + kWave < top) {
        const uint64_t yes = __ballot((double(float_of(near - kWave / 2 + lane)) - m) * scale >= least);
        const int first = yes ? __builtin_ctzll(yes) : kWave;
        if (first < kWave)
            top = near - kWave / 2 + first;
        if (first > 0)
            low = near - kWave / 2 + first - 1;
    }
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

// The larger one; NaN if either is.
__device__ __forceinline__ float larger(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A value of another lane by kCtrl, or 0 (the lane's own with kOwn) where there is none or kRows leaves the row of 16 out.
template <int kCtrl, int kRows, bool kOwn = false> __device__ __forceinline__ unsigned moved(unsigned v) {
    return unsigned(__builtin_amdgcn_update_dpp(kOwn ? int(v) : 0, int(v), kCtrl, kRows, 0xf, false));
}
template <int kCtrl, int kRows, bool kOwn = false> __device__ __forceinline__ uint64_t moved(uint64_t v) {
    return uint64_t(moved<kCtrl, kRows, kOwn>(unsigned(v >> 32))) << 32 | moved<kCtrl, kRows, kOwn>(unsigned(v));
}
template <int kCtrl, int kRows> __device__ __forceinline__ double moved(double v) {
    return __longlong_as_double(moved<kCtrl, kRows>(uint64_t(__double_as_longlong(v))));
}

// Sums over the lanes up to and with this one: within rows of 16, then the rows' ends are added to the rows behind them.
template <typename V> __device__ __forceinline__ V wave_scan(V v) {
    v += moved<0x111, 0xf>(v); // from 1, 2, 4 and 8 lanes before
    v += moved<0x112, 0xf>(v);
    v += moved<0x114, 0xf>(v);
    v += moved<0x118, 0xf>(v);
    v += moved<0x142, 0xa>(v); // the last lane of a row, to the second and fourth
    v += moved<0x143, 0xc>(v); // that of the first half, to the second
    return v;
}
__device__ __forceinline__ uint64_t last_lane(uint64_t v) {
    return uint64_t(unsigned(__builtin_amdgcn_readlane(int(v >> 32), kWave - 1))) << 32 |
           unsigned(__builtin_amdgcn_readlane(int(unsigned(v)), kWave - 1));
}
__device__ __forceinline__ double last_lane(double v) { return __longlong_as_double(last_lane(uint64_t(__double_as_longlong(v)))); }
template <typename V> __device__ __forceinline__ V wave_sum(V v) { return last_lane(wave_scan(v)); }

// Over the 16 lanes of a row, by rotations of 8, 4, 2 and 1.
template <int kCtrl> __device__ __forceinline__ int rotated(int v) { return __builtin_amdgcn_mov_dpp(v, kCtrl, 0xf, 0xf, true); }
template <int kCtrl> __device__ __forceinline__ float rotated(float v) { return __int_as_float(rotated<kCtrl>(__float_as_int(v))); }
template <int kCtrl> __device__ __forceinline__ double rotated(double v) {
    return __hiloint2double(rotated<kCtrl>(__double2hiint(v)), rotated<kCtrl>(__double2loint(v)));
}
__device__ __forceinline__ float row_max(float v) {
    v = larger(v, rotated<0x128>(v));
    v = larger(v, rotated<0x124>(v));
    v = larger(v, rotated<0x122>(v));
    return larger(v, rotated<0x121>(v));
}
__device__ __forceinline__ double row_sum(double v) {
    v += rotated<0x128>(v);
    v += rotated<0x124>(v);
    v += rotated<0x122>(v);
    return v + rotated<0x121>(v);
}
// A row's lanes hold the same: the other rows' too.
__device__ __forceinline__ float of_row(float v, int row) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * row)); }
__device__ __forceinline__ double of_row(double v, int row) {
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), 16 * row), __builtin_amdgcn_readlane(__double2loint(v), 16 * row));
}

template <int kCtrl, int kRows = 0xf> __device__ __forceinline__ float moved_larger(float v) {
    return larger(v, __uint_as_float(moved<kCtrl, kRows, true>(__float_as_uint(v))));
}
template <int kCtrl, int kRows = 0xf> __device__ __forceinline__ uint64_t moved_larger(uint64_t v) {
    return std::max(v, moved<kCtrl, kRows, true>(v));
}
__device__ __forceinline__ float last_lane(float v) {
    return __uint_as_float(unsigned(__builtin_amdgcn_readlane(int(__float_as_uint(v)), kWave - 1)));
}
template <typename V> __device__ __forceinline__ V wave_max(V v) {
    v = moved_larger<0x111>(v);
    v = moved_larger<0x112>(v);
    v = moved_larger<0x114>(v);
    v = moved_larger<0x118>(v);
    v = moved_larger<0x142, 0xa>(v);
    v = moved_larger<0x143, 0xc>(v);
    return last_lane(v);
}

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
    __device__ __forceinline__ Row(float top, double scale_, int shift_)
        : m(double(top)), scale(scale_), c(scale_ * kLog2e), far(-128.0 * __builtin_amdgcn_rcp(scale_)), shift(shift_) {}
    // The weight in units, not rounded. Masked logits are taken at `far`: 2^31 times e^-128 is still nothing to the smallest float.
    __device__ __forceinline__ double power(float x) const { return power_of(fmax(double(x) - m, far), c, shift); }
    __device__ __forceinline__ uint64_t weight(float x) const { return whole_of(power(x)); }
    __device__ __forceinline__ uint64_t key_weight(uint32_t k) const { return weight(float_of(k)); }
};

// Weights in single precision, of which a sum has the relative error of their own: the exponents' factor is taken in two parts, both of
// them positive, so that distances beyond the floats and masked logits' count as 0. For scales of 2^-100 to 2^100.
struct Quick {
    float m, c, rest;
    __device__ __forceinline__ Quick(float top, double scale) : m(top) {
        const double exact = scale * kLog2e;
        c = float(exact * (1.0 - 0x1p-23)); // below it, however that is rounded
        rest = float(exact - double(c));
    }
    __device__ __forceinline__ float power(float x) const {
        const float d = x - m;
        return __builtin_amdgcn_exp2f(fmaf(d, c, d * rest));
    }
};

// The token, its log-probability, and the logarithm of the kept share from the weights kept and not kept (in units): the
// latter by itself, however small it is, and 0 exactly where there is nothing of it.
__device__ __forceinline__ void finish_row(const Args &a, int64_t row, const Row &r, int token, float x, double kept, double dropped) {
    a.tokens[row] = token;
    if (a.logp)
        a.logp[row] = float((double(x) - r.m) * r.scale - log_of(kept + dropped) + r.shift * 0.6931471805599453);
    if (a.log_kept) {
        const double d = ratio(dropped, kept + dropped);
        a.log_kept[row] = float(d < 0x1p-16 ? -fma(d, fma(d, 1.0 / 3, 0.5) * d, d) : log_of(1.0 - d));
    }
}
__device__ __forceinline__ void finish_without(const Args &a, int64_t row, bool bad) {
    if (threadIdx.x == 0)
        store_row(a, row, -1, bad ? NAN : -INFINITY, bad ? NAN : 0.0f);
}

// Entries are in the order of the logits: a larger one comes first. A token is kept if its entry is at least that of the
// last one kept.
__device__ __forceinline__ uint64_t entry_of(uint32_t key, int index) { return uint64_t(key) << 32 | uint32_t(~index); }
__device__ __forceinline__ int index_of(uint64_t entry) { return int(~uint32_t(entry)); }
__device__ __forceinline__ uint32_t key_in(uint64_t entry) { return uint32_t(entry >> 32); }

// The logit and the index of the last one kept; entry 0 keeps all.
struct Last {
    float value;
    int index;
    __device__ __forceinline__ explicit Last(uint64_t entry) : value(entry ? float_of(key_in(entry)) : -INFINITY), index(index_of(entry)) {}
    __device__ __forceinline__ bool keeps(float v, int i) const { return v > value || (v == value && unsigned(i) <= unsigned(index)); }
};

constexpr int kBins = 256;

// Sums over kT threads and the search for a place by all of them.
template <int kT> struct Block {
    static constexpr int kWaves = kT / kWave;
    struct Shared {
        uint64_t part[kWaves];
        double real[kWaves];
        float max[kWaves];
        uint64_t left;
        uint32_t digit;
    };

    // The sum over all threads.
    static __device__ __forceinline__ uint64_t sum(uint64_t v, Shared &s) {
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
    static __device__ __forceinline__ double sum(double v, Shared &s) {
        v = wave_sum(v);
        if constexpr (kWaves == 1)
            return v;
        __syncthreads();
        if (threadIdx.x % kWave == 0)
            s.real[threadIdx.x / kWave] = v;
        __syncthreads();
        v = 0.0;
        for (int w = 0; w < kWaves; ++w)
            v += s.real[w];
        return v;
    }

    // The sum over the threads before this one; `total` receives that over all.
    static __device__ __forceinline__ uint64_t before(uint64_t v, uint64_t &total, Shared &s) {
        const uint64_t with = wave_scan(v);
        if constexpr (kWaves == 1) {
            total = last_lane(with);
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

    static __device__ __forceinline__ float max(float v, Shared &s) {
        v = wave_max(v);
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

    // The entry at which the count (kByMass: the weights) of the logits from the top down to `least` reaches `target`, which it
    // does; `inside` receives the weights down to it. Eight bits of the keys at a time, from histograms, and then its index.
    template <bool kByMass, typename T>
    static __device__ uint64_t place_of(const T *x, int V, const Row &r, float least, uint64_t target, uint64_t &inside, uint64_t *mass,
                                        uint32_t *count, Shared &s) {
        uint32_t key = 0;
        uint64_t spare = target, above = 0;
        for (int bit = 24; bit >= 0; bit -= 8) {
            __syncthreads();
            for (int i = threadIdx.x; i < kBins; i += kT)
                mass[i] = count[i] = 0;
            __syncthreads();
            for (int64_t i = threadIdx.x; i < V; i += kT) {
                const float v = float(x[i]);
                const uint32_t k = key_of(v);
                if (!(v >= least) || (bit < 24 && (k ^ key) >> (bit + 8)))
                    continue;
                const int bin = k >> bit & (kBins - 1);
                atomicAdd(&count[bin], 1u);
                atomicAdd(reinterpret_cast<unsigned long long *>(&mass[bin]), (unsigned long long)r.weight(v));
            }
            __syncthreads();
            if (threadIdx.x == 0) {
                uint64_t left = spare, over = 0;
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
            key |= s.digit << bit;
            spare = s.left;
            above += s.part[0];
        }
        const uint64_t level = r.key_weight(key);
        if (kByMass) // the weight that is left, in tokens of this one's
            spare = level ? (spare + level - 1) / level : 1;
        inside = above + spare * level;
        // the index of the last of them: threads take stretches
        const int each = (V - 1) / kT + 1;
        const int64_t from = std::min(int64_t(threadIdx.x) * each, int64_t(V)), to = std::min(from + each, int64_t(V));
        const float value = float_of(key);
        uint64_t same = 0, unused;
        for (int64_t i = from; i < to; ++i)
            same += float(x[i]) == value;
        uint64_t rank = before(same, unused, s);
        if (rank < spare && spare <= rank + same)
            for (int64_t i = from; i < to; ++i) {
                rank += float(x[i]) == value;
                if (rank == spare) {
                    s.digit = uint32_t(i);
                    break;
                }
            }
        __syncthreads();
        const uint64_t entry = entry_of(key, int(s.digit));
        __syncthreads();
        return entry;
    }
};

// ------------------------------------------------------------------------------------------------
// lists of entries in LDS
// ------------------------------------------------------------------------------------------------
enum class Order { kLogits, kVocabulary };

constexpr int kList = 512;     // candidates of pick_kernel; C took 124, 112 and 119 us with 256, 512 and 1,024
constexpr int kMembers = 4096; // of a bin; one of E may have more than 2,048, and its row is then read once more, for 30 us

// An entry as the order has it, the first one the largest, without the bits that all entries of lists have alike: those of indexes
// beyond 2^kBits, and of keys those that T has not. The fewer steps a search takes: the two of 240 fp16
// candidates, many of them equal, 4 us instead of up to 11, and C 105 us instead of 113.
constexpr int kIndexBits = 19;
template <typename T> constexpr int kKeyDrop = 0;
template <> constexpr int kKeyDrop<__bf16> = 16;
template <> constexpr int kKeyDrop<_Float16> = 13;
template <Order kOrder, typename T, int kBits = kIndexBits> __device__ __forceinline__ uint64_t ordered(uint64_t entry) {
    const uint64_t index = entry & ((1u << kBits) - 1);
    return kOrder == Order::kLogits ? entry >> (32 + kKeyDrop<T>) << kBits | index : index;
}

template <int kT> struct List {
    using B = Block<kT>;
    struct Shared {
        uint64_t mass[kT];
        uint32_t count[kT];
        uint64_t high[B::kWaves], low[B::kWaves];
        uint64_t left, above, entry;
        uint32_t digit;
    };

    // The entry of list[0, n) at which the count (by_mass: the weights) of those of at least `least` reaches `target`, which it
    // does; `inside` receives the weights down to it. By bins of the range that the entries have, as many as there are
    // threads, and then of the range of the bin that holds it, until it is alone.
    // `high` and `low`: bounds of the entries as the order has them, or 0 and 0.
    template <Order kOrder, typename T, int kBits = kIndexBits>
    static __device__ __forceinline__ uint64_t find(bool by_mass, uint64_t target, const uint64_t *list, int n, uint64_t least, uint64_t high,
                                                    uint64_t low, const Row &r, uint64_t &inside, Shared &s, typename B::Shared &block) {
        const int tid = threadIdx.x;
        if (high == 0) {
            low = ~uint64_t(0);
            for (int i = tid; i < n; i += kT)
                if (list[i] >= least) {
                    high = std::max(high, ordered<kOrder, T, kBits>(list[i]));
                    low = std::min(low, ordered<kOrder, T, kBits>(list[i]));
                }
            high = wave_max(high);
            low = ~wave_max(~low);
            if constexpr (B::kWaves > 1) {
                __syncthreads();
                if (tid % kWave == 0) {
                    s.high[tid / kWave] = high;
                    s.low[tid / kWave] = low;
                }
                __syncthreads();
                for (int w = 0; w < B::kWaves; ++w) {
                    high = std::max(high, s.high[w]);
                    low = std::min(low, s.low[w]);
                }
            }
        }
        uint64_t above = 0;
        for (;;) {
            const uint64_t span = high - low;
            const int shift = span < kT ? 0 : 64 - __builtin_clzll(span) - (31 - __builtin_clz(kT));
            __syncthreads();
            s.mass[tid] = s.count[tid] = 0;
            __syncthreads();
            for (int i = tid; i < n; i += kT) {
                const uint64_t e = ordered<kOrder, T, kBits>(list[i]);
                if (list[i] >= least && e <= high && e >= low) {
                    const int bin = int((high - e) >> shift);
                    atomicAdd(&s.count[bin], 1u);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[bin]), (unsigned long long)r.key_weight(key_in(list[i])));
                }
            }
            __syncthreads();
            const uint64_t mass = s.mass[tid], mine = by_mass ? mass : s.count[tid];
            uint64_t unused;
            const uint64_t mass_before = B::before(mass, unused, block), before = by_mass ? mass_before : B::before(mine, unused, block);
            if (before < target && target <= before + mine) {
                s.digit = tid;
                s.left = target - before;
                s.above = mass_before;
            }
            __syncthreads();
            const int bin = int(s.digit);
            target = s.left;
            above += s.above;
            high -= uint64_t(bin) << shift;
            low = high - std::min(high - low, (uint64_t(1) << shift) - 1);
            if (s.count[bin] == 1 || shift == 0) {
                inside = above + s.mass[bin];
                break;
            }
        }
        for (int i = tid; i < n; i += kT)
            if (list[i] >= least && ordered<kOrder, T, kBits>(list[i]) <= high && ordered<kOrder, T, kBits>(list[i]) >= low)
                s.entry = list[i];
        __syncthreads();
        return s.entry;
    }

    // The weights of the entries below `end`, in units, added in whole numbers of 2^-51 of the largest of them: exact in any order, and
    // in proportion to itself, as what is not kept has to be.
    static __device__ __forceinline__ double below(const uint64_t *list, int n, uint64_t end, const Row &r, typename B::Shared &block) {
        static_assert(kMembers <= 1 << 12, "sums are below 2^64");
        float top = -INFINITY;
        for (int i = threadIdx.x; i < n; i += kT)
            top = list[i] < end ? larger(top, float_of(key_in(list[i]))) : top;
        top = B::max(top, block);
        const Row own(top, r.scale, 51);
        uint64_t sum = 0;
        for (int i = threadIdx.x; i < n; i += kT)
            sum += list[i] < end ? own.key_weight(key_in(list[i])) : 0;
        return double(B::sum(sum, block)) * 0x1p-51 * r.power(top);
    }
};

// ------------------------------------------------------------------------------------------------
// short rows
// ------------------------------------------------------------------------------------------------
// A workgroup holds a row's logits and weights in registers, kOwn to a thread, stretches of the vocabulary so that the search
// for the token is a scan over threads. 6,144 x 136 fp32 take 6.8 us, 200,000 x 136 bf16 with top-k and top-p 3.0 ns a row: instructions, 360 of a wave
// where nothing is cut off, more with the lists' searches; the logits themselves would take 0.5 us.
template <typename T, int kT, int kOwn>
__global__ void __launch_bounds__(kT) __attribute__((amdgpu_waves_per_eu(kOwn == 4 ? 4 : 3))) small_kernel(const T *logits, Args a) {
    using B = Block<kT>;
    using L = List<kT>;
    constexpr int kBits = 31 - __builtin_clz(kOwn * kT); // of an index
    __shared__ typename B::Shared s;
    __shared__ typename L::Shared find;
    __shared__ uint64_t list[kOwn * kT];
    const int tid = threadIdx.x, each = (a.V + kT - 1) / kT, from = tid * each;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *x = logits + row * a.stride;
        float v[kOwn], m = -INFINITY;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            v[i] = i < each && from + i < a.V ? float(x[from + i]) : -INFINITY;
            m = larger(m, v[i]);
        }
        const Params p = params_of(a, row);
        m = B::max(m, s);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        const Row r(m, p.scale, a.shift);
        const uint32_t floor = floor_key(r.m, p.scale, p.least, key_of(m));
        uint64_t w[kOwn];
#pragma unroll
        for (int i = 0; i < kOwn; ++i)
            w[i] = i < each && from + i < a.V ? r.weight(v[i]) : 0;
        uint64_t lowest = entry_of(floor, -1); // entries from here on are kept
        if (p.top_k < a.V || p.fraction < kOne) {
            __syncthreads();
            uint64_t inside = 0, there = 0;
#pragma unroll
            for (int i = 0; i < kOwn; ++i)
                if (i < each && from + i < a.V) {
                    const uint64_t e = entry_of(key_of(v[i]), from + i);
                    list[from + i] = e;
                    inside += e >= lowest ? w[i] : 0;
                    there += e >= lowest;
                }
            inside = B::sum(inside, s);
            there = B::sum(there, s);
            __syncthreads();
            if (uint64_t(p.top_k) < there)
                lowest = L::template find<Order::kLogits, T, kBits>(false, uint64_t(p.top_k), list, a.V, lowest, 0, 0, r, inside, find, s);
            uint64_t unused;
            if (p.fraction < kOne)
                lowest = L::template find<Order::kLogits, T, kBits>(true, std::max(share_up(inside, p.fraction), uint64_t(1)), list, a.V, lowest, 0, 0, r, unused, find, s);
        }
        uint64_t mine = 0;
        double lost = 0.0;
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
            if (entry_of(key_of(v[i]), from + i) < lowest) {
                w[i] = 0;
                if (wants_logp(a) && v[i] > -INFINITY)
                    lost += r.power(v[i]);
            }
            mine += w[i];
        }
        if (wants_logp(a) && lowest)
            lost = B::sum(lost, s);
        uint64_t kept;
        uint64_t sum = B::before(mine, kept, s);
        const uint64_t target = share_down(kept, p.at);
        int token = -1;
        float at = 0.0f;
        if (sum <= target && target < sum + mine)
#pragma unroll
            for (int i = 0; i < kOwn; ++i) {
                if (sum <= target && target < sum + w[i]) {
                    token = from + i;
                    at = v[i];
                }
                sum += w[i];
            }
        if (token >= 0)
            finish_row(a, row, r, token, at, double(kept), lost);
    }
}

// ------------------------------------------------------------------------------------------------
// the digest of a row
// ------------------------------------------------------------------------------------------------
constexpr int kPart = 2048, kSeg = 128, kSegs = kPart / kSeg;
constexpr int kMostParts = (1 << kIndexBits) / kPart; // longer rows go to long_kernel

// 16 bytes of logits. A row may start anywhere, so what it is read through claims no alignment.
template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef type unaligned __attribute__((aligned(sizeof(T))));
};

// Up to N logits from p on, -inf beyond the first `len`.
template <typename T> __device__ __forceinline__ typename Vec<T>::type read_vec(const T *p, int len) {
    if (len >= Vec<T>::N)
        return *reinterpret_cast<const typename Vec<T>::unaligned *>(p);
    typename Vec<T>::type q(T(-INFINITY));
#pragma unroll
    for (int i = 0; i < Vec<T>::N; ++i)
        if (i < len)
            q[i] = p[i];
    return q;
}

// The N logits from element `at` on of a row of at least N, or its last ones; `first` receives the first one's index. Those
// before `at` are replaced by -inf.
template <typename T> __device__ __forceinline__ typename Vec<T>::type read_at(const T *x, int V, int at, int &first) {
    first = std::min(at, V - Vec<T>::N);
    typename Vec<T>::type q = *reinterpret_cast<const typename Vec<T>::unaligned *>(x + first);
    if (first < at)
#pragma unroll
        for (int i = 0; i < Vec<T>::N; ++i)
            q[i] = first + i < at ? T(-INFINITY) : q[i];
    return q;
}

// A wave reads a part in kLoads loads of 64 vectors; the 16 lanes of a quarter hold a segment in kSame of them: one of
// 2-byte logits, two of 4-byte ones.
template <typename T> struct Part {
    static constexpr int N = Vec<T>::N, kLoads = kPart / kWave / N, kSame = kLoads / 4;
    // the lane's first element of a load
    static __device__ __forceinline__ int at(int load, int lane) { return (load * kWave + lane) * N; }
    static __device__ __forceinline__ void read(const T *x, int len, int lane, typename Vec<T>::type (&q)[kLoads]) {
        if (len >= kPart) {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                q[j] = *reinterpret_cast<const typename Vec<T>::unaligned *>(x + at(j, lane));
        } else {
#pragma unroll
            for (int j = 0; j < kLoads; ++j)
                q[j] = read_vec(x + at(j, lane), len - at(j, lane));
        }
    }
};

// A row that pick_kernel leaves to the two kernels behind it.
struct WideRow {
    int64_t row;
    float top, least;
    uint64_t last;  // the entry of the last kept token, where `bin` is kNoBin
    uint64_t left;  // otherwise it is in this bin, where the count (by_mass: the weights) reaches this
    int bin, members;
    bool by_mass, fine; // fine: the bin is one of kFine of a bin
    unsigned arrived[2], listed;
};

// What the kernels leave for the next ones.
struct Digest {
    double *mass;      // [n][parts]: weights relative to the part's own largest logit, in units
    float *top;        // [n][parts]
    float *seg;        // [n][parts][kSegs]
    unsigned *wide;    // the number of rows left
    WideRow *rows;     // [n]
    // where several workgroups share a row:
    uint64_t *bins;    // [kShared][kFine]: weights, and
    unsigned *members; // [kShared][kFine]: the numbers of tokens; set to 0 by pick_kernel
    uint64_t *kept;    // [kShared][kMostParts]: weights above the bin, and
    double *lost;      // [kShared][kMostParts]: below it
    uint64_t *list;    // [kShared][kMembers]: the bin's entries
    int parts;
};

// A wave takes a part of a row: all its loads are on their way before the first is used, and the weights relative to the
// part's own largest logit, so that no wave waits for another's. Bound by instructions: 705 of a wave, 22 a logit, where weights
// are exact, which are 18.8 us of B's 28.4 if each takes four cycles of a SIMD, and longer as some of the 64-bit ones take more; its 66 MB would
// take 9.5 us at 6.9 TB/s. 12 a logit in single precision (D: 33 us for 131 MB; with exact weights 47, C 48 instead of 38.5). E, half of
// which 33 MB stay in the caches: 11.3. Double-precision multiply-adds cost what single ones do here, and exp2 two of them. Kept weights are never from
// this sum alone where a list holds the tokens, so its roundings, in an order that is always the same, do not add up with theirs.
template <typename T>
__global__ void __launch_bounds__(256) scan_kernel(const T *logits, Args a, Digest g) {
    using P = Part<T>;
    constexpr int kN = P::kLoads * P::N;
    const int lane = threadIdx.x % kWave;
    if (blockIdx.x == 0 && threadIdx.x == 0)
        *g.wide = 0;
    const int each = (g.parts + 3) / 4; // workgroups of a row
    const int wave = __builtin_amdgcn_readfirstlane(int(threadIdx.x) / kWave);
    for (int64_t at = blockIdx.x; at < a.n * each; at += gridDim.x) {
        const int64_t row = at / each;
        const int part = int(at - row * each) * 4 + wave;
        if (part >= g.parts)
            continue;
        const int64_t item = row * g.parts + part;
        typename Vec<T>::type q[P::kLoads];
        P::read(logits + row * a.stride + part * kPart, a.V - part * kPart, lane, q);
        float v[kN], m = -INFINITY, mine = -INFINITY;
#pragma unroll
        for (int k = 0; k < kN; ++k)
            v[k] = float(q[k / P::N][k % P::N]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            constexpr int kSome = P::kSame * P::N;
            float top = v[i * kSome];
#pragma unroll
            for (int k = 1; k < kSome; ++k)
                top = larger(top, v[i * kSome + k]);
            top = row_max(top);
            mine = lane % 16 == i ? top : mine;
            m = larger(m, top);
        }
        m = larger(larger(of_row(m, 0), of_row(m, 1)), larger(of_row(m, 2), of_row(m, 3)));
        if (lane % 16 < 4)
            g.seg[item * kSegs + lane % 16 * 4 + lane / 16] = mine;
        double mass = 0.0;
        const double scale = scale_of(a, row);
        const Mass kind = mass_of(a, row);
        if (kind != Mass::kNone && scale != 0.0 && m < INFINITY && m > -INFINITY) {
            if (kind == Mass::kExact) {
                const Row r(m, scale, a.shift);
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    mass += r.power(v[k]);
            } else {
                const Quick w(m, scale);
#pragma unroll
                for (int k = 0; k < kN; ++k)
                    mass += double(w.power(v[k]));
                mass *= double(int64_t(1) << a.shift);
            }
            mass = row_sum(mass);
            mass = (of_row(mass, 0) + of_row(mass, 1)) + (of_row(mass, 2) + of_row(mass, 3));
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
constexpr int kFine = 1024;    // bins; E takes 75 us, and 81 with 2,048
constexpr int kShared = 256;   // wide rows that workgroups may share

// What finish_row takes, from whichever thread finds it.
struct Outcome {
    int token;
    float x;
    double kept, dropped;
};

// The token among the logits of one part, as far into the sum of its kept weights there as `ask` is in `of`.
template <typename T, int kT>
__device__ __forceinline__ void pick_in_part(const Args &a, const T *x, int part, const Row &own, Last last, uint64_t ask, uint64_t of,
                                             Outcome &out, typename Block<kT>::Shared &s) {
    constexpr int kEach = kPart / kT;
    const int from = part * kPart + threadIdx.x * kEach;
    float v[kEach];
    uint64_t w[kEach], mine = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i)
        v[i] = from + i < a.V ? float(x[from + i]) : -INFINITY;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        w[i] = last.keeps(v[i], from + i) ? own.weight(v[i]) : 0;
        mine += w[i];
    }
    uint64_t sum = Block<kT>::before(mine, all, s);
    const uint64_t target = all == of ? ask : std::min(uint64_t(double(ask) / double(of) * double(all)), all - 1);
    if (sum <= target && target < sum + mine)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (sum <= target && target < sum + w[i]) {
                out.token = from + i;
                out.x = v[i];
            }
            sum += w[i];
        }
}

constexpr int kPick = 256;
using PickBlock = Block<kPick>;

struct Weighed {
    uint64_t entry, weight;
};
constexpr int kAhead = 8;

struct PickShared {
    uint64_t list[kList];
    union {
        Weighed weighed[kWave + kAhead];
        List<kPick>::Shared find;
    };
    uint64_t bins[kPick];
    float tops[kPick];      // of the parts
    uint64_t listed[kPick]; // weights of a part's tokens in the list, in 2^-51 of its largest
    PickBlock::Shared block;
    uint64_t found_mass, found_left;
    float found_top;
    int found, n;
    bool little;
    Outcome out;
    int ge[2][PickBlock::kWaves];
};
// Behind it in LDS, for as many segments as there are: the keys of their largest logits, of which thread t has every kPick-th
// from t on, and a list of some of the segments.
constexpr int kSegBytes = kSegs * int(sizeof(uint32_t) + sizeof(uint16_t)); // of a part

// The number of segments whose largest logit has a key of at least k.
__device__ __forceinline__ int segments_from(const uint32_t *keys, int segs, uint32_t k, int step, PickShared &s) {
    int n = 0;
    for (int i = threadIdx.x; i < segs; i += kPick)
        n += keys[i] >= k;
    n = int(wave_sum(uint64_t(n)));
    if (threadIdx.x % kWave == 0)
        s.ge[step & 1][threadIdx.x / kWave] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < PickBlock::kWaves; ++w)
        n += s.ge[step & 1][w];
    return n;
}

// Calls f for s.weighed[0, n), of which there is room for kAhead more: that many are on their way from LDS at a time.
template <typename F> __device__ __forceinline__ void for_entries(const PickShared &s, int n, F &&f) {
    for (int i = 0; i < n; i += kAhead) {
        Weighed o[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            o[k] = s.weighed[i + k];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
            if (i + k < n)
                f(o[k]);
    }
}

// The token from s.list[0, n), which holds every token down to some place of the order. `whole`: all that min_p and top_k
// leave is among them; otherwise `total` is the weight of all that top_p is a share of. `rest`: the weights of the tokens
// beyond the list. False where the list ends before the last kept token does.
template <typename T>
__device__ __forceinline__ bool pick_from_list(const Args &a, const Row &r, const Params &p, uint32_t low, int n, bool whole, uint64_t total,
                                               double rest, PickShared &s) {
    using L = List<kPick>;
    uint64_t kept = 0, end = 0, unused;
    for (int i = threadIdx.x; i < n; i += kPick)
        kept += r.key_weight(key_in(s.list[i]));
    kept = PickBlock::sum(kept, s.block);
#pragma unroll 1
    for (int pass = 0; pass < 2; ++pass) { // top_k, then top_p of what it leaves
        if (pass ? p.fraction == kOne : p.top_k >= n)
            continue;
        const uint64_t target = pass ? std::max(share_up(whole ? kept : total, p.fraction), uint64_t(1)) : uint64_t(p.top_k);
        if (pass && kept < target)
            return false;
        end = L::find<Order::kLogits, T>(pass, target, s.list, n, end, ordered<Order::kLogits, T>(entry_of(key_of(float(r.m)), 0)),
                                         ordered<Order::kLogits, T>(entry_of(low, -1)), r, kept, s.find,
                                      s.block);
    }
    const double lost = wants_logp(a) && end ? L::below(s.list, n, end, r, s.block) : 0.0;
    // sums are whole numbers: past the random share of them is to reach the next one
    const uint64_t token = L::find<Order::kVocabulary, T>(true, share_down(kept, p.at) + 1, s.list, n, end, ordered<Order::kVocabulary, T>(entry_of(0, 0)),
                                                              ordered<Order::kVocabulary, T>(entry_of(0, a.V - 1)), r, unused, s.find, s.block);
    if (threadIdx.x == 0)
        s.out = {index_of(token), float_of(key_in(token)), double(kept), rest + lost};
    return true;
}

// The same of up to 64 entries, by the first wave alone and so without barriers: every lane reads the others' entries, in no
// order, and adds what comes before its own.
__device__ __forceinline__ bool pick_from_few(const Args &a, const Row &r, const Params &p, int n, bool whole, uint64_t total, double rest,
                                              PickShared &s) {
    const int lane = threadIdx.x;
    const auto wait = [] { // for the wave's own LDS accesses, which are in order
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    bool keep = lane < n;
    const uint64_t mine = keep ? s.list[lane] : 0;
    const uint64_t w = keep ? r.key_weight(key_in(mine)) : 0;
    if (keep)
        s.weighed[lane] = {mine, w};
    wait();
    if (p.top_k < n || p.fraction < kOne) {
        uint64_t before = 0;
        int rank = 0;
        for_entries(s, n, [&](const Weighed &o) {
            before += o.entry > mine ? o.weight : 0;
            rank += o.entry > mine;
        });
        keep = keep && rank < p.top_k;
        if (p.fraction < kOne) {
            const uint64_t inside = wave_sum(keep ? w : 0);
            const uint64_t target = std::max(share_up(whole ? inside : total, p.fraction), uint64_t(1));
            if (inside < target)
                return false;
            keep = keep && before < target;
        }
        wait();
        if (lane < n)
            s.weighed[lane].weight = keep ? w : 0;
        wait();
    }
    const uint64_t kept = wave_sum(keep ? w : 0), target = share_down(kept, p.at);
    double lost = 0.0; // as List::below has it
    if (wants_logp(a)) {
        const bool is_lost = lane < n && !keep;
        const float x = float_of(key_in(mine)), top = wave_max(is_lost ? x : -INFINITY);
        const Row own(top, r.scale, 51);
        lost = double(wave_sum(is_lost ? own.weight(x) : 0)) * 0x1p-51 * r.power(top);
    }
    uint64_t before = 0;
    for_entries(s, n, [&](const Weighed &o) {
        before += uint32_t(o.entry) > uint32_t(mine) ? o.weight : 0; // indices before this one's
    });
    if (keep && before <= target && target < before + w)
        s.out = {index_of(mine), float_of(key_in(mine)), double(kept), rest + lost};
    return true;
}

// A key down to which the segments' largest logits are `target` at least (by_mass: have at least that weight), and not many
// more: from bins of their distance from the largest of all, as far as weights reach, or, where one of those holds too many,
// by halving. 0 where their weights are less than that.
__device__ __forceinline__ uint32_t key_reached(bool by_mass, uint64_t target, const uint32_t *keys, int segs, float m, const Row &r,
                                                PickShared &s) {
    const int tid = threadIdx.x;
    const float step = kPick / fminf(32.0f / float(r.scale), 64.0f);
    __syncthreads();
    s.bins[tid] = 0;
    if (tid == 0)
        s.found = -1;
    __syncthreads();
#pragma unroll 1
    for (int i = tid; i < segs; i += kPick) {
        const float x = float_of(keys[i]), d = (m - x) * step;
        if (d < float(kPick))
            atomicAdd(reinterpret_cast<unsigned long long *>(&s.bins[int(d)]), by_mass ? (unsigned long long)r.weight(x) : 1ull);
    }
    __syncthreads();
    const uint64_t mine = s.bins[tid];
    uint64_t all;
    const uint64_t sum = PickBlock::before(mine, all, s.block);
    if (sum < target && target <= sum + mine && (by_mass || sum + mine <= 2 * target + 64))
        s.found = tid;
    __syncthreads();
    if (s.found >= 0) {
        // a little below the bin's end, whatever the roundings on the way
        const float end = m - float(s.found + 1) / step;
        return key_of(end - 1e-6f * fmaxf(fabsf(end), fabsf(m)));
    }
    if (by_mass)
        return 0;
    uint32_t from = 0, to = key_of(m) + 1;
    const int want = int(target);
    for (int at = 0; to - from > 1; ++at) {
        const uint32_t k = from + (to - from) / 2;
        const int n = segments_from(keys, segs, k, at, s);
        if (n >= want)
            from = k;
        else
            to = k;
        if (n >= want && n <= want + want / 8 + 8)
            break;
    }
    return std::max(from, key_of(-INFINITY));
}

// What is left of a part's sum without `n` of its tokens is off by up to (n + 20) 2^-52 of the sum: half a unit of 2^-51 for each of the
// tokens, and the 38 roundings on the way to any lane's share of the sum. Below this share of the sum that is more than 2^-19 of what is left.
__device__ __forceinline__ double little_from(int n) { return double(n + 20) * 0x1p-33; }

constexpr int kSegLoads = 4; // of a quarter of a wave, which takes a segment, on their way at a time

// The j-th of kSegLoads vectors that the thread's quarter of a wave has from some[i] on of `many` segments, in steps of as many as there are
// quarters: `at` receives where it begins, `first` its first element's index. Elements before `at`, or all beyond the last segment, are -inf.
template <typename T>
__device__ __forceinline__ typename Vec<T>::type read_seg(const T *x, int V, const uint16_t *some, int many, int i, int j, int &at, int &first) {
    const int k = i + j / Part<T>::kSame * (kPick / 16);
    const int seg = k < many ? some[k] : 0, quarter = seg % 4, load = seg / 4 % 4 * Part<T>::kSame;
    at = k < many ? seg / kSegs * kPart + Part<T>::at(load + j % Part<T>::kSame, quarter * 16 + threadIdx.x % 16) : V;
    return read_at(x, V, at, first);
}
template <typename T> constexpr int kSegStep = kPick / 16 * (kSegLoads / Part<T>::kSame);

// The weights below `lowest`, in units, of the parts whose threads want them, which hold a token that is likeliest by far, or a few that
// a mask leaves over. `some` has room for the list of their segments, whose order makes that of the sum.
// 64 rows of 128,000 bf16 with 100 tokens each that a mask leaves, in 50 parts or so, take 27 us under top_k 50; by a wave a
// part 42, and 24 if what is left is taken as it is.
template <typename T>
__device__ __forceinline__ double little_of(const T *x, int V, const uint32_t *keys, uint16_t *some, int segs, float lowest, const Row &r, bool wanted,
                                            PickShared &s) {
    const int tid = threadIdx.x;
    s.listed[tid] = wanted;
    __syncthreads();
    const auto takes = [&](int i) { return s.listed[i / kSegs] && keys[i] > key_of(-INFINITY); };
    uint64_t mine = 0, many;
    for (int i = tid; i < segs; i += kPick)
        mine += takes(i);
    int to = int(PickBlock::before(mine, many, s.block));
    for (int i = tid; i < segs; i += kPick)
        if (takes(i))
            some[to++] = uint16_t(i);
    __syncthreads();
    double sum = 0.0;
    const auto counts = [&](float v) { return v < lowest && v > -INFINITY; };
    for (int i = tid / 16; i < int(many); i += kSegStep<T>) {
        int at, first;
        bool any = false;
#pragma unroll
        for (int j = 0; j < kSegLoads; ++j) {
            const auto q = read_seg(x, V, some, int(many), i, j, at, first);
#pragma unroll
            for (int k = 0; k < Part<T>::N; ++k)
                any = any || counts(float(q[k]));
        }
        if (any)
#pragma unroll 1
            for (int j = 0; j < kSegLoads; ++j) { // once more, as there are as a rule none
                const auto q = read_seg(x, V, some, int(many), i, j, at, first);
#pragma unroll
                for (int k = 0; k < Part<T>::N; ++k)
                    sum += counts(float(q[k])) ? r.power(float(q[k])) : 0.0;
            }
    }
    return PickBlock::sum(sum, s.block);
}

// A workgroup takes a row. Bound by the latency of its steps one after another (the digest, the search for the lowest segment, the
// segments, the list's searches) and by fetching instructions that run once: 11.5 us for a row alone (A; lists of up to 64 by
// pick_from_list too: 14.7), 5.7 where nothing is cut off (B), 25 for the 2,048 rows of D and in C. Three waves of a SIMD have the
// registers they need: D takes 67 us as a whole, 72 with four and 89 with five, 84 with 512 threads a row. Four loads of a quarter
// of a wave at a time: 66.7, eight: 70.8.
template <typename T>
__global__ void __launch_bounds__(kPick) __attribute__((amdgpu_waves_per_eu(3))) pick_kernel(const T *logits, Args a, Digest g) {
    __shared__ PickShared s;
    extern __shared__ uint32_t keys[];
    static_assert(kMostParts <= kPick, "a part a thread");
    const int tid = threadIdx.x, segs = g.parts * kSegs;
    uint16_t *some = reinterpret_cast<uint16_t *>(keys + segs); // of the segments
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const T *x = logits + row * a.stride;
        const float top = tid < g.parts ? g.top[row * g.parts + tid] : -INFINITY;
        const double part_mass = tid < g.parts ? g.mass[row * g.parts + tid] : 0.0;
        const Params p = params_of(a, row);
        const bool cut = p.top_k < a.V || p.fraction < kOne || p.least != -INFINITY;
        if (cut)
#pragma unroll 4
            for (int i = tid; i < segs; i += kPick)
                keys[i] = key_of(g.seg[row * segs + i]);
        const float m = PickBlock::max(top, s.block);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        const Row r(m, p.scale, a.shift);
        // the parts' weights, relative to the row's largest logit
        const double factor = power_of(fmax(double(top) - r.m, r.far), r.c, 0);
        const uint64_t mine = uint64_t(rint(part_mass * factor));
        uint64_t total;
        const uint64_t sum = PickBlock::before(mine, total, s.block);
        if (!cut) {
            const uint64_t target = share_down(total, p.at);
            if (sum <= target && target < sum + mine) {
                s.found = tid;
                s.found_top = top;
                s.found_left = target - sum;
                s.found_mass = mine;
            }
            __syncthreads();
            const Row own(s.found_top, p.scale, a.shift);
            pick_in_part<T, kPick>(a, x, s.found, own, Last(0), s.found_left, s.found_mass, s.out, s.block);
            __syncthreads();
            if (tid == 0)
                finish_row(a, row, r, s.out.token, s.out.x, double(total), 0.0);
            continue;
        }
        uint32_t low = floor_key(r.m, p.scale, p.least, key_of(m));
        const float least = low ? float_of(low) : -INFINITY;
        bool wide = false, whole = true;
        if (p.top_k < a.V) {
            if (p.top_k <= segs / 2)
                low = std::max(low, key_reached(false, uint64_t(p.top_k), keys, segs, m, r, s));
            else
                wide = low == 0;
        } else if (low == 0) {
            low = key_reached(true, std::max(share_up(total, p.fraction), uint64_t(1)), keys, segs, m, r, s);
            whole = false;
            wide = low == 0;
        }
        if (!wide) {
            // segments that have a candidate, and their candidates
            __syncthreads();
            if (tid == 0)
                s.found = s.n = s.little = 0;
            s.tops[tid] = top;
            s.listed[tid] = 0;
            __syncthreads();
            for (int i = tid; i < segs; i += kPick)
                if (keys[i] >= low)
                    some[atomicAdd(&s.found, 1)] = uint16_t(i);
            __syncthreads();
            const int many = s.found <= kList ? s.found : 0; // each has a candidate: of more there is no list
            wide = s.found > kList;
            const float lowest = float_of(low);
            for (int i = tid / 16; i < many; i += kSegStep<T>) {
                typename Vec<T>::type q[kSegLoads];
                int at[kSegLoads], first[kSegLoads];
#pragma unroll
                for (int j = 0; j < kSegLoads; ++j)
                    q[j] = read_seg(x, a.V, some, many, i, j, at[j], first[j]);
#pragma unroll
                for (int j = 0; j < kSegLoads; ++j) {
                    unsigned hits = 0;
#pragma unroll
                    for (int k = 0; k < Part<T>::N; ++k)
                        hits |= float(q[j][k]) >= lowest ? 1u << k : 0;
                    hits &= at[j] - first[j] < Part<T>::N ? ~0u << (at[j] - first[j]) : 0;
                    while (hits) {
                        const int k = __builtin_ctz(hits), to = atomicAdd(&s.n, 1);
                        hits &= hits - 1;
                        if (to < kList)
                            s.list[to] = entry_of(key_of(float(x[first[j] + k])), first[j] + k);
                    }
                }
            }
            __syncthreads();
            const int n = s.n;
            wide = wide || n > kList;
            double rest = 0.0;
            if (!wide && wants_logp(a)) {
                // what a part has beside the list's tokens, whose weights are those that its sum was made of
                const bool quick = mass_of(a, row) == Mass::kQuick;
                for (int i = tid; i < n; i += kPick) {
                    const int part = index_of(s.list[i]) / kPart;
                    const float v = float_of(key_in(s.list[i])), own = s.tops[part];
                    const double w = quick ? ldexp(double(Quick(own, p.scale).power(v)), 51)
                                           : power_of(fmax(double(v) - double(own), r.far), r.c, 51);
                    atomicAdd(reinterpret_cast<unsigned long long *>(&s.listed[part]), (unsigned long long)whole_of(w));
                }
                __syncthreads();
                const double left = part_mass - ldexp(double(s.listed[tid]), a.shift - 51);
                const bool little = s.listed[tid] != 0 && left < part_mass * little_from(n);
                const double ample = little ? 0.0 : left * factor;
                if (little)
                    s.little = true;
                rest = PickBlock::sum(ample, s.block);
                if (s.little)
                    rest += little_of(x, a.V, keys, some, segs, lowest, r, little, s);
            }
            if (!wide && n <= kWave)
                wide = __syncthreads_or(tid < kWave && !pick_from_few(a, r, p, n, whole, total, rest, s));
            else if (!wide)
                wide = !pick_from_list<T>(a, r, p, low, n, whole, total, rest, s);
        }
        __syncthreads();
        if (!wide) {
            if (tid == 0)
                finish_row(a, row, r, s.out.token, s.out.x, s.out.kept, s.out.dropped);
            continue;
        }
        if (tid == 0) {
            s.found = int(atomicAdd(g.wide, 1u));
            WideRow &w = g.rows[s.found];
            w.row = row;
            w.top = m;
            w.least = least;
            w.arrived[0] = w.arrived[1] = w.listed = 0;
        }
        __syncthreads();
        if (s.found < kShared)
            for (int i = tid; i < kFine; i += kPick)
                g.bins[int64_t(s.found) * kFine + i] = g.members[int64_t(s.found) * kFine + i] = 0;
    }
}

// ------------------------------------------------------------------------------------------------
// rows of which more tokens are kept than a list holds
// ------------------------------------------------------------------------------------------------
constexpr int kWide = 512;
constexpr int kMostShares = 16;
using WideBlock = Block<kWide>;

// Workgroups that share a row, so that a few wide rows have many and many have one each. 128,000 fp32 logits, top-p 0.98, take 47 us
// for one row, 49 for 16, 71 for 64, 151 for 200 and 253 for 400; with a workgroup a row always 135, 139, 147, 164 and 251.
__device__ __forceinline__ int shares_of(unsigned wide, int parts) {
    return wide > kShared ? 1 : std::max(1, std::min(std::min(int(2 * kShared / wide), kMostShares), parts / 4));
}

struct WideShared {
    uint64_t mass[kFine];
    uint32_t count[kFine];
    uint64_t list[kMembers];
    uint64_t kept[kMostParts];
    double lost[kMostParts];
    WideBlock::Shared block;
    List<kWide>::Shared find;
    uint64_t found_mass, found_left;
    int found, n;
    Outcome out;
    bool last;
};

// The bin of a logit by its distance from the largest, which never decreases as logits do; kNoBin: beyond 63 in units of the
// exponent, where a token has no part in what is kept. Halves, because the distance itself may be no float.
// Fine ones are kFine to each of the others, exactly, since a power of two scales the distance.
constexpr int kNoBin = kFine * kFine;
struct Bins {
    float half, step, end;
    __device__ __forceinline__ Bins(const Row &r, bool fine = false)
        : half(float(r.m) * 0.5f), step(fminf(float(r.scale) * (2.0f * kFine / 63.0f), 3.402823466e38f)), end(fine ? kFine * kFine : kFine) {
        step *= fine ? float(kFine) : 1.0f;
    }
    __device__ __forceinline__ bool have_fine() const { return step < 0x1p100f; }
    __device__ __forceinline__ int of(float x) const {
        const float d = (half - x * 0.5f) * step;
        return d < end ? int(d) : kNoBin;
    }
};

// Calls f(logit, index) for a share of a row's vectors, some of the last of them twice, with -inf.
template <typename T, typename F> __device__ __forceinline__ void for_share(const T *x, int V, int share, int shares, F &&f) {
    constexpr int N = Vec<T>::N;
    const int vecs = (V + N - 1) / N, each = (vecs + shares - 1) / shares, end = std::min(vecs, (share + 1) * each);
    constexpr int kLoads = 4; // on their way at a time
    for (int i = share * each + int(threadIdx.x); i < end; i += kLoads * kWide) {
        typename Vec<T>::type q[kLoads];
        int first[kLoads];
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (i + j * kWide < end)
                q[j] = read_at(x, V, (i + j * kWide) * N, first[j]);
#pragma unroll
        for (int j = 0; j < kLoads; ++j)
            if (i + j * kWide < end)
#pragma unroll
                for (int k = 0; k < N; ++k)
                    f(float(q[j][k]), first[j] + k);
    }
}

// Counts and weights of a share of the logits in each bin, or in each fine one of a bin, `first` on.
template <typename T>
__device__ __forceinline__ void fill_bins(const T *x, int V, int share, int shares, const Row &r, const Bins &bins, int first, float least,
                                          WideShared &s) {
    __syncthreads();
    for (int i = threadIdx.x; i < kFine; i += kWide)
        s.mass[i] = s.count[i] = 0;
    __syncthreads();
    for_share(x, V, share, shares, [&](float v, int) {
        const int bin = bins.of(v) - first;
        if (unsigned(bin) < unsigned(kFine) && v >= least) {
            atomicAdd(&s.count[bin], 1u);
            atomicAdd(reinterpret_cast<unsigned long long *>(&s.mass[bin]), (unsigned long long)r.weight(v));
        }
    });
    __syncthreads();
}

// The bin in which the count (by_mass: the weights) from the top reaches `target`, which it does within the bins; `left`
// receives what is left of the target there, `above` the weights of the bins above.
__device__ __forceinline__ int bin_of(bool by_mass, uint64_t target, uint64_t &left, uint64_t &above, WideShared &s) {
    constexpr int kEach = kFine / kWide;
    uint64_t mine = 0, mine_mass = 0, all;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int b = threadIdx.x * kEach + i;
        mine += by_mass ? s.mass[b] : s.count[b];
        mine_mass += s.mass[b];
    }
    uint64_t sum = WideBlock::before(mine, all, s.block);
    uint64_t sum_mass = WideBlock::before(mine_mass, all, s.block);
    if (sum < target && target <= sum + mine)
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int b = threadIdx.x * kEach + i;
            const uint64_t here = by_mass ? s.mass[b] : s.count[b];
            if (sum < target && target <= sum + here) {
                s.found = b;
                s.found_left = target - sum;
                s.found_mass = sum_mass;
            }
            sum += here;
            sum_mass += s.mass[b];
        }
    __syncthreads();
    left = s.found_left;
    above = s.found_mass;
    return s.found;
}

// The same bin, and where it has more entries than a list the fine one, for which the row is read once more.
struct Place {
    uint64_t left, above;
    int bin, members;
    bool fine;
};
template <typename T>
__device__ __forceinline__ Place place_in_bins(const T *x, int V, const Row &r, float least, bool by_mass, uint64_t target, WideShared &s) {
    Place p;
    p.fine = false;
    p.bin = bin_of(by_mass, target, p.left, p.above, s);
    p.members = int(s.count[p.bin]);
    const Bins bins(r, true);
    if (p.members > kMembers && bins.have_fine()) {
        uint64_t above;
        fill_bins(x, V, 0, 1, r, bins, p.bin * kFine, least, s);
        const int bin = bin_of(by_mass, p.left, p.left, above, s);
        p.members = int(s.count[bin]);
        p.bin = p.bin * kFine + bin;
        p.above += above;
        p.fine = true;
    }
    return p;
}

// What workgroups of a row leave for the last of them goes past their caches, each of which belongs to some of them only.
template <typename V> __device__ __forceinline__ void leave(V *p, V v) { __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
template <typename V> __device__ __forceinline__ V left_at(const V *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of `shares` to come here, so that what the others left is there. Every wave waits for its
// stores before the arrival is counted; fences, which write back and empty a whole cache, took 40 us of 64 rows in 8 shares.
__device__ __forceinline__ bool is_last(unsigned *arrived, int shares, WideShared &s) {
    if (shares == 1)
        return true;
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
    if (threadIdx.x == 0)
        s.last = atomicAdd(arrived, 1u) == unsigned(shares - 1);
    __syncthreads();
    return s.last;
}

// Where the last kept token is: counts and weights in bins of the distance from the largest logit say in which. Bound by latency,
// the row's loads and the bins' sums in LDS and then over workgroups: 12 us for the ten rows of C that come here, 19 for the 64 of E,
// whose 33 MB would take 5.
template <typename T>
__global__ void __launch_bounds__(kWide) __attribute__((amdgpu_waves_per_eu(4))) wide_place_kernel(const T *logits, Args a, Digest g) {
    __shared__ WideShared s;
    const int tid = threadIdx.x;
    const unsigned wide = *g.wide;
    if (wide == 0)
        return;
    const int shares = shares_of(wide, g.parts);
    const int64_t items = int64_t(wide) * shares;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t slot = item / shares;
        WideRow &w = g.rows[slot];
        const int64_t row = w.row;
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        const float least = w.least;
        const Row r(w.top, p.scale, a.shift);
        const Bins bins(r);
        uint64_t last = least == -INFINITY ? 0 : entry_of(key_of(least), -1);
        Place place{0, 0, kNoBin, 0, false};
        bool by_mass = false;
        if (p.top_k < a.V || p.fraction < kOne) {
            fill_bins(x, a.V, int(item - slot * shares), shares, r, bins, 0, least, s);
            if (shares > 1) {
                uint64_t *all = g.bins + slot * kFine;
                unsigned *number = g.members + slot * kFine;
                for (int i = tid; i < kFine; i += kWide)
                    if (s.count[i]) {
                        atomicAdd(number + i, s.count[i]);
                        atomicAdd(reinterpret_cast<unsigned long long *>(all + i), (unsigned long long)s.mass[i]);
                    }
                if (!is_last(&w.arrived[0], shares, s))
                    continue;
                for (int i = tid; i < kFine; i += kWide) {
                    s.mass[i] = left_at(all + i);
                    s.count[i] = left_at(number + i);
                }
                __syncthreads();
            }
            uint64_t there = 0, inside = 0;
            for (int i = tid; i < kFine; i += kWide) {
                there += s.count[i];
                inside += s.mass[i];
            }
            there = WideBlock::sum(there, s.block);
            inside = WideBlock::sum(inside, s.block);
            const bool cut = uint64_t(p.top_k) < there; // otherwise what it cuts off is beyond the bins
            if (cut)
                place = place_in_bins(x, a.V, r, least, false, uint64_t(p.top_k), s);
            else if (p.top_k < a.V && p.fraction == kOne && wants_logp(a)) { // the share of what it cuts off there, which has no part in the token
                uint64_t all = 0;
                for_share(x, a.V, 0, 1, [&](float v, int) { all += v >= least && v > -INFINITY; });
                if (uint64_t(p.top_k) < WideBlock::sum(all, s.block))
                    last = WideBlock::place_of<false>(x, a.V, r, least, uint64_t(p.top_k), inside, s.mass, s.count, s.block);
            }
            if (cut && p.fraction < kOne) { // what top_p is a share of has to be known
                const bool read_again = place.fine || place.members > kMembers;
                if (place.members > kMembers)
                    last = WideBlock::place_of<false>(x, a.V, r, least, uint64_t(p.top_k), inside, s.mass, s.count, s.block);
                else {
                    const Bins fine(r, place.fine);
                    __syncthreads();
                    if (tid == 0)
                        s.n = 0;
                    __syncthreads();
                    for_share(x, a.V, 0, 1, [&](float v, int i) {
                        if (fine.of(v) == place.bin && v >= least)
                            s.list[atomicAdd(&s.n, 1)] = entry_of(key_of(v), i);
                    });
                    __syncthreads();
                    List<kWide>::find<Order::kLogits, T>(false, place.left, s.list, place.members, 0, 0, 0, r, inside, s.find, s.block);
                    inside += place.above;
                    __syncthreads();
                }
                if (read_again)
                    fill_bins(x, a.V, 0, 1, r, bins, 0, least, s);
            }
            if (p.fraction < kOne) {
                by_mass = true;
                place = place_in_bins(x, a.V, r, least, true, std::max(share_up(inside, p.fraction), uint64_t(1)), s);
            }
            if (place.members > kMembers) { // a great many equals, or as good as equal
                __syncthreads();
                const uint64_t target = by_mass ? std::max(share_up(inside, p.fraction), uint64_t(1)) : uint64_t(p.top_k);
                uint64_t unused;
                last = by_mass ? WideBlock::place_of<true>(x, a.V, r, least, target, unused, s.mass, s.count, s.block)
                               : WideBlock::place_of<false>(x, a.V, r, least, target, unused, s.mass, s.count, s.block);
                place.bin = kNoBin;
            }
        }
        if (tid == 0) {
            w.last = last;
            w.left = place.left;
            w.bin = place.bin;
            w.members = place.members;
            w.by_mass = by_mass;
            w.fine = place.fine;
        }
        __syncthreads();
    }
}

// The kept weights of every part, the bin's entries, and the token. 20 us for the rows of C, 36 for those of E: the weights again,
// then a chain of latency in the last workgroup of every row (the bin's entries back from memory, the place among them, the part, the
// token). With the registers of two or three waves of a SIMD C took 107 us instead of 111 and E 82 instead of 75. Four
// loads at a time instead of a part's eight: E 74 instead of 76.
template <typename T>
__global__ void __launch_bounds__(kWide) __attribute__((amdgpu_waves_per_eu(4))) wide_pick_kernel(const T *logits, Args a, Digest g) {
    __shared__ WideShared s;
    using P = Part<T>;
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    const unsigned wide = *g.wide;
    if (wide == 0)
        return;
    const int shares = shares_of(wide, g.parts);
    const int64_t items = int64_t(wide) * shares;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int64_t slot = item / shares;
        WideRow &w = g.rows[slot];
        const int64_t row = w.row;
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        const Row r(w.top, p.scale, a.shift);
        const Bins bins(r, w.fine);
        const float least = w.least;
        const int bin = w.bin;
        const bool exact = bin == kNoBin;
        const Last last(w.last);
        uint64_t *list = g.list + slot * kMembers, *kept_of = g.kept + slot * kMostParts; // where the row is shared
        double *lost_of = g.lost + slot * kMostParts;
        const bool wants = wants_logp(a);
        if (tid == 0)
            s.n = 0;
        __syncthreads();
        for (int part = int(item - slot * shares) + wave * shares; part < g.parts; part += shares * WideBlock::kWaves) {
            uint64_t mass = 0;
            double lost = 0.0;
            constexpr int kLoads = 4; // on their way at a time
#pragma unroll 1
            for (int i = 0; i < P::kLoads; i += kLoads) {
                typename Vec<T>::type q[kLoads];
                int at[kLoads];
#pragma unroll
                for (int j = 0; j < kLoads; ++j)
                    q[j] = read_at(x, a.V, part * kPart + P::at(i + j, lane), at[j]);
#pragma unroll
                for (int j = 0; j < kLoads; ++j)
#pragma unroll
                    for (int k = 0; k < P::N; ++k) {
                        const float v = float(q[j][k]);
                        const int mine = bins.of(v);
                        const bool in = v >= least;
                        const bool keep = exact ? last.keeps(v, at[j] + k) : in && mine < bin;
                        if (!exact && in && mine == bin)
                            s.list[atomicAdd(&s.n, 1)] = entry_of(key_of(v), at[j] + k);
                        else if (keep || wants) {
                            const double w = r.power(v);
                            mass += keep ? whole_of(w) : 0;
                            lost += keep || v == -INFINITY ? 0.0 : w;
                        }
                    }
            }
            mass = wave_sum(mass);
            lost = wave_sum(lost);
            if (lane == 0) {
                if (shares > 1) {
                    leave(kept_of + part, mass);
                    leave(lost_of + part, lost);
                } else {
                    s.kept[part] = mass;
                    s.lost[part] = lost;
                }
            }
        }
        if (shares > 1) {
            __syncthreads();
            if (tid == 0)
                s.found = int(atomicAdd(&w.listed, unsigned(s.n)));
            __syncthreads();
            for (int i = tid; i < s.n; i += kWide)
                leave(list + s.found + i, s.list[i]);
        }
        if (!is_last(&w.arrived[1], shares, s))
            continue;
        __syncthreads();
        uint64_t end = w.last;
        if (shares > 1 && tid < g.parts) {
            s.kept[tid] = left_at(kept_of + tid);
            s.lost[tid] = left_at(lost_of + tid);
        }
        double below = 0.0; // of the bin's entries that are not kept
        if (!exact) {
            const int n = w.members;
            if (shares > 1)
                for (int i = tid; i < n; i += kWide)
                    s.list[i] = left_at(list + i);
            uint64_t unused;
            __syncthreads();
            end = List<kWide>::find<Order::kLogits, T>(w.by_mass, w.left, s.list, n, 0, 0, 0, r, unused, s.find, s.block);
            for (int i = tid; i < n; i += kWide) {
                const uint64_t e = s.list[i];
                if (e >= end)
                    atomicAdd(reinterpret_cast<unsigned long long *>(&s.kept[index_of(e) / kPart]), (unsigned long long)r.key_weight(key_in(e)));
            }
            if (wants)
                below = List<kWide>::below(s.list, n, end, r, s.block);
        }
        __syncthreads();
        uint64_t kept;
        const uint64_t mine = tid < g.parts ? s.kept[tid] : 0;
        const uint64_t sum = WideBlock::before(mine, kept, s.block);
        const double dropped = WideBlock::sum(tid < g.parts ? s.lost[tid] : 0.0, s.block) + below;
        const uint64_t target = share_down(kept, p.at);
        if (sum <= target && target < sum + mine) {
            s.found = tid;
            s.found_left = target - sum;
            s.found_mass = mine;
        }
        __syncthreads();
        pick_in_part<T, kWide>(a, x, s.found, r, Last(end), s.found_left, s.found_mass, s.out, s.block);
        __syncthreads();
        if (tid == 0)
            finish_row(a, row, r, s.out.token, s.out.x, double(kept), dropped);
    }
}

// ------------------------------------------------------------------------------------------------
// rows too long for a digest
// ------------------------------------------------------------------------------------------------
constexpr int kLong = 1024;

// The plain way, for vocabularies beyond what there are: a workgroup reads the row once for its largest logit, once for its weights,
// five times for each place and twice for the token.
template <typename T>
__global__ void __launch_bounds__(kLong) long_kernel(const T *logits, Args a) {
    using B = Block<kLong>;
    __shared__ B::Shared s;
    __shared__ uint64_t mass[kBins];
    __shared__ uint32_t count[kBins];
    __shared__ uint64_t part[B::kWaves];
    const int tid = threadIdx.x, lane = tid % kWave, wave = tid / kWave;
    for (int64_t row = blockIdx.x; row < a.n; row += gridDim.x) {
        const Params p = params_of(a, row);
        const T *x = logits + row * a.stride;
        float m = -INFINITY;
        for (int64_t i = tid; i < a.V; i += kLong)
            m = larger(m, float(x[i]));
        m = B::max(m, s);
        if (p.scale == 0.0 || !(m < INFINITY) || m == -INFINITY) {
            finish_without(a, row, p.scale == 0.0 || m != -INFINITY);
            continue;
        }
        const Row r(m, p.scale, a.shift);
        const uint32_t floor = floor_key(r.m, p.scale, p.least, key_of(m));
        const float least = floor ? float_of(floor) : -INFINITY;
        uint64_t inside = 0, there = 0, unused;
        for (int64_t i = tid; i < a.V; i += kLong) {
            const float v = float(x[i]);
            inside += v >= least ? r.weight(v) : 0;
            there += v >= least;
        }
        inside = B::sum(inside, s);
        there = B::sum(there, s);
        uint64_t end = floor ? entry_of(floor, -1) : 0;
        if (uint64_t(p.top_k) < there)
            end = B::template place_of<false>(x, a.V, r, least, uint64_t(p.top_k), inside, mass, count, s);
        if (p.fraction < kOne)
            end = B::template place_of<true>(x, a.V, r, least, std::max(share_up(inside, p.fraction), uint64_t(1)), unused, mass, count, s);
        const Last last(end);
        // waves take stretches of the vocabulary
        const int64_t each = int64_t((a.V - 1) / kLong + 1) * kWave;
        const int64_t from = std::min(wave * each, int64_t(a.V)), to = std::min(from + each, int64_t(a.V));
        uint64_t mine = 0;
        double lost = 0.0;
        for (int64_t i = from + lane; i < to; i += kWave) {
            const float v = float(x[i]);
            const bool keep = last.keeps(v, int(i));
            const double w = r.power(v);
            mine += keep ? whole_of(w) : 0;
            lost += keep || v == -INFINITY ? 0.0 : w;
        }
        lost = B::sum(lost, s);
        mine = wave_sum(mine);
        __syncthreads();
        if (lane == 0)
            part[wave] = mine;
        __syncthreads();
        uint64_t kept = 0, sum = 0;
        for (int w = 0; w < B::kWaves; ++w) {
            sum = w == wave ? kept : sum;
            kept += part[w];
        }
        const uint64_t target = share_down(kept, p.at);
        const bool first = sum <= target;
        for (int64_t i = from + lane; i - lane < to && sum <= target; i += kWave) {
            const float v = i < to ? float(x[i]) : -INFINITY;
            const uint64_t with = sum + wave_scan(i < to && last.keeps(v, int(i)) ? r.weight(v) : 0);
            const uint64_t past = __ballot(with > target);
            if (first && past && lane == __builtin_ctzll(past))
                finish_row(a, row, r, int(i), v, double(kept), lost);
            sum = last_lane(with);
        }
        __syncthreads();
    }
}

// How rows of V tokens are taken, whatever their number. By a wave where it holds the row: 20,000 x 500 bf16, top-k and top-p, take
// 136 us, with 256 threads to a row 307, but 64 of them 19 and 14; 200,000 x 136 take 602 us with four logits a thread, 631 with eight,
// 2,412 with 256 threads. By 256 threads up to 2,048: 2,000 x 2,000 take 69 us, by way of a digest 155, and 64 of them 21 and 39.
struct Plan {
    int group, own; // of small_kernel; 0: a digest
    int parts;      // 0 and no group: long_kernel
};

Plan plan_of(int64_t V) {
    if (V <= 4 * kWave)
        return {kWave, 4, 0};
    if (V <= 8 * kWave)
        return {kWave, 8, 0};
    if (V <= 8 * 256)
        return {256, 8, 0};
    if (V >= int64_t(kMostParts) * kPart)
        return {0, 0, 0};
    return {0, 0, int((V + kPart - 1) / kPart)};
}

// What the kernels leave for the next ones, behind each other in the workspace.
struct Space {
    char *at;
    int64_t bytes = 0;
    template <typename T> T *take(int64_t count) {
        T *p = reinterpret_cast<T *>(at + bytes);
        bytes += (count * int64_t(sizeof(T)) + 15) / 16 * 16;
        return p;
    }
};

// Its bytes, and where its parts are in a workspace at `at`.
int64_t lay_out(const Plan &p, int64_t n, char *at, Digest &g) {
    Space s{at};
    g.parts = p.parts;
    if (!p.parts)
        return 0;
    g.wide = s.take<unsigned>(1);
    g.rows = s.take<WideRow>(n);
    g.mass = s.take<double>(n * p.parts);
    g.top = s.take<float>(n * p.parts);
    g.seg = s.take<float>(n * p.parts * kSegs);
    const int64_t slots = std::min<int64_t>(n, kShared);
    g.bins = s.take<uint64_t>(slots * kFine);
    g.members = s.take<unsigned>(slots * kFine);
    g.kept = s.take<uint64_t>(slots * kMostParts);
    g.lost = s.take<double>(slots * kMostParts);
    g.list = s.take<uint64_t>(slots * kMembers);
    return s.bytes;
}

int size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }

using treeens::set_error;

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

int check_sizes(int32_t dtype, int64_t n, int64_t V) {
    if (dtype != TREE_ENS_F32 && dtype != TREE_ENS_BF16 && dtype != TREE_ENS_F16)
        return set_error(TREE_ENS_E_ARG, "dtype must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
    if (n < 0 || V < 1 || V > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and n_vocab in [1, INT32_MAX]");
    if (n > INT64_MAX / 1024 / kMostParts)
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
    Digest g;
    if (n_tokens > 0)
        *bytes = lay_out(plan_of(n_vocab), n_tokens, nullptr, g);
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
    Digest g;
    if (const int64_t need = lay_out(plan, n_tokens, static_cast<char *>(workspace), g)) {
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
        if (plan.group) {
            const auto kernel = plan.group == 256 ? small_kernel<T, 256, 8> : plan.own == 8 ? small_kernel<T, kWave, 8> : small_kernel<T, kWave, 4>;
            hipLaunchKernelGGL(kernel, rows, dim3(unsigned(plan.group)), 0, s, x, a);
        } else if (plan.parts) {
            const int64_t blocks = n_tokens * ((plan.parts + 3) / 4);
            hipLaunchKernelGGL(scan_kernel<T>, dim3(unsigned(std::min(blocks, kMaxBlocks))), dim3(256), 0, s, x, a, g);
            hipLaunchKernelGGL(pick_kernel<T>, rows, dim3(kPick), unsigned(plan.parts * kSegBytes), s, x, a, g);
            if (!row_top_k && !row_top_p && !row_min_p && a.top_k == 0 && top_p == 1.0f && min_p == 0.0f)
                return; // no row is cut off
            const dim3 wide(unsigned(std::min<int64_t>(n_tokens * kMostShares, 2 * kShared)));
            hipLaunchKernelGGL(wide_place_kernel<T>, wide, dim3(kWide), 0, s, x, a, g);
            hipLaunchKernelGGL(wide_pick_kernel<T>, wide, dim3(kWide), 0, s, x, a, g);
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
