// losses.hip -- losses over packed sequences of token log-probabilities, with their gradients, and
// advantages of scores relative to their group, on gfx950.
//
// Segments: sequence s owns tokens [seq_offsets[s], seq_offsets[s+1]), group g owns sequences
// [group_offsets[g], group_offsets[g+1]). Sums over tokens and over pairs are held in double.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <string>

#include "status.hpp"
#include "tree_ens.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;
constexpr int kWaves = kThreads / kWave;
constexpr int64_t kMaxBlocks = 1 << 20; // segments beyond this many are taken in turn

struct Span {
    int64_t a, b;
};

// Segment i of `offsets`, clamped into [0, n].
__device__ __forceinline__ Span span_of(const int64_t *offsets, int64_t i, int64_t n) {
    const int64_t a = min(max(offsets[i], int64_t(0)), n);
    return {a, min(max(offsets[i + 1], a), n)};
}

__device__ __forceinline__ double wave_sum(double v) {
    for (int off = kWave / 2; off; off >>= 1)
        v += __shfl_xor(v, off);
    return v;
}

// Sum over the workgroup, in a fixed order, for every thread.
__device__ __forceinline__ double block_sum(double v, double *part) {
    v = wave_sum(v);
    __syncthreads(); // part may still be read for the sum before
    if (threadIdx.x % kWave == 0)
        part[threadIdx.x / kWave] = v;
    __syncthreads();
    v = part[0];
    for (int w = 1; w < kWaves; ++w)
        v += part[w];
    return v;
}

// Zero what lies before the first and after the last of n segments (all of it without any).
__device__ __forceinline__ void zero_outside(float *out, int64_t size, const int64_t *offsets, int64_t i, int64_t n, Span s) {
    if (i == 0)
        for (int64_t t = threadIdx.x; t < s.a; t += kThreads)
            out[t] = 0.0f;
    if (i == n - 1)
        for (int64_t t = s.b + threadIdx.x; t < size; t += kThreads)
            out[t] = 0.0f;
}

__global__ void __launch_bounds__(kThreads) zero_kernel(float *out, int64_t size) {
    for (int64_t t = blockIdx.x * int64_t(kThreads) + threadIdx.x; t < size; t += int64_t(gridDim.x) * kThreads)
        out[t] = 0.0f;
}

struct Tokens {
    const float *logp, *ref;
    const uint8_t *mask;
    int64_t n;
    const int64_t *offsets;
    int64_t n_seqs;
    __device__ __forceinline__ bool counts(int64_t t) const { return !mask || mask[t]; }
};

// ---------------------------------------------------------------------------------------------
// Tiles of tokens
//
// Sums over sequences of any lengths read the tokens in tiles of equal size, eight neighbours a thread,
// so no workgroup waits for a long sequence. A thread finds the sequence of its first token by search
// and walks on; what a sequence leaves open at a thread's end is carried to the next one by a segmented
// scan over the workgroup. A sequence inside one tile has its sum stored by the tile; one that goes on
// leaves the tile's `tail` where it begins and `head` in every later tile, added up afterwards in order.
// ---------------------------------------------------------------------------------------------
constexpr int kEach = 8;
constexpr int kTile = kThreads * kEach;

struct Pair {
    double a, b;
};
__device__ __forceinline__ Pair operator+(Pair x, Pair y) { return {x.a + y.a, x.b + y.b}; }

// Two sums per sequence and two per tile.
struct Sums {
    Pair *inside; // [n_seqs], of sequences inside one tile
    Pair *head;   // [tiles]
    Pair *tail;   // [tiles]
};

// The last s in [-1, n_seqs] with offsets[s] <= t (-1: none), by 64 pivots at a time. Offsets that
// decrease give some index of the range.
__device__ __forceinline__ int64_t sequence_at(const int64_t *offsets, int64_t n_seqs, int64_t t) {
    int64_t lo = -1, hi = n_seqs + 1; // offsets[lo] <= t < offsets[hi]
    while (hi - lo > 1) {
        const int64_t step = (hi - lo + kWave) / (kWave + 1), p = lo + (threadIdx.x % kWave + 1) * step;
        lo += __popcll(__ballot(p < hi && offsets[p] <= t)) * step;
        hi = min(hi, lo + step);
    }
    return lo;
}

// The sequence of a token, while the token moves on inside a tile. -1 and n_seqs stand for the tokens
// before the first and after the last sequence.
struct Walk {
    const int64_t *offsets;
    int64_t n_seqs, n, last, s, end; // last: the sequence of the tile's last token
    __device__ __forceinline__ bool inside() const { return s >= 0 && s < n_seqs; }
    __device__ __forceinline__ int64_t start() const { return s < 0 ? 0 : max(offsets[s], int64_t(0)); }
    __device__ __forceinline__ int64_t end_of(int64_t i) const { return i < n_seqs ? min(offsets[i + 1], n) : n; }
    // s: a sequence at or before that of t
    __device__ __forceinline__ void place(int64_t t) {
        int64_t lo = s, hi = last;
        while (lo < hi) {
            const int64_t mid = lo + (hi - lo + 1) / 2;
            if (offsets[mid] <= t)
                lo = mid;
            else
                hi = mid - 1;
        }
        s = lo;
        end = end_of(s);
    }
};

__device__ __forceinline__ Walk walk_from(const Tokens &in, int64_t first, int64_t count) {
    Walk w{in.offsets, in.n_seqs, in.n, 0, 0, 0};
    w.s = sequence_at(in.offsets, in.n_seqs, first);
    w.last = sequence_at(in.offsets, in.n_seqs, first + count - 1);
    return w;
}

typedef float float4_ __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned char byte8_ __attribute__((ext_vector_type(8), aligned(1)));

// A thread's tokens [t, t + count) of an array.
__device__ __forceinline__ void load_tokens(const float *p, int64_t t, int count, float (&x)[kEach]) {
    if (count == kEach) {
        const float4_ a = *reinterpret_cast<const float4_ *>(p + t), b = *reinterpret_cast<const float4_ *>(p + t + 4);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            x[k] = a[k];
            x[k + 4] = b[k];
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        x[k] = k < count ? p[t + k] : 0.0f;
}

__device__ __forceinline__ void store_tokens(float *p, int64_t t, int count, const float (&x)[kEach]) {
    if (count == kEach) {
        *reinterpret_cast<float4_ *>(p + t) = float4_{x[0], x[1], x[2], x[3]};
        *reinterpret_cast<float4_ *>(p + t + 4) = float4_{x[4], x[5], x[6], x[7]};
        return;
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k)
        if (k < count)
            p[t + k] = x[k];
}

// Bit k: token t + k counts.
__device__ __forceinline__ unsigned load_mask(const uint8_t *mask, int64_t t, int count) {
    unsigned bits = 0;
    if (!mask || count <= 0)
        return count <= 0 ? 0u : (1u << count) - 1;
    if (count == kEach) {
        const byte8_ m = *reinterpret_cast<const byte8_ *>(mask + t);
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            bits |= unsigned(m[k] != 0) << k;
        return bits;
    }
    for (int k = 0; k < count; ++k)
        bits |= unsigned(mask[t + k] != 0) << k;
    return bits;
}

__device__ __forceinline__ Pair shuffle_up(Pair x, int by) { return {__shfl_up(x.a, by), __shfl_up(x.b, by)}; }

// Adds up value(k) of the tile's tokens by sequence and stores the sums. enter() is called when the
// walk has come to another sequence, before the value of its first token is asked for.
template <typename Enter, typename Value>
__device__ __forceinline__ void sum_tile(const Sums &out, int64_t tile, int64_t n, Walk w, Enter &&enter, Value &&value) {
    __shared__ Pair part[kWaves];
    __shared__ bool closed[kWaves];
    const int64_t first = tile * kTile, t = first + threadIdx.x * kEach;
    const int count = int(max(int64_t(0), min(int64_t(kEach), n - t)));
    Pair open{0.0, 0.0}, head{0.0, 0.0}; // of the sequence being walked; of the one that the thread began in
    bool ended = false;                  // some sequence ended in this thread
    int64_t head_s = -1;                 // the one that the thread began in, if it ends here
    bool head_before = false;            // and began before the tile
    if (count > 0) {
        w.place(t);
        enter(w);
        bool own = w.start() >= t; // the walked sequence began in this thread
        const bool before = w.start() < first;
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (k < count) {
                if (t + k >= w.end) {
                    w.s += 1;
                    w.place(t + k);
                    enter(w);
                }
                const Pair v = value(k);
                open = open + v;
                if (t + k + 1 >= w.end) {
                    if (w.inside()) {
                        if (own) {
                            out.inside[w.s] = open;
                        } else {
                            head = open;
                            head_s = w.s;
                            head_before = before;
                        }
                    }
                    open = {0.0, 0.0};
                    ended = own = true;
                }
            }
        }
    }
    // inclusive scan of what is open, restarted wherever a sequence ended
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    Pair run = open;
    bool stop = ended;
#pragma unroll
    for (int off = 1; off < kWave; off <<= 1) {
        const Pair p = shuffle_up(run, off);
        const bool q = __shfl_up(int(stop), off);
        if (lane >= off && !stop) {
            run = run + p;
            stop = q;
        }
    }
    __syncthreads(); // the tile before has been read
    if (lane == kWave - 1) {
        part[wave] = run;
        closed[wave] = stop;
    }
    __syncthreads();
    Pair carry = shuffle_up(run, 1);
    bool stopped = __shfl_up(int(stop), 1);
    if (lane == 0) {
        carry = {0.0, 0.0};
        stopped = false;
    }
    for (int k = wave - 1; k >= 0 && !stopped; --k) {
        carry = part[k] + carry;
        stopped = closed[k];
    }
    if (head_s >= 0)
        (head_before ? out.head[tile] : out.inside[head_s]) = carry + head;
    if (threadIdx.x == kThreads - 1) { // a sequence that goes on in the next tile
        const int64_t end = min(first + kTile, n);
        w.s = w.last;
        if (w.inside() && w.end_of(w.s) > end)
            (w.start() < first ? out.head : out.tail)[tile] = ended ? open : carry + open;
    }
}

// The sums of a sequence, from the tiles.
__device__ __forceinline__ Pair joined(const Sums &in, int64_t s, Span q) {
    if (q.a == q.b)
        return {0.0, 0.0};
    const int64_t first = q.a / kTile, last = (q.b - 1) / kTile;
    if (first == last)
        return in.inside[s];
    Pair sum = in.tail[first];
#pragma unroll 4
    for (int64_t k = first + 1; k <= last; ++k)
        sum = sum + in.head[k];
    return sum;
}

// ---------------------------------------------------------------------------------------------
// Preference loss
// ---------------------------------------------------------------------------------------------

// Sums of a sequence's log ratios, and how many count.
__global__ void __launch_bounds__(kThreads) ratio_tile_kernel(Tokens in, Sums out) {
    const int64_t tiles = (in.n + kTile - 1) / kTile;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t first = tile * kTile, t = first + threadIdx.x * kEach;
        const int count = int(max(int64_t(0), min(int64_t(kEach), in.n - t)));
        float x[kEach], r[kEach] = {};
        load_tokens(in.logp, t, count, x);
        if (in.ref)
            load_tokens(in.ref, t, count, r);
        const unsigned use = load_mask(in.mask, t, count);
        sum_tile(out, tile, in.n, walk_from(in, first, min(int64_t(kTile), in.n - first)), [](const Walk &) {},
                 [&](int k) { return use >> k & 1u ? Pair{double(x[k] - r[k]), 1.0} : Pair{0.0, 0.0}; });
    }
}

struct Preference {
    const float *scores;
    const int64_t *groups;
    int64_t n_groups;
    float beta, smoothing, grad_scale;
    bool mean;
    float *loss, *margins, *weights; // weights: dh / dlogp of a counted token, then the loss's gradient
};

// Margins and weights of the sequences [a, b), by the threads of a workgroup.
__device__ __forceinline__ void join_margins(const Tokens &in, const Sums &sums, const Preference &p, int64_t a, int64_t b, bool alone) {
    for (int64_t s = a + threadIdx.x; s < b; s += kThreads) {
        const Pair v = joined(sums, s, span_of(in.offsets, s, in.n));
        const double w = p.mean ? double(p.beta) / fmax(v.b, 1.0) : double(p.beta);
        p.margins[s] = float(w * v.a);
        p.weights[s] = alone ? 0.0f : float(w); // alone: in no group
    }
}

// softplus(-d) = max(-d, 0) + log1p(e) and sigmoid(-d) of e = exp(-|d|).
struct Logistic {
    float softplus, sigmoid;
};
__device__ __forceinline__ Logistic logistic(float d) {
    const float e = __builtin_amdgcn_exp2f(-1.44269504088896340736f * fabsf(d));
    const float u = 1.0f + e, r = __builtin_amdgcn_rcpf(u);
    // log1p(e) = log u + log(1 + rest / u), with the rest that u was rounded by
    const float l = fmaf(e - (u - 1.0f), r, 0.69314718055994530942f * __builtin_amdgcn_logf(u));
    return {(d < 0.0f ? -d : 0.0f) + l, d >= 0.0f ? e * r : r};
}

// Loss of a group, and weights times the loss's gradient with respect to the margins. With d the
// margin of a pair, l = softplus(-d) + smoothing d and dl/dd = smoothing - sigmoid(-d). Every candidate
// meets every other one, so each pair is met twice and nothing is added atomically.
__global__ void __launch_bounds__(kThreads) pairs_kernel(Tokens in, Sums sums, Preference p) {
    __shared__ double part[kWaves];
    __shared__ float2 other[kThreads]; // (margin, score) of the candidates that are met
    __shared__ float slopes[kThreads];
    for (int64_t g = blockIdx.x; g < max(p.n_groups, int64_t(1)); g += gridDim.x) {
        Span q{in.n_seqs, in.n_seqs}; // without groups, every sequence is before the first one
        if (p.n_groups > 0)
            q = span_of(p.groups, g, in.n_seqs);
        if (g == 0)
            join_margins(in, sums, p, 0, q.a, true);
        if (g == p.n_groups - 1)
            join_margins(in, sums, p, q.b, in.n_seqs, true);
        if (p.n_groups == 0)
            return;
        join_margins(in, sums, p, q.a, q.b, false);
        __syncthreads();
        // as many candidates at a time as fit, each by the same number of threads
        const int64_t n = q.b - q.a;
        const int rows = int(max(int64_t(1), min(n, int64_t(kThreads)))), shares = kThreads / rows;
        const int row = threadIdx.x % rows, share = threadIdx.x / rows;
        double total = 0.0, pairs = 0.0;
        for (int64_t i0 = 0; i0 < n; i0 += rows) {
            const int64_t i = i0 + row;
            const bool mine = i < n && share < shares;
            const float h = mine ? p.margins[q.a + i] : 0.0f, r = mine ? p.scores[q.a + i] : 0.0f;
            float slope = 0.0f;
            for (int64_t j0 = 0; j0 < n; j0 += kThreads) {
                __syncthreads();
                if (j0 + threadIdx.x < n)
                    other[threadIdx.x] = make_float2(p.margins[q.a + j0 + threadIdx.x], p.scores[q.a + j0 + threadIdx.x]);
                __syncthreads();
                if (!mine)
                    continue;
                const int met = int(min(int64_t(kThreads), n - j0));
                float sum = 0.0f;
                int found = 0;
                for (int j = share; j < met; j += shares) {
                    const float2 o = other[j];
                    const bool ahead = r > o.y, behind = r < o.y;
                    if (!ahead && !behind)
                        continue;
                    const float d = ahead ? h - o.x : o.x - h;
                    const Logistic l = logistic(d);
                    const float dl = p.smoothing - l.sigmoid;
                    slope += ahead ? dl : -dl;
                    if (ahead) {
                        sum += l.softplus;
                        if (p.smoothing > 0.0f)
                            sum = fmaf(p.smoothing, d, sum);
                        ++found;
                    }
                }
                total += sum;
                pairs += found;
            }
            if (p.grad_scale != 0.0f) { // raw slopes; the number of pairs is not known yet
                __syncthreads();
                slopes[threadIdx.x] = slope;
                __syncthreads();
                if (threadIdx.x < rows && i < n) {
                    double sum = slope;
                    for (int k = 1; k < shares; ++k)
                        sum += slopes[k * rows + row];
                    p.weights[q.a + i] = float(p.weights[q.a + i] * sum);
                }
            }
        }
        total = block_sum(total, part);
        pairs = block_sum(pairs, part);
        if (threadIdx.x == 0)
            p.loss[g] = float(total / fmax(pairs, 1.0));
        const double by = double(p.grad_scale) / fmax(pairs, 1.0);
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            p.weights[i] = float(p.weights[i] * by);
        __syncthreads();
    }
}

// grad[t] = the sequence's weight at its counted tokens.
__global__ void __launch_bounds__(kThreads) spread_tile_kernel(Tokens in, const float *weights, float *grad) {
    const int64_t tiles = (in.n + kTile - 1) / kTile;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t first = tile * kTile, t = first + threadIdx.x * kEach;
        const int count = int(max(int64_t(0), min(int64_t(kEach), in.n - t)));
        const unsigned use = load_mask(in.mask, t, count);
        Walk w = walk_from(in, first, min(int64_t(kTile), in.n - first));
        if (count <= 0)
            continue;
        w.place(t);
        float x = w.inside() ? weights[w.s] : 0.0f, d[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            if (k < count && t + k >= w.end) {
                w.s += 1;
                w.place(t + k);
                x = w.inside() ? weights[w.s] : 0.0f;
            }
            d[k] = use >> k & 1u ? x : 0.0f;
        }
        store_tokens(grad, t, count, d);
    }
}

__global__ void __launch_bounds__(kThreads)
advantage_kernel(const float *scores, int64_t n, const int64_t *groups, int64_t n_groups, float eps, bool center,
                 float *out) {
    __shared__ double part[kWaves];
    for (int64_t g = blockIdx.x; g < n_groups; g += gridDim.x) {
        const Span q = span_of(groups, g, n);
        const double count = fmax(double(q.b - q.a), 1.0);
        double sum = 0.0, squares = 0.0;
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            sum += scores[i];
        const double mean = block_sum(sum, part) / count;
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            squares += (scores[i] - mean) * (scores[i] - mean);
        const double std = sqrt(block_sum(squares, part) / count);
        const double by = center ? 1.0 : 1.0 / (std + eps);
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            out[i] = float((scores[i] - mean) * by);
        zero_outside(out, n, groups, g, n_groups, q);
    }
}

// exp(q) - q - 1: the sum of q^k / k! from k = 2 where the difference would cancel. Below 1/2 the
// terms up to k = 9 leave out less than 2e-9 of it.
__device__ __forceinline__ float exp_less_tangent(float q) {
    if (!(fabsf(q) < 0.5f))
        return expf(q) - q - 1.0f;
    float s = 1.0f / 362880.0f;
    s = fmaf(s, q, 1.0f / 40320.0f);
    s = fmaf(s, q, 1.0f / 5040.0f);
    s = fmaf(s, q, 1.0f / 720.0f);
    s = fmaf(s, q, 1.0f / 120.0f);
    s = fmaf(s, q, 1.0f / 24.0f);
    s = fmaf(s, q, 1.0f / 6.0f);
    s = fmaf(s, q, 0.5f);
    return s * q * q;
}

struct Policy {
    const float *old_logp, *advantages;
    float low, high, kl_coef, grad_scale;
    bool mean;
    float *loss, *kl, *grad;
};

__global__ void __launch_bounds__(kThreads) policy_kernel(Tokens in, Policy p) {
    __shared__ double part[kWaves];
    for (int64_t s = blockIdx.x; s < in.n_seqs; s += gridDim.x) {
        const Span q = span_of(in.offsets, s, in.n);
        const float a = p.advantages[s];
        double share = 1.0;
        if (p.mean) {
            double count = 0.0;
            for (int64_t t = q.a + threadIdx.x; t < q.b; t += kThreads)
                count += in.counts(t) ? 1.0 : 0.0;
            share = 1.0 / fmax(block_sum(count, part), 1.0);
        }
        const float w = float(p.grad_scale * share);
        double loss = 0.0, kl = 0.0;
        for (int64_t t = q.a + threadIdx.x; t < q.b; t += kThreads) {
            float d = 0.0f;
            if (in.counts(t)) {
                const float lp = in.logp[t];
                const float ratio = p.old_logp ? expf(lp - p.old_logp[t]) : 1.0f;
                // comparisons that a NaN ratio passes unchanged
                const bool clipped = a >= 0.0f ? ratio > p.high : ratio < p.low;
                loss -= (clipped ? (a >= 0.0f ? p.high : p.low) : ratio) * a;
                d = clipped ? 0.0f : -a * ratio;
                if (in.ref) {
                    const float x = in.ref[t] - lp, k = exp_less_tangent(x);
                    kl += k;
                    d -= p.kl_coef * (k + x);
                }
            }
            if (p.grad)
                p.grad[t] = w * d;
        }
        loss = block_sum(loss, part);
        kl = block_sum(kl, part);
        if (threadIdx.x == 0) {
            p.loss[s] = float(share * (loss + p.kl_coef * kl));
            if (p.kl)
                p.kl[s] = float(share * kl);
        }
        if (p.grad)
            zero_outside(p.grad, in.n, in.offsets, s, in.n_seqs, q);
    }
}

using treeens::set_error;

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

unsigned blocks_for(int64_t n) { return unsigned(std::min(std::max<int64_t>(n, 1), kMaxBlocks)); }

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(TREE_ENS_E_DEVICE, std::string(what) + " launch: " + hipGetErrorString(e));
    return TREE_ENS_OK;
}

int check_counts(int64_t n_tokens, int64_t n_seqs, int64_t n_groups) {
    if (n_tokens < 0 || n_tokens > INT64_MAX / 64)
        return set_error(TREE_ENS_E_ARG, "n_tokens must be >= 0 and within memory");
    if (n_seqs < 0 || n_seqs > INT32_MAX || n_groups < 0 || n_groups > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "sequence and group counts must be >= 0 and fit int32");
    return TREE_ENS_OK;
}

int check_workspace(const void *workspace, int64_t bytes, int64_t needed) {
    if (needed > 0 && (!workspace || bytes < needed))
        return set_error(TREE_ENS_E_ARG, "workspace is NULL or smaller than " + std::to_string(needed) + " bytes");
    if (needed > 0 && misaligned(workspace, 16))
        return set_error(TREE_ENS_E_ARG, "workspace must be 16-byte aligned");
    return TREE_ENS_OK;
}

// The tokens of both losses: logp and offsets where there are any.
int check_tokens(const float *logp, int64_t n_tokens, const int64_t *seq_offsets, int64_t n_seqs) {
    if ((n_tokens > 0 && !logp) || (n_seqs > 0 && !seq_offsets))
        return set_error(TREE_ENS_E_ARG, "logp or seq_offsets is NULL");
    if (misaligned(logp, 4) || misaligned(seq_offsets, 8))
        return set_error(TREE_ENS_E_ARG, "logp or seq_offsets is misaligned");
    return TREE_ENS_OK;
}

int64_t tiles_of(int64_t n_tokens) { return (n_tokens + kTile - 1) / kTile; }

// Two sums per sequence and tile, 16 bytes each.
int64_t sums_bytes(int64_t n_tokens, int64_t n_seqs) { return 16 * (n_seqs + 2 * tiles_of(n_tokens)); }

Sums sums_at(void *workspace, int64_t n_tokens, int64_t n_seqs) {
    Pair *p = static_cast<Pair *>(workspace);
    return {p, p + n_seqs, p + n_seqs + tiles_of(n_tokens)};
}

int64_t preference_bytes(int64_t n_tokens, int64_t n_seqs) {
    return sums_bytes(n_tokens, n_seqs) + (n_seqs * 4 + 15) / 16 * 16;
}

} // namespace

extern "C" {

int tree_ens_preference_workspace(int64_t n_tokens, int64_t n_seqs, int64_t n_groups, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (int rc = check_counts(n_tokens, n_seqs, n_groups))
        return rc;
    *bytes = preference_bytes(n_tokens, n_seqs);
    return TREE_ENS_OK;
}

int tree_ens_preference_loss(void *stream, const float *logp, const float *ref_logp, const uint8_t *mask,
                             int64_t n_tokens, const int64_t *seq_offsets, int64_t n_seqs, const float *scores,
                             const int64_t *group_offsets, int64_t n_groups, float beta, float smoothing,
                             float grad_scale, uint32_t flags, float *loss, float *margins, float *grad_logp,
                             void *workspace, int64_t workspace_bytes) {
    treeens::clear_error();
    if (int rc = check_counts(n_tokens, n_seqs, n_groups))
        return rc;
    if (!std::isfinite(beta) || !std::isfinite(grad_scale) || !(smoothing >= 0.0f && smoothing < 1.0f))
        return set_error(TREE_ENS_E_ARG, "beta and grad_scale must be finite, smoothing in [0, 1)");
    if (flags & ~TREE_ENS_SEQ_MEAN)
        return set_error(TREE_ENS_E_ARG, "unknown flag bits");
    if (int rc = check_tokens(logp, n_tokens, seq_offsets, n_seqs))
        return rc;
    if ((n_seqs > 0 && (!scores || !margins)) || (n_groups > 0 && (!group_offsets || !loss)))
        return set_error(TREE_ENS_E_ARG, "scores, margins, group_offsets or loss is NULL");
    if (misaligned(ref_logp, 4) || misaligned(scores, 4) || misaligned(group_offsets, 8) || misaligned(loss, 4) ||
        misaligned(margins, 4) || misaligned(grad_logp, 4))
        return set_error(TREE_ENS_E_ARG, "a pointer is misaligned for its type");
    if (int rc = check_workspace(workspace, workspace_bytes, preference_bytes(n_tokens, n_seqs)))
        return rc;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Tokens in{logp, ref_logp, mask, n_tokens, seq_offsets, n_seqs};
    const Sums sums = sums_at(workspace, n_tokens, n_seqs);
    float *weights = reinterpret_cast<float *>(static_cast<char *>(workspace) + sums_bytes(n_tokens, n_seqs));
    const Preference p{scores, group_offsets, n_groups, beta, smoothing, grad_scale, (flags & TREE_ENS_SEQ_MEAN) != 0,
                       loss, margins, weights};
    (void)hipGetLastError();
    if (n_seqs > 0 && n_tokens > 0)
        hipLaunchKernelGGL(ratio_tile_kernel, dim3(blocks_for(tiles_of(n_tokens))), dim3(kThreads), 0, s, in, sums);
    if (n_seqs > 0 || n_groups > 0)
        hipLaunchKernelGGL(pairs_kernel, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, in, sums, p);
    if (grad_logp && n_tokens > 0) {
        if (n_seqs > 0)
            hipLaunchKernelGGL(spread_tile_kernel, dim3(blocks_for(tiles_of(n_tokens))), dim3(kThreads), 0, s, in, weights, grad_logp);
        else
            hipLaunchKernelGGL(zero_kernel, dim3(blocks_for((n_tokens + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                               grad_logp, n_tokens);
    }
    return launched("preference loss");
}

int tree_ens_group_advantage(void *stream, const float *scores, int64_t n_docs, const int64_t *group_offsets,
                             int64_t n_groups, float eps, uint32_t flags, float *advantages) {
    treeens::clear_error();
    if (int rc = check_counts(0, n_docs, n_groups))
        return rc;
    if (!std::isfinite(eps) || !(eps > 0.0f))
        return set_error(TREE_ENS_E_ARG, "eps must be finite and > 0");
    if (flags & ~TREE_ENS_CENTER_ONLY)
        return set_error(TREE_ENS_E_ARG, "unknown flag bits");
    if (n_docs == 0)
        return TREE_ENS_OK;
    if (!scores || !advantages || (n_groups > 0 && !group_offsets))
        return set_error(TREE_ENS_E_ARG, "scores, group_offsets or advantages is NULL");
    if (misaligned(scores, 4) || misaligned(advantages, 4) || misaligned(group_offsets, 8))
        return set_error(TREE_ENS_E_ARG, "a pointer is misaligned for its type");
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    (void)hipGetLastError();
    if (n_groups > 0)
        hipLaunchKernelGGL(advantage_kernel, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, scores, n_docs,
                           group_offsets, n_groups, eps, (flags & TREE_ENS_CENTER_ONLY) != 0, advantages);
    else
        hipLaunchKernelGGL(zero_kernel, dim3(blocks_for((n_docs + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                           advantages, n_docs);
    return launched("group advantage");
}

int tree_ens_policy_workspace(int64_t n_tokens, int64_t n_seqs, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    return check_counts(n_tokens, n_seqs, 0);
}

int tree_ens_policy_loss(void *stream, const float *logp, const float *old_logp, const float *ref_logp,
                         const uint8_t *mask, int64_t n_tokens, const int64_t *seq_offsets, int64_t n_seqs,
                         const float *advantages, float clip_low, float clip_high, float kl_coef, float grad_scale,
                         uint32_t flags, float *loss, float *kl, float *grad_logp, void *workspace,
                         int64_t workspace_bytes) {
    treeens::clear_error();
    if (int rc = check_counts(n_tokens, n_seqs, 0))
        return rc;
    if (!(clip_low >= 0.0f && clip_low <= 1.0f) || !(clip_high >= 0.0f) || !std::isfinite(clip_high) ||
        !std::isfinite(kl_coef) || !std::isfinite(grad_scale))
        return set_error(TREE_ENS_E_ARG, "clip_low must be in [0, 1], clip_high >= 0, kl_coef and grad_scale finite");
    if (!ref_logp && kl_coef != 0.0f && n_tokens > 0)
        return set_error(TREE_ENS_E_ARG, "kl_coef needs ref_logp");
    if (flags & ~TREE_ENS_SEQ_MEAN)
        return set_error(TREE_ENS_E_ARG, "unknown flag bits");
    if (int rc = check_tokens(logp, n_tokens, seq_offsets, n_seqs))
        return rc;
    if (n_seqs > 0 && (!advantages || !loss))
        return set_error(TREE_ENS_E_ARG, "advantages or loss is NULL");
    if (misaligned(old_logp, 4) || misaligned(ref_logp, 4) || misaligned(advantages, 4) || misaligned(loss, 4) ||
        misaligned(kl, 4) || misaligned(grad_logp, 4))
        return set_error(TREE_ENS_E_ARG, "a pointer is misaligned for its type");
    (void)workspace;
    (void)workspace_bytes;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Tokens in{logp, ref_logp, mask, n_tokens, seq_offsets, n_seqs};
    const Policy p{old_logp, advantages, 1.0f - clip_low, 1.0f + clip_high, kl_coef, grad_scale,
                   (flags & TREE_ENS_SEQ_MEAN) != 0, loss, kl, grad_logp};
    (void)hipGetLastError();
    if (n_seqs > 0)
        hipLaunchKernelGGL(policy_kernel, dim3(blocks_for(n_seqs)), dim3(kThreads), 0, s, in, p);
    else if (grad_logp && n_tokens > 0)
        hipLaunchKernelGGL(zero_kernel, dim3(blocks_for((n_tokens + kThreads - 1) / kThreads)), dim3(kThreads), 0, s,
                           grad_logp, n_tokens);
    return launched("policy loss");
}

} // extern "C"
