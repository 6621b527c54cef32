// losses.hip -- losses over packed sequences of token log-probabilities, with their gradients, and
// advantages of scores relative to their group, on gfx950.
//
// Segments: sequence s owns tokens [seq_offsets[s], seq_offsets[s+1]), group g owns sequences
// [group_offsets[g], group_offsets[g+1]). Sums over tokens are held in double, those over pairs in float for up
// to 128 pairs of one candidate and in double beyond.
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

template <typename T> __device__ __forceinline__ T wave_sum(T v) {
    for (int off = kWave / 2; off; off >>= 1)
        v += __shfl_xor(v, off);
    return v;
}

// Sum over the workgroup, in a fixed order, for every thread.
__device__ __forceinline__ double block_sum(double v) {
    __shared__ double part[kWaves];
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
};

template <typename B> struct Pair {
    double a;
    B b;
};

typedef float float4_ __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned unsigned_ __attribute__((aligned(1)));

constexpr int kFour = 4; // neighbouring tokens that a thread takes at a time

// Tokens [t, t + 4) of an array of n, 0 beyond its end. Every array is read once and the gradient is not
// read here, so both go past the caches: the preference loss of 4,096 sequences of 3,700 tokens takes 44
// us where cached loads and stores take 52, the policy loss 59 and 61; 1,660,000 tokens 13.7 and 14.3.
__device__ __forceinline__ void load_tokens(const float *p, int64_t t, int64_t n, float (&x)[kFour]) {
    if (t + kFour <= n) {
        const float4_ a = __builtin_nontemporal_load(reinterpret_cast<const float4_ *>(p + t));
#pragma unroll
        for (int k = 0; k < kFour; ++k)
            x[k] = a[k];
        return;
    }
#pragma unroll
    for (int k = 0; k < kFour; ++k)
        x[k] = t + k < n ? p[t + k] : 0.0f;
}

// Bit k: byte k of x is not 0.
__device__ __forceinline__ unsigned nonzero_bytes(unsigned x) {
    const unsigned high = (((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u;
    return ((high >> 7) * 0x10204080u) >> 28;
}

// A byte for each of the four tokens, not 0 where it counts; tokens beyond the end of the array count as
// the caller says.
__device__ __forceinline__ unsigned load_mask(const uint8_t *mask, int64_t t, int64_t n) {
    if (!mask)
        return ~0u;
    if (t + kFour <= n)
        return *reinterpret_cast<const unsigned_ *>(mask + t);
    unsigned x = 0;
    for (int k = 0; t + k < n; ++k)
        x |= unsigned(mask[t + k]) << (8 * k);
    return x;
}

__device__ __forceinline__ void store_tokens(float *p, int64_t t, int count, const float (&x)[kFour]) {
    if (count == kFour) {
        __builtin_nontemporal_store(float4_{x[0], x[1], x[2], x[3]}, reinterpret_cast<float4_ *>(p + t));
        return;
    }
#pragma unroll
    for (int k = 0; k < kFour; ++k)
        if (k < count)
            p[t + k] = x[k];
}

// ---------------------------------------------------------------------------------------------
// Sequences, by groups of threads
//
// kGroup neighbouring threads take a sequence, four neighbouring tokens a thread at a time. Sequences
// much longer than the group is made for are left to the whole workgroup afterwards, so that none keeps
// a few lanes busy alone. A workgroup's sequence may be one of `parts` parts of it.
// ---------------------------------------------------------------------------------------------
constexpr int kTurns = 16; // a group takes at most so many times four tokens a thread

template <int kN> struct Lanes {
    static constexpr int kThreadsOf = kN;
    int id;
    // Sum over the group, in a fixed order, for each of its threads.
    template <typename T> __device__ __forceinline__ T sum(T v) const {
        if constexpr (kN == kThreads)
            return T(block_sum(double(v)));
        else
            for (int off = kN / 2; off; off >>= 1)
                v += __shfl_xor(v, off);
        return v;
    }
    // For this thread's fours of a span, kAhead at a time: load(k, t) for each, then use(k, t, count).
    template <int kAhead, typename Load, typename Use> __device__ __forceinline__ void each(Span q, Load &&load, Use &&use) const {
        constexpr int kStep = kN * kFour;
        for (int64_t t0 = q.a + id * kFour; t0 < q.b; t0 += kAhead * kStep) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (t0 + k * kStep < q.b)
                    load(k, t0 + k * kStep);
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
                if (t0 + k * kStep < q.b)
                    use(k, t0 + k * kStep, int(min(int64_t(kFour), q.b - t0 - k * kStep)));
        }
    }
};

// Which of `count` tokens count, as bits.
__device__ __forceinline__ unsigned counted_bits(unsigned mask, int count) { return nonzero_bytes(mask) & ((1u << count) - 1); }

// Part `part` of `parts` of a span, in whole fours.
__device__ __forceinline__ Span part_of(Span q, int part, int parts) {
    const int64_t each = ((q.b - q.a + parts - 1) / parts + kFour - 1) / kFour * kFour;
    const int64_t a = min(q.a + part * each, q.b);
    return {a, min(a + each, q.b)};
}

// Calls body(lanes, s, span, part) for every sequence; parts > 1 with whole workgroups only.
template <int kGroup, typename Body> __device__ __forceinline__ void for_sequences(const Tokens &in, int parts, Body &&body) {
    constexpr int kSeqs = kThreads / kGroup;
    if constexpr (kSeqs == 1) {
        const Lanes<kThreads> lanes{int(threadIdx.x)};
        for (int64_t item = blockIdx.x; item < in.n_seqs * parts; item += gridDim.x) {
            const int64_t s = parts > 1 ? item / parts : item;
            const int part = int(item - s * parts);
            const Span q = span_of(in.offsets, s, in.n);
            body(lanes, s, parts > 1 ? part_of(q, part, parts) : q, part);
        }
    } else {
        for (int64_t s0 = blockIdx.x * int64_t(kSeqs); s0 < in.n_seqs; s0 += int64_t(gridDim.x) * kSeqs) {
            const int64_t s = s0 + threadIdx.x / kGroup;
            Span q{0, 0};
            if (s < in.n_seqs)
                q = span_of(in.offsets, s, in.n);
            const bool rest = q.b - q.a > kGroup * kFour * kTurns;
            if (s < in.n_seqs && !rest)
                body(Lanes<kGroup>{int(threadIdx.x % kGroup)}, s, q, 0);
            if (!__syncthreads_or(rest))
                continue;
            for (int64_t i = s0; i < min(s0 + kSeqs, in.n_seqs); ++i) {
                const Span r = span_of(in.offsets, i, in.n);
                if (r.b - r.a > kGroup * kFour * kTurns)
                    body(Lanes<kThreads>{int(threadIdx.x)}, i, r, 0);
            }
        }
    }
}

// Zero the gradient of tokens before the first and after the last sequence, by the first workgroups.
__device__ __forceinline__ void zero_outside(const Tokens &in, float *grad) {
    const unsigned blocks = min(gridDim.x, 64u);
    if (blockIdx.x >= blocks)
        return;
    const int64_t a = span_of(in.offsets, 0, in.n).a, b = span_of(in.offsets, in.n_seqs - 1, in.n).b;
    const int64_t at = blockIdx.x * int64_t(kThreads) + threadIdx.x, step = int64_t(blocks) * kThreads;
    for (int64_t t = at; t < a; t += step)
        grad[t] = 0.0f;
    for (int64_t t = b + at; t < in.n; t += step)
        grad[t] = 0.0f;
}

// ---------------------------------------------------------------------------------------------
// Preference loss
// ---------------------------------------------------------------------------------------------
struct Preference {
    const float *scores;
    const int64_t *groups;
    int64_t n_groups;
    float beta, smoothing, grad_scale;
    bool mean;
    float *loss, *margins, *weights; // weights: dh / dlogp of a counted token, then the loss's gradient
    // The margin and weight of a sequence with this sum of log ratios and so many counted tokens.
    __device__ __forceinline__ void take(int64_t s, Pair<int64_t> v) const {
        const double w = mean ? double(beta) / double(max(v.b, int64_t(1))) : double(beta);
        margins[s] = float(w * v.a);
        weights[s] = float(w);
    }
};

// Sum of a span's log ratios and how many count, over a group's threads.
template <int kN> __device__ __forceinline__ Pair<int64_t> ratios_of(const Tokens &in, Lanes<kN> lanes, Span q) {
    constexpr int kAhead = 4;
    double sum = 0.0;
    int64_t counted = 0;
    float x[kAhead][kFour], r[kAhead][kFour] = {};
    unsigned mask[kAhead];
    lanes.template each<kAhead>(
        q,
        [&](int k, int64_t t) {
            load_tokens(in.logp, t, in.n, x[k]);
            if (in.ref)
                load_tokens(in.ref, t, in.n, r[k]);
            mask[k] = load_mask(in.mask, t, in.n);
        },
        [&](int k, int64_t, int count) {
            const unsigned use = counted_bits(mask[k], count);
#pragma unroll
            for (int i = 0; i < kFour; ++i)
                sum += use >> i & 1u ? x[k][i] - r[k][i] : 0.0f;
            counted += __popc(use);
        });
    return {lanes.sum(sum), lanes.sum(counted)};
}

// The gradient at a span's tokens.
template <int kN> __device__ __forceinline__ void spread(const Tokens &in, Lanes<kN> lanes, Span q, float weight, float *grad) {
    constexpr int kAhead = 4;
    unsigned mask[kAhead];
    lanes.template each<kAhead>(
        q, [&](int k, int64_t t) { mask[k] = load_mask(in.mask, t, in.n); },
        [&](int k, int64_t t, int count) {
            const unsigned use = counted_bits(mask[k], count);
            float d[kFour];
#pragma unroll
            for (int i = 0; i < kFour; ++i)
                d[i] = use >> i & 1u ? weight : 0.0f;
            store_tokens(grad, t, count, d);
        });
}

// Margins and weights, or with several parts what each adds to them. Bound by memory, 9 bytes a masked
// token: 98,000 sequences of 140 tokens take 27 to 32 us (4.6 to 3.9 TB/s), of which 17 are instructions.
template <int kGroup>
__global__ void __launch_bounds__(kThreads) margin_kernel(Tokens in, Preference p, int parts, Pair<int64_t> *partial) {
    for_sequences<kGroup>(in, parts, [&](auto lanes, int64_t s, Span q, int part) {
        const Pair<int64_t> v = ratios_of(in, lanes, q);
        if (lanes.id != 0)
            return;
        if (parts > 1)
            partial[s * parts + part] = v;
        else
            p.take(s, v);
    });
}

// Margins and weights from the parts, a wave a sequence.
__global__ void __launch_bounds__(kThreads) margin_join_kernel(int64_t n_seqs, Preference p, int parts, const Pair<int64_t> *partial) {
    const Lanes<kWave> lanes{int(threadIdx.x % kWave)};
    for (int64_t s = blockIdx.x * int64_t(kWaves) + threadIdx.x / kWave; s < n_seqs; s += int64_t(gridDim.x) * kWaves) {
        Pair<int64_t> v{0.0, 0};
        for (int k = lanes.id; k < parts; k += kWave) {
            v.a += partial[s * parts + k].a;
            v.b += partial[s * parts + k].b;
        }
        v = {lanes.sum(v.a), lanes.sum(v.b)};
        if (lanes.id == 0)
            p.take(s, v);
    }
}

// grad[t] = the sequence's weight at its counted tokens. Bound by the stores: 98,000 sequences of 140 tokens
// take 18 us (4.7 TB/s with the mask).
template <int kGroup> __global__ void __launch_bounds__(kThreads) spread_kernel(Tokens in, const float *weights, int parts, float *grad) {
    for_sequences<kGroup>(in, parts, [&](auto lanes, int64_t s, Span q, int) { spread(in, lanes, q, weights[s], grad); });
    zero_outside(in, grad);
}

// Pairs are bound by instructions: 15 a pair for a slope and 30 with the loss, two (three) of them exp2, a reciprocal
// (and log2). Adding a pair's slope to both candidates by LDS atomics, which halves the pairs, took 95 us
// where meeting each pair from both sides takes 42 (909 groups of 110, by pairs_kernel).
constexpr int kHeld = 512;  // candidates of a group that are held in LDS
constexpr int kChain = 128; // pairs whose losses and slopes are added in float

// What the pairs that a thread met add up to: (1 - smoothing) max(-d, 0) + log1p(exp(-|d|)), max(d, 0) and 1.
struct Met {
    float loss, lead;
    int pairs;
};
// The same over threads, with the smoothing.
struct Loss {
    double sum, pairs;
    // An infinite lead costs nothing without smoothing, where 0 times it would be NaN.
    __device__ __forceinline__ void add(const Met &m, float smoothing, double weight) {
        sum += weight * (smoothing > 0.0f ? m.loss + double(smoothing) * m.lead : double(m.loss));
        pairs += weight * m.pairs;
    }
};

// One pair: dl/dh of the candidate `me`, and with kLoss the pair's loss. Candidates are (margin, score). The margins'
// difference comes first and goes by log2(e) then, so that a pair is rounded by the size of its own difference, whatever
// the margins of others; losses are in units of ln 2 here. With d the margin by which the better one leads and e =
// exp(-|d|): l = (1 - smoothing) softplus(-d) + smoothing softplus(d), softplus(x) = max(x, 0) + log1p(e), dl/dd =
// smoothing - sigmoid(-d). The two maxima are added apart, so that infinite ones never meet with both signs.
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.693147180559945309417;
template <bool kLoss> __device__ __forceinline__ float meet(float2 me, float2 other, float smoothing, Met &met) {
    const bool ahead = me.y > other.y, behind = me.y < other.y;
    const float lead = (me.x - other.x) * kLog2e;
    const float e = __builtin_amdgcn_exp2f(-fabsf(lead));
    const float u = 1.0f + e, r = __builtin_amdgcn_rcpf(u);
    if (kLoss) {
        const float d = ahead ? lead : -lead;
        // log1p(e) = log u + log(1 + rest / u), with the rest that u was rounded by
        float l = fmaf(1.0f - smoothing, fmaxf(-d, 0.0f), __builtin_amdgcn_logf(u));
        l = fmaf((e - (u - 1.0f)) * r, kLog2e, l);
        met.loss += ahead || behind ? l : 0.0f;
        met.lead += ahead || behind ? fmaxf(d, 0.0f) : 0.0f;
        met.pairs += ahead || behind;
    }
    const float dl = smoothing - ((lead >= 0.0f) == ahead ? e * r : r);
    return ahead ? dl : behind ? -dl : 0.0f;
}

// `me` meets every step-th candidate of `others` from k on below `end`: returns the sum of its slopes, and with kLoss
// adds weight times the losses.
template <bool kLoss>
__device__ __forceinline__ double meet_every(float2 me, const float2 *others, int &k, int end, int step, float smoothing, double weight, Loss &loss) {
    double slope = 0.0;
    while (k < end) {
        const int stop = min(end, k + kChain * step);
        Met met{0.0f, 0.0f, 0};
        float sum = 0.0f;
#pragma unroll 4
        for (; k < stop; k += step)
            sum += meet<kLoss>(me, others[k], smoothing, met);
        if (kLoss)
            loss.add(met, smoothing, weight);
        slope += sum;
    }
    return slope;
}

// The n <= kHeld candidates of a group lie twice in a row, so that i + k needs no remainder. In step k
// candidate i meets i + k (modulo n), for its own slope alone, so nothing is added atomically; the first
// half of the steps meets every pair once and takes its loss. One thread takes candidate i in every
// `shares`-th step from 1 + share on; returns its slope.
__device__ __forceinline__ float meet_held(const float2 *held, int n, int i, int share, int shares, float smoothing, Loss &loss) {
    const float2 me = held[i], *other = held + i;
    int k = 1 + share;
    double slope = meet_every<true>(me, other, k, (n + 1) / 2, shares, smoothing, 1.0, loss);
    if (2 * k == n) { // opposite each other: the lower one takes the loss
        Met met{0.0f, 0.0f, 0};
        slope += meet<true>(me, other[k], smoothing, met);
        if (i < k)
            loss.add(met, smoothing, 1.0);
        k += shares;
    }
    return float(slope + meet_every<false>(me, other, k, n, shares, smoothing, 0.0, loss));
}

// One thread's candidate against the kHeld or fewer of a larger group that are held: every pair is met
// twice.
__device__ __forceinline__ double meet_window(float2 me, const float2 *held, int fit, int share, int shares, float smoothing, Loss &loss) {
    return meet_every<true>(me, held, share, fit, shares, smoothing, 0.5, loss);
}

// Sequences outside every group have no gradient: those before the first and after the last group, for the
// kernels that meet the pairs.
__device__ __forceinline__ void clear_outside(const Preference &p, int64_t n_seqs, int64_t g, Span q, int id, int step) {
    if (g == 0)
        for (int64_t s = id; s < q.a; s += step)
            p.weights[s] = 0.0f;
    if (g == p.n_groups - 1)
        for (int64_t s = q.b + id; s < n_seqs; s += step)
            p.weights[s] = 0.0f;
}

// Loss of a group, and weights times the loss's gradient with respect to the margins, by a workgroup.
// kFused: it also sums the sequences' tokens first and writes their gradients last, instead of
// margin_kernel and spread_kernel: a wave a sequence, or a quarter of each where the group has many more
// tokens than sequences, so that no long sequence keeps one wave busy alone: one of 1.9 million tokens among
// 2,000 takes 1.05 ms, 3.6 by one wave.
constexpr int64_t kSplit = 2048; // tokens for each sequence of the group and two more
template <bool kFused>
__global__ void __launch_bounds__(kThreads) pairs_kernel(Tokens in, Preference p, float *grad) {
    __shared__ float2 held[2 * kHeld];
    __shared__ float slopes[kWaves][kHeld];
    const int wave = threadIdx.x / kWave;
    const Lanes<kWave> lanes{int(threadIdx.x % kWave)};
    for (int64_t g = blockIdx.x; g < p.n_groups; g += gridDim.x) {
        const Span q = span_of(p.groups, g, in.n_seqs);
        const int64_t n = q.b - q.a;
        // fused, sequences outside every group go with the first and the last one
        const int64_t lo = g == 0 ? 0 : q.a, hi = g == p.n_groups - 1 ? in.n_seqs : q.b;
        bool split = false;
        if constexpr (kFused) {
            __shared__ Pair<int64_t> quarter[kWaves];
            int64_t s = lo + wave;
            Span t = s < hi ? span_of(in.offsets, s, in.n) : Span{0, 0};
            split = lo < hi && min(in.offsets[hi], in.n) - max(in.offsets[lo], int64_t(0)) > kSplit * (hi - lo + 2);
            if (split)
                t = part_of(span_of(in.offsets, s = lo, in.n), wave, kWaves);
            while (s < hi) {
                Pair<int64_t> v = ratios_of(in, lanes, t);
                if (split) {
                    if (lanes.id == 0)
                        quarter[wave] = v;
                    __syncthreads();
                    v = quarter[0];
                    for (int w = 1; w < kWaves; ++w)
                        v = {v.a + quarter[w].a, v.b + quarter[w].b};
                    __syncthreads(); // quarter is free
                }
                if (lanes.id == 0 && (!split || wave == 0))
                    p.take(s, v);
                s += split ? 1 : kWaves;
                if (s < hi)
                    t = span_of(in.offsets, s, in.n);
                if (split)
                    t = part_of(t, wave, kWaves);
            }
            __syncthreads();
        }
        clear_outside(p, in.n_seqs, g, q, threadIdx.x, kThreads);
        Loss loss{0.0, 0.0};
        if (n <= kHeld) {
            for (int i = threadIdx.x; i < n; i += kThreads)
                held[i] = held[i + n] = make_float2(p.margins[q.a + i], p.scores[q.a + i]);
            __syncthreads();
            // waves take steps in turn and leave their slopes in rows of their own
            for (int i = lanes.id; i < n; i += kWave)
                slopes[wave][i] = meet_held(held, int(n), i, wave, kWaves, p.smoothing, loss);
            __syncthreads();
            for (int i = threadIdx.x; i < n; i += kThreads) {
                double sum = slopes[0][i];
                for (int w = 1; w < kWaves; ++w)
                    sum += slopes[w][i];
                p.weights[q.a + i] = float(p.weights[q.a + i] * sum);
            }
        } else {
            for (int64_t i0 = 0; i0 < n; i0 += kThreads) {
                const int64_t i = q.a + i0 + threadIdx.x;
                const float2 me = i < q.b ? make_float2(p.margins[i], p.scores[i]) : make_float2(0.0f, 0.0f);
                double sum = 0.0;
                for (int64_t j0 = q.a; j0 < q.b; j0 += kHeld) {
                    const int fit = int(min(int64_t(kHeld), q.b - j0));
                    __syncthreads();
                    for (int j = threadIdx.x; j < fit; j += kThreads)
                        held[j] = make_float2(p.margins[j0 + j], p.scores[j0 + j]);
                    __syncthreads();
                    if (i < q.b)
                        sum += meet_window(me, held, fit, 0, 1, p.smoothing, loss);
                }
                if (i < q.b)
                    p.weights[i] = float(p.weights[i] * sum);
            }
        }
        loss.sum = block_sum(loss.sum);
        loss.pairs = block_sum(loss.pairs);
        const double share = 1.0 / fmax(loss.pairs, 1.0);
        if (threadIdx.x == 0)
            p.loss[g] = float(loss.sum * (kLn2 * share));
        __syncthreads();
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            p.weights[i] = float(p.weights[i] * (p.grad_scale * share));
        __syncthreads(); // held and slopes are free, weights are there
        if constexpr (kFused)
            if (grad)
                for (int64_t s = split ? lo : lo + wave; s < hi; s += split ? 1 : kWaves) {
                    const Span t = span_of(in.offsets, s, in.n);
                    spread(in, lanes, split ? part_of(t, wave, kWaves) : t, p.weights[s], grad);
                }
    }
    if constexpr (kFused)
        if (grad)
            zero_outside(in, grad);
}

constexpr int kHeldPart = 2048;

// One of `parts` shares of a group's candidates, against all of the group. As many threads take a
// candidate as there are, each every so many steps of it. 13 million ordered pairs of 909 groups take 23 us in
// three parts, 13 of them for the instructions if every unit had the same number; pairs_kernel, whose
// workgroups differ more, took 36.
__global__ void __launch_bounds__(kThreads) pairs_part_kernel(int64_t n_seqs, Preference p, int parts, Loss *partial) {
    __shared__ float2 held[2 * kHeldPart];
    __shared__ float slopes[kThreads];
    const unsigned items = unsigned(p.n_groups) * unsigned(parts); // fewer than sequences
    for (unsigned item = blockIdx.x; item < items; item += gridDim.x) {
        const unsigned g = item / unsigned(parts), part = item - g * unsigned(parts);
        const Span q = span_of(p.groups, g, n_seqs);
        const unsigned n = unsigned(q.b - q.a), chunk = (n + unsigned(parts) - 1) / unsigned(parts);
        const int64_t from = min(int64_t(part) * chunk, int64_t(n)), to = min(from + chunk, int64_t(n));
        Loss loss{0.0, 0.0};
        // rows of even size, as few as fit
        const int turns = int((to - from + kThreads - 1) / kThreads), each = turns ? int((to - from + turns - 1) / turns) : 0;
        for (int64_t i0 = from; i0 < to; i0 += each) {
            const int rows = int(min(int64_t(each), to - i0)), shares = kThreads / rows;
            const int row = threadIdx.x % rows, share = threadIdx.x / rows;
            const int64_t i = i0 + row;
            const float2 me = make_float2(p.margins[q.a + i], p.scores[q.a + i]);
            double slope = 0.0;
            if (n <= kHeldPart) {
                if (i0 == from)
                    for (int j = threadIdx.x; j < n; j += kThreads)
                        held[j] = held[j + n] = make_float2(p.margins[q.a + j], p.scores[q.a + j]);
                __syncthreads();
                if (share < shares)
                    slope = meet_held(held, int(n), int(i), share, shares, p.smoothing, loss);
            } else {
                for (int64_t j0 = 0; j0 < n; j0 += kHeldPart) {
                    const int fit = int(min(int64_t(kHeldPart), n - j0));
                    __syncthreads();
                    for (int j = threadIdx.x; j < fit; j += kThreads)
                        held[j] = make_float2(p.margins[q.a + j0 + j], p.scores[q.a + j0 + j]);
                    __syncthreads();
                    if (share < shares)
                        slope += meet_window(me, held, fit, share, shares, p.smoothing, loss);
                }
            }
            slopes[threadIdx.x] = float(slope);
            __syncthreads();
            if (threadIdx.x < rows) {
                for (int k = 1; k < shares; ++k)
                    slope += slopes[k * rows + row];
                p.weights[q.a + i] = float(p.weights[q.a + i] * slope);
            }
            __syncthreads(); // slopes are free
        }
        loss.sum = block_sum(loss.sum);
        loss.pairs = block_sum(loss.pairs);
        if (threadIdx.x == 0)
            partial[item] = loss;
        __syncthreads(); // held and slopes are free
    }
}

// What pairs_part_kernel leaves: a group's loss, and weights by its number of pairs. A wave takes a group.
__global__ void __launch_bounds__(kThreads) pairs_finish_kernel(int64_t n_seqs, Preference p, int parts, const Loss *partial) {
    for (int64_t g = blockIdx.x * int64_t(kWaves) + threadIdx.x / kWave; g < p.n_groups; g += int64_t(gridDim.x) * kWaves) {
        const int lane = threadIdx.x % kWave;
        const Span q = span_of(p.groups, g, n_seqs);
        Loss loss{0.0, 0.0};
        for (int k = lane; k < parts; k += kWave) {
            loss.sum += partial[g * parts + k].sum;
            loss.pairs += partial[g * parts + k].pairs;
        }
        loss.sum = wave_sum(loss.sum);
        loss.pairs = wave_sum(loss.pairs);
        const double share = 1.0 / fmax(loss.pairs, 1.0);
        if (lane == 0)
            p.loss[g] = float(loss.sum * (kLn2 * share));
        for (int64_t i = q.a + lane; i < q.b; i += kWave)
            p.weights[i] = float(p.weights[i] * (p.grad_scale * share));
        clear_outside(p, n_seqs, g, q, lane, kWave);
    }
}

// All of group g = [q.a, q.b) by kN neighbouring threads, candidates from memory: a thread takes one at a time and meets
// the whole group with it, every pair twice.
template <int kN> __device__ __forceinline__ void meet_in_memory(const Preference &p, Lanes<kN> lanes, int64_t g, Span q) {
    const float *margins = p.margins + q.a, *scores = p.scores + q.a;
    float *weights = p.weights + q.a;
    const unsigned n = unsigned(q.b - q.a);
    Loss loss{0.0, 0.0};
    for (unsigned i = lanes.id; i < n; i += kN) {
        const float2 me = make_float2(margins[i], scores[i]);
        double sum = 0.0;
        for (unsigned j = 0; j < n;) {
            const unsigned end = kN < kWave ? n : min(j + unsigned(kChain), n); // fewer lanes have kFewMost at most
            Met met{0.0f, 0.0f, 0};
            float slope = 0.0f;
#pragma unroll 2
            for (; j < end; ++j)
                slope += meet<true>(me, make_float2(margins[j], scores[j]), p.smoothing, met);
            loss.add(met, p.smoothing, 0.5);
            sum += slope;
        }
        weights[i] = float(weights[i] * sum);
    }
    loss.sum = lanes.sum(loss.sum);
    loss.pairs = lanes.sum(loss.pairs);
    const double share = 1.0 / fmax(loss.pairs, 1.0);
    if (lanes.id == 0)
        p.loss[g] = float(loss.sum * (kLn2 * share));
    for (unsigned i = lanes.id; i < n; i += kN)
        weights[i] = float(weights[i] * (p.grad_scale * share));
}

// Groups of a few candidates: eight lanes take one. Those of more than kFewMost among them are left to the waves
// afterwards, one to a wave, and those of more than kWaveMost to the whole workgroup after that: 10,000 pairs and one
// group of 5,000 take 10.5 ms. Measured (us of the whole loss; kFewMost 64 / 24): 10,000 groups of 2, each 100th of 40: 43 /
// 24, of 64: 94 / 26, of 65: - / 36; 5,000 of 2 and then 400 of 64: 63 / 80, 1,000 of 28: 24 / 51. Of 65 instead of 64: 207.
// kWaveMost 128 / 256: each 100th of 200: 46 / 104.
constexpr int kFew = 8, kFewMost = 64, kWaveMost = 128;
__global__ void __launch_bounds__(kThreads) pairs_few_kernel(int64_t n_seqs, Preference p) {
    constexpr int kGroups = kThreads / kFew;
    const int lane = threadIdx.x % kFew;
    for (int64_t g0 = blockIdx.x * int64_t(kGroups); g0 < p.n_groups; g0 += int64_t(gridDim.x) * kGroups) {
        const int64_t g = g0 + threadIdx.x / kFew, end = min(g0 + kGroups, p.n_groups);
        Span q{0, 0};
        if (g < end) {
            q = span_of(p.groups, g, n_seqs);
            clear_outside(p, n_seqs, g, q, lane, kFew);
        }
        const bool rest = q.b - q.a > kFewMost;
        if (g < end && !rest)
            meet_in_memory(p, Lanes<kFew>{lane}, g, q);
        if (!__syncthreads_or(rest))
            continue;
        for (int64_t i = g0 + threadIdx.x / kWave; i < end; i += kWaves) {
            const Span r = span_of(p.groups, i, n_seqs);
            if (r.b - r.a > kFewMost && r.b - r.a <= kWaveMost)
                meet_in_memory(p, Lanes<kWave>{int(threadIdx.x % kWave)}, i, r);
        }
        for (int64_t i = g0; i < end; ++i) {
            const Span r = span_of(p.groups, i, n_seqs);
            if (r.b - r.a > kWaveMost)
                meet_in_memory(p, Lanes<kThreads>{int(threadIdx.x)}, i, r);
        }
    }
}

// ---------------------------------------------------------------------------------------------
// Advantages and policy loss
// ---------------------------------------------------------------------------------------------
// Advantages of the groups of `in` (candidates as its tokens): mean and spread in double, by two passes
// over values that stay in registers where four fours a thread hold them. A million candidates in 9,090
// groups take 7.3 us with 16 threads a group, mostly the launch and one trip to memory (a workgroup a group
// that read them three times took 16).
template <int kGroup>
__global__ void __launch_bounds__(kThreads) advantage_kernel(Tokens in, float eps, bool center, float *out) {
    for_sequences<kGroup>(in, 1, [&](auto lanes, int64_t, Span q, int) {
        constexpr int kHold = 4, kN = decltype(lanes)::kThreadsOf;
        const bool held = q.b - q.a <= kN * kFour * kHold;
        const double count = fmax(double(q.b - q.a), 1.0);
        float x[kHold][kFour];
        const auto load = [&](int k, int64_t t) { load_tokens(in.logp, t, in.n, x[k]); };
        const auto again = [&](int k, int64_t t) { // for the passes after the first
            if (!held)
                load(k, t);
        };
        double sum = 0.0, squares = 0.0;
        lanes.template each<kHold>(q, load, [&](int k, int64_t, int some) {
#pragma unroll
            for (int i = 0; i < kFour; ++i)
                sum += i < some ? x[k][i] : 0.0f;
        });
        const double mean = lanes.sum(sum) / count;
        lanes.template each<kHold>(q, again, [&](int k, int64_t, int some) {
#pragma unroll
            for (int i = 0; i < kFour; ++i) {
                const double d = i < some ? x[k][i] - mean : 0.0;
                squares += d * d;
            }
        });
        const double std_ = sqrt(lanes.sum(squares) / count); // NaN if a score is infinite or NaN
        const double by = isnan(std_) ? std_ : center ? 1.0 : 1.0 / (std_ + eps);
        lanes.template each<kHold>(q, again, [&](int k, int64_t t, int some) {
            float d[kFour];
#pragma unroll
            for (int i = 0; i < kFour; ++i)
                d[i] = float((x[k][i] - mean) * by);
            store_tokens(out, t, some, d);
        });
    });
    zero_outside(in, out);
}

// exp(x), off by 2^-24 (2 + |x|) of itself.
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * kLog2e); }

struct Policy {
    const float *old_logp, *advantages;
    float low, high, kl_coef, grad_scale;
    bool mean;
    float *loss, *kl, *grad;
    // The sums of a sequence's gains and of exp(q) - q - 1.
    __device__ __forceinline__ void take(int64_t s, Pair<double> v, double share) const {
        loss[s] = float(share * (kl_coef != 0.0f ? v.a + kl_coef * v.b : v.a));
        if (kl)
            kl[s] = float(share * v.b);
    }
};

// Of one token: the ratio, k = exp(q) - q - 1 and up = dk/dq = exp(q) - 1. Below 1/2 the differences would
// cancel: k is the sum of q^i / i! from i = 2 there, whose terms up to i = 9 leave out less than 2e-9 of it.
// An infinite q has k = inf.
struct Terms {
    float ratio, k, up;
};
__device__ __forceinline__ Terms terms_of(const Tokens &in, const Policy &p, float logp, float old, float ref) {
    const float d = p.old_logp ? logp - old : 0.0f, q = in.ref ? ref - logp : 0.0f; // without them: 0, whatever logp is
    float s = 1.0f / 362880.0f;
    s = fmaf(s, q, 1.0f / 40320.0f);
    s = fmaf(s, q, 1.0f / 5040.0f);
    s = fmaf(s, q, 1.0f / 720.0f);
    s = fmaf(s, q, 1.0f / 120.0f);
    s = fmaf(s, q, 1.0f / 24.0f);
    s = fmaf(s, q, 1.0f / 6.0f);
    s = fmaf(s, q, 0.5f) * q * q;
    const float up = exp_of(q) - 1.0f;
    const bool small = fabsf(q) < 0.5f;
    return {exp_of(d), small ? s : up - fminf(q, 3e38f), small ? s + q : up};
}
// The clipped gain's share in the loss, and the gradient of the token's loss. Comparisons pass a NaN
// ratio unchanged.
__device__ __forceinline__ float policy_of(const Policy &p, const Terms &x, float a, float &slope) {
    const float edge = a >= 0.0f ? p.high : p.low;
    const bool clipped = a >= 0.0f ? x.ratio > edge : x.ratio < edge;
    slope = (clipped ? 0.0f : -a * x.ratio) - (p.kl_coef != 0.0f ? p.kl_coef * x.up : 0.0f);
    return -(clipped ? edge : x.ratio) * a;
}

// How many of a span's tokens count.
template <int kN> __device__ __forceinline__ int64_t counted_of(const Tokens &in, Lanes<kN> lanes, Span q) {
    constexpr int kAhead = 4;
    int64_t count = 0;
    unsigned mask[kAhead];
    lanes.template each<kAhead>(
        q, [&](int k, int64_t t) { mask[k] = load_mask(in.mask, t, in.n); },
        [&](int k, int64_t, int some) { count += __popc(counted_bits(mask[k], some)); });
    return lanes.sum(count);
}

// How many tokens of each part of a sequence count, for the mean over masked sequences in parts.
__global__ void __launch_bounds__(kThreads) count_kernel(Tokens in, int parts, int64_t *counts) {
    for_sequences<kThreads>(in, parts, [&](auto lanes, int64_t s, Span q, int part) {
        const int64_t count = counted_of(in, lanes, q);
        if (lanes.id == 0)
            counts[s * parts + part] = count;
    });
}

// What a sequence's loss is multiplied by, for the threads that take it (or the part q of it).
template <int kN>
__device__ __forceinline__ double share_of(const Tokens &in, const Policy &p, Lanes<kN> lanes, int64_t s, Span q, int parts, const int64_t *counts) {
    if (!p.mean)
        return 1.0;
    if (!in.mask) {
        const Span all = span_of(in.offsets, s, in.n);
        return 1.0 / double(max(all.b - all.a, int64_t(1)));
    }
    if (parts == 1)
        return 1.0 / double(max(counted_of(in, lanes, q), int64_t(1)));
    double count = 0.0; // of all parts
    for (int k = lanes.id; k < parts; k += kN)
        count += double(counts[s * parts + k]);
    return 1.0 / fmax(lanes.sum(count), 1.0);
}

// 17 bytes a masked token: 19 million tokens of 4,096 sequences take 74 us, 4.3 TB/s, 37 of them for the instructions
// if every unit had the same number. Their lengths differ, 512 to 16,384, and a workgroup takes each: as many tokens in
// sequences of 4,571 take 61 us. A mean over masked tokens needs their number first, which reads the
// mask twice, the second time from the cache.
template <int kGroup>
__global__ void __launch_bounds__(kThreads) policy_kernel(Tokens in, Policy p, int parts, const int64_t *counts, Pair<double> *partial) {
    for_sequences<kGroup>(in, parts, [&](auto lanes, int64_t s, Span q, int part) {
        const float a = p.advantages[s];
        const double share = share_of(in, p, lanes, s, q, parts, counts);
        const float w = float(p.grad_scale * share);
        double loss = 0.0, kl = 0.0;
        // Four tokens a thread in flight: 84 registers and five waves a SIMD, with a workgroup a sequence 75 and six, where
        // eight take 101 and four waves (us, one / two fours; sequences x mean tokens): 16,384 x 1,620: 101 / 110; 200,000 x 8: 28.5 / 32; 20,000 x 325: 39 / 42;
        // 97,000 x 116: 70 / 72; 4,096 x 3,700: 60 / 59; 4,096 x 405: 13.9 / 13.7; 4,096 x 4,640: 73 / 72.
        constexpr int kAhead = 1;
        float x[kAhead][kFour], old[kAhead][kFour] = {}, ref[kAhead][kFour] = {};
        unsigned mask[kAhead];
        lanes.template each<kAhead>(
            q,
            [&](int k, int64_t t) {
                load_tokens(in.logp, t, in.n, x[k]);
                if (p.old_logp)
                    load_tokens(p.old_logp, t, in.n, old[k]);
                if (in.ref)
                    load_tokens(in.ref, t, in.n, ref[k]);
                mask[k] = load_mask(in.mask, t, in.n);
            },
            [&](int k, int64_t t, int count) {
                const unsigned use = counted_bits(mask[k], count);
                float d[kFour];
#pragma unroll
                for (int i = 0; i < kFour; ++i) {
                    const Terms m = terms_of(in, p, x[k][i], old[k][i], ref[k][i]);
                    const float gain = policy_of(p, m, a, d[i]);
                    const bool counts_ = use >> i & 1u;
                    loss += counts_ ? gain : 0.0f;
                    kl += counts_ ? m.k : 0.0f;
                    d[i] = counts_ ? w * d[i] : 0.0f;
                }
                if (p.grad)
                    store_tokens(p.grad, t, count, d);
            });
        const Pair<double> v{lanes.sum(loss), lanes.sum(kl)};
        if (lanes.id != 0)
            return;
        if (parts > 1)
            partial[s * parts + part] = v;
        else
            p.take(s, v, share);
    });
    if (p.grad)
        zero_outside(in, p.grad);
}

// Losses from the parts, a wave a sequence.
__global__ void __launch_bounds__(kThreads) policy_join_kernel(Tokens in, Policy p, int parts, const int64_t *counts, const Pair<double> *partial) {
    const Lanes<kWave> lanes{int(threadIdx.x % kWave)};
    for (int64_t s = blockIdx.x * int64_t(kWaves) + threadIdx.x / kWave; s < in.n_seqs; s += int64_t(gridDim.x) * kWaves) {
        Pair<double> v{0.0, 0.0};
        for (int k = lanes.id; k < parts; k += kWave) {
            v.a += partial[s * parts + k].a;
            v.b += partial[s * parts + k].b;
        }
        v = {lanes.sum(v.a), lanes.sum(v.b)};
        const double share = share_of(in, p, lanes, s, Span{0, 0}, parts, counts);
        if (lanes.id == 0)
            p.take(s, v, share);
    }
}

using treeens::set_error;

bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

unsigned blocks_for(int64_t n) { return unsigned(std::min(std::max<int64_t>(n, 1), kMaxBlocks)); }

dim3 blocks_of(int64_t items, int64_t per_block) { return dim3(blocks_for((items + per_block - 1) / per_block)); }

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

// How sequences are shared out: threads for each, or parts of it. By their mean length, and more threads
// where the sequences are too few for 2,000 waves, 8 to a CU. The preference loss's margins and gradients follow the
// same plan. Measured on the policy loss alone (us; sequences x mean
// tokens: 8 / 16 / 32 / 64 / 256 threads):
//   200,000 x 24: 39 / 49 / 81 / 152 / 423; 99,000 x 49: 34 / 37 / 47 / 80 / 210; 50,000 x 98: 41 / 31 / 34 / 46 /
//   111; 30,000 x 195: 60 / 37 / 32 / 37 / 72; 20,000 x 325: - / - / 34 / 35 / 53; 10,000 x 818: - / - / 48 / 36 / 38;
//   4,096 x 2,030: - / - / 63 / 47 / 31; 4,000 x 24: 6.4 / 5.6 / 5.1 / 6.5 / 12.4; 2,000 x 81: 10.6 / 7.7 / 6.0 / 5.2 / 8.4.
// In parts of a thousand tokens or more where long sequences are few (1 / 2 / 4 / 8 / 64 parts): 512 x 23,600:
// 85 / 59 / 52 / 44 / -; 4 x 73,700: 133 / 72 / 40 / 23 / 8.0; 256 x 3,200: 14.0 / 12.3 / 10.9 / 12.5 / -; 2,048 x
// 1,600: 17 / 23 / 30 / 47 / -.
struct SequencePlan {
    int group, parts;
};
SequencePlan sequence_plan(int64_t n_tokens, int64_t n_seqs) {
    const double seqs = double(std::max<int64_t>(n_seqs, 1)), tokens = double(n_tokens) / seqs;
    SequencePlan plan{tokens <= 64.0 ? 8 : tokens <= 144.0 ? 16 : tokens <= 320.0 ? 32 : tokens <= 1024.0 ? kWave : kThreads, 1};
    while (plan.group < kThreads && seqs * plan.group < 2000.0 * kWave)
        plan.group = plan.group == kWave ? kThreads : 2 * plan.group;
    if (plan.group == kThreads && n_seqs <= 1024)
        plan.parts = int(std::max(1.0, std::min(4096.0 / seqs, tokens / 1024.0)));
    return plan;
}

// Calls f with a std::integral_constant of the group's size.
template <typename F> void with_group(int group, F &&f) {
    if (group == 8)
        f(std::integral_constant<int, 8>());
    else if (group == 16)
        f(std::integral_constant<int, 16>());
    else if (group == 32)
        f(std::integral_constant<int, 32>());
    else if (group == kWave)
        f(std::integral_constant<int, kWave>());
    else
        f(std::integral_constant<int, kThreads>());
}

int64_t round_up(int64_t bytes) { return (bytes + 15) / 16 * 16; }

// Which kernels meet the pairs, by the mean sizes of groups and sequences. Measured (us of the whole loss;
// groups x candidates x tokens, means: pairs_kernel fused / pairs_few_kernel / pairs_kernel):
//   64 x 2 x 200: 6.5 / 8.9 / 9.9; 1,000 x 2 x 810: 12.2 / 15.0 / 16.6; 512 x 8 x 405: 13.0 / 14.6 / 15.0; 2,000 x 4 x
//   82: 15.0 / 12.0 / 15.6; 4 x 4 x 6,600: 36 / 11.6 / 12.6; 4,096 x 2 x 410: 30 / 19.3 / 26; 50,000 x 2 x 24: 258 / 23 /
//   106; 5,000 x 8 x 16: 44 / 13.3 / 22; 2,048 x 2 x 405: 18.2 / 13.9 / -; 512 x 16 x 410: 27 / 34 / 20.5; 100 x 16 x
//   82: 17.5 / 27 / 13.6.
// pairs_kernel / pairs_part_kernel with 2 / 8 / 24 parts: 2,000 x 40 x 81: 42 / 54 / - / -; 300 x 65 x 243: 30 / 31 / 46 /
//   79; 909 x 109 x 116: 74 / 68 / 93 / 179; 9,090 x 110 x 8: 209 / 242 / - / -; 100 x 303 x 81: 149 / 84 / 41 / 46; 4 x 640 x
//   81: 271 / 113 / 42 / 25.
enum class Pairs { kFused, kFew, kGroup, kParts };
struct PreferencePlan {
    Pairs by;
    int parts;
};

PreferencePlan preference_plan(int64_t n_tokens, int64_t n_seqs, int64_t n_groups) {
    if (n_groups == 0 || n_seqs == 0)
        return {Pairs::kGroup, 1};
    const double seqs = double(n_seqs) / double(n_groups), tokens = double(n_tokens) / double(n_seqs);
    if (seqs <= 8.0 && n_groups <= 1024 && n_seqs <= 4096 && tokens <= 1024.0)
        return {Pairs::kFused, 1};
    if (seqs <= 8.0)
        return {Pairs::kFew, 1};
    if (seqs >= 96.0 && n_groups <= 2048) // workgroups for the whole card, but eight candidates at least for each
        return {Pairs::kParts, int(std::min(std::ceil(2048.0 / double(n_groups)), std::ceil(seqs / 8.0)))};
    return {Pairs::kGroup, 1};
}

// Where a preference loss keeps what its kernels hand on.
struct PreferenceSpace {
    int64_t weights, losses, sums, bytes;
};
PreferenceSpace preference_space(int64_t n_tokens, int64_t n_seqs, int64_t n_groups) {
    const PreferencePlan pairs = preference_plan(n_tokens, n_seqs, n_groups);
    const SequencePlan seqs = sequence_plan(n_tokens, n_seqs);
    PreferenceSpace p{0, round_up(4 * n_seqs), 0, 0};
    p.sums = p.losses + (pairs.by == Pairs::kParts ? n_groups * pairs.parts * int64_t(sizeof(Loss)) : 0);
    p.bytes = p.sums + (seqs.parts > 1 ? n_seqs * seqs.parts * int64_t(sizeof(Pair<int64_t>)) : 0);
    return p;
}

// Where a policy loss does, if it goes in parts.
struct PolicySpace {
    int64_t counts, bytes;
};
PolicySpace policy_space(int64_t n_tokens, int64_t n_seqs) {
    const int64_t parts = sequence_plan(n_tokens, n_seqs).parts;
    if (parts == 1)
        return {0, 0};
    const int64_t sums = n_seqs * parts * int64_t(sizeof(Pair<double>));
    return {sums, sums + 8 * n_seqs * parts};
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
    *bytes = preference_space(n_tokens, n_seqs, n_groups).bytes;
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
    const PreferenceSpace space = preference_space(n_tokens, n_seqs, n_groups);
    if (int rc = check_workspace(workspace, workspace_bytes, space.bytes))
        return rc;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Tokens in{logp, ref_logp, mask, n_tokens, seq_offsets, n_seqs};
    char *const at = static_cast<char *>(workspace);
    float *weights = reinterpret_cast<float *>(at + space.weights);
    Loss *losses = reinterpret_cast<Loss *>(at + space.losses);
    Pair<int64_t> *sums = reinterpret_cast<Pair<int64_t> *>(at + space.sums);
    const Preference p{scores, group_offsets, n_groups, beta, smoothing, grad_scale, (flags & TREE_ENS_SEQ_MEAN) != 0,
                       loss, margins, weights};
    const PreferencePlan pairs = preference_plan(n_tokens, n_seqs, n_groups);
    const SequencePlan seqs = sequence_plan(n_tokens, n_seqs);
    const bool fused = pairs.by == Pairs::kFused;
    (void)hipGetLastError();
    if (n_seqs > 0 && !fused) {
        with_group(seqs.group, [&](auto group) {
            hipLaunchKernelGGL(margin_kernel<decltype(group)::value>, blocks_of(n_seqs * seqs.parts, kThreads / seqs.group),
                               dim3(kThreads), 0, s, in, p, seqs.parts, sums);
        });
        if (seqs.parts > 1)
            hipLaunchKernelGGL(margin_join_kernel, blocks_of(n_seqs, kWaves), dim3(kThreads), 0, s, n_seqs, p, seqs.parts, sums);
    }
    if (n_groups == 0) {
        // no pair, no gradient
    } else if (fused) {
        hipLaunchKernelGGL(pairs_kernel<true>, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, in, p, grad_logp);
    } else if (pairs.by == Pairs::kFew) {
        hipLaunchKernelGGL(pairs_few_kernel, blocks_of(n_groups, kThreads / kFew), dim3(kThreads), 0, s, n_seqs, p);
    } else if (pairs.by == Pairs::kParts) {
        hipLaunchKernelGGL(pairs_part_kernel, dim3(blocks_for(n_groups * pairs.parts)), dim3(kThreads), 0, s, n_seqs, p,
                           pairs.parts, losses);
        hipLaunchKernelGGL(pairs_finish_kernel, blocks_of(n_groups, kWaves), dim3(kThreads), 0, s, n_seqs, p, pairs.parts, losses);
    } else {
        hipLaunchKernelGGL(pairs_kernel<false>, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, in, p, nullptr);
    }
    if (grad_logp && n_tokens > 0 && !fused) {
        if (n_seqs > 0 && n_groups > 0)
            with_group(seqs.group, [&](auto group) {
                hipLaunchKernelGGL(spread_kernel<decltype(group)::value>, blocks_of(n_seqs * seqs.parts, kThreads / seqs.group),
                                   dim3(kThreads), 0, s, in, weights, seqs.parts, grad_logp);
            });
        else
            hipLaunchKernelGGL(zero_kernel, blocks_of(n_tokens, kThreads), dim3(kThreads), 0, s, grad_logp, n_tokens);
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
    if (n_groups > 0) {
        const Tokens in{scores, nullptr, nullptr, n_docs, group_offsets, n_groups};
        // threads enough to hold a group of twice the mean size
        const double mean = double(n_docs) / double(n_groups);
        const int lanes = mean <= 64.0 ? 8 : mean <= 128.0 ? 16 : mean <= 256.0 ? 32 : mean <= 512.0 ? kWave : kThreads;
        with_group(lanes, [&](auto group) {
            hipLaunchKernelGGL(advantage_kernel<decltype(group)::value>, blocks_of(n_groups, kThreads / lanes), dim3(kThreads), 0, s,
                               in, eps, (flags & TREE_ENS_CENTER_ONLY) != 0, advantages);
        });
    } else {
        hipLaunchKernelGGL(zero_kernel, blocks_of(n_docs, kThreads), dim3(kThreads), 0, s, advantages, n_docs);
    }
    return launched("group advantage");
}

int tree_ens_policy_workspace(int64_t n_tokens, int64_t n_seqs, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (int rc = check_counts(n_tokens, n_seqs, 0))
        return rc;
    *bytes = policy_space(n_tokens, n_seqs).bytes;
    return TREE_ENS_OK;
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
    const PolicySpace space = policy_space(n_tokens, n_seqs);
    if (int rc = check_workspace(workspace, workspace_bytes, space.bytes))
        return rc;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Tokens in{logp, ref_logp, mask, n_tokens, seq_offsets, n_seqs};
    const Policy p{old_logp, advantages, 1.0f - clip_low, 1.0f + clip_high, kl_coef, grad_scale,
                   (flags & TREE_ENS_SEQ_MEAN) != 0, loss, kl, grad_logp};
    const SequencePlan seqs = sequence_plan(n_tokens, n_seqs);
    Pair<double> *sums = static_cast<Pair<double> *>(workspace);
    int64_t *counts = reinterpret_cast<int64_t *>(static_cast<char *>(workspace) + space.counts);
    (void)hipGetLastError();
    if (n_seqs == 0) {
        if (grad_logp && n_tokens > 0)
            hipLaunchKernelGGL(zero_kernel, blocks_of(n_tokens, kThreads), dim3(kThreads), 0, s, grad_logp, n_tokens);
        return launched("policy loss");
    }
    if (seqs.parts > 1 && p.mean && mask)
        hipLaunchKernelGGL(count_kernel, blocks_of(n_seqs * seqs.parts, 1), dim3(kThreads), 0, s, in, seqs.parts, counts);
    with_group(seqs.group, [&](auto group) {
        hipLaunchKernelGGL(policy_kernel<decltype(group)::value>, blocks_of(n_seqs * seqs.parts, kThreads / seqs.group),
                           dim3(kThreads), 0, s, in, p, seqs.parts, counts, sums);
    });
    if (seqs.parts > 1)
        hipLaunchKernelGGL(policy_join_kernel, blocks_of(n_seqs, kWaves), dim3(kThreads), 0, s, in, p, seqs.parts, counts, sums);
    return launched("policy loss");
}

} // extern "C"
