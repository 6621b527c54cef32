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
// Sums over sequences of any lengths read the tokens in tiles of equal size, neighbours a thread,
// so no workgroup waits for a long sequence. A thread finds the sequence of its first token by search
// and walks on; what a sequence leaves open at a thread's end is carried to the next one by a segmented
// scan over the workgroup. A sequence inside one tile has its sum stored by the tile; one that goes on
// leaves the tile's `tail` where it begins and `head` in every later tile, added up afterwards in order.
// ---------------------------------------------------------------------------------------------
constexpr int kEach = 16;
constexpr int kTile = kThreads * kEach;

template <typename B> struct Pair {
    double a;
    B b;
};
template <typename B> __device__ __forceinline__ Pair<B> operator+(Pair<B> x, Pair<B> y) { return {x.a + y.a, x.b + y.b}; }

// Two sums per sequence and two per tile.
template <typename B> struct Sums {
    Pair<B> *inside; // [n_seqs], of sequences inside one tile
    Pair<B> *head;   // [tiles]
    Pair<B> *tail;   // [tiles]
};

// The sequences of a tile's first and last token: the last s in [-1, n_seqs] with offsets[s] <= the
// token (-1: none), by one wave with 64 pivots at a time. Offsets that decrease give some indices of the
// range.
__device__ __forceinline__ int2 sequences_of(const int64_t *offsets, int n_seqs, int64_t first, int64_t last) {
    unsigned lo[2] = {0, 0}, hi[2] = {unsigned(n_seqs) + 2, unsigned(n_seqs) + 2}; // from -1 on
    const unsigned lane = threadIdx.x % kWave + 1;
    while (hi[0] - lo[0] > 1 || hi[1] - lo[1] > 1) { // offsets[lo - 1] <= the token < offsets[hi - 1]
        unsigned step[2];
        bool before[2] = {false, false};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            step[e] = (hi[e] - lo[e] + kWave) / (kWave + 1);
            // in 64 bits: the pivots beyond hi may pass 32
            const uint64_t p = lo[e] + uint64_t(lane) * step[e];
            if (p < hi[e])
                before[e] = offsets[p - 1] <= (e ? last : first);
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            lo[e] += unsigned(__popcll(__ballot(before[e]))) * step[e];
            hi[e] = step[e] < hi[e] - lo[e] ? lo[e] + step[e] : hi[e];
        }
    }
    return make_int2(int(lo[0]) - 1, int(lo[1]) - 1);
}

// The sequence of a token, while the token moves on inside a tile. Positions count from the tile's
// first token, sequences from that token's; those without one (before the first, after the last
// sequence) have indices outside [0, n_seqs) too.
constexpr int kStaged = 512; // offsets of a tile that are held in LDS
struct Walk {
    const int64_t *offsets;
    const int *staged; // offsets of the tile's sequences, within [-1, count]
    int64_t n_seqs, first, s0;
    int last, count; // last: the sequence of the tile's last token
    bool goes_on;    // past the tile
    int s, end;
    __device__ __forceinline__ int64_t sequence() const { return s0 + s; }
    __device__ __forceinline__ bool inside() const { return sequence() >= 0 && sequence() < n_seqs; }
    __device__ __forceinline__ int fetch(int i) const { // where sequence i begins
        if (s0 + i < 0)
            return first == 0 ? 0 : -1;
        if (s0 + i > n_seqs)
            return count;
        return int(max(int64_t(-1), min(max(offsets[s0 + i], int64_t(0)) - first, int64_t(count))));
    }
    __device__ __forceinline__ int start_of(int i) const { return i < kStaged ? staged[i] : fetch(i); }
    // s: a sequence at or before that of t
    __device__ __forceinline__ void place(int t) {
        int lo = s, hi = last;
        while (lo < hi) {
            const int mid = lo + (hi - lo + 1) / 2;
            if (start_of(mid) <= t)
                lo = mid;
            else
                hi = mid - 1;
        }
        s = lo;
        end = s < last ? start_of(s + 1) : goes_on ? INT32_MAX : count;
    }
};

// Called by every thread of the workgroup; `q`: the sequences of the tile's first and last token.
__device__ __forceinline__ Walk walk_of(const Tokens &in, int64_t first, int64_t count, int2 q, int *staged) {
    Walk w{in.offsets, staged, in.n_seqs, first, q.x, max(q.y - q.x, 0), int(count), true, 0, 0};
    const int64_t at = w.s0 + w.last;
    if (at >= 0 && at < in.n_seqs)
        w.goes_on = min(in.offsets[at + 1], in.n) > first + count;
    __syncthreads(); // the tile before has been walked
    for (int i = threadIdx.x; i <= w.last && i < kStaged; i += kThreads)
        staged[i] = w.fetch(i);
    __syncthreads();
    return w;
}

typedef float float4_ __attribute__((ext_vector_type(4), aligned(4)));
typedef unsigned unsigned_ __attribute__((aligned(1)));

// A thread's tokens [t, t + count) of an array.
template <int E> __device__ __forceinline__ void load_tokens(const float *p, int64_t t, int count, float (&x)[E]) {
    if (count == E) {
#pragma unroll
        for (int v = 0; v < E; v += 4) {
            const float4_ a = *reinterpret_cast<const float4_ *>(p + t + v);
#pragma unroll
            for (int k = 0; k < 4; ++k)
                x[v + k] = a[k];
        }
        return;
    }
#pragma unroll
    for (int k = 0; k < E; ++k)
        x[k] = k < count ? p[t + k] : 0.0f;
}

template <int E> __device__ __forceinline__ void store_tokens(float *p, int64_t t, int count, const float (&x)[E]) {
    if (count == E) {
#pragma unroll
        for (int v = 0; v < E; v += 4)
            *reinterpret_cast<float4_ *>(p + t + v) = float4_{x[v], x[v + 1], x[v + 2], x[v + 3]};
        return;
    }
#pragma unroll
    for (int k = 0; k < E; ++k)
        if (k < count)
            p[t + k] = x[k];
}

// Bit k: byte k of x is not 0.
__device__ __forceinline__ unsigned nonzero_bytes(unsigned x) {
    const unsigned high = (((x & 0x7f7f7f7fu) + 0x7f7f7f7fu) | x) & 0x80808080u;
    return ((high >> 7) * 0x10204080u) >> 28;
}

// Bit k: token t + k counts.
template <int E> __device__ __forceinline__ unsigned load_mask(const uint8_t *mask, int64_t t, int count) {
    if (count <= 0)
        return 0u;
    const unsigned all = (1u << count) - 1;
    if (!mask)
        return all;
    unsigned bits = 0;
    if (count == E) {
#pragma unroll
        for (int v = 0; v < E; v += 4)
            bits |= nonzero_bytes(*reinterpret_cast<const unsigned_ *>(mask + t + v)) << v;
        return bits;
    }
    for (int k = 0; k < count; ++k)
        bits |= unsigned(mask[t + k] != 0) << k;
    return bits;
}

// Lanes' values moved by a DPP control; 0 where no lane is the source.
template <int kControl, int kRows> __device__ __forceinline__ int moved(int x) {
    return __builtin_amdgcn_update_dpp(0, x, kControl, kRows, 0xf, false);
}
template <int kControl, int kRows> __device__ __forceinline__ double moved(double x) {
    const long long u = __double_as_longlong(x);
    const unsigned lo = unsigned(moved<kControl, kRows>(int(u))), hi = unsigned(moved<kControl, kRows>(int(u >> 32)));
    return __longlong_as_double(static_cast<long long>(static_cast<unsigned long long>(hi) << 32 | lo));
}

// One step of an inclusive scan over the wave that starts again wherever a sequence ended.
template <int kControl, int kRows, typename B> __device__ __forceinline__ void scan_step(Pair<B> &run, int &stop) {
    const Pair<B> p{moved<kControl, kRows>(run.a), moved<kControl, kRows>(run.b)};
    const int q = moved<kControl, kRows>(stop);
    if (!stop)
        run = p + run;
    stop |= q;
}

// Adds up the tile's tokens by sequence: x and, counted, y (one of them per token if it has none).
// Stores the sums. Tokens that do not count hold 0.
template <typename B, typename Y>
__device__ __forceinline__ void sum_tile(const Sums<B> &out, int64_t tile, Walk w, float (&x)[kEach], Y &&y) {
    __shared__ Pair<B> part[kWaves];
    __shared__ int closed[kWaves];
    const int t = threadIdx.x * kEach, count = min(kEach, w.count - t);
    Pair<B> open{0, 0}, head{0, 0}; // of the sequence being walked; of the one that the thread began in
    int ended = 0;                  // some sequence ended in this thread
    int64_t head_s = -1;            // the one that the thread began in, if it ends here
    bool head_before = false;       // and began before the tile
    if (count > 0) {
        w.place(t);
        const int start = w.start_of(w.s);
        bool own = start >= t; // the walked sequence began in this thread
        const auto close = [&] {
            if (w.inside()) {
                if (own) {
                    out.inside[w.sequence()] = open;
                } else {
                    head = open;
                    head_s = w.sequence();
                    head_before = start < 0;
                }
            }
            open = {0, 0};
            ended = 1;
            own = true;
        };
        int k = 0;
        while (t + count > w.end) { // some tokens are the next sequence's
            const int to = w.end - t;
#pragma unroll
            for (int i = 0; i < kEach; ++i) {
                open.a += i < to ? x[i] : 0.0f;
                x[i] = i < to ? 0.0f : x[i];
            }
            open.b = y(k, to);
            close();
            k = to;
            w.s += 1;
            w.place(t + to);
        }
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            open.a += x[i];
        open.b = y(k, count);
        if (t + count == w.end)
            close();
    }
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
    Pair<B> run = open;
    int stop = ended;
    scan_step<0x111, 0xf>(run, stop); // row_shr 1, 2, 4, 8: within 16 lanes
    scan_step<0x112, 0xf>(run, stop);
    scan_step<0x114, 0xf>(run, stop);
    scan_step<0x118, 0xf>(run, stop);
    scan_step<0x142, 0xa>(run, stop); // row_bcast 15: into the second and fourth 16
    scan_step<0x143, 0xc>(run, stop); // row_bcast 31: into the upper 32
    __syncthreads();                  // the tile before has been read
    if (lane == kWave - 1) {
        part[wave] = run;
        closed[wave] = stop;
    }
    __syncthreads();
    Pair<B> carry{__shfl_up(run.a, 1), __shfl_up(run.b, 1)};
    int stopped = __shfl_up(stop, 1);
    if (lane == 0) {
        carry = {0, 0};
        stopped = 0;
    }
    for (int k = wave - 1; k >= 0 && !stopped; --k) {
        carry = part[k] + carry;
        stopped = closed[k];
    }
    if (head_s >= 0)
        (head_before ? out.head[tile] : out.inside[head_s]) = carry + head;
    w.s = w.last;
    if (threadIdx.x == kThreads - 1 && w.goes_on && w.inside())
        (w.start_of(w.s) < 0 ? out.head : out.tail)[tile] = ended ? open : carry + open;
}

// The sums of a sequence, from the tiles.
template <typename B> __device__ __forceinline__ Pair<B> joined(const Sums<B> &in, int64_t s, Span q) {
    if (q.a == q.b)
        return {0, 0};
    const int64_t first = q.a / kTile, last = (q.b - 1) / kTile;
    if (first == last)
        return in.inside[s];
    Pair<B> sum = in.tail[first];
#pragma unroll 4
    for (int64_t k = first + 1; k <= last; ++k)
        sum = sum + in.head[k];
    return sum;
}

// ---------------------------------------------------------------------------------------------
// Preference loss
// ---------------------------------------------------------------------------------------------

// Sums of a sequence's log ratios, and how many count; and the tiles' sequences, for spread_tile_kernel.
__global__ void __launch_bounds__(kThreads) ratio_tile_kernel(Tokens in, Sums<int> out, int2 *bounds) {
    __shared__ int staged[kStaged];
    const int64_t tiles = (in.n + kTile - 1) / kTile;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t first = tile * kTile, size = min(int64_t(kTile), in.n - first), t = first + threadIdx.x * kEach;
        const int count = int(min(int64_t(kEach), in.n - t));
        float x[kEach], r[kEach] = {};
        load_tokens(in.logp, t, count, x);
        if (in.ref)
            load_tokens(in.ref, t, count, r);
        const unsigned use = load_mask<kEach>(in.mask, t, count);
        __shared__ int2 found;
        if (threadIdx.x < kWave) {
            const int2 q = sequences_of(in.offsets, int(in.n_seqs), first, first + size - 1);
            if (threadIdx.x == 0)
                bounds[tile] = found = q;
        }
        __syncthreads();
        const int2 q = found;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
            x[k] = use >> k & 1u ? x[k] - r[k] : 0.0f;
        sum_tile(out, tile, walk_of(in, first, size, q, staged), x,
                 [&](int k, int to) { return __popc(use & (2u << (to - 1)) - (1u << k)); });
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

constexpr int kFour = 4; // neighbours that a lane takes of a sequence that is its wave's

// Sum of a sequence's log ratios and how many count, by a wave.
__device__ __forceinline__ Pair<int> ratios_of(const Tokens &in, Span q) {
    double sum = 0.0;
    int counted = 0;
#pragma unroll 2
    for (int64_t t = q.a + threadIdx.x % kWave * kFour; t < q.b; t += kWave * kFour) {
        const int count = int(min(int64_t(kFour), q.b - t));
        float x[kFour], r[kFour] = {};
        load_tokens(in.logp, t, count, x);
        if (in.ref)
            load_tokens(in.ref, t, count, r);
        const unsigned use = load_mask<kFour>(in.mask, t, count);
#pragma unroll
        for (int k = 0; k < kFour; ++k)
            sum += use >> k & 1u ? x[k] - r[k] : 0.0f;
        counted += __popc(use);
    }
    return {wave_sum(sum), wave_sum(counted)};
}

// The gradient at a sequence's tokens, by a wave.
__device__ __forceinline__ void spread(const Tokens &in, Span q, float weight, float *grad) {
    for (int64_t t = q.a + threadIdx.x % kWave * kFour; t < q.b; t += kWave * kFour) {
        const int count = int(min(int64_t(kFour), q.b - t));
        const unsigned use = load_mask<kFour>(in.mask, t, count);
        float d[kFour];
#pragma unroll
        for (int k = 0; k < kFour; ++k)
            d[k] = use >> k & 1u ? weight : 0.0f;
        store_tokens(grad, t, count, d);
    }
}

__device__ __forceinline__ void spread_zero(float *grad, int64_t a, int64_t b) {
    for (int64_t t = a + threadIdx.x % kWave; t < b; t += kWave)
        grad[t] = 0.0f;
}

constexpr int kHeld = 512; // candidates of a group that are held in LDS

// What the pairs that a thread met add up to: softplus(-d), d and 1.
struct Met {
    float loss, lead;
    int pairs;
};
// The same over threads, with the smoothing.
struct Loss {
    double sum, pairs;
    // Margins that are infinite have no smoothed loss that is finite, but may have a plain one.
    __device__ __forceinline__ void add(const Met &m, float smoothing, double weight) {
        sum += weight * (smoothing > 0.0f ? m.loss + double(smoothing) * m.lead : double(m.loss));
        pairs += weight * m.pairs;
    }
};

// One pair: dl/dh of the candidate `me`, and with kLoss the pair's loss. Candidates are (margin, score),
// margins and losses in units of ln 2 here. With d the margin by which the better one leads and e =
// exp(-|d|): l = softplus(-d) + smoothing d, softplus(-d) = max(-d, 0) + log1p(e), dl/dd = smoothing -
// sigmoid(-d).
constexpr float kLog2e = 1.44269504088896340736f;
constexpr double kLn2 = 0.693147180559945309417;
template <bool kLoss> __device__ __forceinline__ float meet(float2 me, float2 other, float smoothing, Met &met) {
    const bool ahead = me.y > other.y, behind = me.y < other.y;
    const float lead = me.x - other.x;
    const float e = __builtin_amdgcn_exp2f(-fabsf(lead));
    const float u = 1.0f + e, r = __builtin_amdgcn_rcpf(u);
    if (kLoss) {
        const float d = ahead ? lead : -lead;
        // log1p(e) = log u + log(1 + rest / u), with the rest that u was rounded by
        float l = __builtin_amdgcn_logf(u) + fmaxf(-d, 0.0f);
        l = fmaf((e - (u - 1.0f)) * r, kLog2e, l);
        met.loss += ahead || behind ? l : 0.0f;
        met.lead += ahead || behind ? d : 0.0f;
        met.pairs += ahead || behind;
    }
    const float dl = smoothing - ((lead >= 0.0f) == ahead ? e * r : r);
    return ahead ? dl : behind ? -dl : 0.0f;
}

// The n <= kHeld candidates of a group lie twice in a row, so that i + k needs no remainder. In step k
// candidate i meets i + k (modulo n), for its own slope alone, so nothing is added atomically; the first
// half of the steps meets every pair once and takes its loss. One thread takes candidate i in every
// `shares`-th step from 1 + share on; returns its slope.
__device__ __forceinline__ float meet_held(const float2 *held, int n, int i, int share, int shares, float smoothing, Loss &loss) {
    const float2 me = held[i], *other = held + i;
    Met met{0.0f, 0.0f, 0}, unused = met;
    float slope = 0.0f;
    int k = 1 + share;
#pragma unroll 4
    for (; k <= (n - 1) / 2; k += shares)
        slope += meet<true>(me, other[k], smoothing, met);
    if (2 * k == n) { // opposite each other: the lower one takes the loss
        slope += meet<true>(me, other[k], smoothing, i < k ? met : unused);
        k += shares;
    }
#pragma unroll 4
    for (; k < n; k += shares)
        slope += meet<false>(me, other[k], smoothing, met);
    loss.add(met, smoothing, 1.0);
    return slope;
}

// One thread's candidate against the kHeld or fewer of a larger group that are held: every pair is met
// twice.
__device__ __forceinline__ float meet_window(float2 me, const float2 *held, int fit, int share, int shares, float smoothing, Loss &loss) {
    Met met{0.0f, 0.0f, 0};
    float slope = 0.0f;
#pragma unroll 4
    for (int j = share; j < fit; j += shares)
        slope += meet<true>(me, held[j], smoothing, met);
    loss.add(met, smoothing, 0.5);
    return slope;
}

// Loss of a group, and weights times the loss's gradient with respect to the margins, by a workgroup.
// kFused: it also sums the sequences' tokens first and writes their gradients last, instead of the tile
// kernels.
template <bool kFused>
__global__ void __launch_bounds__(kThreads) pairs_kernel(Tokens in, Sums<int> sums, Preference p, float *grad) {
    __shared__ float2 held[2 * kHeld];
    __shared__ float slopes[kWaves][kHeld];
    const int wave = threadIdx.x / kWave, lane = threadIdx.x % kWave;
    for (int64_t g = blockIdx.x; g < max(p.n_groups, int64_t(1)); g += gridDim.x) {
        Span q{in.n_seqs, in.n_seqs}; // without groups, every sequence is before the first one
        if (p.n_groups > 0)
            q = span_of(p.groups, g, in.n_seqs);
        // sequences outside every group go with the first and the last one; their gradient is 0
        const int64_t lo = g == 0 ? 0 : q.a, hi = g >= p.n_groups - 1 ? in.n_seqs : q.b;
        const int64_t n = q.b - q.a;
        __syncthreads(); // held may still be read for the group before
        const auto take = [&](int64_t s, Pair<int> v) {
            const double w = p.mean ? double(p.beta) / max(v.b, 1) : double(p.beta);
            const float h = float(w * v.a);
            p.margins[s] = h;
            p.weights[s] = s < q.a || s >= q.b ? 0.0f : float(w);
            if (n <= kHeld && s >= q.a && s < q.b)
                held[s - q.a] = held[s - q.a + n] = make_float2(h * kLog2e, p.scores[s]);
        };
        if constexpr (kFused) {
            for (int64_t s = lo + wave; s < hi; s += kWaves) {
                const Pair<int> v = ratios_of(in, span_of(in.offsets, s, in.n));
                if (lane == 0)
                    take(s, v);
            }
        } else {
            for (int64_t s = lo + threadIdx.x; s < hi; s += kThreads)
                take(s, joined(sums, s, span_of(in.offsets, s, in.n)));
        }
        __syncthreads();
        Loss loss{0.0, 0.0};
        if (n <= kHeld) {
            // waves take steps in turn and leave their slopes in rows of their own
            for (int i = lane; i < n; i += kWave)
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
                const float2 me = i < q.b ? make_float2(p.margins[i] * kLog2e, p.scores[i]) : make_float2(0.0f, 0.0f);
                double sum = 0.0;
                for (int64_t j0 = q.a; j0 < q.b; j0 += kHeld) {
                    const int fit = int(min(int64_t(kHeld), q.b - j0));
                    __syncthreads();
                    for (int j = threadIdx.x; j < fit; j += kThreads)
                        held[j] = make_float2(p.margins[j0 + j] * kLog2e, p.scores[j0 + j]);
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
        if (threadIdx.x == 0 && p.n_groups > 0)
            p.loss[g] = float(loss.sum * (kLn2 * share));
        __syncthreads();
        if constexpr (kFused) {
            if (!grad)
                continue;
            for (int64_t s = lo + wave; s < hi; s += kWaves) {
                const Span t = span_of(in.offsets, s, in.n);
                spread(in, t, float(p.weights[s] * (p.grad_scale * share)), grad);
                if (s == 0)
                    spread_zero(grad, 0, t.a);
                if (s == in.n_seqs - 1)
                    spread_zero(grad, t.b, in.n);
            }
        } else {
            for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
                p.weights[i] = float(p.weights[i] * (p.grad_scale * share));
        }
    }
}

// Margins and weights, a thread a sequence, where pairs_part_kernel needs them all before it starts.
__global__ void __launch_bounds__(kThreads) join_kernel(Tokens in, Sums<int> sums, Preference p) {
    for (int64_t s = blockIdx.x * int64_t(kThreads) + threadIdx.x; s < in.n_seqs; s += int64_t(gridDim.x) * kThreads) {
        const Pair<int> v = joined(sums, s, span_of(in.offsets, s, in.n));
        const double w = p.mean ? double(p.beta) / max(v.b, 1) : double(p.beta);
        p.margins[s] = float(w * v.a);
        p.weights[s] = float(w);
    }
}

constexpr int kHeldPart = 2048;

// One of `parts` shares of a group's candidates, against all of the group. As many threads take a
// candidate as there are, each every so many steps of it.
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
            const float2 me = make_float2(p.margins[q.a + i] * kLog2e, p.scores[q.a + i]);
            double slope = 0.0;
            if (n <= kHeldPart) {
                if (i0 == from)
                    for (int j = threadIdx.x; j < n; j += kThreads)
                        held[j] = held[j + n] = make_float2(p.margins[q.a + j] * kLog2e, p.scores[q.a + j]);
                __syncthreads();
                if (share < shares)
                    slope = meet_held(held, int(n), int(i), share, shares, p.smoothing, loss);
            } else {
                for (int64_t j0 = 0; j0 < n; j0 += kHeldPart) {
                    const int fit = int(min(int64_t(kHeldPart), n - j0));
                    __syncthreads();
                    for (int j = threadIdx.x; j < fit; j += kThreads)
                        held[j] = make_float2(p.margins[q.a + j0 + j] * kLog2e, p.scores[q.a + j0 + j]);
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
        // sequences outside every group
        if (g == 0)
            for (int64_t i = lane; i < q.a; i += kWave)
                p.weights[i] = 0.0f;
        if (g == p.n_groups - 1)
            for (int64_t i = q.b + lane; i < n_seqs; i += kWave)
                p.weights[i] = 0.0f;
    }
}

// Groups of a few candidates: eight lanes take one. Larger ones among them are met from memory.
constexpr int kFew = 8;
__global__ void __launch_bounds__(kThreads) pairs_few_kernel(Tokens in, Sums<int> sums, Preference p) {
    constexpr int kGroups = kThreads / kFew;
    const int lane = threadIdx.x % kFew;
    for (int64_t g0 = blockIdx.x * int64_t(kGroups); g0 < p.n_groups; g0 += int64_t(gridDim.x) * kGroups) {
        const int64_t g = g0 + threadIdx.x / kFew;
        if (g >= p.n_groups)
            continue;
        const Span q = span_of(p.groups, g, in.n_seqs);
        const int64_t lo = g == 0 ? 0 : q.a, hi = g == p.n_groups - 1 ? in.n_seqs : q.b;
        for (int64_t s = lo + lane; s < hi; s += kFew) {
            const bool member = s >= q.a && s < q.b;
            const Pair<int> v = joined(sums, s, span_of(in.offsets, s, in.n));
            const double by = p.mean ? double(p.beta) / max(v.b, 1) : double(p.beta);
            p.margins[s] = float(by * v.a);
            p.weights[s] = member ? float(by) : 0.0f;
        }
        __threadfence_block(); // the group's lanes are of one wave
        Loss loss{0.0, 0.0};
        for (int64_t i = q.a + lane; i < q.b; i += kFew) {
            const float2 me = make_float2(p.margins[i] * kLog2e, p.scores[i]);
            Met met{0.0f, 0.0f, 0};
            float slope = 0.0f;
#pragma unroll 2
            for (int64_t j = q.a; j < q.b; ++j)
                slope += meet<true>(me, make_float2(p.margins[j] * kLog2e, p.scores[j]), p.smoothing, met);
            loss.add(met, p.smoothing, 0.5);
            p.weights[i] = float(p.weights[i] * slope);
        }
        for (int off = kFew / 2; off; off >>= 1) {
            loss.sum += __shfl_xor(loss.sum, off);
            loss.pairs += __shfl_xor(loss.pairs, off);
        }
        const double share = 1.0 / fmax(loss.pairs, 1.0);
        if (lane == 0)
            p.loss[g] = float(loss.sum * (kLn2 * share));
        for (int64_t i = q.a + lane; i < q.b; i += kFew)
            p.weights[i] = float(p.weights[i] * (p.grad_scale * share));
    }
}

// Stores a tile of kEach neighbours a thread, through LDS so that a wave's stores are neighbours.
__device__ __forceinline__ void store_tile(float *out, int64_t first, int size, const float (&d)[kEach]) {
    constexpr int kPad = kEach + 4; // rows of other banks
    __shared__ float rows[kThreads * kPad];
    __syncthreads(); // the tile before has been stored
#pragma unroll
    for (int v = 0; v < kEach; v += 4)
        *reinterpret_cast<float4 *>(rows + threadIdx.x * kPad + v) = make_float4(d[v], d[v + 1], d[v + 2], d[v + 3]);
    __syncthreads();
#pragma unroll
    for (int v = 0; v < kEach; v += 4) {
        const int t = v * kThreads + threadIdx.x * 4;
        const float4 q = *reinterpret_cast<const float4 *>(rows + t / kEach * kPad + t % kEach);
        if (t + 4 <= size)
            *reinterpret_cast<float4_ *>(out + first + t) = float4_{q.x, q.y, q.z, q.w};
        else
            for (int k = 0; t + k < size; ++k)
                out[first + t + k] = rows[t / kEach * kPad + t % kEach + k];
    }
}

// grad[t] = the sequence's weight at its counted tokens.
__global__ void __launch_bounds__(kThreads) spread_tile_kernel(Tokens in, const int2 *bounds, const float *weights, float *grad) {
    __shared__ int staged[kStaged];
    const int64_t tiles = (in.n + kTile - 1) / kTile;
    for (int64_t tile = blockIdx.x; tile < tiles; tile += gridDim.x) {
        const int64_t first = tile * kTile;
        const int size = int(min(int64_t(kTile), in.n - first)), t = threadIdx.x * kEach, count = min(kEach, size - t);
        const unsigned use = load_mask<kEach>(in.mask, first + t, count);
        Walk w = walk_of(in, first, size, bounds[tile], staged);
        float d[kEach] = {};
        for (int k = 0; k < count;) {
            w.place(t + k);
            const float x = w.inside() ? weights[w.sequence()] : 0.0f;
            const int to = min(w.end - t, count);
#pragma unroll
            for (int i = 0; i < kEach; ++i)
                d[i] = i >= k && use >> i & 1u ? x : d[i];
            k = to;
            w.s += 1;
        }
        store_tile(grad, first, size, d);
    }
}

__global__ void __launch_bounds__(kThreads)
advantage_kernel(const float *scores, int64_t n, const int64_t *groups, int64_t n_groups, float eps, bool center,
                 float *out) {
    for (int64_t g = blockIdx.x; g < n_groups; g += gridDim.x) {
        const Span q = span_of(groups, g, n);
        const double count = fmax(double(q.b - q.a), 1.0);
        double sum = 0.0, squares = 0.0;
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            sum += scores[i];
        const double mean = block_sum(sum) / count;
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads)
            squares += (scores[i] - mean) * (scores[i] - mean);
        const double std = sqrt(block_sum(squares) / count);
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
    for (int64_t s = blockIdx.x; s < in.n_seqs; s += gridDim.x) {
        const Span q = span_of(in.offsets, s, in.n);
        const float a = p.advantages[s];
        double share = 1.0;
        if (p.mean) {
            double count = 0.0;
            for (int64_t t = q.a + threadIdx.x; t < q.b; t += kThreads)
                count += in.counts(t) ? 1.0 : 0.0;
            share = 1.0 / fmax(block_sum(count), 1.0);
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
        loss = block_sum(loss);
        kl = block_sum(kl);
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
int64_t bounds_bytes(int64_t n_tokens) { return 8 * tiles_of(n_tokens); }

template <typename B> Sums<B> sums_at(void *workspace, int64_t n_tokens, int64_t n_seqs) {
    static_assert(sizeof(Pair<B>) == 16, "as sums_bytes counts");
    Pair<B> *p = static_cast<Pair<B> *>(workspace);
    return {p, p + n_seqs, p + n_seqs + tiles_of(n_tokens)};
}

// Which kernels meet the pairs, by the mean sizes of groups and sequences. Measured (us of the whole loss;
// groups x candidates x tokens; pairs_kernel fused / tile kernels with pairs_few_kernel / with pairs_kernel /
// with pairs_part_kernel):
//   64 x 2 x 250: 7.1 / 14.9 / 15.6; 512 x 2 x 500: 10.2 / 16.0 / 16.5; 512 x 8 x 500: 18.9 / 19.7 / 20.4;
//   4,096 x 2 x 500: 39 / 23.9 / 34; 50,000 x 2 x 30: 272 / 29 / 153; 2 x 2 x 60,000: 451 / 12.9 / 14.2;
//   5,000 x 8 x 20: 47 / 25.6 / 37; 512 x 16 x 500: 44 / 41 / 25.2; 2,000 x 40 x 100: - / - / 48 / 58;
//   909 x 110 x 143: - / - / 79 / 75; 100 x 300 x 100: - / - / 137 / 45; 9,090 x 110 x 10: - / - / 190 / 210.
enum class Pairs { kFused, kFew, kGroup, kParts };
struct PreferencePlan {
    Pairs by;
    int parts;
};

PreferencePlan preference_plan(int64_t n_tokens, int64_t n_seqs, int64_t n_groups) {
    if (n_groups == 0 || n_seqs == 0)
        return {Pairs::kGroup, 1};
    const double seqs = double(n_seqs) / double(n_groups), tokens = double(n_tokens) / double(n_seqs);
    if (seqs <= 8.0 && n_seqs <= 4096 && tokens <= 1024.0)
        return {Pairs::kFused, 1};
    if (seqs <= 8.0)
        return {Pairs::kFew, 1};
    if (seqs >= 96.0 && n_groups <= 2048) // workgroups for the whole card, but eight candidates at least for each
        return {Pairs::kParts, int(std::min(std::ceil(2048.0 / double(n_groups)), std::ceil(seqs / 8.0)))};
    return {Pairs::kGroup, 1};
}

// Where a preference loss keeps what its kernels hand on.
struct PreferenceSpace {
    int64_t sums, bounds, weights, partial, bytes;
};
PreferenceSpace preference_space(int64_t n_tokens, int64_t n_seqs, int64_t n_groups) {
    const PreferencePlan plan = preference_plan(n_tokens, n_seqs, n_groups);
    const auto round = [](int64_t b) { return (b + 15) / 16 * 16; };
    PreferenceSpace p{0, sums_bytes(n_tokens, n_seqs), 0, 0, 0};
    p.weights = p.bounds + round(bounds_bytes(n_tokens));
    p.partial = p.weights + round(4 * n_seqs);
    p.bytes = p.partial + (plan.by == Pairs::kParts ? n_groups * plan.parts * int64_t(sizeof(Loss)) : 0);
    return p;
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
    const Sums<int> sums = sums_at<int>(at + space.sums, n_tokens, n_seqs);
    int2 *bounds = reinterpret_cast<int2 *>(at + space.bounds);
    float *weights = reinterpret_cast<float *>(at + space.weights);
    Loss *partial = reinterpret_cast<Loss *>(at + space.partial);
    const Preference p{scores, group_offsets, n_groups, beta, smoothing, grad_scale, (flags & TREE_ENS_SEQ_MEAN) != 0,
                       loss, margins, weights};
    const PreferencePlan plan = preference_plan(n_tokens, n_seqs, n_groups);
    const bool fused = plan.by == Pairs::kFused;
    const auto blocks = [](int64_t items, int64_t per_block) { return dim3(blocks_for((items + per_block - 1) / per_block)); };
    (void)hipGetLastError();
    if (!fused && n_seqs > 0 && n_tokens > 0)
        hipLaunchKernelGGL(ratio_tile_kernel, blocks(n_tokens, kTile), dim3(kThreads), 0, s, in, sums, bounds);
    if (fused) {
        hipLaunchKernelGGL(pairs_kernel<true>, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, in, sums, p, grad_logp);
    } else if (plan.by == Pairs::kFew) {
        hipLaunchKernelGGL(pairs_few_kernel, blocks(n_groups, kThreads / kFew), dim3(kThreads), 0, s, in, sums, p);
    } else if (plan.by == Pairs::kParts) {
        hipLaunchKernelGGL(join_kernel, blocks(n_seqs, kThreads), dim3(kThreads), 0, s, in, sums, p);
        hipLaunchKernelGGL(pairs_part_kernel, dim3(blocks_for(n_groups * plan.parts)), dim3(kThreads), 0, s, n_seqs, p, plan.parts,
                           partial);
        hipLaunchKernelGGL(pairs_finish_kernel, blocks(n_groups, kWaves), dim3(kThreads), 0, s, n_seqs, p, plan.parts, partial);
    } else if (n_seqs > 0 || n_groups > 0) {
        hipLaunchKernelGGL(pairs_kernel<false>, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, in, sums, p, nullptr);
    }
    if (!fused && grad_logp && n_tokens > 0) {
        if (n_seqs > 0)
            hipLaunchKernelGGL(spread_tile_kernel, blocks(n_tokens, kTile), dim3(kThreads), 0, s, in, bounds, weights, grad_logp);
        else
            hipLaunchKernelGGL(zero_kernel, blocks(n_tokens, kThreads), dim3(kThreads), 0, s, grad_logp, n_tokens);
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
