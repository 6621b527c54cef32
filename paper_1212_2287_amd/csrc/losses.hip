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

// Margins h, and weights dh / dlogp of a sequence's counted tokens.
__global__ void __launch_bounds__(kThreads)
margin_kernel(Tokens in, float beta, bool mean, float *margins, float *weights) {
    __shared__ double part[kWaves];
    for (int64_t s = blockIdx.x; s < in.n_seqs; s += gridDim.x) {
        const Span q = span_of(in.offsets, s, in.n);
        double sum = 0.0, count = 0.0;
        for (int64_t t = q.a + threadIdx.x; t < q.b; t += kThreads)
            if (in.counts(t)) {
                sum += in.ref ? in.logp[t] - in.ref[t] : in.logp[t];
                count += 1.0;
            }
        sum = block_sum(sum, part);
        count = block_sum(count, part);
        const double w = mean ? double(beta) / fmax(count, 1.0) : double(beta);
        if (threadIdx.x == 0) {
            margins[s] = float(w * sum);
            weights[s] = float(w);
        }
    }
}

// Loss of a group, and weights times the loss's gradient with respect to the margins. With d the
// margin of a pair, l = softplus(-d) + smoothing d and dl/dd = smoothing - sigmoid(-d). Each thread
// takes candidates and meets every other one, so nothing is added atomically.
__global__ void __launch_bounds__(kThreads)
pairs_kernel(const float *scores, int64_t n_seqs, const int64_t *groups, int64_t n_groups, const float *margins,
             float smoothing, float grad_scale, float *loss, float *weights) {
    __shared__ double part[kWaves];
    for (int64_t g = blockIdx.x; g < n_groups; g += gridDim.x) {
        const Span q = span_of(groups, g, n_seqs);
        if (weights)
            zero_outside(weights, n_seqs, groups, g, n_groups, q);
        double sum = 0.0, pairs = 0.0;
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads) {
            const float r = scores[i], h = margins[i];
            for (int64_t j = q.a; j < q.b; ++j)
                if (r > scores[j]) {
                    const float d = h - margins[j];
                    sum += fmaxf(-d, 0.0f) + log1pf(expf(-fabsf(d)));
                    if (smoothing > 0.0f)
                        sum += smoothing * d;
                    pairs += 1.0;
                }
        }
        sum = block_sum(sum, part);
        pairs = block_sum(pairs, part);
        if (threadIdx.x == 0)
            loss[g] = float(sum / fmax(pairs, 1.0));
        if (!weights)
            continue;
        const double share = double(grad_scale) / fmax(pairs, 1.0);
        for (int64_t i = q.a + threadIdx.x; i < q.b; i += kThreads) {
            const float r = scores[i], h = margins[i];
            double slope = 0.0;
            for (int64_t j = q.a; j < q.b; ++j) {
                const bool ahead = r > scores[j], behind = r < scores[j];
                if (!ahead && !behind)
                    continue;
                const float d = ahead ? h - margins[j] : margins[j] - h;
                const float e = expf(-fabsf(d));
                const float dl = smoothing - (d >= 0.0f ? e : 1.0f) / (1.0f + e);
                slope += ahead ? dl : -dl;
            }
            weights[i] = float(weights[i] * (share * slope));
        }
    }
}

// grad[t] = the sequence's weight at its counted tokens.
__global__ void __launch_bounds__(kThreads) spread_kernel(Tokens in, const float *weights, float *grad) {
    for (int64_t s = blockIdx.x; s < in.n_seqs; s += gridDim.x) {
        const Span q = span_of(in.offsets, s, in.n);
        zero_outside(grad, in.n, in.offsets, s, in.n_seqs, q);
        const float w = weights[s];
        for (int64_t t = q.a + threadIdx.x; t < q.b; t += kThreads)
            grad[t] = in.counts(t) ? w : 0.0f;
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

int64_t preference_bytes(int64_t n_seqs) { return (n_seqs * 4 + 15) / 16 * 16; }

} // namespace

extern "C" {

int tree_ens_preference_workspace(int64_t n_tokens, int64_t n_seqs, int64_t n_groups, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (int rc = check_counts(n_tokens, n_seqs, n_groups))
        return rc;
    *bytes = preference_bytes(n_seqs);
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
    if (int rc = check_workspace(workspace, workspace_bytes, preference_bytes(n_seqs)))
        return rc;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    const Tokens in{logp, ref_logp, mask, n_tokens, seq_offsets, n_seqs};
    float *weights = static_cast<float *>(workspace);
    (void)hipGetLastError();
    if (n_seqs > 0)
        hipLaunchKernelGGL(margin_kernel, dim3(blocks_for(n_seqs)), dim3(kThreads), 0, s, in, beta,
                           (flags & TREE_ENS_SEQ_MEAN) != 0, margins, weights);
    if (n_groups > 0)
        hipLaunchKernelGGL(pairs_kernel, dim3(blocks_for(n_groups)), dim3(kThreads), 0, s, scores, n_seqs, group_offsets,
                           n_groups, margins, smoothing, grad_scale, loss, grad_logp ? weights : nullptr);
    if (grad_logp && n_tokens > 0) {
        if (n_seqs > 0 && n_groups > 0)
            hipLaunchKernelGGL(spread_kernel, dim3(blocks_for(n_seqs)), dim3(kThreads), 0, s, in, weights, grad_logp);
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
