// grads.hip -- the norm of many tensors together and their scaling to a norm allowed, on gfx950.
//
// The tensors' addresses, sizes and types go to a kernel as its arguments, kTensors at a time, so that nothing
// has to be copied or kept for it, and a captured call replays on the same tensors. Elements are cut into
// chunks that never cross a tensor's end; a workgroup takes every gridDim-th chunk and finds the tensor of
// each from the running number of chunks.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <new>
#include <string>
#include <type_traits>
#include <utility>
#include <vector>

#include "status.hpp"
#include "tree_ens.h"

namespace {

constexpr int kThreads = 256;
constexpr int kWave = 64;
constexpr int kTensors = 128;    // of one launch: its arguments stay below 4,096 bytes
constexpr int kMaxBlocks = 2048; // 8 workgroups to a CU

struct Tensors {
    const void *in[kTensors];
    void *out[kTensors]; // nullptr where there is none
    int64_t n[kTensors];
    int first[kTensors + 1]; // first chunk of each
    int chunk;               // elements
    unsigned char dtype[kTensors];
    int count;
};
static_assert(sizeof(Tensors) <= 4000, "kernel arguments");

template <typename T> struct Vec {
    static constexpr int N = 16 / sizeof(T);
    typedef T type __attribute__((ext_vector_type(16 / sizeof(T))));
    typedef type unaligned __attribute__((aligned(sizeof(T))));
};

// Elements of `p` before the first 16-byte boundary.
template <typename T> __device__ __forceinline__ int lead_of(const T *p) {
    return int((16u - unsigned(reinterpret_cast<uintptr_t>(p) & 15u)) & 15u) / int(sizeof(T));
}

// The last tensor that begins at the chunk or before it, from tensor `low` on, which does. Tensors without elements begin where
// the next one does.
__device__ __forceinline__ int tensor_of(const Tensors &t, int chunk, int low) {
    int high = t.count;
    if (low + 1 < high && t.first[low + 1] > chunk)
        return low;
    while (high - low > 1) {
        const int mid = (low + high) / 2;
        (t.first[mid] <= chunk ? low : high) = mid;
    }
    return low;
}

template <typename F> __device__ __forceinline__ void with_type(int dtype, F &&f) {
    if (dtype == TREE_ENS_F32)
        f(static_cast<float *>(nullptr));
    else if (dtype == TREE_ENS_BF16)
        f(static_cast<__bf16 *>(nullptr));
    else
        f(static_cast<_Float16 *>(nullptr));
}

// Calls f(type, in, out, elements) for every chunk of this workgroup.
template <typename F> __device__ __forceinline__ void for_chunks(const Tensors &t, F &&f) {
    const int chunks = t.first[t.count];
    for (int c = blockIdx.x, k = 0; c < chunks; c += gridDim.x) {
        k = tensor_of(t, c, k);
        const int64_t at = int64_t(c - t.first[k]) * t.chunk;
        const int n = int(min(int64_t(t.chunk), t.n[k] - at));
        with_type(t.dtype[k], [&](auto *type) {
            using T = std::decay_t<decltype(*type)>;
            f(static_cast<const T *>(t.in[k]) + at, static_cast<T *>(t.out[k]) + at, n);
        });
    }
}

template <bool kFar, typename V> __device__ __forceinline__ V load(const V *p) {
    if constexpr (kFar)
        return __builtin_nontemporal_load(p);
    return *p;
}

constexpr int kAhead = 4; // loads of a thread on their way at a time

// sqrt(sum of x^2): squares are taken and added in double, so neither the largest nor the smallest float's square is lost, a
// conversion and a multiply-add an element, which this card does at the rate of single precision. Bound by reading: 2.0 GB of a
// billion bf16 elements in 313 us with the join, 6.3 TB/s. Two sums a thread, because a single one is a chain as long as the chunk.
template <bool kFar>
__global__ void __launch_bounds__(kThreads) norm_part_kernel(Tensors t, double *partial) {
    const int tid = threadIdx.x;
    double sums[2] = {0.0, 0.0};
    const auto add = [&](double v, int k) { sums[k & 1] = fma(v, v, sums[k & 1]); };
    for_chunks(t, [&](auto *x, auto *, int n) {
        using T = std::remove_const_t<std::remove_pointer_t<decltype(x)>>;
        using V = Vec<T>;
        const int lead = min(lead_of(x), n), vecs = (n - lead) / V::N, rest = n - vecs * V::N;
        const auto *v = reinterpret_cast<const typename V::type *>(x + lead);
        int i = tid;
        for (; i + (kAhead - 1) * kThreads < vecs; i += kAhead * kThreads) {
            typename V::type q[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                q[j] = load<kFar>(v + i + j * kThreads);
#pragma unroll
            for (int k = 0; k < kAhead * V::N; ++k)
                add(double(float(q[k / V::N][k % V::N])), k);
        }
        for (; i < vecs; i += kThreads) {
            const typename V::type q = load<kFar>(v + i);
#pragma unroll
            for (int k = 0; k < V::N; ++k)
                add(double(float(q[k])), k);
        }
        if (tid < rest)
            add(double(float(x[tid < lead ? tid : tid + vecs * V::N])), 0);
    });
    double sum = sums[0] + sums[1];
    for (int off = kWave / 2; off; off >>= 1)
        sum += __shfl_xor(sum, off);
    __shared__ double part[kThreads / kWave];
    if (tid % kWave == 0)
        part[tid / kWave] = sum;
    __syncthreads();
    if (tid == 0)
        partial[blockIdx.x] = (part[0] + part[1]) + (part[2] + part[3]);
}

constexpr int kJoin = 1024;

// The workgroups' sums, always in the same order. A trip to memory or two, since the loads of a thread do not wait for each other:
// 8,192 sums take 2.8 us, with 256 threads and a load at a time 9.2.
__global__ void __launch_bounds__(kJoin) norm_join_kernel(const double *partial, int64_t n, float *norm) {
    const int tid = threadIdx.x;
    double sum = 0.0;
    for (int64_t i = tid; i < n; i += kAhead * kJoin) {
        double q[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j)
            q[j] = i + j * kJoin < n ? partial[i + j * kJoin] : 0.0;
        sum += (q[0] + q[1]) + (q[2] + q[3]);
    }
    for (int off = kWave / 2; off; off >>= 1)
        sum += __shfl_xor(sum, off);
    __shared__ double part[kJoin / kWave];
    if (tid % kWave == 0)
        part[tid / kWave] = sum;
    __syncthreads();
    if (tid < kWave) {
        sum = tid < kJoin / kWave ? part[tid] : 0.0;
        for (int off = kWave / 2; off; off >>= 1)
            sum += __shfl_xor(sum, off);
        if (tid == 0)
            *norm = float(sqrt(sum));
    }
}

// x min(1, max_norm / (norm + eps)), the factor in single precision, each product rounded once to its type. Bound by reading and
// writing: 3.7 GB of two billion elements take 1.40 ms, 5.3 TB/s both ways, where torch's copy of 4 GiB reaches 4.8. Vectors are aligned
// to the written tensor; what is read may start elsewhere.
template <bool kFarIn, bool kFarOut>
__global__ void __launch_bounds__(kThreads) clip_kernel(Tensors t, const float *norm, float max_norm, float eps) {
    const float bound = *norm + eps, ratio = max_norm / bound;
    const float factor = ratio >= 1.0f || bound == 0.0f ? 1.0f : ratio; // NaN stays; without a norm everything is 0
    for_chunks(t, [&](auto *x, auto *y, int n) {
        using T = std::remove_pointer_t<decltype(y)>;
        using V = Vec<T>;
        if (x == y && factor == 1.0f)
            return;
        const int tid = threadIdx.x;
        const int lead = min(lead_of(y), n), vecs = (n - lead) / V::N, rest = n - vecs * V::N;
        const auto *v = reinterpret_cast<const typename V::unaligned *>(x + lead);
        auto *o = reinterpret_cast<typename V::type *>(y + lead);
        const auto read = [&](int at) -> typename V::type {
            if constexpr (kFarIn)
                return __builtin_nontemporal_load(v + at);
            else
                return v[at];
        };
        const auto scale = [&](typename V::type q, int at) {
#pragma unroll
            for (int k = 0; k < V::N; ++k)
                q[k] = T(float(q[k]) * factor);
            if constexpr (kFarOut)
                __builtin_nontemporal_store(q, o + at);
            else
                o[at] = q;
        };
        int i = tid;
        for (; i + (kAhead - 1) * kThreads < vecs; i += kAhead * kThreads) {
            typename V::type q[kAhead];
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                q[j] = read(i + j * kThreads);
#pragma unroll
            for (int j = 0; j < kAhead; ++j)
                scale(q[j], i + j * kThreads);
        }
        for (; i < vecs; i += kThreads)
            scale(read(i), i);
        if (tid < rest) {
            const int one = tid < lead ? tid : tid + vecs * V::N;
            y[one] = T(float(x[one]) * factor);
        }
    });
}

using treeens::set_error;

int64_t size_of(int32_t dtype) { return dtype == TREE_ENS_F32 ? 4 : 2; }
bool misaligned(const void *p, unsigned a) { return reinterpret_cast<uintptr_t>(p) % a != 0; }

constexpr int64_t kMostElements = int64_t(1) << 48; // of all tensors, so that no number of bytes or chunks overflows

int check_tensors(int64_t n, const void *const *grads, const int64_t *counts, const int32_t *dtypes) {
    if (n < 0 || n > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tensors must be in [0, INT32_MAX]");
    if (n > 0 && (!grads || !counts || !dtypes))
        return set_error(TREE_ENS_E_ARG, "grads, counts or dtypes is NULL");
    int64_t all = 0;
    for (int64_t i = 0; i < n; ++i) {
        if (dtypes[i] != TREE_ENS_F32 && dtypes[i] != TREE_ENS_BF16 && dtypes[i] != TREE_ENS_F16)
            return set_error(TREE_ENS_E_ARG, "dtypes must be TREE_ENS_F32, TREE_ENS_BF16 or TREE_ENS_F16");
        if (counts[i] < 0 || counts[i] > kMostElements || (all += counts[i]) > kMostElements)
            return set_error(TREE_ENS_E_ARG, "counts must be >= 0 and the tensors within memory");
        if (counts[i] > 0 && !grads[i])
            return set_error(TREE_ENS_E_ARG, "a tensor with elements is NULL");
        if (misaligned(grads[i], unsigned(size_of(dtypes[i]))))
            return set_error(TREE_ENS_E_ARG, "a tensor is misaligned for its type");
    }
    return TREE_ENS_OK;
}

// Elements of a chunk: enough chunks for every CU where the tensors are small, larger ones where they are not. A billion bf16
// elements take 328, 318 and 317 us in chunks of up to 16,384, 32,768 and 65,536.
int64_t chunk_of(int64_t elements) {
    int64_t chunk = 2048;
    while (chunk < 32768 && elements / chunk > 2 * kMaxBlocks)
        chunk *= 2;
    while (elements / chunk > INT32_MAX / 2)
        chunk *= 2;
    return chunk;
}

// Calls launch(tensors, workgroups) for kTensors tensors after kTensors.
template <typename F>
void for_launches(int64_t n, const void *const *in, void *const *out, const int64_t *counts, const int32_t *dtypes, F &&launch) {
    for (int64_t at = 0; at < n; at += kTensors) {
        Tensors t;
        t.count = int(std::min<int64_t>(kTensors, n - at));
        int64_t elements = 0;
        for (int k = 0; k < t.count; ++k)
            elements += counts[at + k];
        const int64_t chunk = chunk_of(elements);
        t.chunk = int(chunk);
        t.first[0] = 0;
        for (int k = 0; k < t.count; ++k) {
            t.in[k] = in[at + k];
            t.out[k] = out ? out[at + k] : nullptr;
            t.n[k] = counts[at + k];
            t.dtype[k] = static_cast<unsigned char>(dtypes[at + k]);
            t.first[k + 1] = t.first[k] + int((counts[at + k] + chunk - 1) / chunk);
        }
        launch(t, std::min(t.first[t.count], kMaxBlocks));
    }
}

int64_t bytes_of(int64_t n, const int64_t *counts, const int32_t *dtypes) {
    int64_t bytes = 0;
    for (int64_t i = 0; i < n; ++i)
        bytes += counts[i] * size_of(dtypes[i]);
    return bytes;
}

// From these sizes on, loads and stores go past the caches. A norm of 2 GB takes 363 us with cached loads and 328 past
// them; 166 MB, normed and then clipped into other tensors, take 88 us with cached loads, which find them there the second time,
// and 102 past them. Stores past the caches leave those to the loads (111 us without).
constexpr int64_t kFarLoads = int64_t(192) << 20, kFarStores = int64_t(64) << 20;

int launched(const char *what) {
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess)
        return set_error(TREE_ENS_E_DEVICE, std::string(what) + " launch: " + hipGetErrorString(e));
    return TREE_ENS_OK;
}

int64_t partial_bytes(int64_t n) { return (n + kTensors - 1) / kTensors * kMaxBlocks * int64_t(sizeof(double)); }

struct Range {
    uintptr_t begin, end;
};

// Whether an `out` overlaps another, one of `in` that is not its own, or the norm.
bool overlapping(int64_t n, const void *const *in, void *const *out, const int64_t *counts, const int32_t *dtypes, const float *norm) {
    std::vector<Range> outs;
    outs.reserve(size_t(n));
    const auto range = [&](const void *p, int64_t i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p);
        return Range{at, at + uintptr_t(counts[i] * size_of(dtypes[i]))};
    };
    for (int64_t i = 0; i < n; ++i)
        if (counts[i] > 0)
            outs.push_back(range(out[i], i));
    std::sort(outs.begin(), outs.end(), [](const Range &a, const Range &b) { return a.begin < b.begin; });
    for (size_t k = 1; k < outs.size(); ++k)
        if (outs[k].begin < outs[k - 1].end)
            return true;
    const auto meets = [&](const Range &r) { // the first `out` that ends behind r's beginning does
        const auto o = std::upper_bound(outs.begin(), outs.end(), r.begin, [](uintptr_t at, const Range &b) { return at < b.end; });
        return o != outs.end() && o->begin < r.end;
    };
    for (int64_t i = 0; i < n; ++i)
        if (counts[i] > 0 && in[i] != out[i] && meets(range(in[i], i)))
            return true;
    return meets({reinterpret_cast<uintptr_t>(norm), reinterpret_cast<uintptr_t>(norm) + sizeof(float)});
}

} // namespace

extern "C" {

int tree_ens_grad_norm_workspace(int64_t n_tensors, int64_t *bytes) {
    treeens::clear_error();
    if (!bytes)
        return set_error(TREE_ENS_E_ARG, "bytes is NULL");
    *bytes = 0;
    if (n_tensors < 0 || n_tensors > INT32_MAX)
        return set_error(TREE_ENS_E_ARG, "n_tensors must be in [0, INT32_MAX]");
    *bytes = partial_bytes(n_tensors);
    return TREE_ENS_OK;
}

int tree_ens_grad_norm(void *stream, int64_t n_tensors, const void *const *grads, const int64_t *counts,
                       const int32_t *dtypes, float *norm, void *workspace, int64_t workspace_bytes) {
    treeens::clear_error();
    if (int rc = check_tensors(n_tensors, grads, counts, dtypes))
        return rc;
    if (!norm)
        return set_error(TREE_ENS_E_ARG, "norm is NULL");
    if (misaligned(norm, 4))
        return set_error(TREE_ENS_E_ARG, "norm is misaligned");
    if (const int64_t need = partial_bytes(n_tensors)) {
        if (!workspace || workspace_bytes < need)
            return set_error(TREE_ENS_E_ARG, "workspace is NULL or smaller than " + std::to_string(need) + " bytes");
        if (misaligned(workspace, 16))
            return set_error(TREE_ENS_E_ARG, "workspace must be 16-byte aligned");
    }
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    double *partial = static_cast<double *>(workspace);
    int64_t parts = 0;
    const int64_t bytes = bytes_of(n_tensors, counts, dtypes);
    (void)hipGetLastError();
    for_launches(n_tensors, grads, nullptr, counts, dtypes, [&](const Tensors &t, int blocks) {
        if (blocks > 0)
            hipLaunchKernelGGL(bytes > kFarLoads ? norm_part_kernel<true> : norm_part_kernel<false>, dim3(unsigned(blocks)), dim3(kThreads), 0, s, t, partial + parts);
        parts += blocks;
    });
    hipLaunchKernelGGL(norm_join_kernel, dim3(1), dim3(kJoin), 0, s, partial, parts, norm);
    return launched("gradient norm");
}

int tree_ens_grad_clip(void *stream, int64_t n_tensors, const void *const *grads, const int64_t *counts,
                       const int32_t *dtypes, const float *norm, float max_norm, float eps, void *const *out) {
    treeens::clear_error();
    if (int rc = check_tensors(n_tensors, grads, counts, dtypes))
        return rc;
    if (!(max_norm >= 0.0f) || !std::isfinite(max_norm) || !(eps >= 0.0f) || !std::isfinite(eps))
        return set_error(TREE_ENS_E_ARG, "max_norm and eps must be finite and >= 0");
    if (n_tensors == 0)
        return TREE_ENS_OK;
    if (!norm || !out)
        return set_error(TREE_ENS_E_ARG, "norm or out is NULL");
    if (misaligned(norm, 4))
        return set_error(TREE_ENS_E_ARG, "norm is misaligned");
    for (int64_t i = 0; i < n_tensors; ++i) {
        if (counts[i] > 0 && !out[i])
            return set_error(TREE_ENS_E_ARG, "a tensor of out with elements is NULL");
        if (misaligned(out[i], unsigned(size_of(dtypes[i]))))
            return set_error(TREE_ENS_E_ARG, "a tensor of out is misaligned for its type");
    }
    try {
        if (overlapping(n_tensors, grads, out, counts, dtypes, norm))
            return set_error(TREE_ENS_E_ARG, "a tensor of out overlaps another tensor or the norm");
    } catch (const std::bad_alloc &) {
        return set_error(TREE_ENS_E_NOMEM, "no host memory for the tensors' places");
    }
    const int64_t bytes = bytes_of(n_tensors, counts, dtypes);
    (void)hipGetLastError();
    for_launches(n_tensors, grads, out, counts, dtypes, [&](const Tensors &t, int blocks) {
        if (blocks > 0)
            hipLaunchKernelGGL((bytes > kFarLoads ? clip_kernel<true, true> : bytes > kFarStores ? clip_kernel<false, true> : clip_kernel<false, false>),
                               dim3(unsigned(blocks)), dim3(kThreads), 0, reinterpret_cast<hipStream_t>(stream), t,
                               norm, max_norm, eps);
    });
    return launched("gradient clipping");
}

} // extern "C"
