// Norm of many gradient tensors together, and clipping by it.
//
// sum g^2 reads every item once; scaling reads and writes every item once.  Both are bound by memory.  Squares and their sum
// are double: a square of an fp32 or bf16 item leaves the range of fp32 at both ends.  The tensors' addresses and sizes
// travel in the kernels' arguments, as many as fit into one launch at a time, so that nothing is staged.
#include "cham_device.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kThreads = 256;
constexpr int kChunk = 1 << 14;            // items of a chunk: a workgroup takes one at a time
constexpr int kMostTensors = 120;          // of a launch: 4 KiB of arguments
constexpr int kBlocks = 1024;              // workgroups of all launches of a call together, but one each at least

struct Tensors {
    const void *from[kMostTensors];
    void *to[kMostTensors];
    int64_t numel[kMostTensors];
    int first[kMostTensors + 1];           // chunk at which a tensor begins
    uint8_t type[kMostTensors];
    int n;
};
static_assert(sizeof(Tensors) <= 4000, "arguments within 4 KiB, with what goes beside them");

// Tensor of a chunk.
__device__ __forceinline__ int tensor_of(const Tensors &t, int chunk)
{
    int lo = 0, hi = t.n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (t.first[mid] <= chunk) lo = mid;
        else hi = mid;
    }
    return lo;
}

// Total of a block's doubles, in every thread.
__device__ __forceinline__ double block_sum(double v)
{
    __shared__ double lds[kThreads / 64];
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    double s = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) s += lds[w];
    return s;
}

template <typename T>
__device__ __forceinline__ double chunk_squares(const void *from, int n)
{
    const typename T::item *p = static_cast<const typename T::item *>(from);
    const int head = (int)items_to_boundary<T>(p, n), n_vec = (n - head) / T::kVec, tail = head + n_vec * T::kVec;
    const uint4 *body = reinterpret_cast<const uint4 *>(p + head);
    double s = 0.0;
    if ((int)threadIdx.x < head) {
        const double x = (double)T::get(p[threadIdx.x]);
        s += x * x;
    }
    if ((int)threadIdx.x < n - tail) {
        const double x = (double)T::get(p[tail + threadIdx.x]);
        s += x * x;
    }
    for (int i = threadIdx.x; i < n_vec; i += kThreads) {
        float x[T::kVec];
        T::unpack(body[i], x);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) s = __builtin_fma((double)x[j], (double)x[j], s);
    }
    return s;
}

__global__ void __launch_bounds__(kThreads) grad_squares_kernel(const Tensors t, double *parts)
{
    double s = 0.0;
    for (int c = (int)blockIdx.x; c < t.first[t.n]; c += (int)gridDim.x) {
        const int i = tensor_of(t, c);
        const int64_t at = (int64_t)(c - t.first[i]) * kChunk;
        const int64_t left = t.numel[i] - at;
        const int n = left < kChunk ? (int)left : kChunk;
        if (t.type[i] == 0) s += chunk_squares<F32>(static_cast<const float *>(t.from[i]) + at, n);
        else if (t.type[i] == 1) s += chunk_squares<BF16>(static_cast<const __bf16 *>(t.from[i]) + at, n);
        else s += chunk_squares<F16>(static_cast<const _Float16 *>(t.from[i]) + at, n);
    }
    s = block_sum(s);
    if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__device__ __forceinline__ double norm_of(const double *parts, int n_parts)
{
    double s = 0.0;
    for (int i = threadIdx.x; i < n_parts; i += kThreads) s += parts[i];
    return sqrt(block_sum(s));
}

__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const double *parts, int n_parts, double *norm)
{
    const double v = norm_of(parts, n_parts);
    if (threadIdx.x == 0) *norm = v;
}

template <typename T>
__device__ __forceinline__ void chunk_scale(const void *from, void *to, int n, float f)
{
    const typename T::item *p = static_cast<const typename T::item *>(from);
    typename T::item *q = static_cast<typename T::item *>(to);
    if (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(q)) & 15) != 0) {      // boundaries at different items
        for (int i = threadIdx.x; i < n; i += kThreads) q[i] = T::put(T::get(p[i]) * f);
        return;
    }
    const int head = (int)items_to_boundary<T>(p, n), n_vec = (n - head) / T::kVec, tail = head + n_vec * T::kVec;
    const uint4 *body = reinterpret_cast<const uint4 *>(p + head);
    uint4 *out = reinterpret_cast<uint4 *>(q + head);
    if ((int)threadIdx.x < head) q[threadIdx.x] = T::put(T::get(p[threadIdx.x]) * f);
    if ((int)threadIdx.x < n - tail) q[tail + threadIdx.x] = T::put(T::get(p[tail + threadIdx.x]) * f);
    for (int i = threadIdx.x; i < n_vec; i += kThreads) {
        float x[T::kVec];
        T::unpack(body[i], x);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) x[j] *= f;
        out[i] = T::pack(x);
    }
}

// parts: the sums of squares of this call (block 0 of the first launch notes the norm); null: *norm is given.
__global__ void __launch_bounds__(kThreads) grad_clip_kernel(const Tensors t, double max_norm, const double *parts, int n_parts, double *norm, int first)
{
    double v;
    if (parts) {
        v = norm_of(parts, n_parts);
        if (first && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    } else {
        v = *norm;
    }
    const bool whole = v + 1e-6 <= max_norm;
    const float f = whole ? 1.0f : (float)(max_norm / (v + 1e-6));
    // from the last chunk to the first: what the sum of squares has read last is still in cache
    for (int c = t.first[t.n] - 1 - (int)blockIdx.x; c >= 0; c -= (int)gridDim.x) {
        const int i = tensor_of(t, c);
        if (whole && t.from[i] == t.to[i]) continue;
        const int64_t at = (int64_t)(c - t.first[i]) * kChunk;
        const int64_t left = t.numel[i] - at;
        const int n = left < kChunk ? (int)left : kChunk;
        if (t.type[i] == 0) chunk_scale<F32>(static_cast<const float *>(t.from[i]) + at, static_cast<float *>(t.to[i]) + at, n, f);
        else if (t.type[i] == 1) chunk_scale<BF16>(static_cast<const __bf16 *>(t.from[i]) + at, static_cast<__bf16 *>(t.to[i]) + at, n, f);
        else chunk_scale<F16>(static_cast<const _Float16 *>(t.from[i]) + at, static_cast<_Float16 *>(t.to[i]) + at, n, f);
    }
}

// The tensors from `i` on that go into one launch (empty ones left out); returns the first that does not.
int gather(Tensors &t, int i, const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n)
{
    t.n = 0;
    t.first[0] = 0;
    for (; i < n && t.n < kMostTensors; ++i) {
        if (numels[i] == 0) continue;
        t.from[t.n] = grads ? grads[i] : nullptr;
        t.to[t.n] = outs ? outs[i] : const_cast<void *>(t.from[t.n]);
        t.numel[t.n] = numels[i];
        t.type[t.n] = (uint8_t)types[i];
        const int64_t end = t.first[t.n] + (numels[i] + kChunk - 1) / kChunk;
        t.first[++t.n] = (int)end;                 // at most 2^40 / kChunk + kMostTensors chunks: below 2^31
    }
    return i;
}

int64_t chunks_of(const int64_t *numels, int n)
{
    int64_t c = 0;
    for (int i = 0; i < n; ++i) c += (numels[i] + kChunk - 1) / kChunk;
    return c;
}

// Workgroups of a launch: one a chunk, or its share of kBlocks.
int blocks_of(const Tensors &t, int64_t all_chunks)
{
    const int64_t c = t.first[t.n];
    if (all_chunks <= kBlocks || c == 0) return (int)c;
    const int64_t share = c * kBlocks / all_chunks;
    return share > 0 ? (int)share : 1;
}

}  // namespace

int grad_parts(const int64_t *numels, const int32_t *types, int n)
{
    Tensors t;
    const int64_t all = chunks_of(numels, n);
    int parts = 0;
    for (int i = 0; i < n;) {
        i = gather(t, i, nullptr, nullptr, numels, types, n);
        parts += blocks_of(t, all);
    }
    return parts;
}

hipError_t launch_grad_norm(const void *const *grads, const int64_t *numels, const int32_t *types, int n, double *parts, int n_parts,
                            double *norm, hipStream_t s)
{
    Tensors t;
    const int64_t all = chunks_of(numels, n);
    int at = 0;
    for (int i = 0; i < n;) {
        i = gather(t, i, grads, nullptr, numels, types, n);
        if (t.n == 0) break;
        const int blocks = blocks_of(t, all);
        hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, parts + at);
        at += blocks;
    }
    if (norm) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, s, parts, n_parts, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n,
                            double max_norm, double *norm, const double *parts, int n_parts, hipStream_t s)
{
    Tensors t;
    const int64_t all = chunks_of(numels, n);
    int first = 1;
    for (int i = 0; i < n;) {
        i = gather(t, i, grads, outs, numels, types, n);
        if (t.n == 0) break;
        hipLaunchKernelGGL(grad_clip_kernel, dim3((unsigned)blocks_of(t, all)), dim3(kThreads), 0, s, t, max_norm, parts, n_parts, norm, first);
        first = 0;
    }
    return hipGetLastError();
}

}  // namespace cham
