// Norm of many gradient tensors together, and clipping by it.
//
// sum g^2 reads every item once; scaling reads and writes every item once.  Both are bound by memory (218 tensors, 2.7 GB bf16: squares 443 us,
// 6.1 TB/s; scaling 940 us, 5.7 TB/s, where a 1 GiB copy reaches 5.1 to 5.5), a small network's by two launches.  Squares and their sum
// are double: a square of an fp32 or bf16 item leaves the range of fp32 at both ends.  The tensors' addresses and sizes
// travel in the kernels' arguments, as many as fit into one launch at a time, so that nothing is staged.
#include "cham_device.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kThreads = 512;
constexpr int kPieces = 4;                 // of 16 bytes that a thread asks for at a time
constexpr int kChunkBytes = kThreads * kPieces * 16;
// Tensors of a launch: 4 KiB of arguments.  A launch more is 4 us of host time (191 small tensors in two and two launches 21.6 us, in one and two 16).
constexpr int kMostRead = 280, kMostScaled = 180;
constexpr int kFewTensors = 12;            // of a launch with a tenth of that to write and to copy (a call of six tensors: 10.9 -> 10.4 us)
constexpr int kBlocks = 1024;              // workgroups that sum squares, of all launches of a call together (what is on the chip at a time), one each at least
constexpr int kMostBlocks = 1 << 20;       // of a launch: 2^32 threads are refused (32 GiB of chunks; beyond, a workgroup takes several)

template <int MOST, bool OUT>
struct Tensors {
    const void *from[MOST];
    void *to[OUT ? MOST : 1];              // OUT: where the scaled items go
    int first[MOST + 1];                   // chunk at which a tensor begins
    uint16_t tail[MOST];                   // items of a tensor's last chunk less one, times four; and its type
    int n;
};
static_assert(kChunkBytes / 2 <= 1 << 14, "a chunk's items less one in fourteen bits");
static_assert(sizeof(Tensors<kMostRead, false>) <= 4000 && sizeof(Tensors<kMostScaled, true>) <= 4000, "arguments within 4 KiB, with what goes beside them");

// Tensor of a chunk.
template <int MOST, bool OUT>
__device__ __forceinline__ int tensor_of(const Tensors<MOST, OUT> &t, int chunk)
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

// A chunk's 16-byte pieces may begin at any item: the hardware takes that, and no sum depends on where a tensor lies.
template <typename T>
__device__ __forceinline__ uint4 piece(const typename T::item *p, int i)
{
    const typename T::words w = *reinterpret_cast<const typename T::words *>(p + i * T::kVec);
    return make_uint4(w.x, w.y, w.z, w.w);
}

template <typename T>
__device__ __forceinline__ void add_squares(const uint4 &raw, double (&s)[4])
{
    float x[T::kVec];
    T::unpack(raw, x);
#pragma unroll
    for (int j = 0; j < T::kVec; ++j) s[j % 4] = __builtin_fma((double)x[j], (double)x[j], s[j % 4]);
}

template <typename T>
__device__ __forceinline__ void chunk_squares(const void *from, int n, double (&s)[4])
{
    const typename T::item *p = static_cast<const typename T::item *>(from);
    const int tid = threadIdx.x, n_vec = n / T::kVec;
    uint4 held[kPieces];
    if (n_vec == kThreads * kPieces) {
#pragma unroll
        for (int k = 0; k < kPieces; ++k) held[k] = piece<T>(p, tid + k * kThreads);
#pragma unroll
        for (int k = 0; k < kPieces; ++k) add_squares<T>(held[k], s);
        return;
    }
#pragma unroll
    for (int k = 0; k < kPieces; ++k) {
        held[k] = make_uint4(0, 0, 0, 0);
        if (tid + k * kThreads < n_vec) held[k] = piece<T>(p, tid + k * kThreads);
    }
    double x = 0.0;
    if (tid < n - n_vec * T::kVec) x = (double)T::get(p[n_vec * T::kVec + tid]);
#pragma unroll
    for (int k = 0; k < kPieces; ++k) add_squares<T>(held[k], s);
    s[0] = __builtin_fma(x, x, s[0]);
}

// The chunks [lo, hi) of a block: consecutive ones, so that a tensor is looked up once and then followed.
template <int MOST, bool OUT>
__device__ __forceinline__ void share_of(const Tensors<MOST, OUT> &t, int &lo, int &hi)
{
    const int64_t n = t.first[t.n];
    lo = (int)(n * blockIdx.x / gridDim.x);
    hi = (int)(n * (blockIdx.x + 1) / gridDim.x);
}

struct Chunk {
    int64_t at;                            // first item
    int n, type;
};
template <int MOST, bool OUT>
__device__ __forceinline__ Chunk chunk_of(const Tensors<MOST, OUT> &t, int tensor, int chunk)
{
    const int tail = t.tail[tensor], type = tail & 3, items = kChunkBytes / (type == 0 ? 4 : 2);
    return {(int64_t)(chunk - t.first[tensor]) * items, chunk + 1 == t.first[tensor + 1] ? (tail >> 2) + 1 : items, type};
}

template <int MOST>
__global__ void __launch_bounds__(kThreads, 8) grad_squares_kernel(const Tensors<MOST, false> t, double *parts)
{
    double s[4] = {};
    int lo, hi;
    share_of(t, lo, hi);
    for (int c = lo, i = tensor_of(t, lo); c < hi; ++c) {
        while (c >= t.first[i + 1]) ++i;
        const Chunk k = chunk_of(t, i, c);
        if (k.type == 0) chunk_squares<F32>(static_cast<const float *>(t.from[i]) + k.at, k.n, s);
        else if (k.type == 1) chunk_squares<BF16>(static_cast<const __bf16 *>(t.from[i]) + k.at, k.n, s);
        else chunk_squares<F16>(static_cast<const _Float16 *>(t.from[i]) + k.at, k.n, s);
    }
    const double sum = block_sum((s[0] + s[1]) + (s[2] + s[3]));
    if (threadIdx.x == 0) parts[blockIdx.x] = sum;
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
__device__ __forceinline__ void scale_piece(typename T::item *q, int i, const uint4 &raw, float f)
{
    float x[T::kVec];
    T::unpack(raw, x);
#pragma unroll
    for (int j = 0; j < T::kVec; ++j) x[j] *= f;
    const uint4 v = T::pack(x);
    const typename T::words w = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(w, reinterpret_cast<typename T::words *>(q + i * T::kVec));
}
// Products by the factor f: in fp32, or, where that has no normal number for it, in double, an item at a time (the code of pieces for both cost
// small lists 3 %, a choice in every piece large ones 1 %).
template <typename T>
__device__ __forceinline__ void chunk_scale(const void *from, void *to, const Chunk &c, double f, bool far)
{
    const typename T::item *p = static_cast<const typename T::item *>(from) + c.at;
    typename T::item *q = static_cast<typename T::item *>(to) + c.at;
    const int tid = threadIdx.x, n_vec = c.n / T::kVec, at = n_vec * T::kVec + tid;
    if (far) {
#pragma unroll 1
        for (int i = tid; i < c.n; i += kThreads) q[i] = T::put((float)((double)T::get(p[i]) * f));
        return;
    }
    uint4 held[kPieces];
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        if (tid + k * kThreads < n_vec) held[k] = piece<T>(p, tid + k * kThreads);
    typename T::item last{};
    if (at < c.n) last = p[at];
#pragma unroll
    for (int k = 0; k < kPieces; ++k)
        if (tid + k * kThreads < n_vec) scale_piece<T>(q, tid + k * kThreads, held[k], (float)f);
    if (at < c.n) q[at] = T::put(T::get(last) * (float)f);
}

// parts: the sums of squares of this call (block 0 of the first launch notes the norm); null: *norm is given.
template <int MOST>
__global__ void __launch_bounds__(kThreads, 8) grad_clip_kernel(const Tensors<MOST, true> t, double max_norm, const double *parts, int n_parts, double *norm, int first)
{
    double v;
    if (parts) {
        v = norm_of(parts, n_parts);
        if (first && blockIdx.x == 0 && threadIdx.x == 0) *norm = v;
    } else {
        v = *norm;
    }
    const bool whole = v + 1e-6 <= max_norm;
    const double f = whole ? 1.0 : max_norm / (v + 1e-6);
    const bool far = f < 0x1p-126 && f > 0.0;
    int lo, hi;
    share_of(t, lo, hi);
    // from the last chunk to the first: what the sum of squares has read last is still in cache
    for (int c = hi - 1, i = lo < hi ? tensor_of(t, hi - 1) : 0; c >= lo; --c) {
        while (c < t.first[i]) --i;
        if (whole && t.from[i] == t.to[i]) continue;
        const Chunk k = chunk_of(t, i, c);
        if (k.type == 0) chunk_scale<F32>(t.from[i], t.to[i], k, f, far);
        else if (k.type == 1) chunk_scale<BF16>(t.from[i], t.to[i], k, f, far);
        else chunk_scale<F16>(t.from[i], t.to[i], k, f, far);
    }
}

// Items of a chunk are a power of two: no division for each of many tensors.
constexpr int shift_of(int type) { return type == 0 ? 13 : 14; }
static_assert(kChunkBytes == 4 << shift_of(0) && kChunkBytes == 2 << shift_of(1), "items of a chunk");
int64_t chunks_in(int64_t numel, int type) { return (numel + (int64_t(1) << shift_of(type)) - 1) >> shift_of(type); }

// The tensors from `i` on that go into one launch (empty ones left out); returns the first that does not.
template <int MOST, bool OUT>
int gather(Tensors<MOST, OUT> &t, int i, const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n)
{
    t.n = 0;
    t.first[0] = 0;
    for (; i < n && t.n < MOST; ++i) {
        if (numels[i] == 0) continue;
        t.from[t.n] = grads ? grads[i] : nullptr;
        if (OUT) t.to[t.n] = outs ? outs[i] : const_cast<void *>(grads[i]);
        const int64_t end = t.first[t.n] + chunks_in(numels[i], types[i]);
        t.tail[t.n] = (uint16_t)(((numels[i] - 1) & ((int64_t(1) << shift_of(types[i])) - 1)) * 4 + types[i]);
        t.first[++t.n] = (int)end;                 // of 2^40 items at most: below 2^28
    }
    return i;
}

int64_t chunks_of(const int64_t *numels, const int32_t *types, int n)
{
    int64_t c = 0;
    for (int i = 0; i < n; ++i) c += chunks_in(numels[i], types[i]);
    return c;
}

// Workgroups of a launch: one a chunk, or its share of kBlocks, with consecutive chunks each.
template <int MOST, bool OUT>
int blocks_of(const Tensors<MOST, OUT> &t, int64_t all_chunks)
{
    const int64_t c = t.first[t.n];
    if (all_chunks <= kBlocks || c == 0) return (int)c;
    const int64_t share = c * kBlocks / all_chunks;
    return share > 0 ? (int)share : 1;
}

template <int MOST>
int parts_of(const int64_t *numels, const int32_t *types, int n)
{
    Tensors<MOST, false> t;
    const int64_t all = chunks_of(numels, types, n);
    int parts = 0;
    for (int i = 0; i < n;) {
        i = gather(t, i, nullptr, nullptr, numels, types, n);
        parts += blocks_of(t, all);
    }
    return parts;
}

template <int MOST>
void launch_squares(const void *const *grads, const int64_t *numels, const int32_t *types, int n, double *parts, hipStream_t s)
{
    Tensors<MOST, false> t;
    const int64_t all = chunks_of(numels, types, n);
    int at = 0;
    for (int i = 0; i < n;) {
        i = gather(t, i, grads, nullptr, numels, types, n);
        if (t.n == 0) break;
        const int blocks = blocks_of(t, all);
        hipLaunchKernelGGL(grad_squares_kernel<MOST>, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, parts + at);
        at += blocks;
    }
}

template <int MOST>
void launch_scale(const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n, double max_norm, double *norm,
                  const double *parts, int n_parts, hipStream_t s)
{
    Tensors<MOST, true> t;
    const int64_t all = chunks_of(numels, types, n);
    int first = 1;
    // the last tensors first, as the chunks within a launch
    for (int end = n; end > 0;) {
        int begin = end;
        for (int most = MOST; begin > 0 && most > 0; --begin) most -= numels[begin - 1] != 0;
        gather(t, begin, grads, outs, numels, types, end);
        end = begin;
        if (t.n == 0) break;
        // Many chunks: a workgroup each, so that the chip walks through memory in order (us a call, spans of kBlocks / one each: 2.7 GB
        // 1580 / 1383, 640 MB 352 / 300, 150 MB 83 / 80).  80 MB, which the caches hold, 41 / 45: the end of a span is still there.
        const int chunks = t.first[t.n], blocks = all <= 4 * kBlocks ? blocks_of(t, all) : chunks < kMostBlocks ? chunks : kMostBlocks;
        hipLaunchKernelGGL(grad_clip_kernel<MOST>, dim3((unsigned)blocks), dim3(kThreads), 0, s, t, max_norm, parts, n_parts, norm, first);
        first = 0;
    }
}

}  // namespace

int grad_parts(const int64_t *numels, const int32_t *types, int n)
{
    return n <= kFewTensors ? parts_of<kFewTensors>(numels, types, n) : parts_of<kMostRead>(numels, types, n);
}

hipError_t launch_grad_norm(const void *const *grads, const int64_t *numels, const int32_t *types, int n, double *parts, int n_parts,
                            double *norm, hipStream_t s)
{
    if (n <= kFewTensors) launch_squares<kFewTensors>(grads, numels, types, n, parts, s);
    else launch_squares<kMostRead>(grads, numels, types, n, parts, s);
    if (norm) hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(kThreads), 0, s, parts, n_parts, norm);
    return hipGetLastError();
}

hipError_t launch_grad_clip(const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n,
                            double max_norm, double *norm, const double *parts, int n_parts, hipStream_t s)
{
    if (n <= kFewTensors) launch_scale<kFewTensors>(grads, outs, numels, types, n, max_norm, norm, parts, n_parts, s);
    else launch_scale<kMostScaled>(grads, outs, numels, types, n, max_norm, norm, parts, n_parts, s);
    return hipGetLastError();
}

}  // namespace cham
