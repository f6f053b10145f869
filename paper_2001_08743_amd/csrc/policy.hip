// Log-probabilities of actions and the clipped policy loss with its gradients (Sec. 3.4: the exploration agent is trained
// with clipped policy updates).
//
// Per head of V logits x:  m = max x, s = sum e^(x-m), t = sum e^(x-m) (x-m);  log p_v = x_v - m - log s,
// H = log s - t / s.  Per decision, lp = sum over heads of log p_action, and with ratio rho = e^(lp - old)
//   L = w (-min(rho A, clip(rho) A) + c_v value - c_H H + c_kl (e^d - d - 1)),   d = ref - lp
//   dL/dlp = D = w (-rho A [unclipped side] + c_kl (1 - e^d)),   dL/dx_v = D ([v = a] - p_v) + w c_H p_v (log p_v + H).
// Exponentials and their sums are fp32 (logits have at most 24 bits), everything per decision double.
#include "cham_device.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kThreads = 256;
constexpr float kLowest = -3.402823466e38f;     // maximum of nothing: finite, so that -inf - kLowest is not a NaN
constexpr float kFar = -200.0f;                 // e^x is 0 in fp32 below; keeps 0 * (-inf) out of the sums

__device__ __forceinline__ float exp_fast(float z) { return __builtin_amdgcn_exp2f(z * 1.44269504f); }

// Running maximum and sums of a head.
struct Soft {
    float m, s, t;
};
__device__ __forceinline__ Soft soft_none() { return {kLowest, 0.0f, 0.0f}; }
// A NaN in x does not reach m (the maximum passes it by) but s, by its exponential.
__device__ __forceinline__ void soft_raise(Soft &a, float m)
{
    if (m > a.m) {
        const float d = a.m - m, f = exp_fast(d);
        a.t = f > 0.0f ? f * (a.t + a.s * d) : 0.0f;
        a.s *= f;
        a.m = m;
    }
}
__device__ __forceinline__ void soft_add(Soft &a, float x)
{
    const float z = x - a.m, e = exp_fast(z);
    a.s += e;
    a.t += e * fmaxf(z, kFar);
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b)
{
    const float m = fmaxf(a.m, b.m);
    soft_raise(a, m);
    soft_raise(b, m);
    return {m, a.s + b.s, a.t + b.t};
}
__device__ __forceinline__ Soft soft_wave(Soft a)
{
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) a = soft_join(a, {__shfl_xor(a.m, o), __shfl_xor(a.s, o), __shfl_xor(a.t, o)});
    return a;
}

// Choice of an action: -1 = its head is left out, V = outside the choices.
__device__ __forceinline__ int choice_of(const PolicyArgs &a, int64_t i)
{
    const int64_t x = a.abytes == 1   ? (int64_t)static_cast<const int8_t *>(a.actions)[i]
                      : a.abytes == 4 ? (int64_t)static_cast<const int32_t *>(a.actions)[i]
                                      : static_cast<const int64_t *>(a.actions)[i];
    if (x < a.first) return -1;
    const uint64_t c = (uint64_t)x - (uint64_t)a.first;
    return c < (uint64_t)a.V ? (int)c : a.V;
}

__device__ __forceinline__ bool counts(const PolicyArgs &a, int64_t r) { return !a.weights || a.weights[r] != 0.0f; }

// One decision: writes its outputs, adds its terms, returns (D, w c_H).
__device__ __forceinline__ float2 decide(const PolicyArgs &a, int64_t r, bool in, double lp, double H, double (&sum)[kPolicySums])
{
    if (a.logp) a.logp[r] = in ? (float)lp : 0.0f;
    if (a.entropy) a.entropy[r] = in ? (float)H : 0.0f;
    if (!a.old_logp) return make_float2(0.0f, 0.0f);
    if (!in) {
        if (a.grad_values) a.grad_values[r] = 0.0f;
        return make_float2(0.0f, 0.0f);
    }
    const double w = a.weights ? (double)a.weights[r] : a.w_all;
    const double A = (double)a.adv[r];
    const double rho = exp(lp - (double)a.old_logp[r]);
    const double held_rho = rho < a.lo ? a.lo : rho > a.hi ? a.hi : rho;
    const double free = rho * A, held = held_rho * A;
    const bool clipped = free > held;
    sum[0] -= w * (clipped ? held : free);
    double D = clipped ? 0.0 : -free;
    if (a.values) {
        const double v = (double)a.values[r], ret = (double)a.returns[r];
        const double near = (v - ret) * (v - ret);
        double kept = near;
        if (a.old_values) {
            const double o = (double)a.old_values[r], d = v - o;
            const double k = o + (d < -a.value_clip ? -a.value_clip : d > a.value_clip ? a.value_clip : d) - ret;
            kept = k * k;
        }
        sum[1] += w * 0.5 * (near < kept ? kept : near);
        if (a.grad_values) a.grad_values[r] = near < kept || a.c_value == 0.0 ? 0.0f : (float)(w * a.c_value * (v - ret));
    } else if (a.grad_values) {
        a.grad_values[r] = 0.0f;
    }
    sum[2] += w * H;
    if (a.ref) {
        const double d = (double)a.ref[r] - lp, e = expm1(d);
        sum[3] += w * (e < __builtin_inf() ? e - d : e);      // an action that the policy has lost: infinite, not inf - inf
        if (a.c_kl != 0.0) D -= a.c_kl * e;
    }
    if (clipped) sum[4] += w;
    return make_float2((float)(w * D), (float)(w * a.c_entropy));
}

// Sums of the waves of a block into the block's place; blocks are joined by policy_terms_kernel.
template <int WAVES>
__device__ __forceinline__ void store_sums(const PolicyArgs &a, const double (&sum)[kPolicySums])
{
    __shared__ double lds[WAVES][kPolicySums];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        const double v = wave_sum(sum[i]);
        if (lane == 0) lds[wave][i] = v;
    }
    __syncthreads();
    if (threadIdx.x < kPolicySums) {
        double v = 0.0;
        for (int w = 0; w < WAVES; ++w) v += lds[w][threadIdx.x];
        a.sums[(int64_t)blockIdx.x * kPolicySums + threadIdx.x] = v;
    }
}

// Terms from the blocks' sums, in a fixed order.  Zeros where there are no blocks.
__global__ void __launch_bounds__(kThreads) policy_terms_kernel(const PolicyArgs a, int blocks)
{
    __shared__ double lds[kThreads / 64][kPolicySums];
    double v[kPolicySums] = {};
    for (int b = threadIdx.x; b < blocks; b += kThreads)
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) v[i] += a.sums[(int64_t)b * kPolicySums + i];
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        v[i] = wave_sum(v[i]);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6][i] = v[i];
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPolicySums; ++i) {
            v[i] = 0.0;
            for (int w = 0; w < kThreads / 64; ++w) v[i] += lds[w][i];
            a.terms[1 + i] = (float)v[i];
        }
        double total = v[0];
        if (a.c_value != 0.0) total += a.c_value * v[1];
        if (a.c_entropy != 0.0) total -= a.c_entropy * v[2];
        if (a.c_kl != 0.0) total += a.c_kl * v[3];
        a.terms[0] = (float)total;
    }
}

// --- few choices a head: a workgroup takes whole decisions, a thread whole heads

constexpr int kTileHeads = 1024;                // at most: kHeadsPerThread of each thread
constexpr int kHeadsPerThread = kTileHeads / kThreads;
constexpr int kTileItems = 8448;                // fp32 logits in LDS, 33 KiB: four workgroups share a compute unit
constexpr int kTileChoices = 32;                // beyond, a tile has fewer heads than threads

struct TileShape {
    int per_tile;           // decisions of a tile
    int stride;             // of a head's logits in LDS: odd, so that the threads of a wave read different banks
    unsigned inv_v, inv_gv; // ceil(2^32 / V), ceil(2^32 / (G V)): quotients of item numbers below 2^16
    int dense;              // the logits of a tile are one run of items
    int gdense;             // its gradients are
};

__device__ __forceinline__ int quotient(int i, unsigned inv, int by) { return by == 1 ? i : (int)__umulhi((unsigned)i, inv); }

// Items of a run of n at p, f(index, value), 16 bytes at a time.
template <typename T, typename F>
__device__ __forceinline__ void read_run(const typename T::item *p, int n, F &&f)
{
    const int head = (int)items_to_boundary<T>(p, n), n_vec = (n - head) / T::kVec, tail = head + n_vec * T::kVec;
    if ((int)threadIdx.x < head) f((int)threadIdx.x, T::get(p[threadIdx.x]));
    if ((int)threadIdx.x < n - tail) f(tail + (int)threadIdx.x, T::get(p[tail + threadIdx.x]));
    const uint4 *body = reinterpret_cast<const uint4 *>(p + head);
    for (int i = threadIdx.x; i < n_vec; i += kThreads) {
        float x[T::kVec];
        T::unpack(body[i], x);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) f(head + i * T::kVec + j, x[j]);
    }
}
template <typename T, typename F>
__device__ __forceinline__ void write_run(typename T::item *p, int n, F &&f)
{
    const int head = (int)items_to_boundary<T>(p, n), n_vec = (n - head) / T::kVec, tail = head + n_vec * T::kVec;
    if ((int)threadIdx.x < head) p[threadIdx.x] = T::put(f((int)threadIdx.x));
    if ((int)threadIdx.x < n - tail) p[tail + threadIdx.x] = T::put(f(tail + (int)threadIdx.x));
    uint4 *body = reinterpret_cast<uint4 *>(p + head);
    for (int i = threadIdx.x; i < n_vec; i += kThreads) {
        float x[T::kVec];
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) x[j] = f(head + i * T::kVec + j);
        body[i] = T::pack(x);
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_tile_kernel(const PolicyArgs a, const TileShape k)
{
    __shared__ float x[kTileItems];
    __shared__ float2 one[kTileHeads];          // log-probability and entropy of a head
    __shared__ float2 dec[kTileHeads];          // of a decision: (D, w c_H)
    __shared__ uint8_t in[kTileHeads];
    const int tid = threadIdx.x;
    const int gv = a.G * a.V;
    double sum[kPolicySums] = {};
    for (int64_t r0 = (int64_t)blockIdx.x * k.per_tile; r0 < a.R; r0 += (int64_t)gridDim.x * k.per_tile) {
        const int nr = a.R - r0 < k.per_tile ? (int)(a.R - r0) : k.per_tile;
        const int heads = nr * a.G, items = nr * gv;
        auto at = [&](int i) {                  // where item i of the tile stands in LDS
            const int h = k.stride == a.V ? 0 : quotient(i, k.inv_v, a.V);
            return i + h;
        };
        auto offset = [&](int i, int64_t ld_r, int64_t ld_g) {
            const int h = quotient(i, k.inv_v, a.V), r = quotient(i, k.inv_gv, gv);
            return (r0 + r) * ld_r + (h - r * a.G) * ld_g + (i - h * a.V);
        };
        const typename T::item *logits = static_cast<const typename T::item *>(a.logits);
        if (k.dense)
            read_run<T>(logits + r0 * gv, items, [&](int i, float v) { x[at(i)] = v; });
        else
            for (int i = tid; i < items; i += kThreads) x[at(i)] = T::get(logits[offset(i, a.ld_r, a.ld_g)]);
        __syncthreads();

        float m[kHeadsPerThread], ls[kHeadsPerThread], ent[kHeadsPerThread];
        int c[kHeadsPerThread];
#pragma unroll
        for (int u = 0; u < kHeadsPerThread; ++u) {
            const int h = tid + u * kThreads;
            m[u] = ls[u] = ent[u] = 0.0f;
            c[u] = -1;
            if (h >= heads) continue;
            const float *xh = x + h * k.stride;
            c[u] = choice_of(a, r0 * a.G + h);
            float lp = 0.0f;
            if (c[u] == a.V) {
                c[u] = 0;
                ls[u] = ent[u] = lp = __builtin_nanf("");
            } else if (c[u] >= 0) {
                Soft v = soft_none();
                for (int j = 0; j < a.V; ++j) v.m = fmaxf(v.m, xh[j]);
                for (int j = 0; j < a.V; ++j) soft_add(v, xh[j]);
                if (v.s != 0.0f) {
                    m[u] = v.m;
                    ls[u] = logf(v.s);
                    ent[u] = ls[u] - v.t / v.s;
                    lp = xh[c[u]] - v.m - ls[u];
                } else {
                    c[u] = -1;                  // every choice is masked
                }
            }
            one[h] = make_float2(lp, ent[u]);
            in[h] = c[u] >= 0;
        }
        __syncthreads();
        for (int r = tid; r < nr; r += kThreads) {
            double lp = 0.0, H = 0.0;
            bool any = false;
            if (counts(a, r0 + r))
                for (int g = 0; g < a.G; ++g) {
                    const float2 o = one[r * a.G + g];
                    lp += (double)o.x;
                    H += (double)o.y;
                    any = any || in[r * a.G + g] != 0;
                }
            dec[r] = decide(a, r0 + r, any, lp, H, sum);
            if (!any)                           // also of weight 0: zeros, whatever the logits are
                for (int g = 0; g < a.G; ++g) in[r * a.G + g] = 0;
        }
        if (!a.grad) {
            __syncthreads();
            continue;
        }
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kHeadsPerThread; ++u) {
            const int h = tid + u * kThreads;
            if (h >= heads) continue;
            float *xh = x + h * k.stride;
            if (!in[h]) {
                for (int j = 0; j < a.V; ++j) xh[j] = 0.0f;
                continue;
            }
            const float2 d = dec[a.G == 1 ? h : h / a.G];
            for (int j = 0; j < a.V; ++j) {
                const float z = xh[j] - m[u] - ls[u], p = exp_fast(z);
                xh[j] = (j == c[u] ? d.x : 0.0f) - p * (d.x - d.y * (fmaxf(z, kFar) + ent[u]));
            }
        }
        __syncthreads();
        typename T::item *grad = static_cast<typename T::item *>(a.grad);
        if (k.gdense)
            write_run<T>(grad + r0 * gv, items, [&](int i) { return x[at(i)]; });
        else
            for (int i = tid; i < items; i += kThreads) grad[offset(i, a.gld_r, a.gld_g)] = T::put(x[at(i)]);
        __syncthreads();
    }
    if (a.old_logp) store_sums<kThreads / 64>(a, sum);
}

// --- any number of heads and choices, in three steps: sums of parts of heads, decisions, gradient

// Visits the items [lo, hi) of a row, 16 bytes at a time from the first boundary on; f(index, value).
template <typename T, typename F>
__device__ __forceinline__ void for_items(const typename T::item *row, int lo, int hi, F &&f)
{
    const int head = (int)items_to_boundary<T>(row + lo, hi - lo);
    const int n_vec = (hi - lo - head) / T::kVec;
    if ((int)threadIdx.x < head) f(lo + (int)threadIdx.x, T::get(row[lo + threadIdx.x]));
    const uint4 *body = reinterpret_cast<const uint4 *>(row + lo + head);
    for (int i = threadIdx.x; i < n_vec; i += kThreads) {
        float x[T::kVec];
        T::unpack(body[i], x);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) f(lo + head + i * T::kVec + j, x[j]);
    }
    const int tail = lo + head + n_vec * T::kVec;
    if ((int)threadIdx.x < hi - tail) f(tail + (int)threadIdx.x, T::get(row[tail + threadIdx.x]));
}

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_part_kernel(const PolicyArgs a, int splits, int chunk)
{
    __shared__ Soft lds[kThreads / 64];
    const int64_t units = a.R * a.G * splits;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t h = u / splits, r = h / a.G;
        if (!counts(a, r)) continue;
        const int c = choice_of(a, h);
        if (c < 0 || c == a.V) continue;
        const int g = (int)(h - r * a.G), lo = (int)(u - h * splits) * chunk;
        const int hi = lo + chunk < a.V ? lo + chunk : a.V;
        const typename T::item *row = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
        Soft v = soft_none();
        for_items<T>(row, lo, hi, [&](int, float x) {
            soft_raise(v, x);
            soft_add(v, x);
        });
        v = soft_wave(v);
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kThreads / 64; ++w) v = soft_join(v, lds[w]);
            reinterpret_cast<float4 *>(a.part)[u] = make_float4(v.m, v.s, v.t, 0.0f);
        }
        __syncthreads();
    }
}

// A wave per decision: its heads one after the other, the parts of a head over the lanes.
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_join_kernel(const PolicyArgs a, int splits)
{
    const int lane = threadIdx.x & 63;
    double sum[kPolicySums] = {};
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6); r < a.R; r += (int64_t)gridDim.x * (kThreads / 64)) {
        double lp = 0.0, H = 0.0;
        bool in = false;
        if (counts(a, r)) {
            for (int g = 0; g < a.G; ++g) {
                const int64_t h = r * a.G + g;
                const int c = choice_of(a, h);
                float4 out = make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
                if (c == a.V) {
                    lp = H = __builtin_nan("");
                    out = make_float4(0.0f, __builtin_nanf(""), 0.0f, __int_as_float(0));
                    in = true;
                } else if (c >= 0) {
                    Soft v = soft_none();
                    for (int i = lane; i < splits; i += 64) {
                        const float4 p = reinterpret_cast<const float4 *>(a.part)[h * splits + i];
                        v = soft_join(v, {p.x, p.y, p.z});
                    }
                    v = soft_wave(v);
                    if (v.s != 0.0f) {                     // 0: every choice is masked
                        const float ls = logf(v.s), e = ls - v.t / v.s;
                        const float x = T::get(static_cast<const typename T::item *>(a.logits)[r * a.ld_r + g * a.ld_g + c]);
                        lp += (double)x - (double)v.m - (double)ls;
                        H += (double)e;
                        out = make_float4(v.m, ls, e, __int_as_float(c));
                        in = true;
                    }
                }
                if (a.grad && lane == 0) a.head[h] = out;
            }
        }
        if (lane == 0) {
            const float2 d = decide(a, r, in, lp, H, sum);
            if (a.grad) a.dec[r] = d;
        }
    }
    if (a.old_logp) store_sums<kThreads / 64>(a, sum);
}

template <typename T>
__global__ void __launch_bounds__(kThreads) policy_grad_kernel(const PolicyArgs a, int splits, int chunk)
{
    const int64_t units = a.R * a.G * splits;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t h = u / splits, r = h / a.G;
        const int g = (int)(h - r * a.G), lo = (int)(u - h * splits) * chunk;
        const int hi = lo + chunk < a.V ? lo + chunk : a.V;
        typename T::item *to = static_cast<typename T::item *>(a.grad) + r * a.gld_r + g * a.gld_g;
        const float4 k = counts(a, r) ? a.head[h] : make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
        const int c = __float_as_int(k.w);
        if (c < 0) {
            for (int v = lo + threadIdx.x; v < hi; v += kThreads) to[v] = T::put(0.0f);
            continue;
        }
        const float2 d = a.dec[r];
        const typename T::item *row = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
        for_items<T>(row, lo, hi, [&](int v, float x) {
            const float z = x - k.x - k.y, p = exp_fast(z);
            to[v] = T::put((v == c ? d.x : 0.0f) - p * (d.x - d.y * (fmaxf(z, kFar) + k.z)));
        });
    }
}

constexpr int kJoinBlocks = 1024;
constexpr int kTileBlocks = 1024;               // what is on the chip at a time
constexpr unsigned kMostBlocks = 1u << 20;

unsigned blocks_for(int64_t n) { return (unsigned)(n < (int64_t)kMostBlocks ? n : (int64_t)kMostBlocks); }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

template <typename T>
hipError_t launch_typed(PolicyArgs &a, const PolicyPlan &p, hipStream_t s)
{
    if (p.tile) {
        const int gv = a.G * a.V;
        TileShape k;
        k.per_tile = p.tile;
        k.stride = a.V | 1;
        k.inv_v = (unsigned)((((uint64_t)1 << 32) + a.V - 1) / a.V);
        k.inv_gv = (unsigned)((((uint64_t)1 << 32) + gv - 1) / gv);
        k.dense = (a.G == 1 || a.ld_g == a.V) && (a.R == 1 || a.ld_r == gv);
        k.gdense = (a.G == 1 || a.gld_g == a.V) && (a.R == 1 || a.gld_r == gv);
        const int64_t tiles = (a.R + p.tile - 1) / p.tile;
        const unsigned blocks = (unsigned)(tiles < kTileBlocks ? tiles : kTileBlocks);
        if (a.R > 0) hipLaunchKernelGGL(policy_tile_kernel<T>, dim3(blocks), dim3(kThreads), 0, s, a, k);
        if (a.old_logp) hipLaunchKernelGGL(policy_terms_kernel, dim3(1), dim3(kThreads), 0, s, a, (int)blocks);
        return hipGetLastError();
    }
    const int64_t units = a.R * a.G * p.splits;
    const unsigned join = (unsigned)((a.R + 3) / 4 < kJoinBlocks ? (a.R + 3) / 4 : kJoinBlocks);
    if (a.R > 0) {
        hipLaunchKernelGGL(policy_part_kernel<T>, dim3(blocks_for(units)), dim3(kThreads), 0, s, a, p.splits, p.chunk);
        hipLaunchKernelGGL(policy_join_kernel<T>, dim3(join), dim3(kThreads), 0, s, a, p.splits);
        if (a.grad) hipLaunchKernelGGL(policy_grad_kernel<T>, dim3(blocks_for(units)), dim3(kThreads), 0, s, a, p.splits, p.chunk);
    }
    if (a.old_logp) hipLaunchKernelGGL(policy_terms_kernel, dim3(1), dim3(kThreads), 0, s, a, (int)join);
    return hipGetLastError();
}

}  // namespace

PolicyPlan plan_policy(int64_t R, int G, int V, int type, bool grad)
{
    PolicyPlan p{};
    if (V <= kTileChoices && G <= kTileHeads && (int64_t)G * (V | 1) <= kTileItems) {
        const int by_heads = kTileHeads / G, by_items = kTileItems / (G * (V | 1));
        p.tile = by_heads < by_items ? by_heads : by_items;
        p.bytes = (int64_t)kTileBlocks * kPolicySums * 8;
        return p;
    }
    // parts of a head: of at least 4096 choices, until there are 1024 workgroups
    const int64_t heads = R * G;
    int64_t most = ((int64_t)V + 4095) / 4096;
    int64_t want = heads > 0 ? (1024 + heads - 1) / heads : 1;
    int64_t n = want < most ? want : most;
    p.chunk = (int)((((int64_t)V + n - 1) / n + 7) / 8 * 8);
    p.splits = (V + p.chunk - 1) / p.chunk;
    p.o_sums = 0;
    p.o_part = up256((int64_t)kJoinBlocks * kPolicySums * 8);
    p.o_head = p.o_part + up256(heads * p.splits * 16);
    p.o_dec = p.o_head + (grad ? up256(heads * 16) : 0);
    p.bytes = p.o_dec + (grad ? up256(R * 8) : 0);
    return p;
}

hipError_t launch_policy(PolicyArgs a, int type, void *workspace, hipStream_t s)
{
    const PolicyPlan p = plan_policy(a.R, a.G, a.V, type, a.grad != nullptr);
    char *w = static_cast<char *>(workspace);
    a.sums = reinterpret_cast<double *>(w + p.o_sums);
    a.part = reinterpret_cast<float *>(w + p.o_part);
    a.head = reinterpret_cast<float4 *>(w + p.o_head);
    a.dec = reinterpret_cast<float2 *>(w + p.o_dec);
    return type == 0 ? launch_typed<F32>(a, p, s) : type == 1 ? launch_typed<BF16>(a, p, s) : launch_typed<F16>(a, p, s);
}

}  // namespace cham
