// Advantages and returns of trajectories (generalised advantage estimation).
//
// A_t = b_t + c_t A_{t+1} with b_t = r_t + gamma n_t V_{t+1} - V_t and c_t = gamma lambda n_t is a composition of affine
// maps: steps t .. u make of the advantage behind them q + p A_{u+1}, and two runs (p1, q1), (p2, q2), the second later, join
// to (p1 p2, q1 + p1 q2).  So every thread folds a few consecutive steps, the runs of a workgroup are scanned from the end, and
// every thread walks its steps once more with the advantage behind them known.
#include "cham_device.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kThreads = 256;
constexpr int kSteps = 8;                 // consecutive steps of a thread
constexpr int kTile = kThreads * kSteps;

struct Run {
    double p, q;                          // factor and summand
};
__device__ __forceinline__ Run run_join(const Run &first, const Run &later) { return {first.p * later.p, first.q + first.p * later.q}; }
__device__ __forceinline__ Run run_down(const Run &r, int by) { return {__shfl_down(r.p, by), __shfl_down(r.q, by)}; }

// Steps [t0, t1) of trajectory b from its end backwards, in tiles; `behind` is the advantage at t1.  WRITE: outputs; otherwise only
// what the steps make of the advantage behind them, returned by thread 0.
template <typename T, bool WRITE>
__device__ Run walk(const GaeArgs &a, int64_t b, int64_t t0, int64_t t1, int64_t len, double behind)
{
    __shared__ Run waves[kThreads / 64];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const typename T::item *rew = static_cast<const typename T::item *>(a.rewards) + b * a.r_ldb;
    const typename T::item *val = static_cast<const typename T::item *>(a.values) + b * a.v_ldb;
    const uint8_t *done = a.dones ? a.dones + b * a.d_ldb : nullptr;
    const double boot = a.bootstrap ? (double)a.bootstrap[b] : 0.0;
    const double gl = a.gamma * a.lambda;
    Run all{1.0, 0.0};
    for (int64_t hi = t1; hi > t0; hi -= kTile) {
        const int64_t base = hi - kTile + (int64_t)tid * kSteps;       // may begin before t0
        double c[kSteps], d[kSteps], v[kSteps];
        double next = 0.0;
        if (base + kSteps > t0) next = base + kSteps < len ? (double)T::get(val[(base + kSteps) * a.v_lds]) : boot;
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) {
            const int64_t t = base + i;
            c[i] = 1.0;
            d[i] = v[i] = 0.0;
            if (t >= t0) {
                const double n = done && done[t * a.d_lds] ? 0.0 : 1.0;
                v[i] = (double)T::get(val[t * a.v_lds]);
                d[i] = (double)T::get(rew[t * a.r_lds]) + a.gamma * n * next - v[i];
                c[i] = gl * n;
                next = v[i];
            }
        }
        Run own{1.0, 0.0};
#pragma unroll
        for (int i = kSteps - 1; i >= 0; --i) own = run_join({c[i], d[i]}, own);
        Run scan = own;                                                // this lane's steps and all behind them in the wave
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const Run r = run_down(scan, o);
            if (lane + o < 64) scan = run_join(scan, r);
        }
        if (lane == 0) waves[wave] = scan;
        Run later = run_down(scan, 1);
        if (lane == 63) later = {1.0, 0.0};
        __syncthreads();
        Run rest{1.0, 0.0}, tile{1.0, 0.0};
        for (int w = kThreads / 64 - 1; w >= 0; --w) {
            if (w == wave) rest = tile;
            tile = run_join(waves[w], tile);
        }
        if (WRITE) {
            const Run r = run_join(later, rest);
            double adv = r.q + r.p * behind;
#pragma unroll
            for (int i = kSteps - 1; i >= 0; --i) {
                const int64_t t = base + i;
                adv = d[i] + c[i] * adv;
                if (t >= t0) {
                    a.adv[b * a.o_ldb + t * a.o_lds] = (float)adv;
                    if (a.ret) a.ret[b * a.o_ldb + t * a.o_lds] = (float)(adv + v[i]);
                }
            }
            behind = tile.q + tile.p * behind;
        }
        all = run_join(tile, all);
        __syncthreads();
    }
    return all;
}

__device__ __forceinline__ int64_t length_of(const GaeArgs &a, int64_t b)
{
    if (!a.lengths) return a.S;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n < a.S ? n : a.S;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) gae_kernel(const GaeArgs a)
{
    for (int64_t b = blockIdx.x; b < a.B; b += gridDim.x) {
        const int64_t len = length_of(a, b);
        walk<T, true>(a, b, 0, len, len, 0.0);
    }
}

// Few long trajectories: chunks of one fold by themselves (gae_fold_kernel), then every chunk takes the advantage behind it from
// the later ones' runs.
template <typename T>
__global__ void __launch_bounds__(kThreads) gae_fold_kernel(const GaeArgs a)
{
    for (int64_t u = blockIdx.x; u < a.B * a.chunks; u += gridDim.x) {
        const int64_t b = u / a.chunks, t0 = (u - b * a.chunks) * a.chunk, len = length_of(a, b);
        const int64_t t1 = t0 + a.chunk < len ? t0 + a.chunk : len;
        const Run r = walk<T, false>(a, b, t0, t1, len, 0.0);
        if (threadIdx.x == 0) a.runs[u] = make_double2(r.p, r.q);
    }
}
template <typename T>
__global__ void __launch_bounds__(kThreads) gae_chunk_kernel(const GaeArgs a)
{
    for (int64_t u = blockIdx.x; u < a.B * a.chunks; u += gridDim.x) {
        const int64_t b = u / a.chunks, i = u - b * a.chunks, t0 = i * a.chunk, len = length_of(a, b);
        const int64_t t1 = t0 + a.chunk < len ? t0 + a.chunk : len;
        double behind = 0.0;
        for (int64_t j = a.chunks - 1; j > i; --j) {
            const double2 r = a.runs[b * a.chunks + j];
            behind = r.y + r.x * behind;
        }
        walk<T, true>(a, b, t0, t1, len, behind);
    }
}

template <typename T>
hipError_t launch_typed(const GaeArgs &a, hipStream_t s)
{
    const int64_t units = a.B * a.chunks;
    const dim3 grid((unsigned)(units < (1 << 20) ? units : (1 << 20)));
    if (a.chunks == 1) {
        hipLaunchKernelGGL(gae_kernel<T>, grid, dim3(kThreads), 0, s, a);
    } else {
        hipLaunchKernelGGL(gae_fold_kernel<T>, grid, dim3(kThreads), 0, s, a);
        hipLaunchKernelGGL(gae_chunk_kernel<T>, grid, dim3(kThreads), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace

GaePlan plan_gae(int64_t B, int64_t S)
{
    // chunks of whole tiles, until there are 512 workgroups
    const int64_t tiles = (S + kTile - 1) / kTile;
    const int64_t want = B > 0 ? (512 + B - 1) / B : 1;
    int64_t n = want < tiles ? want : tiles;
    if (n < 1) n = 1;
    const int64_t per = (tiles + n - 1) / n;
    GaePlan p;
    p.chunk = (per > 0 ? per : 1) * kTile;
    p.chunks = tiles > 0 ? (int)((tiles + per - 1) / per) : 1;
    p.bytes = p.chunks > 1 ? (B * p.chunks * 16 + 255) / 256 * 256 : 0;
    return p;
}

hipError_t launch_gae(GaeArgs a, int type, hipStream_t s)
{
    if (a.B == 0 || a.S == 0) return hipSuccess;
    return type == 0 ? launch_typed<F32>(a, s) : type == 1 ? launch_typed<BF16>(a, s) : launch_typed<F16>(a, s);
}

}  // namespace cham
