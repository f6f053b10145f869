// Advantages and returns of trajectories (generalised advantage estimation).
//
// A_t = b_t + c_t A_{t+1} with b_t = r_t + gamma n_t V_{t+1} - V_t and c_t = gamma lambda n_t is a composition of affine
// maps: steps t .. u make of the advantage behind them q + p A_{u+1}, and two runs (p1, q1), (p2, q2), the second later, join
// to (p1 p2, q1 + p1 q2).  So every thread folds eight consecutive steps, the runs of a workgroup's threads are scanned from the end,
// and every thread walks its steps once more with the advantage behind them known: one read of everything, one write.  In
// double: the sum over a long trajectory keeps its small terms.
// Bound by latency: a workgroup's loads, its join (shuffles and a barrier) and its stores follow each other (bf16 512 x 8192 ragged
// 11 us, 2.2 TB/s; fp32 128 x 500 step by step 8.9 us).  Few long trajectories are cut into chunks of their own workgroups and read twice.
#include "cham_device.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kSteps = 8;                 // consecutive steps of a thread

struct Run {
    double p, q;                          // factor and summand
};
// q + p x.  CUT (where episodes end inside): q alone where p is 0, so that an episode takes nothing from the next one, not even a NaN.
// A factor is 0 by an episode's end, never by underflow: it stays at 1e-300, so that an infinity behind a run is one in front of it.
template <bool CUT>
__device__ __forceinline__ double apply(double p, double x, double q) { return CUT && p == 0.0 ? q : __builtin_fma(p, x, q); }
template <bool CUT>
__device__ __forceinline__ double factor_join(double a, double b) { return CUT && (a == 0.0 || b == 0.0) ? 0.0 : fmax(a * b, 1e-300); }
template <bool CUT>
__device__ __forceinline__ Run run_join(const Run &first, const Run &later) { return {factor_join<CUT>(first.p, later.p), apply<CUT>(first.p, later.q, first.q)}; }
__device__ __forceinline__ Run run_down(const Run &r, int by) { return {__shfl_down(r.p, by), __shfl_down(r.q, by)}; }

__device__ __forceinline__ int64_t length_of(const GaeArgs &a, int64_t b)
{
    if (!a.lengths) return a.S;
    const int64_t n = a.lengths[b];
    return n < 0 ? 0 : n < a.S ? n : a.S;
}

// Eight steps of a thread from `base` on; those at and behind `end` are none.
struct Steps {
    float v[kSteps];
    double d[kSteps];                     // b_t
    uint32_t done;                        // a bit each
    int end;
};

// Items base .. base + 7 of a row, and of its dones.
template <typename T>
__device__ __forceinline__ void load_eight(const typename T::item *p, float (&x)[kSteps])
{
#pragma unroll
    for (int k = 0; k < kSteps / T::kVec; ++k) {
        const typename T::words w = *reinterpret_cast<const typename T::words *>(p + k * T::kVec);
        float y[T::kVec];
        T::unpack(make_uint4(w.x, w.y, w.z, w.w), y);
#pragma unroll
        for (int j = 0; j < T::kVec; ++j) x[k * T::kVec + j] = y[j];
    }
}
__device__ __forceinline__ uint32_t load_dones(const uint8_t *p)
{
    typedef unsigned words __attribute__((ext_vector_type(2), aligned(1)));
    const words w = *reinterpret_cast<const words *>(p);
    uint32_t bits = 0;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) bits |= (((i < 4 ? w.x : w.y) >> (8 * (i & 3))) & 0xffu) != 0 ? 1u << i : 0u;
    return bits;
}

// Steps [base, base + 8) of trajectory b as far as they are below `top`, at most its length.  Steps that are not there have b_t = 0: they
// stand behind the last one, where the advantage is 0, so their factor does not matter.
template <typename T, bool DENSE, bool DONES>
__device__ __forceinline__ Steps load_steps(const GaeArgs &a, int64_t b, int64_t base, int64_t top, int64_t len)
{
    Steps s;
    const int64_t left = top - base;
    s.end = left < 0 ? 0 : left > kSteps ? kSteps : (int)left;
    s.done = 0;
    float r[kSteps], next = 0.0f, boot = 0.0f;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) r[i] = s.v[i] = 0.0f;
    int boot_at = -1;
    if (s.end > 0) {
        const typename T::item *rew = static_cast<const typename T::item *>(a.rewards) + b * a.r_ldb + base * a.r_lds;
        const typename T::item *val = static_cast<const typename T::item *>(a.values) + b * a.v_ldb + base * a.v_lds;
        const uint8_t *done = DONES ? a.dones + b * a.d_ldb + base * a.d_lds : nullptr;
        if (base + kSteps < len) next = T::get(val[kSteps * a.v_lds]);
        else boot_at = (int)(len - 1 - base);
        if (boot_at >= 0 && a.bootstrap) boot = a.bootstrap[b];
        if (s.end == kSteps) {
            if (DENSE) {
                load_eight<T>(rew, r);
                load_eight<T>(val, s.v);
                if (DONES) s.done = load_dones(done);
            } else {
                typename T::item x[kSteps], y[kSteps];
                uint8_t z[kSteps];
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    x[i] = rew[i * a.r_lds];
                    y[i] = val[i * a.v_lds];
                    z[i] = DONES ? done[i * a.d_lds] : 0;
                }
#pragma unroll
                for (int i = 0; i < kSteps; ++i) {
                    r[i] = T::get(x[i]);
                    s.v[i] = T::get(y[i]);
                    s.done |= z[i] != 0 ? 1u << i : 0u;
                }
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSteps - 1; ++i)
                if (i < s.end) {
                    r[i] = T::get(rew[i * a.r_lds]);
                    s.v[i] = T::get(val[i * a.v_lds]);
                    if (DONES && done[i * a.d_lds]) s.done |= 1u << i;
                }
        }
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
        float n = i + 1 < kSteps ? s.v[i + 1 < kSteps ? i + 1 : i] : next;
        n = i == boot_at ? boot : n;
        if (DONES) n = (s.done >> i) & 1 ? 0.0f : n;
        s.d[i] = __builtin_fma(a.gamma, (double)n, (double)r[i] - (double)s.v[i]);
    }
    return s;
}

template <bool DONES>
__device__ __forceinline__ double factor_of(const GaeArgs &a, const Steps &s, int i) { return DONES && (s.done >> i) & 1 ? 0.0 : a.gamma_lambda; }

template <bool DONES>
__device__ __forceinline__ Run fold(const GaeArgs &a, const Steps &s)
{
    double q = s.d[kSteps - 1];
#pragma unroll
    for (int i = kSteps - 2; i >= 0; --i) q = apply<DONES>(factor_of<DONES>(a, s, i), q, s.d[i]);
    return {DONES && s.done != 0 ? 0.0 : a.factor_eight, q};
}
template <bool DENSE, bool DONES>
__device__ __forceinline__ void store_steps(const GaeArgs &a, int64_t b, const Steps &s, int64_t base, double behind)
{
    float adv[kSteps], ret[kSteps];
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
        behind = apply<DONES>(factor_of<DONES>(a, s, i), behind, s.d[i]);
        adv[i] = (float)behind;
        ret[i] = (float)(behind + (double)s.v[i]);
    }
    const int64_t at = b * a.o_ldb + base * a.o_lds;
    if (s.end == kSteps) {
        if (DENSE) {
            typedef float words __attribute__((ext_vector_type(4), aligned(4)));
#pragma unroll
            for (int i = 0; i < kSteps; i += 4) {
                *reinterpret_cast<words *>(a.adv + at + i) = words{adv[i], adv[i + 1], adv[i + 2], adv[i + 3]};
                if (a.ret) *reinterpret_cast<words *>(a.ret + at + i) = words{ret[i], ret[i + 1], ret[i + 2], ret[i + 3]};
            }
        } else {
#pragma unroll
            for (int i = 0; i < kSteps; ++i) a.adv[at + i * a.o_lds] = adv[i];
            if (a.ret)
#pragma unroll
                for (int i = 0; i < kSteps; ++i) a.ret[at + i * a.o_lds] = ret[i];
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < kSteps - 1; ++i)
        if (i < s.end) {
            a.adv[at + i * a.o_lds] = adv[i];
            if (a.ret) a.ret[at + i * a.o_lds] = ret[i];
        }
}

// Runs of a workgroup's threads joined: `later`: those of the threads behind this one (of the same trajectory), `all`: of all.  WIDTH
// trajectories side by side in a wave, lane = time group * WIDTH + trajectory; waves in order of time.
template <int THREADS, int WIDTH, bool CUT>
__device__ __forceinline__ void join_block(const Run &own, Run &later, Run &all)
{
    constexpr int kWaves = THREADS / 64, kGroups = 64 / WIDTH;
    __shared__ Run waves[kWaves][WIDTH];
    const int lane = threadIdx.x & 63, wave = threadIdx.x % THREADS >> 6, group = lane / WIDTH, col = lane % WIDTH;
    Run scan = own;                                                    // this thread's and all behind it in the wave
#pragma unroll
    for (int o = WIDTH; o < 64; o <<= 1) {
        const Run r = run_down(scan, o);
        if (lane + o < 64) scan = run_join<CUT>(scan, r);
    }
    later = run_down(scan, WIDTH & 63);
    if (group == kGroups - 1) later = {1.0, 0.0};
    if (kWaves == 1) {
        all = {__shfl(scan.p, col), __shfl(scan.q, col)};
        return;
    }
    if (group == 0) waves[wave][col] = scan;
    __syncthreads();
    Run rest{1.0, 0.0};
    all = {1.0, 0.0};
#pragma unroll 2
    for (int w = kWaves - 1; w >= 0; --w) {
        if (w == wave) rest = all;
        all = run_join<CUT>(waves[w][col], all);
    }
    later = run_join<CUT>(later, rest);
    __syncthreads();
}

// WIDTH trajectories side by side in a wave (1: a wave along time).  A workgroup of THREADS walks steps
// [t0, t1) of its trajectories from the end in tiles that begin at t0 + n tiles, so that only the last one has steps missing, behind
// the trajectory's end; `behind`: the advantage at t1, 0 unless t1 - t0 is whole tiles.  WRITE: outputs; otherwise what the steps make of the
// advantage behind them is returned by the threads of time group 0 of wave 0.
template <typename T, int THREADS, int WIDTH, bool DENSE, bool DONES, bool WRITE>
__device__ Run walk(const GaeArgs &a, int64_t b, int64_t t0, int64_t t1, int64_t len, int64_t last, double behind)
{
    constexpr int kWaves = THREADS / 64, kGroups = 64 / WIDTH, kTile = kWaves * kGroups * kSteps;
    const int lane = threadIdx.x & 63, wave = threadIdx.x % THREADS >> 6, group = lane / WIDTH;
    const int64_t all_steps = (t1 < last ? t1 : last) - t0;            // of the longest of the trajectories side by side
    const int64_t top = t1 < len ? t1 : len;
    Run all{1.0, 0.0};
    for (int64_t lo = t0 + (all_steps - 1) / kTile * kTile; all_steps > 0 && lo >= t0; lo -= kTile) {
        const int64_t base = lo + (wave * kGroups + group) * kSteps;
        const Steps s = load_steps<T, DENSE, DONES>(a, b, base, top, len);
        Run later, tile;
        join_block<THREADS, WIDTH, DONES>(fold<DONES>(a, s), later, tile);
        if (WRITE) {
            if (s.end > 0) store_steps<DENSE, DONES>(a, b, s, base, apply<DONES>(later.p, behind, later.q));
            behind = apply<DONES>(tile.p, behind, tile.q);
        }
        all = run_join<DONES>(tile, all);
    }
    return all;
}

// The advantage behind chunk i of a trajectory, from the runs of the later ones: a thread joins some consecutive ones, then the threads.
template <int THREADS, int WIDTH, bool CUT>
__device__ __forceinline__ double behind_chunk(const GaeArgs &a, int64_t b, int i)
{
    constexpr int kShares = THREADS / WIDTH;
    const int share = threadIdx.x % THREADS / WIDTH, n = a.chunks - 1 - i, per = (n + kShares - 1) / kShares;
    Run own{1.0, 0.0}, later, all;
    for (int k = per - 1; k >= 0; --k) {
        const int j = i + 1 + share * per + k;
        if (j < a.chunks && b < a.B) {
            const double2 x = a.runs[WIDTH == 1 ? b * a.chunks + j : j * a.B + b];
            own = run_join<CUT>({x.x, x.y}, own);
        }
    }
    join_block<THREADS, WIDTH, CUT>(own, later, all);
    return all.q;
}

// MODE 0: whole trajectories.  Few long ones are cut into chunks: 1 folds each by itself, 2 takes the advantage behind a chunk from the runs of
// the later ones and writes.
template <typename T, int THREADS, bool DENSE, bool DONES, int MODE>
__global__ void __launch_bounds__(THREADS < 256 ? 256 : THREADS, THREADS > 64 ? 4 : 2) gae_row_kernel(const GaeArgs a)
{
    constexpr int kRows = THREADS < 256 ? 256 / THREADS : 1;
    static_assert(THREADS == 64 || kRows == 1, "a wave needs no barrier with its neighbours");
    const int row = kRows > 1 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0;
    const int64_t units = a.B * a.chunks;
    for (int64_t u = (int64_t)blockIdx.x * kRows + row; u < units; u += (int64_t)gridDim.x * kRows) {
        const int64_t b = MODE == 0 ? u : u / a.chunks;
        const int i = MODE == 0 ? 0 : (int)(u - b * a.chunks);
        const int64_t t0 = i * a.chunk, t1 = MODE == 0 ? a.S : t0 + a.chunk, len = length_of(a, b);
        if (MODE == 1) {
            const Run r = walk<T, THREADS, 1, DENSE, DONES, false>(a, b, t0, t1, len, len, 0.0);
            if (threadIdx.x % THREADS == 0) a.runs[u] = make_double2(r.p, r.q);
        } else {
            walk<T, THREADS, 1, DENSE, DONES, true>(a, b, t0, t1, len, len, MODE == 2 ? behind_chunk<THREADS, 1, DONES>(a, b, i) : 0.0);
        }
    }
}

// Trajectories side by side in memory, steps one after the other: WIDTH trajectories a workgroup, whose items of a step are one run.
// Two workgroups share a compute unit, so that one loads while the other joins (1024 threads,
// one workgroup: 726 x 4630 fp32 45 us / 38, 64 x 65536 30 / 22).
constexpr int kSideThreads = 512;
template <typename T, int WIDTH, bool DONES, int MODE>
__global__ void __launch_bounds__(kSideThreads) gae_side_kernel(const GaeArgs a)
{
    const int64_t sets = (a.B + WIDTH - 1) / WIDTH, units = sets * a.chunks;
    const int col = threadIdx.x % WIDTH;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int64_t set = MODE == 0 ? u : u / a.chunks, b = set * WIDTH + col;
        const int i = (int)(u - set * a.chunks);
        const int64_t len = b < a.B ? length_of(a, b) : 0;              // 0: nothing of it is read or written
        int64_t last = len;                                             // the longest of those side by side
#pragma unroll
        for (int o = 1; o < WIDTH; o <<= 1) {
            const int64_t x = __shfl_xor(last, o);
            last = x > last ? x : last;
        }
        const int64_t t0 = i * a.chunk, t1 = MODE == 0 ? a.S : t0 + a.chunk;
        if (MODE == 1) {
            const Run r = walk<T, kSideThreads, WIDTH, false, DONES, false>(a, b, t0, t1, len, last, 0.0);
            if (threadIdx.x < WIDTH && b < a.B) a.runs[i * a.B + b] = make_double2(r.p, r.q);
        } else {
            const double behind = MODE == 2 ? behind_chunk<kSideThreads, WIDTH, DONES>(a, b, i) : 0.0;
            walk<T, kSideThreads, WIDTH, false, DONES, true>(a, b, t0, t1, len, last, behind);
        }
    }
}

constexpr int64_t kMostBlocks = 1 << 20;
unsigned blocks_for(int64_t n) { return (unsigned)(n < kMostBlocks ? n : kMostBlocks); }

template <typename T, int THREADS, bool DENSE, bool DONES>
void launch_row(const GaeArgs &a, hipStream_t s)
{
    constexpr int kBlock = THREADS < 256 ? 256 : THREADS, kRows = kBlock / THREADS;
    const dim3 grid(blocks_for((a.B * a.chunks + kRows - 1) / kRows));
    if (THREADS == 64 || a.chunks == 1) {                 // a wave's trajectories are one tile
        hipLaunchKernelGGL((gae_row_kernel<T, THREADS, DENSE, DONES, 0>), grid, dim3(kBlock), 0, s, a);
    } else if constexpr (THREADS > 64) {
        hipLaunchKernelGGL((gae_row_kernel<T, THREADS, DENSE, DONES, 1>), grid, dim3(kBlock), 0, s, a);
        hipLaunchKernelGGL((gae_row_kernel<T, THREADS, DENSE, DONES, 2>), grid, dim3(kBlock), 0, s, a);
    }
}
template <typename T, int WIDTH, bool DONES>
void launch_side(const GaeArgs &a, hipStream_t s)
{
    const dim3 grid(blocks_for((a.B + WIDTH - 1) / WIDTH * a.chunks)), block(kSideThreads);
    if (a.chunks == 1) {
        hipLaunchKernelGGL((gae_side_kernel<T, WIDTH, DONES, 0>), grid, block, 0, s, a);
    } else {
        hipLaunchKernelGGL((gae_side_kernel<T, WIDTH, DONES, 1>), grid, block, 0, s, a);
        hipLaunchKernelGGL((gae_side_kernel<T, WIDTH, DONES, 2>), grid, block, 0, s, a);
    }
}
template <typename T, bool DONES>
void launch_of(const GaeArgs &a, hipStream_t s)
{
    if (a.layout == kGaeSide && a.width == 16) launch_side<T, 16, DONES>(a, s);
    else if (a.layout == kGaeSide) launch_side<T, 64, DONES>(a, s);
    else if (a.layout == kGaeStrided) launch_row<T, 256, false, DONES>(a, s);
    else if (a.threads == 64) launch_row<T, 64, true, DONES>(a, s);
    else if (a.threads == 256) launch_row<T, 256, true, DONES>(a, s);
    else launch_row<T, 512, true, DONES>(a, s);
}
template <typename T>
hipError_t launch_typed(const GaeArgs &a, hipStream_t s)
{
    if (a.dones) launch_of<T, true>(a, s);
    else launch_of<T, false>(a, s);
    return hipGetLastError();
}

}  // namespace

GaePlan plan_gae(int64_t B, int64_t S, int layout)
{
    GaePlan p;
    // Dense rows: a wave up to 512 steps, four to 2048, eight beyond so that two rows share a compute unit (512 x up to 8192 16 us; sixteen
    // waves, one row, 18).  Few long rows: chunks of four waves' tiles (3 x 200003 12 us; of sixteen waves' 16), until there are two workgroups
    // for every compute unit.  A plan knows of no device, as the workspace is asked for ahead of it: it is made for the 256 units of the whole card.
    p.threads = layout == kGaeSide ? kSideThreads
                : layout == kGaeStrided ? 256
                : S <= 64 * kSteps ? 64
                : S <= 256 * kSteps || B * ((S + 4095) / 4096) < 256 ? 256 : 512;
    // Side by side: sixteen trajectories a workgroup and tiles of 256 steps, which few trajectories are cut into; many with more steps than a tile go by 64,
    // 256 contiguous bytes of each step (fp32, ragged with dones, us at 16 / 64: 726 x 4630 44 / 34, 2048 x 2048 40 / 33; 200 x 8000 19 / 24, 64 x 65536
    // 29 / 45).  Two tiles are walked in one launch rather than cut (128 x 500 12.1 / 9.6; of four 128 x 1024 12.5 / 15.8).
    p.width = layout != kGaeSide ? 1 : B >= 512 && S > kSideThreads / 16 * kSteps ? 64 : 16;
    const int64_t tile = (int64_t)p.threads / p.width * kSteps;
    const int64_t tiles = (S + tile - 1) / tile, units = (B + p.width - 1) / p.width;
    const int64_t want = units > 0 ? (512 + units - 1) / units : 1;
    int64_t n = want < tiles ? want : tiles;
    if (p.width == 16 && tiles <= 2) n = 1;
    if (n < 1) n = 1;
    const int64_t per = tiles > 0 ? (tiles + n - 1) / n : 1;
    p.chunk = per * tile;
    p.chunks = tiles > 0 ? (int)((tiles + per - 1) / per) : 1;
    p.bytes = p.chunks > 1 ? (B * p.chunks * 16 + 255) / 256 * 256 : 0;
    return p;
}

hipError_t launch_gae(const GaeArgs &a, int type, hipStream_t s)
{
    return type == 0 ? launch_typed<F32>(a, s) : type == 1 ? launch_typed<BF16>(a, s) : launch_typed<F16>(a, s);
}

}  // namespace cham
