// Log-probabilities of actions and the clipped policy loss with its gradients (Sec. 3.4: the exploration agent is trained
// with clipped policy updates).
//
// Per head of V logits x:  m = max x, s = sum e^(x-m), t = sum e^(x-m) (x-m);  log p_v = x_v - m - log s,
// H = log s - t / s.  Per decision, lp = sum over heads of log p_action, and with ratio rho = e^(lp - old)
//   L = w (-min(rho A, clip(rho) A) + c_v value - c_H H + c_kl (e^d - d - 1)),   d = ref - lp
//   dL/dlp = D = w (-rho A [unclipped side] + c_kl (1 - e^d)),   dL/dx_v = D ([v = a] - p_v) + w c_H p_v (log p_v + H).
// Exponentials are fp32 (logits have at most 24 bits), and so are the sums of a head, its reciprocal (within an ulp) and, where one lane has a whole
// head, its log-probability; differences, products and sums per decision and beyond are double, with the ratio's and the divergence's exponential of fp32's
// significand and double's range.  Double exp and expm1 there would change nothing that a log-probability from fp32 sums does not
// blur, and their constants spill registers (us a loss, so / with them: 64000 x 24 x 3 20.5 / 21.7, 16384 x 1000 29.6 / 38.0, bf16 4096 x 131072 433 / 485,
// 4096 x 24 x 100 31.8 / 32.3).
#include "cham_device.h"
#include "cham_internal.h"
#include "explore.h"
#include "explore_items.h"

namespace cham {

namespace {

constexpr int kThreads = 256;
constexpr float kLowest = -3.402823466e38f;     // maximum of nothing: finite, so that -inf - kLowest is not a NaN
constexpr float kFar = -300.0f;                 // 2^x is 0 in fp32 below; keeps 0 * (-inf) out of the sums
constexpr float kLog2e = 1.44269504f, kLn2 = 0.693147181f;

__device__ __forceinline__ float exp2_fast(float z) { return __builtin_amdgcn_exp2f(z); }

// Exponents are taken to the base 2: z = (x - m) log2 e.  The difference comes first, rounded relative to itself, so that no result depends on
// where a head's logits lie.  (x log2 e - m log2 e in one fused operation saves an instruction but carries the rounding of m log2 e, half a
// step of a number that may be far from 0, into every exponential: the sum over equal logits of -1e9 was off by 2^18.)
__device__ __forceinline__ float exponent(float x, float m) { return (x - m) * kLog2e; }

// Running maximum and sums of a head: of 2^z and of z 2^z.
struct Soft {
    float m, s, t;
};
__device__ __forceinline__ Soft soft_none() { return {kLowest, 0.0f, 0.0f}; }
// A NaN in x does not reach m (the maximum passes it by) but s, by its exponential.
__device__ __forceinline__ void soft_raise(Soft &a, float m)
{
    if (m > a.m) {
        const float d = (a.m - m) * kLog2e, f = exp2_fast(d);
        a.t = f > 0.0f ? f * (a.t + a.s * d) : 0.0f;
        a.s *= f;
        a.m = m;
    }
}
__device__ __forceinline__ void soft_add(Soft &a, float x)
{
    const float z = exponent(x, a.m), e = exp2_fast(z);
    a.s += e;
    a.t = __builtin_fmaf(e, fmaxf(z, kFar), a.t);
}
// N items more.  m is raised when an item is more than 8 above it and not before: e^8 times V (e^16 V where the sum a.m + 8 is rounded up) stays far
// inside fp32, and lanes that each find a new maximum now and then would have the wave rescale all the time.
template <int N>
__device__ __forceinline__ void soft_add_all(Soft &a, const float (&x)[N])
{
    float m = x[0];
#pragma unroll
    for (int j = 1; j < N; ++j) m = fmaxf(m, x[j]);
    if (m > a.m + 8.0f) soft_raise(a, m);
#pragma unroll
    for (int j = 0; j < N; ++j) soft_add(a, x[j]);
}
__device__ __forceinline__ Soft soft_join(Soft a, Soft b)
{
    const float m = fmaxf(a.m, b.m);
    soft_raise(a, m);
    soft_raise(b, m);
    return {m, a.s + b.s, a.t + b.t};
}

// log s and entropy of a head's sums (s > 0).
__device__ __forceinline__ float2 log_and_entropy(const Soft &v)
{
    const float ls = logf(v.s);
    return make_float2(ls, ls - v.t * kLn2 * __builtin_amdgcn_rcpf(v.s));
}

// Gradient by a head's logits: 2^z (c0 + c1 z), and D more at the action.
struct Slope {
    float m, c0, c1;
};
__device__ __forceinline__ Slope slope_of(float m, float s, float ls, float entropy, float2 d)
{
    const float inv = __builtin_amdgcn_rcpf(s);              // within an ulp; s is at least 1 and at most e^16 V
    return {m, (d.y * (entropy - ls) - d.x) * inv, d.y * kLn2 * inv};
}
template <bool ENT>
__device__ __forceinline__ float slope_at(const Slope &f, float x)
{
    const float z = exponent(x, f.m), e = exp2_fast(z);
    return ENT ? e * __builtin_fmaf(fmaxf(z, kFar), f.c1, f.c0) : e * f.c0;
}

// Maximum and sum over a wave, in every lane: within rows of sixteen lanes, then across rows, by lane shifts.
template <int CTRL, int ROWS>
__device__ __forceinline__ float shifted(float x, float none)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(none), __float_as_int(x), CTRL, ROWS, 0xf, false));
}
__device__ __forceinline__ float wave_max(float x)
{
    x = fmaxf(x, shifted<0x111, 0xf>(x, x));       // row_shr 1, 2, 4, 8
    x = fmaxf(x, shifted<0x112, 0xf>(x, x));
    x = fmaxf(x, shifted<0x114, 0xf>(x, x));
    x = fmaxf(x, shifted<0x118, 0xf>(x, x));
    x = fmaxf(x, shifted<0x142, 0xa>(x, x));       // row_bcast 15, 31
    x = fmaxf(x, shifted<0x143, 0xc>(x, x));
    return readlane_f(x, 63);
}
__device__ __forceinline__ float wave_sum_f(float x)
{
    x += shifted<0x111, 0xf>(x, 0.0f);
    x += shifted<0x112, 0xf>(x, 0.0f);
    x += shifted<0x114, 0xf>(x, 0.0f);
    x += shifted<0x118, 0xf>(x, 0.0f);
    x += shifted<0x142, 0xa>(x, 0.0f);
    x += shifted<0x143, 0xc>(x, 0.0f);
    return readlane_f(x, 63);
}
// One maximum for all lanes first, so that each rescales its sums once.
__device__ __forceinline__ Soft soft_wave(Soft a)
{
    soft_raise(a, wave_max(a.m));
    return {a.m, wave_sum_f(a.s), wave_sum_f(a.t)};
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

// e^x with the significand of an fp32 exponential (within two steps) and the range of a double: ratios beyond 2^127 are ordinary numbers as long as
// their products are.
__device__ __forceinline__ double exp_wide(double x)
{
    double z = x * 1.4426950408889634;
    z = z > 1200.0 ? 1200.0 : z < -1200.0 ? -1200.0 : z;          // infinite, 0; a NaN stays
    const double n = rint(z);
    return ldexp((double)exp2_fast((float)(z - n)), z == z ? (int)n : 0);
}

// e^d - 1 and e^d - 1 - d.  Near 0 by their series, which lose nothing to the difference (|d| <= 1/4: the first term left out is
// below 2^-24 of the sum).
struct Gap {
    double less1, rest;
};
__device__ __forceinline__ Gap gap_of(double d)
{
    if (fabs(d) <= 0.25) {
        const float f = (float)d;
        float p = 1.0f / 40320.0f;
        p = __builtin_fmaf(p, f, 1.0f / 5040.0f);
        p = __builtin_fmaf(p, f, 1.0f / 720.0f);
        p = __builtin_fmaf(p, f, 1.0f / 120.0f);
        p = __builtin_fmaf(p, f, 1.0f / 24.0f);
        p = __builtin_fmaf(p, f, 1.0f / 6.0f);
        p = __builtin_fmaf(p, f, 0.5f);
        const double rest = (double)p * d * d;
        return {d + rest, rest};
    }
    const double e = exp_wide(d);
    return {e - 1.0, e < __builtin_inf() ? e - 1.0 - d : e};      // an action that the policy has lost: infinite, not inf - inf
}

// What a decision is compared with.
struct Given {
    float w, adv, old, ref, value, old_value, ret;
};
template <typename LOAD>
__device__ __forceinline__ Given given_of(const PolicyArgs &a, int64_t r, LOAD &&load)
{
    Given g{};
    if (!a.old_logp) return g;
    g.old = load(a.old_logp, r);
    g.adv = load(a.adv, r);
    if (a.weights) g.w = load(a.weights, r);
    if (a.ref) g.ref = load(a.ref, r);
    if (a.values) {
        g.value = load(a.values, r);
        g.ret = load(a.returns, r);
        if (a.old_values) g.old_value = load(a.old_values, r);
    }
    return g;
}
__device__ __forceinline__ float load_plain(const float *p, int64_t i) { return p[i]; }
// By way of the scalar cache: for a decision that all lanes share.  Nothing that this reads is written by the kernel.
__device__ __forceinline__ float load_shared(const float *p, int64_t i) { return reinterpret_cast<const __attribute__((address_space(4))) float *>((uintptr_t)p)[i]; }

// One decision: writes its outputs, adds its terms, returns (D, w c_H).
__device__ __forceinline__ float2 decide(const PolicyArgs &a, int64_t r, const Given &in, bool on, double lp, double H, double *sum)
{
    if (a.logp) a.logp[r] = on ? (float)lp : 0.0f;
    if (a.entropy) a.entropy[r] = on ? (float)H : 0.0f;
    if (!a.old_logp) return make_float2(0.0f, 0.0f);
    if (!on) {
        if (a.grad_values) a.grad_values[r] = 0.0f;
        return make_float2(0.0f, 0.0f);
    }
    const double w = a.weights ? (double)in.w : a.w_all;
    const double A = (double)in.adv;
    const double rho = exp_wide(lp - (double)in.old);
    const double held_rho = rho < a.lo ? a.lo : rho > a.hi ? a.hi : rho;
    const double free = rho * A, held = held_rho * A;
    const bool clipped = free > held;
    sum[0] -= w * (clipped ? held : free);
    double D = clipped ? 0.0 : -free;
    if (a.values) {
        const double v = (double)in.value, ret = (double)in.ret;
        const double near = (v - ret) * (v - ret);
        double kept = near;
        if (a.old_values) {
            const double o = (double)in.old_value, d = v - o;
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
        const Gap gap = gap_of((double)in.ref - lp);
        sum[3] += w * gap.rest;
        if (a.c_kl != 0.0) D -= a.c_kl * gap.less1;
    }
    if (clipped) sum[4] += w;
    return make_float2((float)(w * D), (float)(w * a.c_entropy));
}

// Terms of the loss from the sums over all decisions.
__device__ __forceinline__ void write_terms(const PolicyArgs &a, const double *v)
{
    double total = v[0];
    if (a.c_value != 0.0) total += a.c_value * v[1];
    if (a.c_entropy != 0.0) total -= a.c_entropy * v[2];
    if (a.c_kl != 0.0) total += a.c_kl * v[3];
    a.terms[0] = (float)total;
    for (int i = 0; i < kPolicySums; ++i) a.terms[1 + i] = (float)v[i];
}

// A block's sums, from n partial ones in LDS, to the block's place, where policy_terms_kernel joins them; the only block of a launch writes the
// terms itself.  Ends without a barrier.
__device__ __forceinline__ void store_partials(const PolicyArgs &a, const double (*lds)[kPolicySums], int n, bool only)
{
    if (threadIdx.x != 0) return;
    double v[kPolicySums];
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        v[i] = 0.0;
        for (int w = 0; w < n; ++w) v[i] += lds[w][i];
    }
    if (only) {
        write_terms(a, v);
    } else {
#pragma unroll
        for (int i = 0; i < kPolicySums; ++i) a.sums[(int64_t)blockIdx.x * kPolicySums + i] = v[i];
    }
}

template <int WAVES>
__device__ __forceinline__ void store_sums(const PolicyArgs &a, const double (&sum)[kPolicySums], bool only)
{
    __shared__ double lds[WAVES][kPolicySums];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int i = 0; i < kPolicySums; ++i) {
        const double v = wave_sum(sum[i]);
        if (lane == 0) lds[wave][i] = v;
    }
    __syncthreads();
    store_partials(a, lds, WAVES, only);
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
        }
        write_terms(a, v);
    }
}

// --- few choices a head: a workgroup takes whole decisions, a thread whole heads

constexpr int kTileHeads = 1024;                // at most: kHeadsPerThread of each thread
constexpr int kHeadsPerThread = kTileHeads / kThreads;
constexpr int kTileItems = 8448;                // fp32 logits in LDS, 33 KiB: with 17 KiB of the heads' three workgroups share a compute unit
constexpr int kTileChoices = 32;                // beyond, a tile has fewer heads than threads
constexpr int kLaneChoices = 64;                // what a lane's registers hold

struct TileShape {
    int per_tile;           // decisions of a tile
    int stride;             // of a head's logits in LDS: odd, so that the threads of a wave read different banks
    unsigned inv_v, inv_g;  // ceil(2^32 / V), ceil(2^32 / G): quotients of numbers below 2^16
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

// Sums of a tile's decisions over their heads, in LDS, and what follows from them: dec, and in[] of the heads whose decision does not count.
// given: of decision tid, asked for ahead of the heads.
template <int HEADS>
struct TileHeads {
    float2 one[HEADS];          // log-probability and entropy of a head
    float2 dec[HEADS];          // of a decision: (D, w c_H)
    uint8_t in[HEADS];
};
template <int HEADS>
__device__ __forceinline__ void decide_tile(const PolicyArgs &a, TileHeads<HEADS> &t, int64_t r0, int nr, const Given &given, double *sum)
{
    for (int r = threadIdx.x; r < nr; r += kThreads) {
        double lp = 0.0, H = 0.0;
        bool any = false;
        if (counts(a, r0 + r))
#pragma unroll 4
            for (int g = 0; g < a.G; ++g) {
                const float2 o = t.one[r * a.G + g];
                lp += (double)o.x;
                H += (double)o.y;
                any = any || t.in[r * a.G + g] != 0;
            }
        t.dec[r] = decide(a, r0 + r, r < kThreads ? given : given_of(a, r0 + r, load_plain), any, lp, H, sum);
        if (!any)                           // also of weight 0: zeros, whatever the logits are
            for (int g = 0; g < a.G; ++g) t.in[r * a.G + g] = 0;
    }
}

// A head's log-probability from its sums; c = -1: left out.
__device__ __forceinline__ float2 head_of(const PolicyArgs &a, Soft &v, float xa, int &c, float2 &le)
{
    if (c < 0) return make_float2(0.0f, 0.0f);
    if (c == a.V) {
        c = 0;
        le.x = le.y = v.s = __builtin_nanf("");
        return le;
    }
    if (v.s == 0.0f) {
        c = -1;                                 // every choice is masked
        return make_float2(0.0f, 0.0f);
    }
    le = log_and_entropy(v);
    return make_float2(xa - v.m - le.x, le.y);
}

// A lane holds HEADS consecutive heads of up to VP choices in registers (four heads of up to four choices, one of up to 64); as many lanes as
// that takes side by side are a decision, and a wave takes as many decisions as fit (24 heads of 3: six lanes, ten
// decisions).  Nothing goes through LDS and no wave waits for another.  Choices from V to VP are masked ones.
// fp32 64000 x 24 x 3 with gradients 18.6 us, of which the vector instructions are 8 and 40 MB of memory 8: the chain of loads, exponentials,
// shuffles and the decision in double, twice per wave.  The tile kernel below took 24 us, more than 1024 workgroups 21.
// V = VP is known at compile time up to four, where a lane's heads are one run of items.
template <typename T>
__device__ __forceinline__ void read_head(const typename T::item *p, int n, float *x, int vp)
{
    typedef typename T::item items __attribute__((ext_vector_type(4)));
    typedef items loose __attribute__((aligned(sizeof(typename T::item))));
#pragma unroll
    for (int q = 0; q < vp; q += 4) {
        if (q + 4 <= n) {
            const items w = *reinterpret_cast<const loose *>(p + q);
#pragma unroll
            for (int j = 0; j < 4; ++j) x[q + j] = T::get(w[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) x[q + j] = q + j < n ? T::get(p[q + j]) : -__builtin_inff();
        }
    }
}
template <typename T>
__device__ __forceinline__ void write_head(typename T::item *p, int n, const float *y, int vp)
{
    typedef typename T::item items __attribute__((ext_vector_type(4)));
    typedef items loose __attribute__((aligned(sizeof(typename T::item))));
#pragma unroll
    for (int q = 0; q < vp; q += 4) {
        if (q + 4 <= n) {
            const items w = {T::put(y[q]), T::put(y[q + 1]), T::put(y[q + 2]), T::put(y[q + 3])};
            *reinterpret_cast<loose *>(p + q) = w;
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (q + j < n) p[q + j] = T::put(y[q + j]);
        }
    }
}

template <typename T, int VP, int HEADS>
__global__ void __launch_bounds__(kThreads, VP > 32 ? 2 : VP > 16 ? 3 : 4) policy_lane_kernel(const PolicyArgs a, int lanes)
{
    constexpr bool kExact = VP <= 4;
    const int V = kExact ? VP : a.V;
    const int lane = threadIdx.x & 63, per_wave = 64 / lanes, mine = lane / lanes, part = lane - mine * lanes;
    const int64_t step = (int64_t)gridDim.x * (kThreads / 64) * per_wave;
    const int h0 = part * HEADS, n = mine < per_wave ? (a.G - h0 < HEADS ? a.G - h0 : HEADS) : 0;      // heads of this lane
    const bool dense = (a.G == 1 || a.ld_g == V) && n == HEADS, gdense = (a.G == 1 || a.gld_g == V) && n == HEADS;
    double sum[kPolicySums] = {};
    for (int64_t r0 = ((int64_t)blockIdx.x * (kThreads / 64) + (threadIdx.x >> 6)) * per_wave; r0 < a.R; r0 += step) {
        const int64_t r = r0 + mine;
        const int here = r < a.R ? n : 0;
        float x[HEADS][VP];
        int c[HEADS];
        Given given{};
        bool on = false;
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            c[u] = -1;
#pragma unroll
            for (int j = 0; j < VP; ++j) x[u][j] = 0.0f;
        }
        if (here > 0) {
            const typename T::item *p = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + h0 * a.ld_g;
            if (!kExact) {
                read_head<T>(p, V, x[0], VP);
            } else if (dense) {
                typename T::item y[HEADS * VP];
#pragma unroll
                for (int i = 0; i < HEADS * VP; ++i) y[i] = p[i];
#pragma unroll
                for (int i = 0; i < HEADS * VP; ++i) x[i / VP][i % VP] = T::get(y[i]);
            } else {
#pragma unroll
                for (int u = 0; u < HEADS; ++u)
                    if (u < here)
#pragma unroll
                        for (int j = 0; j < VP; ++j) x[u][j] = T::get(p[u * a.ld_g + j]);
            }
#pragma unroll
            for (int u = 0; u < HEADS; ++u)
                if (u < here) c[u] = choice_of(a, r * a.G + h0 + u);
            if (part == 0) given = given_of(a, r, load_plain);
            on = counts(a, r);
        }
        Soft v[HEADS];
        float2 le[HEADS];
        double lp = 0.0, H = 0.0;
        bool any = false;
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            v[u] = soft_none();
            le[u] = make_float2(0.0f, 0.0f);
            float xa = 0.0f;
#pragma unroll
            for (int j = 0; j < VP; ++j) {
                v[u].m = fmaxf(v[u].m, x[u][j]);
                xa = j == c[u] ? x[u][j] : xa;
            }
#pragma unroll
            for (int j = 0; j < VP; ++j) soft_add(v[u], x[u][j]);
            const float2 one = head_of(a, v[u], xa, c[u], le[u]);
            lp += (double)one.x;
            H += (double)one.y;
            any = any || c[u] >= 0;
        }
        // the decision's lanes joined into its first one
        for (int o = 1; o < lanes; o <<= 1) {
            const double l2 = __shfl_down(lp, o), H2 = __shfl_down(H, o);
            const int a2 = __shfl_down((int)any, o);
            if (part + o < lanes) {
                lp += l2;
                H += H2;
                any = any || a2;
            }
        }
        float2 d = make_float2(0.0f, 0.0f);
        on = on && any;
        if (part == 0 && here > 0) d = decide(a, r, given, on, on ? lp : 0.0, on ? H : 0.0, sum);
        if (!a.grad) continue;
        const int first = lane - part;
        d = make_float2(__shfl(d.x, first), __shfl(d.y, first));
        on = __shfl((int)on, first);
        if (here == 0) continue;
        typename T::item *p = static_cast<typename T::item *>(a.grad) + r * a.gld_r + h0 * a.gld_g;
#pragma unroll
        for (int u = 0; u < HEADS; ++u) {
            const bool in = on && c[u] >= 0;
            const Slope f = slope_of(v[u].m, v[u].s, le[u].x, le[u].y, d);
#pragma unroll
            for (int j = 0; j < VP; ++j) x[u][j] = in ? slope_at<true>(f, x[u][j]) + (j == c[u] ? d.x : 0.0f) : 0.0f;
        }
        if (!kExact) {
            write_head<T>(p, V, x[0], VP);
        } else if (gdense) {
#pragma unroll
            for (int i = 0; i < HEADS * VP; ++i) p[i] = T::put(x[i / VP][i % VP]);
        } else {
#pragma unroll
            for (int u = 0; u < HEADS; ++u)
                if (u < here)
#pragma unroll
                    for (int j = 0; j < VP; ++j) p[u * a.gld_g + j] = T::put(x[u][j]);
        }
    }
    if (a.old_logp) store_sums<kThreads / 64>(a, sum, gridDim.x == 1);
}

// More heads: the tile's logits in LDS, eight at a time in a thread's registers; bound by LDS and its four barriers (fp32 4096 x 128 x 10 with
// gradients 29 us, 1.5 TB/s).
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_tile_kernel(const PolicyArgs a, const TileShape k)
{
    __shared__ float x[kTileItems];
    __shared__ TileHeads<kTileHeads> t;
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
            const int h = quotient(i, k.inv_v, a.V), r = quotient(h, k.inv_g, a.G);
            return (r0 + r) * ld_r + (h - r * a.G) * ld_g + (i - h * a.V);
        };
        int c[kHeadsPerThread];
#pragma unroll
        for (int u = 0; u < kHeadsPerThread; ++u) {
            const int h = tid + u * kThreads;
            c[u] = h < heads ? choice_of(a, r0 * a.G + h) : -1;
        }
        Given given{};
        if (tid < nr) given = given_of(a, r0 + tid, load_plain);
        const typename T::item *logits = static_cast<const typename T::item *>(a.logits);
        if (k.dense)
            read_run<T>(logits + r0 * gv, items, [&](int i, float v) { x[at(i)] = v; });
        else
            for (int i = tid; i < items; i += kThreads) x[at(i)] = T::get(logits[offset(i, a.ld_r, a.ld_g)]);
        __syncthreads();

        Soft v[kHeadsPerThread];
        float2 le[kHeadsPerThread];
#pragma unroll
        for (int u = 0; u < kHeadsPerThread; ++u) {
            const int h = tid + u * kThreads;
            v[u] = soft_none();
            le[u] = make_float2(0.0f, 0.0f);
            if (h >= heads) continue;
            const float *xh = x + h * k.stride;
            for (int j0 = 0; j0 < a.V; j0 += 8) {
                float y[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) y[j] = j0 + j < a.V ? xh[j0 + j] : -__builtin_inff();
                soft_add_all(v[u], y);
            }
            const float xa = c[u] >= 0 && c[u] < a.V ? xh[c[u]] : 0.0f;
            t.one[h] = head_of(a, v[u], xa, c[u], le[u]);
            t.in[h] = c[u] >= 0;
        }
        __syncthreads();
        decide_tile(a, t, r0, nr, given, sum);
        __syncthreads();
        if (!a.grad) continue;
#pragma unroll
        for (int u = 0; u < kHeadsPerThread; ++u) {
            const int h = tid + u * kThreads;
            if (h >= heads) continue;
            float *xh = x + h * k.stride;
            const bool in = t.in[h] != 0;
            const float2 d = t.dec[quotient(h, k.inv_g, a.G)];
            const Slope f = slope_of(v[u].m, v[u].s, le[u].x, le[u].y, d);
#pragma unroll 4
            for (int j = 0; j < a.V; ++j) xh[j] = in ? slope_at<true>(f, xh[j]) : 0.0f;
            if (in) xh[c[u]] += d.x;
        }
        __syncthreads();
        typename T::item *grad = static_cast<typename T::item *>(a.grad);
        if (k.gdense)
            write_run<T>(grad + r0 * gv, items, [&](int i) { return x[at(i)]; });
        else
            for (int i = tid; i < items; i += kThreads) grad[offset(i, a.gld_r, a.gld_g)] = T::put(x[at(i)]);
        __syncthreads();
    }
    if (a.old_logp) store_sums<kThreads / 64>(a, sum, gridDim.x == 1);
}

// --- one head of more choices: a row stays in the registers of a wave or a workgroup between its sums and its gradient

// Waves of a SIMD that n pieces a thread leave room for (in registers; beyond eight in LDS).
constexpr int row_waves(int n) { return n > 8 ? 4 : n == 8 ? 5 : 6; }

template <typename T>
__device__ __forceinline__ uint4 masked_items()          // 16 bytes of -inf
{
    const uint32_t w = sizeof(typename T::item) == 4 ? 0xff800000u : T::kMasked * 0x10001u;
    return make_uint4(w, w, w, w);
}

// Unpacked items are not carried from one use to the next: they would take twice the registers.
__device__ __forceinline__ void keep_packed(uint4 &v) { asm volatile("" : "+v"(v.x), "+v"(v.y), "+v"(v.z), "+v"(v.w)); }

// Sums of a thread's items joined over the THREADS of a row; every thread returns the row's.
template <int THREADS>
__device__ __forceinline__ Soft soft_row(Soft v, Soft *lds)
{
    v = soft_wave(v);
    if (THREADS == 64) return v;
    if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
    __syncthreads();
    float m = kLowest, sum = 0.0f, t = 0.0f;
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) m = fmaxf(m, lds[w].m);
#pragma unroll
    for (int w = 0; w < THREADS / 64; ++w) {
        Soft o = lds[w];
        soft_raise(o, m);
        sum += o.s;
        t += o.t;
    }
    return {m, sum, t};
}

// A gradient is not read again here: it goes past the caches, which then hold what rows longer than the registers are read from a second time
// (fp32 4096 x 50021 398 -> 355 us, 1024 x 131072 311 -> 256, bf16 4096 x 131072 533 -> 508).
// Its 16 bytes may begin at any item: the hardware takes that, only slower.
template <typename T>
__device__ __forceinline__ void store_past(typename T::item *p, const uint4 &v)
{
    const typename T::words w = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(w, reinterpret_cast<typename T::words *>(p));
}

// Where the items of a decision's row stand: an unaligned head and tail around pieces of 16 bytes.
struct RowAt {
    int choice;                                          // of its action; -1: left out
    int head, n_vec, tail;
};

// THREADS of a row hold N x 16 bytes of it each in registers and L x 16 in LDS, and its ends up to the first and from the last 16-byte boundary
// an item each; what is left of longer rows is read once for the sums and once for the gradient.  A workgroup stays, and asks for a
// piece of its next row's N as soon as it is done with that of the present one, so that loads are under way while sums are joined and gradients
// stored.
template <typename T, int THREADS, int N, int L, bool GRAD, bool ENT>
__global__ void __launch_bounds__(THREADS < kThreads ? kThreads : THREADS, row_waves(N + L)) policy_row_kernel(const PolicyArgs a)
{
    constexpr int kBlock = THREADS < kThreads ? kThreads : THREADS, kRows = kBlock / THREADS;
    constexpr int kHeld = (N + L) * THREADS;             // pieces of a row that are read once
    __shared__ uint4 stash[L > 0 ? L : 1][L > 0 ? kBlock : 1];
    __shared__ Soft lds[THREADS / 64];
    __shared__ float2 dec;
    __shared__ double sum[kRows][kPolicySums];           // of the rows of a group so far, by its first thread
    const int tid = threadIdx.x % THREADS, group = THREADS == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0;
    if (tid < kPolicySums) sum[group][tid] = 0.0;
    __syncthreads();
    const int64_t step = (int64_t)gridDim.x * kRows;
    const auto row_of = [&](int64_t r) { return static_cast<const typename T::item *>(a.logits) + r * a.ld_r; };
    const auto look_up = [&](int64_t r) {
        RowAt at{-1, 0, 0, 0};
        if (r < a.R) {
            at.choice = counts(a, r) ? choice_of(a, r) : -1;
            at.head = (int)items_to_boundary<T>(row_of(r), a.V);
            at.n_vec = (a.V - at.head) / T::kVec;
            at.tail = a.V - at.head - at.n_vec * T::kVec;
        }
        return at;
    };
    uint4 held[N];
    const auto ask = [&](int64_t r, const RowAt &at, int k) {
        const uint4 *body = reinterpret_cast<const uint4 *>(row_of(r) + at.head);
        held[k] = masked_items<T>();
        if (at.choice >= 0 && tid + k * THREADS < at.n_vec) held[k] = body[tid + k * THREADS];
    };
    int64_t r = (int64_t)blockIdx.x * kRows + group;
    RowAt now = look_up(r);
#pragma unroll
    for (int k = 0; k < N; ++k) ask(r, now, k);
    for (; r < a.R; r += step) {
        const typename T::item *row = row_of(r);
        typename T::item *to = GRAD ? static_cast<typename T::item *>(a.grad) + r * a.gld_r : nullptr;
        const int c = now.choice, head = now.head, n_vec = now.n_vec;
        const uint4 *body = reinterpret_cast<const uint4 *>(row + head);
        const int end_at = tid < head ? tid : tid < head + now.tail ? n_vec * T::kVec + tid : -1;
        float end[1] = {-__builtin_inff()}, xa = 0.0f;
        if (c >= 0 && end_at >= 0) end[0] = T::get(row[end_at]);
        if (c >= 0 && c < a.V) xa = T::get(row[c]);      // before a gradient in place
        const RowAt next = look_up(r + step);
        const Given given = given_of(a, r, load_shared);
        Soft v = soft_none();
        if (c >= 0) {
            uint4 rest[L > 0 ? L : 1];
#pragma unroll
            for (int l = 0; l < L; ++l) {
                rest[l] = masked_items<T>();
                if (tid + (N + l) * THREADS < n_vec) rest[l] = body[tid + (N + l) * THREADS];
            }
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (k * THREADS < n_vec) {               // of all threads
                    float x[T::kVec];
                    T::unpack(held[k], x);
                    soft_add_all(v, x);
                }
                if (!GRAD) ask(r + step, next, k);
                else keep_packed(held[k]);
            }
#pragma unroll
            for (int l = 0; l < L; ++l)
                if ((N + l) * THREADS < n_vec) {
                    float x[T::kVec];
                    T::unpack(rest[l], x);
                    soft_add_all(v, x);
                    if (GRAD) stash[l][threadIdx.x] = rest[l];
                }
            for (int i = tid + kHeld; i < n_vec; i += THREADS) {
                float x[T::kVec];
                T::unpack(body[i], x);
                soft_add_all(v, x);
            }
            soft_add_all(v, end);
        } else if (!GRAD) {
#pragma unroll
            for (int k = 0; k < N; ++k) ask(r + step, next, k);
        }
        v = soft_row<THREADS>(v, lds);
        bool in = c >= 0 && v.s != 0.0f;                 // 0: every choice is masked
        if (c == a.V) {
            in = true;
            v.s = __builtin_nanf("");
        }
        const float2 le = log_and_entropy(v);
        float2 d = make_float2(0.0f, 0.0f);
        if (tid == 0) d = decide(a, r, given, in, in ? (double)xa - (double)v.m - (double)le.x : 0.0, in ? (double)le.y : 0.0, sum[group]);
        if (THREADS == 64) {
            d.x = readlane_f(d.x, 0);
            d.y = readlane_f(d.y, 0);
        } else {
            if (tid == 0) dec = d;
            __syncthreads();                             // lds is written again, too
            d = dec;
        }
        if (GRAD) {
            const Slope f = slope_of(v.m, v.s, le.x, le.y, d);
            auto write = [&](int i, const uint4 &raw) {
                float x[T::kVec];
                T::unpack(raw, x);
#pragma unroll
                for (int j = 0; j < T::kVec; ++j) x[j] = slope_at<ENT>(f, x[j]);
                store_past<T>(to + head + i * T::kVec, T::pack(x));
            };
            // the next row's pieces are asked for as this one's registers come free
#pragma unroll
            for (int k = 0; k < N; ++k) {
                if (in && tid + k * THREADS < n_vec) write(tid + k * THREADS, held[k]);
                ask(r + step, next, k);
            }
            if (in) {
#pragma unroll
                for (int l = 0; l < L; ++l)
                    if (tid + (N + l) * THREADS < n_vec) write(tid + (N + l) * THREADS, stash[l][threadIdx.x]);
                for (int i = tid + kHeld; i < n_vec; i += THREADS) write(i, body[i]);
                if (end_at >= 0) to[end_at] = T::put(slope_at<ENT>(f, end[0]));
                // the action's item once more, by the thread that has written it
                const bool owner = c < head || c >= head + n_vec * T::kVec ? end_at == c : (c - head) / T::kVec % THREADS == tid;
                if (owner && c < a.V) to[c] = T::put(slope_at<ENT>(f, xa) + d.x);
            } else {
                for (int i = tid; i < n_vec; i += THREADS) store_past<T>(to + head + i * T::kVec, make_uint4(0, 0, 0, 0));
                if (end_at >= 0) to[end_at] = T::put(0.0f);
            }
        }
        now = next;
    }
    __syncthreads();
    if (a.old_logp) store_partials(a, sum, kRows, gridDim.x == 1);
}

// --- any number of heads and choices, in three steps: sums of parts of heads, decisions, gradient.  Three launches (two for very few
// rows of one head) and a second read; for few rows of long heads bound by latency (fp32 9 x 50021: 12 us), for many by memory and the instructions around each head
// (bf16 4096 x 24 x 1000 123 us, 3.2 TB/s).

// THREADS of a part: a wave of short heads, a workgroup of parts of long ones.
template <typename T, int THREADS>
__global__ void __launch_bounds__(kThreads) policy_part_kernel(const PolicyArgs a, int splits, int chunk)
{
    constexpr int kParts = kThreads / THREADS;
    __shared__ Soft lds[kThreads / 64];
    const int tid = threadIdx.x % THREADS, group = THREADS == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0;
    const int64_t units = a.R * a.G * splits;
    for (int64_t u = (int64_t)blockIdx.x * kParts + group; u < units; u += (int64_t)gridDim.x * kParts) {
        const int64_t h = splits == 1 ? u : u / splits, r = a.G == 1 ? h : h / a.G;
        if (!counts(a, r)) continue;
        const int c = choice_of(a, h);
        if (c < 0 || c == a.V) continue;
        const int g = (int)(h - r * a.G), lo = (int)(u - h * splits) * chunk;
        const int hi = lo + chunk < a.V ? lo + chunk : a.V;
        const typename T::item *row = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
        Soft v = soft_none();
        const int head = (int)items_to_boundary<T>(row + lo, hi - lo), n_vec = (hi - lo - head) / T::kVec, tail = lo + head + n_vec * T::kVec;
        const uint4 *body = reinterpret_cast<const uint4 *>(row + lo + head);
        float end[2] = {-__builtin_inff(), -__builtin_inff()};
        if (tid < head) end[0] = T::get(row[lo + tid]);
        if (tid < hi - tail) end[1] = T::get(row[tail + tid]);
        const float xa = c >= lo && c < hi ? T::get(row[c]) : 0.0f;
        soft_add_all(v, end);
        for (int i = tid; i < n_vec; i += THREADS) {
            float x[T::kVec];
            T::unpack(body[i], x);
            soft_add_all(v, x);
        }
        v = soft_wave(v);
        if (THREADS > 64) {
            if ((tid & 63) == 0) lds[tid >> 6] = v;
            __syncthreads();
            if (tid == 0)
                for (int w = 1; w < THREADS / 64; ++w) v = soft_join(v, lds[w]);
        }
        if (tid == 0) reinterpret_cast<float4 *>(a.part)[u] = make_float4(v.m, v.s, v.t, xa);
        if (THREADS > 64) __syncthreads();
    }
}

// A head of a decision from the sums of its parts and its action's logit x: what it adds to the decision, and what its gradient needs.
__device__ __forceinline__ float4 join_head(const PolicyArgs &a, int c, float x, const Soft &v, double &lp, double &H, bool &in)
{
    if (c == a.V) {
        lp = H = __builtin_nan("");
        in = true;
        return make_float4(0.0f, __builtin_nanf(""), 0.0f, __int_as_float(0));
    }
    if (c < 0 || v.s == 0.0f) return make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));       // 0: every choice is masked
    const float2 le = log_and_entropy(v);
    lp += (double)x - (double)v.m - (double)le.x;
    H += (double)le.y;
    in = true;
    return make_float4(v.m, v.s, le.y, __int_as_float(c));
}

// A head's sums and, as x, its action's logit from its parts, over a wave.  c: its choice, within the choices.
__device__ __forceinline__ Soft soft_parts(const PolicyArgs &a, int64_t h, int c, int splits, int chunk, float &x)
{
    const float4 *parts = reinterpret_cast<const float4 *>(a.part) + h * splits;
    Soft v = soft_none();
    x = parts[c / chunk].w;
    for (int i = threadIdx.x & 63; i < splits; i += 64) {
        const float4 p = parts[i];
        v = soft_join(v, {p.x, p.y, p.z});
    }
    return soft_wave(v);
}

// Decisions, a wave each.  Heads of one part: a lane each; of several: the heads one after the other, their parts over the lanes.
// LAST: nothing reads what a gradient needs of them.
template <int WAVES, bool LAST>
__device__ __forceinline__ void join_rows(const PolicyArgs &a, int splits, int chunk, int64_t first, int64_t step, double (&sum)[kPolicySums])
{
    const int lane = threadIdx.x & 63;
    for (int64_t r = first + (threadIdx.x >> 6); r < a.R; r += step) {
        double lp = 0.0, H = 0.0;
        bool in = false;
        const Given given = given_of(a, r, load_plain);        // asked for ahead of the sums
        if (counts(a, r)) {
            if (splits == 1) {
                for (int g = lane; g < a.G; g += 64) {
                    const int64_t h = r * a.G + g;
                    const int c = choice_of(a, h);
                    float4 p = make_float4(kLowest, 0.0f, 0.0f, 0.0f);
                    if (c >= 0 && c < a.V) p = reinterpret_cast<const float4 *>(a.part)[h];
                    const float4 out = join_head(a, c, p.w, {p.x, p.y, p.z}, lp, H, in);
                    if (!LAST && a.grad) a.head[h] = out;
                }
                lp = wave_sum(lp);
                H = wave_sum(H);
                in = __any(in);
            } else {
                for (int g = 0; g < a.G; ++g) {
                    const int64_t h = r * a.G + g;
                    const int c = choice_of(a, h);
                    Soft v = soft_none();
                    float x = 0.0f;
                    if (c >= 0 && c < a.V) v = soft_parts(a, h, c, splits, chunk, x);
                    const float4 out = join_head(a, c, x, v, lp, H, in);
                    if (!LAST && a.grad && lane == 0) a.head[h] = out;
                }
            }
        }
        if (lane == 0) {
            const float2 d = decide(a, r, given, in, lp, H, sum);
            if (!LAST && a.grad) a.dec[r] = d;
        }
    }
}

template <int WAVES>
__global__ void __launch_bounds__(WAVES * 64) policy_join_kernel(const PolicyArgs a, int splits, int chunk)
{
    double sum[kPolicySums] = {};
    join_rows<WAVES, false>(a, splits, chunk, (int64_t)blockIdx.x * WAVES, (int64_t)gridDim.x * WAVES, sum);
    if (a.old_logp) store_sums<WAVES>(a, sum, gridDim.x == 1);
}

// JOIN (one head, few decisions): there is no join before it.  Every wave joins its row's parts and takes the decision for itself; what decisions
// write, and the terms, are left to the last workgroup.
template <typename T, int THREADS, bool JOIN>
__global__ void __launch_bounds__(kThreads) policy_grad_kernel(const PolicyArgs a, int splits, int chunk)
{
    constexpr int kParts = kThreads / THREADS;
    const int tid = threadIdx.x % THREADS, group = THREADS == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x / THREADS) : 0;
    const int64_t blocks = (int64_t)gridDim.x - JOIN;
    if (JOIN && blockIdx.x == blocks) {
        double sum[kPolicySums] = {};
        join_rows<kThreads / 64, true>(a, splits, chunk, 0, kThreads / 64, sum);
        store_sums<kThreads / 64>(a, sum, true);
        return;
    }
    const int64_t units = a.R * a.G * splits;
    for (int64_t u = (int64_t)blockIdx.x * kParts + group; u < units; u += blocks * kParts) {
        const int64_t h = splits == 1 ? u : u / splits, r = a.G == 1 ? h : h / a.G;
        const int g = (int)(h - r * a.G), lo = (int)(u - h * splits) * chunk;
        const int hi = lo + chunk < a.V ? lo + chunk : a.V;
        typename T::item *to = static_cast<typename T::item *>(a.grad) + r * a.gld_r + g * a.gld_g;
        float4 k = make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
        float2 d = make_float2(0.0f, 0.0f);
        if (counts(a, r)) {
            if (JOIN) {
                PolicyArgs quiet = a;
                quiet.logp = quiet.entropy = quiet.grad_values = nullptr;
                double lp = 0.0, H = 0.0, sum[kPolicySums] = {};
                bool in = false;
                const int c = choice_of(a, h);
                const Given given = given_of(a, r, load_plain);
                Soft v = soft_none();
                float x = 0.0f;
                if (c >= 0 && c < a.V) v = soft_parts(a, h, c, splits, chunk, x);
                k = join_head(a, c, x, v, lp, H, in);
                d = decide(quiet, r, given, in, lp, H, sum);
            } else {
                k = a.head[h];
                d = a.dec[r];
            }
        }
        const int c = __float_as_int(k.w);
        if (c < 0) {
            for (int v = lo + tid; v < hi; v += THREADS) to[v] = T::put(0.0f);
            continue;
        }
        const typename T::item *row = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
        const Slope f = slope_of(k.x, k.y, logf(k.y), k.z, d);
        const int head = (int)items_to_boundary<T>(row + lo, hi - lo), n_vec = (hi - lo - head) / T::kVec, tail = lo + head + n_vec * T::kVec;
        auto one = [&](int v) { to[v] = T::put(slope_at<true>(f, T::get(row[v])) + (v == c ? d.x : 0.0f)); };
        if (tid < head) one(lo + tid);
        if (tid < hi - tail) one(tail + tid);
        for (int i = tid; i < n_vec; i += THREADS) {
            const int at = lo + head + i * T::kVec;
            float x[T::kVec];
            T::unpack(*reinterpret_cast<const uint4 *>(row + at), x);
#pragma unroll
            for (int j = 0; j < T::kVec; ++j) x[j] = slope_at<true>(f, x[j]) + (at + j == c ? d.x : 0.0f);
            store_past<T>(to + at, T::pack(x));
        }
    }
}

// --- several heads of more choices, many decisions: a wave takes a decision, sixteen lanes a head

constexpr int kGroup = 16;
constexpr int kGroupHeads = 256;                 // at most: what LDS holds of the four decisions of a workgroup
constexpr int kGroupChoices = 512, kGroupRows = 256;
// Decisions from which this is faster than three steps.  A wave walks its decision's heads four at a time, each in so many pieces a lane, whatever the
// number of decisions (up to 4096 on the chip), and three steps spread heads over the chip: eight decisions for every piece and head of up to 64.
// us a loss, in three steps / so: bf16 4096 x 24 x 70 98 / 30, x 150 102 / 40, x 500 101 / 62, x 1000 123 / 144; 1024 x 24 x 150 34 / 23, x 500 37 / 40; 1024 x 128 x 70
// 124 / 72, x 500 127 / 184; 2048 x 128 x 500 270 / 304; 512 x 250 x 70 124 / 132, x 500 127 / 339; 256 x 2 x 70 15 / 10; fp32 1024 x 128 x 500 2.5
// times as long so, 4096 x 24 x 500 1.2 times (the rows of all waves leave the caches before their second read), 4096 x 250 x 70 0.4 times.
inline int64_t group_rows(int G, int V, int type)
{
    const int64_t pieces = (V / (16 / type_bytes(type)) + kGroup - 1) / kGroup, rows = 8 * pieces * (G < 64 ? G : 64);
    return rows > kGroupRows ? rows : kGroupRows;
}

// Maximum and sum over sixteen lanes, in each of them, by rotations.
__device__ __forceinline__ Soft soft_group(Soft v)
{
    float m = v.m;
    m = fmaxf(m, shifted<0x121, 0xf>(m, m));       // row_ror 1, 2, 4, 8
    m = fmaxf(m, shifted<0x122, 0xf>(m, m));
    m = fmaxf(m, shifted<0x124, 0xf>(m, m));
    m = fmaxf(m, shifted<0x128, 0xf>(m, m));
    soft_raise(v, m);
    v.s += shifted<0x121, 0xf>(v.s, 0.0f);
    v.s += shifted<0x122, 0xf>(v.s, 0.0f);
    v.s += shifted<0x124, 0xf>(v.s, 0.0f);
    v.s += shifted<0x128, 0xf>(v.s, 0.0f);
    v.t += shifted<0x121, 0xf>(v.t, 0.0f);
    v.t += shifted<0x122, 0xf>(v.t, 0.0f);
    v.t += shifted<0x124, 0xf>(v.t, 0.0f);
    v.t += shifted<0x128, 0xf>(v.t, 0.0f);
    return v;
}

// A decision's logits are read for the sums and, out of the caches, for the gradient.  A head's pieces of 16 bytes begin at its first item, wherever
// that lies; what a head leaves of a last piece is read by item.  Bound by the instructions around short heads and by latency (bf16 4096 x 24 x 100
// with gradients 32 us, 1.2 TB/s).
template <typename T>
__global__ void __launch_bounds__(kThreads) policy_group_kernel(const PolicyArgs a)
{
    constexpr int kGroups = 64 / kGroup;
    __shared__ float4 state[kThreads / 64][kGroupHeads];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, group = lane / kGroup, l = lane % kGroup;
    const int n_vec = a.V / T::kVec, tail = n_vec * T::kVec + l;
    double sum[kPolicySums] = {};
    for (int64_t r = (int64_t)blockIdx.x * (kThreads / 64) + wave; r < a.R; r += (int64_t)gridDim.x * (kThreads / 64)) {
        const bool on = counts(a, r);
        double lp = 0.0, H = 0.0;
        bool in = false;
        Given given{};
        if (lane == 0) given = given_of(a, r, load_plain);
        if (on)
            for (int g0 = 0; g0 < a.G; g0 += kGroups) {
                const int g = g0 + group, c = g < a.G ? choice_of(a, r * a.G + g) : -1;
                Soft v = soft_none();
                float xa = 0.0f;
                if (c >= 0 && c < a.V) {
                    const typename T::item *p = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
                    xa = T::get(p[c]);
                    float end[1] = {-__builtin_inff()};
                    if (tail < a.V) end[0] = T::get(p[tail]);
                    for (int i = l; i < n_vec; i += kGroup) {
                        float x[T::kVec];
                        const typename T::words w = *reinterpret_cast<const typename T::words *>(p + i * T::kVec);
                        T::unpack(make_uint4(w.x, w.y, w.z, w.w), x);
                        soft_add_all(v, x);
                    }
                    soft_add_all(v, end);
                }
                v = soft_group(v);
                if (l == 0 && g < a.G) state[wave][g] = join_head(a, c, xa, v, lp, H, in);
            }
        lp = wave_sum(lp);
        H = wave_sum(H);
        in = __any(in);
        float2 d = make_float2(0.0f, 0.0f);
        if (lane == 0) d = decide(a, r, given, in, lp, H, sum);
        if (!a.grad) continue;
        d.x = readlane_f(d.x, 0);
        d.y = readlane_f(d.y, 0);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // state, written by other lanes of this wave
        for (int g = group; g < a.G; g += kGroups) {
            typename T::item *to = static_cast<typename T::item *>(a.grad) + r * a.gld_r + g * a.gld_g;
            const typename T::item *p = static_cast<const typename T::item *>(a.logits) + r * a.ld_r + g * a.ld_g;
            const float4 k = on ? state[wave][g] : make_float4(0.0f, 0.0f, 0.0f, __int_as_float(-1));
            const int c = __float_as_int(k.w);
            const Slope f = slope_of(k.x, k.y, logf(k.y), k.z, d);
            for (int i = l; i < n_vec; i += kGroup) {
                float x[T::kVec] = {};
                if (c >= 0) {
                    const typename T::words w = *reinterpret_cast<const typename T::words *>(p + i * T::kVec);
                    T::unpack(make_uint4(w.x, w.y, w.z, w.w), x);
#pragma unroll
                    for (int j = 0; j < T::kVec; ++j) x[j] = slope_at<true>(f, x[j]) + (i * T::kVec + j == c ? d.x : 0.0f);
                }
                const uint4 y = T::pack(x);
                *reinterpret_cast<typename T::words *>(to + i * T::kVec) = typename T::words{y.x, y.y, y.z, y.w};
            }
            if (tail < a.V) to[tail] = T::put(c >= 0 ? slope_at<true>(f, T::get(p[tail])) + (tail == c ? d.x : 0.0f) : 0.0f);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");       // before the next decision's state
    }
    if (a.old_logp) store_sums<kThreads / 64>(a, sum, gridDim.x == 1);
}

constexpr int kJoinBlocks = 1024;
constexpr int kTileBlocks = 1024;               // what is on the chip at a time
constexpr int kUnits = 256;                     // compute units of the whole card: what a plan, which knows of no device, is made for
constexpr int kRowBlocks = 6 * kUnits;          // workgroups at most that stay on the device's own units
constexpr int kWaveChunk = 2048;                // choices of a part that a wave takes
// Decisions that one workgroup joins, a wave each; with gradients of one head, beside the gradient's workgroups (us a loss, three launches / two: fp32 1 x 50021
// 12.7 / 9.1, 9 x 50021 14.0 / 12.2, 16 x 131072 15.5 / 15.5, 32 x 131072 18.0 / 23.7).
constexpr int kJoinFew = 16;

// A wave or a workgroup per row, by its pieces of 16 bytes: 64 threads up to 1024 pieces (four rows a workgroup, no barrier), 256 up to
// 4096, 512 to 8192, 1024 beyond, up to sixteen pieces a thread, of which eight in registers and eight in LDS (sixteen in registers: bf16 8192 x
// 20001 146 us / 137, 4096 x 50021 186 / 178, fp32 16384 x 4000 105 / 100, and with 1024 threads they spill).  us a loss, bf16, 64 / 256 threads: 6001 x 8191
// 42 / 49, 16384 x 4096 64 / 81; 256 / 512: 4096 x 65536 249 / 213; 512 / 1024: 4096 x 65536 213 / 237, 4096 x 131072 483 / 413 (the rest of a
// row read twice; a copy of as many bytes 390), fp32 4096 x 50021 341 / 330, 1024 x 131072 249 / 236.
// Fewer rows than what fills the chip take the next size, as a row is then all latency: 512 x 8192 15.0 / 11.5, 1024 x 8192
// 17.0 / 16.6, 1024 x 4096 12.1 / 12.9; fp32 256 x 16384 (4096 pieces; 256 / 1024) 15.6 / 14.3, bf16 (2048 pieces) 12.1 / 12.5.
// Beyond 4096 pieces log-probabilities alone take a row in parts, which a workgroup reads without holding it (bf16 4096 x 131072,
// row / parts, 245 / 194 us, fp32 1024 x 50021 40 / 36; at 4096 pieces, 2048 x 32768, 26 / 28), and gradients do so for few rows:
// the row is read twice, but by many workgroups: 9 x 131072 bf16 24 / 15, 64 26 / 23, 128 30 / 31; fp32 32 x 50021 19 / 17, 128 23 / 26.
// (All pairs: before the exponents' difference became an instruction of its own, which adds 0 to 5 % to either side.)
constexpr int kWideRow = 4096;
constexpr int kFewRows = 1024, kVeryFewRows = 256;
constexpr unsigned kMostBlocks = 1u << 20;

unsigned blocks_for(int64_t n) { return (unsigned)(n < (int64_t)kMostBlocks ? n : (int64_t)kMostBlocks); }
int64_t up256(int64_t v) { return (v + 255) / 256 * 256; }

// The terms of a loss, unless its only workgroup has written them.
hipError_t launch_terms(const PolicyArgs &a, unsigned blocks, hipStream_t s)
{
    if (a.old_logp && (a.R == 0 || blocks > 1))
        hipLaunchKernelGGL(policy_terms_kernel, dim3(1), dim3(kThreads), 0, s, a, a.R > 0 ? (int)blocks : 0);
    return hipGetLastError();
}

template <typename T, int THREADS, int N>
void launch_row_of(const PolicyArgs &a, unsigned blocks, hipStream_t s)
{
    constexpr int kRegisters = N < 8 ? N : 8, kLds = N - kRegisters;
    const dim3 block(THREADS < kThreads ? kThreads : THREADS);
    if constexpr (THREADS * N <= kWideRow)                // longer rows without gradients go by parts
        if (!a.grad) {
            hipLaunchKernelGGL((policy_row_kernel<T, THREADS, kRegisters, 0, false, false>), dim3(blocks), block, 0, s, a);
            return;
        }
    if (a.c_entropy != 0.0) hipLaunchKernelGGL((policy_row_kernel<T, THREADS, kRegisters, kLds, true, true>), dim3(blocks), block, 0, s, a);
    else hipLaunchKernelGGL((policy_row_kernel<T, THREADS, kRegisters, kLds, true, false>), dim3(blocks), block, 0, s, a);
}
template <typename T>
void launch_row(const PolicyArgs &a, const PolicyPlan &p, unsigned blocks, hipStream_t s)
{
    switch (p.threads + p.row) {
    case 64 + 1: return launch_row_of<T, 64, 1>(a, blocks, s);
    case 64 + 2: return launch_row_of<T, 64, 2>(a, blocks, s);
    case 64 + 4: return launch_row_of<T, 64, 4>(a, blocks, s);
    case 64 + 8: return launch_row_of<T, 64, 8>(a, blocks, s);
    case 64 + 16: return launch_row_of<T, 64, 16>(a, blocks, s);
    case 256 + 4: return launch_row_of<T, 256, 4>(a, blocks, s);
    case 256 + 8: return launch_row_of<T, 256, 8>(a, blocks, s);
    case 256 + 16: return launch_row_of<T, 256, 16>(a, blocks, s);
    case 512 + 8: return launch_row_of<T, 512, 8>(a, blocks, s);
    case 512 + 16: return launch_row_of<T, 512, 16>(a, blocks, s);
    default: return launch_row_of<T, 1024, 16>(a, blocks, s);
    }
}

template <typename T, int HEADS>
void launch_lane(const PolicyArgs &a, unsigned blocks, int lanes, hipStream_t s)
{
    const dim3 grid(blocks), block(kThreads);
    if (a.V == 1) hipLaunchKernelGGL((policy_lane_kernel<T, 1, HEADS>), grid, block, 0, s, a, lanes);
    else if (a.V == 2) hipLaunchKernelGGL((policy_lane_kernel<T, 2, HEADS>), grid, block, 0, s, a, lanes);
    else if (a.V == 3) hipLaunchKernelGGL((policy_lane_kernel<T, 3, HEADS>), grid, block, 0, s, a, lanes);
    else hipLaunchKernelGGL((policy_lane_kernel<T, 4, HEADS>), grid, block, 0, s, a, lanes);
}
template <typename T>
void launch_lane_of(const PolicyArgs &a, unsigned blocks, int lanes, hipStream_t s)
{
    const dim3 grid(blocks), block(kThreads);
    if (a.V > 32) hipLaunchKernelGGL((policy_lane_kernel<T, 64, 1>), grid, block, 0, s, a, lanes);
    else if (a.V > 16) hipLaunchKernelGGL((policy_lane_kernel<T, 32, 1>), grid, block, 0, s, a, lanes);
    else if (a.V > 8) hipLaunchKernelGGL((policy_lane_kernel<T, 16, 1>), grid, block, 0, s, a, lanes);
    else if (a.V > 4) hipLaunchKernelGGL((policy_lane_kernel<T, 8, 1>), grid, block, 0, s, a, lanes);
    else if (a.G == 1) launch_lane<T, 1>(a, blocks, lanes, s);
    else if (a.G == 2) launch_lane<T, 2>(a, blocks, lanes, s);
    else launch_lane<T, 4>(a, blocks, lanes, s);
}

template <typename T>
hipError_t launch_typed(PolicyArgs &a, const PolicyPlan &p, hipStream_t s)
{
    if (p.lanes) {
        const int64_t per_block = (int64_t)(kThreads / 64) * (64 / p.lanes), groups = (a.R + per_block - 1) / per_block;
        const unsigned blocks = (unsigned)(groups < kTileBlocks ? groups : kTileBlocks);
        if (a.R > 0) launch_lane_of<T>(a, blocks, p.lanes, s);
        return launch_terms(a, blocks, s);
    }
    if (p.tile) {
        const int gv = a.G * a.V;
        TileShape k;
        k.per_tile = p.tile;
        k.stride = a.V | 1;
        k.inv_v = (unsigned)((((uint64_t)1 << 32) + a.V - 1) / a.V);
        k.inv_g = (unsigned)((((uint64_t)1 << 32) + a.G - 1) / a.G);
        k.dense = (a.G == 1 || a.ld_g == a.V) && (a.R == 1 || a.ld_r == gv);
        k.gdense = (a.G == 1 || a.gld_g == a.V) && (a.R == 1 || a.gld_r == gv);
        const int64_t tiles = (a.R + p.tile - 1) / p.tile;
        const unsigned blocks = (unsigned)(tiles < kTileBlocks ? tiles : kTileBlocks);
        if (a.R > 0) {
            const dim3 grid(blocks), block(kThreads);
            hipLaunchKernelGGL(policy_tile_kernel<T>, grid, block, 0, s, a, k);
        }
        return launch_terms(a, blocks, s);
    }
    if (p.row) {
        const int rows = p.threads < kThreads ? kThreads / p.threads : 1;
        const int64_t groups = (a.R + rows - 1) / rows;
        int cus = 0;
        const hipError_t e = compute_units(cus);
        if (e != hipSuccess) return e;
        if (cus > kUnits) cus = kUnits;
        const int64_t resident = (int64_t)cus * (row_waves(p.row) * 4 / (p.threads < kThreads ? kThreads / 64 : p.threads / 64));
        // Log-probabilities alone: a workgroup for every long row, which the hardware spreads better than a fixed share (us, bf16, share / each:
        // 4096 x 32768 52.2 / 46.5, 16384 x 16384 113 / 101; by waves 6001 x 8191 22.4 / 23.8).  With gradients, whose stores the next row's
        // loads run under, and a loss's sums, a share (4096 x 131072 440 / 474, 16384 x 1000 22.7 / 26.5).
        const bool each = !a.old_logp && p.threads >= kThreads;
        const unsigned blocks = each ? blocks_for(groups) : (unsigned)(groups < resident ? groups : resident);
        if (a.R > 0) launch_row<T>(a, p, blocks, s);
        return launch_terms(a, blocks, s);
    }
    if (p.group) {
        const int64_t groups = (a.R + kThreads / 64 - 1) / (kThreads / 64);
        const unsigned blocks = (unsigned)(groups < kTileBlocks ? groups : kTileBlocks);
        hipLaunchKernelGGL(policy_group_kernel<T>, dim3(blocks), dim3(kThreads), 0, s, a);
        return launch_terms(a, blocks, s);
    }
    const int64_t units = a.R * a.G * p.splits;
    const bool fused = a.grad && a.G == 1 && a.R <= kJoinFew;
    const unsigned join = (unsigned)(a.R <= kJoinFew ? 1 : (a.R + 3) / 4 < kJoinBlocks ? (a.R + 3) / 4 : kJoinBlocks);
    if (a.R > 0) {
        const bool wave = p.chunk <= kWaveChunk;
        const dim3 grid(blocks_for(wave ? (units + 3) / 4 : units)), more(grid.x + 1), block(kThreads);
        if (wave) hipLaunchKernelGGL((policy_part_kernel<T, 64>), grid, block, 0, s, a, p.splits, p.chunk);
        else hipLaunchKernelGGL((policy_part_kernel<T, kThreads>), grid, block, 0, s, a, p.splits, p.chunk);
        if (fused) {
            hipLaunchKernelGGL((policy_grad_kernel<T, kThreads, true>), more, block, 0, s, a, p.splits, p.chunk);
            return hipGetLastError();
        }
        if (join == 1) hipLaunchKernelGGL(policy_join_kernel<kJoinFew>, dim3(1), dim3(kJoinFew * 64), 0, s, a, p.splits, p.chunk);
        else hipLaunchKernelGGL(policy_join_kernel<kThreads / 64>, dim3(join), block, 0, s, a, p.splits, p.chunk);
        if (a.grad && wave) hipLaunchKernelGGL((policy_grad_kernel<T, 64, false>), grid, block, 0, s, a, p.splits, p.chunk);
        else if (a.grad) hipLaunchKernelGGL((policy_grad_kernel<T, kThreads, false>), grid, block, 0, s, a, p.splits, p.chunk);
    }
    return launch_terms(a, join, s);
}

}  // namespace

PolicyPlan plan_policy(int64_t R, int G, int V, int type, bool grad)
{
    PolicyPlan p{};
    if (V <= 4 ? G <= 256 : V <= kLaneChoices && G <= 64 && (G > 1 || V <= 32)) {
        p.lanes = V > 4 ? G : G <= 2 ? 1 : (G + 3) / 4;
        p.bytes = (int64_t)kTileBlocks * kPolicySums * 8;
        return p;
    }
    if (V <= kTileChoices && G <= kTileHeads && (int64_t)G * (V | 1) <= kTileItems) {
        const int by_heads = kTileHeads / G, by_items = kTileItems / (G * (V | 1));
        p.tile = by_heads < by_items ? by_heads : by_items;
        // fewer decisions a tile where that leaves compute units without one
        const int64_t spread = (R + 2 * kUnits - 1) / (2 * kUnits);
        if (spread < p.tile) p.tile = spread > 1 ? (int)spread : 1;
        p.bytes = (int64_t)kTileBlocks * kPolicySums * 8;
        return p;
    }
    const int vecs = V / (16 / type_bytes(type));
    if (G == 1 && (vecs <= kWideRow || (grad && R * 256 > vecs))) {
        p.threads = vecs <= 1024 ? 64 : vecs <= kWideRow ? 256 : vecs <= 2 * kWideRow ? 512 : 1024;
        if (R < kFewRows && vecs > 256 && vecs <= 1024) p.threads = 256;
        if (R <= kVeryFewRows && vecs > 2048 && vecs <= kWideRow) p.threads = 512;
        const int n = (vecs + p.threads - 1) / p.threads;
        p.row = n <= 1 ? 1 : n <= 2 ? 2 : n <= 4 ? 4 : n <= 8 ? 8 : 16;
        if (p.threads == 256 && p.row < 4) p.row = 4;
        if (p.threads == 512 && p.row < 8) p.row = 8;
        if (p.threads == 1024) p.row = 16;
        p.bytes = (int64_t)kRowBlocks * kPolicySums * 8;
        return p;
    }
    if (G > 1 && G <= kGroupHeads && V <= kGroupChoices && R >= group_rows(G, V, type)) {
        p.group = kGroup;
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
