// C ABI of the agent's update: argument checks and workspace carving of cham_policy_logp, cham_policy_loss, cham_gae,
// cham_grad_norm and cham_clip_grads (paper Sec. 3.4).
#include "../../include/cham.h"

#include <math.h>

#include "explore.h"
#include "explore_items.h"

using namespace cham;

namespace {

constexpr int64_t kMostItems = (int64_t)1 << 40;

bool aligned(const void *p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) % to) == 0; }
bool float_type(int32_t t) { return t == CHAM_TYPE_F32 || t == CHAM_TYPE_BF16 || t == CHAM_TYPE_F16; }
bool workspace_ok(const void *w, int64_t have, int64_t need) { return need == 0 || (w && aligned(w, 256) && have >= need); }

// Whether n1 runs at stride ld1 of n2 runs at stride ld2 of `run` consecutive items lie apart, in either order; extent: items from the
// first to behind the last.
bool apart(int64_t n1, int64_t ld1, int64_t n2, int64_t ld2, int64_t run, int64_t &extent)
{
    if (n1 <= 1) ld1 = 0;
    if (n2 <= 1) ld2 = 0;
    if (ld1 < 0 || ld2 < 0 || ld1 > kMostItems || ld2 > kMostItems) return false;
    int64_t e1, e2;
    if (__builtin_mul_overflow(n1 > 0 ? n1 - 1 : 0, ld1, &e1) || __builtin_mul_overflow(n2 > 0 ? n2 - 1 : 0, ld2, &e2) ||
        __builtin_add_overflow(e1, e2, &extent) || __builtin_add_overflow(extent, run, &extent) || extent > ((int64_t)1 << 59))
        return false;
    if (n1 <= 1 && n2 <= 1) return true;
    if (n1 <= 1) return ld2 >= run;
    if (n2 <= 1) return ld1 >= run;
    return (ld2 >= run && ld1 >= e2 + run) || (ld1 >= run && ld2 >= e1 + run);
}

int32_t check_sizes(int64_t R, int32_t G, int32_t V, int32_t type)
{
    if (R < 0 || G < 1 || G > 65536 || V < 1 || V > (1 << 24) || R > kMostItems / G) return CHAM_E_BAD_DIM;
    return float_type(type) ? CHAM_OK : CHAM_E_BAD_TYPE;
}

// The arguments that both policy entry points take; extent: items of the logits.
int32_t check_policy(PolicyArgs &a, const void *logits, int32_t type, int64_t R, int32_t G, int32_t V, int64_t ld_r, int64_t ld_g,
                     const void *actions, int32_t action_type, int64_t first_action, const float *weights, float *logp,
                     float *entropy, int64_t &extent)
{
    const int32_t e = check_sizes(R, G, V, type);
    if (e != CHAM_OK) return e;
    if (action_type != CHAM_TYPE_I8 && action_type != CHAM_TYPE_I32 && action_type != CHAM_TYPE_I64) return CHAM_E_BAD_TYPE;
    if (R > 0 && (!logits || !actions)) return CHAM_E_NULL;
    a = PolicyArgs{};
    a.abytes = action_type == CHAM_TYPE_I8 ? 1 : action_type == CHAM_TYPE_I32 ? 4 : 8;
    if (!apart(R, ld_r, G, ld_g, V, extent)) return CHAM_E_BAD_DIM;
    if (!aligned(logits, type_bytes(type)) || !aligned(actions, a.abytes) || !aligned(weights, 4) || !aligned(logp, 4) || !aligned(entropy, 4))
        return CHAM_E_BAD_DIM;
    a.logits = logits;
    a.R = R;
    a.G = G;
    a.V = V;
    a.ld_r = R > 1 ? ld_r : 0;
    a.ld_g = G > 1 ? ld_g : 0;
    a.actions = actions;
    a.first = first_action;
    a.weights = weights;
    a.logp = logp;
    a.entropy = entropy;
    return CHAM_OK;
}

// Addresses of a dense argument; empty without one.
struct Span {
    uintptr_t lo, hi;
};
Span span(const void *p, int64_t bytes)
{
    const uintptr_t at = reinterpret_cast<uintptr_t>(p);
    return p && bytes > 0 ? Span{at, at + (uintptr_t)bytes} : Span{0, 0};
}
bool crosses(const Span &a, const Span &b) { return a.lo < b.hi && b.lo < a.hi; }
// Whether one of the first n_out spans, which are written, crosses another span.
template <int N>
bool shared(const Span (&spans)[N], int n_out)
{
    for (int i = 0; i < n_out; ++i)
        for (int j = i + 1; j < N; ++j)
            if (crosses(spans[i], spans[j])) return true;
    return false;
}

bool factor(double x) { return x >= 0.0 && x <= 1.7976931348623157e308; }       // not NaN, not infinite

}  // namespace

extern "C" {

int64_t cham_policy_workspace_bytes(int64_t R, int32_t G, int32_t V, int32_t type, int32_t want_grad)
{
    const int32_t e = check_sizes(R, G, V, type);
    if (e != CHAM_OK) return e;
    // with gradients: enough for either call
    const int64_t without = plan_policy(R, G, V, type, false).bytes, with = want_grad ? plan_policy(R, G, V, type, true).bytes : 0;
    return with > without ? with : without;
}

int32_t cham_policy_logp(const void *logits, int32_t type, int64_t R, int32_t G, int32_t V, int64_t ld_r, int64_t ld_g,
                         const void *actions, int32_t action_type, int64_t first_action, const float *weights,
                         float *logp, float *entropy, void *workspace, int64_t workspace_bytes, void *stream)
{
    PolicyArgs a;
    int64_t extent;
    const int32_t e = check_policy(a, logits, type, R, G, V, ld_r, ld_g, actions, action_type, first_action, weights, logp, entropy, extent);
    if (e != CHAM_OK) return e;
    if (R == 0) return CHAM_OK;
    if (!logp) return CHAM_E_NULL;
    const int64_t need = plan_policy(R, G, V, type, false).bytes, heads = R * G;
    if (!workspace_ok(workspace, workspace_bytes, need)) return CHAM_E_WORKSPACE;
    const Span spans[] = {span(logp, 4 * R), span(entropy, 4 * R), span(workspace, need), span(weights, 4 * R), span(actions, heads * a.abytes),
                          span(logits, extent == heads * V ? extent * type_bytes(type) : 0)};
    if (shared(spans, 3)) return CHAM_E_BAD_DIM;
    const hipError_t h = launch_policy(a, type, workspace, reinterpret_cast<hipStream_t>(stream));
    return h == hipSuccess ? CHAM_OK : hip_fail(h);
}

int32_t cham_policy_loss(const void *logits, int32_t type, int64_t R, int32_t G, int32_t V, int64_t ld_r, int64_t ld_g,
                         const void *actions, int32_t action_type, int64_t first_action, const float *weights,
                         const float *old_logp, const float *advantages, const float *ref_logp,
                         const float *values, const float *old_values, const float *returns,
                         const cham_policy_coef *coef, float *terms, float *logp, float *entropy,
                         void *grad_logits, int64_t gld_r, int64_t gld_g, float *grad_values,
                         void *workspace, int64_t workspace_bytes, void *stream)
{
    PolicyArgs a;
    int64_t extent, g_extent;
    const int32_t e = check_policy(a, logits, type, R, G, V, ld_r, ld_g, actions, action_type, first_action, weights, logp, entropy, extent);
    if (e != CHAM_OK) return e;
    if (!coef || !terms || (R > 0 && (!old_logp || !advantages))) return CHAM_E_NULL;
    if (!factor(coef->clip_low) || !factor(coef->clip_high) || !factor(coef->value) || !factor(coef->entropy) || !factor(coef->kl) ||
        (old_values && !factor(coef->value_clip)))
        return CHAM_E_BAD_COEF;
    if (R > 0 && ((values != nullptr) != (returns != nullptr) || (!values && (old_values || coef->value != 0.0)) || (!ref_logp && coef->kl != 0.0)))
        return CHAM_E_NULL;
    if (!aligned(old_logp, 4) || !aligned(advantages, 4) || !aligned(ref_logp, 4) || !aligned(values, 4) || !aligned(old_values, 4) ||
        !aligned(returns, 4) || !aligned(terms, 4) || !aligned(grad_values, 4))
        return CHAM_E_BAD_DIM;
    if (grad_logits) {
        const int bytes = type_bytes(type);
        if (!aligned(grad_logits, bytes) || !apart(R, gld_r, G, gld_g, V, g_extent)) return CHAM_E_BAD_DIM;
        const uintptr_t l0 = reinterpret_cast<uintptr_t>(logits), l1 = l0 + (uintptr_t)extent * bytes;
        const uintptr_t g0 = reinterpret_cast<uintptr_t>(grad_logits), g1 = g0 + (uintptr_t)g_extent * bytes;
        const bool same = l0 == g0 && (R <= 1 || ld_r == gld_r) && (G <= 1 || ld_g == gld_g);
        if (R > 0 && !same && l0 < g1 && g0 < l1) return CHAM_E_BAD_DIM;
        a.grad = grad_logits;
        a.gld_r = R > 1 ? gld_r : 0;
        a.gld_g = G > 1 ? gld_g : 0;
    }
    const int64_t need = plan_policy(R, G, V, type, grad_logits != nullptr).bytes, heads = R * G;
    if (!workspace_ok(workspace, workspace_bytes, need)) return CHAM_E_WORKSPACE;
    if (R > 0) {
        // logits and their gradients have been compared above; here where they are dense, as others may stand between their strides
        const bool gdense = grad_logits && grad_logits != logits && g_extent == heads * V;
        const Span spans[] = {span(terms, 4 * CHAM_TERMS), span(logp, 4 * R), span(entropy, 4 * R), span(grad_values, 4 * R), span(workspace, need),
                              span(weights, 4 * R), span(old_logp, 4 * R), span(advantages, 4 * R), span(ref_logp, 4 * R), span(values, 4 * R),
                              span(old_values, 4 * R), span(returns, 4 * R), span(actions, heads * a.abytes),
                              span(logits, extent == heads * V ? extent * type_bytes(type) : 0)};
        if (shared(spans, 5)) return CHAM_E_BAD_DIM;
        const Span grad = span(gdense || (grad_logits == logits && extent == heads * V) ? grad_logits : nullptr, heads * V * type_bytes(type));
        for (int i = 0; i < 13; ++i)
            if (crosses(grad, spans[i])) return CHAM_E_BAD_DIM;
    }
    a.w_all = R > 0 ? 1.0 / (double)R : 0.0;
    // without decisions the pointer only says that this is a loss
    a.old_logp = old_logp ? old_logp : terms;
    a.adv = advantages;
    a.ref = ref_logp;
    a.values = values;
    a.old_values = old_values;
    a.returns = returns;
    a.lo = 1.0 - coef->clip_low;
    a.hi = 1.0 + coef->clip_high;
    a.c_value = coef->value;
    a.c_entropy = coef->entropy;
    a.c_kl = coef->kl;
    a.value_clip = coef->value_clip;
    a.terms = terms;
    a.grad_values = grad_values;
    const hipError_t h = launch_policy(a, type, workspace, reinterpret_cast<hipStream_t>(stream));
    return h == hipSuccess ? CHAM_OK : hip_fail(h);
}

int64_t cham_gae_workspace_bytes(int64_t B, int64_t S)
{
    if (B < 0 || S < 0 || S > 0x7fffffff || (S > 0 && B > kMostItems / S)) return CHAM_E_BAD_DIM;
    // the largest one: the query does not ask for the layout
    int64_t most = 0;
    for (int layout = kGaeDense; layout <= kGaeStrided; ++layout) {
        const int64_t n = plan_gae(B, S, layout).bytes;
        most = n > most ? n : most;
    }
    return most;
}

int32_t cham_gae(int32_t type, int64_t B, int64_t S, const void *rewards, int64_t r_ldb, int64_t r_lds,
                 const void *values, int64_t v_ldb, int64_t v_lds, const uint8_t *dones, int64_t d_ldb, int64_t d_lds,
                 const float *bootstrap, const int32_t *lengths, double gamma, double lambda,
                 float *advantages, float *returns, int64_t o_ldb, int64_t o_lds,
                 void *workspace, int64_t workspace_bytes, void *stream)
{
    if (!float_type(type)) return CHAM_E_BAD_TYPE;
    const int64_t need = cham_gae_workspace_bytes(B, S);
    if (need < 0) return (int32_t)need;
    if (!(gamma >= 0.0 && gamma <= 1.0) || !(lambda >= 0.0 && lambda <= 1.0)) return CHAM_E_BAD_COEF;
    if (B == 0 || S == 0) return CHAM_OK;
    if (!rewards || !values || !advantages) return CHAM_E_NULL;
    const int64_t ld[6] = {r_ldb, r_lds, v_ldb, v_lds, dones ? d_ldb : 0, dones ? d_lds : 0};
    for (int i = 0; i < 6; ++i)
        if (ld[i] < 0 || ld[i] > kMostItems) return CHAM_E_BAD_DIM;
    for (int i = 0; i < 6; i += 2) {
        int64_t eb, es;
        if (__builtin_mul_overflow(B - 1, ld[i], &eb) || __builtin_mul_overflow(S - 1, ld[i + 1], &es) || __builtin_add_overflow(eb, es, &eb) ||
            eb > ((int64_t)1 << 59))
            return CHAM_E_BAD_DIM;
    }
    int64_t extent;                                        // items from the first to behind the last output
    if (!apart(B, o_ldb, S, o_lds, 1, extent)) return CHAM_E_BAD_DIM;
    if (!aligned(rewards, type_bytes(type)) || !aligned(values, type_bytes(type)) || !aligned(bootstrap, 4) || !aligned(lengths, 4) ||
        !aligned(advantages, 4) || !aligned(returns, 4))
        return CHAM_E_BAD_DIM;
    if (!workspace_ok(workspace, workspace_bytes, need)) return CHAM_E_WORKSPACE;
    // Arrays without gaps are compared as a whole; others may lie between each other's strides and are compared where they begin.
    const int64_t n = B * S;
    const auto array = [&](const void *p, int64_t ldb, int64_t lds, int bytes) {
        return p ? span(p, bytes * ((B - 1) * ldb + (S - 1) * lds + 1 == n ? n : 1)) : Span{0, 0};       // strides of nothing are not looked at
    };
    const bool dense_out = extent == n;
    const Span out[] = {span(advantages, dense_out ? 4 * n : 4), span(returns, dense_out ? 4 * n : 4), span(workspace, need)};
    const Span in[] = {array(rewards, r_ldb, r_lds, type_bytes(type)), array(values, v_ldb, v_lds, type_bytes(type)), array(dones, d_ldb, d_lds, 1),
                       span(bootstrap, 4 * B), span(lengths, 4 * B)};
    if (shared(out, 3)) return CHAM_E_BAD_DIM;
    for (const Span &o : out)
        for (const Span &i : in)
            if (crosses(o, i)) return CHAM_E_BAD_DIM;
    // side by side: of rewards, values and outputs the same step of all trajectories stands closer together than the steps of one
    const bool dense = r_lds == 1 && v_lds == 1 && (!dones || d_lds == 1) && o_lds == 1;
    const int layout = B >= 8 && r_ldb < r_lds && v_ldb < v_lds && o_ldb < o_lds ? kGaeSide : dense ? kGaeDense : kGaeStrided;
    const GaePlan p = plan_gae(B, S, layout);
    GaeArgs a{};
    a.B = B;
    a.S = S;
    a.rewards = rewards;
    a.values = values;
    a.dones = dones;
    a.r_ldb = r_ldb;
    a.r_lds = r_lds;
    a.v_ldb = v_ldb;
    a.v_lds = v_lds;
    a.d_ldb = d_ldb;
    a.d_lds = d_lds;
    a.o_ldb = B > 1 ? o_ldb : 0;
    a.o_lds = S > 1 ? o_lds : 0;
    a.bootstrap = bootstrap;
    a.lengths = lengths;
    a.gamma = gamma;
    // a factor of 0 stands for an episode's end, and for nothing else: 1e-300 times an advantage is below what a float resolves
    const double gl = fmax(gamma * lambda, 1e-300), gl2 = gl * gl, gl4 = gl2 * gl2;
    a.gamma_lambda = gl;
    a.factor_eight = fmax(gl4 * gl4, 1e-300);
    a.adv = advantages;
    a.ret = returns;
    a.runs = static_cast<double2 *>(workspace);
    a.chunk = p.chunk;
    a.chunks = p.chunks;
    a.threads = p.threads;
    a.width = p.width;
    a.layout = layout;
    const hipError_t h = launch_gae(a, type, reinterpret_cast<hipStream_t>(stream));
    return h == hipSuccess ? CHAM_OK : hip_fail(h);
}

int64_t cham_grad_workspace_bytes(const int64_t *numels, const int32_t *types, int32_t n)
{
    if (n < 0) return CHAM_E_BAD_DIM;
    if (n > 0 && (!numels || !types)) return CHAM_E_NULL;
    int64_t all = 0;
    for (int32_t i = 0; i < n; ++i) {
        if (!float_type(types[i])) return CHAM_E_BAD_TYPE;
        if (numels[i] < 0 || numels[i] > kMostItems - all) return CHAM_E_BAD_DIM;
        all += numels[i];
    }
    return ((int64_t)grad_parts(numels, types, n) * 8 + 255) / 256 * 256;
}

static int32_t check_tensors(const void *const *p, const int64_t *numels, const int32_t *types, int32_t n)
{
    if (n > 0 && !p) return CHAM_E_NULL;
    for (int32_t i = 0; i < n; ++i) {
        if (numels[i] == 0) continue;
        if (!p[i]) return CHAM_E_NULL;
        if (!aligned(p[i], type_bytes(types[i]))) return CHAM_E_BAD_DIM;
    }
    return CHAM_OK;
}

int32_t cham_grad_norm(const void *const *grads, const int64_t *numels, const int32_t *types, int32_t n, double *norm,
                       void *workspace, int64_t workspace_bytes, void *stream)
{
    const int64_t need = cham_grad_workspace_bytes(numels, types, n);
    if (need < 0) return (int32_t)need;
    if (!norm) return CHAM_E_NULL;
    if (!aligned(norm, 8)) return CHAM_E_BAD_DIM;
    const int32_t e = check_tensors(grads, numels, types, n);
    if (e != CHAM_OK) return e;
    if (!workspace_ok(workspace, workspace_bytes, need)) return CHAM_E_WORKSPACE;
    const hipError_t h = launch_grad_norm(grads, numels, types, n, static_cast<double *>(workspace), grad_parts(numels, types, n), norm,
                                          reinterpret_cast<hipStream_t>(stream));
    return h == hipSuccess ? CHAM_OK : hip_fail(h);
}

int32_t cham_clip_grads(const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int32_t n,
                        double max_norm, double *norm, void *workspace, int64_t workspace_bytes, int32_t flags,
                        void *stream)
{
    if (flags & ~CHAM_F_NORM_GIVEN) return CHAM_E_BAD_FLAG;
    const int64_t need = cham_grad_workspace_bytes(numels, types, n);
    if (need < 0) return (int32_t)need;
    if (!norm) return CHAM_E_NULL;
    if (!aligned(norm, 8)) return CHAM_E_BAD_DIM;
    if (!(max_norm >= 0.0)) return CHAM_E_BAD_COEF;
    int32_t e = check_tensors(grads, numels, types, n);
    if (e == CHAM_OK && outs) e = check_tensors(outs, numels, types, n);
    if (e != CHAM_OK) return e;
    const bool given = (flags & CHAM_F_NORM_GIVEN) != 0;
    if (!given && !workspace_ok(workspace, workspace_bytes, need)) return CHAM_E_WORKSPACE;
    const hipStream_t s = reinterpret_cast<hipStream_t>(stream);
    double *parts = given ? nullptr : static_cast<double *>(workspace);
    const int n_parts = given ? 0 : grad_parts(numels, types, n);
    hipError_t h = hipSuccess;
    // the kernels that scale note the norm themselves, if there are any
    if (!given) h = launch_grad_norm(grads, numels, types, n, parts, n_parts, n_parts == 0 ? norm : nullptr, s);
    if (h == hipSuccess) h = launch_grad_clip(grads, outs, numels, types, n, max_norm, norm, parts, n_parts, s);
    return h == hipSuccess ? CHAM_OK : hip_fail(h);
}

}  // extern "C"
