// Host/device shared declarations of the agent's update (policy loss, advantages, gradient norm).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace cham {

int32_t hip_fail(hipError_t e);        // notes the code for cham_last_hip_error, returns CHAM_E_HIP

constexpr int kPolicySums = 5;         // policy, value, entropy, kl, clipped

// Arguments of the policy kernels.  Pointers are device pointers; those of a loss are null for log-probabilities alone.
struct PolicyArgs {
    const void *logits;
    int64_t R;
    int G, V;
    int64_t ld_r, ld_g;
    const void *actions;           // [R][G] of abytes bytes each, signed
    int abytes;
    int64_t first;
    const float *weights;          // or null: w_all each
    double w_all;
    const float *old_logp;         // null: no loss
    const float *adv, *ref, *values, *old_values, *returns;
    double lo, hi;                 // the ratio counts within
    double c_value, c_entropy, c_kl, value_clip;
    float *terms, *logp, *entropy;
    void *grad;
    int64_t gld_r, gld_g;
    float *grad_values;
    double *sums;                  // [blocks][kPolicySums] partial sums of the terms
    float *part;                   // [R*G][splits][4] maximum, sum of exponentials, sum of exponential x exponent, logit of the action (in its part)
    float4 *head;                  // [R*G] maximum, sum of exponentials, entropy, choice of the action (int bits; negative: left out)
    float2 *dec;                   // [R] derivative by the log-probability, factor of the entropy's derivative
};

// How a call is run; a function of its sizes and type alone, so that the workspace can be asked for ahead of it.
struct PolicyPlan {
    int lanes;                     // up to 64 choices a head: lanes of a decision, four heads each up to four choices; 0 elsewhere
    int tile;                      // few choices a head: decisions of a tile; 0 elsewhere
    int row, threads;              // one head: 16-byte pieces of a row that each of so many threads holds; 0 elsewhere
    int group;                     // several heads of many decisions: lanes that take one at a time; 0 elsewhere
    int splits;                    // workgroups a head is split over
    int chunk;                     // choices each of them takes
    int64_t o_sums, o_part, o_head, o_dec, bytes;
};
PolicyPlan plan_policy(int64_t R, int G, int V, int type, bool grad);
hipError_t launch_policy(PolicyArgs a, int type, void *workspace, hipStream_t s);

struct GaeArgs {
    int64_t B, S;
    const void *rewards, *values;
    const uint8_t *dones;
    int64_t r_ldb, r_lds, v_ldb, v_lds, d_ldb, d_lds, o_ldb, o_lds;
    const float *bootstrap;
    const int *lengths;
    double gamma, gamma_lambda, factor_eight;      // gamma, gamma lambda, its eighth power
    float *adv, *ret;
    double2 *runs;                 // what a chunk makes of the advantage behind it: factor, summand; [B][chunks], side by side [chunks][B]
    int64_t chunk;                 // steps of a chunk (S rounded up: one chunk)
    int chunks;
    int threads;                   // of a workgroup's trajectories
    int width;                     // trajectories side by side in a wave
    int layout;
};
// How trajectories lie in memory: the steps of each one run of items, the same step of all, or neither.
constexpr int kGaeDense = 0, kGaeSide = 1, kGaeStrided = 2;
struct GaePlan {
    int threads, width, chunks;
    int64_t chunk, bytes;
};
GaePlan plan_gae(int64_t B, int64_t S, int layout);
hipError_t launch_gae(const GaeArgs &a, int type, hipStream_t s);

int grad_parts(const int64_t *numels, const int32_t *types, int n);     // partial sums a norm needs room for
hipError_t launch_grad_norm(const void *const *grads, const int64_t *numels, const int32_t *types, int n, double *parts, int n_parts,
                            double *norm, hipStream_t s);
hipError_t launch_grad_clip(const void *const *grads, void *const *outs, const int64_t *numels, const int32_t *types, int n,
                            double max_norm, double *norm, const double *parts, int n_parts, hipStream_t s);

}  // namespace cham
