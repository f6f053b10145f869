/* Driver for the launches of the agent's update (development check, built and run by the tests; not part of libcham): the HIP
 * entry points that a launch goes through are defined here and note its geometry, so that calls of any size go all the way
 * without a GPU.  A launch holds fewer than 2^32 threads a dimension, at least one workgroup, and its workspace is large
 * enough by the library's own answer.  Device pointers are placeholders that nothing looks behind. */
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "cham.h"

typedef struct {
    uint32_t x, y, z;
} dim3_t;

static dim3_t g_grid, g_block;
static size_t g_shared;
static void *g_stream;
static int launches, fails;
static uint32_t first_grid;                /* of a call */
static const char *what = "";

int __hipPushCallConfiguration(dim3_t grid, dim3_t block, size_t shared, void *stream)
{
    g_grid = grid;
    g_block = block;
    g_shared = shared;
    g_stream = stream;
    return 0;
}
int __hipPopCallConfiguration(dim3_t *grid, dim3_t *block, size_t *shared, void **stream)
{
    *grid = g_grid;
    *block = g_block;
    *shared = g_shared;
    *stream = g_stream;
    return 0;
}
int hipLaunchKernel(const void *kernel, dim3_t grid, dim3_t block, void **args, size_t shared, void *stream)
{
    (void)kernel, (void)args, (void)shared, (void)stream;
    if (launches++ == 0) first_grid = grid.x;
    const int ok = grid.x > 0 && block.x > 0 && block.x <= 1024 && (uint64_t)grid.x * block.x < (1ull << 32) && grid.y == 1 && grid.z == 1 &&
                   block.y == 1 && block.z == 1;
    if (!ok) {
        fprintf(stderr, "explore_launch_check: %s: %u workgroups of %u\n", what, grid.x, block.x);
        ++fails;
    }
    return ok ? 0 : 9;                     /* hipErrorInvalidConfiguration */
}
int hipGetLastError(void) { return 0; }
static int cus = 256;
int hipGetDevice(int *device)
{
    *device = 0;
    return 0;
}
int hipDeviceGetAttribute(int *value, int attribute, int device)
{
    (void)attribute, (void)device;         /* the library asks for the compute units alone */
    *value = cus;
    return 0;
}

static void *const kAt = (void *)(uintptr_t)0x100000;
#define AT(i) ((void *)((uintptr_t)(i) << 53))       /* arguments far apart */

static void expect(int32_t rc, int at_least)
{
    if (rc != CHAM_OK || launches < at_least) {
        fprintf(stderr, "explore_launch_check: %s: code %d, %d launches\n", what, rc, launches);
        ++fails;
    }
    launches = 0;
}

int main(void)
{
    char text[128];
    what = text;
    /* tensors: more than 2^32 threads' worth of chunks in one launch, in several, beside small ones */
    const int64_t sizes[] = {1, 16385, (int64_t)1 << 28, ((int64_t)1 << 37) - 1, ((int64_t)1 << 37) + 5, (int64_t)1 << 39, (int64_t)1 << 40};
    for (int i = 0; i < 7; ++i)
        for (int type = 0; type < 3; ++type)
            for (int n = 1; n <= 700; n = n * 24 + 1) {
                int64_t *numels = malloc(sizeof(int64_t) * (size_t)n);
                int32_t *types = malloc(sizeof(int32_t) * (size_t)n);
                const void **p = malloc(sizeof(void *) * (size_t)n);
                for (int k = 0; k < n; ++k) {
                    numels[k] = sizes[i] / n + (k % 3 == 0 && sizes[i] > n);
                    if (sizes[i] == ((int64_t)1 << 40)) numels[k] = sizes[i] / n;
                    types[k] = type;
                    p[k] = kAt;
                }
                const int64_t bytes = cham_grad_workspace_bytes(numels, types, n);
                snprintf(text, sizeof text, "gradients, %d of %lld items together, type %d", n, (long long)sizes[i], type);
                expect(cham_grad_norm(p, numels, types, n, kAt, kAt, bytes, 0), 1);
                expect(cham_clip_grads(p, NULL, numels, types, n, 1.0, kAt, kAt, bytes, 0, 0), 1);
                expect(cham_clip_grads(p, NULL, numels, types, n, 1.0, kAt, NULL, 0, CHAM_F_NORM_GIVEN, 0), sizes[i] >= n ? 1 : 0);
                free(numels);
                free(types);
                free(p);
            }
    const int64_t rows[] = {1, 17, 1025, 65537, (int64_t)1 << 31, (int64_t)1 << 34};
    const int32_t heads[] = {1, 3, 24, 300, 65536}, choices[] = {1, 3, 24, 100, 700, 9001, 70001, 1 << 24};
    const cham_policy_coef c = {0.2, 0.2, 0.5, 0.1, 0.1, 0.2};
    for (int i = 0; i < 6; ++i)
        for (int j = 0; j < 5; ++j)
            for (int k = 0; k < 8; ++k)
                for (int type = 0; type < 3; ++type) {
                    const int64_t R = rows[i], V = choices[k], G = heads[j];
                    if (R > ((int64_t)1 << 40) / G || (double)R * (double)G * (double)V > 1e15) continue;
                    const int64_t bytes = cham_policy_workspace_bytes(R, (int32_t)G, (int32_t)V, type, 1);
                    snprintf(text, sizeof text, "policy %lld x %lld x %lld, type %d", (long long)R, (long long)G, (long long)V, type);
                    expect(cham_policy_logp(AT(1), type, R, (int32_t)G, (int32_t)V, G * V, V, AT(2), CHAM_TYPE_I8, 0, 0, AT(3), AT(4), AT(5), bytes, 0), 1);
                    for (int grad = 0; grad < 2; ++grad)
                        expect(cham_policy_loss(AT(1), type, R, (int32_t)G, (int32_t)V, G * V, V, AT(2), CHAM_TYPE_I8, 0, 0, AT(3), AT(4), AT(5), AT(6), AT(7),
                                                AT(8), &c, AT(9), AT(10), AT(11), grad ? AT(12) : 0, G * V, V, grad ? AT(13) : 0, AT(14), bytes, 0), 1);
                }
    const int64_t trajectories[] = {1, 9, 700, 100003, (int64_t)1 << 33}, steps[] = {1, 100, 513, 9000, 2000003, 0x7fffffff};
    for (int i = 0; i < 5; ++i)
        for (int j = 0; j < 6; ++j)
            for (int side = 0; side < 3; ++side) {
                const int64_t B = trajectories[i], S = steps[j], b = side == 0 ? S : side == 1 ? 1 : 2 * S, s = side == 0 ? 1 : side == 1 ? B : 2;
                if (B > ((int64_t)1 << 40) / S) continue;
                const int64_t bytes = cham_gae_workspace_bytes(B, S);
                snprintf(text, sizeof text, "advantages %lld x %lld, strides %lld %lld", (long long)B, (long long)S, (long long)b, (long long)s);
                expect(cham_gae(0, B, S, AT(1), b, s, AT(2), b, s, AT(3), b, s, AT(4), AT(5), 0.9, 0.9, AT(6), AT(7), b, s, AT(8), bytes, 0), 1);
            }
    /* rows that stay in a workgroup: as many workgroups as the device's units hold */
    const int32_t rows_of[] = {1000, 8191, 32768, 131072};
    for (int i = 0; i < 4; ++i) {
        uint32_t grids[3];
        const int units[3] = {256, 32, 512};
        for (int k = 0; k < 3; ++k) {
            cus = units[k];
            const int64_t bytes = cham_policy_workspace_bytes(100000, 1, rows_of[i], CHAM_TYPE_BF16, 1);
            snprintf(text, sizeof text, "rows of %d on %d units", rows_of[i], cus);
            expect(cham_policy_loss(AT(1), CHAM_TYPE_BF16, 100000, 1, rows_of[i], rows_of[i], 0, AT(2), CHAM_TYPE_I32, 0, 0, AT(3), AT(4), AT(5), AT(6), AT(7), AT(8),
                                    &c, AT(9), AT(10), AT(11), AT(12), rows_of[i], 0, AT(13), AT(14), bytes, 0), 2);
            grids[k] = first_grid;
        }
        if (grids[0] != 8 * grids[1] || grids[2] != grids[0] || (int64_t)grids[0] * 40 > cham_policy_workspace_bytes(100000, 1, rows_of[i], CHAM_TYPE_BF16, 1)) {
            fprintf(stderr, "explore_launch_check: rows of %d: %u, %u, %u workgroups\n", rows_of[i], grids[0], grids[1], grids[2]);
            ++fails;
        }
    }
    cus = 256;
    if (fails) return 1;
    printf("explore_launch_check ok\n");
    return 0;
}
