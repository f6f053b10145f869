/* Driver for a sanitizer build of the host code behind the agent's update (development check, built and run by the tests;
 * not part of libcham): workspace queries over wide ranges, and calls that stop at an argument or at the workspace.  Nothing
 * reaches a kernel launch; device pointers are placeholders. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include "cham.h"

static int fails = 0;
#define EXPECT(cond)                                                               \
    do {                                                                           \
        if (!(cond)) {                                                             \
            fprintf(stderr, "explore_host_check: line %d: %s\n", __LINE__, #cond); \
            ++fails;                                                               \
        }                                                                          \
    } while (0)

int main(void)
{
    float *f = (float *)(uintptr_t)0x100000;
    double *d = (double *)(uintptr_t)0x200000;
    const int64_t rows[] = {0, 1, 2, 63, 4096, 64000, (int64_t)1 << 24};
    const int32_t heads[] = {1, 2, 24, 65536}, choices[] = {1, 2, 3, 64, 65, 1000, 50021, 131072, 1 << 24};
    for (int i = 0; i < 7; ++i)
        for (int j = 0; j < 4; ++j)
            for (int k = 0; k < 9; ++k)
                for (int type = 0; type < 3; ++type) {
                    const int64_t a = cham_policy_workspace_bytes(rows[i], heads[j], choices[k], type, 0);
                    const int64_t b = cham_policy_workspace_bytes(rows[i], heads[j], choices[k], type, 1);
                    EXPECT(a >= 0 && b >= a);
                }
    EXPECT(cham_policy_workspace_bytes((int64_t)1 << 62, 65536, 1, 0, 0) == CHAM_E_BAD_DIM);
    cham_policy_coef c = {0.2, 0.2, 0.0, 0.0, 0.0, 0.0};
    EXPECT(cham_policy_loss(f, 0, INT64_MAX, 2, 3, INT64_MAX, INT64_MAX, f, 16, INT64_MIN, 0, f, f, 0, 0, 0, 0, &c, f, f, f, 0, 0, 0, 0, 0, 0, 0) ==
           CHAM_E_BAD_DIM);
    EXPECT(cham_policy_loss(f, 0, 5, 2, 3, INT64_MAX, INT64_MAX, f, 16, INT64_MIN, 0, f, f, 0, 0, 0, 0, &c, f, f, f, 0, 0, 0, 0, 0, 0, 0) ==
           CHAM_E_BAD_DIM);
    for (int64_t B = 0; B < ((int64_t)1 << 34); B = 3 * B + 1)
        for (int64_t S = 0; S <= 0x7fffffff; S = 5 * S + 1) {
            const int64_t n = cham_gae_workspace_bytes(B, S);
            EXPECT(n >= 0 || (n == CHAM_E_BAD_DIM && (double)B * (double)S > 1e12));
        }
    EXPECT(cham_gae(0, 3, 4, f, INT64_MAX, 1, f, 1, 3, 0, 0, 0, 0, 0, 0.5, 0.5, f, f, 1, 3, 0, 0, 0) == CHAM_E_BAD_DIM);
    for (int n = 0; n <= 3000; n = n * 2 + 1) {
        int64_t *numels = (int64_t *)malloc(sizeof(int64_t) * (size_t)(n + 1));
        int32_t *types = (int32_t *)malloc(sizeof(int32_t) * (size_t)(n + 1));
        const void **p = (const void **)malloc(sizeof(void *) * (size_t)(n + 1));
        for (int i = 0; i < n; ++i) {
            numels[i] = i % 5 == 0 ? 0 : i % 5 == 1 ? (int64_t)1 << 28 : i;
            types[i] = i % 3;
            p[i] = numels[i] ? f : NULL;
        }
        const int64_t need = cham_grad_workspace_bytes(numels, types, n);
        EXPECT(need >= 0 && need <= 8 * (1024 + (int64_t)n) * 2 + 256);
        if (need > 0) {
            EXPECT(cham_grad_norm(p, numels, types, n, d, NULL, need, 0) == CHAM_E_WORKSPACE);
            EXPECT(cham_clip_grads(p, NULL, numels, types, n, 1.0, d, f, need - 1, 0, 0) == CHAM_E_WORKSPACE);
        }
        EXPECT(cham_clip_grads(p, NULL, numels, types, n, NAN, d, f, need, 0, 0) == CHAM_E_BAD_COEF);
        free(numels);
        free(types);
        free(p);
    }
    if (fails) return 1;
    printf("explore_host_check ok\n");
    return 0;
}
