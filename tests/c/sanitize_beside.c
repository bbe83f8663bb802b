/* The host code of norms with rotary positions, token probabilities and pages under -fsanitize=address,undefined (see sanitize_step.c): size functions at the
 * edges of their ranges, and launching calls that are refused before any device call. tests/test_beside_sanitizers.py compares the values. */
#include <stdio.h>

#include "loza_ssa.h"

int main(void)
{
    const int big[] = {1, 2, 63, 64, 65, 1024, 65535, 65536, 2147483647};
    const int64_t far[] = {1, 2, 64, 8192, 2147483519LL, 2147483647LL, INT64_MAX};
    long long acc = 0;
    for (int a = 0; a < 9; ++a)
        for (int b = 0; b < 9; ++b)
            for (int c = 0; c < 9; ++c) {
                acc += (long long)(loza_ssa_token_probs_workspace_bytes(big[a], big[b], big[c]) % 1000);
                for (int x = 0; x < 7; ++x) acc += (long long)(loza_ssa_norm_rope_backward_workspace_bytes(far[x], big[a], big[b], big[c]) % 1000);
            }
    for (int x = 0; x < 7; ++x) acc += (long long)(loza_ssa_pages_free_workspace_bytes(far[x]) % 1000 + loza_ssa_pages_compact_workspace_bytes(far[x]) % 1000);
    printf("edges %lld\n", acc);
    char buf[96];
    void *p = (void *)(((uintptr_t)buf + 15) & ~(uintptr_t)15);
    int32_t *i = (int32_t *)p;
    float *f = (float *)p;
    const int m1 = 2147483647;
    const int64_t m2 = INT64_MAX;
    printf("refused %d %d %d %d %d %d %d %d %d\n",
           loza_ssa_norm_rope(p, f, i, (double *)p, p, m1, m1, m1, m2, m2, m2, m2, m1, m1, 1.0f, m1, 64, 1, 1.0f, NULL),
           loza_ssa_norm_rope(p, f, i, (double *)p, (char *)p + 2, m1, 1, 64, m2, 0, m2, m2, 0, 64, 1.0f, 0, 64, 1, 1.0f, NULL),
           loza_ssa_norm_rope_backward(p, p, f, i, (double *)p, p, f, m1, m1, m1, m2, m2, m2, m2, m2, m2, m1, m1, 1.0f, m1, 64, 1, 1.0f, p, (size_t)-1, NULL),
           loza_ssa_norm_rope_append(p, f, (char *)p + 2, f, (char *)p + 4, i, i, (double *)p, p, p, p, m1, m1, m1, m1, m1, m1, m2, m2, m2, m2, m2, m2, m2, m2, m2, m1, m1, m1, m1, 1.0f, m1, m1,
                                     64, 1, 1.0f, NULL),
           loza_ssa_token_probs(p, m2, i, i, (int64_t *)p, (uint16_t *)p, m2, f, f, f, f, i, f, m1, i, f, m1, m1, m1, p, (size_t)-1, NULL),
           loza_ssa_count_tokens(i, i, i, i, i, (uint16_t *)p, m2, m1, m1, m1, NULL),
           loza_ssa_pages_fork(i, i, i, i, i, i, i, i, m1, m2, m2, 64, m1, m2, m2, i, i, i, i, i, i, i, i, i, NULL),
           loza_ssa_pages_copy(p, NULL, i, i, i, i, m2, m1, m2, m1, m2, m2, NULL),
           loza_ssa_pages_compact(i, i, i, i, m1, m2, m2, m1, i, i, i, i, i, i, i, p, (size_t)-1, NULL));
    /* within all limits but that results lie on each other */
    printf("overlap %d %d\n",
           loza_ssa_pages_fork(i, i, i, i, i, i, i, i, 65536, 2147483647LL, 2147483647LL, 32, 60000000, m2, m2, i, i, i, i, i, i, i, i, i, NULL),
           loza_ssa_pages_free(i, i, i, i, i, i, i, i, 65536, 2147483647LL, 2147483647LL, 32, 60000000, m2, m2, m2, i, i, i, i, i, p, (size_t)-1, NULL));
    return 0;
}
