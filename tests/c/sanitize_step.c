/* The host code of the calls around the attention under -fsanitize=address,undefined (see sanitize_host.c): size functions at the edges of their
 * ranges, and launching calls that are refused before any device call. tests/test_step_sanitizers.py compares the values with the ordinary build's. */
#include <stdio.h>

#include "loza_ssa.h"

int main(void)
{
    const int big[] = {1, 2, 63, 64, 65, 65536, 2147483647};
    const int64_t far[] = {1, 64, 8192, 2147483519LL, INT64_MAX};
    long long acc = 0;
    for (int b = 0; b < 7; ++b)
        for (int h = 0; h < 7; ++h)
            for (int n = 0; n < 7; ++n)
                for (int x = 0; x < 5; ++x) {
                    for (int wide = 0; wide < 2; ++wide) {
                        int k = 0;
                        const int d = wide ? 576 : 128;
                        acc += loza_ssa_extend_tree_kernel(big[b], big[h], 1, far[x], big[n], d, far[(x + b) % 5], far[(x + h) % 5], far[(x + n) % 5], b & 1, &k) + k;
                        acc += (long long)(loza_ssa_extend_tree_workspace_bytes(big[b], big[h], big[h], far[x], big[n], d, wide ? 512 : 128, far[(x + b) % 5],
                                                                                far[(x + h) % 5], far[(x + n) % 5]) % 1000);
                    }
                    acc += (long long)(loza_ssa_verify_tree_workspace_bytes(big[b], big[n], big[h]) % 1000);
                }
    printf("edges %lld\n", acc);
    char buf[96];
    void *p = (void *)(((uintptr_t)buf + 15) & ~(uintptr_t)15);
    int32_t *i = (int32_t *)p;
    double freq[512];
    float m = 0;
    const int m1 = 2147483647;
    const int64_t m2 = INT64_MAX;
    printf("frequencies %d %d %d", loza_ssa_rope_frequencies(1024, 1e300, 1e300, m2, 0.0, 1e300, freq, &m), loza_ssa_rope_frequencies(m1, 2, 1, 0, 0, 0, freq, &m),
           loza_ssa_rope_frequencies(64, 1e4, 32, 32768, 1, 32, freq, &m));
    printf(" %.17g %.9g\n", freq[31], (double)m);
    printf("refused %d %d %d %d %d %d %d %d %d\n",
           loza_ssa_step_tables(i, i, i, i, i, i, m1, 8, 8, 8, 64, 8, i, i, i, i, (int64_t *)p, i, NULL),
           loza_ssa_step_tables(i, i, NULL, i, i, i, 8, m1, 8, m2, 64, m1, i, i, i, i, NULL, i, NULL),
           loza_ssa_rope(p, i, (double *)p, p, m1, m1, m1, m2, m2, m2, m2, m1, 64, 1, 0, 1.0f, NULL),
           loza_ssa_rope(p, i, (double *)p, (char *)p + 2, m1, 1, 64, m2, 0, m2, m2, 0, 64, 1, 0, 1.0f, NULL),
           loza_ssa_rope(p, i, (double *)p, (char *)p + 2, 3, 8, 64, 0, 0, m2 / 4, m2 / 4, 0, 64, 1, 0, 1.0f, NULL),
           loza_ssa_rope_append(p, (char *)p + 2, (char *)p + 4, i, i, (double *)p, p, p, p, m1, m1, m1, m1, m1, m1, m2, m2, m2, m2, m2, m2, m2, m2, m2, 0, 0, 64, 1, 1.0f, NULL),
           loza_ssa_extend_tree(p, p, p, i, i, i, (int64_t *)p, p, (float *)p, m1, m1, 1, m2, m2, m1, m1, 64, 576, 512, m2, m2, m2, 1.0f, p, 16, NULL),
           loza_ssa_verify_tree((float *)p, NULL, i, i, i, (float *)p, (float *)p, i, i, i, m1, 64, m1, p, 16, NULL),
           loza_ssa_keep_accepted(p, NULL, i, i, i, m1, 64, m1, m2, m2, m2, NULL));
    return 0;
}
