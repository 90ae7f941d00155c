/* oracle_delta_f64 on buffers of exact size for a sanitizer build: ordinary,
 * empty and single-element shapes, with and without gates and outputs; a prefix
 * and its continuation equal the whole.  Test infrastructure only. */
#include <math.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

int oracle_delta_f64(int64_t T, int64_t Hk, int64_t Hv, int64_t K, int64_t V, const double *q, const double *k,
                     const double *v, const double *g, const double *beta, double *S, double *o, int norm,
                     double eps, double scale);

static int failures = 0;
#define CHECK(c)                                                            \
    do {                                                                    \
        if (!(c)) {                                                         \
            fprintf(stderr, "check failed at line %d: %s\n", __LINE__, #c); \
            ++failures;                                                     \
        }                                                                   \
    } while (0)

static uint64_t state = 88172645463325252ull;
static double rnd(void)
{
    state ^= state << 13;
    state ^= state >> 7;
    state ^= state << 17;
    return (double)(state >> 11) / 9007199254740992.0 - 0.5;
}
static double *draw(int64_t n)
{
    double *p = (double *)malloc(sizeof(double) * (n > 0 ? n : 1));
    for (int64_t i = 0; i < n; ++i)
        p[i] = rnd();
    return p;
}

static void run(int64_t T, int64_t Hk, int64_t Hv, int64_t K, int64_t V, int gates, int out)
{
    double *q = draw(T * Hk * K), *k = draw(T * Hk * K), *v = draw(T * Hv * V), *g = draw(T * Hv), *b = draw(T * Hv);
    double *S = draw(Hv * K * V), *S2 = draw(Hv * K * V), *o = draw(T * Hv * V), *o2 = draw(T * Hv * V);
    memcpy(S2, S, sizeof(double) * Hv * K * V);
    for (int64_t i = 0; i < T * Hv; ++i)
        g[i] = -fabs(g[i]);
    CHECK(oracle_delta_f64(T, Hk, Hv, K, V, q, k, v, gates ? g : NULL, gates ? b : NULL, S, out ? o : NULL, 1, 1e-6,
                           1.0) == 0);
    const int64_t h = T / 2;
    CHECK(oracle_delta_f64(h, Hk, Hv, K, V, q, k, v, gates ? g : NULL, gates ? b : NULL, S2, out ? o2 : NULL, 1, 1e-6,
                           1.0) == 0);
    CHECK(oracle_delta_f64(T - h, Hk, Hv, K, V, q + h * Hk * K, k + h * Hk * K, v + h * Hv * V,
                           gates ? g + h * Hv : NULL, gates ? b + h * Hv : NULL, S2, out ? o2 + h * Hv * V : NULL, 1,
                           1e-6, 1.0) == 0);
    CHECK(memcmp(S, S2, sizeof(double) * Hv * K * V) == 0);
    CHECK(!out || memcmp(o, o2, sizeof(double) * T * Hv * V) == 0);
    free(q); free(k); free(v); free(g); free(b); free(S); free(S2); free(o); free(o2);
}

int main(void)
{
    for (int gates = 0; gates < 2; ++gates)
        for (int out = 0; out < 2; ++out) {
            run(9, 2, 4, 5, 3, gates, out);
            run(1, 1, 1, 1, 1, gates, out);
            run(0, 1, 3, 4, 2, gates, out);
        }
    CHECK(oracle_delta_f64(1, 2, 3, 1, 1, NULL, NULL, NULL, NULL, NULL, NULL, NULL, 0, 0, 1) == 1);
    if (failures)
        return 1;
    puts("all checks passed");
    return 0;
}
