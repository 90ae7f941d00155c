/*
 * PRECOG reference oracle -- TEST INFRASTRUCTURE ONLY.
 *
 * Plain, slow, sequential fp64 implementations of what the GPU path computes.
 * Only the test suite, the smoke check and the benchmark's CPU-baseline leg
 * may load this library.  It shares no code, header, table or constant with
 * the HIP kernels under paper_2608_02560_amd/csrc.
 *
 * Every input arrives as fp64 (the caller widens bf16 / fp16 / fp32 values,
 * which is exact).  No -ffast-math: libm exp() is called as is.
 *
 * Functions
 *   oracle_scan_f64     Eq. 1 (Sec. 3) rolled over the sequence as in the
 *                       rollout S(h, x_1:T) of App. A, with the final state
 *                       captured (Sec. 4.2, offline indexing) and the gated
 *                       readout y = (C_t . h_t + Dskip x_t) * silu(z_t).
 *   oracle_top1_f64     Cosine top-1 over unit-norm keys (Sec. 4.2, query-time
 *                       injection): fp64 inner products summed in index order,
 *                       argmax with the lowest index winning ties.
 *   oracle_trajectory_f64  SMC per-step trajectory (Sec. 5.1, Eq. smc-trajectory)
 *                       thinned by the fidelity dial K (Sec. 5.2): every k-th
 *                       state h_k, h_2k, ... plus nothing else.
 *   oracle_scan_complex_f64  Eq. 1 with the diagonal complex A of Sec. 3,
 *                       A_k = a_k + i w_k (a_k > 0 in this sign convention):
 *                       complex state, real input term, readout of the real
 *                       part of C_t . h_t.
 *   oracle_delta_f64    the gated delta rule over one sequence, from and to
 *                       matrix states.
 *
 * Rows (b, d) of the scan are independent (the recurrence is diagonal in the
 * state, Eq. 1), so the driver may hand disjoint row ranges to threads; each
 * row is still computed strictly in time order.
 */
#include <complex.h>
#include <math.h>
#include <pthread.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

/* ------------------------------------------------------------------------- */
/* Selective-SSM scan                                                         */
/* ------------------------------------------------------------------------- */

typedef struct {
    int64_t B, L, D, N;
    const double *x, *dt, *A, *Bm, *Cm, *z, *Dskip, *h0;
    double *y, *hT;
    int64_t row_begin, row_end; /* rows r = b*D + d */
} scan_job;

/* One (b, d) row: the recurrence of Eq. 1 with real, positive A (decay
 * exp(-dt*A) < 1, the stable reading), rolled from h0 over t = 0..L-1.
 * h_t is the state after token t; y_t reads h_t. */
static void scan_row(const scan_job *j, int64_t b, int64_t d, double *h)
{
    const int64_t L = j->L, D = j->D, N = j->N;
    for (int64_t n = 0; n < N; ++n)
        h[n] = j->h0 ? j->h0[(b * D + d) * N + n] : 0.0;

    for (int64_t t = 0; t < L; ++t) {
        const int64_t td = (b * L + t) * D + d; /* [B, L, D] */
        const int64_t tn = (b * L + t) * N;     /* [B, L, N] */
        const double dt = j->dt[td];
        const double xv = j->x[td];
        for (int64_t n = 0; n < N; ++n) {
            const double decay = exp(-dt * j->A[d * N + n]);
            h[n] = decay * h[n] + j->Bm[tn + n] * xv * dt;
        }
        if (j->y) {
            double acc = 0.0;
            for (int64_t n = 0; n < N; ++n)
                acc += j->Cm[tn + n] * h[n];
            double out = acc + (j->Dskip ? j->Dskip[d] * xv : 0.0);
            if (j->z) {
                const double zv = j->z[td];
                out *= zv / (1.0 + exp(-zv)); /* silu */
            }
            j->y[td] = out;
        }
    }
    if (j->hT)
        for (int64_t n = 0; n < N; ++n)
            j->hT[(b * D + d) * N + n] = h[n];
}

static void *scan_worker(void *arg)
{
    const scan_job *j = (const scan_job *)arg;
    double *h = (double *)malloc((size_t)j->N * sizeof(double));
    if (!h)
        return (void *)1;
    for (int64_t r = j->row_begin; r < j->row_end; ++r)
        scan_row(j, r / j->D, r % j->D, h);
    free(h);
    return NULL;
}

/* Returns 0 on success, nonzero on bad arguments or allocation failure.
 * Layouts (row-major, last index fastest):
 *   x, dt, z, y : [B, L, D]     A : [D, N]     Bm, Cm : [B, L, N]
 *   Dskip : [D]                 h0, hT : [B, D, N]
 * z, Dskip, h0, y, hT may be NULL (no gate / zero skip / zero state /
 * no readout / no capture). */
int oracle_scan_f64(int64_t B, int64_t L, int64_t D, int64_t N,
                    const double *x, const double *dt, const double *A,
                    const double *Bm, const double *Cm, const double *z,
                    const double *Dskip, const double *h0, double *y,
                    double *hT, int nthreads)
{
    if (B < 0 || L < 0 || D < 0 || N <= 0)
        return 1;
    if ((L > 0 && (!x || !dt || !Bm)) || !A)
        return 2;
    if (y && L > 0 && !Cm)
        return 3;
    const int64_t rows = B * D;
    if (nthreads < 1)
        nthreads = 1;
    if (nthreads > rows)
        nthreads = rows > 0 ? (int)rows : 1;

    scan_job base = {B, L, D, N, x, dt, A, Bm, Cm, z, Dskip, h0, y, hT, 0, 0};
    if (nthreads == 1) {
        base.row_begin = 0;
        base.row_end = rows;
        return scan_worker(&base) ? 4 : 0;
    }
    pthread_t *th = (pthread_t *)malloc(sizeof(pthread_t) * nthreads);
    scan_job *jobs = (scan_job *)malloc(sizeof(scan_job) * nthreads);
    if (!th || !jobs) {
        free(th);
        free(jobs);
        return 4;
    }
    int rc = 0;
    for (int i = 0; i < nthreads; ++i) {
        jobs[i] = base;
        jobs[i].row_begin = rows * i / nthreads;
        jobs[i].row_end = rows * (i + 1) / nthreads;
        pthread_create(&th[i], NULL, scan_worker, &jobs[i]);
    }
    for (int i = 0; i < nthreads; ++i) {
        void *ret = NULL;
        pthread_join(th[i], &ret);
        if (ret)
            rc = 4;
    }
    free(th);
    free(jobs);
    return rc;
}

/* ------------------------------------------------------------------------- */
/* Complex diagonal A                                                         */
/* ------------------------------------------------------------------------- */

/* h_t[n] = exp(-dt_t (a[n] + i w[n])) h_{t-1}[n] + B_t[n] x_t dt_t   (complex)
 * y_t    = (sum_n C_t[n] Re(h_t[n]) + Dskip x_t) * silu(z_t)
 * h0, hT : [B, D, N, 2] with (real, imaginary) interleaved; h0 NULL = 0.
 * Arguments otherwise as oracle_scan_f64 (y and hT may be NULL). */
int oracle_scan_complex_f64(int64_t B, int64_t L, int64_t D, int64_t N,
                            const double *x, const double *dt, const double *Are,
                            const double *Aim, const double *Bm, const double *Cm,
                            const double *z, const double *Dskip, const double *h0,
                            double *y, double *hT)
{
    if (B < 0 || L < 0 || D < 0 || N <= 0 || !Are || !Aim)
        return 1;
    if (L > 0 && (!x || !dt || !Bm))
        return 2;
    if (y && L > 0 && !Cm)
        return 3;
    double complex *h = (double complex *)malloc((size_t)N * sizeof(double complex));
    if (!h)
        return 4;
    for (int64_t b = 0; b < B; ++b)
        for (int64_t d = 0; d < D; ++d) {
            for (int64_t n = 0; n < N; ++n) {
                const int64_t o = ((b * D + d) * N + n) * 2;
                h[n] = h0 ? h0[o] + I * h0[o + 1] : 0.0;
            }
            for (int64_t t = 0; t < L; ++t) {
                const int64_t td = (b * L + t) * D + d;
                const int64_t tn = (b * L + t) * N;
                for (int64_t n = 0; n < N; ++n) {
                    const double complex A = Are[d * N + n] + I * Aim[d * N + n];
                    h[n] = cexp(-dt[td] * A) * h[n] + Bm[tn + n] * x[td] * dt[td];
                }
                if (y) {
                    double acc = 0.0;
                    for (int64_t n = 0; n < N; ++n)
                        acc += Cm[tn + n] * creal(h[n]);
                    double out = acc + (Dskip ? Dskip[d] * x[td] : 0.0);
                    if (z) {
                        const double zv = z[td];
                        out *= zv / (1.0 + exp(-zv));
                    }
                    y[td] = out;
                }
            }
            if (hT)
                for (int64_t n = 0; n < N; ++n) {
                    const int64_t o = ((b * D + d) * N + n) * 2;
                    hT[o] = creal(h[n]);
                    hT[o + 1] = cimag(h[n]);
                }
        }
    free(h);
    return 0;
}

/* ------------------------------------------------------------------------- */
/* SMC trajectory with the fidelity dial                                      */
/* ------------------------------------------------------------------------- */

/* Keeps h_t for every t with (t + 1) % k == 0, i.e. the states after tokens
 * k, 2k, ... (1-based), as in "every k-th state is retained".  k = 1 keeps
 * the whole trajectory (K = N_c); k = L keeps only the final state (K = 1).
 * traj : [B, floor(L / k), D, N].  Same recurrence as oracle_scan_f64. */
int oracle_trajectory_f64(int64_t B, int64_t L, int64_t D, int64_t N, int64_t k,
                          const double *x, const double *dt, const double *A,
                          const double *Bm, const double *h0, double *traj)
{
    if (B < 0 || L < 0 || D < 0 || N <= 0 || k <= 0 || !A)
        return 1;
    const int64_t K = L / k;
    double *h = (double *)malloc((size_t)N * sizeof(double));
    if (!h)
        return 4;
    for (int64_t b = 0; b < B; ++b)
        for (int64_t d = 0; d < D; ++d) {
            for (int64_t n = 0; n < N; ++n)
                h[n] = h0 ? h0[(b * D + d) * N + n] : 0.0;
            for (int64_t t = 0; t < L; ++t) {
                const int64_t td = (b * L + t) * D + d;
                const int64_t tn = (b * L + t) * N;
                for (int64_t n = 0; n < N; ++n)
                    h[n] = exp(-dt[td] * A[d * N + n]) * h[n] +
                           Bm[tn + n] * x[td] * dt[td];
                if ((t + 1) % k == 0) {
                    const int64_t s = (t + 1) / k - 1;
                    if (s < K)
                        for (int64_t n = 0; n < N; ++n)
                            traj[((b * K + s) * D + d) * N + n] = h[n];
                }
            }
        }
    free(h);
    return 0;
}

/* ------------------------------------------------------------------------- */
/* Cosine top-1 retrieval                                                     */
/* ------------------------------------------------------------------------- */

typedef struct {
    int64_t M, E;
    const float *q, *K;
    int32_t *idx;
    double *best;
    int64_t q_begin, q_end;
} top1_job;

static void *top1_worker(void *arg)
{
    const top1_job *j = (const top1_job *)arg;
    for (int64_t qi = j->q_begin; qi < j->q_end; ++qi) {
        const float *qv = j->q + qi * j->E;
        double best = -INFINITY;
        int64_t arg_best = -1;
        for (int64_t i = 0; i < j->M; ++i) {
            const float *kv = j->K + i * j->E;
            double s = 0.0;
            for (int64_t e = 0; e < j->E; ++e)
                s += (double)qv[e] * (double)kv[e];
            if (arg_best < 0 || s > best) { /* strict: earliest index keeps ties */
                best = s;
                arg_best = i;
            }
        }
        j->idx[qi] = (int32_t)arg_best;
        if (j->best)
            j->best[qi] = best;
    }
    return NULL;
}

/* q : [Q, E] fp32, K : [M, E] fp32 (unit-norm rows, so the inner product is
 * the cosine).  idx[q] = smallest i attaining the maximum fp64 score;
 * best (nullable) receives that score.  M = 0 gives idx = -1. */
int oracle_top1_f64(int64_t Q, int64_t M, int64_t E, const float *q,
                    const float *K, int32_t *idx, double *best, int nthreads)
{
    if (Q < 0 || M < 0 || E < 0 || (Q > 0 && (!q || !idx)) || (M > 0 && !K))
        return 1;
    if (nthreads < 1)
        nthreads = 1;
    if (nthreads > Q)
        nthreads = Q > 0 ? (int)Q : 1;
    top1_job base = {M, E, q, K, idx, best, 0, Q};
    if (nthreads == 1) {
        top1_worker(&base);
        return 0;
    }
    pthread_t *th = (pthread_t *)malloc(sizeof(pthread_t) * nthreads);
    top1_job *jobs = (top1_job *)malloc(sizeof(top1_job) * nthreads);
    if (!th || !jobs) {
        free(th);
        free(jobs);
        return 4;
    }
    for (int i = 0; i < nthreads; ++i) {
        jobs[i] = base;
        jobs[i].q_begin = Q * i / nthreads;
        jobs[i].q_end = Q * (i + 1) / nthreads;
        pthread_create(&th[i], NULL, top1_worker, &jobs[i]);
    }
    for (int i = 0; i < nthreads; ++i)
        pthread_join(th[i], NULL);
    free(th);
    free(jobs);
    return 0;
}

/* ------------------------------------------------------------------------- */
/* Gated delta rule                                                           */
/* ------------------------------------------------------------------------- */

/* One sequence of T tokens, every value head in turn:
 *   u = beta_t (v_t - (a_t S)^T k_t),  S <- a_t S + k_t u^T,  a_t = exp(g_t),
 *   o_t = scale S^T q_t
 * q, k : [T, Hk, K], v : [T, Hv, V], g, beta (nullable: 0, 1) : [T, Hv],
 * S : [Hv, K, V] initial state in, final state out, o (nullable) : [T, Hv, V].
 * Head h reads query/key head h / (Hv / Hk); norm divides q and k of a token
 * and head by sqrt(sum of squares + eps). */
int oracle_delta_f64(int64_t T, int64_t Hk, int64_t Hv, int64_t K, int64_t V, const double *q,
                     const double *k, const double *v, const double *g, const double *beta,
                     double *S, double *o, int norm, double eps, double scale)
{
    if (T < 0 || Hk < 1 || Hv < 1 || Hv % Hk || K < 1 || V < 1 || !S || (T > 0 && (!k || !v)) ||
        (T > 0 && o && !q))
        return 1;
    double *kn = (double *)malloc(sizeof(double) * K);
    double *qn = (double *)malloc(sizeof(double) * K);
    if (!kn || !qn) {
        free(kn);
        free(qn);
        return 4;
    }
    for (int64_t h = 0; h < Hv; ++h) {
        double *Sh = S + h * K * V;
        const int64_t hk = h / (Hv / Hk);
        for (int64_t t = 0; t < T; ++t) {
            const double *kt = k + (t * Hk + hk) * K;
            const double *qt = o ? q + (t * Hk + hk) * K : NULL;
            const double *vt = v + (t * Hv + h) * V;
            double k2 = 0.0, q2 = 0.0;
            for (int64_t i = 0; i < K; ++i) {
                k2 += kt[i] * kt[i];
                if (qt)
                    q2 += qt[i] * qt[i];
            }
            for (int64_t i = 0; i < K; ++i) {
                kn[i] = norm ? kt[i] / sqrt(k2 + eps) : kt[i];
                qn[i] = !qt ? 0.0 : norm ? qt[i] / sqrt(q2 + eps) : qt[i];
            }
            const double a = g ? exp(g[t * Hv + h]) : 1.0;
            const double b = beta ? beta[t * Hv + h] : 1.0;
            for (int64_t j = 0; j < V; ++j) {
                double seen = 0.0;
                for (int64_t i = 0; i < K; ++i)
                    seen += a * Sh[i * V + j] * kn[i];
                const double u = b * (vt[j] - seen);
                double out = 0.0;
                for (int64_t i = 0; i < K; ++i) {
                    Sh[i * V + j] = a * Sh[i * V + j] + kn[i] * u;
                    out += Sh[i * V + j] * qn[i];
                }
                if (o)
                    o[(t * Hv + h) * V + j] = scale * out;
            }
        }
    }
    free(kn);
    free(qn);
    return 0;
}
