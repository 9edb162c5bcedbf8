/*
 * sample_ref.c -- CPU oracle of the token drawing, TEST INFRASTRUCTURE ONLY.
 *
 * The plain statement of the operation sequence: sort the row's tokens by
 * descending logit (equal ones by index), weigh each, cut the prefix that each
 * filter keeps, and walk to the draw.  It shares no code with the GPU path.
 *
 * Build: gcc -std=c11 -O2 -ffp-contract=off -fno-fast-math -mfma.
 */
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

typedef struct { float l; int64_t j; } tok;

static int by_logit(const void *pa, const void *pb)
{
    const tok *a = (const tok *)pa, *b = (const tok *)pb;
    if (a->l != b->l) return a->l > b->l ? -1 : 1;
    return a->j < b->j ? -1 : a->j > b->j;
}

/* exp(d) 2^43 for d in [-31, 0], by the stated sequence. */
static double exp43(double d)
{
    const double n = rint(d * 1.4426950408889634);
    const double ln2_hi = 0x1.62e42fefa3p-1, ln2_lo = 0x1.3de6af278ece6p-42;
    double r = fma(n, -ln2_hi, d);
    r = fma(n, -ln2_lo, r);
    double fact = 39916800.0, p = 1.0 / fact; /* 11! */
    for (int i = 10; i >= 0; --i) {
        fact = fact / (double)(i + 1);
        p = fma(p, r, 1.0 / fact);
    }
    return ldexp(p, (int)n + 43);
}

/* w = rint(exp(d) 2^43): exp(-b/64) exp(d + b/64); 0 for d <= -31 or NaN. */
uint64_t sample_ref_weight(double d)
{
    if (!(d > -31.0)) return 0;
    const double b = rint(d * -64.0);
    const double r = fma(b, 1.0 / 64.0, d);
    const double f[6] = {1.0, 1.0, 1.0 / 2.0, 1.0 / 6.0, 1.0 / 24.0, 1.0 / 120.0};
    double p = f[5];
    for (int i = 4; i >= 0; --i) p = fma(p, r, f[i]);
    /* one rounding of the product to an integer */
    return (uint64_t)(fma(exp43(b * (-1.0 / 64.0)), p, 0x1p52) - 0x1p52);
}

double sample_ref_log(float m)
{
    int e;
    double f = frexp((double)m, &e); /* [1/2, 1) */
    f = f * 2.0;
    e = e - 1;
    if (f > sqrt(2.0)) { f = f * 0.5; e = e + 1; }
    const double s = (f - 1.0) / (f + 1.0), q = s * s;
    double p = 1.0 / 19.0;
    for (int i = 17; i >= 1; i -= 2) p = fma(p, q, 1.0 / (double)i);
    return fma((double)e, 0x1.62e42fefa39efp-1, (s + s) * p);
}

/* One row; returns the token and stores its probability. */
int32_t sample_ref_row(int64_t n, const float *l, float u, float temperature, int32_t top_k,
                       float top_p, float min_p, float *prob)
{
    *prob = 0.0f;
    for (int64_t j = 0; j < n; ++j)
        if (isnan(l[j])) { *prob = NAN; return -1; }
    tok *t = (tok *)malloc(sizeof(tok) * (size_t)(n > 0 ? n : 1));
    uint64_t *w = (uint64_t *)malloc(8 * (size_t)(n > 0 ? n : 1));
    double *d = (double *)malloc(8 * (size_t)(n > 0 ? n : 1));
    if (!t || !w || !d) abort();
    int32_t token = -1;
    for (int64_t j = 0; j < n; ++j) { t[j].l = l[j]; t[j].j = j; }
    qsort(t, (size_t)n, sizeof(tok), by_logit);
    if (n > 0 && t[0].l != -INFINITY) {
        if (!(temperature > 0.0f)) {
            token = (int32_t)t[0].j;
            *prob = 1.0f;
        } else {
            const double it = 1.0 / (double)temperature, m = (double)t[0].l;
            int64_t keep = n;
            for (int64_t i = 0; i < n; ++i) {
                d[i] = t[i].l == t[0].l ? 0.0 : ((double)t[i].l - m) * it;
                w[i] = sample_ref_weight(d[i]);
            }
            if (top_k > 0 && top_k < keep) keep = top_k;
            if (top_p < 1.0f) {
                uint64_t total = 0, before = 0, limit = 1;
                for (int64_t i = 0; i < keep; ++i) total += w[i];
                if (top_p > 0.0f) {
                    const double x = ceil((double)top_p * (double)total);
                    if (x > 1.0) limit = (uint64_t)x;
                }
                int64_t i = 0;
                while (i < keep && (i == 0 || before < limit)) before += w[i++];
                keep = i;
            }
            if (min_p > 0.0f) {
                const double cut = min_p >= 1.0f ? 0.0 : sample_ref_log(min_p);
                int64_t i = 1;
                while (i < keep && d[i] >= cut) ++i;
                keep = i;
            }
            uint64_t kept = 0, run = 0, at = 0;
            for (int64_t i = 0; i < keep; ++i) kept += w[i];
            if (u >= 1.0f) at = kept - 1;
            else if (u > 0.0f) at = (uint64_t)((double)u * (double)kept);
            if (at > kept - 1) at = kept - 1;
            int64_t i = 0;
            while (run + w[i] <= at) run += w[i++];
            token = (int32_t)t[i].j;
            *prob = (float)((double)w[i] / (double)kept);
        }
    }
    free(t); free(w); free(d);
    return token;
}
