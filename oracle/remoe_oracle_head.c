/*
 * CPU oracle, fourth file: what is computed over the vocabulary (log probabilities of given tokens,
 * entropy, top alternatives, distillation from a teacher's top logits, and the gradients of both).
 *
 * TEST INFRASTRUCTURE ONLY (see remoe_oracle.c).  fp64 throughout, from the logits widened to fp32
 * (exactly, where they are bf16); every value is its definition written as loops over one row:
 *
 *   m = max_v z_v,  d_v = (z_v - m) / tau,  S = sum_v exp(d_v),  ln p_v = d_v - ln S
 *   rest = S - 1 summed without the first largest logit, ln S = log1p(rest)
 *   logprob = ln p_target (0 where the target lies outside the vocabulary)
 *   entropy = ln S - sum_v d_v exp(d_v) / S
 *   alternatives: the n largest logits, ties to the lower id; NaN ranks above +inf
 *   q over a teacher's K listed logits t (entries outside the vocabulary are absent):
 *     softmax(t / tau) over the list, or exp(t / tau - lse)
 *   loss = sum_j q_j (ln q_j - ln p_id(j)), 0 where q_j = 0
 *
 * Conventions where the formulas leave a case open: a row whose logits are all -inf has rest = -1, ln p = -inf
 * for every token, entropy 0 and gradient 0; a row that holds NaN or +inf is NaN throughout.
 *
 * Parity status: pinned by the CPU tests (torch's log_softmax, entr and kl_div in fp64, reverse-mode
 * differentiation of those, central differences, closed forms).
 */
#include <math.h>
#include <stdint.h>
#include <stdlib.h>

typedef struct { double m, rest; int bad, empty; } row_stats;

static row_stats stats_of(const float *z, int64_t V, double tau)
{
    row_stats s = {-INFINITY, 0.0, 0, 0};
    int64_t at = 0;
    for (int64_t v = 0; v < V; ++v) {
        if (isnan(z[v]) || z[v] == INFINITY) s.bad = 1;
        if ((double)z[v] > s.m) { s.m = z[v]; at = v; }
    }
    s.empty = !s.bad && s.m == -INFINITY;
    if (s.bad) s.rest = NAN;
    else if (s.empty) s.rest = -1.0;
    else
        for (int64_t v = 0; v < V; ++v)
            if (v != at) s.rest += exp(((double)z[v] - s.m) / tau);
    return s;
}

static double log_p(const row_stats *s, float z, double tau)
{
    if (s->bad) return NAN;
    if (s->empty) return -INFINITY;
    return ((double)z - s->m) / tau - log1p(s->rest);
}

/* z[a] comes before z[b] among the alternatives */
static int ahead(const float *z, int64_t a, int64_t b)
{
    const int na = isnan(z[a]), nb = isnan(z[b]);
    if (na || nb) return na != nb ? na : a < b;
    return z[a] != z[b] ? z[a] > z[b] : a < b;
}

int oracle_token_logprobs(const float *logits, int64_t T, int64_t V, double tau, const int32_t *targets, int n, double *logprob,
                          double *entropy, int32_t *top_idx, double *top_logprob, double *stats)
{
    if (!logits || V < 1 || !(tau > 0.0) || n < 0 || n > V) return -1;
    for (int64_t t = 0; t < T; ++t) {
        const float *z = logits + t * V;
        const row_stats s = stats_of(z, V, tau);
        if (stats) { stats[2 * t] = s.m; stats[2 * t + 1] = s.rest; }
        if (targets && logprob) logprob[t] = targets[t] >= 0 && targets[t] < V ? log_p(&s, z[targets[t]], tau) : 0.0;
        if (entropy) {
            double a = 0.0;
            if (!s.bad && !s.empty)
                for (int64_t v = 0; v < V; ++v) {
                    const double d = ((double)z[v] - s.m) / tau, e = exp(d);
                    if (e > 0.0) a += d * e;
                }
            entropy[t] = s.bad ? NAN : s.empty ? 0.0 : log1p(s.rest) - a / (1.0 + s.rest);
        }
        /* insertion into a list of n */
        int have = 0;
        int32_t *list = top_idx ? top_idx + t * n : NULL;
        for (int64_t v = 0; list && v < V; ++v) {
            int p = have;
            while (p > 0 && ahead(z, v, list[p - 1])) --p;
            if (p >= n) continue;
            for (int j = have < n ? have : n - 1; j > p; --j) list[j] = list[j - 1];
            list[p] = (int32_t)v;
            if (have < n) ++have;
        }
        for (int j = 0; list && top_logprob && j < n; ++j) top_logprob[t * n + j] = log_p(&s, z[list[j]], tau);
    }
    return 0;
}

int oracle_token_logprobs_grad(const float *logits, int64_t T, int64_t V, double tau, const int32_t *targets, const float *d_logprob,
                               const float *d_entropy, double *dlogits)
{
    if (!logits || !dlogits || V < 1 || !(tau > 0.0)) return -1;
    for (int64_t t = 0; t < T; ++t) {
        const float *z = logits + t * V;
        double *g = dlogits + t * V;
        const row_stats s = stats_of(z, V, tau);
        const int aimed = targets && d_logprob && targets[t] >= 0 && targets[t] < V;
        double h = 0.0;
        for (int64_t v = 0; v < V; ++v) {
            const double lp = log_p(&s, z[v], tau);
            if (exp(lp) > 0.0) h -= exp(lp) * lp;
        }
        for (int64_t v = 0; v < V; ++v) {
            if (s.bad) { g[v] = NAN; continue; }
            const double lp = log_p(&s, z[v], tau), p = exp(lp);
            g[v] = aimed ? (double)d_logprob[t] * (v == targets[t] ? -expm1(lp) : -p) : 0.0;
            if (d_entropy && p > 0.0) g[v] -= (double)d_entropy[t] * p * (lp + h);
            if (s.empty) g[v] = 0.0;
            g[v] /= tau;
        }
    }
    return 0;
}

/* q[j], ln q[j] of one row's list */
static void teacher(const int32_t *id, const float *t, const float *lse, int K, int64_t V, double tau, double *q, double *lq)
{
    double top = -INFINITY, sum = 0.0;
    for (int j = 0; j < K; ++j)
        if (id[j] >= 0 && id[j] < V && (double)t[j] > top) top = t[j];
    for (int j = 0; j < K; ++j)
        if (id[j] >= 0 && id[j] < V && t[j] != -INFINITY) sum += exp(((double)t[j] - top) / tau);
    for (int j = 0; j < K; ++j) {
        const int there = id[j] >= 0 && id[j] < V && t[j] != -INFINITY;
        lq[j] = !there ? -INFINITY : lse ? (double)t[j] / tau - (double)*lse : ((double)t[j] - top) / tau - log(sum);
        q[j] = there ? exp(lq[j]) : 0.0;
    }
}

int oracle_distill(const float *logits, int64_t T, int64_t V, double tau, const int32_t *idx, const float *tl, const float *lse, int K,
                   double *loss, double *stats)
{
    if (!logits || !idx || !tl || V < 1 || K < 1 || !(tau > 0.0)) return -1;
    double *q = (double *)malloc(sizeof(double) * 2 * (size_t)K), *lq = q + K;
    if (!q) return -1;
    for (int64_t t = 0; t < T; ++t) {
        const float *z = logits + t * V;
        const int32_t *id = idx + t * K;
        const row_stats s = stats_of(z, V, tau);
        if (stats) { stats[2 * t] = s.m; stats[2 * t + 1] = s.rest; }
        teacher(id, tl + t * K, lse ? lse + t : NULL, K, V, tau, q, lq);
        loss[t] = s.bad ? NAN : 0.0;
        for (int j = 0; j < K; ++j)
            if (q[j] != 0.0) loss[t] += q[j] * (lq[j] - log_p(&s, z[id[j]], tau));
    }
    free(q);
    return 0;
}

int oracle_distill_grad(const float *logits, int64_t T, int64_t V, double tau, const int32_t *idx, const float *tl, const float *lse, int K,
                        const float *d_loss, double *dlogits)
{
    if (!logits || !idx || !tl || !d_loss || !dlogits || V < 1 || K < 1 || !(tau > 0.0)) return -1;
    double *q = (double *)malloc(sizeof(double) * 2 * (size_t)K), *lq = q + K;
    if (!q) return -1;
    for (int64_t t = 0; t < T; ++t) {
        const float *z = logits + t * V;
        const int32_t *id = idx + t * K;
        double *g = dlogits + t * V;
        const row_stats s = stats_of(z, V, tau);
        teacher(id, tl + t * K, lse ? lse + t : NULL, K, V, tau, q, lq);
        double mass = 0.0;
        for (int j = 0; j < K; ++j) mass += q[j];
        for (int64_t v = 0; v < V; ++v) g[v] = s.bad ? NAN : s.empty ? 0.0 : mass * exp(log_p(&s, z[v], tau));
        for (int j = 0; j < K; ++j)
            if (!s.bad && !s.empty && q[j] != 0.0) g[id[j]] -= q[j];
        for (int64_t v = 0; v < V; ++v) g[v] *= (double)d_loss[t] / tau;
    }
    free(q);
    return 0;
}
