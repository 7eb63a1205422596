// Gradients over the vocabulary, from a row's statistics (m, rest), S = 1 + rest, e_v = exp((z_v - m) / tau), p_v = e_v / S:
//
//   log probabilities:  dz_v = (1/tau) ( g (1[v = target] - p_v) - h p_v (ln p_v + H) )
//   teacher's list:     dz_v = (g/tau) ( M p_v - q_v ),  M = sum_j q_j,  q_v the sum over the entries that name v
//
// A pass over the row writes the terms that every token has; the tokens that are named (the target, the teacher's) are taken
// from their logits in fp64 and written over it: their differences cancel where the model agrees (1 - p_v, M p_v - q_v).
// One workgroup per row, an element at a time.
#include "head_rows.h"

namespace remoe {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

template <int DT> __global__ __launch_bounds__(HEAD_THREADS) void head_grad_kernel(const HeadGradArgs a)
{
    typedef typename LogitOf<DT>::type elem;
    __shared__ double part[HEAD_WAVES];
    __shared__ int ids[HEAD_THREADS];
    __shared__ double qs[HEAD_THREADS];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, V = a.V;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    elem *dz = static_cast<elem *>(a.dlogits) + row * a.ld_d;
    const float m = a.stats[2 * row], rest = a.stats[2 * row + 1];
    const float c = LOG2E / a.tau, inv_s = 1.f / (1.f + rest);
    const bool empty = rest == -1.f;

    // coefficients: dz = p * (k0 + k1 * d) away from the named tokens
    int named = -1;
    double q = 0.0, mass = 0.0;
    float k0, k1 = 0.f, h = 0.f;
    if (a.teacher_idx) {
        const TeacherEntry e = teacher_entry(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, V, a.tau, row, part);
        named = e.id;
        q = e.q;
        mass = block_reduce(q, part, OpSum());
        k0 = (float)((double)a.d_loss[row] * mass / (double)a.tau);
        ids[tid] = named;
        qs[tid] = q;
        __syncthreads();
        if (named >= 0)                  // an id that stands there more than once: its first entry takes them all
            for (int j = 0; j < a.K; ++j)
                if (j != tid && ids[j] == named) {
                    if (j < tid) { named = -1; break; }
                    q += qs[j];
                }
    } else {
        const int t = a.targets ? a.targets[row] : -1;
        const float g = t >= 0 && t < V ? a.d_logprob[row] : 0.f;
        if (tid == 0 && t >= 0 && t < V) named = t;
        k0 = -g / a.tau;
        if (a.d_entropy) {
            h = a.d_entropy[row] / a.tau;
            k0 -= h * (a.entropy[row] - log1pf(rest));
            k1 = -h;
        }
    }
    auto at = [&](float zv) {
        const float x = (zv - m) * c, e = __builtin_amdgcn_exp2f(x);
        float v = e * inv_s * k0;
        if (k1 != 0.f && e > 0.f) v += e * inv_s * (k1 * (x * (1.f / LOG2E)));
        return empty ? 0.f : v;
    };
    // the named token's value, before the pass below may write over its logit
    float exact = 0.f;
    if (named >= 0) {
        const float zv = widen(z[named]);
        if (!empty) {
            const double d = ((double)zv - (double)m) / (double)a.tau, s = 1.0 + (double)rest;
            double v;
            if (a.teacher_idx) v = (double)a.d_loss[row] * ((expm1(d) * mass + (mass - q) - q * (double)rest) / s);
            else {
                v = (double)a.d_logprob[row] * (((double)rest - expm1(d)) / s);
                if (a.d_entropy && exp(d) > 0.0) v -= (double)a.d_entropy[row] * (exp(d) / s) * (d - log1p((double)rest) + (double)a.entropy[row]);
            }
            exact = (float)(v / (double)a.tau);
        }
        if (a.accumulate) exact += widen(dz[named]);
    }
    auto store = [&](int v, float f) {
        if constexpr (DT == REMOE_BF16) dz[v] = (bf16_t)(pack_bf16x2(f, 0.f) & 0xFFFFu);
        else dz[v] = f;
    };
    __syncthreads();
    for (int v = tid; v < V; v += HEAD_THREADS) store(v, at(widen(z[v])) + (a.accumulate ? widen(dz[v]) : 0.f));
    __syncthreads();
    if (named >= 0) store(named, exact);
}

}  // namespace

remoe_status launch_head_backward(const HeadGradArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)a.T), block(HEAD_THREADS);
    hipLaunchKernelGGL(a.dtype == REMOE_BF16 ? head_grad_kernel<REMOE_BF16> : head_grad_kernel<REMOE_F32>, grid, block, 0, stream, a);
    return check_hip(hipGetLastError(), "head gradient kernel launch");
}

}  // namespace remoe
