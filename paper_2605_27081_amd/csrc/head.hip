// Log probabilities of given tokens, entropy and top alternatives of rows of logits; divergence from a teacher's top
// logits.  With m the largest logit of a row and d_v = (z_v - m) / tau:
//
//   S = sum_v exp(d_v) = 1 + rest,  ln p_v = d_v - log1p(rest),  H = log1p(rest) - sum_v d_v exp(d_v) / S
//   loss = sum_j q_j (ln q_j - ln p_id(j))
//
// One workgroup per row: a pass for the maximum, one for the sums, one for each alternative.
#include "head_rows.h"

namespace remoe {

namespace {

constexpr float LOG2E = 1.44269504088896340736f;

// what a row's logits add up to
struct RowSums { float m, rest, dsum; };     // largest, sum without one of the largest, sum of d exp(d)

__device__ __forceinline__ float log_p(const RowSums &r, float z, float tau)
{
    if (r.rest == -1.f) return -__builtin_inff();            // nothing but -inf
    return (z - r.m) / tau - log1pf(r.rest);
}

// Order of the alternatives: larger logits first, NaN above all, the lower id first among equals.
__device__ __forceinline__ uint64_t rank_key(float z, int id)
{
    uint32_t u = __float_as_uint(z + 0.0f);                  // -0 as +0
    u = z != z ? 0xFFFFFFFEu : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
    return (uint64_t)u << 32 | (0xFFFFFFFFu - (uint32_t)id);
}
__device__ __forceinline__ int key_id(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

struct OpMaxKey { __device__ __forceinline__ uint64_t operator()(uint64_t a, uint64_t b) const { return a > b ? a : b; } };

template <int DT> __global__ __launch_bounds__(HEAD_THREADS) void head_rows_kernel(const HeadArgs a)
{
    typedef typename LogitOf<DT>::type elem;
    __shared__ double part[HEAD_WAVES];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, V = a.V;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    const float c = LOG2E / a.tau;

    RowSums r;
    float m = -__builtin_inff();
    for (int v = tid; v < V; v += HEAD_THREADS) m = fmaxf(m, widen(z[v]));
    r.m = m = block_reduce(m, reinterpret_cast<float *>(part), OpMax());
    float rest = 0.f, dsum = 0.f, top = 0.f;
    for (int v = tid; v < V; v += HEAD_THREADS) {
        const float zv = widen(z[v]);
        if (zv == m) { top += 1.f; continue; }
        const float x = (zv - m) * c, e = __builtin_amdgcn_exp2f(x);
        rest += e;
        if (e > 0.f) dsum += x * e;
    }
    rest = block_reduce(rest, reinterpret_cast<float *>(part), OpSum());
    top = block_reduce(top, reinterpret_cast<float *>(part), OpSum());
    r.dsum = block_reduce(dsum, reinterpret_cast<float *>(part), OpSum()) * (1.f / LOG2E);
    if (m == -__builtin_inff()) r.rest = rest - 1.f;         // -1, or NaN
    else r.rest = m < __builtin_inff() ? rest + (top - 1.f) : __builtin_nanf("");

    if (tid == 0) {
        if (a.stats) { a.stats[2 * row] = r.m; a.stats[2 * row + 1] = r.rest; }
        if (a.targets) {
            const int t = a.targets[row];
            a.logprob[row] = t >= 0 && t < V ? log_p(r, widen(z[t]), a.tau) : 0.f;
        }
        if (a.entropy) {
            const float h = r.rest == -1.f ? 0.f : log1pf(r.rest) - r.dsum / (1.f + r.rest);
            a.entropy[row] = h < 0.f ? 0.f : h;
        }
    }
    uint64_t last = ~(uint64_t)0;
    for (int j = 0; j < a.top_n; ++j) {
        uint64_t best = 0;
        for (int v = tid; v < V; v += HEAD_THREADS) {
            const uint64_t k = rank_key(widen(z[v]), v);
            if (k < last && k > best) best = k;
        }
        last = block_reduce(best, reinterpret_cast<uint64_t *>(part), OpMaxKey());
        if (tid == 0) {
            a.top_idx[row * a.top_n + j] = key_id(last);
            a.top_logprob[row * a.top_n + j] = log_p(r, widen(z[key_id(last)]), a.tau);
        }
    }
    if (a.teacher_idx) {
        const TeacherEntry e = teacher_entry(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, V, a.tau, row, part);
        double term = 0.0;
        if (e.q != 0.0) {
            const double lp = r.rest == -1.f ? -(double)__builtin_inff()
                                             : ((double)widen(z[e.id]) - (double)r.m) / (double)a.tau - log1p((double)r.rest);
            term = e.q * (e.log_q - lp);
        }
        const double loss = block_reduce(term, part, OpSum());
        if (tid == 0) a.loss[row] = r.rest != r.rest ? r.rest : (float)loss;
    }
}

}  // namespace

size_t head_workspace_bytes(int dtype, int V, int64_t T, int top_n)
{
    (void)dtype; (void)V; (void)T; (void)top_n;
    return 256;
}

remoe_status launch_head_forward(const HeadArgs &a, hipStream_t stream)
{
    const dim3 grid((unsigned)a.T), block(HEAD_THREADS);
    hipLaunchKernelGGL(a.dtype == REMOE_BF16 ? head_rows_kernel<REMOE_BF16> : head_rows_kernel<REMOE_F32>, grid, block, 0, stream, a);
    return check_hip(hipGetLastError(), "head kernel launch");
}

}  // namespace remoe
