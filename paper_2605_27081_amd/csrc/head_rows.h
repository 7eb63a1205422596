// What the kernels over the vocabulary share (head.hip, head_grad.hip): reading a logit, sums and maxima over a workgroup,
// a teacher's list.  Workgroups have HEAD_THREADS threads throughout.
#pragma once

#include "common.h"

namespace remoe {

constexpr int HEAD_THREADS = 256;
constexpr int HEAD_WAVES = HEAD_THREADS / 64;

template <int DT> struct LogitOf;
template <> struct LogitOf<REMOE_F32> { typedef float type; };
template <> struct LogitOf<REMOE_BF16> { typedef bf16_t type; };

__device__ __forceinline__ float widen(float v) { return v; }
__device__ __forceinline__ float widen(bf16_t v) { return bf16_to_f32(v); }

template <typename V, typename Op> __device__ __forceinline__ V wave_reduce(V v, Op op)
{
#pragma unroll
    for (int off = 32; off >= 1; off >>= 1) v = op(v, (V)__shfl_xor(v, off, 64));
    return v;
}

// over the workgroup, the same value in every thread, in a fixed order; `part` is HEAD_WAVES values of LDS
template <typename V, typename Op> __device__ __forceinline__ V block_reduce(V v, V *part, Op op)
{
    v = wave_reduce(v, op);
    __syncthreads();                    // the previous use of part is over
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    V r = part[0];
#pragma unroll
    for (int w = 1; w < HEAD_WAVES; ++w) r = op(r, part[w]);
    return r;
}

struct OpSum { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct OpMax { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// One entry of a teacher's list, thread j holds entry j: q_j and ln q_j in fp64 (a few values per row, and they are
// subtracted from the model's own).  Entries that are absent have id -1 and q 0.
struct TeacherEntry { int id; double q, log_q; };

__device__ __forceinline__ TeacherEntry teacher_entry(const int32_t *idx, const void *logits, int dtype, const float *lse, int K, int V,
                                                      float tau, int64_t row, double *part)
{
    const int j = threadIdx.x;
    TeacherEntry e{-1, 0.0, 0.0};
    float t = -__builtin_inff();
    if (j < K) {
        const int64_t at = row * K + j;
        const int id = idx[at];
        t = dtype == REMOE_F32 ? static_cast<const float *>(logits)[at] : bf16_to_f32(static_cast<const bf16_t *>(logits)[at]);
        if (id >= 0 && id < V && t != -__builtin_inff()) e.id = id;
        else t = -__builtin_inff();
    }
    if (lse) {
        if (e.id >= 0) e.log_q = (double)t / (double)tau - (double)lse[row];
    } else {
        const float top = block_reduce(t, reinterpret_cast<float *>(part), OpMax());
        const double d = e.id >= 0 ? ((double)t - (double)top) / (double)tau : 0.0;
        const double sum = block_reduce(e.id >= 0 ? exp(d) : 0.0, part, OpSum());
        e.log_q = d - log(sum);
    }
    e.q = e.id >= 0 ? exp(e.log_q) : 0.0;
    return e;
}

}  // namespace remoe
