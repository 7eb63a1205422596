// What the kernels over the vocabulary share (head.hip, head_grad.hip): reading a logit, sums and maxima over a workgroup,
// a teacher's list.  NT is the number of threads of a workgroup.
#pragma once

#include "common.h"

namespace remoe {

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

// over the workgroup, the same value in every thread, in a fixed order; `part` is a value of LDS for every wavefront
template <int NT, typename V, typename Op> __device__ __forceinline__ V block_reduce(V v, V *part, Op op)
{
    v = wave_reduce(v, op);
    __syncthreads();                    // the previous use of part is over
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    V r = part[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = op(r, part[w]);
    return r;
}

struct OpSum { template <typename V> __device__ __forceinline__ V operator()(V a, V b) const { return a + b; } };
struct OpMax { __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); } };

// One entry of a teacher's list, thread j holds entry j (K <= NT): q_j and ln q_j in fp64 (a few values per row, and they are
// subtracted from the model's own).  Entries that are absent have id -1 and q 0.  mass = sum_j q_j: 1 by definition where the
// list is normalised by itself and not empty, and only formed where MASS is set.
struct TeacherEntry { int id; double q, log_q, mass; };

template <int NT, bool MASS>
__device__ __forceinline__ TeacherEntry teacher_entry(const int32_t *idx, const void *logits, int dtype, const float *lse, int K, int V,
                                                      float tau, int64_t row, double *part)
{
    const int j = threadIdx.x;
    TeacherEntry e{-1, 0.0, 0.0, 0.0};
    float t = -__builtin_inff();
    if (j < K) {
        const int64_t at = row * K + j;
        const int id = idx[at];
        t = dtype == REMOE_F32 ? static_cast<const float *>(logits)[at] : bf16_to_f32(static_cast<const bf16_t *>(logits)[at]);
        if (id >= 0 && id < V && t != -__builtin_inff()) e.id = id;
        else t = -__builtin_inff();
    }
    if (lse) {
        if (e.id >= 0) {
            e.log_q = (double)t / (double)tau - (double)lse[row];
            e.q = exp(e.log_q);
        }
        if constexpr (MASS) e.mass = block_reduce<NT>(e.q, part, OpSum());
    } else {
        const float top = block_reduce<NT>(t, reinterpret_cast<float *>(part), OpMax());
        const double d = e.id >= 0 ? ((double)t - (double)top) / (double)tau : 0.0;
        const double q = e.id >= 0 ? exp(d) : 0.0;
        const double sum = block_reduce<NT>(q, part, OpSum());
        if (e.id >= 0) {
            e.q = q / sum;
            e.log_q = d - log(sum);
        }
        e.mass = sum == 0.0 ? 0.0 : sum / sum;              // NaN logits: NaN
    }
    return e;
}

// 16 bytes of logits
typedef u32x4_t __attribute__((aligned(2))) u32x4_any_t;      // at any value's address

template <int DT> struct Piece;
template <> struct Piece<REMOE_F32> {
    static constexpr int N = 4;
    static __device__ __forceinline__ void get(const u32x4_t &r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
    }
    static __device__ __forceinline__ u32x4_t put(const float *v)
    {
        return u32x4_t{__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])};
    }
    static __device__ __forceinline__ u32x4_t lowest()          // -inf throughout
    {
        return u32x4_t{0xFF800000u, 0xFF800000u, 0xFF800000u, 0xFF800000u};
    }
};
template <> struct Piece<REMOE_BF16> {
    static constexpr int N = 8;
    static __device__ __forceinline__ void get(const u32x4_t &r, float *v)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[2 * i] = __uint_as_float(r[i] << 16);
            v[2 * i + 1] = __uint_as_float(r[i] & 0xFFFF0000u);
        }
    }
    static __device__ __forceinline__ u32x4_t put(const float *v)
    {
        return u32x4_t{pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
    }
    static __device__ __forceinline__ u32x4_t lowest()
    {
        return u32x4_t{0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u, 0xFF80FF80u};
    }
};

}  // namespace remoe
