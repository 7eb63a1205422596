// Gradients over the vocabulary, from a row's statistics (m, rest), S = 1 + rest, e_v = exp((z_v - m) / tau), p_v = e_v / S:
//
//   log probabilities:  dz_v = (1/tau) ( g (1[v = target] - p_v) - h p_v (ln p_v + H) )
//   teacher's list:     dz_v = (g/tau) ( M p_v - q_v ),  M = sum_j q_j,  q_v the sum over the entries that name v
//
// A pass over the row writes the terms that every token has; the tokens that are named (the target, the teacher's) are taken
// from their logits in fp64 and written over it: their differences cancel where the model agrees (1 - p_v, M p_v - q_v).
// A workgroup has a stretch of a row's 16-byte pieces, cut where dlogits is aligned, and the named tokens among its values.  The
// first pieces are asked for before the row's terms are known, the next ones before the present ones are used; loads and stores
// go past the caches (4096 rows of 151,936 with a teacher's list: loads 518 -> 498 us, stores 590 -> 498; loads 1-5 % from 512 rows of
// 50,257 on; stores 1000 -> 957 for 8192 of 151,936, and within 8 % either way where a copy of the gradient follows that fits the last level).
//
// Bound by HBM: every logit is read and every gradient written once.  8192 rows of 151,936 bf16 logits 954 us = 5.2 TB/s (a plain
// copy of 4 GiB 4.8), with a list of 128 for 4096 rows 493 us = 5.1 TB/s; 1021 rows of 50,257 37 us.  Accumulated, which reads
// the gradient too: 1414 us = 5.3 TB/s, with the list 700 us = 5.3 TB/s (4096 rows of 65,536 fp32 590 us, 5.5; written only 420, 5.1).
// An element at a time by a workgroup a row took 1853, 998 and 127 us.
#include <type_traits>

#include "head_rows.h"

namespace remoe {

namespace {

constexpr int PIECES = 2;              // 16-byte pieces of a thread that are on their way together

// dz = e * (k0 + k1 x) with x = log2 e, away from the named tokens
struct RowTerms { float m, c, c_low, k0, k1; };

// e^(d) as 2^x.  fp32 gradients: x to more than fp32 (its product's remainder and the low part of c), since at d = -12 the
// rounding of x alone would be 20 steps of e; bf16 ones are rounded to 2^-8 anyway.
template <bool FINE> __device__ __forceinline__ float term(const RowTerms &t, float z)
{
    const float d = fmaxf(z - t.m, -512.f / t.c);             // 2^-512 is 0; -inf would make the products below NaN
    const float x = d * t.c;
    float e = __builtin_amdgcn_exp2f(x);
    if constexpr (FINE) e = fmaf(e, 0.693147180559945f * fmaf(d, t.c_low, fmaf(d, t.c, -x)), e);
    return e * fmaf(t.k1, x, t.k0);
}

__device__ __forceinline__ void put_one(float *p, float v) { *p = v; }
__device__ __forceinline__ void put_one(bf16_t *p, float v) { *p = (bf16_t)(pack_bf16x2(v, 0.f) & 0xFFFFu); }

// KEEP: stores that may stay in the caches
template <int NT, int DT, bool TEACHER, bool ADD, bool KEEP>
__global__ __launch_bounds__(NT) void head_grad_kernel(const HeadGradArgs a, int segs, int seg_pieces)
{
    typedef typename LogitOf<DT>::type elem;
    typedef Piece<DT> P;
    constexpr bool FINE = DT == REMOE_F32;
    const int64_t row = blockIdx.x / (unsigned)segs;
    const int seg = blockIdx.x % (unsigned)segs;
    const int tid = threadIdx.x, V = a.V;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    elem *dz = static_cast<elem *>(a.dlogits) + row * a.ld_d;
    // values in front of the first aligned piece of dlogits, whole pieces, values behind the last
    int head = (int)((16 - ((uintptr_t)dz & 15)) & 15) / (int)sizeof(elem);
    if (head > V) head = V;
    const int pieces = (V - head) / P::N;
    // (the stretches are cut for a row whose first value is aligned: another one may have two pieces less)
    const int p0 = seg * seg_pieces < pieces ? seg * seg_pieces : pieces;
    const int p1 = seg == segs - 1 || p0 + seg_pieces > pieces ? pieces : p0 + seg_pieces;
    const int v0 = seg == 0 ? 0 : head + p0 * P::N, v1 = seg == segs - 1 ? V : head + p1 * P::N;      // this workgroup's values

    // the first pieces are on their way while the row's terms are put together
    const elem *zp = z + head;
    elem *dp = dz + head;
    u32x4_t in[PIECES], old[ADD ? PIECES : 1];
    auto request = [&](int p) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int at = p + u * NT;
            if (at < p1) {
                in[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_any_t *>(zp + (int64_t)at * P::N));
                if constexpr (ADD) old[u] = __builtin_nontemporal_load(reinterpret_cast<const u32x4_t *>(dp + (int64_t)at * P::N));
            }
        }
    };
    request(p0 + tid);

    const float m = a.stats[2 * row], rest = a.stats[2 * row + 1];
    const bool empty = rest == -1.f;
    RowTerms t;
    {
        const double c = 1.4426950408889634074 / (double)a.tau;
        t.c = (float)c;
        t.c_low = (float)(c - (double)t.c);
    }
    t.m = empty ? 0.f : m;
    const float inv_s = empty ? 0.f : 1.f / (1.f + rest);
    t.k0 = t.k1 = 0.f;
    int named = -1;
    double q = 0.0, mass = 0.0;
    if constexpr (TEACHER) {
        __shared__ double part[NT / 64];
        __shared__ __align__(16) int ids[NT];
        __shared__ double qs[NT];
        const TeacherEntry e = teacher_entry<NT, true>(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, V, a.tau, row, part);
        named = e.id;
        q = e.q;
        mass = e.mass;
        t.k0 = (float)((double)a.d_loss[row] * mass / (double)a.tau) * inv_s;
        ids[tid] = named;
        qs[tid] = q;
        __syncthreads();
        if (named < v0 || named >= v1) named = -1;
        if (named >= 0)                  // an id that stands there more than once: its first entry takes them all
            for (int j = 0; j < a.K && named >= 0; j += 4) {     // (threads behind K have id -1)
                const int4 four = *reinterpret_cast<const int4 *>(ids + j);
                const int id[4] = {four.x, four.y, four.z, four.w};
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (id[i] == e.id && j + i != tid) {
                        if (j + i < tid) named = -1;
                        else q += qs[j + i];
                    }
            }
    } else {
        const int target = a.targets ? a.targets[row] : -1;
        const bool there = target >= 0 && target < V;
        const float g = there ? a.d_logprob[row] : 0.f;
        if (tid == 0 && target >= v0 && target < v1) named = target;
        float k0 = -g / a.tau;
        if (a.d_entropy && !empty) {
            const float h = a.d_entropy[row] / a.tau;
            k0 -= h * (a.entropy[row] - log1pf(rest));
            t.k1 = -h * 0.693147180559945f * inv_s;
        }
        t.k0 = k0 * inv_s;
    }
    if (empty) t.k0 = 0.f;               // whatever the gradient of an infinite loss is
    // the named token's value, before the pass below may write over its logit
    float exact = 0.f;
    if (named >= 0) {
        if (!empty) {
            const double d = ((double)widen(z[named]) - (double)m) / (double)a.tau, s = 1.0 + (double)rest;
            double v;
            if constexpr (TEACHER) v = (double)a.d_loss[row] * ((expm1(d) * mass + (mass - q) - q * (double)rest) / s);
            else {
                v = a.d_logprob ? (double)a.d_logprob[row] * (((double)rest - expm1(d)) / s) : 0.0;
                if (a.d_entropy && exp(d) > 0.0) v -= (double)a.d_entropy[row] * (exp(d) / s) * (d - log1p((double)rest) + (double)a.entropy[row]);
            }
            exact = (float)(v / (double)a.tau);
        }
        if (ADD) exact += widen(dz[named]);
    }
    __syncthreads();

    // the values outside whole pieces, one to a thread
    {
        const int behind = head + pieces * P::N;
        int v = -1;
        if (seg == 0 && tid < head) v = tid;
        if (seg == segs - 1 && tid >= 32 && tid - 32 < V - behind) v = behind + tid - 32;
        if (v >= 0) put_one(dz + v, term<FINE>(t, widen(z[v])) + (ADD ? widen(dz[v]) : 0.f));
    }
    for (int p = p0 + tid; p < p1; p += PIECES * NT) {
        u32x4_t now[PIECES], add[ADD ? PIECES : 1];
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            now[u] = in[u];
            if constexpr (ADD) add[u] = old[u];
        }
        request(p + PIECES * NT);
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            if (p + u * NT >= p1) break;
            float v[P::N], w[P::N];
            P::get(now[u], v);
            if constexpr (ADD) P::get(add[u], w);
#pragma unroll
            for (int i = 0; i < P::N; ++i) v[i] = ADD ? term<FINE>(t, v[i]) + w[i] : term<FINE>(t, v[i]);
            u32x4_t *to = reinterpret_cast<u32x4_t *>(dp + (int64_t)(p + u * NT) * P::N);
            if constexpr (KEEP) *to = P::put(v);
            else __builtin_nontemporal_store(P::put(v), to);
        }
    }
    __syncthreads();
    if (named >= 0) put_one(dz + named, exact);
}

}  // namespace

namespace {

// Named tokens are stored a second time, which takes the rest of their line back from memory if it has left the caches: with more
// than one in 256 the stores stay there (past the caches / kept, us: 8192 rows of 2048, 64 listed tokens 26.7 / 22.7; of 8192
// 73 / 65; 333 of 102,400 fp32 52.8 / 56.4; 4096 of 151,936, 128 listed 498 / 590).
constexpr int KEEP_FROM = 256;

template <int NT> remoe_status launch_grad(const HeadGradArgs &a, int64_t segs, int seg_pieces, hipStream_t stream)
{
    auto pick = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (!a.teacher_idx) return a.accumulate ? head_grad_kernel<NT, DT, false, true, false> : head_grad_kernel<NT, DT, false, false, false>;
        if ((int64_t)a.K * KEEP_FROM > a.V) return a.accumulate ? head_grad_kernel<NT, DT, true, true, true> : head_grad_kernel<NT, DT, true, false, true>;
        return a.accumulate ? head_grad_kernel<NT, DT, true, true, false> : head_grad_kernel<NT, DT, true, false, false>;
    };
    auto kernel = a.dtype == REMOE_BF16 ? pick(std::integral_constant<int, REMOE_BF16>()) : pick(std::integral_constant<int, REMOE_F32>());
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * segs)), dim3(NT), 0, stream, a, (int)segs, seg_pieces);
    return check_hip(hipGetLastError(), "head_grad_kernel launch");
}

}  // namespace

// Workgroups of 256 threads, enough of them to even out the compute units, each with at least 2 pieces a thread, or 4 where a
// teacher's list is taken first (1024 rows of 8192: 1 / 2 pieces 9.0 / 8.2 us; 1024 of 32,000, 64 listed tokens: 2 / 4 pieces
// 39.9 / 31.5; 333 of 102,400 fp32: 4096 / 8192 workgroups 59.8 / 52.8).  A wavefront a row where many rows are short: its sums over
// the list wait for no other (256 / 64 threads, 8192 rows of 2048 18.0 / 14.5 us, with 64 listed tokens 39.5 / 26.7; of 8192 46.7 / 52.5);
// a list of more than 64 needs the threads, one an entry.  Every workgroup takes the whole list before it stores, which short rows do
// not hide (8192 bf16 rows, none / 64 / 65 / 128 / 256 listed, us: of 2048 14.4 / 22.9 / 42.3 / 54 / 97; of 8192 47 / 66 / 66 / 75 / 106).
constexpr int WORKGROUPS = 8192, SHORT_PIECES = 512, MANY_ROWS = 1024;

remoe_status launch_head_backward(const HeadGradArgs &a, hipStream_t stream)
{
    const int64_t pieces = ceil_div(a.V, a.dtype == REMOE_BF16 ? 8 : 4);
    const int threads = pieces <= SHORT_PIECES && a.T >= MANY_ROWS && a.K <= 64 ? 64 : 256;
    const int64_t most = ceil_div(pieces, threads * (a.teacher_idx ? 4 : 2));
    int64_t segs = ceil_div(WORKGROUPS, a.T);
    if (segs > most) segs = most;
    const int seg_pieces = (int)ceil_div(pieces, segs);
    segs = ceil_div(pieces, seg_pieces);
    return threads == 64 ? launch_grad<64>(a, segs, seg_pieces, stream) : launch_grad<256>(a, segs, seg_pieces, stream);
}

}  // namespace remoe
