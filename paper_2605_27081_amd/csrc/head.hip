// Log probabilities of given tokens, entropy and top alternatives of rows of logits; divergence from a teacher's top
// logits.  With m the largest logit of a row and d_v = (z_v - m) / tau:
//
//   S = sum_v exp(d_v) = 1 + rest,  ln p_v = d_v - log1p(rest),  H = log1p(rest) - sum_v d_v exp(d_v) / S
//   loss = sum_j q_j (ln q_j - ln p_id(j))
//
// head_scan_kernel reads a row, or a part of one, once: 16-byte pieces dealt out to the threads of a workgroup, each of which keeps
// the largest logit it has seen and the sums of e^d and d e^d relative to it, 32 logits at a time, while the next 32 are on their
// way.  rest leaves out the largest logit's own 1, which a running sum cannot take back: the thread that has the largest logit has
// its pieces read once more, a piece by every thread of the workgroup.
//
// Alternatives: every wavefront has a bound that n / wavefronts of its lanes' maxima reach, so n logits of the row reach the
// least of the bounds, and not many more do.  The maxima of every 32 logits are kept in LDS; those that reach it have their pieces
// read again, and the logits found are ranked by counting the larger ones.  Where too many reach it (ties by the thousand, as under
// a mask that leaves fewer than n tokens), or the row holds NaN, every wavefront keeps a sorted list, an entry per lane, over its
// share of the row.
//
// Long rows that are few are cut into parts; head_join_kernel puts the parts together.
//
// Bound by HBM for many rows: 8192 rows of 151,936 bf16 logits with entropy 381 us = 6.5 TB/s (8192 of 65,536 fp32 318 us, 6.8), where
// the vector instructions (9.7 issue slots a bf16 logit, two of them the exponential) fill nine tenths of the time; by those for less
// than two rows a compute unit (333 rows of 102,400: 16 us); by latency for few (one row with 20 alternatives 9 + 6 us of kernels).  An
// element at a time in three passes took 2530 us, 257 (333 rows) and 1767 (one).
#include <type_traits>

#include "head_plan.h"
#include "head_rows.h"
#include "topk.h"

namespace remoe {

namespace {

constexpr float LN2 = 0.693147180559945309417f;
constexpr float LOWEST = -3.402823466e38f;
constexpr int BATCH = HEAD_BATCH;
constexpr int MAX_N = 64;
constexpr int FOUND = 512;                              // logits that may reach the bound

// ln p of a logit; log_s = log1p(rest).  In fp64: the difference of two fp32 numbers need not be one.  (Code that a row passes once
// is kept short throughout: few rows find none of it in the instruction cache, and 64 bytes of it cost 100 cycles then.)
__device__ __forceinline__ float log_p(const RowSums &r, float log_s, float z, float tau)
{
    return r.rest == -1.f ? -__builtin_inff() : (float)(((double)z - (double)r.m) / (double)tau - (double)log_s);      // (-1: nothing but -inf)
}

// Order of the alternatives: larger logits first, NaN above all, the lower id first among equals.
__device__ __forceinline__ uint32_t order_of(float z)
{
    const uint32_t u = __float_as_uint(z + 0.0f);            // -0 as +0
    return z != z ? 0xFFFFFFFEu : u ^ (u >> 31 ? 0xFFFFFFFFu : 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t order)
{
    return __uint_as_float(order >> 31 ? order ^ 0x80000000u : ~order);
}
__device__ __forceinline__ uint64_t rank_key(float z, int id) { return (uint64_t)order_of(z) << 32 | (0xFFFFFFFFu - (uint32_t)id); }
__device__ __forceinline__ int key_id(uint64_t key) { return (int)(0xFFFFFFFFu - (uint32_t)key); }

// Exponents to base 2.  C = log2 e / tau is not an fp32 number: what is cut off it would make every exponential wrong in the same
// direction, by up to 2^-23 |d|, so it is kept in two.
struct Scale {
    float c, low;                                             // c rounded towards 0; low > 0, so that -inf stays -inf
    __device__ __forceinline__ explicit Scale(float tau)
    {
        const double all = 1.4426950408889634074 / (double)tau;
        c = __double2float_rz(all);
        low = fmaxf((float)(all - (double)c), 1e-30f);
    }
    // C d of a difference of logits
    __device__ __forceinline__ float of_difference(float d) const { return fmaf(d, low, d * c); }
    // C z - ref, each rounded as the result is: two instructions a logit where a difference first takes three
    __device__ __forceinline__ float against(float z, float ref) const { return fmaf(z, low, fmaf(z, c, -ref)); }
    // A reference for sums over logits up to z: C z, to 2^-24 of it.  Beyond 2^26 that would be off by more than a few, which an
    // exponential does not forgive: there it stays at 2^26 and is of no use unless a larger logit takes over.
    __device__ __forceinline__ float reference(float z) const { return __builtin_amdgcn_fmed3f(z * c, -0x1p26f, 0x1p26f); }
    __device__ __forceinline__ bool refers(float z) const { return fabsf(z * c) < 0x1p26f; }
};

// From sums relative to 2^from to sums relative to 2^(from - shift): 2^-512 is 0, and the floor keeps -inf out of products with 0.
struct Rescale {
    float dx, f;
    __device__ __forceinline__ explicit Rescale(float shift) : dx(fmaxf(shift, -512.f)), f(__builtin_amdgcn_exp2f(dx)) {}
};

// The outputs of a row that one thread writes, from its sums.  target, target_z: its token and that one's logit.
__device__ __forceinline__ void finish_row(const HeadArgs &a, int64_t row, const RowSums &r, float log_s, int target, float target_z)
{
    if (a.stats) {
        a.stats[2 * row] = r.m;
        a.stats[2 * row + 1] = r.rest;
    }
    if (a.targets) a.logprob[row] = target >= 0 && target < a.V ? log_p(r, log_s, target_z, a.tau) : 0.f;
    if (a.entropy) {
        const float h = r.rest == -1.f ? 0.f : log_s - r.xsum * LN2 / (1.f + r.rest);
        a.entropy[row] = h < 0.f ? 0.f : h;
    }
}

// The divergence from the teacher's list, by a workgroup of at least K threads.
template <int NT, typename elem>
__device__ __forceinline__ void finish_teacher(const HeadArgs &a, int64_t row, const elem *z, const RowSums &r, double *part)
{
    const TeacherEntry e = teacher_entry<NT, false>(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, a.V, a.tau, row, part);
    double term = 0.0;
    if (e.q != 0.0) {
        const double lp = r.rest == -1.f ? -(double)__builtin_inff()
                                         : ((double)widen(z[e.id]) - (double)r.m) / (double)a.tau - log1p((double)r.rest);
        term = e.q * (e.log_q - lp);
    }
    const double loss = block_reduce<NT>(term, part, OpSum());
    if (threadIdx.x == 0) a.loss[row] = r.rest != r.rest ? r.rest : (float)loss;
}

// The token of a row and its logit, asked for ahead of their use (by every thread: the token is a scalar load then).
template <typename elem> __device__ __forceinline__ void request_target(const HeadArgs &a, int64_t row, const elem *z, int &target, float &target_z)
{
    if (!a.targets) return;
    target = a.targets[row];
    if (target >= 0 && target < a.V) target_z = widen(z[target]);
}

// A bound that at least n of a wavefront's values, one a lane, reach, and no more than a quarter more than n where they differ
// enough: bisection between the smallest and the largest.
__device__ __forceinline__ uint32_t bound_of(uint32_t value, int n)
{
    uint32_t lo = wave_min_u32(value);                        // all reach it
    uint32_t hi = ~wave_min_u32(~value) + 1;                  // none does
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const int reach = __popcll(__ballot(value >= mid));
        if (reach < n) hi = mid;
        else {
            lo = mid;
            if (reach <= n + n / 4) break;
        }
    }
    return lo;
}

// The n largest of `count` keys, all different but for zeros (which are none), in their order: four lanes count the larger ones
// of each, eight on their way at a time.
template <int NT, typename Emit> __device__ __forceinline__ void ranked(const uint64_t *keys, int count, int n, Emit emit)
{
    const int q = threadIdx.x & 3;
    for (int i = threadIdx.x >> 2; i < count; i += NT / 4) {
        const uint64_t key = keys[i];
        int larger = 0;
        for (int j = q; j < count; j += 32) {
            uint64_t other[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) other[u] = keys[j + 4 * u < count ? j + 4 * u : i];      // (not larger than itself)
#pragma unroll
            for (int u = 0; u < 8; ++u) larger += other[u] > key;
        }
        larger += __shfl_xor(larger, 1, 64);
        larger += __shfl_xor(larger, 2, 64);
        if (q == 0 && key && larger < n) emit(larger, key);
    }
}

// A sorted list of a wavefront's n largest keys, lane i holds the i-th.  Any order of the keys will do.
struct SortedList {
    uint64_t mine = 0, least = 0;                             // least: the n-th, which a key has to exceed

    __device__ __forceinline__ static uint64_t from_lane(uint64_t v, int lane)
    {
        return (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)v, lane);
    }
    __device__ __forceinline__ static uint64_t from_left(uint64_t v)          // the lane below's (DPP wave_shr:1)
    {
        const int hi = __builtin_amdgcn_update_dpp(0, (int)(v >> 32), 0x138, 0xF, 0xF, false);
        const int lo = __builtin_amdgcn_update_dpp(0, (int)v, 0x138, 0xF, 0xF, false);
        return (uint64_t)(uint32_t)hi << 32 | (uint32_t)lo;
    }
    // a key of every lane (0: none)
    __device__ __forceinline__ void offer(uint64_t key, int n)
    {
        const int lane = threadIdx.x & 63;
        uint64_t better = __ballot(key > least);
        while (better) {
            const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)better) - 1);
            const uint64_t k = from_lane(key, l);
            const int at = __popcll(__ballot(mine > k));
            const uint64_t below = from_left(mine);
            mine = lane < at ? mine : lane == at ? k : below;
            least = from_lane(mine, n - 1);
            better &= better - 1;
            better &= __ballot(key > least);
        }
    }
};

// The list of pieces [p0, p1); the first value of the first piece of zp has the id id0.
template <int DT> __device__ __forceinline__ void offer_pieces(SortedList &list, const typename LogitOf<DT>::type *zp, int id0, int p0, int p1, int n)
{
    typedef Piece<DT> P;
    constexpr int FLIGHT = 4;                                 // pieces of a lane that are on their way together
    const int lane = threadIdx.x & 63;
    for (int p = p0 + lane; p - lane < p1; p += 64 * FLIGHT) {
        u32x4_t in[FLIGHT];
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            in[u] = P::lowest();
            if (p + 64 * u < p1) in[u] = *reinterpret_cast<const u32x4_t *>(zp + (int64_t)(p + 64 * u) * P::N);
        }
#pragma unroll
        for (int u = 0; u < FLIGHT; ++u) {
            const bool there = p + 64 * u < p1;
            const int id = id0 + (p + 64 * u) * P::N;
            const float least = value_of((uint32_t)(list.least >> 32));       // NaN at first: nothing is below it
            const bool behind = id > key_id(list.least);                      // equals come too late
            float v[P::N];
            P::get(in[u], v);
            bool some = false;
#pragma unroll
            for (int k = 0; k < P::N; ++k) some |= behind ? !(v[k] <= least) : !(v[k] < least);
            if (!__ballot(there && some)) continue;
#pragma unroll 1
            for (int k = 0; k < P::N; ++k) {
                float vk = v[0];
#pragma unroll
                for (int i = 1; i < P::N; ++i) vk = k == i ? v[i] : vk;
                list.offer(there ? rank_key(vk, id + k) : 0, n);
            }
        }
    }
}

struct PartOut {              // a part's results in the workspace
    RowSums *sums;            // [T, parts]
    uint64_t *keys;           // [T, parts, n], descending, 0 where there are fewer
};

// ONCE: loads of the stream that leave nothing in the caches.
template <int NT, int DT, bool ENTROPY, bool TOP, bool TEACHER, bool ONCE>
__global__ __launch_bounds__(NT) void head_scan_kernel(const HeadArgs a, int parts, int part_len, PartOut out)
{
    typedef typename LogitOf<DT>::type elem;
    typedef Piece<DT> P;
    constexpr int PIECES = BATCH / P::N, WAVES = NT / 64;
    extern __shared__ float block_max[];                      // [batches + 1, threads]: the maxima of every 32 logits
    __shared__ double part[TEACHER ? WAVES : 1];
    __shared__ float wave_m[WAVES], sums[3][WAVES];
    __shared__ int wave_first[WAVES], n_found, n_blocks;
    __shared__ uint16_t blocks[TOP ? FOUND : 1];
    __shared__ uint32_t wave_bound[WAVES];
    __shared__ uint64_t found[TOP ? FOUND : 1];
    const int64_t row = blockIdx.x / (unsigned)parts;
    const int p = blockIdx.x % (unsigned)parts;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    const int v0 = p * part_len, len = a.V - v0 < part_len ? a.V - v0 : part_len;
    const elem *zs = z + v0;
    // values in front of the first aligned piece, whole pieces, values behind the last
    int head = (int)((16 - ((uintptr_t)zs & 15)) & 15) / (int)sizeof(elem);
    if (head > len) head = len;
    const int pieces = (len - head) / P::N, behind = head + pieces * P::N;
    const elem *zp = zs + head;
    const int batches = (pieces + PIECES * NT - 1) / (PIECES * NT);
    const Scale c(a.tau);

    u32x4_t next[PIECES];
    // (the last piece again where there is none: no branch, and no registers to be set beforehand)
    auto request = [&](int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int at = (batch * PIECES + u) * NT + tid;
            const auto *from = reinterpret_cast<const u32x4_t *>(reinterpret_cast<const char *>(zp) + (uint32_t)(at < pieces ? at : pieces - 1) * 16u);
            next[u] = ONCE ? __builtin_nontemporal_load(from) : *from;
        }
    };
    if (batches > 0) request(0);
    int target = -1;
    float target_z = 0.f;
    if (parts == 1) request_target(a, row, z, target, target_z);
    // the value outside whole pieces that this thread has
    const int edge_at = tid < head ? tid : tid >= 32 && tid - 32 < len - behind ? behind + tid - 32 : -1;
    const float edge = edge_at >= 0 ? widen(zs[edge_at]) : -__builtin_inff();

    // m: largest so far; s, xs: sum 2^x and sum x 2^x, x relative to ref, which follows m
    float m = edge, ref = c.reference(fmaxf(edge, LOWEST)), s = 0.f, xs = 0.f;
    if (edge_at >= 0) {
        const float x = c.against(edge, ref);
        s = __builtin_amdgcn_exp2f(x);
        if constexpr (ENTROPY) xs = fmaxf(x, -512.f) * s;
    }
    if constexpr (TOP) block_max[batches * NT + tid] = edge;
    for (int b = 0; b < batches; ++b) {
        if (b + 1 == batches)
#pragma unroll
            for (int u = 0; u < PIECES; ++u)
                if ((b * PIECES + u) * NT + tid >= pieces) next[u] = P::lowest();
        float v[BATCH];
#pragma unroll
        for (int u = 0; u < PIECES; ++u) P::get(next[u], v + u * P::N);
#pragma unroll
        for (int i = 0; i < BATCH; ++i) asm volatile("" : "+v"(v[i]));        // taken out of `next` here, so that its registers are free
        if (b + 1 < batches) request(b + 1);
        float bm = v[0];
#pragma unroll
        for (int i = 1; i < BATCH; ++i) bm = fmaxf(bm, v[i]);
        if constexpr (TOP) block_max[b * NT + tid] = bm;
        m = fmaxf(m, bm);
        const float to = c.reference(fmaxf(m, LOWEST));
        const Rescale r(ref - to);
        ref = to;
        if constexpr (ENTROPY) xs = r.f * (xs + r.dx * s);
        s *= r.f;
        float s4[4] = {0.f, 0.f, 0.f, 0.f}, x4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float x = c.against(v[i], to), e = __builtin_amdgcn_exp2f(x);
            s4[i & 3] += e;
            if constexpr (ENTROPY) x4[i & 3] = fmaf(fmaxf(x, -512.f), e, x4[i & 3]);
        }
        s += (s4[0] + s4[1]) + (s4[2] + s4[3]);
        if constexpr (ENTROPY) xs += (x4[0] + x4[1]) + (x4[2] + x4[3]);
    }

    // the largest logit and the first thread that has it; a bound that n threads' maxima reach, if n / WAVES of every wavefront do
    {
        const float wm = wave_max(m);
        const uint64_t has = __ballot(m == wm);
        uint32_t reached = 0;
        if constexpr (TOP) reached = bound_of(order_of(m), (a.top_n + WAVES - 1) / WAVES);
        if (lane == 0) {
            wave_m[wave] = wm;
            wave_first[wave] = has ? __ffsll((unsigned long long)has) - 1 : 0;
            if constexpr (TOP) wave_bound[wave] = reached;
        }
        if constexpr (TOP)
            if (tid == 0) n_found = n_blocks = 0;
    }
    __syncthreads();
    float top = wave_m[0];
    int owner = wave_first[0];
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
        if (wave_m[w] > top) {
            top = wave_m[w];
            owner = w * 64 + wave_first[w];
        }
    u32x4_t own = P::lowest();                                // a piece of the owner's
    if (tid * NT + owner < pieces) own = *reinterpret_cast<const u32x4_t *>(zp + (int64_t)(tid * NT + owner) * P::N);
    float least = 0.f;                                        // logits that reach it may be alternatives
    if constexpr (TOP) {
        uint32_t l = wave_bound[0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) l = min(l, wave_bound[w]);
        least = value_of(l);
        // this thread's blocks of 32 that hold some (the last ones may be nothing but padding)
        if (m >= least) {
            uint32_t hits = 0;
#pragma unroll 4
            for (int b = 0; b < batches; ++b) hits |= (block_max[b * NT + tid] >= least && b * PIECES * NT + tid < pieces ? 1u : 0u) << b;
            while (hits) {
                const int b = __ffs(hits) - 1, at = atomicAdd(&n_blocks, 1);
                hits &= hits - 1;
                if (at < FOUND) blocks[at] = (uint16_t)(b * NT + tid);
            }
            if (edge_at >= 0 && edge >= least) {
                const int at = atomicAdd(&n_found, 1);
                if (at < FOUND) found[at] = rank_key(edge, v0 + edge_at);
            }
        }
    }
    // sums relative to 2^(C top)
    if (c.refers(top)) {
        const float to = c.reference(top);
        const Rescale r((ref - to) - c.against(top, to));
        if constexpr (ENTROPY) xs = r.f * (xs + r.dx * s);
        s *= r.f;
    } else if (top > -__builtin_inff()) {                     // from the differences then, in a pass of its own
        s = xs = 0.f;
        auto add = [&](float z) __attribute__((always_inline)) {
            const float x = c.of_difference(z - top), e = __builtin_amdgcn_exp2f(x);
            s += e;
            if constexpr (ENTROPY) xs = fmaf(fmaxf(x, -512.f), e, xs);
        };
        if (edge_at >= 0) add(edge);
#pragma unroll 1
        for (int i = tid; i < pieces; i += NT) {
            float v[P::N];
            P::get(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)i * P::N), v);
#pragma unroll
            for (int k = 0; k < P::N; ++k) add(v[k]);
        }
    }
    // the owner's logits once more: those below the largest, and how many equal it
    float equal = 0.f, again = 0.f;
    {
        if (tid == owner) {
            s = s == s ? 0.f : s;
            xs = 0.f;
        }
        float v[P::N + 1];
        P::get(own, v);
        v[P::N] = tid == owner ? edge : -__builtin_inff();
#pragma unroll
        for (int k = 0; k <= P::N; ++k) {
            const float x = fmaxf(c.of_difference(v[k] - top), -512.f), e = v[k] < top ? __builtin_amdgcn_exp2f(x) : 0.f;
            again += e;
            if constexpr (ENTROPY) xs = fmaf(x, e, xs);
            equal += v[k] == top ? 1.f : 0.f;
        }
    }
    s = wave_sum(s + again);
    equal = wave_sum(equal);
    if constexpr (ENTROPY) xs = wave_sum(xs);
    if (lane == 0) {
        sums[0][wave] = s;
        sums[1][wave] = equal;
        sums[2][wave] = xs;
    }
    __syncthreads();
    RowSums r;
    r.m = top;
    {
        float others = sums[0][0], same = sums[1][0];
        r.xsum = sums[2][0];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) {
            others += sums[0][w];
            same += sums[1][w];
            r.xsum += sums[2][w];
        }
        r.rest = top == -__builtin_inff() ? others - 1.f : others + (same - 1.f);
    }

    const float log_s = log1pf(r.rest);
    if (tid == NT - 64) {                                     // (the last wavefront has the least to do below)
        if (parts > 1) out.sums[row * parts + p] = r;
        else finish_row(a, row, r, log_s, target, target_z);
    }
    if constexpr (TOP) {
        const int n = a.top_n;
        const int nb = n_blocks;
        const bool few = r.rest == r.rest && nb <= FOUND;
        if (few)
            for (int i = tid; i < nb * PIECES; i += NT) {
                const int block = blocks[i / PIECES], piece = (block / NT * PIECES + i % PIECES) * NT + block % NT;
                if (piece >= pieces) continue;
                float v[P::N];
                P::get(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)piece * P::N), v);
                uint32_t reach = 0;
#pragma unroll
                for (int k = 0; k < P::N; ++k) reach |= v[k] >= least ? 1u << k : 0u;
                while (reach) {
                    const int k = __ffs(reach) - 1, to = atomicAdd(&n_found, 1);
                    reach &= reach - 1;
                    float vk = v[0];
#pragma unroll
                    for (int j = 1; j < P::N; ++j) vk = k == j ? v[j] : vk;
                    if (to < FOUND) found[to] = rank_key(vk, v0 + head + piece * P::N + k);
                }
            }
        __syncthreads();
        int nf = n_found;
        if (!few || nf > FOUND) {
            __syncthreads();                                  // every thread has read n_found
            SortedList list;
            const int share = (pieces + WAVES - 1) / WAVES, p0 = wave * share;
            offer_pieces<DT>(list, zp, v0 + head, p0, p0 + share < pieces ? p0 + share : pieces, n);
            if (wave == 0) list.offer(edge_at >= 0 ? rank_key(edge, v0 + edge_at) : 0, n);
            found[tid] = lane < n ? list.mine : 0;
            nf = NT;
            __syncthreads();
        }
        ranked<NT>(found, nf, n, [&](int rank, uint64_t key) {
            if (parts == 1) {
                a.top_idx[row * n + rank] = key_id(key);
                a.top_logprob[row * n + rank] = log_p(r, log_s, value_of((uint32_t)(key >> 32)), a.tau);
            } else {
                out.keys[(row * parts + p) * n + rank] = key;
            }
        });
        if (parts > 1)                                        // a part shorter than n
            for (int j = len + tid; j < n; j += NT) out.keys[(row * parts + p) * n + j] = 0;
    }
    if constexpr (TEACHER)
        if (parts == 1) finish_teacher<NT>(a, row, z, r, part);
}

// The parts of a row, a lane each.
constexpr int JOIN_THREADS = 256, JOIN_WAVES = JOIN_THREADS / 64;
template <int DT> __global__ __launch_bounds__(JOIN_THREADS) void head_join_kernel(const HeadArgs a, int parts, PartOut in)
{
    typedef typename LogitOf<DT>::type elem;
    __shared__ double part[JOIN_WAVES];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, n = a.top_n;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    const Scale c(a.tau);
    int target = -1;
    float target_z = 0.f;
    request_target(a, row, z, target, target_z);
    RowSums r{-__builtin_inff(), -1.f, 0.f};
    if (lane < parts) r = in.sums[row * parts + lane];
    const float top = wave_max(r.m);
    const uint64_t has = __ballot(r.m == top);
    const int owner = has ? __ffsll((unsigned long long)has) - 1 : 0;
    const Rescale scale(c.of_difference(fmaxf(r.m, LOWEST) - fmaxf(top, LOWEST)));
    const float whole = 1.f + r.rest;
    r.xsum = wave_sum(scale.f * (r.xsum + scale.dx * whole));
    r.rest = wave_sum(lane == owner ? r.rest : whole * scale.f);
    r.m = top;
    const float log_s = log1pf(r.rest);
    if (tid == JOIN_THREADS - 64) finish_row(a, row, r, log_s, target, target_z);
    if (n > 0) {
        __shared__ uint64_t found[HEAD_MAX_PARTS * MAX_N];
        __shared__ uint32_t wave_bound[JOIN_WAVES];
        __shared__ int n_found;
        // all parts' first keys, then their second, ...: a thread's first is its largest or close to it
        auto each_key = [&](auto take) __attribute__((always_inline)) {
            const int dp = JOIN_THREADS % parts, dr = JOIN_THREADS / parts;
#pragma unroll 1
            for (int p = tid % parts, rank = tid / parts; rank < n;) {
                take(in.keys[(row * parts + p) * n + rank]);
                rank += dr + (p + dp >= parts);
                p += p + dp >= parts ? dp - parts : dp;
            }
        };
        uint64_t most = 0;
        each_key([&](uint64_t key) __attribute__((always_inline)) { most = key > most ? key : most; });
        const uint32_t reached = bound_of((uint32_t)(most >> 32), (n + JOIN_WAVES - 1) / JOIN_WAVES);
        if (lane == 0) wave_bound[tid >> 6] = reached;
        if (tid == 0) n_found = 0;
        __syncthreads();
        uint32_t bound = wave_bound[0];
#pragma unroll
        for (int w = 1; w < JOIN_WAVES; ++w) bound = min(bound, wave_bound[w]);
        each_key([&](uint64_t key) __attribute__((always_inline)) {
            if (key && (uint32_t)(key >> 32) >= bound) found[atomicAdd(&n_found, 1)] = key;
        });
        __syncthreads();
        ranked<JOIN_THREADS>(found, n_found, n, [&](int rank, uint64_t k) {
            a.top_idx[row * n + rank] = key_id(k);
            a.top_logprob[row * n + rank] = log_p(r, log_s, value_of((uint32_t)(k >> 32)), a.tau);
        });
    }
    if (a.teacher_idx) finish_teacher<JOIN_THREADS>(a, row, z, r, part);
}

// (seven workgroups a compute unit by the bf16 kernels' registers, five by the fp32 ones')
constexpr int64_t ROWS_UNDER_WAY = 7 * 256, LAST_LEVEL = (int64_t)256 << 20;

template <int NT> remoe_status launch_scan(const HeadArgs &a, const HeadCut &cut, const PartOut &out, hipStream_t stream)
{
    const bool bf16 = a.dtype == REMOE_BF16, entropy = a.entropy != nullptr, top = a.top_n > 0;
    // Loads that leave nothing in the caches, unless alternatives are looked up again and the rows under way at a time fit the last
    // level (with and without, us: 8192 rows of 151,936 391 / 427, of 65,536 fp32 322 / 361; 4096 of 151,936 with a teacher's list
    // 201 / 226; 512 of 50,257 14.6 / 15.2; 256 of 32,000 7.3 / 6.5; 20 alternatives: 2048 of 151,936 114 / 130, 8192 of 32,000 117 / 115;
    // 64: 2048 of 32,000 42.1 / 41.2).  A call alone, that is; logits that fit the last level and are taken to their gradient next gain
    // from loads that stay, which a launch cannot know (both calls: 700 of 151,936 128 / 117, 2048 of 32,000 78 / 73, fp32 153 / 134).
    const int64_t under_way = a.T < ROWS_UNDER_WAY ? a.T : ROWS_UNDER_WAY;
    const bool once = under_way * a.V * (bf16 ? 2 : 4) > LAST_LEVEL;
    auto pick = [&](auto dt) {
        constexpr int DT = decltype(dt)::value;
        if (a.teacher_idx) return head_scan_kernel<NT, DT, false, false, true, true>;
        if (!top) return entropy ? head_scan_kernel<NT, DT, true, false, false, true> : head_scan_kernel<NT, DT, false, false, false, true>;
        if constexpr (NT >= 256)                              // (shorter rows always fit)
            if (once) return entropy ? head_scan_kernel<NT, DT, true, true, false, true> : head_scan_kernel<NT, DT, false, true, false, true>;
        return entropy ? head_scan_kernel<NT, DT, true, true, false, false> : head_scan_kernel<NT, DT, false, true, false, false>;
    };
    auto kernel = bf16 ? pick(std::integral_constant<int, REMOE_BF16>()) : pick(std::integral_constant<int, REMOE_F32>());
    const int64_t longest = cut.len < a.V ? cut.len : a.V;
    const size_t lds = top ? sizeof(float) * NT * (ceil_div(longest, NT * BATCH) + 1) : 0;
    if (a.T * cut.parts * NT > 0xFFFFFFFFll)
        return fail(REMOE_E_UNSUPPORTED, "%lld rows in %d parts are more than one launch can count", (long long)a.T, cut.parts);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * cut.parts)), dim3(NT), lds, stream, a, cut.parts, cut.len, out);
    return check_hip(hipGetLastError(), "head_scan_kernel launch");
}

}  // namespace

remoe_status launch_head_forward(const HeadArgs &a, hipStream_t stream)
{
    const HeadCut cut = head_cut(a.dtype, a.V, a.T, a.top_n, a.K);
    PartOut out{};
    if (cut.parts > 1) {
        out.sums = static_cast<RowSums *>(a.workspace);
        out.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(a.workspace) + head_keys_at(a.T * cut.parts));
    }
    const remoe_status st = cut.threads == 64    ? launch_scan<64>(a, cut, out, stream)
                            : cut.threads == 128 ? launch_scan<128>(a, cut, out, stream)
                            : cut.threads == 256 ? launch_scan<256>(a, cut, out, stream)
                                                 : launch_scan<512>(a, cut, out, stream);
    if (st != REMOE_OK || cut.parts == 1) return st;
    hipLaunchKernelGGL(a.dtype == REMOE_BF16 ? head_join_kernel<REMOE_BF16> : head_join_kernel<REMOE_F32>, dim3((unsigned)a.T), dim3(JOIN_THREADS), 0,
                       stream, a, cut.parts, out);
    return check_hip(hipGetLastError(), "head_join_kernel launch");
}

}  // namespace remoe
