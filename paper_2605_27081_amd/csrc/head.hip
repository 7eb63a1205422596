// Log probabilities of given tokens, entropy and top alternatives of rows of logits; divergence from a teacher's top
// logits.  With m the largest logit of a row and d_v = (z_v - m) / tau:
//
//   S = sum_v exp(d_v) = 1 + rest,  ln p_v = d_v - log1p(rest),  H = log1p(rest) - sum_v d_v exp(d_v) / S
//   loss = sum_j q_j (ln q_j - ln p_id(j))
//
// head_scan_kernel reads a row, or a part of one, once: 16-byte pieces dealt out to 256 threads, each of which keeps the
// largest logit it has seen and the sums of e^d and d e^d relative to it, 32 logits at a time.  rest leaves out the largest
// logit's own 1, which a running sum cannot take back: the thread that has the largest logit has its pieces read once more (a
// piece per thread of the workgroup).
//
// Alternatives: the n-th largest of the threads' maxima is a bound that at least n logits reach, and not many more do, so the
// maxima of every 32 logits are kept in LDS; those that reach the bound have their pieces read again, and the logits found are
// ranked by counting the larger ones.  Where too many reach it (ties by the thousand: a mask that leaves fewer than n tokens), or
// the row holds NaN, every wavefront keeps a sorted list, an entry per lane, over a quarter of the row.
//
// Few rows are cut into parts; head_join_kernel puts the parts together.
#include "head_rows.h"
#include "topk.h"

namespace remoe {

namespace {

#ifndef HS_WORKGROUPS
#define HS_WORKGROUPS 2048
#endif
#ifndef HS_MIN_UNITS
#define HS_MIN_UNITS 2
#endif

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
constexpr float LOWEST = -3.402823466e38f;
constexpr int BATCH = 32;                               // logits of a thread that are taken together
constexpr int MAX_PART = 1 << 18;                       // logits of a part: 32 batches of every thread
constexpr int MAX_PARTS = 64;                           // a lane each in the join
constexpr int MAX_N = 64;
constexpr int FOUND = 1024;                             // logits that may reach the bound

// what the logits of a row, or of a part of it, add up to: largest, sum of the e^d without one of the largest, sum of x 2^x
// (x = log2 e d)
struct RowSums { float m, rest, xsum; };

__device__ __forceinline__ float log_p(const RowSums &r, float z, float tau)
{
    if (r.rest == -1.f) return -__builtin_inff();            // nothing but -inf
    return (z - r.m) / tau - log1pf(r.rest);
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

// The scale from sums relative to `from` to sums relative to `to`, and the shift of x.  2^-512 is 0, and the floor keeps
// -inf out of products with 0.
struct Rescale {
    float dx, f;
    __device__ __forceinline__ Rescale(float from, float to, float c) : dx(fmaxf((from - to) * c, -512.f)), f(__builtin_amdgcn_exp2f(dx)) {}
};

// The outputs of a row by its workgroup, from its sums.  target: thread 0's targets[row] (where there are targets); entry_z:
// this thread's teacher entry's logit comes from z.
template <typename elem>
__device__ __forceinline__ void finish_row(const HeadArgs &a, int64_t row, const elem *z, const RowSums &r, double *part)
{
    const int tid = threadIdx.x;
    if (tid == 0) {
        if (a.stats) {
            a.stats[2 * row] = r.m;
            a.stats[2 * row + 1] = r.rest;
        }
        if (a.targets) {
            const int t = a.targets[row];
            a.logprob[row] = t >= 0 && t < a.V ? log_p(r, widen(z[t]), a.tau) : 0.f;
        }
        if (a.entropy) {
            const float h = r.rest == -1.f ? 0.f : log1pf(r.rest) - r.xsum * LN2 / (1.f + r.rest);
            a.entropy[row] = h < 0.f ? 0.f : h;
        }
    }
    if (a.teacher_idx) {
        const TeacherEntry e = teacher_entry<false>(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, a.V, a.tau, row, part);
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

// A bound that at least n of the 4 x 64 values of a wavefront reach, and no more than a quarter more than n where values
// differ enough: bisection between the smallest and the largest.
__device__ __forceinline__ uint32_t bound_of(const uint32_t *order, int n)
{
    uint32_t least = min(min(order[0], order[1]), min(order[2], order[3])), most = max(max(order[0], order[1]), max(order[2], order[3]));
    least = wave_min_u32(least);
    most = ~wave_min_u32(~most);
    uint32_t lo = least, hi = most + 1;                       // all reach lo, none hi
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        int reach = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) reach += __popcll(__ballot(order[i] >= mid));
        if (reach < n) hi = mid;
        else {
            lo = mid;
            if (reach <= n + n / 4) break;
        }
    }
    return lo;
}

// The n largest keys of a stretch of values, by a wavefront: lane i holds the i-th.  Any order of the values will do.
template <int DT>
__device__ __forceinline__ uint64_t sorted_list(const typename LogitOf<DT>::type *z, int first, int last, int n)
{
    constexpr int N = 8;                                      // values of a lane that are on their way together
    const int lane = threadIdx.x & 63;
    uint64_t mine = 0, least = 0;
    for (int v = first; v < last; v += 64 * N) {
        uint64_t key[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int at = v + 64 * i + lane;
            key[i] = at < last ? rank_key(widen(z[at]), at) : 0;
        }
#pragma unroll
        for (int i = 0; i < N; ++i) {
            uint64_t better = __ballot(key[i] > least);
            while (better) {
                const int l = __ffsll((unsigned long long)better) - 1;
                const uint64_t k = __shfl(key[i], l, 64);
                const int at = __popcll(__ballot(mine > k));
                const uint64_t above = __shfl_up(mine, 1, 64);
                mine = lane < at ? mine : lane == at ? k : above;
                least = __shfl(mine, n - 1, 64);
                better &= better - 1;
                better &= __ballot(key[i] > least);
            }
        }
    }
    return mine;
}

struct PartOut {              // a part's results in the workspace
    RowSums *sums;            // [T, parts]
    uint64_t *keys;           // [T, parts, n], descending, 0 where there are fewer
};

template <int DT, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(HEAD_THREADS) void head_scan_kernel(const HeadArgs a, int parts, int part_len, PartOut out)
{
    typedef typename LogitOf<DT>::type elem;
    typedef Piece<DT> P;
    constexpr int PIECES = BATCH / P::N;
    extern __shared__ float block_max[];                      // [batches + 1, threads]: the maxima of every 32 logits
    __shared__ double part[HEAD_WAVES];
    __shared__ float wave_m[HEAD_WAVES], sums[3][HEAD_WAVES];
    __shared__ int wave_first[HEAD_WAVES];
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
    const int batches = (pieces + PIECES * HEAD_THREADS - 1) / (PIECES * HEAD_THREADS);
    const float c = LOG2E / a.tau;

    u32x4_t next[PIECES];
    auto request = [&](int batch) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int at = (batch * PIECES + u) * HEAD_THREADS + tid;
            next[u] = P::lowest();
            if (at < pieces) next[u] = *reinterpret_cast<const u32x4_t *>(zp + (int64_t)at * P::N);
        }
    };
    request(0);
    // the value outside whole pieces that this thread has
    const int edge_at = tid < head ? tid : tid >= 64 && tid - 64 < len - behind ? behind + tid - 64 : -1;
    const float edge = edge_at >= 0 ? widen(zs[edge_at]) : -__builtin_inff();

    // m: largest so far; s, xs: sums relative to ref, which is m, or the lowest number there is
    float m = edge, ref = fmaxf(edge, LOWEST), s = 0.f, xs = 0.f;
    if (edge_at >= 0) s = __builtin_amdgcn_exp2f((edge - ref) * c);
    if constexpr (TOP) block_max[batches * HEAD_THREADS + tid] = edge;
    for (int b = 0; b < batches; ++b) {
        float v[BATCH];
#pragma unroll
        for (int u = 0; u < PIECES; ++u) P::get(next[u], v + u * P::N);
        if (b + 1 < batches) request(b + 1);
        float bm = v[0];
#pragma unroll
        for (int i = 1; i < BATCH; ++i) bm = fmaxf(bm, v[i]);
        if constexpr (TOP) block_max[b * HEAD_THREADS + tid] = bm;
        m = fmaxf(m, bm);
        const float to = fmaxf(m, LOWEST);
        const Rescale r(ref, to, c);
        ref = to;
        if constexpr (ENTROPY) xs = r.f * (xs + r.dx * s);
        s *= r.f;
        float s4[4] = {0.f, 0.f, 0.f, 0.f}, x4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < BATCH; ++i) {
            const float x = (v[i] - to) * c, e = __builtin_amdgcn_exp2f(x);
            s4[i & 3] += e;
            if constexpr (ENTROPY) x4[i & 3] = fmaf(fmaxf(x, -512.f), e, x4[i & 3]);
        }
        s += (s4[0] + s4[1]) + (s4[2] + s4[3]);
        if constexpr (ENTROPY) xs += (x4[0] + x4[1]) + (x4[2] + x4[3]);
    }

    // the largest logit and the first thread that has it
    __shared__ float thread_m[TOP ? HEAD_THREADS : 1];
    if constexpr (TOP) thread_m[tid] = m;
    {
        const float wm = wave_max(m);
        const uint64_t has = __ballot(m == wm);
        if (lane == 0) {
            wave_m[wave] = wm;
            wave_first[wave] = has ? __ffsll((unsigned long long)has) - 1 : 0;
        }
    }
    __syncthreads();
    float top = wave_m[0];
    int owner = wave_first[0];
#pragma unroll
    for (int w = 1; w < HEAD_WAVES; ++w)
        if (wave_m[w] > top) {
            top = wave_m[w];
            owner = w * 64 + wave_first[w];
        }
    const float to = fmaxf(top, LOWEST);
    {
        const Rescale r(ref, to, c);
        if constexpr (ENTROPY) xs = r.f * (xs + r.dx * s);
        s *= r.f;
    }
    // the owner's logits once more: those below the largest, and how many equal it
    float equal = 0.f;
    {
        if (tid == owner) s = s == s ? 0.f : s;
        float again = 0.f;
        for (int i = tid; i * HEAD_THREADS + owner < pieces; i += HEAD_THREADS) {
            float v[P::N];
            P::get(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)(i * HEAD_THREADS + owner) * P::N), v);
#pragma unroll
            for (int k = 0; k < P::N; ++k) {
                if (v[k] < top) again += __builtin_amdgcn_exp2f((v[k] - to) * c);
                else if (v[k] == top) equal += 1.f;
            }
        }
        if (tid == owner && edge_at >= 0) {
            if (edge < top) again += __builtin_amdgcn_exp2f((edge - to) * c);
            else if (edge == top) equal += 1.f;
        }
        s += again;
    }
    s = wave_sum(s);
    equal = wave_sum(equal);
    if constexpr (ENTROPY) xs = wave_sum(xs);
    if (lane == 0) {
        sums[0][wave] = s;
        sums[1][wave] = equal;
        sums[2][wave] = xs;
    }
    __shared__ uint32_t bound;
    __shared__ int n_blocks, n_found;
    if constexpr (TOP) {
        if (wave == 0) {
            uint32_t order[HEAD_WAVES];
#pragma unroll
            for (int i = 0; i < HEAD_WAVES; ++i) order[i] = order_of(thread_m[i * 64 + lane]);
            const uint32_t l = bound_of(order, a.top_n);
            if (lane == 0) {
                bound = l;
                n_blocks = n_found = 0;
            }
        }
    }
    __syncthreads();
    RowSums r;
    r.m = top;
    {
        const float others = (sums[0][0] + sums[0][1]) + (sums[0][2] + sums[0][3]);
        const float same = (sums[1][0] + sums[1][1]) + (sums[1][2] + sums[1][3]);
        r.rest = top == -__builtin_inff() ? others - 1.f : others + (same - 1.f);
        r.xsum = (sums[2][0] + sums[2][1]) + (sums[2][2] + sums[2][3]);
    }

    if constexpr (TOP) {
        __shared__ uint64_t found[FOUND];
        __shared__ uint16_t blocks[FOUND];
        const int n = a.top_n;
        const float least = value_of(bound);
        for (int i = tid; i < (batches + 1) * HEAD_THREADS; i += HEAD_THREADS)
            if (block_max[i] >= least) {
                const int at = atomicAdd(&n_blocks, 1);
                if (at < FOUND) blocks[at] = (uint16_t)i;
            }
        __syncthreads();
        const int nb = n_blocks;
        bool fits = r.rest == r.rest && nb <= FOUND;
        if (fits)
            for (int i = tid; i < nb * PIECES; i += HEAD_THREADS) {
                const int block = blocks[i / PIECES], u = i % PIECES, b = block / HEAD_THREADS, t = block % HEAD_THREADS;
                auto keep = [&](float v, int at) {
                    if (v >= least) {
                        const int k = atomicAdd(&n_found, 1);
                        if (k < FOUND) found[k] = rank_key(v, v0 + at);
                    }
                };
                if (b == batches) {                           // a value outside whole pieces
                    const int at = t < head ? t : t >= 64 && t - 64 < len - behind ? behind + t - 64 : -1;
                    if (u == 0 && at >= 0) keep(widen(zs[at]), at);
                    continue;
                }
                const int at = (b * PIECES + u) * HEAD_THREADS + t;
                if (at >= pieces) continue;
                float v[P::N];
                P::get(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)at * P::N), v);
#pragma unroll
                for (int k = 0; k < P::N; ++k) keep(v[k], head + at * P::N + k);
            }
        __syncthreads();
        int nf = n_found;
        fits = fits && nf <= FOUND;
        if (!fits) {
            __syncthreads();                                  // every thread has read n_found
            const int quarter = (len + HEAD_WAVES - 1) / HEAD_WAVES;
            const int lo = wave * quarter, hi = lo + quarter < len ? lo + quarter : len;
            const uint64_t mine = sorted_list<DT>(zs, lo, hi, n);
            // (ids of the part so far)
            found[tid] = lane < n && mine ? mine - (uint64_t)v0 : 0;
            nf = HEAD_THREADS;
            __syncthreads();
        }
        for (int i = tid; i < nf; i += HEAD_THREADS) {
            const uint64_t key = found[i];
            if (!key) continue;
            int rank = 0;
            for (int j = 0; j < nf; ++j) rank += found[j] > key;
            if (rank >= n) continue;
            if (parts == 1) {
                a.top_idx[row * n + rank] = key_id(key);
                a.top_logprob[row * n + rank] = log_p(r, widen(z[key_id(key)]), a.tau);
            } else {
                out.keys[((row * parts) + p) * n + rank] = key;
            }
        }
        if (parts > 1)                                        // a part shorter than n
            for (int j = len + tid; j < n; j += HEAD_THREADS) out.keys[((row * parts) + p) * n + j] = 0;
    }
    if (parts > 1) {
        if (tid == 0) out.sums[row * parts + p] = r;
    } else {
        finish_row(a, row, z, r, part);
    }
}

// The parts of a row, a lane each.
template <int DT> __global__ __launch_bounds__(HEAD_THREADS) void head_join_kernel(const HeadArgs a, int parts, PartOut in)
{
    typedef typename LogitOf<DT>::type elem;
    __shared__ double part[HEAD_WAVES];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, n = a.top_n;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    const float c = LOG2E / a.tau;
    RowSums r{-__builtin_inff(), -1.f, 0.f};
    if (lane < parts) r = in.sums[row * parts + lane];
    const float top = wave_max(r.m);
    const uint64_t has = __ballot(r.m == top);
    const int owner = has ? __ffsll((unsigned long long)has) - 1 : 0;
    const Rescale scale(fmaxf(r.m, LOWEST), fmaxf(top, LOWEST), c);
    const float whole = 1.f + r.rest;
    r.xsum = wave_sum(scale.f * (r.xsum + scale.dx * whole));
    r.rest = wave_sum(lane == owner ? r.rest : whole * scale.f);
    r.m = top;
    if (n > 0) {
        __shared__ uint64_t keys[MAX_PARTS * MAX_N];
        for (int i = tid; i < parts * n; i += HEAD_THREADS) keys[i] = in.keys[row * parts * n + i];
        __syncthreads();
        for (int i = tid; i < parts * n; i += HEAD_THREADS) {
            const uint64_t key = keys[i];
            if (!key) continue;
            const int own = i / n;
            int rank = i - own * n;
            for (int p = 0; p < parts && rank < n; ++p) {
                if (p == own) continue;
                const uint64_t *list = keys + p * n;          // descending: how many of it are larger
                int at = 0;
#pragma unroll
                for (int step = MAX_N; step >= 1; step >>= 1)
                    if (at + step <= n && list[at + step - 1] > key) at += step;
                rank += at;
            }
            if (rank >= n) continue;
            a.top_idx[row * n + rank] = key_id(key);
            a.top_logprob[row * n + rank] = log_p(r, widen(z[key_id(key)]), a.tau);
        }
    }
    finish_row(a, row, z, r, part);
}

// Parts of a row: as many as give HS_WORKGROUPS workgroups, none shorter than HS_MIN_UNITS pieces a thread or longer than MAX_PART.
struct Cut { int parts, len; };
Cut cut_rows(int dtype, int V, int64_t T)
{
    const int unit = HEAD_THREADS * (dtype == REMOE_BF16 ? 8 : 4);
    const int64_t least = ceil_div(V, MAX_PART);
    int64_t parts = T > 0 ? ceil_div(HS_WORKGROUPS, T) : MAX_PARTS;
    const int64_t most = ceil_div(V, HS_MIN_UNITS * unit);
    if (parts > most) parts = most;
    if (parts > MAX_PARTS) parts = MAX_PARTS;
    if (parts < least) parts = least;
    int64_t len = align_up(ceil_div(V, parts), unit);
    if (len > MAX_PART) len = MAX_PART;
    return {(int)ceil_div(V, len), (int)len};
}

}  // namespace

// Never less for more tokens: T rows have at most T times the parts of one, and no more than HS_WORKGROUPS + T <= 2 HS_WORKGROUPS
// unless MAX_PART cuts every row (a row that is not cut leaves nothing here).
size_t head_workspace_bytes(int dtype, int V, int64_t T, int top_n)
{
    const Cut one = cut_rows(dtype, V, 1);
    const int64_t least = ceil_div(V, MAX_PART);
    int64_t slots = T * one.parts;
    const int64_t enough = 2 * HS_WORKGROUPS + (least > 1 ? T * least : 0);
    if (slots > enough) slots = enough;
    return align_up(sizeof(RowSums) * (size_t)slots, 256) + align_up(sizeof(uint64_t) * (size_t)slots * top_n, 256) + 256;
}

remoe_status launch_head_forward(const HeadArgs &a, hipStream_t stream)
{
    const Cut cut = cut_rows(a.dtype, a.V, a.T);
    const int per = a.dtype == REMOE_BF16 ? 8 : 4;
    PartOut out{};
    if (cut.parts > 1) {
        out.sums = static_cast<RowSums *>(a.workspace);
        out.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(a.workspace) + align_up(sizeof(RowSums) * (size_t)(a.T * cut.parts), 256));
    }
    const bool bf16 = a.dtype == REMOE_BF16, entropy = a.entropy != nullptr, top = a.top_n > 0;
    auto kernel = [&]() {
        if (bf16) {
            if (top) return entropy ? head_scan_kernel<REMOE_BF16, true, true> : head_scan_kernel<REMOE_BF16, false, true>;
            return entropy ? head_scan_kernel<REMOE_BF16, true, false> : head_scan_kernel<REMOE_BF16, false, false>;
        }
        if (top) return entropy ? head_scan_kernel<REMOE_F32, true, true> : head_scan_kernel<REMOE_F32, false, true>;
        return entropy ? head_scan_kernel<REMOE_F32, true, false> : head_scan_kernel<REMOE_F32, false, false>;
    }();
    const int64_t longest = cut.len < a.V ? cut.len : a.V;
    const size_t lds = top ? sizeof(float) * HEAD_THREADS * (ceil_div(longest / per, HEAD_THREADS * (BATCH / per)) + 1) : 0;
    const dim3 block(HEAD_THREADS);
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * cut.parts)), block, lds, stream, a, cut.parts, cut.len, out);
    if (cut.parts > 1)
        hipLaunchKernelGGL(bf16 ? head_join_kernel<REMOE_BF16> : head_join_kernel<REMOE_F32>, dim3((unsigned)a.T), block, 0, stream, a, cut.parts, out);
    return check_hip(hipGetLastError(), "head kernels launch");
}

}  // namespace remoe
