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
#ifndef HS_NT
#define HS_NT 256
#endif
#ifndef HS_MIN_UNITS
#define HS_MIN_UNITS 2
#endif

constexpr float LOG2E = 1.44269504088896340736f, LN2 = 0.693147180559945309417f;
constexpr float LOWEST = -3.402823466e38f;
constexpr int BATCH = 32;                               // logits of a thread that are taken together
constexpr int MAX_PART = 1 << 18;                       // logits of a part: 8192 batches
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

// The outputs of a row by its workgroup, from its sums.  target, target_z: its token and that one's logit.
template <int NT, typename elem>
__device__ __forceinline__ void finish_row(const HeadArgs &a, int64_t row, const elem *z, const RowSums &r, int target, float target_z, double *part)
{
    const int tid = threadIdx.x;
    if (tid == 0) {
        if (a.stats) {
            a.stats[2 * row] = r.m;
            a.stats[2 * row + 1] = r.rest;
        }
        if (a.targets) a.logprob[row] = target >= 0 && target < a.V ? log_p(r, target_z, a.tau) : 0.f;
        if (a.entropy) {
            const float h = r.rest == -1.f ? 0.f : log1pf(r.rest) - r.xsum * LN2 / (1.f + r.rest);
            a.entropy[row] = h < 0.f ? 0.f : h;
        }
    }
    if (a.teacher_idx) {
        const TeacherEntry e = teacher_entry<NT, false>(a.teacher_idx, a.teacher_logits, a.teacher_dtype, a.teacher_lse, a.K, a.V, a.tau, row, part);
        double term = 0.0;
        if (e.q != 0.0) {
            const double lp = r.rest == -1.f ? -(double)__builtin_inff()
                                             : ((double)widen(z[e.id]) - (double)r.m) / (double)a.tau - log1p((double)r.rest);
            term = e.q * (e.log_q - lp);
        }
        const double loss = block_reduce<NT>(term, part, OpSum());
        if (tid == 0) a.loss[row] = r.rest != r.rest ? r.rest : (float)loss;
    }
}

// The token of a row and its logit, asked for ahead of their use (by every thread: the token is a scalar load then).
template <typename elem> __device__ __forceinline__ void request_target(const HeadArgs &a, int64_t row, const elem *z, int &target, float &target_z)
{
    if (!a.targets) return;
    target = a.targets[row];
    if (target >= 0 && target < a.V) target_z = widen(z[target]);
}

// A bound that at least n of the EACH x 64 values of a wavefront reach, and no more than a quarter more than n where values
// differ enough: bisection between the smallest and the largest.
template <int EACH, typename U> __device__ __forceinline__ U bound_of(const U *value, int n)
{
    U least = value[0], most = value[0];
#pragma unroll
    for (int i = 1; i < EACH; ++i) {
        least = value[i] < least ? value[i] : least;
        most = value[i] > most ? value[i] : most;
    }
    U lo = wave_reduce(least, [](U a, U b) { return a < b ? a : b; });                // all reach it
    U hi = wave_reduce(most, [](U a, U b) { return a > b ? a : b; }) + 1;             // none does
    while (hi - lo > 1) {
        const U mid = lo + (hi - lo) / 2;
        int reach = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) reach += __popcll(__ballot(value[i] >= mid));
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

template <int NT, int DT, bool ENTROPY, bool TOP>
__global__ __launch_bounds__(NT) void head_scan_kernel(const HeadArgs a, int parts, int part_len, PartOut out)
{
    typedef typename LogitOf<DT>::type elem;
    typedef Piece<DT> P;
    constexpr int PIECES = BATCH / P::N, WAVES = NT / 64;
    extern __shared__ float block_max[];                      // [batches + 1, threads]: the maxima of every 32 logits
    __shared__ double part[WAVES];
    __shared__ float wave_m[WAVES], sums[3][WAVES];
    __shared__ int wave_first[WAVES];
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
    const float c = LOG2E / a.tau;

    u32x4_t next[PIECES];
    auto request = [&](int batch) __attribute__((always_inline)) {
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            const int at = (batch * PIECES + u) * NT + tid;
            next[u] = P::lowest();
            if (at < pieces) next[u] = *reinterpret_cast<const u32x4_t *>(zp + (int64_t)at * P::N);
        }
    };
    request(0);
    int target = -1;
    float target_z = 0.f;
    if (parts == 1) request_target(a, row, z, target, target_z);
    // the value outside whole pieces that this thread has
    const int edge_at = tid < head ? tid : tid >= 32 && tid - 32 < len - behind ? behind + tid - 32 : -1;
    const float edge = edge_at >= 0 ? widen(zs[edge_at]) : -__builtin_inff();

    // m: largest so far; s, xs: sums relative to ref, which is m, or the lowest number there is
    float m = edge, ref = fmaxf(edge, LOWEST), s = 0.f, xs = 0.f;
    if (edge_at >= 0) s = __builtin_amdgcn_exp2f((edge - ref) * c);
    if constexpr (TOP) block_max[batches * NT + tid] = edge;
    u32x4_t last[PIECES];
    for (int b = 0; b < batches; ++b) {
        float v[BATCH];
#pragma unroll
        for (int u = 0; u < PIECES; ++u) {
            last[u] = next[u];
            P::get(last[u], v + u * P::N);
        }
        if (b + 1 < batches) request(b + 1);
        float bm = v[0];
#pragma unroll
        for (int i = 1; i < BATCH; ++i) bm = fmaxf(bm, v[i]);
        if constexpr (TOP) block_max[b * NT + tid] = bm;
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
    __shared__ float thread_m[TOP ? NT : 1];
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
    for (int w = 1; w < WAVES; ++w)
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
        auto below = [&](const u32x4_t piece) __attribute__((always_inline)) {
            float v[P::N];
            P::get(piece, v);
#pragma unroll
            for (int k = 0; k < P::N; ++k) {
                const float e = __builtin_amdgcn_exp2f((v[k] - to) * c);
                again += v[k] < top ? e : 0.f;
                equal += v[k] == top ? 1.f : 0.f;
            }
        };
        if (batches > 1) {
            for (int i = tid; i * NT + owner < pieces; i += NT) below(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)(i * NT + owner) * P::N));
        } else if (tid == owner && batches == 1) {            // still at hand
#pragma unroll
            for (int u = 0; u < PIECES; ++u) below(last[u]);
        }
        if (tid == owner && edge_at >= 0) {
            const float e = __builtin_amdgcn_exp2f((edge - to) * c);
            again += edge < top ? e : 0.f;
            equal += edge == top ? 1.f : 0.f;
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
            uint32_t order[WAVES];
#pragma unroll
            for (int i = 0; i < WAVES; ++i) order[i] = order_of(thread_m[i * 64 + lane]);
            const uint32_t l = bound_of<WAVES>(order, a.top_n);
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

    if constexpr (TOP) {
        __shared__ uint64_t found[FOUND];
        __shared__ uint16_t blocks[FOUND];
        const int n = a.top_n;
        const float least = value_of(bound);
        for (int i = tid; i < (batches + 1) * NT; i += NT)
            // (blocks of nothing, the last ones and those of threads without a value of their own in the last row, are passed over)
            if (block_max[i] >= least && (i >= batches * NT ? edge_at >= 0 : i / NT * PIECES * NT + tid < pieces)) {
                const int at = atomicAdd(&n_blocks, 1);
                if (at < FOUND) blocks[at] = (uint16_t)i;
            }
        __syncthreads();
        const int nb = n_blocks;
        bool fits = r.rest == r.rest && nb <= FOUND;
        if (fits)
            for (int i = tid; i < nb * PIECES; i += NT) {
                const int block = blocks[i / PIECES], u = i % PIECES, b = block / NT, t = block % NT;
                float v[P::N];
                int at;                                       // of v[0]
                if (b == batches) {                           // a value outside whole pieces
                    at = t < head ? t : t >= 32 && t - 32 < len - behind ? behind + t - 32 : -1;
                    if (u > 0 || at < 0) continue;
                    v[0] = widen(zs[at]);
#pragma unroll
                    for (int k = 1; k < P::N; ++k) v[k] = __builtin_nanf("");
                } else {
                    const int piece = (b * PIECES + u) * NT + t;
                    if (piece >= pieces) continue;
                    P::get(*reinterpret_cast<const u32x4_t *>(zp + (int64_t)piece * P::N), v);
                    at = head + piece * P::N;
                }
                int reach = 0;
#pragma unroll
                for (int k = 0; k < P::N; ++k) reach += v[k] >= least;
                if (reach == 0) continue;
                int to = atomicAdd(&n_found, reach);
#pragma unroll
                for (int k = 0; k < P::N; ++k)
                    if (v[k] >= least) {
                        if (to < FOUND) found[to] = rank_key(v[k], v0 + at + k);
                        ++to;
                    }
            }
        __syncthreads();
        int nf = n_found;
        fits = fits && nf <= FOUND;
        if (!fits) {
            __syncthreads();                                  // every thread has read n_found
            const int quarter = (len + WAVES - 1) / WAVES;
            const int lo = wave * quarter, hi = lo + quarter < len ? lo + quarter : len;
            const uint64_t mine = sorted_list<DT>(zs, lo, hi, n);
            // (ids of the part so far)
            found[tid] = lane < n && mine ? mine - (uint64_t)v0 : 0;
            nf = NT;
            __syncthreads();
        }
        ranked<NT>(found, nf, n, [&](int rank, uint64_t key) {
            if (parts == 1) {
                a.top_idx[row * n + rank] = key_id(key);
                a.top_logprob[row * n + rank] = log_p(r, value_of((uint32_t)(key >> 32)), a.tau);
            } else {
                out.keys[(row * parts + p) * n + rank] = key;
            }
        });
        if (parts > 1)                                        // a part shorter than n
            for (int j = len + tid; j < n; j += NT) out.keys[(row * parts + p) * n + j] = 0;
    }
    if (parts > 1) {
        if (tid == 0) out.sums[row * parts + p] = r;
    } else {
        finish_row<NT>(a, row, z, r, target, target_z, part);
    }
}

// The parts of a row, a lane each.
constexpr int JOIN_THREADS = 256;
template <int DT> __global__ __launch_bounds__(JOIN_THREADS) void head_join_kernel(const HeadArgs a, int parts, PartOut in)
{
    typedef typename LogitOf<DT>::type elem;
    __shared__ double part[JOIN_THREADS / 64];
    const int64_t row = blockIdx.x;
    const int tid = threadIdx.x, lane = tid & 63, n = a.top_n;
    const elem *z = static_cast<const elem *>(a.logits) + row * a.ld;
    const float c = LOG2E / a.tau;
    int target = -1;
    float target_z = 0.f;
    request_target(a, row, z, target, target_z);
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
        constexpr int EACH = MAX_PARTS * MAX_N / JOIN_THREADS;
        __shared__ uint64_t found[MAX_PARTS * MAX_N], thread_top[JOIN_THREADS], bound;
        __shared__ int n_found;
        uint64_t key[EACH], most = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            // all parts' first keys, then their second, ...: a thread's first is its largest or close to it
            const int at = i * JOIN_THREADS + tid;
            key[i] = at < parts * n ? in.keys[(row * parts + at % parts) * n + at / parts] : 0;
        }
#pragma unroll
        for (int i = 0; i < EACH; ++i) most = key[i] > most ? key[i] : most;
        thread_top[tid] = most;
        if (tid == 0) n_found = 0;
        __syncthreads();
        if (tid < 64) {
            uint64_t value[JOIN_THREADS / 64];
#pragma unroll
            for (int i = 0; i < JOIN_THREADS / 64; ++i) value[i] = thread_top[i * 64 + lane];
            const uint64_t l = bound_of<JOIN_THREADS / 64>(value, n);
            if (lane == 0) bound = l;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (key[i] && key[i] >= bound) found[atomicAdd(&n_found, 1)] = key[i];
        __syncthreads();
        ranked<JOIN_THREADS>(found, n_found, n, [&](int rank, uint64_t k) {
            a.top_idx[row * n + rank] = key_id(k);
            a.top_logprob[row * n + rank] = log_p(r, value_of((uint32_t)(k >> 32)), a.tau);
        });
    }
    finish_row<JOIN_THREADS>(a, row, z, r, target, target_z, part);
}

// How rows are dealt out: threads of a workgroup, parts of a row, logits of a part.
struct Cut { int threads, parts, len; };
Cut cut_rows(int dtype, int V, int64_t T)
{
    const int per = dtype == REMOE_BF16 ? 8 : 4, threads = HS_NT, unit = threads * per;
    const int64_t least = ceil_div(V, MAX_PART);
    int64_t parts = T > 0 ? ceil_div(HS_WORKGROUPS, T) : MAX_PARTS;
    const int64_t most = ceil_div(V, HS_MIN_UNITS * unit);
    if (parts > most) parts = most;
    if (parts > MAX_PARTS) parts = MAX_PARTS;
    if (parts < least) parts = least;
    int64_t len = align_up(ceil_div(V, parts), unit);
    if (len > MAX_PART) len = MAX_PART;
    return {threads, (int)ceil_div(V, len), (int)len};
}

template <int NT> remoe_status launch_scan(const HeadArgs &a, const Cut &cut, const PartOut &out, hipStream_t stream)
{
    const bool bf16 = a.dtype == REMOE_BF16, entropy = a.entropy != nullptr, top = a.top_n > 0;
    auto kernel = [&]() {
        if (bf16) {
            if (top) return entropy ? head_scan_kernel<NT, REMOE_BF16, true, true> : head_scan_kernel<NT, REMOE_BF16, false, true>;
            return entropy ? head_scan_kernel<NT, REMOE_BF16, true, false> : head_scan_kernel<NT, REMOE_BF16, false, false>;
        }
        if (top) return entropy ? head_scan_kernel<NT, REMOE_F32, true, true> : head_scan_kernel<NT, REMOE_F32, false, true>;
        return entropy ? head_scan_kernel<NT, REMOE_F32, true, false> : head_scan_kernel<NT, REMOE_F32, false, false>;
    }();
    const int64_t longest = cut.len < a.V ? cut.len : a.V;
    const size_t lds = top ? sizeof(float) * NT * (ceil_div(longest, NT * BATCH) + 1) : 0;
    hipLaunchKernelGGL(kernel, dim3((unsigned)(a.T * cut.parts)), dim3(NT), lds, stream, a, cut.parts, cut.len, out);
    return check_hip(hipGetLastError(), "head_scan_kernel launch");
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
    PartOut out{};
    if (cut.parts > 1) {
        out.sums = static_cast<RowSums *>(a.workspace);
        out.keys = reinterpret_cast<uint64_t *>(static_cast<char *>(a.workspace) + align_up(sizeof(RowSums) * (size_t)(a.T * cut.parts), 256));
    }
    const remoe_status st = launch_scan<HS_NT>(a, cut, out, stream);
    if (st != REMOE_OK || cut.parts == 1) return st;
    hipLaunchKernelGGL(a.dtype == REMOE_BF16 ? head_join_kernel<REMOE_BF16> : head_join_kernel<REMOE_F32>, dim3((unsigned)a.T), dim3(JOIN_THREADS), 0,
                       stream, a, cut.parts, out);
    return check_hip(hipGetLastError(), "head_join_kernel launch");
}

}  // namespace remoe
