// How the forward calls over the vocabulary deal out a batch of rows, and the workspace that takes: one plan for the launch and
// for remoe_head_workspace_bytes.  Host arithmetic only, for any C++ compiler.
#pragma once

#include <initializer_list>

#include "remoe.h"
#include "sizes.h"

namespace remoe {

constexpr int HEAD_BATCH = 32;                          // logits of a thread that are taken together
constexpr int HEAD_MAX_BATCHES = 32;                    // of a thread: bits of a mask
constexpr int64_t HEAD_MAX_PART = 1 << 18;              // logits of a part
constexpr int HEAD_MAX_PARTS = 64;                      // a lane each in the join

// what the logits of a row, or of a part of it, add up to: largest, sum of the e^d without one of the largest, sum of x 2^x
// (x = log2 e d)
struct RowSums { float m, rest, xsum; };

// Threads of a workgroup, parts of a row, logits of a part.
struct HeadCut { int threads, parts, len; };

// a bit of a mask for every batch of a thread, a thread for every piece of the owner's, no more LDS than lets four share a compute unit
static inline int64_t head_longest_part(int threads, int per)
{
    const int64_t bits = (int64_t)threads * HEAD_BATCH * HEAD_MAX_BATCHES, owners = (int64_t)threads * threads * per;
    return bits < owners ? (bits < HEAD_MAX_PART ? bits : HEAD_MAX_PART) : (owners < HEAD_MAX_PART ? owners : HEAD_MAX_PART);
}

// A row is one workgroup's unless it is long and there are few of it, because a second launch costs what 64 K logits take, and joining
// alternatives as much again.  With entropy, uncut / cut, us, without alternatives and with 20 (n) of them:
//   bf16   65,536: 1 row 7.8 / 9.9, n 10.3 / 12.7;  98,304: 48 rows 10.8 / 9.4, n 13.9 / 14.7;  102,400: 64 rows 11.8 / 9.3, n 15.1 / 16.1,
//          128 rows 12.2 / 12.2, n 16.0 / 20.6;  151,936: 1 row 14.1 / 9.2, n 16.9 / 14.4, 64 rows 15.2 / 11.9, n 18.8 / 20.3,
//          128 rows 15.5 / 15.4, n 19.4 / 25.1;  262,144: 96 rows 21.8 / 16.4
//   fp32   65,536: 1 row 8.1 / 9.3, n 10.1 / 12.6;  98,304: 48 rows 11.2 / 9.6, n 14.5 / 15.3;  102,400: 64 rows 12.6 / 10.4, n 16.0 / 17.3;
//          151,936: 1 row 14.5 / 9.3, n 16.8 / 14.0, 64 rows 16.4 / 13.9, n 20.0 / 22.2, 128 rows 18.4 / 19.1, n 22.8 / 29.7
// One rule for both types, with alternatives and without: it gives away 1-2 us with alternatives where half as many rows as its limit or
// more are cut, and 2-4 us without where 50 to 64 rows of 98,304 to 128,256 are not.
constexpr int HEAD_CUT_FROM = 98304, HEAD_CUT_LEN = 32768, HEAD_CUT_ROWS = 2048;
// A wavefront a row where rows are short and many, since nothing waits at a barrier then (256 / 64 threads, us: 8192 rows of 2048
// 32.5 / 14.8; of 8192 37.4 / 31.4, with 20 alternatives 53.8 / 44.2); not for more alternatives than half its lanes, whose bound would
// be too low (1024 rows of 2048, 64 alternatives: 15.7 / 102).  Rows too short to give the lanes of two wavefronts a piece have one
// whatever is asked for (8192 bf16 rows, 128 / 64 threads: of 600, 33 alternatives 129 / 30, 64 alternatives 162 / 193; of 1000,
// 33 alternatives 34 / 30, 64 alternatives 58 / 232).  Twice the threads for long rows as long as every compute unit has one at most
// (256 / 512 threads: 256 rows of 151,936 18.9 / 17.6, fp32 28.1 / 28.4; 128 of 102,400 13.0 / 12.3, fp32 17.4 / 16.1; 256 fp32 of
// 65,536 14.1 / 15.9; 333 of 102,400 19.2 / 21.1; 64 of 32,000 6.9 / 7.7).
constexpr int HEAD_LONG_ROW = 65536, HEAD_SHORT_ROW = 8192, HEAD_MANY_ROWS = 1024, HEAD_FEW_ROWS = 256;

static inline HeadCut head_cut(int dtype, int V, int64_t T, int top_n, int K)
{
    const int per = dtype == REMOE_BF16 ? 8 : 4;
    int threads = 256;
    if (V >= HEAD_LONG_ROW && T <= HEAD_FEW_ROWS) threads = 512;
    else if (V <= HEAD_SHORT_ROW && T >= HEAD_MANY_ROWS && top_n <= 32) threads = 64;
    while (threads > 64 && V < threads * per) threads >>= 1;  // every lane has a piece
    while (threads < K) threads <<= 1;                        // and a teacher's every entry a thread
    int64_t parts = ceil_div(V, head_longest_part(threads, per));
    const int64_t more = ceil_div(V, HEAD_CUT_LEN);
    if (V >= HEAD_CUT_FROM && T <= V / HEAD_CUT_ROWS && parts < more) parts = more < HEAD_MAX_PARTS ? more : HEAD_MAX_PARTS;
    const int64_t len = (int64_t)align_up(ceil_div(V, parts), threads * per);
    return {threads, (int)ceil_div(V, len), (int)len};
}

// The workspace of so many parts: their sums, and behind them their alternatives' keys.
static inline size_t head_keys_at(int64_t slots) { return align_up(sizeof(RowSums) * (size_t)slots, 256); }

// Parts that T rows or fewer come to at most, so that more tokens never ask for less.  A row's parts depend on T only through which
// side of HEAD_FEW_ROWS (threads, to which parts are aligned) and of V / HEAD_CUT_ROWS it lies on, and in between their number grows with
// T: the most is at T or at one of these.  (Alternatives and the teacher's list only matter to shorter rows.)
static inline int64_t head_slots(int dtype, int V, int64_t T)
{
    int64_t most = 0;
    for (int64_t rows : {T, (int64_t)HEAD_FEW_ROWS, (int64_t)(V / HEAD_CUT_ROWS)}) {
        if (rows > T) rows = T;
        const int parts = head_cut(dtype, V, rows, 0, 0).parts;
        if (parts > 1 && most < rows * parts) most = rows * parts;
    }
    return most;
}

static inline size_t head_workspace_bytes(int dtype, int V, int64_t T, int top_n)
{
    const int64_t slots = head_slots(dtype, V, T);
    return head_keys_at(slots) + align_up(sizeof(uint64_t) * (size_t)slots * top_n, 256) + 256;
}

}  // namespace remoe
