// How the attention over the cache is cut into equal shares: integer arithmetic
// that the kernels run and the host can run too (no HIP types).
//
// A unit is one row block (up to `rows` tokens' query heads of one key/value
// head) of one sequence, as long as the keys that it sees.  All units of a batch
// are laid end to end, sequence by sequence, head by head, block by block, and
// workgroup w of the plan takes keys [w * per, (w + 1) * per) of that line: no
// workgroup waits for a long sequence, whatever the lengths are.  A unit also counts
// what it costs beside its keys (reading its rows, its first tiles' latency, its end).
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define ATP_PLAN_FN __host__ __device__ __forceinline__
#else
#define ATP_PLAN_FN inline
#endif

namespace atp {
namespace plan {

constexpr int kTile = 128;     // keys that shares are cut at, where a unit's line is whole tiles
constexpr int kGroups = 512;   // shares: two workgroups per CU on 256 CUs
constexpr int kLeast = kTile;  // fewest keys of a share
// Units of up to 32 rows and of 128: the keys of a tile, and what a unit costs beside its
// keys, in keys.  Without it 300 short contexts' tokens (8 heads, 10 to 200 keys) take 55 us,
// 51 so (64: 52, 256: 51), 32 sequences of 4 drafts 53 and 52 (52, 49), 16 sequences' 24 rows
// 81 and 79 (83, 81); with 128 rows 24 drafted trees 131 and 116 (128: 124, 448: 116), prompt
// chunks 99 and 87 (94, 88), 128 rows over 131000 keys 183 and 131 (131, 127).
constexpr int kFewTile = 128, kFewExtra = 128;
constexpr int kWideTile = 64, kWideExtra = 320;

ATP_PLAN_FN int64_t whole_tiles(int64_t keys) { return (keys + kTile - 1) / kTile * kTile; }

struct Seq {
    int first, fresh;          // its rows of the step's buffers
    int ctx, keys;             // cached before the step; with the new ones
    int blocks;                // row blocks of a head
    int extra;                 // keys' worth of work that a unit costs beside its keys
};

// ctx, c0, c1: the sequence's ctx, cu_new[s], cu_new[s + 1] as they stand in device
// memory; tokens and cap (max_pages * page_size, <= 2^30) bound what they may name.
ATP_PLAN_FN Seq make_seq(int64_t ctx, int64_t c0, int64_t c1, int64_t tokens, int64_t cap,
                         int rows, int extra) {
    Seq q;
    c0 = c0 < 0 ? 0 : (c0 > tokens ? tokens : c0);
    c1 = c1 < c0 ? c0 : (c1 > tokens ? tokens : c1);
    ctx = ctx < 0 ? 0 : (ctx > cap ? cap : ctx);
    q.first = (int)c0;
    q.fresh = (int)(c1 - c0);
    q.ctx = (int)ctx;
    q.keys = (int)(ctx + q.fresh > cap ? cap : ctx + q.fresh);
    q.blocks = (q.fresh + rows - 1) / rows;
    q.extra = extra;
    return q;
}

// Keys that row block i of a causal sequence can see (all of them otherwise).
ATP_PLAN_FN int block_keys(const Seq& q, int i, int rows, bool causal) {
    if (!causal) return q.keys;
    const int64_t last = (int64_t)q.ctx + (int64_t)(i + 1) * rows;
    return last < q.keys ? (int)last : q.keys;
}

// Length on the line of the first n row blocks of a head: whole tiles of keys, so that
// short units are cut where tiles end; causal blocks of a sequence with several count ctx
// + (i + 1) * rows keys, the last one (or one beyond the table) more than it sees.  No
// division: workgroups find their units by this.
ATP_PLAN_FN int64_t line_of(const Seq& q, int64_t n, int rows, bool causal) {
    if (!causal || q.blocks <= 1) return n * (q.extra + whole_tiles(q.keys));
    return n * (q.extra + q.ctx) + rows * (n * (n + 1) / 2);
}

// The row block of key `at` of a head's line (0 <= at < line_of(blocks)).
ATP_PLAN_FN int block_of(const Seq& q, int64_t at, int rows, bool causal) {
    int lo = 0, hi = q.blocks - 1;      // last block whose start is <= at
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (line_of(q, mid, rows, causal) <= at) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Keys of a workgroup.
ATP_PLAN_FN int64_t share(int64_t total, int groups, int least) {
    const int64_t per = (total + groups - 1) / groups;
    return whole_tiles(per > least ? per : least);
}

// The key of a unit at which a cut at `at` of its line falls: the line begins with the unit's
// extra work, and cuts move up to whole tiles and to what the block sees (lim).
ATP_PLAN_FN int cut_key(int64_t at, int extra, int lim, int tile) {
    const int64_t k = at > extra ? (at - extra + tile - 1) / tile * tile : 0;
    return (int)(k < lim ? k : lim);
}

// Keys [first, last) that a piece [p0, p1) of a unit's line reads; `ends`: p1 is the line's
// end.  A cut that leaves nothing on one side is none: the piece there is empty and nobody
// takes it.
struct Piece {
    int first, last;
};
ATP_PLAN_FN Piece piece_keys(int64_t p0, int64_t p1, int extra, bool ends, int lim, int tile) {
    return Piece{cut_key(p0, extra, lim, tile), ends ? lim : cut_key(p1, extra, lim, tile)};
}

// The share that reads the last keys of a unit whose line is [u0, u1).
ATP_PLAN_FN int64_t last_share(int64_t u0, int64_t u1, int64_t per, int extra, int lim, int tile) {
    int64_t w = (u1 - 1) / per;
    while (w * per > u0 && cut_key(w * per - u0, extra, lim, tile) >= lim) --w;
    return w;
}

}  // namespace plan
}  // namespace atp
