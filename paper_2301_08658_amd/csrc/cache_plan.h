// How the attention over the cache is cut into equal shares: integer arithmetic
// that the kernels run and the host can run too (no HIP types).
//
// A unit is one row block (up to `rows` tokens' query heads of one key/value
// head) of one sequence; its keys are walked in steps of 128.  All units of a
// batch are laid end to end, sequence by sequence, head by head, block by
// block, and workgroup w of the plan takes steps [w * per, (w + 1) * per) of that
// line: no workgroup waits for a long sequence, whatever the lengths are.
#pragma once
#include <stdint.h>

#if defined(__HIPCC__)
#define ATP_PLAN_FN __host__ __device__ __forceinline__
#else
#define ATP_PLAN_FN inline
#endif

namespace atp {
namespace plan {

constexpr int kStep = 128;     // keys per step: 32 for each of four waves

struct Seq {
    int first, fresh;          // its rows of the step's buffers
    int ctx, keys;             // cached before the step; with the new ones
    int blocks;                // row blocks of a head
};

// ctx, c0, c1: the sequence's ctx, cu_new[s], cu_new[s + 1] as they stand in device
// memory; tokens and cap (max_pages * page_size, <= 2^30) bound what they may name.
ATP_PLAN_FN Seq make_seq(int64_t ctx, int64_t c0, int64_t c1, int64_t tokens, int64_t cap,
                         int rows) {
    Seq q;
    c0 = c0 < 0 ? 0 : (c0 > tokens ? tokens : c0);
    c1 = c1 < c0 ? c0 : (c1 > tokens ? tokens : c1);
    ctx = ctx < 0 ? 0 : (ctx > cap ? cap : ctx);
    q.first = (int)c0;
    q.fresh = (int)(c1 - c0);
    q.ctx = (int)ctx;
    q.keys = (int)(ctx + q.fresh > cap ? cap : ctx + q.fresh);
    q.blocks = (q.fresh + rows - 1) / rows;
    return q;
}

// Keys that row block i of a causal sequence can see (all of them otherwise).
ATP_PLAN_FN int block_keys(const Seq& q, int i, int rows, bool causal) {
    if (!causal) return q.keys;
    const int64_t last = (int64_t)q.ctx + (int64_t)(i + 1) * rows;
    return last < q.keys ? (int)last : q.keys;
}

// sum_{j = 1 .. m} ceil(j / q)
ATP_PLAN_FN int64_t ceil_sum(int64_t m, int64_t q) {
    const int64_t k = m / q, r = m - k * q;
    return q * (k * (k + 1) / 2) + r * (k + 1);
}

// Steps of the first n row blocks of a head.  A causal sequence of several blocks
// counts A + ceil((a + j) / q) for block j = 1, 2, .. with ctx = 128 A + a', a =
// ceil(a' / rows) and q = floor(128 / rows): never less than the block's keys
// need, and its sum has a closed form.  The new tokens count up to 128 / 120 of
// what they need (rows = 12), the cached ones exactly.
ATP_PLAN_FN int64_t steps_before(const Seq& q, int64_t n, int rows, bool causal) {
    if (!causal || q.blocks <= 1) {
        const int64_t one = (q.keys + kStep - 1) / kStep;
        return n * (one > 0 ? one : 1);
    }
    const int64_t A = q.ctx / kStep, a = (q.ctx % kStep + rows - 1) / rows, w = kStep / rows;
    return n * A + ceil_sum(a + n, w) - ceil_sum(a, w);
}

// The row block of step `at` of a head (0 <= at < steps_before(blocks)).
ATP_PLAN_FN int block_of(const Seq& q, int64_t at, int rows, bool causal) {
    int lo = 0, hi = q.blocks - 1;      // last block whose start is <= at
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (steps_before(q, mid, rows, causal) <= at) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// Steps of a workgroup.
ATP_PLAN_FN int64_t share(int64_t total, int groups, int least) {
    const int64_t per = (total + groups - 1) / groups;
    return per > least ? per : least;
}

}  // namespace plan
}  // namespace atp
