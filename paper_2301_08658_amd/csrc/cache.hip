// Pages of a key/value cache: reserving (with copies of shared pages), forking,
// releasing, copying and compacting.  The bookkeeping is integer work on
// tables and reference counts whose results do not depend on the order in which
// threads run: pages are handed out by rank (free pages in ascending order
// to the wanted places in ascending order), counts change by additions.  It is
// bound by dependent trips to memory, not by bandwidth: a few of them, and in
// reserving one more, with two barriers, per 4096 pages in front of the last free
// one that it gives (n_pages / 4096 of them in a pool that is nearly full).
// Copying and compacting move 16 bytes per lane and are bound by the rows in flight.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "cache_kernels.h"

namespace atp {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256;
constexpr int kPlan = 1024;          // threads of the reserving workgroup
constexpr int kPlanWaves = kPlan / 64;
// entries of a sequence that one lane looks at by itself (a decode step writes to
// one or two); longer runs (a prompt) are looked at by its wave
constexpr int kShort = 4;
constexpr int64_t kFar = 1 << 30;    // a rank that no pool holds (at most 2^28 pages)

__device__ __forceinline__ bool names_page(int32_t e, int n_pages) { return e >= 0 && e < n_pages; }

// Exclusive prefix of v over the workgroup's threads, and the total.  A wave's sum is below
// 2^32 whatever the lists hold: a sequence wants at most 2^26 pages, and 32-bit lists cannot
// give five neighbours the 2^30 new tokens each that it takes.
__device__ __forceinline__ int64_t block_prefix(uint32_t v, uint32_t* waves, int64_t* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t inc = v;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const uint32_t up = __shfl_up(inc, d);
        if (lane >= d) inc += up;
    }
    if (lane == 63) waves[wave] = inc;
    __syncthreads();
    int64_t before = 0, all = 0;
#pragma unroll
    for (int i = 0; i < kPlanWaves; ++i) {
        if (i < wave) before += waves[i];
        all += waves[i];
    }
    __syncthreads();
    *total = all;
    return before + (inc - v);
}

struct Span {      // table columns [lo, hi) that a sequence's new tokens go to
    int lo, hi, over, ctx;
};
__device__ __forceinline__ Span span_of(const BatchView& b, int shift, int s) {
    Span r = {0, 0, 0, 0};
    const int64_t fresh = (int64_t)b.cu[s + 1] - b.cu[s];
    if (fresh <= 0) return r;
    r.ctx = max(b.ctx[s], 0);
    const int64_t lo = r.ctx >> shift;
    const int64_t hi = (r.ctx + fresh + ((int64_t)1 << shift) - 1) >> shift;
    const int64_t fit = hi < b.max_pages ? hi : b.max_pages;
    r.over = (int)(hi - fit);
    r.hi = (int)fit;
    r.lo = (int)(lo < fit ? lo : fit);
    return r;
}

// One workgroup.  A: what every sequence wants; B: its rank among the wanted
// pages; C: the first free pages; D: they are handed out.
__global__ __launch_bounds__(kPlan) void reserve_kernel(int n_pages, int shift, int32_t* refs,
                                                        BatchView b, int32_t* missing, int32_t* src,
                                                        int32_t* dst, int32_t* rows, int32_t* want,
                                                        int32_t* free_list) {
    __shared__ uint32_t waves[kPlanWaves];
    __shared__ int given;
    const int tid = threadIdx.x, lane = tid & 63;
    auto wanted = [&](int32_t e) { return !names_page(e, n_pages) || refs[e] > 1; };

    // A and B; rounds of 1024 sequences.  want[s]: pages wanted before s; a sequence
    // that its table cannot hold wants none.
    int64_t carry = 0;
    for (int s0 = 0; s0 < b.n_seqs; s0 += kPlan) {
        const int s = s0 + tid;
        Span sp = {0, 0, 0, 0};
        if (s < b.n_seqs) sp = span_of(b, shift, s);
        int n = 0;
        const bool is_long = sp.hi - sp.lo > kShort;
        if (!is_long)
            for (int i = sp.lo; i < sp.hi; ++i) n += wanted(b.table[s * b.ld_table + i]);
        for (uint64_t todo = __builtin_amdgcn_ballot_w64(is_long); todo; todo &= todo - 1) {
            const int who = __ffsll((unsigned long long)todo) - 1;
            const int lo = __shfl(sp.lo, who), hi = __shfl(sp.hi, who);
            const int32_t* row = b.table + (int64_t)(s0 + (tid - lane) + who) * b.ld_table;
            int m = 0;
            for (int i = lo + lane; i < hi; i += 64) m += wanted(row[i]);
#pragma unroll
            for (int d = 32; d > 0; d >>= 1) m += __shfl_xor(m, d);
            if (lane == who) n = m;
        }
        int64_t total;
        const int64_t pre = block_prefix(sp.over ? 0 : n, waves, &total);
        if (s < b.n_seqs) {
            want[s] = (int32_t)min(carry + pre, kFar);
            missing[s] = n + sp.over;
        }
        carry += total;
    }

    // C: free pages in ascending order until there are enough
    int64_t found = 0;
    for (int64_t p0 = 0; p0 < n_pages && found < carry; p0 += 4 * kPlan) {
        const int64_t p = p0 + 4 * tid;
        i32x4 r = {1, 1, 1, 1};
        if (p + 4 <= n_pages) {
            r = *reinterpret_cast<const i32x4*>(refs + p);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (p + e < n_pages) r[e] = refs[p + e];
        }
        int n = 0;
        int64_t total;
#pragma unroll
        for (int e = 0; e < 4; ++e) n += r[e] == 0;
        int64_t at = found + block_prefix(n, waves, &total);
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (r[e] == 0) {
                if (at < carry) free_list[at] = (int32_t)(p + e);
                ++at;
            }
        found += total;
    }
    __syncthreads();      // want and free_list were written by this workgroup

    // D.  What is wanted is decided by the counts of the call's start: a replaced
    // page's number takes the place of its successor in free_list, and its
    // count falls in E.  (The counts of the pages given here were 0, so no entry
    // is wanted or not because of them.)
    if (tid == 0) given = 0;
    __syncthreads();
    for (int s0 = 0; s0 < b.n_seqs; s0 += kPlan) {
        const int s = s0 + tid;
        Span sp = {0, 0, 0, 0};
        int base = 0;
        bool give = false;
        if (s < b.n_seqs) {
            sp = span_of(b, shift, s);
            const int n = missing[s];
            base = want[s];
            give = n > 0 && !sp.over && base + n <= found;
            if (give) {
                missing[s] = 0;
                atomicMax(&given, base + n);
            }
            src[s] = dst[s] = -1;
            rows[s] = 0;
        }
        auto hand_out = [&](int seq, int lo, int ctx, int i, int rank) {
            int32_t* entry = b.table + seq * b.ld_table + i;
            const int32_t page = free_list[rank], old = *entry;
            *entry = page;
            refs[page] = 1;
            free_list[rank] = old;
            const int tail = ctx & ((1 << shift) - 1);
            if (i == lo && tail && names_page(old, n_pages)) {
                src[seq] = old;
                dst[seq] = page;
                rows[seq] = tail;
            }
        };
        const bool is_long = give && sp.hi - sp.lo > kShort;
        if (give && !is_long)
            for (int i = sp.lo, rank = base; i < sp.hi; ++i)
                if (wanted(b.table[s * b.ld_table + i])) hand_out(s, sp.lo, sp.ctx, i, rank++);
        for (uint64_t todo = __builtin_amdgcn_ballot_w64(is_long); todo; todo &= todo - 1) {
            const int who = __ffsll((unsigned long long)todo) - 1;
            const int lo = __shfl(sp.lo, who), hi = __shfl(sp.hi, who);
            const int ctx = __shfl(sp.ctx, who), seq = s0 + (tid - lane) + who;
            int rank = __shfl(base, who);
            for (int i0 = lo; i0 < hi; i0 += 64) {
                const int i = i0 + lane;
                const bool w = i < hi && wanted(b.table[seq * b.ld_table + i]);
                const uint64_t all = __builtin_amdgcn_ballot_w64(w);
                if (w) hand_out(seq, lo, ctx, i, rank + __popcll(all & ((1ull << lane) - 1)));
                rank += __popcll(all);
            }
        }
    }
    __syncthreads();
    // E
    for (int i = tid; i < given; i += kPlan) {
        const int32_t old = free_list[i];
        if (names_page(old, n_pages)) atomicSub(&refs[old], 1);
    }
}

// One workgroup per fork.
__global__ __launch_bounds__(kThreads) void fork_kernel(int n_pages, int shift, int32_t* refs,
                                                        BatchView b, int n, const int32_t* parents,
                                                        const int32_t* children, int32_t* done) {
    const int f = blockIdx.x, tid = threadIdx.x;
    const int32_t from = parents[f], to = children[f];
    bool bad = from < 0 || from >= b.n_seqs || to < 0 || to >= b.n_seqs;
    // the child is no parent and no earlier child of the call, and holds nothing
    for (int i = tid; i < n; i += kThreads)
        bad |= parents[i] == to || (i < f && children[i] == to);
    // rows of other forks' children are not looked at: those are refused above
    if (!bad)
        for (int i = tid; i < b.max_pages; i += kThreads)
            bad |= names_page(b.table[to * b.ld_table + i], n_pages);
    const bool refused = __syncthreads_or(bad);
    if (tid == 0) done[f] = refused;
    if (refused) return;
    const int64_t held = ((int64_t)max(b.ctx[from], 0) + ((int64_t)1 << shift) - 1) >> shift;
    for (int i = tid; i < b.max_pages; i += kThreads) {
        int32_t e = i < held ? b.table[from * b.ld_table + i] : -1;
        if (names_page(e, n_pages)) atomicAdd(&refs[e], 1);
        else e = -1;
        b.table[to * b.ld_table + i] = e;
    }
}

// One workgroup per sequence.
__global__ __launch_bounds__(kThreads) void release_kernel(int n_pages, int shift, int32_t* refs,
                                                           BatchView b, const int32_t* keep) {
    const int s = blockIdx.x;
    const int64_t kept = keep[s];
    if (kept < 0) return;
    int32_t* row = b.table + s * b.ld_table;
    for (int64_t i = ((kept + ((int64_t)1 << shift) - 1) >> shift) + threadIdx.x; i < b.max_pages;
         i += kThreads) {
        const int32_t e = row[i];
        if (names_page(e, n_pages)) atomicSub(&refs[e], 1);
        row[i] = -1;
    }
}

// One workgroup per copied page and half head (keys or values of one head): the
// copied tokens are one run of 256-byte rows.
__global__ __launch_bounds__(kThreads) void copy_kernel(CacheView c, const int32_t* src,
                                                        const int32_t* dst, const int32_t* rows) {
    const int i = blockIdx.x;
    const int32_t a = src[i], z = dst[i];
    const int page = 1 << c.page_shift;
    const int n = rows ? min(rows[i], page) : page;
    if (n <= 0 || a == z || !names_page(a, c.n_pages) || !names_page(z, c.n_pages)) return;
    const int64_t run = (int64_t)page * kHead, halves = 2 * c.kv_heads;
    const u32x4* from = reinterpret_cast<const u32x4*>(c.pages + (a * halves + blockIdx.y) * run);
    u32x4* to = reinterpret_cast<u32x4*>(c.pages + (z * halves + blockIdx.y) * run);
    const int words = n * (kHead / 8);
    constexpr int U = 4;
    for (int w0 = threadIdx.x; w0 < words; w0 += U * kThreads) {
        u32x4 v[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (w0 + u * kThreads < words) v[u] = from[w0 + u * kThreads];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (w0 + u * kThreads < words) to[w0 + u * kThreads] = v[u];
    }
}

// One workgroup per sequence and half head.  Row i comes from keep[i] >= i (the
// indices ascend), so a round's stores touch no row that a later round reads, and
// within a round all rows are read before the first is written.  16 lanes move
// a row, kRows rows per lane in flight.
constexpr int kRows = 8;
__global__ __launch_bounds__(kThreads) void compact_kernel(CacheView c, BatchView b,
                                                           const int32_t* cu_keep,
                                                           const int32_t* keep, int n_keep,
                                                           int32_t* moved) {
    const int s = blockIdx.x, tid = threadIdx.x;
    const int k0 = min(max(cu_keep[s], 0), n_keep), k1 = min(max(cu_keep[s + 1], 0), n_keep);
    const int n = max(k1 - k0, 0);
    keep += k0;
    const int64_t ctx = max(b.ctx[s], 0);
    const int shift = c.page_shift;
    const int32_t* table = b.table + s * b.ld_table;
    auto page_of = [&](int64_t at) {
        const int64_t col = at >> shift;
        const int32_t e = col < b.max_pages ? table[col] : -1;
        return names_page(e, c.n_pages) ? e : -1;
    };
    bool bad = false;
    for (int i = tid; i < n; i += kThreads) {
        const int32_t k = keep[i];
        bad |= k < 0 || (i > 0 && keep[i - 1] >= k) || page_of(ctx + i) < 0 ||
               page_of(ctx + k) < 0;
    }
    bad = __syncthreads_or(bad);
    if (moved && tid == 0 && blockIdx.y == 0) moved[s] = bad ? -1 : n;
    if (bad) return;
    const int64_t halves = 2 * c.kv_heads, page = (int64_t)1 << shift;
    auto row_of = [&](int64_t at) {
        return reinterpret_cast<u32x4*>(
                   c.pages + ((page_of(at) * halves + blockIdx.y) * page + (at & (page - 1))) *
                                 kHead) + (tid & 15);
    };
    for (int i0 = 0; i0 < n; i0 += kRows * (kThreads / 16)) {
        u32x4 v[kRows];
        bool go[kRows];
#pragma unroll
        for (int u = 0; u < kRows; ++u) {
            const int i = i0 + u * (kThreads / 16) + tid / 16;
            go[u] = i < n && keep[i] != i;
            if (go[u]) v[u] = *row_of(ctx + keep[i]);
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // this round's rows have been read
        __syncthreads();
#pragma unroll
        for (int u = 0; u < kRows; ++u)
            if (go[u]) *row_of(ctx + i0 + u * (kThreads / 16) + tid / 16) = v[u];
    }
}

}  // namespace

hipError_t launch_cache_reserve(int n_pages, int page_shift, int32_t* refs, const BatchView& b,
                                int32_t* missing, int32_t* src, int32_t* dst, int32_t* rows,
                                int32_t* ws, hipStream_t s) {
    reserve_kernel<<<1, kPlan, 0, s>>>(n_pages, page_shift, refs, b, missing, src, dst, rows,
                                       ws + n_pages, ws);
    return hipGetLastError();
}

hipError_t launch_cache_fork(int n_pages, int page_shift, int32_t* refs, const BatchView& b, int n,
                             const int32_t* parents, const int32_t* children, int32_t* done,
                             hipStream_t s) {
    fork_kernel<<<n, kThreads, 0, s>>>(n_pages, page_shift, refs, b, n, parents, children, done);
    return hipGetLastError();
}

hipError_t launch_cache_release(int n_pages, int page_shift, int32_t* refs, const BatchView& b,
                                const int32_t* keep, hipStream_t s) {
    release_kernel<<<b.n_seqs, kThreads, 0, s>>>(n_pages, page_shift, refs, b, keep);
    return hipGetLastError();
}

hipError_t launch_cache_copy(const CacheView& c, int n, const int32_t* src, const int32_t* dst,
                             const int32_t* rows, hipStream_t s) {
    copy_kernel<<<dim3(n, 2 * c.kv_heads), kThreads, 0, s>>>(c, src, dst, rows);
    return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheView& c, const BatchView& b, const int32_t* cu_keep,
                                const int32_t* keep, int n_keep, int32_t* moved, hipStream_t s) {
    compact_kernel<<<dim3(b.n_seqs, 2 * c.kv_heads), kThreads, 0, s>>>(c, b, cu_keep, keep, n_keep,
                                                                       moved);
    return hipGetLastError();
}

}  // namespace atp
