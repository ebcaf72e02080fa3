// Embedding of tokens on one device's rows of the table, and its gradient.
//
//   out[t] = scale W[id_t - off] (zeros for tokens of other devices: the partial
//   sum of Y = X W with one-hot rows X, W row-first),
//   dW[v] = scale sum over t with id_t = off + v of dy[t], t ascending.
//
// Forward: a copy, bound by memory.  Backward: the tokens are sorted by their row
// (stable, so the tokens of a row stay in order), the sorted tokens are cut into
// chunks of equal length, a workgroup adds up the runs of equal rows of a chunk and
// some columns in registers, and runs that cross a chunk's end are joined in order.  A row
// that occurs thousands of times is so shared by many workgroups, nothing is added by
// atomics, and the result depends on the sizes and tokens alone.  Bound by memory: dy
// is read once, every row of dW written once (zeros where no token is); 8192 rows of
// 4096 values to fp32 40 us, 4.9 TB/s, the gradient of 4096 rows of 20480 values in 6250
// rows 155 us, 4.4 TB/s.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>

#include "train_kernels.h"
#include "wave_ops.h"

namespace atp {
namespace {

using wave::Eight;

// ------------------------------------------------------------------ forward
struct FwdArgs {
    const int32_t* ids;
    int64_t tokens, vocab, off;
    int vecs;                            // vectors of eight values in a row
    const uint16_t* table; int64_t ldt;
    float scale;
    void* out; int64_t ldo;
};

constexpr int kFwdVecs = 4;              // vectors per thread

int64_t fwd_groups(int64_t tokens, int64_t cols) {
    return (tokens * (cols / 8) + 256 * kFwdVecs - 1) / (256 * kFwdVecs);
}

// A workgroup copies a run of kFwdVecs * 256 vectors of the output, rows in order.
template <class T>
__global__ __launch_bounds__(256) void embed_kernel(FwdArgs A) {
    const int64_t first = (int64_t)blockIdx.x * (kFwdVecs * 256);
    const int64_t row0 = first / A.vecs;             // the same for the workgroup
    const uint32_t rem = (uint32_t)(first - row0 * A.vecs);
    Eight<uint16_t> in[kFwdVecs];
    int64_t row[kFwdVecs];
    int col[kFwdVecs];
    int64_t id[kFwdVecs];
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) {
        const uint32_t at = rem + i * 256 + threadIdx.x;
        const uint32_t down = at / (uint32_t)A.vecs;
        row[i] = row0 + down;
        col[i] = (int)(at - down * A.vecs) * 8;
        id[i] = row[i] < A.tokens ? A.ids[row[i]] - A.off : -1;
    }
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) {
        in[i].w = wave::u32x4{0, 0, 0, 0};
        if (id[i] >= 0 && id[i] < A.vocab) in[i].load(A.table + id[i] * A.ldt + col[i]);
    }
#pragma unroll
    for (int i = 0; i < kFwdVecs; ++i) {
        if (row[i] >= A.tokens) continue;
        float v[8];
        in[i].get(v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] *= A.scale;
        // zeros of other devices' tokens stay zeros under any scale
        if (id[i] < 0 || id[i] >= A.vocab) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = 0.f;
        }
        Eight<T> o;
        o.set(v);
        o.store(static_cast<T*>(A.out) + row[i] * A.ldo + col[i]);
    }
}

// ------------------------------------------------------------------ sorting
// A token's row on this device, or `vocab` (sorted last and left out).
__device__ __forceinline__ uint32_t key_of(const int32_t* ids, int64_t t, int64_t off,
                                           int64_t vocab) {
    const int64_t r = (int64_t)ids[t] - off;
    return (uint32_t)(r >= 0 && r < vocab ? r : vocab);
}

constexpr int kSortThreads = 1024;
constexpr int kSortWaves = kSortThreads / 64;
constexpr int kDigits = 256;

// One pass's ranks for the items of a workgroup, wave by wave and round by round:
// an item's place among the items of its digit in its wave (the lanes with the same
// digit come from eight ballots; the wave's counters hold the rounds before).  Then
// count[w][d] becomes the place of wave w's first item of digit d, from base[d] on.
__device__ __forceinline__ uint32_t digit_of(uint32_t item, int at) {
    return (item >> at) & (kDigits - 1);
}
template <int ROUNDS>
__device__ __forceinline__ void ranks(const uint32_t (&item)[ROUNDS], int at,
                                      uint32_t (&rank)[ROUNDS], uint32_t (*count)[kDigits]) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < kSortWaves * kDigits; i += kSortThreads) (&count[0][0])[i] = 0;
    __syncthreads();
    const uint64_t below = (1ull << lane) - 1;
#pragma unroll
    for (int r = 0; r < ROUNDS; ++r) {
        const uint32_t d = digit_of(item[r], at);
        uint64_t same = ~0ull;
#pragma unroll
        for (int b = 0; b < 8; ++b) {
            const bool bit = (d >> b) & 1;
            const uint64_t on = __builtin_amdgcn_ballot_w64(bit);
            same &= bit ? on : ~on;
        }
        volatile uint32_t* c = &count[w][d];
        const uint32_t before = *c;
        rank[r] = before + __popcll(same & below);
        if ((same & below) == 0) *c = before + __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
}

// Exclusive sums over 256 values of LDS, by one wave.
__device__ __forceinline__ void scan256(uint32_t* v) {
    const int lane = threadIdx.x & 63;
    uint32_t a[4], s = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        a[i] = s;
        s += v[4 * lane + i];
    }
    uint32_t incl = s;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t up = __shfl_up(incl, o);
        if (lane >= o) incl += up;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[4 * lane + i] = a[i] + incl - s;
}

// Few tokens: a token's place is the number of tokens before it in the order of
// (row, index), counted.  A workgroup places TOK tokens; its waves divide the others,
// 64 per register, and compare them with one token at a time (one comparison and a
// count of its bits per 64 pairs).
constexpr int kCountMax = 16384;
template <class K, int REGS, int TOK>
__global__ __launch_bounds__(kSortThreads) void sort_few_kernel(const int32_t* ids, int n,
                                                                int64_t off, int64_t vocab,
                                                                int shift, uint32_t* keys,
                                                                uint32_t* order) {
    __shared__ uint32_t place[kSortWaves][TOK];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    auto item = [&](int t) -> K {
        return t < n ? ((K)key_of(ids, t, off, vocab) << shift) | (K)t : ~(K)0;
    };
    const int t = blockIdx.x * TOK + lane;           // the tokens placed here, one per lane
    const K own = item(t);
    K other[REGS];
#pragma unroll
    for (int i = 0; i < REGS; ++i) other[i] = item((w * REGS + i) * 64 + lane);
    uint32_t found = 0;
#pragma unroll 8
    for (int k = 0; k < TOK; ++k) {
        K one;
        if constexpr (sizeof(K) == 8)
            one = (K)(uint32_t)__builtin_amdgcn_readlane((int)own, k) |
                  (K)(uint32_t)__builtin_amdgcn_readlane((int)(own >> 32), k) << 32;
        else
            one = (K)__builtin_amdgcn_readlane((int)own, k);
        uint32_t c = 0;
#pragma unroll
        for (int i = 0; i < REGS; ++i)
            c += __popcll(__builtin_amdgcn_ballot_w64(other[i] < one));
        found = lane == k ? c : found;
    }
    if (lane < TOK) place[w][lane] = found;
    __syncthreads();
    if (w != 0 || lane >= TOK || t >= n) return;
    uint32_t at = 0;
#pragma unroll
    for (int i = 0; i < kSortWaves; ++i) at += place[i][lane];
    keys[at] = (uint32_t)(own >> shift);
    order[at] = (uint32_t)t;
}

// More tokens: tiles of kTile, a pass of eight bits in three launches.
constexpr int kTileRounds = 8;
constexpr int kTile = kTileRounds * kSortThreads;

struct PassArgs {
    const int32_t* ids;                  // the first pass reads the tokens themselves
    int64_t off, vocab;
    const uint32_t *keys, *order;        // the pass before
    uint32_t *keys_out, *order_out;
    uint32_t* hist;                      // [kDigits][tiles]
    int n, tiles, done;                  // bits sorted before this pass
};
__device__ __forceinline__ uint32_t pass_key(const PassArgs& A, int t) {
    return A.keys ? A.keys[t] : key_of(A.ids, t, A.off, A.vocab);
}

__global__ __launch_bounds__(kSortThreads) void sort_count_kernel(PassArgs A) {
    __shared__ uint32_t h[kDigits];
    if (threadIdx.x < kDigits) h[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int64_t t = (int64_t)blockIdx.x * kTile + r * kSortThreads + threadIdx.x;
        if (t < A.n) atomicAdd(&h[digit_of(pass_key(A, (int)t), A.done)], 1u);
    }
    __syncthreads();
    if (threadIdx.x < kDigits) A.hist[(int64_t)threadIdx.x * A.tiles + blockIdx.x] = h[threadIdx.x];
}

// Exclusive sums over kDigits * tiles counts: a wave takes 16 digits, their tiles in
// rounds of 64.
__global__ __launch_bounds__(kSortThreads) void sort_scan_kernel(uint32_t* hist, int tiles) {
    __shared__ uint32_t base[kDigits];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int d = w; d < kDigits; d += kSortWaves) {
        uint32_t run = 0;
        for (int t0 = 0; t0 < tiles; t0 += 64) {
            const int t = t0 + lane;
            const uint32_t v = t < tiles ? hist[(int64_t)d * tiles + t] : 0;
            uint32_t incl = v;
#pragma unroll
            for (int o = 1; o < 64; o <<= 1) {
                const uint32_t up = __shfl_up(incl, o);
                if (lane >= o) incl += up;
            }
            if (t < tiles) hist[(int64_t)d * tiles + t] = run + incl - v;
            run += __shfl(incl, 63);
        }
        if (lane == 0) base[d] = run;
    }
    __syncthreads();
    if (w == 0) scan256(base);
    __syncthreads();
    for (int d = w; d < kDigits; d += kSortWaves)
        for (int t = lane; t < tiles; t += 64) hist[(int64_t)d * tiles + t] += base[d];
}

__global__ __launch_bounds__(kSortThreads) void sort_place_kernel(PassArgs A) {
    __shared__ uint32_t count[kSortWaves][kDigits];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t key[kTileRounds], rank[kTileRounds];
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int64_t t = (int64_t)blockIdx.x * kTile + (w * kTileRounds + r) * 64 + lane;
        key[r] = t < A.n ? pass_key(A, (int)t) : 0xffffffffu;    // behind all of its digit
    }
    ranks<kTileRounds>(key, A.done, rank, count);
    if (threadIdx.x < kDigits) {
        uint32_t s = A.hist[(int64_t)threadIdx.x * A.tiles + blockIdx.x];
#pragma unroll
        for (int k = 0; k < kSortWaves; ++k) {
            const uint32_t c = count[k][threadIdx.x];
            count[k][threadIdx.x] = s;
            s += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < kTileRounds; ++r) {
        const int64_t t = (int64_t)blockIdx.x * kTile + (w * kTileRounds + r) * 64 + lane;
        if (t >= A.n) continue;
        const uint32_t at = count[w][digit_of(key[r], A.done)] + rank[r];
        A.keys_out[at] = key[r];
        A.order_out[at] = A.order ? A.order[t] : (uint32_t)t;
    }
}

// ------------------------------------------------------------------ sums
struct SumArgs {
    const uint32_t *keys, *order;
    int n, chunk, chunks, col_blocks;
    int lanes;                           // of a workgroup's 256 that take one chunk
    int64_t vocab;
    int cols;
    const uint16_t* dy; int64_t lddy;
    float scale;
    float* dtable; int64_t ldt;
    float* part;                         // [chunks][2][cols]: a run from the chunk before, one
                                         // that goes on in the next
    int accumulate;
    int fill_rows;                       // rows of a wave that writes zeros
};

__device__ __forceinline__ void add_row(float (&s)[8], const float* v) {
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += v[e];
}
__device__ __forceinline__ void put_row(const SumArgs& A, uint32_t key, int c, float (&s)[8]) {
    float* to = A.dtable + (int64_t)key * A.ldt + c;
    Eight<float> o;
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] *= A.scale;
    if (A.accumulate) {
        float old[8];
        o.load(to);
        o.get(old);
        add_row(s, old);
    }
    o.set(s);
    o.store(to);
}

// Zeros for the rows that no token names: a wave looks its rows up one by one, 64
// probes at a time.
__device__ __forceinline__ void fill(const SumArgs& A, int64_t r0) {
    const int lane = threadIdx.x & 63;
    const wave::f32x4 z = {0.f, 0.f, 0.f, 0.f};
    for (int64_t r = r0; r < r0 + A.fill_rows && r < A.vocab; ++r) {
        int lo = 0, len = A.n;           // the first key >= r is in [lo, lo + len]
        while (len > 0) {
            const int step = (len + 63) >> 6;
            const int i = lane * step;
            const bool less = i < len && A.keys[lo + i] < (uint32_t)r;
            const int c = __popcll(__builtin_amdgcn_ballot_w64(less));
            if (c == 0) break;
            const int skip = (c - 1) * step + 1;
            lo += skip;
            len = min(step - 1, len - skip);
        }
        if (lo < A.n && A.keys[lo] == (uint32_t)r) continue;
        float* to = A.dtable + r * A.ldt;
#pragma unroll 4
        for (int c = lane * 4; c < A.cols; c += 256) *reinterpret_cast<wave::f32x4*>(to + c) = z;
    }
}

__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs A, int64_t work) {
    if (blockIdx.x >= work) {
        fill(A, (((int64_t)blockIdx.x - work) * 4 + threadIdx.x / 64) * A.fill_rows);
        return;
    }
    const int ch = __builtin_amdgcn_readfirstlane(
        (int)(blockIdx.x / A.col_blocks) * (256 / A.lanes) + (int)threadIdx.x / A.lanes);
    if (ch >= A.chunks) return;
    const int c =
        ((int)(blockIdx.x % A.col_blocks) * A.lanes + (int)threadIdx.x % A.lanes) * 8;
    if (c >= A.cols) return;
    const int p0 = ch * A.chunk, p1 = min(p0 + A.chunk, A.n);
    const uint32_t none = (uint32_t)A.vocab;
    uint32_t cur = A.keys[p0];
    if (cur == none) return;
    const bool from_before = p0 > 0 && A.keys[p0 - 1] == cur;
    const bool goes_on = p1 < A.n && A.keys[p1] == A.keys[p1 - 1];
    bool head = from_before;             // the run at hand came from the chunk before
    float s[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] = 0.f;
    constexpr int U = 8;                 // rows under way
    for (int p = p0; p < p1; p += U) {
        Eight<uint16_t> in[U];
        uint32_t key[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int q = min(p + u, p1 - 1);
            key[u] = p + u < p1 ? A.keys[q] : none;
            in[u].load(A.dy + (int64_t)A.order[q] * A.lddy + c);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (key[u] != cur && cur != none) {      // a run ends inside the chunk
                if (p + u < p1) {
                    if (head) {
                        Eight<float> o;
                        o.set(s);
                        o.store(A.part + (int64_t)ch * 2 * A.cols + c);
                    } else {
                        put_row(A, cur, c, s);
                    }
                    head = false;
                    cur = key[u];
#pragma unroll
                    for (int e = 0; e < 8; ++e) s[e] = 0.f;
                }
            }
            if (p + u < p1 && cur != none) {
                float v[8];
                in[u].get(v);
                add_row(s, v);
            }
        }
    }
    if (cur == none) return;
    if (head || goes_on) {
        Eight<float> o;
        o.set(s);
        o.store(A.part + ((int64_t)ch * 2 + (head ? 0 : 1)) * A.cols + c);
    } else {
        put_row(A, cur, c, s);
    }
}

// Runs that cross chunks, by the chunk that they begin in.
__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs A) {
    const int ch = __builtin_amdgcn_readfirstlane(
        (int)(blockIdx.x / A.col_blocks) * (256 / A.lanes) + (int)threadIdx.x / A.lanes);
    const int c =
        ((int)(blockIdx.x % A.col_blocks) * A.lanes + (int)threadIdx.x % A.lanes) * 8;
    const int p0 = ch * A.chunk, p1 = p0 + A.chunk;
    if (p1 >= A.n) return;
    const uint32_t k = A.keys[p1 - 1];
    if (k == (uint32_t)A.vocab || A.keys[p1] != k) return;
    if (p0 > 0 && A.keys[p0 - 1] == k) return;       // began earlier (then it fills the chunk)
    if (c >= A.cols) return;
    // the last chunk whose first token is of the run
    int lo = ch + 1, hi = A.chunks - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (A.keys[(int64_t)mid * A.chunk] == k) lo = mid;
        else hi = mid - 1;
    }
    float s[8];
    Eight<float> t;
    t.load(A.part + ((int64_t)ch * 2 + 1) * A.cols + c);
    t.get(s);
#pragma unroll 4
    for (int j = ch + 1; j <= lo; ++j) {
        float v[8];
        Eight<float> u;
        u.load(A.part + (int64_t)j * 2 * A.cols + c);
        u.get(v);
        add_row(s, v);
    }
    put_row(A, k, c, s);
}

// ------------------------------------------------------------------ plan
struct Plan {
    int key_bits;
    bool few;                            // places are counted
    int tiles, chunk, chunks;
    int64_t keys, order, keys2, order2, hist, part, bytes;
};
int bit_length(uint64_t v) { return v ? 64 - __builtin_clzll(v) : 0; }

// Tokens of a chunk.  Short chunks fill the chip, long ones leave fewer runs that cross an
// end.  Gradients with chunks of 8, 16, 32 and 64 tokens, us: 1024 x 2048 values 20, 24, 32,
// 50; 4096 x 4096 33, 32, 37, 54; 4096 x 20480 172, 174, 164, 185; 65536 x 2048 242, 184, 183,
// 168.  No more than kMostChunks, which one run may cross.
constexpr int kMostChunks = 2048;
struct ChunkRule {
    int64_t values;                      // of gradients of fewer values than this
    int chunk;
};
constexpr ChunkRule kChunks[] = {{1 << 22, 8}, {1 << 25, 16}, {1 << 27, 32}, {INT64_MAX, 64}};
int64_t chunk_of(int64_t values) {
    for (const ChunkRule& r : kChunks)
        if (values < r.values) return r.chunk;
    return 0;
}
// Rows of partial sums that any gradient of up to n tokens leaves: longer chunks leave fewer,
// so each rule counts with its most tokens.
int64_t most_chunks(int64_t n, int64_t cols) {
    int64_t most = 0;
    for (const ChunkRule& r : kChunks) {
        const int64_t k = std::min(n, (r.values - 1) / cols);
        most = std::max(most, std::min<int64_t>(kMostChunks, (k + r.chunk - 1) / r.chunk));
    }
    return most;
}

Plan plan_of(int64_t n, int64_t vocab, int64_t cols) {
    Plan p = {};
    p.key_bits = bit_length((uint64_t)vocab);
    p.few = n <= kCountMax;
    p.tiles = (int)((n + kTile - 1) / kTile);
    p.chunk = (int)std::max(chunk_of(n * cols), ((n + kMostChunks - 1) / kMostChunks + 7) / 8 * 8);
    p.chunks = (int)((n + p.chunk - 1) / p.chunk);
    int64_t at = 0;
    auto take = [&](int64_t bytes) {
        const int64_t was = at;
        at += (bytes + 255) / 256 * 256;
        return was;
    };
    p.keys = take(4 * n);
    p.order = take(4 * n);
    if (!p.few) {
        p.keys2 = take(4 * n);
        p.order2 = take(4 * n);
        p.hist = take(4 * (int64_t)kDigits * p.tiles);
    }
    p.part = take(most_chunks(n, cols) * 2 * cols * 4);
    p.bytes = at;
    return p;
}

// Tokens of a workgroup: 16, so that 4096 tokens take every CU (their places 5.2 us; the
// whole gradient of 4096 tokens of 20480 values by counted places 164 us, by the passes
// over digits 212, of 16384 of 4096 73 and 112).
template <class K, int REGS, int TOK>
void few(const EmbeddingBwdProblem& p, int shift, uint32_t* keys, uint32_t* order, hipStream_t s) {
    sort_few_kernel<K, REGS, TOK>
        <<<dim3((unsigned)((p.tokens + TOK - 1) / TOK)), kSortThreads, 0, s>>>(
            p.ids, (int)p.tokens, p.off, p.vocab, shift, keys, order);
}
template <class K>
void few_of(const EmbeddingBwdProblem& p, int shift, uint32_t* keys, uint32_t* order,
            hipStream_t s) {
    if (p.tokens <= 1024) few<K, 1, 16>(p, shift, keys, order, s);
    else if (p.tokens <= 4096) few<K, 4, 16>(p, shift, keys, order, s);
    else if (p.tokens <= 8192) few<K, 8, 32>(p, shift, keys, order, s);
    else few<K, 16, 64>(p, shift, keys, order, s);
}

}  // namespace

int64_t embedding_ws_bytes(int64_t tokens, int64_t vocab, int64_t cols) {
    return plan_of(tokens, vocab, cols).bytes;
}

bool embedding_fits(int64_t tokens, int64_t cols) {
    return fits_launch(fwd_groups(tokens, cols), 256);
}

hipError_t launch_embedding(const EmbeddingProblem& p, hipStream_t s) {
    if (p.tokens == 0) return hipSuccess;
    FwdArgs a;
    a.ids = p.ids;
    a.tokens = p.tokens;
    a.vocab = p.vocab;
    a.off = p.off;
    a.vecs = (int)(p.cols / 8);
    a.table = p.table; a.ldt = p.ldt;
    a.scale = p.scale;
    a.out = p.out; a.ldo = p.ldo;
    const int64_t grid = fwd_groups(p.tokens, p.cols);
    if (p.out_f32) embed_kernel<float><<<dim3((unsigned)grid), 256, 0, s>>>(a);
    else embed_kernel<uint16_t><<<dim3((unsigned)grid), 256, 0, s>>>(a);
    return hipGetLastError();
}

hipError_t launch_embedding_bwd(const EmbeddingBwdProblem& p, hipStream_t s) {
    const Plan f = plan_of(p.tokens, p.vocab, p.cols);
    char* ws = static_cast<char*>(p.ws);
    auto u32 = [&](int64_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
    uint32_t *keys = u32(f.keys), *order = u32(f.order);
    hipError_t e = hipSuccess;
    if (p.tokens > 0 && f.few) {
        const int idx = bit_length((uint64_t)p.tokens);      // one more than the last index
        if (idx + f.key_bits <= 32) few_of<uint32_t>(p, idx, keys, order, s);
        else few_of<uint64_t>(p, idx, keys, order, s);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    } else if (p.tokens > 0) {
        PassArgs a = {};
        a.ids = p.ids;
        a.off = p.off;
        a.vocab = p.vocab;
        a.hist = u32(f.hist);
        a.n = (int)p.tokens;
        a.tiles = f.tiles;
        uint32_t *kout = u32(f.keys2), *oout = u32(f.order2);
        for (a.done = 0; a.done < f.key_bits; a.done += 8) {
            // the two pairs of lists in turn
            a.keys_out = kout;
            a.order_out = oout;
            sort_count_kernel<<<f.tiles, kSortThreads, 0, s>>>(a);
            sort_scan_kernel<<<1, kSortThreads, 0, s>>>(a.hist, a.tiles);
            sort_place_kernel<<<f.tiles, kSortThreads, 0, s>>>(a);
            e = hipGetLastError();
            if (e != hipSuccess) return e;
            a.keys = kout;
            a.order = oout;
            std::swap(keys, kout);
            std::swap(order, oout);
        }
    }
    SumArgs a = {};
    a.keys = keys;
    a.order = order;
    a.n = (int)p.tokens;
    a.chunk = f.chunk;
    a.chunks = f.chunks;
    a.vocab = p.vocab;
    a.cols = (int)p.cols;
    a.dy = p.dy; a.lddy = p.lddy;
    a.scale = p.scale;
    a.dtable = p.dtable; a.ldt = p.ldt;
    a.part = reinterpret_cast<float*>(ws + f.part);
    a.accumulate = p.accumulate;
    const int vecs = a.cols / 8;
    a.lanes = vecs <= 64 ? 64 : vecs <= 128 ? 128 : 256;
    a.col_blocks = (vecs + a.lanes - 1) / a.lanes;
    // rows of zeros for 16 waves per CU, more than one each where there are more rows
    a.fill_rows = (int)std::min<int64_t>(16, (p.vocab + 4095) / 4096);
    const int per = 256 / a.lanes;
    const int64_t work = (int64_t)(f.chunks + per - 1) / per * a.col_blocks;
    const int64_t fills =
        p.accumulate ? 0 : (p.vocab + 4 * a.fill_rows - 1) / (4 * a.fill_rows);
    if (work + fills == 0) return hipSuccess;
    embed_sum_kernel<<<dim3((unsigned)(work + fills)), 256, 0, s>>>(a, work);
    e = hipGetLastError();
    if (e != hipSuccess || f.chunks < 2) return e;
    embed_join_kernel<<<dim3((unsigned)work), 256, 0, s>>>(a);
    return hipGetLastError();
}

}  // namespace atp
