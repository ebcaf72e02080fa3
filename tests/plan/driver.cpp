// Host check of the cached attention's shares (csrc/cache_plan.h): for batches read
// from stdin, walks every share's pieces as the kernel does and the joined units as
// the joining kernel does, and checks that the keys that each (head, row block) sees
// are read exactly once, in whole tiles, and that each cut unit is joined once from all
// of its pieces.
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <set>
#include <tuple>
#include <vector>

#include "../../paper_2301_08658_amd/csrc/cache_plan.h"

using namespace atp::plan;
#define CHECK(c) do { if (!(c)) { printf("line %d: %s\n", __LINE__, #c); exit(1); } } while (0)

int main() {
    long long cases = 0;
    int n_seqs, kv, rows, causal, groups, least, tile, extra;
    long long tokens, cap;
    while (scanf("%d %d %d %d %d %d %d %d %lld %lld", &n_seqs, &kv, &rows, &causal, &groups, &least,
                 &tile, &extra, &tokens, &cap) == 10) {
        std::vector<long long> ctx(n_seqs), cu(n_seqs + 1);
        for (auto& v : ctx) CHECK(scanf("%lld", &v) == 1);
        for (auto& v : cu) CHECK(scanf("%lld", &v) == 1);
        std::vector<Seq> q;
        std::vector<int64_t> start(1, 0);
        for (int s = 0; s < n_seqs; ++s) {
            q.push_back(make_seq(ctx[s], cu[s], cu[s + 1], tokens, cap, rows, extra));
            CHECK(q[s].first >= 0 && q[s].first + q[s].fresh <= tokens && q[s].keys <= cap);
            start.push_back(start[s] + kv * line_of(q[s], q[s].blocks, rows, causal));
        }
        const int64_t total = start[n_seqs];
        ++cases;
        if (total == 0) continue;
        const int64_t per = share(total, groups, least), used = (total + per - 1) / per;
        CHECK(used <= groups);
        // the launch's bound on the shares
        const int64_t units = (n_seqs < tokens ? n_seqs : tokens) + tokens / rows;
        CHECK(used <= units * kv * ((cap + tokens + rows + extra) / least + 2));
        typedef std::tuple<int, int, int> Key;
        std::map<Key, int> read;                           // keys read, in order
        std::map<Key, std::set<int64_t>> pieces, joined;   // shares of cut units
        std::set<int64_t> went_on, left;
        auto unit = [&](int64_t at, int s, int* h, int* b, int64_t* u0, int64_t* u1) {
            const int64_t head = line_of(q[s], q[s].blocks, rows, causal);
            *h = (int)((at - start[s]) / head);
            const int64_t h0 = start[s] + *h * head;
            *b = block_of(q[s], at - h0, rows, causal);
            *u0 = h0 + line_of(q[s], *b, rows, causal);
            *u1 = h0 + line_of(q[s], *b + 1, rows, causal);
            CHECK(*h >= 0 && *h < kv && *b >= 0 && *b < q[s].blocks && *u0 <= at && at < *u1);
        };
        for (int64_t w = 0; w < used; ++w) {
            int64_t at = w * per;
            const int64_t end = at + per < total ? at + per : total;
            CHECK(at < end);
            int s = 0, h, b;
            int64_t u0, u1;
            while (start[s + 1] <= at) ++s;
            while (at < end) {
                if (q[s].blocks == 0) { ++s; continue; }
                unit(at, s, &h, &b, &u0, &u1);
                const int64_t upto = end < u1 ? end : u1;
                const int lim = block_keys(q[s], b, rows, causal);
                CHECK(u1 - u0 >= lim);
                const Piece p = piece_keys(at - u0, upto - u0, extra, upto == u1, lim, tile);
                const Key k(s, h, b);
                CHECK(p.first <= p.last && read[k] == p.first);   // exactly the next keys
                CHECK(p.first % tile == 0 || p.first == lim);
                CHECK(p.last % tile == 0 || p.last == lim);
                read[k] = p.last;
                if (upto == u1) CHECK(read[k] == lim);            // all that the block sees
                if (p.first < p.last) {
                    const bool begins = p.first == 0, whole = begins && p.last == lim;
                    if (!whole) CHECK(pieces[k].insert(w).second);
                    // one unfinished piece of either sort per share
                    if (!begins) CHECK(went_on.insert(w).second);
                    if (begins && !whole) {
                        CHECK(joined.find(k) == joined.end() && left.insert(w).second);
                        for (int64_t j = w; j <= last_share(u0, u1, per, extra, lim, tile); ++j)
                            joined[k].insert(j);
                    }
                }
                at = upto;
                if (at >= start[s + 1]) ++s;
            }
        }
        for (int s = 0; s < n_seqs; ++s)
            for (int h = 0; h < kv; ++h)
                for (int b = 0; b < q[s].blocks; ++b)
                    CHECK(read[Key(s, h, b)] == block_keys(q[s], b, rows, causal));
        CHECK(pieces == joined);
    }
    printf("%lld batches\n", cases);
    return 0;
}
