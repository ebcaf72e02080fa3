// Host check of the cached attention's shares (csrc/cache_plan.h): for batches read
// from stdin, walks every share's pieces as the kernel does and the joined units as
// the joining kernel does, and checks that each (head, row block, step of 128 keys)
// that a row needs is taken exactly once and that each cut unit is joined once from
// all of its pieces.
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
    int n_seqs, kv, rows, causal, groups, least;
    long long tokens, cap;
    while (scanf("%d %d %d %d %d %d %lld %lld", &n_seqs, &kv, &rows, &causal, &groups, &least,
                 &tokens, &cap) == 8) {
        std::vector<long long> ctx(n_seqs), cu(n_seqs + 1);
        for (auto& v : ctx) CHECK(scanf("%lld", &v) == 1);
        for (auto& v : cu) CHECK(scanf("%lld", &v) == 1);
        std::vector<Seq> q;
        std::vector<int64_t> start(1, 0);
        for (int s = 0; s < n_seqs; ++s) {
            q.push_back(make_seq(ctx[s], cu[s], cu[s + 1], tokens, cap, rows));
            CHECK(q[s].first >= 0 && q[s].first + q[s].fresh <= tokens && q[s].keys <= cap);
            start.push_back(start[s] + kv * steps_before(q[s], q[s].blocks, rows, causal));
        }
        const int64_t total = start[n_seqs];
        ++cases;
        if (total == 0) continue;
        const int64_t per = share(total, groups, least), used = (total + per - 1) / per;
        CHECK(used <= groups);
        typedef std::tuple<int, int, int> Key;
        std::map<Key, int64_t> done;                       // steps taken, in order
        std::map<Key, std::set<int64_t>> pieces, joined;   // shares of cut units
        for (int64_t w = 0; w < used; ++w) {
            int64_t at = w * per;
            const int64_t end = at + per < total ? at + per : total;
            CHECK(at < end);
            int s = 0;
            while (start[s + 1] <= at) ++s;
            while (at < end) {
                if (q[s].blocks == 0) { ++s; continue; }
                const int64_t head = steps_before(q[s], q[s].blocks, rows, causal);
                const int h = (int)((at - start[s]) / head);
                CHECK(h >= 0 && h < kv);
                const int64_t h0 = start[s] + h * head;
                const int b = block_of(q[s], at - h0, rows, causal);
                const int64_t u0 = h0 + steps_before(q[s], b, rows, causal);
                const int64_t u1 = h0 + steps_before(q[s], b + 1, rows, causal);
                CHECK(b >= 0 && b < q[s].blocks && u0 <= at && at < u1);
                const int64_t t1 = (end < u1 ? end : u1) - u0;
                const Key k(s, h, b);
                CHECK(done[k] == at - u0);                 // exactly the next steps
                done[k] = t1;
                const bool whole = u0 >= w * per && u1 <= end;
                if (!whole) CHECK(pieces[k].insert(w).second);
                if (t1 == u1 - u0)                         // all keys that the block sees
                    CHECK(t1 * kStep >= block_keys(q[s], b, rows, causal));
                at = u0 + t1;
                if (at >= start[s + 1]) ++s;
            }
            // the joining kernel's share w
            if (end < total) {
                int e = 0;
                while (start[e + 1] <= end - 1) ++e;
                const int64_t head = steps_before(q[e], q[e].blocks, rows, causal);
                const int h = (int)((end - 1 - start[e]) / head);
                const int64_t h0 = start[e] + h * head;
                const int b = block_of(q[e], end - 1 - h0, rows, causal);
                const int64_t u0 = h0 + steps_before(q[e], b, rows, causal);
                const int64_t u1 = h0 + steps_before(q[e], b + 1, rows, causal);
                if (u1 > end && u0 >= w * per) {
                    CHECK(joined.find(Key(e, h, b)) == joined.end());
                    for (int64_t j = w; j <= (u1 - 1) / per; ++j) joined[Key(e, h, b)].insert(j);
                }
            }
        }
        for (int s = 0; s < n_seqs; ++s)
            for (int h = 0; h < kv; ++h)
                for (int b = 0; b < q[s].blocks; ++b)
                    CHECK(done[Key(s, h, b)] ==
                          steps_before(q[s], b + 1, rows, causal) - steps_before(q[s], b, rows, causal));
        CHECK(pieces == joined);
    }
    printf("%lld batches\n", cases);
    return 0;
}
