// Every tile of every unit is taken by exactly one CTA, in order, and the parts of a cut unit know how many they are: random batches
// against units counted one by one.  Prints "ok".
#include <cstdio>
#include <cstdlib>
#include <map>
#include <tuple>
#include <vector>

#include "ha_chunk_plan.h"

using namespace ha;

struct Part { int cta, t0, t1, first, n; };

static int fail(const char *what) {
    std::puts(what);
    return 1;
}

int main() {
    srand(1);
    for (int it = 0; it < 4000; ++it) {
        const int B = 1 + rand() % 6, Hkv = 1 + rand() % 4, lg = rand() % 4, most = 1 + rand() % 160;
        const bool causal = rand() % 2;
        std::vector<int32_t> lens(B), off(B + 1, 0);
        for (int b = 0; b < B; ++b) {
            const int mode = rand() % 4, n = mode == 0 ? rand() % 3 : mode == 1 ? rand() % 300 : rand() % 9000;
            const int c = rand() % 3 == 0 ? 1 : rand() % 3 == 0 ? 0 : rand() % 4 == 0 ? n + rand() % 700 : rand() % (n + 1);
            lens[b] = n;
            off[b + 1] = off[b] + c;
        }
        const int rows = off[B] - (rand() % 10 == 0 ? 1 : 0);        // now and then the last sequence does not fit its rows
        long long W = 0;
        std::vector<long long> before(B), cost(B);
        auto seq = [&](int b) { bool bad; return chunk_seq(lens[b], off[b], off[b + 1], rows, lg, bad); };
        for (int b = 0; b < B; ++b) {
            const ChunkSeq s = seq(b);
            long long c = 0;
            for (int u = 0; u < s.units; ++u) {
                if (chunk_cost_full_units(s, u, lg, causal) != c) return fail("closed form of the units in front");
                c += chunk_unit(s, u, lg, causal).total();
            }
            if (c != chunk_cost_head(s, lg, causal)) return fail("closed form of a head");
            before[b] = W;
            cost[b] = c * Hkv;
            W += cost[b];
        }
        if (W == 0) continue;
        const int C = chunk_ctas(W, most);
        std::map<std::tuple<int, int, int>, std::vector<Part>> got;
        for (int c = 0; c < C; ++c) {
            ChunkWalk w;
            w.W = W; w.C = C; w.log2g = lg; w.B = B; w.Hkv = Hkv; w.n_rows = rows; w.causal = causal;
            w.seq_lens = lens.data(); w.offsets = off.data();
            const long long f = chunk_bound(W, C, c);
            int b = 0;
            while (!(before[b] <= f && f < before[b] + cost[b])) ++b;
            w.begin(c, b, f - before[b]);
            for (int k = 0; w.next(); ++k) {
                // where parts of a cut unit are kept: one of a CTA's two places for its last part, one for its first
                if (w.cut && c == w.first_cta && w.t0 != 0) return fail("first part");
                if (w.cut && c != w.first_cta && k != 0) return fail("later part");
                got[{w.b, w.h, w.u}].push_back(Part{c, w.t0, w.t1, w.cut ? w.first_cta : c, w.cut ? w.n_parts : 1});
            }
        }
        for (int b = 0; b < B; ++b)
            for (int h = 0; h < Hkv; ++h)
                for (int u = 0; u < seq(b).units; ++u) {
                    const auto &v = got[{b, h, u}];
                    int t = 0;
                    for (size_t i = 0; i < v.size(); ++i) {
                        if (v[i].t0 != t || v[i].n != (int)v.size() || v[i].first != v[0].cta || v[i].cta != v[0].cta + (int)i) return fail("parts of a unit");
                        t = v[i].t1;
                    }
                    if (t != chunk_unit(seq(b), u, lg, causal).tiles) return fail("tiles of a unit");
                }
    }
    std::puts("ok");
}
