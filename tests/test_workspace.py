"""The operators' growing workspace (csrc/workspace.h), compiled for the host: no block is given back before the release, since a
captured graph may hold its address, and the outgrown ones stay few and small.  No GPU needed."""
from test_pass_rules import run_host

SOURCE = r"""
#include <cstdio>
#include <cstdlib>
#include <map>
#include "workspace.h"
using namespace moshpit;
#define EXPECT(x) do { if (!(x)) { std::printf("line %d: %s\n", __LINE__, #x); ++bad; } } while (0)
int main()
{
    int bad = 0;
    for (int64_t first : {int64_t(1), int64_t(256), int64_t(1) << 30})
        for (double step : {1.0, 1.001, 1.3, 2.0, 17.0}) {
            Workspace w;
            std::map<void *, int64_t> live;
            int64_t most = int64_t(1) << 62;
            uintptr_t next = 4096;
            auto get = [&](int64_t n) -> void * {
                if (n > most) return nullptr;
                void *p = reinterpret_cast<void *>(next += 4096);
                live[p] = n;
                return p;
            };
            EXPECT(w.reserve(0, get) && !w.block() && live.empty());
            double bytes = static_cast<double>(first);
            for (int call = 0; call < 400 && bytes < 1e14; ++call, bytes = bytes * step + 1.0) {
                const std::map<void *, int64_t> before = live;
                void *was = w.block();
                EXPECT(w.reserve(static_cast<int64_t>(bytes), get));
                EXPECT(live.count(w.block()) && live[w.block()] >= static_cast<int64_t>(bytes));
                for (const auto &b : before) EXPECT(live.count(b.first));            // nothing was given back
                EXPECT(w.block() == was || live.size() == before.size() + 1);
                EXPECT(w.reserve(static_cast<int64_t>(bytes), get) && w.reserve(1, get));
            }
            int64_t all = 0;
            for (const auto &b : live) all += b.second;
            EXPECT(all <= 3 * live[w.block()] + 4 * Workspace::kMost);               // (sizes are whole numbers)
            // near the end of the memory: what is asked for, and no more; beyond it an error, and the block stays
            void *was = w.block();
            const int64_t size = live[was];
            most = size + 1;
            EXPECT(w.reserve(size + 1, get) && live[w.block()] == size + 1);
            was = w.block();
            EXPECT(!w.reserve(size + 2, get) && w.block() == was);
            w.release([&](void *p) { EXPECT(live.erase(p) == 1); });
            EXPECT(live.empty() && !w.block());
            EXPECT(w.reserve(5, get) && live.size() == 1);
            w.release([&](void *p) { EXPECT(live.erase(p) == 1); });
        }
    return bad;
}
"""


def test_blocks_stay_until_the_release(tmp_path):
    out = run_host(tmp_path, SOURCE)
    assert out.returncode == 0, out.stdout
