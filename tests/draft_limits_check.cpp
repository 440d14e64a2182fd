// Walks on the CPU what mom_draft.h says at the largest extents that the calls take: shares of sequences of up to 2^29 tokens, and the workspace of all calls that are no larger than one.
#include "mom_draft.h"

#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>
#include <vector>

using namespace momk;

#define CHECK(x, ...)                             \
    do {                                          \
        if (!(x)) {                               \
            printf("%s: ", #x);                   \
            printf(__VA_ARGS__);                  \
            printf("\n");                         \
            exit(1);                              \
        }                                         \
    } while (0)

static std::mt19937 rng(1);
static int64_t upto(int64_t n) { return (int64_t)(((uint64_t)rng() << 32 | rng()) % (uint64_t)(n + 1)); }

static void check_shares() {
    const uint32_t most = 1u << 24;                     // steps of 2^29 tokens
    for (uint32_t share = 1; share < (1u << 25); share += 1 + share / 9)
        for (uint32_t steps = most; steps > most - 40; --steps) CHECK(draft::shares_of(steps, share) == (steps + share - 1) / share, "shares_of %u %u", steps, share);
    int cuts = 0;
    for (int k = 0; k < 20000; ++k) {
        const int heads[][2] = {{32, 8}, {28, 4}, {16, 1}, {1, 1}, {4, 2}};
        const int* h = heads[upto(4)];
        const int D = 64 << upto(2), group = h[0] / h[1];
        const int64_t B = 1 + upto(upto(1) ? 300 : 20), each = 1 + upto(16), max_kv = ((int64_t)1 << 29) - upto(upto(1) ? 1000 : 1 << 28);
        std::vector<int> ms(B);
        int64_t T = 0;
        for (auto& m : ms) T += m = (int)upto(each);
        if (T == 0) continue;
        const draft::AttentionPlan p = draft::tree_plan(T, B, h[0], h[1], D, max_kv, 0, true);
        if (p.whole) continue;
        struct X { uint32_t tiles, steps; };
        std::vector<X> xs;
        const bool all_long = upto(1);
        for (int m : ms) {
            const mx::Span s = draft::tree_span((int)(all_long ? max_kv - upto(100) : upto(max_kv)), m, 0);
            xs.push_back({mx::tiles_of(m, group, p.rows), (uint32_t)std::max((s.hi + mx::kStep - 1) / mx::kStep - s.lo / mx::kStep, 1)});
        }
        auto sum = [&](auto of) { uint32_t r = 0; for (const X& x : xs) r += of(x); return r; };
        const uint32_t share = draft::shortest_share((uint32_t)p.workgroups, (uint32_t)max_kv / mx::kStep + 1, p.wk, sum);
        uint64_t count = 0, shorter = 0;
        bool cut = false;
        for (const X& x : xs) {
            const uint64_t by = (uint64_t)share * p.wk, less = by - p.wk;
            count += x.tiles * ((x.steps + by - 1) / by), cut |= x.tiles && x.steps > by;
            if (less) shorter += x.tiles * ((x.steps + less - 1) / less);
        }
        cuts += cut;
        // what is cut has room in the workspace; nothing shorter would do
        CHECK(!cut || count <= (uint64_t)p.workgroups, "room T %d B %d kv %d: %d of %d", (int)T, (int)B, (int)max_kv, (int)count, (int)p.workgroups);
        CHECK(share == 1 || shorter > (uint64_t)p.workgroups, "shortest T %d B %d kv %d", (int)T, (int)B, (int)max_kv);
        CHECK(count <= (uint64_t)draft::plan_workgroups(p), "launch T %d B %d kv %d", (int)T, (int)B, (int)max_kv);
    }
    CHECK(cuts > 3000, "cuts %d", cuts);
}

// One buffer for a server's calls: what the largest has asked for is enough where sequences end, rows are fewer, or the window or the cache is shorter.
static void check_workspace() {
    int some = 0;
    for (int k = 0; k < 40000; ++k) {
        const int heads[][2] = {{32, 8}, {28, 4}, {16, 1}, {1, 1}, {8, 8}, {64, 64}};
        const int* h = heads[upto(5)];
        const int D = 64 << upto(2);
        const int64_t B = 1 + upto(upto(1) ? 300 : 20), T = B * (1 + upto(upto(1) ? 8 : 200)), max_kv = upto(upto(1) ? 9000 : 200000);
        const int64_t b = 1 + upto(B - 1), most = 1 + upto(T - 1), t = upto(1) ? most : most < b ? b : most / b * b, kv = upto(1) ? max_kv : upto(max_kv), window = upto(2) ? 0 : 1 + upto(5000);
        const bool listed = t % b ? true : upto(1);
        if (t > T) continue;
        const size_t need = draft::plan_workspace(draft::tree_plan(t, b, h[0], h[1], D, kv, window, listed), h[1], D), has = draft::tree_workspace(T, B, h[0], h[1], D, max_kv);
        CHECK(need <= has, "workspace of T %d B %d kv %d in that of T %d B %d kv %d: heads %d %d, D %d, window %d", (int)t, (int)b, (int)kv, (int)T, (int)B, (int)max_kv, h[0], h[1], D, (int)window);
        CHECK(has <= (size_t)4 * (D + 2) * (8192 + 32 * h[1]), "workspace");
        some += need > 0;
    }
    CHECK(some > 10000, "workspaces %d", some);
}

int main() {
    check_workspace();
    check_shares();
    printf("draft_limits_check: ok\n");
    return 0;
}
