// Walks mom_draft.h on the CPU: bits of masks, what rows see with and without a window against a plain list, that shares cover all of it, the power of two against
// the C library's in more bits, and the workspace of a verification.
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
static int upto(int n) { return (int)(rng() % (unsigned)(n + 1)); }

static void check_bits() {
    for (int lo = -40; lo <= 70; ++lo)
        for (int hi = -40; hi <= 70; ++hi) {
            const uint32_t x = draft::bits_between(lo, hi);
            for (int i = 0; i < 32; ++i) CHECK((x >> i & 1) == (i >= lo && i < hi ? 1u : 0u), "bits %d %d bit %d", lo, hi, i);
        }
    for (int words = 1; words <= 4; ++words) {
        std::vector<uint32_t> mask(words);
        for (auto& w : mask) w = rng();
        for (int j = -80; j <= 32 * words + 80; ++j) {
            const uint32_t x = draft::mask_bits(mask.data(), words, j);
            for (int i = 0; i < 32; ++i) {
                const int at = j + i;
                CHECK((x >> i & 1) == (at >= 0 && at < 32 * words ? mask[at >> 5] >> (at & 31) & 1 : 0u), "mask bit %d of %d words", at, words);
            }
        }
    }
    const int32_t parents[] = {0, 0, 5, -1, 3, 4, 2147483647, -2147483647 - 1};
    const int want[] = {-1, 0, -1, -1, 3, 4, -1, -1};
    for (int j = 0; j < 8; ++j) CHECK(draft::above(parents, j) == want[j] && draft::above(nullptr, j) == j - 1, "above %d", j);
}

// What a row sees, one token after the other.
static std::vector<int> listed(const std::vector<uint32_t>& mask, int n, int m, int window) {
    std::vector<int> r;
    for (int t = 0; t < n; ++t) {
        const int j = t - (n - m);
        if (j < 0 || (j < 32 * (int)mask.size() && (mask[j >> 5] >> (j & 31) & 1))) r.push_back(t);
    }
    if (window > 0 && (int)r.size() > window) r.erase(r.begin(), r.end() - window);
    return r;
}

static void check_sight() {
    for (int k = 0; k < 60000; ++k) {
        const int words = 1 + upto(3), m = 1 + upto(140), n = upto(1) ? upto(300) : upto(2000), window = upto(2) ? 0 : 1 + upto(upto(1) ? 20 : 400);
        std::vector<uint32_t> mask(words);
        const int kind = upto(3);
        for (auto& w : mask) w = kind == 0 ? 0 : kind == 1 ? 0xffffffffu : rng();
        const int base = n - m;
        const draft::Sight s = draft::sight(mask.data(), words, base, m, window);
        std::vector<int> sees;
        for (int t = s.from; t < base; ++t) sees.push_back(t);
        for (int t = std::max(base + s.first, 0); t < n; ++t)
            if (draft::mask_bits(mask.data(), words, t - base) & 1) sees.push_back(t);
        const std::vector<int> want = listed(mask, n, m, window);
        CHECK(sees == want, "sight n %d m %d window %d words %d kind %d: %zu %zu", n, m, window, words, kind, sees.size(), want.size());
        const mx::Span span = draft::tree_span(n, m, window), whole = draft::tree_whole(n, m, window);
        for (int t : want) CHECK(t >= span.lo && t < span.hi, "span n %d m %d window %d token %d", n, m, window, t);
        for (int t = whole.lo; t < whole.hi; ++t) CHECK(std::binary_search(want.begin(), want.end(), t), "whole n %d m %d window %d token %d", n, m, window, t);
        CHECK(whole.hi <= std::max(base, 0), "whole");
        // shares of any length cover the span, one after the other
        const int origin = span.lo / mx::kStep * mx::kStep;
        const uint32_t steps = std::max((span.hi + mx::kStep - 1) / mx::kStep - span.lo / mx::kStep, 1), cut = draft::shares_of(steps, 1 + upto(80)), each = (steps + cut - 1) / cut;
        int covered = span.lo;
        for (uint32_t z = 0; z < cut; ++z) {
            const int lo = std::max(span.lo, origin + (int)(z * each) * mx::kStep), hi = std::max(std::min(span.hi, origin + (int)((z + 1) * each) * mx::kStep), lo);
            if (hi > lo) {
                CHECK(lo == covered, "shares n %d m %d window %d", n, m, window);
                covered = hi;
            }
        }
        CHECK(covered == span.hi || span.hi <= span.lo, "shares cover %d of %d, m %d window %d", covered, span.hi, m, window);
    }
}

static void check_plan() {
    for (uint32_t share = 1; share < 700; share += 1 + share / 20)
        for (int k = 0; k < 300; ++k) {
            const uint32_t steps = k < 100 ? k + 1 : 1 + upto((1 << 24) - 2);
            CHECK(draft::shares_of(steps, share) == (steps + share - 1) / share, "shares_of %u %u", steps, share);
        }
    for (int k = 0; k < 400000; ++k) {
        const uint32_t share = 3 + upto(6), steps = (1 << 24) - 1 - upto(1 << 20);
        CHECK(draft::shares_of(steps, share) == (steps + share - 1) / share, "shares_of %u %u", steps, share);
    }
    CHECK(draft::shares_of(12345, 1u << 27) == 1, "shares_of");
    for (int k = 0; k < 20000; ++k) {
        const int heads[][2] = {{32, 8}, {28, 4}, {8, 8}, {16, 1}, {16, 4}, {1, 1}};
        const int* h = heads[upto(5)];
        const int D = 64 << upto(2), group = h[0] / h[1];
        const int64_t B = 1 + upto(60), each = 1 + upto(upto(1) ? 16 : 300), max_kv = upto(3) ? upto(9000) : upto(200000), window = upto(2) ? 0 : 1 + upto(5000);
        for (int listed = 0; listed < 2; ++listed) {
            struct X { uint32_t tiles, steps; };
            std::vector<int> ms(B);
            int64_t T = 0;
            for (auto& m : ms) T += m = listed ? upto((int)each) : (int)each;
            if (T == 0) continue;
            const draft::AttentionPlan p = draft::tree_plan(T, B, h[0], h[1], D, max_kv, window, listed);
            CHECK(p.rows == 16 * p.qb && p.workgroups >= 1, "plan");
            std::vector<X> xs;
            uint32_t tiles = 0;
            for (int m : ms) {
                const mx::Span s = draft::tree_span(upto((int)max_kv), m, (int)window);
                xs.push_back({mx::tiles_of(m, group, p.rows), (uint32_t)std::max((s.hi + mx::kStep - 1) / mx::kStep - s.lo / mx::kStep, 1)});
                tiles += xs.back().tiles;
            }
            CHECK(tiles <= p.numbers && tiles <= draft::plan_workgroups(p), "plan numbers T %d B %d", (int)T, (int)B);
            CHECK(draft::plan_workspace(p, h[1], D) <= draft::tree_workspace(T, B, h[0], h[1], D, max_kv), "plan workspace T %d B %d heads %d D %d kv %d window %d", (int)T, (int)B, h[0], D, (int)max_kv, (int)window);
            if (p.whole) continue;
            auto sum = [&](auto of) { uint32_t r = 0; for (const X& x : xs) r += of(x); return r; };
            const uint32_t share = draft::shortest_share((uint32_t)p.workgroups, (uint32_t)max_kv / mx::kStep + 1, p.wk, sum), count = sum(draft::ShareCount{share * p.wk});
            bool cut = false, shorter_cuts_less = share > 1 && sum(draft::ShareCount{(share - 1) * p.wk}) <= p.workgroups;
            for (const X& x : xs) cut |= x.tiles && draft::shares_of(x.steps, share * p.wk) > 1;
            // what is cut has room in the workspace; nothing shorter would do
            CHECK(!cut || count <= p.workgroups, "plan share T %d B %d", (int)T, (int)B);
            CHECK(!cut || draft::plan_workspace(p, h[1], D) >= (size_t)count * h[1] * p.rows * (D + 2) * 4, "plan workspace T %d B %d", (int)T, (int)B);
            CHECK(count <= draft::plan_workgroups(p) && !shorter_cuts_less, "plan shares T %d B %d: %u of %d, share %u", (int)T, (int)B, count, (int)p.workgroups, share);
        }
    }
}

static void check_power() {
    double worst = 0;
    for (int k = 0; k < 400000; ++k) {
        const double t = -(double)upto(1 << 30) / (1 << 30) * (k % 3 == 0 ? 1.0 : k % 3 == 1 ? 60.0 : 1000.0);
        const long double want = exp2l((long double)t);
        worst = std::max(worst, fabs((double)(((long double)draft::power_of_two(t) - want) / want)));
    }
    // the first term that is left out, on either side of 0
    CHECK(worst < 3e-13, "power %g", worst);
    CHECK(draft::power_of_two(0.0) == 1.0 && draft::power_of_two(-3.0) == 0.125, "power whole");
    CHECK(draft::power_of_two(-INFINITY) == 0.0 && draft::power_of_two(-1e300) == 0.0 && draft::power_of_two(NAN) == 0.0, "power none");
}

static void check_layout() {
    for (int k = 0; k < 2000; ++k) {
        const int64_t T = 1 + upto(5000), B = 1 + upto(300), V = k % 3 ? 1 + upto(200000) : (1 + upto(40)) * draft::kChunk, cells = T * draft::chunks(V);
        CHECK(draft::chunks(V) * draft::kChunk >= V && (draft::chunks(V) - 1) * draft::kChunk < V, "chunks of %d", (int)V);
        const draft::Layout l = draft::layout(T, B, V);
        const size_t ends[] = {l.target, l.draft, l.rest, l.rows, l.lists, l.bytes};
        const size_t sizes[] = {(size_t)cells * sizeof(draft::Part), (size_t)cells * sizeof(draft::Part), 2 * (size_t)cells * 8, 2 * (size_t)T * sizeof(draft::Row), 2 * (size_t)(T + B) * 4};
        for (int i = 0; i < 5; ++i) CHECK(ends[i] % (i < 4 ? 8 : 4) == 0 && ends[i] + sizes[i] <= ends[i + 1], "layout part %d", i);
        CHECK(l.target % 16 == 0 && l.draft % 16 == 0 && l.bytes % 16 == 0, "layout");
    }
}

int main() {
    check_bits();
    check_sight();
    check_plan();
    check_power();
    check_layout();
    printf("draft_check: ok\n");
    return 0;
}
