// Walks on the CPU what mom_draft.h says of what refusals leave: powers of either sign against the C library's in more bits, weights of masked tokens, and the rest of rows that are
// equal, or nearly so, against sums in more bits.
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

static std::mt19937_64 rng(1);
static double number() { return (double)(rng() >> 11) / ((uint64_t)1 << 53); }
static double normal() { return sqrt(-2 * log(1 - number())) * cos(6.283185307179586 * number()); }

static double table[draft::kPowers];
static draft::Scale scale_of(double t) { return draft::scale_of(1.4426950408889634 / t, t); }

// The numbers are the nearest of 64 bits; a sum that ends at f^n leaves the next term.
static void check_power() {
    double worst = 0, far = 0, worst_scalar = 0;
    for (int k = 0; k < 600000; ++k) {
        const double reach = k % 3 == 0 ? 1.0 : k % 3 == 1 ? 60.0 : 995.0, scale = exp2(normal()) * draft::kPowers, d = (2 * number() - 1) * reach / scale * draft::kPowers;
        const draft::Power y = draft::power(table, d, scale);
        const long double want = exp2l((long double)d * scale / draft::kPowers), off = fabsl((long double)y.two * y.rest / want - 1);
        worst = std::max(worst, (double)off);
        if (k % 3 == 2) far = std::max(far, (double)off);
        const double t = -number() * reach;
        worst_scalar = std::max(worst_scalar, (double)fabsl(draft::power_of_two(t) / exp2l((long double)t) - 1));
    }
    // Taylor's 5.5e-16, the table's half step, the factor's, and theirs; what lies far off is no less exact
    CHECK(far < 5.5e-16 + 5 * 0x1p-53, "far power %g", far);
    CHECK(worst < 5.5e-16 + 5 * 0x1p-53, "power %g", worst);
    CHECK(worst_scalar < 4e-16, "power of two %g", worst_scalar);
    const draft::Scale s = scale_of(0.7);
    CHECK(draft::weight(table, 0.0, s) == 1.0, "weight of nothing off");
    CHECK(draft::weight(table, -INFINITY, s) == 0.0 && draft::weight(table, -3.4e38, s) == 0.0 && draft::weight(table, -1080 / s.k * draft::kPowers, s) == 0.0, "weight of what is masked");
    for (int k = 0; k < 100000; ++k) {
        // down to the smallest number, half a step of which is 2^-1075
        const double d = -1080 * number() / s.k * draft::kPowers;
        const long double want = exp2l((long double)d * s.k / draft::kPowers);
        CHECK(fabsl(draft::weight(table, d, s) - want) <= (5.5e-16 + 6 * 0x1p-53) * want + ldexpl(1.0L, -1075), "weight of what is far below");
    }
    // temperatures without end and next to none
    // many at once: the same numbers, and nothing of what is NaN, masked or far below; where floats lie further apart than that, the nearest alone
    for (int k = 0; k < 200000; ++k) {
        const draft::Scale c = scale_of(exp2(12 * normal()));
        const float top = (float)(normal() * exp2(20 * number())), x = k % 4 ? (float)(top + normal() * 300 / c.k * draft::kPowers) : nextafterf(top, k % 8 ? -INFINITY : INFINITY);
        const draft::Near n = draft::near_of(top, c);
        const double t = ((double)x - top) * c.k / draft::kPowers, w = draft::near_weight(table, x, top, n, c.k);
        CHECK(n.low <= top && n.high >= top && (top - (double)n.low) * c.k <= 1000.0001 * draft::kPowers && ((double)n.high - top) * c.k <= 1000.0001 * draft::kPowers, "near %g", top);
        if (t > -999.9 && t < 999.9) CHECK(w == draft::weight(table, (double)x - top, c), "near weight of %g", t);
        if (t < -1000.1) CHECK(w == 0.0, "near weight of what is masked");
        CHECK(draft::near_weight(table, -INFINITY, top, n, c.k) == 0.0 && draft::near_weight(table, NAN, top, n, c.k) == 0.0 && draft::near_weight(table, top, top, n, c.k) == 1.0, "near weight of what is masked");
    }
    CHECK(draft::near_weight(table, INFINITY, 3.402823466e38f, draft::near_of(3.402823466e38f, s), s.k) == 1.0, "near weight of infinity");
    const draft::Scale flat = scale_of(INFINITY), steep = scale_of(1e-45);
    const draft::Near all = draft::near_of(0.0, flat), one = draft::near_of(1.0, scale_of(1e-45));
    CHECK(draft::near_weight(table, -7.0f, 0.0, all, flat.k) == 1.0 && draft::near_weight(table, -INFINITY, 0.0, all, flat.k) == 0.0 && draft::near_weight(table, 1.0f, 1.0, one, steep.k) == 1.0 && draft::near_weight(table, 0.9999999f, 1.0, one, steep.k) == 0.0, "near weight of a flat row");
    CHECK(draft::weight(table, -7.0, flat) == 1.0 && draft::weight(table, -INFINITY, flat) == 0.0, "weight of a flat row");
    CHECK(draft::weight(table, 0.0, steep) == 1.0 && draft::weight(table, -1e-6, steep) == 0.0, "weight of a steep row");
}

struct Model {
    std::vector<float> logits;
    double top, inverse;
    std::vector<long double> exact;
};

// Sums in the order of lanes: 64 numbers each, then what they have.
static void sum(Model& m, double log2e_by_t, double t) {
    const int V = (int)m.logits.size();
    m.top = m.logits[0];
    std::vector<double> lanes(64, 0.0);
    for (int i = 0; i < V; ++i) {
        const draft::Power y = draft::power(table, (double)m.logits[i] - m.top, log2e_by_t * draft::kPowers);
        lanes[i / 4 % 64] = fma(y.two, y.rest, lanes[i / 4 % 64]);
    }
    double all = 0;
    for (double x : lanes) all += x;
    m.inverse = 1.0 / all;
    long double most = -INFINITY, total = 0;
    for (float x : m.logits) most = std::max(most, (long double)x);
    m.exact.resize(V);
    for (int i = 0; i < V; ++i) total += m.exact[i] = expl((m.logits[i] - most) / (long double)t);
    for (auto& x : m.exact) x /= total;
}

static void check_rest() {
    double worst = 0;
    for (int k = 0; k < 400; ++k) {
        const int V = 4096, kind = k % 4, peak = 1 + (int)(rng() % (V - 1));
        const double t = 0.4 + 0.6 * number(), height = t * (15 + 30 * number());
        Model p, q;
        for (int i = 0; i < V; ++i) {
            p.logits.push_back((float)normal());
            q.logits.push_back(kind == 0 ? p.logits[i] : (float)(p.logits[i] + 0.5 * normal()));
        }
        if (kind == 1) p.logits[peak] = q.logits[peak] = (float)height;
        if (kind == 2) {
            q.logits = p.logits;
            for (Model* m : {&p, &q}) m->logits[peak] = (float)height, m->logits[peak % (V - 1) + 1] = (float)(height - 0.3);
            q.logits[0] -= 3.0f;
        }
        sum(p, 1.4426950408889634 / t, t);
        sum(q, 1.4426950408889634 / t, t);
        draft::Row r = {};
        r.target_top = p.top, r.target_inverse = p.inverse, r.draft_top = q.top, r.draft_inverse = q.inverse, r.cut = 1.0, r.rest = 1.0;
        const draft::Scale s = scale_of(t);
        double rest = 0;
        long double exact = 0;
        for (int i = 0; i < V; ++i) {
            rest += draft::left(table, draft::left_of(r, s), p.logits[i], q.logits[i]);
            exact += std::max(p.exact[i] - q.exact[i], 0.0L);
        }
        if (kind == 0) CHECK(rest == 0.0, "rest of equal rows %g", rest);
        CHECK(fabs(rest - (double)exact) < draft::kNothing / 8, "rest %g of %g", rest, (double)exact);
        worst = std::max(worst, (double)fabsl(rest - exact));
        r.cut = 0.0;
        for (int i = 0; i < V; i += 97) CHECK(fabsl(draft::left(table, draft::left_of(r, s), p.logits[i], q.logits[i]) / p.exact[i] - 1) < 2e-14L, "left of a row without a cut");
    }
    printf("rest off by %g at most\n", worst);
}

int main() {
    for (int j = 0; j < draft::kPowers; ++j) table[j] = __builtin_bit_cast(double, draft::Powers().of[j]);
    check_power();
    check_rest();
    printf("draft_rest_check: ok\n");
    return 0;
}
