// Host-side check of what the four-bit kernels (csrc/mom_mx_*.hip.inc) take from csrc/mom_mx.h:
//   1. a cache block's bytes: what the tokens append fills it, every nibble once, and what attention loads lies inside it;
//   2. scales are the smallest that leave at most 7, and a number that is cut to 32 bits goes to the code of the whole one;
//   3. tile numbers: every tile of every sequence has one of its own, in their order, and the numbers behind them are none's;
//   4. tokens: the steps of the wavefronts over all shares take every token that a tile sees once, pages are looked up inside the table,
//      and the workspace holds the shares of every window.
#include <cmath>
#include <cstdio>
#include <cstring>
#include <limits>
#include <random>
#include <set>
#include <vector>

#include "mom_mx.h"

namespace mx = momk::mx;

static int bad = 0;
#define CHECK(c, ...)                                                                                             \
    do {                                                                                                          \
        if (!(c) && bad++ < 5) { std::printf("%s: ", #c); std::printf(__VA_ARGS__); std::printf("\n"); }          \
    } while (0)

static void layout(int P, int D) {
    const int n = (int)mx::block_bytes(P, D);
    CHECK(n % 16 == 0, "block %d x %d", P, D);
    std::vector<int> nibble(2 * n, 0);
    auto byte = [&](int at, int half) {          // half: 0 low, 1 high, 2 both
        CHECK(at >= 0 && at < n, "append: byte %d of %d (%d x %d)", at, n, P, D);
        if (at < 0 || at >= n) return;
        if (half != 1) ++nibble[2 * at];
        if (half != 0) ++nibble[2 * at + 1];
    };
    for (int at = 0; at < P; ++at)
        for (int chunk = 0; chunk < D / 8; ++chunk) {
            for (int i = 0; i < 4; ++i) byte(mx::key_codes(D, at) + chunk * 4 + i, 2);
            const int group = chunk / 4, high = (chunk >> 1) & 1;
            for (int j = 0; j < 8; ++j) {
                const int l = (chunk & 1) * 8 + j, dim = chunk * 8 + j;
                CHECK(dim == 32 * group + 16 * high + l, "dimension %d", dim);
                byte(mx::value_codes(P, D, at >> 2) + l * (D / 8) + group * 4 + (at & 3), high);
            }
            if (chunk % 4 == 0) {
                byte(mx::key_scales(P, D, at) + group, 2);
                byte(mx::value_scales(P, D, at >> 2) + group * 4 + (at & 3), 2);
            }
        }
    for (int i = 0; i < 2 * n; ++i) CHECK(nibble[i] == 1, "nibble %d of %d x %d filled %d times", i, P, D, nibble[i]);
    for (int at = 0; at < P; at += 16)
        for (int lane = 0; lane < 64; ++lane) {
            const int l = lane & 15, h = lane >> 4;
            const int kc = mx::key_codes(D, at + l) + h * (D / 8), ks = mx::key_scales(P, D, at + l) + (D == 256 ? 2 * h : D == 128 ? h : h >> 1);
            const int vc = mx::value_codes(P, D, (at >> 2) + h) + l * (D / 8), vs = mx::value_scales(P, D, (at >> 2) + h);
            const int align = D / 8 < 16 ? D / 8 : 16;
            CHECK(kc >= 0 && kc + D / 8 <= mx::key_scales(P, D, 0) && kc % align == 0, "keys of lane %d", lane);
            CHECK(ks + (D == 256 ? 2 : 1) <= mx::value_codes(P, D, 0) && (D != 256 || ks % 2 == 0), "key scales of lane %d", lane);
            CHECK(vc >= mx::value_codes(P, D, 0) && vc + D / 8 <= mx::value_scales(P, D, 0) && vc % align == 0, "values of lane %d", lane);
            CHECK(vs >= mx::value_scales(P, D, 0) && vs + D / 8 <= n && vs % align == 0, "value scales of lane %d", lane);
            // the operand's dimensions: word j of a lane's keys is dimensions h D/4 + 8 j ..., in the block that its scale is of
            for (int j = 0; j < D / 32; ++j) {
                const int dim = h * (D / 4) + 8 * j;
                CHECK(dim / 2 == h * (D / 8) + 4 * j, "word %d", j);
                CHECK(dim / 32 == ks - mx::key_scales(P, D, at + l) + (D == 256 ? j / 4 : 0), "scale of word %d", j);
            }
        }
}

// The code of a magnitude in units of the scale, by the definition.
static int code_of(double a) {
    const double mags[8] = {0, 0.5, 1, 1.5, 2, 3, 4, 6};
    int best = 0;
    for (int k = 1; k < 8; ++k) {
        const double o = std::fabs(a - mags[k]), b = std::fabs(a - mags[best]);
        if (o < b || (o == b && k % 2 == 0)) best = k;
    }
    return best;
}

static void encoding(std::mt19937& rng) {
    std::normal_distribution<double> normal(0, 1);
    for (int i = 0; i < 20000; ++i) {
        double x[32], top = 0;
        uint32_t bits = 0;
        const int mode = i % 5, e = i % 7 == 0 ? (int)(rng() % 24) - 140 : (int)(rng() % 200) - 100;
        for (double& v : x) {
            double m = mode == 0 ? normal(rng) : mode == 1 ? (double)(int)(rng() % 57) / 8 : mode == 2 ? (double)(int)(rng() % 29) / 4 : mode == 3 ? 0.0 : 7 * (rng() % 2);
            if (rng() % 8 == 0) m = std::nextafter(m, rng() % 2 ? 8.0 : 0.0);        // right beside a border
            v = std::ldexp(rng() % 2 ? m : -m, mode == 0 ? 0 : e);
            const float f = mx::cut_to_odd(v);
            CHECK(std::signbit(f) == std::signbit(v), "sign of %g", v);
            bits = std::max(bits, mx::magnitude(f));
            top = std::max(top, std::fabs(v));
        }
        CHECK(mx::finite(bits), "finite");
        const int s = mx::scale_exponent(bits);
        if (top > 0) {
            CHECK(top <= std::ldexp(7.0, s), "top %g at scale %d", top, s);
            CHECK(s == mx::kMinExponent || top > std::ldexp(7.0, s - 1), "scale %d is not the smallest of %g", s, top);
        }
        for (double v : x) {
            const double a = std::fabs(std::ldexp(v, -s)), b = std::fabs(std::ldexp((double)mx::cut_to_odd(v), -s));
            CHECK(code_of(a) == code_of(b), "%.17g goes to code %d, in 32 bits to %d", a, code_of(a), code_of(b));
        }
    }
    for (double v : {(double)INFINITY, -(double)INFINITY, (double)NAN}) CHECK(!mx::finite(mx::magnitude(mx::cut_to_odd(v))), "%g is finite", v);
    CHECK(mx::finite(mx::magnitude(mx::cut_to_odd(4e38))), "more than 32 bits hold is finite");
    CHECK(mx::scale_exponent(0) == mx::kMinExponent, "scale of nothing");
    CHECK(mx::scale_exponent(mx::magnitude(std::numeric_limits<float>::max())) == mx::kMaxExponent, "largest scale");
}

static void numbers(std::mt19937& rng) {
    const int B = 1 + rng() % 70, group = 1 + rng() % 16, rows = 16 << (rng() % 5);
    std::vector<int> start(B + 1, 0);
    for (int b = 0; b < B; ++b) start[b + 1] = start[b] + (int)(rng() % 4 == 0 ? 0 : rng() % (rng() % 2 ? 4 : 300));
    const int64_t n = mx::tile_numbers(start[B], B, group, rows);
    // the tile of a number as the kernel finds it: 64 sequences at a time, the first of them that has it
    auto find = [&](const std::vector<int>& at, int64_t number) {
        uint32_t before = 0;
        for (int b = 0; b < B; ++b) {
            const int s0 = std::min(std::max(at[b], 0), start[B]), m = std::min(std::max(at[b + 1], s0), start[B]) - s0;
            const uint32_t tiles = mx::tiles_of(m, group, rows);
            if ((uint32_t)number - before < tiles) return std::make_pair(mx::listed_tile((uint32_t)number, b, before, B, m, group, rows), m);
            before += tiles;
        }
        return std::make_pair(mx::Tile{-1, 0}, 0);
    };
    int64_t next = 0;
    for (int b = 0; b < B; ++b) {
        const int all = (start[b + 1] - start[b]) * group;
        for (int t = 0; t * rows < all; ++t, ++next) {
            CHECK(next < n, "number %lld of %lld", (long long)next, (long long)n);
            const mx::Tile of = find(start, next).first;
            CHECK(of.b == b && of.tile == t, "number %lld is tile %d of sequence %d, not %d of %d", (long long)next, of.tile, of.b, t, b);
        }
    }
    // the numbers behind are none's; starts that are out of order name no sequence that is not there
    std::vector<int> wild(B + 1);
    for (int& s : wild) s = (int)(rng() % (start[B] + 3)) - 1;
    for (int64_t number = 0; number < n; ++number) {
        if (number >= next) CHECK(find(start, number).first.b < 0, "number %lld", (long long)number);
        const auto [of, m] = find(wild, number);
        if (of.b >= 0) CHECK(of.b < B && of.tile >= 0 && (int64_t)of.tile * rows < (int64_t)m * group, "number %lld: tile %d of sequence %d", (long long)number, of.tile, of.b);
        const mx::Tile any = mx::checked_tile(rng() % (2 * B), rng() % 64, B, m, group, rows);
        if (any.b >= 0) CHECK(any.b < B && (int64_t)any.tile * rows < (int64_t)m * group, "tile %d of sequence %d", any.tile, any.b);
    }
    // sequences of m tokens each
    const int m = 1 + rng() % 300, each = (m * group + rows - 1) / rows;
    const int64_t even = (int64_t)B * mx::tiles_of(m, group, rows) + 2;
    std::set<std::pair<int, int>> tiles;
    for (int64_t number = 0; number < even; ++number) {
        const mx::Tile of = mx::even_tile(number, B, m, group, rows);
        if (of.b < 0) continue;
        CHECK(of.b < B && of.tile >= 0 && of.tile < each, "number %lld: tile %d of %d, sequence %d of %d", (long long)number, of.tile, each, of.b, B);
        CHECK(tiles.insert({of.b, of.tile}).second, "tile %d of sequence %d twice", of.tile, of.b);
    }
    CHECK((int)tiles.size() == B * each, "%d tiles of %d", (int)tiles.size(), B * each);
}

static void tokens(std::mt19937& rng) {
    const int D = 64 << (rng() % 3), Hkv = 1 << (rng() % 4), group = 1 + rng() % 8, page = 16 << (rng() % 5);
    const int B = 1 + rng() % 8, m = 1 + rng() % (rng() % 2 ? 4 : 400);
    const int max_kv = rng() % (rng() % 2 ? 300 : 40000), window = rng() % 2 ? 0 : 1 + rng() % 3000;
    const int n = max_kv ? rng() % (max_kv + 1) : 0;
    const mx::AttentionPlan p = mx::attention_plan((int64_t)B * m, B, Hkv * group, Hkv, D, max_kv, window, rng() % 2);
    CHECK(p.share % mx::kStep == 0 && p.share > 0 && p.shares >= 1, "share %lld", (long long)p.share);
    if (p.shares > 1) {
        const size_t need = (size_t)p.shares * B * m * Hkv * group * (D + 2) * 4, have = mx::attention_workspace((int64_t)B * m, B, Hkv * group, Hkv, D, max_kv);
        CHECK(need <= have, "workspace %zu of %zu", need, have);
    }
    CHECK(p.numbers >= (int64_t)B * mx::tiles_of(m, group, p.rows) && p.tiles >= (int64_t)B * Hkv, "numbers %lld, tiles %lld", (long long)p.numbers, (long long)p.tiles);
    const int all = m * group, table = (max_kv + page - 1) / page;
    const int tile = rng() % ((all + p.rows - 1) / p.rows);
    const int last_row = std::min((tile + 1) * p.rows, all) - 1;
    const mx::Span whole = mx::tile_span(n, m, tile * p.rows / group, last_row / group, window);
    for (int wave = 0; wave < (p.wk > 1 ? 1 : mx::kRowWaves); ++wave) {
        const int row0 = tile * p.rows + wave * 16 * p.qb;
        if (row0 >= all) continue;
        const int last = std::min(row0 + 16 * p.qb, all) - 1;
        const mx::Span seen = mx::tile_span(n, m, row0 / group, last / group, window);
        std::vector<int> taken(n + 1, 0);
        for (int z = 0; z < p.shares; ++z) {
            const mx::Span part = mx::share_span(whole, z, p.share);
            const int lo = std::max(part.lo, seen.lo), hi = std::min(part.hi, seen.hi), WK = p.wk;
            // many rows: the workgroup goes through its part 64 tokens at a time, and each wavefront looks at those that it sees
            const int from = WK > 1 ? lo : part.lo, to = WK > 1 ? hi : part.hi, length = WK > 1 ? mx::kStep : 64;
            for (int w = 0; w < WK; ++w) {
                const int token0 = from / mx::kStep * mx::kStep + (WK > 1 ? w * mx::kStep : 0);
                const int steps = to > token0 ? (to - token0 + WK * length - 1) / (WK * length) : 0;
                for (int step = 0; step < steps; ++step)
                    for (int i = 0; i < length; ++i) {
                        const int t = token0 + step * WK * length + i;
                        if (i % 16 == 0) {
                            const int slot = std::min(t, to - 1) / page;
                            CHECK(slot >= 0 && slot < table, "page %d of %d", slot, table);
                        }
                        if (t >= lo && t < hi) ++taken[t];
                    }
            }
        }
        // every row's tokens by the definition are among those taken, each of them once
        for (int t = 0; t < n; ++t) {
            bool visible = false;
            for (int r = row0; r <= last; ++r) {
                const int at = n - m + r / group;
                visible = visible || (t <= at && (window == 0 || t > at - window));
            }
            CHECK(taken[t] <= 1 && (!visible || taken[t] == 1), "token %d of %d taken %d times", t, n, taken[t]);
        }
    }
}

int main() {
    for (int P : {16, 32, 64, 128, 256})
        for (int D : {64, 128, 256}) {
            CHECK(mx::page_served(P) && mx::head_dim_served(D), "served");
            layout(P, D);
        }
    for (int P : {-16, 0, 8, 24, 48, 512}) CHECK(!mx::page_served(P), "page of %d", P);
    std::mt19937 rng(7);
    encoding(rng);
    for (uint32_t group = 1; group < (1 << 15); group += group < 300 ? 1 : 977)
        for (uint32_t r = 0; r < (1 << 16) + (1 << 15); r += r < 2000 ? 1 : 313)
            CHECK(mx::divided(r, mx::inverse_of(group)) == r / group, "divided: %u / %u", r, group);
    for (int i = 0; i < 3000; ++i) numbers(rng);
    for (int i = 0; i < 3000; ++i) tokens(rng);
    if (!bad) std::printf("four-bit layout, encoding, tiles and shares: ok\n");
    return bad != 0;
}
