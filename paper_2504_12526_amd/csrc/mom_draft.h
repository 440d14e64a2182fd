// Drafted tokens in a tree: what a row sees, how the logits are cut into chunks and where their sums lie, and the power of two in 64 bits, as kernels
// (mom_draft.hip.inc, mom_draft_attention.hip.inc), entry points and host programs (tests/draft_*check.cpp) ask.  Plain C++17, no HIP types.
//
// The rows of a sequence are its m new tokens: row i is token n - m + i of the n in the cache.  Bit j of a row's mask says that it sees row j.
#ifndef MOM_DRAFT_H
#define MOM_DRAFT_H

#include <math.h>
#include <stddef.h>
#include <stdint.h>

#include "mom_mx.h"

namespace momk {
namespace draft {

constexpr int kMostRows = 512;                          // rows of a sequence that masks and verification know
constexpr int kMostWords = kMostRows / 32;

// ---- what a row sees ------------------------------------------------------------------------------------------------------

// The row above row j by the list of parents (null: a chain); -1 where there is none, which what is no earlier row says too.
MOM_MX_FN int above(const int32_t* parents, int j) {
    const int p = parents ? parents[j] : j - 1;
    return p >= 0 && p < j ? p : -1;
}

// Bits [lo, hi) of 32, the bounds being any numbers.
MOM_MX_FN uint32_t bits_between(int lo, int hi) {
    if (lo < 0) lo = 0;
    if (hi > 32) hi = 32;
    if (hi <= lo) return 0;
    return (0xffffffffu >> (32 - (hi - lo))) << lo;
}

// The 32 bits of a mask of `words` words from bit j on, which may lie outside of it.
MOM_MX_FN uint32_t mask_bits(const uint32_t* mask, int words, int j) {
    const int w = j >> 5, s = j & 31;
    const uint32_t low = w >= 0 && w < words ? mask[w] : 0, high = s && w + 1 >= 0 && w + 1 < words ? mask[w + 1] : 0;
    return s ? low >> s | high << (32 - s) : low;
}

// With a window a row sees the last `window` (over 0) of what its mask and the tokens before the m rows give it, in the order of the cache: tokens
// [from, base) of those, base = n - m, and of its mask the bits from `first` on.
struct Sight { int from, first; };
MOM_MX_FN Sight sight(const uint32_t* mask, int words, int base, int m, int window) {
    const int lowest = base < 0 ? -base : 0, highest = m < 32 * words ? m : 32 * words;
    if (window <= 0) return {0, lowest};
    int left = window;
    for (int w = (highest - 1) >> 5; w >= 0 && 32 * w + 32 > lowest; --w) {
        uint32_t x = mask[w] & bits_between(lowest - 32 * w, highest - 32 * w);
        const int count = __builtin_popcount(x);
        if (count >= left) {
            for (int i = left; i < count; ++i) x &= x - 1;
            return {base, 32 * w + __builtin_ctz(x)};
        }
        left -= count;
    }
    return {base > left ? base - left : 0, lowest};
}

// The tokens that any row of a sequence sees: what its window leaves of those before the rows (a row without bits has the most of them), and the rows.
MOM_MX_FN mx::Span tree_span(int n, int m, int window) {
    const int lo = window > 0 && n - m > window ? n - m - window : 0;
    if (n <= lo) return {0, 0};
    return {lo, n};
}
// The tokens that all rows see and no mask has a say in: [lo, hi).
MOM_MX_FN mx::Span tree_whole(int n, int m, int window) {
    const int base = n - m;
    int lo = window > 0 ? base - window + (m < window ? m : window) : 0;
    if (lo < 0) lo = 0;
    return {lo, base > 0 ? base : 0};
}
// How attention is launched: tiles of 16 qb rows whose tokens `wk` wavefronts share; their tokens in shares, as many as `workgroups` of a key head that there are at once allow
// (the device knows the lengths); whole: a workgroup a tile, and nothing to join.
struct AttentionPlan {
    int qb, wk, rows;
    bool whole;
    int64_t numbers, workgroups, tiles;                 // numbers: of tiles of a key head at most; tiles: about as many there are, of all heads
};
// Tiles of 16 rows where a sequence has no more, and where all of them together have little to do: a tile of 32 takes longer to begin and to end (8 rows of 32 heads, 8 of them key heads,
// after 317 tokens 7.1 us, 9.0 with 32; after 1536 12.1 and 13.8; of 64 tiles of 16 rows 24.0, 32.5), but turns the tokens into operands once for twice the rows (32 sequences of 4608 tokens
// 34.7 us, 46.1 with 16; 16 rows after 131072 59.6 and 88.1; of 128 tiles and 1024 tokens 16.8 and 17.2).  256 dimensions leave registers for 16.
constexpr int64_t kLittle = 65536;                      // tokens, of all tiles of 16 rows
// Whole tiles: a second launch joins shares, 5 us.  8 tiles of 32 rows and 1024 tokens take 12.7 us whole and 13.5 in shares, 1536 tokens 15.5 and 13.8; 64 tiles of 1024 12.9 and 16.9; as many tiles
// as workgroups at once, of lengths up to 8192, 50.6 and 57.7.
constexpr int kWholeTokens = 1024, kManyWholeTokens = 1536, kManyTiles = 64, kAtOnce = 256;
// Workgroups of a key head, so that there are as many of all heads as the compute units hold at once.
MOM_MX_FN int64_t workgroups_at_once(int qb, int Hkv, int D) { return (kAtOnce * (qb == 1 && D <= 128 ? 2 : 1) + Hkv - 1) / Hkv; }
MOM_MX_FN AttentionPlan tree_plan(int64_t T, int64_t B, int Hq, int Hkv, int D, int64_t max_kv, int64_t window, bool listed) {
    const int group = Hq / Hkv;
    const int64_t average = (T * group + B - 1) / B, rows = listed ? T : T / B;
    int64_t reach = max_kv;
    if (window > 0 && window + rows + mx::kStep < reach) reach = window + rows + mx::kStep;
    AttentionPlan p;
    p.wk = 8;
    p.qb = average <= 16 || D == 256 || (average + 15) / 16 * B * Hkv * reach <= kLittle ? 1 : 2;
    p.rows = 16 * p.qb;
    const int64_t even = B * ((average + p.rows - 1) / p.rows), uneven = (2 * T * group + (B + 1) * p.rows - 1) / (2 * p.rows);
    p.tiles = (!listed ? even : uneven < B ? B : uneven) * Hkv;
    p.numbers = listed ? mx::tile_numbers(T, B, group, p.rows) : even;
    p.workgroups = workgroups_at_once(p.qb, Hkv, D);
    p.whole = reach <= (p.tiles >= kManyTiles ? kManyWholeTokens : kWholeTokens) || p.tiles >= p.workgroups * Hkv || p.numbers >= 2 * p.workgroups;
    return p;
}
// Shares of a tile of `steps` (at least 1, at most 2^24 + 1) that are no longer than `share`.
MOM_MX_FN uint32_t shares_of(uint32_t steps, uint32_t share) {
    uint32_t q = (uint32_t)((float)steps * (1.0f / (float)share));       // two roundings: the quotient cut off, or one less
    q += q * share < steps;
    q += q * share < steps;
    return q < 1 ? 1 : q;
}
// The shortest share, counted in `wk` steps, with which all tiles make no more shares than `workgroups` (or none of them two): sum(f) is the sum of f(x) over all sequences x, x.tiles
// tiles of x.steps steps, at most `most`.
struct ShareCount {
    uint32_t share;
    template <typename X> MOM_MX_FN uint32_t operator()(const X& x) const { return x.tiles * shares_of(x.steps, share); }
};
struct RoundCount {                                     // (in `wk` steps, which 32 bits hold for 2047 tiles of 2^29 tokens)
    uint32_t wk;
    template <typename X> MOM_MX_FN uint32_t operator()(const X& x) const { return x.tiles * ((x.steps + wk - 1) / wk); }
};
struct TileCount { template <typename X> MOM_MX_FN uint32_t operator()(const X& x) const { return x.tiles; } };
template <typename Sum>
MOM_MX_FN uint32_t shortest_share(uint32_t workgroups, uint32_t most, uint32_t wk, const Sum& sum) {
    const uint32_t rounds = sum(RoundCount{wk}), tiles = sum(TileCount());
    uint32_t lo = rounds / workgroups, hi = (most + wk) / wk;
    // a tile makes a share of its own and one for every whole share in it at most: so many steps are enough
    if (tiles < workgroups && rounds / (workgroups - tiles) + 1 < hi) hi = rounds / (workgroups - tiles) + 1;
    if (lo < 1) lo = 1;
    while (lo < hi) {
        const uint32_t mid = (lo + hi) / 2;
        if (sum(ShareCount{mid * wk}) <= workgroups) hi = mid;
        else lo = mid + 1;
    }
    return hi;
}
MOM_MX_FN int64_t plan_workgroups(const AttentionPlan& p) { return p.whole || p.numbers > p.workgroups ? p.numbers : p.workgroups; }
MOM_MX_FN size_t plan_workspace(const AttentionPlan& p, int Hkv, int D) { return p.whole ? 0 : (size_t)p.workgroups * Hkv * p.rows * (D + 2) * 4; }
// That of all calls of no more rows, sequences and tokens (fewer tiles are cut where more are whole), with any window: of either height of tiles.
MOM_MX_FN size_t tree_workspace(int64_t, int64_t, int, int Hkv, int D, int64_t max_kv) {
    if (max_kv <= kWholeTokens) return 0;
    size_t most = 0;
    for (int qb = 1; qb <= 2; ++qb) {
        AttentionPlan p = {};
        p.rows = 16 * qb, p.workgroups = workgroups_at_once(qb, Hkv, D);
        const size_t bytes = qb == 2 && D == 256 ? 0 : plan_workspace(p, Hkv, D);
        most = bytes > most ? bytes : most;
    }
    return most;
}

// ---- verification ---------------------------------------------------------------------------------------------------------

// 2^t in 64 bits for t <= 0: t = n + f with |f| <= 1/2, Taylor's sum of 2^f = e^(f ln 2) to f^13 (the next term is under 5e-18), and n as the exponent: off by the
// roundings, under 4e-16.  Whatever is under 2^-1074 is 0, minus infinity among it.
MOM_MX_FN double power_of_two(double t) {
    t = t > -1100.0 ? t : -1100.0;                      // (NaN too)
    const double n = rint(t), f = t - n;
    constexpr double kLn2 = 0.69314718055994530942;
    constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4, c5 = c4 * kLn2 / 5, c6 = c5 * kLn2 / 6, c7 = c6 * kLn2 / 7, c8 = c7 * kLn2 / 8,
                     c9 = c8 * kLn2 / 9, c10 = c9 * kLn2 / 10;
    constexpr double c11 = c10 * kLn2 / 11, c12 = c11 * kLn2 / 12, c13 = c12 * kLn2 / 13;
    double y = fma(c13, f, c12);
    y = fma(y, f, c11);
    y = fma(y, f, c10);
    y = fma(y, f, c9);
    y = fma(y, f, c8);
    y = fma(y, f, c7);
    y = fma(y, f, c6);
    y = fma(y, f, c5);
    y = fma(y, f, c4);
    y = fma(y, f, c3);
    y = fma(y, f, c2);
    y = fma(y, f, c1);
    y = fma(y, f, 1.0);
    return ldexp(y, (int)n);
}

// 2^t for many t of either sign, t * 1024 given as d k (at most 2^31 in size): t = n + j / 1024 + f, |f| <= 1/2048: 2^(j / 1024) from a table times Taylor's sum to f^3 (the next term is under
// 5.5e-16), n added to the exponent: right between 2^-1022 and 2^1023.  d k is never rounded, f alone is, so distances make nothing less exact.  As two factors, so that a sum takes them in one step:
// 7 instructions in 64 bits, 3 others and a read, where power_of_two has 23 and more.  (480 rows of 128256 logits and 208 of 152064 in bf16: 43.3 and 27.2 us; 45.0 and 28.0 with 128 powers and a
// sum to f^4, off by 1.3e-15.)
constexpr int kPowers = 1024, kPowerBits = 10;
struct Powers {
    unsigned long long of[kPowers];     // the numbers' bits, less j at the place where 1024 n + j is added: that leaves n at the exponent's
    constexpr Powers() : of() {
        // e^(j ln 2 / 1024), Taylor's sum from its end; ln 2 as the part whose products with j are exact, and the rest
        constexpr double kHigh = 0x1.62e42fefap-1, kLow = 0x1.cf79abc9e3b3ap-40;
        for (int j = 0; j < kPowers; ++j) {
            const double x = j * kHigh / kPowers;
            double sum = 1.0;
            for (int n = 24; n >= 2; --n) sum = 1.0 + x / n * sum;
            sum = 1.0 + x * sum + j * kLow / kPowers * (1.0 + x * sum);
            of[j] = __builtin_bit_cast(unsigned long long, sum) - ((unsigned long long)j << (52 - kPowerBits));
        }
    }
};
struct Power { double two, rest; };
struct Split { uint32_t whole; double rest; };          // 1024 t to the nearest, and the power of what that leaves
MOM_MX_FN Split split_power(double d, double k) {
    constexpr double kStep = 0.69314718055994530942 / kPowers, kMagic = 6755399441055744.0;       // 1.5 * 2^52: added, the sum's low word is the nearest whole number
    const double moved = fma(d, k, kMagic), f = fma(d, k, kMagic - moved);
    double y = fma(f, kStep * kStep * kStep / 6, kStep * kStep / 2);
    y = fma(y, f, kStep);
    return {(uint32_t)__builtin_bit_cast(uint64_t, moved), fma(y, f, 1.0)};
}
MOM_MX_FN Power power(const double* table, double d, double k) {
    const Split s = split_power(d, k);
    const uint64_t two = __builtin_bit_cast(uint64_t, table[s.whole & (kPowers - 1)]);
    return {__builtin_bit_cast(double, (uint64_t)((uint32_t)(two >> 32) + (s.whole << (20 - kPowerBits))) << 32 | (uint32_t)two), s.rest};
}
// A logit's weight by its distance from what its row's weights are relative to: 2^(d k / 1024) down to the smallest number there is, 0 under it (what is masked is minus infinity).
struct Scale { double k, limit; };
MOM_MX_FN Scale scale_of(double log2e_by_t, double t) { return {log2e_by_t * kPowers, t * (1100.0 * 0.69314718055994530942)}; }
MOM_MX_FN double weight(const double* table, double d, const Scale& s) {
    const Split x = split_power(fmin(fmax(d, -s.limit), s.limit), s.k);
    const uint32_t j = x.whole & (kPowers - 1);
    const uint64_t two = __builtin_bit_cast(uint64_t, table[j]);
    const double root = __builtin_bit_cast(double, (uint64_t)((uint32_t)(two >> 32) + (j << (20 - kPowerBits))) << 32 | (uint32_t)two);
    return d > -s.limit ? ldexp(root * x.rest, (int32_t)x.whole >> kPowerBits) : 0.0;
}
// The same for many logits at once, down to 2^-1000: those that are nearer to what the weights of their row are relative to than [low, high] says.
struct Near { float low, high; };
MOM_MX_FN Near near_of(double top, const Scale& s) {
    const double low = top - s.limit * (1000.0 / 1100.0), high = top + s.limit * (1000.0 / 1100.0);
    Near n = {low < -3.402823466e38 ? -3.402823466e38f : (float)low, high > 3.402823466e38 ? 3.402823466e38f : (float)high};
    if (n.low < low) n.low = nextafterf(n.low, INFINITY);
    if (n.high > high) n.high = nextafterf(n.high, -INFINITY);
    return n;
}
MOM_MX_FN double near_weight(const double* table, float x, double top, const Near& n, double k) {
    const Power y = power(table, (double)fminf(fmaxf(x, n.low), n.high) - top, k);
    return x >= n.low ? y.two * y.rest : 0.0;           // (NaN as minus infinity)
}
// A rest under this part of p counts as nothing.  p and q are each off by 5.5e-16 by the power's sum and by the roundings of a hundred additions at most, 1.2e-14, so what both leave of one another is off by
// 2.5e-14 of p; that would be the whole of what is drawn from where the rest is no larger.
constexpr double kNothing = 1.0 / ((int64_t)1 << 42);

constexpr int kChunk = 4096;                            // logits of a row that a workgroup sums at once
constexpr int64_t kMostVocabulary = (int64_t)1 << 30;
MOM_MX_FN int64_t chunks(int64_t V) { return (V + kChunk - 1) / kChunk; }

// What lies in the workspace of a verification: sums of the chunks of each row of both models and of what is left there, then what is known of a row.
struct Part { double sum; float most; int32_t place; };                 // of a chunk: sum of 2^((l - most) k), most being its row's first logit, or its own largest; greedy: that and its place
struct Row {
    double target_top, target_inverse;                  // probabilities of the target here: 2^((l - top) k) inverse
    double draft_top, draft_inverse;
    double p, q;                                        // probabilities of this row's token at the row above
    double cut, rest;                                   // what is left here is max(p - cut q, 0) / rest; cut 0: p
    int32_t rank, verdict, place, left;                 // which child it is; kOpen ...; the target's largest logit; refused children that `cut` counts, without a drafting model the row from which on they
                                                        // are taken off
    int32_t again, held;                                // the last child of the same row before it that is the same token, 0: none; where a workgroup has its chunks' rests
};
// What is left of a token's probability at a row, not divided by the rest.  All that has to agree takes it from here: with the same roundings on both sides equal rows leave nothing, and a chunk whose rest is
// above 0 has a token whose is.
struct Left {
    Near target, drafted;
    double target_top, target_inverse, draft_top, draft_inverse, cut, k;
};
MOM_MX_FN Left left_of(const Row& r, const Scale& s) {
    return {near_of(r.target_top, s), near_of(r.draft_top, s), r.target_top, r.target_inverse, r.draft_top, r.draft_inverse, r.cut, s.k};
}
MOM_MX_FN double left(const double* table, const Left& l, float target, float drafted) {
    const double p = near_weight(table, target, l.target_top, l.target, l.k) * l.target_inverse, q = near_weight(table, drafted, l.draft_top, l.drafted, l.k) * l.draft_inverse;
    return fmax(fma(-l.cut, q, p), 0.0);
}
constexpr int kOpen = 0, kTaken = 1, kRefused = 2, kPassed = 3;         // kPassed: not tried
struct Layout { size_t target, draft, rest, rows, lists, bytes; };
MOM_MX_FN Layout layout(int64_t T, int64_t B, int64_t V) {
    const size_t cells = (size_t)T * (size_t)chunks(V);
    Layout l;
    l.target = 0;
    l.draft = l.target + cells * sizeof(Part);
    l.rest = l.draft + cells * sizeof(Part);
    l.rows = l.rest + 2 * cells * sizeof(double);
    l.lists = l.rows + 2 * (size_t)T * sizeof(Row);
    l.bytes = l.lists + 2 * (size_t)(T + B) * sizeof(int32_t);
    l.bytes = (l.bytes + 15) / 16 * 16;
    return l;
}

}  // namespace draft
}  // namespace momk

#endif
