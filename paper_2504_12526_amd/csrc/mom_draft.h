// Drafted tokens in a tree: what a row sees, how the logits are cut into chunks and where their sums lie, and the power of two in 64 bits, as kernels
// (mom_draft.hip.inc, mom_mx_attention.hip.inc), entry points and a host program (tests/draft_check.cpp) ask.  Plain C++17, no HIP types.
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
    // of all heads as many as the compute units hold at once
    const int64_t at_once = kAtOnce * (p.qb == 1 && D <= 128 ? 2 : 1);
    p.workgroups = (at_once + Hkv - 1) / Hkv;
    p.whole = reach <= (p.tiles >= kManyTiles ? kManyWholeTokens : kWholeTokens) || p.tiles >= p.workgroups * Hkv || p.numbers >= 2 * p.workgroups;
    return p;
}
// Shares of a tile of `steps` (at least 1, under 2^24) that are no longer than `share`.
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
struct StepCount { template <typename X> MOM_MX_FN uint32_t operator()(const X& x) const { return x.tiles * x.steps; } };
struct TileCount { template <typename X> MOM_MX_FN uint32_t operator()(const X& x) const { return x.tiles; } };
template <typename Sum>
MOM_MX_FN uint32_t shortest_share(uint32_t workgroups, uint32_t most, uint32_t wk, const Sum& sum) {
    const uint32_t steps = sum(StepCount()), tiles = sum(TileCount());
    uint32_t lo = (steps / workgroups + wk - 1) / wk, hi = (most + wk) / wk;
    // a tile makes a share of its own and one for every whole share in it at most: so many steps are enough
    if (tiles < workgroups && steps / (workgroups - tiles) / wk + 1 < hi) hi = steps / (workgroups - tiles) / wk + 1;
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
// (Fewer tokens or a window may have tiles of 16 rows where more have 32: twice the workgroups, half the rows, and the same bytes.)
MOM_MX_FN size_t tree_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D, int64_t max_kv) {
    const size_t even = plan_workspace(tree_plan(T, B, Hq, Hkv, D, max_kv, 0, false), Hkv, D), uneven = plan_workspace(tree_plan(T, B, Hq, Hkv, D, max_kv, 0, true), Hkv, D);
    return even > uneven ? even : uneven;
}

// ---- verification ---------------------------------------------------------------------------------------------------------

// 2^t in 64 bits for t <= 0: t = n + f with |f| <= 1/2, Taylor's sum of 2^f = e^(f ln 2) to f^10 (the next term is under 2.2e-13 of it), and n as the exponent.  Whatever is under
// 2^-1074 is 0, minus infinity among it.
MOM_MX_FN double power_of_two(double t) {
    t = t > -1100.0 ? t : -1100.0;                      // (NaN too)
    const double n = rint(t), f = t - n;
    constexpr double kLn2 = 0.69314718055994530942;
    constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4, c5 = c4 * kLn2 / 5, c6 = c5 * kLn2 / 6, c7 = c6 * kLn2 / 7, c8 = c7 * kLn2 / 8,
                     c9 = c8 * kLn2 / 9, c10 = c9 * kLn2 / 10;
    double y = fma(c10, f, c9);
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

constexpr int kChunk = 4096;                            // logits of a row that a workgroup sums at once
constexpr int64_t kMostVocabulary = (int64_t)1 << 30;
MOM_MX_FN int64_t chunks(int64_t V) { return (V + kChunk - 1) / kChunk; }

// What lies in the workspace of a verification: sums of the chunks of each row of both models and of what is left there, then what is known of a row.
struct Part { double sum; float most; int32_t place; };                 // of a chunk: its largest logit and that one's place, sum of 2^((l - most) k)
struct Row {
    double target_top, target_inverse;                  // probabilities of the target here: 2^((l - top) k) inverse
    double draft_top, draft_inverse;
    double p, q;                                        // probabilities of this row's token at the row above
    double cut, rest;                                   // what is left here is max(p - cut q, 0) / rest
    int32_t rank, verdict, place, left;                 // which child it is; kOpen ...; the target's largest logit; refused children that `cut` counts
    int32_t again, held;                                // an earlier child of the same row is the same token; where a workgroup has its chunks' rests
};
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
