// Four-bit elements in blocks of 32 with a common power of two (OCP Microscaling: e2m1 elements, one e8m0 scale): their encoding, the layout
// of a block of the paged cache, and how attention over it is cut into tiles and shares, as kernels (mom_mx_*.hip.inc), entry points and a
// host program (tests/mx_check.cpp) ask.  Plain C++17, no HIP types.
//
// A code is sign, two exponent bits, one mantissa bit: 0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; a scale byte b stands for 2^(b - 127),
// 255 for NaN.  gfx950 turns two codes and a scale into two bf16 numbers in one instruction, exactly (8 significant bits hold every product), so
// nothing is rounded between the cache and the matrix cores; and two numbers and a scale into two codes: the nearest, ties to the even one, above 6 the
// largest.
#ifndef MOM_MX_H
#define MOM_MX_H

#include <stddef.h>
#include <stdint.h>
#include <string.h>

#if defined(__HIPCC__)
#define MOM_MX_FN __host__ __device__ inline
#else
#define MOM_MX_FN inline
#endif

namespace momk {
namespace mx {

constexpr int kBlock = 32;                              // elements of a block
constexpr int kScaleNaN = 255;
constexpr int kMinExponent = -125, kMaxExponent = 125;  // of a scale that the library writes: every nonzero value is a normal bf16 number then

// ---- encoding -------------------------------------------------------------------------------------------------------------

// The bits of a magnitude, which order like it, infinities and NaN last.
MOM_MX_FN uint32_t magnitude(float x) {
    uint32_t b;
    memcpy(&b, &x, 4);
    return b & 0x7fffffffu;
}
MOM_MX_FN bool finite(uint32_t magnitude) { return magnitude < 0x7f800000u; }

// Exponent of the scale of a block whose largest magnitude is `top` (finite): the power of two that brings it to at most 7, which is half a step
// away from the largest element 6, so that no element is further than half a step from its code (the rounding down to [4, 8) that is
// also in use cuts off up to a quarter of the largest element).  Above 7 * 2^125
// (the largest number of bf16 is just under 8 * 2^125) 6 * 2^125 stands for everything.
MOM_MX_FN int scale_exponent(uint32_t top) {
    const int e = (int)(top >> 23) - 127 - 2 + ((top & 0x7fffffu) > (3u << 21) ? 1 : 0);
    return e < kMinExponent ? kMinExponent : e > kMaxExponent ? kMaxExponent : e;
}

// x in 32 bits, cut off, the last bit set if anything was: on the same side of every number of fewer bits, borders between codes among them, as x (a
// rounded one may come to lie on a border, whose ties then go the wrong way).
MOM_MX_FN float cut_to_odd(double x) {
    const float f = (float)x;
    const double back = (double)f;
    uint32_t b;
    memcpy(&b, &f, 4);
    if ((back < 0 ? -back : back) > (x < 0 ? -x : x)) b -= 1;
    if (back != x) b |= 1;
    float r;
    memcpy(&r, &b, 4);
    return r;
}

// ---- layout of the paged cache --------------------------------------------------------------------------------------------

// A page holds P tokens for every key head, a block of block_bytes each:
//     key codes     [P][D / 2]            low nibble first
//     key scales    [P][D / 32]
//     value codes   [P / 4][16][D / 32][4]   byte (q, l, g, t): dimension 32 g + l of token 4 q + t, and 32 g + 16 + l in the high nibble
//     value scales  [P / 4][D / 32][4]
// Keys are contracted over the dimensions and values over the tokens, and a lane of the matrix cores takes neighbours along the contracted
// axis: so a lane's operand of either is one run of bytes, and a wavefront's loads of 16 tokens are contiguous.
MOM_MX_FN size_t block_bytes(int P, int D) { return (size_t)P * (size_t)(D + D / 16); }
MOM_MX_FN int key_codes(int D, int at) { return at * (D / 2); }
MOM_MX_FN int key_scales(int P, int D, int at) { return P * (D / 2) + at * (D / 32); }
MOM_MX_FN int value_codes(int P, int D, int quad) { return P * (D / 2 + D / 32) + quad * 2 * D; }
MOM_MX_FN int value_scales(int P, int D, int quad) { return P * (D + D / 32) + quad * (D / 8); }

MOM_MX_FN bool head_dim_served(int64_t D) { return D == 64 || D == 128 || D == 256; }
MOM_MX_FN bool page_served(int64_t P) { return P >= 16 && P <= 256 && (P & (P - 1)) == 0; }

// ---- tiles of attention ---------------------------------------------------------------------------------------------------

// The query rows of a sequence at one key head, `group` query heads for each of its tokens, are cut into tiles of `rows`, numbered sequence by sequence.
// Where the tokens of a sequence start is known on the device only, and with it how many tiles there are: at most tile_numbers, those that are none's last
// (numbers that are none's between the others leave part of the compute units without work, as workgroups are handed out in order: 4 sequences of 8 tokens
// and 8192 in the cache, 32 rows a tile, took 29.5 us where every second number was none's).
// (32 bits hold all of it: up to 2^29 tokens and 2^31 rows of queries.)
MOM_MX_FN uint32_t tiles_of(uint32_t m, uint32_t group, uint32_t rows) { return (m * group + rows - 1) / rows; }
MOM_MX_FN int64_t tile_numbers(int64_t T, int64_t B, int group, int rows) { return T * group / rows + B; }

// The sequence of tile `number`, and which of its tiles it is; b = -1 where the number is no tile's.  Where every sequence has m tokens, and
// of sequence b whose m tokens have `before` tiles in front of them.
struct Tile { int b, tile; };
MOM_MX_FN Tile checked_tile(uint32_t b, uint32_t tile, uint32_t B, uint32_t m, uint32_t group, uint32_t rows) {
    if (b >= B || tile >= tiles_of(m, group, rows)) return {-1, 0};
    return {(int)b, (int)tile};
}
MOM_MX_FN Tile even_tile(uint32_t number, uint32_t B, uint32_t m, uint32_t group, uint32_t rows) {
    const uint32_t tiles = tiles_of(m, group, rows), b = tiles == 1 ? number : number / tiles;
    return checked_tile(b, number - b * tiles, B, m, group, rows);
}
MOM_MX_FN Tile listed_tile(uint32_t number, uint32_t b, uint32_t before, uint32_t B, uint32_t m, uint32_t group, uint32_t rows) {
    return checked_tile(b, number - before, B, m, group, rows);
}

// r / group for r < 2^16 + 2^15 and group < 2^15, by a multiplication: inverse = floor(2^32 / group) + 1 is off by less than 1 in 2^32 / group of it.
MOM_MX_FN uint32_t inverse_of(uint32_t group) { return group == 1 ? 0u : (uint32_t)(((uint64_t)1 << 32) / group) + 1; }
MOM_MX_FN uint32_t divided(uint32_t r, uint32_t inverse) { return inverse ? (uint32_t)(((uint64_t)r * inverse) >> 32) : r; }

// The tokens of the cache that the rows of a tile see: tokens [first, last] of the sequence's m new ones, n in the cache.  Token i stands at
// n - m + i, sees itself and what is before it, and not what is `window` or more before it (0: no window).
struct Span { int lo, hi; };                            // tokens [lo, hi)
MOM_MX_FN Span tile_span(int n, int m, int first, int last, int window) {
    const int p0 = n - m + first, p1 = n - m + last;                                 // p1 < n
    int lo = window > 0 ? p0 - window + 1 : 0, hi = p1 + 1;
    if (lo < 0) lo = 0;
    if (hi <= lo) return {0, 0};
    return {lo, hi};
}

// A step of a wavefront is kStep tokens at a multiple of it, and a share (one workgroup's part of a tile's tokens) `share` of them from the
// step that has the first visible token.
constexpr int kStep = 32;
MOM_MX_FN Span share_span(Span s, int z, int share) {
    const int base = s.lo / kStep * kStep, lo = base + z * share, hi = lo + share;
    const int a = lo > s.lo ? lo : s.lo, b = hi < s.hi ? hi : s.hi;
    if (b <= a) return {0, 0};
    return {a, b};
}

// Tokens that a tile can reach: the rows of `rows / group` tokens (and the two that a tile may cut), their window, and what lies in front of
// the first in its step.
MOM_MX_FN int64_t tile_reach(int64_t max_kv, int64_t window, int group, int rows) {
    if (window <= 0) return max_kv;
    const int64_t r = window + rows / group + 2 + kStep;
    return r < max_kv ? r : max_kv;
}

// How a call is launched: tiles of `rows` query rows, 16 qb for each wavefront; `wk` wavefronts have the same rows and share their tokens (1: each of
// kRowWaves has its own); the tokens of a tile in `shares` of `share`, which mx_join_kernel joins.
struct AttentionPlan {
    int qb, wk, rows, shares;
    int64_t share, numbers, tiles;      // numbers: of tiles of a key head at most; tiles: about as many there are, of all heads
};
// Wavefronts of a workgroup that have rows of their own, two a SIMD, and their blocks of 16: what their registers let them.
constexpr int kRowWaves = 8;
MOM_MX_FN constexpr int row_blocks(int D) { return D == 256 ? 1 : 2; }
MOM_MX_FN constexpr int tile_rows(int qb, int wk) { return 16 * qb * (wk > 1 ? 1 : kRowWaves); }

// Wavefronts that share a tile's tokens: as many as find their registers in half a compute unit (qb = 1 with 64 and 128 dimensions), or in all of it.
// Of qb = 1 four and sixteen each took longer: one sequence of 1024 tokens 9.0 us, 9.7 with four and 10.1 with sixteen, of 131072 37.2, 39.5 and 43.3, 32
// sequences of up to 8192 47.0, 63.0 and 54.1.
constexpr int kSharing = 8;
// Rows of a sequence up to which wavefronts share tokens, not rows (one sequence of 210 rows and 40000 tokens 36.0 us, 40.5 with rows of their own; 2 of 80
// and 9000 21.9 and 28.1), and of them at most 16 a workgroup if there are 256 dimensions (4 sequences of 32 rows and 5000 tokens 17.6 us, 22.1 with 32).
constexpr int kFewRows = 256;
MOM_MX_FN constexpr int few_blocks(int D) { return D == 256 ? 1 : 2; }
// Of qb = 1 with fewer than 256 dimensions four where there are so many tiles that each compute unit has several anyway, and few steps for each wavefront:
// 128 sequences of up to 512 tokens and 8 key heads 15.8 us, 20.1 with eight; of up to 2048 tokens 42.2 and 45.1; 96 sequences of 512 14.7 and 17.5.  Eight
// are ahead with fewer tiles (64 sequences of 512 11.9 us, 12.3 with four), longer reaches (128 of 8192 142 and 149) and 256 dimensions (95 and 102).
constexpr int kNarrow = 4, kManyTiles = 768, kNarrowReach = 2048;

// Shares of a tile of `reach` tokens and qb = 1, `tiles` workgroups without any; more for longer reaches, never fewer.  Joining costs a launch, so short reaches are
// one share: up to 768 tokens of up to 16 tiles (of 8 tiles 512 tokens take 6.8 us, 7.7 in 4 shares; 1024 tokens 9.0, and 8.0 in 8), and up to 1024, or more
// where there are many tiles, of others (64 tiles 9.5 us, 11.0 in 4).  Beyond, a workgroup for every one of 256 compute units, and two or eight shares' worth
// more where that is little: 64 tiles of 4096 tokens take 15.0 us in 8 shares and 17.4 in 4, 256 tiles of up to 8192 47.2 in 2 and 61.8 in 1; of 8 tiles
// 32768 tokens 15.5 in 32 and 17.1 in 64, 131072 37.1 in 64 and 40.9 in 32.  A share has 256 tokens, of few tiles' short reaches 128 (2048 tokens 8.4 us
// in 16 shares, 8.8 in 8).
constexpr int kComputeUnits = 256, kMostShares = 128, kFewTiles = 16;
MOM_MX_FN int64_t most_shares(int64_t reach, int64_t tiles) {
    if (tiles < 1) tiles = 1;
    if (reach <= (tiles <= kFewTiles ? 768 : 1024 * (tiles > 64 ? tiles / 64 : 1))) return 1;
    int64_t s = reach / 2048, least = kComputeUnits / tiles, most = 2 * kComputeUnits / tiles;
    if (least < 8) least = 8;
    if (s < least) s = least;
    if (s > most) s = most;
    int64_t whole = reach / 256;
    if (tiles <= kFewTiles && whole < 16) whole = reach / 128 < 16 ? reach / 128 : 16;
    if (s > whole) s = whole;
    if (s > kMostShares) s = kMostShares;
    return s < 1 ? 1 : s;
}
// Shares of the other tiles, of which a compute unit has one at a time: what the rounds of workgroups take, and what a share costs that is stored and
// joined, as much as 600 tokens' work: the fewest shares of which the sum is smallest, and so no fewer for longer reaches.  It is one whole round where
// that can be: 2048 tokens against 16384 with 256 tiles 499 us in one share, 540 in two, 562 in four; 512 against 32768 with 64 tiles 267 in four, 279 in
// eight, 509 in two; 4 sequences of 64 rows and 16384 tokens 35.2 in four, 42.6 in eight.
constexpr int64_t kShareCost = 600;
MOM_MX_FN int64_t round_shares(int64_t reach, int64_t tiles) {
    int64_t best = 1;
    if (tiles < 1) tiles = 1;
    const auto cost = [&](int64_t s) {                  // times tiles and s (54 bits)
        return (tiles * s + kComputeUnits - 1) / kComputeUnits * kComputeUnits * reach + (s > 1 ? kShareCost * s * s * tiles : 0);
    };
    for (int64_t s = 2; s <= kMostShares && s <= reach / 256 && tiles * s <= 8 * kComputeUnits; ++s)
        if (cost(s) * best < cost(best) * s) best = s;
    return best;
}

MOM_MX_FN int64_t plan_shares(const AttentionPlan& p, int64_t reach) { return p.wk > 1 && p.qb == 1 ? most_shares(reach, p.tiles) : round_shares(reach, p.tiles); }
// `listed`: sequences of their own lengths, whose last tiles are half full, say.
MOM_MX_FN AttentionPlan attention_plan(int64_t T, int64_t B, int Hq, int Hkv, int D, int64_t max_kv, int64_t window, bool listed) {
    const int group = Hq / Hkv;
    const int64_t average = (T * group + B - 1) / B;
    AttentionPlan p;
    p.wk = average > kFewRows ? 1 : kSharing;
    p.qb = average > kFewRows ? row_blocks(D) : average > 16 ? few_blocks(D) : 1;
    p.rows = tile_rows(p.qb, p.wk);
    const int64_t even = B * ((average + p.rows - 1) / p.rows), uneven = (2 * T * group + (B + 1) * p.rows - 1) / (2 * p.rows);
    p.tiles = (!listed ? even : uneven < B ? B : uneven) * Hkv;
    p.numbers = listed ? tile_numbers(T, B, group, p.rows) : even;
    const int64_t reach = tile_reach(max_kv, window, group, p.rows), s = plan_shares(p, reach);
    if (p.wk > 1 && p.qb == 1 && D < 256 && p.tiles >= kManyTiles && reach <= kNarrowReach) p.wk = kNarrow;
    p.share = ((reach + s - 1) / s + kStep - 1) / kStep * kStep;
    if (p.share < kStep) p.share = kStep;
    p.shares = reach > 0 ? (int)((reach + p.share - 1) / p.share) : 1;
    return p;
}
// Bytes of workspace: for every share of every row its sums, maximum and sum of weights.  A window or a shorter reach leaves fewer shares, never more; fewer
// tokens may be cut into more of them.
MOM_MX_FN size_t attention_workspace(int64_t T, int64_t B, int Hq, int Hkv, int D, int64_t max_kv) {
    const int64_t even = plan_shares(attention_plan(T, B, Hq, Hkv, D, max_kv, 0, false), max_kv), uneven = plan_shares(attention_plan(T, B, Hq, Hkv, D, max_kv, 0, true), max_kv);
    const int64_t s = even > uneven ? even : uneven;
    return s <= 1 ? 0 : (size_t)s * (size_t)T * (size_t)Hq * (size_t)(D + 2) * 4;
}

}  // namespace mx
}  // namespace momk

#endif
