// Which kernel a product with 8-bit weights takes: a function of sizes, digits and alignment alone.  Host code without HIP, which a test compiles by
// itself to see that its shapes reach every kernel.
#pragma once
#include <stddef.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace {

constexpr int64_t kI8Step = 256;   // columns that a row is padded to: up to four waves share a step of 64 each

constexpr int64_t i8_row_bytes(int64_t cols) { return (cols + kI8Step - 1) / kI8Step * kI8Step; }
constexpr int64_t i8_pieces(int64_t cols) { return (cols + 63) / 64; }   // of 64 columns, up to the last that has some

// Few rows of a long contraction: behind them lies room for the counters and the partial sums of kI8SplitTiles workgroups of up to 64 x 64 sums
// (a counter for each of the up to two waves that a tile's sums end in: only tiles that two workgroups or more share have them).
constexpr int64_t kI8SplitColumns = 2048, kI8SplitRows = 512, kI8SplitTiles = 256;
inline bool i8_splits(int64_t T, int64_t cols, int digits) { return i8_row_bytes(cols) >= kI8SplitColumns && T * digits <= kI8SplitRows; }

// The tiles and their times on a compute unit, in nanoseconds: a step of 64 columns alone on a chip with few workgroups (waiting; 1.4 times that where the
// weights are read once or come from memory), the same as a share of a chip that is full (throughput; small tiles run side by side on a unit), and what comes around
// the steps, filling and results.  Fitted to some forty shapes.  On 200 others (5 to 16384 rows, 64 to 13824 columns, one and two digits, gated or not, half of
// them with weights that no cache holds), every tile timed with a shared contraction and without: the way with the least sum was the fastest on 140, within 5 % of it
// on 160, within 15 % on 187, and 35 % behind at worst (389 x 67 x 5734 gated 14.7 us instead of 10.9 with 128 x 128 tiles, 3575 x 7716 -> 348 54 instead
// of 41 with 64 x 64); 2.8 % behind in the mean.
struct TileCost {
    int channels, tokens;
    double alone, share, fixed;
};
constexpr TileCost kTiles[7] = {{256, 256, 600, 800, 7000}, {256, 128, 390, 510, 3400}, {128, 128, 200, 300, 1100}, {64, 64, 77, 125, 600},
                                {32, 64, 55, 80, 400},      {32, 32, 35, 60, 300},      {32, 16, 25, 50, 300}};
constexpr TileCost kGatedTiles[7] = {{256, 256, 600, 800, 18000}, {256, 128, 390, 510, 9500}, {128, 128, 200, 300, 5000}, {64, 64, 77, 125, 1500},
                                     {64, 32, 60, 105, 1000},     {64, 32, 60, 105, 1000},    {64, 16, 40, 100, 600}};   // (64 x 32 stands for both small plain ones)

// Few small tiles of a long contraction: several workgroups share a tile's steps, which costs them kJoin ns to join (the product of 4 x 25742 -> 83 in two
// digits 15.8 -> 6.4 us).
constexpr double kJoin = 6000;
struct Choice {
    int tile;
    uint32_t splits;
};
inline Choice cheapest_tile(const TileCost (&tiles)[7], int64_t channels, int64_t rows, bool two_digits, int pieces, bool may_split) {
    Choice best = {0, 1};
    double least = 0;
    const double steps = pieces;
    const bool from_memory = channels * pieces * 64 > (24 << 20);   // (weights that the caches of the XCDs do not hold)
    for (int i = 0; i < (two_digits ? 6 : 7); ++i) {   // (two digits are two blocks of 16 rows)
        const int64_t across = (rows + tiles[i].tokens - 1) / tiles[i].tokens;
        const double n = static_cast<double>((channels + tiles[i].channels - 1) / tiles[i].channels) * static_cast<double>(across);
        const double alone = across == 1 || from_memory ? 1.4 * tiles[i].alone : tiles[i].alone;
        const double rounds = n <= 256 ? n / 256 : std::ceil(n / 256);   // (256 compute units)
        const double cost = std::max(alone, rounds * tiles[i].share) * steps + std::max(1., rounds) * tiles[i].fixed;
        if (i == 0 || cost < least) best = {i, 1}, least = cost;
        if (i < 3 || !may_split) continue;
        const uint32_t splits = static_cast<uint32_t>(std::min({kI8SplitTiles / n, steps / 8, 16.}));
        if (splits < 2) continue;
        const double shared = std::max(alone, n * splits / 256 * tiles[i].share) * steps / splits + tiles[i].fixed + kJoin;
        if (shared < least) best = {i, splits}, least = shared;
    }
    return best;
}

// The tile of T rows in `digits` digits with n outputs (of a gate and an up projection each) over `cols` columns.  room: for a shared contraction's sums
inline Choice i8_choice(int64_t T, int64_t cols, int64_t n, int digits, bool gated, bool room = true) {
    return cheapest_tile(gated ? kGatedTiles : kTiles, (gated ? 2 : 1) * n, digits * T, digits == 2, static_cast<int>(i8_pieces(cols)),
                         room && i8_splits(T, cols, digits));
}

constexpr size_t kLdsBytes = 160 * 1024;   // of a compute unit

// LDS that rows made by the product's workgroups take behind the ring: x, rows of whole KiB; their 8-bit rows; room for scales and partial maxima.
constexpr int64_t own_x_bytes(int64_t d_in) { return (d_in * 2 + 1023) / 1024 * 1024; }
constexpr int64_t own_bytes(int64_t T, int64_t d_in, int64_t ld) { return T * (own_x_bytes(d_in) + ld) + 64 * 4 * 2; }

// Whether the product's workgroups bring the rows to digits themselves: one launch instead of two, but every workgroup does the whole of it.  Times of a
// call in us, with the row kernel -> without, T x d_in -> d_out: 1 x 4096 -> 4096 7.9 -> 5.8, 1 x 4096 -> 11008 12.2 -> 8.9, 1 x 11008 -> 4096 13.2 -> 11.7,
// 2 x 4096 -> 4096 8.0 -> 6.8, 2 x 11008 -> 4096 13.1 -> 13.6, 4 x 1000 -> 1024 8.2 -> 5.9, 4 x 4096 -> 11008 12.4 -> 17.8, 16 x 512 -> 512 8.5 -> 12.9 (tokens are
// taken one after the other); gated, 1 x 4096 x 11008 19.6 -> 17.2, 2 x 4096 x 11008 19.4 -> 21.9.
// Rows read through registers cost more: 1 x 126 -> 292 8.5 -> 5.1, 1 x 566 x 286 gated 8.4 -> 5.4, but 2 x 4095 -> 4096 8.5 either way, 1 x 13823 -> 4096 13.9 -> 15.0,
// 4 x 1001 -> 1024 7.8 -> 8.3.
// 0: the row kernel makes them.  1: the workgroups do, from rows of whole 16-byte pieces (`aligned`: x starts on one); 2: from any rows.
inline int i8_own_rows(int64_t T, int64_t d_in, int digits, bool gated, bool aligned) {
    const bool pieces = d_in % 8 == 0 && aligned;
    const int64_t most = pieces ? (gated ? 6144 : 14336) : (gated ? 2048 : 4096);
    const bool fits = digits == 1 && T <= (pieces ? 4 : 2) && T * d_in <= most &&
                      static_cast<size_t>(own_bytes(T, d_in, i8_row_bytes(d_in))) + 4 * 4 * (gated ? 64 : 32) * 64 <= kLdsBytes;
    return fits ? (pieces ? 1 : 2) : 0;
}

}  // namespace
