// Which kernel a product with 4-bit weights takes: a function of sizes and alignment alone.  Host code without HIP, which a test compiles by itself to see that
// its shapes reach every kernel and to know which of them take the weights as they are.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace {

// The tiles, and their times in microseconds: a step of `parts` blocks of 128 columns where the chip has room for more workgroups (waiting for memory), the same as a
// share of a full compute unit, and what comes around the steps.  Fitted to 17 .. 2048 tokens of 4096 -> 4096, 4096 -> 11008, 11008 -> 4096 and 1000 -> 1000; of the five
// ways the one with the least sum was the fastest on all but three of those 30, and there 5 .. 15 % behind.
enum I4Kernel { kI4Few = 0, kI4Tile32 = 1, kI4Tile64 = 2, kI4Tile128 = 3, kI4Tile256 = 4 };
struct I4Tile {
    int channels, tokens, parts, resident;   // resident: workgroups that a compute unit holds at a time
    double alone, share, fixed;
};
constexpr I4Tile kI4Tiles[5] = {{32, 16, 8, 2, 1.6, 1.7, 3.0},     // kernel for few tokens: the weights as they are, forward
                                {32, 32, 8, 1, 1.6, 2.0, 3.0},     // (gated: 64 channels)
                                {64, 32, 4, 2, 1.1, 1.05, 2.5},
                                {128, 64, 2, 2, 1.15, 1.2, 2.5},
                                {256, 128, 1, 2, 1.3, 1.9, 3.0}};
// The same for rows that no request takes whole, which come through registers.  (The second waits longer than the third: nothing chooses it.)
constexpr I4Tile kI4Unaligned[5] = {{32, 16, 8, 2, 2.0, 2.0, 3.0}, {32, 32, 8, 1, 3.4, 3.4, 3.0}, {64, 32, 4, 2, 1.8, 1.3, 2.5}, {128, 64, 2, 2, 1.75, 1.57, 2.5},
                                    {256, 128, 1, 2, 1.8, 2.5, 3.0}};

constexpr int64_t kI4MostColumns = 1 << 22;   // of a plane: a tile's rows span less than 4 GiB
constexpr int64_t kI4FewTokens = 8;           // up to here a tile's other tokens would be none

inline double i4_cost(const I4Tile& t, int64_t channels, int64_t T, int64_t blocks) {
    const double n = static_cast<double>((channels + t.channels - 1) / t.channels) * static_cast<double>((T + t.tokens - 1) / t.tokens);
    const double rounds = std::ceil(n / (256. * t.resident)), steps = static_cast<double>((blocks + t.parts - 1) / t.parts);
    return t.fixed * rounds + steps * std::max(t.alone * rounds, n / 256 * t.share);
}

// T tokens, k columns of a plane of the contraction, `blocks` of 128 columns in all, n outputs; aligned: rows of whole 16-byte pieces
inline I4Kernel i4_kernel(int64_t T, int64_t k, int64_t blocks, int64_t n, bool gated, bool aligned) {
    if (T <= kI4FewTokens || k < 8 || k > kI4MostColumns) return kI4Few;
    const int64_t channels = gated ? 2 * n : n;
    I4Kernel best = kI4Few;
    double least = i4_cost((aligned ? kI4Tiles : kI4Unaligned)[0], channels, T, blocks);
    for (int i = 1; i < 5; ++i) {
        if (!aligned && i == kI4Tile32) continue;
        I4Tile t = (aligned ? kI4Tiles : kI4Unaligned)[i];
        if (gated && i == kI4Tile32) t.channels = 64, t.share *= 1.3;
        const double cost = i4_cost(t, channels, T, blocks);
        if (cost < least) best = static_cast<I4Kernel>(i), least = cost;
    }
    return best;
}

}  // namespace
