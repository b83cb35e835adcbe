// Which kernel a product with 4-bit weights takes: a function of sizes and alignment alone.  Host code without HIP, which a test compiles by itself to see that
// its shapes reach every kernel and to know which of them take the weights as they are.
#pragma once
#include <stdint.h>

#include <algorithm>
#include <cmath>

namespace {

// The tiles, and their times in microseconds: a step of `parts` blocks of 128 columns where the chip has room for more workgroups, the same as a share of a
// full compute unit, and what comes around the steps of each round of workgroups.  (A step of the small tiles takes its microsecond for bringing the codes to fp16,
// not for waiting: read two or three steps ahead it took as long.)  Fitted to every kernel's times on 318 calls of 9 to 2000 tokens, 512 to 11008 columns and 512 to
// 32000 outputs, with and without zeros: there the pick is behind the best by 0.9 % in the mean and 19 % at worst.
// The 64 x 64 tile brings each code to fp16 once where the 64 x 32 one does twice for 33 to 64 tokens, by eight waves of which each has half of the channels
// (64 x 4096 -> 11008 19 -> 15 us, 33 x 5120 -> 13824 22.9 -> 19.8; on 15 of 117 forward shapes 3 to 25 % ahead of all others, never in the gradient: 36 against 23).
enum I4Kernel { kI4Few = 0, kI4Tile32 = 1, kI4Tile64 = 2, kI4Tile128 = 3, kI4Tile256 = 4, kI4Square64 = 5 };
struct I4Tile {
    int channels, tokens, parts, resident;   // resident: workgroups that a compute unit holds at a time
    double alone, share, fixed;
};
constexpr I4Tile kI4Tiles[6] = {{32, 16, 8, 2, 1.1, 1.67, 2.17},     // kernel for few tokens: the weights as they are, forward
                                {32, 32, 8, 1, 1.02, 1.44, 2.93},    // (gated: 64 channels)
                                {64, 32, 4, 2, 0.94, 1.02, 2.7},
                                {128, 64, 2, 2, 1.13, 1.3, 2.37},
                                {256, 128, 1, 2, 1.46, 2.44, 3.09},
                                {64, 64, 4, 1, 1.1, 1.43, 3.02}};    // forward, one matrix, aligned rows
constexpr I4Tile kI4FewGradient = {32, 16, 8, 2, 1.5, 2.89, 1.0};    // (a scale and a zero for every code)
// The same for rows that no request takes whole, which come through registers (219 calls, 0.5 % and 17 %).  The largest tile's registers do not hold those
// as well as the scales and zeros of groups of 32 along a row (2000 x 11003 -> 4096 380 us, 128 x 64 tiles 284; without zeros 234 and 262).
// Eleven of the largest tile's other forms keep 1 to 16 registers in memory, the aligned ones of groups of 32 with zeros among them, and are counted like the rest.
constexpr I4Tile kI4Unaligned[5] = {{32, 16, 8, 2, 0.24, 3.27, 2.92}, {32, 32, 8, 1, 2.02, 2.14, 5.23}, {64, 32, 4, 2, 1.47, 1.65, 3.57}, {128, 64, 2, 2, 1.74, 1.55, 4.75},
                                    {256, 128, 1, 2, 2.11, 3.0, 4.73}};
constexpr I4Tile kI4UnalignedFewGradient = {32, 16, 8, 2, 0.84, 4.2, 3.44};
constexpr double kI4Launch = 2.5;

constexpr int64_t kI4MostColumns = 1 << 22;   // of a plane: a tile's rows span less than 4 GiB
constexpr int64_t kI4FewTokens = 8;           // up to here a tile's other tokens would be none

inline double i4_cost(const I4Tile& t, int64_t channels, int64_t T, int64_t blocks) {
    const double n = static_cast<double>((channels + t.channels - 1) / t.channels) * static_cast<double>((T + t.tokens - 1) / t.tokens);
    const double rounds = std::ceil(n / (256. * t.resident)), steps = static_cast<double>((blocks + t.parts - 1) / t.parts);
    return kI4Launch + t.fixed * rounds + steps * std::max(t.alone * rounds, n / 256 * t.share);
}

// T tokens, k columns of a plane of the contraction, `blocks` of 128 columns in all, n outputs; aligned: rows of whole 16-byte pieces; fine_zeros: zeros, groups of 32
inline I4Kernel i4_kernel(int64_t T, int64_t k, int64_t blocks, int64_t n, bool gated, bool aligned, bool backward, bool fine_zeros) {
    if (T <= kI4FewTokens || k < 8 || k > kI4MostColumns) return kI4Few;
    const int64_t channels = gated ? 2 * n : n;
    I4Kernel best = kI4Few;
    double least = i4_cost(backward ? (aligned ? kI4FewGradient : kI4UnalignedFewGradient) : (aligned ? kI4Tiles : kI4Unaligned)[kI4Few], channels, T, blocks);
    const int tiles = gated || backward || !aligned ? kI4Square64 : kI4Square64 + 1;
    for (int i = 1; i < tiles; ++i) {
        if (i == kI4Tile256 && !aligned && !backward && fine_zeros) continue;
        I4Tile t = (aligned ? kI4Tiles : kI4Unaligned)[i];
        if (gated && i == kI4Tile32) t.channels = 64, t.share *= 2;
        const double cost = i4_cost(t, channels, T, blocks);
        if (cost < least) best = static_cast<I4Kernel>(i), least = cost;
    }
    return best;
}

}  // namespace
