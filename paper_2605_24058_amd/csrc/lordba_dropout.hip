// Dropout whose mask is a function of the element's index: Philox4x32-10 (J. Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011)
// with the counter (index / 8, offset) and the seed as the key gives 128 bits for eight elements, 16 for each.  Nothing but the tensor moves: the
// backward pass draws the same bits again.
#include <algorithm>
#include <cmath>

#include "lordba_dev_util.h"
#include "lordba_i8.h"

namespace {

struct DropoutArgs {
    const _Float16* x;
    const _Float16* y_base;   // or null
    _Float16* y;
    const uint64_t* offset_dev;   // or null
    uint64_t seed, offset;
    int64_t n;
    int64_t first;   // group of eight elements of this launch's first thread
    uint32_t least;   // what is kept has draws from here on: 0 .. 65536
    float factor;
};

__device__ __forceinline__ u4 philox(uint64_t group, uint64_t offset, uint64_t seed) {
    uint32_t c0 = static_cast<uint32_t>(group), c1 = static_cast<uint32_t>(group >> 32), c2 = static_cast<uint32_t>(offset),
             c3 = static_cast<uint32_t>(offset >> 32), k0 = static_cast<uint32_t>(seed), k1 = static_cast<uint32_t>(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t a = static_cast<uint64_t>(c0) * 0xD2511F53u, b = static_cast<uint64_t>(c2) * 0xCD9E8D57u;
        c0 = static_cast<uint32_t>(b >> 32) ^ c1 ^ k0;
        c1 = static_cast<uint32_t>(b);
        c2 = static_cast<uint32_t>(a >> 32) ^ c3 ^ k1;
        c3 = static_cast<uint32_t>(a);
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u4{c0, c1, c2, c3};
}

template <bool BASE>
__global__ __launch_bounds__(256) void lordba_dropout_kernel(DropoutArgs a) {
    const int64_t group = a.first + static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x, i = 8 * group;
    if (i >= a.n) return;
    const u4 r = philox(static_cast<uint64_t>(group), a.offset + (a.offset_dev ? *a.offset_dev : 0), a.seed);
    const bool whole = i + 8 <= a.n;
    u4 xv = {0u, 0u, 0u, 0u}, bv = {0u, 0u, 0u, 0u};
    if (whole) {
        xv = load16_any_stream(a.x + i);
        if constexpr (BASE) bv = load16_any_stream(a.y_base + i);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < a.n) {
                xv[e >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(a.x)[i + e]) << (16 * (e & 1));
                if constexpr (BASE) bv[e >> 1] |= static_cast<uint32_t>(reinterpret_cast<const uint16_t*>(a.y_base)[i + e]) << (16 * (e & 1));
            }
    }
    const h8 x = as_h8(xv), b = as_h8(bv);
    h8 y;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const uint32_t draw = (r[e >> 1] >> (16 * (e & 1))) & 0xFFFFu;
        float v = draw >= a.least ? static_cast<float>(x[e]) * a.factor : 0.f;   // (chosen, not multiplied: what is dropped may be anything)
        if constexpr (BASE) v += static_cast<float>(b[e]);
        y[e] = static_cast<_Float16>(v);
    }
    const u4 yv = __builtin_bit_cast(u4, y);
    if (whole) {
        store16_any_stream(a.y + i, yv);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (i + e < a.n) reinterpret_cast<uint16_t*>(a.y)[i + e] = static_cast<uint16_t>(yv[e >> 1] >> (16 * (e & 1)));
    }
}

}  // namespace

extern "C" lordba_status lordba_dropout(const void* x, const void* y_base, void* y_out, int64_t n, double p, uint64_t seed, uint64_t offset,
                                        const uint64_t* offset_dev, void* stream) {
    if (n < 0 || n > (static_cast<int64_t>(1) << 38)) return LORDBA_ERR_DIM;
    if (!(p >= 0. && p <= 1.)) return LORDBA_ERR_VALUE;
    if (n == 0) return LORDBA_OK;
    if (!x || !y_out) return LORDBA_ERR_NULL;
    if (i8_misaligned(x, 2) || i8_misaligned(y_base, 2) || i8_misaligned(y_out, 2) || i8_misaligned(offset_dev, 8)) return LORDBA_ERR_ALIGN;
    const size_t bytes = static_cast<size_t>(n) * 2;
    if ((y_out != x && i8_overlap(y_out, bytes, x, bytes)) || (y_out != y_base && i8_overlap(y_out, bytes, y_base, bytes)) ||
        i8_overlap(y_out, bytes, offset_dev, 8))
        return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const uint32_t least = static_cast<uint32_t>(nearbyint(p * 65536.));
    DropoutArgs a = {static_cast<const _Float16*>(x), static_cast<const _Float16*>(y_base), static_cast<_Float16*>(y_out), offset_dev,
                           seed, offset, n, 0, least, least < 65536 ? 65536.f / static_cast<float>(65536 - least) : 0.f};
    const int64_t groups = (n + 7) / 8, most = static_cast<int64_t>(1) << 31;   // (a launch counts threads in 32 bits)
    for (a.first = 0; a.first < groups; a.first += most) {
        const dim3 grid(static_cast<unsigned>((std::min(most, groups - a.first) + 255) / 256));
        if (y_base) hipLaunchKernelGGL(lordba_dropout_kernel<true>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
        else hipLaunchKernelGGL(lordba_dropout_kernel<false>, grid, dim3(256), 0, static_cast<hipStream_t>(stream), a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}
