// Products with 4-bit weights, few tokens: what bounds them is reading the weights.
#include <algorithm>

#include "lordba_i4_product.h"

namespace {

// A workgroup owns CB blocks of 16 weight rows (gated: half of them gate's, half up's) and TB blocks of 16 tokens; its NW waves share the contraction, wave
// w taking the blocks of 128 columns w, w + NW, ...  Operands come straight into registers, one block ahead of the products, and the waves' sums are joined
// through LDS in the waves' order.
// Forward (S > 0 scales along a block of 128 columns): the products run on the whole numbers code - zero, which fp16 holds exactly, and a group's sum is
// multiplied by its scale in fp32, so that nothing is rounded but the sums.  Backward (S = 0): the scales vary along the contraction, so each weight is rounded
// to fp16 before its product (half a step, 2^-11 of the weight).
template <int CB, int TB, int NW, int S, bool ZERO, bool GATED>
__global__ __launch_bounds__(64 * NW) void lordba_i4_few_kernel(I4Args a) {
    constexpr bool BWD = S == 0;
    constexpr int P = GATED ? 2 : 1, CT = CB / P;   // blocks of a half
    static_assert(CB % P == 0 && !(GATED && BWD), "");
    extern __shared__ f4 sums[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int across = (a.tiles + CT - 1) / CT;
    const uint32_t id = a.first + blockIdx.x;
    const int tile0 = static_cast<int>(id % across) * CT;
    const int64_t t0 = static_cast<int64_t>(id / across) * (16 * TB);

    const u4* code[CB];
    const uint16_t *scale[CB], *zero[CB];
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        const int64_t tile = min(tile0 + i % CT, a.tiles - 1) + (i / CT) * a.tiles;
        code[i] = reinterpret_cast<const u4*>(a.codes) + tile * a.blocks * 64 + lane;
        const int64_t at = BWD ? (i4_row(tile, 0) >> a.shift) * a.blocks * kI4Columns + 8 * q : tile * a.groups * 16;
        scale[i] = a.scale + at + (BWD ? 0 : 4 * q);
        zero[i] = ZERO ? a.zero + at + (BWD ? 0 : r) : nullptr;
    }
    const _Float16* row[TB];
#pragma unroll
    for (int j = 0; j < TB; ++j) row[j] = a.x + min(t0 + 16 * j + r, a.T - 1) * a.k;

    constexpr int kScales = BWD ? 4 : S;
    struct Block {
        u4 c[CB], x[TB][4];
        u4 s8[BWD ? CB : 1][4], z8[BWD && ZERO ? CB : 1][4];
        uint2 s4[BWD ? 1 : CB][kScales];
        uint16_t z1[!BWD && ZERO ? CB : 1][kScales];
    };
    auto load = [&](int b, Block& v) {
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            v.c[i] = code[i][static_cast<int64_t>(b) * 64];
            if constexpr (BWD) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    v.s8[i][m] = load16(scale[i] + static_cast<int64_t>(b) * kI4Columns + 32 * m);
                    if constexpr (ZERO) v.z8[i][m] = load16(zero[i] + static_cast<int64_t>(b) * kI4Columns + 32 * m);
                }
            } else {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    v.s4[i][s] = *reinterpret_cast<const uint2*>(scale[i] + (static_cast<int64_t>(b) * S + s) * 16);
                    if constexpr (ZERO) v.z1[i][s] = zero[i][(static_cast<int64_t>(b) * S + s) * 16];
                }
            }
        }
        const int plane = b >= a.plane_blocks ? 1 : 0;
        const int64_t c0 = static_cast<int64_t>(b - plane * a.plane_blocks) * kI4Columns + 8 * q, off = plane * a.T * a.k;
        if (c0 - 8 * q + kI4Columns <= a.k) {
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int m = 0; m < 4; ++m) v.x[j][m] = load16_any(row[j] + off + c0 + 32 * m);
        } else {
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int m = 0; m < 4; ++m) v.x[j][m] = load_part(row[j] + off, c0 + 32 * m, a.k);
        }
    };
    f4 acc[CB][TB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const Block& v) {
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            if constexpr (BWD) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    h8 w;
                    if constexpr (ZERO) w = operand(v.c[i][m], Zero8{v.z8[i][m]});
                    else w = operand(v.c[i][m], Zero1(kZero8));
                    w = w * as_h8(v.s8[i][m]);
#pragma unroll
                    for (int j = 0; j < TB; ++j) acc[i][j] = mfma(w, as_h8(v.x[j][m]), acc[i][j]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    f4 part[TB];
#pragma unroll
                    for (int j = 0; j < TB; ++j) part[j] = f4{0.f, 0.f, 0.f, 0.f};
                    const Zero1 z(ZERO ? v.z1[i][s] : kZero8);
#pragma unroll
                    for (int m = s * (4 / S); m < (s + 1) * (4 / S); ++m) {
                        const h8 w = operand(v.c[i][m], z);
#pragma unroll
                        for (int j = 0; j < TB; ++j) part[j] = mfma(w, as_h8(v.x[j][m]), part[j]);
                    }
                    const h2 s01 = as_h2(v.s4[i][s].x), s23 = as_h2(v.s4[i][s].y);
                    const f4 f = {static_cast<float>(s01[0]), static_cast<float>(s01[1]), static_cast<float>(s23[0]), static_cast<float>(s23[1])};
#pragma unroll
                    for (int j = 0; j < TB; ++j)
#pragma unroll
                        for (int e = 0; e < 4; ++e) acc[i][j][e] = fmaf(f[e], part[j][e], acc[i][j][e]);
                }
            }
        }
    };
    int b = wave;
    if (b < a.blocks) {
        Block now;
        load(b, now);
        while (b + NW < a.blocks) {
            Block next;
            load(b + NW, next);
            multiply(now);
            now = next;
            b += NW;
        }
        multiply(now);
    }
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) sums[(wave * CB * TB + i * TB + j) * 64 + lane] = acc[i][j];
    __syncthreads();
    // Four columns of a token a thread.
    for (int o = threadIdx.x; o < CT * TB * 64; o += 64 * NW) {
        f4 v[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            v[p] = sums[p * CT * TB * 64 + o];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[p] += sums[w * CB * TB * 64 + p * CT * TB * 64 + o];
        }
        const int i = o / (TB * 64), j = o / 64 % TB, l = o & 63;
        const int64_t t = t0 + 16 * j + (l & 15), c = i4_row(tile0 + i, 4 * (l >> 4));
        if (tile0 + i >= a.tiles || t >= a.T) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= a.n) break;
            const int64_t at = t * a.n + c + e, plane = a.T * a.n;
            if constexpr (GATED) {
                float g = v[0][e], u = v[1][e];
                if (a.addends) g += static_cast<float>(a.addends[at]), u += static_cast<float>(a.addends[plane + at]);
                if (a.kept) {
                    a.kept[at] = kept_half(g);
                    a.kept[plane + at] = kept_half(u);
                }
                a.y[at] = static_cast<_Float16>(silu(g) * u);
            } else {
                a.y[at] = static_cast<_Float16>(v[0][e]);
            }
        }
    }
}

template <int CB, int TB, int NW, int S, bool ZERO, bool GATED>
lordba_status few_launch(I4Args a, hipStream_t stream) {
    constexpr size_t kLds = static_cast<size_t>(CB) * TB * NW * 1024;
    static_assert(kLds <= 64 * 1024, "LDS that a launch gets unasked");
    const int64_t across = (a.tiles + CB / (GATED ? 2 : 1) - 1) / (CB / (GATED ? 2 : 1)), n = across * ((a.T + 16 * TB - 1) / (16 * TB));
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / (64 * NW);   // (a launch counts threads in 32 bits)
    if (n > INT32_MAX) return LORDBA_ERR_DIM;
    for (int64_t first = 0; first < n; first += kMost) {
        a.first = static_cast<uint32_t>(first);
        hipLaunchKernelGGL((lordba_i4_few_kernel<CB, TB, NW, S, ZERO, GATED>), dim3(static_cast<unsigned>(std::min(kMost, n - first))), dim3(64 * NW), kLds,
                           stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

template <int S, bool ZERO, bool GATED>
lordba_status few(const I4Args& a, hipStream_t stream) {
    constexpr int P = GATED ? 2 : 1;
    if (a.T <= 16) return few_launch<P, 1, 16, S, ZERO, GATED>(a, stream);
    if (a.T <= 32) return few_launch<2, 2, 8, S, ZERO, GATED>(a, stream);
    return few_launch<2, 4, 8, S, ZERO, GATED>(a, stream);
}
template <int S, bool GATED>
lordba_status few(const I4Args& a, hipStream_t stream) {
    return a.zero ? few<S, true, GATED>(a, stream) : few<S, false, GATED>(a, stream);
}
template <bool GATED>
lordba_status few(const I4Args& a, int64_t group, hipStream_t stream) {
    return group == 32 ? few<4, GATED>(a, stream) : group == 64 ? few<2, GATED>(a, stream) : few<1, GATED>(a, stream);
}

}  // namespace

lordba_status lordba_i4_few(const I4Args& a, int64_t group, bool gated, bool backward, hipStream_t stream) {
    if (backward) return few<0, false>(a, stream);
    return gated ? few<true>(a, group, stream) : few<false>(a, group, stream);
}
