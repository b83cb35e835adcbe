// Products with 4-bit weights, few tokens: what bounds them is reading the weights.
#include <algorithm>

#include "lordba_i4_product.h"

namespace {

// What a workgroup of NW waves keeps of the activations: two of eight waves, or four of four, run on a compute unit side by side.
constexpr int64_t few_lds(int NW) { return NW == 4 ? 32 * 1024 : 64 * 1024; }

// A workgroup owns CB blocks of 16 weight rows (gated: half of them gate's, half up's) and up to 16 tokens; its NW waves share the contraction, wave w
// taking the blocks of 128 columns w, w + NW, ...  The activations are kept in LDS, as many columns of them at a time as fit (`columns`, a multiple of 128),
// rows in 16-byte pieces of which piece p of row t lies at place p ^ t of its sixteen.  So the only requests that are on their way in the
// loop are the weights', D blocks ahead, and what the call waits for is a latency of memory or two.  The waves' sums are joined through LDS in the waves' order.
// Forward (S > 0 scales along a block of 128 columns): the products run on the whole numbers code - zero, which fp16 holds exactly, and a group's sum is
// multiplied by its scale in fp32, so that nothing is rounded but the sums.  Backward (S = 0): the scales vary along the contraction, so each weight is rounded
// to fp16 before its product (half a step, 2^-11 of the weight).
template <int CB, int NW, int D, int S, bool ZERO, bool GATED>
__global__ __launch_bounds__(64 * NW, NW <= 8 ? 4 : 1) void lordba_i4_few_kernel(I4Args a) {
    constexpr bool BWD = S == 0;
    constexpr int P = GATED ? 2 : 1, CT = CB / P;   // blocks of a half
    static_assert(CB % P == 0 && CT <= 2 && !(GATED && BWD), "a half's blocks lie in one pair: one group's rows in the transposed layout");
    extern __shared__ int8_t lds[];
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int across = (a.tiles + CT - 1) / CT;
    const uint32_t id = a.first + blockIdx.x;
    const int tile0 = static_cast<int>(id % across) * CT;
    const int64_t t0 = static_cast<int64_t>(id / across) * 16;
    const int tokens = static_cast<int>(min<int64_t>(16, a.T - t0));

    const u4* code[CB];
    const uint16_t *scale[CB], *zero[CB];   // (backward: the first serves all)
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        const int64_t tile = tile0 + i % CT + (i / CT) * a.tiles;
        code[i] = reinterpret_cast<const u4*>(a.codes) + tile * a.blocks * 64 + lane;
        const int64_t at = BWD ? (i4_row(tile, 0) >> a.shift) * a.blocks * kI4Columns + 8 * q : tile * a.groups * 16;
        scale[i] = a.scale + at + (BWD ? 0 : 4 * q);
        zero[i] = ZERO ? a.zero + at + (BWD ? 0 : r) : nullptr;
    }
    struct Block {
        u4 c[CB], s8[BWD ? 4 : 1], z8[BWD && ZERO ? 4 : 1];
        uint2 s4[BWD ? 1 : CB][BWD ? 1 : S];
        uint16_t z1[!BWD && ZERO ? CB : 1][BWD ? 1 : S];
    };
    auto load = [&](int64_t b, Block& v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CB; ++i) v.c[i] = code[i][b * 64];
        if constexpr (BWD) {
#pragma unroll
            for (int m = 0; m < 4; ++m) {
                v.s8[m] = load16(scale[0] + b * kI4Columns + 32 * m);
                if constexpr (ZERO) v.z8[m] = load16(zero[0] + b * kI4Columns + 32 * m);
            }
        } else {
#pragma unroll
            for (int i = 0; i < CB; ++i)
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    v.s4[i][s] = *reinterpret_cast<const uint2*>(scale[i] + (b * S + s) * 16);
                    if constexpr (ZERO) v.z1[i][s] = zero[i][(b * S + s) * 16];
                }
        }
    };
    f4 acc[CB];
#pragma unroll
    for (int i = 0; i < CB; ++i) acc[i] = f4{0.f, 0.f, 0.f, 0.f};
    const uint32_t exp = exponent();
    const int8_t* const mine = lds + min(r, tokens - 1) * (a.columns * 2);
    const int turn = min(r, tokens - 1);
    auto multiply = [&](int b, const Block& v) __attribute__((always_inline)) {   // b: of those in LDS
        h8 x[4];
#pragma unroll
        for (int m = 0; m < 4; ++m) x[m] = as_h8(*reinterpret_cast<const u4*>(mine + b * 256 + 16 * ((4 * m + q) ^ turn)));
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            if constexpr (BWD) {
#pragma unroll
                for (int m = 0; m < 4; ++m) {
                    h8 w;
                    if constexpr (ZERO) w = operand(v.c[i][m], Zero8{v.z8[m]}, exp);
                    else w = operand(v.c[i][m], Zero1(kZero8), exp);
                    acc[i] = mfma(w * as_h8(v.s8[m]), x[m], acc[i]);
                }
            } else {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    f4 part = {0.f, 0.f, 0.f, 0.f};
                    const Zero1 z(ZERO ? v.z1[i][s] : kZero8);
#pragma unroll
                    for (int m = s * (4 / S); m < (s + 1) * (4 / S); ++m) part = mfma(operand(v.c[i][m], z, exp), x[m], part);
                    const h2 s01 = as_h2(v.s4[i][s].x), s23 = as_h2(v.s4[i][s].y);
                    acc[i][0] = fmaf(static_cast<float>(s01[0]), part[0], acc[i][0]);
                    acc[i][1] = fmaf(static_cast<float>(s01[1]), part[1], acc[i][1]);
                    acc[i][2] = fmaf(static_cast<float>(s23[0]), part[2], acc[i][2]);
                    acc[i][3] = fmaf(static_cast<float>(s23[1]), part[3], acc[i][3]);
                }
            }
        }
    };
    const int there = a.columns / static_cast<int>(kI4Columns);   // blocks that LDS holds
    for (int b0 = 0; b0 < a.blocks; b0 += there) {
        const int blocks = min(there, a.blocks - b0), n = (blocks - wave + NW - 1) / NW;   // in LDS; of this wave
        auto at = [&](int k) { return static_cast<int64_t>(b0 + min(wave + k * NW, blocks - 1)); };   // (behind a wave's last block the last there is)
        Block ring[D];
#pragma unroll
        for (int j = 0; j < D; ++j) load(at(j), ring[j]);
        if (b0 > 0) __syncthreads();   // (everybody has read what lies there)
        // The activations: 256 bytes of a row a time, 16 to a lane, four of those a wave.  What is behind the rows' end is 0.  (All in 32 bits, the division
        // by a product that is exact for the few thousand units there are: with 64-bit steps and a division it took 3 us where the rest takes 5.)
        const int units = tokens * there, columns = static_cast<int>(a.k), last = max(columns - 8, 0);
        const float by = __builtin_amdgcn_rcpf(static_cast<float>(there));
        auto place = [&](int k, const _Float16*& x, int& c) __attribute__((always_inline)) {   // unit k of the workgroup's, this lane's piece: its row, its column
            const int t = static_cast<int>((static_cast<float>(k) + 0.5f) * by), in = b0 + min(k - t * there, blocks - 1);
            const bool second = in >= a.plane_blocks;
            c = (second ? in - a.plane_blocks : in) * static_cast<int>(kI4Columns) + 8 * ((lane & 15) ^ t);
            x = a.x + (t0 + (second ? a.T : 0)) * a.k + static_cast<uint32_t>(t * columns);
        };
        if (a.aligned) {
            for (int k0 = 4 * wave; k0 < units; k0 += 4 * NW) {
                const _Float16* x;
                int c;
                place(min(k0 + q, units - 1), x, c);
                load16_to_lds<false>(base + k0 * 256u, x + min(c, last));
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            for (int k0 = 4 * wave; columns % kI4Columns != 0 && k0 + q < units; k0 += 4 * NW) {
                const _Float16* x;
                int c;
                place(k0 + q, x, c);
                if (c >= columns) *reinterpret_cast<u4*>(lds + (k0 + q) * 256 + 16 * (lane & 15)) = u4{0u, 0u, 0u, 0u};
            }
        } else {
            constexpr int U = 4;   // requested together
            for (int k0 = 4 * wave; k0 < units; k0 += 4 * NW * U) {
                u4 v[U];
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    if (k0 + 4 * NW * u >= units) break;
                    const _Float16* x;
                    int c;
                    place(min(k0 + 4 * NW * u + q, units - 1), x, c);
                    if (columns >= 8) v[u] = load16_any(x + min(c, last));
                    else v[u] = load_part(x, 0, columns);
                }
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int k = k0 + 4 * NW * u + q;
                    if (k >= units) break;
                    const _Float16* x;
                    int c;
                    place(k, x, c);
                    *reinterpret_cast<u4*>(lds + k * 256 + 16 * (lane & 15)) = c > last ? drop_halves(v[u], min(c - last, 8)) : v[u];
                }
            }
        }
        __syncthreads();
        for (int k = 0; k < n; k += D) {
#pragma unroll
            for (int j = 0; j < D; ++j) {
                if (k + j < n) multiply(wave + (k + j) * NW, ring[j]);
                load(at(k + D + j), ring[j]);
            }
        }
    }
    f4* const sums = reinterpret_cast<f4*>(lds);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < CB; ++i) sums[(wave * CB + i) * 64 + lane] = acc[i];
    __syncthreads();
    // Four columns of a token a thread.
    for (int o = threadIdx.x; o < CT * 64; o += 64 * NW) {
        f4 v[P];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            v[p] = sums[p * CT * 64 + o];
#pragma unroll
            for (int w = 1; w < NW; ++w) v[p] += sums[(w * CB + p * CT) * 64 + o];
        }
        const int i = o / 64, l = o & 63;
        const int64_t t = t0 + (l & 15), c = i4_row(tile0 + i, 4 * (l >> 4)), plane = a.T * a.n;
        if (t >= a.T) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            if (c + e >= a.n) break;
            const int64_t to = t * a.n + c + e;
            if constexpr (GATED) {
                float g = v[0][e], u = v[1][e];
                if (a.addends) g += static_cast<float>(a.addends[to]), u += static_cast<float>(a.addends[plane + to]);
                if (a.kept) {
                    a.kept[to] = kept_half(g);
                    a.kept[plane + to] = kept_half(u);
                }
                a.y[to] = static_cast<_Float16>(silu(g) * u);
            } else {
                a.y[to] = static_cast<_Float16>(v[0][e]);
            }
        }
        if constexpr (BWD) {
            if (a.dh && !number(v[0][0])) from_unrounded<4>(a, t, c);
        }
    }
}

template <int CB, int NW, int D, int S, bool ZERO, bool GATED>
lordba_status few_launch(I4Args a, hipStream_t stream) {
    constexpr int CT = CB / (GATED ? 2 : 1);
    // as many columns as fit, in equal parts, whole blocks for every wave where there are that many
    const int64_t tokens = std::min<int64_t>(a.T, 16), most = few_lds(NW) / (tokens * 256), parts = (a.blocks + most - 1) / most;
    int64_t blocks = (a.blocks + parts - 1) / parts;
    if (blocks > NW) blocks = std::min(most, (blocks + NW - 1) / NW * NW);
    a.columns = static_cast<int32_t>(blocks * kI4Columns);
    const size_t lds = static_cast<size_t>(std::max<int64_t>((tokens * blocks * 256 + 1023) / 1024 * 1024, NW * CB * 1024));   // (whole requests of 1 KiB)
    static_assert(NW * CB * 1024 <= few_lds(NW), "room for the sums");
    const int64_t n = (a.tiles + CT - 1) / CT * ((a.T + 15) / 16);
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / (64 * NW);   // (a launch counts threads in 32 bits)
    if (n > INT32_MAX) return LORDBA_ERR_DIM;
    for (int64_t first = 0; first < n; first += kMost) {
        a.first = static_cast<uint32_t>(first);
        hipLaunchKernelGGL((lordba_i4_few_kernel<CB, NW, D, S, ZERO, GATED>), dim3(static_cast<unsigned>(std::min(kMost, n - first))), dim3(64 * NW), lds,
                           stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

template <int S, bool ZERO, bool GATED>
lordba_status few(const I4Args& a, hipStream_t stream) {
    // More blocks of 16 rows than two workgroups of eight waves on every compute unit: four waves, and four workgroups side by side (one token 4096 -> 11008
    // 6.8 us, with eight waves 7.8; 301 -> 13001 4.6 and 6.4; gated 4096 -> 11008 12.8 and 15.4).  No more than compute units: sixteen waves on each (one token
    // 13001 -> 301 6.7, with eight 7.1, with four 9.0), but backward, where a wave's scales take as many registers as its codes, eight (16 x 4096 -> 4096 8.8,
    // with sixteen 10.6).  Between them, and with more tokens, whose staging then is the larger part, eight waves, on two blocks of rows (16 x 4096 -> 11008 18.5 ->
    // 14.8 us).
    // Not all forms have room for their ring in the 128 registers that sixteen waves on a compute unit leave each: gated with groups of 64 and zeros 47 lie in memory, without 12, with zeros and groups of 32
    // or 128 11 and 8, of the gradient on two blocks of rows with zeros 33, of the forward product there with zeros and groups of 32 11.  Shallower rings for these have not been measured.
    constexpr int P = GATED ? 2 : 1, D = S == 0 || S == 4 ? 2 : 4;
    if (a.tiles > 512 && a.T <= 8) return few_launch<P, 4, D, S, ZERO, GATED>(a, stream);
    if constexpr (S > 0 && !GATED) {
        if (a.tiles * ((a.T + 15) / 16) <= 256) return few_launch<1, 16, 2, S, ZERO, GATED>(a, stream);
    }
    if constexpr (!GATED) {
        if (a.tiles > 256 && a.T > 4) return few_launch<2, 8, 2, S, ZERO, GATED>(a, stream);
    }
    return few_launch<P, 8, D, S, ZERO, GATED>(a, stream);
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
