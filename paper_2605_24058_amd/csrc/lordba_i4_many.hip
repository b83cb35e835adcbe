// Products with 4-bit weights, many tokens: what bounds them is the matrix cores.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lordba_i4_product.h"

namespace {

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: every XCD gets a contiguous eighth of the
// tiles, in groups of kTogether tiles along the tokens, so that those it runs at a time share rows of both operands.
constexpr uint32_t kTogether = 4;
struct Tile {
    uint32_t c, t;
};
__device__ __forceinline__ Tile tile_of(uint32_t id, uint32_t nc, uint32_t nt) {
    const uint32_t n = nc * nt, xcd = id & 7, each = n / 8, rest = n % 8;
    const uint32_t i = xcd * each + min(xcd, rest) + (id >> 3);
    const uint32_t g = i / (kTogether * nc), in = i % (kTogether * nc), size = min(kTogether, nt - g * kTogether);
    return {in / size, g * kTogether + in % size};
}

// A workgroup owns 16 CB WC weight rows (gated: half of them gate's, half up's) and 16 TB WT tokens, each of its WC x WT waves CB x TB blocks of 16 x 16.
// A step is a block of 128 columns.  The activations of a step lie in LDS, of which two steps' are held, rows of 256 bytes with their 16-byte piece p
// at place p ^ (row mod 16): sixteen lanes that read one piece of sixteen rows cover all banks.  The weights come from memory straight into the
// registers of the waves that multiply them, a step ahead, and become fp16 there: their scale is multiplied on before the product, which rounds each weight once
// (half a step, 2^-11 of it; scales taken out of the sums instead, as for few tokens, would be exact, but take a multiplication for every accumulator and group).
template <int CB, int TB, int WC, int WT, int S, bool ZERO, bool GATED>
__global__ __launch_bounds__(64 * WC * WT) void lordba_i4_many_kernel(I4Args a) {
    constexpr bool BWD = S == 0;
    constexpr int P = GATED ? 2 : 1, NW = WC * WT, CT = CB / P, kTiles = CT * WC, kTokens = 16 * TB * WT;   // kTiles: blocks of a half
    constexpr int kGroups = BWD ? (16 * kTiles + 31) / 32 : 0;   // most groups across a workgroup's rows
    constexpr uint32_t kX = kTokens * 256u, kS = kGroups * 256u, kBuffer = kX + kS * (ZERO ? 2 : 1);
    static_assert(CT % 2 == 0 && !(GATED && BWD), "pairs of blocks");
    extern __shared__ int8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = lane & 15, q = lane >> 4;
    const int wc = wave % WC, wt = wave / WC;
    const Tile at = tile_of(a.first + blockIdx.x, static_cast<uint32_t>((a.tiles + kTiles - 1) / kTiles), static_cast<uint32_t>((a.T + kTokens - 1) / kTokens));
    const int first_tile = static_cast<int>(at.c) * kTiles, tile0 = first_tile + wc * CT;
    const int64_t first_token = static_cast<int64_t>(at.t) * kTokens;

    const u4* code[CB];
    const uint16_t *scale[CB], *zero[CB];
    uint32_t s_at[CB];   // backward: where in a buffer the scales of the block's group start
    const int group0 = BWD ? static_cast<int>(i4_row(first_tile, 0) >> a.shift) : 0;
#pragma unroll
    for (int i = 0; i < CB; ++i) {
        const int64_t tile = min(tile0 + i % CT, a.tiles - 1) + (i / CT) * a.tiles;
        code[i] = reinterpret_cast<const u4*>(a.codes) + tile * a.blocks * 64 + lane;
        scale[i] = BWD ? nullptr : a.scale + tile * a.groups * 16 + r;
        zero[i] = BWD || !ZERO ? nullptr : a.zero + tile * a.groups * 16 + r;
        s_at[i] = BWD ? static_cast<uint32_t>((i4_row(tile, 0) >> a.shift) - group0) * 256u : 0;
    }
    struct Weights {
        u4 c[CB];
        uint16_t s[BWD ? 1 : CB][BWD ? 1 : S], z[!BWD && ZERO ? CB : 1][BWD ? 1 : S];
    };
    auto load_weights = [&](int b, Weights& w) {
#pragma unroll
        for (int i = 0; i < CB; ++i) {
            w.c[i] = code[i][static_cast<int64_t>(b) * 64];
            if constexpr (!BWD) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    w.s[i][s] = scale[i][(static_cast<int64_t>(b) * S + s) * 16];
                    if constexpr (ZERO) w.z[i][s] = zero[i][(static_cast<int64_t>(b) * S + s) * 16];
                }
            }
        }
    };
    // The activations of step b, and the scales that go with them.  Whole steps of aligned rows go straight into LDS.
    const bool aligned = a.k % 8 == 0 && (reinterpret_cast<uintptr_t>(a.x) & 15) == 0;
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    auto stage = [&](int b, uint32_t buffer) {
        const int plane = b >= a.plane_blocks ? 1 : 0;
        const int64_t c0 = static_cast<int64_t>(b - plane * a.plane_blocks) * kI4Columns;
        const _Float16* const x = a.x + plane * a.T * a.k;
        if (aligned && c0 + kI4Columns <= a.k) {
#pragma unroll
            for (int i = 0; i < kTokens / 4 / NW; ++i) {
                const int row = 4 * (wave + NW * i) + q;
                load16_to_lds<false>(base + buffer + (wave + NW * i) * 1024u, x + min(first_token + row, a.T - 1) * a.k + c0 + 8 * (r ^ (row & 15)));
            }
        } else {
#pragma unroll 4
            for (int i = 0; i < kTokens / 4 / NW; ++i) {
                const int row = 4 * (wave + NW * i) + q;
                const u4 v = load_part(x + min(first_token + row, a.T - 1) * a.k, c0 + 8 * (r ^ (row & 15)), a.k);
                *reinterpret_cast<u4*>(lds + buffer + (wave + NW * i) * 1024u + 16 * lane) = v;
            }
        }
        if constexpr (BWD) {   // (rows of groups that the matrix does not have stay unread)
            const int group = threadIdx.x >> 4, piece = threadIdx.x & 15;
            if (group < kGroups && group0 + group <= static_cast<int>((a.n - 1) >> a.shift)) {
                const int64_t from = (static_cast<int64_t>(group0 + group) * a.blocks + b) * kI4Columns + 8 * piece;
                *reinterpret_cast<u4*>(lds + buffer + kX + group * 256 + 16 * piece) = load16(a.scale + from);
                if constexpr (ZERO) *reinterpret_cast<u4*>(lds + buffer + kX + kS + group * 256 + 16 * piece) = load16(a.zero + from);
            }
        }
    };
    static_assert(!BWD || kGroups * 16 <= 64 * NW, "a thread for each piece");
    f4 acc[CB][TB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    const int8_t* const mine = lds + (wt * TB * 16 + r) * 256;
    auto multiply = [&](uint32_t buffer, const Weights& v) {
#pragma unroll
        for (int m = 0; m < 4; ++m) {
            h8 x[TB], w[CB];
#pragma unroll
            for (int j = 0; j < TB; ++j) x[j] = as_h8(*reinterpret_cast<const u4*>(mine + buffer + j * 4096 + 16 * ((4 * m + q) ^ r)));
#pragma unroll
            for (int i = 0; i < CB; ++i) {
                if constexpr (BWD) {
                    const int8_t* const s = lds + buffer + kX + s_at[i] + 64 * m + 16 * q;
                    if constexpr (ZERO) w[i] = operand(v.c[i][m], Zero8{*reinterpret_cast<const u4*>(s + kS)});
                    else w[i] = operand(v.c[i][m], Zero1(kZero8));
                    w[i] = w[i] * as_h8(*reinterpret_cast<const u4*>(s));
                } else {
                    constexpr int kEach = 4 / (S ? S : 1);
                    w[i] = operand(v.c[i][m], Zero1(ZERO ? v.z[i][m / kEach] : kZero8));
                    const h2 s = both(v.s[i][m / kEach]);
                    w[i] = w[i] * h8{s[0], s[0], s[0], s[0], s[0], s[0], s[0], s[0]};
                }
            }
#pragma unroll
            for (int i = 0; i < CB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] = mfma(w[i], x[j], acc[i][j]);
        }
    };
    // What has been requested has landed, and everybody has read the buffer that comes next.
    auto meet = [] {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    Weights now;
    stage(0, 0);
    load_weights(0, now);
    uint32_t buffer = 0;
    for (int b = 0; b < a.blocks; ++b) {
        meet();
        Weights next = now;
        if (b + 1 < a.blocks) {
            stage(b + 1, kBuffer - buffer);
            load_weights(b + 1, next);
        }
        multiply(buffer, now);
        now = next;
        buffer = kBuffer - buffer;
    }
    // A lane has eight consecutive columns of a token in a pair of blocks.
    auto finish = [&](auto whole, auto odd) {
        constexpr bool FULL = whole.value, ODD = odd.value;
        const int64_t plane = a.T * a.n;
#pragma unroll
        for (int i = 0; i < CT; i += 2) {
            const int64_t c = i4_row(tile0 + i, 4 * q);
            if (!FULL && c >= a.n) continue;
#pragma unroll
            for (int j = 0; j < TB; ++j) {
                const int64_t t = first_token + (wt * TB + j) * 16 + r;
                if (!FULL && t >= a.T) continue;
                float v[P][8];
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[p][e] = acc[p * CT + i + (e >> 2)][j][e & 3];
                if constexpr (GATED) {
                    if (a.addends) {
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            const h8 add = as_h8(load8<FULL>(a.addends + p * plane + t * a.n, c, a.n));
#pragma unroll
                            for (int e = 0; e < 8; ++e) v[p][e] += static_cast<float>(add[e]);
                        }
                    }
                    if (a.kept) {
#pragma unroll
                        for (int p = 0; p < P; ++p) {
                            if constexpr (ODD) store8_odd<true>(a.kept + p * plane + t * a.n + c, v[p]);
                            else store8<FULL, false, true>(a.kept + p * plane + t * a.n, c, a.n, v[p]);
                        }
                    }
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[0][e] = silu(v[0][e]) * v[1][e];
                }
                if constexpr (ODD) store8_odd<false>(a.y + t * a.n + c, v[0]);
                else store8<FULL, false, false>(a.y + t * a.n, c, a.n, v[0]);
            }
        }
    };
    const bool full = (first_tile + kTiles) * 16 <= a.n && first_token + kTokens <= a.T;
    if (!full) finish(std::false_type{}, std::false_type{});
    else if ((a.n & 1) || ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.kept)) & 2)) finish(std::true_type{}, std::true_type{});
    else finish(std::true_type{}, std::false_type{});
}

template <int CB, int TB, int WC, int WT, int S, bool ZERO, bool GATED>
lordba_status many_launch(I4Args a, hipStream_t stream) {
    constexpr int kTiles = CB / (GATED ? 2 : 1) * WC, kTokens = 16 * TB * WT;
    constexpr size_t kScales = S == 0 ? (16 * kTiles + 31) / 32 * 256 * (ZERO ? 2 : 1) : 0, kLds = 2 * (kTokens * 256 + kScales);
    static_assert(kLds <= kLdsBytes, "LDS of a compute unit");
    if (kLds > 64 * 1024) {   // (once for a device: more LDS than a launch gets unasked)
        static std::atomic<uint64_t> asked{0};
        int device = 0;
        if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) return LORDBA_ERR_NO_DEVICE;
        if (!(asked.load(std::memory_order_relaxed) >> device & 1)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(lordba_i4_many_kernel<CB, TB, WC, WT, S, ZERO, GATED>),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kLds)) != hipSuccess) {
                (void)hipGetLastError();
                return LORDBA_ERR_LAUNCH;
            }
            asked.fetch_or(static_cast<uint64_t>(1) << device, std::memory_order_relaxed);
        }
    }
    const int64_t n = static_cast<int64_t>((a.tiles + kTiles - 1) / kTiles) * ((a.T + kTokens - 1) / kTokens);
    if (n > INT32_MAX / 512) return LORDBA_ERR_DIM;
    hipLaunchKernelGGL((lordba_i4_many_kernel<CB, TB, WC, WT, S, ZERO, GATED>), dim3(static_cast<unsigned>(n)), dim3(64 * WC * WT), kLds, stream, a);
    return i8_launched();
}

template <int S, bool ZERO, bool GATED>
lordba_status many(const I4Args& a, hipStream_t stream) {
    const int64_t large = static_cast<int64_t>((a.tiles * (GATED ? 2 : 1) + 15) / 16) * ((a.T + 255) / 256);
    if (large >= 192) return many_launch<4, 8, 4, 2, S, ZERO, GATED>(a, stream);
    return many_launch<4, 4, 2, 2, S, ZERO, GATED>(a, stream);
}
template <int S, bool GATED>
lordba_status many(const I4Args& a, hipStream_t stream) {
    return a.zero ? many<S, true, GATED>(a, stream) : many<S, false, GATED>(a, stream);
}
template <bool GATED>
lordba_status many(const I4Args& a, int64_t group, hipStream_t stream) {
    return group == 32 ? many<4, GATED>(a, stream) : group == 64 ? many<2, GATED>(a, stream) : many<1, GATED>(a, stream);
}

}  // namespace

lordba_status lordba_i4_many(const I4Args& a, int64_t group, bool gated, bool backward, hipStream_t stream) {
    if (backward) return many<0, false>(a, stream);
    return gated ? many<true>(a, group, stream) : many<false>(a, group, stream);
}
