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

typedef float sums16 __attribute__((ext_vector_type(16)));

// A workgroup owns 32 CP WC weight rows (gated: half of them gate's, half up's) and 32 TB WT tokens, each of its WC x WT waves CP x TB blocks of 32 x 32 by
// v_mfma_f32_32x32x16_f16.  A step is a block of 128 columns, eight products deep.
// Activations.  Those of a step lie in LDS, of which two steps' are held, rows of 256 bytes with their 16-byte piece p at place p ^ (row mod 16): sixteen
// lanes that read one piece of sixteen rows cover all banks.
// Weights.  They come from memory straight into the registers of the waves that multiply them, a step ahead.  A pair of 16-row blocks is a 32-row operand: lane
// 32 h + 16 b + r takes from block b what lanes 16 (2 c + h) + r hold (lordba_i4.h), which is row r's columns 32 m + 16 c + 8 h .. + 7 for m = 0 .. 3 and c = 0, 1.
// They become fp16 in the registers, their scale multiplied on before the product, which rounds each weight once (half a step, 2^-11 of it; scales taken out of
// the sums instead, as for few tokens, would be exact, but take a multiplication for every accumulator and group: 64 against 32 for a 32 x 128 block of weights in the
// largest tile at groups of 128, whose registers do not hold a second set of accumulators besides.  In tiles of 32 tokens it would be 16 against 32, which has not been measured).
// While the products of one depth run, the operands of the next are read from LDS and made from the codes.  The barrier stands one depth before a step's
// end: everybody has then read the step's activations, and the next step's have landed.
template <int CP, int TB, int WC, int WT, int WK, int S, bool ZERO, bool GATED, bool BY_REGISTERS>
__global__ __launch_bounds__(64 * WC * WT * WK, 2) void lordba_i4_many_kernel(I4Args a) {
    constexpr bool BWD = S == 0;
    constexpr int P = GATED ? 2 : 1, NW = WC * WT, PW = CP / P, kPairs = PW * WC, kTokens = 32 * TB * WT;   // kPairs: row pairs of a half
    constexpr int kEach = BWD ? (kPairs + 3) / 4 : 0;   // KiB for the scales of the groups across a workgroup's rows
    constexpr uint32_t kX = kTokens * 256u, kS = kEach * 1024u, kBuffer = kX + kS * (ZERO ? 2 : 1);
    static_assert(CP % P == 0 && !(GATED && BWD), "");
    extern __shared__ int8_t all_lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
    const int wk = wave / NW, wi = wave % NW, wc = wi % WC, wt = wi / WC, pairs = a.tiles / 2;
    const Tile at = tile_of(a.first + blockIdx.x, static_cast<uint32_t>((pairs + kPairs - 1) / kPairs), static_cast<uint32_t>((a.T + kTokens - 1) / kTokens));
    int8_t* const lds = all_lds + wk * 2 * kBuffer;
    const int steps = (a.blocks + WK - 1) / WK;
    const int first_pair = static_cast<int>(at.c) * kPairs, pair0 = first_pair + wc * PW;
    const int64_t first_token = static_cast<int64_t>(at.t) * kTokens;

    const u4* code[CP];
    const uint16_t *scale[CP], *zero[CP];
    uint32_t s_at[CP];   // backward: where in a buffer the scales of the pair's group start
    const int group0 = BWD ? (32 * first_pair) >> a.shift : 0;
#pragma unroll
    for (int i = 0; i < CP; ++i) {
        const int pair = min(pair0 + i % PW, pairs - 1) + (i / PW) * pairs;
        const int64_t tile = 2 * static_cast<int64_t>(pair) + (n >> 4);
        code[i] = reinterpret_cast<const u4*>(a.codes) + tile * a.blocks * 64 + 16 * h + (n & 15);
        scale[i] = BWD ? nullptr : a.scale + tile * a.groups * 16 + (n & 15);
        zero[i] = BWD || !ZERO ? nullptr : a.zero + tile * a.groups * 16 + (n & 15);
        s_at[i] = BWD ? static_cast<uint32_t>(((32 * pair) >> a.shift) - group0) * 256u : 0;
    }
    struct Weights {
        u4 c[CP][2];
        uint16_t s[BWD ? 1 : CP][BWD ? 1 : S], z[!BWD && ZERO ? CP : 1][BWD ? 1 : S];
    };
    auto load_weights = [&](int b, Weights& w) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CP; ++i) {
            w.c[i][0] = code[i][static_cast<int64_t>(b) * 64];
            w.c[i][1] = code[i][static_cast<int64_t>(b) * 64 + 32];
            if constexpr (!BWD) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    w.s[i][s] = scale[i][(static_cast<int64_t>(b) * S + s) * 16];
                    if constexpr (ZERO) w.z[i][s] = zero[i][(static_cast<int64_t>(b) * S + s) * 16];
                }
            }
        }
    };
    // The activations of step b, and the scales that go with them, straight into LDS, request by request; pieces behind the rows' end hold what is in front of it
    // and are cleared when they have landed (a NaN among them would pass the weights of 0 there).  Rows that do not consist of aligned pieces (BY_REGISTERS) are
    // requested into registers and stored, moved into place at their end, before the barrier that the step waits for.
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    constexpr int kLoads = kTokens / 4 / NW;
    static_assert(kTokens / 4 % NW == 0, "whole loads per wave");
    const int32_t last_row = static_cast<int32_t>(min<int64_t>(a.T - 1 - first_token, kTokens - 1));
    const int32_t row0 = 4 * wi + (lane >> 4);
    // (a large tile's accumulators leave room for half of a step's activations: those of the next step are requested and stored half by half then)
    constexpr bool HALVES = BY_REGISTERS && CP * TB >= 8;
    constexpr int kHeld = HALVES ? kLoads / 2 : kLoads;
    u4 held[BY_REGISTERS ? kHeld : 1];
    // (of the WK blocks of a step this wave has the wk-th; where there is none, the last stands in, behind the rows' end altogether)
    auto block_of = [&](int step) __attribute__((always_inline)) { return min(step * WK + wk, a.blocks - 1); };
    auto column_of = [&](int b) __attribute__((always_inline)) { return (b >= a.plane_blocks ? b - a.plane_blocks : b) * static_cast<int32_t>(kI4Columns); };
    auto end_of = [&](int step, int w) __attribute__((always_inline)) {   // of the w-th block of a step: its columns
        const int b = step * WK + w;
        return b < a.blocks ? static_cast<int32_t>(a.k) - column_of(b) : 0;
    };
    auto piece_of = [&](int i) __attribute__((always_inline)) { return 8 * ((lane & 15) ^ ((row0 + 4 * NW * i) & 15)); };   // (in halves)
    auto request = [&](int step, uint32_t buffer, int i) __attribute__((always_inline)) {
        const int b = block_of(step);
        const int32_t c0 = column_of(b), k = static_cast<int32_t>(a.k);
        const _Float16* const x = a.x + ((b >= a.plane_blocks ? a.T : 0) + first_token) * a.k;
        // (a tile's rows span less than 4 GiB: what the launch sees to)
        const uint32_t at = (static_cast<uint32_t>(min(row0 + 4 * NW * i, last_row)) * static_cast<uint32_t>(k) + min(c0 + piece_of(i), k - 8)) * 2u;
        if constexpr (BY_REGISTERS) held[i % kHeld] = load16_any(reinterpret_cast<const char*>(x) + at);
        else load16_to_lds_from(base + buffer + (wi + NW * i) * 1024u, x, at);
    };
    auto request_scales = [&](int step, uint32_t buffer) __attribute__((always_inline)) {
        if constexpr (BWD) {   // (a place for each group there may be; groups behind the last are not read by anybody)
            constexpr int kAll = kEach * (ZERO ? 2 : 1);
            static_assert(kAll % NW == 0 || NW % kAll == 0, "a wave for each KiB, or several, or several for each");
#pragma unroll
            for (int j = 0; j < kAll; j += NW) {
                const int p = (wi + j) % kAll, part = p % kEach, group = min(group0 + 4 * part + (lane >> 4), static_cast<int>((a.n - 1) >> a.shift));
                load16_to_lds<false>(base + buffer + kX + p * 1024u,
                                     (p >= kEach ? a.zero : a.scale) + (static_cast<int64_t>(group) * a.blocks + block_of(step)) * kI4Columns + 8 * (lane & 15));
            }
        }
    };
    auto store_held = [&](int step, uint32_t buffer, int first) __attribute__((always_inline)) {
        if constexpr (BY_REGISTERS) {
            const int32_t end = end_of(step, wk);
#pragma unroll
            for (int l = 0; l < kHeld; ++l) {
                const int i = first + l;
                const int32_t over = piece_of(i) - (end - 8);
                if (end < kI4Columns && over > 0) held[l] = drop_halves(held[l], over);
                *reinterpret_cast<u4*>(lds + buffer + (wi + NW * i) * 1024u + 16 * lane) = held[l];
            }
        }
    };
    auto request_some = [&](int step, uint32_t buffer, int first, int n) __attribute__((always_inline)) {
#pragma unroll
        for (int l = 0; l < n; ++l) request(step, buffer, first + l);
    };
    // Pieces of a step behind the rows' end, when everything has landed; whoever requested a piece clears it.
    auto clear_end = [&](int step, uint32_t buffer) __attribute__((always_inline)) {
        if constexpr (!BY_REGISTERS) {
            int32_t least = kI4Columns;
#pragma unroll
            for (int w = 0; w < WK; ++w) least = min(least, end_of(step, w));
            if (least >= kI4Columns) return;
            const int32_t end = end_of(step, wk);
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
                if (piece_of(i) >= end) *reinterpret_cast<u4*>(lds + buffer + (wi + NW * i) * 1024u + 16 * lane) = u4{0u, 0u, 0u, 0u};
            __syncthreads();
        }
    };
    sums16 acc[CP][TB];
#pragma unroll
    for (int i = 0; i < CP; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.f;
    // Operands of depth d = 2 m + c of a step: the activations are read A - 1 depths ahead (a small tile's products of one depth do not last as long as a
    // read of LDS takes), the weights are made from the codes one depth ahead.
    constexpr int A = CP * TB >= 8 ? 2 : CP * TB >= 4 || BWD ? 4 : 8;
    const int8_t* const mine = lds + (wt * TB * 32 + n) * 256;
    h8 x[A][TB], w[2][CP];
    u4 sv[BWD && A > 2 ? A : 1][CP], zv[BWD && A > 2 && ZERO ? A : 1][CP];
    const uint32_t exp = exponent();
    auto read = [&](auto depth, uint32_t buffer) __attribute__((always_inline)) {
        constexpr int d = depth.value, set = d % A;
#pragma unroll
        for (int j = 0; j < TB; ++j) x[set][j] = as_h8(*reinterpret_cast<const u4*>(mine + buffer + j * 8192 + 16 * ((2 * d + h) ^ (n & 15))));
        if constexpr (BWD && A > 2) {
#pragma unroll
            for (int i = 0; i < CP; ++i) {
                const int8_t* const s = lds + buffer + kX + s_at[i] + 32 * d + 16 * h;
                sv[set][i] = *reinterpret_cast<const u4*>(s);
                if constexpr (ZERO) zv[set][i] = *reinterpret_cast<const u4*>(s + kS);
            }
        }
    };
    auto make = [&](auto depth, uint32_t buffer, const Weights& v) __attribute__((always_inline)) {
        constexpr int d = depth.value, m = d >> 1, c = d & 1, set = d & 1, early = A > 2 ? d % A : 0;
#pragma unroll
        for (int i = 0; i < CP; ++i) {
            if constexpr (BWD) {
                const int8_t* const at_s = lds + buffer + kX + s_at[i] + 32 * d + 16 * h;
                const u4 s = A > 2 ? sv[early][i] : *reinterpret_cast<const u4*>(at_s);
                if constexpr (ZERO) w[set][i] = operand(v.c[i][c][m], Zero8{A > 2 ? zv[early][i] : *reinterpret_cast<const u4*>(at_s + kS)}, exp);
                else w[set][i] = operand(v.c[i][c][m], Zero1(kZero8), exp);
                w[set][i] = w[set][i] * as_h8(s);
            } else {
                constexpr int g = m * (S ? S : 1) / 4;
                w[set][i] = operand(v.c[i][c][m], Zero1(ZERO ? v.z[i][g] : kZero8), exp);
                const h2 s = both(v.s[i][g]);
                w[set][i] = w[set][i] * h8{s[0], s[0], s[0], s[0], s[0], s[0], s[0], s[0]};
            }
        }
    };
    auto multiply = [&](auto depth) __attribute__((always_inline)) {
        constexpr int d = depth.value;
#pragma unroll
        for (int i = 0; i < CP; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_f16(w[d & 1][i], x[d % A][j], acc[i][j], 0, 0, 0);
    };
    // between every few products some of the next operands' work
    auto weave = []() __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CP * TB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x2, 16 * CP / (CP * TB), 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    // What has been requested has landed, and everybody has read what was in the other buffer.
    auto meet = []() __attribute__((always_inline)) {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // (the copy is made here, not behind the loads into `next`: their arrival would be waited for with it)
    auto settle = [](Weights& v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CP; ++i) {
            asm volatile("" : "+v"(v.c[i][0]), "+v"(v.c[i][1]));
            if constexpr (!BWD) {
#pragma unroll
                for (int s = 0; s < S; ++s) {
                    asm volatile("" : "+v"(v.s[i][s]));
                    if constexpr (ZERO) asm volatile("" : "+v"(v.z[i][s]));
                }
            }
        }
    };
    using std::integral_constant;
    Weights now, next;
    request_scales(0, 0);
    load_weights(block_of(0), now);
    if constexpr (HALVES) {
        request_some(0, 0, 0, kHeld);
        store_held(0, 0, 0);
        request_some(0, 0, kHeld, kHeld);
        store_held(0, 0, kHeld);
    } else {
        request_some(0, 0, 0, kLoads);
        store_held(0, 0, 0);
    }
    meet();
    clear_end(0, 0);
    request_scales(min(1, steps - 1), kBuffer);
    if constexpr (!HALVES) request_some(min(1, steps - 1), kBuffer, 0, kLoads);
    load_weights(block_of(min(1, steps - 1)), next);
    auto read_first = [&](uint32_t buffer) __attribute__((always_inline)) {   // what depth 0 expects to be there
        read(integral_constant<int, 0>{}, buffer);
        if constexpr (A > 2) {
            read(integral_constant<int, 1>{}, buffer);
            read(integral_constant<int, 2>{}, buffer);
        }
        if constexpr (A > 4) {
            read(integral_constant<int, 3>{}, buffer);
            read(integral_constant<int, 4>{}, buffer);
            read(integral_constant<int, 5>{}, buffer);
            read(integral_constant<int, 6>{}, buffer);
        }
    };
    read_first(0);
    make(integral_constant<int, 0>{}, 0, now);
    uint32_t buffer = 0;
    for (int step = 0; step < steps; ++step) {
        // (Behind the last step what is there is requested once more, operands are made of it, and nobody multiplies them.)
        const int next_step = min(step + 1, steps - 1), behind = min(step + 2, steps - 1);
        auto depth = [&](auto d) __attribute__((always_inline)) {
            if constexpr (d.value + A - 1 < 8) read(integral_constant<int, d.value + A - 1>{}, buffer);
            make(integral_constant<int, d.value + 1>{}, buffer, now);
            multiply(d);
            weave();
        };
        if constexpr (HALVES) request_some(next_step, 0, 0, kHeld);
        depth(integral_constant<int, 0>{});
        depth(integral_constant<int, 1>{});
        depth(integral_constant<int, 2>{});
        if constexpr (HALVES) {
            store_held(next_step, kBuffer - buffer, 0);
            request_some(next_step, 0, kHeld, kHeld);
        }
        depth(integral_constant<int, 3>{});
        depth(integral_constant<int, 4>{});
        depth(integral_constant<int, 5>{});
        depth(integral_constant<int, 6>{});
        // (the operands of depth 7 are made above, not behind the barrier)
#pragma unroll
        for (int i = 0; i < CP; ++i) asm volatile("" : "+v"(w[1][i]));
        store_held(next_step, kBuffer - buffer, kLoads - kHeld);
        meet();
        clear_end(next_step, kBuffer - buffer);
        now = next;
        settle(now);
        load_weights(block_of(behind), next);
        request_scales(behind, buffer);
        const uint32_t freed = buffer;
        buffer = kBuffer - buffer;
        read_first(buffer);
        make(integral_constant<int, 0>{}, buffer, now);
        if constexpr (!HALVES) request_some(behind, freed, 0, kLoads);
        multiply(integral_constant<int, 7>{});
        weave();
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (nothing is on its way into LDS when the workgroup ends, or takes it for its sums)

    // Results of a block, of both halves where there are two: a lane has two times eight consecutive columns of a token.
    const int64_t plane = a.T * a.n;
    uint32_t lost = 0;   // backward: blocks whose first result of this lane's is no number, bit i TB + j
    auto finish = [&](auto whole, auto odd, int i, int j, const sums16 (&sum)[P]) __attribute__((always_inline)) {
        constexpr bool FULL = whole.value, ODD = odd.value;
        const int64_t t = first_token + (wt * TB + j) * 32 + n;
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int64_t c = 32 * static_cast<int64_t>(pair0 + i) + 16 * u + 8 * h;
            if (!FULL && (c >= a.n || t >= a.T)) continue;
            float v[P][8];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) v[p][e] = sum[p][4 * (u + 2 * (e >> 2)) + (e & 3)];
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
                        if constexpr (ODD) store8_odd<true, 32>(a.kept + p * plane + t * a.n + c, v[p]);
                        else store8<FULL, false, true>(a.kept + p * plane + t * a.n, c, a.n, v[p]);
                    }
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[0][e] = silu(v[0][e]) * v[1][e];
            }
            if constexpr (ODD) store8_odd<false, 32>(a.y + t * a.n + c, v[0]);
            else store8<FULL, false, false>(a.y + t * a.n, c, a.n, v[0]);
            if (BWD && u == 0) lost |= number(v[0][0]) ? 0u : 1u << (i * TB + j);
        }
    };
    const bool full = 32 * static_cast<int64_t>(first_pair + kPairs) <= a.n && first_token + kTokens <= a.T;
    const bool odd = (a.n & 1) || ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.kept)) & 2) != 0;
    if constexpr (WK == 1) {
        auto all = [&](auto whole, auto is_odd) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < PW; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) {
                    sums16 sum[P];
#pragma unroll
                    for (int p = 0; p < P; ++p) sum[p] = acc[p * PW + i][j];
                    finish(whole, is_odd, i, j, sum);
                }
        };
        if (!full) all(std::false_type{}, std::false_type{});
        else if (odd) all(std::true_type{}, std::true_type{});
        else all(std::true_type{}, std::false_type{});
    } else {
        // The sums of the WK parts are joined through LDS, in their order, block by block; the parts share the blocks.
        f4* const parts = reinterpret_cast<f4*>(all_lds);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CP; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    parts[((wave * CP + i) * TB + j) * 256 + e * 64 + lane] = f4{acc[i][j][4 * e], acc[i][j][4 * e + 1], acc[i][j][4 * e + 2], acc[i][j][4 * e + 3]};
        __syncthreads();
        for (int o = wk; o < PW * TB; o += WK) {
            sums16 sum[P];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    f4 s = parts[((wi * CP + p * PW) * TB + o) * 256 + e * 64 + lane];
#pragma unroll
                    for (int w = 1; w < WK; ++w) s += parts[(((w * NW + wi) * CP + p * PW) * TB + o) * 256 + e * 64 + lane];
#pragma unroll
                    for (int f = 0; f < 4; ++f) sum[p][4 * e + f] = s[f];
                }
            const int i = o / TB, j = o % TB;
            if (!full) finish(std::false_type{}, std::false_type{}, i, j, sum);
            else if (odd) finish(std::true_type{}, std::true_type{}, i, j, sum);
            else finish(std::true_type{}, std::false_type{}, i, j, sum);
        }
    }
    if constexpr (BWD) {
        if (a.dh && lost) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (where every other row starts in the middle of a word, another lane has stored them)
            const int me = __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u));   // (the lane once more: kept from the start it takes a register of the largest tile that is not there)
            for (; lost; lost &= lost - 1) {
                const int o = __builtin_ctz(lost);
                for (int u = 0; u < 2; ++u)
                    from_unrounded<8>(a, first_token + (wt * TB + o % TB) * 32 + (me & 31), 32 * static_cast<int64_t>(pair0 + o / TB) + 16 * u + 8 * (me >> 5));
            }
        }
    }
}

template <int CP, int TB, int WC, int WT, int WK, int S, bool ZERO, bool GATED, bool BY_REGISTERS>
lordba_status many_launch(I4Args a, hipStream_t stream) {
    constexpr int kPairs = CP / (GATED ? 2 : 1) * WC, kTokens = 32 * TB * WT;
    constexpr size_t kScales = S == 0 ? (kPairs + 3) / 4 * 1024 * (ZERO ? 2 : 1) : 0, kRing = 2 * WK * (kTokens * 256 + kScales);
    constexpr size_t kSums = WK == 1 ? 0 : static_cast<size_t>(WK) * WC * WT * CP * TB * 4096, kLds = kRing > kSums ? kRing : kSums;
    static_assert(kLds <= kLdsBytes, "LDS of a compute unit");
    if (kLds > 64 * 1024) {   // (once for a device: more LDS than a launch gets unasked)
        static std::atomic<uint64_t> asked{0};
        int device = 0;
        if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) return LORDBA_ERR_NO_DEVICE;
        if (!(asked.load(std::memory_order_relaxed) >> device & 1)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(lordba_i4_many_kernel<CP, TB, WC, WT, WK, S, ZERO, GATED, BY_REGISTERS>),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kLds)) != hipSuccess) {
                (void)hipGetLastError();
                return LORDBA_ERR_LAUNCH;
            }
            asked.fetch_or(static_cast<uint64_t>(1) << device, std::memory_order_relaxed);
        }
    }
    const int64_t n = static_cast<int64_t>((a.tiles / 2 + kPairs - 1) / kPairs) * ((a.T + kTokens - 1) / kTokens);
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / (64 * WC * WT * WK);   // (a launch counts threads in 32 bits)
    if (n > INT32_MAX) return LORDBA_ERR_DIM;
    for (int64_t first = 0; first < n; first += kMost) {
        a.first = static_cast<uint32_t>(first);
        hipLaunchKernelGGL((lordba_i4_many_kernel<CP, TB, WC, WT, WK, S, ZERO, GATED, BY_REGISTERS>), dim3(static_cast<unsigned>(std::min(kMost, n - first))), dim3(64 * WC * WT * WK),
                           kLds, stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

template <int S, bool ZERO, bool GATED>
lordba_status many(const I4Args& a, int kernel, hipStream_t stream) {
    if (!a.aligned) {
        if (kernel == kI4Tile32) return many_launch<GATED ? 2 : 1, 1, 1, 1, 8, S, ZERO, GATED, true>(a, stream);
        if (kernel == kI4Tile64) return many_launch<2, 1, 1, 1, 4, S, ZERO, GATED, true>(a, stream);
        if constexpr (!(S == 4 && ZERO)) {
            if (kernel == kI4Tile256) return many_launch<2, 4, 4, 1, 1, S, ZERO, GATED, true>(a, stream);
        }
        return many_launch<2, 2, 2, 1, 2, S, ZERO, GATED, true>(a, stream);
    }
    if constexpr (S > 0 && !GATED) {
        if (kernel == kI4Square64) return many_launch<1, 2, 2, 1, 4, S, ZERO, GATED, false>(a, stream);
    }
    switch (kernel) {
        case kI4Tile32: return many_launch<GATED ? 2 : 1, 1, 1, 1, 8, S, ZERO, GATED, false>(a, stream);
        case kI4Tile64: return many_launch<2, 1, 1, 1, 4, S, ZERO, GATED, false>(a, stream);
        case kI4Tile128: return many_launch<2, 2, 2, 1, 2, S, ZERO, GATED, false>(a, stream);
        default: return many_launch<2, 4, 4, 1, 1, S, ZERO, GATED, false>(a, stream);
    }
}
template <int S, bool GATED>
lordba_status many(const I4Args& a, int kernel, hipStream_t stream) {
    return a.zero ? many<S, true, GATED>(a, kernel, stream) : many<S, false, GATED>(a, kernel, stream);
}
template <bool GATED>
lordba_status many(const I4Args& a, int kernel, int64_t group, hipStream_t stream) {
    return group == 32 ? many<4, GATED>(a, kernel, stream) : group == 64 ? many<2, GATED>(a, kernel, stream) : many<1, GATED>(a, kernel, stream);
}

}  // namespace

lordba_status lordba_i4_many(const I4Args& a, int kernel, int64_t group, bool gated, bool backward, hipStream_t stream) {
    if (backward) return many<0, false>(a, kernel, stream);
    return gated ? many<true>(a, kernel, group, stream) : many<false>(a, kernel, group, stream);
}
