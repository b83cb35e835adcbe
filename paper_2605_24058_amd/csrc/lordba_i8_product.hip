// Products with 8-bit weights: y[t, j] = s_t w_j sum_i q_ti W_ji on v_mfma_i32_16x16x64_i8, plain or as the two projections of a gated block.
//
// The weights' rows are the first operand, the tokens' rows the second, so that a lane's four accumulators are four consecutive
// columns of y for one token.  Blocks of 16 rows are the unit of everything: with two digits the token blocks alternate hi, lo (y takes
// 256 hi + lo of neighbouring accumulators), in the gated block the weight blocks alternate gate, up, so that a lane holds both
// factors of its outputs.
#include <algorithm>
#include <atomic>
#include <type_traits>

#include "lordba_dev_util.h"
#include "lordba_i8.h"
#include "lordba_results.h"

namespace {

typedef int i4 __attribute__((ext_vector_type(4)));

struct ProductArgs {
    const int8_t* w;          // [channels, ld]; gated: [2 n, ld], gate then up
    const int8_t* q;          // [digits, T, ld]
    const float* q_scale;     // [T]
    const float* w_scale;     // [channels], or null: 1
    const _Float16* addends;  // gated: [2, T, n], or null
    _Float16* y;              // [T, n]
    _Float16* kept;           // gated: [2, T, n], or null
    int64_t T, n, ld;
    int pieces;               // of 64 columns that the contraction has (behind them the rows are zeros)
    const _Float16* x;        // OWN_ROWS: [T, d_in], in place of q and q_scale
    int64_t d_in;
    int32_t* parts;           // splits > 1: [splits, tiles, 16 x 16 blocks] sums, behind the tiles' counters of arrivals (zeros)
    uint32_t* arrived;
    uint32_t splits;
    uint32_t first;           // tile of this launch's first workgroup
};

typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));

template <bool FULL>
__device__ __forceinline__ void load8(const float* p, int64_t c, int64_t n, float (&v)[8]) {
    if (FULL || c + 8 <= n) {
        const f4_any a = *reinterpret_cast<const f4_any*>(p + c), b = *reinterpret_cast<const f4_any*>(p + c + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p[min(c + e, n - 1)];
    }
}
// The sums of a lane (CB x TB blocks) to y.  c0, t0: the first column of y and the first token of the wave's part.  A lane has eight
// consecutive columns of a token in a pair of weight blocks (of gate and of up each), see weight_row.  FULL: all columns and tokens exist.
// ODD: n is odd, or y starts in the middle of a word.  LINES: every piece of 32 columns
// is 64 aligned bytes; what is kept then goes past the caches, with STREAM y too.
// addend(p, j, k) gives the lane's eight addends of plane p for its token of block j and its columns of group k.
template <int CB, int TB, int DIG, bool GATED, bool FULL, bool ODD, bool LINES, bool STREAM, class F>
__device__ __forceinline__ void finish(const ProductArgs& a, const i4 (&acc)[CB][TB], int64_t c0, int64_t t0, F addend) {
    constexpr int P = GATED ? 2 : 1, G = 2 * P, J = TB / DIG;
    static_assert(CB % G == 0 && TB % DIG == 0, "whole groups of blocks");
    const int lane = threadIdx.x & 63;
    const int64_t plane = a.T * a.n, t1 = t0 + (lane & 15);
    float s[J];
#pragma unroll
    for (int j = 0; j < J; ++j) s[j] = FULL || t1 + 16 * j < a.T ? a.q_scale[t1 + 16 * j] : 0.f;
#pragma unroll
    for (int cb = 0; cb < CB; cb += G) {
        const int64_t c = c0 + 32 * (cb / G) + 8 * (lane >> 4);
        if (!FULL && c >= a.n) continue;
        float w[P][8];
        constexpr int A = J < 4 ? J : 4;   // tokens whose addends are requested together: what the registers hold
        u4 add[P][A];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (a.w_scale) load8<FULL>(a.w_scale + p * a.n, c, a.n, w[p]);
            else w[p][0] = w[p][1] = w[p][2] = w[p][3] = w[p][4] = w[p][5] = w[p][6] = w[p][7] = 1.f;
        }
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const int64_t t = t1 + 16 * j;
            if constexpr (GATED)
                if (j % A == 0) {
#pragma unroll
                    for (int p = 0; p < P; ++p)
#pragma unroll
                        for (int i = 0; i < A; ++i)
                            add[p][i] = addend(p, j + i, cb / G);
                }
            if (!FULL && t >= a.T) continue;
            float v[P][8];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const int b = cb + (e >> 2) * P + p;
                    float sum = static_cast<float>(acc[b][j * DIG][e & 3]);
                    if constexpr (DIG == 2) sum = fmaf(256.f, sum, static_cast<float>(acc[b][j * DIG + 1][e & 3]));
                    v[p][e] = sum * s[j] * w[p][e];
                    if constexpr (GATED) v[p][e] += static_cast<float>(as_h8(add[p][j % A])[e]);
                }
            if constexpr (GATED) {
                if (a.kept && ODD) {
                    store8_odd<true>(a.kept + t * a.n + c, v[0]);
                    store8_odd<true>(a.kept + plane + t * a.n + c, v[1]);
                } else if (a.kept) {
                    store8<FULL, LINES, true>(a.kept + t * a.n, c, a.n, v[0]);
                    store8<FULL, LINES, true>(a.kept + plane + t * a.n, c, a.n, v[1]);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) v[0][e] = v[0][e] * __builtin_amdgcn_rcpf(1.f + __expf(-v[0][e])) * v[1][e];
            }
            if constexpr (ODD) store8_odd<false>(a.y + t * a.n + c, v[0]);
            else store8<FULL, STREAM, false>(a.y + t * a.n, c, a.n, v[0]);
        }
    }
}

// Row b * 16 + r of the workgroup's weight rows / token rows in memory.  Two weight blocks (gated: two of gate and two of up in turn) hold
// 32 columns such that rows 4 g .. 4 g + 3 of both are columns 8 g .. 8 g + 7: those that lane group g gets of the result.
template <bool GATED>
__device__ __forceinline__ const int8_t* weight_row(const ProductArgs& a, int64_t c0, int b, int r) {
    const int group = GATED ? b >> 2 : b >> 1, half = GATED ? (b >> 1) & 1 : b & 1, up = GATED ? b & 1 : 0;
    return a.w + (up * a.n + min(c0 + group * 32 + (r >> 2) * 8 + half * 4 + (r & 3), a.n - 1)) * a.ld;
}
template <int DIG>
__device__ __forceinline__ const int8_t* token_row(const ProductArgs& a, int64_t t0, int b, int r) {
    if constexpr (DIG == 2) return a.q + ((b & 1) * a.T + min(t0 + (b >> 1) * 16 + r, a.T - 1)) * a.ld;
    else return a.q + min(t0 + b * 16 + r, a.T - 1) * a.ld;
}

// Which tile a workgroup takes.  Workgroups go to the eight XCDs in turn, each with an L2 of its own: every XCD gets a contiguous eighth of the
// tiles, in groups of kGroup tiles along the tokens, so that those it runs at a time share rows of both operands.
constexpr uint32_t kGroup = 4;   // (2 .. 16 measured: 4 and 8 alike, 2 and 16 up to 6 % slower)
struct Tile {
    uint32_t c, t;
};
__device__ __forceinline__ Tile tile_of(uint32_t id, uint32_t nc, uint32_t nt) {
    const uint32_t n = nc * nt, xcd = id & 7, each = n / 8, rest = n % 8;
    const uint32_t i = xcd * each + min(xcd, rest) + (id >> 3);
    const uint32_t g = i / (kGroup * nc), in = i % (kGroup * nc), size = min(kGroup, nt - g * kGroup);
    return {in / size, g * kGroup + in % size};
}

// A few tokens' rows brought to digits by the workgroup itself (OWN_ROWS): x comes into LDS the way of the weights, ahead of them, and its 8-bit rows are
// kept there.  Behind the ring: x, rows of whole KiB; the rows, a.ld bytes each; their scales.  OWN_ROWS = 2: rows that do not consist of aligned 16-byte
// pieces are read through registers, twice, behind the weights that have been requested (loads return in order).
__device__ __forceinline__ int8_t* own_rows_at(const ProductArgs& a, int8_t* lds) { return lds + a.T * own_x_bytes(a.d_in); }
__device__ __forceinline__ float* own_scales_at(const ProductArgs& a, int8_t* lds) { return reinterpret_cast<float*>(own_rows_at(a, lds) + a.T * a.ld); }

template <int THREADS>
__device__ __forceinline__ void own_rows_request(const ProductArgs& a, int8_t* lds) {
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds)), per = static_cast<uint32_t>(own_x_bytes(a.d_in) / 1024);
    const uint32_t last = static_cast<uint32_t>(a.d_in * 2) - 16;   // (whole 16-byte pieces: d_in is a multiple of 8)
    for (uint32_t k = wave; k < per * static_cast<uint32_t>(a.T); k += THREADS / 64) {
        const uint32_t t = k / per, at = min(k % per * 1024u + lane * 16u, last);
        load16_to_lds<false>(base + k * 1024u, reinterpret_cast<const int8_t*>(a.x + t * a.d_in) + at);
    }
}

// LATER: loads that this wave has requested since
template <int THREADS, int LATER, bool PIECES>
__device__ __forceinline__ void own_rows(const ProductArgs& a, int8_t* lds) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    int8_t* const rows = own_rows_at(a, lds);
    float* const scales = own_scales_at(a, lds);
    uint32_t* const part = reinterpret_cast<uint32_t*>(scales + 16);   // [token][wave]
    if constexpr (PIECES) {
        asm volatile("s_waitcnt vmcnt(%0)" :: "n"(LATER) : "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
    const uint32_t groups = static_cast<uint32_t>((a.d_in + 7) / 8), all = static_cast<uint32_t>(a.ld / 8);
    auto group_of = [&](int t, uint32_t k) {
        if constexpr (PIECES) return reinterpret_cast<const u4*>(lds + t * own_x_bytes(a.d_in))[k];
        else return load_part(a.x + t * a.d_in, 8 * static_cast<int64_t>(k), a.d_in);
    };
    for (int t = 0; t < a.T; ++t) {
        uint32_t m = 0;   // (fp16 magnitudes as unsigned numbers, a NaN the largest)
        for (uint32_t k = threadIdx.x; k < groups; k += THREADS) {
            const u4 v = group_of(t, k);
#pragma unroll
            for (int e = 0; e < 4; ++e) m = max(m, max(v[e] & 0x7FFFu, v[e] >> 16 & 0x7FFFu));
        }
#pragma unroll
        for (int s = 32; s > 0; s >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
        if (lane == 0) part[t * (THREADS / 64) + wave] = m;
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);   // (LDS only: the weights stay on their way)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    for (int t = 0; t < a.T; ++t) {
        uint32_t m = part[t * (THREADS / 64)];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) m = max(m, part[t * (THREADS / 64) + w]);
        const RowScale s = scale_of(__float_as_uint(static_cast<float>(__builtin_bit_cast(_Float16, static_cast<uint16_t>(m)))), 127.f);
        if (threadIdx.x == 0) scales[t] = s.scale;
        for (uint32_t k = threadIdx.x; k < all; k += THREADS) {
            const h8 h = as_h8(k < groups ? group_of(t, k) : u4{0u, 0u, 0u, 0u});
            float f[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) f[e] = static_cast<float>(h[e]);
            uint2 q, none;
            digits_of<1>(f, s.inverse, q, none);
            *reinterpret_cast<uint2*>(rows + t * a.ld + 8 * k) = q;
        }
    }
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One workgroup: CT x TT sums (weight rows x token rows) by WC x WT waves; with WK > 1 as many of those side by side, each with its own 64 columns of a
// step (short steps wait for their barrier and for LDS, not for data: few tiles want long ones).  A ring of S slots in LDS holds the steps; the loads
// go straight into it, several steps ahead.
// A step's rows of 64 bytes lie there as four 16-byte pieces, piece p of row r at place p ^ (r / 2 mod 4): eight neighbouring
// lanes of an operand read (eight rows, one piece) then cover all banks (no conflicts counted).  Where a load's data goes follows from
// the lane, so it is the lane's address that is permuted.
// While a step's products run on one set of operand registers, the next step's operands are read into the other.
// The barrier of step k says that step k + 1 has landed and that everybody has read step k, whose slot then takes step k + S.
template <int CT, int TT, int WC, int WT, int WK, int S, int DIG, bool GATED, int OWN_ROWS = 0>
__global__ __launch_bounds__(64 * WC * WT * WK) void lordba_i8_product_kernel(ProductArgs a) {
    constexpr int NW = WC * WT * WK, CB = CT / 16 / WC, TB = TT / 16 / WT, NB = (OWN_ROWS ? CT : CT + TT) / 16, L = NB * WK / NW;
    constexpr uint32_t kPart = NB * 1024u, kSlot = WK * kPart;
    static_assert(NB * WK % NW == 0 && (S == 3 || S == 4), "whole loads per wave; the waits at the end");
    extern __shared__ int8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wt = wave / WC % WT, wk = wave / (WC * WT);
    constexpr int kCols = GATED ? CT / 2 : CT, kTokens = TT / DIG;
    const Tile tile = tile_of(a.first + blockIdx.x, static_cast<uint32_t>((a.n + kCols - 1) / kCols), static_cast<uint32_t>((a.T + kTokens - 1) / kTokens));
    const int64_t c0 = static_cast<int64_t>(tile.c) * kCols, t0 = static_cast<int64_t>(tile.t) * kTokens;
    // (SPLIT: this workgroup has the steps k0 .. k0 + K - 1 of the contraction)
    constexpr bool SPLIT = WC * WT <= 2 && WK > 1 && !OWN_ROWS;
    const int steps = (a.pieces + WK - 1) / WK;
    const int k0 = SPLIT ? static_cast<int>(static_cast<int64_t>(steps) * blockIdx.y / a.splits) : 0;
    const int K = SPLIT ? static_cast<int>(static_cast<int64_t>(steps) * (blockIdx.y + 1) / a.splits) - k0 : steps;

    const int8_t* src[L];
#pragma unroll
    for (int j = 0; j < L; ++j) {
        const int b = (wave * L + j) % NB, part = (wave * L + j) / NB, r = lane >> 2, piece = (lane & 3) ^ ((r >> 1) & 3);
        src[j] = (b < CT / 16 ? weight_row<GATED>(a, c0, b, r) : token_row<DIG>(a, t0, b - CT / 16, r)) + (k0 * WK + part) * 64 + 16 * piece;
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    uint32_t to = base + wave * L * 1024u, from = 0;   // the slot that the next step is requested into, and the one that is read next
    const uint32_t to_end = to + S * kSlot;
    auto request = [&] {
#pragma unroll
        for (int j = 0; j < L; ++j) {
            load16_to_lds<false>(to + j * 1024u, src[j]);
            src[j] += 64 * WK;
        }
        to = to + kSlot == to_end ? to_end - S * kSlot : to + kSlot;
    };
    if constexpr (OWN_ROWS != 0) {
        static_assert(DIG == 1 && TT == 16 && WC == 1 && WT == 1, "one block of tokens, read by every wave");
        if constexpr (OWN_ROWS == 1) own_rows_request<64 * NW>(a, lds + S * kSlot);
    }
#pragma unroll
    for (int k = 0; k < S; ++k)
        if (k < K) request();
    const int8_t* own = nullptr;
    if constexpr (OWN_ROWS != 0) {
        if (K >= S) own_rows<64 * NW, S * L, OWN_ROWS == 1>(a, lds + S * kSlot);
        else own_rows<64 * NW, 0, OWN_ROWS == 1>(a, lds + S * kSlot);
        own = own_rows_at(a, lds + S * kSlot) + min<int64_t>(lane & 15, a.T - 1) * a.ld + 64 * wk + 16 * (lane >> 4);
        a.q_scale = own_scales_at(a, lds + S * kSlot);
    }
    i4 acc[CB][TB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = i4{0, 0, 0, 0};
    i4 fc[2][CB], ft[2][TB];
    const int r = lane & 15, place = 16 * ((lane >> 4) ^ ((r >> 1) & 3));
    const int8_t* const at_c = lds + wk * kPart + wc * CB * 1024 + r * 64 + place;
    const int8_t* const at_t = lds + wk * kPart + (CT / 16 + wt * TB) * 1024 + r * 64 + place;
    auto read = [&](auto set) {
#pragma unroll
        for (int i = 0; i < CB; ++i) fc[set.value][i] = *reinterpret_cast<const i4*>(at_c + from + i * 1024);
        if constexpr (OWN_ROWS != 0) {
            ft[set.value][0] = *reinterpret_cast<const i4*>(own);
            if ((lane & 15) >= a.T) ft[set.value][0] = i4{0, 0, 0, 0};
            own += 64 * WK;
        } else {
#pragma unroll
            for (int i = 0; i < TB; ++i) ft[set.value][i] = *reinterpret_cast<const i4*>(at_t + from + i * 1024);
        }
        from = from + kSlot == S * kSlot ? 0 : from + kSlot;
    };
    auto multiply = [&](auto set) {
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fc[set.value][i], ft[set.value][j], acc[i][j], 0, 0, 0);
    };
    // The addends of a whole tile come the way of the operands: in the last S steps, when there is nothing left to request for the products, each lane
    // requests those that it will add itself (P planes, TB / DIG tokens, kN groups of columns, eight at a time) into its wave's share of the slots that fall
    // free.  The products hide what the loads wait for: with cold
    // weights 2048 x 4096 x 11008 203 -> 193 us, 4096 x 4096 x 11008 434 -> 367.
    constexpr int P = GATED ? 2 : 1, kN = CB / (2 * P), kAddends = P * (TB / DIG) * kN;
    constexpr bool kAhead = GATED && WK == 1 && kAddends <= L * S;
    const int64_t cw = c0 + wc * (kCols / WC), tw = t0 + wt * (kTokens / WT);
    const bool full = c0 + kCols <= a.n && t0 + kTokens <= a.T;
    const bool ahead = kAhead && full && a.addends && K >= S && a.n % 8 == 0 && (reinterpret_cast<uintptr_t>(a.addends) & 15) == 0;
    const _Float16* const mine = a.addends + (tw + (lane & 15)) * a.n + cw + 8 * (lane >> 4);
    auto addend_at = [&](int p, int j, int kn) { return mine + (p * a.T + 16 * j) * a.n + 32 * kn; };
    auto request_addends = [&](int part) {
#pragma unroll
        for (int j = 0; j < L; ++j) {   // (always L loads: the waits count on it)
            const int item = min(part * L + j, kAddends - 1);
            load16_to_lds<true>(to + j * 1024u, addend_at(item % P, item / P % (TB / DIG), item / (P * (TB / DIG))));
        }
        to = to + kSlot == to_end ? to_end - S * kSlot : to + kSlot;
    };
    // Of this wave's loads all but the youngest LATER steps' have landed, and its operands are in registers; then everybody's.  (The builtin, because
    // the compiler counts the reads of LDS along with it; it does not see the loads.)
    auto meet = [&](auto later) {
        constexpr int n = later.value * L;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt((n & 15) | (7 << 4) | ((n >> 4) << 14));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    // one operand read between every few products
    auto weave = [&] {
#pragma unroll
        for (int i = 0; i < CB + TB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, CB * TB / (CB + TB), 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, CB * TB % (CB + TB), 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    using N0 = std::integral_constant<int, 0>;
    using N1 = std::integral_constant<int, 1>;
    using Ring = std::integral_constant<int, S - 2>;
    if (K >= S) meet(Ring{});
    else meet(N0{});
    read(N0{});
    int k = 0;
    for (; k + S + 1 < K; k += 2) {
        meet(Ring{});
        request();
        read(N1{});
        multiply(N0{});
        weave();
        meet(Ring{});
        request();
        read(N0{});
        multiply(N1{});
        weave();
    }
    // The last steps, S + 1 at most: step k + i + 1 has landed when at most as many are on their way as come behind it.
    auto last = [&](auto self, auto i) {
        constexpr int n = i.value;
        using This = std::integral_constant<int, n & 1>;
        using Next = std::integral_constant<int, 1 - (n & 1)>;
        if (k + n + 1 < K) {
            const int behind = ahead ? S : K - 2 - (k + n);
            if (behind >= S - 2) meet(Ring{});
            else if (S > 3 && behind == 1) meet(N1{});
            else meet(N0{});
            if (k + n + S < K) request();
            else if (ahead) request_addends(k + n + S - K);
            read(Next{});
        } else if (ahead) {   // (everybody has the last step's operands)
            meet(Ring{});
            request_addends(S - 1);
        }
        multiply(This{});
        if constexpr (n < S)
            if (k + n + 1 < K) self(self, std::integral_constant<int, n + 1>{});
    };
    last(last, N0{});
    if constexpr (WK > 1) {   // the parts' sums meet in LDS, in the order of the parts
        static_assert((WK - 1) * CT * TT * 4 <= S * kSlot, "the sums fit the ring");
        i4* const sums = reinterpret_cast<i4*>(lds) + (wc + WC * wt) * CB * TB * 64 + lane;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j)
                if (wk > 0) sums[((wk - 1) * WC * WT * CB * TB + i * TB + j) * 64] = acc[i][j];
        __syncthreads();
        if (wk > 0) return;
#pragma unroll
        for (int p = 0; p < WK - 1; ++p)
#pragma unroll
            for (int i = 0; i < CB; ++i)
#pragma unroll
                for (int j = 0; j < TB; ++j) acc[i][j] += sums[(p * WC * WT * CB * TB + i * TB + j) * 64];
    }
    if constexpr (SPLIT) {
        // The last workgroup of a tile to arrive joins the parts (each of its waves its own blocks): whole numbers, any order gives the same sum.  The parts go through the memory that all XCDs
        // share, piece by piece (accesses of agent scope), not by a fence, which would have the XCD's whole L2 written back (3 us more).
        if (a.splits > 1) {
            const uint32_t mine_of = blockIdx.x * (WC * WT) + wave % (WC * WT);
            uint64_t* const parts = reinterpret_cast<uint64_t*>(a.parts) + static_cast<int64_t>(mine_of) * (CB * TB * 128) + lane;
            const int64_t apart = static_cast<int64_t>(gridDim.x) * (WC * WT * CB * TB * 128);
            typedef uint64_t l2v __attribute__((ext_vector_type(2)));
#pragma unroll
            for (int i = 0; i < CB * TB; ++i) {
                const l2v v = __builtin_bit_cast(l2v, acc[i / TB][i % TB]);
#pragma unroll
                for (int k = 0; k < 2; ++k) __hip_atomic_store(parts + blockIdx.y * apart + i * 128 + k * 64, v[k], __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            }
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // (the parts are there before the arrival is counted)
            uint32_t before = 0;
            if (lane == 0) before = __hip_atomic_fetch_add(a.arrived + mine_of, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            if (__builtin_amdgcn_readfirstlane(before) + 1 != a.splits) return;
            asm volatile("" ::: "memory");
            // several parts are on their way at a time: each way takes about a microsecond
            constexpr uint32_t kTogether = CB * TB > 4 ? 4 : 8;
            for (uint32_t p0 = 0; p0 < a.splits; p0 += kTogether) {
                uint64_t v[kTogether][CB * TB][2];
#pragma unroll
                for (uint32_t u = 0; u < kTogether; ++u)
#pragma unroll
                    for (int i = 0; i < CB * TB; ++i)
#pragma unroll
                        for (int k = 0; k < 2; ++k)
                            v[u][i][k] = __hip_atomic_load(parts + min(p0 + u, a.splits - 1) * apart + i * 128 + k * 64, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
                for (uint32_t u = 0; u < kTogether; ++u)
                    if (p0 + u < a.splits && p0 + u != blockIdx.y)
#pragma unroll
                        for (int i = 0; i < CB * TB; ++i) acc[i / TB][i % TB] += __builtin_bit_cast(i4, l2v{v[u][i][0], v[u][i][1]});
            }
        }
    }
    // What only the backward pass wants goes past the caches, which hold rows that the products still need: 512 x 4096 x 11008 60 -> 54 us,
    // 4096 x 4096 x 11008 386 -> 371, 8192 x 1024 x 8192 262 -> 237; pieces of lines that others finish do not (4096 x 500 x 4088 49 -> 69 if they did).
    // y too where it is more than the caches of the XCDs hold twice over.  Plain products take the same time either way.
    auto finish_tile = [&](auto addend) {
        using No = std::false_type;
        using Yes = std::true_type;
        auto go = [&](auto whole, auto odd, auto lines, auto stream) {
            finish<CB, TB, DIG, GATED, whole.value, odd.value, lines.value, stream.value>(a, acc, cw, tw, addend);
        };
        if (!full) go(No{}, No{}, No{}, No{});
        else if ((a.n & 1) || ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.kept)) & 2)) go(Yes{}, Yes{}, No{}, No{});
        else if (!GATED || a.n % 32 != 0 || ((reinterpret_cast<uintptr_t>(a.y) | reinterpret_cast<uintptr_t>(a.kept)) & 63) != 0) go(Yes{}, No{}, No{}, No{});
        else if (TT < 256 || a.T * a.n < (1 << 25)) go(Yes{}, No{}, Yes{}, No{});
        else go(Yes{}, No{}, Yes{}, Yes{});
    };
    auto from_memory = [&](int p, int j, int kn) {
        const int64_t t = tw + (lane & 15) + 16 * j, c = cw + 8 * (lane >> 4) + 32 * kn;
        return a.addends && t < a.T ? load_part(a.addends + (p * a.T + t) * a.n, c, a.n) : u4{0u, 0u, 0u, 0u};
    };
    if constexpr (kAhead) {
        if (ahead) {
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            auto from_lds = [&](int p, int j, int kn) {   // (part 0 lies where the next would go)
                const int item = p + P * (j + TB / DIG * kn);
                const uint32_t at = to + item / L * kSlot;
                return *reinterpret_cast<const u4*>(lds + ((at >= to_end ? at - S * kSlot : at) - base) + item % L * 1024u + lane * 16u);
            };
            finish_tile(from_lds);
            return;
        }
    }
    finish_tile(from_memory);
}

template <int CT, int TT, int WC, int WT, int WK, int S, int DIG, bool GATED, int OWN_ROWS = 0>
lordba_status product_launch(const ProductArgs& a, hipStream_t stream) {
    constexpr int kCols = GATED ? CT / 2 : CT, kTokens = TT / DIG;
    constexpr size_t kRing = S * WK * (OWN_ROWS ? CT : CT + TT) * 64;
    const size_t lds = kRing + (OWN_ROWS ? static_cast<size_t>(own_bytes(a.T, a.d_in, a.ld)) : 0);
    static_assert(kRing <= kLdsBytes, "LDS of a compute unit");
    if (OWN_ROWS || kRing > 64 * 1024) {   // (once for a device: more LDS than a launch gets unasked)
        static std::atomic<uint64_t> asked{0};
        int device = 0;
        if (hipGetDevice(&device) != hipSuccess || device < 0 || device >= 64) return LORDBA_ERR_NO_DEVICE;
        if (!(asked.load(std::memory_order_relaxed) >> device & 1)) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(lordba_i8_product_kernel<CT, TT, WC, WT, WK, S, DIG, GATED, OWN_ROWS>),
                                    hipFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(OWN_ROWS ? kLdsBytes : kRing)) != hipSuccess) {
                (void)hipGetLastError();
                return LORDBA_ERR_LAUNCH;
            }
            asked.fetch_or(static_cast<uint64_t>(1) << device, std::memory_order_relaxed);
        }
    }
    const int64_t tiles = (a.n + kCols - 1) / kCols * ((a.T + kTokens - 1) / kTokens);
    if (tiles > INT32_MAX) return LORDBA_ERR_DIM;
    constexpr int64_t kMost = (static_cast<int64_t>(1) << 31) / (64 * WC * WT * WK);   // (a launch counts threads in 32 bits)
    for (int64_t first = 0; first < tiles; first += kMost) {
        ProductArgs part = a;
        part.first = static_cast<uint32_t>(first);
        hipLaunchKernelGGL((lordba_i8_product_kernel<CT, TT, WC, WT, WK, S, DIG, GATED, OWN_ROWS>),
                           dim3(static_cast<unsigned>(std::min(kMost, tiles - first)), a.splits), dim3(64 * WC * WT * WK), lds, stream, part);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
    }
    return LORDBA_OK;
}

template <int DIG, bool GATED>
lordba_status product(ProductArgs a, hipStream_t stream) {
    const Choice choice = i8_choice(a.T, 64 * static_cast<int64_t>(a.pieces), a.n, DIG, GATED, a.arrived != nullptr);
    a.splits = choice.splits;
    switch (choice.tile) {
        case 0: return product_launch<256, 256, 4, 2, 1, 4, DIG, GATED>(a, stream);
        case 1: return product_launch<256, 128, 4, 2, 1, 4, DIG, GATED>(a, stream);
        case 2: return product_launch<128, 128, 2, 4, 1, 4, DIG, GATED>(a, stream);
        case 3: return product_launch<64, 64, 1, 2, 2, 4, DIG, GATED>(a, stream);
        case 4:
            if constexpr (!GATED) return product_launch<32, 64, 1, 2, 2, 4, DIG, GATED>(a, stream);
            [[fallthrough]];
        case 5: return product_launch<GATED ? 64 : 32, 32, 1, 1, GATED ? 2 : 4, 4, DIG, GATED>(a, stream);
        default:
            if constexpr (DIG == 1) return product_launch<GATED ? 64 : 32, 16, 1, 1, GATED ? 2 : 4, 4, DIG, GATED>(a, stream);
            return LORDBA_ERR_LAUNCH;   // (cheapest_tile does not name it)
    }
}

template <bool GATED>
lordba_status own_rows_product(const ProductArgs& a, int from, hipStream_t stream) {
    if (from == 1) return product_launch<GATED ? 64 : 32, 16, 1, 1, 4, 4, 1, GATED, 1>(a, stream);
    return product_launch<GATED ? 64 : 32, 16, 1, 1, 4, 4, 1, GATED, 2>(a, stream);
}

// What the four entry points check alike.
lordba_status check(int64_t T, int64_t d_in, int64_t d_out, int64_t contracted, int digits) {
    if (T < 0 || T > INT32_MAX || d_in < 1 || d_out < 1 || d_in > (1 << 24) || d_out > (1 << 24) || contracted > LORDBA_I8_MAX_COLUMNS) return LORDBA_ERR_DIM;
    return digits < 1 || digits > 2 ? LORDBA_ERR_VALUE : LORDBA_OK;
}

struct Workspace {
    int8_t* q;
    float* scale;
    uint32_t* arrived;   // counters that the row kernel clears ahead of the product; null: the product's contraction is not shared
    int32_t* parts;
    size_t bytes;        // that the call may write to
};
Workspace split(void* workspace, size_t bytes, int64_t T, int64_t cols, int digits) {
    char* const p = static_cast<char*>(workspace);
    char* const more = p + i8_split_offset(T, cols, digits);
    const bool room = i8_splits(T, cols, digits) && bytes >= i8_workspace_bytes(T, cols, digits);
    return {reinterpret_cast<int8_t*>(p), reinterpret_cast<float*>(p + i8_scale_offset(T, cols, digits)), room ? reinterpret_cast<uint32_t*>(more) : nullptr,
            reinterpret_cast<int32_t*>(more + kI8SplitTiles * 4), room ? i8_workspace_bytes(T, cols, digits) : i8_least_workspace_bytes(T, cols, digits)};
}

// y = x diag(col_scale) W^T diag(w_scale) over `contracted` columns
lordba_status linear(const void* x, const float* col_scale, const int8_t* w, const float* w_scale, void* y, void* workspace, size_t workspace_bytes,
                     int64_t T, int64_t contracted, int64_t n, int digits, void* stream) {
    if (T == 0) return LORDBA_OK;
    const float* scale = col_scale ? col_scale : w_scale;
    if (!x || !w || !scale || !y || !workspace) return LORDBA_ERR_NULL;
    if (workspace_bytes < i8_least_workspace_bytes(T, contracted, digits)) return LORDBA_ERR_WORKSPACE;
    const Workspace ws = split(workspace, workspace_bytes, T, contracted, digits);
    if (i8_misaligned(x, 2) || i8_misaligned(w, 16) || i8_misaligned(scale, 4) || i8_misaligned(y, 2) || i8_misaligned(workspace, 16)) return LORDBA_ERR_ALIGN;
    const Span out[] = {{y, static_cast<size_t>(T) * n * 2}, {workspace, ws.bytes}};
    const Span in[] = {{x, static_cast<size_t>(T) * contracted * 2}, {w, static_cast<size_t>(n) * i8_row_bytes(contracted)},
                       {scale, static_cast<size_t>(col_scale ? contracted : n) * 4}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const ProductArgs a = {w, ws.q, ws.scale, w_scale, nullptr, static_cast<_Float16*>(y), nullptr, T, n, i8_row_bytes(contracted), static_cast<int>(i8_pieces(contracted)),
                           static_cast<const _Float16*>(x), contracted, ws.parts, ws.arrived, 1, 0};
    if (const int own = col_scale ? 0 : i8_own_rows(T, contracted, digits, false, !i8_misaligned(x, 16))) return own_rows_product<false>(a, own, st);
    const lordba_status rows = lordba_i8_quantize(x, col_scale, ws.q, ws.scale, ws.arrived, T, contracted, digits, st);
    if (rows != LORDBA_OK) return rows;
    return digits == 1 ? product<1, false>(a, st) : product<2, false>(a, st);
}

}  // namespace

extern "C" lordba_status lordba_linear_i8(const void* x, const int8_t* W, const float* w_scale, void* y, void* workspace, size_t workspace_bytes,
                                          int64_t T, int64_t d_in, int64_t d_out, int digits, void* stream) {
    const lordba_status st = check(T, d_in, d_out, d_in, digits);
    return st != LORDBA_OK ? st : linear(x, nullptr, W, w_scale, y, workspace, workspace_bytes, T, d_in, d_out, digits, stream);
}

extern "C" lordba_status lordba_linear_i8_backward(const void* g, const int8_t* Wt, const float* w_scale, void* dx, void* workspace,
                                                   size_t workspace_bytes, int64_t T, int64_t d_in, int64_t d_out, int digits, void* stream) {
    const lordba_status st = check(T, d_in, d_out, d_out, digits);
    if (st != LORDBA_OK) return st;
    if (T > 0 && !w_scale) return LORDBA_ERR_NULL;
    return linear(g, w_scale, Wt, nullptr, dx, workspace, workspace_bytes, T, d_out, d_in, digits, stream);
}

extern "C" lordba_status lordba_gated_i8(const void* x, const int8_t* W, const float* w_scale, const void* addends, void* h, void* gate_up,
                                         void* workspace, size_t workspace_bytes, int64_t T, int64_t d_in, int64_t d_ff, int digits, void* stream) {
    lordba_status st = check(T, d_in, d_ff, d_in, digits);
    if (st != LORDBA_OK || T == 0) return st;
    if (!x || !W || !w_scale || !h || !workspace) return LORDBA_ERR_NULL;
    if (workspace_bytes < i8_least_workspace_bytes(T, d_in, digits)) return LORDBA_ERR_WORKSPACE;
    const Workspace ws = split(workspace, workspace_bytes, T, d_in, digits);
    if (i8_misaligned(x, 2) || i8_misaligned(W, 16) || i8_misaligned(w_scale, 4) || i8_misaligned(addends, 2) || i8_misaligned(h, 2) ||
        i8_misaligned(gate_up, 2) || i8_misaligned(workspace, 16))
        return LORDBA_ERR_ALIGN;
    const size_t nh = static_cast<size_t>(T) * d_ff * 2;
    const Span out[] = {{h, nh}, {gate_up, 2 * nh}, {workspace, ws.bytes}};
    const Span in[] = {{x, static_cast<size_t>(T) * d_in * 2}, {W, static_cast<size_t>(2 * d_ff) * i8_row_bytes(d_in)},
                       {w_scale, static_cast<size_t>(2 * d_ff) * 4}, {addends, 2 * nh}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const ProductArgs a = {W, ws.q, ws.scale, w_scale, static_cast<const _Float16*>(addends), static_cast<_Float16*>(h), static_cast<_Float16*>(gate_up),
                           T, d_ff, i8_row_bytes(d_in), static_cast<int>(i8_pieces(d_in)), static_cast<const _Float16*>(x), d_in, ws.parts, ws.arrived, 1, 0};
    if (const int own = i8_own_rows(T, d_in, digits, true, !i8_misaligned(x, 16))) return own_rows_product<true>(a, own, s);
    if ((st = lordba_i8_quantize(x, nullptr, ws.q, ws.scale, ws.arrived, T, d_in, digits, s)) != LORDBA_OK) return st;
    return digits == 1 ? product<1, true>(a, s) : product<2, true>(a, s);
}

extern "C" lordba_status lordba_gated_i8_backward(const void* dh, const void* gate_up, const int8_t* Wt, const float* w_scale, void* dx,
                                                  void* dgate_up, void* workspace, size_t workspace_bytes, int64_t T, int64_t d_in,
                                                  int64_t d_ff, int digits, void* stream) {
    lordba_status st = check(T, d_in, d_ff, 2 * d_ff, digits);
    if (st != LORDBA_OK || T == 0) return st;
    if (!dh || !gate_up || !Wt || !w_scale || !dx || !dgate_up || !workspace) return LORDBA_ERR_NULL;
    if (workspace_bytes < i8_least_workspace_bytes(T, 2 * d_ff, digits)) return LORDBA_ERR_WORKSPACE;
    const Workspace ws = split(workspace, workspace_bytes, T, 2 * d_ff, digits);
    if (i8_misaligned(dh, 2) || i8_misaligned(gate_up, 2) || i8_misaligned(Wt, 16) || i8_misaligned(w_scale, 4) || i8_misaligned(dx, 2) ||
        i8_misaligned(dgate_up, 2) || i8_misaligned(workspace, 16))
        return LORDBA_ERR_ALIGN;
    const size_t nh = static_cast<size_t>(T) * d_ff * 2;
    const Span out[] = {{dx, static_cast<size_t>(T) * d_in * 2}, {dgate_up, 2 * nh}, {workspace, ws.bytes}};
    const Span in[] = {{dh, nh}, {gate_up, 2 * nh}, {Wt, static_cast<size_t>(d_in) * i8_row_bytes(2 * d_ff)}, {w_scale, static_cast<size_t>(2 * d_ff) * 4}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    if ((st = lordba_i8_gated_grad(dh, gate_up, w_scale, dgate_up, ws.q, ws.scale, ws.arrived, T, d_ff, digits, s)) != LORDBA_OK) return st;
    const ProductArgs a = {Wt, ws.q, ws.scale, nullptr, nullptr, static_cast<_Float16*>(dx), nullptr, T, d_in, i8_row_bytes(2 * d_ff), static_cast<int>(i8_pieces(2 * d_ff)), nullptr, 0, ws.parts, ws.arrived, 1, 0};
    return digits == 1 ? product<1, false>(a, s) : product<2, false>(a, s);
}
