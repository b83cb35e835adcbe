// Products with 4-bit weights: arguments, operands and results, shared by the kernels for few tokens and those for many.
//
// The weights' rows are the first operand of v_mfma_f32_16x16x32_f16, the tokens the second, so that a lane's four accumulators are four
// consecutive columns of y for one token.
#pragma once
#include "lordba_dev_util.h"
#include "lordba_i4.h"
#include "lordba_i4_choice.h"
#include "lordba_results.h"

struct I4Args {
    const _Float16* x;         // [planes, T, k]: the activations' rows, `k` columns of each plane
    const uint8_t* codes;      // laid out, see lordba_i4.h
    const uint16_t *scale, *zero;   // zero: null for 8 everywhere
    const _Float16* addends;   // gated: [2, T, n], or null
    _Float16* y;               // [T, n]
    _Float16* kept;            // gated: [2, T, n], or null
    const _Float16 *dh, *gate_up;   // the gated block's gradient: what x was made of, [T, k] and [2, T, k]; otherwise null
    int64_t T, k, n;
    int32_t blocks, plane_blocks;   // of 128 columns: in all, of a plane
    int32_t tiles;             // blocks of 16 rows of a half
    int32_t groups;            // forward: along a row, padding included
    int32_t shift;             // backward: log2 of the group
    int32_t columns;           // few tokens: that LDS holds at a time
    int32_t aligned;           // whether rows of x consist of aligned 16-byte pieces
    uint32_t first;            // tile of this launch's first workgroup
};

namespace {

[[maybe_unused]] constexpr lordba_status (*kCheckDevice)() = check_device;   // (which the entry points alone call)

// Sixteen bytes a lane into LDS, from a uniform base and a byte offset per lane.
__device__ __forceinline__ void load16_to_lds_from(uint32_t lds, const void* base, uint32_t byte_off) {
    const uint64_t b = reinterpret_cast<uint64_t>(base);   // (into scalar registers, also where the compiler does not see that it is uniform)
    const uint64_t u = static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b))) |
                       static_cast<uint64_t>(static_cast<uint32_t>(__builtin_amdgcn_readfirstlane(static_cast<int>(b >> 32)))) << 32;
    asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(byte_off), "s"(u), "{m0}"(lds) : "memory");
}

__device__ __forceinline__ h2 both(uint16_t v) { return as_h2(v * 0x10001u); }

// The eight numbers code - zero of a word, exact in fp16.  With the biased exponent 0x64 a code in the low four bits of a half is 1024 + code, one four
// bits further up 1024 + 16 code; `z` is 1024 + zero, one for all eight (forward) or one each (backward).
struct Zero1 {
    h2 low, high;   // 1024 + zero, -(64 + zero)
    __device__ __forceinline__ explicit Zero1(uint16_t bits) : low(both(bits)), high(h2{static_cast<_Float16>(960), static_cast<_Float16>(960)} - both(bits)) {}
    __device__ __forceinline__ h2 low_of(int) const { return low; }
    __device__ __forceinline__ h2 high_of(int) const { return high; }
};
struct Zero8 {
    u4 z;
    __device__ __forceinline__ h2 low_of(int p) const { return as_h2(z[p]); }
    __device__ __forceinline__ h2 high_of(int p) const { return h2{static_cast<_Float16>(960), static_cast<_Float16>(960)} - as_h2(z[p]); }
};
// The exponent's bits in a vector register: with the mask in a scalar one, "and" and "or" are one instruction (constants in the instruction itself make two).
__device__ __forceinline__ uint32_t exponent() {
    uint32_t v = 0x64006400u;
    asm("" : "+v"(v));
    return v;
}
template <class Z>
__device__ __forceinline__ h8 operand(uint32_t w, const Z& z, uint32_t exp) {
    const h2 sixteenth = {static_cast<_Float16>(0.0625f), static_cast<_Float16>(0.0625f)};
    auto low = [&](uint32_t v, int p) { return as_h2((v & 0x000F000Fu) | exp) - z.low_of(p); };
    auto high = [&](uint32_t v, int p) { return __builtin_elementwise_fma(as_h2((v & 0x00F000F0u) | exp), sixteenth, z.high_of(p)); };
    const h2 a = low(w, 0), b = high(w, 1), c = low(w >> 8, 2), d = high(w >> 8, 3);
    return h8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

__device__ __forceinline__ f4 mfma(h8 a, h8 b, f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// For the backward pass: what passes the range of fp16 is kept as its largest number, a NaN as one.
__device__ __forceinline__ _Float16 kept_half(float v) { return static_cast<_Float16>(v != v ? v : fminf(fmaxf(v, -65504.f), 65504.f)); }

// The gated block's gradient at columns c .. c + N - 1 (c a multiple of N) of token t once more, of dgate and dup before they are rounded to fp16: where one of
// them passes its range, the product has an infinity times every weight, those that are 0 among them, in place of a number, in all of the token's columns.
// One lane alone, in fp32 (weights unrounded), a block of 128 columns by itself so that sums stay short.  What is no number by itself is left as the product gave it.
// 2048 tokens of 4096 <- 2 x 11008, all of them past the range: 54 ms (in range the call takes 0.39, and as long as without the question).
__device__ __forceinline__ bool number(float v) { return fabsf(v) < __builtin_inff(); }
template <int N>
__device__ __forceinline__ void from_unrounded(const I4Args& a, int64_t t, int64_t c) {
    if (c >= a.n) return;
    const int row = static_cast<int>(c & 31), in = 4 * (row >> 3) + (row & 3);   // c's place in a pair of blocks: i4_row() the other way round
    const int64_t tile = 2 * (c >> 5) + (row >> 2 & 1), scales = (c >> a.shift) * a.blocks * kI4Columns;
    const uint32_t* const codes = reinterpret_cast<const uint32_t*>(a.codes);
    float sum[N];
#pragma unroll
    for (int e = 0; e < N; ++e) sum[e] = 0.f;
    for (int b = 0; b < a.blocks; ++b) {
        const int half = b >= a.plane_blocks;
        const int64_t j0 = static_cast<int64_t>(b - half * a.plane_blocks) * kI4Columns;
        const _Float16 *const d = a.dh + t * a.k, *const g = a.gate_up + t * a.k, *const u = g + a.T * a.k;
        float part[N];
#pragma unroll
        for (int e = 0; e < N; ++e) part[e] = 0.f;
        for (int w = 0; w < 16 && j0 + 8 * w < a.k; ++w) {
            const h8 hd = as_h8(load_part(d, j0 + 8 * w, a.k)), hg = as_h8(load_part(g, j0 + 8 * w, a.k)), hu = as_h8(load_part(u, j0 + 8 * w, a.k));
            const int64_t at = scales + static_cast<int64_t>(b) * kI4Columns + 8 * w;
            const h8 s = as_h8(load16(a.scale + at));
            const u4 z = a.zero ? load16(a.zero + at) : u4{kZero8 * 0x10001u, kZero8 * 0x10001u, kZero8 * 0x10001u, kZero8 * 0x10001u};
            float v[8];
            bool numbers = true;
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                float dg, du;
                slopes(static_cast<float>(hd[k]), static_cast<float>(hg[k]), static_cast<float>(hu[k]), dg, du);
                v[k] = half ? du : dg;
                v[k] *= static_cast<float>(s[k]);
                numbers = numbers && number(v[k]);
            }
            if (!numbers) return;
#pragma unroll
            for (int e = 0; e < N; ++e) {
                const int at_row = in + (e & 3);
                const uint32_t code = codes[(((tile + (e >> 2)) * a.blocks + b) * 64 + 16 * (w & 3) + at_row) * 4 + (w >> 2)];
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int zero = z[k >> 1] >> (16 * (k & 1)) & 15;
                    part[e] = fmaf(v[k], static_cast<float>(static_cast<int>(code >> (4 * i4_nibble(k)) & 15) - zero), part[e]);
                }
            }
        }
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] += part[e];
    }
#pragma unroll
    for (int e = 0; e < N; ++e)
        if (c + e < a.n) a.y[t * a.n + c + e] = static_cast<_Float16>(sum[e]);
}

__device__ __forceinline__ float silu(float v) { return v * __builtin_amdgcn_rcpf(1.f + __expf(-v)); }

}  // namespace

// The launches; arguments have been checked.
lordba_status lordba_i4_few(const I4Args& a, int64_t group, bool gated, bool backward, hipStream_t stream);
lordba_status lordba_i4_many(const I4Args& a, int kernel, int64_t group, bool gated, bool backward, hipStream_t stream);
