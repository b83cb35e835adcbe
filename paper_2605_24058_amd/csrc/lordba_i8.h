// 8-bit projections: what the row kernels, the product kernels and their entry points share.
//
// Rows.  A row of numbers v is held as q = rint(v * D / amax), scale = amax / D with amax = max |v| of the row: D = 127 for one digit,
// q in one int8; D = 127 * 256 for two, q = 256 * hi + lo with hi in [-127, 127] and lo in [-128, 127], both int8.  Rows are stored
// i8_row_bytes(columns) apart, zeros behind their last column, so that the product kernels contract whole steps without a test;
// with two digits all rows' hi come first, then all rows' lo.  A row without a number (amax not finite) gets the scale NaN and
// zeros, so that everything that depends on it is NaN; a row of zeros, or one whose largest is below 2^-100 (D / amax would overflow),
// the scale 0.
//
// Sums.  |q| <= 128 and |W| <= 128, so a sum over LORDBA_I8_MAX_COLUMNS = 131071 columns stays inside 32 bits: the contraction is exact, and
// what is rounded is the row (once, above), the scaled sum (fp32) and the result (fp16).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lordba.h"
#include "lordba_dev_util.h"
#include "lordba_host_util.h"
#include "lordba_i8_choice.h"

namespace {

inline size_t i8_scale_offset(int64_t T, int64_t cols, int digits) {   // the rows' scales lie behind the rows in a workspace
    return (static_cast<size_t>(digits) * static_cast<size_t>(T) * static_cast<size_t>(i8_row_bytes(cols)) + 255) / 256 * 256;
}

inline size_t i8_split_offset(int64_t T, int64_t cols, int digits) {
    return (i8_scale_offset(T, cols, digits) + static_cast<size_t>(T) * 4 + 255) / 256 * 256;
}
// What a call needs is up to here; what a contraction's sharing needs on top, it needs only where a contraction is shared.  (The size never falls with T up to here,
// but on the whole, where a longer batch shares nothing: a workspace for the longest batch has to serve shorter ones.)
inline size_t i8_least_workspace_bytes(int64_t T, int64_t cols, int digits) { return i8_split_offset(T, cols, digits); }
inline size_t i8_workspace_bytes(int64_t T, int64_t cols, int digits) {
    return i8_split_offset(T, cols, digits) + (i8_splits(T, cols, digits) ? kI8SplitTiles * (4 + 64 * 64 * 4) : 0);
}

inline bool i8_overlap(const void* p, size_t pn, const void* q, size_t qn) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return p && q && pn && qn && a < b + qn && b < a + pn;
}
inline bool i8_misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Eight numbers of a row from column c < cols on, zeros from column `cols` on.  At a row's end the row's last eight are read and moved down: one
// load, no entry by itself.  Rows of fewer than eight: all requested before the first is looked at.
__device__ __forceinline__ u4 load_part(const _Float16* row, int64_t c, int64_t cols) {
    if (c + 8 <= cols) return load16_any(row + c);
    if (cols >= 8) return drop_halves(load16_any(row + cols - 8), static_cast<int>(c + 8 - cols));
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = reinterpret_cast<const uint16_t*>(row)[min(c + e, cols - 1)];
    u4 v;
#pragma unroll
    for (int e = 0; e < 8; e += 2) v[e >> 1] = (c + e < cols ? h[e] : 0u) | (c + e + 1 < cols ? h[e + 1] << 16 : 0u);
    return v;
}

constexpr uint32_t kInfBits = 0x7F800000u;

struct RowScale {
    float inverse, scale;
};
// D / amax and amax / D, both correctly rounded; zeros and rows without a number as above.
__device__ __forceinline__ RowScale scale_of(uint32_t max_bits, float D) {
    const float amax = __uint_as_float(max_bits);
    if (max_bits >= kInfBits) return {0.f, __uint_as_float(0x7FC00000u)};
    if (amax < 0x1p-100f) return {0.f, 0.f};
    return {D / amax, amax / D};
}

// Eight numbers into their digits: bytes 0..7 of (hi, lo); with one digit all of it in hi.  Adding 1.5 * 2^23 rounds to an integer (ties to even) and
// leaves it in two's complement in the low bits of the sum; a byte permutation gathers the bytes of four sums.
template <int DIG>
__device__ __forceinline__ void digits_of(const float (&v)[8], float inverse, uint2& hi, uint2& lo) {
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        float q = v[e] * inverse;
        asm("" : "+v"(q));   // (two roundings, as the definition has it: not one fused operation)
        b[e] = __float_as_uint(q + 12582912.f);
    }
    auto gather = [](uint32_t b0, uint32_t b1, uint32_t b2, uint32_t b3, uint32_t pair) {   // byte `pair & 0xFF` of each
        return __builtin_amdgcn_perm(__builtin_amdgcn_perm(b3, b2, pair), __builtin_amdgcn_perm(b1, b0, pair), 0x05040100u);
    };
    const bool none = inverse == 0.f;   // (a row of zeros, or without a number: infinity times zero is no zero)
    if constexpr (DIG == 1) {
        hi = make_uint2(gather(b[0], b[1], b[2], b[3], 0x0400u), gather(b[4], b[5], b[6], b[7], 0x0400u));
    } else {
        lo = make_uint2(gather(b[0], b[1], b[2], b[3], 0x0400u), gather(b[4], b[5], b[6], b[7], 0x0400u));
#pragma unroll
        for (int e = 0; e < 8; ++e) b[e] += 128;
        hi = make_uint2(gather(b[0], b[1], b[2], b[3], 0x0501u), gather(b[4], b[5], b[6], b[7], 0x0501u));
        lo = none ? make_uint2(0, 0) : lo;
    }
    hi = none ? make_uint2(0, 0) : hi;
}

inline lordba_status i8_launched() { return hipGetLastError() == hipSuccess ? LORDBA_OK : LORDBA_ERR_LAUNCH; }

}  // namespace

// The steps of the entry points; arguments have been checked.  Each enqueues one kernel.
// `clear`: kI8SplitTiles words that the kernel sets to zero on its way, or null.
lordba_status lordba_i8_quantize(const void* x, const float* col_scale, int8_t* q, float* scale, uint32_t* clear, int64_t rows, int64_t cols,
                                 int digits, hipStream_t stream);
lordba_status lordba_i8_gated_grad(const void* dh, const void* gate_up, const float* w_scale, void* dgate_up, int8_t* q, float* scale,
                                   uint32_t* clear, int64_t T, int64_t d_ff, int digits, hipStream_t stream);
