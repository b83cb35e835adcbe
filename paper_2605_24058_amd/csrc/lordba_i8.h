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

namespace {

constexpr int64_t kI8Step = 256;   // columns that a row is padded to: up to four waves share a step of 64 each

inline int64_t i8_row_bytes(int64_t cols) { return (cols + kI8Step - 1) / kI8Step * kI8Step; }

inline size_t i8_scale_offset(int64_t T, int64_t cols, int digits) {   // the rows' scales lie behind the rows in a workspace
    return (static_cast<size_t>(digits) * static_cast<size_t>(T) * static_cast<size_t>(i8_row_bytes(cols)) + 255) / 256 * 256;
}

inline bool i8_overlap(const void* p, size_t pn, const void* q, size_t qn) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(p), b = reinterpret_cast<uintptr_t>(q);
    return p && q && pn && qn && a < b + qn && b < a + pn;
}
inline bool i8_misaligned(const void* p, uintptr_t bytes) { return (reinterpret_cast<uintptr_t>(p) & (bytes - 1)) != 0; }

// Eight numbers of a row from column c < cols on, zeros from column `cols` on.  At a row's end all of them are requested before the first is
// looked at: one wait, not eight.
__device__ __forceinline__ u4 load_part(const _Float16* row, int64_t c, int64_t cols) {
    if (c + 8 <= cols) return load16_any(row + c);
    uint32_t h[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = reinterpret_cast<const uint16_t*>(row)[min(c + e, cols - 1)];
    u4 v;
#pragma unroll
    for (int e = 0; e < 8; e += 2) v[e >> 1] = (c + e < cols ? h[e] : 0u) | (c + e + 1 < cols ? h[e + 1] << 16 : 0u);
    return v;
}

inline lordba_status i8_launched() { return hipGetLastError() == hipSuccess ? LORDBA_OK : LORDBA_ERR_LAUNCH; }

}  // namespace

// The steps of the entry points; arguments have been checked.  Each enqueues one kernel.
lordba_status lordba_i8_quantize(const void* x, const float* col_scale, int8_t* q, float* scale, int64_t rows, int64_t cols, int digits,
                                 hipStream_t stream);
lordba_status lordba_i8_gated_grad(const void* dh, const void* gate_up, const float* w_scale, void* dgate_up, int8_t* q, float* scale,
                                   int64_t T, int64_t d_ff, int digits, hipStream_t stream);
