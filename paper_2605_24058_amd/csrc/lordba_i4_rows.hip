// 4-bit weights: fp16 weights to codes with group scales, the layout that the products read; the elementwise part of the gated block's backward pass.
// What bounds them is memory; all but the last run once for a program's weights.
#include <algorithm>

#include "lordba_dev_util.h"
#include "lordba_i4.h"
#include "lordba_results.h"

namespace {

typedef uint32_t u2_byte __attribute__((ext_vector_type(2), aligned(1)));   // eight codes

// ---- quantisation: a thread takes eight columns, the 4 to 16 lanes of a group find its range together -------------------
// 11008 x 4096: 54 us (a thread a group read rows 256 bytes apart: 1630).
struct QuantizeArgs {
    const _Float16* w;
    uint8_t* codes;
    _Float16* scale;
    uint8_t* zero;   // or null: symmetric
    int64_t rows, cols, group, groups;
};

__global__ __launch_bounds__(256) void lordba_quantize_i4_kernel(QuantizeArgs a) {
    const int lanes = static_cast<int>(a.group / 8);
    const int64_t per_row = a.groups * lanes, stride = static_cast<int64_t>(gridDim.x) * 256;   // a group's lanes are here or not together
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < a.rows * per_row; k += stride) {
        const int64_t row = k / per_row, c = k % per_row * 8;
        const h8 w = c < a.cols ? as_h8(load_part(a.w + row * a.cols, c, a.cols)) : h8{};   // (0 behind the row's end)
        float low = 0.f, high = 0.f, number = 1.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = static_cast<float>(w[e]);
            low = fminf(low, v), high = fmaxf(high, v);
            if (!(fabsf(v) < __builtin_inff())) number = 0.f;
        }
        for (int d = 1; d < lanes; d *= 2) {
            low = fminf(low, __shfl_xor(low, d)), high = fmaxf(high, __shfl_xor(high, d));
            number = fminf(number, __shfl_xor(number, d));
        }
        const float range = a.zero ? (high - low) / 15.f : fmaxf(high, -low) / 7.f;
        const _Float16 scale = number > 0.f ? static_cast<_Float16>(range) : static_cast<_Float16>(__builtin_nanf(""));
        const float s = static_cast<float>(scale);
        const bool flat = !(s > 0.f);   // (no weight but 0, or a range that fp16 does not hold, or no number)
        const float z = !a.zero ? 8.f : flat ? 0.f : fminf(rintf(-low / s), 15.f);
        if (threadIdx.x % lanes == 0) {
            a.scale[k / lanes] = scale;
            if (a.zero) a.zero[k / lanes] = static_cast<uint8_t>(z);
        }
        uint32_t q[2] = {0, 0};
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float v = flat ? z : rintf(static_cast<float>(w[e]) / s + z);
            q[e >> 2] |= static_cast<uint32_t>(fminf(fmaxf(v, 0.f), 15.f)) << (8 * (e & 3));
        }
        uint8_t* const to = a.codes + row * a.cols + c;
        if (c + 8 <= a.cols) {
            *reinterpret_cast<u2_byte*>(to) = u2_byte{q[0], q[1]};
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c + e < a.cols) to[e] = static_cast<uint8_t>(q[e >> 2] >> (8 * (e & 3)));
        }
    }
}

// ---- layout ---------------------------------------------------------------------------------------------------------
struct LayoutArgs {
    const uint8_t* codes;    // [rows, cols] of W
    const uint16_t* scale;   // [rows, groups]
    const uint8_t* zero;     // [rows, groups], or null
    uint32_t* out;
    uint16_t *out_scale, *out_zero;
    int64_t cols, group, groups;   // of W
    I4Shape s;
    bool transposed;
};

// A thread lays out a word, eight columns of a row, which are eight of W's too, or of a column of W.
// 11008 x 4096: 25 us, transposed 50 (each code's place found by itself: 104).
__global__ __launch_bounds__(256) void lordba_layout_i4_kernel(LayoutArgs a) {
    const int64_t words = a.s.tiles * a.s.blocks * 256, stride = static_cast<int64_t>(gridDim.x) * 256;
    const int64_t row_blocks = a.s.tiles / a.s.row_halves, col_blocks = a.s.blocks / a.s.col_halves;
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < words; k += stride) {
        const int64_t block = k >> 8, tile = block / a.s.blocks, at = block % a.s.blocks;
        const int lane = static_cast<int>(k >> 2) & 63, m = static_cast<int>(k) & 3;
        const int row_half = tile >= row_blocks, col_half = at >= col_blocks;
        const int64_t row = i4_row(tile - row_half * row_blocks, lane & 15);
        const int64_t c0 = (at - col_half * col_blocks) * kI4Columns + 32 * m + 8 * (lane >> 4);
        const int64_t r = row_half * a.s.rows + row, c = col_half * a.s.cols + c0;   // in the unpadded matrix
        const bool there = row < a.s.rows;
        uint32_t code[8];
        // Padding: what stands for 0, 8 where the scale is padding too and behind the end of a row, in a group that it has, the group's zero.
        const bool in_group = there && !a.transposed && a.zero && c < a.groups * a.group;
        const uint32_t none = in_group ? a.zero[r * a.groups + c / a.group] & 15u : 8u;
        if (there && !a.transposed && c0 + 8 <= a.s.cols) {
            const u2_byte q = *reinterpret_cast<const u2_byte*>(a.codes + r * a.cols + c);
#pragma unroll
            for (int e = 0; e < 8; ++e) code[e] = q[e >> 2] >> (8 * (e & 3)) & 15u;
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                code[e] = there && c0 + e < a.s.cols ? a.codes[a.transposed ? (c + e) * a.cols + r : r * a.cols + c + e] & 15u : none;
        }
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) v |= code[e] << (4 * i4_nibble(e));
        a.out[k] = v;
    }
    // Scales.  A padded place has code 8 and zero 8.  A padded group's scale is never NaN.
    const int64_t along = a.transposed ? a.s.blocks * kI4Columns : a.s.groups * 16;
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < a.s.scales; k += stride) {
        int64_t j, i;
        bool there;
        if (a.transposed) {   // [group][column]: any row of the group, here its first
            const int64_t c = k % along, per = a.s.blocks / a.s.col_halves * kI4Columns;
            i = k / along * a.group, j = c / per * a.s.cols + c % per;
            there = c % per < a.s.cols;
        } else {
            const int64_t tile = k / along, per = a.s.tiles / a.s.row_halves;
            const int64_t row = i4_row(tile % per, static_cast<int>(k & 15));
            i = (k % along >> 4) * a.group, j = tile / per * a.s.rows + row;
            there = row < a.s.rows && i < a.cols;
        }
        const int64_t at = there ? j * a.groups + i / a.group : 0;
        a.out_scale[k] = there ? a.scale[at] : 0;
        if (a.out_zero) a.out_zero[k] = there ? static_cast<uint16_t>(0x6400 + (a.zero[at] & 15)) : kZero8;
    }
}

// ---- the gated block's slopes ---------------------------------------------------------------------------------------
struct GatedGradArgs {
    const _Float16 *dh, *gate, *up;
    _Float16 *dgate, *dup;
    int64_t n;   // elements of a plane
};

__global__ __launch_bounds__(256) void lordba_i4_gated_grad_kernel(GatedGradArgs a) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256 * 8;
    for (int64_t k = (static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x) * 8; k < a.n; k += stride) {
        const h8 d = as_h8(load_part(a.dh, k, a.n)), g = as_h8(load_part(a.gate, k, a.n)), u = as_h8(load_part(a.up, k, a.n));
        h8 dg, du;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float vg, vu;
            slopes(static_cast<float>(d[e]), static_cast<float>(g[e]), static_cast<float>(u[e]), vg, vu);
            dg[e] = static_cast<_Float16>(vg), du[e] = static_cast<_Float16>(vu);
        }
        if (k + 8 <= a.n) {
            *reinterpret_cast<u4_any*>(a.dgate + k) = __builtin_bit_cast(u4, dg);
            *reinterpret_cast<u4_any*>(a.dup + k) = __builtin_bit_cast(u4, du);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (k + e < a.n) a.dgate[k + e] = dg[e], a.dup[k + e] = du[e];
        }
    }
}

unsigned grid_for(int64_t threads) { return static_cast<unsigned>(std::min<int64_t>((threads + 255) / 256, 1 << 16)); }

}  // namespace

lordba_status lordba_i4_gated_grad(const void* dh, const void* gate_up, void* dgate_up, int64_t T, int64_t d_ff, hipStream_t stream) {
    const int64_t n = T * d_ff;
    const _Float16* const gu = static_cast<const _Float16*>(gate_up);
    _Float16* const out = static_cast<_Float16*>(dgate_up);
    const GatedGradArgs a = {static_cast<const _Float16*>(dh), gu, gu + n, out, out + n, n};
    hipLaunchKernelGGL(lordba_i4_gated_grad_kernel, dim3(grid_for((n + 7) / 8)), dim3(256), 0, stream, a);
    return i8_launched();
}

extern "C" size_t lordba_i4_code_bytes(int64_t rows, int64_t cols, int halves, int transposed) {
    if (rows < 1 || cols < 1 || rows > kI4Most || cols > kI4Most || halves < 1 || halves > 2 || rows % halves) return 0;
    const I4Shape s = i4_shape(rows, cols, 128, halves, transposed != 0);
    return static_cast<size_t>(s.tiles) * static_cast<size_t>(s.blocks) * 1024;
}

extern "C" size_t lordba_i4_scale_count(int64_t rows, int64_t cols, int64_t group, int halves, int transposed) {
    if (rows < 1 || cols < 1 || rows > kI4Most || cols > kI4Most || halves < 1 || halves > 2 || rows % halves || !i4_group(group)) return 0;
    return static_cast<size_t>(i4_shape(rows, cols, group, halves, transposed != 0).scales);
}

extern "C" lordba_status lordba_quantize_i4(const void* w, uint8_t* codes, void* scale, uint8_t* zero, int64_t rows, int64_t cols, int64_t group,
                                            void* stream) {
    if (rows < 0 || cols < 1 || rows > kI4Most || cols > kI4Most) return LORDBA_ERR_DIM;
    if (!i4_group(group)) return LORDBA_ERR_VALUE;
    if (rows == 0) return LORDBA_OK;
    if (!w || !codes || !scale) return LORDBA_ERR_NULL;
    if (i8_misaligned(w, 2) || i8_misaligned(scale, 2)) return LORDBA_ERR_ALIGN;
    const int64_t groups = (cols + group - 1) / group;
    const size_t n = static_cast<size_t>(rows) * cols, ng = static_cast<size_t>(rows) * groups;
    const Span out[] = {{codes, n}, {scale, 2 * ng}, {zero, ng}};
    const Span in[] = {{w, 2 * n}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const QuantizeArgs a = {static_cast<const _Float16*>(w), codes, static_cast<_Float16*>(scale), zero, rows, cols, group, groups};
    hipLaunchKernelGGL(lordba_quantize_i4_kernel, dim3(grid_for(rows * groups * (group / 8))), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return i8_launched();
}

extern "C" lordba_status lordba_layout_i4(const uint8_t* codes, const void* scale, const uint8_t* zero, uint8_t* out, void* out_scale, void* out_zero,
                                          int64_t rows, int64_t cols, int64_t group, int halves, int transposed, void* stream) {
    if (rows < 1 || cols < 1 || rows > kI4Most || cols > kI4Most) return LORDBA_ERR_DIM;
    if (!i4_group(group) || halves < 1 || halves > 2 || rows % halves) return LORDBA_ERR_VALUE;
    if (!codes || !scale || !out || !out_scale || (zero && !out_zero)) return LORDBA_ERR_NULL;
    if (i8_misaligned(scale, 2) || i8_misaligned(out, 16) || i8_misaligned(out_scale, 16) || i8_misaligned(out_zero, 16)) return LORDBA_ERR_ALIGN;
    const I4Shape s = i4_shape(rows, cols, group, halves, transposed != 0);
    const int64_t groups = (cols + group - 1) / group;
    const size_t ng = static_cast<size_t>(rows) * groups, ns = static_cast<size_t>(s.scales) * 2;
    const Span to[] = {{out, static_cast<size_t>(s.tiles) * s.blocks * 1024}, {out_scale, ns}, {out_zero, ns}};
    const Span from[] = {{codes, static_cast<size_t>(rows) * cols}, {scale, 2 * ng}, {zero, ng}};
    if (aliased(to, from)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const LayoutArgs a = {codes, static_cast<const uint16_t*>(scale), zero, reinterpret_cast<uint32_t*>(out), static_cast<uint16_t*>(out_scale),
                          zero ? static_cast<uint16_t*>(out_zero) : nullptr, cols, group, groups, s, transposed != 0};
    hipLaunchKernelGGL(lordba_layout_i4_kernel, dim3(grid_for(s.tiles * s.blocks * 256)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
    return i8_launched();
}
