// 4-bit weights: fp16 weights to codes with group scales, the layout that the products read; the elementwise part of the gated block's backward pass.
// What bounds them is memory; all but the last run once for a program's weights.
#include <algorithm>

#include "lordba_dev_util.h"
#include "lordba_i4.h"
#include "lordba_results.h"

namespace {

// ---- quantisation: a thread takes a group of a row ------------------------------------------------------------------
struct QuantizeArgs {
    const _Float16* w;
    uint8_t* codes;
    _Float16* scale;
    uint8_t* zero;   // or null: symmetric
    int64_t rows, cols, group, groups;
};

__global__ __launch_bounds__(256) void lordba_quantize_i4_kernel(QuantizeArgs a) {
    const int64_t stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < a.rows * a.groups; k += stride) {
        const int64_t row = k / a.groups, c0 = k % a.groups * a.group, n = min(a.group, a.cols - c0);
        const _Float16* const w = a.w + row * a.cols + c0;
        uint8_t* const to = a.codes + row * a.cols + c0;
        float low = 0.f, high = 0.f;
        bool number = true;
        for (int64_t i = 0; i < n; ++i) {
            const float v = static_cast<float>(w[i]);
            low = fminf(low, v), high = fmaxf(high, v);
            number = number && fabsf(v) < __builtin_inff();
        }
        const float range = a.zero ? (high - low) / 15.f : fmaxf(high, -low) / 7.f;
        const _Float16 scale = number ? static_cast<_Float16>(range) : static_cast<_Float16>(__builtin_nanf(""));
        const float s = static_cast<float>(scale);
        const bool flat = !(s > 0.f);   // (no weight but 0, or a range that fp16 does not hold, or no number)
        const float z = !a.zero ? 8.f : flat ? 0.f : fminf(rintf(-low / s), 15.f);
        a.scale[k] = scale;
        if (a.zero) a.zero[k] = static_cast<uint8_t>(z);
        for (int64_t i = 0; i < n; ++i) {
            const float q = flat ? z : rintf(static_cast<float>(w[i]) / s + z);
            to[i] = static_cast<uint8_t>(fminf(fmaxf(q, 0.f), 15.f));
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

// Position (row, column) of the laid-out matrix, both with padding, in W: false where it is padding.
__device__ __forceinline__ bool source(const LayoutArgs& a, int64_t tile, int r, int64_t c, int64_t& j, int64_t& i) {
    const int64_t per_row = a.s.tiles / a.s.row_halves, per_col = a.s.blocks / a.s.col_halves * kI4Columns;
    const int64_t row = i4_row(tile % per_row, r), col = c % per_col;
    if (row >= a.s.rows || col >= a.s.cols) return false;
    const int64_t full_row = tile / per_row * a.s.rows + row, full_col = c / per_col * a.s.cols + col;
    j = a.transposed ? full_col : full_row, i = a.transposed ? full_row : full_col;
    return true;
}

__global__ __launch_bounds__(256) void lordba_layout_i4_kernel(LayoutArgs a) {
    const int64_t words = a.s.tiles * a.s.blocks * 256, stride = static_cast<int64_t>(gridDim.x) * 256;
    for (int64_t k = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; k < words; k += stride) {
        const int64_t block = k >> 8;
        const int lane = static_cast<int>(k >> 2) & 63, m = static_cast<int>(k) & 3;
        const int64_t tile = block / a.s.blocks, c0 = block % a.s.blocks * kI4Columns + 32 * m + 8 * (lane >> 4);
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            int64_t j, i;
            uint32_t code = 8;   // (stands for 0 where the scale is padding too)
            if (source(a, tile, lane & 15, c0 + e, j, i)) code = a.codes[j * a.cols + i] & 15u;
            // behind the end of a row, in a group that it has: the group's zero
            else if (!a.transposed && a.zero && c0 + e < a.groups * a.group && source(a, tile, lane & 15, 0, j, i)) code = a.zero[j * a.groups + (c0 + e) / a.group] & 15u;
            v |= code << (4 * i4_nibble(e));
        }
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

__device__ __forceinline__ void slopes(float d, float gate, float up, float& dg, float& du) {
    // silu' = sigma (1 + gate (1 - sigma)) with 1 - sigma = e / (1 + e): no cancellation where sigma is near 1
    const float e = __expf(-fabsf(gate)), r = __builtin_amdgcn_rcpf(1.f + e);
    const float sigma = gate < 0.f ? e * r : r, rest = gate < 0.f ? r : e * r;
    dg = d * up * sigma * (1.f + gate * rest);
    du = d * gate * sigma;
}

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
    hipLaunchKernelGGL(lordba_quantize_i4_kernel, dim3(grid_for(rows * groups)), dim3(256), 0, static_cast<hipStream_t>(stream), a);
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
