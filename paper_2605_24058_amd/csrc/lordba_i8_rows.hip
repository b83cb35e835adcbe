// Row kernels of the 8-bit projections: rows of fp16 numbers into one or two digits, the gradient of the gated activation into two,
// the layout of weights.  All of them are bound by memory: each reads its input once and holds it in registers while the row's
// largest magnitude is found.
#include <algorithm>

#include "lordba_dev_util.h"
#include "lordba_i8.h"

namespace {

// The largest of the workgroup's values per row.  Magnitudes are compared as unsigned bits, so that a NaN is the largest of all.
// TPR threads share a row: a wave of its own (TPR = 64, four rows a workgroup) or the whole workgroup.
template <int TPR>
__device__ __forceinline__ uint32_t row_max(uint32_t m) {
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), s)));
    if constexpr (TPR > 64) {
        __shared__ uint32_t part[TPR / 64];
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) m = max(m, part[w]);
    }
    return m;
}

// Eight channel scales from column c < cols on, zeros from column `cols` on.
__device__ __forceinline__ void load_scales(const float* p, int64_t c, int64_t cols, float (&v)[8]) {
    typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));
    if (c + 8 <= cols) {
        const f4_any a = *reinterpret_cast<const f4_any*>(p + c), b = *reinterpret_cast<const f4_any*>(p + c + 4);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = a[e], v[4 + e] = b[e];
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = p[min(c + e, cols - 1)];   // (all requested before the first is looked at)
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? v[e] : 0.f;
    }
}

__device__ __forceinline__ void store_part(_Float16* row, int64_t c, int64_t cols, u4 v) {
    if (c + 8 <= cols) {
        *reinterpret_cast<u4_any*>(row + c) = v;
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c + e < cols) reinterpret_cast<uint16_t*>(row)[c + e] = static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1)));
}

struct QuantizeArgs {
    const _Float16* x;
    const float* col_scale;
    int8_t* q;
    float* scale;
    uint32_t* clear;
    int64_t rows, cols, ld;
    int64_t first;   // row of this launch's first workgroup
};

// kI8SplitTiles counters for the product behind this kernel
__device__ __forceinline__ void clear_counters(uint32_t* p) {
    if (p && blockIdx.x == 0)
        for (int64_t k = threadIdx.x; k < kI8SplitTiles; k += blockDim.x) p[k] = 0;
}

// NV > 0: a thread's numbers stay in registers between the two passes over the row; NV = 0 (more than 32768 columns): they are read again.
template <int TPR, int NV, int DIG, bool CS>
__global__ __launch_bounds__(TPR < 128 ? 256 : TPR) void lordba_quantize_rows_kernel(QuantizeArgs a) {
    const int t = threadIdx.x % TPR;
    const int64_t row = a.first + (TPR < 128 ? static_cast<int64_t>(blockIdx.x) * (256 / TPR) + threadIdx.x / TPR : blockIdx.x);
    clear_counters(a.clear);
    if (row >= a.rows) return;   // (whole waves: a wave has one row)
    const _Float16* x = a.x + row * a.cols;
    const int turns = NV > 0 ? NV : static_cast<int>((a.ld + 8 * TPR - 1) / (8 * TPR));
    u4 raw[NV > 0 ? NV : 1];
    if constexpr (NV > 0) {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int64_t c = 8 * static_cast<int64_t>(t + i * TPR);
            raw[i] = c < a.cols ? load_part(x, c, a.cols) : u4{0u, 0u, 0u, 0u};
        }
    }
    // (with column scales the products are formed again for the second use: kept, they would take twice the registers of the row)
    auto numbers = [&](int i, float (&f)[8]) {
        const int64_t c = 8 * static_cast<int64_t>(t + i * TPR);
        const h8 h = as_h8(NV > 0 ? raw[NV > 0 ? i : 0] : c < a.cols ? load_part(x, c, a.cols) : u4{0u, 0u, 0u, 0u});
        float s[8];
        if constexpr (CS) load_scales(a.col_scale, min(c, a.cols - 1), a.cols, s);   // (behind the last column: the numbers are zeros)
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = CS ? static_cast<float>(h[e]) * s[e] : static_cast<float>(h[e]);
    };
    uint32_t m = 0;
#pragma unroll NV > 0 ? NV : 1
    for (int i = 0; i < turns; ++i) {
        float f[8];
        numbers(i, f);
#pragma unroll
        for (int e = 0; e < 8; ++e) m = max(m, __float_as_uint(f[e]) & 0x7FFFFFFFu);
    }
    const RowScale s = scale_of(row_max<TPR>(m), DIG == 1 ? 127.f : 32512.f);
    if (t == 0) a.scale[row] = s.scale;
#pragma unroll NV > 0 ? NV : 1
    for (int i = 0; i < turns; ++i) {
        const int64_t c = 8 * static_cast<int64_t>(t + i * TPR);
        if (c >= a.ld) break;
        float f[8];
        numbers(i, f);
        uint2 hi, lo;
        digits_of<DIG>(f, s.inverse, hi, lo);
        *reinterpret_cast<uint2*>(a.q + row * a.ld + c) = hi;
        if constexpr (DIG == 2) *reinterpret_cast<uint2*>(a.q + (a.rows + row) * a.ld + c) = lo;
    }
}

constexpr int64_t kRowsPerLaunch = 1 << 21;   // (a launch counts threads in 32 bits, up to 1024 for a row)

template <int TPR, int NV, int DIG, bool CS>
lordba_status quantize_launch(QuantizeArgs a, hipStream_t stream) {
    constexpr int64_t per = TPR < 128 ? 256 / TPR : 1;
    for (a.first = 0; a.first < a.rows; a.first += kRowsPerLaunch) {
        const int64_t n = std::min(kRowsPerLaunch, a.rows - a.first);
        hipLaunchKernelGGL((lordba_quantize_rows_kernel<TPR, NV, DIG, CS>), dim3(static_cast<unsigned>((n + per - 1) / per)),
                           dim3(TPR < 128 ? 256 : TPR), 0, stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
        a.clear = nullptr;
    }
    return LORDBA_OK;
}

template <int DIG, bool CS>
lordba_status quantize(const QuantizeArgs& a, hipStream_t stream) {
    const int64_t vectors = a.ld / 8;
    if (vectors <= 64) return quantize_launch<64, 1, DIG, CS>(a, stream);
    if (vectors <= 128) return quantize_launch<64, 2, DIG, CS>(a, stream);
    if (vectors <= 256 && a.rows >= 1024) return quantize_launch<128, 2, DIG, CS>(a, stream);   // (8192 x 1230 10.9 -> 9.1 us; few rows are done sooner by more waves)
    if (vectors <= 256) return quantize_launch<256, 1, DIG, CS>(a, stream);
    if (vectors <= 512) return quantize_launch<256, 2, DIG, CS>(a, stream);
    if (vectors <= 1024) return quantize_launch<256, 4, DIG, CS>(a, stream);
    if (vectors <= 2048) return quantize_launch<512, 4, DIG, CS>(a, stream);
    if (vectors <= 4096) return quantize_launch<1024, 4, DIG, CS>(a, stream);
    return quantize_launch<1024, 0, DIG, CS>(a, stream);
}

// ---- the gradient of h = g sigma(g) u -----------------------------------------------------------------------------
// dg = dh u sigma(g) (1 + g (1 - sigma(g))), du = dh g sigma(g).  Both are returned in fp16 and, times their weights' channel scales, as the
// digits of one row of 2 d_ff columns: the contraction with both projections' weights has one scale per token.
struct GatedGradArgs {
    const _Float16* dh;
    const _Float16* gate_up;   // [2, T, d_ff]
    const float* w_scale;      // [2 d_ff]
    _Float16* dgate_up;        // [2, T, d_ff]
    int8_t* q;
    float* scale;
    uint32_t* clear;
    int64_t T, d_ff, ld;
    int64_t first;
};

__device__ __forceinline__ void gated_grad(h8 dh, h8 gate, h8 up, float (&dg)[8], float (&du)[8]) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float g = static_cast<float>(gate[e]), u = static_cast<float>(up[e]), d = static_cast<float>(dh[e]);
        const float sigma = __builtin_amdgcn_rcpf(1.f + __expf(-g));   // (to one last place)
        dg[e] = d * u * sigma * (1.f + g * (1.f - sigma));
        du[e] = d * g * sigma;
    }
}

// `n` of eight bytes to any address
__device__ __forceinline__ void store_bytes(int8_t* p, uint2 v, int64_t n) {
    typedef uint32_t u2_byte __attribute__((ext_vector_type(2), aligned(1)));
    if (n >= 8) {
        *reinterpret_cast<u2_byte*>(p) = u2_byte{v.x, v.y};
        return;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < n) p[e] = static_cast<int8_t>((e < 4 ? v.x : v.y) >> (8 * (e & 3)));
}

// Bound by arithmetic (about 30 instructions for a pair of gradients) and memory alike: 2048 rows of 11008 62 us, 315 MB.  NV > 0: a thread's numbers stay in
// registers (formed again for the second use, 77 us); NV = 0 (d_ff > 16384): they are computed again from memory.
template <int TPR, int NV, int DIG>
__global__ __launch_bounds__(TPR < 128 ? 256 : TPR) void lordba_gated_grad_kernel(GatedGradArgs a) {
    const int tid = threadIdx.x % TPR;
    const int64_t row = a.first + (TPR < 128 ? static_cast<int64_t>(blockIdx.x) * (256 / TPR) + threadIdx.x / TPR : blockIdx.x);
    clear_counters(a.clear);
    if (row >= a.T) return;   // (whole waves: a wave has one row)
    const int64_t F = a.d_ff, plane = a.T * F;
    const _Float16 *dh = a.dh + row * F, *gate = a.gate_up + row * F, *up = gate + plane;
    _Float16 *dgate = a.dgate_up + row * F, *dup = dgate + plane;
    // The first of this thread's eight columns, -1: none.  A row's last group ends where the row does: it repeats columns of the one before, with the same results
    // (stored entry by entry the end of a row cost 20 of 86 us at 4096 x 4092).
    auto column = [&](int i) -> int64_t {
        const int64_t c = 8 * static_cast<int64_t>(tid + i * TPR);
        return c >= F ? -1 : F >= 8 ? min(c, F - 8) : c;
    };
    const int turns = NV > 0 ? NV : static_cast<int>((F + 8 * TPR - 1) / (8 * TPR));
    float v[NV > 0 ? NV : 1][2][8];
    uint32_t m = 0;
#pragma unroll NV > 0 ? NV : 1
    for (int i = 0; i < turns; ++i) {
        const int64_t c = column(i);
        if (c < 0) break;
        float dg[8], du[8];
        gated_grad(as_h8(load_part(dh, c, F)), as_h8(load_part(gate, c, F)), as_h8(load_part(up, c, F)), dg, du);
        h8 hg, hu;
        float sg[8], su[8];
        load_scales(a.w_scale, c, F, sg);
        load_scales(a.w_scale + F, c, F, su);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            hg[e] = static_cast<_Float16>(dg[e]);
            hu[e] = static_cast<_Float16>(du[e]);
            dg[e] *= sg[e];
            du[e] *= su[e];
            m = max(m, max(__float_as_uint(dg[e]) & 0x7FFFFFFFu, __float_as_uint(du[e]) & 0x7FFFFFFFu));
            if constexpr (NV > 0) {
                v[i][0][e] = dg[e];
                v[i][1][e] = du[e];
            }
        }
        store_part(dgate, c, F, __builtin_bit_cast(u4, hg));
        store_part(dup, c, F, __builtin_bit_cast(u4, hu));
    }
    const RowScale s = scale_of(row_max<TPR>(m), DIG == 1 ? 127.f : 32512.f);
    if (tid == 0) a.scale[row] = s.scale;
    int8_t* const q = a.q + row * a.ld;
    int8_t* const q_lo = q + a.T * a.ld;
#pragma unroll NV > 0 ? NV : 1
    for (int i = 0; i < turns; ++i) {
        const int64_t c = column(i);
        if (c < 0) break;
        float dg[8], du[8];
        if constexpr (NV > 0) {
#pragma unroll
            for (int e = 0; e < 8; ++e) dg[e] = v[i][0][e], du[e] = v[i][1][e];
        } else {
            gated_grad(as_h8(load_part(dh, c, F)), as_h8(load_part(gate, c, F)), as_h8(load_part(up, c, F)), dg, du);
            float sg[8], su[8];
            load_scales(a.w_scale, c, F, sg);
            load_scales(a.w_scale + F, c, F, su);
#pragma unroll
            for (int e = 0; e < 8; ++e) dg[e] *= sg[e], du[e] *= su[e];
        }
        uint2 hi, lo;
        digits_of<DIG>(dg, s.inverse, hi, lo);
        store_bytes(q + c, hi, F - c);
        if constexpr (DIG == 2) store_bytes(q_lo + c, lo, F - c);
        digits_of<DIG>(du, s.inverse, hi, lo);
        store_bytes(q + F + c, hi, F - c);
        if constexpr (DIG == 2) store_bytes(q_lo + F + c, lo, F - c);
    }
    for (int64_t c = 2 * F + tid; c < a.ld; c += TPR) {
        q[c] = 0;
        if constexpr (DIG == 2) q_lo[c] = 0;
    }
}

template <int TPR, int NV, int DIG>
lordba_status gated_grad_launch(GatedGradArgs a, hipStream_t stream) {
    constexpr int64_t per = TPR < 128 ? 256 / TPR : 1;
    for (a.first = 0; a.first < a.T; a.first += kRowsPerLaunch) {
        const int64_t n = std::min(kRowsPerLaunch, a.T - a.first);
        hipLaunchKernelGGL((lordba_gated_grad_kernel<TPR, NV, DIG>), dim3(static_cast<unsigned>((n + per - 1) / per)), dim3(TPR < 128 ? 256 : TPR), 0,
                           stream, a);
        const lordba_status st = i8_launched();
        if (st != LORDBA_OK) return st;
        a.clear = nullptr;
    }
    return LORDBA_OK;
}

// With many rows of up to 1024 columns a wave has a row of its own (16384 x 320: 58 -> 27 us for the call); few rows are done sooner by more waves (190 x 811
// 8.7 -> 5.8 us, both with row ends stored entry by entry; 4.3 since).  (1024 threads of two groups each, for the longest rows, spilled: 72 us instead of 62 at
// 2048 x 11008.)
template <int DIG>
lordba_status gated_grad(const GatedGradArgs& a, hipStream_t stream) {
    const bool many = a.T >= 512;
    if (many && a.d_ff <= 512) return gated_grad_launch<64, 1, DIG>(a, stream);
    if (many && a.d_ff <= 1024) return gated_grad_launch<64, 2, DIG>(a, stream);
    if (a.d_ff <= 2048) return gated_grad_launch<256, 1, DIG>(a, stream);
    if (a.d_ff <= 4096) return gated_grad_launch<512, 1, DIG>(a, stream);
    if (a.d_ff <= 8192) return gated_grad_launch<512, 2, DIG>(a, stream);
    if (a.d_ff <= 16384) return gated_grad_launch<512, 4, DIG>(a, stream);
    return gated_grad_launch<512, 0, DIG>(a, stream);
}

// ---- layout of weights --------------------------------------------------------------------------------------------
struct LayoutArgs {
    const int8_t* w;
    int8_t* out;
    int64_t rows, cols, ld;   // of w; ld: row bytes of out
};

__global__ __launch_bounds__(256) void lordba_layout_i8_kernel(LayoutArgs a) {
    const int64_t c = (static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x) * 4;
    if (c >= a.ld) return;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (c + e < a.cols) v |= static_cast<uint32_t>(static_cast<uint8_t>(a.w[row * a.cols + c + e])) << (8 * e);
        *reinterpret_cast<uint32_t*>(a.out + row * a.ld + c) = v;
    }
}

// 64 x 64 tiles through LDS: rows of w in, columns out, four entries of an output row per store
__global__ __launch_bounds__(256) void lordba_transpose_i8_kernel(LayoutArgs a) {
    __shared__ int8_t tile[64][68];
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * 64, r0 = static_cast<int64_t>(blockIdx.y) * 64;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int r = w; r < 64; r += 4) tile[r][lane] = r0 + r < a.rows && c0 + lane < a.cols ? a.w[(r0 + r) * a.cols + c0 + lane] : 0;
    __syncthreads();
    for (int k = threadIdx.x; k < 64 * 16; k += 256) {
        const int c = k >> 4, r = (k & 15) * 4;
        if (c0 + c >= a.cols || r0 + r >= a.ld) continue;
        uint32_t v = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) v |= static_cast<uint32_t>(static_cast<uint8_t>(tile[r + e][c])) << (8 * e);
        *reinterpret_cast<uint32_t*>(a.out + (c0 + c) * a.ld + r0 + r) = v;
    }
}

}  // namespace

lordba_status lordba_i8_quantize(const void* x, const float* col_scale, int8_t* q, float* scale, uint32_t* clear, int64_t rows, int64_t cols,
                                 int digits, hipStream_t stream) {
    const QuantizeArgs a = {static_cast<const _Float16*>(x), col_scale, q, scale, clear, rows, cols, i8_row_bytes(cols), 0};
    if (digits == 1) return col_scale ? quantize<1, true>(a, stream) : quantize<1, false>(a, stream);
    return col_scale ? quantize<2, true>(a, stream) : quantize<2, false>(a, stream);
}

lordba_status lordba_i8_gated_grad(const void* dh, const void* gate_up, const float* w_scale, void* dgate_up, int8_t* q, float* scale,
                                   uint32_t* clear, int64_t T, int64_t d_ff, int digits, hipStream_t stream) {
    const GatedGradArgs a = {static_cast<const _Float16*>(dh), static_cast<const _Float16*>(gate_up), w_scale, static_cast<_Float16*>(dgate_up),
                             q, scale, clear, T, d_ff, i8_row_bytes(2 * d_ff), 0};
    return digits == 1 ? gated_grad<1>(a, stream) : gated_grad<2>(a, stream);
}

extern "C" size_t lordba_i8_row_bytes(int64_t cols) {
    return cols < 1 || cols > LORDBA_I8_MAX_COLUMNS ? 0 : static_cast<size_t>(i8_row_bytes(cols));
}

extern "C" size_t lordba_i8_workspace_bytes(int64_t T, int64_t cols, int digits) {
    if (T < 0 || T > INT32_MAX || cols < 1 || cols > LORDBA_I8_MAX_COLUMNS || digits < 1 || digits > 2) return 0;
    return i8_workspace_bytes(T, cols, digits);
}

extern "C" lordba_status lordba_quantize_rows(const void* x, const float* col_scale, int8_t* q, float* scale, int64_t rows, int64_t cols,
                                              int digits, void* stream) {
    if (rows < 0 || rows > INT32_MAX || cols < 1 || cols > LORDBA_I8_MAX_COLUMNS) return LORDBA_ERR_DIM;
    if (digits < 1 || digits > 2) return LORDBA_ERR_VALUE;
    if (rows == 0) return LORDBA_OK;
    if (!x || !q || !scale) return LORDBA_ERR_NULL;
    if (i8_misaligned(x, 2) || i8_misaligned(col_scale, 4) || i8_misaligned(q, 16) || i8_misaligned(scale, 4)) return LORDBA_ERR_ALIGN;
    const size_t nx = static_cast<size_t>(rows) * cols * 2, nq = static_cast<size_t>(digits) * rows * i8_row_bytes(cols), ns = static_cast<size_t>(rows) * 4;
    if (i8_overlap(q, nq, x, nx) || i8_overlap(scale, ns, x, nx) || i8_overlap(q, nq, scale, ns) ||
        i8_overlap(q, nq, col_scale, static_cast<size_t>(cols) * 4) || i8_overlap(scale, ns, col_scale, static_cast<size_t>(cols) * 4))
        return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    return lordba_i8_quantize(x, col_scale, q, scale, nullptr, rows, cols, digits, static_cast<hipStream_t>(stream));
}

extern "C" lordba_status lordba_layout_i8(const int8_t* w, int8_t* out, int64_t rows, int64_t cols, int transposed, void* stream) {
    if (rows < 1 || cols < 1 || rows > (1 << 24) || cols > (1 << 24) || (transposed ? rows : cols) > LORDBA_I8_MAX_COLUMNS) return LORDBA_ERR_DIM;
    if (!w || !out) return LORDBA_ERR_NULL;
    if (i8_misaligned(out, 16)) return LORDBA_ERR_ALIGN;
    const LayoutArgs a = {w, out, rows, cols, i8_row_bytes(transposed ? rows : cols)};
    if (i8_overlap(out, static_cast<size_t>(transposed ? cols : rows) * a.ld, w, static_cast<size_t>(rows) * cols)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    if (transposed)
        hipLaunchKernelGGL(lordba_transpose_i8_kernel, dim3(static_cast<unsigned>((cols + 63) / 64), static_cast<unsigned>((a.ld + 63) / 64)),
                           dim3(256), 0, static_cast<hipStream_t>(stream), a);
    else
        hipLaunchKernelGGL(lordba_layout_i8_kernel, dim3(static_cast<unsigned>(std::min<int64_t>(rows, 1 << 20)), static_cast<unsigned>((a.ld + 1023) / 1024)), dim3(256), 0,
                           static_cast<hipStream_t>(stream), a);
    return i8_launched();
}
