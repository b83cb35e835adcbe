// Products with 8-bit weights: y[t, j] = s_t w_j sum_i q_ti W_ji on v_mfma_i32_16x16x64_i8, plain or as the two projections of a gated block.
//
// The weights' rows are the first operand, the tokens' rows the second, so that a lane's four accumulators are four consecutive
// columns of y for one token.  Blocks of 16 rows are the unit of everything: with two digits the token blocks alternate hi, lo (y takes
// 256 hi + lo of neighbouring accumulators), in the gated block the weight blocks alternate gate, up, so that a lane holds both
// factors of its outputs.
#include <type_traits>

#include "lordba_dev_util.h"
#include "lordba_i8.h"

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
};

typedef uint32_t u2_any __attribute__((ext_vector_type(2), aligned(2)));
typedef float f4_any __attribute__((ext_vector_type(4), aligned(4)));

// Four consecutive entries from column c of n: one access inside the row, single ones at its end.
__device__ __forceinline__ void load4(const _Float16* row, int64_t c, int64_t n, float (&v)[4]) {
    if (c + 4 <= n) {
        const u2_any r = *reinterpret_cast<const u2_any*>(row + c);
        const h2 a = as_h2(r[0]), b = as_h2(r[1]);
        v[0] = a[0], v[1] = a[1], v[2] = b[0], v[3] = b[1];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < n ? static_cast<float>(row[c + i]) : 0.f;
    }
}
__device__ __forceinline__ void load4(const float* p, int64_t c, int64_t n, float (&v)[4]) {
    if (c + 4 <= n) {
        const f4_any r = *reinterpret_cast<const f4_any*>(p + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = r[i];
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = c + i < n ? p[c + i] : 0.f;
    }
}
__device__ __forceinline__ void store4(_Float16* row, int64_t c, int64_t n, const float (&v)[4]) {
    if (c + 4 <= n) {
        const h2 a = {static_cast<_Float16>(v[0]), static_cast<_Float16>(v[1])}, b = {static_cast<_Float16>(v[2]), static_cast<_Float16>(v[3])};
        *reinterpret_cast<u2_any*>(row + c) = u2_any{__builtin_bit_cast(uint32_t, a), __builtin_bit_cast(uint32_t, b)};
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (c + i < n) row[c + i] = static_cast<_Float16>(v[i]);
    }
}

// The sums of a lane (CB x TB blocks) to y.  c0, t0: the first column of y and the first token of the wave's part.
template <int CB, int TB, int DIG, bool GATED>
__device__ __forceinline__ void finish(const ProductArgs& a, const i4 (&acc)[CB][TB], int64_t c0, int64_t t0) {
    constexpr int P = GATED ? 2 : 1;
    static_assert(CB % P == 0 && TB % DIG == 0, "whole pairs of blocks");
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int cb = 0; cb < CB; cb += P) {
        const int64_t c = c0 + 16 * (cb / P) + 4 * (lane >> 4);
        float w[P][4];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            if (a.w_scale) load4(a.w_scale + p * a.n, c, a.n, w[p]);
            else w[p][0] = w[p][1] = w[p][2] = w[p][3] = 1.f;
        }
#pragma unroll
        for (int tb = 0; tb < TB; tb += DIG) {
            const int64_t t = t0 + 16 * (tb / DIG) + (lane & 15);
            if (t >= a.T || c >= a.n) continue;
            const float s = a.q_scale[t];
            float v[P][4];
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float sum = static_cast<float>(acc[cb + p][tb][i]);
                    if constexpr (DIG == 2) sum = fmaf(256.f, sum, static_cast<float>(acc[cb + p][tb + 1][i]));
                    v[p][i] = sum * s * w[p][i];
                }
            if constexpr (GATED) {
                const int64_t plane = a.T * a.n;
                if (a.addends) {
#pragma unroll
                    for (int p = 0; p < 2; ++p) {
                        float add[4];
                        load4(a.addends + p * plane + t * a.n, c, a.n, add);
#pragma unroll
                        for (int i = 0; i < 4; ++i) v[p][i] += add[i];
                    }
                }
                if (a.kept) {
                    store4(a.kept + t * a.n, c, a.n, v[0]);
                    store4(a.kept + plane + t * a.n, c, a.n, v[1]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) v[0][i] = v[0][i] / (1.f + __expf(-v[0][i])) * v[1][i];
            }
            store4(a.y + t * a.n, c, a.n, v[0]);
        }
    }
}

// Row b * 16 + r of the workgroup's weight rows / token rows in memory.
template <bool GATED>
__device__ __forceinline__ const int8_t* weight_row(const ProductArgs& a, int64_t c0, int b, int r) {
    if constexpr (GATED) return a.w + ((b & 1) * a.n + min(c0 + (b >> 1) * 16 + r, a.n - 1)) * a.ld;
    else return a.w + min(c0 + b * 16 + r, a.n - 1) * a.ld;
}
template <int DIG>
__device__ __forceinline__ const int8_t* token_row(const ProductArgs& a, int64_t t0, int b, int r) {
    if constexpr (DIG == 2) return a.q + ((b & 1) * a.T + min(t0 + (b >> 1) * 16 + r, a.T - 1)) * a.ld;
    else return a.q + min(t0 + b * 16 + r, a.T - 1) * a.ld;
}

// One workgroup: CT x TT sums (weight rows x token rows), WC x WT waves, steps of 64 columns through a ring of four slots in LDS.
// A step's rows of 64 bytes lie there as four 16-byte pieces, piece p of row r at place p ^ (r / 2 mod 4): eight neighbouring
// lanes of an operand read (eight rows, one piece) then cover all banks.  The loads go straight into LDS, where the place follows from
// the lane, so it is the lane's address that is permuted.
// While a step's products run on one set of operand registers, the next step's operands are read into the other.
// The barrier of step k says that step k + 1 has landed and that everybody has read step k, whose slot then takes step k + 4.
template <int CT, int TT, int WC, int WT, int DIG, bool GATED>
__global__ __launch_bounds__(64 * WC * WT) void lordba_i8_product_kernel(ProductArgs a) {
    constexpr int NW = WC * WT, CB = CT / 16 / WC, TB = TT / 16 / WT, NB = (CT + TT) / 16, L = NB / NW;
    constexpr uint32_t kSlot = NB * 1024u;
    static_assert(NB % NW == 0, "whole loads per wave");
    extern __shared__ int8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wc = wave % WC, wt = wave / WC;
    constexpr int kCols = GATED ? CT / 2 : CT, kTokens = TT / DIG;
    const int64_t c0 = static_cast<int64_t>(blockIdx.x) * kCols, t0 = static_cast<int64_t>(blockIdx.y) * kTokens;
    const int K = static_cast<int>(a.ld / 64);

    const int8_t* src[L];
#pragma unroll
    for (int j = 0; j < L; ++j) {
        const int b = wave * L + j, r = lane >> 2, piece = (lane & 3) ^ ((r >> 1) & 3);
        src[j] = (b < CT / 16 ? weight_row<GATED>(a, c0, b, r) : token_row<DIG>(a, t0, b - CT / 16, r)) + 16 * piece;
    }
    const uint32_t base = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(lds));
    auto request = [&](int k) {
#pragma unroll
        for (int j = 0; j < L; ++j) {
            load16_to_lds<false>(base + (k & 3) * kSlot + (wave * L + j) * 1024u, src[j]);
            src[j] += 64;
        }
    };
    i4 acc[CB][TB];
#pragma unroll
    for (int i = 0; i < CB; ++i)
#pragma unroll
        for (int j = 0; j < TB; ++j) acc[i][j] = i4{0, 0, 0, 0};
    i4 fc[2][CB], ft[2][TB];
    const int r = lane & 15, place = 16 * ((lane >> 4) ^ ((r >> 1) & 3));
    const int8_t* const at_c = lds + wc * CB * 1024 + r * 64 + place;
    const int8_t* const at_t = lds + (CT / 16 + wt * TB) * 1024 + r * 64 + place;
    auto read = [&](auto set, int k) {
        const uint32_t slot = (k & 3) * kSlot;
#pragma unroll
        for (int i = 0; i < CB; ++i) fc[set.value][i] = *reinterpret_cast<const i4*>(at_c + slot + i * 1024);
#pragma unroll
        for (int i = 0; i < TB; ++i) ft[set.value][i] = *reinterpret_cast<const i4*>(at_t + slot + i * 1024);
    };
    auto multiply = [&](auto set) {
#pragma unroll
        for (int i = 0; i < CB; ++i)
#pragma unroll
            for (int j = 0; j < TB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fc[set.value][i], ft[set.value][j], acc[i][j], 0, 0, 0);
    };
    // Everything up to step k + 1 has landed (this wave's loads; steps up to min(k + 3, K - 1) are requested), and this wave's operands are in
    // registers; then everybody's.
    auto meet = [&](int k) {
        if (k + 3 < K) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(2 * L) : "memory");
        else if (k + 2 < K) asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" :: "n"(L) : "memory");
        else asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    using Set0 = std::integral_constant<int, 0>;
    using Set1 = std::integral_constant<int, 1>;
#pragma unroll
    for (int k = 0; k < 4; ++k)
        if (k < K) request(k);
    meet(-1);
    read(Set0{}, 0);
    for (int k = 0; k < K; k += 2) {   // (K is even)
        meet(k);
        if (k + 4 < K) request(k + 4);
        read(Set1{}, k + 1);
        multiply(Set0{});
        meet(k + 1);
        if (k + 5 < K) request(k + 5);
        if (k + 2 < K) read(Set0{}, k + 2);
        multiply(Set1{});
    }
    finish<CB, TB, DIG, GATED>(a, acc, c0 + wc * (kCols / WC), t0 + wt * (kTokens / WT));
}

template <int CT, int TT, int WC, int WT, int DIG, bool GATED>
lordba_status product_launch(const ProductArgs& a, hipStream_t stream) {
    constexpr int kCols = GATED ? CT / 2 : CT, kTokens = TT / DIG;
    constexpr size_t kLds = 4 * (CT + TT) * 64;
    static_assert(kLds <= 160 * 1024, "LDS of a compute unit");
    if constexpr (kLds > 64 * 1024) {
        if (hipFuncSetAttribute(reinterpret_cast<const void*>(lordba_i8_product_kernel<CT, TT, WC, WT, DIG, GATED>),
                                hipFuncAttributeMaxDynamicSharedMemorySize, kLds) != hipSuccess) {
            (void)hipGetLastError();
            return LORDBA_ERR_LAUNCH;
        }
    }
    const dim3 grid(static_cast<unsigned>((a.n + kCols - 1) / kCols), static_cast<unsigned>((a.T + kTokens - 1) / kTokens));
    hipLaunchKernelGGL((lordba_i8_product_kernel<CT, TT, WC, WT, DIG, GATED>), grid, dim3(64 * WC * WT), kLds, stream, a);
    return i8_launched();
}

template <int DIG, bool GATED>
lordba_status product(const ProductArgs& a, hipStream_t stream) {
    return product_launch<64, 64, 2, 2, DIG, GATED>(a, stream);
}

// What the four entry points check alike.
lordba_status check(int64_t T, int64_t d_in, int64_t d_out, int64_t contracted, int digits) {
    if (T < 0 || T > INT32_MAX || d_in < 1 || d_out < 1 || d_in > (1 << 24) || d_out > (1 << 24) || contracted > LORDBA_I8_MAX_COLUMNS) return LORDBA_ERR_DIM;
    return digits < 1 || digits > 2 ? LORDBA_ERR_VALUE : LORDBA_OK;
}

struct Span {
    const void* p;
    size_t n;
};
// No output may overlap an input or another output.
template <size_t NO, size_t NI>
bool aliased(const Span (&out)[NO], const Span (&in)[NI]) {
    for (size_t i = 0; i < NO; ++i) {
        for (size_t j = 0; j < NI; ++j)
            if (i8_overlap(out[i].p, out[i].n, in[j].p, in[j].n)) return true;
        for (size_t j = i + 1; j < NO; ++j)
            if (i8_overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return true;
    }
    return false;
}

struct Workspace {
    int8_t* q;
    float* scale;
};
Workspace split(void* workspace, int64_t T, int64_t cols, int digits) {
    char* const p = static_cast<char*>(workspace);
    return {reinterpret_cast<int8_t*>(p), reinterpret_cast<float*>(p + i8_scale_offset(T, cols, digits))};
}

// y = x diag(col_scale) W^T diag(w_scale) over `contracted` columns
lordba_status linear(const void* x, const float* col_scale, const int8_t* w, const float* w_scale, void* y, void* workspace, size_t workspace_bytes,
                     int64_t T, int64_t contracted, int64_t n, int digits, void* stream) {
    if (T == 0) return LORDBA_OK;
    const float* scale = col_scale ? col_scale : w_scale;
    if (!x || !w || !scale || !y || !workspace) return LORDBA_ERR_NULL;
    if (workspace_bytes < lordba_i8_workspace_bytes(T, contracted, digits)) return LORDBA_ERR_WORKSPACE;
    if (i8_misaligned(x, 2) || i8_misaligned(w, 16) || i8_misaligned(scale, 4) || i8_misaligned(y, 2) || i8_misaligned(workspace, 16)) return LORDBA_ERR_ALIGN;
    const Span out[] = {{y, static_cast<size_t>(T) * n * 2}, {workspace, lordba_i8_workspace_bytes(T, contracted, digits)}};
    const Span in[] = {{x, static_cast<size_t>(T) * contracted * 2}, {w, static_cast<size_t>(n) * i8_row_bytes(contracted)},
                       {scale, static_cast<size_t>(col_scale ? contracted : n) * 4}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const Workspace ws = split(workspace, T, contracted, digits);
    const lordba_status rows = lordba_i8_quantize(x, col_scale, ws.q, ws.scale, T, contracted, digits, st);
    if (rows != LORDBA_OK) return rows;
    const ProductArgs a = {w, ws.q, ws.scale, w_scale, nullptr, static_cast<_Float16*>(y), nullptr, T, n, i8_row_bytes(contracted)};
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
    if (workspace_bytes < lordba_i8_workspace_bytes(T, d_in, digits)) return LORDBA_ERR_WORKSPACE;
    if (i8_misaligned(x, 2) || i8_misaligned(W, 16) || i8_misaligned(w_scale, 4) || i8_misaligned(addends, 2) || i8_misaligned(h, 2) ||
        i8_misaligned(gate_up, 2) || i8_misaligned(workspace, 16))
        return LORDBA_ERR_ALIGN;
    const size_t nh = static_cast<size_t>(T) * d_ff * 2;
    const Span out[] = {{h, nh}, {gate_up, 2 * nh}, {workspace, lordba_i8_workspace_bytes(T, d_in, digits)}};
    const Span in[] = {{x, static_cast<size_t>(T) * d_in * 2}, {W, static_cast<size_t>(2 * d_ff) * i8_row_bytes(d_in)},
                       {w_scale, static_cast<size_t>(2 * d_ff) * 4}, {addends, 2 * nh}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Workspace ws = split(workspace, T, d_in, digits);
    if ((st = lordba_i8_quantize(x, nullptr, ws.q, ws.scale, T, d_in, digits, s)) != LORDBA_OK) return st;
    const ProductArgs a = {W, ws.q, ws.scale, w_scale, static_cast<const _Float16*>(addends), static_cast<_Float16*>(h), static_cast<_Float16*>(gate_up),
                           T, d_ff, i8_row_bytes(d_in)};
    return digits == 1 ? product<1, true>(a, s) : product<2, true>(a, s);
}

extern "C" lordba_status lordba_gated_i8_backward(const void* dh, const void* gate_up, const int8_t* Wt, const float* w_scale, void* dx,
                                                  void* dgate_up, void* workspace, size_t workspace_bytes, int64_t T, int64_t d_in,
                                                  int64_t d_ff, int digits, void* stream) {
    lordba_status st = check(T, d_in, d_ff, 2 * d_ff, digits);
    if (st != LORDBA_OK || T == 0) return st;
    if (!dh || !gate_up || !Wt || !w_scale || !dx || !dgate_up || !workspace) return LORDBA_ERR_NULL;
    if (workspace_bytes < lordba_i8_workspace_bytes(T, 2 * d_ff, digits)) return LORDBA_ERR_WORKSPACE;
    if (i8_misaligned(dh, 2) || i8_misaligned(gate_up, 2) || i8_misaligned(Wt, 16) || i8_misaligned(w_scale, 4) || i8_misaligned(dx, 2) ||
        i8_misaligned(dgate_up, 2) || i8_misaligned(workspace, 16))
        return LORDBA_ERR_ALIGN;
    const size_t nh = static_cast<size_t>(T) * d_ff * 2;
    const Span out[] = {{dx, static_cast<size_t>(T) * d_in * 2}, {dgate_up, 2 * nh}, {workspace, lordba_i8_workspace_bytes(T, 2 * d_ff, digits)}};
    const Span in[] = {{dh, nh}, {gate_up, 2 * nh}, {Wt, static_cast<size_t>(d_in) * i8_row_bytes(2 * d_ff)}, {w_scale, static_cast<size_t>(2 * d_ff) * 4}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    const Workspace ws = split(workspace, T, 2 * d_ff, digits);
    if ((st = lordba_i8_gated_grad(dh, gate_up, w_scale, dgate_up, ws.q, ws.scale, T, d_ff, digits, s)) != LORDBA_OK) return st;
    const ProductArgs a = {Wt, ws.q, ws.scale, nullptr, nullptr, static_cast<_Float16*>(dx), nullptr, T, d_in, i8_row_bytes(2 * d_ff)};
    return digits == 1 ? product<1, false>(a, s) : product<2, false>(a, s);
}
