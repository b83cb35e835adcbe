// Products with 4-bit weights: the entry points, what they check, and which kernel a call takes.
#include "lordba_i4_product.h"

namespace {

lordba_status check(int64_t T, int64_t d_in, int64_t d_out, int64_t group) {
    if (T < 0 || T > INT32_MAX || d_in < 1 || d_out < 1 || d_in > kI4Most || d_out > kI4Most) return LORDBA_ERR_DIM;
    return i4_group(group) ? LORDBA_OK : LORDBA_ERR_VALUE;
}

struct Weights {
    const uint8_t* codes;
    const void *scale, *zero;
    bool misaligned() const { return i8_misaligned(codes, 16) || i8_misaligned(scale, 16) || i8_misaligned(zero, 16); }
};

lordba_status product(I4Args a, const Weights& w, const I4Shape& s, int64_t group, bool gated, bool backward, void* stream) {
    a.codes = w.codes;
    a.scale = static_cast<const uint16_t*>(w.scale), a.zero = static_cast<const uint16_t*>(w.zero);
    a.blocks = static_cast<int32_t>(s.blocks), a.plane_blocks = static_cast<int32_t>(s.blocks / s.col_halves);
    a.tiles = static_cast<int32_t>(s.tiles / s.row_halves);
    a.groups = static_cast<int32_t>(s.groups);
    a.shift = group == 32 ? 5 : group == 64 ? 6 : 7;
    a.aligned = a.k % 8 == 0 && !i8_misaligned(a.x, 16);
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const I4Kernel kernel = i4_kernel(a.T, a.k, a.blocks, a.n, gated, a.aligned != 0, backward, w.zero != nullptr && group == 32);
    return kernel == kI4Few ? lordba_i4_few(a, group, gated, backward, st) : lordba_i4_many(a, kernel, group, gated, backward, st);
}

size_t bytes_of(const I4Shape& s) { return static_cast<size_t>(s.tiles) * static_cast<size_t>(s.blocks) * 1024; }

lordba_status linear(const void* x, const Weights& w, void* y, int64_t T, int64_t d_in, int64_t d_out, int64_t group, bool backward, void* stream) {
    const lordba_status st = check(T, d_in, d_out, group);
    if (st != LORDBA_OK || T == 0) return st;
    if (!x || !w.codes || !w.scale || !y) return LORDBA_ERR_NULL;
    if (i8_misaligned(x, 2) || w.misaligned() || i8_misaligned(y, 2)) return LORDBA_ERR_ALIGN;
    const I4Shape s = i4_shape(d_out, d_in, group, 1, backward);
    const int64_t k = backward ? d_out : d_in, n = backward ? d_in : d_out;
    const size_t ns = static_cast<size_t>(s.scales) * 2;
    const Span out[] = {{y, static_cast<size_t>(T) * n * 2}};
    const Span in[] = {{x, static_cast<size_t>(T) * k * 2}, {w.codes, bytes_of(s)}, {w.scale, ns}, {w.zero, ns}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    const lordba_status dev = check_device();
    if (dev != LORDBA_OK) return dev;
    I4Args a = {};
    a.x = static_cast<const _Float16*>(x), a.y = static_cast<_Float16*>(y);
    a.T = T, a.k = k, a.n = n;
    return product(a, w, s, group, false, backward, stream);
}

}  // namespace

extern "C" lordba_status lordba_linear_i4(const void* x, const uint8_t* codes, const void* scale, const void* zero, void* y, int64_t T, int64_t d_in,
                                          int64_t d_out, int64_t group, void* stream) {
    return linear(x, {codes, scale, zero}, y, T, d_in, d_out, group, false, stream);
}

extern "C" lordba_status lordba_linear_i4_backward(const void* g, const uint8_t* codes_t, const void* scale_t, const void* zero_t, void* dx, int64_t T,
                                                   int64_t d_in, int64_t d_out, int64_t group, void* stream) {
    return linear(g, {codes_t, scale_t, zero_t}, dx, T, d_in, d_out, group, true, stream);
}

extern "C" lordba_status lordba_gated_i4(const void* x, const uint8_t* codes, const void* scale, const void* zero, const void* addends, void* h,
                                         void* gate_up, int64_t T, int64_t d_in, int64_t d_ff, int64_t group, void* stream) {
    lordba_status st = check(T, d_in, d_ff, group);
    if (st != LORDBA_OK || T == 0) return st;
    if (2 * d_ff > kI4Most) return LORDBA_ERR_DIM;
    const Weights w = {codes, scale, zero};
    if (!x || !codes || !scale || !h) return LORDBA_ERR_NULL;
    if (i8_misaligned(x, 2) || w.misaligned() || i8_misaligned(addends, 2) || i8_misaligned(h, 2) || i8_misaligned(gate_up, 2)) return LORDBA_ERR_ALIGN;
    const I4Shape s = i4_shape(2 * d_ff, d_in, group, 2, false);
    const size_t nh = static_cast<size_t>(T) * d_ff * 2, ns = static_cast<size_t>(s.scales) * 2;
    const Span out[] = {{h, nh}, {gate_up, 2 * nh}};
    const Span in[] = {{x, static_cast<size_t>(T) * d_in * 2}, {codes, bytes_of(s)}, {scale, ns}, {zero, ns}, {addends, 2 * nh}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    I4Args a = {};
    a.x = static_cast<const _Float16*>(x), a.addends = static_cast<const _Float16*>(addends);
    a.y = static_cast<_Float16*>(h), a.kept = static_cast<_Float16*>(gate_up);
    a.T = T, a.k = d_in, a.n = d_ff;
    return product(a, w, s, group, true, false, stream);
}

extern "C" lordba_status lordba_gated_i4_backward(const void* dh, const void* gate_up, const uint8_t* codes_t, const void* scale_t, const void* zero_t,
                                                  void* dx, void* dgate_up, int64_t T, int64_t d_in, int64_t d_ff, int64_t group, void* stream) {
    lordba_status st = check(T, d_in, d_ff, group);
    if (st != LORDBA_OK || T == 0) return st;
    if (2 * d_ff > kI4Most) return LORDBA_ERR_DIM;
    const Weights w = {codes_t, scale_t, zero_t};
    if (!dh || !gate_up || !codes_t || !scale_t || !dx || !dgate_up) return LORDBA_ERR_NULL;
    if (i8_misaligned(dh, 2) || i8_misaligned(gate_up, 2) || w.misaligned() || i8_misaligned(dx, 2) || i8_misaligned(dgate_up, 2)) return LORDBA_ERR_ALIGN;
    const I4Shape s = i4_shape(2 * d_ff, d_in, group, 2, true);
    const size_t nh = static_cast<size_t>(T) * d_ff * 2, ns = static_cast<size_t>(s.scales) * 2;
    const Span out[] = {{dx, static_cast<size_t>(T) * d_in * 2}, {dgate_up, 2 * nh}};
    const Span in[] = {{dh, nh}, {gate_up, 2 * nh}, {codes_t, bytes_of(s)}, {scale_t, ns}, {zero_t, ns}};
    if (aliased(out, in)) return LORDBA_ERR_ALIAS;
    if ((st = check_device()) != LORDBA_OK) return st;
    if ((st = lordba_i4_gated_grad(dh, gate_up, dgate_up, T, d_ff, static_cast<hipStream_t>(stream))) != LORDBA_OK) return st;
    I4Args a = {};
    a.x = static_cast<const _Float16*>(dgate_up), a.y = static_cast<_Float16*>(dx);
    a.dh = static_cast<const _Float16*>(dh), a.gate_up = static_cast<const _Float16*>(gate_up);
    a.T = T, a.k = d_ff, a.n = d_in;
    return product(a, w, s, group, false, true, stream);
}
