// How the products on 8-bit and on 4-bit weights read what they add and store their results, eight fp16 columns of a row at a time; what their entry points
// check of the memory that they are given.
#pragma once
#include "lordba_i8.h"

namespace {

// Eight consecutive entries from column c of n; the part of a row that is there.
template <bool FULL>
__device__ __forceinline__ u4 load8(const _Float16* row, int64_t c, int64_t n) {
    return FULL ? load16_any(row + c) : load_part(row, c, n);
}
// KEPT: for the backward pass.  What passes the range of fp16 is kept as its largest number (a NaN as one): with an infinity the slopes of the gated activation,
// finite numbers here and h's too, would come out as 0 times infinity.
template <bool KEPT>
__device__ __forceinline__ u4 to_halves(const float (&f)[8]) {
    h8 h;
#pragma unroll
    for (int e = 0; e < 8; ++e) h[e] = static_cast<_Float16>(f[e]);
    if constexpr (KEPT) {
        const h8 largest = static_cast<_Float16>(65504);
        h = __builtin_elementwise_minimum(__builtin_elementwise_maximum(h, -largest), largest);
    }
    return __builtin_bit_cast(u4, h);
}
template <bool FULL, bool STREAM, bool KEPT>
__device__ __forceinline__ void store8(_Float16* row, int64_t c, int64_t n, const float (&f)[8]) {
    const u4 v = to_halves<KEPT>(f);
    if (FULL || c + 8 <= n) {
        if constexpr (STREAM) store16_any_stream(row + c, v);
        else *reinterpret_cast<u4_any*>(row + c) = v;
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < n) reinterpret_cast<uint16_t*>(row)[c + e] = static_cast<uint16_t>(v[e >> 1] >> (16 * (e & 1)));
    }
}
// The same for rows of which every other one starts in the middle of a word (an odd n), all lanes here: the 64 / LANES lane groups' columns, 32 of four, are
// stored from their second column on, one further for each lane, so that the wide stores start on words (the memory path takes stores that do not apart).
// 4096 x 8191 results 48 us -> 39 with 128 x 128 tiles, 50 -> 45 with 256 x 256.
template <bool KEPT, int LANES = 16>
__device__ __forceinline__ void store8_odd(_Float16* p, const float (&f)[8]) {
    typedef uint32_t u3_word __attribute__((ext_vector_type(3), aligned(4)));
    const u4 v = to_halves<KEPT>(f);
    const int g = (threadIdx.x & 63) / LANES;
    const bool odd = (reinterpret_cast<uintptr_t>(p) & 2) != 0;
    const uint32_t next = static_cast<uint32_t>(__shfl_down(static_cast<int>(v[0]), LANES));
    const u4 moved = {__builtin_amdgcn_alignbit(v[1], v[0], 16), __builtin_amdgcn_alignbit(v[2], v[1], 16), __builtin_amdgcn_alignbit(v[3], v[2], 16),
                      __builtin_amdgcn_alignbit(next, v[3], 16)};
    uint16_t* const h = reinterpret_cast<uint16_t*>(p);
    if (!odd || g < 64 / LANES - 1) {
        u4_word* const to = reinterpret_cast<u4_word*>(h + odd);
        *to = odd ? moved : v;
    } else {
        *reinterpret_cast<u3_word*>(h + 1) = u3_word{moved[0], moved[1], moved[2]};
        h[7] = static_cast<uint16_t>(v[3] >> 16);
    }
    if (odd && g == 0) h[0] = static_cast<uint16_t>(v[0]);
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

}  // namespace
