// 4-bit projections: the layout of the weights, which the kernels that write it and those that read it share.
//
// W[j, i] = scale[j, i / group] * (code[j, i] - zero[j, i / group]): codes and zeros from 0 to 15 (zeros not given: 8), scales fp16, groups of 32, 64
// or 128 columns of a row.  A product contracts rows of the laid-out matrix with rows of activations; transposed, the laid-out matrix is W^T and the
// groups run across its rows, not along them.
//
// Codes: blocks of 16 rows x 128 columns, 1 KiB each, a row of blocks behind the other.  A block is one 16-byte load of a wave: lane 16 q + r holds row
// r, and its word m the columns 32 m + 8 q .. + 7, the operand of the m-th v_mfma_f32_16x16x32_f16 of the block.  In a word the eight codes lie such
// that two that follow each other are 16 bits apart, four bits further for each pair: a mask and a biased exponent make fp16 pairs of them.
// Rows go to blocks in pairs of 32: row 4 g + e of block 2 p + h is row 32 p + 8 g + 4 h + e of the matrix.  Lane group g then has eight consecutive columns
// of the result in two accumulators.
// Rows are padded to whole pairs of blocks, columns to whole blocks (of each half, where the matrix has two, the gate's and the up projection's) with
// codes that stand for 0.
//
// Scales, and zeros as 1024 + zero in fp16, in the order of the codes' rows: [block row][group][16]; transposed, where they vary along the
// contraction: [group][column].
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "lordba_i8.h"

namespace {

constexpr int64_t kI4Rows = 32, kI4Columns = 128;   // what rows and columns are padded to

struct I4Shape {   // of a laid-out matrix
    int64_t rows, cols;               // of one half's rows and of one half's columns, unpadded
    int row_halves, col_halves;
    int64_t tiles, blocks;            // blocks of 16 rows, blocks of 128 columns, all halves
    int64_t groups, scales;           // groups along a matrix row; scales in all
};
inline I4Shape i4_shape(int64_t rows, int64_t cols, int64_t group, int halves, bool transposed) {   // of W: rows in `halves` parts
    const int64_t part = rows / halves;
    I4Shape s;
    s.rows = transposed ? cols : part;
    s.cols = transposed ? part : cols;
    s.row_halves = transposed ? 1 : halves;
    s.col_halves = transposed ? halves : 1;
    s.tiles = (s.rows + kI4Rows - 1) / kI4Rows * 2 * s.row_halves;
    s.blocks = (s.cols + kI4Columns - 1) / kI4Columns * s.col_halves;
    s.groups = transposed ? (cols + group - 1) / group : s.blocks * (kI4Columns / group);
    s.scales = transposed ? s.groups * s.blocks * kI4Columns : s.tiles * s.groups * 16;
    return s;
}
inline bool i4_group(int64_t group) { return group == 32 || group == 64 || group == 128; }
constexpr int64_t kI4Most = 1 << 24;   // rows and columns

// Nibble of the word that holds code e of its eight.
constexpr int i4_nibble(int e) { return (e & 1) * 4 + (e >> 1); }
// The matrix row (of its half) that row r of block row t holds.
__host__ __device__ constexpr int64_t i4_row(int64_t t, int r) { return 32 * (t >> 1) + 8 * (r >> 2) + 4 * (t & 1) + (r & 3); }

constexpr uint16_t kZero8 = 0x6408;   // 1024 + 8 in fp16

// dgate and dup of the gated block, before they are rounded
__device__ __forceinline__ void slopes(float d, float gate, float up, float& dg, float& du) {
    // silu' = sigma (1 + gate (1 - sigma)) with 1 - sigma = e / (1 + e): no cancellation where sigma is near 1
    const float e = __expf(-fabsf(gate)), r = __builtin_amdgcn_rcpf(1.f + e);
    const float sigma = gate < 0.f ? e * r : r, rest = gate < 0.f ? r : e * r;
    dg = d * up * sigma * (1.f + gate * rest);
    du = d * gate * sigma;
}

}  // namespace

// dgate and dup of the gated block in fp16, [2, T, d_ff]
lordba_status lordba_i4_gated_grad(const void* dh, const void* gate_up, void* dgate_up, int64_t T, int64_t d_ff, hipStream_t stream);
