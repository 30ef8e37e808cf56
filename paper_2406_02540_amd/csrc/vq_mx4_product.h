// What the GEMMs on microscaled 4-bit operands share.
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 rows x 16 rows x 4 blocks: lane l holds one block of row l%16, 16 bytes of codes as
// they lie in memory, and its scale's byte.
#pragma once
#include "vq_gemm_common.h"
#include "vq_mx4.h"

namespace vq {

typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kNowhere = 0x7FFFFFF0;     // an offset behind every buffer: its lanes load zeros

// (4: e2m1; STEP: the byte of the scales)
template <int STEP>
__device__ __forceinline__ v4f mx_mfma(v4i w, int ws, v4i x, int xs, v4f acc) {
    const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, STEP, ws, STEP, xs);
}

// Operands in LDS lie in rows of one line, 128 bytes.  The order of blocks in a product is free as long as both operands agree: of
// a line's eight, lane group g = l/16 takes 2g and 2g + 1 in the line's two steps, so that a lane's two scales are one read.  The
// chunk of 16 bytes of a row lies at chunk ^ this: sixteen lanes that the LDS serves together (rows 0-3 and 12-15 of chunk c and 4-11
// of chunk c ^ 2, or the others) are then in different banks.
__device__ __forceinline__ int line_swizzle(int row) { return (row >> 1) & 5; }

}  // namespace vq
