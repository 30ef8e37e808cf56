// GEMM on microscaled 4-bit operands, few tokens or few channels: the wavefronts of a workgroup divide K.
//
// y[m,n] = sum over blocks of 2^(Ex + Ew) * (sum of 32 products of codes) + bias[n], on v_mfma_scale_f32_16x16x128_f8f6f4: 16
// channels x 16 tokens x 4 blocks, the channels as rows so that a lane ends with four neighbouring channels of
// a token.  Lane l holds the whole block l/16 of row l%16, 16 bytes as they lie in memory, and its scale's byte: operands
// come straight from memory.
#include "vq_internal.h"
#include "vq_mx4.h"

namespace vq {
namespace {

typedef int v8i __attribute__((ext_vector_type(8)));

constexpr int kStepBlocks = 4;    // blocks of K that an MFMA takes

__device__ __forceinline__ v4f mx_mfma(v4i w, int ws, v4i x, int xs, v4f acc) {
    const v8i a = {w[0], w[1], w[2], w[3], 0, 0, 0, 0}, b = {x[0], x[1], x[2], x[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(a, b, acc, 4, 4, 0, ws, 0, xs);   // (4: e2m1)
}

// The block `kb` of a row; behind the row's end zeros, whatever the other operand has there.
__device__ __forceinline__ void load_block(const uint8_t* q, const uint8_t* s, int row, int kb, int K, v4i& v, int& scale) {
    const bool in = kb < K / kMxBlock;
    const int b = in ? kb : 0;
    v = *(const v4i*)(q + (size_t)row * (K / 2) + 16 * b);
    scale = s[(size_t)row * mx_scale_stride(K) + b];
    if (!in) v = v4i{0, 0, 0, 0}, scale = 0;
}

// TT x CC blocks of 16 tokens x 16 channels a workgroup.
template <class TYPE, int TT, int CC, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void mx4_gemm_split(Mx4GemmArgs a) {
    __shared__ v4f part[WAVES][TT * CC][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int tiles_c = (a.N - 1) / (16 * CC) + 1;
    const int row0 = (int)(blockIdx.x / (unsigned)tiles_c) * (16 * TT), col0 = (int)(blockIdx.x % (unsigned)tiles_c) * (16 * CC);
    const int r = lane & 15, g = lane >> 4;
    v4f acc[TT][CC] = {};
    const int steps = (a.K / kMxBlock - 1) / kStepBlocks + 1;
    for (int s = wave; s < steps; s += WAVES) {
        v4i x[TT], w[CC];
        int xs[TT], ws[CC];
#pragma unroll
        for (int c = 0; c < CC; ++c) load_block(a.wq, a.w_scale, min(col0 + 16 * c + r, a.N - 1), kStepBlocks * s + g, a.K, w[c], ws[c]);
#pragma unroll
        for (int t = 0; t < TT; ++t) load_block(a.xq, a.x_scale, min(row0 + 16 * t + r, a.M - 1), kStepBlocks * s + g, a.K, x[t], xs[t]);
#pragma unroll
        for (int t = 0; t < TT; ++t)
#pragma unroll
            for (int c = 0; c < CC; ++c) acc[t][c] = mx_mfma(w[c], ws[c], x[t], xs[t], acc[t][c]);
    }
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int c = 0; c < CC; ++c) part[wave][t * CC + c][lane] = acc[t][c];
    __syncthreads();
    for (int i = threadIdx.x; i < TT * CC * 64; i += 64 * WAVES) {
        const int b = i >> 6, l = i & 63;
        v4f sum = part[0][b][l];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v][b][l];
        const int m = row0 + 16 * (b / CC) + (l & 15), n = col0 + 16 * (b % CC) + 4 * (l >> 4);
        if (m >= a.M) continue;
        typename TYPE::T* y = (typename TYPE::T*)a.y + (size_t)m * a.N + n;
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) y[e] = (typename TYPE::T)(sum[e] + (a.bias ? (float)((const typename TYPE::T*)a.bias)[n + e] : 0.0f));
    }
}

}  // namespace

hipError_t launch_mx4_gemm(const Mx4GemmArgs& a, int dtype, hipStream_t stream) {
    constexpr int TT = 2, CC = 2, WAVES = 4;
    const long tiles = (((long)a.M - 1) / (16 * TT) + 1) * (((long)a.N - 1) / (16 * CC) + 1);
    if (tiles * 64 * WAVES >= 1l << 32) return hipErrorInvalidValue;
    return enqueue(dtype == VQ_F16 ? mx4_gemm_split<F16, TT, CC, WAVES> : mx4_gemm_split<BF16, TT, CC, WAVES>, dim3((unsigned)tiles),
                   dim3(64 * WAVES), stream, a);
}

}  // namespace vq
