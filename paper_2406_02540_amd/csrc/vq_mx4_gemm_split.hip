// GEMM on microscaled 4-bit operands, few tokens or few channels: the wavefronts of a workgroup divide K.  Also the whole layer for up to
// sixteen tokens, which the workgroups quantize for themselves (a block's scale depends on its 32 values only).
#include "vq_internal.h"
#include "vq_mx4_product.h"

namespace vq {
namespace {

// Four channels of a token, with their bias, to memory.
template <class TYPE>
__device__ __forceinline__ void write_four(const Mx4GemmArgs& a, int m, int n, v4f sum) {
    if (m >= a.M) return;
    typename TYPE::T* const y = (typename TYPE::T*)a.y + (size_t)m * a.N + n;
    const typename TYPE::T* const bias = (const typename TYPE::T*)a.bias + n;
    if (a.N % 4 == 0) {
        if (n >= a.N) return;
        float f[4] = {0, 0, 0, 0};
        if (a.bias) {
            const v2i b4 = *(const v2i*)bias;
            TYPE::unpack((unsigned)b4[0], f[0], f[1]);
            TYPE::unpack((unsigned)b4[1], f[2], f[3]);
        }
        *(v2i*)y = v2i{(int)TYPE::pack(sum[0] + f[0], sum[1] + f[1]), (int)TYPE::pack(sum[2] + f[2], sum[3] + f[3])};
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (n + e < a.N) y[e] = (typename TYPE::T)(sum[e] + (a.bias ? (float)bias[e] : 0.0f));
    }
}

// Rows are loaded a whole line (256 codes) at a time, through LDS: operands straight from memory to the lanes that multiply them are 64
// bytes of a row at a time (240 x 4096 -> 2304 17.3 us so, 6.5 as it is).  Every wavefront has a contiguous part of K, LDS of its
// own and no barrier until the sums are joined.  (With two lines on their way at a time a workgroup takes a CU alone: 16 x 65536 -> 512
// 31.8 us, 27.0 with one; 64 x 4096 -> 4096 4.85 and 4.72.)
typedef __attribute__((address_space(3))) char* lds_bytes;

// Where a product's tokens come from: codes, or values that are quantized on the way.
enum XFrom { kCodes, kValues, kMaskedValues };

// Line `l` of the tokens row0 .. row0 + rows - 1 (16 at most), quantized into LDS: 32 lanes a row, eight values each.  The rows that do not
// exist keep what the LDS holds: their sums are not written, and no sum holds two tokens.
template <class TYPE, bool MASK>
__device__ __forceinline__ void quantize_line(const Mx4GemmArgs& a, int row0, int rows, int l, lds_bytes to, lds_bytes scales, int lane) {
    const int piece = lane & 31, k = 256 * l + 8 * piece;
    const bool in = k < a.K;
    float mul[8];
    if (MASK) {
        const v4f* const m = (const v4f*)(a.chan_mul + (in ? k : 0));
        const v4f lo = m[0], hi = m[1];
#pragma unroll
        for (int e = 0; e < 4; ++e) mul[e] = lo[e], mul[4 + e] = hi[e];
    }
    for (int r0 = 0; r0 < rows; r0 += 2) {
        const int r = r0 + (lane >> 5);
        const v4i v = *(const v4i*)((const typename TYPE::T*)a.x + (size_t)(row0 + min(r, rows - 1)) * a.K + (in ? k : 0));
        float t[8];
        unsigned top = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) TYPE::unpack((unsigned)v[e], t[2 * e], t[2 * e + 1]);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (MASK) t[e] *= mul[e];
            top = max(top, magnitude(t[e]));
        }
        top = largest_of_block(top);
        const int byte = in ? mx_scale_of(top) : 0;      // (behind the row's end: codes of zero, a scale that is a number)
        *(__attribute__((address_space(3))) unsigned*)(to + 128 * r + 16 * ((piece >> 2) ^ line_swizzle(r)) + 4 * (piece & 3)) = in ? mx_encode(t, byte) : 0;
        if ((piece & 3) == 0) scales[8 * r + (piece >> 2)] = (char)byte;
    }
}

template <class TYPE, int TT, int CC, int WAVES, XFrom X_FROM>
__global__ __launch_bounds__(64 * WAVES) void mx4_gemm_lines(Mx4GemmArgs a) {
    constexpr int kX = 16 * TT, kRows = 16 * (TT + CC), kLine = kRows * 128;
    constexpr int kOwn = kLine + 8 * kRows, kPart = WAVES * TT * CC * 1024;      // a wavefront's; the sums
    constexpr int kRowTurns = (kRows + 63) / 64;
    __shared__ __align__(128) char lds[WAVES * kOwn > kPart ? WAVES * kOwn : kPart];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int tiles_c = (a.N - 1) / (16 * CC) + 1;
    const int row0 = (int)(blockIdx.x / (unsigned)tiles_c) * kX, col0 = (int)(blockIdx.x % (unsigned)tiles_c) * (16 * CC);
    const int r = lane & 15, g = lane >> 4;
    const int blocks = a.K / kMxBlock, lines = (blocks - 1) / 8 + 1, stride = mx_scale_stride(a.K), row_bytes = a.K / 2;
    const int l1 = (int)((unsigned)lines * (unsigned)(wave + 1) / WAVES);
    const int rows = min(a.M - row0, kX);
    const v4i rx = X_FROM == kCodes ? make_rsrc(a.xq + (size_t)row0 * row_bytes, (unsigned)(rows * row_bytes)) : v4i{0, 0, 0, 0};
    const v4i rw = make_rsrc(a.wq + (size_t)col0 * row_bytes, (unsigned)(min(a.N - col0, 16 * CC) * row_bytes));
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds + wave * kOwn;
    const lds_bytes own = (lds_bytes)lds + wave * kOwn, own_scales = own + kLine;

    v4f acc[TT][CC] = {};
    for (int l = (int)((unsigned)lines * (unsigned)wave / WAVES); l < l1; ++l) {
        unsigned s[kRowTurns][2];           // the line's scales, a row a lane
#pragma unroll
        for (int i = 0; i < kRowTurns; ++i) {
            const int row = 64 * i + lane;
            const bool x = row < kX;
            const int from = x ? row0 + row : col0 + row - kX;
            const uint8_t* const p = (x ? a.x_scale : a.w_scale) + (size_t)from * stride + 8 * l;
#pragma unroll
            for (int d = 0; d < 2; ++d)
                s[i][d] = row < kRows && (X_FROM == kCodes || !x) && from < (x ? a.M : a.N) && 8 * l + 4 * d < stride ? *(const unsigned*)(p + 4 * d) : 0;
        }
#pragma unroll
        for (int i = X_FROM == kCodes ? 0 : kX / 8; i < kRows / 8; ++i) {
            const int row = 8 * i + (lane >> 3), chunk = (lane & 7) ^ line_swizzle(row), at = 128 * l + 16 * chunk;
            const bool x = 8 * i < kX;
            load_to_lds_16(x ? rx : rw, base + 1024 * i, at < row_bytes ? (x ? row : row - kX) * row_bytes + at : kNowhere, 0);
        }
#pragma unroll
        for (int i = 0; i < kRowTurns; ++i)
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                const int n = blocks - 8 * l - 4 * d;     // (blocks behind the row's end: codes of zero, a scale that is a number)
                const unsigned v = n >= 4 ? s[i][d] : n <= 0 ? 0 : s[i][d] & ((1u << 8 * n) - 1);
                if (64 * i + lane < kRows && (X_FROM == kCodes || 64 * i + lane >= kX)) *(__attribute__((address_space(3))) unsigned*)(own_scales + 8 * (64 * i + lane) + 4 * d) = v;
            }
        if constexpr (X_FROM != kCodes) quantize_line<TYPE, X_FROM == kMaskedValues>(a, row0, rows, l, own, own_scales, lane);
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        int xs[TT], ws[CC];
        const lds_bytes sp = own_scales + 8 * r + 2 * g;
#pragma unroll
        for (int t = 0; t < TT; ++t) xs[t] = *(__attribute__((address_space(3))) unsigned short*)(sp + 128 * t);
#pragma unroll
        for (int c = 0; c < CC; ++c) ws[c] = *(__attribute__((address_space(3))) unsigned short*)(sp + 8 * kX + 128 * c);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const lds_bytes at = own + 128 * r + 16 * ((2 * g + j) ^ line_swizzle(r));
            v4i x[TT], w[CC];
#pragma unroll
            for (int t = 0; t < TT; ++t) x[t] = *(__attribute__((address_space(3))) v4i*)(at + 2048 * t);
#pragma unroll
            for (int c = 0; c < CC; ++c) w[c] = *(__attribute__((address_space(3))) v4i*)(at + 128 * kX + 2048 * c);
#pragma unroll
            for (int t = 0; t < TT; ++t)
#pragma unroll
                for (int c = 0; c < CC; ++c)
                    acc[t][c] = j == 0 ? mx_mfma<0>(w[c], ws[c], x[t], xs[t], acc[t][c]) : mx_mfma<1>(w[c], ws[c], x[t], xs[t], acc[t][c]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");     // (read before the next line's loads land there)
    }
    __syncthreads();
    v4f* const part = (v4f*)lds;       // [WAVES][TT * CC][64]
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int c = 0; c < CC; ++c) part[(wave * TT * CC + t * CC + c) * 64 + lane] = acc[t][c];
    __syncthreads();
    for (int i = threadIdx.x; i < TT * CC * 64; i += 64 * WAVES) {
        v4f sum = part[i];
#pragma unroll
        for (int v = 1; v < WAVES; ++v) sum += part[v * TT * CC * 64 + i];
        write_four<TYPE>(a, row0 + 16 * (i / 64 / CC) + (i & 15), col0 + 16 * (i / 64 % CC) + 4 * (i >> 4 & 3), sum);
    }
}

template <class TYPE, int TT, int CC, int WAVES, XFrom X_FROM>
hipError_t launch_lines(const Mx4GemmArgs& a, hipStream_t stream) {
    const long tiles = (((long)a.M - 1) / (16 * TT) + 1) * (((long)a.N - 1) / (16 * CC) + 1);
    if (!mx4_gemm_takes(a.M, a.N) || tiles * 64 * WAVES >= 1l << 32) return hipErrorInvalidValue;
    return enqueue(mx4_gemm_lines<TYPE, TT, CC, WAVES, X_FROM>, dim3((unsigned)tiles), dim3(64 * WAVES), stream, a);
}

template <class TYPE>
hipError_t launch(int tile_t, int tile_c, const Mx4GemmArgs& a, hipStream_t stream) {
    if (tile_t == 48) return launch_lines<TYPE, 3, 3, 8, kCodes>(a, stream);
    if (tile_c == 64) return launch_lines<TYPE, 2, 4, 8, kCodes>(a, stream);
    return launch_lines<TYPE, 2, 2, 8, kCodes>(a, stream);
}
template <class TYPE>
hipError_t launch_layer(const Mx4GemmArgs& a, hipStream_t stream) {
    return a.chan_mul ? launch_lines<TYPE, 1, 1, 8, kMaskedValues>(a, stream) : launch_lines<TYPE, 1, 1, 8, kValues>(a, stream);
}

}  // namespace

hipError_t launch_mx4_gemm_lines(int tile_t, int tile_c, const Mx4GemmArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch<F16>(tile_t, tile_c, a, stream) : launch<BF16>(tile_t, tile_c, a, stream);
}

hipError_t launch_mx4_layer_small(const Mx4GemmArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch_layer<F16>(a, stream) : launch_layer<BF16>(a, stream);
}

}  // namespace vq
