// Activations and weights to microscaled 4-bit codes, and back.  Both are one pass over memory: 8192 x 4608 with a mask there and back
// 38.6 us, 3.9 TB/s of the 151 MB outside and 4.9 with the codes between (a copy moves 5.2).
#include "vq_internal.h"
#include "vq_mx4.h"

namespace vq {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = 4;      // rows that a thread has in flight

struct MxArgs {
    const void* x;
    const float* chan_mul;
    uint8_t* xq;
    uint8_t* x_scale;
    int M, K;
    int pieces;               // K / 8: a thread's share of a row is eight values
    int step_group, step_piece;   // what a grid of threads is in groups of rows and pieces of a row
};

// A thread's row group and piece, and the next ones a grid further.
struct Place {
    int group, piece;
    __device__ explicit Place(const MxArgs& a) {
        const unsigned i = blockIdx.x * kThreads + threadIdx.x;
        group = (int)(i / (unsigned)a.pieces);
        piece = (int)(i - (unsigned)group * (unsigned)a.pieces);
    }
    __device__ void step(const MxArgs& a) {
        group += a.step_group;
        piece += a.step_piece;
        if (piece >= a.pieces) {
            piece -= a.pieces;
            ++group;
        }
    }
};

template <class TYPE>
struct Eight {
    v4i v;
    __device__ __forceinline__ void load(const void* x, size_t at) { v = *(const v4i*)((const typename TYPE::T*)x + at); }
    __device__ __forceinline__ void get(float* t) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) TYPE::unpack((unsigned)v[i], t[2 * i], t[2 * i + 1]);
    }
};
struct F32 {};
template <>
struct Eight<F32> {
    v4f lo, hi;
    __device__ __forceinline__ void load(const void* x, size_t at) {
        lo = *(const v4f*)((const float*)x + at);
        hi = *(const v4f*)((const float*)x + at + 4);
    }
    __device__ __forceinline__ void get(float* t) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) t[i] = lo[i], t[4 + i] = hi[i];
    }
};

// Four neighbouring lanes hold a block, eight values each: loads of 16 bytes a lane and stores of 4 are whole lines
// of a wavefront, the largest magnitude takes two exchanges within four lanes.
template <class TYPE, bool MASK>
__global__ __launch_bounds__(kThreads) void mx4_quantize(MxArgs a) {
    const int stride = mx_scale_stride(a.K);
    const int groups = (a.M - 1) / kRows + 1;
    for (Place p(a); p.group < groups; p.step(a)) {
        const int left = a.M - p.group * kRows;
        Eight<TYPE> in[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r)
            in[r].load(a.x, ((size_t)p.group * kRows + min(r, left - 1)) * a.K + 8 * p.piece);
        float mul[8];
        if (MASK) {
            Eight<F32> m;
            m.load(a.chan_mul, 8 * p.piece);
            m.get(mul);
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r >= left) break;     // (the same for the four lanes of a block: they are in one row)
            float t[8];
            in[r].get(t);
            unsigned top = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (MASK) t[i] *= mul[i];
                top = max(top, magnitude(t[i]));
            }
            top = largest_of_block(top);
            const int byte = mx_scale_of(top);
            const size_t row = (size_t)p.group * kRows + r;
            *(unsigned*)(a.xq + row * (a.K / 2) + 4 * p.piece) = mx_encode(t, byte);
            if ((p.piece & 3) == 0) a.x_scale[row * stride + p.piece / 4] = (uint8_t)byte;
            if (p.piece == a.pieces - 1)
                for (int b = a.K / kMxBlock; b < stride; ++b) a.x_scale[row * stride + b] = 0;
        }
    }
}

template <class TYPE>
__device__ __forceinline__ void store_eight(void* x, size_t at, const float* t) {
    v4i o;
#pragma unroll
    for (int i = 0; i < 4; ++i) o[i] = (int)TYPE::pack(t[2 * i], t[2 * i + 1]);
    *(v4i*)((typename TYPE::T*)x + at) = o;
}
template <>
__device__ __forceinline__ void store_eight<F32>(void* x, size_t at, const float* t) {
    *(v4f*)((float*)x + at) = v4f{t[0], t[1], t[2], t[3]};
    *(v4f*)((float*)x + at + 4) = v4f{t[4], t[5], t[6], t[7]};
}

template <class TYPE>
__global__ __launch_bounds__(kThreads) void mx4_dequantize(MxArgs a) {
    const int stride = mx_scale_stride(a.K);
    const int groups = (a.M - 1) / kRows + 1;
    for (Place p(a); p.group < groups; p.step(a)) {
        const int left = a.M - p.group * kRows;
        unsigned code[kRows];
        int byte[kRows];
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            const size_t row = (size_t)p.group * kRows + min(r, left - 1);
            code[r] = *(const unsigned*)(a.xq + row * (a.K / 2) + 4 * p.piece);
            byte[r] = a.x_scale[row * stride + p.piece / 4];
        }
#pragma unroll
        for (int r = 0; r < kRows; ++r) {
            if (r >= left) break;
            // (byte 0 is 2^-127, which no float's exponent field says; byte 255 is NaN, as the float would not be)
            const float scale = byte[r] == 0 ? __builtin_bit_cast(float, 0x00400000)
                                : byte[r] == kMxNan ? __builtin_bit_cast(float, 0x7FC00000)
                                                    : __builtin_bit_cast(float, byte[r] << 23);
            float t[8];
            v2f two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[r], 1.0f, 0);
            t[0] = two[0] * scale, t[1] = two[1] * scale;
            two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[r], 1.0f, 1);
            t[2] = two[0] * scale, t[3] = two[1] * scale;
            two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[r], 1.0f, 2);
            t[4] = two[0] * scale, t[5] = two[1] * scale;
            two = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code[r], 1.0f, 3);
            t[6] = two[0] * scale, t[7] = two[1] * scale;
            store_eight<TYPE>((void*)a.x, ((size_t)p.group * kRows + r) * a.K + 8 * p.piece, t);
        }
    }
}

// Every thread of the grid takes at least one piece of a group of rows, up to some workgroups per CU; more rows are
// further turns.  Whole rows are K / 8 pieces, K / 32 of four lanes each: a block never straddles two wavefronts.
dim3 grid_of(MxArgs& a) {
    a.pieces = a.K / 8;
    const long work = (((long)a.M - 1) / kRows + 1) * a.pieces;
    long blocks = (work + kThreads - 1) / kThreads;
    if (blocks > 1 << 16) blocks = 1 << 16;
    const long threads = blocks * kThreads;
    a.step_group = (int)(threads / a.pieces);
    a.step_piece = (int)(threads % a.pieces);
    return dim3((unsigned)blocks);
}

}  // namespace

hipError_t launch_mx4_quantize(const void* x, int dtype, const float* chan_mul, uint8_t* xq, uint8_t* x_scale, int M, int K,
                               hipStream_t stream) {
    MxArgs a{x, chan_mul, xq, x_scale, M, K, 0, 0, 0};
    const dim3 grid = grid_of(a);
    void (*kernel)(MxArgs) =
        dtype == VQ_F16    ? (chan_mul ? mx4_quantize<F16, true> : mx4_quantize<F16, false>)
        : dtype == VQ_BF16 ? (chan_mul ? mx4_quantize<BF16, true> : mx4_quantize<BF16, false>)
                           : (chan_mul ? mx4_quantize<F32, true> : mx4_quantize<F32, false>);
    return enqueue(kernel, grid, dim3(kThreads), stream, a);
}

hipError_t launch_mx4_dequantize(const uint8_t* xq, const uint8_t* x_scale, void* x, int dtype, int M, int K,
                                 hipStream_t stream) {
    MxArgs a{x, nullptr, const_cast<uint8_t*>(xq), const_cast<uint8_t*>(x_scale), M, K, 0, 0, 0};
    const dim3 grid = grid_of(a);
    void (*kernel)(MxArgs) = dtype == VQ_F16 ? mx4_dequantize<F16> : dtype == VQ_BF16 ? mx4_dequantize<BF16> : mx4_dequantize<F32>;
    return enqueue(kernel, grid, dim3(kThreads), stream, a);
}

}  // namespace vq
