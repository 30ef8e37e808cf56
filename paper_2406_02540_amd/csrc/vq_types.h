// The 16-bit types that entry points take side by side (vq_dtype), and their conversions.  gfx950 only.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace vq {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef int v2i __attribute__((ext_vector_type(2)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef float v2f __attribute__((ext_vector_type(2)));

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));

struct F16 {
    typedef _Float16 T;
    // Two values in a register, low half first: each rounded to nearest even.
    static __device__ __forceinline__ unsigned pack(float a, float b) {
        const half2v h = {(_Float16)a, (_Float16)b};
        return __builtin_bit_cast(unsigned, h);
    }
    static __device__ __forceinline__ void unpack(unsigned v, float& a, float& b) {
        const half2v h = __builtin_bit_cast(half2v, v);
        a = (float)h[0];
        b = (float)h[1];
    }
};
struct BF16 {
    typedef __bf16 T;
    static __device__ __forceinline__ unsigned pack(float a, float b) {
        const v2f f = {a, b};
        return __builtin_bit_cast(unsigned, __builtin_convertvector(f, bf2v));
    }
    static __device__ __forceinline__ void unpack(unsigned v, float& a, float& b) {
        a = __builtin_bit_cast(float, v << 16);
        b = __builtin_bit_cast(float, v & 0xFFFF0000u);
    }
};

}  // namespace vq
