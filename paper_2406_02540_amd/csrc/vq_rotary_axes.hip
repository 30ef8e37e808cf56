// Rotary positions of several axes, and the norm of every head in front of them: a wavefront a head.
#include "vq_internal.h"
#include "vq_types.h"

namespace vq {
namespace {

__device__ __forceinline__ float sum64(float v) {
#pragma unroll
    for (int i = 1; i < 64; i *= 2) v += __shfl_xor(v, i);
    return v;
}

template <class TYPE>
__global__ __launch_bounds__(256) void rotary_axes(RotaryAxesArgs a) {
    typedef typename TYPE::T T;
    __shared__ float head_of[4][VQ_MAX_HEAD_DIM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    float* const y = head_of[wave];
    const long all = (long)a.T * (a.q_heads + a.k_heads);
    const long turns = (all + 4l * gridDim.x - 1) / (4l * gridDim.x);
    for (long n = 0; n < turns; ++n) {
        const long i = (n * gridDim.x + blockIdx.x) * 4 + wave;
        const bool real = i < all;
        const long token = real ? i / (a.q_heads + a.k_heads) : 0;
        int h = real ? (int)(i - token * (a.q_heads + a.k_heads)) : 0;
        const bool is_k = h >= a.q_heads;
        if (is_k) h -= a.q_heads;
        const T* const x = is_k ? (const T*)a.k + token * a.k_token + h * a.k_head : (const T*)a.q + token * a.q_token + h * a.q_head;
        T* const out = is_k ? (T*)a.k_out + token * a.ko_token + h * a.ko_head : (T*)a.q_out + token * a.qo_token + h * a.qo_head;
        float v[2];
        for (int e = 0; e < 2; ++e) v[e] = lane + 64 * e < a.head_dim ? (float)x[lane + 64 * e] : 0.0f;
        if (a.norm) {
            if (a.norm == 1 + VQ_NORM_LAYER) {
                const float mean = sum64(v[0] + v[1]) / a.head_dim;
                for (int e = 0; e < 2; ++e) v[e] = lane + 64 * e < a.head_dim ? v[e] - mean : 0.0f;
            }
            const float scale = 1.0f / sqrtf(sum64(v[0] * v[0] + v[1] * v[1]) / a.head_dim + a.eps);
            for (int e = 0; e < 2; ++e) {
                const int c = lane + 64 * e;
                if (c < a.head_dim) {
                    v[e] *= scale;
                    if (a.weight[is_k]) v[e] *= a.weight[is_k][c];
                    if (a.bias[is_k]) v[e] += a.bias[is_k][c];
                }
            }
        }
        for (int e = 0; e < 2; ++e) y[lane + 64 * e] = v[e];
        __syncthreads();
        if (real) {
            for (int c = 2 * a.pairs + lane; c < a.head_dim; c += 64) out[c] = (T)y[c];
            if (lane < a.pairs) {
                int axis = 0, first = 0;
                while (lane >= first + a.sections[axis]) first += a.sections[axis++];
                const double turns2 = (double)a.positions[axis * (long)a.T + token] * ((double)a.inv_freq[lane] * 0.15915494309189533577);
                float s, c;
                sincospif((float)(2.0 * (turns2 - rint(turns2))), &s, &c);
                c *= a.amplitude, s *= a.amplitude;
                const int i0 = a.pairing == VQ_PAIRS_HALVES ? lane : a.pairing == VQ_PAIRS_NEIGHBOURS ? 2 * lane : first + lane;
                const int i1 = a.pairing == VQ_PAIRS_HALVES ? lane + a.pairs : a.pairing == VQ_PAIRS_NEIGHBOURS ? 2 * lane + 1 : first + lane + a.sections[axis];
                out[i0] = (T)(y[i0] * c - y[i1] * s);
                out[i1] = (T)(y[i1] * c + y[i0] * s);
            }
        }
        __syncthreads();
    }
}

}  // namespace

hipError_t launch_rotary_axes(RotaryAxesArgs a, int dtype, hipStream_t stream) {
    const long blocks = ((long)a.T * (a.q_heads + a.k_heads) + 3) / 4;
    return enqueue(dtype == VQ_F16 ? rotary_axes<F16> : rotary_axes<BF16>, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), stream, a);
}

}  // namespace vq
