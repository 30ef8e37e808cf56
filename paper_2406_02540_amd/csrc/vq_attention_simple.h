// A wavefront a query row: 64 keys at a time, a lane a key for the scores and two channels for the outputs.
#pragma once
#include "vq_attention.h"

namespace vq {

// KEYS(row's token): seen(key), k(key), v(key), count.
template <class TYPE, class ARGS, class KEYS>
__device__ __forceinline__ void attention_simple(const ARGS& a) {
    typedef typename TYPE::T T;
    __shared__ float q_of[4][VQ_MAX_HEAD_DIM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const long rows = (long)a.Tq * a.heads, turns = (rows + 4l * gridDim.x - 1) / (4l * gridDim.x);
    for (long n = 0; n < turns; ++n) {
        const long row = (n * gridDim.x + blockIdx.x) * 4 + wave;
        const int at = row < rows ? (int)(row / a.heads) : 0, head = row < rows ? (int)(row - (long)at * a.heads) : 0;
        int b = a.sequences - 1;
        while (b >= 0) {
            const Span s = span_of(a, b);
            if (at >= s.q0 && at < s.q0 + s.n) break;
            --b;
        }
        const bool real = row < rows && b >= 0;
        const Span s = span_of(a, b < 0 ? 0 : b);
        for (int c = lane; c < a.head_dim; c += 64) q_of[wave][c] = (float)((const T*)a.q)[at * a.q_token + head * a.q_head + c];
        __syncthreads();
        if (real) {
            const KEYS keys(a, s, at - s.q0, head / a.group);
            float m = -__builtin_inff(), l = 0, o[2] = {0, 0};
            for (int k0 = 0; k0 < keys.count; k0 += 64) {
                const int key = k0 + lane;
                const bool seen = key < keys.count && keys.seen(key);
                float score = -__builtin_inff();
                if (seen) {
                    const T* const k = keys.template k<T>(key);
                    score = 0;
                    for (int c = 0; c < a.head_dim; ++c) score += q_of[wave][c] * (float)k[c];
                    score *= a.scale_log2;
                }
                float top = score;
                for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
                if (!__any(seen)) continue;
                const float up = fmaxf(m, top), old = exp2f(m - up), p = exp2f(score - up);
                m = up;
                l = l * old + p;
                o[0] *= old, o[1] *= old;
                for (int i = 0; i < 64; ++i) {
                    const float w = __shfl(p, i);
                    if (w == 0.0f) continue;
                    const T* const v = keys.template v<T>(k0 + i);
                    if (lane < a.head_dim) o[0] += w * (float)v[lane];
                    if (lane + 64 < a.head_dim) o[1] += w * (float)v[lane + 64];
                }
            }
            for (int i = 1; i < 64; i *= 2) l += __shfl_xor(l, i);
            const float inv = l > 0 ? 1.0f / l : 0.0f;      // (a sum that is no number leaves outputs that are none)
            T* const out = (T*)a.out + at * a.o_token + head * a.o_head;
            for (int e = 0; e < 2; ++e)
                if (lane + 64 * e < a.head_dim) out[lane + 64 * e] = (T)(o[e] * inv);
        }
        __syncthreads();
    }
}

}  // namespace vq
