// Rotary positions on views of q and k: out_a = a c - b s, out_b = b c + a s for the pairs of a head's first rot_dim
// channels, the rest copied.  Reads and writes every value once: bound by memory (a copy of 1 GiB moves 5.2 TB/s).
#include "vq_internal.h"
#include "vq_types.h"

namespace vq {
namespace {

constexpr int kThreads = 256;
constexpr int kAtOnce = 4;

// (cos, sin) of position * frequency, times the amplitude.  The angle in turns is a product in 64 bits: its fraction, which is
// all that counts, is off by 2^-53 of the angle, 2^-33 of a turn at position 2^20; in 32 bits it would be an eighth.
__device__ __forceinline__ void rotation(int position, float freq, float amplitude, float& c, float& s) {
    const double turns = (double)position * ((double)freq * 0.15915494309189533577);
    sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
    c *= amplitude;
    s *= amplitude;
}

// A thread takes four neighbouring pairs of a token, computes their angles once and turns them in every `lanes_h`-th head, q's and
// k's one after the other (threads behind the pairs copy eight channels that are not turned).  Neighbouring threads take
// neighbouring pairs, then heads: a wavefront's accesses cover whole rows of a token.
template <class TYPE, bool INTERLEAVED>
__global__ __launch_bounds__(kThreads) void rotary(RotaryArgs a) {
    const int pieces = a.copied_from + a.copied;       // per head: four pairs, or eight channels to copy
    const int heads = a.q_heads + a.k_heads;
    const long step = (long)gridDim.x * kThreads, all = (long)a.T * a.lanes_h * pieces;
    for (long i = (long)blockIdx.x * kThreads + threadIdx.x; i < all; i += step) {
        long rest;
        int piece, h, token;
        if (all < 1l << 32) {      // (a 64-bit division is a hundred instructions)
            const unsigned u = (unsigned)i / (unsigned)pieces;
            piece = (int)((unsigned)i - u * (unsigned)pieces);
            token = (int)(u / (unsigned)a.lanes_h);
            h = (int)(u - (unsigned)token * (unsigned)a.lanes_h);
        } else {
            rest = i / pieces;
            piece = (int)(i - rest * pieces);
            token = (int)(rest / a.lanes_h);
            h = (int)(rest - (long)token * a.lanes_h);
        }
        typedef typename TYPE::T T;
        const T* const q = (const T*)a.q + token * a.q_token;
        const T* const k = (const T*)a.k + token * a.k_token;
        T* const qo = (T*)a.q_out + token * a.qo_token;
        T* const ko = (T*)a.k_out + token * a.ko_token;
        if (piece >= a.copied_from) {
            const int at = a.rot_dim + 8 * (piece - a.copied_from);
            for (; h < heads; h += a.lanes_h) {
                const bool is_q = h < a.q_heads;
                const int hk = h - a.q_heads;
                *(v4i*)((is_q ? qo + h * a.qo_head : ko + hk * a.ko_head) + at) =
                    *(const v4i*)((is_q ? q + h * a.q_head : k + hk * a.k_head) + at);
            }
            continue;
        }
        const int position = a.positions[token];
        const v4f freq = *(const v4f*)(a.inv_freq + 4 * piece);
        float c[4], s[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) rotation(position, freq[e], a.amplitude, c[e], s[e]);
        const int half = a.rot_dim / 2;
        // (kAtOnce heads' loads are on their way together: 32768 tokens, 16 + 16 heads of 72, halves 70 us with one, 65 so,
        // 4.3 and 4.7 TB/s; neighbouring pairs 51.6 and 49.3)
        for (; h < heads; h += kAtOnce * a.lanes_h) {
            v4i in[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int hu = h + u * a.lanes_h;
                if (hu >= heads) break;
                const T* const from = hu < a.q_heads ? q + hu * a.q_head : k + (hu - a.q_heads) * a.k_head;
                if (INTERLEAVED) {
                    in[u] = *(const v4i*)(from + 8 * piece);
                } else {
                    const v2i va = *(const v2i*)(from + 4 * piece), vb = *(const v2i*)(from + half + 4 * piece);
                    in[u] = v4i{va[0], va[1], vb[0], vb[1]};
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int hu = h + u * a.lanes_h;
                if (hu >= heads) break;
                T* const out = hu < a.q_heads ? qo + hu * a.qo_head : ko + (hu - a.q_heads) * a.ko_head;
                float x[4], y[4];
                v4i o;
                if (INTERLEAVED) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        TYPE::unpack((unsigned)in[u][e], x[e], y[e]);
                        o[e] = (int)TYPE::pack(x[e] * c[e] - y[e] * s[e], y[e] * c[e] + x[e] * s[e]);
                    }
                    *(v4i*)(out + 8 * piece) = o;
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int i0 = 2 * e, i1 = 2 * e + 1;
                        TYPE::unpack((unsigned)in[u][e], x[i0], x[i1]);
                        TYPE::unpack((unsigned)in[u][2 + e], y[i0], y[i1]);
                        o[e] = (int)TYPE::pack(x[i0] * c[i0] - y[i0] * s[i0], x[i1] * c[i1] - y[i1] * s[i1]);
                        o[2 + e] = (int)TYPE::pack(y[i0] * c[i0] + x[i0] * s[i0], y[i1] * c[i1] + x[i1] * s[i1]);
                    }
                    *(v2i*)(out + 4 * piece) = v2i{o[0], o[1]};
                    *(v2i*)(out + half + 4 * piece) = v2i{o[2], o[3]};
                }
            }
        }
    }
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int dtype, int interleaved, hipStream_t stream) {
    const bool in_place = a.q == a.q_out && (a.k_heads == 0 || a.k == a.k_out);
    a.copied_from = a.rot_dim / 8;
    a.copied = in_place ? 0 : (a.head_dim - a.rot_dim) / 8;
    const int pieces = a.copied_from + a.copied, heads = a.q_heads + a.k_heads;
    // heads that a thread turns one after another: as many as leave the chip full
    int turns = 8;
    while (turns > 1 && (long)a.T * pieces * heads / turns < 256l * 2048) turns /= 2;
    a.lanes_h = (heads + turns - 1) / turns;
    const long all = (long)a.T * a.lanes_h * pieces;
    long blocks = (all + kThreads - 1) / kThreads;
    if (blocks > 1 << 20) blocks = 1 << 20;
    void (*kernel)(RotaryArgs) = dtype == VQ_F16 ? (interleaved ? rotary<F16, true> : rotary<F16, false>)
                                                 : (interleaved ? rotary<BF16, true> : rotary<BF16, false>);
    return enqueue(kernel, dim3((unsigned)blocks), dim3(kThreads), stream, a);
}

}  // namespace vq
