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

// A thread takes PAIRS neighbouring pairs of a token, computes their angles once and turns them in every `lanes_h`-th head, q's and
// k's one after the other (threads behind the pairs copy as many channels that are not turned).  Neighbouring threads take
// neighbouring pairs, then heads: a wavefront's accesses cover whole rows of a token.  Four pairs where the heads' turned part
// divides by them, else two, else one: the second halves start at rot_dim / 2, and with them the accesses' alignment.  (32768 tokens, 16 + 16 heads of 72, halves, out of place:
// all 72 channels turned 70 us, 36 of them 117, 18 159: the bytes are the same, in accesses of 4 and 2 bytes a lane instead of 8.)
template <class TYPE, bool INTERLEAVED, int PAIRS>
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
        typedef int Piece __attribute__((ext_vector_type(PAIRS)));          // a piece's channels, neighbours in pairs
        typedef short Half __attribute__((ext_vector_type(PAIRS)));         // those of one half
        typedef short Both __attribute__((ext_vector_type(2 * PAIRS)));
        typedef float Angles __attribute__((ext_vector_type(PAIRS)));
        const T* const q = (const T*)a.q + token * a.q_token;
        const T* const k = (const T*)a.k + token * a.k_token;
        T* const qo = (T*)a.q_out + token * a.qo_token;
        T* const ko = (T*)a.k_out + token * a.ko_token;
        if (piece >= a.copied_from) {
            const int at = a.rot_dim + 2 * PAIRS * (piece - a.copied_from);
            for (; h < heads; h += a.lanes_h) {
                const bool is_q = h < a.q_heads;
                const int hk = h - a.q_heads;
                *(Piece*)((is_q ? qo + h * a.qo_head : ko + hk * a.ko_head) + at) =
                    *(const Piece*)((is_q ? q + h * a.q_head : k + hk * a.k_head) + at);
            }
            continue;
        }
        const int position = a.positions[token];
        const Angles freq = *(const Angles*)(a.inv_freq + PAIRS * piece);
        float c[PAIRS], s[PAIRS];
#pragma unroll
        for (int e = 0; e < PAIRS; ++e) rotation(position, freq[e], a.amplitude, c[e], s[e]);
        const int half = a.rot_dim / 2;
        // (kAtOnce heads' loads are on their way together: 32768 tokens, 16 + 16 heads of 72, halves 73.3 us with one, 70.0 so, 4.3 TB/s;
        // neighbouring pairs 64.7 and 60.8, 5.0 TB/s; captured, inputs that are not in the caches)
        for (; h < heads; h += kAtOnce * a.lanes_h) {
            Piece in[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int hu = h + u * a.lanes_h;
                if (hu >= heads) break;
                const T* const from = hu < a.q_heads ? q + hu * a.q_head : k + (hu - a.q_heads) * a.k_head;
                if (INTERLEAVED) {
                    in[u] = *(const Piece*)(from + 2 * PAIRS * piece);
                } else {
                    const Half first = *(const Half*)(from + PAIRS * piece), second = *(const Half*)(from + half + PAIRS * piece);
                    Both both;
#pragma unroll
                    for (int e = 0; e < PAIRS; ++e) both[e] = first[e], both[PAIRS + e] = second[e];
                    in[u] = __builtin_bit_cast(Piece, both);
                }
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int hu = h + u * a.lanes_h;
                if (hu >= heads) break;
                T* const out = hu < a.q_heads ? qo + hu * a.qo_head : ko + (hu - a.q_heads) * a.ko_head;
                float x[PAIRS], y[PAIRS];
                Piece o;
                if (INTERLEAVED || PAIRS == 1) {
#pragma unroll
                    for (int e = 0; e < PAIRS; ++e) {
                        TYPE::unpack((unsigned)in[u][e], x[e], y[e]);
                        o[e] = (int)TYPE::pack(x[e] * c[e] - y[e] * s[e], y[e] * c[e] + x[e] * s[e]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < PAIRS / 2; ++e) {
                        const int i0 = 2 * e, i1 = 2 * e + 1, b = PAIRS / 2 + e;
                        TYPE::unpack((unsigned)in[u][e], x[i0], x[i1]);
                        TYPE::unpack((unsigned)in[u][b], y[i0], y[i1]);
                        o[e] = (int)TYPE::pack(x[i0] * c[i0] - y[i0] * s[i0], x[i1] * c[i1] - y[i1] * s[i1]);
                        o[b] = (int)TYPE::pack(y[i0] * c[i0] + x[i0] * s[i0], y[i1] * c[i1] + x[i1] * s[i1]);
                    }
                }
                if (INTERLEAVED) {
                    *(Piece*)(out + 2 * PAIRS * piece) = o;
                } else {
                    const Both both = __builtin_bit_cast(Both, o);
                    Half first, second;
#pragma unroll
                    for (int e = 0; e < PAIRS; ++e) first[e] = both[e], second[e] = both[PAIRS + e];
                    *(Half*)(out + PAIRS * piece) = first;
                    *(Half*)(out + half + PAIRS * piece) = second;
                }
            }
        }
    }
}

template <class TYPE, bool INTERLEAVED>
void (*kernel_of(int pairs))(RotaryArgs) {
    return pairs == 4 ? rotary<TYPE, INTERLEAVED, 4> : pairs == 2 ? rotary<TYPE, INTERLEAVED, 2> : rotary<TYPE, INTERLEAVED, 1>;
}

}  // namespace

hipError_t launch_rotary(RotaryArgs a, int dtype, int interleaved, hipStream_t stream) {
    const bool in_place = a.q == a.q_out && (a.k_heads == 0 || a.k == a.k_out);
    const int pairs = a.rot_dim % 8 == 0 ? 4 : a.rot_dim % 4 == 0 ? 2 : 1;
    a.copied_from = a.rot_dim / (2 * pairs);
    a.copied = in_place ? 0 : (a.head_dim - a.rot_dim) / (2 * pairs);
    const int pieces = a.copied_from + a.copied, heads = a.q_heads + a.k_heads;
    // heads that a thread turns one after another: as many as leave the chip full
    int turns = 8;
    while (turns > 1 && (long)a.T * pieces * heads / turns < 256l * 2048) turns /= 2;
    a.lanes_h = (heads + turns - 1) / turns;
    const long all = (long)a.T * a.lanes_h * pieces;
    long blocks = (all + kThreads - 1) / kThreads;
    if (blocks > 1 << 20) blocks = 1 << 20;
    void (*kernel)(RotaryArgs) = dtype == VQ_F16 ? (interleaved ? kernel_of<F16, true>(pairs) : kernel_of<F16, false>(pairs))
                                                 : (interleaved ? kernel_of<BF16, true>(pairs) : kernel_of<BF16, false>(pairs));
    return enqueue(kernel, dim3((unsigned)blocks), dim3(kThreads), stream, a);
}

}  // namespace vq
