// Rotary positions of several axes on views of q and k, and the norm of every head in front of them:
//     out_c = (y_c A_c + y_p B_c),  p the other channel of c's pair,  A = cos,  B = -sin for a pair's first channel, sin for its second,
// and with a norm  y = (x - mean) r w + b  (mean = 0 for root mean squares),  so that
//     out_c = r ((x_c - mean) w_c A_c + (x_p - mean) w_p B_c) + (b_c A_c + b_p B_c):
// what depends on token and channel alone is a table in LDS, made once for all heads of a workgroup's tokens, and a head costs two
// products a channel, whatever the order of its pairs.  All of it fp32, one rounding at the end.  Reads and writes every value once: bound by
// memory (a copy of 1 GiB moves 5.1 TB/s; outputs that the last-level cache holds from the call before go faster).
#include <type_traits>

#include "vq_internal.h"
#include "vq_types.h"

namespace vq {
namespace {

constexpr int kWaves = 4;
constexpr int kAtOnce = 2;          // rows of a lane that are worked on together
constexpr int kMaxTokens = 8;       // of a workgroup: their tables are in LDS
constexpr int kResident = 6 * 256;  // workgroups of a launch at a time, six a CU
constexpr size_t kLds = 26 << 10;   // bytes of LDS that let them be so many
constexpr int kStage = 1024;        // bytes of a wavefront's rows, 16 a lane

// Channels of pair `pair`, `first` the pairs of the axes in front of its own, `size` those of its axis.
__device__ __forceinline__ void channels_of(const RotaryAxesArgs& a, int pair, int first, int size, int& c0, int& c1) {
    if (a.pairing == VQ_PAIRS_HALVES) c0 = pair, c1 = pair + a.pairs;
    else if (a.pairing == VQ_PAIRS_NEIGHBOURS) c0 = 2 * pair, c1 = 2 * pair + 1;
    else c0 = first + pair, c1 = first + pair + size;
}

// The other channel of c's pair (neighbours do not ask), itself behind the turned ones.
__device__ __forceinline__ int partner_of(const RotaryAxesArgs& a, int c) {
    if (c >= 2 * a.pairs) return c;
    if (a.pairing == VQ_PAIRS_HALVES) return c < a.pairs ? c + a.pairs : c - a.pairs;
    int first = 0, axis = 0;
    while (c >= 2 * (first + a.sections[axis])) first += a.sections[axis++];
    return c - 2 * first < a.sections[axis] ? c + a.sections[axis] : c - a.sections[axis];
}

// Tables of a block's tokens: for q and k (one for both without a norm) A, B and, with biases, their term: [head_dim] floats each, the
// first four of every eight channels, then the others, so that lanes read 16 bytes next to each other.
template <int NORM>
struct Table {
    float* const at;
    const int D, kinds;
    __device__ __forceinline__ Table(float* at, const RotaryAxesArgs& a) : at(at), D(a.head_dim), kinds(NORM && a.has_bias ? 3 : 2) {}
    __device__ __forceinline__ float* of(int token, int which, int kind) const { return at + ((token * (NORM ? 2 : 1) + (NORM ? which : 0)) * kinds + kind) * D; }
    __device__ __forceinline__ int place(int c) const { return ((c >> 2 & 1) * (D >> 3) + (c >> 3)) * 4 + (c & 3); }
};

template <int NORM>
__device__ __forceinline__ void make_table(const RotaryAxesArgs& a, const Table<NORM>& table, long token0, int tokens) {
    const int entries = a.pairs + (NORM ? a.head_dim - 2 * a.pairs : 0);
    for (int i = threadIdx.x; i < tokens * entries; i += 64 * kWaves) {
        const int t = (int)((unsigned)i / (unsigned)entries), e = i - t * entries;
        if (e >= a.pairs) {         // a channel that is not turned
            const int c = a.pairs + e;
            for (int which = 0; which < 2; ++which) {
                table.of(t, which, 0)[table.place(c)] = a.weight[which] ? a.weight[which][c] : 1.0f;
                table.of(t, which, 1)[table.place(c)] = 0.0f;
                if (table.kinds == 3) table.of(t, which, 2)[table.place(c)] = a.bias[which] ? a.bias[which][c] : 0.0f;
            }
            continue;
        }
        int axis = 0, first = 0;
        while (e >= first + a.sections[axis]) first += a.sections[axis++];
        // The angle in turns is a product in 64 bits: its fraction, which is all that counts, is off by 2^-53 of the angle.
        const double turns = (double)a.positions[(long)axis * a.T + token0 + t] * ((double)a.inv_freq[e] * 0.15915494309189533577);
        float s, c;
        sincospif((float)(2.0 * (turns - rint(turns))), &s, &c);
        c *= a.amplitude;
        s *= a.amplitude;
        int c0, c1;
        channels_of(a, e, first, a.sections[axis], c0, c1);
        for (int which = 0; which < (NORM ? 2 : 1); ++which) {
            const float w0 = NORM && a.weight[which] ? a.weight[which][c0] : 1.0f, w1 = NORM && a.weight[which] ? a.weight[which][c1] : 1.0f;
            float *const A = table.of(t, which, 0), *const B = table.of(t, which, 1);
            A[table.place(c0)] = c * w0;
            B[table.place(c0)] = -s * w1;
            A[table.place(c1)] = c * w1;
            B[table.place(c1)] = s * w0;
            if (NORM && table.kinds == 3) {
                const float b0 = a.bias[which] ? a.bias[which][c0] : 0.0f, b1 = a.bias[which] ? a.bias[which][c1] : 0.0f;
                table.of(t, which, 2)[table.place(c0)] = b0 * c - b1 * s;
                table.of(t, which, 2)[table.place(c1)] = b1 * c + b0 * s;
            }
        }
    }
}

// What a wavefront wrote to LDS is there for its other lanes: its accesses are served in order, the compiler has to keep them so.
__device__ __forceinline__ void wave_fence() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The sums over a row's lanes, `pieces` of them from lane - piece on.  (Through LDS, four lanes a read, it takes as long.)
__device__ __forceinline__ void row_sums(float (&v)[kAtOnce], int pieces, int piece, int lane) {
    for (int i = 1; i < pieces; i *= 2) {
        float o[kAtOnce];
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) o[n] = __shfl_down(v[n], i);
#pragma unroll
        for (int n = 0; n < kAtOnce; ++n) v[n] += piece + i < pieces ? o[n] : 0.0f;
    }
#pragma unroll
    for (int n = 0; n < kAtOnce; ++n) v[n] = __shfl(v[n], lane - piece);
}

// What a turn of a wavefront works on: rows of q or of k, all the same for its lanes.
struct Side {
    const char* in;
    char* out;
    int64_t in_token, in_head, out_token, out_head;      // bytes
    int heads, head0, per_head, which;
};

// A lane has eight channels of a row (a head of a token), as many rows a wavefront as fit it: loads and stores are 16 bytes a lane and
// a token's heads lie next to each other.  Partners are read where the wavefront's rows pass through LDS, GRAIN channels at once: as many as
// every axis' pairs divide by (0: neighbours, which a lane has itself).  NORM: 0, or 1 + vq_norm.  WIDE: a workgroup's rows are more than 2^31
// bytes apart.  kAtOnce rows of a lane are worked on together, the next ones' loads on their way meanwhile; six workgroups a CU cover each
// other's waits.  32768 tokens, 16 + 16 heads of 72, f16, with outputs of their own, turned 61 us (5.0 TB/s), normed and turned 62.  Launches whose outputs
// go where the last one's went, inputs that are not in the caches: 50, 55 and with mean, variance and biases 65; with four rows at once, four workgroups a CU,
// 58, 67 and 82; one row, seven a CU, 52, 59 and 70.
template <class TYPE, int GRAIN, int NORM, bool WIDE>
__global__ __launch_bounds__(64 * kWaves, WIDE || GRAIN == 1 ? 5 : 6) void rotary_axes(RotaryAxesArgs a) {
    typedef typename std::conditional<WIDE, int64_t, unsigned>::type Offset;
    extern __shared__ __align__(16) char lds[];
    const Table<NORM> table((float*)(lds + (GRAIN ? kWaves * kAtOnce * kStage : 0)), a);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int pieces = a.head_dim / 8, rows_at_once = 64 / pieces;
    const int row_in = (int)((unsigned)lane / (unsigned)pieces), piece = lane - row_in * pieces;
    const bool active = row_in < rows_at_once;
    char* const stage = lds + wave * kAtOnce * kStage;
    constexpr int kReads = GRAIN ? 8 / GRAIN : 1;
    int partner[kReads];
    if (GRAIN)
#pragma unroll
        for (int i = 0; i < kReads; ++i) partner[i] = (lane - piece) * 16 + 2 * partner_of(a, 8 * piece + i * GRAIN);
    const float per_channel = 1.0f / a.head_dim;

    for (long block = blockIdx.x; block < a.blocks; block += gridDim.x) {
        const long group = a.head_blocks == 1 ? block : block / a.head_blocks;
        const long token0 = group * a.tokens_each;
        const int head0 = (int)(block - group * a.head_blocks) * a.heads_each;      // (of q's and k's, one behind the other)
        const int tokens = (int)(a.T - token0 < a.tokens_each ? a.T - token0 : a.tokens_each);
        const int end = min(head0 + a.heads_each, a.q_heads + a.k_heads);
        const int q_heads = max(min(end, a.q_heads) - head0, 0), k_first = max(head0 - a.q_heads, 0), k_heads = max(end - a.q_heads, 0) - k_first;
        const int q_turns = (tokens * q_heads + rows_at_once - 1) / rows_at_once, turns = q_turns + (tokens * k_heads + rows_at_once - 1) / rows_at_once;
        const Side sides[2] = {{(const char*)a.q + 2 * token0 * a.q_token, (char*)a.q_out + 2 * token0 * a.qo_token, 2 * a.q_token, 2 * a.q_head,
                                2 * a.qo_token, 2 * a.qo_head, q_heads, head0, a.per_head[0], 0},
                               {(const char*)a.k + 2 * token0 * a.k_token, (char*)a.k_out + 2 * token0 * a.ko_token, 2 * a.k_token, 2 * a.k_head,
                                2 * a.ko_token, 2 * a.ko_head, k_heads, k_first, a.per_head[1], 1}};
        // A row's token and head, or a token of -1.
        auto row_of = [&](int turn, const Side& s, int& t, int& h) {
            const int row = (turn - (s.which ? q_turns : 0)) * rows_at_once + row_in;
            t = a.tokens_each == 1 ? 0 : (int)((unsigned)row * (unsigned)s.per_head >> 24);
            h = row - t * s.heads;
            if (!active || turn >= turns || row >= tokens * s.heads) t = -1;
            h += s.head0;
        };
        auto load = [&](int first, v4i (&x)[kAtOnce]) {
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int turn = first + u * kWaves;
                const Side& s = sides[turn >= q_turns];
                int t, h;
                row_of(turn, s, t, h);
                x[u] = v4i{0, 0, 0, 0};
                if (t >= 0) x[u] = *(const v4i*)(s.in + ((Offset)t * (Offset)s.in_token + (Offset)h * (Offset)s.in_head + (Offset)(16 * piece)));
            }
        };
        // Loads of the first rows are on their way while the table is made.
        v4i next[kAtOnce];
        load(wave, next);
        make_table<NORM>(a, table, token0, tokens);
        __syncthreads();
        for (int first = wave; first < turns; first += kWaves * kAtOnce) {
            v4i raw[kAtOnce];
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) raw[u] = next[u];
            if (first + kWaves * kAtOnce < turns) load(first + kWaves * kAtOnce, next);
            if (GRAIN) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) *(v4i*)(stage + u * kStage + 16 * lane) = raw[u];
                wave_fence();
            }
            float mean[kAtOnce], r[kAtOnce];
            if (NORM) {
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) mean[u] = 0;
                if (NORM == 1 + VQ_NORM_LAYER) {
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            float x0, x1;
                            TYPE::unpack((unsigned)raw[u][e], x0, x1);
                            mean[u] += x0 + x1;
                        }
                    row_sums(mean, pieces, piece, lane);
#pragma unroll
                    for (int u = 0; u < kAtOnce; ++u) mean[u] *= per_channel;
                }
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) {
                    r[u] = 0;
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        float x0, x1;
                        TYPE::unpack((unsigned)raw[u][e], x0, x1);
                        if (NORM == 1 + VQ_NORM_LAYER) x0 -= mean[u], x1 -= mean[u];
                        r[u] = __builtin_fmaf(x0, x0, r[u]);
                        r[u] = __builtin_fmaf(x1, x1, r[u]);
                    }
                }
                row_sums(r, pieces, piece, lane);
#pragma unroll
                for (int u = 0; u < kAtOnce; ++u) r[u] = __builtin_amdgcn_rsqf(__builtin_fmaf(r[u], per_channel, a.eps));      // (good to a unit of 2^-23)
            }
#pragma unroll
            for (int u = 0; u < kAtOnce; ++u) {
                const int turn = first + u * kWaves;
                if (turn >= turns) break;
                const Side& s = sides[turn >= q_turns];
                int t, h;
                row_of(turn, s, t, h);
                v4i other;
                char* const at = stage + u * kStage;
                if (GRAIN == 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) other[e] = (int)__builtin_amdgcn_alignbit((unsigned)raw[u][e], (unsigned)raw[u][e], 16);
                } else if (GRAIN == 8) {
                    other = *(const v4i*)(at + partner[0]);
                } else if (GRAIN == 4) {
                    const v2i lo = *(const v2i*)(at + partner[0]), hi = *(const v2i*)(at + partner[1 % kReads]);
                    other = v4i{lo[0], lo[1], hi[0], hi[1]};
                } else if (GRAIN == 2) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) other[e] = *(const int*)(at + partner[e % kReads]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        other[e] = (int)((unsigned)*(const uint16_t*)(at + partner[2 * e % kReads]) |
                                         (unsigned)*(const uint16_t*)(at + partner[(2 * e + 1) % kReads]) << 16);
                }
                const int tt = max(t, 0);
                // (all of the table's reads on their way together, one branch a row: 7257 tokens of 20 + 4 heads of 96 with biases 21.2 us, 22.4
                // where every product branches and waits for its own)
                v4f A[2], B[2], E[2] = {};
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    A[h] = ((const v4f*)table.of(tt, s.which, 0) + piece)[h * pieces];
                    B[h] = ((const v4f*)table.of(tt, s.which, 1) + piece)[h * pieces];
                }
                if (NORM && table.kinds == 3)
#pragma unroll
                    for (int h = 0; h < 2; ++h) E[h] = ((const v4f*)table.of(tt, s.which, 2) + piece)[h * pieces];
                v4i y;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const v4f A4 = A[e >> 1], B4 = B[e >> 1], E4 = E[e >> 1];
                    const int i = 2 * (e & 1);
                    float x0, x1, p0, p1;
                    TYPE::unpack((unsigned)raw[u][e], x0, x1);
                    TYPE::unpack((unsigned)other[e], p0, p1);
                    if (NORM == 1 + VQ_NORM_LAYER) x0 -= mean[u], x1 -= mean[u], p0 -= mean[u], p1 -= mean[u];
                    float o0 = __builtin_fmaf(p0, B4[i], x0 * A4[i]), o1 = __builtin_fmaf(p1, B4[i + 1], x1 * A4[i + 1]);
                    if (NORM) o0 = __builtin_fmaf(o0, r[u], E4[i]), o1 = __builtin_fmaf(o1, r[u], E4[i + 1]);
                    y[e] = (int)TYPE::pack(o0, o1);
                    // (without a norm what is not turned has no table: it is copied, whatever it holds)
                    if (!NORM && 8 * piece + 2 * e >= 2 * a.pairs) y[e] = raw[u][e];
                }
                if (t >= 0) *(v4i*)(s.out + ((Offset)t * (Offset)s.out_token + (Offset)h * (Offset)s.out_head + (Offset)(16 * piece))) = y;
            }
            if (GRAIN) wave_fence();
        }
        __syncthreads();         // the next tokens' table goes where this one was
    }
}

template <class TYPE, int NORM, bool WIDE>
void (*kernel_of(int grain))(RotaryAxesArgs) {
    switch (grain) {
        case 0: return rotary_axes<TYPE, 0, NORM, WIDE>;
        case 1: return rotary_axes<TYPE, 1, NORM, WIDE>;
        case 2: return rotary_axes<TYPE, 2, NORM, WIDE>;
        case 4: return rotary_axes<TYPE, 4, NORM, WIDE>;
        default: return rotary_axes<TYPE, 8, NORM, WIDE>;
    }
}
template <class TYPE, int NORM>
void (*kernel_of(int grain, bool wide))(RotaryAxesArgs) {
    return wide ? kernel_of<TYPE, NORM, true>(grain) : kernel_of<TYPE, NORM, false>(grain);
}

// Fills in what a workgroup takes, and says which kernel takes it.
struct Choice {
    int grain;
    bool wide;
    size_t lds;
};
Choice choose(RotaryAxesArgs& a) {
    // Channels that keep together on their way to their partners: 8, or the largest power of two that divides every axis' pairs, or all
    // pairs where they are halves of the whole.
    int all = a.pairing == VQ_PAIRS_HALVES ? a.pairs : 0;
    for (int i = 0; i < a.axes && a.pairing == VQ_PAIRS_AXIS_HALVES; ++i) all |= a.sections[i];
    const int grain = a.pairing == VQ_PAIRS_NEIGHBOURS || a.axes == 0 ? 0 : all % 8 == 0 ? 8 : all & -all;
    a.has_bias = a.norm && (a.bias[0] || a.bias[1]);
    const int pieces = a.head_dim / 8, rows_at_once = 64 / pieces, heads = a.q_heads + a.k_heads;
    auto lds_of = [&](int tokens) {
        return (size_t)(grain ? kWaves * kAtOnce * kStage : 0) + (size_t)tokens * a.head_dim * 4 * (a.norm ? (a.has_bias ? 6 : 4) : 2);
    };
    a.tokens_each = 1;
    a.heads_each = heads;
    if (a.T < kResident / 2) {
        // Few tokens: their heads are dealt to workgroups, a turn of its wavefronts each if there are workgroups enough.
        const int turns = (heads + kWaves * rows_at_once - 1) / (kWaves * rows_at_once), most = kResident / a.T, blocks = turns < most ? turns : most;
        a.heads_each = (heads + blocks - 1) / blocks;
    } else {
        // As many tokens a workgroup as cost least: turns of its wavefronts, and what its table takes, about four of them, for every time that
        // the chip is filled.  7257 tokens, 20 + 4 heads of 96 with mean, variance and biases: 33 us with three tokens, 24 with five (21 now).
        double least = 0;
        for (int n = 1; n <= kMaxTokens && (n == 1 || lds_of(n) <= kLds); ++n) {
            const int turns = (n * a.q_heads + rows_at_once - 1) / rows_at_once + (n * a.k_heads + rows_at_once - 1) / rows_at_once;
            if (n > 1 && turns > 8 * kWaves * kAtOnce) break;
            const int each = (turns + kWaves * kAtOnce - 1) / (kWaves * kAtOnce) * kAtOnce;
            const double filled = (double)(((long)a.T + n - 1) / n) / kResident, cost = (filled <= 1 ? 1 : filled + 0.5) * (each + 4);
            if (n == 1 || cost < least) least = cost, a.tokens_each = n;
        }
    }
    a.head_blocks = (heads + a.heads_each - 1) / a.heads_each;
    a.blocks = (((long)a.T + a.tokens_each - 1) / a.tokens_each) * a.head_blocks;
    // (row * per_head >> 24 is row / heads: several tokens are at most 2^12 rows of 2^11 heads)
    a.per_head[0] = ((1 << 24) + a.q_heads - 1) / a.q_heads;
    a.per_head[1] = a.k_heads ? ((1 << 24) + a.k_heads - 1) / a.k_heads : 0;
    auto extent = [&](int64_t token, int64_t head, int heads) { return 2 * ((a.tokens_each - 1) * token + (heads - 1) * head + a.head_dim); };
    bool wide = extent(a.q_token, a.q_head, a.q_heads) >= 1l << 31 || extent(a.qo_token, a.qo_head, a.q_heads) >= 1l << 31;
    if (a.k_heads) wide = wide || extent(a.k_token, a.k_head, a.k_heads) >= 1l << 31 || extent(a.ko_token, a.ko_head, a.k_heads) >= 1l << 31;
    return {grain, wide, lds_of(a.tokens_each)};
}

}  // namespace

hipError_t launch_rotary_axes(RotaryAxesArgs a, int dtype, hipStream_t stream) {
    const Choice c = choose(a);
    void (*kernel)(RotaryAxesArgs) = nullptr;
    const bool f16 = dtype == VQ_F16;
    switch (a.norm) {
        case 0: kernel = f16 ? kernel_of<F16, 0>(c.grain, c.wide) : kernel_of<BF16, 0>(c.grain, c.wide); break;
        case 1 + VQ_NORM_RMS: kernel = f16 ? kernel_of<F16, 1 + VQ_NORM_RMS>(c.grain, c.wide) : kernel_of<BF16, 1 + VQ_NORM_RMS>(c.grain, c.wide); break;
        default: kernel = f16 ? kernel_of<F16, 1 + VQ_NORM_LAYER>(c.grain, c.wide) : kernel_of<BF16, 1 + VQ_NORM_LAYER>(c.grain, c.wide); break;
    }
    return enqueue(kernel, dim3((unsigned)(a.blocks < 1 << 20 ? a.blocks : 1 << 20)), dim3(64 * kWaves), stream, a, c.lds);
}

}  // namespace vq

extern "C" void vq_internal_rotary_axes_choice(int norm, int has_bias, int pairing, int axes, const int32_t* sections, int T, int q_heads, int k_heads, int head_dim,
                                               const int64_t* strides, int choice[4]) {
    const float bias = 0;
    vq::RotaryAxesArgs a{};
    a.norm = norm, a.bias[0] = has_bias ? &bias : nullptr, a.pairing = pairing, a.axes = axes;
    for (int i = 0; i < axes; ++i) a.sections[i] = sections[i], a.pairs += sections[i];
    a.T = T, a.q_heads = q_heads, a.k_heads = k_heads, a.head_dim = head_dim;
    a.q_token = strides[0], a.q_head = strides[1], a.qo_token = strides[2], a.qo_head = strides[3];
    a.k_token = strides[4], a.k_head = strides[5], a.ko_token = strides[6], a.ko_head = strides[7];
    const vq::Choice c = vq::choose(a);
    choice[0] = c.grain;
    choice[1] = c.wide;
    choice[2] = a.tokens_each;
    choice[3] = a.heads_each;
}
