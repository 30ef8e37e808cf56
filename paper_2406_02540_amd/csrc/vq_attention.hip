// Attention whose wavefronts divide the keys: few query rows per sequence (new tokens, short sequences).
#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kRows = 32;       // query rows of a tile: the columns of an MFMA block
constexpr int kKeys = 32;       // keys of a wavefront's tile
constexpr float kInf = __builtin_inff();

// Eight channels of a row: normalised to the output.
template <class TYPE>
__device__ __forceinline__ void write_outputs(const AttentionArgs& a, int token, int head, int c, const float* o, float l) {
    const float inv = l > 0 ? 1.0f / l : 0.0f;
    v4i y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (int)TYPE::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    *(v4i*)((typename TYPE::T*)a.out + token * a.o_token + head * a.o_head + c) = y;
}
// Or as they are, where other workgroups have more of the row's keys.
template <class TYPE>
__device__ __forceinline__ void write_eight_of_row(const AttentionArgs& a, int token, int head, int split, int c, const float* o, float m, float l) {
    if (a.split_shift == 0) return write_outputs<TYPE>(a, token, head, c, o, l);
    const size_t slot = ((size_t)split * a.Tq + token) * a.heads + head;
    *(v4f*)(a.part_o + slot * a.head_dim + c) = v4f{o[0], o[1], o[2], o[3]};
    *(v4f*)(a.part_o + slot * a.head_dim + c + 4) = v4f{o[4], o[5], o[6], o[7]};
    if (c == 0) *(v2f*)(a.part_ml + slot * 2) = v2f{m, l};
}

// Every wavefront takes tiles of 32 keys of its own, every WAVES-th of the workgroup's: loads into LDS of its own, no
// barrier; at the end the wavefronts' rows are joined.  A key is multiplied by 32 rows, however few there are: bound by the reads of K
// and V.  16 sequences of one token over up to 32768 keys, 32 heads on 8 of 128, 170 us, 4.7 TB/s of 791 MB (a copy moves 5.2); 64 over
// 4096 215 us, 5.0 TB/s; one over 32768 39 us, 3.4 TB/s.  CHUNKS: 16-byte chunks of a key in LDS (8, 12, 16); STEPS: of 16 channels;
// STAGES: tiles of a wavefront in LDS.
template <class TYPE, int CHUNKS, int STEPS, int WAVES, int STAGES>
__global__ __launch_bounds__(64 * WAVES) void attention_rows(AttentionArgs a) {
    constexpr int BLOCKS = CHUNKS / 4;                 // of 32 channels
    constexpr int kTile = kKeys * CHUNKS * 16;         // bytes
    constexpr int kStage = 2 * kTile;                  // K, V
    constexpr int kPitch = 32 * BLOCKS + 4;            // floats of a row where the wavefronts' sums meet
    constexpr int kLoads = 2 * kKeys * CHUNKS / 64;    // of a stage, per lane
    constexpr int kBytes = WAVES * STAGES * kStage;
    static_assert(WAVES == 1 || WAVES * kRows * (kPitch + 2) * 4 <= kBytes, "the sums fit where the stages were");
    __shared__ __align__(16) char lds[kBytes];
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5;
    int kv, item;
    if (!place_of(a, kv, item)) return;
    const int split = item & ((1 << a.split_shift) - 1), b = item >> a.split_shift;
    const Span s = span_of(a, b);
    const int rows = s.n * a.group;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    lds_bytes const own = (lds_bytes)lds + wave * STAGES * kStage;
    const unsigned base = (unsigned)(uintptr_t)own;
    const TileLoader<CHUNKS, kKeys, 64, false> k_load((int)(2 * a.k_token), head_bytes, lane);
    const TileLoader<CHUNKS, kKeys, 64, true> v_load((int)(2 * a.v_token), head_bytes, lane);
    const KeyReader<CHUNKS, STEPS> k_read(own, lane);
    const ValueReader<CHUNKS> v_read(own, lane);

    for (int row0 = 0; row0 < rows; row0 += kRows) {
        const int r = min(row0 + (lane & 31), rows - 1);
        const bool real = row0 + (lane & 31) < rows;
        const int token = token_of(a, r), head = kv * a.group + r - token * a.group;
        // keys: this lane's row's, the tile's most
        const int visible = keys_seen(a, s, token);
        const int end = __builtin_amdgcn_readfirstlane(keys_seen(a, s, token_of(a, min(row0 + kRows, rows) - 1)));
        const int tiles = (end + kKeys - 1) / kKeys;
        const int t0 = split_begin(a, tiles, split), t1 = split_begin(a, tiles, split + 1);

        auto ask = [&](int t, int to) {
            const int left = s.m - t * kKeys;
            const unsigned at = base + to * kStage;
            k_load.ask(k + (long)t * kKeys * a.k_token, at, left, lane);
            v_load.ask(v + (long)t * kKeys * a.v_token, at + kTile, left, lane);
        };
        if (t0 + wave < t1) ask(t0 + wave, 0);
        v8s q[STEPS];
        const T* const qr = (const T*)a.q + (s.q0 + token) * a.q_token + head * a.q_head;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 16 * i + 8 * half;
            q[i] = c < a.head_dim ? *(const v8s*)(qr + c) : v8s{0, 0, 0, 0, 0, 0, 0, 0};
        }
        // (the compiler does not know of the loads into LDS: it has to see q arrive in front of those that are counted)
#pragma unroll
        for (int i = 0; i < STEPS; ++i) asm volatile("" : "+v"(q[i]));
        v16f o[BLOCKS] = {};
        float m = -kInf, l = 0;
        int stage = 0;
        for (int t = t0 + wave; t < t1; t += WAVES) {
            const bool more = t + WAVES < t1;
            if (STAGES == 2 && more) {
                // (the reads of the stage that is overwritten are done: what they fed has been computed)
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                ask(t + WAVES, stage ^ 1);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            const int at = stage * kStage;
            v16f sc = {};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) sc = mfma<TYPE>(k_read.read(at, 0, i), q[i], sc);
            const int first = t * kKeys + 4 * half;
            float top = -kInf;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[i] = first + key_of(i) < visible ? sc[i] * a.scale_log2 : -kInf;
                top = fmaxf(top, sc[i]);
            }
            top = fmaxf(top, other_half(top));
            const float up = fmaxf(m, top);
            const float ref = up == -kInf ? 0.0f : up;                // (no key yet: every weight is exp2(-inf) = 0)
            const float old = __builtin_amdgcn_exp2f(m - ref);
            m = up;
            float sum = 0;
            unsigned p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(sc[2 * i] - ref), p1 = __builtin_amdgcn_exp2f(sc[2 * i + 1] - ref);
                sum += p0 + p1;
                p[i] = TYPE::pack(p0, p1);
            }
            l = l * old + sum;
#pragma unroll
            for (int c = 0; c < BLOCKS; ++c) o[c] *= old;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v4i pp = {(int)p[4 * i], (int)p[4 * i + 1], (int)p[4 * i + 2], (int)p[4 * i + 3]};
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c)
                    o[c] = mfma<TYPE>(v_read.read(at + kTile, 16 * i, c), __builtin_bit_cast(v8s, pp), o[c]);
            }
            if (STAGES == 2) {
                stage ^= 1;
            } else if (more) {
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                ask(t + WAVES, 0);
            }
        }
        l += other_half(l);
        if constexpr (WAVES == 1) {
            write_rows<TYPE, BLOCKS>(a, o, m, l, s.q0 + token, head, split, real, half);
            continue;
        }

        // Join the wavefronts: sums and weights relative to the largest maximum of a row.
        float* const sums = (float*)lds;                        // [WAVES][kRows][kPitch]
        float* const ml = sums + WAVES * kRows * kPitch;        // [WAVES][kRows][2]
        __syncthreads();
        if (half == 0) {
            ml[(wave * kRows + lane) * 2] = m;
            ml[(wave * kRows + lane) * 2 + 1] = l;
        }
        float* const mine = sums + (wave * kRows + (lane & 31)) * kPitch;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(v4f*)(mine + 32 * c + 8 * i + 4 * half) = v4f{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
        __syncthreads();
        const int pieces = a.head_dim / 8, count = min(kRows, rows - row0);
        for (int i = threadIdx.x; i < count * pieces; i += 64 * WAVES) {
            const int row = (int)((unsigned)i / (unsigned)pieces), c = 8 * (i - row * pieces);
            float top = -kInf, sum = 0, out[8] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[(w * kRows + row) * 2]);
            const float ref = top == -kInf ? 0.0f : top;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[(w * kRows + row) * 2] - ref);
                sum += ml[(w * kRows + row) * 2 + 1] * f;
                const float* from = sums + (w * kRows + row) * kPitch + c;
#pragma unroll
                for (int e = 0; e < 8; ++e) out[e] += from[e] * f;
            }
            const int tk = token_of(a, row0 + row), hd = kv * a.group + row0 + row - tk * a.group;
            write_eight_of_row<TYPE>(a, s.q0 + tk, hd, split, c, out, top, sum);
        }
        __syncthreads();      // the next tile's loads go where the sums were
    }
}

// Joins the parts of the rows whose keys were divided among workgroups: a wavefront a row, a lane first the weight of one of at most 64
// parts, then eight channels of every fourth part.  (A thread for eight channels and the parts one after another: 68 us instead of 32 for
// one token over 32768 keys with both kernels, inputs in the caches.)
template <class TYPE>
__global__ __launch_bounds__(256) void attention_join(AttentionArgs a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, parts = 1 << a.split_shift;
    const int first = min(max(a.cu_q[0], 0), a.Tq), last = min(max(a.cu_q[a.sequences], 0), a.Tq);
    const size_t next = (size_t)a.Tq * a.heads;
    const int piece = lane & 15, group = lane >> 4;
    for (unsigned row = (unsigned)first * a.heads + blockIdx.x * 4 + wave; row < (unsigned)last * a.heads; row += gridDim.x * 4) {
        const v2f ml = lane < parts ? *(const v2f*)(a.part_ml + (lane * next + row) * 2) : v2f{-kInf, 0.0f};
        float top = ml[0];
#pragma unroll
        for (int i = 1; i < 64; i *= 2) top = fmaxf(top, __shfl_xor(top, i));
        const float weight = __builtin_amdgcn_exp2f(ml[0] - (top == -kInf ? 0.0f : top));
        float l = ml[1] * weight;
#pragma unroll
        for (int i = 1; i < 64; i *= 2) l += __shfl_xor(l, i);
        float o[8] = {};
        const bool in = 8 * piece < a.head_dim;
        for (int s0 = 0; s0 < parts; s0 += 16) {
            v4f lo[4], hi[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int s = s0 + 4 * u + group;
                const v4f* from = (const v4f*)(a.part_o + ((s < parts ? s : 0) * next + row) * a.head_dim + (in ? 8 * piece : 0));
                lo[u] = from[0], hi[u] = from[1];
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int s = s0 + 4 * u + group;
                const float w = __shfl(weight, s & 63), f = s < parts ? w : 0.0f;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += s < parts ? lo[u][e] * f : 0.0f, o[4 + e] += s < parts ? hi[u][e] * f : 0.0f;
            }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            o[e] += __shfl_xor(o[e], 16);
            o[e] += __shfl_xor(o[e], 32);
        }
        const int token = (int)(row / (unsigned)a.heads);
        if (group == 0 && in) write_outputs<TYPE>(a, token, (int)(row - (unsigned)token * a.heads), 8 * piece, o, l);
    }
}

template <class TYPE, int WAVES, int STAGES>
hipError_t launch_rows(AttentionArgs a, hipStream_t stream) {
    const unsigned blocks = attention_grid(a, a.sequences);
    void (*kernel)(AttentionArgs) = a.head_dim <= 64   ? attention_rows<TYPE, 8, 4, WAVES, STAGES>
                                    : a.head_dim <= 80 ? attention_rows<TYPE, 12, 5, WAVES, STAGES>
                                    : a.head_dim <= 96 ? attention_rows<TYPE, 12, 6, WAVES, STAGES>
                                                       : attention_rows<TYPE, 16, 8, WAVES, STAGES>;
    return enqueue(kernel, dim3(blocks), dim3(64 * WAVES), stream, a);
}
}  // namespace

AttentionChoice choose_attention(int sequences, int Tq, int Tk, int heads, int kv_heads) {
    const int group = heads / kv_heads;
    const long keys = (long)Tk / sequences;
    // Rows of the average sequence: up to 32, one MFMA block of them.  With all in tiles 16 single tokens over long keys take 230 us instead
    // of 170 and 2048 sequences of 16 239 instead of 84 (64 equal ones over 4096 keys 191 and 215); with up to 64 by rows 16 sequences of 64
    // rows over 4096 keys 151 instead of 71 and 512 sequences of 64 91 instead of 75.
    const bool rows = (long)Tq * group <= 32l * sequences;
    // Parts of at least 256 keys of the average sequence, and workgroups for eight turns of the chip, or one of tiles.  Undivided and
    // divided (us, captured, inputs that are not in the caches): a token of one sequence over 32768 keys 437 and 39, of 16 ragged ones
    // 442 and 170, 512 queries over 32768 584 and 280, 64 tokens of 2 sequences over 8192 156 and 35.  Eight turns are for ragged sequences,
    // where the longest decides: workgroups for two make those 16 199, but 64 equal ones over 4096 keys 190 instead of 215.
    const long tiles = rows ? (long)sequences : attention_items(sequences, Tq, group), items = tiles * kv_heads;
    int shift = 0;
    while (shift < 6 && (items << shift) < (rows ? 2048 : 512) && keys >> (shift + 1) >= 256) ++shift;
    // A wavefront alone, one tile of keys at a time, where the average sequence has a few tiles and there are sequences enough: 2048
    // sequences of 16, 16 heads of 72, 84 us, by four wavefronts 542, most of which have no keys.
    const bool alone = rows && shift == 0 && keys <= 64 && (long)sequences * kv_heads >= 2048;
    // (HIP takes less than 2^32 threads; the items of a kernel are rounded up to whole groups of XCDs)
    const long most = ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads;
    return {!rows ? kAttentionTiles : alone ? kAttentionRowsAlone : kAttentionRows, shift, most * (alone ? 64 : 256) < 1l << 32};
}

hipError_t launch_attention(const AttentionArgs& a, AttentionKernel kernel, int dtype, hipStream_t stream) {
    const bool f16 = dtype == VQ_F16;
    if (kernel == kAttentionRowsAlone) return f16 ? launch_rows<F16, 1, 1>(a, stream) : launch_rows<BF16, 1, 1>(a, stream);
    const hipError_t e = kernel == kAttentionTiles ? launch_attention_tiles(a, dtype, stream)
                         : f16                     ? launch_rows<F16, 4, 2>(a, stream)
                                                   : launch_rows<BF16, 4, 2>(a, stream);
    if (e != hipSuccess || a.split_shift == 0) return e;
    const long join = ((long)a.Tq * a.heads + 3) / 4;
    return enqueue(f16 ? attention_join<F16> : attention_join<BF16>, dim3((unsigned)(join < 1 << 20 ? join : 1 << 20)), dim3(256), stream, a);
}

}  // namespace vq

extern "C" void vq_internal_attention_choice(int sequences, int Tq, int Tk, int heads, int kv_heads, int choice[2]) {
    const vq::AttentionChoice c = vq::choose_attention(sequences, Tq, Tk, heads, kv_heads);
    choice[0] = c.kernel;
    choice[1] = c.split_shift;
}
