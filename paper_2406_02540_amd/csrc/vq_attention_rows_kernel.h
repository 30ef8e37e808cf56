// The kernels whose wavefronts divide the keys, and the one that joins parts of rows.  ARGS says which keys there are, as in
// vq_attention_tiles_kernel.h.
#pragma once
#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kRows = 32;       // query rows of a tile: the columns of an MFMA block
constexpr int kOwnRows = 64;    // of a workgroup of a part of the sequences' own keys, one tile behind the other
constexpr int kRowKeys = 32;       // keys of a wavefront's tile

// Eight channels of a row: normalised to the output.
template <class TYPE, class ARGS>
__device__ __forceinline__ void write_outputs(const ARGS& a, int token, int head, int c, const float* o, float l) {
    const float inv = l > 0 ? 1.0f / l : 0.0f;
    v4i y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (int)TYPE::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
    *(v4i*)((typename TYPE::T*)a.out + token * a.o_token + head * a.o_head + c) = y;
}
// Or as they are, where other workgroups have more of the row's keys.
template <class TYPE, class ARGS>
__device__ __forceinline__ void write_eight_of_row(const ARGS& a, int token, int head, int split, int c, const float* o, float m, float l) {
    if (!writes_parts(a)) return write_outputs<TYPE>(a, token, head, c, o, l);
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
template <int CHUNKS, int WAVES, int STAGES>
constexpr int kRowsBytes = [] {       // of LDS: the stages, or where the wavefronts' sums meet
    constexpr int stages = WAVES * STAGES * 2 * kRowKeys * CHUNKS * 16, sums = WAVES == 1 ? 0 : WAVES * kRows * (8 * CHUNKS + 4 + 2) * 4;
    return stages > sums ? stages : sums;
}();

// A workgroup's sequence and rows: all of them, or a block (its number less than 2^24; the last ones see the most keys and go first).  Blocks that no
// sequence has cost their workgroups' start: 200 x 16 tokens behind 2000 keys, 16 heads on 8 of 128, 106 us by sequences, 108 in blocks of 64
// rows, 121 of 32; 20 x 25 behind 6000, 32 heads, 91, 85 and 79.
struct RowsTaken {
    int sequence, first, count;
};
__device__ __forceinline__ RowsTaken rows_taken(const AttentionArgs&, int item) { return {item, 0, 0x7FFFFFFF}; }
__device__ __forceinline__ RowsTaken rows_taken(const AttentionOwnArgs& a, int item) {
    if (!a.by_blocks) return {item, 0, 0x7FFFFFFF};
    int block;
    const int b = find_sequence<kOwnRows>(a, a.tiles - 1 - item, block);
    return {b, max(block, 0) * kOwnRows, block < 0 ? 0 : kOwnRows};
}

// Workgroup `block` of a launch's.
template <class TYPE, int CHUNKS, int STEPS, int WAVES, int STAGES, class ARGS>
__device__ __forceinline__ void rows_of(const ARGS& a, unsigned block, char* lds) {
    constexpr int BLOCKS = CHUNKS / 4;                 // of 32 channels
    constexpr int kTile = kRowKeys * CHUNKS * 16;         // bytes
    constexpr int kStage = 2 * kTile;                  // K, V
    constexpr int kPitch = 32 * BLOCKS + 4;            // floats of a row where the wavefronts' sums meet
    constexpr int kLoads = 2 * kRowKeys * CHUNKS / 64;    // of a stage, per lane
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5;
    int kv, item;
    if (!place_of(a, block, kv, item)) return;
    const int split = item & ((1 << a.split_shift) - 1);
    const RowsTaken taken = rows_taken(a, item >> a.split_shift);
    const Span s = span_of(a, taken.sequence);
    const int rows = s.n * a.group, end = taken.count < rows - taken.first ? taken.first + taken.count : rows;
    const int head_bytes = 2 * a.head_dim;
    lds_bytes const mine_in_lds = (lds_bytes)lds + wave * STAGES * kStage;
    const unsigned base = (unsigned)(uintptr_t)mine_in_lds;
    typedef TileLoader<CHUNKS, kRowKeys, 64, false> LoaderK;
    typedef TileLoader<CHUNKS, kRowKeys, 64, true> LoaderV;
    LoaderK k_load((int)(2 * a.k_token), head_bytes, lane);
    LoaderV v_load((int)(2 * a.v_token), head_bytes, lane);
    const KeyReader<CHUNKS, STEPS> k_read(mine_in_lds, lane);
    const ValueReader<CHUNKS> v_read(mine_in_lds, lane);

    for (int row0 = taken.first; row0 < end; row0 += kRows) {
        const int r = min(row0 + (lane & 31), rows - 1);
        const bool real = row0 + (lane & 31) < rows;
        const int token = token_of(a, r), head = kv * a.group + r - token * a.group;
        // keys: the tile's, this lane's row's
        typedef Keys<ARGS, T, kRowKeys> KeysOf;
        const KeysOf keys(a, s, kv, token_of(a, row0), token_of(a, min(row0 + kRows, rows) - 1));
        const typename KeysOf::Row sight(a, s, token);
        const int t0 = split_begin(a, keys.tiles, split), t1 = split_begin(a, keys.tiles, split + 1);

        bool own = true;            // whether the loaders are those of the sequence's own keys
        if constexpr (KeysOf::kTwoTensors) {
            own = t0 + wave >= keys.first_tiles;      // (another block of rows may have left the others)
            k_load = LoaderK((int)(2 * (own ? a.k_token : a.pk_token)), head_bytes, lane);
            v_load = LoaderV((int)(2 * (own ? a.v_token : a.pv_token)), head_bytes, lane);
        }
        auto ask = [&](int t, int to) {
            if constexpr (KeysOf::kTwoTensors)
                if (!own && t >= keys.first_tiles) {
                    own = true;
                    k_load = LoaderK((int)(2 * a.k_token), head_bytes, lane);
                    v_load = LoaderV((int)(2 * a.v_token), head_bytes, lane);
                }
            const int left = keys.left(t);
            const unsigned at = base + to * kStage;
            k_load.ask(keys.k_of(a, t), at, left, lane);
            v_load.ask(keys.v_of(a, t), at + kTile, left, lane);
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
            float top = -kInf;
            if constexpr (KeysOf::kStretches) {
                const unsigned seen = (unsigned)(keys.seen(sight, t) >> (4 * half));
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[i] = seen_or_hidden(sc[i] * a.scale_log2, seen, key_of(i));
                    top = fmaxf(top, sc[i]);
                }
            } else {
                const int first = keys.key_of_tile(t) + 4 * half;
                const typename KeysOf::Row here = keys.within(sight, t);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[i] = keys.sees(here, first + key_of(i)) ? sc[i] * a.scale_log2 : -kInf;
                    top = fmaxf(top, sc[i]);
                }
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

template <class TYPE, int CHUNKS, int STEPS, int WAVES, int STAGES, class ARGS>
__global__ __launch_bounds__(64 * WAVES) void attention_rows(ARGS a) {
    __shared__ __align__(16) char lds[kRowsBytes<CHUNKS, WAVES, STAGES>];
    rows_of<TYPE, CHUNKS, STEPS, WAVES, STAGES>(a, blockIdx.x, lds);
}

// Joins the parts of the rows whose keys were divided among workgroups: a wavefront a row, a lane first the weight of one of at most 64
// parts, then eight channels of every fourth part.  (A thread for eight channels and the parts one after another: 68 us instead of 32 for
// one token over 32768 keys with both kernels, inputs in the caches.)
__device__ __forceinline__ int parts_of(const AttentionArgs& a) { return 1 << a.split_shift; }
__device__ __forceinline__ int parts_of(const AttentionPrefixArgs& a) { return a.parts; }
template <class TYPE, class ARGS>
__global__ __launch_bounds__(256) void attention_join(ARGS a) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, parts = parts_of(a);
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

template <class TYPE, int WAVES, int STAGES, class ARGS>
hipError_t launch_rows(ARGS a, hipStream_t stream) {
    const unsigned blocks = attention_grid(a, a.sequences);
    void (*kernel)(ARGS) = a.head_dim <= 64   ? attention_rows<TYPE, 8, 4, WAVES, STAGES, ARGS>
                                    : a.head_dim <= 80 ? attention_rows<TYPE, 12, 5, WAVES, STAGES, ARGS>
                                    : a.head_dim <= 96 ? attention_rows<TYPE, 12, 6, WAVES, STAGES, ARGS>
                                                       : attention_rows<TYPE, 16, 8, WAVES, STAGES, ARGS>;
    return enqueue(kernel, dim3(blocks), dim3(64 * WAVES), stream, a);
}
template <class ARGS>
hipError_t launch_join(const ARGS& a, int dtype, hipStream_t stream) {
    const long join = ((long)a.Tq * a.heads + 3) / 4;
    return enqueue(dtype == VQ_F16 ? attention_join<F16, ARGS> : attention_join<BF16, ARGS>, dim3((unsigned)(join < 1 << 20 ? join : 1 << 20)), dim3(256),
                   stream, a);
}

}  // namespace
}  // namespace vq
