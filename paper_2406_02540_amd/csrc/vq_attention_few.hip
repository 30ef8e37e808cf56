// Attention of many queries to few keys (captions): a workgroup keeps 128 keys of a sequence in LDS and goes through up to 1024 query
// rows, each of its wavefronts through tiles of 32 by itself.
//
// The tiles of vq_attention_tiles.hip load the keys again for every 128 rows, and most of a workgroup's time is the way of its first
// loads: 2 x 16384 queries on 120 keys, 16 heads of 72, 42 us so, 35 as it is; heads of 128 on 128 keys 43
// and 37.  Here a tile's queries are asked for when the one before has its scores.  Sequences of more keys go through them 128 at a time, for every 128 rows anew.
#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 128, kKeyBlocks = kKeys / 32;
constexpr float kInf = __builtin_inff();

template <class TYPE, int CHUNKS, int STEPS>
__global__ __launch_bounds__(64 * kWaves, STEPS == 5 ? 3 : 2) void attention_few_keys(AttentionArgs a) {
    constexpr int BLOCKS = CHUNKS / 4;
    constexpr int kTile = kKeys * CHUNKS * 16;
    constexpr bool kSumColumn = STEPS == 5;
    __shared__ __align__(16) char lds[2 * kTile];       // K, V
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    int kv, item, tile;
    if (!place_of(a, kv, item)) return;
    const int b = find_sequence(a, item, a.tile_shift, tile);
    const Span s = span_of(a, b);
    const int rows = s.n * a.group;
    if (tile < 0 || (unsigned)tile << a.tile_shift >= (unsigned)rows) return;
    const int row0 = tile << a.tile_shift, row1 = rows - row0 > 1 << a.tile_shift ? row0 + (1 << a.tile_shift) : rows;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds + 1024 * wave;
    auto ask = [&](int key0) {         // (rarely more than once: places of loads are not kept)
        const int thread = opaque(threadIdx.x);
        const TileLoader<CHUNKS, kKeys, 64 * kWaves, false> k_load((int)(2 * a.k_token), head_bytes, thread);
        const TileLoader<CHUNKS, kKeys, 64 * kWaves, true> v_load((int)(2 * a.v_token), head_bytes, thread);
        k_load.ask(k + (long)key0 * a.k_token, base, s.m - key0, thread);
        v_load.template ask<kSumColumn>(v + (long)key0 * a.v_token, base + kTile, s.m - key0, thread);
    };
    if (s.m > 0) ask(0);
    if (kSumColumn) write_sum_column<TYPE, CHUNKS>((lds_bytes)lds + kTile, kKeys, a.head_dim / 8, threadIdx.x, 64 * kWaves);

    const KeyReader<CHUNKS, STEPS> k_read((lds_bytes)lds, lane);
    const ValueReader<CHUNKS> v_read((lds_bytes)lds + kTile, lane);
    v8s q[STEPS];
    auto ask_q = [&](int first) {      // the 32 rows from `first` on; the last one for those that do not exist
        const int at = opaque(lane), r = min(first + (at & 31), rows - 1), token = token_of(a, r);
        const T* const from = (const T*)a.q + (s.q0 + token) * a.q_token + (kv * a.group + r - token * a.group) * a.q_head;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 16 * i + 8 * (at >> 5);
            q[i] = c < a.head_dim ? *(const v8s*)(from + c) : v8s{0, 0, 0, 0, 0, 0, 0, 0};
        }
    };
    ask_q(row0 + 32 * wave);
    wait_loads_and_barrier();
    for (int first = row0; first < row1; first += 32 * kWaves) {       // (the same turns for all wavefronts: they meet where keys are loaded)
        v16f o[BLOCKS] = {};
        float m = -kInf, l = 0;
        for (int key0 = 0; key0 < s.m; key0 += kKeys) {
            if (s.m > kKeys && (key0 > 0 || first > row0)) {
                wait_lds_and_barrier();
                ask(key0);
                wait_loads_and_barrier();
            }
            const int left = s.m - key0;
            v16f sc[kKeyBlocks];
#pragma unroll
            for (int j = 0; j < kKeyBlocks; ++j) {
                sc[j] = v16f{};
                if (32 * j < left)
#pragma unroll
                    for (int i = 0; i < STEPS; ++i) sc[j] = mfma<TYPE>(k_read.read(0, 32 * j, i), q[i], sc[j]);
            }
            const bool next = left <= kKeys && first + 32 * kWaves < row1;
            if (next) ask_q(first + 32 * kWaves + 32 * wave);
            float top = -kInf;
#pragma unroll
            for (int j = 0; j < kKeyBlocks; ++j) {
                if (32 * j + 32 > left)
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[j][i] = 32 * j + 4 * half + key_of(i) < left ? sc[j][i] : -kInf;
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[j][i]);
            }
            top = fmaxf(top, other_half(top)) * a.scale_log2;      // (there is a key: it is a number, or what the inputs made of it)
            const float up = fmaxf(m, top), old = __builtin_amdgcn_exp2f(m - up);
            m = up;
            if (key0 > 0) {
                l *= old;
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c) o[c] *= old;
            }
#pragma unroll
            for (int j = 0; j < kKeyBlocks; ++j) {
                if (32 * j >= left) break;
                v4i p[2];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float p0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][2 * i], a.scale_log2, -m));
                    const float p1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[j][2 * i + 1], a.scale_log2, -m));
                    if (!kSumColumn) l += p0 + p1;
                    p[i >> 2][i & 3] = (int)TYPE::pack(p0, p1);
                }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int c = 0; c < BLOCKS; ++c)
                        o[c] = mfma<TYPE>(v_read.read(0, 32 * j + 16 * i, c), __builtin_bit_cast(v8s, p[i]), o[c]);
            }
        }
        l = kSumColumn ? sum_of_column<BLOCKS>(o, a.head_dim, half) : l + other_half(l);
        const int at = opaque(lane), r = first + 32 * wave + (at & 31), row = min(r, rows - 1), token = token_of(a, row);
        write_rows<TYPE, BLOCKS>(a, o, m, l, s.q0 + token, kv * a.group + row - token * a.group, 0, r < row1, at >> 5);
    }
}

template <class TYPE>
hipError_t launch(AttentionArgs a, hipStream_t stream) {
    // rows of a workgroup: as many as leave two workgroups a CU
    a.tile_shift = 7;
    while (a.tile_shift < 10 && (attention_items(a.sequences, a.Tq, a.group, a.tile_shift + 1) * a.kv_heads) >= 512) ++a.tile_shift;
    const unsigned blocks = attention_grid(a, attention_items(a.sequences, a.Tq, a.group, a.tile_shift), 64 * kWaves);
    if (!blocks) return hipErrorInvalidValue;
    void (*kernel)(AttentionArgs) = a.head_dim <= 64   ? attention_few_keys<TYPE, 8, 4>
                                    : a.head_dim <= 80 ? attention_few_keys<TYPE, 12, 5>
                                    : a.head_dim <= 96 ? attention_few_keys<TYPE, 12, 6>
                                                       : attention_few_keys<TYPE, 16, 8>;
    return enqueue(kernel, dim3(blocks), dim3(64 * kWaves), stream, a);
}

}  // namespace

hipError_t launch_attention_few_keys(const AttentionArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace vq
