// The kernel whose wavefronts share the keys: 128 query rows a workgroup, 32 a wavefront, tiles of 64 keys.  ARGS says which keys there are:
// all of a sequence (AttentionArgs), those of a window (AttentionWindowArgs), or a prefix and then a sequence's own (AttentionPrefixArgs).
#pragma once
#include <type_traits>

#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kTileWaves = 4;
constexpr int kTileKeys = 64;
constexpr float kSlack = 8.0f;    // base 2: how far a score may exceed the reference before sums and outputs are rescaled

template <int CHUNKS>
constexpr int kTilesBytes = 4 * kTileKeys * CHUNKS * 16;      // of LDS: two tiles of K, two of V

// Workgroup `block` of a launch's.
template <class TYPE, int CHUNKS, int STEPS, class ARGS>
__device__ __forceinline__ void tiles_of(const ARGS& a, unsigned block, char* lds) {
    constexpr int BLOCKS = CHUNKS / 4;
    constexpr int kTile = kTileKeys * CHUNKS * 16;
    constexpr bool kSumColumn = STEPS == 5;             // heads of 72 and 80 channels leave a part of their last block free
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    int kv, item;
    if (!place_of(a, block, kv, item)) return;
    const int split = item & ((1 << a.split_shift) - 1);
    int tile;
    // (the last tiles of a sequence see the most keys: they go first)
    const int b = find_sequence<kTileRows>(a, a.tiles - 1 - (item >> a.split_shift), tile);
    const Span s = span_of(a, b);
    const int rows = s.n * a.group;
    if (tile < 0 || (unsigned)tile * kTileRows >= (unsigned)rows) return;
    const int row0 = tile * kTileRows;
    const int head_bytes = 2 * a.head_dim;
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds + 1024 * wave;

    const int r = min(row0 + 32 * wave + (lane & 31), rows - 1);
    const int token = token_of(a, r), head = kv * a.group + r - token * a.group;
    // keys: the workgroup's, this lane's row's, those that all of the wavefront's rows see
    typedef Keys<ARGS, T, kTileKeys> KeysOf;
    const KeysOf keys(a, s, kv, token_of(a, row0), token_of(a, min(row0 + kTileRows, rows) - 1));
    const typename KeysOf::Row sight(a, s, token);
    const typename KeysOf::Rows seen_by_all(a, s, token_of(a, min(row0 + 32 * wave, rows - 1)), token_of(a, min(row0 + 32 * wave + 32, rows) - 1));
    const int t0 = split_begin(a, keys.tiles, split), t1 = split_begin(a, keys.tiles, split + 1);

    typedef TileLoader<CHUNKS, kTileKeys, 64 * kTileWaves, false> LoaderK;
    typedef TileLoader<CHUNKS, kTileKeys, 64 * kTileWaves, true> LoaderV;
    LoaderK k_load((int)(2 * a.k_token), head_bytes, threadIdx.x);
    LoaderV v_load((int)(2 * a.v_token), head_bytes, threadIdx.x);
    if constexpr (KeysOf::kTwoTensors)
        if (t0 < keys.first_tiles) {
            k_load = LoaderK((int)(2 * a.pk_token), head_bytes, threadIdx.x);
            v_load = LoaderV((int)(2 * a.pv_token), head_bytes, threadIdx.x);
        }
    // tile t into the buffer `to`, 0 or 1; tiles are asked for in turn
    auto ask_k = [&](int t, int to) {
        if constexpr (KeysOf::kTwoTensors)
            if (t == keys.first_tiles) k_load = LoaderK((int)(2 * a.k_token), head_bytes, threadIdx.x);
        k_load.ask(keys.k_of(a, t), base + to * kTile, keys.left(t), threadIdx.x);
    };
    auto ask_v = [&](int t, int to) {
        if constexpr (KeysOf::kTwoTensors)
            if (t == keys.first_tiles) v_load = LoaderV((int)(2 * a.v_token), head_bytes, threadIdx.x);
        v_load.template ask<kSumColumn>(keys.v_of(a, t), base + (2 + to) * kTile, keys.left(t), threadIdx.x);
    };
    // The sum of a row's weights as one more channel: V's first column behind the head is ones, which stay in LDS (and whatever the keys
    // behind a sequence's end have there, their weights are zero).
    if (kSumColumn) {
        const int first = a.head_dim / 8;
        for (int i = threadIdx.x; i < 2 * kTileKeys * (CHUNKS - first); i += 64 * kTileWaves) {
            const int key = i / (CHUNKS - first), c = first + i % (CHUNKS - first);
            const int one = c == first ? (int)(TYPE::pack(1.0f, 0.0f)) : 0;
            *(__attribute__((address_space(3))) v4i*)((lds_bytes)lds + 2 * kTile + (key * CHUNKS + c) * 16) = v4i{one, 0, 0, 0};
        }
    }
    if (t0 < t1) {
        ask_k(t0, 0);
        ask_v(t0, 0);
        if (t0 + 1 < t1) ask_k(t0 + 1, 1);
    }
    v8s q[STEPS];
    const T* const qr = (const T*)a.q + (s.q0 + token) * a.q_token + head * a.q_head;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = 16 * i + 8 * half;
        q[i] = c < a.head_dim ? *(const v8s*)(qr + c) : v8s{0, 0, 0, 0, 0, 0, 0, 0};
    }
    v16f o[BLOCKS] = {};
    float ref = 0, l = 0;         // exponents are relative to ref
    bool late = false;            // no key seen yet, and ref stands for nothing
    v16f sc[2];
    const KeyReader<CHUNKS, STEPS> k_read((lds_bytes)lds, lane);
    const ValueReader<CHUNKS> v_read((lds_bytes)lds + 2 * kTile, lane);
    auto hide = [&](int t) {
        if constexpr (KeysOf::kStretches) {
            const uint64_t seen = keys.seen(sight, t) >> (4 * half);
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[j][i] = seen_or_hidden(sc[j][i], (unsigned)(seen >> (32 * j)), key_of(i));
        } else {
            const typename KeysOf::Row here = keys.within(sight, t);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int first = keys.key_of_tile(t) + 32 * j + 4 * half;
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[j][i] = keys.sees(here, first + key_of(i)) ? sc[j][i] : -kInf;
            }
        }
    };
    auto relative = [&](int j) {
        float top = -kInf;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            sc[j][i] = __builtin_fmaf(sc[j][i], a.scale_log2, -ref);
            top = fmaxf(top, sc[j][i]);
        }
        return top;
    };
    auto weight_pair = [&](int j, int i, v4i* p) {
        const float p0 = __builtin_amdgcn_exp2f(sc[j][2 * i]), p1 = __builtin_amdgcn_exp2f(sc[j][2 * i + 1]);
        if (!kSumColumn) l += p0 + p1;
        p[i >> 2][i & 3] = (int)TYPE::pack(p0, p1);
    };
    // Products in pairs: the outputs of block j of tile t, and the scores of block j of tile t + 1 (MORE), with `between` in the gaps.  Operands
    // are read kAhead pairs ahead.
    auto products = [&](int buffer, int j, const v4i* p, auto more, auto between) {
        constexpr bool MORE = decltype(more)::value;
        const int k_at = (buffer ^ 1) * kTile, v_at = buffer * kTile;
        constexpr int kPairs = MORE && STEPS > 2 * BLOCKS ? STEPS : 2 * BLOCKS, kAhead = STEPS == 6 ? 1 : 2;
        v8s kf[kAhead + 1], vf[kAhead + 1];
        auto fetch = [&](int n) {
            if (MORE && n < STEPS) kf[n % (kAhead + 1)] = k_read.read(k_at, 32 * j, n);
            if (n < 2 * BLOCKS) vf[n % (kAhead + 1)] = v_read.read(v_at, 32 * j + 16 * (n / BLOCKS), n % BLOCKS);
        };
        v16f next = {};
#pragma unroll
        for (int n = 0; n < kAhead; ++n) fetch(n);
#pragma unroll
        for (int n = 0; n < kPairs; ++n) {
            if (n + kAhead < kPairs) fetch(n + kAhead);
            if (n < 2 * BLOCKS) o[n % BLOCKS] = mfma<TYPE>(vf[n % (kAhead + 1)], __builtin_bit_cast(v8s, p[n / BLOCKS]), o[n % BLOCKS]);
            between(n, kPairs);
            if (MORE && n < STEPS) next = mfma<TYPE>(kf[n % (kAhead + 1)], q[n], next);
            __builtin_amdgcn_sched_barrier(0);      // (the scheduler would put an operand's read right in front of its product)
        }
        if (MORE) sc[j] = next;
    };
    // Tile t, whose scores are in sc, block 0 of them relative to ref with `top` the largest: weights, sums, outputs, and under them the
    // scores of the next tile, block by block as they are used up.
    float top;
    auto step = [&](int t, auto more) {
        const int buffer = (t - t0) & 1;
        constexpr bool MORE = decltype(more)::value;
        if (!keys.whole(seen_by_all, t)) {
            hide(t);
            top = -kInf;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[0][i]);
        }
        top = fmaxf(top, relative(1));
        top = fmaxf(top, other_half(top));
        if (__any(top > kSlack || (!KeysOf::kFirstSeen && late && top > -kInf))) {
            float up = fmaxf(top, 0.0f);
            if (!KeysOf::kFirstSeen && late && top > -kInf) up = top;
            const float f = !KeysOf::kFirstSeen && late ? 1.0f : __builtin_amdgcn_exp2f(-up);       // (nothing to rescale: sums and outputs are zero)
            if (!KeysOf::kFirstSeen) late = late && top == -kInf;
            ref += up;
            l *= f;
#pragma unroll
            for (int c = 0; c < BLOCKS; ++c) o[c] *= f;
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] -= up;
        }
        v4i p[2][2];
#pragma unroll
        for (int i = 0; i < 8; ++i) weight_pair(0, i, p[0]);
        wait_loads_and_barrier();
        if constexpr (MORE) {
            if (t + 2 < t1) ask_k(t + 2, buffer);
            ask_v(t + 1, buffer ^ 1);
        }
        products(buffer, 0, p[0], more, [&](int n, int pairs) {
#pragma unroll
            for (int i = n * 8 / pairs; i < (n + 1) * 8 / pairs; ++i) weight_pair(1, i, p[1]);
        });
        if constexpr (MORE) top = -kInf;
        products(buffer, 1, p[1], more, [&](int n, int pairs) {
            if constexpr (MORE)
#pragma unroll
                for (int i = n * 16 / pairs; i < (n + 1) * 16 / pairs; ++i) {
                    sc[0][i] = __builtin_fmaf(sc[0][i], a.scale_log2, -ref);
                    top = fmaxf(top, sc[0][i]);
                }
        });
    };
    if (t0 < t1) {
        wait_loads_and_barrier();
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            sc[j] = v16f{};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) sc[j] = mfma<TYPE>(k_read.read(0, 32 * j, i), q[i], sc[j]);
        }
        hide(t0);
        // the reference is the first tile's largest score (a row that sees any key sees the first of its first tile)
        top = -kInf;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[j][i]);
        top = fmaxf(top, other_half(top));
        ref = top == -kInf ? 0.0f : top * a.scale_log2;
        if (!KeysOf::kFirstSeen) late = top == -kInf;
        top = relative(0);
        int t = t0;
        for (; t + 1 < t1; ++t) step(t, std::true_type{});
        step(t, std::false_type{});
    }
    if (kSumColumn) {       // (channel head_dim, 8 or 16 of the last block, in the lower half)
        const float sum = a.head_dim == 72 ? o[BLOCKS - 1][4] : o[BLOCKS - 1][8], other = other_half(sum);
        l = half ? other : sum;
    } else {
        l += other_half(l);
    }
    // (the row's token and head once more: kept through the loop they would be registers that it does not have)
    const int last_lane = opaque(lane), row = min(row0 + 32 * wave + (last_lane & 31), rows - 1), its_token = token_of(a, row);
    write_rows<TYPE, BLOCKS>(a, o, ref, l, s.q0 + its_token, kv * a.group + row - its_token * a.group, split,
                             row0 + 32 * wave + (last_lane & 31) < rows, last_lane >> 5);
}

template <class TYPE, int CHUNKS, int STEPS, class ARGS>
__global__ __launch_bounds__(64 * kTileWaves, CHUNKS == 16 ? 2 : 3) void attention_tiles(ARGS a) {
    __shared__ __align__(16) char lds[kTilesBytes<CHUNKS>];
    tiles_of<TYPE, CHUNKS, STEPS>(a, blockIdx.x, lds);
}

template <class TYPE, class ARGS>
hipError_t launch_tiles(ARGS a, hipStream_t stream) {
    const unsigned blocks = attention_grid(a, attention_items(a.sequences, a.Tq, a.group));
    void (*kernel)(ARGS) = a.head_dim <= 64   ? attention_tiles<TYPE, 8, 4, ARGS>
                                    : a.head_dim <= 80 ? attention_tiles<TYPE, 12, 5, ARGS>
                                    : a.head_dim <= 96 ? attention_tiles<TYPE, 12, 6, ARGS>
                                                       : attention_tiles<TYPE, 16, 8, ARGS>;
    return enqueue(kernel, dim3(blocks), dim3(64 * kTileWaves), stream, a);
}

}  // namespace
}  // namespace vq
