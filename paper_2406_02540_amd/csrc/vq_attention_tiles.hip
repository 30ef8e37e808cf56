// Attention whose wavefronts share the keys: 128 query rows a workgroup, 32 a wavefront, tiles of 64 keys.
//
// Bound by the sum of matrix and vector time: a wavefront's exponentials and its products do not overlap much, and the clock falls under
// both (2 x 4096, 16 heads of 72: matrix units busy 48 % of the cycles at 1.8 GHz; causal prompts of up to 8192, heads of 128: 53 % at 1.7 GHz; no
// LDS conflicts to speak of).  Measured (captured, inputs that are not in the caches): 4 x 4096, 16 heads of 128 524 us (1048 TFLOP/s), heads of
// 64 322 (853); 2 x 4096, 16 heads of 72 207 (747; its heads' last block of 32 channels is a fourth full); 256 rows a workgroup are slower.
// With few keys bound by the way of the first loads: 2 x 16384 queries on 120 keys 57 us, 2.6 TB/s of 151 MB (50 us on a chip that has been busy
// for a second: the clock dips when work begins).
#include <type_traits>

#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kWaves = 4;
constexpr int kKeys = 64;
constexpr float kInf = __builtin_inff();
constexpr float kSlack = 8.0f;    // base 2: how far a score may exceed the reference before sums and outputs are rescaled

// Tiles of all sequences are numbered so that a sequence's first is floor(cu * group / rows) + b, at least the tiles of the
// sequences in front of it (floor(x + y) - floor(x) + 1 >= ceil(y)): a sequence is found by bisection, and a number that no tile has
// is a workgroup that ends at once.
__device__ __forceinline__ int find_sequence(const AttentionArgs& a, int item, int& tile) {
    int lo = 0, hi = a.sequences - 1;
    auto first = [&](int b) { return (int)((unsigned)(min(max(a.cu_q[b], 0), a.Tq) * a.group) / kTileRows) + b; };
    while (lo < hi) {
        const int mid = lo + (hi - lo + 1) / 2;
        if (first(mid) <= item) lo = mid;
        else hi = mid - 1;
    }
    tile = item - first(lo);
    return lo;
}

template <class TYPE, int CHUNKS, int STEPS>
__global__ __launch_bounds__(64 * kWaves, CHUNKS == 16 ? 2 : 3) void attention_tiles(AttentionArgs a) {
    constexpr int BLOCKS = CHUNKS / 4;
    constexpr int kTile = kKeys * CHUNKS * 16;
    constexpr bool kSumColumn = STEPS == 5;             // heads of 72 and 80 channels leave a part of their last block free
    __shared__ __align__(16) char lds[4 * kTile];       // two tiles of K, two of V
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    int kv, item;
    if (!place_of(a, kv, item)) return;
    const int split = item & ((1 << a.split_shift) - 1);
    int tile;
    // (the last tiles of a sequence see the most keys: they go first)
    const int b = find_sequence(a, a.tiles - 1 - (item >> a.split_shift), tile);
    const Span s = span_of(a, b);
    const int rows = s.n * a.group;
    if (tile < 0 || (unsigned)tile * kTileRows >= (unsigned)rows) return;
    const int row0 = tile * kTileRows;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds + 1024 * wave;

    const int r = min(row0 + 32 * wave + (lane & 31), rows - 1);
    const int token = token_of(a, r), head = kv * a.group + r - token * a.group;
    // keys: this lane's row's, the wavefront's fewest, the workgroup's most
    const int visible = keys_seen(a, s, token);
    const int least = __builtin_amdgcn_readfirstlane(keys_seen(a, s, token_of(a, min(row0 + 32 * wave, rows - 1))));
    const int end = __builtin_amdgcn_readfirstlane(keys_seen(a, s, token_of(a, min(row0 + kTileRows, rows) - 1)));
    const int tiles = (end + kKeys - 1) / kKeys;
    const int t0 = split_begin(a, tiles, split), t1 = split_begin(a, tiles, split + 1);

    const TileLoader<CHUNKS, kKeys, 64 * kWaves, false> k_load((int)(2 * a.k_token), head_bytes, threadIdx.x);
    const TileLoader<CHUNKS, kKeys, 64 * kWaves, true> v_load((int)(2 * a.v_token), head_bytes, threadIdx.x);
    // tile t into the buffer `to`, 0 or 1
    auto ask_k = [&](int t, int to) { k_load.ask(k + (long)t * kKeys * a.k_token, base + to * kTile, s.m - t * kKeys, threadIdx.x); };
    auto ask_v = [&](int t, int to) {
        v_load.template ask<kSumColumn>(v + (long)t * kKeys * a.v_token, base + (2 + to) * kTile, s.m - t * kKeys, threadIdx.x);
    };
    // The sum of a row's weights as one more channel: V's first column behind the head is ones, which stay in LDS (and whatever the keys
    // behind a sequence's end have there, their weights are zero).
    if (kSumColumn) {
        const int first = a.head_dim / 8;
        for (int i = threadIdx.x; i < 2 * kKeys * (CHUNKS - first); i += 64 * kWaves) {
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
    v16f sc[2];
    const KeyReader<CHUNKS, STEPS> k_read((lds_bytes)lds, lane);
    const ValueReader<CHUNKS> v_read((lds_bytes)lds + 2 * kTile, lane);
    auto hide = [&](int t, int j) {
        const int first = t * kKeys + 32 * j + 4 * half;
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[j][i] = first + key_of(i) < visible ? sc[j][i] : -kInf;
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
        if (t * kKeys + kKeys > least) {
            hide(t, 0);
            hide(t, 1);
            top = -kInf;
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[0][i]);
        }
        top = fmaxf(top, relative(1));
        top = fmaxf(top, other_half(top));
        if (__any(top > kSlack)) {
            const float up = fmaxf(top, 0.0f), f = __builtin_amdgcn_exp2f(-up);
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
            hide(t0, j);
        }
        // the reference is the first tile's largest score (a row that sees any key sees the first of its first tile)
        top = -kInf;
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, sc[j][i]);
        top = fmaxf(top, other_half(top));
        ref = top == -kInf ? 0.0f : top * a.scale_log2;
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

template <class TYPE>
hipError_t launch(AttentionArgs a, hipStream_t stream) {
    const unsigned blocks = attention_grid(a, attention_items(a.sequences, a.Tq, a.group));
    void (*kernel)(AttentionArgs) = a.head_dim <= 64   ? attention_tiles<TYPE, 8, 4>
                                    : a.head_dim <= 80 ? attention_tiles<TYPE, 12, 5>
                                    : a.head_dim <= 96 ? attention_tiles<TYPE, 12, 6>
                                                       : attention_tiles<TYPE, 16, 8>;
    return enqueue(kernel, dim3(blocks), dim3(64 * kWaves), stream, a);
}

}  // namespace

hipError_t launch_attention_tiles(const AttentionArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace vq
