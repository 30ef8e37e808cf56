// Attention whose wavefronts share the keys: 128 query rows a workgroup, 32 a wavefront, tiles of 64 keys.
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
__global__ __launch_bounds__(64 * kWaves, 2) void attention_tiles(AttentionArgs a) {
    constexpr int BLOCKS = CHUNKS / 4;
    constexpr int kTile = kKeys * CHUNKS * 16, kStage = 2 * kTile;
    __shared__ __align__(16) char lds[2 * kStage];
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5;
    const int kv = (int)(blockIdx.x % (unsigned)a.kv_heads);
    const unsigned rest = blockIdx.x / (unsigned)a.kv_heads;
    const int split = (int)rest & ((1 << a.split_shift) - 1);
    int tile;
    // (the last tiles of a sequence see the most keys: they go first)
    const int b = find_sequence(a, a.items - 1 - (int)(rest >> a.split_shift), tile);
    const Span s = span_of(a, b);
    const int rows = s.n * a.group, row0 = tile * kTileRows;
    if (tile < 0 || row0 >= rows) return;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    const int k_stride = (int)(2 * a.k_token), v_stride = (int)(2 * a.v_token);
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds;

    const int r = min(row0 + 32 * wave + (lane & 31), rows - 1);
    const bool real = row0 + 32 * wave + (lane & 31) < rows;
    const int token = token_of(a, r), head = kv * a.group + r - token * a.group;
    // keys: this lane's row's, the wavefront's fewest, the workgroup's most
    const int visible = keys_seen(a, s, token);
    const int least = __builtin_amdgcn_readfirstlane(keys_seen(a, s, token_of(a, min(row0 + 32 * wave, rows - 1))));
    const int end = __builtin_amdgcn_readfirstlane(keys_seen(a, s, token_of(a, min(row0 + kTileRows, rows) - 1)));
    const int tiles = (end + kKeys - 1) / kKeys;
    const int t0 = split_begin(a, tiles, split), t1 = split_begin(a, tiles, split + 1);

    auto ask = [&](int t, int to) {
        const int left = s.m - t * kKeys;
        const unsigned at = base + to * kStage;
        load_tile<CHUNKS, kKeys, 64 * kWaves, false>(k + (long)t * kKeys * a.k_token, at, k_stride, left, head_bytes, threadIdx.x);
        load_tile<CHUNKS, kKeys, 64 * kWaves, true>(v + (long)t * kKeys * a.v_token, at + kTile, v_stride, left, head_bytes, threadIdx.x);
    };
    if (t0 < t1) ask(t0, 0);
    v8s q[STEPS];
    const T* const qr = (const T*)a.q + (s.q0 + token) * a.q_token + head * a.q_head;
#pragma unroll
    for (int i = 0; i < STEPS; ++i) {
        const int c = 16 * i + 8 * half;
        q[i] = c < a.head_dim ? *(const v8s*)(qr + c) : v8s{0, 0, 0, 0, 0, 0, 0, 0};
    }
    v16f o[BLOCKS] = {};
    float ref = 0, l = 0;         // exponents are relative to ref
    for (int t = t0; t < t1; ++t) {
        wait_loads_and_barrier();
        const int stage = (t - t0) & 1;
        if (t + 1 < t1) ask(t + 1, stage ^ 1);
        lds_bytes const kt = (lds_bytes)lds + stage * kStage, vt = kt + kTile;
        v16f sc[2] = {};
#pragma unroll
        for (int i = 0; i < STEPS; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] = mfma<TYPE>(read_k<CHUNKS>(kt, 32 * j, i, lane), q[i], sc[j]);
        float top = -kInf;
        if (t * kKeys + kKeys <= least) {
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[j][i] = __builtin_fmaf(sc[j][i], a.scale_log2, -ref);
                    top = fmaxf(top, sc[j][i]);
                }
        } else {
            const int first = t * kKeys + 4 * half;
#pragma unroll
            for (int j = 0; j < 2; ++j)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[j][i] = first + 32 * j + key_of(i) < visible ? __builtin_fmaf(sc[j][i], a.scale_log2, -ref) : -kInf;
                    top = fmaxf(top, sc[j][i]);
                }
        }
        top = fmaxf(top, other_half(top));
        // (a row that sees any key sees the first of its first tile)
        if (t == t0 || __any(top > kSlack)) {
            const float up = t == t0 ? (top == -kInf ? 0.0f : top) : fmaxf(top, 0.0f);
            const float f = __builtin_amdgcn_exp2f(-up);
            ref += up;
            l *= f;
#pragma unroll
            for (int c = 0; c < BLOCKS; ++c) o[c] *= f;
#pragma unroll
            for (int j = 0; j < 2; ++j) sc[j] -= up;
        }
        unsigned p[2][8];
#pragma unroll
        for (int j = 0; j < 2; ++j)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(sc[j][2 * i]), p1 = __builtin_amdgcn_exp2f(sc[j][2 * i + 1]);
                l += p0 + p1;
                p[j][i] = TYPE::pack(p0, p1);
            }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned* pi = p[i >> 1] + 4 * (i & 1);
            const v4i pp = {(int)pi[0], (int)pi[1], (int)pi[2], (int)pi[3]};
#pragma unroll
            for (int c = 0; c < BLOCKS; ++c) o[c] = mfma<TYPE>(read_v<CHUNKS>(vt, 16 * i, c, lane), __builtin_bit_cast(v8s, pp), o[c]);
        }
    }
    l += other_half(l);
    write_rows<TYPE, BLOCKS>(a, o, ref, l, s.q0 + token, head, split, real, half);
}

template <class TYPE>
hipError_t launch(AttentionArgs a, hipStream_t stream) {
    const long items = attention_items(a.sequences, a.Tq, a.group), blocks = (items << a.split_shift) * a.kv_heads;
    a.items = (int)items;
    if (items > 0x7FFFFFFF || blocks * 64 * kWaves >= 1l << 32) return hipErrorInvalidValue;
    void (*kernel)(AttentionArgs) = a.head_dim <= 64   ? attention_tiles<TYPE, 8, 4>
                                    : a.head_dim <= 80 ? attention_tiles<TYPE, 12, 5>
                                    : a.head_dim <= 96 ? attention_tiles<TYPE, 12, 6>
                                                       : attention_tiles<TYPE, 16, 8>;
    return enqueue(kernel, dim3((unsigned)blocks), dim3(64 * kWaves), stream, a);
}

}  // namespace

hipError_t launch_attention_tiles(const AttentionArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch<F16>(a, stream) : launch<BF16>(a, stream);
}

}  // namespace vq
