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
__device__ __forceinline__ int find_sequence(const AttentionArgs& a, long item, long& tile) {
    int lo = 0, hi = a.sequences - 1;
    auto first = [&](int b) { return (long)min(max(a.cu_q[b], 0), a.Tq) * a.group / kTileRows + b; };
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
    const int split = (int)(rest % (unsigned)a.splits);
    long tile;
    // (the last tiles of a sequence see the most keys: they go first)
    const int b = find_sequence(a, a.items - 1 - rest / (unsigned)a.splits, tile);
    const Span s = span_of(a, b);
    const long rows = (long)s.n * a.group, row0 = tile * kTileRows;
    if (tile < 0 || row0 >= rows) return;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    const int k_stride = (int)(2 * a.k_token), v_stride = (int)(2 * a.v_token);
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)lds;

    const long r = min(row0 + 32 * wave + (lane & 31), rows - 1);
    const bool real = row0 + 32 * wave + (lane & 31) < rows;
    const int token = (int)(r / a.group), head = kv * a.group + (int)(r - (long)token * a.group);
    // keys that a token sees: this lane's row's, the wavefront's fewest, the workgroup's most
    auto sees = [&](long t) { return a.causal ? (int)min((long)s.m, max(0l, (long)s.m - s.n + t + 1)) : s.m; };
    const int visible = sees(token);
    const int least = __builtin_amdgcn_readfirstlane(sees(min(row0 + 32 * wave, rows - 1) / a.group));
    const int end = sees((min(row0 + kTileRows, rows) - 1) / a.group);
    const int tiles = (end + kKeys - 1) / kKeys;
    const int t0 = (int)((long)tiles * split / a.splits), t1 = (int)((long)tiles * (split + 1) / a.splits);

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
    if (a.splits == 1) {
        const float inv = l > 0 ? 1.0f / l : 0.0f;
        T* const y = (T*)a.out + (s.q0 + token) * a.o_token + head * a.o_head;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                // a lane has four channels of every eight, the other half of the wavefront the rest: one takes this eight, one the next
                unsigned x0 = TYPE::pack(o[c][4 * i] * inv, o[c][4 * i + 1] * inv), x1 = TYPE::pack(o[c][4 * i + 2] * inv, o[c][4 * i + 3] * inv);
                unsigned y0 = TYPE::pack(o[c][4 * i + 4] * inv, o[c][4 * i + 5] * inv), y1 = TYPE::pack(o[c][4 * i + 6] * inv, o[c][4 * i + 7] * inv);
                const auto s0 = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
                const int at = 32 * c + 8 * (i + half);
                if (real && at < a.head_dim) *(v4i*)(y + at) = v4i{(int)s0[0], (int)s1[0], (int)s0[1], (int)s1[1]};
            }
    } else if (real) {
        const size_t slot = ((size_t)split * a.Tq + s.q0 + token) * a.heads + head;
        float* const y = a.part_o + slot * a.head_dim;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 32 * c + 8 * i + 4 * half;
                if (at < a.head_dim) *(v4f*)(y + at) = v4f{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
            }
        if (half == 0) *(v2f*)(a.part_ml + slot * 2) = v2f{l > 0 ? ref : -kInf, l};
    }
}

template <class TYPE>
hipError_t launch(AttentionArgs a, hipStream_t stream) {
    a.items = attention_items(a.sequences, a.Tq, a.group);
    const long blocks = a.items * a.splits * a.kv_heads;
    if (blocks * 64 * kWaves >= 1l << 32) return hipErrorInvalidValue;
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
