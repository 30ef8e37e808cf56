// Attention whose wavefronts divide the keys: few query rows per sequence (new tokens, short sequences).
#include "vq_attention.h"

namespace vq {
namespace {

constexpr int kRows = 32;       // query rows of a tile: the columns of an MFMA block
constexpr int kKeys = 32;       // keys of a wavefront's tile
constexpr float kInf = __builtin_inff();

// A wavefront's running maximum (base 2, scaled), sum and output of a query row; its other half holds the other keys and channels.
template <int BLOCKS>
struct Row {
    float m = -kInf, l = 0;
    v16f o[BLOCKS] = {};
};

// Every wavefront takes tiles of 32 keys of its own, every WAVES-th of the workgroup's: loads into LDS of its own, no
// barrier; at the end the wavefronts' rows are joined.  CHUNKS: 16-byte chunks of a key in LDS (8, 12, 16); STEPS: of 16 channels.
template <class TYPE, int CHUNKS, int STEPS, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void attention_rows(AttentionArgs a) {
    constexpr int BLOCKS = CHUNKS / 4;                 // of 32 channels
    constexpr int kTile = kKeys * CHUNKS * 16;         // bytes
    constexpr int kStage = 2 * kTile;                  // K, V
    constexpr int kPitch = 32 * BLOCKS + 4;            // floats of a row where the wavefronts' sums meet
    constexpr int kLoads = 2 * kKeys * CHUNKS / 64;    // of a stage, per lane
    constexpr int kBytes = WAVES * 2 * kStage;
    static_assert(WAVES * kRows * (kPitch + 2) * 4 <= kBytes, "the sums fit where the stages were");
    __shared__ __align__(16) char lds[kBytes];
    typedef typename TYPE::T T;

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int half = lane >> 5;
    const int kv = (int)(blockIdx.x % (unsigned)a.kv_heads);
    const unsigned item = blockIdx.x / (unsigned)a.kv_heads;
    const int split = (int)(item % (unsigned)a.splits), b = (int)(item / (unsigned)a.splits);
    const Span s = span_of(a, b);
    const long rows = (long)s.n * a.group;
    const int head_bytes = 2 * a.head_dim;
    const T* const k = (const T*)a.k + s.k0 * a.k_token + kv * a.k_head;
    const T* const v = (const T*)a.v + s.k0 * a.v_token + kv * a.v_head;
    const int k_stride = (int)(2 * a.k_token), v_stride = (int)(2 * a.v_token);
    const unsigned base = (unsigned)(uintptr_t)(lds_bytes)(lds) + wave * 2 * kStage;

    for (long row0 = 0; row0 < rows; row0 += kRows) {
        const long r = row0 + (lane & 31);
        const bool real = r < rows;
        const int token = (int)((real ? r : rows - 1) / a.group), head = kv * a.group + (int)((real ? r : rows - 1) % a.group);
        // keys that this lane's row sees, and those that the tile and this workgroup go through
        const int visible = a.causal ? (int)min((long)s.m, max(0l, (long)s.m - s.n + token + 1)) : s.m;
        const int last_token = (int)(min(row0 + kRows, rows) - 1) / a.group;
        const int end_all = a.causal ? (int)min((long)s.m, max(0l, (long)s.m - s.n + last_token + 1)) : s.m;
        const int tiles = (end_all + kKeys - 1) / kKeys;
        const int t0 = (int)((long)tiles * split / a.splits), t1 = (int)((long)tiles * (split + 1) / a.splits);

        v8s q[STEPS];
        const T* const qr = (const T*)a.q + (s.q0 + token) * a.q_token + head * a.q_head;
#pragma unroll
        for (int i = 0; i < STEPS; ++i) {
            const int c = 16 * i + 8 * half;
            q[i] = c < a.head_dim ? *(const v8s*)(qr + c) : v8s{0, 0, 0, 0, 0, 0, 0, 0};
        }
        Row<BLOCKS> st;
        int stage = 0;
        auto ask = [&](int t, int to) {
            const int left = s.m - t * kKeys;
            const unsigned at = base + to * kStage;
            load_tile<CHUNKS, kKeys, 64, false>(k + (long)t * kKeys * a.k_token, at, k_stride, left, head_bytes, lane);
            load_tile<CHUNKS, kKeys, 64, true>(v + (long)t * kKeys * a.v_token, at + kTile, v_stride, left, head_bytes, lane);
        };
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        if (t0 + wave < t1) ask(t0 + wave, 0);
        for (int t = t0 + wave; t < t1; t += WAVES) {
            const bool more = t + WAVES < t1;
            // (the reads of the stage that is overwritten are done: what they fed has been computed)
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            if (more) {
                ask(t + WAVES, stage ^ 1);
                asm volatile("s_waitcnt vmcnt(%0)" ::"n"(kLoads) : "memory");
            } else {
                asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
            }
            lds_bytes const tile = (lds_bytes)lds + (wave * 2 + stage) * kStage;
            v16f sc = {};
#pragma unroll
            for (int i = 0; i < STEPS; ++i) sc = mfma<TYPE>(read_k<CHUNKS>(tile, 0, i, lane), q[i], sc);
            const int first = t * kKeys + 4 * half;
            float top = -kInf;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                sc[i] = first + key_of(i) < visible ? sc[i] * a.scale_log2 : -kInf;
                top = fmaxf(top, sc[i]);
            }
            top = fmaxf(top, other_half(top));
            const float m = fmaxf(st.m, top);
            const float ref = m == -kInf ? 0.0f : m;                  // (no key yet: every weight is exp2(-inf) = 0)
            const float old = __builtin_amdgcn_exp2f(st.m - ref);
            st.m = m;
            float sum = 0;
            unsigned p[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float p0 = __builtin_amdgcn_exp2f(sc[2 * i] - ref), p1 = __builtin_amdgcn_exp2f(sc[2 * i + 1] - ref);
                sum += p0 + p1;
                p[i] = TYPE::pack(p0, p1);
            }
            st.l = st.l * old + sum;
#pragma unroll
            for (int c = 0; c < BLOCKS; ++c) st.o[c] *= old;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const v4i pp = {(int)p[4 * i], (int)p[4 * i + 1], (int)p[4 * i + 2], (int)p[4 * i + 3]};
#pragma unroll
                for (int c = 0; c < BLOCKS; ++c)
                    st.o[c] = mfma<TYPE>(read_v<CHUNKS>(tile + kTile, 16 * i, c, lane), __builtin_bit_cast(v8s, pp), st.o[c]);
            }
            stage ^= 1;
        }
        st.l += other_half(st.l);

        // Join the wavefronts: sums and weights relative to the largest maximum of a row.
        float* const sums = (float*)lds;                        // [WAVES][kRows][kPitch]
        float* const ml = sums + WAVES * kRows * kPitch;        // [WAVES][kRows][2]
        __syncthreads();
        if (half == 0) {
            ml[(wave * kRows + lane) * 2] = st.m;
            ml[(wave * kRows + lane) * 2 + 1] = st.l;
        }
        float* const mine = sums + (wave * kRows + (lane & 31)) * kPitch;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *(v4f*)(mine + 32 * c + 8 * i + 4 * half) = v4f{st.o[c][4 * i], st.o[c][4 * i + 1], st.o[c][4 * i + 2], st.o[c][4 * i + 3]};
        __syncthreads();
        const int pieces = a.head_dim / 8, count = (int)min((long)kRows, rows - row0);
        for (int i = threadIdx.x; i < count * pieces; i += 64 * WAVES) {
            const int row = i / pieces, c = 8 * (i - row * pieces);
            float m = -kInf, l = 0, o[8] = {};
#pragma unroll
            for (int w = 0; w < WAVES; ++w) m = fmaxf(m, ml[(w * kRows + row) * 2]);
            const float ref = m == -kInf ? 0.0f : m;
#pragma unroll
            for (int w = 0; w < WAVES; ++w) {
                const float f = __builtin_amdgcn_exp2f(ml[(w * kRows + row) * 2] - ref);
                l += ml[(w * kRows + row) * 2 + 1] * f;
                const float* from = sums + (w * kRows + row) * kPitch + c;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] += from[e] * f;
            }
            const long rr = row0 + row;
            const int tk = s.q0 + (int)(rr / a.group), hd = kv * a.group + (int)(rr % a.group);
            if (a.splits == 1) {
                const float inv = l > 0 ? 1.0f / l : 0.0f;
                v4i y;
#pragma unroll
                for (int e = 0; e < 4; ++e) y[e] = (int)TYPE::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
                *(v4i*)((T*)a.out + tk * a.o_token + hd * a.o_head + c) = y;
            } else {
                const size_t slot = ((size_t)split * a.Tq + tk) * a.heads + hd;
                *(v4f*)(a.part_o + slot * a.head_dim + c) = v4f{o[0], o[1], o[2], o[3]};
                *(v4f*)(a.part_o + slot * a.head_dim + c + 4) = v4f{o[4], o[5], o[6], o[7]};
                if (c == 0) *(v2f*)(a.part_ml + slot * 2) = v2f{m, l};
            }
        }
        __syncthreads();      // the next tile's loads go where the sums were
    }
}

// Joins the parts of the rows whose keys were divided among workgroups: a thread takes eight channels of a row.
template <class TYPE>
__global__ __launch_bounds__(256) void attention_join(AttentionArgs a) {
    typedef typename TYPE::T T;
    const int pieces = a.head_dim / 8;
    const int first = min(max(a.cu_q[0], 0), a.Tq), last = min(max(a.cu_q[a.sequences], 0), a.Tq);
    const long all = (long)(last - first) * a.heads * pieces;
    for (long i = (long)blockIdx.x * 256 + threadIdx.x; i < all; i += (long)gridDim.x * 256) {
        const long row = (long)first * a.heads + i / pieces;
        const int c = 8 * (int)(i % pieces);
        const size_t next = (size_t)a.Tq * a.heads;
        float m = -kInf;
        for (int s = 0; s < a.splits; ++s) m = fmaxf(m, a.part_ml[(s * next + row) * 2]);
        const float ref = m == -kInf ? 0.0f : m;
        float l = 0, o[8] = {};
        for (int s = 0; s < a.splits; ++s) {
            const v2f ml = *(const v2f*)(a.part_ml + (s * next + row) * 2);
            const float f = __builtin_amdgcn_exp2f(ml[0] - ref);
            l += ml[1] * f;
            const v4f* from = (const v4f*)(a.part_o + (s * next + row) * a.head_dim + c);
            const v4f lo = from[0], hi = from[1];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += lo[e] * f, o[4 + e] += hi[e] * f;
        }
        const float inv = l > 0 ? 1.0f / l : 0.0f;
        v4i y;
#pragma unroll
        for (int e = 0; e < 4; ++e) y[e] = (int)TYPE::pack(o[2 * e] * inv, o[2 * e + 1] * inv);
        const long token = row / a.heads;
        *(v4i*)((T*)a.out + token * a.o_token + (row - token * a.heads) * a.o_head + c) = y;
    }
}

template <class TYPE>
hipError_t launch_rows(const AttentionArgs& a, hipStream_t stream) {
    const long blocks = (long)a.sequences * a.splits * a.kv_heads;
    constexpr int WAVES = 4;
    if (blocks * 64 * WAVES >= 1l << 32) return hipErrorInvalidValue;
    void (*kernel)(AttentionArgs) = a.head_dim <= 64   ? attention_rows<TYPE, 8, 4, WAVES>
                                    : a.head_dim <= 80 ? attention_rows<TYPE, 12, 5, WAVES>
                                    : a.head_dim <= 96 ? attention_rows<TYPE, 12, 6, WAVES>
                                                       : attention_rows<TYPE, 16, 8, WAVES>;
    return enqueue(kernel, dim3((unsigned)blocks), dim3(64 * WAVES), stream, a);
}

}  // namespace

int attention_splits(int sequences, int Tq, int Tk, int heads, int kv_heads) {
    const int group = heads / kv_heads;
    const long keys = (long)Tk / sequences;
    const bool rows = attention_by_rows(sequences, Tq, group);
    // parts of at least 512 keys of the average sequence, and workgroups for four turns of the chip, or one of tiles
    const long items = (rows ? (long)sequences : attention_items(sequences, Tq, group)) * kv_heads;
    long splits = (rows ? 1024 : 512) / items;
    if (splits > keys / 512) splits = keys / 512;
    return splits < 1 ? 1 : splits > 64 ? 64 : (int)splits;
}

hipError_t launch_attention(const AttentionArgs& a, int dtype, hipStream_t stream) {
    const hipError_t e = !attention_by_rows(a.sequences, a.Tq, a.group) ? launch_attention_tiles(a, dtype, stream)
                         : dtype == VQ_F16                              ? launch_rows<F16>(a, stream)
                                                                        : launch_rows<BF16>(a, stream);
    if (e != hipSuccess || a.splits == 1) return e;
    const long join = ((long)a.Tq * a.heads * (a.head_dim / 8) + 255) / 256;
    return enqueue(dtype == VQ_F16 ? attention_join<F16> : attention_join<BF16>, dim3((unsigned)(join < 1 << 20 ? join : 1 << 20)),
                   dim3(256), stream, a);
}

}  // namespace vq
