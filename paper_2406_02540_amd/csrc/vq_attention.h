// Attention over packed sequences: what its kernels share.  gfx950 only.
//
// For the query rows of a tile and the keys in turn, with m the largest score of a row so far:
//     S = scale * Q K^T,  m' = max(m, rowmax S),  P = exp(S - m'),  l = l exp(m - m') + rowsum P,  O = O exp(m - m') + P V
// and O / l at the end: one pass over K and V, nothing of S leaves the registers.
//
// m, l and O are fp32; P goes into the second product rounded to the type of V, since a matrix instruction takes one type.  Relative error
// of fp16 outputs against 64 bits, where their own rounding alone makes 2.07e-4: 2 x 4096, 16 heads of 72 2.9e-4; 2 x 16384 queries on 120 keys 2.5e-4;
// 16 single tokens over up to 32768 keys 2.6e-4.  A second product, with what the rounding left of P, makes each of them 2.07e-4 and takes 283 us
// instead of 207, 61 to 66 instead of 57, 175 instead of 170; 4 x 4096, 16 heads of 128 706 instead of 524, 16 x 64 rows over 4096 keys 76 to 80
// instead of 69 (captured, inputs that are not in the caches).
//
// The matrix cores compute S^T = K Q^T and O^T = V^T P^T in blocks of 32 x 32 x 16: a lane's column is a query row, so that a
// row's maximum and sum are a lane's own values and one exchange with the other half of the wavefront, and
// the P^T that it holds after the exponentials is the operand of the second product as it lies: a lane has keys 8i + 4h + 0..3
// (h its half), and since the order of keys in a product is free, V^T is read in that order too (transposed on its way from
// LDS, four keys a read).
//
// Query heads that share a head of K and V are rows of one tile: row r of a sequence is token r / group, head r % group.
#pragma once
#include "vq_gemm_common.h"
#include "vq_internal.h"
#include "vq_types.h"

namespace vq {

typedef float v16f __attribute__((ext_vector_type(16)));
typedef short v4s __attribute__((ext_vector_type(4)));
typedef short v8s __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char* lds_bytes;

// ---- sequences -----------------------------------------------------------------------------------------------

// What a workgroup works on.  The offsets come from device memory: whatever they are, rows stay within the tensors.
struct Span {
    int q0, n, k0, m;       // first query row and rows, first key and keys
};
__device__ __forceinline__ Span span_of(const AttentionArgs& a, int b) {
    Span s;
    s.q0 = min(max(a.cu_q[b], 0), a.Tq);
    s.n = min(max(a.cu_q[b + 1], s.q0), a.Tq) - s.q0;
    s.k0 = min(max(a.cu_k[b], 0), a.Tk);
    s.m = min(max(a.cu_k[b + 1], s.k0), a.Tk) - s.k0;
    return s;
}

__device__ __forceinline__ int token_of(const AttentionArgs& a, int row) {
    return a.group_shift >= 0 ? row >> a.group_shift : (int)((unsigned)row / (unsigned)a.group);
}
// Keys of its sequence that a token sees.
__device__ __forceinline__ int keys_seen(const AttentionArgs& a, const Span& s, int token) {
    return a.causal ? min(s.m, max(0, s.m - s.n + token + 1)) : s.m;
}
// Tiles of keys of a workgroup among those that divide `tiles` (less than 2^26 of them; at most 2^6 workgroups).
__device__ __forceinline__ int split_begin(const AttentionArgs& a, int tiles, int split) {
    return (int)((unsigned)tiles * (unsigned)split >> a.split_shift);
}

// Which item a workgroup takes (false: none), and which head of K and V.  Workgroup ids are dealt round-robin to the XCDs.  A head's
// items go to one XCD (as far as the heads are a multiple of them), whose L2 then has its keys, or all heads of an item, whose
// rows share memory lines of q and out where a head is no whole lines: with few keys those are the traffic, and a line that is written
// from two XCDs is written in pieces.  2 x 16384 queries on 120 keys, 16 heads of 72: 65.6 us by heads, 59.5 together (captured, inputs
// that are not in the caches); 2048 sequences of 16 93.7 and 84; heads of 96 34.9 and 33.9.  With many keys they are better by heads: 32
// sequences of 1024 223 and 232; so are heads of whole lines: of 128 on 128 keys 43 and 45 (both with inputs in the caches).
constexpr int kAttentionXcds = 8;
__device__ __forceinline__ bool place_of(const AttentionArgs& a, int& kv, int& item) {
    if (a.heads_together) {
        const unsigned j = blockIdx.x / kAttentionXcds, group = j / (unsigned)a.kv_heads;
        kv = (int)(j - group * (unsigned)a.kv_heads);
        item = (int)(group * kAttentionXcds + blockIdx.x % kAttentionXcds);
    } else {
        const unsigned j = blockIdx.x / (unsigned)a.kv_heads;
        kv = (int)(blockIdx.x - j * (unsigned)a.kv_heads);
        item = (int)j;
    }
    return item < a.items;
}
// The workgroups that place_of() has in mind (choose_attention() has seen that a launch takes them).
inline unsigned attention_grid(AttentionArgs& a, long tiles) {
    a.tiles = (int)tiles;
    a.items = (int)(tiles << a.split_shift);
    a.heads_together = a.Tk / a.sequences <= 512 && a.head_dim % 64 != 0;
    const long items = a.heads_together ? ((long)a.items + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds : a.items;
    return (unsigned)(items * a.kv_heads);
}

// ---- tiles of K and V in LDS ---------------------------------------------------------------------------------
// [key][CHUNKS of 16 bytes], the chunk of a key at chunk ^ swizzle(key), so that what the LDS serves at once lies in different banks:
// K is read 16 bytes a lane, one chunk of 32 keys at a time (sixteen lanes are served together: keys 0-3, 12-15 and 20-27, or the
// others); V transposed, 8 bytes a lane, 64 bytes of keys 4i .. 4i+3 at a time.
template <int CHUNKS>
__device__ __forceinline__ int k_swizzle(int key) {
    return CHUNKS == 16 ? key & 15 : CHUNKS == 12 ? (key >> 2) & 3 : (key >> 1) & 7;
}
template <int CHUNKS>
__device__ __forceinline__ int v_swizzle(int key) {
    return CHUNKS == 16 ? (key & 3) << 2 : CHUNKS == 12 ? 0 : (key >> 1 & 1) << 2;
}

constexpr int kBehind = 0x7FFFFFF0;        // an offset that no buffer reaches: its lanes load zeros

// What a thread loads of KEYS rows of K or V, THREADS threads together.  Rows are at most 2^24 bytes apart.
template <int CHUNKS, int KEYS, int THREADS, bool IS_V>
struct TileLoader {
    static_assert(KEYS * CHUNKS % THREADS == 0, "whole turns");
    static constexpr int kTurns = KEYS * CHUNKS / THREADS;
    int at[kTurns];          // from the tile's first row; kBehind behind the head's channels
    __device__ __forceinline__ TileLoader(int stride, int head_bytes, int thread) {
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            const int p = i * THREADS + thread, key = p / CHUNKS, slot = p % CHUNKS;
            const int c = slot ^ (IS_V ? v_swizzle<CHUNKS>(key) : k_swizzle<CHUNKS>(key));
            at[i] = opaque(16 * c < head_bytes ? key * stride + 16 * c : kBehind);
        }
    }
    // Asks for the rows from `base` on, into LDS from `lds` (this wavefront's share: its first thread's 16 bytes).  Rows from `left` on come
    // as zeros.  KEEP: what lies behind the head's channels in LDS stays.
    template <bool KEEP = false>
    __device__ __forceinline__ void ask(const void* base, unsigned lds, int left, int thread) const {
        const v4i rsrc = make_rsrc(base, 0x7FFFFF00u);
#pragma unroll
        for (int i = 0; i < kTurns; ++i) {
            if (KEEP && at[i] == kBehind) continue;
            if (left >= KEYS) load_to_lds_16(rsrc, lds + i * THREADS * 16, at[i], 0);
            else load_to_lds_16(rsrc, lds + i * THREADS * 16, (i * THREADS + thread) / CHUNKS < left ? at[i] : kBehind, 0);
        }
    }
};

template <class TYPE>
__device__ __forceinline__ v16f mfma(v8s a, v8s b, v16f c);
template <>
__device__ __forceinline__ v16f mfma<F16>(v8s a, v8s b, v16f c) {
    typedef _Float16 h8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8, a), __builtin_bit_cast(h8, b), c, 0, 0, 0);
}
template <>
__device__ __forceinline__ v16f mfma<BF16>(v8s a, v8s b, v16f c) {
    typedef __bf16 b8 __attribute__((ext_vector_type(8)));
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8, a), __builtin_bit_cast(b8, b), c, 0, 0, 0);
}

// Where a lane reads K: rows `lane % 32` of 32 keys, channels 16 step + 8 (lane / 32) .. + 7.  The swizzle is an exclusive or on the
// chunk's number: with 12 chunks on its lower two bits, so that the steps are two places and constants; otherwise a place for every step.
template <int CHUNKS, int STEPS>
struct KeyReader {
    static constexpr int kPlaces = CHUNKS == 12 ? 2 : STEPS;
    lds_bytes at[kPlaces];
    __device__ __forceinline__ KeyReader(lds_bytes tile, int lane) {
        const int key = lane & 31, half = lane >> 5, s = k_swizzle<CHUNKS>(key);
#pragma unroll
        for (int i = 0; i < kPlaces; ++i)
            at[i] = (lds_bytes)(uintptr_t)(unsigned)opaque((int)(unsigned)(uintptr_t)(tile + key * CHUNKS * 16 + ((2 * i + half) ^ s) * 16));
    }
    // 32 keys from key0, of a tile `offset` bytes behind the one named above
    __device__ __forceinline__ v8s read(int offset, int key0, int step) const {
        lds_bytes const p = CHUNKS == 12 ? at[step & 1] + 64 * (step >> 1) : at[CHUNKS == 12 ? 0 : step];
        return *(__attribute__((address_space(3))) v8s*)(p + offset + key0 * CHUNKS * 16);
    }
};

// And V, transposed: channel 32 block + lane % 32 of keys key0 + 4h .. + 3 and key0 + 8 + 4h .. + 3, h = lane / 32.  In a transposed
// read sixteen lanes name four rows of sixteen channels, four lanes a row, and each receives a column.
template <int CHUNKS>
struct ValueReader {
    static constexpr int kPlaces = CHUNKS == 12 ? 1 : CHUNKS / 4;
    lds_bytes at[kPlaces];
    __device__ __forceinline__ ValueReader(lds_bytes tile, int lane) {
        const int in16 = lane & 15, key = 4 * (lane >> 5) + (in16 >> 2), c = 2 * (lane >> 4 & 1) + (in16 >> 1 & 1);
#pragma unroll
        for (int i = 0; i < kPlaces; ++i)
            at[i] = (lds_bytes)(uintptr_t)(unsigned)opaque(
                (int)(unsigned)(uintptr_t)(tile + (key * CHUNKS + ((4 * i + c) ^ v_swizzle<CHUNKS>(key))) * 16 + 8 * (in16 & 1)));
    }
    __device__ __forceinline__ v8s read(int offset, int key0, int block) const {
        // (key0 a multiple of 8: the swizzle is the same)
        lds_bytes const p = (CHUNKS == 12 ? at[0] + 64 * block : at[CHUNKS == 12 ? 0 : block]) + offset + key0 * CHUNKS * 16;
        const v4s lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)p);
        const v4s hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) v4s*)(p + 8 * CHUNKS * 16));
        return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// The key of register r of a block of S^T, less the block's first.
__device__ __forceinline__ constexpr int key_of(int r) { return (r & 3) + 8 * (r >> 2); }   // + 4 (lane / 32)

// A wavefront's 32 rows of outputs, whose lanes' sums l and outputs o (relative to ref) are complete: normalised to `out`, or as they are
// to the parts.  `row`: token (of all) and head of the lane's row.
template <class TYPE, int BLOCKS>
__device__ __forceinline__ void write_rows(const AttentionArgs& a, const v16f* o, float ref, float l, int token, int head, int split, bool real, int half) {
    typedef typename TYPE::T T;
    if (a.split_shift == 0) {
        const float inv = l > 0 ? 1.0f / l : 0.0f;
        T* const y = (T*)a.out + token * a.o_token + head * a.o_head;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                // a lane has four channels of every eight, the other half of the wavefront the rest: one takes this eight, one the next
                const unsigned x0 = TYPE::pack(o[c][4 * i] * inv, o[c][4 * i + 1] * inv), x1 = TYPE::pack(o[c][4 * i + 2] * inv, o[c][4 * i + 3] * inv);
                const unsigned y0 = TYPE::pack(o[c][4 * i + 4] * inv, o[c][4 * i + 5] * inv), y1 = TYPE::pack(o[c][4 * i + 6] * inv, o[c][4 * i + 7] * inv);
                const auto s0 = __builtin_amdgcn_permlane32_swap(x0, y0, false, false);
                const auto s1 = __builtin_amdgcn_permlane32_swap(x1, y1, false, false);
                const int at = 32 * c + 8 * (i + half);
                if (real && at < a.head_dim) *(v4i*)(y + at) = v4i{(int)s0[0], (int)s1[0], (int)s0[1], (int)s1[1]};
            }
    } else if (real) {
        const size_t slot = ((size_t)split * a.Tq + token) * a.heads + head;
        float* const y = a.part_o + slot * a.head_dim;
#pragma unroll
        for (int c = 0; c < BLOCKS; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int at = 32 * c + 8 * i + 4 * half;
                if (at < a.head_dim) *(v4f*)(y + at) = v4f{o[c][4 * i], o[c][4 * i + 1], o[c][4 * i + 2], o[c][4 * i + 3]};
            }
        if (half == 0) *(v2f*)(a.part_ml + slot * 2) = v2f{l > 0 ? ref : -__builtin_inff(), l};
    }
}

__device__ __forceinline__ float other_half(float v) {
    const unsigned u = __builtin_bit_cast(unsigned, v);
    const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
    // (r[0]: the low half's value in both halves, r[1]: the high half's)
    return __builtin_bit_cast(float, (threadIdx.x & 32) ? r[0] : r[1]);
}

}  // namespace vq
