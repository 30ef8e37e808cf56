// Attention of sequences behind keys that all of them share.  In one pass, the shared keys first, by tiles of query rows or by rows; or, where a
// sequence has few rows and the shared keys are many, in parts: all sequences' rows together with the shared keys, which so are read once for
// all, and in the same launch each sequence's with its own, then a join.
#include "vq_attention_rows_kernel.h"
#include "vq_attention_tiles_kernel.h"

namespace vq {

AttentionPrefixChoice choose_attention_prefix(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads, int head_dim) {
    const int group = heads / kv_heads;
    const long rows = (long)Tq * group;          // of all sequences
    AttentionPrefixChoice c{};
    auto groups = [&](long tiles, int shift) { return ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads; };
    // What one pass reads of the shared keys more than once.
    const long again = (long)(sequences - 1) * prefix * kv_heads * head_dim * 4;
    if (rows > 64l * sequences || again < 8l << 20) {
        c.pass = rows > 32l * sequences ? kAttentionTiles : kAttentionRows;
        const long keys = (long)Tk / sequences + prefix, tiles = c.pass == kAttentionTiles ? attention_items(sequences, Tq, group) : sequences;
        if (c.pass == kAttentionRows) c.split_shift = split_of_equal(tiles * kv_heads, keys);
        while (c.pass == kAttentionTiles && c.split_shift < 6 && (tiles * kv_heads << c.split_shift) < 512 && keys >> (c.split_shift + 1) >= 256) ++c.split_shift;
        c.fits = groups(tiles, c.split_shift) * 256 < 1l << 32;
        return c;
    }
    c.in_parts = true;
    const long own = (long)Tk / sequences, own_items = (long)sequences * kv_heads;
    while (c.split_shift < 5 && (own_items << c.split_shift) < 512 && own >> (c.split_shift + 1) >= 256) ++c.split_shift;
    c.pass = rows <= 32 ? kAttentionRows : kAttentionTiles;
    const long tiles = c.pass == kAttentionRows ? 1 : (rows + kTileRows - 1) / kTileRows;
    while (c.shared_shift < 5 && (tiles * kv_heads << c.shared_shift) < (own_items >= 256 ? 128 : 384) && (long)prefix >> (c.shared_shift + 1) >= 256) ++c.shared_shift;
    c.fits = (groups(sequences, c.split_shift) + shared_blocks(tiles, c.shared_shift, kv_heads)) * 256 < 1l << 32;
    return c;
}

namespace {

struct PartsArgs {
    AttentionSharedArgs shared;
    AttentionOwnArgs own;
    unsigned shared_blocks;
};

// Both kinds of parts in one launch: neither fills the chip for long.  PASS: the kernel of the shared keys.
template <class TYPE, int CHUNKS, int STEPS, AttentionKernel PASS>
__global__ __launch_bounds__(256, 2) void attention_parts(PartsArgs a) {
    constexpr int rows = kRowsBytes<CHUNKS, 4, 1>, tiles = PASS == kAttentionTiles ? kTilesBytes<CHUNKS> : 0;
    __shared__ __align__(16) char lds[rows > tiles ? rows : tiles];
    if (blockIdx.x >= a.shared_blocks) rows_of<TYPE, CHUNKS, STEPS, 4, 1>(a.own, blockIdx.x - a.shared_blocks, lds);
    else if constexpr (PASS == kAttentionTiles) tiles_of<TYPE, CHUNKS, STEPS>(a.shared, blockIdx.x, lds);
    else rows_of<TYPE, CHUNKS, STEPS, 4, 1>(a.shared, blockIdx.x, lds);
}

template <class TYPE, AttentionKernel PASS>
hipError_t launch_parts(const PartsArgs& a, unsigned blocks, hipStream_t stream) {
    const int D = a.own.head_dim;
    void (*kernel)(PartsArgs) = D <= 64   ? attention_parts<TYPE, 8, 4, PASS>
                                : D <= 80 ? attention_parts<TYPE, 12, 5, PASS>
                                : D <= 96 ? attention_parts<TYPE, 12, 6, PASS>
                                          : attention_parts<TYPE, 16, 8, PASS>;
    return enqueue(kernel, dim3(blocks), dim3(256), stream, a);
}

template <class TYPE>
hipError_t launch(const AttentionPrefixArgs& a, const AttentionPrefixChoice& choice, int dtype, hipStream_t stream) {
    if (!choice.in_parts) {
        const hipError_t e = choice.pass == kAttentionTiles ? launch_tiles<TYPE>(a, stream) : launch_rows<TYPE, 4, 2>(a, stream);
        return e != hipSuccess || a.split_shift == 0 ? e : launch_join<AttentionArgs>(a, dtype, stream);
    }
    PartsArgs p{{a}, {a}, 0};
    AttentionSharedArgs& s = p.shared;
    s.k = a.prefix_k, s.v = a.prefix_v, s.Tk = a.prefix, s.causal = 0, s.split_shift = choice.shared_shift;
    s.k_token = a.pk_token, s.k_head = a.pk_head, s.v_token = a.pv_token, s.v_head = a.pv_head;
    s.tiles = choice.pass == kAttentionTiles ? (int)(((long)a.Tq * a.group + kTileRows - 1) / kTileRows) : 1;
    p.shared_blocks = (unsigned)shared_blocks(s.tiles, s.split_shift, a.kv_heads);
    const size_t behind = ((size_t)a.Tq << choice.shared_shift) * a.heads;
    p.own.part_o += behind * a.head_dim, p.own.part_ml += behind * 2;
    const unsigned blocks = p.shared_blocks + attention_grid(p.own, a.sequences);
    const hipError_t e = choice.pass == kAttentionTiles ? launch_parts<TYPE, kAttentionTiles>(p, blocks, stream) : launch_parts<TYPE, kAttentionRows>(p, blocks, stream);
    if (e != hipSuccess) return e;
    AttentionPrefixArgs join = a;
    join.parts = choice.parts();
    return launch_join(join, dtype, stream);
}

}  // namespace

hipError_t launch_attention_prefix(const AttentionPrefixArgs& a, const AttentionPrefixChoice& choice, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch<F16>(a, choice, dtype, stream) : launch<BF16>(a, choice, dtype, stream);
}

}  // namespace vq

extern "C" void vq_internal_attention_prefix_choice(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads, int head_dim, int choice[4]) {
    const vq::AttentionPrefixChoice c = vq::choose_attention_prefix(sequences, Tq, prefix, Tk, heads, kv_heads, head_dim);
    choice[0] = c.in_parts;
    choice[1] = c.pass;
    choice[2] = c.split_shift;
    choice[3] = c.shared_shift;
}
