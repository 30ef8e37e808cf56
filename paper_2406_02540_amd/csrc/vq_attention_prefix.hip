// Attention of sequences behind keys that all of them share.  In one pass, the shared keys first, by tiles of query rows or by rows; or, where a
// sequence has few rows and the shared keys are many, in parts: all sequences' rows together with the shared keys, which so are read once for
// all, and in the same launch each sequence's with its own, then a join.
//
// One pass by tiles is bound as vq_attention's: 6 images of 4096 tokens behind 300, 16 heads of 72, 615 us (810 TFLOP/s; matrix units busy 51 % of the cycles
// at 1.6 GHz).  In parts: 64 single tokens behind 8192 keys and up to 700 of their own, 32 heads on 8 of 128, 36 us (99 MB, 19 us at a copy's rate): 31 for the
// parts, of which the shared keys alone take 26 (two tiles of 128 rows a head) and the own ones 19 (a few tiles of keys a workgroup: waits for first loads), 5 for the join;
// as a part of every sequence's own keys they are 2.2 GB.  In two launches, one behind the other, it took 54.
#include "vq_attention_rows_kernel.h"
#include "vq_attention_tiles_kernel.h"

namespace vq {

AttentionPrefixChoice choose_attention_prefix(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads, int head_dim) {
    const int group = heads / kv_heads;
    const long rows = (long)Tq * group;          // of all sequences
    auto groups = [&](long tiles, int shift) { return ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads; };
    // In parts where one pass would read at least 8 MB of shared keys over and over, and a sequence's rows leave tiles of 128 as empty as the parts'
    // own traffic weighs.  Parts and one pass (us; heads on heads of k and v): 8 single tokens behind 4096 keys, 32 on 8 of 128, 15 and 26; 16 behind 512
    // 13.3 and 16.3; 2 behind 8192 17.7 and 19.0; 3 x 4 behind 4096, 16 on 2 of 64 (4 MB), 12.6 and 12.1; 12 x 30 behind 3000, 16 on 8 of 64, 25 and 41, x 64 37 and
    // 47; 64 x 100 behind 4000, 8 of 128, 153 and 208; 200 x 64 behind 1000, 16 of 72, 228 and 170.
    const double again = 4.0 * (sequences - 1) * prefix * kv_heads * head_dim;       // (beyond 2^63 where sizes are the largest)
    const long own = (long)Tk / sequences;
    auto one_pass = [&] {
        AttentionPrefixChoice c{};
        c.pass = rows > 32l * sequences ? kAttentionTiles : kAttentionRows;
        const long keys = own + prefix, tiles = c.pass == kAttentionTiles ? attention_items(sequences, Tq, group) : sequences;
        // (sequences are about equal where the prefix is most of what they have. 16 single tokens of up to 32768 keys, 12000 on average, 32 heads on 8
        // of 128, behind 16 others, divided as equal and as ragged ones: 257 us and 170; 48 571 and 457; 32 of up to 8000 129 and 103)
        c.split_shift = c.pass == kAttentionRows && prefix >= own ? split_of_equal(tiles * kv_heads, keys)
                                                                  : split_for(c.pass == kAttentionRows ? kRaggedWorkgroups : 512, tiles * kv_heads, keys);
        c.fits = groups(tiles, c.split_shift) * 256 < 1l << 32;
        return c;
    };
    if (again < 8 << 20 || (rows > 32l * sequences && (rows > 128l * sequences || prefix < 2048 || own > prefix / 4))) return one_pass();
    AttentionPrefixChoice c{};
    c.in_parts = true;
    // Where there are more than single tokens, a workgroup for every block of rows: a prompt among single tokens would take all of its own one after another.
    // 63 single tokens and a prompt of 1900 behind 4000 keys, 32 heads on 8 of 128, 3370 us by sequences and 233, a prompt of 400 295 and 62.
    c.by_blocks = Tq > sequences;
    const long own_blocks = c.by_blocks ? rows / kOwnRows + sequences : sequences, own_items = own_blocks * kv_heads;
    // Own keys of few rows are divided as vq_attention's (at most 32 parts of them and 32 of the shared ones): single tokens of up to 32768 keys, 12000 on
    // average, 32 heads on 8 of 128, behind 4096 others with workgroups for two turns of the chip and for eight, 16 sequences 237 us and 182, 48 583 and 481;
    // 32 of up to 8000 behind 2048 110 and 91; 8 equal ones of 16000 behind 8192 114 and 117, 64 of 4096 220 and 224.
    c.split_shift = split_for(rows <= 32l * sequences ? kRaggedWorkgroups : 512, own_items, own, 5);
    // Parts of the shared keys for half of the chip where the sequences' own workgroups fill it by themselves: 64 single tokens behind 8192 keys
    // with 4, 8, 16 and 32 of them 53, 37, 43 and 52 us; 5 x 7 behind 30011, where they do not, with 8, 16, 32 and 64 56, 34, 24.5 and 25.6.
    c.pass = rows <= 32 ? kAttentionRows : kAttentionTiles;
    const long tiles = c.pass == kAttentionRows ? 1 : (rows + kTileRows - 1) / kTileRows;
    while (c.shared_shift < 5 && (tiles * kv_heads << c.shared_shift) < ((long)sequences * kv_heads >= 256 ? 128 : 384) && (long)prefix >> (c.shared_shift + 1) >= 256) ++c.shared_shift;
    // (parts take more workgroups than one pass: where a launch does not hold them it is one pass)
    if ((groups(own_blocks, c.split_shift) + shared_blocks(tiles, c.shared_shift, kv_heads)) * 256 >= 1l << 32) return one_pass();
    c.fits = true;
    c.own_items = (int)own_blocks;
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
    PartsArgs p{{a}, {a, 0}, 0};
    AttentionSharedArgs& s = p.shared;
    s.k = a.prefix_k, s.v = a.prefix_v, s.Tk = a.prefix, s.causal = 0, s.split_shift = choice.shared_shift;
    s.k_token = a.pk_token, s.k_head = a.pk_head, s.v_token = a.pv_token, s.v_head = a.pv_head;
    s.tiles = choice.pass == kAttentionTiles ? (int)(((long)a.Tq * a.group + kTileRows - 1) / kTileRows) : 1;
    p.shared_blocks = (unsigned)shared_blocks(s.tiles, s.split_shift, a.kv_heads);
    const size_t behind = ((size_t)a.Tq << choice.shared_shift) * a.heads;
    p.own.part_o += behind * a.head_dim, p.own.part_ml += behind * 2;
    p.own.by_blocks = choice.by_blocks;
    const unsigned blocks = p.shared_blocks + attention_grid(p.own, choice.own_items);
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
extern "C" int vq_internal_attention_prefix_own_items(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads, int head_dim) {
    return vq::choose_attention_prefix(sequences, Tq, prefix, Tk, heads, kv_heads, head_dim).own_items;
}
