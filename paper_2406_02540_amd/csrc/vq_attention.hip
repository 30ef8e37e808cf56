// Attention whose wavefronts divide the keys: few query rows per sequence (new tokens, short sequences).
#include "vq_attention_rows_kernel.h"

namespace vq {

AttentionChoice choose_attention(int sequences, int Tq, int Tk, int heads, int kv_heads) {
    const int group = heads / kv_heads;
    const long keys = (long)Tk / sequences;
    // Rows of the average sequence: up to 32, one MFMA block of them.  With all in tiles 16 single tokens over long keys take 230 us instead
    // of 170 and 2048 sequences of 16 239 instead of 84 (64 equal ones over 4096 keys 191 and 215); with up to 64 by rows 16 sequences of 64
    // rows over 4096 keys 151 instead of 71 and 512 sequences of 64 91 instead of 75.
    const bool rows = (long)Tq * group <= 32l * sequences;
    // Parts of at least 256 keys of the average sequence, and workgroups for eight turns of the chip, or one of tiles.  Undivided and
    // divided (us, captured, inputs that are not in the caches): a token of one sequence over 32768 keys 437 and 39, of 16 ragged ones
    // 442 and 170, 512 queries over 32768 584 and 280, 64 tokens of 2 sequences over 8192 156 and 35.  Eight turns are for ragged sequences,
    // where the longest decides: workgroups for two make those 16 199, but 64 equal ones over 4096 keys 190 instead of 215.
    const long tiles = rows ? (long)sequences : attention_items(sequences, Tq, group), items = tiles * kv_heads;
    const int shift = split_for(rows ? kRaggedWorkgroups : 512, items, keys);
    // A wavefront alone, one tile of keys at a time, where the average sequence has a few tiles and there are sequences enough: 2048
    // sequences of 16, 16 heads of 72, 84 us, by four wavefronts 542, most of which have no keys.
    const bool alone = rows && shift == 0 && keys <= 64 && (long)sequences * kv_heads >= 2048;
    // (HIP takes less than 2^32 threads; the items of a kernel are rounded up to whole groups of XCDs)
    const long most = ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads;
    return {!rows ? kAttentionTiles : alone ? kAttentionRowsAlone : kAttentionRows, shift, most * (alone ? 64 : 256) < 1l << 32};
}

hipError_t launch_attention(const AttentionArgs& a, AttentionKernel kernel, int dtype, hipStream_t stream) {
    const bool f16 = dtype == VQ_F16;
    if (kernel == kAttentionRowsAlone) return f16 ? launch_rows<F16, 1, 1>(a, stream) : launch_rows<BF16, 1, 1>(a, stream);
    const hipError_t e = kernel == kAttentionTiles ? launch_attention_tiles(a, dtype, stream)
                         : f16                     ? launch_rows<F16, 4, 2>(a, stream)
                                                   : launch_rows<BF16, 4, 2>(a, stream);
    if (e != hipSuccess || a.split_shift == 0) return e;
    return launch_join(a, dtype, stream);
}

}  // namespace vq

extern "C" void vq_internal_attention_choice(int sequences, int Tq, int Tk, int heads, int kv_heads, int choice[2]) {
    const vq::AttentionChoice c = vq::choose_attention(sequences, Tq, Tk, heads, kv_heads);
    choice[0] = c.kernel;
    choice[1] = c.split_shift;
}
