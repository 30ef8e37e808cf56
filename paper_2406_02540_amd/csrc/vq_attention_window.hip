// Attention in a sliding window with first keys that stay visible: the kernels of vq_attention on the tiles of keys that a block of query rows
// sees (Keys<AttentionWindowArgs>, vq_attention.h).
//
// Tiles are bound as vq_attention's, by matrix and vector time one behind the other; a block of rows works on the union of its rows' windows, rounded up to
// tiles of 64, and first keys in tiles of their own: 35 tiles where 32.5 are seen of 2 x 16384 tokens, 16 heads of 72, windows of 2049 and 32 first keys,
// 442 us (689 TFLOP/s, matrix units busy 47 % of the cycles at 1.8 GHz); 18 where 16 are of prompts of up to 8192, 32 heads on 8 of 128, windows of 1024, 4 first
// keys, 243 us (782).  With small windows the rows themselves count: q and out of 2 x 8192 tokens, 32 heads of 128, are 268 MB, and a window of 64 takes 88 us.
// By rows bound by memory: 48 single tokens on 4100 keys, 32 heads on 8 of 128, 143 us (747 MB, 5.2 TB/s).
#include "vq_attention_rows_kernel.h"
#include "vq_attention_tiles_kernel.h"

namespace vq {

long keys_in_window(int sequences, int Tq, int Tk, int group, int causal, int left, int right, int sinks) {
    const long all = (long)Tk / sequences, queries = ((long)Tq + sequences - 1) / sequences;
    const long block = ((long)Tq * group <= 32l * sequences ? 32 : kTileRows) / group + 1;       // tokens of a block of rows
    if (left < 0 || (right < 0 && !causal)) return all;
    const long keys = (queries < block ? queries : block) + left + (causal ? 0 : right) + sinks;
    return keys < all ? keys : all;
}

// As choose_attention(), with the keys that a block of rows works on in the place of the sequence's: a window makes them equal.
AttentionChoice choose_attention_window(int sequences, int Tq, int Tk, int heads, int kv_heads, int causal, int left, int right, int sinks) {
    const int group = heads / kv_heads;
    const long keys = keys_in_window(sequences, Tq, Tk, group, causal, left, right, sinks);
    const bool rows = (long)Tq * group <= 32l * sequences;
    const long tiles = rows ? (long)sequences : attention_items(sequences, Tq, group), items = tiles * kv_heads;
    int shift = rows ? split_of_equal(items, keys) : 0;
    while (!rows && shift < 6 && (items << shift) < 512 && keys >> (shift + 1) >= 256) ++shift;
    const bool alone = rows && shift == 0 && keys <= 64 && (long)sequences * kv_heads >= 2048;
    const long most = ((tiles << shift) + kItemsRounded) * kv_heads;
    return {!rows ? kAttentionTiles : alone ? kAttentionRowsAlone : kAttentionRows, shift, most * (alone ? 64 : 256) < 1l << 32};
}

hipError_t launch_attention_window(const AttentionWindowArgs& a, AttentionKernel kernel, int dtype, hipStream_t stream) {
    const bool f16 = dtype == VQ_F16;
    if (kernel == kAttentionRowsAlone) return f16 ? launch_rows<F16, 1, 1>(a, stream) : launch_rows<BF16, 1, 1>(a, stream);
    const hipError_t e = kernel == kAttentionTiles ? (f16 ? launch_tiles<F16>(a, stream) : launch_tiles<BF16>(a, stream))
                         : f16                     ? launch_rows<F16, 4, 2>(a, stream)
                                                   : launch_rows<BF16, 4, 2>(a, stream);
    return e != hipSuccess || a.split_shift == 0 ? e : launch_join<AttentionArgs>(a, dtype, stream);
}

}  // namespace vq

extern "C" void vq_internal_attention_window_choice(int sequences, int Tq, int Tk, int heads, int kv_heads, int causal, int left, int right, int sinks, int choice[2]) {
    const vq::AttentionChoice c = vq::choose_attention_window(sequences, Tq, Tk, heads, kv_heads, causal, left, right, sinks);
    choice[0] = c.kernel;
    choice[1] = c.split_shift;
}
