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

namespace {
// Keys that a block of rows would work on if its sequence had them.
long window_of(int sequences, int Tq, int group, int causal, int left, int right, int sinks) {
    if (left < 0 || (right < 0 && !causal)) return 1l << 40;      // (more than any)
    const long queries = ((long)Tq + sequences - 1) / sequences;
    const long block = ((long)Tq * group <= 32l * sequences ? 32 : kTileRows) / group + 1;       // tokens of a block of rows
    return (queries < block ? queries : block) + left + (causal ? 0 : right) + sinks;
}
}  // namespace

long keys_in_window(int sequences, int Tq, int Tk, int group, int causal, int left, int right, int sinks) {
    const long all = (long)Tk / sequences, keys = window_of(sequences, Tq, group, causal, left, right, sinks);
    return keys < all ? keys : all;
}

// As choose_attention(), with the keys that a block of rows works on in the place of the sequence's. A window makes sequences equal, one that is long
// beside the average leaves them as ragged as they are. Single tokens of up to 32768 keys (12000 on average), 32 heads on 8 of 128, divided as equal
// and as ragged ones (us): no window, 16 sequences 256 and 169, 48 570 and 456; windows of twice the average 198 and 155, 507 and 430, of one and a half
// 154 and 137, 453 and 388, of the average 113 and 117, 337 and 316, of half of it 70 and 91, 197 and 214. Of up to 8000 (2900), 32 sequences: no
// window 127 and 100, twice 99 and 95, one and a half 79 and 90, the average 61 and 79. 4 of up to 32768: 80 and 85, 80 and 85, 68 and 83, 53 and 76.
AttentionChoice choose_attention_window(int sequences, int Tq, int Tk, int heads, int kv_heads, int causal, int left, int right, int sinks) {
    const int group = heads / kv_heads;
    const long keys = keys_in_window(sequences, Tq, Tk, group, causal, left, right, sinks);
    const bool rows = (long)Tq * group <= 32l * sequences;
    const long tiles = rows ? (long)sequences : attention_items(sequences, Tq, group), items = tiles * kv_heads;
    const bool equal = 2 * window_of(sequences, Tq, group, causal, left, right, sinks) < 3 * ((long)Tk / sequences);
    const int shift = rows && equal ? split_of_equal(items, keys) : split_for(rows ? kRaggedWorkgroups : 512, items, keys);
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
