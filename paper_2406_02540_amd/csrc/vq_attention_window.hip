// Attention in a sliding window with first keys that stay visible: the kernels of vq_attention on the tiles of keys that a block of query rows sees.
#include "vq_attention_rows_kernel.h"
#include "vq_attention_tiles_kernel.h"

namespace vq {

AttentionChoice choose_attention_window(int sequences, int Tq, int Tk, int heads, int kv_heads, int causal, int left, int right, int sinks) {
    const int group = heads / kv_heads;
    // Keys that a block of the average sequence's rows works on.
    const long all = (long)Tk / sequences, queries = ((long)Tq + sequences - 1) / sequences;
    const bool rows = (long)Tq * group <= 32l * sequences;
    const long tokens = rows ? (queries < 32 / group + 1 ? queries : 32 / group + 1) : queries < kTileRows / group + 1 ? queries : kTileRows / group + 1;
    long keys = sinks + tokens;
    keys = left < 0 ? all : keys + left;
    if (!causal) keys = right < 0 ? all : keys + right;
    if (keys > all) keys = all;
    const long tiles = rows ? (long)sequences : attention_items(sequences, Tq, group), items = tiles * kv_heads;
    int shift = 0;
    while (shift < 6 && (items << shift) < (rows ? 2048 : 512) && keys >> (shift + 1) >= 256) ++shift;
    const bool alone = rows && shift == 0 && keys <= 64 && (long)sequences * kv_heads >= 2048;
    const long most = ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads;
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
