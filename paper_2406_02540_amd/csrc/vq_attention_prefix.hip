// Attention of sequences behind keys that all of them share: by tiles of query rows in one pass, the shared keys first; or, where a sequence has
// few rows, all sequences' rows together with the shared keys, which so are read once for all, each sequence's with its own, and a join.
#include "vq_attention_rows_kernel.h"
#include "vq_attention_tiles_kernel.h"

namespace vq {

AttentionPrefixChoice choose_attention_prefix(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads) {
    const int group = heads / kv_heads;
    AttentionPrefixChoice c{};
    c.one_pass = (long)Tq * group > 32l * sequences;
    auto groups = [&](long tiles, int shift) { return ((tiles << shift) + kAttentionXcds - 1) / kAttentionXcds * kAttentionXcds * kv_heads; };
    if (c.one_pass) {
        const long keys = (long)Tk / sequences + prefix, tiles = attention_items(sequences, Tq, group), items = tiles * kv_heads;
        while (c.split_shift < 6 && (items << c.split_shift) < 512 && keys >> (c.split_shift + 1) >= 256) ++c.split_shift;
        c.fits = groups(tiles, c.split_shift) * 256 < 1l << 32;
        return c;
    }
    const long own = (long)Tk / sequences, own_items = (long)sequences * kv_heads;
    while (c.split_shift < 5 && (own_items << c.split_shift) < 2048 && own >> (c.split_shift + 1) >= 256) ++c.split_shift;
    c.shared_by_rows = (long)Tq * group <= 32;
    const long tiles = c.shared_by_rows ? 1 : attention_items(1, Tq, group), items = tiles * kv_heads;
    while (c.shared_shift < 5 && (items << c.shared_shift) < 512 && (long)prefix >> (c.shared_shift + 1) >= 256) ++c.shared_shift;
    c.fits = groups(sequences, c.split_shift) * 256 < 1l << 32 && groups(tiles, c.shared_shift) * 256 < 1l << 32;
    return c;
}

namespace {

template <class TYPE>
hipError_t launch(const AttentionPrefixArgs& a, const AttentionPrefixChoice& choice, int dtype, hipStream_t stream) {
    if (choice.one_pass) {
        const hipError_t e = launch_tiles<TYPE>(a, stream);
        return e != hipSuccess || a.split_shift == 0 ? e : launch_join<AttentionArgs>(a, dtype, stream);
    }
    AttentionSharedArgs shared{a};
    shared.k = a.prefix_k, shared.v = a.prefix_v, shared.sequences = 1, shared.Tk = a.prefix, shared.causal = 0, shared.split_shift = choice.shared_shift;
    shared.k_token = a.pk_token, shared.k_head = a.pk_head, shared.v_token = a.pv_token, shared.v_head = a.pv_head;
    hipError_t e = choice.shared_by_rows ? launch_rows<TYPE, 4, 2>(shared, stream) : launch_tiles<TYPE>(shared, stream);
    if (e != hipSuccess) return e;
    AttentionOwnArgs own{a};
    const size_t behind = ((size_t)a.Tq << choice.shared_shift) * a.heads;
    own.part_o += behind * a.head_dim, own.part_ml += behind * 2;
    e = launch_rows<TYPE, 4, 2>(own, stream);
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

extern "C" void vq_internal_attention_prefix_choice(int sequences, int Tq, int prefix, int Tk, int heads, int kv_heads, int choice[4]) {
    const vq::AttentionPrefixChoice c = vq::choose_attention_prefix(sequences, Tq, prefix, Tk, heads, kv_heads);
    choice[0] = c.one_pass;
    choice[1] = c.shared_by_rows;
    choice[2] = c.split_shift;
    choice[3] = c.shared_shift;
}
