// Attention of sequences behind keys that all of them share.
#include "vq_attention_simple.h"

namespace vq {
namespace {

struct PrefixKeys {
    const AttentionPrefixArgs& a;
    const Span& s;
    int kv, count;
    __device__ PrefixKeys(const AttentionPrefixArgs& a, const Span& s, int token, int kv) : a(a), s(s), kv(kv), count(a.prefix + keys_seen(a, s, token)) {}
    __device__ bool seen(int) const { return true; }
    template <class T>
    __device__ const T* k(int key) const {
        return key < a.prefix ? (const T*)a.prefix_k + key * a.pk_token + kv * a.pk_head
                              : (const T*)a.k + (s.k0 + key - a.prefix) * a.k_token + kv * a.k_head;
    }
    template <class T>
    __device__ const T* v(int key) const {
        return key < a.prefix ? (const T*)a.prefix_v + key * a.pv_token + kv * a.pv_head
                              : (const T*)a.v + (s.k0 + key - a.prefix) * a.v_token + kv * a.v_head;
    }
};

template <class TYPE>
__global__ __launch_bounds__(256) void attention_prefix(AttentionPrefixArgs a) {
    attention_simple<TYPE, AttentionPrefixArgs, PrefixKeys>(a);
}

}  // namespace

hipError_t launch_attention_prefix(const AttentionPrefixArgs& a, int dtype, hipStream_t stream) {
    const long blocks = ((long)a.Tq * a.heads + 3) / 4;
    return enqueue(dtype == VQ_F16 ? attention_prefix<F16> : attention_prefix<BF16>, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), stream, a);
}

}  // namespace vq
