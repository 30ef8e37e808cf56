// Attention in a sliding window with first keys that stay visible.
#include "vq_attention_simple.h"

namespace vq {
namespace {

struct WindowKeys {
    const AttentionWindowArgs& a;
    const Span& s;
    int kv, p, count;
    __device__ WindowKeys(const AttentionWindowArgs& a, const Span& s, int token, int kv) : a(a), s(s), kv(kv), p(token + s.m - s.n), count(s.m) {}
    __device__ bool seen(int key) const {
        const long d = (long)key - p;
        return ((d >= -a.left && (a.right < 0 || d <= a.right)) || key < a.sinks) && !(a.causal && d > 0);
    }
    template <class T>
    __device__ const T* k(int key) const { return (const T*)a.k + (s.k0 + key) * a.k_token + kv * a.k_head; }
    template <class T>
    __device__ const T* v(int key) const { return (const T*)a.v + (s.k0 + key) * a.v_token + kv * a.v_head; }
};

template <class TYPE>
__global__ __launch_bounds__(256) void attention_window(AttentionWindowArgs a) {
    attention_simple<TYPE, AttentionWindowArgs, WindowKeys>(a);
}

}  // namespace

AttentionChoice choose_attention_window(int, int, int, int, int, int, int, int, int) { return {kAttentionRows, 0, true}; }

hipError_t launch_attention_window(const AttentionWindowArgs& a, AttentionKernel, int dtype, hipStream_t stream) {
    const long blocks = ((long)a.Tq * a.heads + 3) / 4;
    return enqueue(dtype == VQ_F16 ? attention_window<F16> : attention_window<BF16>, dim3((unsigned)(blocks < 1 << 20 ? blocks : 1 << 20)), dim3(256), stream, a);
}

}  // namespace vq
