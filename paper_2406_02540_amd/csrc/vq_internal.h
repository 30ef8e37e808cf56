// Internal launch interface between the C-ABI front end (vq_api.hip) and the
// gfx950 kernels.  Every launcher enqueues on `stream` and returns the HIP
// error of the launch; arguments were validated by the caller.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "vq.h"

namespace vq {

// A kernel of one argument.  (An argument costs the host 0.04 us, the <<<>>> stub 0.15 us beyond the 2.1 that a launch
// takes; small layers are host-bound.)
template <class Args>
inline hipError_t enqueue(void (*kernel)(Args), dim3 grid, dim3 block, hipStream_t stream, const Args& a) {
    void* args[] = {const_cast<Args*>(&a)};
    const hipError_t e = hipLaunchKernel((const void*)kernel, grid, block, args, 0, stream);
    if (e != hipSuccess) (void)hipGetLastError();   // (reported here, not once more by the next call)
    return e;
}

hipError_t launch_quantize_per_token(const void* x_f16, const float* chan_mul, int8_t* xq,
                                     float* x_scale, int M, int K, hipStream_t stream);

// Its part for rows of whole chunks (vq_fused.hip): K % 8 == 0, K <= 8192, 16-byte aligned.
hipError_t launch_plain_quantize(const void* x_f16, const float* chan_mul, int8_t* xq, float* x_scale, int M, int K,
                                 hipStream_t stream);

// What runs in front of the quantizer, and its operands (those that it does not have stay null).
enum Producer { kGeluErf = 0, kGeluTanh = 1, kLayerNorm = 2, kResidual = 3, kHadamard = 4, kPlain = 5 };
struct ProducerArgs {
    int producer;
    const void* x;            // fp16 [M,K]
    const float* chan_mul;    // Eq. 3's factor [K], or null
    const void* y;            // residual: the branch output, fp16 [M,K]
    void* r;                  // residual: the sum, fp16 [M,K]
    const float* mod_a;       // LayerNorm: scale [B,K]; residual: gate [B,K]; or null
    const float* mod_b;       // LayerNorm: shift [B,K]; or null
    int tokens_per_sample;    // >= 1
    float eps;
};

// The quantizer behind its producer (vq_fused.hip; kPlain goes to launch_quantize_per_token):
// K % 8 == 0, K <= 8192 (Hadamard: K % 128 == 0).
hipError_t launch_producer_quantize(const ProducerArgs& p, int8_t* xq, float* x_scale, int M, int K, hipStream_t stream);
hipError_t launch_rotate_weight(const float* w, const float* chan_s, float* w_rot, int N, int K,
                                hipStream_t stream);                  // K % 128 == 0, K <= 8192

// Calibration of Eq. 3's mask: column absmax of fp16 (is_f32 = 0) or fp32 rows, and the mask itself.
hipError_t launch_channel_absmax(const void* a, int is_f32, float* amax, int R, int K, int accumulate,
                                 hipStream_t stream);
hipError_t launch_balance_mask(const float* amax_x, const float* amax_w, float alpha, float* s, float* chan_mul,
                               int K, hipStream_t stream);

hipError_t launch_quantize_static(const void* x_f16, const float* chan_mul, float inv_scale, int8_t* xq,
                                  int M, int K, hipStream_t stream);

hipError_t launch_quantize_weight(const float* w, const float* chan_s, int w_bits, void* wq_out,
                                  float* w_scale, int N, int K, hipStream_t stream);

// w_bits 8: w is int8 [N,K]; 4: w is packed nibbles [N,K/2]; 16: the fp16 comparison layer, xq and w
// are fp16 [M,K] and [N,K], x_scale and w_scale are not read, acc_out must be null.  num_cus: compute units of
// the device the stream belongs to (the kernel is persistent, one workgroup per CU).
hipError_t launch_gemm(const int8_t* xq, const float* x_scale, const void* w, int w_bits,
                       const float* w_scale, const void* bias_f16, void* y_f16, int32_t* acc_out,
                       int M, int N, int K, int num_cus, hipStream_t stream);

// The kernel that launch_gemm takes: tiles of tokens x channels, and the number of wavefronts that divide K (0:
// the workgroup shares the tile; with 256 tokens it is the persistent kernel).
struct GemmChoice { int tile_t, tile_c, waves; };
GemmChoice choose_gemm(int w_bits, int M, int N, int K, int num_cus);

// A layer of few tokens in one launch (vq_linear_small.hip): quantizer, with its producer, and GEMM.
// small_layer: whether it is the faster way for these sizes.
bool small_layer(int producer, int M, int N, int K, int num_cus);
hipError_t launch_linear_small(const ProducerArgs& p, const void* w, int w_bits, const float* w_scale, const void* bias_f16,
                               void* y_f16, int M, int N, int K, hipStream_t stream);

// ---- microscaled 4-bit floating point (vq_mx4_quantize.hip, vq_mx4_gemm_split.hip) -----------------------------
hipError_t launch_mx4_quantize(const void* x, int dtype, const float* chan_mul, uint8_t* xq, uint8_t* x_scale, int M, int K,
                               hipStream_t stream);
hipError_t launch_mx4_dequantize(const uint8_t* xq, const uint8_t* x_scale, void* x, int dtype, int M, int K,
                                 hipStream_t stream);
struct Mx4GemmArgs {
    const uint8_t* xq;
    const uint8_t* x_scale;
    const uint8_t* wq;
    const uint8_t* w_scale;
    const void* bias;         // or null
    void* y;
    int M, N, K;
    const void* x;            // launch_mx4_layer_small: the activations, and their factors or null
    const float* chan_mul;
};
// The kernel that a product takes: tiles of tokens x channels, shared by their wavefronts (vq_mx4_gemm.hip) or with the wavefronts
// dividing K (vq_mx4_gemm_split.hip: 32 x 32, 48 x 48, 32 x 64).
struct Mx4Choice { int tile_t, tile_c; bool divide_k; };
Mx4Choice choose_mx4_gemm(int M, int N, int K, int num_cus);
bool mx4_gemm_takes(int M, int N);      // whether launch_mx4_gemm has a kernel for these sizes
hipError_t launch_mx4_gemm(const Mx4GemmArgs& a, int dtype, int num_cus, hipStream_t stream);
hipError_t launch_mx4_gemm_lines(int tile_t, int tile_c, const Mx4GemmArgs& a, int dtype, hipStream_t stream);
// A layer of few tokens in one launch, from x instead of xq; small_mx4_layer: whether it is the faster way.
bool small_mx4_layer(int M, int N, int K);
hipError_t launch_mx4_layer_small(const Mx4GemmArgs& a, int dtype, hipStream_t stream);

// ---- rotary positions (vq_rotary.hip) and attention (vq_attention.hip) -----------------------------------------
struct RotaryArgs {
    const void* q;
    void* q_out;
    const void* k;
    void* k_out;
    const int32_t* positions;
    const float* inv_freq;
    float amplitude;
    int T, q_heads, k_heads, head_dim, rot_dim;
    int64_t q_token, q_head, qo_token, qo_head, k_token, k_head, ko_token, ko_head;   // strides in elements
    int copied_from, copied, lanes_h;    // the launch's: pieces of a head, and threads that share its heads
};
hipError_t launch_rotary(RotaryArgs a, int dtype, int interleaved, hipStream_t stream);

struct AttentionArgs {
    const void* q;
    const void* k;
    const void* v;
    void* out;
    const int32_t* cu_q;
    const int32_t* cu_k;
    int sequences, Tq, Tk, heads, kv_heads, head_dim, causal;
    int group, group_shift;   // heads / kv_heads, and its logarithm if it is a power of two, else -1
    int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;       // strides in elements
    float scale_log2;         // softmax_scale / ln 2
    float* part_o;            // [splits][Tq * heads][head_dim] and [splits][Tq * heads][2]: sums, maxima and weights
    float* part_ml;
    int split_shift;          // 2^split_shift workgroups divide the keys of a tile
    int tiles;                // the launch's: tiles of query rows (attention_items()) or sequences,
    int items;                // these for every part of their keys,
    int heads_together;       // and whether an item's heads of K and V go to one XCD, or a head's items
};
// Its kernels: tiles of kTileRows query rows (vq_attention_tiles.hip), at most attention_items() of them for a head of K and V, or few rows a
// sequence (vq_attention.hip), by four wavefronts or by one; and how often the keys of a tile are divided among workgroups, from the
// sizes alone.  Tq * heads < 2^31.
enum AttentionKernel { kAttentionTiles = 0, kAttentionRows = 1, kAttentionRowsAlone = 2 };
struct AttentionChoice {
    AttentionKernel kernel;
    int split_shift;          // the logarithm of the workgroups that divide the keys
    bool fits;                // in one launch
};
AttentionChoice choose_attention(int sequences, int Tq, int Tk, int heads, int kv_heads);
hipError_t launch_attention(const AttentionArgs& a, AttentionKernel kernel, int dtype, hipStream_t stream);
constexpr int kTileRows = 128;
inline long attention_items(int sequences, int Tq, int group) { return (long)Tq * group / kTileRows + sequences; }
hipError_t launch_attention_tiles(const AttentionArgs& a, int dtype, hipStream_t stream);

}  // namespace vq

// For the tests, which name the kernels that they mean to reach: choose_gemm, and how the persistent kernel
// writes its rows (Out, vq_gemm_common.h).  Not a part of vq.h.
extern "C" void vq_internal_gemm_choice(int w_bits, int M, int N, int K, int num_cus, int choice[3]);
extern "C" void vq_internal_mx4_choice(int M, int N, int K, int num_cus, int choice[3]);
extern "C" void vq_internal_attention_choice(int sequences, int Tq, int Tk, int heads, int kv_heads, int choice[2]);
extern "C" int vq_internal_gemm_out(int N, const void* y, const void* acc_out);
