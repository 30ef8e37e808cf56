// Attention whose wavefronts share the keys: 128 query rows a workgroup, 32 a wavefront, tiles of 64 keys.
//
// Bound by the sum of matrix and vector time: a wavefront's exponentials and its products do not overlap much, and the clock falls under
// both (2 x 4096, 16 heads of 72: matrix units busy 48 % of the cycles at 1.8 GHz; causal prompts of up to 8192, heads of 128: 53 % at 1.7 GHz; no
// LDS conflicts to speak of).  Measured (captured, inputs that are not in the caches): 4 x 4096, 16 heads of 128 524 us (1048 TFLOP/s), heads of
// 64 322 (853); 2 x 4096, 16 heads of 72 207 (747; its heads' last block of 32 channels is a fourth full); 256 rows a workgroup are slower.
// With few keys bound by the way of the first loads: 2 x 16384 queries on 120 keys 57 us, 2.6 TB/s of 151 MB (50 us on a chip that has been busy
// for a second: the clock dips when work begins).
#include "vq_attention_tiles_kernel.h"

namespace vq {

hipError_t launch_attention_tiles(const AttentionArgs& a, int dtype, hipStream_t stream) {
    return dtype == VQ_F16 ? launch_tiles<F16>(a, stream) : launch_tiles<BF16>(a, stream);
}

}  // namespace vq
