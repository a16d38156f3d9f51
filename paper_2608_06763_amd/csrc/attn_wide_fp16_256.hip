// attn_wide_256.h for FP16 heads of 256.
#include "attn_wide_256.h"

namespace cq {

hipError_t attn_wide_fp16_256(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    return attn_wide_256_dim<1>(w, p, stream);
}

}  // namespace cq
