// attn_wide.h for FP16 heads of 64.
#include "attn_wide.h"

namespace cq {

hipError_t attn_wide_fp16_64(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    return attn_wide_dim<1, 64>(w, p, stream);
}

}  // namespace cq
