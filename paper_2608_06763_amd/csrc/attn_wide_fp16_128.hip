// attn_wide.h for FP16 heads of 128.
#include "attn_wide.h"

namespace cq {

hipError_t attn_wide_fp16_128(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    return attn_wide_dim<1, 128>(w, p, stream);
}

}  // namespace cq
