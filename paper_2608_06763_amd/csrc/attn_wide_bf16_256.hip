// attn_wide.h for BF16 heads of 256.
#include "attn_wide.h"

namespace cq {

hipError_t attn_wide_bf16_256(const wide_plan &w, const attn_params &p, hipStream_t stream) {
    return attn_wide_dim<0, 256>(w, p, stream);
}

}  // namespace cq
