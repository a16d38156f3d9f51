// attn_shared.h for FP16 heads of 256.
#include "attn_shared.h"

namespace cq {

hipError_t attn_shared_fp16_256(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                               hipStream_t stream) {
    return attn_shared_dim<1, 256>(w, flat, r, own, stream);
}

}  // namespace cq
