// attn_rows.h for FP16 heads of 256.
#include "attn_rows.h"

namespace cq {

hipError_t attn_rows_fp16_256(const rows_plan &r, const attn_params &p, hipStream_t stream) {
    return attn_rows_dim<1, 256>(r, p, stream);
}

}  // namespace cq
