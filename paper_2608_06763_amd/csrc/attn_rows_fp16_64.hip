// attn_rows.h for FP16 heads of 64.
#include "attn_rows.h"

namespace cq {

hipError_t attn_rows_fp16_64(const rows_plan &r, const attn_params &p, hipStream_t stream) {
    return attn_rows_dim<1, 64>(r, p, stream);
}

}  // namespace cq
