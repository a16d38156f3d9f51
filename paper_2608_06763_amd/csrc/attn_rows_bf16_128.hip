// attn_rows.h for BF16 heads of 128.
#include "attn_rows.h"

namespace cq {

hipError_t attn_rows_bf16_128(const rows_plan &r, const attn_params &p, hipStream_t stream) {
    return attn_rows_dim<0, 128>(r, p, stream);
}

}  // namespace cq
