// attn_shared.h for BF16 heads of 128.
#include "attn_shared.h"

namespace cq {

hipError_t attn_shared_bf16_128(const wide_plan &w, const attn_params &flat, const rows_plan &r, const attn_params &own,
                               hipStream_t stream) {
    return attn_shared_dim<0, 128>(w, flat, r, own, stream);
}

}  // namespace cq
