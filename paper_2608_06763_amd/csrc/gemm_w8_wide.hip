// 8-bit product of many rows: the tiles (gemm_w8_wide.h).
#include "gemm_w8_wide.h"

namespace cq {

namespace w8 {

hipError_t launch_wide(const params &p, bool routed, const choice &c, hipStream_t stream) {
    if (c.height == 256) return routed ? wide_run<4, 4, 2, true>(p, stream) : wide_run<4, 4, 2, false>(p, stream);
    if (c.height == 128 && c.width == 256) return routed ? wide_run<2, 4, 3, true>(p, stream) : wide_run<2, 4, 3, false>(p, stream);
    if (c.height == 128 && c.depth == 4) return routed ? wide_run<2, 2, 4, true>(p, stream) : wide_run<2, 2, 4, false>(p, stream);
    if (c.height == 128) return routed ? wide_run<2, 2, 2, true>(p, stream) : wide_run<2, 2, 2, false>(p, stream);
    if (!routed) return wide_run<1, 2, 4, false>(p, stream);
    if (c.depth == 4) return wide_run<1, 2, 4, true>(p, stream);
    return c.width == 256 ? wide_run<1, 4, 2, true>(p, stream) : wide_run<1, 2, 2, true>(p, stream);
}

hipError_t launch_wide_far(const params &p, hipStream_t stream) { return wide_run<2, 2, 2, true, true>(p, stream); }

}  // namespace w8

}  // namespace cq
