// Choice of the kernel for an 8-bit product.
#include "gemm_w8.h"

namespace cq {

namespace {

w8::params make(const cq_w8_args &a, bool routed) {
    w8::params p = {};
    p.x8 = a.x8;
    p.dx = a.dx;
    p.w8 = a.w8;
    p.dw = a.dw;
    p.bias = a.bias;
    p.y = a.y;
    p.plan = a.plan;
    p.rows = a.rows;
    p.routes = routed ? a.routes : a.rows;
    p.n = int(a.n);
    p.k = int(a.k);
    p.experts = routed ? a.experts : 1;
    p.fan = routed ? a.fan : 1;
    p.y_dt = a.y_dtype;
    if (p.fan > 1) {
        // r / fan exactly for r < 2^31: ceil(2^(32 + s) / fan) with 2^s >= fan / 2
        int s = 0;
        while ((int64_t(2) << s) < p.fan) ++s;
        p.fan_mul = uint32_t(((uint64_t(1) << (32 + s)) + uint64_t(p.fan) - 1) / uint64_t(p.fan));
        p.fan_shift = s;
    }
    return p;
}

}  // namespace

bool w8_fits(const cq_w8_args &a, bool routed) {
    // workgroups of the smallest tiles, 16 rows by 16 channels
    const int64_t most = int64_t(1) << 31;
    const int64_t tiles = routed ? w8::most_tiles(a.routes, a.experts, 16) : (a.rows + 15) / 16;
    return tiles < most / ((a.n + 15) / 16);
}

hipError_t launch_gemm_w8(const cq_w8_args &a, bool routed, hipStream_t stream) {
    const w8::params p = make(a, routed);
    const int64_t rows = routed ? (a.routes + a.experts - 1) / a.experts : a.rows;
    return rows <= 64 ? w8::launch_rows(p, routed, stream) : w8::launch_tile(p, routed, stream);
}

}  // namespace cq
