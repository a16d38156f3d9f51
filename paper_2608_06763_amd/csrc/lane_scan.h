// Running sums over the lanes of a wavefront.
#pragma once

#include "cq_device.h"

namespace cq {

// Sum of the lanes up to this one (modulo 2^32), all lanes active: shifts inside rows of
// sixteen, then the last lane of a row to the next row, and of the first half to the second.
__device__ __forceinline__ uint32_t wave_scan(uint32_t v) {
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x111, 0xf, 0xf, false));  // row_shr 1, 2, 4, 8
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x112, 0xf, 0xf, false));
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x114, 0xf, 0xf, false));
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x118, 0xf, 0xf, false));
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x142, 0xa, 0xf, false));  // row_bcast 15 to rows 1 and 3
    v += uint32_t(__builtin_amdgcn_update_dpp(0, int(v), 0x143, 0xc, 0xf, false));  // row_bcast 31 to rows 2 and 3
    return v;
}

}  // namespace cq
