// What the offsets of a plan say of an expert's routes.  Offsets are device data that
// nobody has checked, so whatever they hold ends inside the plan.  Plain constexpr C++,
// which the device takes as it is and a host compiler too.
#pragma once

#include <stdint.h>

namespace cq {

// Places first .. first + count - 1 of the routes' order.
struct plan_run {
    int first, count;
};

// The run from one offset to the next, each cut to 0 .. routes before their difference is
// taken: that of two offsets as they are can pass 32 bits and come out positive.
constexpr plan_run run_of(int32_t from, int32_t to, int32_t routes) {
    const int32_t lo = from < 0 ? 0 : from > routes ? routes : from;
    const int32_t hi = to < 0 ? 0 : to > routes ? routes : to;
    return {lo, hi > lo ? hi - lo : 0};
}

// Tiles of `tile` routes that a run takes (routes < 2^31 - tile).
constexpr uint32_t tiles_of(plan_run run, int tile) { return uint32_t(run.count + tile - 1) / uint32_t(tile); }

// Tile n of a run, for n below tiles_of: inside the run.
constexpr plan_run tile_of(plan_run run, uint32_t n, int tile) {
    const int past = int(n) * tile, left = run.count - past;
    return {run.first + past, left < tile ? left : tile};
}

}  // namespace cq
