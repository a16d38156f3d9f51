// Choice of the kernel for an 8-bit product.
#include "gemm_w8.h"

#include <algorithm>
#include <cmath>

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

// Time of a product in tiles, us: rounds over the workgroups that the card holds at once, by
// what a round takes for its way in and out and for each stage of 128 codes of K, fitted to
// 5302 x 9458 with 256 to 2048 codes, 2000 x 2000 with 256 to 4096, 8192 x 8192 and 256 x 28672
// with 8192.  (64 x 128 tiles wait for memory, 256 x 256 are bound by the matrix cores; two
// shallow 128 x 128 ones a compute unit hide each other's way in and out.  A single round of
// those has other figures.)
struct tile_t {
    int height, width, depth;
    double slots, fixed, stage, fixed_alone, stage_alone;
};
constexpr tile_t kTiles[] = {{64, 128, 4, 256, 3.0, 0.43, 3.0, 0.43},
                             {128, 128, 4, 256, 4.5, 0.57, 4.5, 0.57},
                             {128, 128, 2, 512, 4.8, 1.0, 3.0, 1.2},
                             {128, 256, 3, 256, 8.0, 1.08, 8.0, 1.08},
                             {256, 256, 2, 256, 12.0, 1.55, 12.0, 1.55}};

w8::choice tiles(const tile_t &t) { return {CQ_W8_TILES, t.height, t.width, t.depth}; }

w8::choice dense(const w8::params &p) {
    if (p.rows <= 8) return w8::few_rows_choice(p, false);
    auto cells = [&](int m, int n) { return double((p.rows + m - 1) / m) * double((p.n + n - 1) / n); };
    const double stages = (p.k + 127) / 128;
    const tile_t *best = nullptr;
    double least = 0.0;
    for (const tile_t &t : kTiles) {
        const double rounds = std::ceil(cells(t.height, t.width) / t.slots);
        const double cost = rounds == 1.0 ? t.fixed_alone + stages * t.stage_alone : rounds * (t.fixed + stages * t.stage);
        if (!best || cost < least) {
            best = &t;
            least = cost;
        }
    }
    // Where tiles would leave the card empty, however many rows: K shared out over a
    // workgroup's waves, whose stage is a step of each wave's eighth of K (weights from memory,
    // us: 45 rows of 4096 x 14336 18.6, in tiles 50; 48 of 14336 x 4096 28 and 20; 1300 of 384 x
    // 5872 20.8 and 23).  Up to 16 rows that is the better kernel for all.
    if (p.rows <= 16 || 1.0 + 0.2 * stages * std::max(1.0, cells(32, 32) / 256.0) < least) return w8::rows_choice(p);
    return tiles(*best);
}

w8::choice routed(const w8::params &p) {
    if (p.rows * p.k >= int64_t(1) << 31) return {CQ_W8_TILES_FAR, 128, 128, 2};
    // routes of an expert, were all taken alike
    const double each = double(p.routes) / p.experts;
    if (each <= 5.0) return w8::few_rows_choice(p, true);
    // 128 experts of 2048 x 2048, us: 6 routes each 102 in tiles of 64 x 128 (117 by the few
    // rows' kernel), 37 each 139 (64 x 256: 140), 62 each 161 (150); 64 experts of 4096 x
    // 4096: 62 each 289 (265; 128 x 256: 267), 250 each 468 in 128 x 256 (256 x 256: 488),
    // 500 each 773 (739).
    // With short rows tiles that share a compute unit hide each other's way in and out.
    const bool brief = p.k <= 1024 && each > 80.0;
    const int m = each <= 80.0 ? 64 : each < 400.0 || brief ? 128 : 256, n = each <= 40.0 || brief ? 128 : 256;
    // a tile of each expert is half full, on average
    auto cells = [&](int tm, int tn) {
        return (double(p.routes) / tm + 0.5 * double(std::min<int64_t>(p.experts, p.routes))) * ((p.n + tn - 1) / tn);
    };
    if (cells(m, n) >= 256.0) return {CQ_W8_TILES, m, n, m == 128 && n == 256 ? 3 : 2};
    // few tiles: the deeper ones, 64 or 128 rows high
    const double stages = (p.k + 127) / 128;
    auto cost = [&](const tile_t &t) {
        return std::max(1.0, cells(t.height, t.width) / t.slots) * (t.fixed + stages * t.stage);
    };
    return tiles(cost(kTiles[0]) <= cost(kTiles[1]) ? kTiles[0] : kTiles[1]);
}

w8::choice choose(const w8::params &p, bool with_routes) { return with_routes ? routed(p) : dense(p); }

}  // namespace

bool w8_fits(const cq_w8_args &a, bool routed) {
    // of the smallest of launch_wide's tiles, whose threads along x stay below 2^32
    const int64_t tiles = routed ? w8::most_tiles(a.routes, a.experts, 64) : (a.rows + 63) / 64;
    return tiles < (int64_t(1) << 23) / ((a.n + 127) / 128);
}

int w8_kernel(const cq_w8_args &a, bool with_routes, int32_t *tile) {
    const w8::choice c = choose(make(a, with_routes), with_routes);
    tile[0] = c.height;
    tile[1] = c.width;
    tile[2] = c.depth;
    return c.kind;
}

hipError_t launch_gemm_w8(const cq_w8_args &a, bool with_routes, hipStream_t stream) {
    const w8::params p = make(a, with_routes);
    const w8::choice c = choose(p, with_routes);
    switch (c.kind) {
        case CQ_W8_FEW: return w8::launch_few(p, with_routes, c, stream);
        case CQ_W8_ROWS: return w8::launch_rows(p, c, stream);
        case CQ_W8_TILES: return w8::launch_wide(p, with_routes, c, stream);
    }
    return w8::launch_wide_far(p, stream);
}

}  // namespace cq
