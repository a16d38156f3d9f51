// 8-bit product of many rows on gfx950 matrix cores.
//
// A workgroup of four waves (2 x 2) owns 64 TM rows of x by 64 TN channels, a wave
// 32 TM by 32 TN of them, whose INT32 sums stay in registers.  A stage is 128 codes of K:
// it goes from memory straight into one of two places in LDS, whole cache lines a row.
// Operands of a slice of 32 codes are read into registers while the slice before is
// multiplied, so that neither the LDS nor the barrier between two stages (one for each)
// holds up the matrix cores; loads are requested a stage before they are waited for.
//
// v_mfma_i32_32x32x32_i8 takes half the operand reads of the 16x16 form for the same work.
// Lane l supplies row l % 32 with codes 16 (l / 32) .. +15 of a slice of 32; chunk c of 16
// codes of row r lies at place c ^ ((r / 2) % 8) of the row's eight, so that sixteen
// neighbouring lanes reach all 64 banks.  The weights are the first operand: lane l holds
// four neighbouring channels 8 g + 4 (l / 32) .. of row l % 32 in each group g of registers.
//
// What bounds it: 256 x 256 tiles the card's power.  8192^3 443 us, 2480 TOP/s (a library's
// product of these integers 2480), the matrix cores busy for 65% of the cycles at 1.77 GHz, no
// bank conflicts; with operands always in the nearest cache 431.  (Cards differ: others take
// 462 to 468 us.)  7013 x 28672 x 8192 1.41 to 1.49 ms, 2210 to 2330 TOP/s.  Routed: 8191 tokens
// of 4 experts of 48, 4096 x 4096, 670 to 706 us, 1560 to 1640 TOP/s, as tiles that an expert's
// last routes fill in part cost whole ones (a path of half the rows for them gave 1%), and as a
// tile's way in and out, by the fit in gemm_w8.hip a fifth of its time with 32 stages, has
// nothing beside it: the tile fills its compute unit.  Small tiles wait for memory: 512 x 4096 x
// 4096 15.5 us with four stages in flight, 21.4 with two.
#pragma once

#include "gemm_w8.h"

namespace cq {

namespace w8 {

typedef int i32x16 __attribute__((ext_vector_type(16)));

constexpr int kStage = 128;  // codes of K

// Scales and biases of the channels 8 g + 4 (l / 32) .. +3 behind n, in the order of the
// sums; past the last channel any.
template <int YDT>
__device__ __forceinline__ void load_channels(const params &p, int expert, int n, float (&dw)[16], float (&bias)[16]) {
    const int half = (threadIdx.x & 63) >> 5;
    const int64_t first = int64_t(expert) * p.n;
    if (n + 32 <= p.n) {
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int64_t c = first + n + 8 * g + 4 * half;
            const float4 d = load4(p.dw, c);
            dw[4 * g] = d.x; dw[4 * g + 1] = d.y; dw[4 * g + 2] = d.z; dw[4 * g + 3] = d.w;
#pragma unroll
            for (int e = 0; e < 4; ++e) bias[4 * g + e] = p.bias ? load_bias<YDT>(p.bias, c + e) : 0.f;
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) {
        const int64_t c = first + min(n + 8 * (e >> 2) + 4 * half + (e & 3), p.n - 1);
        dw[e] = p.dw[c];
        bias[e] = p.bias ? load_bias<YDT>(p.bias, c) : 0.f;
    }
}

// Outputs of a wave's 32 x 32 tile: row `row` in this lane and channels from n on.  Lanes
// l and l + 32 exchange halves of two groups, so that each stores eight neighbours.
template <int YDT>
__device__ __forceinline__ void store_tile(const params &p, const i32x16 &sum, const float (&dw)[16], const float (&bias)[16],
                                           float dx, int64_t row, bool there, int n) {
    const int half = (threadIdx.x & 63) >> 5;
    float v[16];
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = __builtin_fmaf(float(sum[e]), dx * dw[e], bias[e]);
    if (YDT == 2 || n + 32 > p.n) {
        if (!there) return;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            const int at = n + 8 * g + 4 * half;
            if (at < p.n) store4<YDT>(p.y, row * p.n + at, v + 4 * g, min(4, p.n - at));
        }
    } else if constexpr (YDT != 2) {
        uint32_t h[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) h[e] = pack_out<YDT>(v[2 * e], v[2 * e + 1]);
#pragma unroll
        for (int g = 0; g < 4; g += 2) {
            const auto a = __builtin_amdgcn_permlane32_swap(h[2 * g], h[2 * g + 2], false, false);
            const auto b = __builtin_amdgcn_permlane32_swap(h[2 * g + 1], h[2 * g + 3], false, false);
            const uint4 o = make_uint4(a[0], b[0], a[1], b[1]);
            if (there) __builtin_memcpy(static_cast<uint16_t *>(p.y) + row * p.n + n + 8 * (g + half), &o, 16);
        }
    }
}

// NS stages in LDS.  FAR: routed rows of x lie behind 2 GiB.
template <int TM, int TN, int NS, bool ROUTED, bool FAR>
__global__ void __launch_bounds__(256, TM * TN > 4 || NS * (TM + TN) > 10 ? 1 : 2) w8_wide_kernel(params p, int tiles_m, int tiles_n) {
    constexpr int kM = 64 * TM, kN = 64 * TN, NX = kM / 32, NW = kN / 32;
    constexpr int kX = kM * kStage, kW = kN * kStage;
    __shared__ __attribute__((aligned(1024))) uint8_t xs0[kX];
    __shared__ __attribute__((aligned(1024))) uint8_t xs1[kX];
    __shared__ __attribute__((aligned(1024))) uint8_t xs2[NS > 2 ? kX : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t xs3[NS > 3 ? kX : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t ws0[kW];
    __shared__ __attribute__((aligned(1024))) uint8_t ws1[kW];
    __shared__ __attribute__((aligned(1024))) uint8_t ws2[NS > 2 ? kW : 16];
    __shared__ __attribute__((aligned(1024))) uint8_t ws3[NS > 3 ? kW : 16];
    auto xbuf = [&](auto s_c) __attribute__((always_inline)) -> uint8_t * {
        constexpr int S = decltype(s_c)::value % NS;
        if constexpr (S == 0) return xs0;
        else if constexpr (S == 1) return xs1;
        else if constexpr (S == 2) return xs2;
        else return xs3;
    };
    auto wbuf = [&](auto s_c) __attribute__((always_inline)) -> uint8_t * {
        constexpr int S = decltype(s_c)::value % NS;
        if constexpr (S == 0) return ws0;
        else if constexpr (S == 1) return ws1;
        else if constexpr (S == 2) return ws2;
        else return ws3;
    };
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);

    // Those of one XCD (blockIdx modulo 8) take consecutive tiles, which walk kBand row
    // tiles by all channel tiles, so that the tiles that run together share their operands
    // (8192^3: 443 us, 456 in bands of 8; 2000 tokens of 8 experts of 64, 4096 x 4096: 456 us,
    // 478 in bands of 4).
    constexpr int kBand = ROUTED ? 8 : 4;
    const int wg = xcd_tile(tiles_m * tiles_n);
    const int band = wg / (kBand * tiles_n), in_band = wg - band * (kBand * tiles_n);
    const int high = min(kBand, tiles_m - kBand * band);
    const int tile_n = in_band / high, tile_m = kBand * band + (in_band - tile_n * high);
    const int n0 = tile_n * kN;
    place at = {0, 0, 0};
    if constexpr (ROUTED) {
        at = find_tile(p, tile_m, kM);
    } else {
        at.first = tile_m * kM;
        at.count = int(min(p.rows - at.first, int64_t(kM)));
    }
    if (at.count <= 0) return;

    // pieces of 1 KB, 8 rows each: lane l brings place l % 8 of row l / 8
    const int sub = lane >> 3;
    const auto rx = rows_from<ROUTED>(p, at);
    const int8_t *far[FAR ? NX : 1];
    uint32_t xoff[NX], woff[NW];
    const int chunk = 16 * ((lane & 7) ^ (((8 * wave + sub) >> 1) & 7));  // of all its pieces
#pragma unroll
    for (int t = 0; t < NX; ++t) {
        int row = min(8 * (4 * t + wave) + sub, at.count - 1);
        if constexpr (ROUTED) row = row_of(p, max(route_at(p, at.first + row), 0));
        if constexpr (FAR) far[t] = p.x8 + int64_t(row) * p.k;
        xoff[t] = uint32_t(row) * uint32_t(p.k) + uint32_t(chunk);
    }
    // weights behind the last channel and behind a row's end are zeros
    const int channels = min(p.n - n0, kN);
    const auto rw = weights_from(p, at.expert, n0, channels);
#pragma unroll
    for (int t = 0; t < NW; ++t) woff[t] = uint32_t(8 * (4 * t + wave) + sub) * uint32_t(p.k) + uint32_t(chunk);
    const int stages = (p.k + kStage - 1) / kStage;
    // stages behind the last are zeros
    auto load = [&](int st, uint8_t *xb, uint8_t *wb) __attribute__((always_inline)) {
        const int k = kStage * st;
        const bool in = k + chunk < p.k;
#pragma unroll
        for (int t = 0; t < NX; ++t) {
            uint8_t *to = xb + 1024 * (4 * t + wave);
            if constexpr (FAR) {
                __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)(far[t] + (in ? k + chunk : 0)),
                                                 (__attribute__((address_space(3))) void *)to, 16, 0, 0);
            } else {
                load_lds16(rx, to, in ? xoff[t] + uint32_t(k) : kOobOffset);
            }
        }
#pragma unroll
        for (int t = 0; t < NW; ++t) load_lds16(rw, wb + 1024 * (4 * t + wave), in ? woff[t] + uint32_t(k) : kOobOffset);
    };

    const int wm = wave >> 1, wn = wave & 1;
    // place of chunk 2 s + l / 32 of row l % 32: (2 s) ^ own
    const int own = (lane >> 5) ^ ((lane >> 1) & 7);
    const uint32_t xrow = uint32_t(32 * TM * wm + (lane & 31)) * kStage, wrow = uint32_t(32 * TN * wn + (lane & 31)) * kStage;
    struct slice_t {
        i32x4 x[TM], w[TN];
    };
    auto read = [&](auto s_c, const uint8_t *xb, const uint8_t *wb, slice_t &o) __attribute__((always_inline)) {
        constexpr int S = decltype(s_c)::value;
        const uint32_t c = 16u * uint32_t((2 * S) ^ own);
        unroll<0, TM>([&](auto i_c) __attribute__((always_inline)) {
            constexpr int I = decltype(i_c)::value;
            o.x[I] = *reinterpret_cast<const i32x4 *>(xb + xrow + 32 * kStage * I + c);
        });
        unroll<0, TN>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int J = decltype(j_c)::value;
            o.w[J] = *reinterpret_cast<const i32x4 *>(wb + wrow + 32 * kStage * J + c);
        });
    };
    i32x16 sum[TM][TN] = {};
    auto multiply = [&](const slice_t &o) __attribute__((always_inline)) {
        unroll<0, TM * TN>([&](auto t_c) __attribute__((always_inline)) {
            constexpr int I = decltype(t_c)::value / TN, J = decltype(t_c)::value % TN;
            sum[I][J] = __builtin_amdgcn_mfma_i32_32x32x32_i8(o.w[J], o.x[I], sum[I][J], 0, 0, 0);
        });
    };
    // reads (and loads) one beside each product, as far as they go
    auto weave = [&](auto l_c) __attribute__((always_inline)) {
        constexpr int L = decltype(l_c)::value;
        unroll<0, TM * TN>([&](auto t_c) __attribute__((always_inline)) {
            constexpr int T = decltype(t_c)::value;
            if constexpr (T < TM + TN) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            if constexpr (T < L) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        });
        __builtin_amdgcn_sched_barrier(0);
    };

    slice_t a, b;
    using S0 = std::integral_constant<int, 0>;
    using S1 = std::integral_constant<int, 1>;
    using S2 = std::integral_constant<int, 2>;
    using S3 = std::integral_constant<int, 3>;
    using none = std::integral_constant<int, 0>;
    // Stage st in buffer S, its first slice in a.
    auto do_stage = [&](int st, auto s_c) __attribute__((always_inline)) {
        constexpr int S = decltype(s_c)::value;
        uint8_t *xb = xbuf(s_c), *wb = wbuf(s_c);
        using next = std::integral_constant<int, S + 1>;
        read(S1{}, xb, wb, b);
        multiply(a);
        weave(none{});
        read(S2{}, xb, wb, a);
        multiply(b);
        weave(none{});
        read(S3{}, xb, wb, b);
        multiply(a);
        weave(none{});
        // the next stage has landed, and every wave has read all of this one
        wait_loads<(NS - 2) * (NX + NW)>();
        __builtin_amdgcn_s_barrier();
        vmem_order();
        load(st + NS, xb, wb);
        read(S0{}, xbuf(next{}), wbuf(next{}), a);
        multiply(b);
        weave(std::integral_constant<int, NX + NW>{});
        vmem_order();
    };
    unroll<0, NS>([&](auto s_c) __attribute__((always_inline)) { load(decltype(s_c)::value, xbuf(s_c), wbuf(s_c)); });
    wait_loads<(NS - 1) * (NX + NW)>();
    __builtin_amdgcn_s_barrier();
    vmem_order();
    read(S0{}, xs0, ws0, a);
    // As many stages a turn as there are buffers, with one way out of the loop (with more,
    // 256 x 256 sums find no registers to meet in); the last turn may end in zeros.
    for (int st = 0; st < stages; st += NS)
        unroll<0, NS>([&](auto s_c) __attribute__((always_inline)) { do_stage(st + decltype(s_c)::value, s_c); });
    wait_loads<0>();

    float dx[TM];
    int64_t out[TM];
    bool there[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const int m = 32 * (TM * wm + i) + (lane & 31);
        there[i] = m < at.count;
        int row = at.first + min(m, at.count - 1);
        out[i] = row;
        if constexpr (ROUTED) {
            out[i] = route_at(p, row);
            there[i] = there[i] && out[i] >= 0;
            row = row_of(p, max(int(out[i]), 0));
        }
        dx[i] = p.dx[row];
    }
    auto finish = [&](auto y_c) __attribute__((always_inline)) {
        constexpr int YDT = decltype(y_c)::value;
        unroll<0, TN>([&](auto j_c) __attribute__((always_inline)) {
            constexpr int J = decltype(j_c)::value;
            const int n = n0 + 32 * (TN * wn + J);
            if (n >= p.n) return;
            float dw[16], bias[16];
            load_channels<YDT>(p, at.expert, n, dw, bias);
            unroll<0, TM>([&](auto i_c) __attribute__((always_inline)) {
                constexpr int I = decltype(i_c)::value;
                // the sums stay in accumulation registers up to here: without this they are
                // all moved out at once behind the loop, and what lives across it is spilled
                i32x16 &t = sum[I][J];
                __asm__ volatile("" : "+a"(t));
                store_tile<YDT>(p, t, dw, bias, dx[I], out[I], there[I], n);
                __builtin_amdgcn_sched_barrier(0);
            });
        });
    };
    if (p.y_dt == 0) finish(std::integral_constant<int, 0>{});
    else if (p.y_dt == 1) finish(std::integral_constant<int, 1>{});
    else finish(std::integral_constant<int, 2>{});
}

template <int TM, int TN, int NS, bool ROUTED, bool FAR = false>
hipError_t wide_run(const params &p, hipStream_t stream) {
    const int64_t tiles_n = (p.n + 64 * TN - 1) / (64 * TN);
    const int64_t tiles_m = ROUTED ? most_tiles(p.routes, p.experts, 64 * TM) : (p.rows + 64 * TM - 1) / (64 * TM);
    hipLaunchKernelGGL((w8_wide_kernel<TM, TN, NS, ROUTED, FAR>), dim3(uint32_t(tiles_m * tiles_n)), dim3(256), 0, stream, p,
                       int(tiles_m), int(tiles_n));
    return hipGetLastError();
}

}  // namespace w8

}  // namespace cq
