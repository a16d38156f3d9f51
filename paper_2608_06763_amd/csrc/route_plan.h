// Routes in the order of their experts: a stable counting sort, so that the order is
// the map's alone.
//
// Routes are counted by expert in rows of a table, one row for each run of them.  A
// workgroup places the routes of a few neighbouring rows: its first place in each expert
// is what the rows before hold, each of its waves comes behind the waves before, and a
// wave takes 64 routes at a time, whose lanes of one expert find each other by ballots
// over the expert's bits.
#pragma once

#include "cq_device.h"
#include "experts_internal.h"
#include "lane_scan.h"

namespace cq {

constexpr int kPlanWaves = 8, kPlanThreads = kPlanWaves * kWave;
constexpr int kPlanExperts = 1024;  // most

// Rows that a placing workgroup adds up by itself.  Above it a launch of its own turns
// the table into sums first, since the adding grows with the square of the rows.
constexpr int kPlanRows = 512;

struct plan_params {
    int32_t *plan;
    int32_t *table;   // [rows + 1, experts]: counts; above kPlanRows, what the rows before hold
    int64_t routes;
    int row;          // routes of a row
    int rows, group;  // rows of the table; of a placing workgroup
    int experts, bits;
};

inline int plan_bits(int experts) {  // of 0 .. experts
    int bits = 0;
    while ((experts >> bits) != 0) ++bits;
    return bits;
}

// LDS of a placing workgroup: the waves' places (to whole 16 bytes), sums of threads,
// and sums of slices of the table, 8 for each thread at most.
__host__ __device__ inline int plan_pitch(int experts) { return (kPlanWaves * (experts + 1) + 3) & ~3; }
inline size_t plan_lds(int experts, bool alone) {
    return sizeof(int) * (size_t(plan_pitch(experts)) + (alone ? 1 : 9) * kPlanThreads);
}

// Lanes of the wave that hold the same value as this one (of `bits` bits).
__device__ __forceinline__ uint64_t same_value(int v, int bits) {
    uint64_t same = __ballot(1);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((v >> b) & 1);
        same &= (v >> b) & 1 ? set : ~set;
    }
    return same;
}

__device__ __forceinline__ int plan_bucket(int e, int experts) {
    return uint32_t(e) < uint32_t(experts) ? e : experts;
}

// Places of the routes first .. first + count - 1 of the map; expert_of(i) is the expert of
// route first + i, or `experts`.  ALONE: there are no other routes, and no table.
template <bool ALONE, typename F>
__device__ __forceinline__ void plan_place(const plan_params &p, int block, int64_t first, int count, int *lds, F expert_of) {
    int *place = lds;  // [wave][expert]: the wave's routes, then the expert's next place
    int *part = lds + plan_pitch(p.experts);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pitch = p.experts + 1;
    // a wave's routes are neighbours
    const int share = ((count + kPlanThreads - 1) / kPlanThreads) * kWave, begin = wave * share;
    const int end = min(begin + share, count);
    for (int i = tid; i < kPlanWaves * pitch; i += kPlanThreads) place[i] = 0;
    // the first routes of a lane stay in registers, asked for together
    constexpr int kKeep = 8;
    int keep[kKeep];
#pragma unroll
    for (int n = 0; n < kKeep; ++n) keep[n] = begin + n * kWave + lane < end ? expert_of(begin + n * kWave + lane) : p.experts;
    // Routes of the rows before this workgroup's, and of all rows, by expert: asked for
    // before the workgroup's own are counted.
    constexpr int kPer = kPlanExperts / kPlanThreads;
    const int per = (p.experts + kPlanThreads - 1) / kPlanThreads;
    int before[kPer] = {}, all[kPer] = {};
    const int row0 = block * p.group;
    int *sums = part + kPlanThreads;  // of slices of the table: [2][slices][experts]
    int slices = 0;
    if constexpr (!ALONE) {
        if (p.rows > kPlanRows) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = tid * per + i;
                if (i >= per || e >= p.experts) continue;
                before[i] = p.table[int64_t(row0) * p.experts + e];
                all[i] = p.table[int64_t(p.rows) * p.experts + e];
            }
        } else if (p.experts % 4 == 0) {
            // four experts a thread, of a slice of neighbouring rows; the slices' sums meet in
            // LDS.  Most slices lie whole before this workgroup's rows, or behind.
            const int quads = p.experts / 4;
            slices = min(kPlanThreads / quads, 16);
            const int s = tid / quads, e = 4 * (tid - s * quads), each = (p.rows + slices - 1) / slices;
            int4 some = make_int4(0, 0, 0, 0), early = some;
            auto add = [](int4 &to, const int4 &c) {
                to.x += c.x; to.y += c.y; to.z += c.z; to.w += c.w;
            };
            const int end_row = s < slices ? min((s + 1) * each, p.rows) : 0;
            constexpr int kTurn = 32;
            for (int b0 = s * each; b0 < end_row; b0 += kTurn) {
                const int32_t *from = p.table + b0 * p.experts + e;
                int4 c[kTurn];
#pragma unroll
                for (int i = 0; i < kTurn; ++i) {
                    c[i] = make_int4(0, 0, 0, 0);
                    if (b0 + i < end_row) c[i] = *reinterpret_cast<const int4 *>(from);
                    from += p.experts;
                }
                if (b0 < row0 && row0 < b0 + kTurn) {
#pragma unroll
                    for (int i = 0; i < kTurn; ++i)
                        if (b0 + i < row0) add(early, c[i]);
                }
                int4 turn = make_int4(0, 0, 0, 0);
#pragma unroll
                for (int i = 0; i < kTurn; ++i) add(turn, c[i]);
                add(some, turn);
                if (b0 + kTurn <= row0) add(early, turn);
            }
            if (s < slices) {
                *reinterpret_cast<int4 *>(sums + s * p.experts + e) = some;
                *reinterpret_cast<int4 *>(sums + (slices + s) * p.experts + e) = early;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = tid * per + i;
                if (i >= per || e >= p.experts) continue;
#pragma unroll 16
                for (int b = 0; b < p.rows; ++b) {
                    const int c = p.table[b * p.experts + e];
                    all[i] += c;
                    before[i] += b < row0 ? c : 0;
                }
            }
        }
    }
    __syncthreads();
#pragma unroll
    for (int n = 0; n < kKeep; ++n)
        if (begin + n * kWave + lane < end) atomicAdd(&place[wave * pitch + keep[n]], 1);
    for (int i = begin + kKeep * kWave + lane; i < end; i += kWave) atomicAdd(&place[wave * pitch + expert_of(i)], 1);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = tid * per + i;
        if (i >= per || e >= p.experts) continue;
        for (int s = 0; s < slices; ++s) {
            all[i] += sums[s * p.experts + e];
            before[i] += sums[(slices + s) * p.experts + e];
        }
    }
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = tid * per + i;
        if (i >= per || e >= p.experts) continue;
        if constexpr (ALONE) {
#pragma unroll
            for (int w = 0; w < kPlanWaves; ++w) all[i] += place[w * pitch + e];
        }
        sum += all[i];
    }
    // offsets of the experts: sums over the lanes of a wave, then over the waves
    const int upto = int(wave_scan(uint32_t(sum)));
    if (lane == 63) part[wave] = upto;
    __syncthreads();
    int at = upto - sum, total = 0;
#pragma unroll
    for (int w = 0; w < kPlanWaves; ++w) {
        const int v = part[w];
        at += w < wave ? v : 0;
        total += v;
    }
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int e = tid * per + i;
        if (i >= per || e >= p.experts) continue;
        if (block == 0) p.plan[e] = at;
        int to = at + before[i];
#pragma unroll
        for (int w = 0; w < kPlanWaves; ++w) {
            const int c = place[w * pitch + e];
            place[w * pitch + e] = to;
            to += c;
        }
        at += all[i];
    }
    if (block == 0 && tid == 0) p.plan[p.experts] = total;
    __syncthreads();
    int32_t *order = p.plan + p.experts + 1;
    auto put = [&](int i, int e) __attribute__((always_inline)) {
        const uint64_t same = same_value(e, p.bits);
        const int rank = __builtin_popcountll(same & ((uint64_t(1) << lane) - 1));
        const int to = place[wave * pitch + e] + rank;
        if (e < p.experts) order[to] = int32_t(first + i);
        // every lane has read its place before the first of its expert moves it on
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (rank == 0) place[wave * pitch + e] = to + __builtin_popcountll(same);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        // behind the routes that have a place
        if (i < end && first + i >= total) order[first + i] = -1;
    };
#pragma unroll
    for (int n = 0; n < kKeep; ++n)
        if (begin + n * kWave < end) put(begin + n * kWave + lane, keep[n]);
    for (int base = begin + kKeep * kWave; base < end; base += kWave)
        put(base + lane, base + lane < end ? expert_of(base + lane) : p.experts);
}

// Bytes of the table of counts.
inline int64_t plan_table_bytes(int64_t rows, int experts) { return (rows + 1) * experts * 4; }

// Placing of counted routes; p.group is set here.
hipError_t launch_plan_place(plan_params p, const int32_t *chosen, hipStream_t stream);

}  // namespace cq
