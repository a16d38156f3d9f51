// Attention over a paged cache: which kernels a call runs, and where its parts
// lie in the workspace.
#include "attn_common.h"

#include <cmath>

namespace cq {

namespace {

// The rows kernel for `sequences` of at most `rows` rows and `tokens` tokens.
rows_plan plan_rows(int dim, int64_t sequences, int kv_heads, int64_t rows, int64_t tokens, bool keep, bool beside) {
    rows_plan r;
    r.nt = rows <= 16 ? 1 : 2;
    r.numbers = sequences * kv_heads;
    const int64_t units = tokens > 32 ? (tokens + 31) / 32 : 1;
    // workgroups that LDS and registers let run at once
    const int64_t most = int64_t(device_cu_count()) * (dim == 256 || beside ? 1 : 2);
    // Up to 1024 tokens one workgroup takes a row tile whole: 800 tokens 12.6 us,
    // 15.3 split and joined (2000 tokens 22.4 and 16.1).  Up to 2048 where the tiles
    // alone fill the chip: 90 sequences of up to 1200 tokens 3 us less.
    r.split = units > (r.numbers >= most ? 64 : 32);
    const int64_t need = (r.numbers * units + kRunUnits - 1) / kRunUnits;
    r.grid = int(r.split ? (need < most ? need : most) : r.numbers);
    r.slots = (r.split ? 2 * int64_t(r.grid) : 0) + (keep ? r.numbers : 0);
    return r;
}

// The wide kernel: at most `tiles` row tiles in all, few of which leave compute
// units idle unless their tokens are split.
wide_plan plan_wide(int64_t sequences, int kv_heads, int64_t rows, int64_t all_rows, int64_t tokens, bool keep,
                    bool beside) {
    wide_plan w;
    w.tiles = all_rows / 128 + sequences;
    const int64_t most = sequences * ((rows + 127) / 128);
    if (w.tiles > most) w.tiles = most;
    // Splitting n tiles of 64 tokens s ways takes 1.1 us n (1 - 1 / s) off a workgroup
    // and costs, for each part, the round trip of its rows through the workspace
    // (0.35 ns a row and 0.1 us), and 5 us of the join's launch where none runs
    // anyway.  With 8192 rows and 8 tiles a split of 2 took 22 us against 18 without;
    // 256 rows of 4 key heads over 16000 tokens took 30 us split 31 ways, 38 split 62.
    const int64_t groups = w.tiles * kv_heads, cus = device_cu_count();
    const double n = double(tokens) / 64, part = 0.1 + 0.00035 * double(all_rows) * kv_heads;
    int64_t splits = int64_t(std::sqrt(1.1 * n / part) + 0.5);
    const int64_t slots = beside ? cus : 2 * cus;
    if (splits > slots / groups) splits = slots / groups;
    if (splits < 2 || groups >= cus || 1.1 * n * (1.0 - 1.0 / splits) < (keep ? 0.0 : 5.0) + part * splits) splits = 1;
    w.splits = int(splits > 64 ? 64 : splits);
    w.part_rows = w.splits > 1 || keep ? w.splits * all_rows * kv_heads : 0;
    return w;
}

constexpr int64_t kRowsMost = 32;  // rows of a sequence that the rows kernel takes

// One pass over tokens: by the rows kernel, or by the wide one.
struct pass_plan {
    bool wide, keep;
    rows_plan rows;
    wide_plan tall;
    int64_t o, ml, shares;  // bytes of the workspace
    int64_t bytes() const { return o + ml + shares; }
};

pass_plan plan_pass(bool wide, int dim, int64_t sequences, int kv_heads, int64_t rows, int64_t all_rows, int64_t tokens,
                    bool keep, bool beside) {
    pass_plan t;
    t.keep = keep;
    t.wide = wide;
    int64_t part_rows = 0;
    t.shares = 0;
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    if (t.wide) {
        t.tall = plan_wide(sequences, kv_heads, rows, all_rows, tokens, keep, beside);
        part_rows = t.tall.part_rows;
    } else {
        t.rows = plan_rows(dim, sequences, kv_heads, rows, tokens, keep, beside);
        if (t.rows.split || keep) {
            part_rows = t.rows.slots * 16 * t.rows.nt;
            t.shares = up(t.rows.numbers * int64_t(sizeof(int2)));
        }
    }
    t.o = up(part_rows * dim * 4);
    t.ml = up(part_rows * 8);
    return t;
}

// Points a pass's parts at `ws`, and the join at them.
join_source place(const pass_plan &t, attn_params &p, uint8_t *ws) {
    join_source join = {};
    join.o = p.part_o = reinterpret_cast<float *>(ws);
    join.ml = p.part_ml = reinterpret_cast<float *>(ws + t.o);
    p.keep_parts = t.keep;
    if (t.wide) {
        join.splits = t.tall.part_rows ? t.tall.splits : 0;
        return join;
    }
    p.shares = t.shares ? reinterpret_cast<int2 *>(ws + t.o + t.ml) : nullptr;
    join.shares = p.shares;
    join.rows = t.shares ? 16 * t.rows.nt : 0;
    join.grid = t.rows.grid;
    join.first = !t.keep ? -1 : t.rows.split ? 2 * int64_t(t.rows.grid) : 0;
    return join;
}

int dim_index(int dim) { return dim == 64 ? 0 : dim == 128 ? 1 : 2; }

hipError_t launch_pass(int dt, int dim, const pass_plan &t, const attn_params &p, hipStream_t stream) {
    typedef hipError_t (*rows_fn)(const rows_plan &, const attn_params &, hipStream_t);
    typedef hipError_t (*wide_fn)(const wide_plan &, const attn_params &, hipStream_t);
    static constexpr rows_fn rows_of[2][3] = {{attn_rows_bf16_64, attn_rows_bf16_128, attn_rows_bf16_256},
                                              {attn_rows_fp16_64, attn_rows_fp16_128, attn_rows_fp16_256}};
    static constexpr wide_fn wide_of[2][3] = {{attn_wide_bf16_64, attn_wide_bf16_128, attn_wide_bf16_256},
                                              {attn_wide_fp16_64, attn_wide_fp16_128, attn_wide_fp16_256}};
    const int d = dim_index(dim);
    return t.wide ? wide_of[dt][d](t.tall, p, stream) : rows_of[dt][d](t.rows, p, stream);
}

hipError_t launch_both(int dt, int dim, const pass_plan &f, const attn_params &flat, const pass_plan &o,
                       const attn_params &own, hipStream_t stream) {
    typedef hipError_t (*fn)(const wide_plan &, const attn_params &, const rows_plan &, const attn_params &,
                             hipStream_t);
    static constexpr fn of[2][3] = {{attn_shared_bf16_64, attn_shared_bf16_128, attn_shared_bf16_256},
                                    {attn_shared_fp16_64, attn_shared_fp16_128, attn_shared_fp16_256}};
    return of[dt][dim_index(dim)](f.tall, flat, o.rows, own, stream);
}

struct plan_t {
    pass_plan own, flat;
    bool shared, together;
    int64_t max_kv, flat_bytes;
};

plan_t make_plan(const cq_kv_cache &c, const cq_attn_args &a) {
    plan_t t;
    const int64_t group = a.heads / c.kv_heads, held = int64_t(a.table_width) * c.page;
    t.max_kv = a.max_kv < held ? a.max_kv : held;
    t.shared = a.prefix_len > 0;
    const int64_t rows = a.tokens * group;
    const bool wide = a.max_q * group > kRowsMost;
    // The prefix always takes the wide kernel, which with few rows is bound by memory
    // too; where the own tokens take the rows kernel both go in one launch: 2 to 8
    // sequences behind 1500 tokens took 24-28 us with two launches of the rows kernel,
    // 16 so.
    t.together = t.shared && !wide;
    t.own = plan_pass(wide, c.dim, a.batch, c.kv_heads, a.max_q * group, rows, t.max_kv, t.shared, t.together);
    t.flat_bytes = 0;
    if (t.shared) {
        t.flat = plan_pass(true, c.dim, 1, c.kv_heads, rows, rows, a.prefix_len, true, t.together);
        t.flat_bytes = t.flat.bytes();
    }
    return t;
}

}  // namespace

bool attn_fits(const cq_kv_cache &c, const cq_attn_args &a) {
    const plan_t t = make_plan(c, a);
    const auto groups = [&](const pass_plan &p) {
        return p.wide ? p.tall.tiles * c.kv_heads * (t.together ? p.tall.splits : 1) : p.rows.grid;
    };
    constexpr int64_t kMost = int64_t(1) << 24;  // of 256 threads, which a launch counts in 32 bits
    const int64_t own = groups(t.own), flat = t.shared ? groups(t.flat) : 0;
    return t.together ? own + flat < kMost : own < kMost && flat < kMost;
}

int64_t attn_workspace_bytes(const cq_kv_cache &c, const cq_attn_args &a) {
    const plan_t t = make_plan(c, a);
    return t.own.bytes() + t.flat_bytes;
}

hipError_t launch_attn(const cq_kv_cache &c, const cq_attn_args &a, void *workspace, hipStream_t stream) {
    const plan_t t = make_plan(c, a);
    attn_params p = {};
    p.q = static_cast<const uint16_t *>(a.q);
    p.k = static_cast<const uint16_t *>(c.k);
    p.v = static_cast<const uint16_t *>(c.v);
    p.out = static_cast<uint16_t *>(a.out);
    p.q_stride = a.q_stride;
    p.tokens = a.tokens;
    p.heads = a.heads;
    p.kv_heads = c.kv_heads;
    p.group = a.heads / c.kv_heads;
    p.batch = a.batch;
    p.q_starts = a.q_starts;
    p.tables = a.tables;
    p.kv_lens = a.kv_lens;
    p.bidir = a.bidir;
    p.slopes = a.slopes;
    p.table_width = a.table_width;
    p.max_kv = int(t.max_kv);
    p.max_q = a.max_q;
    p.page_shift = __builtin_ctz(unsigned(c.page));
    p.pages = uint32_t(c.pages);
    p.window = a.window < t.max_kv ? a.window : 0;  // a longer one hides nothing
    p.scale = a.scale;
    p.softcap = a.softcap;
    if (a.softcap > 0.f) {
        // finite for the smallest caps, so that a score of 0 stays one
        const float rate = (a.softcap <= kNearCap ? 2.f * kLog2e : 1.f) * a.scale / a.softcap;
        p.cap_rate = rate < 3.0e38f ? rate : 3.0e38f;
    }

    uint8_t *ws = static_cast<uint8_t *>(workspace);
    const int dt = int(c.dtype);
    join_source flat = {};
    const join_source own = place(t.own, p, ws);
    hipError_t e;
    if (t.shared) {
        attn_params f = p;
        f.flat = 1;
        f.flat_len = int(a.prefix_len);
        f.tables = a.prefix_table;
        f.kv_lens = f.q_starts = nullptr;
        f.batch = 1;
        f.max_q = int(a.tokens);
        f.shares = nullptr;
        flat = place(t.flat, f, ws + t.own.bytes());
        if (t.together) {
            e = launch_both(dt, c.dim, t.flat, f, t.own, p, stream);
        } else {
            e = launch_pass(dt, c.dim, t.flat, f, stream);
            if (e == hipSuccess) e = launch_pass(dt, c.dim, t.own, p, stream);
        }
    } else {
        e = launch_pass(dt, c.dim, t.own, p, stream);
    }
    if (e != hipSuccess || (!own.rows && !own.splits)) return e;
    return launch_attn_join(dt, c.dim, p, own, flat, p.tokens * p.heads >= 4096, stream);
}

}  // namespace cq
