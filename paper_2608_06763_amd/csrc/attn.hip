// Attention over a paged cache: which kernels a call runs, and where its parts
// lie in the workspace.
#include "attn_common.h"

namespace cq {

namespace {

// The rows kernel for `sequences` of at most `rows` rows and `tokens` tokens.
rows_plan plan_rows(int dim, int64_t sequences, int kv_heads, int64_t rows, int64_t tokens, bool keep) {
    rows_plan r;
    r.nt = rows <= 16 ? 1 : rows <= 32 || dim == 256 ? 2 : 4;
    r.row_tiles = int((rows + 16 * r.nt - 1) / (16 * r.nt));
    r.numbers = sequences * kv_heads * r.row_tiles;
    const int64_t units = tokens > 32 ? (tokens + 31) / 32 : 1;
    r.min_units = 4;
    r.split = units > 8;
    // workgroups that LDS and registers let run at once
    const int64_t most = int64_t(device_cu_count()) * (dim == 256 || r.nt == 4 ? 1 : 2);
    const int64_t need = (r.numbers * units + r.min_units - 1) / r.min_units;
    r.grid = int(r.split ? (need < most ? need : most) : r.numbers);
    r.slots = (r.split ? 2 * int64_t(r.grid) : 0) + (keep ? r.numbers : 0);
    return r;
}

struct source_bytes {
    int64_t o, ml, shares;
    int64_t all() const { return o + ml + shares; }
};
source_bytes bytes_of(const rows_plan &r, int dim, bool keep) {
    const auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
    if (!r.split && !keep) return {0, 0, 0};
    const int64_t rows = r.slots * 16 * r.nt;
    return {up(rows * dim * 4), up(rows * 8), up(r.numbers * int64_t(sizeof(int2)))};
}

// Points a launch's parts at `ws`, and the join at them.
join_source place(attn_params &p, const rows_plan &r, const source_bytes &n, bool keep, uint8_t *ws) {
    p.part_o = reinterpret_cast<float *>(ws);
    p.part_ml = reinterpret_cast<float *>(ws + n.o);
    p.shares = n.shares ? reinterpret_cast<int2 *>(ws + n.o + n.ml) : nullptr;
    p.row_tiles = r.row_tiles;
    p.min_units = r.min_units;
    p.keep_parts = keep;
    join_source j = {p.part_o, p.part_ml, p.shares, n.shares ? 16 * r.nt : 0, r.row_tiles, r.grid, 0, -1};
    if (keep) j.first = r.split ? 2 * int64_t(r.grid) : 0;
    return j;
}

hipError_t launch_rows(int dt, int dim, const rows_plan &r, const attn_params &p, hipStream_t stream) {
    if (dt == 0) {
        if (dim == 64) return attn_rows_bf16_64(r, p, stream);
        return dim == 128 ? attn_rows_bf16_128(r, p, stream) : attn_rows_bf16_256(r, p, stream);
    }
    if (dim == 64) return attn_rows_fp16_64(r, p, stream);
    return dim == 128 ? attn_rows_fp16_128(r, p, stream) : attn_rows_fp16_256(r, p, stream);
}

struct plan_t {
    rows_plan own, flat;
    source_bytes own_bytes, flat_bytes;
    bool shared;
    int64_t max_kv;
};

plan_t make_plan(const cq_kv_cache &c, const cq_attn_args &a) {
    plan_t t;
    const int64_t group = a.heads / c.kv_heads, held = int64_t(a.table_width) * c.page;
    t.max_kv = a.max_kv < held ? a.max_kv : held;
    t.shared = a.prefix_len > 0;
    t.own = plan_rows(c.dim, a.batch, c.kv_heads, a.max_q * group, t.max_kv, t.shared);
    t.own_bytes = bytes_of(t.own, c.dim, t.shared);
    t.flat_bytes = {0, 0, 0};
    if (t.shared) {
        t.flat = plan_rows(c.dim, 1, c.kv_heads, a.tokens * group, a.prefix_len, true);
        t.flat_bytes = bytes_of(t.flat, c.dim, true);
    }
    return t;
}

}  // namespace

int64_t attn_workspace_bytes(const cq_kv_cache &c, const cq_attn_args &a) {
    const plan_t t = make_plan(c, a);
    return t.own_bytes.all() + t.flat_bytes.all();
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
    p.window = a.window;
    p.scale = a.scale;
    p.softcap = a.softcap;

    uint8_t *ws = static_cast<uint8_t *>(workspace);
    join_source flat = {};
    if (t.shared) {
        attn_params f = p;
        f.flat = 1;
        f.flat_len = int(a.prefix_len);
        f.tables = a.prefix_table;
        f.kv_lens = f.bidir = nullptr;
        f.q_starts = nullptr;
        f.batch = 1;
        flat = place(f, t.flat, t.flat_bytes, true, ws + t.own_bytes.all());
        const hipError_t e = launch_rows(int(c.dtype), c.dim, t.flat, f, stream);
        if (e != hipSuccess) return e;
    }
    const join_source own = place(p, t.own, t.own_bytes, t.shared, ws);
    const hipError_t e = launch_rows(int(c.dtype), c.dim, t.own, p, stream);
    if (e != hipSuccess || !own.rows) return e;
    return launch_attn_join(int(c.dtype), c.dim, p, own, flat, stream);
}

}  // namespace cq
