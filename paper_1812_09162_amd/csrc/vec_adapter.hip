// vec_adapter and vec_adapter_grad: checks, plans and launches (kernels: vec_adapter.h).
#include "vec_adapter_launch.h"

// vec_lookup.hip: the stable sort of positions by id; ids outside 0..rows-1 come last, with key `rows`
size_t qadc_vec_sort_bytes(int64_t n, int64_t rows);
void qadc_vec_sort(const void *ids, int id_bytes, int64_t n, int64_t rows, char *ws, const uint32_t **keys, const uint32_t **pos, hipStream_t s);

// The rules between the forms.  Times of whole calls in a graph, us, bfloat16 unless said.
//
// Rows that are not sorted: each reads its adapter for itself, mostly from the caches.  Of 16 adapters, sorted / not: 128 x 4096 at rank 16 18.7 / 13.4, 256 x 4096 20.6 / 19.5, 300 x 4096
// 20.0 / 29.2, 128 x 2048 at rank 64 29.7 / 13.0, 256 24.3 / 18.8, 512 x 2048 at rank 16 15.8 / 21.9.  Of less than two rows an adapter none are sorted, which up to about 1000 rows is
// the faster side and beyond the slower one: 300 x 4096 of 300 at rank 16 44 / 32, 600 x 2048 of 500 at rank 32 39 / 40, 1000 x 4096 of 1000 at rank 16 72 / 69, 1999 x 4096 of 1000
// 104 / 124, 4000 x 2048 of 3000 98 / 147, 8000 x 512 of 7000 65 / 89.
#define AD_FEW_ROWS 256
// Single rows in one launch: what they read of A altogether, mostly from the L2 cache, and how many they are (of one adapter the other form has whole tiles).  By two kernels / by one:
// 64 x 4096 at rank 16 (67 MB) 9.7 / 8.3, 128 (134 MB) 13.5 / 13.4, 128 x 2048 at rank 64 (134 MB) 12.8 / 14.4, 512 x 1024 at rank 16 (34 MB) 15.4 / 8.3, 1024 (67 MB) 16.0 / 14.0, 2048 (134
// MB) 17.0 / 25.4, 2048 x 256 at rank 8 14.8 / 11.4, 4096 15.5 / 20.3; of one adapter 16 x 4096 8.9 / 5.6, 256 x 1024 (17 MB) 8.3 / 5.3, 256 x 2048 (67 MB) 8.4 / 9.5.
#define AD_ONE_BYTES (72 << 20)
#define AD_ONE_SAME_BYTES (40 << 20)
#define AD_ONE_ROWS 2048
#define AD_ONE_SAME 256
// `down`: a wave takes an adapter of the tile where adapters have few rows (rows an adapter times columns), unless one wave would have too many columns.  Together / a wave each:
// 4096 rows of 1000 adapters at rank 16, 512 columns 36.5 / 28.9, 2048 69 / 58; 16,384 of 2000 at rank 8, 1024 columns, 81 / 66; beyond the rule, where it would still be faster, 4096
// columns 124 / 112 and 16,384 of 1000, 2048 columns, 99 / 91.
#define AD_OWN 32768
#define AD_OWN_COLUMNS 2048
// `up`: rows an adapter times ranks below which it runs on the vector units.  Matrix cores / vector units: 8192 of 500 at rank 8, 1001 fp16 columns, 43 / 37;
// 4096 of 1000 at rank 16, 512 columns, 36 / 29, 4096 columns 128 / 122; 16,384 of 1000, 4096 columns, 179 / 236; 16,384 of 500 at rank 32, 1024 columns, 51 / 97.
#define AD_UP_FEW 256
// Tiles of 32 and 64 positions only if so many are left: of short rows more, since a tile is little work.  At least 256 / 64 tiles: 4096 x 1024 of 8 at rank 16 19.0 / 22.0,
// 4096 x 4096 38 / 32, 8192 x 4096 53 / 50, 8192 x 2048 34.3 / 33.2, 2048 x 4096 float32 42 / 38.
#define AD_TILES(din, dout) ((din) + (dout) < 4096 ? 256 : 64)
// Slabs of `down` where there are fewer waves than this (with 512 / 1024 / 2048 / 4096: 1024 x 4096 of 8 at rank 16 22.2 / 20.7 / 19.2 / 23.2; 512 x 4096 17.8 / 16.9 / 18.3 / 18.3; 8192 x 2048 33.1 / 33.3 / 33.4 / 36.0).
#define AD_WAVES 1024
#define AD_MAX_SLABS 16

struct AdPlan {
    bool sorted, grouped;      // grouped: by k_vec_ad_group
    bool few;                  // `up` on the vector units
    bool one;                  // single rows in one launch
    int tp, tp_up;             // positions of a tile of `down`, of `up`
    int rp;                    // ranks of a row of partial sums
    int waves, slabs, per;     // of the contraction over columns
    bool own;                  // its waves take an adapter each
    int len_a, len_b;          // positions of a piece of the sums over rows
    int dpad_a, dpad_b;
    bool keeps;                // `outer` keeps the mask's bits for `up`
    size_t part, part_a, part_b, bits, total;  // bytes from the workspace's start
};

// Positions of a block of `outer`: fewer where there would be few blocks (us, whole gradients, with 128 / 64 / 32 / 16: 10,000 x (1001 + 700) fp16 of 200 adapters at rank 12
// 61 / 63 / 66 / 80; 79 x (84 + 6403) of 38 at rank 8 69 / 60 / 47 / 44; 2000 x (1024 + 1024) of 8 at rank 16 27 / 26 / 27 / 33).
static int ad_len(int64_t n, int64_t each, int d, int other, int rank) {
    const int64_t across = (int64_t)ad_outer_blocks(d, other) * ((rank + 63) / 64);
    int len = AD_MAX_LEN;
    while (len > (each < 16 ? 16 : 32) && (n + len - 1) / len * across < 400) len /= 2;
    return len;
}

static AdPlan ad_plan(int64_t n, int din, int dout, int rank, int adapters, int type, bool grad) {
    AdPlan p = {};
    const int64_t each = n / (adapters > 1 ? adapters : 1);
    // (a row's A is read for each of the column blocks)
    p.one = !grad && adapters > 0 && n <= (adapters > 1 ? AD_ONE_ROWS : AD_ONE_SAME) && rank <= 64 &&
            n * ad_column_blocks(dout, (int)vec_bytes(type)) * rank * din * (int64_t)vec_bytes(type) <= (adapters > 1 ? AD_ONE_BYTES : AD_ONE_SAME_BYTES);
    const bool sort = adapters > 1 && n > AD_FEW_ROWS && each > 1;
    p.sorted = grad || sort;
    // as many positions a tile as two adapters have rows on average, at most (one adapter / two / four: 16,384 x 2048 of 300 at rank 16 65 / 61 / 61, 16,384 x 4096 of 1000 193 / 179 / 173,
    // 8192 x 4096 of 400 at rank 32 121 / 105 / 113, 20,000 x 1024 of 400 54 / 54 / 54).  The average is over the adapters that are there, whether the call names them or not: 16,384 x 4096
    // in sixteen runs, of 64 / of 1000 adapters, at rank 16 97 / 108, at rank 8, where `few` holds for the 1000, 96 / 142.
    p.tp = rank <= 32 && din >= 8 && dout >= 8 ? 64 : 32;  // (of k_vec_ad_up's other form at most 32)
    while (p.tp > 16 && (p.tp > 2 * each || n / p.tp < AD_TILES(din, dout))) p.tp /= 2;
    p.tp_up = p.tp;
    p.few = p.sorted && each * rank < AD_UP_FEW;
    // tiles of up to eight, fewer where there would be too few waves (with 1024 / 2048 / 4096 waves at least: 4096 rows of 500 at rank 8, 1001 fp16 columns, 34 / 31 / 33; 4096 of
    // 1000 at rank 16, 512 columns, 33 / 29 / 29; 8192 of 500 at rank 8, 512 columns, 27 / 24 / 28)
    if (p.few) {
        const int64_t across = ad_column_blocks(grad ? din : dout, (int)vec_bytes(type));
        p.tp_up = AD_FEW_POSITIONS;
        while (p.tp_up > 1 && (n + p.tp_up - 1) / p.tp_up * across < 2048) p.tp_up /= 2;
    }
    if (adapters > 1 && !p.sorted) p.tp = p.tp_up = 1;
    p.grouped = n <= AD_GROUP_ROWS && adapters <= AD_GROUP_ADAPTERS;
    p.rp = (rank + 15) & ~15;
    const int d = grad ? dout : din;
    const int64_t tiles = (n + p.tp - 1) / p.tp;
    p.waves = d >= 1024 && rank <= 64 ? 8 : 4;
    p.own = p.sorted && d <= AD_OWN_COLUMNS && each * d < AD_OWN;
    // A wave of a slab has at least two turns of 64 columns.  Of waves with an adapter each about two have one (one slab / so: 4096 rows of 500 at rank 8, 1001 fp16 columns, 35 / 31; 4096
    // of 1000 at rank 16, 512 columns, 31.5 / 28.7; 8192 of 500, 512 columns, 25.1 / 24.2).
    const int64_t active = tiles * (p.own ? 2 : p.waves);
    int64_t slabs = active >= AD_WAVES ? 1 : AD_WAVES / active;
    const int64_t most = d / (p.own ? 128 : p.waves * 64);
    if (slabs > most) slabs = most;
    if (slabs > AD_MAX_SLABS) slabs = AD_MAX_SLABS;
    if (slabs < 1) slabs = 1;
    const int64_t per = ((d + slabs - 1) / slabs + 127) / 128 * 128;
    p.per = (int)per;
    p.slabs = (int)((d + per - 1) / per);
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += vec_up256(bytes); return was; };
    if (p.sorted) at = p.grouped ? 2 * vec_up256((size_t)n * 4) + vec_up256((size_t)(adapters + 1) * 4) : qadc_vec_sort_bytes(n, adapters);
    p.part = take((size_t)p.slabs * n * p.rp * 4);
    if (grad) {
        p.len_a = ad_len(n, each, din, dout, rank);
        p.len_b = ad_len(n, each, dout, din, rank);
        p.dpad_a = (din + 7) & ~7;
        p.dpad_b = (dout + 7) & ~7;
        p.part_a = take((size_t)((n + p.len_a - 1) / p.len_a) * 2 * rank * p.dpad_a * 4);
        p.part_b = take((size_t)((n + p.len_b - 1) / p.len_b) * 2 * rank * p.dpad_b * 4);
        // (a bit of x each, for the call's duration; where eight columns are no row's end and `outer` has four columns a lane.  Whole gradients with the mask made again in `up` / read, us: 16,384 x 4096 bf16
        // of 8 at rank 16 184 / 181, 16,384 x 2048 at rank 64 153 / 147, 4096 x 1024 of 500 73 / 72)
        p.keeps = din % 8 == 0 && dout >= 4;
        p.bits = take(p.keeps ? (size_t)((n + 3) / 4) * (din / 8) * 4 : 0);
    }
    p.total = at;
    return p;
}

// Returns where the adapters' positions begin (adapters + 1 numbers), or null where that is not known.
static const uint32_t *ad_sort(const AdPlan &p, AdRows &rows, char *ws, hipStream_t s) {
    if (!p.grouped) {
        qadc_vec_sort(rows.ids, rows.id_bytes, rows.n, rows.adapters, ws, &rows.keys, &rows.pos, s);
        return nullptr;
    }
    uint32_t *keys = (uint32_t *)ws, *pos = (uint32_t *)(ws + vec_up256((size_t)rows.n * 4)), *starts = (uint32_t *)(ws + 2 * vec_up256((size_t)rows.n * 4));
    const dim3 grid((unsigned)((rows.n + AD_GROUP_TILE - 1) / AD_GROUP_TILE));
    if (rows.id_bytes == 4) hipLaunchKernelGGL((k_vec_ad_group<int32_t>), grid, dim3(1024), 0, s, (const int32_t *)rows.ids, (int)rows.n, rows.adapters, keys, pos, starts);
    else hipLaunchKernelGGL((k_vec_ad_group<int64_t>), grid, dim3(1024), 0, s, (const int64_t *)rows.ids, (int)rows.n, rows.adapters, keys, pos, starts);
    rows.keys = keys;
    rows.pos = pos;
    return starts;
}

static bool ad_sizes(int64_t n, int din, int dout, int rank, int adapters) {
    return n >= 0 && n <= 0x7fffffffLL && din >= 1 && din <= VEC_MAX_ADAPTER_DIM && dout >= 1 && dout <= VEC_MAX_ADAPTER_DIM && rank >= 1 &&
           rank <= VEC_MAX_RANK && adapters >= 0 && adapters <= VEC_MAX_ADAPTERS;
}

extern "C" size_t vec_adapter_workspace_bytes(int64_t n, int din, int dout, int rank, int adapters, int type) {
    return n > 0 && adapters > 0 && ad_sizes(n, din, dout, rank, adapters) ? ad_plan(n, din, dout, rank, adapters, type, false).total : 0;
}
extern "C" size_t vec_adapter_grad_workspace_bytes(int64_t n, int din, int dout, int rank, int adapters, int type) {
    return n > 0 && adapters > 0 && ad_sizes(n, din, dout, rank, adapters) ? ad_plan(n, din, dout, rank, adapters, type, true).total : 0;
}

// column blocks of `up`: fewer than hold the columns where there are many tiles, each then takes some in turn
static int ad_up_blocks(int64_t n, int tp, int d, int type) {
    const int64_t tiles = (n + tp - 1) / tp, most = ad_column_blocks(d, (int)vec_bytes(type));
    const int64_t want = tiles >= 2048 ? 1 : (2048 + tiles - 1) / tiles;
    return (int)(want < most ? want : most);
}

static bool ad_fits(const AdPlan &p, int64_t n, int d, int type) {
    return (n + p.tp - 1) / p.tp * p.slabs <= VEC_MAX_BLOCKS && (n + p.tp_up - 1) / p.tp_up * ad_column_blocks(d, (int)vec_bytes(type)) <= VEC_MAX_BLOCKS;
}

#define AD_CHECK(name)                                                                                                                              \
    uint32_t threshold;                                                                                                                             \
    float factor;                                                                                                                                   \
    VEC_REQUIRE(ad_sizes(n, din, dout, rank, adapters), name ": n=%lld, din=%d, dout=%d (1..%d), rank=%d (1..%d), adapters=%d (0..%d)", (long long)n, \
                din, dout, VEC_MAX_ADAPTER_DIM, rank, VEC_MAX_RANK, adapters, VEC_MAX_ADAPTERS);                                                    \
    VEC_REQUIRE(vec_rate(p, &threshold, &factor), name ": p=%g is not in 0..65535/65536", p);                                                       \
    VEC_REQUIRE(vec_is_wide(type), name ": types: %d is not F32, BF16 or F16", type);                                                               \
    VEC_REQUIRE(id_bytes == 4 || id_bytes == 8, name ": ids of %d bytes", id_bytes);                                                                \
    VEC_REQUIRE(threshold == 0 || (state && ((uintptr_t)state & 7u) == 0), name ": state null or misaligned");                                      \
    VEC_REQUIRE(ld_a >= din && ld_b >= dout && stride_a >= 0 && stride_b >= 0, name ": a distance of rows is below their length, or one of adapters below 0")

#define AD_WORKSPACE(name, need)                                                                            \
    do {                                                                                                    \
        VEC_REQUIRE(workspace && ((uintptr_t)workspace & 255u) == 0, name ": workspace null or not 256-byte aligned"); \
        if (workspace_bytes < (need)) {                                                                     \
            qadc_set_error(name ": workspace of %zu bytes, %zu needed", workspace_bytes, (size_t)(need));   \
            return PQ_ENOMEM;                                                                               \
        }                                                                                                   \
    } while (0)

extern "C" int vec_adapter(const void *x, int64_t ld_x, const void *a, int64_t ld_a, int64_t stride_a, const void *b, int64_t ld_b, int64_t stride_b, int type,
                           int adapters, int rank, const float *scales, const void *ids, int id_bytes, int64_t n, int din, int dout, const void *base,
                           int64_t ld_base, void *y, int64_t ld_y, int y_type, double p, const uint64_t *state, uint32_t layer, float *t, void *workspace,
                           size_t workspace_bytes, void *stream) {
    AD_CHECK("vec_adapter");
    VEC_REQUIRE(y_type == type || y_type == VEC_F32, "vec_adapter: types %d and %d (y)", type, y_type);
    VEC_REQUIRE(ld_x >= din && (!base || ld_base >= dout) && ld_y >= dout, "vec_adapter: a distance of rows is below their length");
    VEC_REQUIRE(base != y || !base || ld_base == ld_y, "vec_adapter: y in place of base with other distances of rows");
    if (n == 0) return PQ_OK;
    VEC_REQUIRE(x && y && ids && (adapters == 0 || (a && b)), "vec_adapter: null pointer");
    // (a row's blocks of k_vec_ad_one read all of x's row, while others already write theirs of y)
    VEC_REQUIRE(x != y, "vec_adapter: y in place of x");
    VEC_REQUIRE(vec_aligned(x, type) && vec_aligned(a, type) && vec_aligned(b, type) && vec_aligned(base, y_type) && vec_aligned(y, y_type) &&
                    vec_aligned(scales, VEC_F32) && vec_aligned(t, VEC_F32) && ((uintptr_t)ids & (uintptr_t)(id_bytes - 1)) == 0,
                "vec_adapter: misaligned pointer");
    hipStream_t s = (hipStream_t)stream;
    const AdPlan plan = ad_plan(n, din, dout, rank, adapters, type, false);
    VEC_REQUIRE(ad_fits(plan, n, dout, type), "vec_adapter: n=%lld too large for one call", (long long)n);
    AdRows rows = {ids, id_bytes, plan.tp, n, adapters, nullptr, nullptr};
    char *ws = (char *)workspace;
    float *part = nullptr;
    const VecMask mask = {state, layer, threshold}, none = {nullptr, 0, 0};
    if (adapters > 0) AD_WORKSPACE("vec_adapter", plan.total);
    if (plan.one) {
        const AdMatrix ma = {a, ld_a, stride_a, rank, din}, mb = {b, ld_b, stride_b, rank, dout};
        VEC_TYPED(type, T, AdLaunch<T>::one(rows, x, ld_x, ma, mb, scales, factor, mask, base, ld_base, y, ld_y, y_type == type, t, s));
        QADC_LAUNCH_CHECK("k_vec_ad_one");
        return PQ_OK;
    }
    if (adapters > 0) {
        part = (float *)(ws + plan.part);
        if (plan.sorted) ad_sort(plan, rows, ws, s);
        const AdMatrix m = {a, ld_a, stride_a, rank, din};
        VEC_TYPED(type, T, AdLaunch<T>::down(rows, x, ld_x, m, scales, factor, mask, part, n * plan.rp, plan.rp, plan.waves, plan.slabs, plan.per,
                                             plan.own, plan.slabs == 1 ? t : nullptr, s));
    }
    float *const keep = adapters > 0 && plan.slabs == 1 ? nullptr : t;
    rows.tp = plan.tp_up;
    const AdFactor f = {part, plan.rp, n * plan.rp, plan.slabs};
    const AdMatrix m = {b, ld_b, stride_b, rank, dout};
    VEC_TYPED(type, T, AdLaunch<T>::up(rows, f, m, base, ld_base, y, ld_y, y_type == type, none, nullptr, plan.few, ad_up_blocks(n, plan.tp_up, dout, type), keep, nullptr, s));
    QADC_LAUNCH_CHECK("vec_adapter's kernels");
    return PQ_OK;
}

extern "C" int vec_adapter_grad(const void *dy, int64_t ld_dy, const void *x, int64_t ld_x, const float *t, const void *a, int64_t ld_a, int64_t stride_a,
                                const void *b, int64_t ld_b, int64_t stride_b, int type, int adapters, int rank, const float *scales, const void *ids,
                                int id_bytes, int64_t n, int din, int dout, const void *dx_base, int64_t ld_dx_base, void *dx, int64_t ld_dx, double p,
                                const uint64_t *state, uint32_t layer, int accumulate, void *da, int64_t ld_da, int64_t stride_da, void *db, int64_t ld_db,
                                int64_t stride_db, int grad_type, void *workspace, size_t workspace_bytes, void *stream) {
    AD_CHECK("vec_adapter_grad");
    VEC_REQUIRE(grad_type == type || grad_type == VEC_F32, "vec_adapter_grad: types %d and %d (da, db)", type, grad_type);
    VEC_REQUIRE(dx || !dx_base, "vec_adapter_grad: dx_base without dx");
    VEC_REQUIRE(ld_x >= din && ld_dy >= dout && (!dx || ld_dx >= din) && (!dx_base || ld_dx_base >= din) && ld_da >= din && ld_db >= dout,
                "vec_adapter_grad: a distance of rows is below their length");
    VEC_REQUIRE(adapters <= 1 || (stride_da >= (int64_t)(rank - 1) * ld_da + din && stride_db >= (int64_t)(rank - 1) * ld_db + dout),
                "vec_adapter_grad: the adapters' gradients overlap");
    VEC_REQUIRE(!dx || dx_base != dx || ld_dx_base == ld_dx, "vec_adapter_grad: dx in place of dx_base with other distances of rows");
    VEC_REQUIRE((adapters == 0 || (da && db)) && (n == 0 || (ids && (adapters == 0 || (dy && x && t && a && b)))), "vec_adapter_grad: null pointer");
    VEC_REQUIRE(vec_aligned(dy, type) && vec_aligned(x, type) && vec_aligned(t, VEC_F32) && vec_aligned(a, type) && vec_aligned(b, type) &&
                    vec_aligned(scales, VEC_F32) && vec_aligned(dx_base, type) && vec_aligned(dx, type) && vec_aligned(da, grad_type) && vec_aligned(db, grad_type) &&
                    ((uintptr_t)ids & (uintptr_t)(id_bytes - 1)) == 0, "vec_adapter_grad: misaligned pointer");
    if (n == 0 && (adapters == 0 || accumulate)) return PQ_OK;
    hipStream_t s = (hipStream_t)stream;
    const VecMask mask = {state, layer, threshold}, none = {nullptr, 0, 0};
    const bool narrow = grad_type == type;
    AdRows rows = {ids, id_bytes, 1, n, adapters, nullptr, nullptr};
    AdPlan plan = {};
    plan.len_a = plan.len_b = AD_MAX_LEN;
    plan.dpad_a = (din + 7) & ~7;
    plan.dpad_b = (dout + 7) & ~7;
    const uint32_t *starts = nullptr;
    const AdMatrix ma = {a, ld_a, stride_a, rank, din}, mb = {b, ld_b, stride_b, rank, dout};
    AdFactor u = {};
    uint32_t *bits = nullptr;
    AdOuter oa = {da, ld_da, stride_da, nullptr, plan.dpad_a, accumulate}, ob = {db, ld_db, stride_db, nullptr, plan.dpad_b, accumulate};
    if (n > 0) {
        plan = ad_plan(n, din, dout, rank, adapters, type, true);
        rows.tp = plan.tp;
        VEC_REQUIRE(ad_fits(plan, n, din, type) && (n / plan.len_a + 1) * ad_outer_blocks(din, dout) + (n / plan.len_b + 1) * ad_outer_blocks(dout, din) <= VEC_MAX_BLOCKS, "vec_adapter_grad: n=%lld too large for one call", (long long)n);
        char *ws = (char *)workspace;
        u = {nullptr, plan.rp, n * plan.rp, plan.slabs};
        if (adapters > 0) {
            AD_WORKSPACE("vec_adapter_grad", plan.total);
            float *part = (float *)(ws + plan.part);
            u.p = part;
            bits = plan.keeps && dx && threshold ? (uint32_t *)(ws + plan.bits) : nullptr;
            oa.part = (float *)(ws + plan.part_a);
            ob.part = (float *)(ws + plan.part_b);
            starts = ad_sort(plan, rows, ws, s);
            const AdSide sb = {{t, rank, 0, 1}, dy, ld_dy, dout, plan.len_b, ad_outer_blocks(dout, din), ob}, sa = {u, x, ld_x, din, plan.len_a, ad_outer_blocks(din, dout), oa};
            VEC_TYPED(type, T, AdLaunch<T>::down(rows, dy, ld_dy, mb, scales, factor, none, part, n * plan.rp, plan.rp, plan.waves, plan.slabs, plan.per, plan.own, nullptr, s);
                      AdLaunch<T>::outer(rows, rank, mask, sb, sa, narrow, bits, s));
        }
        rows.tp = plan.tp_up;
    }
    AdJoins joins = {{oa, plan.len_a, din}, {ob, plan.len_b, dout}, starts, rank, narrow, 1};
    const int64_t pieces = (int64_t)rank * ((plan.dpad_a > plan.dpad_b ? plan.dpad_a : plan.dpad_b) / 8);
    // 2 (8192 + adapters) blocks at most: of many adapters most have nothing to join (whole gradients with a block for each 2048 values of each / so, us: 4096 rows of 1000, 4096 columns at
    // rank 16 315 / 286, 16,384 of 4000, 512 columns at rank 64 577 / 466)
    joins.across = (int)((pieces + 255) / 256);
    if (adapters > 0 && joins.across > 8192 / adapters + 1) joins.across = 8192 / adapters + 1;
    if (n > 0 && dx) {
        VEC_TYPED(type, T, AdLaunch<T>::up(rows, u, ma, dx_base, ld_dx_base, dx, ld_dx, true, adapters > 0 ? mask : none, bits, plan.few, ad_up_blocks(n, plan.tp_up, din, type),
                                           nullptr, adapters > 0 ? &joins : nullptr, s));
    } else if (adapters > 0) {
        VEC_TYPED(type, T, AdLaunch<T>::join(rows, joins, s));
    }
    QADC_LAUNCH_CHECK("vec_adapter_grad's kernels");
    return PQ_OK;
}
