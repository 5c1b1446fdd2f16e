// vec_lookup and vec_lookup_grad: rows of a table by id, and the sum of gradients by id.
#include "vec_device.h"

// ------------------------------------------------------------------ look-up --
// out[i] = scale * table[ids[i]].  A block copies `rpb` neighbouring rows of the result as pieces of eight elements; bound by
// memory: every piece is one wide load behind a load of the row's id, four of them in flight per thread.  65,536 rows of 65,536 x 1024 bf16 (some
// rows again and again): 32 us for the 134 MB written, 44 us a call among calls (its neighbours' stores drain); 100 rows 3.6 us, all latency.
template <class TI, class TO, class ID>
__global__ void __launch_bounds__(256)
k_vec_lookup(const TI *__restrict__ table, int64_t rows, int d, int64_t ld_table, const ID *__restrict__ ids, int64_t n,
             float scale, TO *__restrict__ out, int64_t ld_out, int rpb, int pieces, uint32_t magic) {
    const int64_t row0 = vec_block() * rpb;
    const int nrow = (int)(n - row0 < rpb ? n - row0 : rpb);
    const int total = nrow * pieces;  // (0 or less behind the last row)
    for (int e0 = threadIdx.x; e0 < total; e0 += 256 * 4) {
        vec_pack<TI> v[4];
        int64_t to[4];
        int left[4];
        float by[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int e = e0 + u * 256;
            left[u] = 0;
            if (e >= total) continue;
            const int r = rpb == 1 ? 0 : (pieces == 1 ? e : (int)__umulhi((uint32_t)e, magic));  // e / pieces
            const int col = (e - r * pieces) * 8;
            const int64_t id = (int64_t)ids[row0 + r];
            const bool known = id >= 0 && id < rows;
            left[u] = d - col;
            by[u] = known ? scale : 0.0f;  // (zeros of an unknown id take no sign, infinity or NaN of the scale)
            to[u] = (row0 + r) * ld_out + col;
            v[u] = vec_load(table + (known ? id * ld_table + col : 0), known ? left[u] : 0, col);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (left[u] > 0) {
                vec_f8 f = vec_wide<TI>(v[u]);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= by[u];
                vec_store(out + to[u], left[u], f);
            }
    }
}

extern "C" int vec_lookup(const void *table, int64_t rows, int d, int64_t ld_table, int table_type, const void *ids,
                          int id_bytes, int64_t n, float scale, void *out, int64_t ld_out, int out_type, void *stream) {
    VEC_REQUIRE(n >= 0 && rows >= 0 && d >= 1 && d <= VEC_MAX_ROW_DIM, "vec_lookup: n=%lld, rows=%lld, d=%d", (long long)n, (long long)rows, d);
    VEC_REQUIRE(vec_is_wide(table_type) && vec_is_wide(out_type), "vec_lookup: types %d and %d are not F32, BF16 or F16", table_type, out_type);
    VEC_REQUIRE(id_bytes == 4 || id_bytes == 8, "vec_lookup: ids of %d bytes", id_bytes);
    VEC_REQUIRE(ld_table >= d && ld_out >= d, "vec_lookup: rows of %lld and %lld elements hold no %d", (long long)ld_table, (long long)ld_out, d);
    if (n == 0) return PQ_OK;
    VEC_REQUIRE((table || rows == 0) && ids && out, "vec_lookup: null pointer");
    VEC_REQUIRE(vec_aligned(table, table_type) && vec_aligned(out, out_type) && ((uintptr_t)ids & (uintptr_t)(id_bytes - 1)) == 0, "vec_lookup: misaligned pointer");
    const int pieces = (d + 7) / 8;
    // 1024 pieces a block, whole rows; a row of more is a block of its own
    const int rpb = pieces >= 1024 ? 1 : 1024 / pieces;
    const int64_t blocks = (n + rpb - 1) / rpb;
    VEC_REQUIRE(blocks <= VEC_MAX_BLOCKS, "vec_lookup: n=%lld too large for one call", (long long)n);
    // e / pieces for e < 1024, pieces > 1: exact as 1024 pieces < 2^32
    const uint32_t magic = (uint32_t)((((uint64_t)1 << 32) + pieces - 1) / pieces);
    hipStream_t s = (hipStream_t)stream;
#define GO(TI, TO, ID)                                                                                                    \
    hipLaunchKernelGGL((k_vec_lookup<TI, TO, ID>), vec_grid(blocks, 256), dim3(256), 0, s, (const TI *)table, rows, d,    \
                       ld_table, (const ID *)ids, n, scale, (TO *)out, ld_out, rpb, pieces, magic)
    VEC_TYPED(table_type, TI, VEC_TYPED(out_type, TO, if (id_bytes == 4) GO(TI, TO, int32_t); else GO(TI, TO, int64_t)));
#undef GO
    QADC_LAUNCH_CHECK("k_vec_lookup");
    return PQ_OK;
}

// ----------------------------------------------------------------- gradient --
// table_grad[v] = base + scale * sum of the rows of grad whose id is v.  Positions with the same id are summed in ascending
// order in float32, in pieces that do not depend on which block ran first.
//
// Few ids (n <= GRAD_FEW): one launch.  Every block owns some rows of the table, dealt out in turn since frequent ids are often
// neighbours; it goes through all ids, keeps the positions of its own in order, and writes its rows, zeros or sums.  The ids
// are read once per block, from the L2 cache.  2,048 ids into 65,536 x 256 float32: 20 us, of which the 67 MB of zeros are 14 at the rate of a large copy.
//
// Many: the positions are sorted by id (a stable radix sort of up to 2^GRAD_BITS buckets a pass), then summed in pieces
// of at most GRAD_CHUNK sorted positions, whatever ids they hold, so that a frequent id is no wave's alone; sums of ids that cross
// a piece's ends are joined by a last kernel.  k_vec_grad_place waits for memory most of the time: blocks beside its own clear the
// table meanwhile, a share in each pass (in k_vec_grad_count too: 262,144 ids into 900,000 x 100 85 us, 79 without).  262,144 ids into 100,003 x 512 (bf16, 373 MB, log-uniform): two passes of 5 + 15 us, in which the 102 MB are
// cleared, sums 74 (271 MB read and 56 written, 4.4 TB/s), joins 9: 131 us a call.
//
// A row is spread over the 64 lanes of a wave, E elements each (2, 4 or 8, the fewest that hold it, else 64 E columns at a time).
// us, one launch / sorted: 2,048 ids into 65,536 x 256 21 / 60, 4,096 25 / 57, 8,192 44 / 46; tables that one pass sorts: 883 into 623 x 2944 21 / 43,
// 4,000 54 / 43, 4,000 into 623 x 128 20 / 22
#define GRAD_POS 12  // bits of a position
#define GRAD_FEW (1 << GRAD_POS)
#define GRAD_BITS 10
#define GRAD_TILE 4096   // keys that a block of 1024 threads of the sort takes
#define GRAD_TILES_ALONE 128  // tiles of the sort whose counts every block adds up itself
#define GRAD_CHUNK 64    // at most: shorter pieces, more waves where there are few (16,384 ids into 65,536 x 256: 18 us with 64)

#define GRAD_WIDTHS(d, ...)          \
    do {                             \
        if ((d) <= 128) {            \
            constexpr int E = 2;     \
            __VA_ARGS__;             \
        } else if ((d) <= 256) {     \
            constexpr int E = 4;     \
            __VA_ARGS__;             \
        } else {                     \
            constexpr int E = 8;     \
            __VA_ARGS__;             \
        }                            \
    } while (0)

struct GradPlan {
    bool few;
    int passes, bits;   // of the sort
    int tiles, chunks;  // blocks of a pass; pieces of the sum,
    int len;            // so many positions each
    int seg, segs;      // tiles of a segment, and segments, where the counts become running sums first; else 0
    int dpad;           // floats of a partial row
    size_t key0, key1, pos0, pos1, counts, sums, begins, part, total;
};

static GradPlan grad_plan(int64_t n, int64_t rows, int d) {
    GradPlan p = {};
    p.few = n <= (rows < (1 << GRAD_BITS) ? GRAD_FEW / 2 : GRAD_FEW);
    if (p.few) return p;
    int bits = 1;
    while (((int64_t)1 << bits) <= rows) ++bits;  // ids 0..rows, `rows` standing for those that take no part
    p.passes = (bits + GRAD_BITS - 1) / GRAD_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = (int)((n + GRAD_TILE - 1) / GRAD_TILE);
    p.len = n <= 32768 ? GRAD_CHUNK / 4 : (n <= 131072 ? GRAD_CHUNK / 2 : GRAD_CHUNK);
    p.chunks = (int)((n + p.len - 1) / p.len);
    if (p.tiles > GRAD_TILES_ALONE) {
        p.seg = 1;
        while ((int64_t)p.seg * p.seg < p.tiles) p.seg *= 2;
        p.segs = (p.tiles + p.seg - 1) / p.seg;
    }
    p.dpad = (d + 7) & ~7;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += vec_up256(bytes); return was; };
    p.key0 = take((size_t)n * 4);
    p.key1 = take((size_t)n * 4);
    p.pos0 = take((size_t)n * 4);
    p.pos1 = take((size_t)n * 4);
    p.counts = take(((size_t)p.tiles << p.bits) * 4);
    p.sums = p.segs > 0 ? take(((size_t)(p.segs + 1) << p.bits) * 4) : 0;
    p.begins = take((size_t)rows * 4);
    p.part = take((size_t)p.chunks * 2 * p.dpad * 4);
    p.total = at;
    return p;
}

extern "C" size_t vec_lookup_grad_workspace_bytes(int64_t n, int64_t rows, int d) {
    return n <= 0 || rows <= 0 || d <= 0 || n > 0x7fffffffLL || rows > 0x7ffffffeLL ? 0 : grad_plan(n, rows, d).total;
}

template <class TT, int E>
__device__ __forceinline__ void grad_write(TT *__restrict__ row, int64_t col, int64_t left, vec_f<E> acc, float scale, int accumulate) {
    if (left <= 0) return;
    vec_f<E> f;
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = acc[i] * scale;
    if (accumulate) f += vec_wide<TT, E>(vec_load<TT, E>(row + col, left, col));
    vec_store<TT, E>(row + col, left, f);
}

// Zeros in the first `cols` columns of those of `nrow` rows whose bit of `has` is not set; row(r): where the r-th begins.
template <class TT, int NT, class ROW>
__device__ __forceinline__ void grad_zeros(int nrow, int cols, const uint32_t *has, ROW row) {
    const int pieces = (cols + 7) / 8;
    int r = threadIdx.x / pieces, c = threadIdx.x - r * pieces;
    const int dr = NT / pieces, dc = NT - dr * pieces;
    while (r < nrow) {
        if (!(has[r >> 5] >> (r & 31) & 1)) vec_store<TT>(row(r) + c * 8, cols - c * 8, (vec_f8)0.0f);
        r += dr;
        c += dc;
        if (c >= pieces) c -= pieces, ++r;
    }
}

// Adds to acc the rows of grad at the positions (low GRAD_POS bits) of those of list[0 .. m - 1] that are of row r (the bits above), in order.
template <class TG, int E>
__device__ __forceinline__ void grad_pick(const TG *__restrict__ grad, int64_t ld, int64_t col, int64_t left, const uint32_t *list, int m,
                                          uint32_t r, vec_f<E> &acc) {
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < m; i0 += 64) {
        const uint32_t e = i0 + lane < m ? list[i0 + lane] : 0xffffffffu;
        uint64_t hits = __ballot(e >> GRAD_POS == r);
        while (hits) {
            constexpr int B = sizeof(TG) * E <= 16 ? 16 : 8;  // rows on their way
            vec_pack<TG, E> v[B];
            int k = 0;
#pragma unroll
            for (int u = 0; u < B; ++u) {
                const int at = hits ? __builtin_ctzll(hits) : 0;
                const bool more = hits != 0;
                hits &= hits - 1;
                const uint32_t pos = __builtin_amdgcn_readlane(e, at) & (GRAD_FEW - 1);
                k += more;
                v[u] = vec_load<TG, E>(grad + (int64_t)pos * ld + col, more ? left : 0, col);
            }
#pragma unroll
            for (int u = 0; u < B; ++u)
                if (u < k) acc += vec_wide<TG, E>(v[u]);
        }
    }
}

// The block's rows: groups of 2^group neighbouring rows are dealt out over 2^deal blocks.  Its columns: 64 E from blockIdx.y 64 E on.
template <class TG, class TT, class ID, int E>
__global__ void __launch_bounds__(256)
k_vec_grad_few(const TG *__restrict__ grad, int n, int d, int64_t ld_grad, const ID *__restrict__ ids, float scale,
               int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table, int group, int deal, int rpb) {
    constexpr int WAVES = 4;  // (sixteen: twice the time, 2,048 ids into 65,536 x 256 43 us)
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t *has = (uint32_t *)smem;           // [(rpb + 31) / 32]
    uint32_t *list = has + (rpb + 31) / 32;     // [n, up to the next 64 WAVES] row of the block << GRAD_POS | position
    __shared__ int count[WAVES];
    __shared__ vec_f<E> share[WAVES][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int col0 = (int)blockIdx.y * 64 * E, col = col0 + lane * E, cols = d - col0 < 64 * E ? d - col0 : 64 * E;
    // row r of the block is row of(r) of the table; its rows below `rows` come first
    auto of = [&](int r) { return ((((int64_t)(r >> group) << deal) + blockIdx.x) << group) + (r & ((1 << group) - 1)); };
    int nrow = rpb;
    while (nrow > 0 && of(nrow - 1) >= rows) --nrow;
    for (int i = threadIdx.x; i < (rpb + 31) / 32; i += 64 * WAVES) has[i] = 0;
    __syncthreads();
    // each wave takes its share of the positions, sixteen loads at once, and keeps the block's own, in order, in its share of the list
    const int per = (n + 64 * WAVES - 1) / (64 * WAVES) * 64, from = wave * per;
    int m = 0;
    for (int i0 = from; i0 < from + per; i0 += 1024) {
        int64_t id[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const int i = i0 + u * 64 + lane;
            id[u] = i < from + per && i < n ? (int64_t)ids[i] : -1;
        }
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            const bool mine = id[u] >= 0 && id[u] < rows && ((id[u] >> group) & ((1 << deal) - 1)) == blockIdx.x;
            const uint64_t b = __ballot(mine);
            if (!b) continue;
            if (mine) {
                const int r = (int)(id[u] >> (group + deal) << group) + (int)(id[u] & ((1 << group) - 1));
                list[from + m + __popcll(b & ((1ull << lane) - 1))] = (uint32_t)r << GRAD_POS | (uint32_t)(i0 + u * 64 + lane);
                atomicOr(&has[r >> 5], 1u << (r & 31));
            }
            m += __popcll(b);
        }
    }
    if (lane == 0) count[wave] = m;
    __syncthreads();
    int all = 0;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) all += count[q];
    int turn = 0;
    for (int w = 0; w < (nrow + 31) / 32; ++w) {
        for (uint32_t bits = has[w]; bits; bits &= bits - 1) {
            const int r = w * 32 + __builtin_ctz(bits);
            TT *row = table + of(r) * ld_table;
            vec_f<E> acc = (vec_f<E>)0.0f;
            if (all <= 64) {  // a wave per row
                if ((turn++ & (WAVES - 1)) != wave) continue;
                for (int q = 0; q < WAVES; ++q) grad_pick<TG, E>(grad, ld_grad, col, d - col, list + q * per, count[q], r, acc);
                grad_write<TT, E>(row, col, d - col, acc, scale, accumulate);
            } else {  // frequent ids: each wave its share of the positions
                grad_pick<TG, E>(grad, ld_grad, col, d - col, list + from, m, r, acc);
                share[wave][lane] = acc;
                __syncthreads();
                if (wave == 0) {
#pragma unroll
                    for (int q = 1; q < WAVES; ++q) acc += share[q][lane];
                    grad_write<TT, E>(row, col, d - col, acc, scale, accumulate);
                }
                __syncthreads();
            }
        }
    }
    // (behind the sums, whose reads would wait for these stores)
    if (!accumulate) grad_zeros<TT, 64 * WAVES>(nrow, cols, has, [&](int r) { return table + of(r) * ld_table + col0; });
}

// --- the sort.  counts[tile][bucket]

// Clears rows: the blocks of a launch from `after` on take `each` rows, from `lo` on.
struct GradClear {
    void *table;
    int64_t lo, hi, ld;
    int d, each, after;
};
template <class TT>
__device__ __forceinline__ bool grad_clear(const GradClear &z) {
    if ((int)blockIdx.x < z.after) return false;
    const int64_t lo = z.lo + (int64_t)((int)blockIdx.x - z.after) * z.each, hi = lo + z.each < z.hi ? lo + z.each : z.hi;
    const int pieces = (z.d + 7) / 8;
    TT *row = (TT *)z.table + lo * z.ld;
    int r = threadIdx.x / pieces, c = threadIdx.x - r * pieces;
    const int dr = 1024 / pieces, dc = 1024 - dr * pieces;
    while (r < hi - lo) {
        vec_store<TT>(row + r * z.ld + c * 8, z.d - c * 8, (vec_f8)0.0f);
        r += dr;
        c += dc;
        if (c >= pieces) c -= pieces, ++r;
    }
    return true;
}

template <class ID>
__device__ __forceinline__ uint32_t grad_key(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t i, int64_t rows) {
    if (keys) return keys[i];
    const int64_t id = (int64_t)ids[i];
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

#define GRAD_PER (GRAD_TILE / 1024)
template <class ID>
__global__ void __launch_bounds__(1024)
k_vec_grad_count(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t n, int64_t rows, int shift, int bits,
                 uint32_t *__restrict__ counts) {
    __shared__ uint32_t h[1 << GRAD_BITS];
    const int nb = 1 << bits;
    const int64_t first = (int64_t)blockIdx.x * GRAD_TILE + threadIdx.x;
    uint32_t key[GRAD_PER];
#pragma unroll
    for (int u = 0; u < GRAD_PER; ++u) key[u] = first + u * 1024 < n ? grad_key(ids, keys, first + u * 1024, rows) : 0;
    if ((int)threadIdx.x < nb) h[threadIdx.x] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < GRAD_PER; ++u)
        if (first + u * 1024 < n) atomicAdd(&h[key[u] >> shift & (nb - 1)], 1u);
    __syncthreads();
    if ((int)threadIdx.x < nb) counts[((size_t)blockIdx.x << bits) + threadIdx.x] = h[threadIdx.x];
}

// Running sums of the counts over many tiles, in place: a block takes a segment of them, thread b bucket b; sums[segment][bucket] becomes the segment's.
// Sixteen counts are read before any is written.
__global__ void __launch_bounds__(1024)
k_vec_grad_running(uint32_t *counts, int tiles, int seg, int bits, uint32_t *__restrict__ sums) {
    if (threadIdx.x >> bits) return;
    const int t0 = blockIdx.x * seg, t1 = t0 + seg < tiles ? t0 + seg : tiles;
    uint32_t *const c = counts + threadIdx.x;
    uint32_t sum = 0;
    for (int t = t0; t < t1; t += 16) {
        uint32_t v[16];
#pragma unroll
        for (int u = 0; u < 16; ++u) v[u] = t + u < t1 ? c[(size_t)(t + u) << bits] : 0;
#pragma unroll
        for (int u = 0; u < 16; ++u) {
            if (t + u < t1) c[(size_t)(t + u) << bits] = sum;
            sum += v[u];
        }
    }
    sums[((size_t)blockIdx.x << bits) + threadIdx.x] = sum;
}

// A tile's keys to their places: those of one bucket keep their order.  Thread b adds up the sizes of bucket b over the tiles, of those
// before this one and of all; running sums over the buckets then say where the tile's keys go.  (A kernel of its own for these sums
// took 5 us, the loads here about 2 with 64 tiles.  They grow with the square of the tiles, so that more than GRAD_TILES_ALONE have k_vec_grad_running make them, over the tiles
// of a segment and then over the segments.  us, by the blocks / by k_vec_grad_running: into 900,000 x 8, 64 tiles 70 / 74, 128 98 / 95, 256 168 / 152,
// 1024 760 / 442; into 500 x 64 37 / 39, 52 / 52, 88 / 84, 382 / 303.)  Wave w holds the tile's w-th sixteenth, 64 keys at a time; a key's rank among them is
// the number of lower lanes with the same bucket, found bit by bit with ballots.
template <class ID, class TT>
__global__ void __launch_bounds__(1024)
k_vec_grad_place(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos, int64_t n,
                 int64_t rows, int shift, int bits, const uint32_t *__restrict__ counts, int tiles, int seg, const uint32_t *__restrict__ sums,
                 const uint32_t *__restrict__ totals, uint32_t *__restrict__ keys_out, uint32_t *__restrict__ pos_out, GradClear z) {
    if (grad_clear<TT>(z)) return;
    extern __shared__ uint32_t next[];  // [16 waves][buckets]: a wave's keys of a bucket, then where its next one goes
    __shared__ uint32_t part[16];
    const int nb = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t first = (int64_t)blockIdx.x * GRAD_TILE + wave * (GRAD_TILE / 16) + lane;
    uint32_t key[GRAD_PER], from[GRAD_PER];
#pragma unroll
    for (int u = 0; u < GRAD_PER; ++u) {
        const int64_t i = first + u * 64;
        key[u] = i < n ? grad_key(ids, keys, i, rows) : 0;
        from[u] = i < n && pos ? pos[i] : (uint32_t)i;
    }
    uint32_t before_tile = 0, total = 0;
    if (seg > 0) {
        if ((int)threadIdx.x < nb) {
            before_tile = counts[((size_t)blockIdx.x << bits) + threadIdx.x] + sums[((size_t)(blockIdx.x / seg) << bits) + threadIdx.x];
            total = totals[threadIdx.x];
        }
    } else if ((int)threadIdx.x < nb) {
        const uint32_t *c = counts + threadIdx.x;
#pragma unroll 16
        for (int t = 0; t < tiles; ++t) {
            const uint32_t v = c[(size_t)t << bits];
            total += v;
            before_tile += t < (int)blockIdx.x ? v : 0;
        }
    }
    for (int i = threadIdx.x; i < 16 * nb; i += 1024) next[i] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < GRAD_PER; ++u)
        if (first + u * 64 < n) atomicAdd(&next[(wave << bits) + (key[u] >> shift & (nb - 1))], 1u);
    uint32_t s = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(s, o);
        if (lane >= o) s += x;
    }
    if (lane == 63) part[wave] = s;
    __syncthreads();
    if ((int)threadIdx.x < nb) {
        uint32_t at = s - total + before_tile;
        for (int w = 0; w < wave; ++w) at += part[w];
#pragma unroll
        for (int w = 0; w < 16; ++w) {
            const uint32_t c = next[(w << bits) + threadIdx.x];
            next[(w << bits) + threadIdx.x] = at;
            at += c;
        }
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < GRAD_PER; ++u) {
        const bool in = first + u * 64 < n;
        const uint32_t bucket = key[u] >> shift & (nb - 1);
        uint32_t *mine = &next[(wave << bits) + bucket];
        uint64_t same = __ballot(in);
        for (int b = 0; b < bits; ++b) {
            const uint64_t x = __ballot(bucket >> b & 1);
            same &= bucket >> b & 1 ? x : ~x;
        }
        if (in) {
            const uint32_t at = *mine + __popcll(same & ((1ull << lane) - 1));
            keys_out[at] = key[u];
            pos_out[at] = from[u];
        }
        __builtin_amdgcn_wave_barrier();  // the reads above come before the wave's own update
        if (in && (same >> lane) == 1) *mine += __popcll(same);  // the bucket's last lane
        __builtin_amdgcn_wave_barrier();
    }
}

// --- the sums.  A wave per piece of `len` sorted positions and 64 E columns: ids that lie within the piece are written to
// the table; the sum of one that began before goes to part[chunk][0], that of one that begins here and goes on to part[chunk][1].  begins[v]: first sorted position of id v.
// Rows are requested eight at a time, whatever ids they are of, eight ahead of those that are added.
template <class TG, class TT, int E>
__global__ void __launch_bounds__(256)
k_vec_grad_chunks(const TG *__restrict__ grad, int d, int64_t ld_grad, const uint32_t *__restrict__ keys,
                  const uint32_t *__restrict__ pos, int64_t n, int64_t rows, float scale, int accumulate,
                  TT *__restrict__ table, int64_t ld_table, uint32_t *__restrict__ begins, float *__restrict__ part, int dpad, int chunks, int len) {
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (chunk >= chunks) return;
    const int64_t first = (int64_t)chunk * len;
    int m = (int)(n - first < len ? n - first : len);
    const uint32_t none = 0xffffffffu;
    const uint32_t key = lane < m ? keys[first + lane] : none, p = lane < m ? pos[first + lane] : 0;
    const uint32_t prev = lane < m && first + lane > 0 ? keys[first + lane - 1] : none;
    const uint32_t next = lane < m && first + lane + 1 < n ? keys[first + lane + 1] : none;
    const bool head = lane < m && key != prev, tail = lane < m && key != next;
    if (blockIdx.y == 0 && head && key < (uint64_t)rows) begins[key] = (uint32_t)(first + lane);
    const uint64_t heads = __ballot(head), tails = __ballot(tail);
    m = __popcll(__ballot(key < (uint64_t)rows));  // (ids that take no part come last)
    const int col = (int)blockIdx.y * 64 * E + lane * E, left = d - col;
    const TG *g = grad + col;
    vec_pack<TG, E> v[8], ahead[8];
    auto request = [&](int i0) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            ahead[u] = vec_load<TG, E>(g + (int64_t)__builtin_amdgcn_readlane(p, (i0 + u) & 63) * ld_grad, i0 + u < m ? left : 0, col);
    };
    vec_f<E> acc = (vec_f<E>)0.0f;
    bool whole = heads & 1;  // the run that is being added has begun here
    if (m > 0) request(0);
    for (int i0 = 0; i0 < m; i0 += 8) {
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = ahead[u];
        if (i0 + 8 < m) request(i0 + 8);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const int i = i0 + u;
            if (i >= m) break;
            acc += vec_wide<TG, E>(v[u]);
            if (tails >> i & 1) {
                if (whole) grad_write<TT, E>(table + (int64_t)__builtin_amdgcn_readlane(key, i) * ld_table, col, left, acc, scale, accumulate);
                else if (left > 0) *(vec_f<E> *)(part + (int64_t)chunk * 2 * dpad + col) = acc;  // (began before this piece)
                acc = (vec_f<E>)0.0f;
                whole = true;
            }
        }
    }
    if (m > 0 && !(tails >> (m - 1) & 1) && left > 0)  // goes on behind this piece
        *(vec_f<E> *)(part + ((int64_t)chunk * 2 + (whole ? 1 : 0)) * dpad + col) = acc;
}

// The run that ends in a piece and began before it: its partial sums added in order, by a wave, or by the block, a share of them per
// wave, if they are many.  64 E columns from blockIdx.y 64 E on.
#define GRAD_JOIN_ALONE 16
#define GRAD_JOIN_WAVES 8  // (us with 4 / 8 / 16: 262,144 ids into 500 x 64 42.3 / 39.7 / 40.6, 5,000 into 65,536 x 256 43.0 / 43.7 / 45.1)
template <class TT, int E>
__global__ void __launch_bounds__(64 * GRAD_JOIN_WAVES)
k_vec_grad_join(const uint32_t *__restrict__ keys, int64_t n, const uint32_t *__restrict__ begins, const float *__restrict__ part, int dpad,
                int d, float scale, int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table, int chunks, int len) {
    __shared__ vec_f<E> share[GRAD_JOIN_WAVES][64];
    __shared__ int many[GRAD_JOIN_WAVES];  // a wave's run, if the block is to take it: its first piece
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, first_chunk = blockIdx.x * GRAD_JOIN_WAVES + 1, chunk = first_chunk + wave;
    const int col = (int)blockIdx.y * 64 * E + lane * E;
    auto sum = [&](int c0, int from, int to) {
        vec_f<E> acc = (vec_f<E>)0.0f;
        if (col < d) {
#pragma unroll 8
            for (int c = from; c < to; ++c) acc += *(const vec_f<E> *)(part + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * dpad + col);
        }
        return acc;
    };
    auto write = [&](int c, vec_f<E> acc) {
        grad_write<TT, E>(table + (int64_t)keys[(int64_t)c * len] * ld_table, col, d - col, acc, scale, accumulate);
    };
    int c0 = -1;
    if (chunk < chunks) {
        const int64_t first = (int64_t)chunk * len, behind = first + len;
        const uint32_t key = keys[first], prev = keys[first - 1], last = behind < n ? keys[behind - 1] : 0, next = behind < n ? keys[behind] : 1;
        // (a run that goes on is a later piece's)
        if (key < (uint64_t)rows && prev == key && !(last == key && next == key)) c0 = (int)(begins[key] / (uint32_t)len);
    }
    const bool all = c0 >= 0 && chunk - c0 >= GRAD_JOIN_ALONE;
    if (lane == 0) many[wave] = all ? c0 : -1;
    if (c0 >= 0 && !all) write(chunk, sum(c0, c0, chunk + 1));
    __syncthreads();
    for (int w = 0; w < GRAD_JOIN_WAVES; ++w) {
        const int at = many[w], c1 = first_chunk + w + 1;
        if (at < 0) continue;
        const int each = (c1 - at + GRAD_JOIN_WAVES - 1) / GRAD_JOIN_WAVES, from = at + wave * each;
        vec_f<E> acc = sum(at, from < c1 ? from : c1, from + each < c1 ? from + each : c1);
        share[wave][lane] = acc;
        __syncthreads();
        if (wave == 0) {
#pragma unroll
            for (int q = 1; q < GRAD_JOIN_WAVES; ++q) acc += share[q][lane];
            write(c1 - 1, acc);
        }
        __syncthreads();
    }
}

extern "C" int vec_lookup_grad(const void *grad, int64_t n, int d, int64_t ld_grad, int grad_type, const void *ids, int id_bytes,
                               float scale, int accumulate, void *table_grad, int64_t rows, int64_t ld_table, int table_type,
                               void *workspace, size_t workspace_bytes, void *stream) {
    VEC_REQUIRE(n >= 0 && rows >= 0 && d >= 1 && d <= VEC_MAX_ROW_DIM && n <= 0x7fffffffLL && rows <= 0x7ffffffeLL, "vec_lookup_grad: n=%lld, rows=%lld, d=%d",
                (long long)n, (long long)rows, d);
    VEC_REQUIRE(vec_is_wide(grad_type) && vec_is_wide(table_type), "vec_lookup_grad: types %d and %d are not F32, BF16 or F16", grad_type, table_type);
    VEC_REQUIRE(id_bytes == 4 || id_bytes == 8, "vec_lookup_grad: ids of %d bytes", id_bytes);
    VEC_REQUIRE(ld_grad >= d && ld_table >= d, "vec_lookup_grad: rows of %lld and %lld elements hold no %d", (long long)ld_grad, (long long)ld_table, d);
    if (rows == 0 || (n == 0 && accumulate)) return PQ_OK;
    VEC_REQUIRE(table_grad && (n == 0 || (grad && ids)), "vec_lookup_grad: null pointer");
    VEC_REQUIRE(vec_aligned(grad, grad_type) && vec_aligned(table_grad, table_type) && ((uintptr_t)ids & (uintptr_t)(id_bytes - 1)) == 0,
                "vec_lookup_grad: misaligned pointer");
    const GradPlan p = grad_plan(n, rows, d);
    if (p.total > 0) {
        VEC_REQUIRE(workspace && ((uintptr_t)workspace & 255u) == 0, "vec_lookup_grad: workspace null or not 256-byte aligned");
        if (workspace_bytes < p.total) {
            qadc_set_error("vec_lookup_grad: workspace of %zu bytes, %zu needed", workspace_bytes, p.total);
            return PQ_ENOMEM;
        }
    }
    hipStream_t s = (hipStream_t)stream;
    if (p.few) {
        // 512 bytes of neighbouring rows together; at least about 1024 blocks (at most 2^15 rows each, a group more: a row of a block shares a word with a position)
        int group = 0, deal = 0;
        while (group < 5 && ((int64_t)vec_bytes(table_type) * d << group) < 512) ++group;
        const int tiles = (d + 511) / 512;  // (of 64 E columns: d > 256 has E = 8)
        while (((int64_t)tiles << deal) < 1024 && ((int64_t)4 << group << deal) < rows) ++deal;
        while ((rows >> (deal + 15)) > 0) ++deal;
        const int64_t groups = (rows + ((int64_t)1 << group) - 1) >> group, each = (groups + ((int64_t)1 << deal) - 1) >> deal;
        const int rpb = (int)(each << group);
        const size_t lds = (size_t)((rpb + 31) / 32) * 4 + (size_t)(n + 255) / 256 * 256 * 4;
#define GO(TG, TT, ID, E)                                                                                                  \
    hipLaunchKernelGGL((k_vec_grad_few<TG, TT, ID, E>), dim3(1u << deal, (unsigned)tiles), dim3(256), lds, s, (const TG *)grad, (int)n, d, \
                       ld_grad, (const ID *)ids, scale, accumulate, (TT *)table_grad, rows, ld_table, group, deal, rpb)
        VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, if (id_bytes == 4) GO(TG, TT, int32_t, E); else GO(TG, TT, int64_t, E))));
#undef GO
        QADC_LAUNCH_CHECK("k_vec_grad_few");
        return PQ_OK;
    }
    char *ws = (char *)workspace;
    uint32_t *key[2] = {(uint32_t *)(ws + p.key0), (uint32_t *)(ws + p.key1)}, *pos[2] = {(uint32_t *)(ws + p.pos0), (uint32_t *)(ws + p.pos1)};
    uint32_t *counts = (uint32_t *)(ws + p.counts);
    uint32_t *sums = (uint32_t *)(ws + p.sums), *totals = sums + ((size_t)p.segs << p.bits);
    uint32_t *begins = (uint32_t *)(ws + p.begins);
    float *part = (float *)(ws + p.part);
    // a pass's share of the rows to clear, 32 KB and more a block
    const size_t row_bytes = vec_bytes(table_type) * (size_t)d;
    GradClear z = {table_grad, 0, 0, ld_table, d, (int)(row_bytes >= 32768 ? 1 : 32768 / row_bytes), 0};
    auto share = [&](int pass, unsigned own) {
        z.after = (int)own;
        z.lo = z.hi;
        z.hi = accumulate ? 0 : rows * (pass + 1) / p.passes;
        int64_t blocks = (z.hi - z.lo + z.each - 1) / z.each;
        while (blocks > (1 << 20)) {
            z.each *= 2;
            blocks = (z.hi - z.lo + z.each - 1) / z.each;
        }
        return dim3(own + (unsigned)blocks);
    };
    for (int pass = 0; pass < p.passes; ++pass) {
        const uint32_t *ki = pass ? key[(pass - 1) & 1] : nullptr, *pi = pass ? pos[(pass - 1) & 1] : nullptr;
        const int shift = pass * p.bits;
        if (id_bytes == 4)
            hipLaunchKernelGGL((k_vec_grad_count<int32_t>), dim3((unsigned)p.tiles), dim3(1024), 0, s, (const int32_t *)ids, ki, n, rows, shift, p.bits, counts);
        else
            hipLaunchKernelGGL((k_vec_grad_count<int64_t>), dim3((unsigned)p.tiles), dim3(1024), 0, s, (const int64_t *)ids, ki, n, rows, shift, p.bits, counts);
        if (p.segs > 0) {
            const dim3 threads(p.bits < 6 ? 64 : 1u << p.bits);
            hipLaunchKernelGGL(k_vec_grad_running, dim3((unsigned)p.segs), threads, 0, s, counts, p.tiles, p.seg, p.bits, sums);
            hipLaunchKernelGGL(k_vec_grad_running, dim3(1), threads, 0, s, sums, p.segs, p.segs, p.bits, totals);
        }
        const dim3 grid = share(pass, (unsigned)p.tiles);
#define GO(ID, TT)                                                                                                         \
    hipLaunchKernelGGL((k_vec_grad_place<ID, TT>), grid, dim3(1024), (size_t)64 << p.bits, s, (const ID *)ids, ki, pi, n, rows, shift, p.bits, \
                       counts, p.tiles, p.seg, sums, totals, key[pass & 1], pos[pass & 1], z)
        VEC_TYPED(table_type, TT, if (id_bytes == 4) GO(int32_t, TT); else GO(int64_t, TT));
#undef GO
    }
    const uint32_t *ks = key[(p.passes - 1) & 1], *ps = pos[(p.passes - 1) & 1];
    VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, hipLaunchKernelGGL(
        (k_vec_grad_chunks<TG, TT, E>), dim3((unsigned)((p.chunks + 3) / 4), (unsigned)((d + 64 * E - 1) / (64 * E))), dim3(256), 0, s, (const TG *)grad,
        d, ld_grad, ks, ps, n, rows, scale, accumulate, (TT *)table_grad, ld_table, begins, part, p.dpad, p.chunks, p.len))));
    VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, hipLaunchKernelGGL((k_vec_grad_join<TT, E>), dim3((unsigned)((p.chunks + GRAD_JOIN_WAVES - 2) / GRAD_JOIN_WAVES), (unsigned)((d + 64 * E - 1) / (64 * E))),
                                                                dim3(64 * GRAD_JOIN_WAVES), 0, s, ks, n, begins, part, p.dpad, d, scale, accumulate, (TT *)table_grad, rows, ld_table, p.chunks, p.len)));
    QADC_LAUNCH_CHECK("vec_lookup_grad's kernels");
    return PQ_OK;
}
