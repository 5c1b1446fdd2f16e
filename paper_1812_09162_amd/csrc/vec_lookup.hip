// vec_lookup and vec_lookup_grad: rows of a table by id, and the sum of gradients by id.
#include "vec_device.h"

// ------------------------------------------------------------------ look-up --
// out[i] = scale * table[ids[i]].  A block copies `rpb` neighbouring rows of the result as pieces of eight elements; bound by
// memory: every piece is one wide load behind a load of the row's id, eight of them in flight per thread.
template <class TI, class TO, class ID>
__global__ void __launch_bounds__(256)
k_vec_lookup(const TI *__restrict__ table, int64_t rows, int d, int64_t ld_table, const ID *__restrict__ ids, int64_t n,
             float scale, TO *__restrict__ out, int64_t ld_out, int rpb, int pieces, uint32_t magic) {
    const int64_t row0 = (int64_t)blockIdx.x * rpb;
    const int nrow = (int)(n - row0 < rpb ? n - row0 : rpb);
    const int total = nrow * pieces;
    for (int e0 = threadIdx.x; e0 < total; e0 += 256 * 4) {
        vec_pack<TI> v[4];
        int64_t to[4];
        int left[4];
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
            to[u] = (row0 + r) * ld_out + col;
            v[u] = vec_load(table + (known ? id * ld_table + col : 0), known ? left[u] : 0);
        }
#pragma unroll
        for (int u = 0; u < 4; ++u)
            if (left[u] > 0) {
                vec_f8 f = vec_wide<TI>(v[u]);
#pragma unroll
                for (int i = 0; i < 8; ++i) f[i] *= scale;
                vec_store(out + to[u], left[u], f);
            }
    }
}

extern "C" int vec_lookup(const void *table, int64_t rows, int d, int64_t ld_table, int table_type, const void *ids,
                          int id_bytes, int64_t n, float scale, void *out, int64_t ld_out, int out_type, void *stream) {
    VEC_REQUIRE(n >= 0 && rows >= 0 && d >= 1, "vec_lookup: n=%lld, rows=%lld, d=%d", (long long)n, (long long)rows, d);
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
    VEC_REQUIRE(blocks <= 0x7fffffffLL, "vec_lookup: n=%lld too large for one call", (long long)n);
    // e / pieces for e < 1024, pieces > 1: exact as 1024 pieces < 2^32
    const uint32_t magic = (uint32_t)((((uint64_t)1 << 32) + pieces - 1) / pieces);
    hipStream_t s = (hipStream_t)stream;
#define GO(TI, TO, ID)                                                                                                    \
    hipLaunchKernelGGL((k_vec_lookup<TI, TO, ID>), dim3((unsigned)blocks), dim3(256), 0, s, (const TI *)table, rows, d,    \
                       ld_table, (const ID *)ids, n, scale, (TO *)out, ld_out, rpb, pieces, magic)
    VEC_TYPED(table_type, TI, VEC_TYPED(out_type, TO, if (id_bytes == 4) GO(TI, TO, int32_t); else GO(TI, TO, int64_t)));
#undef GO
    QADC_LAUNCH_CHECK("k_vec_lookup");
    return PQ_OK;
}

// ----------------------------------------------------------------- gradient --
// table_grad[v] = base + scale * sum of the rows of grad whose id is v.  Positions with the same id are summed in ascending
// order in float32, so that a result does not depend on which block ran first.
//
// Few ids (n <= GRAD_FEW): one launch.  Every block owns a range of table rows, goes through all ids, keeps the positions
// of its own in order, and writes its rows, zeros or sums.  The ids are read once per block, from the L2 cache.
//
// Many: the positions are sorted by id (a stable radix sort of up to 2^GRAD_BITS buckets a pass), then summed in pieces
// of GRAD_CHUNK sorted positions, whatever ids they hold, so that a frequent id is no wave's alone; sums of ids that cross
// a piece's ends are joined by the kernel that also writes the rows without an id.
#define GRAD_FEW 4096
#define GRAD_BITS 10
#define GRAD_TILE 1024   // keys a block of the sort takes: four per thread
#define GRAD_CHUNK 64

struct GradPlan {
    bool few;
    int passes, bits;   // of the sort
    int tiles, chunks;  // blocks of a pass; pieces of the sum
    int dpad;           // floats of a partial row
    size_t key0, key1, pos0, pos1, counts, totals, bounds, part, total;
};

static GradPlan grad_plan(int64_t n, int64_t rows, int d) {
    GradPlan p = {};
    p.few = n <= GRAD_FEW;
    if (p.few) return p;
    int bits = 1;
    while (((int64_t)1 << bits) <= rows) ++bits;  // ids 0..rows, `rows` standing for those that take no part
    p.passes = (bits + GRAD_BITS - 1) / GRAD_BITS;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.tiles = (int)((n + GRAD_TILE - 1) / GRAD_TILE);
    p.chunks = (int)((n + GRAD_CHUNK - 1) / GRAD_CHUNK);
    p.dpad = (d + 7) & ~7;
    size_t at = 0;
    auto take = [&](size_t bytes) { const size_t was = at; at += vec_up256(bytes); return was; };
    p.key0 = take((size_t)n * 4);
    p.key1 = take((size_t)n * 4);
    p.pos0 = take((size_t)n * 4);
    p.pos1 = take((size_t)n * 4);
    p.counts = take(((size_t)p.tiles << p.bits) * 4);
    p.totals = take(((size_t)1 << p.bits) * 4);
    p.bounds = take((size_t)rows * 8);
    p.part = take((size_t)p.chunks * 2 * p.dpad * 4);
    p.total = at;
    return p;
}

extern "C" size_t vec_lookup_grad_workspace_bytes(int64_t n, int64_t rows, int d) {
    return n <= 0 || rows <= 0 || d <= 0 || n > 0x7fffffffLL || rows > 0x7ffffffeLL ? 0 : grad_plan(n, rows, d).total;
}

// Adds the rows of grad at the positions pos(0) .. pos(m - 1), eight columns from col on, in this order to acc.
template <class TG, class POS>
__device__ __forceinline__ void grad_sum(const TG *__restrict__ grad, int64_t ld, int64_t col, int64_t left, int m, POS pos, vec_f8 &acc) {
    int i = 0;
    for (; i + 8 <= m; i += 8) {
        vec_pack<TG> v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = vec_load(grad + (int64_t)pos(i + u) * ld + col, left);
#pragma unroll
        for (int u = 0; u < 8; ++u) acc += vec_wide<TG>(v[u]);
    }
    for (; i < m; ++i) acc += vec_wide<TG>(vec_load(grad + (int64_t)pos(i) * ld + col, left));
}

template <class TT>
__device__ __forceinline__ void grad_write(TT *__restrict__ row, int64_t col, int64_t left, vec_f8 acc, float scale, int accumulate) {
    vec_f8 f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = acc[i] * scale;
    if (accumulate) f += vec_wide<TT>(vec_load(row + col, left));
    vec_store(row + col, left, f);
}

// Zeros in the rows lo .. lo + nrow - 1 whose bit of `has` is not set.
template <class TT>
__device__ __forceinline__ void grad_zeros(TT *__restrict__ table, int64_t lo, int nrow, int d, int64_t ld, const uint32_t *has) {
    const int pieces = (d + 7) / 8;
    int r = threadIdx.x / pieces, c = threadIdx.x - r * pieces;
    const int dr = 256 / pieces, dc = 256 - dr * pieces;
    for (; r < nrow;) {
        if (!(has[r >> 5] >> (r & 31) & 1)) vec_store<TT>(table + (lo + r) * ld + c * 8, d - c * 8, (vec_f8)0.0f);
        r += dr;
        c += dc;
        if (c >= pieces) c -= pieces, ++r;
    }
}

template <class TG, class TT, class ID>
__global__ void __launch_bounds__(256)
k_vec_grad_few(const TG *__restrict__ grad, int n, int d, int64_t ld_grad, const ID *__restrict__ ids, float scale,
               int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table, int rpb) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t *has = (uint32_t *)smem;                      // [(rpb + 31) / 32]
    uint32_t *list = has + (rpb + 31) / 32;                // [GRAD_FEW] row of the block << 12 | position
    uint16_t *picked = (uint16_t *)(list + GRAD_FEW);      // [4 waves][GRAD_FEW / 4 ...] see below
    __shared__ int count[4];
    const int64_t lo = (int64_t)blockIdx.x * rpb;
    const int nrow = (int)(rows - lo < rpb ? rows - lo : rpb);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < (rpb + 31) / 32; i += 256) has[i] = 0;
    __syncthreads();
    // each wave takes a quarter of the positions and keeps the block's own, in order, in its quarter of the list
    const int quarter = (n + 3) / 4;
    const int from = wave * quarter, to = from + quarter < n ? from + quarter : n;
    int m = 0;
    for (int i0 = from; i0 < to; i0 += 64) {
        const int i = i0 + lane;
        const int64_t id = i < to ? (int64_t)ids[i] : -1;
        const bool mine = id >= lo && id < lo + nrow;
        const uint64_t b = __ballot(mine);
        if (mine) {
            const int r = (int)(id - lo);
            list[from + m + __popcll(b & ((1ull << lane) - 1))] = (uint32_t)r << 12 | (uint32_t)i;
            atomicOr(&has[r >> 5], 1u << (r & 31));
        }
        m += __popcll(b);
    }
    if (lane == 0) count[wave] = m;
    __syncthreads();
    if (!accumulate) grad_zeros(table, lo, nrow, d, ld_table, has);
    // rows with an id: one per wave in turn.  A wave picks the row's positions out of the lists, then sums.
    uint16_t *mine = picked + wave * GRAD_FEW;
    int turn = 0;
    for (int w = 0; w < (nrow + 31) / 32; ++w) {
        uint32_t bits = has[w];
        while (bits) {
            const int r = w * 32 + __builtin_ctz(bits);
            bits &= bits - 1;
            if ((turn++ & 3) != wave) continue;
            int k = 0;
            for (int q = 0; q < 4; ++q)
                for (int i0 = 0; i0 < count[q]; i0 += 64) {
                    const uint32_t e = i0 + lane < count[q] ? list[q * quarter + i0 + lane] : 0xffffffffu;
                    const bool hit = e >> 12 == (uint32_t)r;
                    const uint64_t b = __ballot(hit);
                    if (hit) mine[k + __popcll(b & ((1ull << lane) - 1))] = (uint16_t)(e & 4095u);
                    k += __popcll(b);
                }
            for (int col = lane * 8; col < d; col += 512) {
                vec_f8 acc = (vec_f8)0.0f;
                grad_sum(grad, ld_grad, col, d - col, k, [&](int i) { return mine[i]; }, acc);
                grad_write(table + (lo + r) * ld_table, col, d - col, acc, scale, accumulate);
            }
        }
    }
}

// --- the sort.  counts[bucket][tile] -> where a tile's keys of a bucket go within it; totals[bucket] -> where a bucket begins
template <class ID>
__device__ __forceinline__ uint32_t grad_key(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t i, int64_t rows) {
    if (keys) return keys[i];
    const int64_t id = (int64_t)ids[i];
    return id >= 0 && id < rows ? (uint32_t)id : (uint32_t)rows;
}

template <class ID>
__global__ void __launch_bounds__(256)
k_vec_grad_count(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, int64_t n, int64_t rows, int shift, int bits,
                 uint32_t *__restrict__ counts, int tiles, uint2 *__restrict__ bounds) {
    __shared__ uint32_t h[1 << GRAD_BITS];
    const int nb = 1 << bits;
    for (int i = threadIdx.x; i < nb; i += 256) h[i] = 0;
    __syncthreads();
    for (int u = 0; u < GRAD_TILE / 256; ++u) {
        const int64_t i = (int64_t)blockIdx.x * GRAD_TILE + u * 256 + threadIdx.x;
        if (i < n) atomicAdd(&h[grad_key(ids, keys, i, rows) >> shift & (nb - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < nb; i += 256) counts[(size_t)i * tiles + blockIdx.x] = h[i];
    if (bounds)  // (first pass: no row has an id yet)
        for (int64_t v = (int64_t)blockIdx.x * 256 + threadIdx.x; v < rows; v += (int64_t)gridDim.x * 256) bounds[v] = make_uint2(0, 0);
}

// a wave per bucket: running sums over the tiles
__global__ void __launch_bounds__(256)
k_vec_grad_scan(uint32_t *__restrict__ counts, int tiles, int nb, uint32_t *__restrict__ totals) {
    const int b = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= nb) return;
    uint32_t *c = counts + (size_t)b * tiles, sum = 0;
    for (int t0 = 0; t0 < tiles; t0 += 64) {
        const uint32_t v = t0 + lane < tiles ? c[t0 + lane] : 0;
        uint32_t s = v;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) {
            const uint32_t x = __shfl_up(s, o);
            if (lane >= o) s += x;
        }
        if (t0 + lane < tiles) c[t0 + lane] = sum + s - v;
        sum += __shfl(s, 63);
    }
    if (lane == 0) totals[b] = sum;
}

// A tile's keys to their places: those of one bucket keep their order.  Wave w holds the tile's w-th quarter, 64 keys at a
// time; a key's rank among them is the number of lower lanes with the same bucket, found bit by bit with ballots.
template <class ID>
__global__ void __launch_bounds__(256)
k_vec_grad_place(const ID *__restrict__ ids, const uint32_t *__restrict__ keys, const uint32_t *__restrict__ pos, int64_t n,
                 int64_t rows, int shift, int bits, const uint32_t *__restrict__ counts, int tiles,
                 const uint32_t *__restrict__ totals, uint32_t *__restrict__ keys_out, uint32_t *__restrict__ pos_out) {
    __shared__ uint32_t next[4][1 << GRAD_BITS];  // per wave: where its next key of a bucket goes
    __shared__ uint32_t part[4];
    const int nb = 1 << bits, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    for (int i = threadIdx.x; i < 4 * nb; i += 256) next[i >> bits][i & (nb - 1)] = 0;
    __syncthreads();
    const int64_t first = (int64_t)blockIdx.x * GRAD_TILE + wave * (GRAD_TILE / 4);
    uint32_t key[GRAD_TILE / 256], bucket[GRAD_TILE / 256];
#pragma unroll
    for (int u = 0; u < GRAD_TILE / 256; ++u) {
        const int64_t i = first + u * 64 + lane;
        key[u] = i < n ? grad_key(ids, keys, i, rows) : 0;
        bucket[u] = key[u] >> shift & (nb - 1);
        if (i < n) atomicAdd(&next[wave][bucket[u]], 1u);
    }
    __syncthreads();
    // where each bucket begins: running sums over the totals, four buckets per thread at most
    const int per = (nb + 255) / 256;
    uint32_t mine[(1 << GRAD_BITS) / 256], sum = 0;
#pragma unroll
    for (int j = 0; j < (1 << GRAD_BITS) / 256; ++j) {
        const int b = threadIdx.x * per + j;
        mine[j] = j < per && b < nb ? totals[b] : 0;
        sum += mine[j];
    }
    uint32_t s = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t x = __shfl_up(s, o);
        if (lane >= o) s += x;
    }
    if (lane == 63) part[wave] = s;
    __syncthreads();
    uint32_t before = s - sum;
    for (int w = 0; w < wave; ++w) before += part[w];
#pragma unroll
    for (int j = 0; j < (1 << GRAD_BITS) / 256; ++j) {
        const int b = threadIdx.x * per + j;
        if (j < per && b < nb) {
            uint32_t at = before + counts[(size_t)b * tiles + blockIdx.x];
            for (int w = 0; w < 4; ++w) {
                const uint32_t c = next[w][b];
                next[w][b] = at;
                at += c;
            }
        }
        before += mine[j];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < GRAD_TILE / 256; ++u) {
        const int64_t i = first + u * 64 + lane;
        const bool in = i < n;
        uint64_t same = __ballot(in);
        for (int b = 0; b < bits; ++b) {
            const uint64_t x = __ballot(bucket[u] >> b & 1);
            same &= bucket[u] >> b & 1 ? x : ~x;
        }
        if (in) {
            const int rank = __popcll(same & ((1ull << lane) - 1));
            const uint32_t at = next[wave][bucket[u]] + rank;
            keys_out[at] = key[u];
            pos_out[at] = pos ? pos[i] : (uint32_t)i;
        }
        __builtin_amdgcn_wave_barrier();  // the reads above come before the wave's own update
        if (in && (same >> lane) == 1) next[wave][bucket[u]] += __popcll(same);  // the bucket's last lane
        __builtin_amdgcn_wave_barrier();
    }
}

// --- the sums.  A wave per piece of GRAD_CHUNK sorted positions and 512 columns: ids that lie within the piece are written to
// the table; the sum of the one that the piece begins with, if it began before, goes to part[chunk][0]; that of the one it ends
// with, if it goes on, to part[chunk][1] (to [0] if it is the same).  bounds[v]: first and last + 1 sorted position of id v.
template <class TG, class TT>
__global__ void __launch_bounds__(256)
k_vec_grad_chunks(const TG *__restrict__ grad, int d, int64_t ld_grad, const uint32_t *__restrict__ keys,
                  const uint32_t *__restrict__ pos, int64_t n, int64_t rows, float scale, int accumulate,
                  TT *__restrict__ table, int64_t ld_table, uint2 *__restrict__ bounds, float *__restrict__ part, int dpad, int chunks) {
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (chunk >= chunks) return;
    const int64_t first = (int64_t)chunk * GRAD_CHUNK;
    const int m = (int)(n - first < GRAD_CHUNK ? n - first : GRAD_CHUNK);
    const uint32_t none = 0xffffffffu;
    const uint32_t key = lane < m ? keys[first + lane] : none, p = lane < m ? pos[first + lane] : 0;
    const uint32_t prev = lane < m && first + lane > 0 ? keys[first + lane - 1] : none;
    const uint32_t next = lane < m && first + lane + 1 < n ? keys[first + lane + 1] : none;
    const bool begins = lane < m && key != prev, ends = lane < m && key != next;
    if (blockIdx.y == 0 && key < (uint64_t)rows) {
        if (begins) bounds[key].x = (uint32_t)(first + lane);
        if (ends) bounds[key].y = (uint32_t)(first + lane) + 1;
    }
    uint64_t heads = __ballot(begins) | 1ull;  // where an id's run within the piece starts
    const bool first_whole = __ballot(begins) & 1, last_whole = __ballot(ends) >> (m - 1) & 1;
    const int col = blockIdx.y * 512 + lane * 8;
    while (heads) {
        const int at = __builtin_ctzll(heads);
        heads &= heads - 1;
        const int to = heads ? __builtin_ctzll(heads) : m;
        const uint32_t k = __builtin_amdgcn_readlane(key, at);
        if (k >= (uint64_t)rows) break;  // ids that take no part come last
        vec_f8 acc = (vec_f8)0.0f;
        if (col < d) grad_sum(grad, ld_grad, col, d - col, to - at, [&](int i) { return __builtin_amdgcn_readlane(p, at + i); }, acc);
        const bool whole = (at > 0 || first_whole) && (to < m || last_whole);
        if (col >= d) continue;
        if (whole) grad_write(table + (int64_t)k * ld_table, col, d - col, acc, scale, accumulate);
        else *(vec_f8 *)(part + ((int64_t)chunk * 2 + (at > 0)) * dpad + col) = acc;
    }
}

// Rows without an id, and those whose run crosses the end of a piece: partial sums in order, a quarter of them per wave.
#define GRAD_END_ROWS 64
template <class TT>
__global__ void __launch_bounds__(256)
k_vec_grad_end(const uint2 *__restrict__ bounds, const float *__restrict__ part, int dpad, int d, float scale,
               int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table) {
    __shared__ uint32_t has[GRAD_END_ROWS / 32], cross[GRAD_END_ROWS / 32];
    __shared__ uint2 bound[GRAD_END_ROWS];
    __shared__ vec_f8 quarter[4][64];
    const int64_t lo = (int64_t)blockIdx.x * GRAD_END_ROWS;
    const int nrow = (int)(rows - lo < GRAD_END_ROWS ? rows - lo : GRAD_END_ROWS);
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if (threadIdx.x < 64) {
        const uint2 b = lane < nrow ? bounds[lo + lane] : make_uint2(0, 0);
        bound[lane] = b;
        const uint64_t h = __ballot(b.y > b.x), c = __ballot(b.y > b.x && b.x / GRAD_CHUNK != (b.y - 1) / GRAD_CHUNK);
        if (lane < 2) has[lane] = (uint32_t)(h >> (32 * lane)), cross[lane] = (uint32_t)(c >> (32 * lane));
    }
    __syncthreads();
    if (!accumulate) grad_zeros(table, lo, nrow, d, ld_table, has);
    for (int r = 0; r < nrow; ++r) {
        if (!(cross[r >> 5] >> (r & 31) & 1)) continue;
        const int c0 = (int)(bound[r].x / GRAD_CHUNK), c1 = (int)((bound[r].y - 1) / GRAD_CHUNK);
        // a run is the piece's second part where it starts within it, else its first
        const int slot0 = bound[r].x % GRAD_CHUNK ? 1 : 0;
        const int cnt = c1 - c0 + 1, each = (cnt + 3) / 4;
        const int a = c0 + wave * each, b = a + each < c1 + 1 ? a + each : c1 + 1;
        for (int col0 = 0; col0 < d; col0 += 512) {
            const int col = col0 + lane * 8;
            vec_f8 acc = (vec_f8)0.0f;
            if (col < d) {
                const float *p = part + col;
#pragma unroll 4
                for (int c = a; c < b; ++c) acc += *(const vec_f8 *)(p + ((int64_t)c * 2 + (c == c0 ? slot0 : 0)) * dpad);
            }
            quarter[wave][lane] = acc;
            __syncthreads();
            if (wave == 0 && col < d) {
#pragma unroll
                for (int w = 1; w < 4; ++w) acc += quarter[w][lane];
                grad_write(table + (lo + r) * ld_table, col, d - col, acc, scale, accumulate);
            }
            __syncthreads();
        }
    }
}

extern "C" int vec_lookup_grad(const void *grad, int64_t n, int d, int64_t ld_grad, int grad_type, const void *ids, int id_bytes,
                               float scale, int accumulate, void *table_grad, int64_t rows, int64_t ld_table, int table_type,
                               void *workspace, size_t workspace_bytes, void *stream) {
    VEC_REQUIRE(n >= 0 && rows >= 0 && d >= 1 && n <= 0x7fffffffLL && rows <= 0x7ffffffeLL, "vec_lookup_grad: n=%lld, rows=%lld, d=%d",
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
        // 1024 blocks, four per CU; the row of a block and a position share a word, so at most 2^19 rows a block
        int64_t rpb = (rows + 1023) / 1024;
        if (rpb < 8) rpb = 8;
        if (rpb > 65536) rpb = 65536;
        const int64_t blocks = (rows + rpb - 1) / rpb;
        const size_t lds = (size_t)((rpb + 31) / 32) * 4 + GRAD_FEW * 4 + 4 * GRAD_FEW * 2;
#define GO(TG, TT, ID)                                                                                                     \
    do {                                                                                                                   \
        if (lds > 64 * 1024)                                                                                               \
            QADC_HIP_TRY(hipFuncSetAttribute((const void *)k_vec_grad_few<TG, TT, ID>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds)); \
        hipLaunchKernelGGL((k_vec_grad_few<TG, TT, ID>), dim3((unsigned)blocks), dim3(256), lds, s, (const TG *)grad, (int)n, d, \
                           ld_grad, (const ID *)ids, scale, accumulate, (TT *)table_grad, rows, ld_table, (int)rpb);        \
    } while (0)
        VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, if (id_bytes == 4) GO(TG, TT, int32_t); else GO(TG, TT, int64_t)));
#undef GO
        QADC_LAUNCH_CHECK("k_vec_grad_few");
        return PQ_OK;
    }
    char *ws = (char *)workspace;
    uint32_t *key[2] = {(uint32_t *)(ws + p.key0), (uint32_t *)(ws + p.key1)}, *pos[2] = {(uint32_t *)(ws + p.pos0), (uint32_t *)(ws + p.pos1)};
    uint32_t *counts = (uint32_t *)(ws + p.counts), *totals = (uint32_t *)(ws + p.totals);
    uint2 *bounds = (uint2 *)(ws + p.bounds);
    float *part = (float *)(ws + p.part);
    const int nb = 1 << p.bits;
    for (int pass = 0; pass < p.passes; ++pass) {
        const uint32_t *ki = pass ? key[(pass - 1) & 1] : nullptr, *pi = pass ? pos[(pass - 1) & 1] : nullptr;
        const int shift = pass * p.bits;
#define GO(ID)                                                                                                             \
    do {                                                                                                                   \
        hipLaunchKernelGGL(k_vec_grad_count<ID>, dim3(p.tiles), dim3(256), 0, s, (const ID *)ids, ki, n, rows, shift, p.bits, counts, \
                           p.tiles, pass ? (uint2 *)nullptr : bounds);                                                     \
        hipLaunchKernelGGL(k_vec_grad_scan, dim3((nb + 3) / 4), dim3(256), 0, s, counts, p.tiles, nb, totals);             \
        hipLaunchKernelGGL(k_vec_grad_place<ID>, dim3(p.tiles), dim3(256), 0, s, (const ID *)ids, ki, pi, n, rows, shift, p.bits, \
                           counts, p.tiles, totals, key[pass & 1], pos[pass & 1]);                                         \
    } while (0)
        if (id_bytes == 4) GO(int32_t);
        else GO(int64_t);
#undef GO
    }
    const uint32_t *ks = key[(p.passes - 1) & 1], *ps = pos[(p.passes - 1) & 1];
    const dim3 grid((unsigned)((p.chunks + 3) / 4), (unsigned)((d + 511) / 512));
    VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, hipLaunchKernelGGL((k_vec_grad_chunks<TG, TT>), grid, dim3(256), 0, s, (const TG *)grad, d,
                                                                         ld_grad, ks, ps, n, rows, scale, accumulate, (TT *)table_grad, ld_table,
                                                                         bounds, part, p.dpad, p.chunks)));
    VEC_TYPED(table_type, TT, hipLaunchKernelGGL((k_vec_grad_end<TT>), dim3((unsigned)((rows + GRAD_END_ROWS - 1) / GRAD_END_ROWS)), dim3(256), 0, s,
                                                 bounds, part, p.dpad, d, scale, accumulate, (TT *)table_grad, rows, ld_table));
    QADC_LAUNCH_CHECK("vec_lookup_grad's kernels");
    return PQ_OK;
}
