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
// order in float32, in pieces that do not depend on which block ran first.
//
// Few ids (n <= GRAD_FEW): one launch.  Every block owns some rows of the table, dealt out in turn since frequent ids are often
// neighbours; it goes through all ids, keeps the positions of its own in order, and writes its rows, zeros or sums.  The ids
// are read once per block, from the L2 cache.
//
// Many: the positions are sorted by id (a stable radix sort of up to 2^GRAD_BITS buckets a pass), then summed in pieces
// of GRAD_CHUNK sorted positions, whatever ids they hold, so that a frequent id is no wave's alone; sums of ids that cross
// a piece's ends are joined by the kernel that also writes the rows without an id.
//
// A row is spread over the 64 lanes of a wave, E elements each (2, 4 or 8, the fewest that hold it, else 64 E columns at a time).
#define GRAD_FEW 4096
#define GRAD_BITS 10
#define GRAD_TILE 1024   // keys a block of the sort takes: four per thread
#define GRAD_CHUNK 64

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

template <class TT, int E>
__device__ __forceinline__ void grad_write(TT *__restrict__ row, int64_t col, int64_t left, vec_f<E> acc, float scale, int accumulate) {
    if (left <= 0) return;
    vec_f<E> f;
#pragma unroll
    for (int i = 0; i < E; ++i) f[i] = acc[i] * scale;
    if (accumulate) f += vec_wide<TT, E>(vec_load<TT, E>(row + col, left));
    vec_store<TT, E>(row + col, left, f);
}

// Zeros in those of `nrow` rows whose bit of `has` is not set; row(r): address of the r-th.
template <class TT, class ROW>
__device__ __forceinline__ void grad_zeros(int nrow, int d, const uint32_t *has, ROW row) {
    const int pieces = (d + 7) / 8;
    int r = threadIdx.x / pieces, c = threadIdx.x - r * pieces;
    const int dr = 256 / pieces, dc = 256 - dr * pieces;
    while (r < nrow) {
        if (!(has[r >> 5] >> (r & 31) & 1)) vec_store<TT>(row(r) + c * 8, d - c * 8, (vec_f8)0.0f);
        r += dr;
        c += dc;
        if (c >= pieces) c -= pieces, ++r;
    }
}

// Adds to acc the rows of grad at the positions (low 12 bits) of those of list[0 .. m - 1] that are of row r (the bits above), in order.
template <class TG, int E>
__device__ __forceinline__ void grad_pick(const TG *__restrict__ grad, int64_t ld, int64_t col, int64_t left, const uint32_t *list, int m,
                                          uint32_t r, vec_f<E> &acc) {
    const int lane = threadIdx.x & 63;
    for (int i0 = 0; i0 < m; i0 += 64) {
        const uint32_t e = i0 + lane < m ? list[i0 + lane] : 0xffffffffu;
        uint64_t hits = __ballot(e >> 12 == r);
        while (hits) {
            vec_pack<TG, E> v[8];
            int k = 0;
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                const int at = hits ? __builtin_ctzll(hits) : 0;
                const bool more = hits != 0;
                hits &= hits - 1;
                const uint32_t pos = __builtin_amdgcn_readlane(e, at) & 4095u;
                k += more;
                v[u] = vec_load<TG, E>(grad + (int64_t)pos * ld + col, more ? left : 0);
            }
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (u < k) acc += vec_wide<TG, E>(v[u]);
        }
    }
}

// The block's rows: groups of 2^group neighbouring rows are dealt out over 2^deal blocks.
template <class TG, class TT, class ID, int E>
__global__ void __launch_bounds__(256)
k_vec_grad_few(const TG *__restrict__ grad, int n, int d, int64_t ld_grad, const ID *__restrict__ ids, float scale,
               int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table, int group, int deal, int rpb) {
    extern __shared__ __align__(16) unsigned char smem[];
    uint32_t *has = (uint32_t *)smem;           // [(rpb + 31) / 32]
    uint32_t *list = has + (rpb + 31) / 32;     // [GRAD_FEW] row of the block << 12 | position
    __shared__ int count[4];
    __shared__ vec_f<E> quarter[4][64];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    // row r of the block is row of(r) of the table; its rows below `rows` come first
    auto of = [&](int r) { return ((((int64_t)(r >> group) << deal) + blockIdx.x) << group) + (r & ((1 << group) - 1)); };
    int nrow = rpb;
    while (nrow > 0 && of(nrow - 1) >= rows) --nrow;
    for (int i = threadIdx.x; i < (rpb + 31) / 32; i += 256) has[i] = 0;
    // each wave takes a quarter of the positions, all loads at once, and keeps the block's own, in order, in its quarter of the list
    const int per = (n + 255) / 256 * 64, from = wave * per;
    int64_t id[GRAD_FEW / 256];
#pragma unroll
    for (int u = 0; u < GRAD_FEW / 256; ++u) {
        const int i = from + u * 64 + lane;
        id[u] = u * 64 < per && i < n ? (int64_t)ids[i] : -1;
    }
    __syncthreads();
    int m = 0;
#pragma unroll
    for (int u = 0; u < GRAD_FEW / 256; ++u) {
        const bool mine = id[u] >= 0 && id[u] < rows && ((id[u] >> group) & ((1 << deal) - 1)) == blockIdx.x;
        const uint64_t b = __ballot(mine);
        if (!b) continue;
        if (mine) {
            const int r = (int)(id[u] >> (group + deal) << group) + (int)(id[u] & ((1 << group) - 1));
            list[from + m + __popcll(b & ((1ull << lane) - 1))] = (uint32_t)r << 12 | (uint32_t)(from + u * 64 + lane);
            atomicOr(&has[r >> 5], 1u << (r & 31));
        }
        m += __popcll(b);
    }
    if (lane == 0) count[wave] = m;
    __syncthreads();
    if (!accumulate) grad_zeros<TT>(nrow, d, has, [&](int r) { return table + of(r) * ld_table; });
    const int all = count[0] + count[1] + count[2] + count[3];
    if (all == 0) return;
    int turn = 0;
    for (int w = 0; w < (nrow + 31) / 32; ++w) {
        for (uint32_t bits = has[w]; bits; bits &= bits - 1) {
            const int r = w * 32 + __builtin_ctz(bits);
            TT *row = table + of(r) * ld_table;
            if (all <= 64) {  // a wave per row
                if ((turn++ & 3) != wave) continue;
                for (int col0 = 0; col0 < d; col0 += 64 * E) {
                    const int col = col0 + lane * E;
                    vec_f<E> acc = (vec_f<E>)0.0f;
                    for (int q = 0; q < 4; ++q) grad_pick<TG, E>(grad, ld_grad, col, d - col, list + q * per, count[q], r, acc);
                    grad_write<TT, E>(row, col, d - col, acc, scale, accumulate);
                }
            } else {  // frequent ids: each wave its quarter of the positions
                for (int col0 = 0; col0 < d; col0 += 64 * E) {
                    const int col = col0 + lane * E;
                    vec_f<E> acc = (vec_f<E>)0.0f;
                    grad_pick<TG, E>(grad, ld_grad, col, d - col, list + from, m, r, acc);
                    quarter[wave][lane] = acc;
                    __syncthreads();
                    if (wave == 0) {
#pragma unroll
                        for (int q = 1; q < 4; ++q) acc += quarter[q][lane];
                        grad_write<TT, E>(row, col, d - col, acc, scale, accumulate);
                    }
                    __syncthreads();
                }
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

// --- the sums.  A wave per piece of GRAD_CHUNK sorted positions and 64 E columns: ids that lie within the piece are written to
// the table; the sum of one that began before goes to part[chunk][0], that of one that begins here and goes on to part[chunk][1].  bounds[v]: first and last + 1 sorted position of id v.
// Rows are requested eight at a time, whatever ids they are of, eight ahead of those that are added.
template <class TG, class TT, int E>
__global__ void __launch_bounds__(256)
k_vec_grad_chunks(const TG *__restrict__ grad, int d, int64_t ld_grad, const uint32_t *__restrict__ keys,
                  const uint32_t *__restrict__ pos, int64_t n, int64_t rows, float scale, int accumulate,
                  TT *__restrict__ table, int64_t ld_table, uint2 *__restrict__ bounds, float *__restrict__ part, int dpad, int chunks) {
    const int chunk = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (chunk >= chunks) return;
    const int64_t first = (int64_t)chunk * GRAD_CHUNK;
    int m = (int)(n - first < GRAD_CHUNK ? n - first : GRAD_CHUNK);
    const uint32_t none = 0xffffffffu;
    const uint32_t key = lane < m ? keys[first + lane] : none, p = lane < m ? pos[first + lane] : 0;
    const uint32_t prev = lane < m && first + lane > 0 ? keys[first + lane - 1] : none;
    const uint32_t next = lane < m && first + lane + 1 < n ? keys[first + lane + 1] : none;
    const bool begins = lane < m && key != prev, ends = lane < m && key != next;
    if (blockIdx.y == 0 && key < (uint64_t)rows) {
        if (begins) bounds[key].x = (uint32_t)(first + lane);
        if (ends) bounds[key].y = (uint32_t)(first + lane) + 1;
    }
    const uint64_t heads = __ballot(begins), tails = __ballot(ends);
    m = __popcll(__ballot(key < (uint64_t)rows));  // (ids that take no part come last)
    const int col = (int)blockIdx.y * 64 * E + lane * E, left = d - col;
    const TG *g = grad + col;
    vec_pack<TG, E> v[8], ahead[8];
    auto request = [&](int i0) {
#pragma unroll
        for (int u = 0; u < 8; ++u)
            ahead[u] = vec_load<TG, E>(g + (int64_t)__builtin_amdgcn_readlane(p, (i0 + u) & 63) * ld_grad, i0 + u < m ? left : 0);
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

// The first `chunks` blocks of a row of the grid: the run that ends in the piece and began before it, its partial sums added in order, a
// quarter of them per wave if they are many.  The other blocks: the rows without an id, GRAD_END_ROWS each.
#define GRAD_END_ROWS 64
template <class TT, int E>
__global__ void __launch_bounds__(256)
k_vec_grad_end(const uint32_t *__restrict__ keys, int64_t n, const uint2 *__restrict__ bounds, const float *__restrict__ part, int dpad,
               int d, float scale, int accumulate, TT *__restrict__ table, int64_t rows, int64_t ld_table, int chunks) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    if ((int64_t)blockIdx.x >= chunks) {
        __shared__ uint32_t has[GRAD_END_ROWS / 32];
        const int64_t lo = ((int64_t)blockIdx.x - chunks) * GRAD_END_ROWS;
        const int nrow = (int)(rows - lo < GRAD_END_ROWS ? rows - lo : GRAD_END_ROWS);
        if (threadIdx.x < 64) {
            const uint2 b = lane < nrow ? bounds[lo + lane] : make_uint2(0, 0);
            const uint64_t h = __ballot(b.y > b.x);
            if (lane < 2) has[lane] = (uint32_t)(h >> (32 * lane));
        }
        __syncthreads();
        grad_zeros<TT>(nrow, d, has, [&](int r) { return table + (lo + r) * ld_table; });
        return;
    }
    __shared__ vec_f<E> quarter[4][64];
    const int chunk = blockIdx.x;
    const int64_t first = (int64_t)chunk * GRAD_CHUNK;
    const uint32_t key = keys[first];
    if (chunk == 0 || key >= (uint64_t)rows || keys[first - 1] != key) return;
    const uint2 b = bounds[key];
    if ((b.y - 1) / GRAD_CHUNK != (uint32_t)chunk) return;  // (a later block's)
    const int c0 = (int)(b.x / GRAD_CHUNK);
    const int cnt = chunk - c0 + 1, each = cnt <= 8 ? cnt : (cnt + 3) / 4;
    if (cnt <= 8 && wave > 0) return;
    const int from = c0 + wave * each, to = from + each < chunk + 1 ? from + each : chunk + 1;
    for (int col0 = 0; col0 < d; col0 += 64 * E) {
        const int col = col0 + lane * E;
        vec_f<E> acc = (vec_f<E>)0.0f;
        if (col < d) {
#pragma unroll 8
            for (int c = from; c < to; ++c) acc += *(const vec_f<E> *)(part + ((int64_t)c * 2 + (c == c0 ? 1 : 0)) * dpad + col);
        }
        if (cnt > 8) {
            quarter[wave][lane] = acc;
            __syncthreads();
            if (wave == 0)
#pragma unroll
                for (int w = 1; w < 4; ++w) acc += quarter[w][lane];
        }
        if (wave == 0) grad_write<TT, E>(table + (int64_t)key * ld_table, col, d - col, acc, scale, accumulate);
        if (cnt > 8) __syncthreads();
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
        // 512 bytes of neighbouring rows together; about 1024 blocks (at most 2^16 rows each: a row of a block shares a word with a position)
        int group = 0, deal = 0;
        while (group < 5 && ((int64_t)vec_bytes(table_type) * d << group) < 512) ++group;
        while (deal < 10 && ((int64_t)4 << group << deal) < rows) ++deal;
        while ((rows >> (deal + 15)) > 0) ++deal;
        const int64_t groups = (rows + ((int64_t)1 << group) - 1) >> group, each = (groups + ((int64_t)1 << deal) - 1) >> deal;
        const int rpb = (int)(each << group);
        const size_t lds = (size_t)((rpb + 31) / 32) * 4 + GRAD_FEW * 4;
#define GO(TG, TT, ID, E)                                                                                                  \
    hipLaunchKernelGGL((k_vec_grad_few<TG, TT, ID, E>), dim3(1u << deal), dim3(256), lds, s, (const TG *)grad, (int)n, d,  \
                       ld_grad, (const ID *)ids, scale, accumulate, (TT *)table_grad, rows, ld_table, group, deal, rpb)
        VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, if (id_bytes == 4) GO(TG, TT, int32_t, E); else GO(TG, TT, int64_t, E))));
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
    VEC_TYPED(grad_type, TG, VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, hipLaunchKernelGGL(
        (k_vec_grad_chunks<TG, TT, E>), dim3((unsigned)((p.chunks + 3) / 4), (unsigned)((d + 64 * E - 1) / (64 * E))), dim3(256), 0, s, (const TG *)grad,
        d, ld_grad, ks, ps, n, rows, scale, accumulate, (TT *)table_grad, ld_table, bounds, part, p.dpad, p.chunks))));
    const int64_t zeros = accumulate ? 0 : (rows + GRAD_END_ROWS - 1) / GRAD_END_ROWS;
    VEC_TYPED(table_type, TT, GRAD_WIDTHS(d, hipLaunchKernelGGL((k_vec_grad_end<TT, E>), dim3((unsigned)(p.chunks + zeros)), dim3(256), 0, s, ks, n,
                                                                bounds, part, p.dpad, d, scale, accumulate, (TT *)table_grad, rows, ld_table, p.chunks)));
    QADC_LAUNCH_CHECK("vec_lookup_grad's kernels");
    return PQ_OK;
}
