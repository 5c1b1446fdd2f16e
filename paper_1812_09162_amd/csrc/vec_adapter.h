// vec_adapter and vec_adapter_grad: the kernels.  Rows x_i have an adapter e = id_i each, a pair of matrices A [rank][din], B [rank][dout]:
//   down   t_i = x_i A_e^T              contraction over columns: 64 rows' loads feed the matrix cores as they come
//   up     y_i = base_i + t_i B_e       contraction over ranks
//   outer  G_e = sum over the rows of e of t_i^T x_i   contraction over rows
// The gradient is the same three: u = dy B^T down, dx = u A up, dA = u^T x and dB = t^T dy outer; both factors lie along the long side, so
// that one form of each serves both.
//
// Rows of one adapter meet in a tile: the rows are sorted by id (k_vec_grad_place, stable) or taken as they come, and a block goes through
// the different ids among its positions, whatever their order, so that tiles need no list and no padding.
//
// t and u are sums and stay in float32.  Where they are factors, of bfloat16 and fp16 matrices, they are three bfloat16 numbers that hold all their 24
// bits, and an fp16 factor is two: the matrix cores have far more products than these operators need (at rank 16 a read byte takes 16 of
// 500 possible operations), and results in float32 stay as near as float32 sums come.  float32 matrices take the float32 instructions.
#pragma once
#include "vec_random.h"

#define AD_COLS(T) (16 / (int)sizeof(T))  // columns that a lane holds in `up` and `outer`: sixteen bytes

struct AdRows {
    const void *ids;
    int id_bytes, tp;             // tp: positions of a tile
    int64_t n;
    int adapters;
    const uint32_t *keys, *pos;   // sorted: position p holds row pos[p] of adapter keys[p] (= adapters: none); null: rows as they come
};
// float32 factors: the sum of `slabs` parts, times scales[e] factor
struct AdFactor {
    const float *p;
    int64_t ld, stride;
    int slabs;
    const float *scales;
    float factor;
};
struct AdMatrix {
    const void *p;
    int64_t ld, stride;  // of rows, of adapters
    int rank, d;
};

__device__ __forceinline__ int ad_id(const AdRows &r, int64_t p) {
    if (r.keys) return (int)r.keys[p];
    const int64_t id = r.id_bytes == 4 ? (int64_t)((const int32_t *)r.ids)[p] : ((const int64_t *)r.ids)[p];
    return id >= 0 && id < r.adapters ? (int)id : r.adapters;
}
__device__ __forceinline__ uint32_t ad_row(const AdRows &r, int64_t p) { return r.pos ? r.pos[p] : (uint32_t)p; }

typedef __bf16 ad_b8 __attribute__((ext_vector_type(8)));
typedef _Float16 ad_h8 __attribute__((ext_vector_type(8)));
typedef uint32_t ad_u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ vec_f4 ad_mma(ad_b8 a, ad_b8 b, vec_f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ vec_f4 ad_mma(ad_h8 a, ad_h8 b, vec_f4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// Products of values of the matrices' own type: eight k a lane (its 8 (lane / 16) and on), for rows lane % 16 of either factor.
template <class T>
__device__ __forceinline__ vec_f4 ad_mul(vec_pack<T> a, vec_pack<T> b, vec_f4 c) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
        return c;
    } else if constexpr (__is_same(T, __bf16)) {
        return ad_mma(__builtin_bit_cast(ad_b8, a), __builtin_bit_cast(ad_b8, b), c);
    } else {
        return ad_mma(__builtin_bit_cast(ad_h8, a), __builtin_bit_cast(ad_h8, b), c);
    }
}

__device__ __forceinline__ uint32_t ad_high(float hi, float lo) {  // the upper halves of two
    return __builtin_amdgcn_perm(__float_as_uint(hi), __float_as_uint(lo), 0x07060302u);
}
__device__ __forceinline__ float ad_cut(float f) { return __uint_as_float(__float_as_uint(f) & 0xffff0000u); }

// A float32 factor as the matrix cores take it beside values of T.
template <class T>
struct AdWide {  // bfloat16, fp16: f = p[0] + p[1] + p[2], each the upper eight bits of what the ones before leave
    static constexpr int parts = 3;
    ad_u4 p[3];
    __device__ __forceinline__ void set(vec_f8 f) {
#pragma unroll
        for (int s = 0; s < 3; ++s)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[s][i] = ad_high(f[2 * i + 1], f[2 * i]);
                f[2 * i] -= ad_cut(f[2 * i]);
                f[2 * i + 1] -= ad_cut(f[2 * i + 1]);
            }
    }
};
template <>
struct AdWide<float> {
    static constexpr int parts = 2;
    ad_u4 p[2];
    __device__ __forceinline__ void set(vec_f8 f) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i >> 2][i & 3] = __float_as_uint(f[i]);
    }
};
// Eight values of T (along the contraction) for it: fp16 as two bfloat16 numbers.
template <class T>
struct AdNarrow {
    ad_u4 p[1];
};
template <>
struct AdNarrow<_Float16> {
    ad_u4 p[2];
};
template <>
struct AdNarrow<float> {
    float p[8];
};
// Rows raw[0..7], AD_COLS(T) columns each: column m.
template <class T>
__device__ __forceinline__ AdNarrow<T> ad_column(const vec_pack<T, AD_COLS(T)> *raw, int m) {
    AdNarrow<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int q = 0; q < 8; ++q) o.p[q] = raw[q][m];
    } else {
        ad_u4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            u[i] = __builtin_amdgcn_perm(__builtin_bit_cast(ad_u4, raw[2 * i + 1])[m >> 1], __builtin_bit_cast(ad_u4, raw[2 * i])[m >> 1], m & 1 ? 0x07060302u : 0x05040100u);
        if constexpr (__is_same(T, __bf16)) {
            o.p[0] = u;
        } else {
            const ad_h8 h = __builtin_bit_cast(ad_h8, u);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float a = (float)h[2 * i], b = (float)h[2 * i + 1];
                o.p[0][i] = ad_high(b, a);
                o.p[1][i] = ad_high(b - ad_cut(b), a - ad_cut(a));
            }
        }
    }
    return o;
}
// c += narrow factor (rows of the result) times wide one (its columns), or, WIDE_FIRST, the other way round
template <class T, bool WIDE_FIRST>
__device__ __forceinline__ vec_f4 ad_mul(const AdNarrow<T> &n, const AdWide<T> &w, vec_f4 c) {
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const float f = __uint_as_float(w.p[q >> 2][q & 3]);
            c = WIDE_FIRST ? __builtin_amdgcn_mfma_f32_16x16x4f32(f, n.p[q], c, 0, 0, 0) : __builtin_amdgcn_mfma_f32_16x16x4f32(n.p[q], f, c, 0, 0, 0);
        }
    } else {
        auto one = [&](ad_u4 a, ad_u4 b) {
            c = WIDE_FIRST ? ad_mma(__builtin_bit_cast(ad_b8, b), __builtin_bit_cast(ad_b8, a), c) : ad_mma(__builtin_bit_cast(ad_b8, a), __builtin_bit_cast(ad_b8, b), c);
        };
        if constexpr (__is_same(T, _Float16)) {  // (smallest first; the product of the last parts is below float32's last bit)
            one(n.p[1], w.p[1]);
            one(n.p[0], w.p[2]);
            one(n.p[1], w.p[0]);
        } else {
            one(n.p[0], w.p[2]);
        }
        one(n.p[0], w.p[1]);
        one(n.p[0], w.p[0]);
    }
    return c;
}

// Elements of a mask of eight columns that hold E columns from the one at `col` on.
template <class T, int E>
__device__ __forceinline__ vec_pack<T, E> ad_drop(vec_pack<T, E> v, vec_i4 kept, int64_t col) {
    if constexpr (E == 8) {
        return vec_drop<T>(v, kept);
    } else {
        static_assert(E == 4 && sizeof(T) == 4, "");
        const bool second = col & 4;
        const int a = second ? kept[2] : kept[0], b = second ? kept[3] : kept[1];
        v[0] = a & 1 ? v[0] : 0.0f;
        v[1] = a >> 16 & 1 ? v[1] : 0.0f;
        v[2] = b & 1 ? v[2] : 0.0f;
        v[3] = b >> 16 & 1 ? v[3] : 0.0f;
        return v;
    }
}

// ------------------------------------------------------------------- tiles --
// The positions of a tile, a lane each: rows and adapters (`adapters` behind the last and for none).
struct AdTile {
    int id;
    uint32_t row;
    bool in;
};
__device__ __forceinline__ AdTile ad_tile(const AdRows &r, int lane) {
    const int64_t p = vec_block() * r.tp + lane;
    AdTile t = {r.adapters, 0, lane < r.tp && p < r.n};
    if (t.in) {
        t.id = ad_id(r, p);
        t.row = ad_row(r, p);
    }
    return t;
}
// Rows of those lanes whose bit is set, in order, in a wave's own list; returns how many.
__device__ __forceinline__ int ad_list(uint64_t bits, uint32_t row, uint32_t *list, int lane) {
    if (bits >> lane & 1) list[__popcll(bits & ((1ull << lane) - 1))] = row;
    __builtin_amdgcn_wave_barrier();
    return __popcll(bits);
}

// -------------------------------------------------------------------- down --
// part[slab][row][rank] = sum over the slab's columns of (kept) x_row W_e^T, rows padded to `rp` ranks, with zeros.  A block takes a
// tile of positions, 16 RK ranks and a slab of columns; its four waves take turns at 32 columns each and join their sums through LDS.  W's rows are the
// instruction's first factor, so that a lane holds four neighbouring ranks of a row.  Rows of x go to registers as the matrix cores want them, without LDS.
template <class T, int RK, int NT, bool MASK>
__device__ __forceinline__ void ad_down(const T *__restrict__ x, int64_t ld_x, const T *__restrict__ w, int64_t ld_w, int d, int kb, int ke, int rank, int j0,
                                        const uint32_t *list, int count, const VecMask &mask, VecKey key, vec_f4 *red, float *__restrict__ part, int rp) {
    constexpr int U = sizeof(T) == 4 ? 1 : 2;  // steps on their way
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const T *xp[NT], *wp[RK];
    uint32_t row[NT];
    // (lanes without a row or a rank read another's: what they give is not stored)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        row[t] = list[16 * t + c < count ? 16 * t + c : 0];
        xp[t] = x + (int64_t)row[t] * ld_x;
    }
#pragma unroll
    for (int j = 0; j < RK; ++j) wp[j] = w + (int64_t)(j0 + 16 * j + c < rank ? j0 + 16 * j + c : rank - 1) * ld_w;
    vec_f4 acc[NT][RK];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < RK; ++j) acc[t][j] = (vec_f4)0.0f;
    auto step = [&](vec_pack<T> *xv, const vec_pack<T> *wv, int k) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            if (MASK) xv[t] = vec_drop<T>(xv[t], vec_kept(vec_random(key, mask.layer, row[t], (uint32_t)k >> 3), mask.threshold));
#pragma unroll
            for (int j = 0; j < RK; ++j) acc[t][j] = ad_mul<T>(wv[j], xv[t], acc[t][j]);
        }
    };
    const int whole = ke < d ? ke : d / 32 * 32;  // steps that begin below hold 32 columns
    int k = kb + 32 * wave;
    for (; k + (U - 1) * 128 + 32 <= whole; k += 128 * U) {
        vec_pack<T> xv[U][NT], wv[U][RK];
#pragma unroll
        for (int u = 0; u < U; ++u) {
#pragma unroll
            for (int t = 0; t < NT; ++t) xv[u][t] = *(const vec_pack<T> *)(xp[t] + k + 128 * u + 8 * g);
#pragma unroll
            for (int j = 0; j < RK; ++j) wv[u][j] = *(const vec_pack<T> *)(wp[j] + k + 128 * u + 8 * g);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) step(xv[u], wv[u], k + 128 * u + 8 * g);
    }
    for (; k < ke; k += 128) {
        vec_pack<T> xv[NT], wv[RK];
        const int col = k + 8 * g;
#pragma unroll
        for (int t = 0; t < NT; ++t) xv[t] = vec_load(xp[t] + (col < d ? col : 0), d - col, col);
#pragma unroll
        for (int j = 0; j < RK; ++j) wv[j] = vec_load(wp[j] + (col < d ? col : 0), d - col, col);
        step(xv, wv, col);
    }
    // sums of the four waves, TR tiles' a round
    constexpr int TR = NT * RK <= 8 ? NT : (RK <= 4 ? 8 / RK : 1);
#pragma unroll
    for (int t0 = 0; t0 < NT; t0 += TR) {
        __syncthreads();
#pragma unroll
        for (int t = 0; t < TR; ++t)
#pragma unroll
            for (int j = 0; j < RK; ++j) red[((wave * TR + t) * RK + j) * 64 + lane] = acc[t0 + t][j];
        __syncthreads();
        for (int i = threadIdx.x; i < TR * RK * 64; i += 256) {
            const int l = i & 63, j = (i >> 6) % RK, t = (i >> 6) / RK;
            const int at = 16 * (t0 + t) + (l & 15), to = j0 + 16 * j + 4 * (l >> 4);
            if (at >= count || to >= rp) continue;
            vec_f4 s = red[i];
#pragma unroll
            for (int v = 1; v < 4; ++v) s += red[v * TR * RK * 64 + i];
#pragma unroll
            for (int q = 0; q < 4; ++q) s[q] = to + q < rank ? s[q] : 0.0f;
            *(vec_f4 *)(part + (int64_t)list[at] * rp + to) = s;
        }
    }
}

template <class T, int RK, bool MASK>
__global__ void __launch_bounds__(256)
k_vec_ad_down(AdRows rows, const T *__restrict__ x, int64_t ld_x, AdMatrix m, VecMask mask, float *__restrict__ part, int64_t part_stride, int rp, int per) {
    __shared__ uint32_t lists[4][64];
    __shared__ vec_f4 red[4 * (RK == 1 ? 4 : 8) * 64];
    const int lane = threadIdx.x & 63;
    uint32_t *list = lists[threadIdx.x >> 6];
    const AdTile tile = ad_tile(rows, lane);
    VecKey key = {0, 0, 0};
    if (MASK) key = vec_key(mask);
    const int kb = blockIdx.z * per, ke = kb + per < m.d ? kb + per : m.d;
    part += blockIdx.z * part_stride;
    uint64_t todo = __ballot(tile.id < rows.adapters);
    while (todo) {
        const int e = __builtin_amdgcn_readlane(tile.id, __builtin_ctzll(todo));
        const uint64_t bits = __ballot(tile.id == e);
        todo &= ~bits;
        const int count = ad_list(bits, tile.row, list, lane);
        const T *w = (const T *)m.p + e * m.stride;
        for (int j0 = 0; j0 < m.rank; j0 += 16 * RK) {
            if (RK <= 2 && count > 32) ad_down<T, RK, RK <= 2 ? 4 : 1, MASK>(x, ld_x, w, m.ld, m.d, kb, ke, m.rank, j0, list, count, mask, key, red, part, rp);
            else if (count > 16) ad_down<T, RK, 2, MASK>(x, ld_x, w, m.ld, m.d, kb, ke, m.rank, j0, list, count, mask, key, red, part, rp);
            else ad_down<T, RK, 1, MASK>(x, ld_x, w, m.ld, m.d, kb, ke, m.rank, j0, list, count, mask, key, red, part, rp);
        }
        __syncthreads();  // (other waves read their lists' rows for the last stores; these are equal, the sums' buffer is not)
    }
}

// ---------------------------------------------------------------------- up --
// y_row = base_row + (kept) f_row W_e.  A block takes a tile of positions and 64 AD_COLS columns at a time, a quarter a wave.  The factor f is made ready
// in LDS once (its parts as the matrix cores take them); a lane reads eight ranks of AD_COLS columns of W, whose columns are put together from
// their halves by byte permutations.  Lane c reads column group 4 (c % 4) + c / 4, so that the four lanes of a row hold neighbouring groups of the result.
template <class T, class Y, bool MASK>
struct AdUp {
    static constexpr int E = AD_COLS(T);
    const Y *base;
    Y *y;
    int64_t ld_base, ld_y;
    int d, c0;
    VecMask mask;
    VecKey key;

    __device__ __forceinline__ void write(const vec_f4 *acc, uint32_t row) const {  // acc: a lane's groups 4 i + lane / 16, column m of each
        const int g = (threadIdx.x & 63) >> 4;
        vec_pack<Y, E> b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = c0 + E * (4 * i + g);
            if (base) b[i] = vec_load<Y, E>(base + row * ld_base + (col < d ? col : 0), d - col, col);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = c0 + E * (4 * i + g);
            if (col >= d) continue;
            vec_pack<float, E> f;
#pragma unroll
            for (int m = 0; m < E; ++m) f[m] = acc[m][i];
            if (MASK) {
                const vec_i4 kept = vec_kept(vec_random(key, mask.layer, row, (uint32_t)col >> 3), mask.threshold);
#pragma unroll
                for (int m = 0; m < E; ++m) {
                    const int at = (col & 7) + m;
                    const int word = E == 8 ? kept[m >> 1] : (col & 4 ? kept[2 + (m >> 1)] : kept[m >> 1]);
                    f[m] = word >> (16 * (at & 1)) & 1 ? f[m] : 0.0f;
                }
            }
            vec_f<E> v = f;
            if (base) v += vec_wide<Y, E>(b[i]);
            vec_store<Y, E>(y + row * ld_y + col, d - col, v);
        }
    }
};

// f of the list's rows, 32 ranks (chunk kc) a slot: lane holds row lane % 16 of the tile and ranks 8 (lane / 16) and on.
template <class T>
__device__ __forceinline__ void ad_ready(const AdFactor &f, float by, int rank, int chunks, const uint32_t *list, int count, int tiles, ad_u4 *ready, float *keep, int64_t ld_keep) {
    constexpr int P = AdWide<T>::parts;
    for (int i = threadIdx.x; i < tiles * chunks * 64; i += 256) {
        const int l = i & 63, t = (i >> 6) % tiles, kc = (i >> 6) / tiles;
        const int at = 16 * t + (l & 15), r0 = 32 * kc + 8 * (l >> 4);
        vec_f8 v = (vec_f8)0.0f;
        if (at < count && r0 < rank) {
            const float *p = f.p + (int64_t)list[at] * f.ld + r0;
            for (int s = 0; s < f.slabs; ++s) {
                const vec_f4 a = *(const vec_f4 *)p, b = *(const vec_f4 *)(p + 4);  // (rows are padded to sixteen ranks, with zeros)
#pragma unroll
                for (int q = 0; q < 4; ++q) v[q] += a[q], v[4 + q] += b[q];
                p += f.stride;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = r0 + q < rank ? v[q] * by : 0.0f;
            if (keep) vec_store<float>(keep + (int64_t)list[at] * ld_keep + r0, rank - r0, v);
        }
        AdWide<T> o;
        o.set(v);
#pragma unroll
        for (int s = 0; s < P; ++s) ready[(((kc * tiles + t) * P) + s) * 64 + l] = o.p[s];
    }
}

template <class T, class Y, bool MASK, bool ONE>  // ONE: at most 32 ranks
__global__ void __launch_bounds__(256)
k_vec_ad_up(AdRows rows, AdFactor f, AdMatrix m, const Y *base, int64_t ld_base, Y *y, int64_t ld_y, VecMask mask, float *__restrict__ keep) {
    constexpr int E = AD_COLS(T), P = AdWide<T>::parts;
    extern __shared__ __align__(16) unsigned char smem[];
    ad_u4 *ready = (ad_u4 *)smem;  // [chunk][tile][part][lane]
    __shared__ uint32_t lists[4][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    uint32_t *list = lists[wave];
    const AdTile tile = ad_tile(rows, lane);
    const int chunks = ONE ? 1 : (m.rank + 31) / 32;
    AdUp<T, Y, MASK> up = {base, y, ld_base, ld_y, m.d, 0, mask, {0, 0, 0}};
    if (MASK) up.key = vec_key(mask);
    uint64_t todo = __ballot(tile.in);
    while (todo) {
        const int e = __builtin_amdgcn_readlane(tile.id, __builtin_ctzll(todo));
        const uint64_t bits = __ballot(tile.in && tile.id == e);
        todo &= ~bits;
        const bool none = e == rows.adapters;
        if (none && base == y && !keep) continue;
        const int count = ad_list(bits, tile.row, list, lane), tiles = (count + 15) / 16;
        float *const kept = blockIdx.z == 0 ? keep : nullptr;
        if (none) {
            if (kept)
                for (int i = threadIdx.x; i < count * m.rank; i += 256) kept[(int64_t)list[i / m.rank] * m.rank + i % m.rank] = 0.0f;
            if (base == y) continue;
        } else {
            const float by = f.scales ? f.scales[e] * f.factor : f.factor;
            ad_ready<T>(f, by, m.rank, chunks, list, count, tiles, ready, kept, m.rank);
            __syncthreads();
        }
        const T *w = (const T *)m.p + (none ? 0 : e * m.stride);
        for (up.c0 = (blockIdx.z * 4 + wave) * 16 * E; up.c0 < m.d; up.c0 += gridDim.z * 64 * E) {
            const int col = up.c0 + E * (4 * (c & 3) + (c >> 2));
            auto weights = [&](int kc, AdNarrow<T> *o) {
                vec_pack<T, E> raw[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int r = 32 * kc + 8 * g + q;
                    raw[q] = vec_load<T, E>(w + (r < m.rank && col < m.d ? r * m.ld + col : 0), r < m.rank ? m.d - col : 0, col);
                }
#pragma unroll
                for (int i = 0; i < E; ++i) o[i] = ad_column<T>(raw, i);
            };
            auto factor = [&](int kc, int t) {
                AdWide<T> o;
#pragma unroll
                for (int s = 0; s < P; ++s) o.p[s] = ready[((kc * tiles + t) * P + s) * 64 + lane];
                return o;
            };
            if (none) {
                vec_f4 acc[E];
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] = (vec_f4)0.0f;
                for (int t = 0; t < tiles; ++t)
                    if (16 * t + c < count) up.write(acc, list[16 * t + c]);
            } else if (ONE) {
                AdNarrow<T> o[E];
                weights(0, o);
                for (int t = 0; t < tiles; ++t) {
                    const AdWide<T> a = factor(0, t);
                    vec_f4 acc[E];
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[i] = ad_mul<T, false>(o[i], a, (vec_f4)0.0f);
                    if (16 * t + c < count) up.write(acc, list[16 * t + c]);
                }
            } else {  // (tiles of at most 32 positions)
                vec_f4 acc[2][E];
#pragma unroll
                for (int i = 0; i < E; ++i) acc[0][i] = acc[1][i] = (vec_f4)0.0f;
                for (int kc = 0; kc < chunks; ++kc) {
                    AdNarrow<T> o[E];
                    weights(kc, o);
                    const AdWide<T> a = factor(kc, 0);
#pragma unroll
                    for (int i = 0; i < E; ++i) acc[0][i] = ad_mul<T, false>(o[i], a, acc[0][i]);
                    if (tiles > 1) {
                        const AdWide<T> b = factor(kc, 1);
#pragma unroll
                        for (int i = 0; i < E; ++i) acc[1][i] = ad_mul<T, false>(o[i], b, acc[1][i]);
                    }
                }
                if (c < count) up.write(acc[0], list[c]);
                if (16 + c < count) up.write(acc[1], list[16 + c]);
            }
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------- outer --
// G_e[j][col] = sum over the rows of e of f_row[j] (kept) x_row[col].  A block takes `len` sorted positions and 64 AD_COLS columns, a quarter a wave, and goes through
// the runs of equal ids among them.  Runs that lie within the block's positions are written; the others' sums go to part[chunk][0] (began before)
// or part[chunk][1], which k_vec_ad_join adds up in order.  Per step a lane reads eight rows of AD_COLS columns.
#define AD_STAGE 128  // positions whose factors are made ready at once
struct AdOuter {
    void *out;
    int64_t ld, stride;   // of rows, of adapters
    float *part;          // [chunk][2][rank][dpad]
    int dpad, accumulate;
};
template <class O, int E>
__device__ __forceinline__ void ad_put(O *p, int64_t left, vec_f<E> v, int64_t before, bool accumulate) {
    if (accumulate) v += vec_wide<O, E>(vec_load<O, E>(p, left, before));
    vec_store<O, E>(p, left, v);
}

template <class T, class O, int RK, bool MASK>
__global__ void __launch_bounds__(256)
k_vec_ad_outer(AdRows rows, int len, AdFactor f, int rank, const T *__restrict__ x, int64_t ld_x, int d, VecMask mask, AdOuter o) {
    constexpr int E = AD_COLS(T), P = AdWide<T>::parts, STEPS = AD_STAGE / 32;
    __shared__ ad_u4 ready[STEPS][RK][P][64];
    __shared__ uint32_t at[AD_STAGE];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, c = lane & 15, g = lane >> 4;
    const int64_t chunk = blockIdx.x, p0 = chunk * len, p1 = p0 + len < rows.n ? p0 + len : rows.n;
    const int col = (blockIdx.y * 4 + wave) * 16 * E + E * c, j0 = blockIdx.z * 16 * RK;
    VecKey key = {0, 0, 0};
    if (MASK) key = vec_key(mask);
    for (int64_t a = p0; a < p1;) {
        const uint32_t e = rows.keys[a];
        if (e >= (uint32_t)rows.adapters) break;  // (rows without an adapter come last)
        int64_t b = a + 1;
        for (;;) {  // the run's end
            const uint64_t other = __ballot(b + lane >= p1 || rows.keys[b + lane] != e);
            if (other) {
                b += __builtin_ctzll(other);
                break;
            }
            b += 64;
        }
        const float by = f.scales ? f.scales[e] * f.factor : f.factor;
        vec_f4 acc[RK][E];
#pragma unroll
        for (int j = 0; j < RK; ++j)
#pragma unroll
            for (int i = 0; i < E; ++i) acc[j][i] = (vec_f4)0.0f;
        for (int64_t s0 = a; s0 < b; s0 += AD_STAGE) {
            const int m = (int)(b - s0 < AD_STAGE ? b - s0 : AD_STAGE);
            __syncthreads();
            if (threadIdx.x < AD_STAGE) at[threadIdx.x] = (int)threadIdx.x < m ? rows.pos[s0 + threadIdx.x] : 0;
            __syncthreads();
            for (int i = threadIdx.x; i < STEPS * RK * 64; i += 256) {
                const int l = i & 63, j = (i >> 6) % RK, st = (i >> 6) / RK;
                const int r = j0 + 16 * j + (l & 15), q0 = 32 * st + 8 * (l >> 4);
                vec_f8 v;
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    float sum = 0.0f;
                    if (q0 + q < m && r < rank) {
                        const float *p = f.p + (int64_t)at[q0 + q] * f.ld + r;
                        for (int s = 0; s < f.slabs; ++s) sum += p[s * f.stride];
                        sum *= by;
                    }
                    v[q] = sum;
                }
                AdWide<T> w;
                w.set(v);
#pragma unroll
                for (int s = 0; s < P; ++s) ready[st][j][s][l] = w.p[s];
            }
            __syncthreads();
            for (int st = 0; 32 * st < m; ++st) {
                vec_pack<T, E> raw[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const int i = 32 * st + 8 * g + q;
                    const bool in = i < m && col < d;
                    const uint32_t row = at[i];
                    raw[q] = vec_load<T, E>(x + (in ? row * ld_x + col : 0), in ? d - col : 0, col);
                    if (MASK && in) raw[q] = ad_drop<T, E>(raw[q], vec_kept(vec_random(key, mask.layer, row, (uint32_t)col >> 3), mask.threshold), col);
                }
                AdWide<T> w[RK];
#pragma unroll
                for (int j = 0; j < RK; ++j)
#pragma unroll
                    for (int s = 0; s < P; ++s) w[j].p[s] = ready[st][j][s][lane];
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const AdNarrow<T> v = ad_column<T>(raw, i);
#pragma unroll
                    for (int j = 0; j < RK; ++j) acc[j][i] = ad_mul<T, true>(v, w[j], acc[j][i]);
                }
            }
        }
        const bool before = a == p0 && p0 > 0 && rows.keys[p0 - 1] == e, behind = b == p1 && p1 < rows.n && rows.keys[p1] == e;
#pragma unroll
        for (int j = 0; j < RK; ++j)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int r = j0 + 16 * j + 4 * g + q;
                if (r >= rank || col >= d) continue;
                vec_f<E> v;
#pragma unroll
                for (int i = 0; i < E; ++i) v[i] = acc[j][i][q];
                if (before || behind) vec_store<float, E>(o.part + ((chunk * 2 + (before ? 0 : 1)) * rank + r) * (int64_t)o.dpad + col, o.dpad - col, v);
                else ad_put<O, E>((O *)o.out + e * o.stride + r * o.ld + col, d - col, v, col, o.accumulate);
            }
        a = b;
    }
}

// The sums of ids whose positions several blocks held, and zeros for those without a row.
template <class O>
__global__ void __launch_bounds__(256)
k_vec_ad_join(AdRows rows, int len, int rank, int d, AdOuter o) {
    const int64_t n = rows.n;
    const uint32_t e = blockIdx.y;
    auto first = [&](uint32_t key) {  // the first position whose key is at least this
        int64_t lo = 0, hi = n;
        while (lo < hi) {
            const int64_t mid = (lo + hi) >> 1;
            if (rows.keys[mid] < key) lo = mid + 1;
            else hi = mid;
        }
        return lo;
    };
    const int64_t lo = first(e), hi = first(e + 1);
    const int64_t from = lo / len, to = lo < hi ? (hi - 1) / len : 0;
    if (lo < hi ? from == to : o.accumulate) return;
    const int pieces = o.dpad / 8;
    for (int64_t i = blockIdx.x * 256 + threadIdx.x; i < (int64_t)rank * pieces; i += gridDim.x * 256) {
        const int r = (int)(i / pieces), col = (int)(i - (int64_t)r * pieces) * 8;
        vec_f8 sum = (vec_f8)0.0f;
        if (lo < hi) {
            const int64_t each = 2 * (int64_t)rank * o.dpad;
            const float *p = o.part + (int64_t)r * o.dpad + col;
            sum = *(const vec_f8 *)(p + from * each + each / 2);
#pragma unroll 8
            for (int64_t k = from + 1; k <= to; ++k) sum += *(const vec_f8 *)(p + k * each);
        }
        ad_put<O, 8>((O *)o.out + e * o.stride + r * o.ld + col, d - col, sum, col, o.accumulate);
    }
}
