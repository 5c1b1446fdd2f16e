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

#define AD_COLS(T) (16 / (int)sizeof(T))  // columns that a lane holds: sixteen bytes (in `outer` four columns; one where the matrix has fewer)

struct AdRows {
    const void *ids;
    int id_bytes, tp;             // tp: positions of a tile
    int64_t n;
    int adapters;
    const uint32_t *keys, *pos;   // sorted: position p holds row pos[p] of adapter keys[p] (= adapters: none); null: rows as they come
};
// float32 factors: the sum of `slabs` parts
struct AdFactor {
    const float *p;
    int64_t ld, stride;
    int slabs;
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
template <int N>
struct AdWords {
    typedef uint32_t type __attribute__((ext_vector_type(N)));
};
template <int N>
using ad_words = typename AdWords<N>::type;

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

// Some of eight values along the contraction: all bits of those, none of the others'.
template <class T>
struct AdNamed {
    ad_u4 m;
    __device__ __forceinline__ void set(uint32_t bits) {
#pragma unroll
        for (int i = 0; i < 4; ++i) m[i] = (bits >> (2 * i) & 1 ? 0xffffu : 0u) | (bits >> (2 * i + 1) & 1 ? 0xffff0000u : 0u);
    }
};
template <>
struct AdNamed<float> {
    uint32_t m;
    __device__ __forceinline__ void set(uint32_t bits) { m = bits; }
};
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
    // zeros for those of the eight values that are not named
    __device__ __forceinline__ void only(const AdNamed<T> &in) {
#pragma unroll
        for (int s = 0; s < 3; ++s) p[s] &= in.m;
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
    __device__ __forceinline__ void only(const AdNamed<float> &in) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i >> 2][i & 3] = in.m >> i & 1 ? p[i >> 2][i & 3] : 0u;
    }
};
// Eight values of T (along the contraction) for it: fp16 as two bfloat16 numbers.
template <class T>
struct AdNarrow {
    ad_u4 p[1];
    __device__ __forceinline__ void only(const AdNamed<T> &in) { p[0] &= in.m; }
};
template <>
struct AdNarrow<_Float16> {
    ad_u4 p[2];
    __device__ __forceinline__ void only(const AdNamed<_Float16> &in) { p[0] &= in.m, p[1] &= in.m; }
};
template <>
struct AdNarrow<float> {
    float p[8];
    __device__ __forceinline__ void only(const AdNamed<float> &in) {
#pragma unroll
        for (int i = 0; i < 8; ++i) p[i] = in.m >> i & 1 ? p[i] : 0.0f;
    }
};
// Rows raw[0..7], E columns each: column m.
template <class T, int E>
__device__ __forceinline__ AdNarrow<T> ad_column(const vec_pack<T, E> *raw, int m) {
    AdNarrow<T> o;
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int q = 0; q < 8; ++q) o.p[q] = raw[q][m];
    } else {
        ad_u4 u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 1)
                u[i] = (uint32_t)__builtin_bit_cast(uint16_t, (T)raw[2 * i + 1][0]) << 16 | __builtin_bit_cast(uint16_t, (T)raw[2 * i][0]);
            else
                u[i] = __builtin_amdgcn_perm(__builtin_bit_cast(ad_words<E / 2>, raw[2 * i + 1])[m >> 1], __builtin_bit_cast(ad_words<E / 2>, raw[2 * i])[m >> 1],
                                             m & 1 ? 0x07060302u : 0x05040100u);
        }
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
        if constexpr (__is_same(T, _Float16)) {  // (smallest first; the product of the last parts, left out, is below 2^-22 of the whole)
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

// Which of the eight columns 8 col8 and on are kept, a bit each.
__device__ __forceinline__ uint32_t ad_bits(VecKey key, const VecMask &mask, uint32_t row, uint32_t col8) {
    const vec_i4 k = vec_random(key, mask.layer, row, col8);
    uint32_t b = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        const uint32_t u = (uint32_t)k[w];
        b |= ((u & 0xffffu) >= mask.threshold ? 1u : 0u) << (2 * w) | ((u >> 16) >= mask.threshold ? 2u : 0u) << (2 * w);
    }
    return b;
}
// The same of the E columns from `from` on (a lane's own, or at the matrix's end any).
template <int E>
__device__ __forceinline__ uint32_t ad_kept(VecKey key, const VecMask &mask, uint32_t row, int from) {
    const int shift = from & 7;
    uint32_t b = ad_bits(key, mask, row, (uint32_t)from >> 3);
    if (shift + E > 8) b |= ad_bits(key, mask, row, ((uint32_t)from >> 3) + 1) << 8;
    return b >> shift;
}
// The same of a position, where `outer` has kept them: a word has eight columns of four positions, [position / 4][column / 8].
__device__ __forceinline__ uint32_t ad_bits_of(const uint32_t *bits, int64_t position, int d, int from) {
    return bits[(position >> 2) * (d / 8) + (from >> 3)] >> (8 * ((int)position & 3) + (from & 7));
}
// Zeros in place of what is dropped.
template <class T, int E>
__device__ __forceinline__ vec_pack<T, E> ad_drop(vec_pack<T, E> v, uint32_t kept) {
    if constexpr (E > 1 && sizeof(T) == 2) {
        auto u = __builtin_bit_cast(ad_words<E / 2>, v);
#pragma unroll
        for (int w = 0; w < E / 2; ++w) u[w] &= (kept >> (2 * w) & 1 ? 0xffffu : 0u) | (kept >> (2 * w + 1) & 1 ? 0xffff0000u : 0u);
        return __builtin_bit_cast(vec_pack<T, E>, u);
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (!(kept >> i & 1)) v[i] = 0;
        return v;
    }
}
// The same for eight rows.  whole: lanes have their own columns, all that are stored; neighbouring lanes that hold halves of eight columns then make four rows' bits each, and
// `store` takes these.
template <class T, int E, class ROW, class STORE>
__device__ __forceinline__ void ad_drop8(vec_pack<T, E> *v, VecKey key, const VecMask &mask, ROW row, int from, bool whole, STORE store) {
    if (E == 4 && whole) {
        const int half = threadIdx.x & 1;
        uint32_t mine = 0;
#pragma unroll
        for (int q = 0; q < 4; ++q) mine |= ad_bits(key, mask, row(4 * half + q), (uint32_t)from >> 3) << (8 * q);
        store(half, mine);
        const uint32_t other = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)mine, 0xb1, 0xf, 0xf, true);  // (of the lane beside)
        const uint32_t low = half ? other : mine, high = half ? mine : other;
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = ad_drop<T, E>(v[q], (q < 4 ? low : high) >> (8 * (q & 3) + 4 * half));
    } else {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] = ad_drop<T, E>(v[q], ad_kept<E>(key, mask, row(q), from));
    }
}

// A lane's E columns from col on, where the matrix ends: every lane reads E columns, those at the end the last E (d >= E; matrices of fewer
// columns take E = 1), and writes what is its own of them.  (Reads of part of the columns cost the loops twice their registers.)
template <int E>
__device__ __forceinline__ int ad_from(int col, int d) { return col + E <= d ? col : d - E; }
template <class T, int E>
__device__ __forceinline__ vec_pack<T, E> ad_load(const T *row, int from) { return *(const vec_pack<T, E> *)(row + from); }
template <class T, int E>
__device__ __forceinline__ void ad_store(T *row, int col, int d, vec_f<E> v) {
    const vec_pack<T, E> o = __builtin_convertvector(v, vec_pack<T, E>);
    const int from = ad_from<E>(col, d);
    if (from == col) {
        *(vec_pack<T, E> *)(row + col) = o;
    } else {
#pragma unroll
        for (int i = 0; i < E; ++i)
            if (from + i >= col) row[from + i] = o[i];
    }
}

// ------------------------------------------------------------------- tiles --
// The positions of a tile, a lane each: rows and adapters (`adapters` behind the last and for none).
struct AdTile {
    int id;
    uint32_t row;
    bool in;
};
__device__ __forceinline__ AdTile ad_tile(const AdRows &r, int64_t tile, int lane) {
    const int64_t p = tile * r.tp + lane;
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
// part[slab][row][rank] = by the sum over the slab's columns of (kept) x_row W_e^T, rows padded to `rp` ranks, with zeros.  A block takes a
// tile of positions and a slab of columns (one slab unless there are few rows); its waves take turns at 128 bytes of the rows each and join their sums
// through LDS, or, where adapters have few rows, take an adapter of the tile each (`own`), without a wait.  W's rows are the instruction's first factor, so that a lane holds four neighbouring ranks of a row.
//
// Eight neighbouring lanes read 128 bytes of a row, sixteen bytes each, and pass them through LDS to the lanes that the matrix cores want them in (rows of 128 bytes whose
// sixteen-byte pieces are exchanged by the row's number, so that neither side meets bank conflicts); read directly in that order, neighbouring lanes
// would hold different rows, and the L1 cache take four times the accesses: 16,384 x 4096 bf16 at rank 16 44 us, 40 this way (134 MB, 3.4 TB/s);
// 4096 x 2048 at rank 64 24 and 15.  Bound by waits, not by memory's rate: at 16,384 x 4096 waves wait 57% of their time, vector instructions take 5% of the cycles and the matrix
// cores 3%, with one block a CU (84 KB of LDS each), two waves a SIMD; above 64 ranks 300 registers leave one.  Neighbouring blocks begin at different columns: rows are
// often a multiple of 4 KB apart, and blocks that read the same columns at the same time would ask few of the memory's channels.
#define AD_DOWN_WAVES 8
// (rows without an adapter)
__device__ __forceinline__ void ad_zeros(uint64_t bits, uint32_t row, uint32_t *list, int rank, float *__restrict__ keep) {
    if (!bits) return;
    const int count = ad_list(bits, row, list, threadIdx.x & 63);
    for (int i = threadIdx.x; i < count * rank; i += blockDim.x) keep[(int64_t)list[i / rank] * rank + i % rank] = 0.0f;
    __builtin_amdgcn_wave_barrier();
}
// where the sixteen-byte piece p of row r lies
__device__ __forceinline__ int ad_slot(int r, int p) { return r * 8 + (p ^ (r >> 1 & 7)); }

template <class T, int RK, int NT, bool MASK>
__device__ __forceinline__ void ad_down(const T *__restrict__ x, int64_t ld_x, const T *__restrict__ w, int64_t ld_w, int d, int kb, int ke, int turn, int rank, int j0, float by,
                                        const uint32_t *list, int count, const VecMask &mask, VecKey key, ad_u4 *lds, int wave, int waves, float *__restrict__ part, int rp,
                                        float *__restrict__ keep) {
    constexpr int E = AD_COLS(T), COLS = 8 * E, KS = COLS / 32, N = NT + RK;  // columns of a piece and of a turn; instructions' worth; tiles
    const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, lr = lane >> 3, lp = lane & 7;
    ad_u4 *mine = lds + wave * N * 128;  // [tile][16 rows][8 pieces]
    // (rows without a position and ranks behind the last read another's: what they give is not stored)
    const T *from[N][2];
    uint32_t row[NT][2];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const int i = 16 * t + 8 * h + lr;
            row[t][h] = list[i < count ? i : 0];
            from[t][h] = x + (int64_t)row[t][h] * ld_x;
        }
#pragma unroll
        for (int j = 0; j < RK; ++j) {
            const int i = j0 + 16 * j + 8 * h + lr;
            from[NT + j][h] = w + (int64_t)(i < rank ? i : rank - 1) * ld_w;
        }
    }
    vec_f4 acc[NT][RK];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int j = 0; j < RK; ++j) acc[t][j] = (vec_f4)0.0f;
    vec_pack<T, E> v[N][2];
    auto put = [&](int col) {  // (col: the lane's)
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                vec_pack<T, E> o = v[t][h];
                if (MASK && t < NT) o = ad_drop<T, E>(o, ad_bits(key, mask, row[t < NT ? t : 0][h], (uint32_t)col >> 3) >> (E == 4 ? col & 4 : 0));
                mine[t * 128 + ad_slot(8 * h + lr, lp)] = __builtin_bit_cast(ad_u4, o);
            }
    };
    auto multiply = [&]() {
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            auto operand = [&](int t) {
                const ad_u4 *at = mine + t * 128;
                if constexpr (sizeof(T) == 2) {
                    return __builtin_bit_cast(vec_pack<T>, at[ad_slot(c, 4 * ks + g)]);
                } else {
                    vec_pack<T> o;
                    const vec_f4 lo = __builtin_bit_cast(vec_f4, at[ad_slot(c, 2 * g)]), hi = __builtin_bit_cast(vec_f4, at[ad_slot(c, 2 * g + 1)]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) o[i] = lo[i], o[4 + i] = hi[i];
                    return o;
                }
            };
            vec_pack<T> wv[RK];
#pragma unroll
            for (int j = 0; j < RK; ++j) wv[j] = operand(NT + j);
#pragma unroll
            for (int t = 0; t < NT; ++t) {
                const vec_pack<T> xv = operand(t);
#pragma unroll
                for (int j = 0; j < RK; ++j) acc[t][j] = ad_mul<T>(wv[j], xv, acc[t][j]);
            }
        }
    };
    const int span = waves * COLS, first = kb + COLS * wave, end = ke < d ? ke : d;
    const int whole = first + COLS <= end ? (end - first - COLS) / span + 1 : 0;  // the wave's turns whose columns are all there
    if (whole > 0) {
        turn %= whole;
        int col = first + turn * span + E * lp;
        auto request = [&]() {
#pragma unroll
            for (int t = 0; t < N; ++t)
#pragma unroll
                for (int h = 0; h < 2; ++h) v[t][h] = ad_load<T, E>(from[t][h], col);
        };
        request();
        for (int i = 0; i < whole; ++i) {
            put(col);
            if (++turn == whole) turn = 0;
            col = first + turn * span + E * lp;
            if (i + 1 < whole) request();
            multiply();
        }
    }
    if (first + whole * span < end) {
        const int col = first + whole * span + E * lp;
#pragma unroll
        for (int t = 0; t < N; ++t)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[t][h] = vec_load<T, E>(from[t][h] + (col < end ? col : 0), end - col, col);
        put(col);
        multiply();
    }
    auto store = [&](vec_f4 s, int at, int to) {  // ranks to .. + 3 of a row
        if (at >= count || to >= rp) return;
#pragma unroll
        for (int r = 0; r < 4; ++r) s[r] = to + r < rank ? s[r] * by : 0.0f;
        *(vec_f4 *)(part + (int64_t)list[at] * rp + to) = s;
        if (keep) vec_store<float, 4>(keep + (int64_t)list[at] * rank + to, rank - to, s);
    };
    if (waves == 1) {
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
            for (int j = 0; j < RK; ++j) store(acc[t][j], 16 * t + c, j0 + 16 * j + 4 * g);
        return;
    }
    // sums of the waves, G pairs of tiles a round
    constexpr int G = NT * RK < 4 ? NT * RK : 4;
    vec_f4 *red = (vec_f4 *)lds;
#pragma unroll
    for (int p0 = 0; p0 < NT * RK; p0 += G) {
        __syncthreads();
#pragma unroll
        for (int q = 0; q < G; ++q) red[(wave * G + q) * 64 + lane] = acc[(p0 + q) / RK][(p0 + q) % RK];
        __syncthreads();
        for (int i = threadIdx.x; i < G * 64; i += blockDim.x) {
            const int l = i & 63, q = p0 + (i >> 6);
            vec_f4 s = red[i];
            for (int u = 1; u < waves; ++u) s += red[u * G * 64 + i];
            store(s, 16 * (q / RK) + (l & 15), j0 + 16 * (q % RK) + 4 * (l >> 4));
        }
    }
    __syncthreads();
}

template <class T, int RK, bool MASK>
__global__ void __launch_bounds__(64 * (RK == 8 ? 4 : AD_DOWN_WAVES))
k_vec_ad_down(AdRows rows, const T *__restrict__ x, int64_t ld_x, AdMatrix m, const float *__restrict__ scales, float factor, VecMask mask, float *__restrict__ part,
              int64_t part_stride, int rp, int slabs, int per, int own, float *__restrict__ keep) {
    __shared__ uint32_t lists[AD_DOWN_WAVES][64];
    extern __shared__ __align__(16) unsigned char smem[];  // [waves][tiles of x and W][128] pieces of sixteen bytes; [waves][4][64] sums
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
    uint32_t *list = lists[wave];
    const int64_t block = vec_block(), at = slabs == 1 ? block : block / slabs;
    const int slab = (int)(block - at * slabs);
    const AdTile tile = ad_tile(rows, at, lane);
    VecKey key = {0, 0, 0};
    if (MASK) key = vec_key(mask);
    const int kb = slab * per, ke = kb + per < m.d ? kb + per : m.d;
    part += slab * part_stride;
    if (keep) ad_zeros(__ballot(tile.in && tile.id == rows.adapters), tile.row, list, m.rank, keep);
    const int room = ((rows.tp > 32 ? 4 : (rows.tp > 16 ? 2 : 1)) + RK) * 128;  // a wave's LDS: of its largest form, since others may be in another
    uint64_t todo = __ballot(tile.id < rows.adapters);
    for (int i = 0; todo; ++i) {
        const int e = __builtin_amdgcn_readlane(tile.id, __builtin_ctzll(todo));
        const uint64_t bits = __ballot(tile.id == e);
        todo &= ~bits;
        if (own && i % waves != wave) continue;
        const int count = ad_list(bits, tile.row, list, lane);
        const T *w = (const T *)m.p + e * m.stride;
        const float by = scales ? scales[e] * factor : factor;
        for (int j0 = 0; j0 < m.rank; j0 += 16 * RK) {
            // (its own wave: LDS and columns as a block of one)
#define GO(NT)                                                                                                                                          \
    ad_down<T, RK, NT, MASK>(x, ld_x, w, m.ld, m.d, kb, ke, (int)(at & 0xffff), m.rank, j0, by, list, count, mask, key,                                 \
                             (ad_u4 *)smem + (own ? wave * room : 0), own ? 0 : wave, own ? 1 : waves, part, rp, keep)
            if (RK <= 2 && count > 32) GO(RK <= 2 ? 4 : 1);
            else if (count > 16) GO(2);
            else GO(1);
#undef GO
        }
    }
}

// -------------------------------------------------------------------- join --
// What `outer` leaves of a gradient: sums of parts of a run.
struct AdOuter {
    void *out;
    int64_t ld, stride;   // of rows, of adapters
    float *part;          // [chunk][2][rank][dpad]
    int dpad, accumulate;
};
// The sums of ids whose positions several blocks held, and zeros for those without a row; both gradients in one launch, of its own or behind `up`'s blocks.
struct AdJoin {
    AdOuter o;
    int len, d;
};
struct AdJoins {
    AdJoin a, b;
    const uint32_t *starts;  // where the adapters' positions begin, or null
    int rank, narrow;        // narrow: the gradients are of type T, else float32
    int across;              // blocks of an adapter
};
template <class O>
__device__ __forceinline__ void ad_join_write(O *out, int left, int col, vec_f8 sum, bool accumulate) {
    if (accumulate) sum += vec_wide<O>(vec_load<O>(out, left, col));
    vec_store<O>(out, left, sum);
}
template <class T>
__device__ __forceinline__ void ad_join(const AdRows &rows, const AdJoins &js, int64_t block) {
    const int64_t per = (int64_t)js.across * rows.adapters;
    if (block >= 2 * per) return;
    const AdJoin &j = block >= per ? js.b : js.a;
    if (block >= per) block -= per;
    const AdOuter &o = j.o;
    __shared__ int64_t found[2];
    const uint32_t e = (uint32_t)(block / js.across), part = (uint32_t)(block - (int64_t)e * js.across);
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (js.starts) {
        if (threadIdx.x < 2) found[threadIdx.x] = js.starts[e + threadIdx.x];
    } else if (wave < 2) {  // the first position whose key is at least e (at least e + 1), a 64th of what is left a round
        int64_t lo = 0, hi = rows.n;
        while (lo < hi) {
            const int64_t step = (hi - lo + 63) / 64, p = lo + lane * step;
            const uint64_t below = __ballot(p < hi && rows.keys[p < hi ? p : lo] < e + wave);  // (a prefix of the lanes)
            const int k = __popcll(below);
            if (k == 0) break;
            hi = lo + k * step < hi ? lo + k * step : hi;
            lo += (k - 1) * step + 1;
        }
        if (lane == 0) found[wave] = lo;
    }
    __syncthreads();
    const int64_t lo = found[0], hi = found[1];
    // (len is a power of two)
    const int shift = __builtin_ctz(j.len);
    const int64_t from = lo >> shift, to = lo < hi ? (hi - 1) >> shift : 0;
    if (lo < hi ? from == to : o.accumulate) return;
    const int pieces = o.dpad / 8;
    for (uint32_t i = part * 256 + threadIdx.x; i < (uint32_t)js.rank * pieces; i += js.across * 256) {  // (at most 2^25)
        const int r = (int)(i / (uint32_t)pieces), col = (int)(i - (uint32_t)r * pieces) * 8;
        vec_f8 sum = (vec_f8)0.0f;
        if (lo < hi) {
            const int64_t each = 2 * (int64_t)js.rank * o.dpad;
            const float *p = o.part + (int64_t)r * o.dpad + col;
            sum = *(const vec_f8 *)(p + from * each + each / 2);
            int64_t k = from + 1;
            for (; k + 8 <= to + 1; k += 8) {
                vec_f8 v[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) v[u] = *(const vec_f8 *)(p + (k + u) * each);
#pragma unroll
                for (int u = 0; u < 8; ++u) sum += v[u];
            }
            for (; k <= to; ++k) sum += *(const vec_f8 *)(p + k * each);
        }
        const int64_t at = e * o.stride + r * o.ld + col;
        if (js.narrow) ad_join_write((T *)o.out + at, j.d - col, col, sum, o.accumulate);
        else ad_join_write((float *)o.out + at, j.d - col, col, sum, o.accumulate);
    }
}
template <class T>
__global__ void __launch_bounds__(256)
k_vec_ad_join(AdRows rows, AdJoins js) {
    ad_join<T>(rows, js, vec_block());
}

// ---------------------------------------------------------------------- up --
// y_row = base_row + (kept) f_row W_e.  A block takes a tile of positions and 64 AD_COLS columns at a time, a quarter a wave.  The factor f is made ready
// in LDS once (its parts as the matrix cores take them); a lane reads eight ranks of AD_COLS columns of W, whose columns are put together from
// their halves by byte permutations.  The products' 16 rows pass through LDS, so that sixteen neighbouring lanes read and write a row's 256 bytes: from
// the matrix cores' own order, where neighbouring lanes hold different rows, every sixteen bytes would be an access of their own (16,384 x 4096 bf16 at rank 16 60 us, 53
// this way: 268 MB, the rate of a large copy).
// MASK: 0 without dropout, 1 the mask is made here, 2 its bits are read.
template <class T, class Y, int MASK, int E>
struct AdUp {
    static constexpr int LD = 16 * E + 4;  // floats between two rows in LDS (lanes of a quarter wave then write to different banks)
    const Y *base;
    Y *y;
    int64_t ld_base, ld_y;
    int d;
    VecMask mask;
    const uint32_t *bits;
    VecKey key;
    float *lds;  // the wave's own [16][LD]

    // a lane's part of four rows: row 4 i + lane / 16, columns c0 + E (lane % 16) and on
    __device__ __forceinline__ int column(int c0) const { return c0 + E * (threadIdx.x & 15); }
    __device__ __forceinline__ void read(vec_pack<Y, E> *b, const uint32_t *rows, int c0) const {
        if (!base) return;
        const int from = ad_from<E>(column(c0), d);
#pragma unroll
        for (int i = 0; i < 4; ++i) b[i] = ad_load<Y, E>(base + (int64_t)rows[i] * ld_base, from);
    }
    // acc[m][i]: of row lane % 16, column E (4 (lane / 16) + i) + m
    __device__ __forceinline__ void write(const vec_f4 *acc, const vec_pack<Y, E> *b, const uint32_t *mask_bits, const uint32_t *rows, int left, int c0) const {
        const int lane = threadIdx.x & 63, c = lane & 15, g = lane >> 4, col = column(c0);
        float *to = lds + c * LD + 4 * E * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (E == 1) {
                to[i] = acc[0][i];
            } else {
#pragma unroll
                for (int m = 0; m < E; m += 4) *(vec_f4 *)(to + E * i + m) = (vec_f4){acc[m][i], acc[m + 1][i], acc[m + 2][i], acc[m + 3][i]};
            }
        }
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            vec_f<E> f;
            const float *at = lds + (4 * i + g) * LD + E * c;
            if constexpr (E == 1) {
                f[0] = at[0];
            } else {
#pragma unroll
                for (int m = 0; m < E; m += 4) {
                    const vec_f4 u = *(const vec_f4 *)(at + m);
#pragma unroll
                    for (int k = 0; k < 4; ++k) f[m + k] = u[k];
                }
            }
            if (4 * i + g >= left || col >= d) continue;
            if (MASK) {
                const uint32_t kept = MASK == 2 ? mask_bits[i] : ad_kept<E>(key, mask, rows[i], ad_from<E>(col, d));
#pragma unroll
                for (int m = 0; m < E; ++m) f[m] = kept >> m & 1 ? f[m] : 0.0f;
            }
            if (base) f += vec_wide<Y, E>(b[i]);
            ad_store<Y, E>(y + (int64_t)rows[i] * ld_y, col, d, f);
        }
        __builtin_amdgcn_wave_barrier();
    }
};

// f of the list's rows, 32 ranks (chunk kc) a slot: lane holds row lane % 16 of the tile and ranks 8 (lane / 16) and on.
template <class T>
__device__ __forceinline__ void ad_ready(const AdFactor &f, int rank, int chunks, const uint32_t *list, int count, int tiles, ad_u4 *ready, float *__restrict__ keep) {
    constexpr int P = AdWide<T>::parts;
    for (int i = threadIdx.x; i < tiles * chunks * 64; i += 256) {
        const int l = i & 63, t = (i >> 6) % tiles, kc = (i >> 6) / tiles;
        const int at = 16 * t + (l & 15), r0 = 32 * kc + 8 * (l >> 4);
        vec_f8 v = (vec_f8)0.0f;
        if (at < count && r0 < f.ld) {  // (rows are padded to sixteen ranks, with zeros)
            const float *p = f.p + (int64_t)list[at] * f.ld + r0;
            v = *(const vec_f8 *)p;
            for (int s = 1; s < f.slabs; s += 3) {  // three on their way
                vec_f8 w[3];
#pragma unroll
                for (int u = 0; u < 3; ++u) w[u] = *(const vec_f8 *)(p + (s + u < f.slabs ? s + u : 0) * f.stride);
#pragma unroll
                for (int u = 0; u < 3; ++u)
                    if (s + u < f.slabs) v += w[u];
            }
            if (keep) vec_store<float>(keep + (int64_t)list[at] * rank + r0, rank - r0, v);
        }
        AdWide<T> o;
        o.set(v);
#pragma unroll
        for (int s = 0; s < P; ++s) ready[(((kc * tiles + t) * P) + s) * 64 + l] = o.p[s];
    }
}

// The rows of a list and a wave's 16 E columns from c0 on: requested, then computed.
template <class T, class Y, int MASK, bool ONE, int E>
struct AdUpPass {
    static constexpr int P = AdWide<T>::parts;
    const AdUp<T, Y, MASK, E> &up;
    const AdMatrix &m;
    const T *w;  // null: no adapter
    const uint32_t *list, *place;
    int count, chunks, c0;
    vec_pack<T, E> raw[8];
    vec_pack<Y, E> b[4];
    uint32_t at[4], kept[4];  // the rows of b, their bits of the mask

    // (lanes without a rank read the last one's: their part of the factor is zero)
    __device__ __forceinline__ void weights(int kc) {
        const int g = (threadIdx.x & 63) >> 4, from = ad_from<E>(up.column(c0), m.d);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int r = 32 * kc + 8 * g + q;
            raw[q] = ad_load<T, E>(w + (int64_t)(r < m.rank ? r : m.rank - 1) * m.ld, from);
        }
    }
    __device__ __forceinline__ int entry(int t, int i) const {
        const int k = 16 * t + 4 * i + ((threadIdx.x & 63) >> 4);
        return k < count ? k : 0;
    }
    __device__ __forceinline__ void rows(int t, uint32_t *to) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = list[entry(t, i)];
    }
    __device__ __forceinline__ void masks(int t, uint32_t *to) const {
        if (MASK != 2) return;
        const int from = ad_from<E>(up.column(c0), m.d);
#pragma unroll
        for (int i = 0; i < 4; ++i) to[i] = ad_bits_of(up.bits, place[entry(t, i)], m.d, from);
    }
    __device__ __forceinline__ void request(int from) {
        c0 = from;
        if (w) weights(0);
        rows(0, at);
        if (ONE) masks(0, kept);
        up.read(b, at, c0);
    }
    __device__ __forceinline__ void run(const ad_u4 *ready) {
        const int lane = threadIdx.x & 63, tiles = (count + 15) / 16;
        auto factor = [&](int kc, int t) {
            AdWide<T> o;
#pragma unroll
            for (int s = 0; s < P; ++s) o.p[s] = ready[((kc * tiles + t) * P + s) * 64 + lane];
            return o;
        };
        if constexpr (ONE) {
            for (int t = 0; t < tiles; ++t) {
                vec_pack<Y, E> next[4];
                uint32_t then[4], more[4];
                if (t + 1 < tiles) {
                    rows(t + 1, then);
                    masks(t + 1, more);
                    up.read(next, then, c0);
                }
                vec_f4 acc[E];
#pragma unroll
                for (int i = 0; i < E; ++i) acc[i] = (vec_f4)0.0f;
                if (w) {
                    const AdWide<T> a = factor(0, t);
                    if constexpr (sizeof(T) == 2 && E > 1)  // (fp16 columns as two bfloat16 numbers, all at once, are registers that the rows on their way need)
#pragma unroll
                        for (int q = 0; q < 8; ++q) asm volatile("" : "+v"(raw[q]));
#pragma unroll
                    for (int i = 0; i < E; ++i) {
                        acc[i] = ad_mul<T, false>(ad_column<T, E>(raw, i), a, acc[i]);
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                up.write(acc, b, kept, at, count - 16 * t, c0);
#pragma unroll
                for (int i = 0; i < 4; ++i) b[i] = next[i], at[i] = then[i], kept[i] = more[i];
            }
        } else {  // (tiles of at most 32 positions)
            vec_f4 acc[2][E];
#pragma unroll
            for (int i = 0; i < E; ++i) acc[0][i] = acc[1][i] = (vec_f4)0.0f;
            for (int kc = 0; kc < (w ? chunks : 0); ++kc) {
                vec_pack<T, E> here[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) here[q] = raw[q];
                if (kc + 1 < chunks) weights(kc + 1);
                const AdWide<T> a = factor(kc, 0), a1 = factor(kc, tiles > 1 ? 1 : 0);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const AdNarrow<T> o = ad_column<T, E>(here, i);
                    acc[0][i] = ad_mul<T, false>(o, a, acc[0][i]);
                    if (tiles > 1) acc[1][i] = ad_mul<T, false>(o, a1, acc[1][i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
            masks(0, kept);
            up.write(acc[0], b, kept, at, count, c0);
            if (tiles > 1) {
                rows(1, at);
                masks(1, kept);
                up.read(b, at, c0);
                up.write(acc[1], b, kept, at, count - 16, c0);
            }
        }
    }
};

// ONE: at most 32 ranks.  JOIN: blocks behind `blocks` join the gradients of the factors, which nothing here reads, so that a launch is saved.
template <class T, class Y, int MASK, bool ONE, int E, bool JOIN>
__global__ void __launch_bounds__(256, 2)
k_vec_ad_up(AdRows rows, AdFactor f, AdMatrix m, const Y *base, int64_t ld_base, Y *y, int64_t ld_y, VecMask mask, int column_blocks, float *__restrict__ keep,
            const uint32_t *__restrict__ bits, int64_t blocks, AdJoins js) {
    if (JOIN && vec_block() >= blocks) return ad_join<T>(rows, js, vec_block() - blocks);
    extern __shared__ __align__(16) unsigned char smem[];
    ad_u4 *ready = (ad_u4 *)smem;  // [chunk][tile][part][lane]
    __shared__ uint32_t lists[4][64], places[4][MASK == 2 ? 64 : 1];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    uint32_t *list = lists[wave];
    const int64_t block = vec_block(), at = block / column_blocks;
    const int first = (int)(block - at * column_blocks) * 64 * E + wave * 16 * E, step = column_blocks * 64 * E;
    const AdTile tile = ad_tile(rows, at, lane);
    const int chunks = ONE ? 1 : (m.rank + 31) / 32;
    __shared__ __align__(16) float out[4][16 * AdUp<T, Y, MASK, E>::LD];
    AdUp<T, Y, MASK, E> up = {base, y, ld_base, ld_y, m.d, mask, bits, {0, 0, 0}, out[wave]};
    if (MASK == 1) up.key = vec_key(mask);
    if (block != at * column_blocks) keep = nullptr;  // (a tile's first block writes it)
    if (keep) ad_zeros(__ballot(tile.in && tile.id == rows.adapters), tile.row, list, m.rank, keep);
    uint64_t todo = __ballot(tile.in);
    while (todo) {
        const int e = __builtin_amdgcn_readlane(tile.id, __builtin_ctzll(todo));
        const uint64_t same = __ballot(tile.in && tile.id == e);
        todo &= ~same;
        const bool none = e == rows.adapters;
        if (none && base == y) continue;
        const int count = ad_list(same, tile.row, list, lane), tiles = (count + 15) / 16;
        if (MASK == 2) ad_list(same, (uint32_t)(at * rows.tp + lane), places[wave], lane);
        const T *w = none ? nullptr : (const T *)m.p + e * m.stride;
        // what the first tile needs is asked for before the factor is made ready
        AdUpPass<T, Y, MASK, ONE, E> pass = {up, m, w, list, places[wave], count, chunks};
        if (first < m.d) pass.request(first);
        if (!none) {
            ad_ready<T>(f, m.rank, chunks, list, count, tiles, ready, keep);
            __syncthreads();
        }
        for (int c0 = first; c0 < m.d; c0 += step) {
            if (c0 != first) pass.request(c0);
            pass.run(ready);
        }
        if (todo) __syncthreads();
    }
}

// The same for few rows of an adapter: on the vector units, without a wait between waves.  A wave takes a tile of at most eight positions and 64 E columns, E a lane;
// four rows of one adapter share what it reads of W.  Where a tile of the matrix cores would hold three rows of sixteen, the rest of the form above (the parts of the
// factor, columns put together, LDS) costs more than these products: 8192 mixed rows of 500 adapters, 1001 fp16
// columns at rank 8: 26 us above, 21 here; 16,384 of 1000, 4096 bf16 columns at rank 16: 91 above, 151 here.
#define AD_FEW_POSITIONS 8
template <class T, class Y, int MASK, int E, bool JOIN>
__global__ void __launch_bounds__(256, 2)
k_vec_ad_up_few(AdRows rows, const float *__restrict__ f, int64_t ld_f, int64_t f_stride, int f_slabs, AdMatrix m, const Y *base, int64_t ld_base, Y *y, int64_t ld_y,
                VecMask mask, int column_blocks, float *__restrict__ keep, const uint32_t *__restrict__ bits, int64_t blocks, AdJoins js) {
    if (JOIN && vec_block() >= blocks) return ad_join<T>(rows, js, vec_block() - blocks);
    const int lane = threadIdx.x & 63;
    const int64_t item = vec_block() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), at = item / column_blocks;
    if (at * rows.tp >= rows.n) return;
    const int slab = (int)(item - at * column_blocks), col = slab * 64 * E + E * lane, from = ad_from<E>(col, m.d);
    const AdTile tile = ad_tile(rows, at, lane);
    VecKey key = {0, 0, 0};
    if (MASK == 1) key = vec_key(mask);
    uint64_t todo = __ballot(tile.in);
    while (todo) {
        const int e = __builtin_amdgcn_readlane(tile.id, __builtin_ctzll(todo));
        const uint64_t same = __ballot(tile.in && tile.id == e);
        const bool none = e == rows.adapters;
        const T *w = (const T *)m.p + (none ? 0 : e * m.stride) + from;
        // the first four rows of e
        int row[4], place[4], count = 0;
        uint64_t mine = todo & same;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            count += mine != 0;
            place[k] = mine ? __builtin_ctzll(mine) : __builtin_ctzll(same);
            row[k] = __builtin_amdgcn_readlane((int)tile.row, place[k]);
            todo &= ~(mine & -mine);
            mine &= mine - 1;
        }
        vec_f<E> acc[4];
        vec_pack<Y, E> b[4];
        uint32_t kept[4];
        if (MASK == 2)
#pragma unroll
            for (int k = 0; k < 4; ++k) kept[k] = ad_bits_of(bits, at * rows.tp + place[k], m.d, from);
        if (base && !(none && base == y))
#pragma unroll
            for (int k = 0; k < 4; ++k) b[k] = ad_load<Y, E>(base + (uint32_t)row[k] * ld_base, from);
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[k] = (vec_f<E>)0.0f;
        for (int r64 = 0; r64 < m.rank; r64 += 64) {
            if (none && !(keep && slab == 0)) break;
            vec_pack<T, E> raw[8];
            auto request = [&](int r0) {  // (behind the last rank that one again, beside zeros of the factor)
#pragma unroll
                for (int q = 0; q < 8; ++q) raw[q] = *(const vec_pack<T, E> *)(w + (int64_t)(r0 + q < m.rank ? r0 + q : m.rank - 1) * m.ld);
            };
            if (!none) request(r64);
            // a lane has one rank of the factor, the sum of its parts
            float t[4] = {};
            const int r = r64 + lane;
            if (!none && r < ld_f) {
                for (int s = 0; s < f_slabs; s += 4) {  // four on their way
                    float part[4][4];
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int u = 0; u < 4; ++u) part[k][u] = k < count ? f[(s + u < f_slabs ? s + u : s) * f_stride + (uint32_t)row[k] * ld_f + r] : 0.0f;
#pragma unroll
                    for (int k = 0; k < 4; ++k)
#pragma unroll
                        for (int u = 0; u < 4; ++u) t[k] += s + u < f_slabs ? part[k][u] : 0.0f;
                }
            }
            if (keep && slab == 0 && r < m.rank)
#pragma unroll
                for (int k = 0; k < 4; ++k)
                    if (k < count) keep[(int64_t)row[k] * m.rank + r] = t[k];
            if (none) continue;
            for (int r0 = 0; r0 < 64 && r64 + r0 < m.rank; r0 += 8) {
                vec_pack<T, E> here[8];
#pragma unroll
                for (int q = 0; q < 8; ++q) here[q] = raw[q];
                if (r0 + 8 < 64 && r64 + r0 + 8 < m.rank) request(r64 + r0 + 8);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const vec_f<E> v = vec_wide<T, E>(here[q]);
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        if (k < count) {
                            const float by = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(t[k]), r0 + q));
#pragma unroll
                            for (int i = 0; i < E; ++i) acc[k][i] = __fmaf_rn(by, v[i], acc[k][i]);
                        }
                }
            }
        }
        if (none && base == y) continue;
        if (col >= m.d) continue;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            if (k >= count) break;
            if (MASK) {
                if (MASK == 1) kept[k] = ad_kept<E>(key, mask, (uint32_t)row[k], from);
#pragma unroll
                for (int i = 0; i < E; ++i) acc[k][i] = kept[k] >> i & 1 ? acc[k][i] : 0.0f;
            }
            if (base) acc[k] += vec_wide<Y, E>(b[k]);
            ad_store<Y, E>(y + (uint32_t)row[k] * ld_y, col, m.d, acc[k]);
        }
    }
}

// ------------------------------------------------------------ single tokens --
// Both products in one launch, for rows of their own adapters: a block takes a row and 64 AD_COLS columns of the result, and makes the row's t itself, so
// that A is read once for each of these (from the L2 cache).  Its eight waves share the columns of x, AD_ONE_TILES KB of A on their way each, then the ranks of B, which is asked
// for before.  4096 x 4096 bf16 at rank 16, us in a graph by two kernels / by this: 1 row 8.8 / 5.4, 16 9.1 / 5.6, 32 (33 MB of A read) 8.6 / 5.9 (7.0 with a row's blocks on all
// XCDs, each of which then fetches A), 64 (67 MB) 9.7 / 8.5 (12.5); 16 rows at rank 64 10.7 / 10.3.
#define AD_ONE_TILES 4
template <class T, class Y, int RK, int E>
__global__ void __launch_bounds__(512)
k_vec_ad_one(AdRows rows, const T *__restrict__ x, int64_t ld_x, AdMatrix ma, AdMatrix mb, const float *__restrict__ scales, float factor, VecMask mask, const Y *base,
             int64_t ld_base, Y *y, int64_t ld_y, float *__restrict__ keep, int column_blocks) {
    constexpr int EA = AD_COLS(T), COLS = 8 * EA, KS = COLS / 32, U = AD_ONE_TILES / RK, BR = 2 * RK;  // U: turns on their way; BR: ranks of B a wave
    constexpr int LDS = 8 * U * RK * 128;
    __shared__ ad_u4 tiles[LDS > 32 * E * 4 ? LDS : 32 * E * 4];  // [wave][turn][16 ranks][16 rows][8 pieces]; [wave][64 E] sums
    __shared__ float sums[8][16 * RK], t[16 * RK];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 15, g = lane >> 4, lr = lane >> 3, lp = lane & 7;
    // (eight rows in turn, so that the blocks of a row are on one XCD, whose L2 cache reads A once for them)
    const int block = (int)vec_block(), eight = block / (8 * column_blocks) * 8, r = block - eight * column_blocks, many = rows.n - eight < 8 ? (int)rows.n - eight : 8;
    if (eight >= rows.n) return;
    const int slab = r / many, row = eight + r - slab * many, c0 = slab * 64 * E, d = ma.d, rank = ma.rank;
    const int e = __builtin_amdgcn_readfirstlane(ad_id(rows, row));
    const bool none = e == rows.adapters;
    const int own = c0 + (int)threadIdx.x;  // the thread's column of the result
    const bool writes = threadIdx.x < 64 * E && own < mb.d;
    float old = 0.0f;
    if (writes && base) old = (float)base[row * ld_base + own];
    if (keep && slab == 0 && none && (int)threadIdx.x < rank) keep[row * rank + threadIdx.x] = 0.0f;
    if (none) {
        if (writes && base != y) y[row * ld_y + own] = (Y)old;
        return;
    }
    const T *a = (const T *)ma.p + e * ma.stride, *b = (const T *)mb.p + e * mb.stride;
    const T *xr = x + row * ld_x;
    const int from = ad_from<E>(c0 + E * lane, mb.d);
    vec_pack<T, E> bv[BR];  // ranks wave BR and on (behind the last that one again)
#pragma unroll
    for (int q = 0; q < BR; ++q) bv[q] = ad_load<T, E>(b + (int64_t)(wave * BR + q < rank ? wave * BR + q : rank - 1) * mb.ld, from);
    ad_u4 *mine = tiles + wave * U * RK * 128;
    vec_f4 acc[RK];
#pragma unroll
    for (int j = 0; j < RK; ++j) acc[j] = (vec_f4)0.0f;
    const T *ar[RK][2];
#pragma unroll
    for (int j = 0; j < RK; ++j)
#pragma unroll
        for (int h = 0; h < 2; ++h) ar[j][h] = a + (int64_t)(16 * j + 8 * h + lr < rank ? 16 * j + 8 * h + lr : rank - 1) * ma.ld;
    vec_pack<T, EA> v[U][RK][2];
    vec_pack<T> xv[U][KS];
    VecKey key = {0, 0, 0};
    if (mask.threshold) key = vec_key(mask);
    auto multiply = [&](int u, int k) {  // k: the turn's first column
        if (mask.threshold)
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) xv[u][ks] = vec_drop<T>(xv[u][ks], vec_kept(vec_random(key, mask.layer, (uint32_t)row, (uint32_t)(k + 32 * ks + 8 * g) >> 3), mask.threshold));
#pragma unroll
        for (int ks = 0; ks < KS; ++ks)
#pragma unroll
            for (int j = 0; j < RK; ++j) {
                const ad_u4 *at = mine + (u * RK + j) * 128;
                vec_pack<T> w;
                if constexpr (sizeof(T) == 2) {
                    w = __builtin_bit_cast(vec_pack<T>, at[ad_slot(c, 4 * ks + g)]);
                } else {
                    const vec_f4 lo = __builtin_bit_cast(vec_f4, at[ad_slot(c, 2 * g)]), hi = __builtin_bit_cast(vec_f4, at[ad_slot(c, 2 * g + 1)]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) w[i] = lo[i], w[4 + i] = hi[i];
                }
                acc[j] = ad_mul<T>(w, xv[u][ks], acc[j]);
            }
    };
    auto put = [&](int u) {
#pragma unroll
        for (int j = 0; j < RK; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) mine[(u * RK + j) * 128 + ad_slot(8 * h + lr, lp)] = __builtin_bit_cast(ad_u4, v[u][j][h]);
    };
    const int first = COLS * wave, span = 8 * COLS, whole = first + COLS <= d ? (d - first - COLS) / span + 1 : 0;
    for (int i = 0; i < whole; i += U) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (i + u >= whole) continue;
            const int k = first + (i + u) * span;
#pragma unroll
            for (int j = 0; j < RK; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) v[u][j][h] = ad_load<T, EA>(ar[j][h], k + EA * lp);
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) xv[u][ks] = *(const vec_pack<T> *)(xr + k + 32 * ks + 8 * g);
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u < whole) put(u);
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (i + u < whole) multiply(u, first + (i + u) * span);
    }
    if (first + whole * span < d) {
        const int k = first + whole * span, ca = k + EA * lp;
#pragma unroll
        for (int j = 0; j < RK; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) v[0][j][h] = vec_load<T, EA>(ar[j][h] + (ca < d ? ca : 0), d - ca, ca);
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            const int cx = k + 32 * ks + 8 * g;
            xv[0][ks] = vec_load<T>(xr + (cx < d ? cx : 0), d - cx, cx);
        }
        put(0);
        multiply(0, k);
    }
    if (c == 0)  // (all sixteen columns of the products are the row)
#pragma unroll
        for (int j = 0; j < RK; ++j) *(vec_f4 *)&sums[wave][16 * j + 4 * g] = acc[j];
    __syncthreads();
    if (threadIdx.x < 16 * RK) {
        float s = 0.0f;
#pragma unroll
        for (int u = 0; u < 8; ++u) s += sums[u][threadIdx.x];
        s = (int)threadIdx.x < rank ? s * (scales ? scales[e] * factor : factor) : 0.0f;
        t[threadIdx.x] = s;
        if (keep && slab == 0 && (int)threadIdx.x < rank) keep[row * rank + threadIdx.x] = s;
    }
    __syncthreads();
    float *part = (float *)tiles;  // [wave][64 E]
    vec_f<E> f = (vec_f<E>)0.0f;
#pragma unroll
    for (int q = 0; q < BR; ++q) {
        const vec_f<E> w = vec_wide<T, E>(bv[q]);
        const float by = t[wave * BR + q];
#pragma unroll
        for (int i = 0; i < E; ++i) f[i] = __fmaf_rn(by, w[i], f[i]);
    }
#pragma unroll
    for (int i = 0; i < E; ++i) part[wave * 64 * E + lane * E + i] = f[i];
    __syncthreads();
    if (!writes) return;
    // column `own` is value i of lane l, whose columns begin at its `from`
    const int l = (int)threadIdx.x / E, i = own - ad_from<E>(c0 + E * l, mb.d);
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < 8; ++u) s += part[u * 64 * E + l * E + i];
    y[row * ld_y + own] = (Y)(old + s);
}

// ------------------------------------------------------------------- outer --
// G_e[j][col] = sum over the rows of e of f_row[j] (kept) x_row[col].  A block takes `len` sorted positions and 256 columns, a quarter a wave, in steps of 32
// positions whatever runs of equal ids these hold: the rows of a step are read once, and each run among them takes its own and zeros for the others.  Runs that lie within the block's positions are written; the others' sums go to part[chunk][0] (began before)
// or part[chunk][1], which the join adds up in order.  Per step a lane reads eight rows of four columns.  Bound by the vector units, which put columns together and make the mask:
// 16,384 x (4096 + 4096) bf16 at rank 16 with dropout 81 us (288 MB read, 66% of the cycles with a vector instruction), 10,000 x (1001 + 700) fp16 of 200
// adapters 27 (34 with columns put together for each run of a step, not once), 1024 x (256 + 96) float32 8.
#define AD_STAGE 128  // positions whose factors are made ready at once
template <class O, int E>
__device__ __forceinline__ void ad_put(O *row, int col, int d, vec_f<E> v, bool accumulate) {
    if (accumulate) v += vec_wide<O, E>(ad_load<O, E>(row, ad_from<E>(col, d)));
    ad_store<O, E>(row, col, d, v);
}

// Both gradients are one launch: db's blocks first, then da's, whose rows are masked.
#define AD_MAX_LEN 1024  // positions of a block at most
struct AdSide {
    AdFactor f;
    const void *x;
    int64_t ld_x;
    int d, len, column_blocks;  // len: positions of a block
    AdOuter o;
};
template <class T, class O, int RK, bool MASK, int E>
__global__ void __launch_bounds__(256, sizeof(T) == 4 && RK == 4 ? 1 : 2)
k_vec_ad_outer(AdRows rows, int rank, VecMask mask, AdSide sb, AdSide sa, int64_t blocks_b, uint32_t *__restrict__ bits) {
    constexpr int P = AdWide<T>::parts;
    int64_t block = vec_block();
    const bool masked = block >= blocks_b;
    const AdSide &side = masked ? sa : sb;
    if (masked) block -= blocks_b;
    const AdFactor f = side.f;
    const AdOuter o = side.o;
    const T *__restrict__ const x = (const T *)side.x;
    const int64_t ld_x = side.ld_x;
    const int d = side.d, len = side.len, column_blocks = side.column_blocks;
    __shared__ ad_u4 ready[AD_STAGE / 32 * RK * P * 64];  // [step][16 ranks][part][lane]
    __shared__ uint32_t keys[AD_MAX_LEN], at[AD_MAX_LEN];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane >> 4;
    const int64_t chunk = block / column_blocks, p0 = chunk * len;
    if (p0 >= rows.n) return;
    const int size = (int)(rows.n - p0 < len ? rows.n - p0 : len);
    const int c0 = ((int)(block - chunk * column_blocks) * 4 + wave) * 16 * E, col = c0 + E * (lane & 15), from = ad_from<E>(col, d), j0 = blockIdx.z * 16 * RK;
    VecKey key = {0, 0, 0};
    if (MASK && masked) key = vec_key(mask);
    int total = size;
    if (size > 0 && rows.keys[p0 + size - 1] >= (uint32_t)rows.adapters) {  // (rows without an adapter come last)
        total = 0;
        for (int i = lane; i < (size + 63) / 64 * 64; i += 64) total += __popcll(__ballot(i < size && rows.keys[p0 + (i < size ? i : 0)] < (uint32_t)rows.adapters));
    }
    if (total == 0) return;
    for (int i = threadIdx.x; i < total; i += 256) {
        keys[i] = rows.keys[p0 + i];
        at[i] = rows.pos[p0 + i];
    }
    const uint32_t before_key = p0 > 0 ? rows.keys[p0 - 1] : 0xffffffffu, behind_key = p0 + total < rows.n ? rows.keys[p0 + total] : 0xffffffffu;
    __syncthreads();
    auto request = [&](vec_pack<T, E> *v, int s0) {  // positions s0 + 8 g and on; behind the last that one again, beside zeros of the factor
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            const int i = s0 + 8 * g + q;
            v[q] = ad_load<T, E>(x + (int64_t)at[i < total ? i : total - 1] * ld_x, from);
        }
    };
    vec_f4 acc[RK][E];
    auto clear = [&]() {
#pragma unroll
        for (int j = 0; j < RK; ++j)
#pragma unroll
            for (int i = 0; i < E; ++i) acc[j][i] = (vec_f4)0.0f;
    };
    clear();
    vec_pack<T, E> raw[8];
    request(raw, 0);
    const bool whole = __builtin_amdgcn_readfirstlane(c0) + 16 * E <= d || d % 8 == 0;  // (then neighbours end together)
    int a = 0;  // where the run in hand begins
    for (int s0 = 0; s0 < total; s0 += AD_STAGE) {
        const int m = total - s0 < AD_STAGE ? total - s0 : AD_STAGE;
        __syncthreads();
        for (int i = threadIdx.x; i < (m + 31) / 32 * RK * 64; i += 256) {
            const int l = i & 63, j = (i >> 6) % RK, st = (i >> 6) / RK;
            const int r = j0 + 16 * j + (l & 15), q0 = 32 * st + 8 * (l >> 4);
            const float *p = f.p + (r < rank ? r : 0);
            vec_f8 v;
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = p[(int64_t)at[s0 + (q0 + q < m ? q0 + q : 0)] * f.ld];
            for (int s = 1; s < f.slabs; s += 4) {  // four parts on their way
                float more[4][8];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int q = 0; q < 8; ++q) more[u][q] = p[(s + u < f.slabs ? s + u : 0) * f.stride + (int64_t)at[s0 + (q0 + q < m ? q0 + q : 0)] * f.ld];
#pragma unroll
                for (int u = 0; u < 4; ++u)
#pragma unroll
                    for (int q = 0; q < 8; ++q) v[q] += s + u < f.slabs ? more[u][q] : 0.0f;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = q0 + q < m && r < rank ? __builtin_canonicalizef(v[q]) : 0.0f;
            AdWide<T> w;
            w.set(v);
#pragma unroll
            for (int s = 0; s < P; ++s) ready[((st * RK + j) * P + s) * 64 + l] = w.p[s];
        }
        __syncthreads();
        for (int st = 0; 32 * st < m; ++st) {
            const int here = s0 + 32 * st, behind = here + 32 < total ? here + 32 : total;
            vec_pack<T, E> next[8];
            if (here + 32 < total) request(next, here + 32);
            if (MASK && masked)
                ad_drop8<T, E>(raw, key, mask, [&](int q) { return at[here + 8 * g + q < total ? here + 8 * g + q : total - 1]; }, from, whole, [&](int half, uint32_t word) {
                    const int i = here + 8 * g + 4 * half;
                    if (bits && blockIdx.z == 0 && col < d && i < total) bits[((p0 + i) >> 2) * (d / 8) + (col >> 3)] = word;
                });
            // the runs that the step holds, or parts of
            const uint32_t mine = keys[here + (lane & 31) < behind ? here + (lane & 31) : behind - 1];
            const uint64_t heads = __ballot(lane < behind - here && (here + lane == 0 || keys[here + lane > 0 ? here + lane - 1 : 0] != mine)) | 1ull << (behind - here);
            AdNarrow<T> v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) v[i] = ad_column<T, E>(raw, i);
            for (int lo = here; lo < behind;) {
                const int hi = here + __builtin_ctzll(heads >> (lo - here + 1)) + (lo - here + 1);
                auto factor = [&](int j) {
                    AdWide<T> w;
#pragma unroll
                    for (int s = 0; s < P; ++s) w.p[s] = ready[((st * RK + j) * P + s) * 64 + lane];
                    return w;
                };
                if (lo == here && hi == behind) {  // all of the step's rows are of this run
#pragma unroll
                    for (int j = 0; j < RK; ++j) {
                        const AdWide<T> w = factor(j);
#pragma unroll
                        for (int i = 0; i < E; ++i) acc[j][i] = ad_mul<T, true>(v[i], w, acc[j][i]);
                        __builtin_amdgcn_sched_barrier(0);  // (all ranks' factors at once are registers that the rows on their way need)
                    }
                } else {  // others' rows take no part, whatever they hold
                    uint32_t in = 0;
#pragma unroll
                    for (int q = 0; q < 8; ++q) in |= (here + 8 * g + q >= lo && here + 8 * g + q < hi ? 1u : 0u) << q;
                    AdNamed<T> its;
                    its.set(in);
#pragma unroll
                    for (int j = 0; j < RK; ++j) {
                        AdWide<T> w = factor(j);
                        w.only(its);
#pragma unroll
                        for (int i = 0; i < E; ++i) {
                            AdNarrow<T> o = v[i];
                            o.only(its);
                            acc[j][i] = ad_mul<T, true>(o, w, acc[j][i]);
                        }
                        __builtin_amdgcn_sched_barrier(0);
                    }
                }
                const uint32_t e = keys[lo];
                const bool goes_on = hi < total ? keys[hi] == e : behind_key == e;
                if (hi == total || !goes_on) {  // write the run's sum, or the block's part of it
                    const bool before = a == 0 && before_key == e;
                    int r0 = j0 + 4 * g;
                    asm volatile("" : "+v"(r0));  // (addresses of all ranks are made here, not kept over the loops)
#pragma unroll
                    for (int j = 0; j < RK; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const int r = r0 + 16 * j + q;
                            if (r >= rank || col >= d) continue;
                            vec_f<E> v;
#pragma unroll
                            for (int i = 0; i < E; ++i) v[i] = acc[j][i][q];
                            if (before || goes_on) ad_store<float, E>(o.part + ((chunk * 2 + (before ? 0 : 1)) * rank + r) * (int64_t)o.dpad, col, d, v);
                            else ad_put<O, E>((O *)o.out + e * o.stride + r * o.ld, col, d, v, o.accumulate);
                        }
                    clear();
                    a = hi;
                }
                lo = hi;
            }
#pragma unroll
            for (int q = 0; q < 8; ++q) raw[q] = next[q];
        }
    }
}

// ----------------------------------------------------------------- grouping --
// Positions sorted by id (stable), up to AD_GROUP_ROWS rows and AD_GROUP_ADAPTERS adapters: one launch.  A block places AD_GROUP_TILE positions.  It counts all ids itself,
// those before its own apart (16,384 ids are 128 KB from the L2 cache); of sixty-four neighbours those of two ids count at once, so that runs and few ids do not queue for
// one counter.  16,384 ids 8.2 us (two ids at random 9.0), 1024 4.2: two round trips to memory, and the instructions of sixteen waves on a CU.
#define AD_GROUP_TILE 256
#define AD_GROUP_ROWS 65536
#define AD_GROUP_ADAPTERS 4095
template <class ID>
__global__ void __launch_bounds__(1024)
k_vec_ad_group(const ID *__restrict__ ids, int n, int adapters, uint32_t *__restrict__ keys, uint32_t *__restrict__ pos, uint32_t *__restrict__ starts) {
    __shared__ uint32_t early[AD_GROUP_ADAPTERS + 1], late[AD_GROUP_ADAPTERS + 1], wide[16];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, first = blockIdx.x * AD_GROUP_TILE;
    auto norm = [&](ID id) { return id >= 0 && id < adapters ? (uint32_t)id : (uint32_t)adapters; };
    for (int i = threadIdx.x; i <= adapters; i += 1024) early[i] = late[i] = 0;
    __syncthreads();
    for (int i0 = wave * 64; i0 < n; i0 += 4 * 1024) {
        ID id[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) id[u] = ids[i0 + u * 1024 + lane < n ? i0 + u * 1024 + lane : n - 1];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const int at = i0 + u * 1024;
            if (at >= n) break;
            const uint32_t key = norm(id[u]);
            uint32_t *count = at < first ? early : late;
            uint64_t todo = __ballot(at + lane < n);
#pragma unroll
            for (int t = 0; t < 2; ++t) {  // those of the first lane's id, and of the first other
                if (!todo) continue;
                const uint32_t one = (uint32_t)__builtin_amdgcn_readlane((int)key, __builtin_ctzll(todo));
                const uint64_t same = __ballot(key == one) & todo;
                if (lane == 0) atomicAdd(&count[one], (uint32_t)__popcll(same));
                todo &= ~same;
            }
            if (todo >> lane & 1) atomicAdd(&count[key], 1u);
        }
    }
    __syncthreads();
    // where the block's first position of each id goes: the ids below it, and those before it
    uint32_t mine[4], sum = 0;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int b = threadIdx.x * 4 + u;
        mine[u] = b <= adapters ? early[b] + late[b] : 0;
        sum += mine[u];
    }
    uint32_t s = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t v = __shfl_up(s, o);
        if (lane >= o) s += v;
    }
    if (lane == 63) wide[wave] = s;
    __syncthreads();
    uint32_t at = s - sum;
    for (int v = 0; v < wave; ++v) at += wide[v];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int b = threadIdx.x * 4 + u;
        if (b <= adapters) {
            early[b] += at;
            if (starts && blockIdx.x == 0) starts[b] = at;
        }
        at += mine[u];
    }
    __syncthreads();
    const int i = first + (int)threadIdx.x;
    const bool in = threadIdx.x < AD_GROUP_TILE && i < n;
    const uint32_t key = in ? norm(ids[i]) : 0;
    uint64_t same = __ballot(in);
    for (int b = 0; adapters >> b; ++b) {
        const uint64_t v = __ballot(key >> b & 1);
        same &= key >> b & 1 ? v : ~v;
    }
#pragma unroll
    for (int v = 0; v < AD_GROUP_TILE / 64; ++v) {  // a wave after the other
        if (wave == v && in) {
            const uint32_t to = early[key] + __popcll(same & ((1ull << lane) - 1));
            keys[to] = key;
            pos[to] = (uint32_t)i;
        }
        __syncthreads();
        if (wave == v && in && (same >> lane) == 1) early[key] += __popcll(same);  // the id's last lane
        __syncthreads();
    }
}
