// The launches of vec_adapter's and vec_adapter_grad's kernels for matrices of type T (a source each).
#pragma once
#include "vec_adapter.h"

// blocks of `up` (16 bytes a lane) and `outer` (four columns a lane) that hold d columns
static inline int ad_blocks(int d, int lane_columns) { return (d + 64 * lane_columns - 1) / (64 * lane_columns); }
static inline int ad_column_blocks(int d, int bytes) { return ad_blocks(d, d < 16 / bytes ? 1 : 16 / bytes); }
static inline int ad_outer_blocks(int d, int other) { return ad_blocks(d, d < 4 || other < 4 ? 1 : 4); }  // (one form for both gradients)

template <class T>
struct AdLaunch {
    static void down(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &m, const float *scales, float factor, const VecMask &mask, float *part,
                     int64_t part_stride, int rp, int waves, int slabs, int per, bool own, float *keep, hipStream_t s);
    // narrow: the result is of type T, else float32; joins: of the gradients of the factors in the same launch, or null; a mask or joins only with
    // a narrow result, a mask only with joins (a gradient of x); bits: the mask as `outer` kept it (of 8 columns and more), or null
    static void up(const AdRows &rows, const AdFactor &f, const AdMatrix &m, const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow,
                   const VecMask &mask, const uint32_t *bits, bool few, int column_blocks, float *keep, const AdJoins *joins, hipStream_t s);
    // both products for single rows, of at most 64 ranks
    static void one(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &a, const AdMatrix &b, const float *scales, float factor, const VecMask &mask,
                    const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow, float *keep, hipStream_t s);
    static void join(const AdRows &rows, const AdJoins &joins, hipStream_t s);
    static void outer(const AdRows &rows, int rank, const VecMask &mask, const AdSide &b, const AdSide &a, bool narrow, uint32_t *bits, hipStream_t s);
};

#ifdef VEC_ADAPTER_SOURCE
static dim3 ad_grid(const AdRows &rows, int parts, int threads) { return vec_grid((rows.n + rows.tp - 1) / rows.tp * parts, threads); }

template <class T>
void AdLaunch<T>::down(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &m, const float *scales, float factor, const VecMask &mask, float *part,
                       int64_t part_stride, int rp, int waves, int slabs, int per, bool own, float *keep, hipStream_t s) {
    const dim3 grid = ad_grid(rows, slabs, 64 * waves);
    // tiles of x and W, and at least the sums' four kilobytes a wave
    auto lds = [&](int rk) {
        const int nt = rows.tp > 32 ? 4 : (rows.tp > 16 ? 2 : 1);
        return (size_t)waves * (nt + rk) * 2048;
    };
#define GO2(RK, M)                                                                                                         \
    do {                                                                                                                   \
        void (*const k)(AdRows, const T *, int64_t, AdMatrix, const float *, float, VecMask, float *, int64_t, int, int, int, int, float *) = &k_vec_ad_down<T, RK, M>; \
        if (lds(RK) > 65536) (void)hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds(RK)); \
        hipLaunchKernelGGL(k, grid, dim3(64 * waves), lds(RK), s, rows, (const T *)x, ld_x, m, scales, factor, mask, part, part_stride, rp, slabs, per, (int)own, keep); \
    } while (0)
#define GO(RK)                           \
    do {                                 \
        if (mask.threshold) GO2(RK, true); \
        else GO2(RK, false);             \
    } while (0)
    if (m.rank <= 16) GO(1);
    else if (m.rank <= 32) GO(2);
    else if (m.rank <= 64) GO(4);
    else GO(8);
#undef GO
#undef GO2
}

static int64_t ad_join_blocks(const AdRows &rows, const AdJoins &joins) { return 2ll * joins.across * rows.adapters; }

template <class T>
void AdLaunch<T>::join(const AdRows &rows, const AdJoins &joins, hipStream_t s) {
    hipLaunchKernelGGL((k_vec_ad_join<T>), vec_grid(ad_join_blocks(rows, joins), 256), dim3(256), 0, s, rows, joins);
}

template <class T>
void AdLaunch<T>::up(const AdRows &rows, const AdFactor &f, const AdMatrix &m, const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow,
                     const VecMask &mask, const uint32_t *bits, bool few, int column_blocks, float *keep, const AdJoins *joins, hipStream_t s) {
    const int64_t tiles = (rows.n + rows.tp - 1) / rows.tp;
    const AdJoins js = joins ? *joins : AdJoins{};
    const int64_t more = joins ? ad_join_blocks(rows, js) : 0;
    if (few) {
        const int cb = ad_column_blocks(m.d, (int)sizeof(T));
        const int64_t blocks = (tiles * cb + 3) / 4;
        const dim3 grid = vec_grid(blocks + more, 256);
#define GO(Y, M, E, J)                                                                                                     \
    hipLaunchKernelGGL((k_vec_ad_up_few<T, Y, M, E, J>), grid, dim3(256), 0, s, rows, f.p, f.ld, f.stride, f.slabs, m, (const Y *)base, ld_base, (Y *)y, \
                       ld_y, mask, cb, keep, bits, blocks, js)
#define GO2(Y, M, J)                                           \
    do {                                                       \
        if (m.d < AD_COLS(T)) GO(Y, M, 1, J);                  \
        else GO(Y, M, AD_COLS(T), J);                          \
    } while (0)
        if (joins) {
            if (bits) GO(T, 2, AD_COLS(T), true);
            else if (mask.threshold) GO2(T, 1, true);
            else GO2(T, 0, true);
        } else if (narrow) GO2(T, 0, false);
        else GO2(float, 0, false);
#undef GO2
#undef GO
        return;
    }
    // Eight bytes a lane where sixteen leave few blocks: half the registers and twice the waves.  Whole calls, us, with sixteen / eight: 16,384 x 2048 of one at rank 32 (1024 blocks) 44.6 / 39.6,
    // 10,000 x 1001 fp16 of 200 at rank 12 (1252) 45 / 42; 16,384 x 4096 at rank 16 (2048) 96.5 / 97.4, of 1000 adapters (4096) 179 / 189.  With a mask each of two neighbouring lanes would make it.
    const bool half = sizeof(T) == 2 && m.rank <= 32 && !mask.threshold && m.d >= AD_COLS(T) && rows.tp >= 16 && tiles * ad_column_blocks(m.d, 2) < 2048;
    if (half) column_blocks = ad_blocks(m.d, 4);
    const int64_t blocks = tiles * column_blocks;
    const dim3 grid = vec_grid(blocks + more, 256);
    const size_t lds = (size_t)((m.rank + 31) / 32) * ((rows.tp + 15) / 16) * AdWide<T>::parts * 1024;
#define GO(Y, M, ONE, E, J)                                                                                                \
    hipLaunchKernelGGL((k_vec_ad_up<T, Y, M, ONE, E, J>), grid, dim3(256), lds, s, rows, f, m, (const Y *)base, ld_base, (Y *)y, ld_y, mask, column_blocks, keep, bits, blocks, js)
#define GO2(Y, M, J)                                                                                                       \
    do {                                                                                                                   \
        if (m.d < AD_COLS(T)) GO(Y, M, false, 1, J);                                                                       \
        else if (m.rank <= 32) GO(Y, M, true, AD_COLS(T), J);                                                              \
        else GO(Y, M, false, AD_COLS(T), J);                                                                               \
    } while (0)
    if (half) {
        if (joins) GO(T, 0, true, 4, true);
        else if (narrow) GO(T, 0, true, 4, false);
        else GO(float, 0, true, 4, false);
    } else if (joins) {
        if (bits && m.rank <= 32) GO(T, 2, true, AD_COLS(T), true);
        else if (bits) GO(T, 2, false, AD_COLS(T), true);
        else if (mask.threshold) GO2(T, 1, true);
        else GO2(T, 0, true);
    } else if (narrow) GO2(T, 0, false);
    else GO2(float, 0, false);
#undef GO2
#undef GO
}

template <class T>
void AdLaunch<T>::one(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &a, const AdMatrix &b, const float *scales, float factor, const VecMask &mask,
                      const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow, float *keep, hipStream_t s) {
    const int cb = ad_column_blocks(b.d, (int)sizeof(T));
    const dim3 grid = vec_grid(rows.n * cb, 512);
#define GO(Y, RK, E)                                                                                                       \
    hipLaunchKernelGGL((k_vec_ad_one<T, Y, RK, E>), grid, dim3(512), 0, s, rows, (const T *)x, ld_x, a, b, scales, factor, mask, (const Y *)base, ld_base, (Y *)y, ld_y, \
                       keep, cb)
#define GO2(Y)                                                 \
    do {                                                       \
        if (b.d < AD_COLS(T)) GO(Y, 4, 1);                     \
        else if (a.rank <= 16) GO(Y, 1, AD_COLS(T));           \
        else if (a.rank <= 32) GO(Y, 2, AD_COLS(T));           \
        else GO(Y, 4, AD_COLS(T));                             \
    } while (0)
    if (narrow) GO2(T);
    else GO2(float);
#undef GO2
#undef GO
}

template <class T>
void AdLaunch<T>::outer(const AdRows &rows, int rank, const VecMask &mask, const AdSide &b, const AdSide &a, bool narrow, uint32_t *bits, hipStream_t s) {
    auto blocks = [&](const AdSide &side) { return (rows.n + side.len - 1) / side.len * side.column_blocks; };
    const int64_t blocks_b = blocks(b);
    dim3 grid = vec_grid(blocks_b + blocks(a), 256);
#define GO(O, RK, M, E)                                                                                                    \
    do {                                                                                                                   \
        grid.z = (unsigned)((rank + 16 * RK - 1) / (16 * RK));                                                             \
        hipLaunchKernelGGL((k_vec_ad_outer<T, O, RK, M, E>), grid, dim3(256), 0, s, rows, rank, mask, b, a, blocks_b, bits);      \
    } while (0)
#define GO2(O, M)                                                                                                          \
    do {                                                                                                                   \
        if (a.d < 4 || b.d < 4) GO(O, 1, M, 1);                                                                                         \
        else if (rank <= 16) GO(O, 1, M, 4);                                                                               \
        else if (rank <= 32) GO(O, 2, M, 4);                                                                               \
        else GO(O, 4, M, 4);                                                                                                  \
    } while (0)
    if (mask.threshold) {
        if (narrow) GO2(T, true);
        else GO2(float, true);
    } else {
        if (narrow) GO2(T, false);
        else GO2(float, false);
    }
#undef GO2
#undef GO
}

template struct AdLaunch<VEC_ADAPTER_SOURCE>;
#endif
