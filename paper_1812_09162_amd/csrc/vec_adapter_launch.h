// The launches of vec_adapter's and vec_adapter_grad's kernels for matrices of type T (a source each).
#pragma once
#include "vec_adapter.h"

template <class T>
struct AdLaunch {
    static void down(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &m, const VecMask &mask, float *part, int64_t part_stride, int rp,
                     int slabs, int per, hipStream_t s);
    // narrow: the result is of type T, else float32
    static void up(const AdRows &rows, const AdFactor &f, const AdMatrix &m, const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow,
                   const VecMask &mask, float *keep, int column_blocks, hipStream_t s);
    static void outer(const AdRows &rows, int len, const AdFactor &f, int rank, const void *x, int64_t ld_x, int d, const VecMask &mask, const AdOuter &o,
                      bool narrow, hipStream_t s);
};

#ifdef VEC_ADAPTER_SOURCE
static dim3 ad_grid(const AdRows &rows, int z) {
    dim3 g = vec_grid((rows.n + rows.tp - 1) / rows.tp, 256);
    g.z = (unsigned)z;
    return g;
}

template <class T>
void AdLaunch<T>::down(const AdRows &rows, const void *x, int64_t ld_x, const AdMatrix &m, const VecMask &mask, float *part, int64_t part_stride, int rp,
                       int slabs, int per, hipStream_t s) {
    const dim3 grid = ad_grid(rows, slabs);
#define GO(RK)                                                                                                             \
    do {                                                                                                                   \
        if (mask.threshold)                                                                                                \
            hipLaunchKernelGGL((k_vec_ad_down<T, RK, true>), grid, dim3(256), 0, s, rows, (const T *)x, ld_x, m, mask, part, part_stride, rp, per);  \
        else                                                                                                               \
            hipLaunchKernelGGL((k_vec_ad_down<T, RK, false>), grid, dim3(256), 0, s, rows, (const T *)x, ld_x, m, mask, part, part_stride, rp, per); \
    } while (0)
    if (m.rank <= 16) GO(1);
    else if (m.rank <= 32) GO(2);
    else if (m.rank <= 64) GO(4);
    else GO(8);
#undef GO
}

template <class T>
void AdLaunch<T>::up(const AdRows &rows, const AdFactor &f, const AdMatrix &m, const void *base, int64_t ld_base, void *y, int64_t ld_y, bool narrow,
                     const VecMask &mask, float *keep, int column_blocks, hipStream_t s) {
    const dim3 grid = ad_grid(rows, column_blocks);
    const size_t lds = (size_t)((m.rank + 31) / 32) * ((rows.tp + 15) / 16) * AdWide<T>::parts * 1024;
#define GO(Y, M, ONE)                                                                                                      \
    hipLaunchKernelGGL((k_vec_ad_up<T, Y, M, ONE>), grid, dim3(256), lds, s, rows, f, m, (const Y *)base, ld_base, (Y *)y, ld_y, mask, keep)
#define GO2(Y, M)                                                                                                          \
    do {                                                                                                                   \
        if (m.rank <= 32) GO(Y, M, true);                                                                                  \
        else GO(Y, M, false);                                                                                              \
    } while (0)
    if (mask.threshold) GO2(T, true);  // (a gradient of x, which is of its type)
    else if (narrow) GO2(T, false);
    else GO2(float, false);
#undef GO2
#undef GO
}

template <class T>
void AdLaunch<T>::outer(const AdRows &rows, int len, const AdFactor &f, int rank, const void *x, int64_t ld_x, int d, const VecMask &mask, const AdOuter &o,
                        bool narrow, hipStream_t s) {
    constexpr int cols = 64 * AD_COLS(T);
    const unsigned chunks = (unsigned)((rows.n + len - 1) / len), cb = (unsigned)((d + cols - 1) / cols);
#define GO(O, RK, M)                                                                                                       \
    hipLaunchKernelGGL((k_vec_ad_outer<T, O, RK, M>), dim3(chunks, cb, (unsigned)((rank + 16 * RK - 1) / (16 * RK))), dim3(256), 0, s, rows, len, f, \
                       rank, (const T *)x, ld_x, d, mask, o)
#define GO2(O, M)                                                                                                          \
    do {                                                                                                                   \
        if (rank <= 16) GO(O, 1, M);                                                                                       \
        else if (rank <= 32) GO(O, 2, M);                                                                                  \
        else GO(O, 4, M);                                                                                                  \
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
