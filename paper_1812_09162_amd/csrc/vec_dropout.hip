// vec_dropout: elements dropped by a counter-based generator, with the residual's addition.
//
// y = residual + (kept ? factor x : 0); the mask is made where it is used and never stored, so the gradient is the same call on dy.
// A block takes 1024 pieces of eight elements (whole rows, or part of one), four of them in flight per thread; bound by memory:
// 16,384 x 2048 bf16 with a residual 35 us (201 MB, 5.7 TB/s, part of it from the caches); 10,000 x 1001 fp16 11, 1024 x 256 float32 4.6 (one round trip and a launch).
#include "vec_random.h"

template <class T, bool RESIDUAL>
__global__ void __launch_bounds__(256)
k_vec_dropout(const T *x, int64_t ld_x, const T *residual, int64_t ld_r, int64_t n, int64_t d, VecMask mask, float factor,
              T *y, int64_t ld_y, int rpb, int pieces, int parts, uint32_t magic) {
    // rows of up to 1024 pieces: rpb of them; of more: part blockIdx % parts of one
    const int64_t block = vec_block(), row0 = parts > 1 ? block / parts : block * rpb;
    const int64_t piece0 = parts > 1 ? (block - row0 * parts) * 1024 : 0;
    if (row0 >= n) return;
    const int nrow = (int)(n - row0 < rpb ? n - row0 : rpb);
    const int total = parts > 1 ? 1024 : nrow * pieces;
    VecKey key = {0, 0, 0};
    if (mask.threshold) key = vec_key(mask);
    vec_pack<T> v[4], w[4];
    int r[4];
    int64_t col[4], left[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        const int e = threadIdx.x + u * 256;
        r[u] = parts > 1 || rpb == 1 ? 0 : (pieces == 1 ? e : (int)__umulhi((uint32_t)e, magic));  // e / pieces
        col[u] = (piece0 + e - r[u] * pieces) * 8;
        left[u] = e < total ? d - col[u] : 0;
        const bool in = left[u] > 0;
        v[u] = vec_load(x + (in ? (row0 + r[u]) * ld_x + col[u] : 0), in ? left[u] : 0, col[u]);
        if (RESIDUAL) w[u] = vec_load(residual + (in ? (row0 + r[u]) * ld_r + col[u] : 0), in ? left[u] : 0, col[u]);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        if (left[u] <= 0) continue;
        vec_pack<T> a = v[u];
        if (mask.threshold) a = vec_drop<T>(a, vec_kept(vec_random(key, mask.layer, (uint32_t)(row0 + r[u]), (uint32_t)(col[u] >> 3)), mask.threshold));
        vec_f8 f = vec_wide<T>(a);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= factor;
        if (RESIDUAL) f += vec_wide<T>(w[u]);
        vec_store(y + (row0 + r[u]) * ld_y + col[u], left[u], f);
    }
}

extern "C" int vec_dropout(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, int type, int64_t n, int64_t d, double p,
                           const uint64_t *state, uint32_t layer, void *y, int64_t ld_y, void *stream) {
    uint32_t threshold;
    float factor;
    VEC_REQUIRE(n >= 0 && n <= 0xffffffffLL && d >= 1 && d <= VEC_MAX_ROW_DIM, "vec_dropout: n=%lld, d=%lld", (long long)n, (long long)d);
    VEC_REQUIRE(vec_rate(p, &threshold, &factor), "vec_dropout: p=%g is not in 0..65535/65536", p);
    VEC_REQUIRE(vec_is_wide(type), "vec_dropout: type %d is not F32, BF16 or F16", type);
    VEC_REQUIRE(ld_x >= d && (!residual || ld_residual >= d) && ld_y >= d, "vec_dropout: a distance of rows is below their length %lld", (long long)d);
    VEC_REQUIRE(threshold == 0 || (state && ((uintptr_t)state & 7u) == 0), "vec_dropout: state null or misaligned");
    if (n == 0) return PQ_OK;
    VEC_REQUIRE(x && y, "vec_dropout: null pointer");
    // (a row of y would lie over others that are still to be read)
    VEC_REQUIRE(n <= 1 || ((x != y || ld_x == ld_y) && (residual != y || ld_residual == ld_y)), "vec_dropout: y in place of x or residual with another distance of rows");
    VEC_REQUIRE(vec_aligned(x, type) && vec_aligned(residual, type) && vec_aligned(y, type), "vec_dropout: misaligned pointer");
    const int pieces = (int)((d + 7) / 8), rpb = pieces >= 1024 ? 1 : 1024 / pieces, parts = (pieces + 1023) / 1024;
    const int64_t blocks = parts > 1 ? n * parts : (n + rpb - 1) / rpb;
    VEC_REQUIRE(blocks <= VEC_MAX_BLOCKS, "vec_dropout: n=%lld, d=%lld too large for one call", (long long)n, (long long)d);
    const uint32_t magic = (uint32_t)((((uint64_t)1 << 32) + pieces - 1) / pieces);  // e / pieces for e < 1024, pieces > 1: exact as 1024 pieces < 2^32
    const VecMask mask = {state, layer, threshold};
    hipStream_t s = (hipStream_t)stream;
#define GO(T, R)                                                                                                           \
    hipLaunchKernelGGL((k_vec_dropout<T, R>), vec_grid(blocks, 256), dim3(256), 0, s, (const T *)x, ld_x, (const T *)residual, ld_residual, \
                       n, d, mask, factor, (T *)y, ld_y, rpb, pieces, parts, magic)
    VEC_TYPED(type, T, if (residual) GO(T, true); else GO(T, false));
#undef GO
    QADC_LAUNCH_CHECK("k_vec_dropout");
    return PQ_OK;
}
