// vec_quantize_blocks: 8-bit values with a scale for each block of 128.
#include "vec_device.h"

struct QuantOut {
    uint8_t *q;
    void *scales;
    int64_t ld_q, ld_scales;
    int e5m2, pow2;
};

// Blocks along a row: sixteen lanes hold one, eight values each; a thread block takes sixteen neighbouring blocks of the matrix.  Bound by
// memory: 32,768 x 2048 bf16 34 us for 201 MB, part of which the caches keep from call to call.
template <class T>
__global__ void __launch_bounds__(256)
k_vec_quantize(const T *__restrict__ x, int64_t ld, int64_t n, int64_t d, int64_t nb, QuantOut o) {
    const int64_t b = vec_block() * 16 + threadIdx.x / 16;  // block of the matrix
    const int64_t row = b / nb, col = (b - row * nb) * VEC_BLOCK + (threadIdx.x & 15) * 8;
    const bool in = row < n;
    const vec_f8 f = vec_wide<T>(vec_load(x + (in ? row * ld + col : 0), in ? d - col : 0, col));
    const VecScale s = vec_scale(vec_max16(vec_top(f)), o.e5m2, o.pow2);
    if (!in) return;
    if (col < d) vec_store_bytes(o.q + row * o.ld_q + col, d - col, vec_to8(f, s, o.e5m2, o.pow2));
    if ((threadIdx.x & 15) == 0) vec_put_scale(o.scales, row * o.ld_scales + col / VEC_BLOCK, s, o.pow2);
}

// Blocks along a column, written transposed: a thread block takes 128 rows of 128 columns.  Thread t holds rows 8 (t / 16) ..+7
// of columns 8 (t % 16) ..+7, so that what it makes of a column are eight neighbouring bytes of the result; they meet in LDS
// and leave as whole rows.  Bound by memory: 32,768 x 2048 bf16 41 us for 201 MB (4.9 TB/s), F32 scales.
#define QT_LD 136  // bytes between two columns in LDS: 34 words, so that eight lanes' columns start in different banks
template <class T>
__global__ void __launch_bounds__(256)
k_vec_quantize_t(const T *__restrict__ x, int64_t ld, int64_t n, int64_t d, int64_t ncol, QuantOut o) {
    __shared__ float top[16][VEC_BLOCK];
    __shared__ __align__(16) uint8_t tile[VEC_BLOCK * QT_LD];
    const int64_t b = vec_block(), rb = b / ncol, row0 = rb * VEC_BLOCK, col0 = (b - rb * ncol) * VEC_BLOCK;
    if (row0 >= n) return;
    const int tr = threadIdx.x / 16, tc = threadIdx.x & 15;
    vec_pack<T> v[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int64_t row = row0 + tr * 8 + i, col = col0 + tc * 8;
        v[i] = vec_load(x + (row < n ? row * ld + col : 0), row < n ? d - col : 0, col);
    }
    vec_f8 m = (vec_f8)0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const vec_f8 f = vec_wide<T>(v[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float a = fabsf(f[j]);
            m[j] = fmaxf(m[j], a < INFINITY ? a : 0.0f);
        }
    }
    *(vec_f8 *)&top[tr][tc * 8] = m;
    __syncthreads();
    if (threadIdx.x < VEC_BLOCK) {
        float t = 0.0f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t = fmaxf(t, top[i][threadIdx.x]);
        top[0][threadIdx.x] = t;
        if (col0 + threadIdx.x < d) {
            const VecScale s = vec_scale(t, o.e5m2, o.pow2);
            vec_put_scale(o.scales, (col0 + threadIdx.x) * o.ld_scales + rb, s, o.pow2);
        }
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const VecScale s = vec_scale(top[0][tc * 8 + j], o.e5m2, o.pow2);
        vec_f8 f;
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = (float)v[i][j];
        *(uint64_t *)(tile + (tc * 8 + j) * QT_LD + tr * 8) = vec_to8(f, s, o.e5m2, o.pow2);
    }
    __syncthreads();
    const int64_t left = n - row0;
#pragma unroll
    for (int u = 0; u < VEC_BLOCK * 8 / 256; ++u) {
        const int e = u * 256 + threadIdx.x, c = e / 8, p = (e & 7) * 16;
        typedef int at8 __attribute__((ext_vector_type(4), aligned(8)));
        if (col0 + c < d && p < left) vec_store_bytes(o.q + (col0 + c) * o.ld_q + row0 + p, left - p, (vec_i4) * (at8 *)(tile + c * QT_LD + p));
    }
}

extern "C" int vec_quantize_blocks(const void *x, int64_t ld_x, int type, int64_t n, int64_t d, int transposed, void *q, int64_t ld_q,
                                   int q_type, void *scales, int64_t ld_scales, int scale_type, void *stream) {
    VEC_REQUIRE(n >= 0 && d >= 0 && (transposed == 0 || transposed == 1), "vec_quantize_blocks: n=%lld, d=%lld, transposed=%d", (long long)n,
                (long long)d, transposed);
    VEC_REQUIRE(vec_is_wide(type) && vec_is_8bit(q_type) && vec_is_scale(scale_type), "vec_quantize_blocks: type %d to %d with scales of type %d", type,
                q_type, scale_type);
    const int64_t along = transposed ? n : d, nb = (along + VEC_BLOCK - 1) / VEC_BLOCK;
    VEC_REQUIRE(ld_x >= d && ld_q >= along && ld_scales >= nb, "vec_quantize_blocks: a distance of rows is below their length");
    if (n == 0 || d == 0) return PQ_OK;
    VEC_REQUIRE(x && q && scales, "vec_quantize_blocks: null pointer");
    VEC_REQUIRE(vec_aligned(x, type) && vec_aligned(scales, scale_type), "vec_quantize_blocks: misaligned pointer");
    const QuantOut o = {(uint8_t *)q, scales, ld_q, ld_scales, q_type == VEC_E5M2, scale_type == VEC_E8M0};
    hipStream_t s = (hipStream_t)stream;
    const int64_t ncol = (d + VEC_BLOCK - 1) / VEC_BLOCK;
    VEC_REQUIRE(n < ((int64_t)1 << 40) && d < ((int64_t)1 << 40) && nb <= ((int64_t)1 << 40) / (transposed ? ncol : n), "vec_quantize_blocks: n=%lld, d=%lld too large",
                (long long)n, (long long)d);
    const int64_t blocks = transposed ? nb * ncol : (n * nb + 15) / 16;
    VEC_REQUIRE(blocks <= VEC_MAX_BLOCKS, "vec_quantize_blocks: n=%lld, d=%lld too large for one call", (long long)n, (long long)d);
    if (transposed)
        VEC_TYPED(type, T, hipLaunchKernelGGL((k_vec_quantize_t<T>), vec_grid(blocks, 256), dim3(256), 0, s, (const T *)x, ld_x, n, d, ncol, o));
    else
        VEC_TYPED(type, T, hipLaunchKernelGGL((k_vec_quantize<T>), vec_grid(blocks, 256), dim3(256), 0, s, (const T *)x, ld_x, n, d, nb, o));
    QADC_LAUNCH_CHECK(transposed ? "k_vec_quantize_t" : "k_vec_quantize");
    return PQ_OK;
}
