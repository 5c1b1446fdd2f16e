// vec_norm and vec_norm_grad: root-mean-square norm of rows, with the residual's addition and an 8-bit result.
//
// LANES lanes hold a row, eight elements in each of CH pieces: piece c of lane l starts at column 8 (c LANES + l), so that
// sixteen neighbouring lanes hold the 128 values of a block's scale.  A wave holds 64 / LANES rows (LANES <= 64, four waves a
// block), or a block of 256 or 512 threads one row.  Everything is read once and stays in registers; bound by memory.  16,384 x 2048 bf16 with residual and
// 8-bit result: 42 us for 235 MB (5.6 TB/s; 48 a call among calls, the rate of a large copy); one row 5 us, all latency.  (Outputs that
// may be inputs in place are not __restrict__: a row is read whole before it is written.)
#include "vec_device.h"

#define NORM_BLOCKS 2048

// Sum over a row's lanes; over the block, through LDS (two calls in a row need two buffers), where it has more than a wave.
template <int LANES>
__device__ __forceinline__ float norm_sum(float v, float *buf) {
    if constexpr (LANES <= 64) {
        return vec_sum<LANES>(v);
    } else {
        v = vec_sum<64>(v);
        if ((threadIdx.x & 63) == 0) buf[threadIdx.x >> 6] = v;
        __syncthreads();
        v = (buf[0] + buf[1]) + (buf[2] + buf[3]);
        if constexpr (LANES == 512) v += (buf[4] + buf[5]) + (buf[6] + buf[7]);
        return v;
    }
}
template <int LANES>
constexpr int norm_threads = LANES > 256 ? LANES : 256;

struct NormOut {
    void *h, *y;
    uint8_t *q;
    void *scales;
    int64_t ld_h, ld_y, ld_q, ld_scales;
    int e5m2, pow2;
};

template <class T, class W, int LANES, int CH>
__global__ void __launch_bounds__(norm_threads<LANES>)
k_vec_norm(const T *x, int64_t ld_x, const T *residual, int64_t ld_r, const W *__restrict__ weight,
           int64_t n, int d, float eps, NormOut o) {
    __shared__ float buf[2][8];
    constexpr int ROWS = norm_threads<LANES> / LANES;
    const int lane = threadIdx.x % LANES;
    vec_pack<W> w[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) w[c] = vec_load(weight + 8 * (c * LANES + lane), d - 8 * (c * LANES + lane), 8 * (c * LANES + lane));
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < n; row0 += (int64_t)gridDim.x * ROWS, turn ^= 1) {
        const int64_t row = row0 + threadIdx.x / LANES;
        const bool in = row < n;
        vec_f8 h[CH];
        {
            vec_pack<T> a[CH], b[CH];
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                const int col = 8 * (c * LANES + lane);
                a[c] = vec_load(x + (in ? row * ld_x + col : 0), in ? d - col : 0, col);
                if (residual) b[c] = vec_load(residual + (in ? row * ld_r + col : 0), in ? d - col : 0, col);
            }
#pragma unroll
            for (int c = 0; c < CH; ++c) {
                h[c] = vec_wide<T>(a[c]);
                if (residual) {
                    // (the norm is of the rounded sum: it is what the residual stream carries on, and what the gradient sees)
                    h[c] = vec_wide<T>(__builtin_convertvector(h[c] + vec_wide<T>(b[c]), vec_pack<T>));
                    const int col = 8 * (c * LANES + lane);
                    if (in) vec_store((T *)o.h + row * o.ld_h + col, d - col, h[c]);
                }
            }
        }
        float sum = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = __fmaf_rn(h[c][i], h[c][i], sum);
        sum = norm_sum<LANES>(sum, buf[turn]);
        const float r = rsqrtf(sum / (float)d + eps);
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = 8 * (c * LANES + lane);
            const vec_f8 g = vec_wide<W>(w[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) h[c][i] = h[c][i] * r * g[i];
            if (o.y && in) vec_store((T *)o.y + row * o.ld_y + col, d - col, h[c]);
            if (o.q) {
                const VecScale s = vec_scale(vec_max16(vec_top(h[c])), o.e5m2, o.pow2);
                if (in && col < d) {
                    vec_store_bytes(o.q + row * o.ld_q + col, d - col, vec_to8(h[c], s, o.e5m2, o.pow2));
                    if ((lane & 15) == 0) vec_put_scale(o.scales, row * o.ld_scales + (col >> 7), s, o.pow2);
                }
            }
        }
    }
}

// The smallest form whose lanes and pieces hold a row.
#define NORM_FORMS(d, GO)                \
    do {                                 \
        if ((d) <= 128) GO(16, 1);       \
        else if ((d) <= 256) GO(32, 1);  \
        else if ((d) <= 512) GO(64, 1);  \
        else if ((d) <= 1024) GO(64, 2); \
        else if ((d) <= 2048) GO(64, 4); \
        else if ((d) <= 4096) GO(256, 2); \
        else if ((d) <= 8192) GO(256, 4); \
        else GO(512, 4);                 \
    } while (0)

extern "C" int vec_norm(const void *x, int64_t ld_x, const void *residual, int64_t ld_residual, int type, const void *weight,
                        int weight_type, int64_t n, int d, float eps, void *h, int64_t ld_h, void *y, int64_t ld_y, void *q,
                        int64_t ld_q, int q_type, void *scales, int64_t ld_scales, int scale_type, void *stream) {
    VEC_REQUIRE(n >= 0 && d >= 1 && d <= VEC_MAX_NORM_DIM && eps >= 0.0f, "vec_norm: n=%lld, d=%d (1..%d), eps=%g", (long long)n, d, VEC_MAX_NORM_DIM, eps);
    VEC_REQUIRE(vec_is_wide(type) && (weight_type == type || weight_type == VEC_F32), "vec_norm: types %d and %d (weight)", type, weight_type);
    VEC_REQUIRE((residual != nullptr) == (h != nullptr), "vec_norm: residual and h go together");
    VEC_REQUIRE((q != nullptr) == (scales != nullptr), "vec_norm: q and scales go together");
    VEC_REQUIRE(y || q || n == 0, "vec_norm: neither y nor q wanted");
    VEC_REQUIRE(!q || (vec_is_8bit(q_type) && vec_is_scale(scale_type)), "vec_norm: q of type %d with scales of type %d", q_type, scale_type);
    VEC_REQUIRE(ld_x >= d && (!residual || (ld_residual >= d && ld_h >= d)) && (!y || ld_y >= d) && (!q || (ld_q >= d && ld_scales >= (d + 127) / 128)),
                "vec_norm: a distance of rows is below their length %d", d);
    if (n == 0) return PQ_OK;
    VEC_REQUIRE(x && weight, "vec_norm: null pointer");
    VEC_REQUIRE(vec_aligned(x, type) && vec_aligned(residual, type) && vec_aligned(h, type) && vec_aligned(y, type) && vec_aligned(weight, weight_type) &&
                    (!q || vec_aligned(scales, scale_type)), "vec_norm: misaligned pointer");
    const NormOut o = {h, y, (uint8_t *)q, scales, ld_h, ld_y, ld_q, ld_scales, q_type == VEC_E5M2, scale_type == VEC_E8M0};
    hipStream_t s = (hipStream_t)stream;
#define GO(LANES, CH)                                                                                                     \
    do {                                                                                                                  \
        constexpr int rows = norm_threads<LANES> / LANES;                                                                 \
        const int64_t need = (n + rows - 1) / rows;                                                                       \
        const unsigned blocks = (unsigned)(need < NORM_BLOCKS ? need : NORM_BLOCKS);                                      \
        if (weight_type == type)                                                                                          \
            hipLaunchKernelGGL((k_vec_norm<T, T, LANES, CH>), dim3(blocks), dim3(norm_threads<LANES>), 0, s, (const T *)x, ld_x,          \
                               (const T *)residual, ld_residual, (const T *)weight, n, d, eps, o);                        \
        else                                                                                                              \
            hipLaunchKernelGGL((k_vec_norm<T, float, LANES, CH>), dim3(blocks), dim3(norm_threads<LANES>), 0, s, (const T *)x, ld_x,      \
                               (const T *)residual, ld_residual, (const float *)weight, n, d, eps, o);                    \
    } while (0)
    VEC_TYPED(type, T, NORM_FORMS(d, GO));
#undef GO
    QADC_LAUNCH_CHECK("k_vec_norm");
    return PQ_OK;
}

// ----------------------------------------------------------------- gradient --
// The same layout.  Every lane sums its columns of dweight over the rows that it meets (a fixed set), the block joins its rows
// through LDS and writes a row of partial sums, which k_vec_norm_join adds up in order.  Bound by memory: 16,384 x 2048 bf16 44 us for 268 MB (6.1 TB/s), the join 5,
// 55 a call among calls; 10,000 x 1001 fp16 15 and 5 us.
//
// More blocks hide the latency of a row, but each writes a row of partial sums.  us with 256 / 512 / 1024 blocks: 32,768 x 128 bf16
// 12.5 / 12.3 / 12.5; 32,768 x 257 66.8 / 39.4 / 28.2; 10,000 x 1001 fp16 31.1 / 22.9 / 21.9; 16,384 x 2048 bf16 56.2 / 51.4 / 55.3; 8192 x 4096
// 63.6 / 51.9 / 55.3; 1000 x 16,384 41.7 / 51.5 / 70.4.  What one block does in two rounds (four of narrow rows)
// it does alone, writing dweight itself, without the join: 8 x 2048 13.6 -> 11.5 a call, which waits for the host's launches, and 6.3 -> 5.7 in a graph; 16 x 2048
// in four rounds 8.5 there, so not more.
static int norm_grad_blocks(int64_t n, int d) {
    const int rows = d <= 128 ? 16 : (d <= 256 ? 8 : (d <= 2048 ? 4 : 1));  // a block holds at once
    const int64_t need = (n + rows - 1) / rows, most = rows == 4 && d <= 1024 ? 1024 : (rows == 1 && n < 2048 ? 256 : 512);
    return (int)(need <= (d <= 256 ? 4 : 2) ? 1 : (need < most ? need : most));
}
extern "C" size_t vec_norm_grad_workspace_bytes(int64_t n, int d) {
    return n <= 0 || d <= 0 ? 0 : vec_up256((size_t)norm_grad_blocks(n, d) * ((d + 7) & ~7) * 4);
}

template <class T, class W, int LANES, int CH>
__global__ void __launch_bounds__(norm_threads<LANES>)
k_vec_norm_grad(const T *dy, int64_t ld_dy, const T *hs, int64_t ld_h, const T *dh, int64_t ld_dh,
                const W *__restrict__ weight, int64_t n, int d, float eps, T *dx, int64_t ld_dx,
                float *__restrict__ part, int dpad) {  // part: a row of dpad sums a block
    __shared__ float buf[4][8];
    constexpr int ROWS = norm_threads<LANES> / LANES;
    const int lane = threadIdx.x % LANES;
    vec_pack<W> w[CH];
    vec_f8 dw[CH];
#pragma unroll
    for (int c = 0; c < CH; ++c) {
        w[c] = vec_load(weight + 8 * (c * LANES + lane), d - 8 * (c * LANES + lane), 8 * (c * LANES + lane));
        dw[c] = (vec_f8)0.0f;
    }
    int turn = 0;
    for (int64_t row0 = (int64_t)blockIdx.x * ROWS; row0 < n; row0 += (int64_t)gridDim.x * ROWS, turn ^= 2) {
        const int64_t row = row0 + threadIdx.x / LANES;
        const bool in = row < n;
        vec_pack<T> a[CH], b[CH], e[CH];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = 8 * (c * LANES + lane);
            const int64_t left = in ? d - col : 0;
            a[c] = vec_load(dy + (in ? row * ld_dy + col : 0), left, col);
            b[c] = vec_load(hs + (in ? row * ld_h + col : 0), left, col);
            if (dh) e[c] = vec_load(dh + (in ? row * ld_dh + col : 0), left, col);
        }
        float sq = 0.0f, dot = 0.0f;
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const vec_f8 g = vec_wide<W>(w[c]), h = vec_wide<T>(b[c]), y = vec_wide<T>(a[c]);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sq = __fmaf_rn(h[i], h[i], sq);
                dot = __fmaf_rn(y[i] * g[i], h[i], dot);
            }
        }
        sq = norm_sum<LANES>(sq, buf[turn]);
        dot = norm_sum<LANES>(dot, buf[turn + 1]);
        const float r = in ? rsqrtf(sq / (float)d + eps) : 0.0f;  // (a row behind the last would bring 0 / 0 into dweight where eps is 0)
        const float k = r * (r * (dot / (float)d));  // (h r and r h are near one, so that nothing here leaves float32's range early: r^3 did, for h of 1e13 and of 1e-13)
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            const int col = 8 * (c * LANES + lane);
            const vec_f8 g = vec_wide<W>(w[c]), h = vec_wide<T>(b[c]), y = vec_wide<T>(a[c]);
            vec_f8 f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hr = h[i] * r;
                f[i] = __fmaf_rn(-hr, k, r * (y[i] * g[i]));
                dw[c][i] = __fmaf_rn(y[i], hr, dw[c][i]);
            }
            if (dh) f += vec_wide<T>(e[c]);
            if (in) vec_store(dx + row * ld_dx + col, d - col, f);
        }
    }
    float *mine = part + (int64_t)blockIdx.x * dpad;
    if constexpr (LANES >= 256) {
#pragma unroll
        for (int c = 0; c < CH; ++c)
            vec_store(mine + 8 * (c * LANES + lane), dpad - 8 * (c * LANES + lane), dw[c]);
    } else {
        __shared__ vec_f8 all[ROWS][LANES];
#pragma unroll
        for (int c = 0; c < CH; ++c) {
            __syncthreads();
            all[threadIdx.x / LANES][lane] = dw[c];
            __syncthreads();
            if (threadIdx.x < LANES) {
                vec_f8 sum = all[0][lane];
                for (int r = 1; r < ROWS; ++r) sum += all[r][lane];
                vec_store(mine + 8 * (c * LANES + lane), dpad - 8 * (c * LANES + lane), sum);
            }
        }
    }
}

// dweight from the blocks' partial sums: sixteen columns a block, sixteen threads each
__global__ void __launch_bounds__(256)
k_vec_norm_join(const float *__restrict__ part, int dpad, int blocks, int d, float *__restrict__ dweight) {
    __shared__ float s[16][17];
    const int col = blockIdx.x * 16 + (threadIdx.x & 15), g = threadIdx.x >> 4;
    float sum = 0.0f;
    if (col < d)
#pragma unroll 8
        for (int b = g; b < blocks; b += 16) sum += part[(int64_t)b * dpad + col];
    s[g][threadIdx.x & 15] = sum;
    __syncthreads();
    if (g == 0 && col < d) {
        for (int i = 1; i < 16; ++i) sum += s[i][threadIdx.x & 15];
        dweight[col] = sum;
    }
}

extern "C" int vec_norm_grad(const void *dy, int64_t ld_dy, const void *h, int64_t ld_h, const void *dh, int64_t ld_dh, int type,
                             const void *weight, int weight_type, int64_t n, int d, float eps, void *dx, int64_t ld_dx, float *dweight,
                             void *workspace, size_t workspace_bytes, void *stream) {
    VEC_REQUIRE(n >= 0 && d >= 1 && d <= VEC_MAX_NORM_DIM && eps >= 0.0f, "vec_norm_grad: n=%lld, d=%d (1..%d), eps=%g", (long long)n, d, VEC_MAX_NORM_DIM, eps);
    VEC_REQUIRE(vec_is_wide(type) && (weight_type == type || weight_type == VEC_F32), "vec_norm_grad: types %d and %d (weight)", type, weight_type);
    VEC_REQUIRE(ld_dy >= d && ld_h >= d && (!dh || ld_dh >= d) && ld_dx >= d, "vec_norm_grad: a distance of rows is below their length %d", d);
    VEC_REQUIRE(dweight && (n == 0 || (dy && h && weight && dx)), "vec_norm_grad: null pointer");
    VEC_REQUIRE(vec_aligned(dy, type) && vec_aligned(h, type) && vec_aligned(dh, type) && vec_aligned(dx, type) && vec_aligned(weight, weight_type) &&
                    vec_aligned(dweight, VEC_F32), "vec_norm_grad: misaligned pointer");
    hipStream_t s = (hipStream_t)stream;
    int dpad = (d + 7) & ~7;
    unsigned blocks = 0;
    float *part = (float *)workspace;
    if (n > 0) {
        const size_t need = vec_norm_grad_workspace_bytes(n, d);
        VEC_REQUIRE(workspace && ((uintptr_t)workspace & 255u) == 0, "vec_norm_grad: workspace null or not 256-byte aligned");
        if (workspace_bytes < need) {
            qadc_set_error("vec_norm_grad: workspace of %zu bytes, %zu needed", workspace_bytes, need);
            return PQ_ENOMEM;
        }
        blocks = (unsigned)norm_grad_blocks(n, d);
        if (blocks == 1) part = dweight, dpad = d;
#define GO(LANES, CH)                                                                                                     \
    do {                                                                                                                  \
        if (weight_type == type)                                                                                          \
            hipLaunchKernelGGL((k_vec_norm_grad<T, T, LANES, CH>), dim3(blocks), dim3(norm_threads<LANES>), 0, s, (const T *)dy, ld_dy,   \
                               (const T *)h, ld_h, (const T *)dh, ld_dh, (const T *)weight, n, d, eps, (T *)dx, ld_dx,    \
                               part, dpad);                                                                               \
        else                                                                                                              \
            hipLaunchKernelGGL((k_vec_norm_grad<T, float, LANES, CH>), dim3(blocks), dim3(norm_threads<LANES>), 0, s, (const T *)dy,      \
                               ld_dy, (const T *)h, ld_h, (const T *)dh, ld_dh, (const float *)weight, n, d, eps, (T *)dx, \
                               ld_dx, part, dpad);                                                                        \
    } while (0)
        VEC_TYPED(type, T, NORM_FORMS(d, GO));
#undef GO
    }
    if (blocks != 1)
        hipLaunchKernelGGL(k_vec_norm_join, dim3((unsigned)((d + 15) / 16)), dim3(256), 0, s, part, dpad, (int)blocks, d, dweight);
    QADC_LAUNCH_CHECK("vec_norm_grad's kernels");
    return PQ_OK;
}
