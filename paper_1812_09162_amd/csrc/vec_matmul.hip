// vec_matmul_blocks: the entry point, the choice of a form, and the joining of split products.
#include "vec_matmul.h"

// c from the splits' partial products, in order
__global__ void __launch_bounds__(256) k_vec_mat_join(const MatArgs p) {
    const int64_t quads = (p.n + 3) / 4, e = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t row = e / quads, col = (e - row * quads) * 4;
    if (row >= p.m) return;
    typedef float f4u __attribute__((ext_vector_type(4), aligned(4)));
    vec_f4 sum = (vec_f4)0.0f;
    const float *q = p.part + row * p.n + col;
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s, q += p.m * p.n) {
        if (col + 4 <= p.n) {
            sum += *(const f4u *)q;
        } else {
            for (int i = 0; i < 3; ++i)
                if (col + i < p.n) sum[i] += q[i];
        }
    }
    mat_store(p, row, col, sum);
}

// The form of a product, by what each was measured to take (us; E8M0 scales unless said otherwise).
//   Tiles: 5, and for a step of 128 columns 1.15 (128 x 128, one tile on a CU; 0.92 per tile with more; F32 scales 1.45 and 1.25) or 3.1
//   (256 x 256), so that large tiles win by a sixth where they fill the CUs; k is split into shares where tiles are too few
//   for that, at the price of a launch and of partial results written and read (4.5 TB/s).
//   Up to 32 rows of a, each wave sixteen rows of b: 2.5, and b at 4.6 TB/s for one row, 3.1 up to 16, 2.1 (F32 scales 1.75) up to 32 (rows of a are read again by
//   every wave): 16 x 4096 x 4096 9.3 against 13.4 in tiles, 32 11.5 / 14.0, but 16 x 65,536 x 4096 88 / 59 and 64 x 4096 x 4096 17.4 / 16.2.
static MatPlan mat_plan(int64_t m, int64_t n, int64_t k, bool pow2, bool async) {
    MatPlan p = {};
    const int64_t steps = (k + VEC_BLOCK - 1) / VEC_BLOCK;
    double best = 1e300;
    // (the large tile has no registers to spare for a detour through them, nor for sums of a block)
    for (int tile = MAT_128; tile <= (async && pow2 ? MAT_256 : MAT_128); ++tile) {
        const int side = tile == MAT_256 ? 256 : 128;
        const int64_t tm = (m + side - 1) / side, tn = (n + side - 1) / side;
        if (tm * tn * (tile == MAT_256 ? 512 : 256) > 0xffffffffLL) continue;  // (threads of a launch)
        for (int64_t s = 1; s <= 32 && (s == 1 || (s * 4 <= steps && tm * tn * s <= 512)); ++s) {
            const int64_t per = (steps + s - 1) / s, rounds = (tm * tn * s + 255) / 256;
            const bool one = rounds == 1;
            const double step = tile == MAT_256 ? 3.1 : (pow2 ? (one ? 1.15 : 0.92) : (one ? 1.45 : 1.25));
            const double us = 5.0 + (double)(rounds * per) * step + (s > 1 ? 4.0 + (double)s * (double)m * (double)n * 8 / 4.5e6 : 0.0);
            if (us >= best) continue;
            best = us;
            p.tile = tile;
            p.tm = (int)tm;
            p.tn = (int)tn;
            p.per = (int)per;
            p.splits = per > 0 ? (int)((steps + per - 1) / per) : 1;
        }
    }
    if (m <= 32 && 2.5 + (double)n * (double)k / (m == 1 ? 4.6e6 : (m <= 16 ? 3.1e6 : (pow2 ? 2.1e6 : 1.75e6))) < best) {
        p.few = m <= 16 ? 1 : 2;
        p.splits = 1;
        p.kshare = 1;
        while (p.kshare < MAT_FEW_WAVES && p.kshare * 2 <= steps && (n + 15) / 16 * p.kshare < 4096) p.kshare *= 2;
    }
    if (p.splits > 1) p.workspace = vec_up256((size_t)p.splits * (size_t)m * (size_t)n * 4);
    return p;
}

static bool mat_sizes(int64_t m, int64_t n, int64_t k) {
    return m >= 0 && n >= 0 && k >= 0 && m <= 0x7fffffffLL && n <= 0x7fffffffLL && k <= 0x7fffffffLL;
}
extern "C" size_t vec_matmul_blocks_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    if (!mat_sizes(m, n, k) || m == 0 || n == 0) return 0;
    size_t most = 0;  // of all types and alignments
    for (int form = 0; form < 4; ++form) {
        const size_t need = mat_plan(m, n, k, form & 1, form & 2).workspace;
        most = need > most ? need : most;
    }
    return most;
}

extern "C" int vec_matmul_blocks(const void *a, int64_t ld_a, int a_type, const void *a_scales, int64_t ld_a_scales, const void *b,
                                 int64_t ld_b, int b_type, const void *b_scales, int64_t ld_b_scales, int scale_type, int64_t m,
                                 int64_t n, int64_t k, void *c, int64_t ld_c, int c_type, void *workspace, size_t workspace_bytes,
                                 void *stream) {
    VEC_REQUIRE(mat_sizes(m, n, k), "vec_matmul_blocks: m=%lld, n=%lld, k=%lld", (long long)m, (long long)n, (long long)k);
    VEC_REQUIRE(vec_is_8bit(a_type) && vec_is_8bit(b_type) && vec_is_scale(scale_type) && vec_is_wide(c_type),
                "vec_matmul_blocks: types %d and %d, scales %d, result %d", a_type, b_type, scale_type, c_type);
    const int64_t steps = (k + VEC_BLOCK - 1) / VEC_BLOCK;
    VEC_REQUIRE(ld_a >= k && ld_b >= k && ld_a_scales >= steps && ld_b_scales >= steps && ld_c >= n, "vec_matmul_blocks: a distance of rows is below their length");
    if (m == 0 || n == 0) return PQ_OK;
    VEC_REQUIRE(c && (k == 0 || (a && b && a_scales && b_scales)), "vec_matmul_blocks: null pointer");
    VEC_REQUIRE(vec_aligned(c, c_type) && vec_aligned(a_scales, scale_type) && vec_aligned(b_scales, scale_type), "vec_matmul_blocks: misaligned pointer");
    const bool pow2 = scale_type == VEC_E8M0;
    const bool async = (((uintptr_t)a | (uintptr_t)b | (uintptr_t)ld_a | (uintptr_t)ld_b) & 15u) == 0 && ld_a < (1 << 23) && ld_b < (1 << 23) &&
                       ld_a_scales < (1 << 21) && ld_b_scales < (1 << 21);
    const MatPlan plan = mat_plan(m, n, k, pow2, async);
    if (plan.workspace > 0) {
        const size_t need = vec_matmul_blocks_workspace_bytes(m, n, k);
        VEC_REQUIRE(workspace && ((uintptr_t)workspace & 255u) == 0, "vec_matmul_blocks: workspace null or not 256-byte aligned");
        if (workspace_bytes < need) {
            qadc_set_error("vec_matmul_blocks: workspace of %zu bytes, %zu needed", workspace_bytes, need);
            return PQ_ENOMEM;
        }
    }
    VEC_REQUIRE(plan.few > 0 || plan.tm > 0, "vec_matmul_blocks: m=%lld, n=%lld too large for one call",
                (long long)m, (long long)n);
    const MatArgs p = {(const uint8_t *)a, (const uint8_t *)b, a_scales, b_scales, ld_a, ld_b, ld_a_scales, ld_b_scales, m, n, k,
                       c, ld_c, c_type, (float *)workspace, plan.splits, plan.per, plan.tm, plan.tn};
    hipStream_t s = (hipStream_t)stream;
    const bool a5 = a_type == VEC_E5M2, b5 = b_type == VEC_E5M2;
    const int rc = a5 ? (b5 ? qadc_vec_mat_launch<1, 1>(p, plan, pow2, async, s) : qadc_vec_mat_launch<1, 0>(p, plan, pow2, async, s))
                      : (b5 ? qadc_vec_mat_launch<0, 1>(p, plan, pow2, async, s) : qadc_vec_mat_launch<0, 0>(p, plan, pow2, async, s));
    if (rc != PQ_OK || plan.splits == 1) return rc;
    const int64_t blocks = (m * ((n + 3) / 4) + 255) / 256;
    VEC_REQUIRE(blocks <= 0x7fffffffLL, "vec_matmul_blocks: m=%lld, n=%lld too large for one call", (long long)m, (long long)n);
    hipLaunchKernelGGL(k_vec_mat_join, dim3((unsigned)blocks), dim3(256), 0, s, p);
    QADC_LAUNCH_CHECK("k_vec_mat_join");
    return PQ_OK;
}
