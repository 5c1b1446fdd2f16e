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

static MatPlan mat_plan(int64_t m, int64_t n, int64_t k) {
    MatPlan p = {};
    const int64_t steps = (k + VEC_BLOCK - 1) / VEC_BLOCK;
    p.splits = 1;
    p.per = (int)steps;
    if (m <= 64) {
        p.few = m <= 16 ? 1 : (m <= 32 ? 2 : 4);
        const int64_t tiles = (n + 15) / 16;
        p.kshare = 1;
        while (p.kshare < MAT_FEW_WAVES && p.kshare * 2 <= steps && tiles * p.kshare < 4096) p.kshare *= 2;
        return p;
    }
    const int64_t big = ((m + 255) / 256) * ((n + 255) / 256);
    p.big = big >= 192;
    const int side = p.big ? 256 : 128;
    const int64_t tm = (m + side - 1) / side, tn = (n + side - 1) / side, tiles = tm * tn;
    p.tm = (int)tm;
    p.tn = (int)tn;
    if (!p.big && tiles < 384 && steps >= 8) {
        int64_t s = (512 + tiles - 1) / tiles;
        if (s > steps / 4) s = steps / 4;
        p.per = (int)((steps + s - 1) / s);
        p.splits = (int)((steps + p.per - 1) / p.per);
    }
    if (p.splits > 1) p.workspace = vec_up256((size_t)p.splits * (size_t)m * (size_t)n * 4);
    return p;
}

static bool mat_sizes(int64_t m, int64_t n, int64_t k) {
    return m >= 0 && n >= 0 && k >= 0 && m <= 0x7fffffffLL && n <= 0x7fffffffLL && k <= 0x7fffffffLL;
}
extern "C" size_t vec_matmul_blocks_workspace_bytes(int64_t m, int64_t n, int64_t k) {
    return !mat_sizes(m, n, k) || m == 0 || n == 0 ? 0 : mat_plan(m, n, k).workspace;
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
    MatPlan plan = mat_plan(m, n, k);
    if (plan.workspace > 0) {
        VEC_REQUIRE(workspace && ((uintptr_t)workspace & 255u) == 0, "vec_matmul_blocks: workspace null or not 256-byte aligned");
        if (workspace_bytes < plan.workspace) {
            qadc_set_error("vec_matmul_blocks: workspace of %zu bytes, %zu needed", workspace_bytes, plan.workspace);
            return PQ_ENOMEM;
        }
    }
    const bool async = (((uintptr_t)a | (uintptr_t)b | (uintptr_t)ld_a | (uintptr_t)ld_b) & 15u) == 0 && ld_a < (1 << 23) && ld_b < (1 << 23);
    if (plan.big && !(async && scale_type == VEC_E8M0)) {  // the large tile has no registers to spare for a detour, nor for sums of a block
        plan.big = false;
        plan.tm = (int)((m + 127) / 128);
        plan.tn = (int)((n + 127) / 128);
    }
    VEC_REQUIRE(plan.few ? (n + 15) / 16 <= 0x7fffffffLL : (int64_t)plan.tm * plan.tn <= 0x7fffffffLL / plan.splits, "vec_matmul_blocks: m=%lld, n=%lld too large for one call",
                (long long)m, (long long)n);
    const MatArgs p = {(const uint8_t *)a, (const uint8_t *)b, a_scales, b_scales, ld_a, ld_b, ld_a_scales, ld_b_scales, m, n, k,
                       c, ld_c, c_type, (float *)workspace, plan.splits, plan.per, plan.tm, plan.tn};
    hipStream_t s = (hipStream_t)stream;
    const bool pow2 = scale_type == VEC_E8M0, a5 = a_type == VEC_E5M2, b5 = b_type == VEC_E5M2;
    const int rc = a5 ? (b5 ? qadc_vec_mat_launch<1, 1>(p, plan, pow2, async, s) : qadc_vec_mat_launch<1, 0>(p, plan, pow2, async, s))
                      : (b5 ? qadc_vec_mat_launch<0, 1>(p, plan, pow2, async, s) : qadc_vec_mat_launch<0, 0>(p, plan, pow2, async, s));
    if (rc != PQ_OK || plan.splits == 1) return rc;
    const int64_t blocks = (m * ((n + 3) / 4) + 255) / 256;
    VEC_REQUIRE(blocks <= 0x7fffffffLL, "vec_matmul_blocks: m=%lld, n=%lld too large for one call", (long long)m, (long long)n);
    hipLaunchKernelGGL(k_vec_mat_join, dim3((unsigned)blocks), dim3(256), 0, s, p);
    QADC_LAUNCH_CHECK("k_vec_mat_join");
    return PQ_OK;
}
