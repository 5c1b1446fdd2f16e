// One translation unit per pair of factor types: MAT_FA and MAT_FB are 1 for E5M2.
#include "vec_matmul.h"

template <bool P2, bool ASYNC, int WM, int WN, int MI, int NI>
static int go_tiles(const MatArgs &p, hipStream_t s) {
    constexpr int rows = WM * MI * 16 + WN * NI * 16, lds = 2 * rows * 132;
    void (*const k)(MatArgs) = &k_vec_mat<MAT_FA, MAT_FB, P2, ASYNC, WM, WN, MI, NI>;
    QADC_HIP_TRY(hipFuncSetAttribute((const void *)k, hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    hipLaunchKernelGGL(k, dim3((unsigned)p.tm * (unsigned)p.tn * (unsigned)p.splits), dim3(64 * WM * WN), lds, s, p);
    QADC_LAUNCH_CHECK("k_vec_mat");
    return PQ_OK;
}
template <bool P2, int MF>
static int go_few(const MatArgs &p, const MatPlan &plan, hipStream_t s) {
    const int64_t tiles = (p.n + 15) / 16, per = MAT_FEW_WAVES / plan.kshare;
    hipLaunchKernelGGL((k_vec_mat_few<MAT_FA, MAT_FB, P2, MF>), vec_grid((tiles + per - 1) / per, 64 * MAT_FEW_WAVES), dim3(64 * MAT_FEW_WAVES), 0, s, p, plan.kshare);
    QADC_LAUNCH_CHECK("k_vec_mat_few");
    return PQ_OK;
}
template <bool P2>
static int go(const MatArgs &p, const MatPlan &plan, bool async, hipStream_t s) {
    if (plan.few == 1) return go_few<P2, 1>(p, plan, s);
    if (plan.few == 2) return go_few<P2, 2>(p, plan, s);
    if (!async) return go_tiles<P2, false, 2, 2, 4, 4>(p, s);
    if constexpr (P2)
        if (plan.tile == MAT_256) return go_tiles<P2, true, 2, 4, 8, 4>(p, s);
    return go_tiles<P2, true, 2, 2, 4, 4>(p, s);
}
template <>
int qadc_vec_mat_launch<MAT_FA, MAT_FB>(const MatArgs &p, const MatPlan &plan, bool pow2, bool async, hipStream_t s) {
    return pow2 ? go<true>(p, plan, async, s) : go<false>(p, plan, async, s);
}
