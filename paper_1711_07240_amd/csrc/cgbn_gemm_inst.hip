// The matrix-product kernels of one element type and form (CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED): see cgbn_gemm.h.
#include "cgbn_gemm.h"
#include "cgbn_gemm_plan.h"

namespace cgbn {

template <> hipError_t launch_gemm<CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED>(const GemmPlan& p, GemmArgs G, hipStream_t st)
{
    G.ti = p.ti; G.tj = p.tj; G.splits = p.splits; G.per = p.per;
    const dim3 grid((unsigned)((long long)p.ti * p.tj * p.splits * G.batch));
#define CGBN_TILE_CASE(n_, BI_, BJ_, WI_, WJ_)                                                                                   \
    case n_:                                                                                                                     \
        if (p.splits > 1)                                                                                                        \
            hipLaunchKernelGGL((gemm_tile<CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED, true, BI_, BJ_, WI_, WJ_>), grid,        \
                               dim3(WI_ * WJ_ * kWave), 0, st, G);                                                               \
        else                                                                                                                     \
            hipLaunchKernelGGL((gemm_tile<CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED, false, BI_, BJ_, WI_, WJ_>), grid,       \
                               dim3(WI_ * WJ_ * kWave), 0, st, G);                                                               \
        break;
    switch (p.shape) { CGBN_TILE_SHAPES(CGBN_TILE_CASE) }
#undef CGBN_TILE_CASE
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.splits == 1) return e;
    const long long values = (long long)G.I * G.J * (CGBN_INST_GATED ? 1 : G.batch);
    if (G.J % 4 == 0)
        hipLaunchKernelGGL((gemm_join<CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED, 4>), dim3((unsigned)((values / 4 + kThreads - 1) / kThreads)),
                           dim3(kThreads), 0, st, G);
    else
        hipLaunchKernelGGL((gemm_join<CGBN_INST_T, CGBN_INST_FORM, CGBN_INST_GATED, 1>), dim3((unsigned)((values + kThreads - 1) / kThreads)),
                           dim3(kThreads), 0, st, G);
    return hipGetLastError();
}

}  // namespace cgbn
