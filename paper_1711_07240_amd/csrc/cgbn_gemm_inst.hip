// The matrix-product kernels of one element type and form: see cgbn_gemm.h.  The build passes CGBN_INST_T and CGBN_INST_FORM; 0: the
// forward product, 1: the gated pair, 2: the two of a backward pass, together and each by itself.
#include "cgbn_gemm.h"
#include "cgbn_gemm_plan.h"

namespace cgbn {
namespace {

void take(const GemmPlan& p, GemmArgs* G)
{
    G->ti = p.ti; G->tj = p.tj; G->splits = p.splits; G->per = p.per;
    // Results of more than the caches next to the compute units hold go past them (268800 x 128 x 512 with dx as the result 121 us
    // against 87, 67200 x 256 x 1024 with a residual 115 against 94); smaller ones stay there for whoever reads them next.
    G->nt = (double)G->I * G->J * p.elem > 32e6;
}

unsigned groups_of(const GemmArgs& G) { return (unsigned)((long long)G.ti * G.tj * G.splits * G.batch); }

template <typename T, int FORM, bool GATED> hipError_t join(const GemmArgs& G, hipStream_t st)
{
    if (G.splits == 1) return hipSuccess;
    const int n = G.J % 4 == 0 ? 4 : 1;
    const long long threads = (long long)G.I * G.J * (GATED ? 1 : G.batch) / n;
    int lanes = 1;
    while (lanes < 16 && lanes * 4 <= G.splits && threads * lanes < 128 * 1024) lanes *= 2;
    const dim3 grid((unsigned)((threads * lanes + kThreads - 1) / kThreads));
    if (n == 4) hipLaunchKernelGGL((gemm_join<T, FORM, GATED, 4>), grid, dim3(kThreads), 0, st, G, lanes);
    else hipLaunchKernelGGL((gemm_join<T, FORM, GATED, 1>), grid, dim3(kThreads), 0, st, G, lanes);
    return hipGetLastError();
}

template <typename T, int FORM, bool GATED> hipError_t launch_one(const GemmPlan& p, GemmArgs G, hipStream_t st)
{
    take(p, &G);
    if constexpr (sizeof(T) == 2 && FORM == FORM_NT && !GATED) {
        if (short_shape(p.shape, G.splits, G.I, G.J, G.R, G.residual != nullptr)) {
            G.ti = (G.I + kShortI - 1) / kShortI;
            G.tj = (G.J + kShortJ - 1) / kShortJ;
            if (G.residual) hipLaunchKernelGGL((gemm_short<T, kShortI, kShortJ, 2, 2, true>), dim3(groups_of(G)), dim3(4 * kWave), 0, st, G);
            else hipLaunchKernelGGL((gemm_short<T, kShortI, kShortJ, 2, 2, false>), dim3(groups_of(G)), dim3(4 * kWave), 0, st, G);
            return hipGetLastError();
        }
    }
#define CGBN_CASE(n_, BI_, BJ_, WI_, WJ_) \
    case n_: hipLaunchKernelGGL((gemm_tile<T, FORM, GATED, BI_, BJ_, WI_, WJ_>), dim3(groups_of(G)), dim3(WI_ * WJ_ * kWave), 0, st, G); break;
    if constexpr (sizeof(T) == 2) switch (p.shape) { CGBN_TILE_SHAPES(CGBN_CASE) }
    else switch (p.shape) { CGBN_TILE_SHAPES_FLOAT(CGBN_CASE) }
#undef CGBN_CASE
    const hipError_t e = hipGetLastError();
    return e != hipSuccess ? e : join<T, FORM, GATED>(G, st);
}

template <typename T> void two(int shape, const GemmArgs& X, const GemmArgs& W, int nx, unsigned n, hipStream_t st)
{
#define CGBN_CASE(n_, BI_, BJ_, WI_, WJ_) \
    case n_: hipLaunchKernelGGL((gemm_two<T, BI_, BJ_, WI_, WJ_>), dim3(n), dim3(WI_ * WJ_ * kWave), 0, st, X, W, nx); break;
    if constexpr (sizeof(T) == 2) switch (shape) { CGBN_TILE_SHAPES(CGBN_CASE) }
    else switch (shape) { CGBN_TILE_SHAPES_FLOAT(CGBN_CASE) }
#undef CGBN_CASE
}

}  // namespace

#if CGBN_INST_FORM == 0
template <> hipError_t launch_gemm<CGBN_INST_T, FORM_NT, false>(const GemmPlan& p, GemmArgs G, hipStream_t st) { return launch_one<CGBN_INST_T, FORM_NT, false>(p, G, st); }
template <> hipError_t launch_join<CGBN_INST_T, false>(const GemmArgs& G, hipStream_t st) { return join<CGBN_INST_T, FORM_NT, false>(G, st); }
#elif CGBN_INST_FORM == 1
template <> hipError_t launch_join<CGBN_INST_T, true>(const GemmArgs& G, hipStream_t st) { return join<CGBN_INST_T, FORM_NT, true>(G, st); }
template <> hipError_t launch_gemm<CGBN_INST_T, FORM_NT, true>(const GemmPlan& p, GemmArgs G, hipStream_t st) { return launch_one<CGBN_INST_T, FORM_NT, true>(p, G, st); }
#else
template <> hipError_t launch_gemm<CGBN_INST_T, FORM_NN, false>(const GemmPlan& p, GemmArgs G, hipStream_t st) { return launch_one<CGBN_INST_T, FORM_NN, false>(p, G, st); }
template <> hipError_t launch_gemm<CGBN_INST_T, FORM_TN, false>(const GemmPlan& p, GemmArgs G, hipStream_t st) { return launch_one<CGBN_INST_T, FORM_TN, false>(p, G, st); }
template <> hipError_t launch_two<CGBN_INST_T>(const GemmPlan& px, GemmArgs X, const GemmPlan& pw, GemmArgs W, hipStream_t st)
{
    take(px, &X);
    take(pw, &W);
    const unsigned nx = groups_of(X), nw = groups_of(W);
    two<CGBN_INST_T>(px.shape, X, W, (int)nx, nx + nw, st);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) e = join<CGBN_INST_T, FORM_NN, false>(X, st);
    return e != hipSuccess ? e : join<CGBN_INST_T, FORM_TN, false>(W, st);
}
#endif

}  // namespace cgbn
