// The attention kernels of one element type (CGBN_INST_T).
#include "cgbn.h"
#include "cgbn_attention.h"

namespace cgbn {

template <typename T, int DP> static void launch_width(const AttendArgs& A, int way, hipStream_t st)
{
    const dim3 grid((unsigned)A.jobs);
    switch (way) {
    case WAY_16_16: hipLaunchKernelGGL((attend_keys<T, DP, 1, 1, 1, 1>), grid, dim3(kThreads), 0, st, A); break;
    case WAY_32_16: hipLaunchKernelGGL((attend_keys<T, DP, 1, 2, 1, 1>), grid, dim3(kThreads), 0, st, A); break;
    case WAY_128_16: hipLaunchKernelGGL((attend_keys<T, DP, 4, 2, 1, 1>), grid, dim3(kThreads), 0, st, A); break;
    case WAY_32_32: hipLaunchKernelGGL((attend_keys<T, DP, 1, 2, 1, 2>), grid, dim3(kThreads), 0, st, A); break;
    case WAY_128_32: hipLaunchKernelGGL((attend_keys<T, DP, 4, 2, 1, 2>), grid, dim3(kThreads), 0, st, A); break;
    case WAY_128_128: hipLaunchKernelGGL((attend_keys<T, DP, 4, 2, 4, 2>), grid, dim3(kThreads), 0, st, A); break;
    }
}

template <> cgbn_status launch_attend<CGBN_INST_T>(const AttendArgs& A, int way, hipStream_t st)
{
    typedef CGBN_INST_T T;
    if (A.D <= 32) launch_width<T, 32>(A, way, st);
    else if (A.D <= 64) launch_width<T, 64>(A, way, st);
    else if (A.D <= 96) launch_width<T, 96>(A, way, st);
    else if (A.D <= 128) launch_width<T, 128>(A, way, st);
    else if (A.D <= 192) launch_width<T, 192>(A, way, st);
    else launch_width<T, 256>(A, way, st);
    if (hipGetLastError() != hipSuccess) return CGBN_ERR_HIP;
    if (!A.direct) {
        const long long rows = A.T * A.Hq;
        hipLaunchKernelGGL(attend_join<T>, dim3((unsigned)((rows + 3) / 4)), dim3(kThreads), 0, st, A);
        if (hipGetLastError() != hipSuccess) return CGBN_ERR_HIP;
    }
    return CGBN_OK;
}

}  // namespace cgbn
