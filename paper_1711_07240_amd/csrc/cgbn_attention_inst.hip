// The attention kernels of one element type (CGBN_INST_T).
#include "cgbn.h"
#include "cgbn_attention.h"

namespace cgbn {

template <typename T, int DP> static void launch_width(const AttendArgs& A, int prefix, int own, hipStream_t st)
{
    const dim3 grid((unsigned)A.jobs);
#define CGBN_CASE(prefix_, own_) \
    if (prefix == prefix_ && own == own_) hipLaunchKernelGGL((attend_keys<T, DP, prefix_, own_>), grid, dim3(kThreads), 0, st, A);
    if constexpr (may_stream(DP, sizeof(T))) {
        CGBN_CASE(STREAM, STREAM)
        CGBN_CASE(FEW, STREAM)
        CGBN_CASE(SOME, STREAM)
        CGBN_CASE(MANY, STREAM)
    }
    CGBN_CASE(FEW, FEW)
    CGBN_CASE(SOME, FEW)
    CGBN_CASE(MANY, FEW)
    CGBN_CASE(SOME, SOME)
    CGBN_CASE(MANY, SOME)
    CGBN_CASE(MANY, MANY)
#undef CGBN_CASE
}

// a workgroup to a row where it may have many parts, and rows are few enough for that
template <typename T, int LANES> static void launch_join(const AttendArgs& A, int tile, hipStream_t st)
{
    const long long rows = A.T * A.Hq;
    if (A.prefix_splits + A.own_splits > 8 && rows < (1 << 14)) hipLaunchKernelGGL((attend_join<T, LANES, 4>), dim3((unsigned)rows), dim3(kThreads), 0, st, A, tile);
    else hipLaunchKernelGGL((attend_join<T, LANES, 1>), dim3((unsigned)((rows + 3) / 4)), dim3(kThreads), 0, st, A, tile);
}

template <> cgbn_status launch_attend<CGBN_INST_T>(const AttendArgs& A, int prefix, int own, hipStream_t st)
{
    typedef CGBN_INST_T T;
    switch (width_of(A.D)) {
    case 32: launch_width<T, 32>(A, prefix, own, st); break;
    case 64: launch_width<T, 64>(A, prefix, own, st); break;
    case 96: launch_width<T, 96>(A, prefix, own, st); break;
    case 128: launch_width<T, 128>(A, prefix, own, st); break;
    case 192: launch_width<T, 192>(A, prefix, own, st); break;
    default: launch_width<T, 256>(A, prefix, own, st);
    }
    if (hipGetLastError() != hipSuccess) return CGBN_ERR_HIP;
    const int tile = rows_of(own, line_of(width_of(A.D), sizeof(T)), sizeof(T));
    if (A.whole && A.tail_splits > 1) {
        const int tiles = (A.jobs - A.cut) / A.tail_splits;
        hipLaunchKernelGGL(attend_join_tail<T>, dim3((unsigned)(tiles * (tile / kTailRows))), dim3(kThreads), 0, st, A, tile);
        if (hipGetLastError() != hipSuccess) return CGBN_ERR_HIP;
    }
    if (!A.direct) {
        if (A.D <= 32) launch_join<T, 8>(A, tile, st);
        else if (A.D <= 64) launch_join<T, 16>(A, tile, st);
        else if (A.D <= 128) launch_join<T, 32>(A, tile, st);
        else launch_join<T, 64>(A, tile, st);
        if (hipGetLastError() != hipSuccess) return CGBN_ERR_HIP;
    }
    return CGBN_OK;
}

}  // namespace cgbn
