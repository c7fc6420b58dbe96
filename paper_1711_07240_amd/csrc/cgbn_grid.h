// Launches of many workgroups.  Along each of its axes a launch has less than 2^32 threads; of more the runtime starts some, without an error.
#pragma once

#include <hip/hip_runtime.h>

namespace cgbn {

// Workgroups that know themselves by workgroup(): along two axes where one does not hold them, the last ones beyond the work.
constexpr long long kGridX = 1 << 21;              // (of up to 1024 threads)
__device__ __forceinline__ long long workgroup() { return (long long)blockIdx.y * kGridX + blockIdx.x; }
inline dim3 grid_of(long long groups)
{
    return groups <= kGridX ? dim3((unsigned)groups) : dim3((unsigned)kGridX, (unsigned)((groups + kGridX - 1) / kGridX));
}

}  // namespace cgbn
