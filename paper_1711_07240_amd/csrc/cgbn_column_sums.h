// The last step of a gradient that is summed over rows: partial sums of the workgroups, added in a fixed order.
#pragma once

#include "cgbn_kernels.h"

namespace cgbn {
namespace {

// Sums over `rows` of part[row * ld + n], n < N, in double precision: n < n0 to out0, the others to out1.  A workgroup takes 16 columns (a
// line of 64 bytes a row) with 16 threads each.
__global__ __launch_bounds__(kThreads) void column_sums(const float* part, int rows, int ld, int N, float* out0, int n0, float* out1)
{
    __shared__ double red[16][17];
    const int c = (int)threadIdx.x & 15, k = (int)threadIdx.x >> 4, n = (int)blockIdx.x * 16 + c;
    double s = 0.;
    if (n < N)
        for (int r = k; r < rows; r += 16) s += (double)part[(long long)r * ld + n];
    red[k][c] = s;
    __syncthreads();
    if (k != 0 || n >= N) return;
    for (int x = 1; x < 16; ++x) s += red[x][c];
    if (n < n0) out0[n] = (float)s;
    else out1[n - n0] = (float)s;
}

}  // namespace
}  // namespace cgbn
