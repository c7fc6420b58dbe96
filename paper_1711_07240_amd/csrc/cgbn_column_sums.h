// The last step of a gradient that is summed over rows: partial sums of the workgroups, added in a fixed order.
#pragma once

#include "cgbn_kernels.h"

namespace cgbn {
namespace {

// Sums over `rows` of part[row * ld + n], n < N, in double precision: n < n0 to out0, the others to out1.  A workgroup takes 16
// columns (64 bytes a row) with 64 threads each, a thread's rows eight at a time: the sums are few and what they take is the
// loads' way (1023 rows of 128: 7 us, 512 of 160: 4.7; a launch is 3 of them).
constexpr int kSumThreads = 1024;
__global__ __launch_bounds__(kSumThreads) void column_sums(const float* part, int rows, int ld, int N, float* out0, int n0, float* out1)
{
    __shared__ double red[64][17];
    const int c = (int)threadIdx.x & 15, k = (int)threadIdx.x >> 4, n = (int)blockIdx.x * 16 + c;
    double s = 0.;
    if (n < N) {
        for (int r0 = k; r0 < rows; r0 += 64 * 8) {
            float v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) v[u] = r0 + u * 64 < rows ? part[(long long)(r0 + u * 64) * ld + n] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; ++u) s += (double)v[u];
        }
    }
    red[k][c] = s;
    __syncthreads();
    for (int half = 32; half >= 1; half /= 2) {
        if (k < half) red[k][c] += red[k + half][c];
        __syncthreads();
    }
    if (k != 0 || n >= N) return;
    if (n < n0) out0[n] = (float)red[0][c];
    else out1[n - n0] = (float)red[0][c];
}

}  // namespace
}  // namespace cgbn
