// The matrix product of a layer for few rows (one token ... a few dozen): y = act(x W^T + ...), the gated pair likewise.
//
// What such a call has to do is read W once; its products are nothing.  A workgroup takes 16 rows of W (of both matrices of a
// gated pair) and its wavefronts share the reduction, 128 bytes of every row at a time in turn, so the workgroup walks 16 (32)
// streams of whole lines.  W goes from memory straight to the registers that the matrix instruction reads: lane l holds 16 bytes of
// row l % 16, the four lanes of a row 64 neighbouring ones, several steps in flight.  x is small and comes
// from the caches.  The wavefronts' sums meet in LDS and are added in wavefront order.  Where W has few rows and long ones, several
// workgroups share them, and gemm_join adds their sums.  Bound by that read: 16 x 4096 x 4096 10.3 us, 3.3 TB/s (the smallest kernels take 2.4 of them);
// the gated pair, 4 x 4096 x 11264, 37.4 us, 4.9 TB/s; 1 x 1024 x 1024 3.3 us, which is a launch and one trip to memory.
#pragma once

#include "cgbn_gemm.h"

namespace cgbn {

// 16 bytes of an operand's row of which `left` elements remain (none or fewer: the row ended before); zeros beyond.  What is not there is the row's
// last element again, so that no branch keeps one load from following the other.
template <typename T> __device__ __forceinline__ u32x4 row_chunk(const T* p, int left)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (left >= E) return *reinterpret_cast<const u32x4_any*>(p);
    uint32_t t[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 2) t[e] = p[min(e, left - 1)].bits;
        else t[e] = __float_as_uint(p[min(e, left - 1)]);
    }
    u32x4 v;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) v[k] = (2 * k < left ? t[2 * k] : 0) | (2 * k + 1 < left ? t[2 * k + 1] << 16 : 0);
        else v[k] = k < left ? t[k] : 0;
    }
    return v;
}

// 16 bytes of an operand's row, of a step that lies within the row.  HALF: of rows of an odd number of bfloat16, every other one of which starts
// between two words, where a load takes twice as long.  The words from the one it starts in, and one more, which holds the row's own last value of
// the 8 and the next (the row has one: its length is odd, whole steps are even); rows that start on a word ask for their last word again instead.
template <typename T, bool HALF> struct RowPiece {
    u32x4 v;
    uint32_t next;
    __device__ __forceinline__ void load(const T* p)
    {
        if constexpr (HALF) {
            typedef uint32_t u32x4_word __attribute__((ext_vector_type(4), aligned(4)));
            const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 2;
            const char* const a = reinterpret_cast<const char*>(p) - off;
            v = *reinterpret_cast<const u32x4_word*>(a);
            next = *reinterpret_cast<const uint32_t*>(a + 12 + 2 * off);
        } else {
            v = *reinterpret_cast<const u32x4_any*>(p);
        }
    }
    __device__ __forceinline__ u32x4 get(const T* p) const
    {
        if constexpr (HALF) {
            const uint32_t off = (uint32_t)reinterpret_cast<uintptr_t>(p) & 2;
            return u32x4{__builtin_amdgcn_alignbyte(v[1], v[0], off), __builtin_amdgcn_alignbyte(v[2], v[1], off), __builtin_amdgcn_alignbyte(v[3], v[2], off),
                         __builtin_amdgcn_alignbyte(next, v[3], off)};
        } else {
            return v;
        }
    }
};

// FM: 16-row blocks of x; NW: wavefronts; HALF: see RowPiece
template <typename T, bool GATED, int FM, int NW, bool HALF>
__global__ __launch_bounds__(NW * kWave) void gemm_rows(const GemmArgs G)
{
    constexpr int E = 16 / (int)sizeof(T), STEP = 8 * E, P = GATED ? 2 : 1, U = FM == 1 && !GATED ? 4 : 2;
    __shared__ f32x4 sums[NW][FM * P][kWave];
    const int l = (int)threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave), t = l & 15, q = l >> 4;
    const int j0 = (int)blockIdx.x * 16;
    const T *pw[P], *px[FM];
#pragma unroll
    for (int p = 0; p < P; ++p) pw[p] = static_cast<const T*>(G.B[p]) + (long long)min(j0 + t, G.J - 1) * G.ldb + q * E;
#pragma unroll
    for (int m = 0; m < FM; ++m) px[m] = static_cast<const T*>(G.A[0]) + (long long)min(m * 16 + t, G.I - 1) * G.lda + q * E;

    f32x4 acc[P][FM];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int m = 0; m < FM; ++m) acc[p][m] = f32x4{0.f, 0.f, 0.f, 0.f};
    const int begin = (int)blockIdx.y * G.per, steps = min(begin + G.per, (G.R + STEP - 1) / STEP), full = min(steps, G.R / STEP);
    int s = begin + wave;
    for (; s + (U - 1) * NW < full; s += U * NW) {
        RowPiece<T, HALF> w[U][P][2], x[U][FM][2];
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = (s + u * NW) * STEP + h * 4 * E;
#pragma unroll
                for (int p = 0; p < P; ++p) w[u][p][h].load(pw[p] + r);
#pragma unroll
                for (int m = 0; m < FM; ++m) x[u][m][h].load(px[m] + r);
            }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int m = 0; m < FM; ++m) acc[p][m] = multiply<T>(w[u][p][h].get(pw[p]), x[u][m][h].get(px[m]), acc[p][m]);
    }
    for (; s < steps; s += NW) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int r = s * STEP + h * 4 * E, left = G.R - r - q * E;
            const bool whole = HALF && s < full;
            auto chunk = [&](const T* row) {
                if (!whole) return row_chunk<T>(row + r, left);
                RowPiece<T, HALF> piece;
                piece.load(row + r);
                return piece.get(row);
            };
            u32x4 x[FM];
#pragma unroll
            for (int m = 0; m < FM; ++m) x[m] = chunk(px[m]);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const u32x4 w = chunk(pw[p]);
#pragma unroll
                for (int m = 0; m < FM; ++m) acc[p][m] = multiply<T>(w, x[m], acc[p][m]);
            }
        }
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int m = 0; m < FM; ++m) sums[wave][p * FM + m][l] = acc[p][m];
    __syncthreads();
    if (wave >= FM) return;
    const int m = wave, i = m * 16 + t, j = j0 + q * 4;
    if (i >= G.I || j >= G.J) return;
    float v[P][4];
#pragma unroll
    for (int p = 0; p < P; ++p) {
        f32x4 a = sums[0][p * FM + m][l];
#pragma unroll
        for (int k = 1; k < NW; ++k) a += sums[k][p * FM + m][l];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[p][k] = a[k];
    }
    if (G.splits > 1) {
#pragma unroll
        for (int p = 0; p < P; ++p) store_run<float, 4>(G.part + (((long long)blockIdx.y * P + p) * G.I + i) * G.J + j, v[p], G.J - j);
        return;
    }
    const long long o = (long long)i * G.ldc + j;
    float extra[4];
    if constexpr (!GATED) {
        float bias[4];
        load_bias<4>(G, bias, j, G.J - j);
        load_extras<T, 4>(G, extra, bias, o, G.J - j);
    }
    if constexpr (GATED) finish_gated<T, 4>(G, v[0], v[1], o, G.J - j);
    else finish_linear<T, 4>(G, v[0], extra, o, G.J - j);
}

}  // namespace cgbn
