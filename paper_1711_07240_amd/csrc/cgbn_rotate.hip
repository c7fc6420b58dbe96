// The rotation of queries and keys by position, forward and backward, without a norm, with angles formed here.
//
//   (a, b) -> m (a cos t - b sin t, b cos t + a sin t),  t = position * frequency;  backward the same with -t
//
// Bound by memory: q and k are read and written once.  A wavefront takes heads of one token; its lanes first form the token's R/2 angles,
// one each, into LDS, from where all heads take them.  Of the far positions of long contexts a product in 32 bits would be off by whole
// hundredths of a turn (2^20 positions: 2^-4 radians), and a table of cosines and sines for each of them would be 512 bytes a position of a head of
// 128 to read; so the turns are counted in 64 bits, which the vector unit has at half rate, and only the rest, within an eighth of a turn, goes on in 32.
//
// Measured: 40 heads of 128 bfloat16, 32768 tokens, 121 us, 5.5 TB/s; float backward, 40 heads of 80, 32 turned, 8191 tokens, 38 us, 5.5; 8 tokens 4.2 us, a
// launch.  Rows go in chunks of 16 bytes, 8, two values or one, as rows, strides, addresses and halves allow (144 heads of 45 bfloat16, 23233 tokens, one by one,
// 195 us, 3.1 TB/s).
#include "cgbn.h"
#include "cgbn_grid.h"
#include "cgbn_heads.h"

#include <cmath>
#include <cstring>

namespace cgbn {
namespace {

struct RotateArgs {
    const void* x[2];              // q, k or their gradients
    void* out[2];
    long long ldx[2], ldo[2];
    const int* positions;
    const double* freq;
    long long T;
    int H[2], D, R;
    float magnitude;
    int turned, per;               // items of a head: those that are turned, all (in place: the same)
    int step, far;                 // values from one turned item to the next, and from an item's first chunk to its second (0: it has none)
    int parts;                     // wavefronts that share a token's heads
};

constexpr int kMaxHalf = 512;      // angles of a token

// cos and sin of a quarter turn times x, |x| <= 1/2, by their Taylor polynomials: off by less than 1.75 units of 2^-24 (1.5 the sine), with the rounding of x to float:
// the largest over 6e7 angles
__device__ __forceinline__ void quarter(float x, float* c, float* s)
{
    const float t = x * 1.5707963267948966f, u = t * t;
    *s = fmaf(t * u, fmaf(u, fmaf(u, fmaf(u, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f), t);
    *c = fmaf(u, fmaf(u, fmaf(u, fmaf(u, fmaf(u, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f), 1.f);
}

// cos and sin of t radians: whole and quarter turns taken off in 64 bits, exactly, once they are counted (t, the constant and their product: off by less than 1.3 * 2^-52 of t)
__device__ __forceinline__ void cos_sin(double t, float* c, float* s)
{
    double turns = t * 0.15915494309189535;
    turns = 4. * (turns - rint(turns));
    const double n = rint(turns);
    float u, v;
    quarter((float)(turns - n), &u, &v);
    const int quadrant = (int)n & 3;
    const float a = quadrant & 1 ? v : u, b = quadrant & 1 ? u : v;
    *c = quadrant == 1 || quadrant == 2 ? -a : a;
    *s = quadrant >= 2 ? -b : b;
}

// FAR: an item is two chunks, the values of the one turned with the other's (halves, or chunks of one value); else one of neighbouring pairs.
// SIGN 1: turn, -1: turn back; NT: results go past the caches
template <typename T, int E, bool FAR, int SIGN, bool NT> __global__ __launch_bounds__(kThreads) void rotate(const RotateArgs A)
{
    __shared__ __attribute__((aligned(16))) float cosines[kThreads / kWave][kMaxHalf], sines[kThreads / kWave][kMaxHalf];
    constexpr int AHEAD = 4, PAIRS = FAR ? E : E / 2 > 0 ? E / 2 : 1;
    const int lane = (int)threadIdx.x % kWave, w = (int)threadIdx.x / kWave;
    const long long wave = workgroup() * (kThreads / kWave) + w, token = wave / A.parts;
    const int part = (int)(wave - token * A.parts);
    if (token >= A.T) return;
    const double position = A.positions ? (double)A.positions[token] : (double)token;
    const int half = A.R / 2;
    for (int i = lane; i < half; i += kWave) {
        float c, s;
        cos_sin(position * A.freq[i], &c, &s);
        cosines[w][i] = c * A.magnitude;
        sines[w][i] = s * (SIGN * A.magnitude);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the lanes of a wavefront read each other's)
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const T* const x = static_cast<const T*>(A.x[t]) + token * A.ldx[t];
        T* const y = static_cast<T*>(A.out[t]) + token * A.ldo[t];
        const int items = A.H[t] * A.per;
        for (int i0 = part * kWave + lane; i0 < items; i0 += AHEAD * kWave * A.parts) {
            typename Chunk<T, E>::Raw ra[AHEAD], rb[AHEAD];
            int at[AHEAD], item[AHEAD];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = i0 + k * kWave * A.parts;
                if (i >= items) continue;
                const int h = (unsigned)i / (unsigned)A.per;
                item[k] = i - h * A.per;
                // behind the turned ones the others, in order
                at[k] = h * A.D + (item[k] < A.turned ? item[k] * A.step : FAR ? A.R + (item[k] - A.turned) * E : item[k] * E);
                ra[k] = Chunk<T, E>::load(x + at[k]);
                if (FAR && item[k] < A.turned) rb[k] = Chunk<T, E>::load(x + at[k] + A.far);
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (i0 + k * kWave * A.parts >= items) continue;
                float a[E], b[E];
                Chunk<T, E>::unpack(ra[k], a);
                if (item[k] < A.turned) {
                    float c[PAIRS], s[PAIRS];
                    if constexpr (FAR) {
                        load_floats<PAIRS>(&cosines[w][item[k] * E], c);
                        load_floats<PAIRS>(&sines[w][item[k] * E], s);
                        Chunk<T, E>::unpack(rb[k], b);
#pragma unroll
                        for (int e = 0; e < E; ++e) {
                            const float u = a[e], v = b[e];
                            a[e] = u * c[e] - v * s[e];
                            b[e] = v * c[e] + u * s[e];
                        }
                        Chunk<T, E>::template store<NT>(y + at[k] + A.far, b);
                    } else {
#pragma unroll
                        for (int e = 0; e < PAIRS; ++e) {
                            const int i = item[k] * PAIRS + e;          // (the last chunk may be turned in part)
                            if (i >= half) continue;
                            c[e] = cosines[w][i];
                            s[e] = sines[w][i];
                            const float u = a[2 * e], v = a[2 * e + 1];
                            a[2 * e] = u * c[e] - v * s[e];
                            a[2 * e + 1] = v * c[e] + u * s[e];
                        }
                    }
                }
                Chunk<T, E>::template store<NT>(y + at[k], a);
            }
        }
    }
}

// ---- host ----

cgbn_status launched() { return hipGetLastError() == hipSuccess ? CGBN_OK : CGBN_ERR_HIP; }

constexpr long long kMaxTokens = 1ll << 30, kMaxStride = 1ll << 32;
constexpr int kMaxHeads = 1 << 14, kMaxD = 2 * kMaxHalf;

// rows in chunks of E values
template <typename T> bool chunks_fit(const RotateArgs& A, int E, bool halves)
{
    const size_t bytes = E * sizeof(T);
    if (A.D % E != 0 || (halves && (A.R / 2) % E != 0)) return false;
    for (int t = 0; t < (A.H[1] ? 2 : 1); ++t)
        if (reinterpret_cast<uintptr_t>(A.x[t]) % bytes || reinterpret_cast<uintptr_t>(A.out[t]) % bytes || A.ldx[t] % E != 0 || A.ldo[t] % E != 0) return false;
    return true;
}

template <typename T, int E, int SIGN, bool NT> cgbn_status launch(RotateArgs& A, bool halves, hipStream_t st)
{
    const bool far = halves || E == 1;
    const int count = far ? A.R / 2 / E : (A.R + E - 1) / E;
    A.turned = count;
    A.step = halves ? E : far ? 2 : E;
    A.far = halves ? A.R / 2 : 1;
    const bool in_place = A.out[0] == A.x[0] && (!A.H[1] || A.out[1] == A.x[1]);
    A.per = in_place ? count : far ? count + (A.D - A.R) / E : A.D / E;
    if (A.per == 0) return CGBN_OK;
    const long long most = ((long long)(A.H[0] > A.H[1] ? A.H[0] : A.H[1]) * A.per + kWave - 1) / kWave;
    A.parts = 1;
    while (A.parts < most && A.T * A.parts < 4096) A.parts *= 2;
    if (A.parts > most) A.parts = (int)most;
    const dim3 grid = grid_of((A.T * A.parts + 3) / 4);
    if (far) hipLaunchKernelGGL((rotate<T, E, true, SIGN, NT>), grid, dim3(kThreads), 0, st, A);
    else if constexpr (E > 1) hipLaunchKernelGGL((rotate<T, E, false, SIGN, NT>), grid, dim3(kThreads), 0, st, A);
    return launched();
}

template <typename T, int SIGN> cgbn_status run(RotateArgs& A, bool halves, hipStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    // Results of more than the caches next to the compute units hold go past them, as the head norm's do
    const bool past = (double)A.T * (A.H[0] + A.H[1]) * A.D * sizeof(T) > 32e6;
    if (chunks_fit<T>(A, E, halves)) return past ? launch<T, E, SIGN, true>(A, halves, st) : launch<T, E, SIGN, false>(A, halves, st);
    if (sizeof(T) == 2 && chunks_fit<T>(A, 4, halves)) return launch<T, 4, SIGN, false>(A, halves, st);
    if (chunks_fit<T>(A, 2, halves)) return launch<T, 2, SIGN, false>(A, halves, st);
    return launch<T, 1, SIGN, false>(A, halves, st);
}

template <int SIGN> cgbn_status call(RotateArgs& A, cgbn_rotation style, cgbn_dtype dtype, void* stream)
{
    if (dtype != CGBN_F32 && dtype != CGBN_BF16) return CGBN_ERR_ENUM;
    if (style != CGBN_ROTATE_HALVES && style != CGBN_ROTATE_PAIRS) return CGBN_ERR_ACTIVATION;
    if (A.T < 0 || A.T > kMaxTokens || A.H[0] < 1 || A.H[0] > kMaxHeads || A.H[1] < 0 || A.H[1] > kMaxHeads || A.D < 1 || A.D > kMaxD) return CGBN_ERR_SHAPE;
    if (A.T * (A.H[0] + A.H[1]) > (1ll << 33) || A.R < 0 || A.R > A.D || A.R % 2 != 0) return CGBN_ERR_SHAPE;
    if (A.T == 0) return CGBN_OK;
    if (A.R && !A.freq) return CGBN_ERR_NULL;
    const size_t elem = dtype == CGBN_F32 ? 4 : 2;
    for (int t = 0; t < (A.H[1] ? 2 : 1); ++t) {
        if (!A.x[t] || !A.out[t]) return CGBN_ERR_NULL;
        const long long width = (long long)A.H[t] * A.D;
        if (A.ldx[t] > kMaxStride || A.ldo[t] > kMaxStride) return CGBN_ERR_SHAPE;
        if (A.T > 1 && (A.ldx[t] < width || A.ldo[t] < width)) return CGBN_ERR_STRIDE;
        if (reinterpret_cast<uintptr_t>(A.x[t]) % elem || reinterpret_cast<uintptr_t>(A.out[t]) % elem) return CGBN_ERR_ALIGN;
        if (A.out[t] == A.x[t] && A.T > 1 && A.ldo[t] != A.ldx[t]) return CGBN_ERR_ALIAS;
        if (A.R && (A.out[t] == A.freq || (A.positions && A.out[t] == A.positions))) return CGBN_ERR_ALIAS;
    }
    if (reinterpret_cast<uintptr_t>(A.freq) % 8 || reinterpret_cast<uintptr_t>(A.positions) % 4) return CGBN_ERR_ALIGN;
    if (A.H[1] && (A.out[0] == A.out[1] || A.out[0] == A.x[1] || A.out[1] == A.x[0])) return CGBN_ERR_ALIAS;
    const bool halves = style == CGBN_ROTATE_HALVES;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == CGBN_F32 ? run<float, SIGN>(A, halves, st) : run<bf16_t, SIGN>(A, halves, st);
}

RotateArgs args(const void* q, long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk, int D, int R, const int* positions,
                const double* freq, float magnitude, void* yq, long long ldyq, void* yk, long long ldyk)
{
    RotateArgs A;
    std::memset(&A, 0, sizeof(A));
    A.x[0] = q; A.x[1] = k; A.out[0] = yq; A.out[1] = yk;
    A.ldx[0] = ldq; A.ldx[1] = ldk; A.ldo[0] = ldyq; A.ldo[1] = ldyk;
    A.positions = positions; A.freq = freq; A.T = T; A.H[0] = Hq; A.H[1] = Hk; A.D = D; A.R = R; A.magnitude = magnitude;
    return A;
}

}  // namespace
}  // namespace cgbn

using namespace cgbn;

extern "C" {

cgbn_status cgbn_rotary_frequencies(int R, double base, cgbn_scaling scaling, double factor, double trained, double fast, double slow, double* freq)
{
    if (scaling < CGBN_SCALE_NONE || scaling > CGBN_SCALE_PARTS) return CGBN_ERR_ACTIVATION;
    if (R < 0 || R > kMaxD || R % 2 != 0 || !(base > 1.) || std::isinf(base)) return CGBN_ERR_SHAPE;
    if (scaling != CGBN_SCALE_NONE && (!(factor >= 1.) || std::isinf(factor))) return CGBN_ERR_SHAPE;
    if (scaling == CGBN_SCALE_PARTS && (!(trained >= 1.) || std::isinf(trained) || !(slow >= 0.) || !(fast > slow) || std::isinf(fast))) return CGBN_ERR_SHAPE;
    if (R && !freq) return CGBN_ERR_NULL;
    if (scaling == CGBN_SCALE_BASE && R > 2) base *= std::pow(factor, (double)R / (R - 2));
    for (int i = 0; i < R / 2; ++i) {
        double f = std::pow(base, -2. * i / R);
        if (scaling == CGBN_SCALE_POSITIONS) f /= factor;
        if (scaling == CGBN_SCALE_PARTS) {
            double keep = (trained * f / 6.283185307179586 - slow) / (fast - slow);
            keep = keep < 0. ? 0. : keep > 1. ? 1. : keep;
            f = f * keep + f / factor * (1. - keep);
        }
        freq[i] = f;
    }
    return CGBN_OK;
}

cgbn_status cgbn_rotate_forward(const void* q, long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk, int D, int R, cgbn_rotation style,
                                const int* positions, const double* freq, float magnitude, void* yq, long long ldyq, void* yk, long long ldyk,
                                cgbn_dtype dtype, void* stream)
{
    RotateArgs A = args(q, ldq, k, ldk, T, Hq, Hk, D, R, positions, freq, magnitude, yq, ldyq, yk, ldyk);
    return call<1>(A, style, dtype, stream);
}

cgbn_status cgbn_rotate_backward(const void* dyq, long long lddyq, const void* dyk, long long lddyk, long long T, int Hq, int Hk, int D, int R,
                                 cgbn_rotation style, const int* positions, const double* freq, float magnitude, void* dq, long long lddq, void* dk,
                                 long long lddk, cgbn_dtype dtype, void* stream)
{
    RotateArgs A = args(dyq, lddyq, dyk, lddyk, T, Hq, Hk, D, R, positions, freq, magnitude, dq, lddq, dk, lddk);
    return call<-1>(A, style, dtype, stream);
}

}  // extern "C"
