// The norm of queries and keys, head by head, with the rotation by position in the same pass, and its backward.
//
//   forward   r = 1 / sqrt(mean(x^2) + eps);  n = w x r;  y = rotation(n)
//   backward  e = inverse rotation(dy);  dw = sum over rows of e x r;  t = e w;  dx = r (t - x r mean(t x r))
//
// Bound by memory: forward one read and one write of q and k, backward two reads and one write (r comes from x again: reading
// a stored r would save nothing, x is read anyway).  A row of D values is held by a group of lanes, two 16-byte chunks a
// lane, chosen so that the values that are turned together are in the same lane: with halves, chunk c and the one R/2 values
// on; with pairs any two.  So nothing but the row's sums crosses lanes.  A wavefront takes heads of ONE token: cosines and sines,
// which in float are twice the bytes of a bfloat16 row, and the weights are fetched once for all of them.
// Chunks are as wide as rows, strides, addresses and halves allow, 16 bytes, 8, two values or one (value by value a wavefront to a row, and
// in chunks: 144 heads of 80 bfloat16, 40 turned, 5845 tokens, 348 and 65 us; 24 of 82, 40 turned, 8000 tokens, 77 and 21, backward 230 and 48;
// 80 of 39, 15994 tokens, 276 and 70, backward 606 and 170).  Rows of more than 64 pairs of chunks a wavefront takes one at a time, a value a
// lane and step, and reads partners again from the cache (`_any`).
//
// Measured: 40 heads of 128 bfloat16, 32768 tokens, 119 us, 5.8 TB/s, more than a copy's rate; float backward, 40 heads of 80, 8191 tokens,
// 71.5 us with the weights' sums, 4.4 TB/s, 57 of them this kernel's, 5.6; 8 tokens 3.9 us, two trips to memory and a launch.
//
// Sums are float: a row's over at most 16 values a lane, then a fixed tree; the weights' gradients per lane over the rows a wavefront
// walks, then over wavefronts in order, then over workgroups in double precision.  No atomics.
#include "cgbn.h"
#include "cgbn_column_sums.h"
#include "cgbn_grid.h"
#include "cgbn_heads.h"

#include <cmath>
#include <cstring>

namespace cgbn {
namespace {

struct HeadArgs {
    const void *x[2], *dy[2];          // q, k
    void* out[2];                      // yq, yk or dq, dk
    long long ldx[2], lddy[2], ldo[2];
    const float *w[2], *cos, *sin;
    const int* positions;
    float* part;                       // backward: [workgroups][2][D]
    long long T;
    int H[2], D, R, table;
    int style;                         // CGBN_ROTATE_*
    float eps, inv_D;
    int pairs, lead, step, far, rest;  // chunk pairs of a row; those turned together, chunks from one to the next and within one; see chunks_of()
    int parts;                         // wavefronts that share a token's heads
};

// The sum over the L lanes of a group (a power of two, groups aligned): every lane gets it, whatever its place, in the same order.
template <int L> __device__ __forceinline__ float group_sum(float v)
{
#define CGBN_DPP_ADD(ctrl_) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl_, 0xf, 0xf, true))
    if constexpr (L >= 2) CGBN_DPP_ADD(0xB1);      // lane ^ 1
    if constexpr (L >= 4) CGBN_DPP_ADD(0x4E);      // lane ^ 2
    if constexpr (L >= 8) CGBN_DPP_ADD(0x141);     // the other half of 8
    if constexpr (L >= 16) CGBN_DPP_ADD(0x140);    // the other half of 16
#undef CGBN_DPP_ADD
    if constexpr (L >= 32) v += __shfl_xor(v, 16);
    if constexpr (L >= 64) v += __shfl_xor(v, 32);
    return v;
}

// The first elements of a lane's two chunks (-1: none).  Turned together as halves, or chunks of one value: `lead` pairs of chunks `far`
// apart, then the `rest` chunks that are not turned, first half with second half.
template <int E> __device__ __forceinline__ void chunks_of(const HeadArgs& A, int p, int* c0, int* c1)
{
    *c0 = *c1 = -1;
    if (p >= A.pairs) return;
    if (p < A.lead) {
        *c0 = p * A.step * E;
        *c1 = *c0 + A.far * E;
    } else {
        const int k = p - A.lead, first = 2 * A.lead, half = (A.rest + 1) / 2;
        *c0 = (first + k) * E;
        if (k + half < A.rest) *c1 = (first + k + half) * E;
    }
}

// cosines and sines of a lane's chunks.  Halves: of value e of both chunks; pairs: of values 2e, 2e + 1 of chunk 0 in the first
// half, of chunk 1 in the second.  Chunks of one value are turned as halves are.  Not turned: 1 and 0.
template <int E> struct Turn {
    float c[E], s[E];
    static __device__ __forceinline__ bool across(int style) { return E == 1 || style == CGBN_ROTATE_HALVES; }
    __device__ __forceinline__ void load(const HeadArgs& A, long long token, int p, int c0, int c1)
    {
#pragma unroll
        for (int e = 0; e < E; ++e) { c[e] = 1.f; s[e] = 0.f; }
        if (A.R == 0) return;
        const long long pos = A.positions ? (long long)A.positions[token] : token;
        const bool in = pos >= 0 && pos < A.table;
        const long long row = in ? pos * (A.R / 2) : 0;
        const float bad = __int_as_float(0x7fc00000);
        if (across(A.style)) {
            if (c0 < 0 || p >= A.lead) return;
            load_floats<E>(A.cos + row + p * E, c);
            load_floats<E>(A.sin + row + p * E, s);
        } else if constexpr (E > 1) {
            // (chunks that are turned in part: the angles of those of their pairs that are)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int first = h ? c1 : c0, n = first < 0 ? 0 : (A.R - first) / 2;
                if (n >= E / 2) {
                    load_floats<E / 2>(A.cos + row + first / 2, *reinterpret_cast<float(*)[E / 2]>(c + h * (E / 2)));
                    load_floats<E / 2>(A.sin + row + first / 2, *reinterpret_cast<float(*)[E / 2]>(s + h * (E / 2)));
                } else {
#pragma unroll
                    for (int e = 0; e < E / 2; ++e) {
                        if (e >= n) continue;
                        c[h * (E / 2) + e] = A.cos[row + first / 2 + e];
                        s[h * (E / 2) + e] = A.sin[row + first / 2 + e];
                    }
                }
            }
        }
        if (!in) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const bool turned = across(A.style) || (e < E / 2 ? c0 >= 0 && c0 + 2 * e < A.R : c1 >= 0 && c1 + 2 * (e - E / 2) < A.R);
                if (turned) c[e] = s[e] = bad;
            }
        }
    }
    // sign 1: turn; -1: turn back
    template <int SIGN> __device__ __forceinline__ void apply(int style, float (&a)[E], float (&b)[E]) const
    {
        if (across(style)) {
#pragma unroll
            for (int e = 0; e < E; ++e) {
                const float u = a[e], v = b[e], t = SIGN * s[e];
                a[e] = u * c[e] - v * t;
                b[e] = v * c[e] + u * t;
            }
        } else if constexpr (E > 1) {
#pragma unroll
            for (int e = 0; e < E / 2; ++e) {
                const float t = SIGN * s[e], u = a[2 * e], v = a[2 * e + 1];
                a[2 * e] = u * c[e] - v * t;
                a[2 * e + 1] = v * c[e] + u * t;
                const float t2 = SIGN * s[E / 2 + e], u2 = b[2 * e], v2 = b[2 * e + 1];
                b[2 * e] = u2 * c[E / 2 + e] - v2 * t2;
                b[2 * e + 1] = v2 * c[E / 2 + e] + u2 * t2;
            }
        }
    }
};

template <int E> __device__ __forceinline__ void load_weights(const float* w, int c0, int c1, float (&w0)[E], float (&w1)[E])
{
#pragma unroll
    for (int e = 0; e < E; ++e) w0[e] = w1[e] = 0.f;
    if (c0 >= 0) load_floats<E>(w + c0, w0);
    if (c1 >= 0) load_floats<E>(w + c1, w1);
}

// Rows whose chunks are asked for before the first of them is used: with one at a time 4.4 TB/s forward and 2.6 backward, with
// four, and angles and weights by vectors, 5.4 and 4.5 (bfloat16, 40 heads of 128 values; 32768 and 16384 tokens).
constexpr int kAhead = 4;

// L: lanes of a row; NT: results go past the caches
template <typename T, int E, int L, bool NT> __global__ __launch_bounds__(kThreads) void head_forward(const HeadArgs A)
{
    constexpr int G = kWave / L;
    const int lane = (int)threadIdx.x % kWave, p = lane % L, g = lane / L;
    const long long wave = workgroup() * (kThreads / kWave) + threadIdx.x / kWave;
    const long long token = wave / A.parts;
    const int part = (int)(wave - token * A.parts);
    if (token >= A.T) return;
    int c0, c1;
    chunks_of<E>(A, p, &c0, &c1);
    Turn<E> turn;
    turn.load(A, token, p, c0, c1);
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        if (part * G >= A.H[t]) continue;
        float w0[E], w1[E];
        load_weights<E>(A.w[t], c0, c1, w0, w1);
        const T* const x = static_cast<const T*>(A.x[t]) + token * A.ldx[t];
        T* const y = static_cast<T*>(A.out[t]) + token * A.ldo[t];
        const int stride = A.parts * G;
        for (int h0 = part * G + g; h0 < A.H[t]; h0 += kAhead * stride) {
            typename Chunk<T, E>::Raw ra[kAhead], rb[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int h = h0 + k * stride;
                if (h >= A.H[t]) continue;
                ra[k] = load_chunk<T, E>(x + (long long)h * A.D, c0);
                rb[k] = load_chunk<T, E>(x + (long long)h * A.D, c1);
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const int h = h0 + k * stride;
                if (h >= A.H[t]) continue;
                float a[E], b[E], s = 0.f;
                Chunk<T, E>::unpack(ra[k], a);
                Chunk<T, E>::unpack(rb[k], b);
#pragma unroll
                for (int e = 0; e < E; ++e) s += a[e] * a[e] + b[e] * b[e];
                const float r = 1.f / sqrtf(group_sum<L>(s) * A.inv_D + A.eps);
#pragma unroll
                for (int e = 0; e < E; ++e) { a[e] *= r * w0[e]; b[e] *= r * w1[e]; }
                turn.template apply<1>(A.style, a, b);
                if (c0 >= 0) Chunk<T, E>::template store<NT>(y + (long long)h * A.D + c0, a);
                if (c1 >= 0) Chunk<T, E>::template store<NT>(y + (long long)h * A.D + c1, b);
            }
        }
    }
}

// A workgroup's sums of dw, from the wavefronts' (LDS, [4][D]) to its row of `part`
__device__ __forceinline__ void store_dw(const HeadArgs& A, const float* red, int t)
{
    __syncthreads();
    for (int d = (int)threadIdx.x; d < A.D; d += kThreads)
        A.part[((long long)blockIdx.x * 2 + t) * A.D + d] = ((red[d] + red[A.D + d]) + red[2 * A.D + d]) + red[3 * A.D + d];
    __syncthreads();
}

template <typename T, int E, int L, bool NT> __global__ __launch_bounds__(kThreads, 2) void head_backward(const HeadArgs A)
{
    constexpr int G = kWave / L;
    extern __shared__ float red[];                    // [4][D]
    const int lane = (int)threadIdx.x % kWave, p = lane % L, g = lane / L, wave = (int)threadIdx.x / kWave;
    int c0, c1;
    chunks_of<E>(A, p, &c0, &c1);
    for (int t = 0; t < 2; ++t) {
        float w0[E], w1[E], dw0[E], dw1[E];
        load_weights<E>(A.w[t], A.H[t] ? c0 : -1, A.H[t] ? c1 : -1, w0, w1);
#pragma unroll
        for (int e = 0; e < E; ++e) dw0[e] = dw1[e] = 0.f;
        const long long waves = (long long)gridDim.x * (kThreads / kWave);
        for (long long u = (long long)blockIdx.x * (kThreads / kWave) + wave; u < A.T * A.parts; u += waves) {
            const long long token = u / A.parts;
            const int part = (int)(u - token * A.parts);
            if (part * G >= A.H[t]) continue;
            Turn<E> turn;
            turn.load(A, token, p, c0, c1);
            const T* const x = static_cast<const T*>(A.x[t]) + token * A.ldx[t];
            const T* const dy = static_cast<const T*>(A.dy[t]) + token * A.lddy[t];
            T* const dx = static_cast<T*>(A.out[t]) + token * A.ldo[t];
            const int stride = A.parts * G;
            for (int h0 = part * G + g; h0 < A.H[t]; h0 += kAhead * stride) {
                typename Chunk<T, E>::Raw ra[kAhead], rb[kAhead], rc[kAhead], rd[kAhead];
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int h = h0 + k * stride;
                    if (h >= A.H[t]) continue;
                    const long long o = (long long)h * A.D;
                    ra[k] = load_chunk<T, E>(x + o, c0);
                    rb[k] = load_chunk<T, E>(x + o, c1);
                    rc[k] = load_chunk<T, E>(dy + o, c0);
                    rd[k] = load_chunk<T, E>(dy + o, c1);
                }
#pragma unroll
                for (int k = 0; k < kAhead; ++k) {
                    const int h = h0 + k * stride;
                    if (h >= A.H[t]) continue;
                    float a[E], b[E], ea[E], eb[E], s = 0.f, m = 0.f;
                    Chunk<T, E>::unpack(ra[k], a);
                    Chunk<T, E>::unpack(rb[k], b);
                    Chunk<T, E>::unpack(rc[k], ea);
                    Chunk<T, E>::unpack(rd[k], eb);
                    turn.template apply<-1>(A.style, ea, eb);
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        s += a[e] * a[e] + b[e] * b[e];
                        m += ea[e] * w0[e] * a[e] + eb[e] * w1[e] * b[e];
                    }
                    const float r = 1.f / sqrtf(group_sum<L>(s) * A.inv_D + A.eps);
                    const float f = group_sum<L>(m) * r * r * A.inv_D;          // mean(t x r) r
#pragma unroll
                    for (int e = 0; e < E; ++e) {
                        dw0[e] += ea[e] * (a[e] * r);
                        dw1[e] += eb[e] * (b[e] * r);
                        a[e] = r * (ea[e] * w0[e] - a[e] * f);
                        b[e] = r * (eb[e] * w1[e] - b[e] * f);
                    }
                    if (c0 >= 0) Chunk<T, E>::template store<NT>(dx + (long long)h * A.D + c0, a);
                    if (c1 >= 0) Chunk<T, E>::template store<NT>(dx + (long long)h * A.D + c1, b);
                }
            }
        }
        // over the groups of the wavefront (fixed order), then over wavefronts
#pragma unroll
        for (int e = 0; e < E; ++e) {
#pragma unroll
            for (int o = L; o < kWave; o *= 2) { dw0[e] += __shfl_xor(dw0[e], o); dw1[e] += __shfl_xor(dw1[e], o); }
            if (g == 0 && c0 >= 0) red[wave * A.D + c0 + e] = dw0[e];
            if (g == 0 && c1 >= 0) red[wave * A.D + c1 + e] = dw1[e];
        }
        store_dw(A, red, t);
    }
}

// ---- one value a lane and step: any length, stride and alignment ----

constexpr int kMaxD = 1024;

// the value turned together with value d (R > d), whether d is the first of the two, and the angle's index
__device__ __forceinline__ int partner_of(const HeadArgs& A, int d, bool* is_first, int* angle)
{
    if (A.style == CGBN_ROTATE_HALVES) {
        const int half = A.R / 2;
        *is_first = d < half;
        *angle = d < half ? d : d - half;
        return d < half ? d + half : d - half;
    }
    *is_first = (d & 1) == 0;
    *angle = d / 2;
    return d ^ 1;
}

struct Angles {
    long long row;
    bool in;
    __device__ __forceinline__ Angles(const HeadArgs& A, long long token)
    {
        const long long pos = A.positions && A.R ? (long long)A.positions[token] : token;
        in = pos >= 0 && pos < A.table;
        row = in ? pos * (A.R / 2) : 0;
    }
    __device__ __forceinline__ float cos(const HeadArgs& A, int k) const { return in ? A.cos[row + k] : __int_as_float(0x7fc00000); }
    __device__ __forceinline__ float sin(const HeadArgs& A, int k) const { return in ? A.sin[row + k] : __int_as_float(0x7fc00000); }
};

// kSlots: values a lane
// in place (out == x) every value is read, partners too, before the row's first is written
template <typename T, int kSlots> __global__ __launch_bounds__(kThreads) void head_forward_any(const HeadArgs A)
{
    const int lane = (int)threadIdx.x % kWave, heads = A.H[0] + A.H[1];
    const long long row = workgroup() * (kThreads / kWave) + threadIdx.x / kWave;
    if (row >= A.T * heads) return;
    const long long token = row / heads;
    int h = (int)(row - token * heads);
    const int t = h >= A.H[0];
    if (t) h -= A.H[0];
    const T* x = static_cast<const T*>(A.x[t]) + token * A.ldx[t] + (long long)h * A.D;
    T* y = static_cast<T*>(A.out[t]) + token * A.ldo[t] + (long long)h * A.D;
    const Angles ang(A, token);
    float v[kSlots], s = 0.f;
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const int d = k * kWave + lane;
        v[k] = d < A.D ? Elem<T>::load1(x + d) : 0.f;
        s += v[k] * v[k];
    }
    const float r = 1.f / sqrtf(group_sum<kWave>(s) * A.inv_D + A.eps);
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const int d = k * kWave + lane;
        if (d >= A.D) continue;
        v[k] *= r * A.w[t][d];
        if (d < A.R) {
            bool first;
            int angle;
            const int o = partner_of(A, d, &first, &angle);
            const float other = Elem<T>::load1(x + o) * (r * A.w[t][o]), sn = ang.sin(A, angle);
            v[k] = v[k] * ang.cos(A, angle) + (first ? -other * sn : other * sn);
        }
    }
    // partners' values are in registers by now: the loads above feed the values that are stored, but those of other lanes
    // may still be on their way while this lane stores, so all of them are waited for
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int k = 0; k < kSlots; ++k) {
        const int d = k * kWave + lane;
        if (d < A.D) Elem<T>::store1(y + d, v[k]);
    }
}

template <typename T, int kSlots> __global__ __launch_bounds__(kThreads) void head_backward_any(const HeadArgs A)
{
    extern __shared__ float red[];                    // [4][D]
    const int lane = (int)threadIdx.x % kWave, wave = (int)threadIdx.x / kWave;
    const long long waves = (long long)gridDim.x * (kThreads / kWave);
    for (int t = 0; t < 2; ++t) {
        float dw[kSlots];
#pragma unroll
        for (int k = 0; k < kSlots; ++k) dw[k] = 0.f;
        for (long long row = (long long)blockIdx.x * (kThreads / kWave) + wave; row < A.T * A.H[t]; row += waves) {
            const long long token = row / A.H[t];
            const int h = (int)(row - token * A.H[t]);
            const T* x = static_cast<const T*>(A.x[t]) + token * A.ldx[t] + (long long)h * A.D;
            const T* dy = static_cast<const T*>(A.dy[t]) + token * A.lddy[t] + (long long)h * A.D;
            T* dx = static_cast<T*>(A.out[t]) + token * A.ldo[t] + (long long)h * A.D;
            const Angles ang(A, token);
            float v[kSlots], e[kSlots], s = 0.f, m = 0.f;
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const int d = k * kWave + lane;
                v[k] = e[k] = 0.f;
                if (d >= A.D) continue;
                v[k] = Elem<T>::load1(x + d);
                e[k] = Elem<T>::load1(dy + d);
                if (d < A.R) {
                    bool first;
                    int angle;
                    const int o = partner_of(A, d, &first, &angle);
                    const float other = Elem<T>::load1(dy + o), sn = ang.sin(A, angle);
                    e[k] = e[k] * ang.cos(A, angle) + (first ? other * sn : -other * sn);
                }
                s += v[k] * v[k];
                m += e[k] * A.w[t][d] * v[k];
            }
            const float r = 1.f / sqrtf(group_sum<kWave>(s) * A.inv_D + A.eps);
            const float f = group_sum<kWave>(m) * r * r * A.inv_D;
            asm volatile("s_waitcnt vmcnt(0)" ::: "memory");          // as above: dx may be dy
#pragma unroll
            for (int k = 0; k < kSlots; ++k) {
                const int d = k * kWave + lane;
                if (d >= A.D) continue;
                dw[k] += e[k] * (v[k] * r);
                Elem<T>::store1(dx + d, r * (e[k] * A.w[t][d] - v[k] * f));
            }
        }
#pragma unroll
        for (int k = 0; k < kSlots; ++k)
            if (k * kWave + lane < A.D) red[wave * A.D + k * kWave + lane] = dw[k];
        store_dw(A, red, t);
    }
}

// ---- host ----

cgbn_status launched() { return hipGetLastError() == hipSuccess ? CGBN_OK : CGBN_ERR_HIP; }

constexpr long long kMaxTokens = 1ll << 30, kMaxStride = 1ll << 32;
constexpr int kMaxHeads = 1 << 14;
constexpr int kBackwardGroups = 512;          // two workgroups a compute unit, all there at once: each ends with a row of sums

cgbn_status check_sizes(long long T, int Hq, int Hk, int D, int dtype)
{
    if (dtype != CGBN_F32 && dtype != CGBN_BF16) return CGBN_ERR_ENUM;
    if (T < 0 || T > kMaxTokens || Hq < 1 || Hq > kMaxHeads || Hk < 0 || Hk > kMaxHeads || D < 1 || D > kMaxD) return CGBN_ERR_SHAPE;
    if (T * (Hq + Hk) > (1ll << 33)) return CGBN_ERR_SHAPE;            // 2^31 workgroups at the most
    return CGBN_OK;
}

// workgroups of a backward call
int backward_groups(long long T, int Hq, int Hk)
{
    const long long rows = T * (Hq + Hk), groups = (rows + 15) / 16;   // (at least four rows a wavefront, but for the last)
    return (int)(groups < kBackwardGroups ? (groups < 1 ? 1 : groups) : kBackwardGroups);
}

// bytes of a backward call's partial sums
size_t partial_sums(long long T, int Hq, int Hk, int D) { return (size_t)backward_groups(T, Hq, Hk) * 2 * D * sizeof(float); }

// rows in chunks of E values
template <typename T> bool plan_chunks(HeadArgs* A, int E, bool backward)
{
    const size_t bytes = E * sizeof(T);
    if (A->D % E != 0) return false;
    for (int t = 0; t < (A->H[1] ? 2 : 1); ++t) {
        if (reinterpret_cast<uintptr_t>(A->x[t]) % bytes || reinterpret_cast<uintptr_t>(A->out[t]) % bytes || A->ldx[t] % E != 0 || A->ldo[t] % E != 0)
            return false;
        if (backward && (reinterpret_cast<uintptr_t>(A->dy[t]) % bytes || A->lddy[t] % E != 0)) return false;
    }
    const int chunks = A->D / E;
    A->lead = A->far = 0;
    A->step = 1;
    if (A->style == CGBN_ROTATE_HALVES && A->R) {
        if ((A->R / 2) % E != 0) return false;
        A->lead = A->far = A->R / 2 / E;
    } else if (E == 1 && A->R) {                // a pair is two chunks side by side
        A->lead = A->R / 2;
        A->step = 2;
        A->far = 1;
    }
    A->rest = chunks - 2 * A->lead;
    A->pairs = A->lead + (A->rest + 1) / 2;
    return A->pairs <= kWave;
}

// (rows in chunks of one or two values are no shorter than that: where one is, its lanes idle)
template <int E> int lanes_of(int pairs)
{
    int l = E <= 2 ? 16 : 1;
    while (l < pairs) l *= 2;
    return l;
}

#define CGBN_LANES(X_) X_(1) X_(2) X_(4) X_(8)
#define CGBN_LANES_LONG(X_) X_(16) X_(32) X_(64)

// a wavefront takes all heads of its token unless there are too few tokens to fill the device with
void deal_heads(HeadArgs* A, int G)
{
    const int most = ((A->H[0] > A->H[1] ? A->H[0] : A->H[1]) + G - 1) / G;
    A->parts = 1;
    while (A->parts < most && A->T * A->parts < 4096) A->parts *= 2;
    if (A->parts > most) A->parts = most;
}

template <typename T, int E, bool NT> void launch_forward(HeadArgs& A, hipStream_t st)
{
    const int L = lanes_of<E>(A.pairs);
    deal_heads(&A, kWave / L);
    const dim3 grid = grid_of((A.T * A.parts + 3) / 4);
#define CGBN_CASE(L_) \
    case L_: hipLaunchKernelGGL((head_forward<T, E, L_, NT>), grid, dim3(kThreads), 0, st, A); break;
    if constexpr (E <= 2) switch (L) { CGBN_LANES_LONG(CGBN_CASE) }
    else switch (L) { CGBN_LANES(CGBN_CASE) CGBN_LANES_LONG(CGBN_CASE) }
#undef CGBN_CASE
}

template <typename T, int E, bool NT> void launch_backward(HeadArgs& A, int groups, size_t lds, hipStream_t st)
{
    const int L = lanes_of<E>(A.pairs);
    deal_heads(&A, kWave / L);
#define CGBN_CASE(L_) \
    case L_: hipLaunchKernelGGL((head_backward<T, E, L_, NT>), dim3((unsigned)groups), dim3(kThreads), lds, st, A); break;
    if constexpr (E <= 2) switch (L) { CGBN_LANES_LONG(CGBN_CASE) }
    else switch (L) { CGBN_LANES(CGBN_CASE) CGBN_LANES_LONG(CGBN_CASE) }
#undef CGBN_CASE
}

#define CGBN_ANY(kernel_, grid_, lds_)                                                                                 \
    do {                                                                                                               \
        const dim3 g_ = grid_;                                                                                         \
        if (A.D <= 64) hipLaunchKernelGGL((kernel_<T, 1>), g_, dim3(kThreads), lds_, st, A);                           \
        else if (A.D <= 128) hipLaunchKernelGGL((kernel_<T, 2>), g_, dim3(kThreads), lds_, st, A);                     \
        else if (A.D <= 256) hipLaunchKernelGGL((kernel_<T, 4>), g_, dim3(kThreads), lds_, st, A);                     \
        else hipLaunchKernelGGL((kernel_<T, kMaxD / kWave>), g_, dim3(kThreads), lds_, st, A);                         \
    } while (0)

// Results of more than the caches next to the compute units hold go past them: 119 against 127 us, backward 106 against 112 (40 heads of
// 128 bfloat16; 32768 and 16384 tokens); smaller ones stay there for whoever reads them next.  Not from chunks of 8 bytes: 65 us through
// the caches, 72 past them (5845 tokens, 144 heads of 80).
template <typename T> bool past_caches(const HeadArgs& A) { return (double)A.T * (A.H[0] + A.H[1]) * A.D * sizeof(T) > 32e6; }

template <typename T> cgbn_status run_forward(HeadArgs& A, hipStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    if (plan_chunks<T>(&A, E, false)) past_caches<T>(A) ? launch_forward<T, E, true>(A, st) : launch_forward<T, E, false>(A, st);
    else if (sizeof(T) == 2 && plan_chunks<T>(&A, 4, false)) launch_forward<T, 4, false>(A, st);
    else if (plan_chunks<T>(&A, 2, false)) launch_forward<T, 2, false>(A, st);
    else if (plan_chunks<T>(&A, 1, false)) launch_forward<T, 1, false>(A, st);
    else CGBN_ANY(head_forward_any, grid_of((A.T * (A.H[0] + A.H[1]) + 3) / 4), 0);
    return launched();
}

template <typename T> cgbn_status run_backward(HeadArgs& A, float* dwq, float* dwk, hipStream_t st)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int groups = backward_groups(A.T, A.H[0], A.H[1]);
    const size_t lds = (size_t)4 * A.D * sizeof(float);
    if (plan_chunks<T>(&A, E, true)) past_caches<T>(A) ? launch_backward<T, E, true>(A, groups, lds, st) : launch_backward<T, E, false>(A, groups, lds, st);
    else if (sizeof(T) == 2 && plan_chunks<T>(&A, 4, true)) launch_backward<T, 4, false>(A, groups, lds, st);
    else if (plan_chunks<T>(&A, 2, true)) launch_backward<T, 2, false>(A, groups, lds, st);
    else if (plan_chunks<T>(&A, 1, true)) launch_backward<T, 1, false>(A, groups, lds, st);
    else CGBN_ANY(head_backward_any, dim3((unsigned)groups), lds);
    if (launched() != CGBN_OK) return CGBN_ERR_HIP;
    const int n = A.H[1] ? 2 * A.D : A.D;
    // (a workgroup's row of partial sums has both weights' side by side; without keys the second half is zero and stays unread)
    hipLaunchKernelGGL(column_sums, dim3((unsigned)((n + 15) / 16)), dim3(kSumThreads), 0, st, A.part, groups, 2 * A.D, n, dwq, A.D, dwk);
    return launched();
}

cgbn_status check_call(const HeadArgs& A, cgbn_dtype dtype, cgbn_rotation style, bool backward)
{
    const cgbn_status s = check_sizes(A.T, A.H[0], A.H[1], A.D, dtype);
    if (s != CGBN_OK) return s;
    if (style != CGBN_ROTATE_HALVES && style != CGBN_ROTATE_PAIRS) return CGBN_ERR_ACTIVATION;
    if (A.R < 0 || A.R > A.D || A.R % 2 != 0 || (A.R && A.table < 1)) return CGBN_ERR_SHAPE;
    if (!(A.eps > 0.f) || std::isinf(A.eps)) return CGBN_ERR_EPS;
    if (A.R && A.T && (!A.cos || !A.sin)) return CGBN_ERR_NULL;
    const size_t elem = dtype == CGBN_F32 ? 4 : 2;
    for (int t = 0; t < (A.H[1] ? 2 : 1); ++t) {
        if (!A.w[t] || (A.T && (!A.x[t] || !A.out[t] || (backward && !A.dy[t])))) return CGBN_ERR_NULL;
        const long long width = (long long)A.H[t] * A.D;
        if (A.ldx[t] > kMaxStride || A.ldo[t] > kMaxStride || (backward && A.lddy[t] > kMaxStride)) return CGBN_ERR_SHAPE;
        if (A.T > 1 && (A.ldx[t] < width || A.ldo[t] < width || (backward && A.lddy[t] < width))) return CGBN_ERR_STRIDE;
        if (reinterpret_cast<uintptr_t>(A.x[t]) % elem || reinterpret_cast<uintptr_t>(A.out[t]) % elem ||
            (backward && reinterpret_cast<uintptr_t>(A.dy[t]) % elem))
            return CGBN_ERR_ALIGN;
        // in place: row for row
        const void* in = backward ? A.dy[t] : A.x[t];
        const long long ld = backward ? A.lddy[t] : A.ldx[t];
        if (A.T && A.out[t] == in && A.T > 1 && A.ldo[t] != ld) return CGBN_ERR_ALIAS;
        if (A.T && backward && A.out[t] == A.x[t] && A.T > 1 && A.ldo[t] != A.ldx[t]) return CGBN_ERR_ALIAS;
    }
    if (A.T && A.H[1]) {
        if (A.out[0] == A.out[1]) return CGBN_ERR_ALIAS;
        // the one's results over what the other's come from
        for (int t = 0; t < 2; ++t)
            if (A.out[t] == A.x[1 - t] || (backward && A.out[t] == A.dy[1 - t])) return CGBN_ERR_ALIAS;
    }
    for (int t = 0; A.T && t < (A.H[1] ? 2 : 1); ++t) {
        const void* const out = A.out[t];
        if (out == A.w[0] || (A.H[1] && out == A.w[1]) || (A.R && (out == A.cos || out == A.sin || (A.positions && out == A.positions))))
            return CGBN_ERR_ALIAS;
    }
    return CGBN_OK;
}

}  // namespace
}  // namespace cgbn

using namespace cgbn;

extern "C" {

cgbn_status cgbn_head_norm_forward(const void* q, long long ldq, const void* k, long long ldk, long long T, int Hq, int Hk, int D, int R,
                                   cgbn_rotation style, const int* positions, const float* cos, const float* sin, int table_rows, const float* wq,
                                   const float* wk, float eps, void* yq, long long ldyq, void* yk, long long ldyk, cgbn_dtype dtype, void* stream)
{
    HeadArgs A;
    std::memset(&A, 0, sizeof(A));
    A.x[0] = q; A.x[1] = k; A.out[0] = yq; A.out[1] = yk;
    A.ldx[0] = ldq; A.ldx[1] = ldk; A.ldo[0] = ldyq; A.ldo[1] = ldyk;
    A.w[0] = wq; A.w[1] = wk; A.cos = cos; A.sin = sin; A.positions = positions;
    A.T = T; A.H[0] = Hq; A.H[1] = Hk; A.D = D; A.R = R; A.table = table_rows; A.style = style; A.eps = eps;
    const cgbn_status s = check_call(A, dtype, style, false);
    if (s != CGBN_OK || T == 0) return s;
    A.inv_D = 1.f / (float)D;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == CGBN_F32 ? run_forward<float>(A, st) : run_forward<bf16_t>(A, st);
}

size_t cgbn_head_norm_workspace_bytes(long long T, int Hq, int Hk, int D, cgbn_dtype dtype)
{
    if (check_sizes(T, Hq, Hk, D, dtype) != CGBN_OK) return 0;
    const size_t bytes = (partial_sums(T, Hq, Hk, D) + 255) / 256 * 256;
    return bytes > 256 ? bytes : 512;          // (of 256 or less a program may pass none)
}

cgbn_status cgbn_head_norm_backward(const void* dyq, long long lddyq, const void* dyk, long long lddyk, const void* q, long long ldq, const void* k,
                                    long long ldk, long long T, int Hq, int Hk, int D, int R, cgbn_rotation style, const int* positions,
                                    const float* cos, const float* sin, int table_rows, const float* wq, const float* wk, float eps, void* dq,
                                    long long lddq, void* dk, long long lddk, float* dwq, float* dwk, cgbn_dtype dtype, void* workspace,
                                    size_t workspace_bytes, void* stream)
{
    HeadArgs A;
    std::memset(&A, 0, sizeof(A));
    A.x[0] = q; A.x[1] = k; A.dy[0] = dyq; A.dy[1] = dyk; A.out[0] = dq; A.out[1] = dk;
    A.ldx[0] = ldq; A.ldx[1] = ldk; A.lddy[0] = lddyq; A.lddy[1] = lddyk; A.ldo[0] = lddq; A.ldo[1] = lddk;
    A.w[0] = wq; A.w[1] = wk; A.cos = cos; A.sin = sin; A.positions = positions;
    A.T = T; A.H[0] = Hq; A.H[1] = Hk; A.D = D; A.R = R; A.table = table_rows; A.style = style; A.eps = eps;
    const cgbn_status s = check_call(A, dtype, style, true);
    if (s != CGBN_OK) return s;
    if (!dwq || (Hk && !dwk)) return CGBN_ERR_NULL;
    if (dwq == dwk) return CGBN_ERR_ALIAS;
    for (int t = 0; T && t < (Hk ? 2 : 1); ++t)
        if (A.out[t] == dwq || (Hk && A.out[t] == dwk)) return CGBN_ERR_ALIAS;
    const size_t need = partial_sums(T, Hq, Hk, D);
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need) return CGBN_ERR_WORKSPACE;
    A.part = static_cast<float*>(workspace);
    A.inv_D = 1.f / (float)D;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == CGBN_F32 ? run_backward<float>(A, dwq, dwk, st) : run_backward<bf16_t>(A, dwq, dwk, st);
}

}  // extern "C"
