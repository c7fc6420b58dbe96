// Matrix products of libcgbn for gfx950: C[i][j] = sum over r of A(i, r) B(j, r), on the matrix cores, with bias, residual,
// activation or a gated product applied to the accumulators before they are rounded and stored.
//
// An operand lies in memory either with its reduction index innermost ("rows": p[i * ld + r]) or outermost ("columns":
// p[r * ld + i]).  Three forms serve a layer:
//   FORM_NT  rows x rows        z  = x W^T          (forward)
//   FORM_NN  rows x columns     dx = dz W
//   FORM_TN  columns x columns  dW = dz^T x
//
// A workgroup owns a BI x BJ tile of C in its accumulator registers and walks the reduction in steps of 128 bytes of r (64
// bfloat16, 32 float), two steps' operands in LDS: while one is multiplied the next travels from memory to LDS directly, 16
// bytes a lane, without passing registers.  Such a load writes its wavefront's lanes side by side, so bank conflicts cannot be
// avoided by padding; instead each lane fetches another 16-byte chunk of its row (chunk index xor a key of the row, `row_key`,
// `col_key`) and the readers apply the same xor.  "Rows" operands are read back as 16-byte fragments; "columns" operands of
// bfloat16 by the LDS reads that transpose 4 x 16 blocks, so no operand is ever transposed in memory.
//
// The product is formed as C^T (B is the matrix instruction's first operand), so that a lane's four accumulators are
// neighbours in a row of C.
//
// What bounds it: long reductions the matrix cores (8192 x 8192 x 8192 bfloat16 772 us, 1425 TF; they are busy 65% of the gated product of
// 8192 x 4096 x 14336, 1430 us, 1345 TF); short ones with wide results the results' way to memory (16384 x 2048 x 8192 with z kept 518 us, 1061 TF and
// 537 MB written; 67200 x 256 x 1024 with a residual 93.5 us, 3.3 TB/s, the matrix cores busy 15%).  Tiles of 256 x 256 read the least from
// LDS for each product, but fill a compute unit alone, so that nothing is multiplied while their results leave; smaller ones run side by
// side.  No bank conflicts (counted).  Float, three bfloat16 parts a value: 8192 x 8192 x 2048 1382 us, 199 TF, 12544-long 512 x 1024 87 us, 152 TF.
//
// Sums are held in 32 bits throughout.  Where tiles are too few for 256 compute units the reduction is split and the partial
// sums, float, are joined by gemm_join in split order: results never depend on the order in which workgroups end.
#pragma once

#include "cgbn_kernels.h"

#include <type_traits>

namespace cgbn {

enum { FORM_NT = 0, FORM_NN = 1, FORM_TN = 2 };
enum { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_SILU = 3 };

struct GemmArgs {
    const void* A[2];           // second entries: the second segment of the reduction, or the second product of a batch
    const void* B[2];           // gated: the two weight matrices
    void* C[2];                 // gated: h
    void* Z[2];                 // linear: z or null in [0]; gated: gate, up or null
    const float* bias;          // may be null
    const void* residual;       // may be null
    float* part;                // partial sums of a split reduction
    long long lda, ldb, ldc;    // elements from row to row
    int I, J, R;                // R: up to a multiple of 16 bytes where an operand is in rows (the filling is zero)
    int segs, batch;            // segments of the reduction; products side by side
    int ti, tj, splits, per;    // tiles; splits of the reduction and steps (of 128 bytes) in each
    int act;
    int nt;                     // results go past the caches
};

// ---- activations, on 32-bit values ----
//
// FINE: for float results, which show what the shorter forms leave out.  Those are for bfloat16, at most 2.7e-7 off (GELU, near zero).

// exp(x): the hardware's 2^y
__device__ __forceinline__ float exp_of(float x) { return __builtin_amdgcn_exp2f(x * 1.4426950408889634f); }

// exp(x) with what is lost of the product, and of log2(e), made good; x within [-150, 100], beyond which it is 0 and infinity
__device__ __forceinline__ float exp_fine(float x)
{
    x = __builtin_amdgcn_fmed3f(x, -150.f, 100.f);
    const float y = x * 1.4426950408889634f, lost = fmaf(x, 1.9259629911266175e-8f, fmaf(x, 1.4426950408889634f, -y));
    return __builtin_amdgcn_exp2f(y) * fmaf(lost, 0.6931471805599453f, 1.f);
}

// exp(-z^2 / 2)
template <bool FINE> __device__ __forceinline__ float bell(float z)
{
    if constexpr (!FINE) return __builtin_amdgcn_exp2f(z * z * -0.72134752044448170f);
    z = fminf(fabsf(z), 30.f);
    const float s = z * z, y = s * -0.72134752044448170f;
    const float lost = fmaf(fmaf(z, z, -s), -0.72134752044448170f, fmaf(s, -9.629814955633087e-9f, fmaf(s, -0.72134752044448170f, -y)));
    return __builtin_amdgcn_exp2f(y) * fmaf(lost, 0.6931471805599453f, 1.f);
}

// Phi(-|z|), e being exp(-z^2 / 2).  Short: the rational approximation of the complementary error function that Abramowitz and Stegun give as
// 7.1.26 (after Hastings).  It counts: an epilogue is bound by its instructions, 14 a value for GELU, 40 us of 520 at 16384 x 2048 x 8192 (the
// library's erff cost about three times as much).  Fine: of the same form, t = 1 / (1 + 0.35 |z|), a polynomial of degree 8 fitted to Phi(-z) / (e t) over z in
// [0, 14] for the least largest relative error, 3.2e-8; evaluated in 32 bits it is off by 7 units of 2^-24 of itself.
template <bool FINE> __device__ __forceinline__ float normal_tail(float z, float e)
{
    if constexpr (!FINE) {
        const float t = __builtin_amdgcn_rcpf(fmaf(0.23164189f, fabsf(z), 1.f));         // 0.3275911 / sqrt(2)
        return e * (t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 0.5307027145f, -0.7265760135f), 0.7107068705f), -0.142248368f), 0.127414796f));
    }
    const float t = __builtin_amdgcn_rcpf(fmaf(0.35f, fminf(fabsf(z), 30.f), 1.f));
    constexpr float c[9] = {0.13962140679359436f, 0.13986186683177948f, 0.11983287334442139f, 0.1055079847574234f, -0.023109780624508858f,
                            0.1591740846633911f, -0.25571417808532715f, 0.14397166669368744f, -0.029145922511816025f};
    float p = c[8];
#pragma unroll
    for (int k = 7; k >= 0; --k) p = fmaf(t, p, c[k]);
    return e * (t * p);
}

template <bool FINE> __device__ __forceinline__ float act_apply(float z, int act)
{
    if (act == ACT_RELU) return z < 0.f ? 0.f : z;
    // z Phi(z), which is z - z Phi(-z); the positive part by its bits, as an integer (where z is NaN the other term is).  Where z is large the tail is
    // zero, and what it is multiplied by is kept finite, by its bits too, for an infinite z.
    if (act == ACT_GELU) {
        const float finite = FINE ? (z > 1e30f ? 1e30f : z) : __int_as_float(min(__float_as_int(z), 0x7149f2ca));
        return fmaf(-fabsf(finite), normal_tail<FINE>(z, bell<FINE>(z)), __int_as_float(max(__float_as_int(z), 0)));
    }
    if (act == ACT_SILU) return FINE ? z / (1.f + exp_fine(-z)) : z * __builtin_amdgcn_rcpf(1.f + exp_of(-z));
    return z;
}

// act'(z)
template <bool FINE> __device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (act == ACT_GELU) {
        const float e = bell<FINE>(z);
        const float p = normal_tail<FINE>(z, e);
        return (z < 0.f ? p : 1.f - p) + z * 0.39894228040143268f * e;
    }
    if (act == ACT_SILU) {
        if constexpr (FINE) {
            // (1 - s is e s: where z is positive the difference would lose its bits)
            const float e = exp_fine(-z), s = 1.f / (1.f + e);
            return fmaf(z * s, z > 0.f ? e * s : 1.f - s, s);
        }
        const float s = __builtin_amdgcn_rcpf(1.f + exp_of(-z));
        return s + z * s * (1.f - s);
    }
    return 1.f;
}

// ---- runs of neighbouring values, of which `valid` lie within the row ----

// 16 and 8 bytes at any address that a value can have: rows of odd lengths start anywhere, and the memory instructions take that
typedef u32x4 u32x4_any __attribute__((aligned(2)));
typedef uint32_t u32x2_any __attribute__((ext_vector_type(2), aligned(2)));

// a whole 16 bytes
template <typename T> __device__ __forceinline__ void unpack_run(const u32x4 w, float (&v)[16 / sizeof(T)])
{
    if constexpr (sizeof(T) == 2) Elem<T>::unpack(w, v);
    else Elem<T>::unpack(__builtin_bit_cast(f32x4, w), v);
}

// 16 bytes that are read once
template <typename T> __device__ __forceinline__ u32x4 load_once(const T* p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4_any*>(p)); }

template <typename T, int N> __device__ __forceinline__ void load_run(const T* p, float (&v)[N], int valid)
{
    constexpr int V = Elem<T>::VEC;
    if (valid >= N && N >= 4) {
        if constexpr (N % V == 0) {
#pragma unroll
            for (int k = 0; k < N; k += V) {
                float t[V];
                unpack_run<T>(*reinterpret_cast<const u32x4_any*>(p + k), t);
#pragma unroll
                for (int e = 0; e < V; ++e) v[k + e] = t[e];
            }
        } else if constexpr (N == 4) {                 // 4 bfloat16
            const u32x2_any w = *reinterpret_cast<const u32x2_any*>(p);
            v[0] = __uint_as_float(w.x << 16); v[1] = __uint_as_float(w.x & 0xffff0000u);
            v[2] = __uint_as_float(w.y << 16); v[3] = __uint_as_float(w.y & 0xffff0000u);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = k < valid ? Elem<T>::load1(p + k) : 0.f;
    }
}

// NT: past the caches (a choice of the compiler's, not of the program's: of two stores under a condition it makes one without)
template <typename T, int N, bool NT = false> __device__ __forceinline__ void store_run(T* p, const float (&v)[N], int valid)
{
    constexpr int V = Elem<T>::VEC;
    if (valid >= N && N >= 4) {
        if constexpr (N % V == 0) {
#pragma unroll
            for (int k = 0; k < N; k += V) {
                u32x4 w;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (sizeof(T) == 2) w[e] = f32x2_to_bf16x2(v[k + 2 * e], v[k + 2 * e + 1]);
                    else w[e] = __float_as_uint(v[k + e]);
                }
                if constexpr (NT) __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any*>(p + k));
                else *reinterpret_cast<u32x4_any*>(p + k) = w;
            }
        } else if constexpr (N == 4) {
            u32x2_any w;
            w.x = f32x2_to_bf16x2(v[0], v[1]);
            w.y = f32x2_to_bf16x2(v[2], v[3]);
            *reinterpret_cast<u32x2_any*>(p) = w;
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k)
            if (k < valid) Elem<T>::store1(p + k, v[k]);
    }
}

// ---- memory to LDS ----

// 16 bytes a lane from base + off to LDS at `lds` + 16 * lane.  Written out because the compiler, which cannot tell the two
// halves of the buffer apart, would have every LDS read wait for the loads in flight into the other half.  No register is
// written but m0, which the compiler reserves: it writes it before each use of its own and keeps nothing in it (nor does it take it for a clobber).
// dma_wait_and_meet() below makes the bytes visible.  The wait state is what the load needs after m0 is written.  Five are needed after the VECTOR unit
// has written a scalar of the address, where a spilled one is brought back, say; waited for here, in every load, that is 2% of a product
// (8192 x 8192 x 8192 774 and 794 us).  No kernel does so: tests/test_product_code.py reads it from their code.
__device__ __forceinline__ void dma16(uint32_t lds, const char* base, uint32_t off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
// every load of this wavefront has landed, every LDS read of it has returned; then the workgroup meets
__device__ __forceinline__ void dma_wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_hw __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// xor key of a row of an operand in rows (8 chunks of 16 bytes a row): the rows that a fragment read touches at once spread over all banks
__device__ __forceinline__ int row_key(int row) { return row & 7; }

// xor key, in 16-byte chunks, of a row of an operand in columns with CR chunks a row
template <typename T, int CR> __device__ __forceinline__ int col_key(int row)
{
    if constexpr (sizeof(T) == 2)
        return CR >= 16 ? ((row & 3) | ((row >> 3) & 1) << 2) << 1 : (((row >> 1) & 1) | ((row >> 3) & 1) << 1) << 1;
    else
        return ((row >> 2) & 3) << 2;
}

// One operand's share of a step: ROWS (of i or j) x 128 bytes of r, staged by NT threads.
template <typename T, bool COLS, int ROWS, int NT, bool PAIR> struct Operand {
    static constexpr int E = 16 / (int)sizeof(T);           // elements of a chunk
    static constexpr int STEP = 128 / (int)sizeof(T);       // r of a step
    static constexpr int CR = COLS ? ROWS / E : 8;          // chunks of a row of the tile in LDS
    static constexpr int BYTES = ROWS * 128;
    static constexpr int IT = BYTES / 16 / NT;
    static constexpr int HALF = ROWS / 2;
    static_assert(BYTES % (16 * NT) == 0, "whole passes");
    static_assert(!PAIR || HALF % (NT / 8) == 0, "a pass stays within one of the two matrices");

    uint32_t off[IT];

    // row of the tile in LDS and chunk of that row's data that this thread fetches in pass `it`
    static __device__ __forceinline__ int row_of(int it) { return (it * NT + (int)threadIdx.x) / CR; }
    static __device__ __forceinline__ int chunk_of(int it)
    {
        const int slot = (it * NT + (int)threadIdx.x) % CR;
        if constexpr (COLS) return slot ^ col_key<T, CR>(row_of(it));
        else return slot ^ row_key(row_of(it));
    }
    // first: the tile's first i; n: how many there are (rows and chunks beyond are read at the last one: results unused)
    __device__ __forceinline__ void init(int first, int n, long long ld)
    {
#pragma unroll
        for (int it = 0; it < IT; ++it) {
            if constexpr (COLS) {
                const int c = min(first / E + chunk_of(it), (n + E - 1) / E - 1) - first / E;
                off[it] = (uint32_t)(row_of(it) * ld * (int)sizeof(T)) + c * 16;
            } else {
                const int r = PAIR ? row_of(it) % HALF : row_of(it);
                off[it] = (uint32_t)((min(first + r, n - 1) - first) * ld * (int)sizeof(T)) + chunk_of(it) * 16;
            }
        }
    }
    static __device__ __forceinline__ const char* at(const void* p, int first, int step, long long ld)
    {
        return static_cast<const char*>(p) + (COLS ? (long long)step * STEP * ld + first : (long long)first * ld + (long long)step * STEP) * (int)sizeof(T);
    }
    // bytes from one step to the next
    static __device__ __forceinline__ long long advance(long long ld) { return COLS ? STEP * ld * (int)sizeof(T) : 128; }
    // Pass `it` of a step whose data starts at b0 (gated: of the second matrix at b1); lds: where the wavefront's share of the tile goes.
    __device__ __forceinline__ void pass(int it, uint32_t lds, const char* b0, const char* b1) const
    {
        dma16(lds + it * NT * 16, PAIR && it * (NT / 8) >= HALF ? b1 : b0, off[it]);
    }
    // ... with only `left` r of the operand remaining: zeros for what lies beyond (a lane that is switched off leaves its 16
    // bytes of LDS alone)
    __device__ __forceinline__ void last_pass(int it, uint32_t lds, lds_char* tile, const char* b0, const char* b1, int left) const
    {
        if ((COLS ? row_of(it) : chunk_of(it) * E) < left) pass(it, lds, b0, b1);
        else *reinterpret_cast<__attribute__((address_space(3))) u32x4*>(tile + (it * NT + (int)threadIdx.x) * 16) = u32x4{0, 0, 0, 0};
    }
};

// A fragment: 16 rows of i x 16 bytes of r a lane, that is lane l holds row l % 16 and chunk 4 * ks + l / 16 of the step.
// (bfloat16: what one matrix instruction takes; float: four of them, r being dealt to them in the same way on both sides.)
// base: the first of the rows that are walked, within the tile; f: which of their fragments.
template <typename T, bool COLS, int ROWS>
__device__ __forceinline__ u32x4 fragment(const lds_char* tile, int base, int f, int ks)
{
    const int l = (int)threadIdx.x % kWave, t = l & 15, q = l >> 4;
    if constexpr (!COLS) {
        const int row = base + f * 16 + t;
        return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + row * 128 + (((ks * 4 + q) ^ row_key(row)) << 4));
    } else {
        constexpr int RB = ROWS * (int)sizeof(T), CR = RB / 16;
        if constexpr (sizeof(T) == 2) {
            const int row = ks * 32 + q * 8 + (t >> 2), chunk = (base + f * 16) / 8;
            const lds_char* p = tile + row * RB + ((chunk ^ col_key<T, CR>(row)) << 4) + (t & 3) * 8;
            // (the key of row + 4 is that of row where CR >= 16, and otherwise too: it takes bits 0, 1 and 3 of the row)
            typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p);
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 4 * RB));
            const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
            return u32x4{a.x, a.y, b.x, b.y};
        } else {
            const int row = 4 * (4 * ks + q), chunk = (base + f * 16) / 4 + (t >> 2);
            const lds_char* p = tile + row * RB + ((chunk ^ col_key<T, CR>(row)) << 4) + (t & 3) * 4;
            typedef const __attribute__((address_space(3))) uint32_t lds_u32;
            return u32x4{*(lds_u32*)p, *(lds_u32*)(p + RB), *(lds_u32*)(p + 2 * RB), *(lds_u32*)(p + 3 * RB)};
        }
    }
}

template <typename T> __device__ __forceinline__ f32x4 multiply(const u32x4& a, const u32x4& b, f32x4 c)
{
    if constexpr (sizeof(T) == 2) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_hw, a), __builtin_bit_cast(bf16x8_hw, b), c, 0, 0, 0);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
        return c;
    }
}

// Float values as sums of three bfloat16, which is exact: the first is cut off (rounded, the type's largest values would become infinities), the second
// is what is left rounded to nearest, so that the third has either sign and what a product drops no preferred one.
// (Parts below the smallest normal number are lost: values under 1e-33 have fewer than 24 bits.)  8 values of a lane, from two chunks.
// QUIET: a NaN whose upper half alone would be an infinity stays a NaN: the bit that makes it quiet is in the upper half.
template <bool QUIET> __device__ __forceinline__ void split_float(const u32x4& lo, const u32x4& hi, u32x4 (&part)[3])
{
    auto value = [](uint32_t v) { return QUIET ? __builtin_canonicalizef(__uint_as_float(v)) : __uint_as_float(v); };
    auto upper = [](float v) { return __uint_as_float(__float_as_uint(v) & 0xffff0000u); };
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const float x = value(k < 2 ? lo[2 * k] : hi[2 * k - 4]), y = value(k < 2 ? lo[2 * k + 1] : hi[2 * k - 3]);
        const float xr = x - upper(x), yr = y - upper(y);
        const uint32_t mid = f32x2_to_bf16x2(xr, yr);
        const float xs = xr - __uint_as_float(mid << 16), ys = yr - __uint_as_float(mid & 0xffff0000u);
        part[0][k] = __builtin_amdgcn_perm(__float_as_uint(y), __float_as_uint(x), 0x07060302);           // the upper halves of both
        part[1][k] = mid;
        part[2][k] = __builtin_amdgcn_perm(__float_as_uint(ys), __float_as_uint(xs), 0x07060302);
    }
}

// Which tile a workgroup takes.  Consecutive workgroups go to the 8 dies in turn, so each die is given a run of consecutive
// work of its own; within it tiles go in blocks of 8 rows of tiles, column by column, so that the ones in flight at a time share operands in
// the die's L2.
struct TileId { int i, j, split, z; };
__device__ __forceinline__ TileId tile_of(const GemmArgs& G, int id, int n)
{
    const int die = id & 7, q = n >> 3, r = n & 7;
    int w = (die < r ? die * (q + 1) : r * (q + 1) + (die - r) * q) + (id >> 3);
    TileId t;
    const int tiles = G.ti * G.tj;
    t.z = w / (tiles * G.splits);
    w -= t.z * tiles * G.splits;
    t.split = w / tiles;
    w -= t.split * tiles;
    const int band = w / (8 * G.tj), rows = min(8, G.ti - band * 8);
    w -= band * 8 * G.tj;
    t.j = w / rows;
    t.i = band * 8 + (w - t.j * rows);
    return t;
}

// ---- epilogues: a run of N neighbours of a row ----

template <bool FINE, int N> __device__ __forceinline__ void activate(float (&v)[N], int act)
{
#define CGBN_ACTIVATE(act_)                                   \
    if (act == act_) {                                        \
        _Pragma("unroll") for (int k = 0; k < N; ++k) v[k] = act_apply<FINE>(v[k], act_); \
    }
    CGBN_ACTIVATE(ACT_RELU)
    CGBN_ACTIVATE(ACT_GELU)
    CGBN_ACTIVATE(ACT_SILU)
#undef CGBN_ACTIVATE
}

// v: the products; r: bias and residual.  o: the run's first element in the outputs
template <typename T, int N, bool NT = false>
__device__ __forceinline__ void finish_linear(const GemmArgs& G, float (&v)[N], const float (&r)[N], long long o, int valid)
{
    if (G.bias || G.residual) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += r[k];
    }
    if (G.Z[0]) store_run<T, N, NT>(static_cast<T*>(G.Z[0]) + o, v, valid);
    activate<sizeof(T) == 4>(v, G.act);
    store_run<T, N, NT>(static_cast<T*>(G.C[0]) + o, v, valid);
}

// what finish_linear adds
template <int N> __device__ __forceinline__ void load_bias(const GemmArgs& G, float (&b)[N], int j, int valid)
{
#pragma unroll
    for (int k = 0; k < N; ++k) b[k] = G.bias && k < valid ? G.bias[j + k] : 0.f;
}
template <typename T, int N> __device__ __forceinline__ void load_extras(const GemmArgs& G, float (&r)[N], const float (&b)[N], long long o, int valid)
{
    if (G.residual) {
        load_run<T, N>(static_cast<const T*>(G.residual) + o, r, valid);
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] += b[k];
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) r[k] = b[k];
    }
}

template <typename T, int N, bool NT = false> __device__ __forceinline__ void finish_gated(const GemmArgs& G, float (&g)[N], const float (&u)[N], long long o, int valid)
{
    if (G.Z[0]) {
        store_run<T, N, NT>(static_cast<T*>(G.Z[0]) + o, g, valid);
        store_run<T, N, NT>(static_cast<T*>(G.Z[1]) + o, u, valid);
    }
    activate<sizeof(T) == 4>(g, G.act);
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] *= u[k];
    store_run<T, N, NT>(static_cast<T*>(G.C[0]) + o, g, valid);
}

// ---- the product ----

// (float: and a word of each wavefront)
constexpr int tile_lds(int bi, int bj, int elem) { return 2 * (bi + bj) * 128 + (elem == 4 ? 16 : 0); }
// wavefronts that a vector unit must have registers for, by the values that one accumulates
constexpr int tile_waves(int values) { return values > 96 * 64 ? 1 : 2; }

// One workgroup's share, number `id` of `n`.  EARLY: see below
constexpr bool early_fits(int ti, int tj, int elem) { return ti * tj * elem / kWave <= 128; }
template <typename T, int FORM, bool GATED, int BI, int BJ, int WI, int WJ, bool EARLY = FORM == FORM_NT && !GATED && early_fits(BI / WI, BJ / WJ, sizeof(T))>
__device__ __forceinline__ void tile_product(const GemmArgs& G, char* lds, int id, int n)
{
    constexpr int NT = WI * WJ * kWave, TI = BI / WI, FI = TI / 16, TJ = BJ / WJ, FJ = TJ / 16;
    constexpr bool ACOLS = FORM == FORM_TN, BCOLS = FORM != FORM_NT;
    typedef Operand<T, ACOLS, BI, NT, false> OA;
    typedef Operand<T, BCOLS, BJ, NT, GATED> OB;
    constexpr int STAGE = OA::BYTES + OB::BYTES;
    static_assert(2 * STAGE == tile_lds(BI, BJ, 2) && WI * WJ <= 4, "two steps");
    lds_char* const tile = (lds_char*)lds;
    const uint32_t lds0 = (uint32_t)(uintptr_t)tile;

    const TileId w = tile_of(G, id, n);
    const int i0 = w.i * BI, j0 = w.j * (GATED ? BJ / 2 : BJ);
    OA a;
    OB b;
    a.init(i0, G.I, G.lda);
    b.init(j0, G.J, G.ldb);
    const int seg_steps = (G.R + OA::STEP - 1) / OA::STEP;
    const int first = w.split * G.per, last = min(first + G.per, seg_steps * G.segs);

    // The next step to be staged: where its data starts, and the r that remain in its segment.
    int seg, left;
    const char *pa, *pb, *pb2;
    auto from_the_first = [&] {
        seg = first >= seg_steps;
        left = G.R - (first - seg * seg_steps) * OA::STEP;
        pa = OA::at(G.A[seg + w.z], i0, first - seg * seg_steps, G.lda);
        pb = OB::at(GATED ? G.B[0] : G.B[seg + w.z], j0, first - seg * seg_steps, G.ldb);
        pb2 = GATED ? OB::at(G.B[1], j0, first, G.ldb) : pb;
        // (an address must not be read by a load within five wait states of the vector unit's writing it; from here on only the scalar
        // unit touches these)
        asm volatile("s_nop 4" : "+s"(pa), "+s"(pb), "+s"(pb2));
    };
    from_the_first();
    const char *const next_a = OA::at(G.A[1], i0, 0, G.lda), *const next_b = OB::at(G.B[1], j0, 0, G.ldb);
    const long long da = OA::advance(G.lda), db = OB::advance(G.ldb);
    auto staged = [&] {
        pa += da; pb += db; pb2 += db;
        left -= OA::STEP;
        if (!GATED && left <= 0) { pa = next_a; pb = next_b; left = G.R; }          // (a second segment, or nothing more to stage)
    };
    constexpr int PASSES = OA::IT + OB::IT;
    const uint32_t lds_wave = lds0 + __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave) * (kWave * 16);
    auto pass = [&](int buf, int p, bool whole) {
        const uint32_t to = buf * STAGE + (p < OA::IT ? 0 : OA::BYTES);
        if (p < OA::IT) {
            if (whole) a.pass(p, lds_wave + to, pa, nullptr);
            else a.last_pass(p, lds_wave + to, tile + to, pa, nullptr, left);
        } else {
            if (whole) b.pass(p - OA::IT, lds_wave + to, pb, pb2);
            else b.last_pass(p - OA::IT, lds_wave + to, tile + to, pb, pb2, left);
        }
    };
    auto stage = [&](int buf) {
        const bool whole = left >= OA::STEP;
#pragma unroll
        for (int p = 0; p < PASSES; ++p) pass(buf, p, whole);
        staged();
    };

    const int wave = (int)threadIdx.x / kWave, wi = wave / WJ, wj = wave % WJ;
    // A tile's residual is asked for before anything else where registers are left for it: with few steps there is nothing to hide
    // its way behind at the end.  (Laid out as store_round below takes it.)
    constexpr int EV = Elem<T>::VEC, ELANES = TJ / EV, EROWS = kWave / ELANES, EARLY_N = EARLY ? TI / EROWS : 1;
    u32x4 early[EARLY_N];
    if constexpr (EARLY) {
        const int j = j0 + wj * TJ + ((int)threadIdx.x % ELANES) * EV;
        if (G.residual && G.splits == 1) {
#pragma unroll
            for (int k = 0; k < EARLY_N; ++k) {
                const int i = i0 + wi * TI + k * EROWS + (int)threadIdx.x % kWave / ELANES;
                if (i < G.I && j + EV <= G.J) early[k] = load_once(static_cast<const T*>(G.residual) + (long long)i * G.ldc + j);
            }
        }
    }
    const int abase = wi * TI, bbase = wj * (GATED ? TJ / 2 : TJ);
    f32x4 acc[FI][FJ];
#pragma unroll
    for (int x = 0; x < FI; ++x)
#pragma unroll
        for (int y = 0; y < FJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};

    typedef std::integral_constant<bool, true> yes;
    typedef std::integral_constant<bool, false> no;
    if constexpr (sizeof(T) == 4) {
        // Float: each value as three bfloat16 (split_float), of whose nine products the six that count run on the bfloat16
        // instructions, 16 times the rate of those for float.  What is dropped, second by third parts, is below 2^-22 of a product (2^-7 by 2^-16 of its
        // factors, twice), on either side.
        // The leading products have accumulators of their own: where an infinity makes one of those infinite, the others, in which it may
        // have met a zero, have no say.
        f32x4 rest[FI][FJ];
        auto sums = [&](auto QUIET) {
#pragma unroll
            for (int x = 0; x < FI; ++x)
#pragma unroll
                for (int y = 0; y < FJ; ++y) acc[x][y] = rest[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (first < last) stage(0);
            for (int s = first, buf = 0; s < last; ++s, buf ^= 1) {
                dma_wait_and_meet();
                if (s + 1 < last) stage(buf ^ 1);
                const lds_char* const ta = tile + buf * STAGE;
                u32x4 pb[FJ][3];
#pragma unroll
                for (int y = 0; y < FJ; ++y) {
                    const int at = bbase + (GATED && y >= FJ / 2 ? BJ / 2 : 0), f = GATED ? y % (FJ / 2) : y;
                    split_float<QUIET()>(fragment<T, BCOLS, BJ>(ta + OA::BYTES, at, f, 0), fragment<T, BCOLS, BJ>(ta + OA::BYTES, at, f, 1), pb[y]);
                }
#pragma unroll
                for (int x = 0; x < FI; ++x) {
                    u32x4 pa[3];
                    split_float<QUIET()>(fragment<T, ACOLS, BI>(ta, abase, x, 0), fragment<T, ACOLS, BI>(ta, abase, x, 1), pa);
#pragma unroll
                    for (int k = 0; k < 6; ++k) {
                        constexpr int ka[6] = {0, 2, 1, 0, 1, 0}, kb[6] = {2, 0, 1, 1, 0, 0};          // small ones first
#pragma unroll
                        for (int y = 0; y < FJ; ++y) {
                            f32x4& to = k == 5 ? acc[x][y] : rest[x][y];
                            to = multiply<bf16_t>(pb[y][kb[k]], pa[ka[k]], to);
                        }
                    }
                }
            }
        };
        sums(no());
        // A leading sum that is not finite may hold a NaN that was cut to an infinity: where a workgroup has one it forms its sums once more, of values
        // that are made quiet.  (In every sum that takes an instruction a value, 5% of a product.)
        f32x4 finite = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < FI; ++x)
#pragma unroll
            for (int y = 0; y < FJ; ++y)
#pragma unroll
                for (int k = 0; k < 4; ++k) finite[k] = fmaf(acc[x][y][k], 0.f, finite[k]);
        typedef __attribute__((address_space(3))) uint32_t lds_word;
        lds_word* const doubts = (lds_word*)(tile + 2 * STAGE);
        const bool doubt = __any(!(finite[0] + finite[1] + finite[2] + finite[3] == 0.f));
        if ((int)threadIdx.x % kWave == 0) doubts[wave] = doubt;
        dma_wait_and_meet();                            // ... and everyone has read the last step
        uint32_t again = 0;
#pragma unroll
        for (int k = 0; k < WI * WJ; ++k) again |= doubts[k];
        if (__builtin_amdgcn_readfirstlane(again)) {
            from_the_first();
            sums(yes());
        }
#pragma unroll
        for (int x = 0; x < FI; ++x)
#pragma unroll
            for (int y = 0; y < FJ; ++y)
#pragma unroll
                for (int k = 0; k < 4; ++k) acc[x][y][k] = fabsf(acc[x][y][k]) < INFINITY ? acc[x][y][k] + rest[x][y][k] : acc[x][y][k];
    } else {
        // A step is multiplied in two halves (ks), row of fragments by row.  What a half needs is read from LDS during the half before:
        // B's fragments into a second set of registers, A's into the row just multiplied.  Where the step's own reads end, one or two
        // rows into the second half, the workgroup meets; the loads of the step after next are issued between the rows that
        // follow, and have a whole step to arrive.
        constexpr int LAG = FI >= 4 ? 2 : 1;
        u32x4 fa[FI], fb[2][FJ];
        auto read_a = [&](int buf, int ks, int x) { fa[x] = fragment<T, ACOLS, BI>(tile + buf * STAGE, abase, x, ks); };
        auto read_b = [&](int buf, int ks) {
#pragma unroll
            for (int y = 0; y < FJ; ++y) fb[ks][y] = fragment<T, BCOLS, BJ>(tile + buf * STAGE + OA::BYTES, bbase + (GATED && y >= FJ / 2 ? BJ / 2 : 0), GATED ? y % (FJ / 2) : y, ks);
        };
        auto multiply_row = [&](int ks, int x) {
#pragma unroll
            for (int y = 0; y < FJ; ++y) acc[x][y] = multiply<T>(fb[ks][y], fa[x], acc[x][y]);
        };
        if (first < last) {
            stage(0);
            if (first + 1 < last) stage(1);
            dma_wait_and_meet();                // (both: with few steps it is the trips to memory one after another that take the time)
            read_b(0, 0);
#pragma unroll
            for (int x = 0; x < FI; ++x) read_a(0, 0, x);
        }
        // NEXT: another step follows; MORE: and yet another, whose loads start here; WHOLE: it is a whole one
        auto step = [&](int buf, auto NEXT, auto MORE, auto WHOLE) {
            read_b(buf, 1);
#pragma unroll
            for (int x = 0; x < FI; ++x) {
                multiply_row(0, x);
                read_a(buf, 1, x);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int x = 0; x < LAG; ++x) multiply_row(1, x);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (NEXT()) {
                dma_wait_and_meet();                // the next step is in LDS, and everyone has read this one
                read_b(buf ^ 1, 0);
#pragma unroll
                for (int x = 0; x < LAG; ++x) read_a(buf ^ 1, 0, x);
            }
#pragma unroll
            for (int x = LAG; x < FI; ++x) {
                if constexpr (MORE()) {
#pragma unroll
                    for (int p = (x - LAG) * PASSES / (FI - LAG); p < (x - LAG + 1) * PASSES / (FI - LAG); ++p) pass(buf, p, WHOLE());
                    __builtin_amdgcn_sched_barrier(0);
                }
                multiply_row(1, x);
                if constexpr (NEXT()) read_a(buf ^ 1, 0, x);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (MORE()) staged();
        };
        int buf = 0, s = first;
        while (s + 2 < last) {
            for (; s + 2 < last && left >= OA::STEP; ++s, buf ^= 1) step(buf, yes(), yes(), yes());
            if (s + 2 < last) {                     // the end of a segment
                step(buf, yes(), yes(), no());
                ++s, buf ^= 1;
            }
        }
        if (s + 1 < last) {
            step(buf, yes(), no(), no());
            buf ^= 1;
        }
        if (first < last) step(buf, no(), no(), no());
    }

    // The accumulators go to memory through LDS, each wavefront through its own part of it, in as many rounds as that takes: a lane
    // holds 4 columns of one row of each fragment, and would fetch and store 16 rows of 32 bytes; from LDS it takes a run
    // of N columns, 16 bytes of the output, beside its neighbours'.
    constexpr int WIDE = GATED ? TJ / 2 : TJ, ROOM = 2 * STAGE / (WI * WJ) / (TJ * 4) / 16;
    constexpr int FX = ROOM >= FI ? FI : ROOM >= FI / 2 ? FI / 2 : FI / 4;                  // rows of fragments in a round
    static_assert(FX >= 1 && FX <= ROOM, "a round fits");
    const int l = (int)threadIdx.x % kWave, t = l & 15, q = l >> 4;
    lds_char* const mine = tile + wave * (FX * 16 * TJ * 4);
    typedef __attribute__((address_space(3))) f32x4 lds_f32x4;
    auto store_round = [&](int x0, auto PART, auto NT) {
        const int i_first = i0 + wi * TI + x0 * 16;
        constexpr int N = PART() ? 4 : Elem<T>::VEC, LANES = WIDE / N, ROWS = kWave / LANES, RUNS = FX * 16 / ROWS, U = RUNS < 4 ? RUNS : RUNS % 4 == 0 ? 4 : 3;
        static_assert(FX * 16 % (ROWS * U) == 0, "whole rounds");
        constexpr bool EXTRAS = FORM == FORM_NT && !PART() && !GATED;
        const int j = j0 + wj * WIDE + (l % LANES) * N, valid = G.J - j;
        float bias[N];
        if constexpr (EXTRAS) load_bias<N>(G, bias, j, valid);
        constexpr int BATCHES = FX * 16 / (ROWS * U);
        auto batch = [&](int b0) {
            const int r0 = b0 + l / LANES;
            float extra[U][N];
            if constexpr (EXTRAS) {
#pragma unroll
                for (int u = 0; u < U; ++u) {
                    const int i = i_first + r0 + u * ROWS;
                    if (i >= G.I || valid <= 0) continue;
                    if (EARLY && G.residual && valid >= N) {
                        if constexpr (EARLY) unpack_run<T>(early[(x0 * 16 + b0) / ROWS + u], extra[u]);
#pragma unroll
                        for (int k = 0; k < N; ++k) extra[u][k] += bias[k];
                    } else {
                        load_extras<T, N>(G, extra[u], bias, (long long)i * G.ldc + j, valid);
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int r = r0 + u * ROWS, i = i_first + r;
                if (i >= G.I || valid <= 0) continue;
                float v[N], up[N];
#pragma unroll
                for (int k = 0; k < N; k += 4) {
                    const int c = ((l % LANES) * N + k) / 4;
                    const f32x4 a4 = *(lds_f32x4*)(mine + r * (TJ * 4) + ((c ^ (r & 7)) << 4));
                    v[k] = a4.x; v[k + 1] = a4.y; v[k + 2] = a4.z; v[k + 3] = a4.w;
                    if constexpr (GATED) {
                        const f32x4 u4 = *(lds_f32x4*)(mine + r * (TJ * 4) + (((c + WIDE / 4) ^ (r & 7)) << 4));
                        up[k] = u4.x; up[k + 1] = u4.y; up[k + 2] = u4.z; up[k + 3] = u4.w;
                    }
                }
                const long long o = (long long)i * G.ldc + j;
                if constexpr (PART()) {
                    float* p = G.part + ((long long)(GATED ? 2 * w.split : w.split * G.batch + w.z) * G.I + i) * G.J + j;
                    store_run<float, N>(p, v, valid);
                    if constexpr (GATED) store_run<float, N>(p + (long long)G.I * G.J, up, valid);
                } else if constexpr (GATED) {
                    finish_gated<T, N, NT()>(G, v, up, o, valid);
                } else if constexpr (FORM == FORM_NT) {
                    finish_linear<T, N, NT()>(G, v, extra[u], o, valid);
                } else {
                    store_run<T, N, NT()>(static_cast<T*>(G.C[w.z]) + o, v, valid);
                }
            }
        };
        if constexpr (EARLY && EXTRAS) {            // (registers cannot be indexed in a loop)
#pragma unroll
            for (int k = 0; k < BATCHES; ++k) batch(k * ROWS * U);
        } else {
            for (int k = 0; k < BATCHES; ++k) batch(k * ROWS * U);
        }
    };
    dma_wait_and_meet();                            // everyone has read the last step
#pragma unroll
    for (int x0 = 0; x0 < FI; x0 += FX) {
        // (16-byte chunk c of a row lies at c ^ (row & 7): rows are a multiple of all banks long)
#pragma unroll
        for (int x = 0; x < FX; ++x)
#pragma unroll
            for (int y = 0; y < FJ; ++y) *(lds_f32x4*)(mine + (x * 16 + t) * (TJ * 4) + (((y * 4 + q) ^ (t & 7)) << 4)) = acc[x0 + x][y];
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the lanes of a wavefront read each other's)
        if (G.splits > 1) store_round(x0, yes(), no());
        else if (G.nt) store_round(x0, no(), yes());
        else store_round(x0, no(), no());
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
}

template <typename T, int FORM, bool GATED, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * kWave, tile_waves(BI * BJ / (WI * WJ))) void gemm_tile(const GemmArgs G)
{
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds(BI, BJ, sizeof(T))];
    tile_product<T, FORM, GATED, BI, BJ, WI, WJ>(G, lds, (int)blockIdx.x, (int)gridDim.x);
}

// The same for a forward product with many tiles and a short reduction (short_shape says when).  Its epilogue counts, so a residual, asked for
// early, has a kernel of its own: without one the registers are better left free (67200 x 64 x 1024 50 us, and 56 with them).
template <typename T, int BI, int BJ, int WI, int WJ, bool RESIDUAL>
__global__ __launch_bounds__(WI * WJ * kWave, tile_waves(BI * BJ / (WI * WJ))) void gemm_short(const GemmArgs G)
{
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds(BI, BJ, sizeof(T))];
    tile_product<T, FORM_NT, false, BI, BJ, WI, WJ, RESIDUAL>(G, lds, (int)blockIdx.x, (int)gridDim.x);
}

// dx = dz W and dW = dz^T x in one launch: neither needs the other, and the second's workgroups fill the compute units that
// the first's last round leaves idle.  268800 x 512 x 128: 160 us, 440 TF, bound by dx's 275 MB on their way out beside two reads of dz; 5003 x
// 2048 x 5461, both projections: 400 us, 1120 TF, bound by the matrix cores (busy 60%).
template <typename T, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * kWave, tile_waves(BI * BJ / (WI * WJ))) void gemm_two(const GemmArgs X, const GemmArgs W, int nx)
{
    __shared__ __attribute__((aligned(1024))) char lds[tile_lds(BI, BJ, sizeof(T))];
    if ((int)blockIdx.x < nx) tile_product<T, FORM_NN, false, BI, BJ, WI, WJ>(X, lds, (int)blockIdx.x, nx);
    else tile_product<T, FORM_TN, false, BI, BJ, WI, WJ>(W, lds, (int)blockIdx.x - nx, (int)gridDim.x - nx);
}

// Partial sums of a split reduction, added in a fixed order, then the epilogue.  N values a thread (4 where J allows whole vectors).
// Where there are few values and many splits, `lanes` threads (a power of two) share a value's splits: 128 x 512 values of 120
// splits took 31 us with one thread each, 7 with several; 512 x 1024 values of few splits want one (85 us with the product, 90 with two).
template <typename T, int FORM, bool GATED, int N>
__global__ __launch_bounds__(kThreads) void gemm_join(const GemmArgs G, int lanes)
{
    constexpr int P = GATED ? 2 : 1, U = 4;
    __shared__ float red[kThreads * N * P];
    const long long plane = (long long)G.I * G.J, planes = GATED ? 2 : G.batch, total = GATED ? plane : plane * planes;
    const int across = kThreads / lanes, lane = (int)threadIdx.x / across, at = (int)threadIdx.x % across;
    const long long e = ((long long)blockIdx.x * across + at) * N;
    float v[P][N];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int k = 0; k < N; ++k) v[p][k] = 0.f;
    if (e < total) {
        for (int s0 = lane; s0 < G.splits; s0 += U * lanes) {
            float t[U][P][N];
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int p = 0; p < P; ++p)
                    load_run<float, N>(G.part + e + (s0 + u * lanes) * plane * planes + p * plane, t[u][p], s0 + u * lanes < G.splits ? N : 0);
#pragma unroll
            for (int u = 0; u < U; ++u)
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int k = 0; k < N; ++k) v[p][k] += t[u][p][k];
        }
    }
    if (lanes > 1) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int k = 0; k < N; ++k) red[(p * N + k) * kThreads + threadIdx.x] = v[p][k];
        __syncthreads();
        if (lane != 0) return;
        for (int o = 1; o < lanes; ++o)
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int k = 0; k < N; ++k) v[p][k] += red[(p * N + k) * kThreads + o * across + at];
    }
    if (e >= total) return;
    const long long z = GATED ? 0 : e / plane, o = e - z * plane;        // (outputs are dense)
    if constexpr (GATED) {
        finish_gated<T, N>(G, v[0], v[1], o, N);
    } else if constexpr (FORM == FORM_NT) {
        float bias[N], extra[N];
        load_bias<N>(G, bias, (int)(o % G.J), N);
        load_extras<T, N>(G, extra, bias, o, N);
        finish_linear<T, N>(G, v[0], extra, o, N);
    } else {
        store_run<T, N>(static_cast<T*>(G.C[z]) + o, v[0], N);
    }
}

}  // namespace cgbn
