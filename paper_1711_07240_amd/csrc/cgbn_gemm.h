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
// neighbours in a row of C.  Where B is in rows, which of its rows feed which row of which fragment is free: they are dealt so that a
// lane ends up with 16 neighbours (8 + 8 of a gated pair), which makes the epilogue's loads and stores 16 bytes wide.
//
// Sums are held in 32 bits throughout.  Where tiles are too few for 256 compute units the reduction is split and the partial
// sums, float, are joined by gemm_join in split order: results never depend on the order in which workgroups end.
#pragma once

#include "cgbn_kernels.h"

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
};

// ---- activations, on 32-bit values ----

__device__ __forceinline__ float act_apply(float z, int act)
{
    if (act == ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    if (act == ACT_GELU) return z * (0.5f + 0.5f * erff(z * 0.70710678118654752f));
    if (act == ACT_SILU) return z / (1.f + expf(-z));
    return z;
}

// act'(z)
__device__ __forceinline__ float act_slope(float z, int act)
{
    if (act == ACT_RELU) return z > 0.f ? 1.f : 0.f;
    if (act == ACT_GELU) return 0.5f + 0.5f * erff(z * 0.70710678118654752f) + z * 0.39894228040143268f * expf(-0.5f * z * z);
    if (act == ACT_SILU) {
        const float s = 1.f / (1.f + expf(-z));
        return s + z * s * (1.f - s);
    }
    return 1.f;
}

// ---- runs of neighbouring values ----

template <typename T, int N> __device__ __forceinline__ void load_run(const T* p, float (&v)[N], int valid, bool whole)
{
    constexpr int V = Elem<T>::VEC < N ? Elem<T>::VEC : N;
    if (whole) {
        if constexpr (V == Elem<T>::VEC) {
#pragma unroll
            for (int k = 0; k < N; k += V) {
                float t[V];
                Elem<T>::loadv(p + k, t);
#pragma unroll
                for (int e = 0; e < V; ++e) v[k + e] = t[e];
            }
        } else if constexpr (N == 4) {                 // 4 bfloat16
            const uint2 w = *reinterpret_cast<const uint2*>(p);
            v[0] = bf16_to_f32(w.x & 0xffffu); v[1] = bf16_to_f32(w.x >> 16);
            v[2] = bf16_to_f32(w.y & 0xffffu); v[3] = bf16_to_f32(w.y >> 16);
        }
    } else {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = k < valid ? Elem<T>::load1(p + k) : 0.f;
    }
}

template <typename T, int N> __device__ __forceinline__ void store_run(T* p, const float (&v)[N], int valid, bool whole)
{
    constexpr int V = Elem<T>::VEC < N ? Elem<T>::VEC : N;
    if (whole) {
        if constexpr (V == Elem<T>::VEC) {
#pragma unroll
            for (int k = 0; k < N; k += V) {
                float t[V];
#pragma unroll
                for (int e = 0; e < V; ++e) t[e] = v[k + e];
                Elem<T>::storev(p + k, t, 0);
            }
        } else if constexpr (N == 4) {
            uint2 w;
            w.x = f32x2_to_bf16x2(v[0], v[1]); w.y = f32x2_to_bf16x2(v[2], v[3]);
            *reinterpret_cast<uint2*>(p) = w;
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
// written (but m0, in which the compiler keeps nothing); dma_wait_and_meet() below makes the bytes visible.  The wait states
// are those that m0, and an address in scalar registers that the vector unit may have written, need before the load.
__device__ __forceinline__ void dma16(uint32_t lds, const char* base, uint32_t off)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void dma16(uint32_t lds, const char* p)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}
// every load of this wavefront has landed, every LDS read of it has returned; then the workgroup meets
__device__ __forceinline__ void dma_wait_and_meet()
{
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
}

__device__ __attribute__((aligned(16))) const uint32_t gemm_zeros[4] = {0, 0, 0, 0};

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_hw __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) char lds_char;

// How the rows of B (operand in rows) are dealt to fragments: lane t of a fragment's 16 rows, fragment f of 4.
enum { DEAL_PLAIN = 0, DEAL_16 = 1, DEAL_GATED = 2 };

// xor key of a row of an operand in rows (8 chunks of 16 bytes a row): the 16 rows that a fragment read touches at once spread over all banks
template <int DEAL> __device__ __forceinline__ int row_key(int row)
{
    if constexpr (DEAL == DEAL_16) return (row & 3) | ((row >> 4) & 1) << 2;
    if constexpr (DEAL == DEAL_GATED) return (row & 3) | ((row >> 3) & 1) << 2;
    return row & 7;
}

// xor key, in 16-byte chunks, of a row of an operand in columns with CR chunks a row
template <typename T, int CR> __device__ __forceinline__ int col_key(int row)
{
    if constexpr (sizeof(T) == 2)
        return CR >= 16 ? ((row & 3) | ((row >> 3) & 1) << 2) << 1 : (((row >> 1) & 1) | ((row >> 3) & 1) << 1) << 1;
    else
        return ((row >> 2) & 3) << 2;
}

// One operand's share of a step: ROWS (of i or j) x 128 bytes of r, staged by NT threads.
template <typename T, bool COLS, int ROWS, int NT, int DEAL> struct Operand {
    static constexpr int E = 16 / (int)sizeof(T);           // elements of a chunk
    static constexpr int STEP = 128 / (int)sizeof(T);       // r of a step
    static constexpr int CR = COLS ? ROWS / E : 8;          // chunks of a row of the tile in LDS
    static constexpr int BYTES = ROWS * 128;
    static constexpr int IT = BYTES / 16 / NT;
    static constexpr int HALF = ROWS / 2;
    static_assert(BYTES % (16 * NT) == 0, "whole passes");
    static_assert(DEAL != DEAL_GATED || HALF % (NT / 8) == 0, "a pass stays within one of the two matrices");

    uint32_t off[IT];

    // row of the tile in LDS and chunk of that row's data that this thread fetches in pass `it`
    static __device__ __forceinline__ int row_of(int it) { return (it * NT + (int)threadIdx.x) / CR; }
    static __device__ __forceinline__ int chunk_of(int it)
    {
        const int slot = (it * NT + (int)threadIdx.x) % CR;
        if constexpr (COLS) return slot ^ col_key<T, CR>(row_of(it));
        else return slot ^ row_key<DEAL>(row_of(it));
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
                const int r = DEAL == DEAL_GATED ? row_of(it) % HALF : row_of(it);
                off[it] = (uint32_t)((min(first + r, n - 1) - first) * ld * (int)sizeof(T)) + chunk_of(it) * 16;
            }
        }
    }
    static __device__ __forceinline__ const char* at(const void* p, int first, int step, long long ld)
    {
        return static_cast<const char*>(p) + (COLS ? (long long)step * STEP * ld + first : (long long)first * ld + (long long)step * STEP) * (int)sizeof(T);
    }
    // p1: the second matrix of a gated pair.  lds: where the tile goes.  left: r that remain from this step on
    __device__ __forceinline__ void stage(uint32_t lds, const void* p0, const void* p1, int first, int step, long long ld, int left) const
    {
        const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x / kWave);
        const char* b0 = at(p0, first, step, ld);
        const char* b1 = DEAL == DEAL_GATED ? at(p1, first, step, ld) : b0;
        if (left >= STEP) {
#pragma unroll
            for (int it = 0; it < IT; ++it)
                dma16(lds + (it * NT + wave * kWave) * 16, DEAL == DEAL_GATED && it * (NT / 8) >= HALF ? b1 : b0, off[it]);
        } else {
#pragma unroll
            for (int it = 0; it < IT; ++it) {
                const bool in = (COLS ? row_of(it) : chunk_of(it) * E) < left;
                const char* b = DEAL == DEAL_GATED && it * (NT / 8) >= HALF ? b1 : b0;
                dma16(lds + (it * NT + wave * kWave) * 16, in ? b + off[it] : reinterpret_cast<const char*>(gemm_zeros));
            }
        }
    }
};

// A fragment: 16 rows of i x 16 bytes of r a lane, that is lane l holds row l % 16 and chunk 4 * ks + l / 16 of the step.
// (bfloat16: what one matrix instruction takes; float: four of them, r being dealt to them in the same way on both sides.)
// first: the fragment's first row within the tile (a multiple of 16), or its column group where rows are dealt.
template <typename T, bool COLS, int ROWS, int DEAL>
__device__ __forceinline__ u32x4 fragment(const lds_char* tile, int base, int f, int ks)
{
    const int l = (int)threadIdx.x % kWave, t = l & 15, q = l >> 4;
    if constexpr (!COLS) {
        int row;
        if constexpr (DEAL == DEAL_16) row = base + (t >> 2) * 16 + f * 4 + (t & 3);
        else if constexpr (DEAL == DEAL_GATED) row = (f >> 1) * (ROWS / 2) + base + (t >> 2) * 8 + (f & 1) * 4 + (t & 3);
        else row = base + f * 16 + t;
        return *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + row * 128 + (((ks * 4 + q) ^ row_key<DEAL>(row)) << 4));
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

// Which tile a workgroup takes.  Consecutive workgroups go to the 8 dies in turn, so each die is given a run of consecutive
// work of its own; within it tiles go in blocks of 8 rows of tiles, column by column, so that the ones in flight at a time share operands in
// the die's L2.
struct TileId { int i, j, split, z; };
__device__ __forceinline__ TileId tile_of(const GemmArgs& G)
{
    const int n = (int)gridDim.x, id = (int)blockIdx.x, die = id & 7, q = n >> 3, r = n & 7;
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

template <typename T, int N> __device__ __forceinline__ void finish_linear(const GemmArgs& G, float (&v)[N], int i, int j, bool whole)
{
    const int valid = G.J - j;
    const long long o = (long long)i * G.ldc + j;
    if (G.bias) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += k < valid ? G.bias[j + k] : 0.f;
    }
    if (G.residual) {
        float r[N];
        load_run<T, N>(static_cast<const T*>(G.residual) + o, r, valid, whole);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += r[k];
    }
    if (G.Z[0]) store_run<T, N>(static_cast<T*>(G.Z[0]) + o, v, valid, whole);
    if (G.act == ACT_RELU) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = act_apply(v[k], ACT_RELU);
    } else if (G.act == ACT_GELU) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = act_apply(v[k], ACT_GELU);
    } else if (G.act == ACT_SILU) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = act_apply(v[k], ACT_SILU);
    }
    store_run<T, N>(static_cast<T*>(G.C[0]) + o, v, valid, whole);
}

template <typename T, int N> __device__ __forceinline__ void finish_gated(const GemmArgs& G, float (&g)[N], const float (&u)[N], int i, int j, bool whole)
{
    const int valid = G.J - j;
    const long long o = (long long)i * G.ldc + j;
    if (G.Z[0]) {
        store_run<T, N>(static_cast<T*>(G.Z[0]) + o, g, valid, whole);
        store_run<T, N>(static_cast<T*>(G.Z[1]) + o, u, valid, whole);
    }
    if (G.act == ACT_RELU) {
#pragma unroll
        for (int k = 0; k < N; ++k) g[k] = act_apply(g[k], ACT_RELU);
    } else if (G.act == ACT_GELU) {
#pragma unroll
        for (int k = 0; k < N; ++k) g[k] = act_apply(g[k], ACT_GELU);
    } else if (G.act == ACT_SILU) {
#pragma unroll
        for (int k = 0; k < N; ++k) g[k] = act_apply(g[k], ACT_SILU);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) g[k] *= u[k];
    store_run<T, N>(static_cast<T*>(G.C[0]) + o, g, valid, whole);
}

// ---- the product ----

template <typename T, int FORM, bool GATED, bool PART, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * kWave) void gemm_tile(const GemmArgs G)
{
    constexpr int NT = WI * WJ * kWave, TI = BI / WI, FI = TI / 16, FJ = 4;
    static_assert(BJ / WJ == 64 && TI % 16 == 0, "a wavefront's share is 64 columns wide");
    constexpr bool ACOLS = FORM == FORM_TN, BCOLS = FORM != FORM_NT;
    constexpr int DEAL = BCOLS ? DEAL_PLAIN : (GATED ? DEAL_GATED : DEAL_16);
    typedef Operand<T, ACOLS, BI, NT, DEAL_PLAIN> OA;
    typedef Operand<T, BCOLS, BJ, NT, DEAL> OB;
    constexpr int STAGE = OA::BYTES + OB::BYTES;
    __shared__ __attribute__((aligned(1024))) char lds[2 * STAGE];
    lds_char* const tile = (lds_char*)lds;
    const uint32_t lds0 = (uint32_t)(uintptr_t)tile;

    const TileId w = tile_of(G);
    const int i0 = w.i * BI, j0 = w.j * (GATED ? BJ / 2 : BJ);
    OA a;
    OB b;
    a.init(i0, G.I, G.lda);
    b.init(j0, G.J, G.ldb);
    const int seg_steps = (G.R + OA::STEP - 1) / OA::STEP;
    const int first = w.split * G.per, last = min(first + G.per, seg_steps * G.segs);

    auto stage = [&](int s, int buf) {
        const int seg = s >= seg_steps, step = s - seg * seg_steps, which = seg + w.z, left = G.R - step * OA::STEP;
        const uint32_t to = lds0 + buf * STAGE;
        a.stage(to, G.A[which], nullptr, i0, step, G.lda, left);
        b.stage(to + OA::BYTES, GATED ? G.B[0] : G.B[which], G.B[1], j0, step, G.ldb, left);
    };

    const int wave = (int)threadIdx.x / kWave, wi = wave / WJ, wj = wave % WJ;
    const int abase = wi * TI, bbase = wj * (GATED ? 32 : 64);
    f32x4 acc[FI][FJ];
#pragma unroll
    for (int x = 0; x < FI; ++x)
#pragma unroll
        for (int y = 0; y < FJ; ++y) acc[x][y] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (first < last) stage(first, 0);
    for (int s = first; s < last; ++s) {
        dma_wait_and_meet();
        const int buf = (s - first) & 1;
        if (s + 1 < last) stage(s + 1, buf ^ 1);
        const lds_char* ta = tile + buf * STAGE;
        const lds_char* tb = ta + OA::BYTES;
#pragma unroll
        for (int ks = 0; ks < 2; ++ks) {
            u32x4 fb[FJ], fa[FI];
#pragma unroll
            for (int y = 0; y < FJ; ++y) fb[y] = fragment<T, BCOLS, BJ, DEAL>(tb, bbase, y, ks);
#pragma unroll
            for (int x = 0; x < FI; ++x) fa[x] = fragment<T, ACOLS, BI, DEAL_PLAIN>(ta, abase, x, ks);
#pragma unroll
            for (int x = 0; x < FI; ++x)
#pragma unroll
                for (int y = 0; y < FJ; ++y) acc[x][y] = multiply<T>(fb[y], fa[x], acc[x][y]);
        }
    }

    const int l = (int)threadIdx.x % kWave, t = l & 15, q = l >> 4;
#pragma unroll
    for (int x = 0; x < FI; ++x) {
        const int i = i0 + wi * TI + x * 16 + t;
        if (i >= G.I) continue;
        if constexpr (GATED) {
            const int j = j0 + wj * 32 + q * 8;
            if (j >= G.J) continue;
            float g[8], u[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) { g[k] = acc[x][k >> 2][k & 3]; u[k] = acc[x][2 + (k >> 2)][k & 3]; }
            if constexpr (PART) {
                const bool whole = j + 8 <= G.J && G.J % 4 == 0;
                float* p = G.part + ((long long)w.split * 2 * G.I + i) * G.J + j;
                store_run<float, 8>(p, g, G.J - j, whole);
                store_run<float, 8>(p + (long long)G.I * G.J, u, G.J - j, whole);
            } else {
                finish_gated<T, 8>(G, g, u, i, j, j + 8 <= G.J && G.J % 8 == 0);
            }
        } else if constexpr (FORM == FORM_NT) {
            const int j = j0 + wj * 64 + q * 16;
            if (j >= G.J) continue;
            float v[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) v[k] = acc[x][k >> 2][k & 3];
            if constexpr (PART) store_run<float, 16>(G.part + ((long long)w.split * G.I + i) * G.J + j, v, G.J - j, j + 16 <= G.J && G.J % 4 == 0);
            else finish_linear<T, 16>(G, v, i, j, j + 16 <= G.J && G.J % 8 == 0);
        } else {
#pragma unroll
            for (int y = 0; y < FJ; ++y) {
                const int j = j0 + wj * 64 + y * 16 + q * 4;
                if (j >= G.J) continue;
                float v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) v[k] = acc[x][y][k];
                const bool whole = j + 4 <= G.J && G.J % 4 == 0;
                if constexpr (PART) store_run<float, 4>(G.part + ((long long)(w.split * G.batch + w.z) * G.I + i) * G.J + j, v, G.J - j, whole);
                else store_run<T, 4>(static_cast<T*>(G.C[w.z]) + (long long)i * G.ldc + j, v, G.J - j, whole);
            }
        }
    }
}

// Partial sums of a split reduction, added in split order, then the epilogue.  N values a thread (4 where J allows whole vectors).
template <typename T, int FORM, bool GATED, int N>
__global__ __launch_bounds__(kThreads) void gemm_join(const GemmArgs G)
{
    const long long plane = (long long)G.I * G.J, planes = GATED ? 2 : G.batch;
    const long long e = ((long long)blockIdx.x * kThreads + threadIdx.x) * N;
    const long long total = GATED ? plane : plane * planes;
    if (e >= total) return;
    const float* p = G.part + e;
    float v[N], u[N];
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = u[k] = 0.f;
    for (int s = 0; s < G.splits; ++s, p += plane * planes) {
        float t[N];
        load_run<float, N>(p, t, N, N == 4);
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] += t[k];
        if constexpr (GATED) {
            load_run<float, N>(p + plane, t, N, N == 4);
#pragma unroll
            for (int k = 0; k < N; ++k) u[k] += t[k];
        }
    }
    const long long z = GATED ? 0 : e / plane, o = e - z * plane;
    const int i = (int)(o / G.J), j = (int)(o - (long long)i * G.J);
    if constexpr (GATED) finish_gated<T, N>(G, v, u, i, j, N == 4);
    else if constexpr (FORM == FORM_NT) finish_linear<T, N>(G, v, i, j, N == 4);
    else store_run<T, N>(static_cast<T*>(G.C[z]) + (long long)i * G.ldc + j, v, N, N == 4);
}

}  // namespace cgbn
