// The layers beside the normalization: matrix product with bias, residual and activation, and the gated feed-forward block,
// forward and backward.  Argument checks, workspace layout, launches; the products themselves are in cgbn_gemm.h (tiles) and
// cgbn_gemm_rows.h (few rows).
#include "cgbn.h"
#include "cgbn_gemm_plan.h"
#include "cgbn_gemm_rows.h"
#include "cgbn_column_sums.h"
#include "cgbn_grid.h"

#include <cstring>

namespace cgbn {
namespace {

// ---- small kernels around the products ----

// A row's last values: `valid` of them, at least one and fewer than E; zeros for the others.  The last one is asked for again where there is none,
// without a branch: all of the loads are on their way before the first is waited for.
template <typename T, int E> __device__ __forceinline__ void load_end(const T* p, float (&v)[E], int valid)
{
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = Elem<T>::load1(p + min(k, valid - 1));
#pragma unroll
    for (int k = 0; k < E; ++k) v[k] = k < valid ? v[k] : 0.f;
}

// Rows of n elements to rows of np, the filling zero: operands whose rows do not start on 16 bytes, which a load to LDS has to.  All operands of a
// call in one launch.  Bound by memory where it is not the launch, 3 us (6832 x 267 float, 7.3 MB read and written, 5.8 us).
struct PadArgs {
    const void* src[3];
    void* dst[3];
    long long end[3];              // 16-byte chunks up to the end of each operand
    int n, np;
};
template <typename T> __global__ __launch_bounds__(kThreads) void pad_rows(const PadArgs A)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int chunks = A.np / E;
    long long id = workgroup() * kThreads + threadIdx.x;
    if (id >= A.end[2]) return;
    const int k = id < A.end[0] ? 0 : id < A.end[1] ? 1 : 2;
    id -= k == 0 ? 0 : k == 1 ? A.end[0] : A.end[1];
    const T* const src = static_cast<const T*>(k == 0 ? A.src[0] : k == 1 ? A.src[1] : A.src[2]);
    T* const dst = static_cast<T*>(k == 0 ? A.dst[0] : k == 1 ? A.dst[1] : A.dst[2]);
    const long long r = id / chunks;
    const int c = (int)(id - r * chunks) * E, valid = A.n - c;
    float v[E];
    if (valid >= E) load_run<T, E>(src + r * A.n + c, v, valid);
    else load_end<T, E>(src + r * A.n + c, v, valid);
    store_run<T, E>(dst + r * A.np + c, v, E);
}

// the E values of a run: one decision for all of them
#define CGBN_EACH(act_, which_, ...)                          \
    if (act_ == which_) {                                     \
        _Pragma("unroll") for (int e = 0; e < E; ++e) { __VA_ARGS__; } \
    }

struct DzArgs {
    const void *dy, *saved;        // [M][N]; saved null: act none
    void *dz, *dresidual;          // [M][ld], [M][N]; either may be null
    float* part;                   // [row blocks][N] column sums, or null
    long long M;
    int N, ld, act;
    int tw, rows;                  // vectors of a row that a workgroup covers (a power of two, at most 64); rows of a block
};

// dz = dy * act'(saved), and its column sums.  Memory bound: one read of dy and saved, one write of dz (268800 x 128 bfloat16, ReLU: 38
// us, 5.4 TB/s).  A thread stays in one column vector and walks rows; its sums are of at most rows * tw / 256 values, in float, and column_sums
// adds those of the workgroups.  dz is rounded to the operands' type, which is what the matrix cores multiply: half the bytes of a float dz,
// written once and read twice; the column sums are of the values before it.
// ENDS: rows are no whole number of vectors.  (A kernel each: the registers that ends are loaded to cost the others 209 us for 205.)
template <typename T, bool ENDS> __global__ __launch_bounds__(kThreads) void linear_dz(const DzArgs A)
{
    constexpr int E = 16 / (int)sizeof(T);
    __shared__ float red[kThreads * E];
    const int tw = A.tw, c = ((int)blockIdx.x * tw + (int)threadIdx.x % tw) * E, first = (int)threadIdx.x / tw, stride = kThreads / tw;
    const bool in = c < A.ld;
    const int valid = A.N - c;
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.f;
    const long long r0 = (long long)blockIdx.y * A.rows, r1 = min(r0 + A.rows, A.M);
    if (in) {
        const T *const dy = static_cast<const T*>(A.dy) + c, *const saved = static_cast<const T*>(A.saved) + c;
        auto row = [&](long long r, float (&g)[E], const float (&z)[E]) {
            // (where ReLU passes nothing dz is zero, not dy * 0: an infinity there does not become NaN)
            if (A.saved) {
                CGBN_EACH(A.act, ACT_RELU, g[e] = z[e] > 0.f ? g[e] : 0.f)
                CGBN_EACH(A.act, ACT_GELU, g[e] *= act_slope<sizeof(T) == 4>(z[e], ACT_GELU))
                CGBN_EACH(A.act, ACT_SILU, g[e] *= act_slope<sizeof(T) == 4>(z[e], ACT_SILU))
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += g[e];
            // (beyond the row the filling is zero: what was loaded there is)
            if (A.dz) store_run<T, E>(static_cast<T*>(A.dz) + r * A.ld + c, g, E);
            if (A.dresidual) store_run<T, E>(static_cast<T*>(A.dresidual) + r * A.N + c, g, valid);
        };
        // four rows at a time: the loads of all before the first is used (the last row's again where there are fewer)
        constexpr int U = 4;
        for (long long r = r0 + first; r < r1; r += U * stride) {
            u32x4 wg[U], wz[U];
            auto load = [&](const T* p, u32x4 (&w)[U]) {
                if (!ENDS || valid >= E) {
#pragma unroll
                    for (int u = 0; u < U; ++u) w[u] = load_once(p + min(r + u * stride, r1 - 1) * A.N);
                } else {
#pragma unroll
                    for (int u = 0; u < U; ++u) w[u] = row_chunk<T>(p + min(r + u * stride, r1 - 1) * A.N, valid);
                }
            };
            load(dy, wg);
            if (A.saved) load(saved, wz);
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float g[E], z[E];
                unpack_run<T>(wg[u], g);
                unpack_run<T>(wz[u], z);
                if (r + u * stride < r1) row(r + u * stride, g, z);
            }
        }
    }
    if (!A.part) return;
#pragma unroll
    for (int e = 0; e < E; ++e) red[threadIdx.x * E + e] = sum[e];
    __syncthreads();
    for (int v = (int)threadIdx.x; v < tw * E; v += kThreads) {
        float s = 0.f;
        for (int k = 0; k < stride; ++k) s += red[k * tw * E + v];
        const int n = (int)blockIdx.x * tw * E + v;
        if (n < A.N) A.part[(long long)blockIdx.y * A.N + n] = s;
    }
}

struct GateArgs {
    const void *dh, *gate, *up;    // [M][F]
    void *dg, *du;                 // [M][ld]
    long long M;
    int F, ld, act;
};

// dg = dh * up * act'(gate), du = dh * act(gate), rounded to the operands' type for the products that follow (as they would be
// had they been tensors of the layer): memory bound, three reads and two writes (5003 x 5461 bfloat16, rows on no 16 bytes, GELU: 48 us, 5.7 TB/s).
template <typename T> __global__ __launch_bounds__(kThreads) void gated_dz(const GateArgs A)
{
    constexpr int E = 16 / (int)sizeof(T);
    const int chunks = A.ld / E;
    const long long total = A.M * chunks;
    for (long long id = (long long)blockIdx.x * kThreads + threadIdx.x; id < total; id += (long long)gridDim.x * kThreads) {
        const long long r = id / chunks;
        const int c = (int)(id - r * chunks) * E, valid = A.F - c;
        const long long o = r * A.F + c;
        const T *const ph = static_cast<const T*>(A.dh) + o, *const pg = static_cast<const T*>(A.gate) + o, *const pu = static_cast<const T*>(A.up) + o;
        float h[E], g[E], u[E];
        if (valid >= E) {
            const u32x4 wh = load_once(ph), wg = load_once(pg), wu = load_once(pu);
            unpack_run<T>(wh, h);
            unpack_run<T>(wg, g);
            unpack_run<T>(wu, u);
        } else {
            load_end<T, E>(ph, h, valid);
            load_end<T, E>(pg, g, valid);
            load_end<T, E>(pu, u, valid);
        }
        CGBN_EACH(A.act, ACT_NONE, const float a = g[e]; g[e] = h[e] * u[e]; u[e] = h[e] * a)
        CGBN_EACH(A.act, ACT_RELU, const float a = act_apply<sizeof(T) == 4>(g[e], ACT_RELU); g[e] = g[e] > 0.f ? h[e] * u[e] : 0.f; u[e] = h[e] * a)
        CGBN_EACH(A.act, ACT_GELU, const float z = g[e]; g[e] = h[e] * u[e] * act_slope<sizeof(T) == 4>(z, ACT_GELU); u[e] = h[e] * act_apply<sizeof(T) == 4>(z, ACT_GELU))
        CGBN_EACH(A.act, ACT_SILU, const float z = g[e]; g[e] = h[e] * u[e] * act_slope<sizeof(T) == 4>(z, ACT_SILU); u[e] = h[e] * act_apply<sizeof(T) == 4>(z, ACT_SILU))
        store_run<T, E>(static_cast<T*>(A.dg) + r * A.ld + c, g, E);
        store_run<T, E>(static_cast<T*>(A.du) + r * A.ld + c, u, E);
    }
}

template <typename T> __global__ __launch_bounds__(kThreads) void fill_zero(T* p, long long n)
{
    const long long i = workgroup() * kThreads + threadIdx.x;
    if (i < n) p[i] = T{};
}

// ---- host ----

#define CGBN_TRY(call_)                                  \
    do {                                                 \
        const cgbn_status s_ = (call_);                  \
        if (s_ != CGBN_OK) return s_;                    \
    } while (0)
#define CGBN_HIP(call_)                                  \
    do {                                                 \
        if ((call_) != hipSuccess) return CGBN_ERR_HIP;  \
    } while (0)

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
size_t round256(size_t n) { return (n + 255) / 256 * 256; }

constexpr int kMaxWidth = 1 << 20;                  // of N, K, F: a tile's byte offsets stay within 32 bits
constexpr long long kMaxRows = 1ll << 30;
constexpr long long kMaxElements = 1ll << 38;       // of a matrix: grids stay within 31 bits (and what a product's tiles have for threads, see plan_with)

// Whether a product takes gemm_rows.  Up to 16 rows it does: the gated pair 38 against 49 us with tiles (4096 x 11264, 16 rows), 61
// against 49 with 32.  Beyond them it pays for every row again with all of the weights, so these have to be small.  bfloat16, against
// tiles: 5.0 and 7.3 us (32 rows, 1024 x 1024), 11.1 and 12.1 (17, 4096 x 4096), 12.4 and 12.4 (24), 13.7 and 12.8 (32), 31 and 26.5
// (17, 12288 x 4096).  Float, whose tiles multiply six times: 27 and 26.6 (32, 4096 x 4096), 58 and 64 (17, 12288 x 4096), 64.5 and
// 64.3 (24), 73 and 66 (32).
bool few_rows(long long M, int N, int K, int elem, bool gated)
{
    if (M <= 16) return true;
    return !gated && M <= 32 && (double)M * N * K * elem <= (elem == 2 ? 0.8e9 : 4e9);
}

cgbn_status check_sizes(long long M, int N, int K, int dtype)
{
    if (dtype != CGBN_F32 && dtype != CGBN_BF16) return CGBN_ERR_ENUM;
    if (M < 0 || M > kMaxRows || N < 1 || N > kMaxWidth || K < 1 || K > kMaxWidth) return CGBN_ERR_SHAPE;
    if (M * N > kMaxElements || M * K > kMaxElements || (long long)N * K > kMaxElements) return CGBN_ERR_SHAPE;
    return CGBN_OK;
}

// How a call uses its workspace: byte offsets of its parts, 0 bytes for those it needs not.
struct Layout {
    size_t at = 0;
    size_t take(size_t bytes)
    {
        const size_t o = at;
        at += round256(bytes);
        return o;
    }
};

struct Widths {
    int elem, E;
    explicit Widths(int dtype) : elem(dtype == CGBN_F32 ? 4 : 2), E(16 / elem) {}
    int padded(int n) const { return (n + E - 1) / E * E; }
    bool odd(int n) const { return n % E != 0; }
};

struct ForwardPlan {
    bool rows;                  // gemm_rows
    bool none;                  // more tiles than a launch has
    GemmPlan g;
    size_t x, w, part, bytes;   // padded copies of x and of the weights; partial sums
};

ForwardPlan plan_forward(long long M, int N, int K, int dtype, bool gated)
{
    const Widths W(dtype);
    ForwardPlan p{};
    p.rows = few_rows(M, N, K, W.elem, gated);
    Layout l;
    if (p.rows) {
        // Workgroups of 16 weight rows; where those are too few for the device and long, several share them: 23.4 us by 4 workgroups,
        // 7.2 by 40 (the gated pair, 2 x 5248 x 64, float); bfloat16, 1 x 4096 x 64 6.5 and 5.4, 16 x 4096 x 256 9.1 and 6.4, gated 13.2 and
        // 8.0.  Not for less: 16 x 3008 x 256 is 7.4 and 7.0, 1 x 2048 x 256 4.5 and 5.3.  Where only two can, the joining has to pay: 1 x 4096 x 2048 7.3
        // and 9.3; 1 x 8192 x 1024 11.5 and 9.4.
        const int steps = (K * W.elem + 127) / 128, groups = (N + 15) / 16;
        int want = groups <= 128 && steps >= (groups <= 64 || gated ? 48 : 96) ? 256 / groups : 1;
        if (want > steps / 16) want = steps / 16 > 1 ? steps / 16 : 1;
        p.g.per = (steps + want - 1) / want;
        p.g.splits = (steps + p.g.per - 1) / p.g.per;
        p.part = l.take(p.g.splits > 1 ? (size_t)p.g.splits * (gated ? 2 : 1) * M * N * sizeof(float) : 0);
        p.bytes = l.at;
        return p;
    }
    p.g = plan_gemm(W.elem, gated, M, N, K, 1, 1);
    p.none = p.g.ti == 0;
    if (W.odd(K)) {
        p.x = l.take((size_t)M * W.padded(K) * W.elem);
        p.w = l.take((size_t)N * W.padded(K) * W.elem * (gated ? 2 : 1));
    }
    p.part = l.take(p.g.part_bytes);
    p.bytes = l.at;
    return p;
}

struct BackwardPlan {
    GemmPlan dx, dw;
    size_t dz, x, w, part_x, part_w, sums, bytes;
    int sum_blocks, sum_rows, tw;
    bool none;
};

// (one plan whichever of dx and dW a call wants: it is what the workspace is sized by)
BackwardPlan plan_backward(long long M, int N, int K, int dtype, bool gated)
{
    const Widths W(dtype);
    BackwardPlan p{};
    plan_two(W.elem, M, N, K, gated ? 2 : 1, &p.dx, &p.dw);
    p.none = p.dx.ti == 0;
    Layout l;
    p.dz = l.take((size_t)M * W.padded(N) * W.elem * (gated ? 2 : 1));
    if (W.odd(K)) {
        p.x = l.take((size_t)M * W.padded(K) * W.elem);
        p.w = l.take((size_t)N * W.padded(K) * W.elem * (gated ? 2 : 1));
    }
    p.part_x = l.take(p.dx.part_bytes);
    p.part_w = l.take(p.dw.part_bytes);
    // column sums: enough blocks of rows to fill the device, no block of fewer rows than a workgroup takes at once
    const int vecs = W.padded(N) / W.E;
    p.tw = 1;
    while (p.tw < 64 && p.tw < vecs) p.tw *= 2;
    const long long across = (vecs + p.tw - 1) / p.tw, least = 4ll * (kThreads / p.tw);
    long long blocks = 1024 / across > 1 ? 1024 / across : 1;
    if (blocks > (M + least - 1) / least) blocks = (M + least - 1) / least;
    if (blocks < 1) blocks = 1;
    p.sum_rows = (int)((M + blocks - 1) / blocks);
    p.sum_blocks = p.sum_rows ? (int)((M + p.sum_rows - 1) / p.sum_rows) : 0;
    if (!gated) p.sums = l.take((size_t)p.sum_blocks * N * sizeof(float));
    p.bytes = l.at;
    return p;
}

size_t workspace_of(long long M, int N, int K, int dtype, bool gated, bool backward)
{
    size_t bytes;
    if (backward) {
        const BackwardPlan p = plan_backward(M, N, K, dtype, gated);
        if (p.none) return 0;
        bytes = p.bytes;
    } else {
        const ForwardPlan p = plan_forward(M, N, K, dtype, gated);
        if (p.none) return 0;
        bytes = p.bytes;
    }
    // (256 says that none is needed: a program may then pass none)
    return bytes == 0 ? 256 : bytes > 256 ? bytes : 512;
}

cgbn_status check_workspace(size_t need, const void* workspace, size_t have)
{
    if (need == 0) return CGBN_OK;
    if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || have < need) return CGBN_ERR_WORKSPACE;
    return CGBN_OK;
}

// the operands of a call that are laid out anew, one after the other
struct Pads {
    PadArgs A;
    int count;
    Pads() { std::memset(this, 0, sizeof(*this)); }
    // (three at the most: x and a gated pair's weights)
    const void* add(const void* src, void* dst, long long rows, int chunks)
    {
        A.src[count] = src;
        A.dst[count] = dst;
        for (int k = 2; k > count; --k) A.end[k] += rows * chunks;
        A.end[count++] += rows * chunks;
        return dst;
    }
    template <typename T> hipError_t launch(int n, int np, hipStream_t st)
    {
        if (count == 0) return hipSuccess;
        A.n = n;
        A.np = np;
        hipLaunchKernelGGL(pad_rows<T>, grid_of((A.end[2] + kThreads - 1) / kThreads), dim3(kThreads), 0, st, A);
        return hipGetLastError();
    }
};

template <typename T, bool GATED> hipError_t launch_rows(const GemmArgs& G, hipStream_t st)
{
    const dim3 grid((unsigned)((G.J + 15) / 16), (unsigned)G.splits);
    // 16 wavefronts, each with all of its loads in flight at once or twice, where there are steps for them: 8.0 against 8.5 us with 8 of
    // them (one row, 4096 x 4096); with few steps they only wait for each other: 3.3 with 4 against 3.6 us (1024 x 1024)
    const bool many = (long long)G.R * (int)sizeof(T) >= 32 * 128;
    const bool half = sizeof(T) == 2 && G.R % 2 != 0;
#define CGBN_ROWS(FM_, NW_)                                                                                             \
    do {                                                                                                                \
        if (sizeof(T) == 2 && half) hipLaunchKernelGGL((gemm_rows<T, GATED, FM_, NW_, sizeof(T) == 2>), grid, dim3(NW_ * kWave), 0, st, G); \
        else hipLaunchKernelGGL((gemm_rows<T, GATED, FM_, NW_, false>), grid, dim3(NW_ * kWave), 0, st, G);              \
    } while (0)
    if (G.I <= 16 && many && sizeof(T) == 4) CGBN_ROWS(1, 8);          // 16.9 against 18.3 us (8 rows, 4096 x 4096)
    else if (G.I <= 16 && many) CGBN_ROWS(1, 16);
    else if (G.I <= 16) CGBN_ROWS(1, 4);
    else if constexpr (!GATED) CGBN_ROWS(2, 16);
#undef CGBN_ROWS
    return hipGetLastError();
}

template <typename T, bool GATED>
cgbn_status forward(GemmArgs G, const ForwardPlan& p, char* ws, hipStream_t st)
{
    const int K = G.R;
    const Widths W(sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16);
    G.segs = G.batch = 1;
    G.lda = G.ldb = K;
    G.ldc = G.J;
    G.part = reinterpret_cast<float*>(ws + p.part);
    if (p.rows) {
        G.splits = p.g.splits;
        G.per = p.g.per;
        CGBN_HIP((launch_rows<T, GATED>(G, st)));
        if (G.splits > 1) CGBN_HIP((launch_join<T, GATED>(G, st)));
        return CGBN_OK;
    }
    if (W.odd(K)) {
        const int kp = W.padded(K), chunks = kp / W.E;
        Pads pads;
        G.A[0] = pads.add(G.A[0], ws + p.x, G.I, chunks);
        for (int k = 0; k < (GATED ? 2 : 1); ++k) G.B[k] = pads.add(G.B[k], ws + p.w + (size_t)k * G.J * kp * sizeof(T), G.J, chunks);
        CGBN_HIP(pads.launch<T>(K, kp, st));
        G.lda = G.ldb = kp;
    }
    CGBN_HIP((launch_gemm<T, FORM_NT, GATED>(p.g, G, st)));
    return CGBN_OK;
}

// dx = dz W (two pairs: summed) and dW = dz^T x (two: side by side), dz rows of `ldz` elements
template <typename T>
cgbn_status products(const void* const dz[2], int ldz, int pairs, const void* x, const void* const w[2], long long M, int N, int K, void* dx,
                     void* const dw[2], const BackwardPlan& p, char* ws, hipStream_t st)
{
    const Widths W(sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16);
    const int kp = W.padded(K);
    Pads pads;
    GemmArgs X, G;              // dx, dW
    std::memset(&X, 0, sizeof(X));
    X.J = K;
    X.lda = ldz;
    X.ldb = kp;
    X.ldc = K;
    G = X;
    for (int k = 0; k < pairs; ++k) X.A[k] = G.A[k] = dz[k];
    if (dx) {
        for (int k = 0; k < pairs; ++k) X.B[k] = W.odd(K) ? pads.add(w[k], ws + p.w + (size_t)k * N * kp * sizeof(T), N, kp / W.E) : w[k];
        X.C[0] = dx;
        X.I = (int)M;
        X.R = N;
        X.segs = pairs;
        X.batch = 1;
        X.part = reinterpret_cast<float*>(ws + p.part_x);
    }
    if (dw[0]) {
        if (W.odd(K)) x = pads.add(x, ws + p.x, M, kp / W.E);
        for (int k = 0; k < pairs; ++k) {
            G.B[k] = x;
            G.C[k] = dw[k];
        }
        G.I = N;
        G.R = (int)M;
        G.segs = 1;
        G.batch = pairs;
        G.part = reinterpret_cast<float*>(ws + p.part_w);
    }
    CGBN_HIP(pads.launch<T>(K, kp, st));
    if (dx && dw[0]) CGBN_HIP(launch_two<T>(p.dx, X, p.dw, G, st));
    else if (dx) CGBN_HIP((launch_gemm<T, FORM_NN, false>(p.dx, X, st)));
    else if (dw[0]) CGBN_HIP((launch_gemm<T, FORM_TN, false>(p.dw, G, st)));
    return CGBN_OK;
}

template <typename T> hipError_t zero(void* p, long long n, hipStream_t st)
{
    if (!p || n == 0) return hipSuccess;
    hipLaunchKernelGGL(fill_zero<T>, grid_of((n + kThreads - 1) / kThreads), dim3(kThreads), 0, st, static_cast<T*>(p), n);
    return hipGetLastError();
}

template <typename T>
cgbn_status linear_backward(const void* dy, const void* x, const void* w, const void* saved, long long M, int N, int K, int act, void* dx, void* dw,
                            float* dbias, void* dresidual, char* ws, hipStream_t st)
{
    if (M == 0) {
        CGBN_HIP(zero<T>(dw, (long long)N * K, st));
        CGBN_HIP(zero<float>(dbias, N, st));
        return CGBN_OK;
    }
    const Widths W(sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16);
    const int dtype = sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16;
    const BackwardPlan p = plan_backward(M, N, K, dtype, false);
    const int np = W.padded(N);
    const void* dz = dy;
    const bool products_follow = dx || dw, changes = act != ACT_NONE || W.odd(N);
    DzArgs A;
    std::memset(&A, 0, sizeof(A));
    if (dresidual && dresidual != dy && !W.odd(N)) {
        A.dz = dresidual;                         // dz is what the residual's gradient is: one buffer serves both
        dz = dresidual;
    } else {
        if (products_follow && changes) {
            A.dz = ws + p.dz;
            dz = ws + p.dz;
        }
        // (in place: an element is read before the same thread writes it)
        if (dresidual && (dresidual != dy || act != ACT_NONE)) A.dresidual = dresidual;
    }
    if (A.dz || A.dresidual || dbias) {
        A.dy = dy;
        A.saved = act == ACT_NONE ? nullptr : saved;
        A.part = dbias ? reinterpret_cast<float*>(ws + p.sums) : nullptr;
        A.M = M; A.N = N; A.ld = np; A.act = act;
        A.tw = p.tw; A.rows = p.sum_rows;
        const int vecs = np / W.E;
        const dim3 grid((unsigned)((vecs + p.tw - 1) / p.tw), (unsigned)p.sum_blocks);
        if (W.odd(N)) hipLaunchKernelGGL((linear_dz<T, true>), grid, dim3(kThreads), 0, st, A);
        else hipLaunchKernelGGL((linear_dz<T, false>), grid, dim3(kThreads), 0, st, A);
        CGBN_HIP(hipGetLastError());
        if (dbias) {
            hipLaunchKernelGGL(column_sums, dim3((unsigned)((N + 15) / 16)), dim3(kSumThreads), 0, st, A.part, p.sum_blocks, N, N, dbias, N, nullptr);
            CGBN_HIP(hipGetLastError());
        }
    }
    const void *dzs[2] = {dz, nullptr}, *ws_[2] = {w, nullptr};
    void* dws[2] = {dw, nullptr};
    return products<T>(dzs, np, 1, x, ws_, M, N, K, dx, dws, p, ws, st);
}

template <typename T>
cgbn_status gated_backward(const void* dh, const void* x, const void* wg, const void* wu, const void* gate, const void* up, long long M, int F, int K,
                           int act, void* dx, void* dwg, void* dwu, char* ws, hipStream_t st)
{
    if (M == 0) {
        CGBN_HIP(zero<T>(dwg, (long long)F * K, st));
        CGBN_HIP(zero<T>(dwu, (long long)F * K, st));
        return CGBN_OK;
    }
    const Widths W(sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16);
    const BackwardPlan p = plan_backward(M, F, K, sizeof(T) == 4 ? CGBN_F32 : CGBN_BF16, true);
    const int fp = W.padded(F);
    char* dg = ws + p.dz;
    char* du = dg + (size_t)M * fp * sizeof(T);
    const GateArgs A = {dh, gate, up, dg, du, M, F, fp, act};
    const long long ids = M * (fp / W.E), groups = (ids + kThreads - 1) / kThreads;
    const dim3 grid((unsigned)(groups < 8192 ? groups : 8192));
    hipLaunchKernelGGL(gated_dz<T>, grid, dim3(kThreads), 0, st, A);
    CGBN_HIP(hipGetLastError());
    const void *dzs[2] = {dg, du}, *ws_[2] = {wg, wu};
    void* dws[2] = {dwg, dwu};
    return products<T>(dzs, fp, 2, x, ws_, M, F, K, dx, dws, p, ws, st);
}

}  // namespace
}  // namespace cgbn

using namespace cgbn;

extern "C" {

size_t cgbn_linear_workspace_bytes(long long M, int N, int K, cgbn_dtype dtype, int backward)
{
    if (check_sizes(M, N, K, dtype) != CGBN_OK) return 0;
    if (M == 0) return 256;
    return workspace_of(M, N, K, dtype, false, backward);
}

cgbn_status cgbn_linear_forward(const void* x, const void* w, const float* bias, const void* residual, long long M, int N, int K, cgbn_activation act,
                                void* y, void* z, cgbn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!w || (M != 0 && (!x || !y))) return CGBN_ERR_NULL;          // (no rows, no tensors)
    CGBN_TRY(check_sizes(M, N, K, dtype));
    if (act < CGBN_ACT_NONE || act > CGBN_ACT_SILU) return CGBN_ERR_ACTIVATION;
    if (M == 0) return CGBN_OK;
    if (!aligned16(x) || !aligned16(w) || !aligned16(y) || !aligned16(residual) || !aligned16(z)) return CGBN_ERR_ALIGN;
    if (y == z || y == x || z == x || y == w || z == w || (bias && (y == bias || z == bias))) return CGBN_ERR_ALIAS;
    const ForwardPlan p = plan_forward(M, N, K, dtype, false);
    if (p.none) return CGBN_ERR_SHAPE;
    CGBN_TRY(check_workspace(p.bytes, workspace, workspace_bytes));
    GemmArgs G;
    std::memset(&G, 0, sizeof(G));
    G.A[0] = x; G.B[0] = w; G.C[0] = y; G.Z[0] = z; G.bias = bias; G.residual = residual;
    G.I = (int)M; G.J = N; G.R = K; G.act = act;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == CGBN_F32 ? forward<float, false>(G, p, ws, st) : forward<bf16_t, false>(G, p, ws, st);
}

cgbn_status cgbn_linear_backward(const void* dy, const void* x, const void* w, const void* saved, long long M, int N, int K, cgbn_activation act,
                                 void* dx, void* dw, float* dbias, void* dresidual, cgbn_dtype dtype, void* workspace, size_t workspace_bytes,
                                 void* stream)
{
    if (!w || (M != 0 && (!dy || !x))) return CGBN_ERR_NULL;
    CGBN_TRY(check_sizes(M, N, K, dtype));
    if (act < CGBN_ACT_NONE || act > CGBN_ACT_SILU) return CGBN_ERR_ACTIVATION;
    if (act != CGBN_ACT_NONE && M != 0 && !saved) return CGBN_ERR_NULL;
    if (!aligned16(dy) || !aligned16(x) || !aligned16(w) || !aligned16(saved) || !aligned16(dx) || !aligned16(dw) || !aligned16(dresidual))
        return CGBN_ERR_ALIGN;
    if (M != 0 && dx && (dx == dw || dx == dresidual || dx == dy || dx == x || dx == w)) return CGBN_ERR_ALIAS;
    if (M != 0 && dw && (dw == dresidual || dw == dy || dw == x || dw == w)) return CGBN_ERR_ALIAS;
    if (M != 0 && dresidual && (dresidual == x || dresidual == w)) return CGBN_ERR_ALIAS;
    // (without rows, too: these are set to zero)
    if (dw && dw == w) return CGBN_ERR_ALIAS;
    if (dbias && (dbias == w || dbias == dw)) return CGBN_ERR_ALIAS;
    if (M != 0 && dbias && (dbias == dx || dbias == dresidual || dbias == dy || dbias == x || (act != CGBN_ACT_NONE && dbias == saved))) return CGBN_ERR_ALIAS;
    if (M > 0) {
        const BackwardPlan p = plan_backward(M, N, K, dtype, false);
        if (p.none) return CGBN_ERR_SHAPE;
        CGBN_TRY(check_workspace(p.bytes, workspace, workspace_bytes));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == CGBN_F32 ? linear_backward<float>(dy, x, w, saved, M, N, K, act, dx, dw, dbias, dresidual, ws, st)
                             : linear_backward<bf16_t>(dy, x, w, saved, M, N, K, act, dx, dw, dbias, dresidual, ws, st);
}

size_t cgbn_gated_workspace_bytes(long long M, int F, int K, cgbn_dtype dtype, int backward)
{
    if (check_sizes(M, F, K, dtype) != CGBN_OK) return 0;
    if (M == 0) return 256;
    return workspace_of(M, F, K, dtype, true, backward);
}

cgbn_status cgbn_gated_forward(const void* x, const void* w_gate, const void* w_up, long long M, int F, int K, cgbn_activation act, void* h,
                               void* gate, void* up, cgbn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (!w_gate || !w_up || (M != 0 && (!x || !h || !gate != !up))) return CGBN_ERR_NULL;
    CGBN_TRY(check_sizes(M, F, K, dtype));
    if (act < CGBN_ACT_NONE || act > CGBN_ACT_SILU) return CGBN_ERR_ACTIVATION;
    if (M == 0) return CGBN_OK;
    if (!aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(h) || !aligned16(gate) || !aligned16(up)) return CGBN_ERR_ALIGN;
    const void* const outs[3] = {h, gate, up};
    for (int k = 0; k < 3; ++k)
        if (outs[k] && (outs[k] == x || outs[k] == w_gate || outs[k] == w_up || outs[k] == outs[(k + 1) % 3])) return CGBN_ERR_ALIAS;
    const ForwardPlan p = plan_forward(M, F, K, dtype, true);
    if (p.none) return CGBN_ERR_SHAPE;
    CGBN_TRY(check_workspace(p.bytes, workspace, workspace_bytes));
    GemmArgs G;
    std::memset(&G, 0, sizeof(G));
    G.A[0] = x; G.B[0] = w_gate; G.B[1] = w_up; G.C[0] = h; G.Z[0] = gate; G.Z[1] = up;
    G.I = (int)M; G.J = F; G.R = K; G.act = act;
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == CGBN_F32 ? forward<float, true>(G, p, ws, st) : forward<bf16_t, true>(G, p, ws, st);
}

cgbn_status cgbn_gated_backward(const void* dh, const void* x, const void* w_gate, const void* w_up, const void* gate, const void* up, long long M,
                                int F, int K, cgbn_activation act, void* dx, void* dw_gate, void* dw_up, cgbn_dtype dtype, void* workspace,
                                size_t workspace_bytes, void* stream)
{
    if (!w_gate || !w_up || !dw_gate != !dw_up || (M != 0 && (!dh || !x || !gate || !up))) return CGBN_ERR_NULL;
    CGBN_TRY(check_sizes(M, F, K, dtype));
    if (act < CGBN_ACT_NONE || act > CGBN_ACT_SILU) return CGBN_ERR_ACTIVATION;
    if (!aligned16(dh) || !aligned16(x) || !aligned16(w_gate) || !aligned16(w_up) || !aligned16(gate) || !aligned16(up) || !aligned16(dx) ||
        !aligned16(dw_gate) || !aligned16(dw_up))
        return CGBN_ERR_ALIGN;
    const void* const outs[3] = {dx, dw_gate, dw_up};
    for (int k = 0; k < 3; ++k)
        if (outs[k] && (outs[k] == x || outs[k] == w_gate || outs[k] == w_up || outs[k] == dh || outs[k] == gate || outs[k] == up ||
                        outs[k] == outs[(k + 1) % 3]))
            return CGBN_ERR_ALIAS;
    if (M > 0) {
        const BackwardPlan p = plan_backward(M, F, K, dtype, true);
        if (p.none) return CGBN_ERR_SHAPE;
        CGBN_TRY(check_workspace(p.bytes, workspace, workspace_bytes));
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    char* ws = static_cast<char*>(workspace);
    return dtype == CGBN_F32 ? gated_backward<float>(dh, x, w_gate, w_up, gate, up, M, F, K, act, dx, dw_gate, dw_up, ws, st)
                             : gated_backward<bf16_t>(dh, x, w_gate, w_up, gate, up, M, F, K, act, dx, dw_gate, dw_up, ws, st);
}

}  // extern "C"
