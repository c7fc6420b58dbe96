// Attention of new tokens over a prefix that all requests share and over pages of their own, for gfx950.
//
//   o = sum over visible keys of softmax(scale q.k) v,   lse = log sum exp(scale q.k)
//
// The prefix's keys are the same for every row, so its products are formed with all requests' rows side by side: a workgroup takes a tile of rows (a
// row is one head of one token; the Hq / Hk heads that share keys lie side by side) and a range of keys, which it reads once for all of them.  A request's own keys are
// met by its own rows alone.  Both are split over ranges of keys where there are few rows; the parts carry their largest score m, the sum l of
// exp(score - m) and the products o, all in 32 bits, and are joined in a fixed order.
//
// One pass over the keys: scores of a tile, their largest, exponentials, and the products with v are formed before the next tile is read; o and l
// are scaled down when the largest score grows.  Scores are formed as K Q^T, so that a lane holds one row's scores for four
// neighbouring keys of each 16: rounded to bfloat16 they are, as they are, the second operand of V^T P^T, if the keys of two such
// tiles are dealt to the reduction in the order that the lanes hold them; V is read from LDS in the same order (bfloat16: by the reads that
// transpose 4 x 16 blocks).  No score crosses lanes but for its row's maximum and sum.
#pragma once

#include "cgbn_gemm.h"

namespace cgbn {

struct AttendArgs {
    const char *q, *k_pages, *v_pages;
    char* out;
    float* lse;                        // may be null
    float* part_o;                     // [parts][T][Hq][D], not divided by l
    float2* part_ml;                   // [parts][T][Hq]
    const int *rows, *lengths, *prefix_table, *table;
    long long ldq, ldo, T;             // elements from row to row
    int B, Hq, Hk, g, D, pages, page_bits, prefix, max_pages;
    int prefix_splits, prefix_per, own_splits;
    int prefix_tiles, own_tiles;       // tiles of rows
    int prefix_jobs, jobs;             // workgroups, those of the prefix first
    int whole;                         // a workgroup takes the prefix and then its request's own keys
    int direct;                        // there is one part: it is the result
    float scale;                       // times log2(e)
};

// T: element type; DP: D up to the next tile width; WR: wavefronts side by side in rows (the others side by side in keys); QT: 16-row tiles of a wavefront
template <typename T, int DP, int WR, int QT> struct Attend {
    static constexpr int EB = (int)sizeof(T), WK = 4 / WR, ROWS = WR * QT * 16;
    static constexpr int KW = (WK == 1 ? 128 : 64) / EB, KT = KW * WK;          // keys of a wavefront, of a tile
    static constexpr int KROW = DP * EB + 16, VROW = DP * EB + (EB == 2 ? 32 : 16);        // rows apart in banks, see the reads
    static constexpr int CH = DP * EB / 16, KS = DP * EB / 64, NT = KW / 16, ND = DP / 16;
    static constexpr int V0 = KT * KROW, FLAGS = V0 + KT * VROW, KEYS = FLAGS + KT * 4;
    static constexpr int MERGE = WK == 1 ? 0 : 4 * QT * 16 * (DP + 2) * 4;
    static constexpr int LDS = KEYS > MERGE ? KEYS : MERGE;
};

__device__ __forceinline__ bool finite16(uint32_t pair, int hi) { return ((pair >> (hi ? 16 : 0)) & 0x7f80u) != 0x7f80u; }
template <typename T> __device__ __forceinline__ bool all_finite(const u32x4& v)
{
    bool ok = true;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) ok = ok && finite16(v[k], 0) && finite16(v[k], 1);
        else ok = ok && (v[k] & 0x7f800000u) != 0x7f800000u;
    }
    return ok;
}
template <typename T> __device__ __forceinline__ u32x4 only_finite(u32x4 v)
{
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 2) v[k] = (finite16(v[k], 0) ? v[k] & 0xffffu : 0u) | (finite16(v[k], 1) ? v[k] & 0xffff0000u : 0u);
        else if ((v[k] & 0x7f800000u) == 0x7f800000u) v[k] = 0;
    }
    return v;
}

// address of a key's row of one head, or null where its page is none
template <typename T> __device__ __forceinline__ long long key_at(const AttendArgs& A, const int* table, int head, int key)
{
    const int page = table[key >> A.page_bits];
    if (page < 0 || page >= A.pages) return -1;
    return (((((long long)page * A.Hk + head) << A.page_bits) + (key & ((1 << A.page_bits) - 1))) * A.D) * (long long)sizeof(T);
}

// The first request whose tiles begin behind tile i, less one: request b's begin at floor(rows[b] g / ROWS) + b, which leaves room for all of them.
__device__ __forceinline__ long long tiles_before(const AttendArgs& A, int b, int rows_of_a_tile)
{
    const long long r = min(max((long long)A.rows[b], 0ll), A.T);
    return r * A.g / rows_of_a_tile + b;
}
__device__ __forceinline__ int request_of_tile(const AttendArgs& A, int i, int rows_of_a_tile)
{
    int lo = 0, hi = A.B;          // 64 places are looked at in each step
    const int lane = (int)threadIdx.x % kWave;
    while (hi - lo > 1) {
        const int step = (hi - lo + kWave - 1) / kWave, b = lo + lane * step;
        const unsigned long long in = __ballot(b < hi && tiles_before(A, b, rows_of_a_tile) <= i);
        const int n = __popcll(in);                      // (ascending: those that are in come first)
        const int at = lo + (n ? n - 1 : 0) * step;
        hi = min(hi, at + step);
        lo = at;
    }
    return __builtin_amdgcn_readfirstlane(lo);
}

template <typename T, int DP, int WR, int QT> __device__ void attend(const AttendArgs& A, char* lds, int id, bool prefix_job)
{
    typedef Attend<T, DP, WR, QT> C;
    const int tid = (int)threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave), wr = w % WR, wk = w / WR, col = lane & 15, grp = lane >> 4;
    lds_char* const tile = (lds_char*)lds;
    const int head = id % A.Hk;
    id /= A.Hk;

    // the rows of this workgroup: from r0 on, of `count`; token0: the token of row 0
    int r0, count, token0, length, fresh, split, b = 0;
    if (prefix_job) {
        r0 = id % A.prefix_tiles * C::ROWS;
        split = id / A.prefix_tiles;
        token0 = 0;
        fresh = A.rows ? (int)min(max((long long)A.rows[A.B], 0ll), A.T) : (int)A.T;
        length = 0;
    } else {
        split = id % A.own_splits;
        const int i = id / A.own_splits;
        if (A.rows) {
            b = request_of_tile(A, i, C::ROWS);
            token0 = (int)min(max((long long)A.rows[b], 0ll), A.T);
            fresh = max((int)min((long long)A.rows[b + 1], A.T) - token0, 0);
            r0 = (i - (int)tiles_before(A, b, C::ROWS)) * C::ROWS;
        } else {
            const int per = (A.g + C::ROWS - 1) / C::ROWS;
            b = i / per;
            token0 = b;
            fresh = 1;
            r0 = (i - b * per) * C::ROWS;
        }
        length = A.max_pages ? (int)min((long long)max(A.lengths[b], 0), (long long)A.max_pages << A.page_bits) : 0;
    }
    count = fresh * A.g;                  // (T * Hq stays below 2^31)
    if (r0 < 0 || r0 >= count) return;

    long long row[QT];                    // of [T][Hq]
    int sees[QT];                         // own keys
    u32x4 Q[QT][C::KS];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = r0 + (wr * QT + t) * 16 + col;
        const bool in = r < count;
        const int token = in ? r / A.g : 0, h = in ? r - token * A.g : 0;
        row[t] = in ? (long long)(token0 + token) * A.Hq + head * A.g + h : -1;
        sees[t] = in ? min(max(length - fresh + token + 1, 0), length) : 0;
        const char* const at = A.q + ((token0 + token) * A.ldq + (long long)(head * A.g + h) * A.D) * C::EB;
#pragma unroll
        for (int s = 0; s < C::KS; ++s) {
            const int c = s * 64 + grp * 16;
            Q[t][s] = u32x4{0, 0, 0, 0};
            if (in && c < A.D * C::EB) Q[t][s] = *reinterpret_cast<const u32x4*>(at + c);
        }
    }

    f32x4 O[QT][C::ND];
    float m[QT], l[QT];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        m[t] = -INFINITY;
        l[t] = 0.f;
#pragma unroll
        for (int d = 0; d < C::ND; ++d) O[t][d] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int dirty_from = 0, dirty_to = 0;     // own keys whose infinities and NaN stay out of the products, see below
    for (int own = prefix_job || A.whole ? 0 : 1; own < (prefix_job ? 1 : 2); ++own) {
        const int* const table = own ? A.table + (long long)b * A.max_pages : A.prefix_table;
        int begin = 0, end, least;        // this workgroup's keys; those below `least` are seen by all of its rows
        if (!own) {
            if (A.whole) {
                end = A.prefix;
            } else {
                begin = split * A.prefix_per;
                end = min(begin + A.prefix_per, A.prefix);
            }
            least = end;
        } else {
            const int last = min(r0 + C::ROWS, count) - 1;
            end = min(max(length - fresh + last / A.g + 1, 0), length);
            least = min(max(length - fresh + r0 / A.g + 1, 0), length);
            if (A.own_splits > 1) {
                const int per = ((end + A.own_splits - 1) / A.own_splits + 127) / 128 * 128;
                begin = min(split * per, end);
                end = min(begin + per, end);
            }
        }
        for (int key0 = begin; key0 < end; key0 += C::KT) {
            __syncthreads();
            const bool edge = own && least < end && key0 + C::KT > least;
            int bad = 0;
            for (int i = tid; i < C::KT * C::CH; i += kThreads) {
                const int r = i / C::CH, c = i % C::CH, key = key0 + r;
                const long long at = key < end ? key_at<T>(A, table, head, key) : -1;
                u32x4 k = {0, 0, 0, 0}, v = {0, 0, 0, 0};
                if (at >= 0 && c * 16 < A.D * C::EB) {
                    k = *reinterpret_cast<const u32x4*>(A.k_pages + at + c * 16);
                    v = *reinterpret_cast<const u32x4*>(A.v_pages + at + c * 16);
                }
                *reinterpret_cast<u32x4*>(lds + r * C::KROW + c * 16) = k;
                *reinterpret_cast<u32x4*>(lds + C::V0 + r * C::VROW + c * 16) = v;
                if (c == 0) *reinterpret_cast<int*>(lds + C::FLAGS + r * 4) = at < 0;
                if (edge) bad |= !all_finite<T>(v);
            }
            // A product with a score of zero would carry an infinity or a NaN of v to rows that do not see its key.  Where rows of the tile see
            // different keys such values are left out of the products and added to the rows that do at the end.
            const bool dirty = edge ? __syncthreads_or(bad) : (__syncthreads(), false);
            if (dirty) {
                if (dirty_to == 0) dirty_from = key0;
                dirty_to = end;
            }

            const int k0 = wk * C::KW;
            f32x4 S[QT][C::NT];
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int n = 0; n < C::NT; ++n) S[t][n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int s = 0; s < C::KS; ++s)
#pragma unroll
                for (int n = 0; n < C::NT; ++n) {
                    const u32x4 k = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + (k0 + n * 16 + col) * C::KROW + s * 64 + grp * 16);
#pragma unroll
                    for (int t = 0; t < QT; ++t) S[t][n] = multiply<T>(k, Q[t][s], S[t][n]);
                }

            u32x4 P[QT][C::EB == 2 ? C::NT / 2 : C::NT];
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                float top = -INFINITY;
#pragma unroll
                for (int n = 0; n < C::NT; ++n) {
                    const u32x4 none = *reinterpret_cast<const __attribute__((address_space(3))) u32x4*>(tile + C::FLAGS + (k0 + n * 16 + grp * 4) * 4);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const int key = key0 + k0 + n * 16 + grp * 4 + e;
                        const bool hidden = none[e] || (own && key >= sees[t]);
                        S[t][n][e] = hidden ? -INFINITY : S[t][n][e] * A.scale;
                        top = fmaxf(top, S[t][n][e]);
                    }
                }
                top = fmaxf(top, __shfl_xor(top, 16));
                top = fmaxf(top, __shfl_xor(top, 32));
                const float most = fmaxf(m[t], top), from = most == -INFINITY ? 0.f : most, down = __builtin_amdgcn_exp2f(m[t] - from);
                m[t] = most;
                float sum = 0.f;
#pragma unroll
                for (int n = 0; n < C::NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        S[t][n][e] = __builtin_amdgcn_exp2f(S[t][n][e] - from);
                        sum += S[t][n][e];
                    }
                l[t] = l[t] * down + sum;
#pragma unroll
                for (int d = 0; d < C::ND; ++d) O[t][d] *= down;
                // bfloat16: the weights are rounded to 8 bits for the products (off by at most 2^-8 of themselves, with no preferred sign); their sum is not
                if constexpr (C::EB == 2) {
#pragma unroll
                    for (int n = 0; n < C::NT / 2; ++n)
                        P[t][n] = u32x4{f32x2_to_bf16x2(S[t][2 * n][0], S[t][2 * n][1]), f32x2_to_bf16x2(S[t][2 * n][2], S[t][2 * n][3]),
                                        f32x2_to_bf16x2(S[t][2 * n + 1][0], S[t][2 * n + 1][1]), f32x2_to_bf16x2(S[t][2 * n + 1][2], S[t][2 * n + 1][3])};
                } else {
#pragma unroll
                    for (int n = 0; n < C::NT; ++n)
                        P[t][n] = u32x4{__float_as_uint(S[t][n][0]), __float_as_uint(S[t][n][1]), __float_as_uint(S[t][n][2]), __float_as_uint(S[t][n][3])};
                }
            }
#pragma unroll
            for (int n = 0; n < (C::EB == 2 ? C::NT / 2 : C::NT); ++n)
#pragma unroll
                for (int d = 0; d < C::ND; ++d) {
                    u32x4 v;
                    if constexpr (C::EB == 2) {
                        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
                        const lds_char* const p = tile + C::V0 + (k0 + n * 32 + grp * 4 + (col >> 2)) * C::VROW + d * 32 + (col & 3) * 8;
                        const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
                        const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * C::VROW)));
                        v = u32x4{lo.x, lo.y, hi.x, hi.y};
                    } else {
                        typedef const __attribute__((address_space(3))) uint32_t lds_u32;
                        const lds_char* const p = tile + C::V0 + (k0 + n * 16 + grp * 4) * C::VROW + (d * 16 + col) * 4;
                        v = u32x4{*(lds_u32*)p, *(lds_u32*)(p + C::VROW), *(lds_u32*)(p + 2 * C::VROW), *(lds_u32*)(p + 3 * C::VROW)};
                    }
                    if (dirty) v = only_finite<T>(v);
#pragma unroll
                    for (int t = 0; t < QT; ++t) O[t][d] = multiply<T>(v, P[t][n], O[t][d]);
                }
        }
    }

#pragma unroll
    for (int t = 0; t < QT; ++t) {
        l[t] += __shfl_xor(l[t], 16);
        l[t] += __shfl_xor(l[t], 32);
    }

    // what was left out of the products: a row's four values from d on of a key that it sees
    auto left_out = [&](int key, int d) {
        f32x4 v = {0.f, 0.f, 0.f, 0.f};
        const long long at = key_at<T>(A, A.table + (long long)b * A.max_pages, head, key);
        if (at < 0 || d >= A.D) return v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = Elem<T>::load1(reinterpret_cast<const T*>(A.v_pages + at) + d + e);
            v[e] = fabsf(x) < INFINITY ? 0.f : x;
        }
        return v;
    };
    // one row's four values from d on: to the result or to this part's place
    const long long part = prefix_job ? split : A.prefix_splits + split;
    auto store = [&](long long r, int d, f32x4 o, float mm, float ll) {
        if (r < 0) return;
        if (d < A.D) {
            if (A.direct) {
                const float by = ll == 0.f ? 0.f : 1.f / ll;
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] = ll == 0.f ? 0.f : o[e] * by;
                const long long token = r / A.Hq;
                T* const to = reinterpret_cast<T*>(A.out) + token * A.ldo + (r - token * A.Hq) * A.D + d;
                if constexpr (C::EB == 2) *reinterpret_cast<uint2*>(to) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
                else *reinterpret_cast<f32x4*>(to) = o;
            } else {
                *reinterpret_cast<f32x4*>(A.part_o + (part * A.T * A.Hq + r) * A.D + d) = o;
            }
        }
        if (d == 0) {
            if (!A.direct) A.part_ml[part * A.T * A.Hq + r] = make_float2(mm, ll);
            else if (A.lse) A.lse[r] = ll == 0.f ? -INFINITY : 0.6931471805599453f * (mm + __builtin_amdgcn_logf(ll));
        }
    };
    if constexpr (C::WK == 1) {
        for (int key = dirty_from; key < dirty_to; ++key)
#pragma unroll
            for (int d = 0; d < C::ND; ++d) {
                const f32x4 v = left_out(key, d * 16 + grp * 4);
#pragma unroll
                for (int t = 0; t < QT; ++t)
                    if (key < sees[t]) O[t][d] += v;
            }
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int d = 0; d < C::ND; ++d) store(row[t], d * 16 + grp * 4, O[t][d], m[t], l[t]);
    } else {
        // the wavefronts' parts, in order
        constexpr int RW = QT * 16;
        float* const o = reinterpret_cast<float*>(lds);
        float* const ml = o + 4 * RW * DP;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int d = 0; d < C::ND; ++d) *reinterpret_cast<f32x4*>(o + ((wk * RW + t * 16 + col) * DP + d * 16 + grp * 4)) = O[t][d];
            if (grp == 0) {
                ml[(wk * RW + t * 16 + col) * 2] = m[t];
                ml[(wk * RW + t * 16 + col) * 2 + 1] = l[t];
            }
        }
        __syncthreads();
        for (int i = tid; i < RW * (DP / 4); i += kThreads) {
            const int r = i / (DP / 4), d = i % (DP / 4) * 4;
            float top = -INFINITY, ll = 0.f;
#pragma unroll
            for (int k = 0; k < C::WK; ++k) top = fmaxf(top, ml[(k * RW + r) * 2]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < C::WK; ++k) {
                if (ml[(k * RW + r) * 2 + 1] == 0.f) continue;          // (no key: what o holds is no sum)
                const float f = __builtin_amdgcn_exp2f(ml[(k * RW + r) * 2] - top);
                ll += f * ml[(k * RW + r) * 2 + 1];
                sum += f * *reinterpret_cast<const f32x4*>(o + (k * RW + r) * DP + d);
            }
            const int at = r0 + r;
            const int token = at / A.g;
            const long long to = at < count ? (long long)(token0 + token) * A.Hq + head * A.g + (at - token * A.g) : -1;
            for (int key = dirty_from; key < min(dirty_to, length - fresh + token + 1); ++key) sum += left_out(key, d);
            store(to, d, sum, top, ll);
        }
    }
}

// WP: the row wavefronts of a prefix tile; WO: of a tile of one request's rows.  One launch for both.
template <typename T, int DP, int WP, int QP, int WO, int QO> __global__ __launch_bounds__(kThreads) void attend_keys(const AttendArgs A)
{
    constexpr int P = Attend<T, DP, WP, QP>::LDS, O = Attend<T, DP, WO, QO>::LDS;
    __shared__ __attribute__((aligned(1024))) char lds[P > O ? P : O];
    const int id = (int)blockIdx.x;
    if constexpr (WP == WO && QP == QO) {
        attend<T, DP, WP, QP>(A, lds, id < A.prefix_jobs ? id : id - A.prefix_jobs, id < A.prefix_jobs);
    } else {
        if (id < A.prefix_jobs) attend<T, DP, WP, QP>(A, lds, id, true);
        else attend<T, DP, WO, QO>(A, lds, id - A.prefix_jobs, false);
    }
}

// Joins a row's parts, a wavefront to a row, in their order.
template <typename T> __global__ __launch_bounds__(kThreads) void attend_join(const AttendArgs A)
{
    const long long r = (long long)blockIdx.x * (kThreads / kWave) + threadIdx.x / kWave, token = r / A.Hq;
    const long long end = A.rows ? min(max((long long)A.rows[A.B], 0ll), A.T) : A.T;
    if (token >= end) return;
    const int lane = (int)threadIdx.x % kWave, parts = A.prefix_splits + A.own_splits, d = lane * 4;
    float top = -INFINITY, sum = 0.f;
    for (int p = 0; p < parts; ++p) {
        const float2 ml = A.part_ml[p * A.T * A.Hq + r];
        if (ml.y != 0.f) top = fmaxf(top, ml.x);
    }
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p = 0; p < parts; ++p) {
        const float2 ml = A.part_ml[p * A.T * A.Hq + r];
        if (ml.y == 0.f) continue;
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        sum += f * ml.y;
        if (d < A.D) o += f * *reinterpret_cast<const f32x4*>(A.part_o + (p * A.T * A.Hq + r) * A.D + d);
    }
    if (d < A.D) {
        const float by = 1.f / sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = sum == 0.f ? 0.f : o[e] * by;
        T* const to = reinterpret_cast<T*>(A.out) + token * A.ldo + (r - token * A.Hq) * A.D + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
        else *reinterpret_cast<f32x4*>(to) = o;
    }
    if (lane == 0 && A.lse) A.lse[r] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (top + __builtin_amdgcn_logf(sum));
}

// ways: which tiles the rows go in, see plan()
enum { WAY_16_16 = 0, WAY_32_16 = 1, WAY_128_16 = 2, WAY_32_32 = 3, WAY_128_32 = 4, WAY_128_128 = 5, WAYS = 6 };
constexpr int kPrefixRows[WAYS] = {16, 32, 128, 32, 128, 128}, kOwnRows[WAYS] = {16, 16, 16, 32, 32, 128};

template <typename T> cgbn_status launch_attend(const AttendArgs& A, int way, hipStream_t st);

}  // namespace cgbn
