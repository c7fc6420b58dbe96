// Attention of new tokens over a prefix that all requests share and over pages of their own, for gfx950.
//
//   o = sum over visible keys of softmax(scale q.k) v,   lse = log sum exp(scale q.k)
//
// The prefix's keys are the same for every row, so its products are formed with all requests' rows side by side: a workgroup takes a tile of rows (a
// row is one head of one token; the Hq / Hk heads that share keys lie side by side) and a range of keys, which it reads once for all of them.  A request's own keys are
// met by its own rows alone.  Both are split over ranges of keys where there are few rows; the parts carry a score m near their largest, the sum l of
// exp(score - m) and the products o, all in 32 bits, and are joined in a fixed order.
//
// One pass over the keys: scores of a tile, their largest, exponentials, and the products with v are formed before the next tile is read; o and l
// are scaled down when the largest score grows.  Scores are formed as K Q^T, so that a lane holds one row's scores for four
// neighbouring keys of each 16: rounded to bfloat16 they are, as they are, the second operand of V^T P^T, if the keys of two such
// tiles are dealt to the reduction in the order that the lanes hold them; V is read from LDS in the same order (bfloat16: by the reads that
// transpose 4 x 16 blocks).  No score crosses lanes but for its row's maximum and sum.
//
// Keys and values go from memory to LDS directly, the next tile's while one is multiplied; scores are one tile ahead of values, so that the vector unit
// forms a tile's weights while the matrix cores form the next one's scores.  Without that order 2919 us for what takes 552 (16 requests of up to 512 new tokens
// behind 8191, 32 heads of 128 on 8, bfloat16).
//
// What bounds it: few rows the read of the keys (4 requests of up to 131072, 1.67 GB, 295 us, 5.7 TB/s, more than a copy's rate); many rows
// the products and the weights' arithmetic together, 960 TF, two thirds of the 1450 that the library's large product reaches on the same card: the matrix cores are busy 41 %
// of the time, the vector unit about as long, at 1.9 to 2.1 GHz, and no single part of the loop taken out gains more than a fifth.  64 rows of
// each key head behind 32768 keys with up to 2048 of their own are both, 99 us for 68 of reading.  Float with few rows reading too (stream(), below); with more the float
// products, a fifth of the matrix cores' bfloat16 rate at best.  Small calls the launch and five trips to memory one after the other, 8 us.
#pragma once

#include "cgbn_gemm.h"

namespace cgbn {

struct AttendArgs {
    const char *q, *k_pages, *v_pages;
    char* out;
    float* lse;                        // may be null
    float* part_o;                     // [parts][T][Hq][D], not divided by l; where own keys are dealt theirs are behind the prefix's, [workgroup][row of a tile][D]
    float2* part_ml;                   // the same of two
    const int *rows, *lengths, *prefix_table, *table;
    long long ldq, ldo, T;             // elements from row to row
    int B, Hq, Hk, g, D, pages, page_bits, prefix, max_pages;
    int prefix_splits, prefix_per;
    int own_splits, own_least;         // parts of a request's own keys at most, and keys of a part at least
    int own_groups;                    // workgroups for them
    float* dense;                      // workspace: parts to a key, as the lengths have it, see deal(); [B]: a request's first workgroup
    int* own_first;
    int prefix_tiles, own_tiles;       // tiles of rows
    int prefix_jobs, jobs;             // workgroups, those of the prefix first
    int whole;                         // a workgroup takes the prefix and then its request's own keys
    int cut, tail_splits;              // whole: from tile-and-head `cut` on workgroups share one, by its keys; their parts are [tile][part][row] from `cut` on
    int direct;                        // there is one part: it is the result (whole: but for the last ones, see `cut`)
    float scale;                       // times log2(e)
};

// How many rows a tile has, and how it is dealt to the four wavefronts: FEW (one row's worth: a request's heads), SOME, MANY.  `line`: bytes from key to key
// in LDS.  Wavefronts side by side in keys (wk of them) read each key once from LDS, and have sums to join at the end; side by side in rows (wr) they
// read the same keys.  A tile's keys and values are 32 KiB, two of them in LDS, so that two workgroups share a compute unit.
// STREAM, float alone: up to four rows without LDS and matrix products, see stream() below.
enum { STREAM = 0, FEW = 1, SOME = 2, MANY = 3 };
constexpr int kStreamRows = 4;
constexpr bool may_stream(int D, int elem) { return elem == 4 && D <= 128; }
constexpr int width_of(int D) { return D <= 32 ? 32 : D <= 64 ? 64 : D <= 96 ? 96 : D <= 128 ? 128 : D <= 192 ? 192 : 256; }
constexpr int line_of(int D, int elem) { return D * elem <= 64 ? 64 : D * elem <= 128 ? 128 : D * elem <= 256 ? 256 : D * elem <= 512 ? 512 : 1024; }
constexpr int keys_of(int kind, int line) { return line >= 256 ? 16384 / line : kind == MANY ? 64 : 128; }
constexpr int wk_of(int kind, int line) { return kind == MANY || line == 1024 ? 1 : line == 512 ? 2 : 4; }
// 16-row tiles of a wavefront: what is left of its registers decides where rows are long
constexpr int qt_of(int kind, int line, int elem) { return kind == FEW ? 1 : line <= 256 ? 2 : kind == MANY && line == 512 && elem == 4 ? 2 : 1; }
constexpr int rows_of(int kind, int line, int elem) { return kind == STREAM ? kStreamRows : 4 / wk_of(kind, line) * qt_of(kind, line, elem) * 16; }

constexpr int kPlaces = 1024;          // pages whose addresses a workgroup has at hand

// T: element type; DP: D up to the next tile width
template <typename T, int DP, int KIND> struct Attend {
    static constexpr int EB = (int)sizeof(T), LINE = line_of(DP, EB), WK = wk_of(KIND, LINE), WR = 4 / WK, QT = qt_of(KIND, LINE, EB), ROWS = rows_of(KIND, LINE, EB);
    static constexpr int KT = keys_of(KIND, LINE), KW = KT / WK;                 // keys of a tile, of a wavefront
    static constexpr int CH = LINE / 16, PASS = kThreads / CH, PASSES = KT / PASS;         // chunks of a line; keys of a pass of the workgroup's loads
    static constexpr int KS = DP * EB / 64, NT = KW / 16, ND = DP / 16, NP = EB == 2 && NT > 1 ? NT / 2 : NT;
    static constexpr int HALF = KT * LINE, STAGE = 2 * HALF, PLACES = 2 * STAGE;
    static constexpr int MERGE = WK == 1 ? 0 : 4 * QT * 16 * (DP + 2) * 4;
    static constexpr int LDS = PLACES + kPlaces * 8 > MERGE ? PLACES + kPlaces * 8 : MERGE;
    static_assert(ROWS == WR * QT * 16 && KT % PASS == 0 && KW % 16 == 0 && KT <= 128, "");
};

// 16 bytes a lane to LDS at `lds` + 16 * lane, from an address of the lane's own; see dma16
__device__ __forceinline__ void dma16_from(uint32_t lds, const char* from)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(from) : "memory");
}

// The larger of the four lanes that hold a row: lanes 16 and 32 apart, by the instructions that swap rows of 16 lanes and halves
__device__ __forceinline__ float row_max(float v)
{
    typedef unsigned u32x2_hw __attribute__((ext_vector_type(2)));
    const u32x2_hw a = __builtin_bit_cast(u32x2_hw, __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    v = fmaxf(__uint_as_float(a.x), __uint_as_float(a.y));
    const u32x2_hw b = __builtin_bit_cast(u32x2_hw, __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false));
    return fmaxf(__uint_as_float(b.x), __uint_as_float(b.y));
}

// xor number of a key's line of 64 ... 1024 bytes: the 16 keys that a read of a fragment touches at once spread over all banks
template <int LINE> __device__ __forceinline__ int line_key(int key) { return LINE >= 256 ? key & 15 : LINE == 128 ? (key >> 1) & 7 : (key >> 2) & 3; }

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

// Tokens of request b's own that have a place in its row of the table: no other keys are looked at
__host__ __device__ __forceinline__ int tokens_of(const AttendArgs& A, int b) { return A.max_pages ? max(A.lengths[b], 0) : 0; }
__host__ __device__ __forceinline__ int keys_of_request(const AttendArgs& A, int b) { return min(tokens_of(A, b), A.max_pages << A.page_bits); }          // (below 2^30)

// A request of the batch: the first of its `fresh` new tokens, its tokens in all, of which the table may hold fewer (keys), tiles of its rows
struct Request {
    int token0, fresh, tokens, keys, tiles;
    __host__ __device__ __forceinline__ Request(const AttendArgs& A, int b, int rows_of_a_tile)
    {
        token0 = b;
        fresh = 1;
        if (A.rows) {
            token0 = (int)min(max((long long)A.rows[b], 0ll), A.T);
            fresh = max((int)min((long long)A.rows[b + 1], A.T) - token0, 0);
        }
        tokens = tokens_of(A, b);
        keys = keys_of_request(A, b);
        tiles = (fresh * A.g + rows_of_a_tile - 1) / rows_of_a_tile;
    }
};

// The rows of a workgroup, from r0 on of `count`: of request b, of whose new tokens token0 is the first and comes behind `before` others, or of all requests (prefix)
struct RowsOf {
    int r0, count, token0, before, keys, b;
    static __host__ __device__ __forceinline__ RowsOf of_prefix(const AttendArgs& A, int r0)
    {
        const int fresh = A.rows ? (int)min(max((long long)A.rows[A.B], 0ll), A.T) : (int)A.T;
        return {r0, fresh * A.g, 0, 0, 0, 0};          // (T * Hq stays below 2^26)
    }
    static __host__ __device__ __forceinline__ RowsOf of_request(const AttendArgs& A, const Request& q, int b, int r0) { return {r0, q.fresh * A.g, q.token0, q.tokens - q.fresh, q.keys, b}; }
    static __device__ __forceinline__ RowsOf of_tile(const AttendArgs& A, int i, int rows_of_a_tile)
    {
        int b, r0;
        if (A.rows) {
            b = request_of_tile(A, i, rows_of_a_tile);
            r0 = (i - (int)tiles_before(A, b, rows_of_a_tile)) * rows_of_a_tile;
        } else {
            const int per = (A.g + rows_of_a_tile - 1) / rows_of_a_tile;
            b = i / per;
            r0 = (i - b * per) * rows_of_a_tile;
        }
        return of_request(A, Request(A, b, rows_of_a_tile), b, r0);
    }
    __host__ __device__ __forceinline__ bool none() const { return r0 < 0 || r0 >= count; }
    // Own keys that row `at` of the tile sees, those that are there of its request's first ones up to itself, and that all rows do together.  (Which is its own goes by
    // the tokens, also by those that the table has no room for: they are the request's last ones.)
    __host__ __device__ __forceinline__ int sees(const AttendArgs& A, int at) const
    {
        const int r = r0 + at;
        return r < count ? min(max(before + r / A.g + 1, 0), keys) : 0;
    }
    __host__ __device__ __forceinline__ int end(const AttendArgs& A, int rows_of_a_tile) const { return sees(A, min(rows_of_a_tile, count - r0) - 1); }
};

// Parts of a request's `length` own keys, if there are to be `dense` of them to a key; keys of one: they are equal
__device__ __forceinline__ int parts_of(const AttendArgs& A, int length, float dense) { return length ? min((int)((float)length * dense) + 1, A.own_splits) : 0; }
__device__ __forceinline__ int keys_of_part(int length, int parts) { return ((length + parts - 1) / parts + 127) / 128 * 128; }

// Requests' own keys in parts.  The host does not know the lengths, so it starts own_groups workgroups, and each finds the part that is its own: of `tiles` tiles of
// rows (with their heads) and K keys for all of them, (own_groups - tiles) / K parts to a key and one to a tile for what is left are no more than there are workgroups.
// One long request among short ones is in as many parts as its keys are worth (64 requests of about 100 bfloat16 keys, one of 65536, 8 heads: 71 us, with equally many parts
// to each 528), and there are few workgroups without any (tables for 65536 keys, all requests short: 30 and 35 us).
// A wavefront looks at 256 requests at a time, four neighbours to a lane.  Rows are left at none if there is no part for workgroup `id`.
template <int N> __device__ __forceinline__ void deal(const AttendArgs& A, int id, int rows_of_a_tile, RowsOf* rows, int* head, int* split, int* parts, int* per)
{
    const int lane = (int)threadIdx.x % kWave;
    float keys = 0.f;
    for (int b0 = lane * N; b0 < A.B; b0 += kWave * N)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const Request q(A, min(b0 + k, A.B - 1), rows_of_a_tile);
            keys += b0 + k < A.B ? (float)q.tiles * (float)q.keys : 0.f;
        }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) keys += __shfl_xor(keys, d);
    // (below the quotient by more than all roundings together, since the sum is over 1024 requests at most, 22 additions deep, so that the parts do not outgrow
    // the workgroups)
    const float dense = fminf((float)(A.own_groups - A.own_tiles * A.Hk) / (keys * (float)A.Hk), 1.f / (float)A.own_least) * (1.f - 0x1p-16f);
    if (id == 0 && threadIdx.x == 0) *A.dense = dense;
    int before = 0;          // (no more than `id`)
    for (int b0 = 0; b0 < A.B; b0 += kWave * N) {
        int jobs[N], all = 0;          // (rows make up own_tiles tiles or fewer, of 64 parts at most, so that a wavefront's sum has room)
#pragma unroll
        for (int k = 0; k < N; ++k) {
            const Request q(A, min(b0 + lane * N + k, A.B - 1), rows_of_a_tile);
            jobs[k] = b0 + lane * N + k < A.B ? q.tiles * parts_of(A, q.keys, dense) * A.Hk : 0;
            all += jobs[k];
        }
        int upto = all;
#pragma unroll
        for (int d = 1; d < kWave; d *= 2) {
            const int o = __shfl_up(upto, d);
            if (lane >= d) upto += o;
        }
        const unsigned long long in = __ballot(before + upto > id);
        if (in) {
            const int at = __ffsll((long long)in) - 1;
            int j = __builtin_amdgcn_readfirstlane(id - before - __shfl(upto - all, at)), b = b0 + at * N;
#pragma unroll
            for (int k = 0; k < N - 1; ++k) {
                const int n = __builtin_amdgcn_readfirstlane(__shfl(jobs[k], at));
                if (b != b0 + at * N + k || j < n) continue;
                j -= n;
                ++b;
            }
            if (j == 0 && threadIdx.x == 0) A.own_first[b] = id;
            const Request q(A, b, rows_of_a_tile);
            *parts = parts_of(A, q.keys, dense);
            *per = keys_of_part(q.keys, *parts);
            *head = j % A.Hk;
            *split = j / A.Hk % *parts;
            *rows = RowsOf::of_request(A, q, b, j / A.Hk / *parts * rows_of_a_tile);
            return;
        }
        before += __builtin_amdgcn_readfirstlane(__shfl(upto, kWave - 1));
    }
}

// Where a workgroup's results go: they are the call's (direct), or a part.
struct Place {
    int id, split;
    bool prefix, direct;

    // Parts of its own keys, before the lengths are looked at.  (A prefix's workgroup has none; what there are of the prefix is in A.direct.)
    static __host__ __device__ __forceinline__ int first_parts(const AttendArgs& A, bool prefix) { return prefix ? 1 : A.own_splits; }
    static __host__ __device__ __forceinline__ bool is_direct(const AttendArgs& A, bool prefix, int parts)
    {
        if (!prefix && !A.whole && A.own_splits > 1) return A.prefix_splits == 0 && parts == 1;
        return A.direct && parts == 1;
    }
    // Row r of [T][Hq], `at` of this workgroup's tile: which row of the parts it is
    __host__ __device__ __forceinline__ long long part_row(const AttendArgs& A, int rows_of_a_tile, long long r, int at) const
    {
        if (A.whole) return (long long)(id - A.cut) * rows_of_a_tile + at;
        if (!prefix && A.own_splits > 1) return (long long)A.prefix_splits * A.T * A.Hq + (long long)id * rows_of_a_tile + at;
        return (long long)(prefix ? split : A.prefix_splits) * A.T * A.Hq + r;
    }
};

// What a workgroup has to do: its rows, its keys, and where its results go.  ROWS: of a tile
template <typename T, int ROWS> struct Job : Place {
    const AttendArgs& A;
    int parts, head, per;              // parts: of its keys, if those are a request's; keys of one
    RowsOf rows;

    __device__ __forceinline__ Job(const AttendArgs& args, int id_, bool prefix_job) : Place{id_, 0, prefix_job, false}, A(args), parts(first_parts(args, prefix_job)), head(0), per(0)
    {
        if (!prefix && !A.whole && A.own_splits > 1) {
            rows = {0, 0, 0, 0, 0, 0};
            if (A.B <= kWave) deal<1>(A, id, ROWS, &rows, &head, &split, &parts, &per);
            else deal<4>(A, id, ROWS, &rows, &head, &split, &parts, &per);
            parts = __builtin_amdgcn_readfirstlane(parts);
        } else {
            int tile_and_head = id;
            split = prefix ? id / A.Hk / A.prefix_tiles : 0;
            if (A.whole && id >= A.cut) {
                tile_and_head = A.cut + (id - A.cut) / A.tail_splits;
                split = (id - A.cut) % A.tail_splits;
                parts = A.tail_splits;
            }
            head = tile_and_head % A.Hk;
            const int tile = tile_and_head / A.Hk;
            rows = prefix ? RowsOf::of_prefix(A, tile % A.prefix_tiles * ROWS) : RowsOf::of_tile(A, tile, ROWS);
        }
        direct = is_direct(A, prefix, parts);
        // (scalars, also where lanes have found them together)
        for (int* v : {&split, &head, &per, &rows.r0, &rows.count, &rows.token0, &rows.before, &rows.keys, &rows.b}) *v = __builtin_amdgcn_readfirstlane(*v);
    }
    __device__ __forceinline__ bool none() const { return rows.none(); }
    // of [T][Hq]; own keys that it sees
    __device__ __forceinline__ long long row(int at) const
    {
        const int r = rows.r0 + at, token = r / A.g;
        return r < rows.count ? (long long)(rows.token0 + token) * A.Hq + head * A.g + (r - token * A.g) : -1;
    }
    __device__ __forceinline__ int sees(int at) const
    {
        return rows.sees(A, at);
    }
    // Its keys, the prefix's or the request's own; those below `least` are seen by all of its rows
    __device__ __forceinline__ void keys(int own, int* begin, int* end, int* least) const
    {
        const int own_end = rows.end(A, ROWS);
        *begin = 0;
        *end = own ? own_end : A.prefix;
        if (prefix) {
            *begin = split * A.prefix_per;
            *end = min(*begin + A.prefix_per, A.prefix);
        } else if (parts > 1) {
            // parts of its own keys, or equal ones of those behind the prefix's (below 2^31 together)
            const int before = A.whole ? A.prefix : 0, all = before + own_end;
            const int n = A.whole ? (int)(((unsigned)all + parts - 1) / parts + 127) / 128 * 128 : per;
            const int from = (int)min((long long)split * n, (long long)all) - (own ? before : 0), to = (int)min((long long)split * n + n, (long long)all) - (own ? before : 0);
            *begin = max(from, 0);
            *end = min(to, *end);
        }
        *least = own ? sees(0) : *end;
    }
    __device__ __forceinline__ const int* table(int own) const { return own ? A.table + (long long)rows.b * A.max_pages : A.prefix_table; }

    // Where row r of [T][Hq], `at` of this workgroup, goes: to the result or to this part's place; its sums
    __device__ __forceinline__ char* place(long long r, int at) const
    {
        const int token = (int)((unsigned)r / (unsigned)A.Hq), h = (int)r - token * A.Hq;
        return direct ? A.out + (token * A.ldo + h * A.D) * (long long)sizeof(T) : reinterpret_cast<char*>(A.part_o + part_row(A, ROWS, r, at) * A.D);
    }
    __device__ __forceinline__ void store_sums(long long r, int at, float m, float l) const
    {
        if (!direct) A.part_ml[part_row(A, ROWS, r, at)] = make_float2(m, l);
        else if (A.lse) A.lse[r] = l == 0.f ? -INFINITY : 0.6931471805599453f * (m + __builtin_amdgcn_logf(l));
    }
    // four values from d on
    __device__ __forceinline__ void store(char* to, int d, f32x4 o, float l) const
    {
        if (d >= A.D) return;
        if (direct) {
            const float by = 1.f / l;
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = l == 0.f ? 0.f : o[e] * by;
            if constexpr (sizeof(T) == 2) {
                *reinterpret_cast<uint2*>(to + d * 2) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
                return;
            }
        }
        *reinterpret_cast<f32x4*>(to + d * 4) = o;
    }
};

template <typename T, int DP, int KIND> __device__ __forceinline__ void attend(const AttendArgs& A, char* lds, int id, bool prefix_job)
{
    typedef Attend<T, DP, KIND> C;
    constexpr int QT = C::QT, WR = C::WR;
    const int tid = (int)threadIdx.x, lane = tid % kWave, w = __builtin_amdgcn_readfirstlane(tid / kWave), wr = w % WR, wk = w / WR, col = lane & 15, grp = lane >> 4;
    const char** const places = reinterpret_cast<const char**>(lds + C::PLACES);
    const Job<T, C::ROWS> job(A, id, prefix_job);
    if (job.none()) return;
    const int count = job.rows.count, r0 = job.rows.r0, head = job.head;

    int sees[QT];                         // own keys
    u32x4 Q[QT][C::KS];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
        const int r = r0 + (wr * QT + t) * 16 + col;
        const bool in = r < count;
        const int token = in ? r / A.g : 0, h = in ? r - token * A.g : 0;
        sees[t] = job.sees((wr * QT + t) * 16 + col);
        const char* const at = A.q + ((job.rows.token0 + token) * A.ldq + (long long)(head * A.g + h) * A.D) * C::EB;
#pragma unroll
        for (int s = 0; s < C::KS; ++s) {
            const int c = s * 64 + grp * 16;
            Q[t][s] = u32x4{0, 0, 0, 0};
            if (in && c < A.D * C::EB && A.scale != 0.f) Q[t][s] = *reinterpret_cast<const u32x4*>(at + c);
            if (A.scale < 0.f) Q[t][s] ^= C::EB == 2 ? 0x80008000u : 0x80000000u;          // the scale's sign goes with the queries, and so does a scale of zero
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

    const float scale = A.scale == 0.f ? 1.f : fabsf(A.scale);

    // this thread's part of a tile's loads: key r0 + pass * PASS, chunk `chunk` of its line, which goes to place tid of the pass.  A load writes its
    // wavefront's lanes side by side, so the chunks of a line change places (xor a number of the key) instead of leaving gaps, for the reads below.
    // Reads of keys meet no bank twice so; those that transpose values do, two lanes to a bank, half of the cycles that they take (bfloat16, 128 wide).
    const int load_row = tid / C::CH, line = A.D * C::EB;
    auto chunk = [&](int pass) { return ((tid % C::CH) ^ line_key<C::LINE>(pass * C::PASS + load_row)) * 16; };
    if (A.D < DP || DP * C::EB < C::LINE) {                       // places that no load reaches
        for (int i = tid; i < 2 * C::STAGE / 16; i += kThreads) *reinterpret_cast<u32x4*>(lds + i * 16) = u32x4{0, 0, 0, 0};
    }
    const long long values = A.v_pages - A.k_pages;
    lds_char* const base = (lds_char*)lds;          // two tiles of keys, two of values
    const int k0 = wk * C::KW;

    int dirty_from = 0, dirty_to = 0;     // own keys whose infinities and NaN stay out of the products, see below
    for (int own = prefix_job || A.whole ? 0 : 1; own < (prefix_job ? 1 : 2); ++own) {
        const int* const table = job.table(own);
        int begin, end, least;
        job.keys(own, &begin, &end, &least);
        if (begin >= end) continue;

        int first = 0, stop = begin;      // keys whose pages' addresses are at hand
        bool holes = false;               // some of those pages are not there
        const char* at[C::PASSES];        // the keys of the last tile whose loads were started: null where there is none
        bool full = false;                // all of them are there
        unsigned long long seen[2] = {0, 0};          // which of them are there, if not all
        const int mask = (1 << A.page_bits) - 1;
        auto load_keys = [&](int key0, int stage) {
            if (key0 + C::KT > stop && stop < end) {
                first = key0 >> A.page_bits;
                const int n = min(kPlaces, ((end - 1) >> A.page_bits) - first + 1);
                stop = min((first + kPlaces) << A.page_bits, end);          // (below 2^30 + 2^20)
                __syncthreads();
                int missing = 0;
                for (int i = tid; i < n; i += kThreads) {
                    const int page = table[first + i];
                    const bool none = page < 0 || page >= A.pages;
                    places[i] = none ? nullptr : A.k_pages + ((((long long)page * A.Hk + head) << A.page_bits) * line);
                    missing |= none;
                }
                holes = __syncthreads_or(missing);
            }
            const uint32_t to = (uint32_t)(uintptr_t)base + stage * C::HALF + w * 1024;
            full = key0 + C::KT <= end && !holes;
            if (full) {
#pragma unroll
                for (int i = 0; i < C::PASSES; ++i) {
                    const int key = key0 + i * C::PASS + load_row;
                    at[i] = places[(key >> A.page_bits) - first] + ((key & mask) * line + chunk(i));
                }
#pragma unroll
                for (int i = 0; i < C::PASSES; ++i)
                    if (chunk(i) < line) dma16_from(to + i * 4096, at[i]);
                return;
            }
#pragma unroll
            for (int h = 0; h < (C::KT + 63) / 64; ++h) {
                const int key = key0 + h * 64 + lane;
                seen[h] = __ballot(h * 64 + lane < C::KT && key < end && places[(min(key, end - 1) >> A.page_bits) - first] != nullptr);
            }
#pragma unroll
            for (int i = 0; i < C::PASSES; ++i) {
                const int key = key0 + i * C::PASS + load_row;
                const char* const place = key < end ? places[(key >> A.page_bits) - first] : nullptr;
                at[i] = place ? place + ((key & mask) * line + chunk(i)) : nullptr;
                if (at[i] && chunk(i) < line) dma16_from(to + i * 4096, at[i]);
                else *reinterpret_cast<u32x4*>(lds + stage * C::HALF + i * 4096 + tid * 16) = u32x4{0, 0, 0, 0};
            }
        };
        // ... of the values of the keys that the last call of load_keys() was for
        auto load_values = [&](int stage) {
            const uint32_t to = (uint32_t)(uintptr_t)base + (2 + stage) * C::HALF + w * 1024;
            if (full) {
#pragma unroll
                for (int i = 0; i < C::PASSES; ++i)
                    if (chunk(i) < line) dma16_from(to + i * 4096, at[i] + values);
                return;
            }
#pragma unroll
            for (int i = 0; i < C::PASSES; ++i) {
                if (at[i] && chunk(i) < line) dma16_from(to + i * 4096, at[i] + values);
                else *reinterpret_cast<u32x4*>(lds + 2 * C::HALF + stage * C::HALF + i * 4096 + tid * 16) = u32x4{0, 0, 0, 0};
            }
        };
        typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
        typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
        typedef __attribute__((address_space(3))) uint32_t lds_u32;
        // where this lane reads: line `col` of 16 keys; the values' line of its keys.  (xor of a chunk's number and xor of an address are the same: lines
        // begin at multiples of their length)
        const int k_from = (k0 + col) * C::LINE + ((grp ^ line_key<C::LINE>(col)) << 4);
        const int v_line = grp * 4 + (C::EB == 2 ? col >> 2 : 0), v_chunk = C::EB == 2 ? (col >> 1) & 1 : col >> 2;
        const int v_from = 2 * C::HALF + (k0 + v_line) * C::LINE + ((v_chunk ^ line_key<C::LINE>(v_line)) << 4) + (C::EB == 2 ? (col & 1) * 8 : (col & 3) * 4);
        // fragment i of a tile's keys (16 of them, 64 bytes of each), of its values (the keys of a weights' register by 16 of D)
        constexpr int K_STEPS = C::KS * C::NT, V_STEPS = C::NP * C::ND, AHEAD = K_STEPS < 4 ? K_STEPS : C::EB == 2 ? 4 : 3;
        auto key_fragment = [&](int stage, int i) {
            return *(const lds_u32x4*)(base + ((k_from + stage * C::HALF) ^ (i / C::NT << 6)) + i % C::NT * 16 * C::LINE);
        };
        auto value_fragment = [&](int stage, int i) {
            const int n = i / C::ND, d = i % C::ND, from = v_from + stage * C::HALF;
            u32x4 v = {0, 0, 0, 0};
            if constexpr (C::EB == 2) {
                lds_char* const p = base + (from ^ (d << 5)) + n * 32 * C::LINE;
                const uint2 lo = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)p));
                v.x = lo.x;
                v.y = lo.y;
                if constexpr (C::NT > 1) {
                    const uint2 hi = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(p + 16 * C::LINE)));
                    v.z = hi.x;
                    v.w = hi.y;
                }
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = *(const lds_u32*)(base + (from ^ (d << 6) ^ (line_key<C::LINE>(e) << 4)) + (n * 16 + e) * C::LINE);
            }
            return v;
        };
        auto largest = [&](const f32x4 (&S)[QT][C::NT], float (&top)[QT]) {
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                top[t] = S[t][0][0];
#pragma unroll
                for (int n = 0; n < C::NT; ++n)
#pragma unroll
                    for (int e = 0; e < 4; ++e) top[t] = fmaxf(top[t], S[t][n][e]);
            }
        };
        // What rows do not see is -infinity, and m follows the largest score, of the tile at key0.  m follows only where that is more than 2^8 times what m stands for: sums
        // hold that and much more in 32 bits, and what is there already is seldom scaled.
        auto settle = [&](int key0, bool all, const unsigned long long (&seen)[2], f32x4 (&S)[QT][C::NT], float (&top)[QT]) {
            const bool edge = own && key0 + C::KT > least;
            if (!all || edge) {
                const unsigned long long there = all ? ~0ull : (C::KT > 64 && k0 >= 64 ? seen[1] : seen[0]) >> (k0 & 63) >> (grp * 4);
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    // bit 16 n + e: key 16 n + e from this lane's first on
                    const int below = own ? sees[t] - (key0 + k0 + grp * 4) : 64;
                    const unsigned long long bits = there & (below <= 0 ? 0ull : below >= 64 ? ~0ull : (1ull << below) - 1);
#pragma unroll
                    for (int n = 0; n < C::NT; ++n)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const unsigned half = n < 2 ? (unsigned)bits : (unsigned)(bits >> 32);
                            S[t][n][e] = half & (1u << (n % 2 * 16 + e)) ? S[t][n][e] : -INFINITY;
                        }
                }
                largest(S, top);
            }
            bool grows = false;
#pragma unroll
            for (int t = 0; t < QT; ++t) grows = grows || top[t] * scale > m[t] + 8.f;
            if (!__any(grows)) return;
#pragma unroll
            for (int t = 0; t < QT; ++t) {
                const float most = fmaxf(m[t], row_max(top[t] * scale)), down = __builtin_amdgcn_exp2f(m[t] - (most == -INFINITY ? 0.f : most));
                m[t] = most;
                l[t] *= down;
#pragma unroll
                for (int d = 0; d < C::ND; ++d) O[t][d] *= down;
            }
        };

        // Keys are one tile ahead of values: while a tile's weights are formed, on the vector unit, and its values multiplied, the next one's scores are.
        f32x4 S[QT][C::NT], next[QT][C::NT];
        float top[QT];
        __syncthreads();                  // (LDS is read no more)
        load_keys(begin, 0);
        const bool all = full;
        const unsigned long long first_seen[2] = {seen[0], seen[1]};
        load_values(0);
        if (begin + C::KT < end) load_keys(begin + C::KT, 1);
        dma_wait_and_meet();
        const bool live = r0 + wr * (QT * 16) < count;          // this wavefront has rows
        if (live) {
#pragma unroll
            for (int i = 0; i < K_STEPS; ++i) {
                const u32x4 k = key_fragment(0, i);
#pragma unroll
                for (int t = 0; t < QT; ++t) S[t][i % C::NT] = multiply<T>(k, Q[t][i / C::NT], i < C::NT ? f32x4{0.f, 0.f, 0.f, 0.f} : S[t][i % C::NT]);
            }
            largest(S, top);
            settle(begin, all, first_seen, S, top);
        }
        int stage = 0;
        for (int key0 = begin; key0 < end; key0 += C::KT, stage ^= 1) {
            dma_wait_and_meet();
            const bool next_all = full;          // of the next tile, before the one after it is asked for
            const unsigned long long next_seen[2] = {seen[0], seen[1]};
            if (key0 + C::KT < end) load_values(stage ^ 1);
            if (key0 + 2 * C::KT < end) load_keys(key0 + 2 * C::KT, stage);
            // A product with a weight of zero would carry an infinity or a NaN of v to rows that do not see its key.  Where rows of the tile see
            // different keys such values are taken out of the tile and added to the rows that do at the end.
            if (own && least < end && key0 + C::KT > least) {
                u32x4 v[C::PASSES];
                int bad = 0;
#pragma unroll
                for (int i = 0; i < C::PASSES; ++i) {
                    v[i] = *reinterpret_cast<const u32x4*>(lds + 2 * C::HALF + stage * C::HALF + i * 4096 + tid * 16);
                    bad |= !all_finite<T>(v[i]);
                }
                if (__syncthreads_or(bad)) {
                    if (dirty_to == 0) dirty_from = key0;
                    dirty_to = end;
#pragma unroll
                    for (int i = 0; i < C::PASSES; ++i) *reinterpret_cast<u32x4*>(lds + 2 * C::HALF + stage * C::HALF + i * 4096 + tid * 16) = only_finite<T>(v[i]);
                    __syncthreads();
                }
            }
            if (!live) continue;

            // The order is held step by step (the compiler by itself asks LDS for an operand right before its product and then waits): operands are read some
            // products ahead, and between the products of the next scores (behind the last tile: of what is there, and not used) goes the weights' arithmetic.
            u32x4 P[QT][C::NP], k[K_STEPS], v[V_STEPS];
            float from[QT];
#pragma unroll
            for (int t = 0; t < QT; ++t) from[t] = m[t] == -INFINITY ? 0.f : m[t];
            constexpr int SLICES = QT * C::NT;
            auto weights = [&](int j) {          // four keys of a row
                const int t = j % QT, n = j / QT;
                f32x4& x = S[t][n];
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = __builtin_amdgcn_exp2f(fmaf(x[e], scale, -from[t]));
                l[t] += (x[0] + x[1]) + (x[2] + x[3]);
                // bfloat16: the weights are rounded to 8 bits for the products (off by at most 2^-8 of themselves, with no preferred sign); their sum is not
                if constexpr (C::EB == 2) {
                    P[t][n / 2][n % 2 * 2] = f32x2_to_bf16x2(x[0], x[1]);
                    P[t][n / 2][n % 2 * 2 + 1] = f32x2_to_bf16x2(x[2], x[3]);
                } else {
                    P[t][n] = u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
                }
            };
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) k[i] = key_fragment(stage ^ 1, i);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < K_STEPS; ++i) {
                if (i + AHEAD < K_STEPS) k[i + AHEAD] = key_fragment(stage ^ 1, i + AHEAD);
                else if (i + AHEAD - K_STEPS < V_STEPS) v[i + AHEAD - K_STEPS] = value_fragment(stage, i + AHEAD - K_STEPS);
#pragma unroll
                for (int t = 0; t < QT; ++t) next[t][i % C::NT] = multiply<T>(k[i], Q[t][i / C::NT], i < C::NT ? f32x4{0.f, 0.f, 0.f, 0.f} : next[t][i % C::NT]);
#pragma unroll
                for (int j = i * SLICES / K_STEPS; j < (i + 1) * SLICES / K_STEPS; ++j) weights(j);
                __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int t = 0; t < QT; ++t) top[t] = next[t][0][0];
#pragma unroll
            for (int i = 0; i < V_STEPS; ++i) {
                if (i + AHEAD < V_STEPS) v[i + AHEAD] = value_fragment(stage, i + AHEAD);
#pragma unroll
                for (int t = 0; t < QT; ++t) {
                    const int n = i / C::ND, d = i % C::ND;
                    if constexpr (C::EB == 2 && C::NT == 1)
                        O[t][d] = __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, make_uint2(v[i].x, v[i].y)),
                                                                            __builtin_bit_cast(s16x4, make_uint2(P[t][n].x, P[t][n].y)), O[t][d], 0, 0, 0);
                    else O[t][d] = multiply<T>(v[i], P[t][n], O[t][d]);
                }
#pragma unroll
                for (int j = i * SLICES / V_STEPS; j < (i + 1) * SLICES / V_STEPS; ++j) {
                    const f32x4 x = next[j % QT][j / QT];
                    top[j % QT] = fmaxf(fmaxf(fmaxf(top[j % QT], x[0]), fmaxf(x[1], x[2])), x[3]);
                }
                __builtin_amdgcn_sched_barrier(0);
            }
            if (key0 + C::KT < end) settle(key0 + C::KT, next_all, next_seen, next, top);
#pragma unroll
            for (int t = 0; t < QT; ++t)
#pragma unroll
                for (int n = 0; n < C::NT; ++n) S[t][n] = next[t][n];
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
        const long long at = key_at<T>(A, job.table(1), head, key);
        if (at < 0 || d >= A.D) return v;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const float x = Elem<T>::load1(reinterpret_cast<const T*>(A.v_pages + at) + d + e);
            v[e] = fabsf(x) < INFINITY ? 0.f : x;
        }
        return v;
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
        for (int t = 0; t < QT; ++t) {
            const int at = (wr * QT + t) * 16 + col;
            const long long row = job.row(at);
            if (row < 0) continue;
            char* const to = job.place(row, at);
#pragma unroll
            for (int d = 0; d < C::ND; ++d) job.store(to, d * 16 + grp * 4, O[t][d], l[t]);
            if (grp == 0) job.store_sums(row, at, m[t], l[t]);
        }
    } else {
        // the wavefronts' parts, in order
        constexpr int RW = QT * 16;
        float* const o = reinterpret_cast<float*>(lds);
        float* const ml = o + 4 * RW * DP;
        __syncthreads();
#pragma unroll
        for (int t = 0; t < QT; ++t) {
#pragma unroll
            for (int d = 0; d < C::ND; ++d) *reinterpret_cast<f32x4*>(o + ((w * RW + t * 16 + col) * DP + d * 16 + grp * 4)) = O[t][d];
            if (grp == 0) {
                ml[(w * RW + t * 16 + col) * 2] = m[t];
                ml[(w * RW + t * 16 + col) * 2 + 1] = l[t];
            }
        }
        __syncthreads();
        for (int i = tid; i < C::ROWS * (DP / 4); i += kThreads) {
            const int r = i / (DP / 4), d = i % (DP / 4) * 4, from = r / RW * RW + r % RW;          // (wavefront k * WR + r / RW has row r for its keys)
            float top = -INFINITY, ll = 0.f;
#pragma unroll
            for (int k = 0; k < C::WK; ++k) top = fmaxf(top, ml[(k * WR * RW + from) * 2]);
            f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < C::WK; ++k) {
                const int at = k * WR * RW + from;
                if (ml[at * 2 + 1] == 0.f) continue;          // (no key: what o holds is no sum)
                const float f = __builtin_amdgcn_exp2f(ml[at * 2] - top);
                ll += f * ml[at * 2 + 1];
                sum += f * *reinterpret_cast<const f32x4*>(o + at * DP + d);
            }
            const long long row = job.row(r);
            if (row < 0) continue;
            for (int key = dirty_from; key < min(dirty_to, job.sees(r)); ++key) sum += left_out(key, d);
            job.store(job.place(row, r), d, sum, ll);
            if (d == 0) job.store_sums(row, r, top, ll);
        }
    }
}

// Up to four rows of float: bound by memory, and by float matrix products if those were formed of 16 rows that are mostly empty.  No LDS, no barrier:
// LANES lanes hold a key, chunks of 16 bytes of it (lane p chunks p, p + LANES, ...), so that they read whole lines; the workgroup takes GROUPS keys at a time,
// and DEPTH such steps' keys and values are on their way to registers while one is used.  A score is the sum over its lanes;
// each group of lanes has maxima, sums and products of its own keys, which meet at the end, in LDS, in a fixed order.
template <int DP> struct Stream {
    static constexpr int LANES = DP == 128 ? 16 : 8, NC = DP / 4 / LANES, GROUPS = kThreads / LANES, DEPTH = NC == 3 ? 3 : 4;
    static constexpr int LDS = GROUPS * kStreamRows * (DP + 2) * 4;
};

// the sum over 8 or 16 lanes; all of them get it
template <int LANES> __device__ __forceinline__ float sum_over(float v)
{
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0xB1, 0xf, 0xf, true));       // lane ^ 1
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x4E, 0xf, 0xf, true));       // lane ^ 2
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x141, 0xf, 0xf, true));      // the other half of 8
    if constexpr (LANES == 16) v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), 0x140, 0xf, 0xf, true));      // the other half of 16
    return v;
}

template <int DP> __device__ __forceinline__ void stream(const AttendArgs& A, char* lds, int id, bool prefix_job)
{
    typedef Stream<DP> C;
    constexpr int R = kStreamRows, NC = C::NC, DEPTH = C::DEPTH, LANES = C::LANES, G = C::GROUPS;
    const int tid = (int)threadIdx.x, p = tid % LANES, slot = tid / LANES;
    const Job<float, R> job(A, id, prefix_job);
    if (job.none()) return;
    const float scale = A.scale;

    f32x4 Q[R][NC], O[R][NC];
    float m[R], l[R];
    int sees[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const long long row = job.row(r), token = row < 0 ? 0 : row / A.Hq;
        sees[r] = job.sees(r);
        const float* const at = reinterpret_cast<const float*>(A.q) + token * A.ldq + (row - token * A.Hq) * A.D;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
            const int d = (c * LANES + p) * 4;
            Q[r][c] = O[r][c] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (row >= 0 && d < A.D && scale != 0.f) Q[r][c] = *reinterpret_cast<const f32x4*>(at + d);
        }
        m[r] = -INFINITY;
        l[r] = 0.f;
    }
    const float factor = scale == 0.f ? 1.f : scale;
    const long long values = A.v_pages - A.k_pages;
    for (int own = prefix_job || A.whole ? 0 : 1; own < (prefix_job ? 1 : 2); ++own) {
        const int* const table = job.table(own);
        int begin, end, least;
        job.keys(own, &begin, &end, &least);
        if (begin >= end) continue;
        f32x4 K[DEPTH][NC], V[DEPTH][NC];
        bool there[DEPTH];
        int pages[DEPTH];
        // a page's number is asked for DEPTH steps before its keys
        auto page_of = [&](int key) { return key < end ? table[key >> A.page_bits] : -1; };
        auto load = [&](int u, int key) {
            const int page = pages[u];
            there[u] = page >= 0 && page < A.pages;
            const char* const at = A.k_pages + (((((long long)page * A.Hk + job.head) << A.page_bits) + (key & ((1 << A.page_bits) - 1))) * A.D + p * 4) * 4;
#pragma unroll
            for (int c = 0; c < NC; ++c) {
                K[u][c] = V[u][c] = f32x4{0.f, 0.f, 0.f, 0.f};
                if (there[u] && (c * LANES + p) * 4 < A.D) {
                    K[u][c] = *reinterpret_cast<const f32x4*>(at + c * (LANES * 16));
                    V[u][c] = *reinterpret_cast<const f32x4*>(at + c * (LANES * 16) + values);
                }
            }
        };
        const int key0 = begin + slot;
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) pages[u] = page_of(key0 + u * G);
#pragma unroll
        for (int u = 0; u < DEPTH; ++u) {
            load(u, key0 + u * G);
            pages[u] = page_of(key0 + (DEPTH + u) * G);
        }
        for (int step = begin; step < end; step += DEPTH * G)
#pragma unroll
            for (int u = 0; u < DEPTH; ++u) {
                const int first = step + u * G, key = first + slot;
                if (first >= end) break;
                const bool edge = own && first + G > least;          // rows see different keys
                float x[R];
                bool hidden[R];
                bool grows = false;
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    float s = 0.f;
#pragma unroll
                    for (int c = 0; c < NC; ++c)
#pragma unroll
                        for (int e = 0; e < 4; ++e) s = fmaf(Q[r][c][e], K[u][c][e], s);
                    float y = sum_over<LANES>(s) * factor;
                    asm("" : "+v"(y));          // (formed in any case: a branch around it is the longer way)
                    hidden[r] = !there[u] || (edge && key >= sees[r]);
                    x[r] = hidden[r] ? -INFINITY : y;
                    grows = grows || x[r] > m[r] + 8.f;
                }
                // m follows only where a score is more than 2^8 times what it stands for, see attend()
                if (__any(grows)) {
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        const float most = fmaxf(m[r], x[r]), down = __builtin_amdgcn_exp2f(m[r] - (most == -INFINITY ? 0.f : most));
                        m[r] = most;
                        l[r] *= down;
#pragma unroll
                        for (int c = 0; c < NC; ++c) O[r][c] *= down;
                    }
                }
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const float w = __builtin_amdgcn_exp2f(x[r] - (m[r] == -INFINITY ? 0.f : m[r]));
                    l[r] += w;
                    x[r] = w;
                }
                if (!edge) {
#pragma unroll
                    for (int r = 0; r < R; ++r)
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) O[r][c][e] = fmaf(x[r], V[u][c][e], O[r][c][e]);
                } else {          // what a row does not see does not reach it, whatever it is
#pragma unroll
                    for (int r = 0; r < R; ++r) {
                        if (hidden[r]) continue;
#pragma unroll
                        for (int c = 0; c < NC; ++c)
#pragma unroll
                            for (int e = 0; e < 4; ++e) O[r][c][e] = fmaf(x[r], V[u][c][e], O[r][c][e]);
                    }
                }
                load(u, key + DEPTH * G);
                pages[u] = page_of(key + 2 * DEPTH * G);
            }
    }

    // The groups' parts: a wavefront to a row for what they weigh, then two threads to four values of a row, half of the groups each
    float* const o = reinterpret_cast<float*>(lds);
    float2* const ml = reinterpret_cast<float2*>(o + G * R * DP);
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int c = 0; c < NC; ++c)
            if ((c * LANES + p) * 4 < DP) *reinterpret_cast<f32x4*>(o + (slot * R + r) * DP + (c * LANES + p) * 4) = O[r][c];
        if (p == 0) ml[r * G + slot] = make_float2(m[r], l[r]);
    }
    __syncthreads();
    static_assert(R == kThreads / kWave, "");
    {
        const int r = tid / kWave, g = tid % G;
        const float2 part = ml[r * G + g];
        float top = part.x, sum;
#pragma unroll
        for (int d = 1; d < G; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        const float f = part.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(part.x - top);
        sum = part.y == 0.f ? 0.f : f * part.y;
#pragma unroll
        for (int d = 1; d < G; d *= 2) sum += __shfl_xor(sum, d);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // (the wavefront's own row)
        ml[r * G + g] = make_float2(part.y == 0.f ? -1.f : f, sum);
        const long long row = job.row(r);
        if (row >= 0 && tid % kWave == 0) job.store_sums(row, r, top, sum);
    }
    __syncthreads();
    for (int i = tid / 2; i < R * (DP / 4); i += kThreads / 2) {
        const int r = i / (DP / 4), d = i % (DP / 4) * 4, g0 = tid % 2 * (G / 2);
        f32x4 all = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < G / 2; ++g) {
            const float f = ml[r * G + g0 + g].x;
            const f32x4 part = *reinterpret_cast<const f32x4*>(o + ((g0 + g) * R + r) * DP + d);
            if (f != -1.f) all += f * part;          // (of no key there is no sum)
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) all[e] += __shfl_xor(all[e], 1);
        const long long row = job.row(r);
        if (row >= 0 && tid % 2 == 0) job.store(job.place(row, r), d, all, ml[r * G].y);
    }
}

template <typename T, int DP, int KIND> constexpr int lds_of()
{
    if constexpr (KIND == STREAM) return Stream<DP>::LDS;
    else return Attend<T, DP, KIND>::LDS;
}
template <typename T, int DP, int KIND> __device__ __forceinline__ void do_job(const AttendArgs& A, char* lds, int id, bool prefix)
{
    if constexpr (KIND == STREAM) stream<DP>(A, lds, id, prefix);
    else attend<T, DP, KIND>(A, lds, id, prefix);
}

// PREFIX: the kind of a tile of the prefix's rows; OWN: of a tile of one request's.  One launch for both.
template <typename T, int DP, int PREFIX, int OWN> __global__ __launch_bounds__(kThreads, 2) void attend_keys(const AttendArgs A)
{
    constexpr int P = lds_of<T, DP, PREFIX>(), O = lds_of<T, DP, OWN>();
    __shared__ __attribute__((aligned(1024))) char lds[P > O ? P : O];
    // Workgroups of both kinds in turns of 256, as many as there are compute units, while there are both: products of the one and reads of the other side by side.
    int id = (int)blockIdx.x;
    const int turns = min(A.prefix_jobs, A.jobs - A.prefix_jobs) / 256, turn = id / 256;
    bool prefix = turn % 2 == 0;
    if (turn < 2 * turns) {
        id = turn / 2 * 256 + id % 256;
    } else {
        id -= turns * 256;
        prefix = id < A.prefix_jobs;
        if (!prefix) id -= A.prefix_jobs - turns * 256;
    }
    if constexpr (PREFIX == OWN) {
        do_job<T, DP, PREFIX>(A, lds, id, prefix);
    } else {
        if (prefix) do_job<T, DP, PREFIX>(A, lds, id, true);
        else do_job<T, DP, OWN>(A, lds, id, false);
    }
}

constexpr int kMaxParts = 128;

// A row's parts: the prefix's, and those of own keys that there are
struct PartsOf {
    int prefix, all, step;             // parts; rows from one of own keys to the next
    long long first, next, row;        // rows: of the first part of own keys; from one of the prefix to the next; in the prefix's
    __device__ __forceinline__ PartsOf(const AttendArgs& A, long long r, int token, int rows_of_a_tile)
    {
        next = A.T * A.Hq;
        row = r;
        prefix = A.prefix_splits;
        first = prefix * next + r;
        step = 0;
        all = prefix + A.own_splits;
        if (A.own_splits <= 1) return;
        int b = token, token0 = token;
        if (A.rows) {          // the last request that starts at this token or before it; 64 are looked at in each step
            int lo = 0, hi = A.B;
            const int lane = (int)threadIdx.x % kWave;
            while (hi - lo > 1) {
                const int step = (hi - lo + kWave - 1) / kWave, c = lo + lane * step, n = __popcll(__ballot(c < hi && A.rows[c] <= token));
                const int at = lo + (n ? n - 1 : 0) * step;
                hi = min(hi, at + step);
                lo = at;
            }
            b = lo;
            token0 = min(max(A.rows[b], 0), token);
        }
        const int parts = parts_of(A, keys_of_request(A, b), *A.dense);
        const int h = (int)(r - (long long)token * A.Hq), head = h / A.g, i = (token - token0) * A.g + h - head * A.g, tile = i / rows_of_a_tile;
        all = prefix + parts;
        // (no workgroup behind the last one, whatever `rows` are)
        const int job = parts ? min(max(A.own_first[b] + tile * parts * A.Hk + head, 0), max(A.own_groups - (parts - 1) * A.Hk - 1, 0)) : 0;
        first = prefix * next + (long long)job * rows_of_a_tile + (i - tile * rows_of_a_tile);
        step = A.Hk * rows_of_a_tile;
    }
    __device__ __forceinline__ long long at(int p) const { return p < prefix ? p * next + row : first + (long long)(p - prefix) * step; }
};

// Joins a row's parts: WAVES wavefronts to a row, lanes in groups of D / 4 (up to a power of two) that take every so manieth part; added part by part
// within a group, then over the groups and the wavefronts in a fixed tree.  All of the parts' sums are fetched at once, and the products of four at a time.
template <typename T, int LANES, int WAVES> __global__ __launch_bounds__(kThreads) void attend_join(const AttendArgs A, int rows_of_a_tile)
{
    constexpr int GROUPS = kWave / LANES, STEP = GROUPS * WAVES, AHEAD = 4;
    __shared__ float weights[4][kMaxParts];
    __shared__ f32x4 joined[WAVES == 1 ? 1 : 4][LANES];
    const int w = (int)threadIdx.x / kWave, lane = (int)threadIdx.x % kWave;
    const long long r = (long long)blockIdx.x * (4 / WAVES) + (WAVES == 1 ? w : 0);
    const int token = (int)((unsigned)r / (unsigned)A.Hq);          // (rows are fewer than 2^26)
    const long long end = A.rows ? min(max((long long)A.rows[A.B], 0ll), A.T) : A.T;
    if (token >= end) return;                                       // (with several wavefronts to a row, all of the workgroup)
    const PartsOf of(A, r, token, rows_of_a_tile);
    const int parts = of.all;
    if (parts == 1 && A.prefix_splits == 0) return;                 // (stored already)
    float top = -INFINITY;
    float2 ml[kMaxParts / kWave];
#pragma unroll
    for (int k = 0; k < kMaxParts / kWave; ++k) {
        ml[k] = make_float2(-INFINITY, 0.f);
        if (k * kWave + lane < parts) ml[k] = A.part_ml[of.at(k * kWave + lane)];
        if (ml[k].y != 0.f) top = fmaxf(top, ml[k].x);
    }
    top = row_max(top);
#pragma unroll
    for (int d = 1; d < 16; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < kMaxParts / kWave; ++k) {
        const float f = ml[k].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[k].x - top);
        sum += ml[k].y == 0.f ? 0.f : f * ml[k].y;
        // (a part without keys weighs nothing, whatever it holds; one whose weight comes out as zero is there all the same)
        weights[w][k * kWave + lane] = ml[k].y == 0.f ? -1.f : f;
    }
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) sum += __shfl_xor(sum, d);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");              // (the lanes of a wavefront read each other's)

    const int d = lane % LANES * 4, g = lane / LANES + (WAVES == 1 ? 0 : w * GROUPS);
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    for (int p0 = g; p0 < parts; p0 += AHEAD * STEP) {
        f32x4 v[AHEAD];
        float f[AHEAD];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int p = p0 + k * STEP;
            f[k] = p < parts ? weights[w][p] : -1.f;
            if (f[k] != -1.f && d < A.D) v[k] = *reinterpret_cast<const f32x4*>(A.part_o + of.at(p) * A.D + d);
            else v[k] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) o += (f[k] == -1.f ? 0.f : f[k]) * v[k];
    }
#pragma unroll
    for (int k = LANES; k < kWave; k *= 2)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], k);
    if constexpr (WAVES > 1) {
        if (lane < LANES) joined[w][lane] = o;
        __syncthreads();
        if (w) return;
        o = (joined[0][lane % LANES] + joined[1][lane % LANES]) + (joined[2][lane % LANES] + joined[3][lane % LANES]);
    }
    if (lane >= LANES) return;
    if (d < A.D) {
        const float by = 1.f / sum;
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = sum == 0.f ? 0.f : o[e] * by;
        T* const to = reinterpret_cast<T*>(A.out) + token * A.ldo + ((int)r - token * A.Hq) * A.D + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
        else *reinterpret_cast<f32x4*>(to) = o;
    }
    if (lane == 0 && A.lse) A.lse[r] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (top + __builtin_amdgcn_logf(sum));
}

// Joins the parts of the tiles that workgroups share by keys: 32 rows of one, eight lanes to a row.
constexpr int kTailRows = 32, kMaxTail = 8;
template <typename T> __global__ __launch_bounds__(kThreads) void attend_join_tail(const AttendArgs A, int rows_of_a_tile)
{
    const int per = rows_of_a_tile / kTailRows, tile = (int)blockIdx.x / per, job = A.cut + tile, head = job % A.Hk;
    const RowsOf w = RowsOf::of_tile(A, job / A.Hk, rows_of_a_tile);
    const int at = (int)blockIdx.x % per * kTailRows + (int)threadIdx.x / 8, r = w.r0 + at;
    if (w.r0 < 0 || r >= w.count) return;
    const long long first = (long long)tile * A.tail_splits * rows_of_a_tile + at;
    float2 ml[kMaxTail];
    float top = -INFINITY, sum = 0.f;
#pragma unroll
    for (int p = 0; p < kMaxTail; ++p) {
        ml[p] = make_float2(-INFINITY, 0.f);
        if (p < A.tail_splits) ml[p] = A.part_ml[first + p * rows_of_a_tile];
        if (ml[p].y != 0.f) top = fmaxf(top, ml[p].x);
    }
#pragma unroll
    for (int p = 0; p < kMaxTail; ++p) {
        ml[p].x = ml[p].y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml[p].x - top);
        if (ml[p].y != 0.f) sum += ml[p].x * ml[p].y;
    }
    const int token = w.token0 + r / A.g, h = head * A.g + r % A.g;
    const float by = 1.f / sum;
    for (int d = (int)threadIdx.x % 8 * 4; d < A.D; d += 32) {
        f32x4 o = {0.f, 0.f, 0.f, 0.f}, v[kMaxTail];
#pragma unroll
        for (int p = 0; p < kMaxTail; ++p) {
            v[p] = f32x4{0.f, 0.f, 0.f, 0.f};
            if (ml[p].y != 0.f) v[p] = *reinterpret_cast<const f32x4*>(A.part_o + (first + p * rows_of_a_tile) * A.D + d);
        }
#pragma unroll
        for (int p = 0; p < kMaxTail; ++p) o += ml[p].x * v[p];
#pragma unroll
        for (int e = 0; e < 4; ++e) o[e] = sum == 0.f ? 0.f : o[e] * by;
        T* const to = reinterpret_cast<T*>(A.out) + token * A.ldo + h * A.D + d;
        if constexpr (sizeof(T) == 2) *reinterpret_cast<uint2*>(to) = make_uint2(f32x2_to_bf16x2(o[0], o[1]), f32x2_to_bf16x2(o[2], o[3]));
        else *reinterpret_cast<f32x4*>(to) = o;
    }
    if (threadIdx.x % 8 == 0 && A.lse) A.lse[(long long)token * A.Hq + h] = sum == 0.f ? -INFINITY : 0.6931471805599453f * (top + __builtin_amdgcn_logf(sum));
}

template <typename T> cgbn_status launch_attend(const AttendArgs& A, int prefix_kind, int own_kind, hipStream_t st);

}  // namespace cgbn
