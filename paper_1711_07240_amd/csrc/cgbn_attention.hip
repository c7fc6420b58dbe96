// Attention over a shared prefix and pages of each request's own: arguments and the choice of tiles.  The kernels are in cgbn_attention.h.
#include "cgbn.h"
#include "cgbn_attention.h"

#include <cstring>

namespace cgbn {
namespace {

constexpr int kMaxHeads = 1 << 10, kMaxRequests = 1 << 20, kMaxPage = 1024, kMaxTable = 1 << 20;
constexpr long long kMaxKeys = 1ll << 30, kMaxRows = 1ll << 26;          // rows: heads of tokens

struct Plan {
    int prefix_kind, own_kind, prefix_splits, prefix_per, own_splits, own_least, own_groups, prefix_tiles, own_tiles, whole, tail_splits;
    long long prefix_jobs, jobs, cut;
    int parts() const { return prefix_splits + own_splits; }
};

bool sizes_fit(long long T, int B, int Hq, int Hk, int D, long long prefix, long long capacity)
{
    if (T < 0 || B < 0 || B > kMaxRequests || Hk < 1 || Hq < Hk || Hq > kMaxHeads || Hq % Hk != 0 || D < 8 || D > 256 || D % 8 != 0) return false;
    return T <= (kMaxRows - 4) / Hq && (long long)B * Hk <= (1 << 22) && prefix >= 0 && prefix < kMaxKeys && capacity >= 0 && capacity < kMaxKeys;
}

long long up(long long a, long long b) { return (a + b - 1) / b; }

// What the device has to know of the lengths stays there: ranges of a request's own keys are cut by its length where they are read, `own_splits` of
// them.  `several`: requests may have more rows than one.
Plan plan(long long T, int B, int Hq, int Hk, int D, int line, int elem, long long prefix, long long capacity, bool several)
{
    Plan p;
    std::memset(&p, 0, sizeof(p));
    const long long g = Hq / Hk, rows = T * g, each = several ? up(rows, B) : g;
    // tiles of rows: no more of them empty than has to be
    auto kind_of = [&](long long n) {
        if (n <= kStreamRows && may_stream(D, elem) && (rows / kStreamRows + B) * Hk < (1 << 22)) return (int)STREAM;          // (fewer than 2^32 threads)
        int kind = n <= rows_of(FEW, line, elem) ? FEW : n <= rows_of(SOME, line, elem) ? SOME : MANY;
        // float products take so much longer than what they are of that keys may as well be read again, if fewer empty rows are multiplied
        auto work = [&](int k) { return up(n, rows_of(k, line, elem)) * qt_of(k, line, elem) * (4 / wk_of(k, line)); };
        if (elem == 4)
            for (int k = kind - 1; k >= FEW; --k)
                if (work(k) < work(kind)) kind = k;
        return kind;
    };
    p.own_kind = kind_of(each);
    p.prefix_kind = kind_of(rows);
    if (p.own_kind > p.prefix_kind) p.own_kind = p.prefix_kind;          // (one request's rows are no more than all rows; the other way there is no kernel)
    const int own_rows = rows_of(p.own_kind, line, elem);
    p.prefix_tiles = (int)up(rows, rows_of(p.prefix_kind, line, elem));
    const long long own_tiles = several ? rows / own_rows + B : B * up(g, own_rows);
    p.own_tiles = (int)own_tiles;
    // A workgroup to a tile of one request's rows and a head, prefix and own keys: where there are many, and where there are so few keys that one launch is the
    // shorter way (3 requests, 100 keys of the prefix and up to 80 of their own: 7 us, in parts 9).
    const long long whole = own_tiles * Hk, slots = 512;
    const bool many = p.own_kind == MANY && whole >= 256;
    if (many || prefix + capacity <= 512) {
        p.whole = p.own_splits = 1;
        p.prefix_kind = p.own_kind;
        p.prefix_tiles = 0;
        p.jobs = p.cut = whole;
        // Two workgroups share each compute unit.  What is left behind the last full round of those is shared by more of them, in parts of 512 keys or more.
        const long long left = whole % slots;
        long long s = left ? 2 * slots / left : 1;
        if (s > (prefix + capacity) / 512) s = (prefix + capacity) / 512;
        if (s > kMaxTail) s = kMaxTail;
        p.tail_splits = 1;
        if (many && s > 1 && left * 4 <= slots * 3) {
            p.tail_splits = (int)s;
            p.cut = whole - left;
            p.jobs = p.cut + left * s;
        }
        return p;
    }
    p.own_splits = prefix ? 0 : 1;         // (without any keys rows are zero)
    // Parts of a request's keys, whose number goes by the lengths, which the host does not know (see deal()): two rounds of the 512 workgroups that the device holds
    // at a time, or 512 more than there are tiles (768 workgroups in all: 24 drafts of up to 1500 float keys, 20 heads, 98 us, 1024: 90; 64 requests of 100
    // bfloat16 keys of which one has 65536, 81 and 73).  With many tiles one part to each is quicker where requests are alike, and no one's end is waited for where
    // they are not (256 requests of 8 heads, one part and several: 2000 keys each 357 and 369 us, 200 keys 52 and 68, one of 32768 among those 532 and 95; with 2000
    // requests of one head 188 and 251, 51 and 123, 376 and 125), so it is both up to 2048 tiles and 1024 requests.  A part has 128 keys or more where tiles are few,
    // 512 where they are many.
    const long long tiles = own_tiles * Hk;
    p.own_least = tiles <= 64 ? 128 : tiles <= 128 ? 256 : 512;
    if (capacity) {
        const long long s = up(capacity, p.own_least);
        p.own_splits = (int)(tiles > 2048 || B > 1024 ? 1 : s > 64 ? 64 : s);
    }
    p.own_groups = (int)(p.own_splits > 1 ? (tiles <= 512 ? 512 : tiles) + 512 : tiles * p.own_splits);
    // Parts of the prefix: a workgroup for each compute unit, which leaves room for one that reads beside it (64 rows, 32768 bfloat16 keys of 8 heads, 128, 256, 512 and
    // 1024 workgroups: 112, 98, 105 and 130 us); with few rows reading is all there is to do, as above
    if (prefix) {
        long long s = (rows > 32 ? 256 : 1024) / ((long long)p.prefix_tiles * Hk);
        if (s > up(prefix, 256)) s = up(prefix, 256);
        s = s < 1 ? 1 : s > 64 ? 64 : s;
        p.prefix_per = (int)up(up(prefix, s), 128) * 128;
        p.prefix_splits = (int)up(prefix, p.prefix_per);
    }
    p.prefix_jobs = (long long)p.prefix_tiles * p.prefix_splits * Hk;
    p.jobs = p.prefix_jobs + p.own_groups;
    return p;
}

// Rows of the parts: where own keys are dealt, a tile for each workgroup, as most requests have far fewer parts than there may be (256 requests of 64 heads in
// tables for 65536 keys: 21 MB, with room for 64 parts of each 545 MB); bytes
long long part_rows(const Plan& p, long long T, int Hq, int line, int elem)
{
    const int tile = rows_of(p.own_kind, line, elem);
    return p.whole ? (p.jobs - p.cut) * tile : p.own_splits > 1 ? p.prefix_splits * T * Hq + (long long)p.own_groups * tile : p.parts() <= 1 ? 0 : p.parts() * T * Hq;
}
size_t scratch(const Plan& p, long long T, int B, int Hq, int D, int line, int elem)
{
    return (size_t)part_rows(p, T, Hq, line, elem) * (D + 2) * sizeof(float) + (p.own_splits > 1 ? (1 + (size_t)B) * sizeof(int) : 0);
}

}  // namespace
}  // namespace cgbn

using namespace cgbn;

extern "C" {

size_t cgbn_prefix_attention_workspace_bytes(long long T, int B, int Hq, int Hk, int D, long long prefix, long long capacity, cgbn_dtype dtype)
{
    if ((dtype != CGBN_F32 && dtype != CGBN_BF16) || !sizes_fit(T, B, Hq, Hk, D, prefix, capacity)) return 0;
    if (T == 0 || B == 0) return 256;
    const int elem = dtype == CGBN_F32 ? 4 : 2, line = line_of(width_of(D), elem);
    // requests of one row each go in other tiles when it is said that they are
    size_t most = scratch(plan(T, B, Hq, Hk, D, line, elem, prefix, capacity, true), T, B, Hq, D, line, elem);
    if (T == B) {
        const size_t single = scratch(plan(T, B, Hq, Hk, D, line, elem, prefix, capacity, false), T, B, Hq, D, line, elem);
        if (single > most) most = single;
    }
    const size_t bytes = (most + 255) / 256 * 256;
    return most == 0 ? 256 : bytes > 256 ? bytes : 512;          // (of 256 or less a program may pass none)
}

cgbn_status cgbn_prefix_attention(const void* q, long long ldq, long long T, int B, const int* rows, const int* lengths, int Hq, int Hk, int D, float scale,
                                  const void* k_pages, const void* v_pages, int pages, int page, const int* prefix_table, int prefix, const int* table,
                                  int max_pages, void* out, long long ldo, float* lse, cgbn_dtype dtype, void* workspace, size_t workspace_bytes, void* stream)
{
    if (dtype != CGBN_F32 && dtype != CGBN_BF16) return CGBN_ERR_ENUM;
    if (page < 1 || page > kMaxPage || (page & (page - 1)) || pages < 0 || (long long)pages * page >= (1ll << 31) || max_pages < 0 || max_pages > kMaxTable) return CGBN_ERR_SHAPE;
    const long long capacity = (long long)max_pages * page;
    if (!sizes_fit(T, B, Hq, Hk, D, prefix, capacity) || (!rows && T != B)) return CGBN_ERR_SHAPE;
    if (T == 0 || B == 0) return CGBN_OK;
    if (!q || !out || (pages && (!k_pages || !v_pages)) || (prefix && !prefix_table) || (max_pages && (!table || !lengths))) return CGBN_ERR_NULL;
    const int elem = dtype == CGBN_F32 ? 4 : 2;
    const long long width = (long long)Hq * D;
    if (ldq > (1ll << 32) || ldo > (1ll << 32)) return CGBN_ERR_SHAPE;
    if (T > 1 && (ldq < width || ldo < width)) return CGBN_ERR_STRIDE;
    const uintptr_t sixteen = reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(out) | reinterpret_cast<uintptr_t>(k_pages) | reinterpret_cast<uintptr_t>(v_pages);
    const uintptr_t four = reinterpret_cast<uintptr_t>(rows) | reinterpret_cast<uintptr_t>(lengths) | reinterpret_cast<uintptr_t>(prefix_table) |
                           reinterpret_cast<uintptr_t>(table) | reinterpret_cast<uintptr_t>(lse);
    if (sixteen % 16 || four % 4 || (T > 1 && (ldq * elem % 16 || ldo * elem % 16))) return CGBN_ERR_ALIGN;
    const void* const in[] = {q, rows, lengths, k_pages, v_pages, prefix_table, table, workspace};
    for (const void* p : in)
        if (p && (p == out || p == lse)) return CGBN_ERR_ALIAS;
    if (out == lse) return CGBN_ERR_ALIAS;
    const int line = line_of(width_of(D), elem);
    const Plan p = plan(T, B, Hq, Hk, D, line, elem, prefix, capacity, rows != nullptr);
    if (p.jobs >= (1ll << 24)) return CGBN_ERR_SHAPE;           // 2^32 threads
    AttendArgs A;
    std::memset(&A, 0, sizeof(A));
    const size_t need = scratch(p, T, B, Hq, D, line, elem);
    if (need && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < need)) return CGBN_ERR_WORKSPACE;
    A.part_o = static_cast<float*>(workspace);
    const long long of_parts = part_rows(p, T, Hq, line, elem);
    A.part_ml = reinterpret_cast<float2*>(A.part_o + of_parts * D);
    A.dense = reinterpret_cast<float*>(A.part_ml + of_parts);
    A.own_first = reinterpret_cast<int*>(A.dense + 1);
    A.q = static_cast<const char*>(q); A.k_pages = static_cast<const char*>(k_pages); A.v_pages = static_cast<const char*>(v_pages);
    A.out = static_cast<char*>(out); A.lse = lse; A.rows = rows; A.lengths = lengths; A.prefix_table = prefix_table; A.table = table;
    A.ldq = ldq; A.ldo = ldo; A.T = T; A.B = B; A.Hq = Hq; A.Hk = Hk; A.g = Hq / Hk; A.D = D; A.pages = pages; A.prefix = prefix; A.max_pages = max_pages;
    while ((1 << A.page_bits) < page) ++A.page_bits;
    A.prefix_splits = p.prefix_splits; A.prefix_per = p.prefix_per; A.own_splits = p.own_splits; A.own_least = p.own_least; A.own_groups = p.own_groups; A.prefix_tiles = p.prefix_tiles; A.own_tiles = p.own_tiles;
    A.prefix_jobs = (int)p.prefix_jobs; A.jobs = (int)p.jobs; A.whole = p.whole; A.cut = (int)p.cut; A.tail_splits = p.tail_splits; A.direct = p.parts() <= 1; A.scale = scale * 1.4426950408889634f;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == CGBN_F32 ? launch_attend<float>(A, p.prefix_kind, p.own_kind, st) : launch_attend<bf16_t>(A, p.prefix_kind, p.own_kind, st);
}

}  // extern "C"
