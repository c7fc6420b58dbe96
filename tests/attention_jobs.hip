// What the attention's workgroups do with the arguments that a call gives them, followed on the host: the entry point is the library's, in the place of
// the launch stands a function that looks where every workgroup would store.  Reads calls from stdin, one a line:
//   elem T B single Hq Hk D prefix max_pages page fresh...           (fresh: new tokens of each request, none if single)
// and answers with a line each: "ok", what it found wrong, or the status if the call is refused.  Or a request's rows, which it answers with the keys that each sees:
//   sees fresh tokens max_pages page g
#include "cgbn.h"
#include "cgbn_attention.h"

#include <algorithm>
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>
#include <vector>

namespace cgbn {

static std::string found;
static size_t workspace_bytes;

static void wrong(const char* what, long long a, long long b)
{
    char text[200];
    std::snprintf(text, sizeof(text), "%s: %lld, %lld", what, a, b);
    if (found.empty()) found = text;
}

// Workgroups of the prefix and, where they are not dealt by the lengths, of own keys: rows that go to parts lie in the workspace, each of them has a place of
// its own, and a call without a join has none
template <typename T> static void look(const AttendArgs& A, int prefix_kind, int own_kind)
{
    const int elem = (int)sizeof(T), line = line_of(width_of(A.D), elem);
    const size_t room = workspace_bytes / sizeof(float);
    const long long parts = reinterpret_cast<float*>(A.part_ml) - A.part_o;          // floats of the parts' products
    const bool dealt = !A.whole && A.own_splits > 1;
    std::vector<char> taken(parts / A.D);
    auto store = [&](const Place& to, int rows_of_a_tile, long long row, int at) {
        if (to.direct) return;
        const long long r = to.part_row(A, rows_of_a_tile, row, at);
        if (r < 0 || (r + 1) * A.D > parts || (size_t)(parts + (r + 1) * 2) > room) return wrong("a part behind the workspace: row, workgroup", r, to.id);
        if (taken[r]++) wrong("two stores to a row of the parts: row, workgroup", r, to.id);
    };
    for (int id = 0; id < A.prefix_jobs; ++id) {
        const int rows = rows_of(prefix_kind, line, elem), split = id / A.Hk / A.prefix_tiles, head = id % A.Hk;
        const RowsOf w = RowsOf::of_prefix(A, id / A.Hk % A.prefix_tiles * rows);
        const Place to = {id, split, true, Place::is_direct(A, true, Place::first_parts(A, true))};
        if (A.direct != to.direct) wrong("a prefix's workgroup stores parts and nothing joins them, or the other way: direct, workgroup", A.direct, id);
        for (int at = 0; at < rows && w.r0 + at < w.count; ++at) {
            const int r = w.r0 + at, token = r / A.g;
            store(to, rows, (long long)token * A.Hq + head * A.g + (r - token * A.g), at);
        }
    }
    if (dealt || A.jobs == A.prefix_jobs) return;
    for (int id = 0; id < A.jobs - A.prefix_jobs; ++id) {
        const int rows = rows_of(own_kind, line, elem);
        Place to = {id, 0, false, false};
        int parts_of_it = Place::first_parts(A, false);
        if (A.whole && id >= A.cut) {
            to.split = (id - A.cut) % A.tail_splits;
            parts_of_it = A.tail_splits;
        }
        to.direct = Place::is_direct(A, false, parts_of_it);
        if (A.whole && to.direct != (id < A.cut || A.tail_splits == 1)) wrong("a tile is shared and its parts are not joined, or the other way: workgroup", id, A.cut);
        if (!A.whole && to.direct != (A.direct != 0)) wrong("own keys go to parts and nothing joins them, or the other way: workgroup", id, A.direct);
        if (!A.whole) {
            // (a tile's rows are its request's; every row of all is some tile's)
            for (int at = 0; !A.rows && at < rows; ++at) {
                const int per = (A.g + rows - 1) / rows, tile = id / A.Hk, r = (tile % per) * rows + at;
                if (r < A.g) store(to, rows, (long long)(tile / per) * A.Hq + id % A.Hk * A.g + r, at);
            }
        } else {
            for (int at = 0; at < rows; ++at) store(to, rows, 0, at);
        }
    }
}

template <> cgbn_status launch_attend<float>(const AttendArgs& A, int prefix, int own, hipStream_t)
{
    look<float>(A, prefix, own);
    return CGBN_OK;
}
template <> cgbn_status launch_attend<bf16_t>(const AttendArgs& A, int prefix, int own, hipStream_t)
{
    look<bf16_t>(A, prefix, own);
    return CGBN_OK;
}

}  // namespace cgbn

#include "cgbn_attention.hip"

static void sees(std::istringstream& in)
{
    std::string word;
    int fresh, tokens, max_pages, page, g;
    in >> word >> fresh >> tokens >> max_pages >> page >> g;
    AttendArgs A;
    std::memset(&A, 0, sizeof(A));
    const int rows[2] = {0, fresh};
    A.rows = rows; A.lengths = &tokens; A.T = fresh; A.B = 1; A.Hk = 1; A.Hq = A.g = g; A.max_pages = max_pages; A.page_bits = __builtin_ctz(page);
    for (int r0 = 0; r0 < fresh * g; r0 += 16) {
        const RowsOf w = RowsOf::of_request(A, Request(A, 0, 16), 0, r0);
        for (int at = 0; at < 16 && r0 + at < fresh * g; ++at) std::printf("%d ", w.sees(A, at));
        if (w.sees(A, std::min(16, fresh * g - r0) - 1) != w.end(A, 16) || w.sees(A, 16 + fresh * g)) std::printf("wrong end of %d ", r0);
    }
    std::printf("\n");
}

int main()
{
    std::string text;
    while (std::getline(std::cin, text)) {
        std::istringstream in(text);
        if (text.compare(0, 4, "sees") == 0) {
            sees(in);
            continue;
        }
        int elem, B, single, Hq, Hk, D, prefix, max_pages, page, n;
        long long T;
        in >> elem >> T >> B >> single >> Hq >> Hk >> D >> prefix >> max_pages >> page;
        std::vector<int> rows(1, 0), lengths(B + 1, 1);
        while (in >> n) rows.push_back(rows.back() + n);
        char* const at = reinterpret_cast<char*>(1ll << 40);          // (addresses that nothing follows)
        const cgbn_dtype dtype = elem == 4 ? CGBN_F32 : CGBN_BF16;
        workspace_bytes = cgbn_prefix_attention_workspace_bytes(T, B, Hq, Hk, D, prefix, (long long)max_pages * page, dtype);
        found.clear();
        // of 256 bytes and less a program may pass none
        const bool none = workspace_bytes <= 256;
        if (none) workspace_bytes = 0;
        const cgbn_status code = cgbn_prefix_attention(at, (long long)Hq * D, T, B, single ? nullptr : rows.data(), lengths.data(), Hq, Hk, D, 1.f, at + (1 << 20),
                                                       at + (2 << 20), 4, page, reinterpret_cast<int*>(at + (3 << 20)), prefix, reinterpret_cast<int*>(at + (4 << 20)),
                                                       max_pages, at + (5 << 20), (long long)Hq * D, reinterpret_cast<float*>(at + (6 << 20)), dtype,
                                                       none ? nullptr : at + (7 << 20), workspace_bytes, nullptr);
        if (code) std::printf("status %d\n", code);
        else std::printf("%s\n", found.empty() ? "ok" : found.c_str());
    }
    return 0;
}
