// Index arithmetic of attention on the host: blocks of rows, pages, and the split of decode, for good tables and for wrong ones.
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "../../paper_2311_09549_amd/csrc/attention.h"

using namespace sck;

#define CHECK(x)                                                  \
    do {                                                          \
        if (!(x)) {                                               \
            printf("%s:%d: %s\n", __FILE__, __LINE__, #x);        \
            exit(1);                                              \
        }                                                         \
    } while (0)

template <int ROWS>
static void blocks_cover(const std::vector<int32_t> &start, int32_t rows, bool in_order)
{
    Sequences s = {};
    s.batch = (int32_t)start.size() - 1;
    s.rows = rows;
    s.row_start = start.data();
    std::vector<int> times(rows, 0);
    for (int32_t n = 0; n < row_blocks<ROWS>(rows, s.batch); ++n) {
        const RowBlock k = row_block<ROWS>(s, n);
        if (k.sequence < 0) continue;
        CHECK(k.sequence < s.batch && k.first >= 0 && k.first < k.end && k.end <= rows && k.end - k.first <= ROWS);
        CHECK(k.begin >= 0 && k.count > 0 && k.begin + (int64_t)k.count <= rows && k.first >= k.begin && k.end <= k.begin + k.count);
        for (int32_t r = k.first; r < k.end; ++r) ++times[r];
        if (in_order)
            for (int32_t r = k.first; r < k.end; ++r) CHECK(sequence_of(s, r) == k.sequence);
    }
    for (int32_t r = 0; in_order && r < rows; ++r) {
        const bool inside = r >= row_begin(s, 0) && r < row_begin(s, s.batch);
        CHECK(times[r] == (inside ? 1 : 0));
        if (!inside) CHECK(sequence_of(s, r) == -1);
    }
    for (int32_t r = 0; r < rows; ++r) {
        const int32_t b = sequence_of(s, r);
        CHECK(b >= -1 && b < s.batch);
    }
}

static void split_covers(const std::vector<int32_t> &length, int32_t segments, int32_t groups_log2)
{
    int64_t units = 0;
    for (const int32_t n : length) units += units_of(n);
    units *= segments;
    const int32_t groups = 1 << groups_log2;
    const auto share_begin = [&](int64_t all, int32_t w, int32_t) { return sck::share_begin(all, w, groups_log2); };
    const auto share_of = [&](int64_t all, int64_t u, int32_t) { return sck::share_of(all, u, groups_log2); };
    CHECK(share_begin(units, 0, groups) == 0 && share_begin(units, groups, groups) == units);
    std::vector<int> slot(2 * groups, 0);
    int64_t first = 0;
    for (const int32_t n : length)
        for (int32_t g = 0; g < segments; ++g) {
            const int32_t u = units_of(n);
            if (u == 0) continue;
            const int32_t w0 = share_of(units, first, groups), w1 = share_of(units, first + u - 1, groups);
            CHECK(0 <= w0 && w0 <= w1 && w1 < groups);
            CHECK(share_begin(units, w0, groups) <= first && first < share_begin(units, w0 + 1, groups));
            CHECK(share_begin(units, w1, groups) < first + u && first + u <= share_begin(units, w1 + 1, groups));
            for (int32_t w = w0; w0 != w1 && w <= w1; ++w) {
                if (share_begin(units, w, groups) == share_begin(units, w + 1, groups)) continue;
                const int32_t at = piece_slot(first, share_begin(units, w, groups), w);
                CHECK(at >= 0 && at < 2 * groups && slot[at]++ == 0);   // no two pieces share a slot
            }
            first += u;
        }
    CHECK(first == units);
}

int main()
{
    std::mt19937 rng(1);
    const auto below = [&](int n) { return (int32_t)(rng() % (uint32_t)n); };
    for (int round = 0; round < 400; ++round) {
        std::vector<int32_t> start = {round % 3 ? 0 : below(5)};
        for (int b = below(20); b >= 0; --b) start.push_back(start.back() + (below(3) ? below(200) : 0));
        const int32_t rows = start.back() + (round % 2 ? 0 : below(70));
        blocks_cover<64>(start, rows, true);
        blocks_cover<128>(start, rows, true);
        blocks_cover<256>(start, rows, true);
        for (int32_t &x : start)   // anything at all
            if (below(3) == 0) x = (int32_t)rng();
        blocks_cover<64>(start, rows, false);
        blocks_cover<256>(start, rows, false);
    }
    for (int round = 0; round < 400; ++round) {
        std::vector<int32_t> length;
        for (int b = below(40); b >= 0; --b) length.push_back(below(4) ? below(round % 5 ? 1000 : 100000) : 0);
        split_covers(length, 1 + below(9), below(round % 2 ? 11 : 4));
    }
    split_covers(std::vector<int32_t>(3, 2147483647), 64, 10);
    for (int round = 0; round < 200000; ++round) {   // quotients below 2^50 of numbers below 2^62
        const auto any = [&](int bits) { return (int64_t)(((uint64_t)rng() << 32 | rng()) >> (64 - bits)); };
        const int64_t y = 1 + any(1 + below(40)), q = any(1 + below(50));
        for (const int64_t r : {(int64_t)0, y - 1, any(62) % y})
            if (q <= (((int64_t)1 << 62) - 1 - r) / y) CHECK(quotient(q * y + r, y) == q);
    }

    const int32_t table[6] = {0, 4, -1, 5, 2147483647, 3}, lengths[4] = {-1, 33, 48, 49};
    Sequences s = {};
    s.batch = 2;
    s.page = table;
    s.page_ld = 3;
    s.page_count = 3;
    s.page_shift = 4;
    s.pages = 5;
    s.length = lengths;
    CHECK(table_room(s) == 48);
    CHECK(page_of(s, 0, 0) == 0 && page_of(s, 0, 15) == 0 && page_of(s, 0, 16) == 4 && page_of(s, 0, 47) == -1);
    CHECK(page_of(s, 1, 0) == -1 && page_of(s, 1, 16) == -1 && page_of(s, 1, 32) == 3);
    CHECK(paged_length(s, 0) == -1 && paged_length(s, 1) == 33 && paged_length(s, 2) == 48 && paged_length(s, 3) == -1);
    s.page_count = 2147483647;
    s.page_shift = 12;
    CHECK(table_room(s) == (int64_t)2147483647 << 12);
    printf("ok\n");
    return 0;
}
