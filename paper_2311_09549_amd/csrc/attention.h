// Attention over packed rows and a paged cache: what the host entry points hand to the kernels, and the index arithmetic that both
// sides (and the host tests) use.  Not part of the public C ABI.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

#include "../../include/sparsecontract.h"

#define ATTN_HD __host__ __device__ __forceinline__

namespace sck {

constexpr int kMaxHeadDim = 256;
constexpr int kMaxPairs = kMaxHeadDim / 2;
constexpr int kHeadTile = 16;      // query heads of one key head that a wavefront of decode works on
constexpr int kDecodeUnit = 128;   // keys: the grain of the split of decode
constexpr int64_t kMaxRows = (1 << 24) - 1;
constexpr int64_t kMaxUnits = (int64_t)1 << 52;   // of decode: 2^10 times as many fit what quotient() takes
constexpr int32_t kMaxKeys = 1 << 30;   // of a sequence: a tile beyond the last one fits 32 bits
constexpr int32_t kMaxBatch = (1 << 20) - 1;
constexpr int kSplitBlocks = 1024;   // of rows of a prompt whose keys are split
constexpr int32_t kMaxNodes = 1024;  // of a tree of drafted rows
constexpr int32_t kMaxGroupsLog2 = 10;   // 2^n workgroups of decode at most

// ------------------------------------------------------------------------------------------
// sequences
// ------------------------------------------------------------------------------------------
struct Sequences {
    int32_t batch;
    int32_t rows;
    const int32_t *row_start;   // null: one row each
    const int32_t *length;      // null: as many keys as rows
    const int32_t *page;
    int64_t page_ld, page_count;
    int32_t page_shift;         // log2 of the rows of a page
    int32_t pages;              // of the cache
};

// First row of sequence b (b == batch: one past the last row), whatever the table holds: within 0..rows.
ATTN_HD int32_t row_begin(const Sequences &s, int32_t b)
{
    const int32_t r = s.row_start ? s.row_start[b] : b;
    return r < 0 ? 0 : r > s.rows ? s.rows : r;
}

// Keys that a sequence's table of pages has room for.
ATTN_HD int64_t table_room(const Sequences &s) { return s.page_count << s.page_shift; }

// Length of a sequence with its keys in pages: -1 for one that the table has no room for.
ATTN_HD int32_t paged_length(const Sequences &s, int32_t b)
{
    const int32_t n = s.length[b];
    return n < 0 || n > table_room(s) || n > kMaxKeys ? -1 : n;
}

// Page of key j of sequence b, -1 for a number that is no page of the cache.  0 <= j < table_room.
ATTN_HD int32_t page_of(const Sequences &s, int32_t b, int32_t j)
{
    const int32_t p = s.page[(int64_t)b * s.page_ld + (j >> s.page_shift)];
    return (uint32_t)p < (uint32_t)s.pages ? p : -1;
}

// Of 64 places base + n * step, n = 0..63, a bit for each that is below `end` and a sequence that begins at row r or before.  On the GPU every lane of
// a wavefront looks at one: a table of 64 is searched in one read's time.
ATTN_HD uint64_t begun(const Sequences &s, int32_t r, int32_t base, int32_t step, int32_t end)
{
#ifdef __HIP_DEVICE_COMPILE__
    const int64_t b = base + (int64_t)(threadIdx.x % 64) * step;
    return __ballot(b < end && row_begin(s, (int32_t)b) <= r);
#else
    uint64_t bits = 0;
    for (int n = 0; n < 64; ++n) {
        const int64_t b = base + (int64_t)n * step;
        if (b < end && row_begin(s, (int32_t)b) <= r) bits |= (uint64_t)1 << n;
    }
    return bits;
#endif
}

// Sequence of row r, which all lanes ask for: the last b whose first row is not after r.  Rows before the first sequence or after the last give
// -1.  For a table that is not in order the answer is some sequence that has the row.
ATTN_HD int32_t sequence_of(const Sequences &s, int32_t r)
{
    if (!s.row_start) return r;
    int32_t base = 0, end = s.batch;
    while (true) {
        const int32_t step = (end - base + 63) / 64;
        const uint64_t bits = begun(s, r, base, step, end);
        if (bits == 0) return -1;
        base += (63 - __builtin_clzll(bits)) * step;
        if (step == 1) break;
        end = end - base < step ? end : base + step;
    }
    return r < row_begin(s, base + 1) ? base : -1;
}

// Blocks of ROWS rows, none across sequences, without a table of them: sequence b is given the numbers from row_begin(b) / ROWS + b
// up to that of b + 1, which is never fewer than it has blocks (floor(y) - floor(x) + 1 >= ceil(y - x)); numbers left over have
// no rows.  rows / ROWS + batch numbers in all.
template <int ROWS>
ATTN_HD int32_t row_blocks(int32_t rows, int32_t batch) { return rows / ROWS + batch; }

template <int ROWS>
ATTN_HD int32_t first_block(const Sequences &s, int32_t b) { return row_begin(s, b) / ROWS + b; }

struct RowBlock {
    int32_t sequence;      // -1: no rows
    int32_t first, end;    // rows of the block [first, end)
    int32_t begin, count;  // rows of its sequence
};

template <int ROWS>
ATTN_HD RowBlock row_block(const Sequences &s, int32_t number)
{
    RowBlock k = {-1, 0, 0, 0, 0};
    int32_t lo = 0, hi = s.batch;   // first_block(lo) <= number
    while (hi - lo > 1) {
        const int32_t mid = lo + ((hi - lo) >> 1);
        if (first_block<ROWS>(s, mid) <= number) lo = mid; else hi = mid;
    }
    const int32_t begin = row_begin(s, lo), end = row_begin(s, lo + 1), at = number - first_block<ROWS>(s, lo);
    if (at < 0 || (int64_t)begin + (int64_t)at * ROWS >= end) return k;
    k.sequence = lo;
    k.begin = begin;
    k.count = end - begin;
    k.first = begin + at * ROWS;
    k.end = k.first + ROWS < end ? k.first + ROWS : end;
    return k;
}

// ------------------------------------------------------------------------------------------
// a window: a row at position p sees keys p - window + 1 .. p, and those of the first `sinks` that are before it
// ------------------------------------------------------------------------------------------

// The first key that a row at position p sees through its window.
ATTN_HD int32_t window_low(int32_t window, int32_t p) { return window > 0 && p >= window ? p - window + 1 : 0; }

// What rows from position p on see of a sequence of `length` keys, as one line: the first keys, up to `first` (whole sixteens, 0 if the line has no gap), then those from
// first + skip on.  Nobody sees the `skip` keys between (whole sixteens too).
struct Span {
    int32_t first, skip, length;   // length: of the line
};

ATTN_HD Span span_of(int32_t length, int32_t window, int32_t sinks, int32_t p)
{
    const int32_t low = window_low(window, p) & ~15;
    if (low > 0 && sinks < low && (sinks + 15 & ~15) < low) {
        const int32_t first = sinks + 15 & ~15;
        return {first, low - first, length - (low - first)};
    }
    return {0, 0, length};
}

// The key at place v of the line.
ATTN_HD int32_t key_at(const Span &s, int32_t v) { return v < s.first ? v : v + s.skip; }

// ------------------------------------------------------------------------------------------
// trees of drafted rows: parent[r] is the row that row r follows, counted from the first row of its sequence, -1 for one that follows what is before the tree
// ------------------------------------------------------------------------------------------

// Whether node i may follow node p.  A number that is neither -1 nor of an earlier row is wrong.
ATTN_HD bool parent_ok(int32_t i, int32_t p) { return p >= -1 && p < i; }

// Depth of node i, or -1 if its chain has a wrong number.  Every step goes to an earlier row.
ATTN_HD int32_t depth_of(const int32_t *parent, int32_t i)
{
    int32_t depth = 0;
    while (true) {
        const int32_t p = parent[i];
        if (!parent_ok(i, p)) return -1;
        if (p < 0) return depth;
        i = p;
        ++depth;
    }
}

// ------------------------------------------------------------------------------------------
// split of decode: the units of all segments (a segment is a sequence and a tile of the heads of one key head) in one
// line, a workgroup takes an equal share of it
// ------------------------------------------------------------------------------------------
ATTN_HD int32_t units_of(int32_t length) { return length <= 0 ? 0 : (length - 1) / kDecodeUnit + 1; }

// x / y, rounded down, for 0 <= x < 2^62, 0 < y and a quotient below 2^50.  A division of 64-bit integers is some hundred instructions on a GPU, and every workgroup makes a few
// before its first load; one in fp64, corrected, is thirty.
ATTN_HD int64_t quotient(int64_t x, int64_t y)
{
    int64_t q = (int64_t)((double)x / (double)y);   // off by one at most
    if (q * y > x) --q;
    if ((q + 1) * y <= x) ++q;
    return q;
}

// First unit of workgroup w of 2^groups_log2: the w-th part of the line, rounded down.
ATTN_HD int64_t share_begin(int64_t units, int32_t w, int32_t groups_log2) { return (units * w) >> groups_log2; }

// The workgroup that has unit u (0 <= u < units): the last w with share_begin(w) < u + 1.
ATTN_HD int32_t share_of(int64_t units, int64_t u, int32_t groups_log2) { return (int32_t)quotient(((u + 1) << groups_log2) - 1, units); }

// A workgroup has at most two segments that others have parts of: the one its share begins in and the one it ends in.  The piece of the
// first goes to slot 2 w, that of another one to 2 w + 1.
ATTN_HD int32_t piece_slot(int64_t segment_first, int64_t share_first, int32_t w) { return 2 * w + (share_first < segment_first ? 1 : 0); }

// ------------------------------------------------------------------------------------------
// arguments of the kernels (strides in elements)
// ------------------------------------------------------------------------------------------
struct Rows {
    void *data;
    int64_t row, head;
};

struct Cache {
    void *keys, *values;
    int64_t page, row, head;
};

struct AppendArgs {
    Sequences s;
    Rows q, k, v, q_out;
    Cache cache;
    int32_t heads, kv_heads, head_dim, pairs, interleaved;
    const int32_t *parent;      // null: rows are in order
    double turns[kMaxPairs];    // turns per position of each pair
};

struct AttendArgs {
    Sequences s;
    Rows q, k, v, out;          // k and v: packed keys
    Cache cache;                // keys in pages
    int32_t heads, kv_heads, group, head_dim, causal;
    float scale_log2;           // scale / ln 2: weights are powers of two
    int32_t groups_log2;        // decode: workgroups
    int32_t head_tiles;         // decode: tiles of kHeadTile heads of one key head
    float *pieces;              // decode: per slot 16 rows of padded head_dim sums, 16 maxima, 16 sums of weights; prompt: null, or room for prompt_tile.h's
    int32_t *cut;               // prompt: blocks that each share has pieces of
    int32_t blocks;             // prompt: numbers of blocks of rows
    int32_t n_cu;
    int32_t window, sinks;      // window 0: every key before a row
    const int32_t *parent;      // trees: null, rows are in order
    int32_t tree;               // rows of trees: no more of them than keys, and no more than kMaxNodes where they have parents
    struct TreeCut *tree_cut;   // trees: the segment that each workgroup leaves to others
};

// The segment that a workgroup began and left to others, for the kernel that joins its pieces: its place in the line and units, and those of the whole line.  No units: none.
struct TreeCut {
    int64_t first, all;
    int32_t units, b, kv, tile;
};

// The accepted rows of trees.
struct AcceptArgs {
    Sequences s;
    Cache cache;
    int32_t kv_heads, head_dim;
    const int32_t *parent, *last;
    int32_t *length_out;        // null: not wanted
};

// Pages of the sequences that come after (new_batch of them) from those that are.
struct ForkArgs {
    int32_t batch, new_batch, columns, pages, page_shift, window, sinks;
    const int32_t *page, *length, *holders;
    int64_t page_ld;
    const int32_t *parent, *wanted;   // wanted null: as many rows as the parent has
    int32_t *page_out, *length_out, *holders_out, *moves;
    int64_t page_out_ld;
    // workspace
    int32_t *keeper;        // per page: the first sequence that keeps it in part
    uint64_t *free_bits;    // per page
    int32_t *free_before;   // per block of pages: how many are free
    int64_t *needed;        // per sequence: pages that those before it take
};

struct CompactArgs {
    int32_t batch, columns, pages, page_shift;
    const int32_t *page, *length, *holders;
    int64_t page_ld;
    int32_t *page_out, *holders_out, *moves;
    int64_t page_out_ld;
    // workspace
    int32_t *to;            // per page: where it goes
    uint64_t *used_bits;    // per page
    int32_t *used_before;   // per block of pages: how many are in use
};

struct CopyArgs {
    Cache cache;
    int32_t kv_heads, head_dim, page_shift, pages;
    const int32_t *moves;
    int64_t count;
};

// Padded head_dim of the kernels.
ATTN_HD int padded_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }
ATTN_HD int piece_floats(int padded) { return kHeadTile * (padded + 2); }

// Workgroups that a split prompt has, and the bytes of its pieces and of its table (0: a type that is not split).
int prompt_shares(int n_cu);
size_t prompt_workspace(sc_dtype dtype, int head_dim, int n_cu);

// The same for trees, and for single rows through a window.  The table of cut segments is behind the pieces.
size_t tree_pieces(int head_dim, int groups_log2);
size_t row_pieces(int head_dim, int groups_log2);
inline size_t cut_bytes(int groups_log2) { return sizeof(TreeCut) << groups_log2; }

// Pages that a workgroup of fork and compact counts.
constexpr int32_t kPagesPerBlock = 4096;
constexpr int32_t kMaxPages = 1 << 30;
inline int32_t blocks_of_pages(int32_t pages) { return (pages + kPagesPerBlock - 1) / kPagesPerBlock; }

hipError_t launch_append(const AppendArgs &a, sc_dtype dtype, hipStream_t stream);
hipError_t launch_prompt(const AttendArgs &a, sc_dtype dtype, bool paged, hipStream_t stream);
hipError_t launch_prompt_window(const AttendArgs &a, sc_dtype dtype, bool paged, hipStream_t stream);
hipError_t launch_prompt_tree(const AttendArgs &a, sc_dtype dtype, hipStream_t stream);   // 16-bit types
hipError_t launch_decode(const AttendArgs &a, sc_dtype dtype, hipStream_t stream);
hipError_t launch_tree(const AttendArgs &a, sc_dtype dtype, hipStream_t stream);
hipError_t launch_accept(const AcceptArgs &a, sc_dtype dtype, hipStream_t stream);
hipError_t launch_fork(const ForkArgs &a, hipStream_t stream);
hipError_t launch_compact(const CompactArgs &a, hipStream_t stream);
hipError_t launch_copy(const CopyArgs &a, sc_dtype dtype, hipStream_t stream);

}  // namespace sck

struct sc_attention {
    sc_dtype dtype;
    int32_t heads, kv_heads, head_dim, page_rows, page_shift, causal;
    float scale_log2;
    int32_t pairs, interleaved;
    double turns[sck::kMaxPairs];
    bool has_device;
    int32_t n_cu;
    int32_t groups_log2;
    size_t ws_bytes, prompt_ws_bytes, tree_ws_bytes;
    int32_t window, sinks;
};
