// Pages of a cache: the accepted rows of trees, the next batch of sequences from the present one, pages moved to the lowest numbers, and copies of pages.
//
// Tables are integers by the thousand and rows are moved as they are: bound by launches and chains of reads, and by memory where pages move.
//
// The next batch of eight beams up to 700 rows in one workgroup 8 us, 23 with the same steps on tables in memory instead of LDS; 384 beams up to 8,191 rows, 32,000 pages, in
// four kernels of 2.5, 7.9, 3.9 and 6.2 us.  130 pages to the lowest numbers 5.3 us; 5,900 pages, of which 1,200 of 512 KB move, 12 us and 135 for the copies, 4.6 TB/s.  Accepted
// paths of one tree 4 us, of 192 trees of up to 63 nodes 7.
#include "attention_device.h"

namespace sck {

namespace {

constexpr int kThreads = 256;
constexpr int32_t kNone = 0x7fffffff;   // no sequence

// -- accepted rows ---------------------------------------------------------------------------------------------------------------
// Rows of a path move to the places 0, 1, .. of their tree, each to its own place or an earlier one.  A thread has 16 bytes of every row: it takes the rows in order, eight on
// their way at a time, so that none is overwritten before it is read.
constexpr int kRowsAhead = 8;

__global__ void __launch_bounds__(kThreads) accept_kernel(AcceptArgs a, int32_t elem_bytes)
{
    __shared__ int32_t path_s[kMaxNodes];
    __shared__ int64_t from_s[kMaxNodes], to_s[kMaxNodes];   // elements; from -1: the row stays, or has no place
    const int32_t b = blockIdx.x;
    const int32_t begin = row_begin(a.s, b), count = row_begin(a.s, b + 1) - begin, length = paged_length(a.s, b), before = length - count;
    const int32_t last = a.last[b];
    // the path, from its end, by every thread alike
    int32_t n = 0;
    bool wrong = length < 0 || before < 0 || count < 0 || count > kMaxNodes || last < -1 || last >= count;
    if (!wrong) {
        for (int32_t i = last; i >= 0; ++n) {
            if (threadIdx.x == 0) path_s[n] = i;
            const int32_t p = a.parent[begin + i];
            if (!parent_ok(i, p)) {
                wrong = true;
                break;
            }
            i = p;
        }
    }
    if (blockIdx.y == 0 && threadIdx.x == 0 && a.length_out) a.length_out[b] = wrong ? -1 : before + n;
    if (wrong) return;
    __syncthreads();
    const auto place = [&](int32_t key) -> int64_t {
        const int32_t page = page_of(a.s, b, key);
        return page < 0 ? -1 : page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row;
    };
    for (int32_t d = threadIdx.x; d < n; d += kThreads) {
        const int32_t i = path_s[n - 1 - d];
        const int64_t to = place(before + d);
        from_s[d] = i == d || to < 0 ? -1 : place(before + i);
        to_s[d] = to;
    }
    __syncthreads();
    const int32_t per_head = a.head_dim * elem_bytes / 16, pieces = a.kv_heads * per_head, x = blockIdx.y * kThreads + threadIdx.x;
    if (x >= 2 * pieces) return;
    const int32_t y = x < pieces ? x : x - pieces, h = y / per_head;
    char *cache = static_cast<char *>(x < pieces ? a.cache.keys : a.cache.values) + h * a.cache.head * elem_bytes + (y - h * per_head) * 16;
    for (int32_t d = 0; d < n; d += kRowsAhead) {
        u32x4 v[kRowsAhead];
#pragma unroll
        for (int k = 0; k < kRowsAhead; ++k)
            if (d + k < n && from_s[d + k] >= 0) v[k] = *reinterpret_cast<const u32x4 *>(cache + from_s[d + k] * elem_bytes);
#pragma unroll
        for (int k = 0; k < kRowsAhead; ++k)
            if (d + k < n && from_s[d + k] >= 0) *reinterpret_cast<u32x4 *>(cache + to_s[d + k] * elem_bytes) = v[k];
    }
}

// -- copies ----------------------------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kThreads) copy_kernel(CopyArgs a, int32_t elem_bytes)
{
    const int64_t move = blockIdx.x;
    const int32_t from = a.moves[3 * move], to = a.moves[3 * move + 1], page_rows = 1 << a.page_shift;
    int32_t rows = a.moves[3 * move + 2];
    if ((uint32_t)from >= (uint32_t)a.pages || (uint32_t)to >= (uint32_t)a.pages || from == to) return;
    rows = rows < page_rows ? rows : page_rows;
    const int32_t per_head = a.head_dim * elem_bytes / 16, per_row = a.kv_heads * per_head;
    const int64_t all = 2 * (int64_t)rows * per_row;
    for (int64_t x = (int64_t)blockIdx.y * kThreads + threadIdx.x; x < all; x += (int64_t)gridDim.y * kThreads) {
        const bool keys = x < all / 2;
        const int32_t y = (int32_t)(keys ? x : x - all / 2), r = y / per_row, z = y - r * per_row, h = z / per_head;
        char *cache = static_cast<char *>(keys ? a.cache.keys : a.cache.values) + (r * a.cache.row + h * a.cache.head) * elem_bytes + (z - h * per_head) * 16;
        *reinterpret_cast<u32x4 *>(cache + to * a.cache.page * elem_bytes) = *reinterpret_cast<const u32x4 *>(cache + from * a.cache.page * elem_bytes);
    }
}

// -- the next batch --------------------------------------------------------------------------------------------------------------
// Fork and compact are a few steps over tables, each of which needs the one before it whole.  Small tables: one workgroup takes all steps; others: a kernel for each.
constexpr int kWide = 1024;   // threads of a workgroup of theirs

// Sum over the threads of a workgroup, and of those before each.
template <typename T>
__device__ __forceinline__ T sum_before(T x, T &all)
{
    __shared__ T wave_s[kWide / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    T upto = x;
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const T y = __shfl_up(upto, d);
        upto += lane >= d ? y : 0;
    }
    __syncthreads();
    if (lane == 63) wave_s[wave] = upto;
    __syncthreads();
    T before = 0;
    all = 0;
#pragma unroll
    for (int k = 0; k < kWide / 64; ++k) {
        before += k < wave ? wave_s[k] : 0;
        all += wave_s[k];
    }
    return before + upto - x;
}

// A bit for each of the kPagesPerBlock pages of a block, and how many are set.
template <typename IS>
__device__ __forceinline__ void count_block(int32_t block, int32_t pages, uint64_t *bits, int32_t *count, const IS &is)
{
    __shared__ int32_t wave_s[kWide / 64];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    int32_t n = 0;
#pragma unroll
    for (int k = 0; k < kPagesPerBlock; k += kWide) {
        const int64_t p = (int64_t)block * kPagesPerBlock + k + threadIdx.x;
        const uint64_t word = __ballot(p < pages && is((int32_t)p));
        if (lane == 0) bits[p / 64] = word;
        n += __popcll(word);
    }
    __syncthreads();
    if (lane == 0) wave_s[wave] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
        n = 0;
        for (int k = 0; k < kWide / 64; ++k) n += wave_s[k];
        count[block] = n;
    }
}

// Of the counts of all blocks: the sum of those before one, and of all.
__device__ __forceinline__ void sum_counts(const int32_t *count, int32_t blocks, int32_t block, int32_t &before, int32_t &all)
{
    before = all = 0;
    for (int32_t k0 = 0; k0 < blocks; k0 += kWide) {
        const int32_t k = k0 + (int32_t)threadIdx.x, n = k < blocks ? count[k] : 0;
        int32_t sum;
        sum_before(k < block ? n : 0, sum);
        before += sum;
        sum_before(n, sum);
        all += sum;
    }
}

// Calls f(page, whether its bit is set, set bits before it) for the pages of a block, of which each wavefront looks at the words by itself.
template <typename F>
__device__ __forceinline__ void each_page(int32_t block, int32_t pages, const uint64_t *bits, int32_t before, const F &f)
{
    static_assert(kPagesPerBlock == 64 * 64, "a word for each lane");
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const uint64_t word = bits[(int64_t)block * 64 + lane];
    int32_t upto = __popcll(word);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        const int32_t y = __shfl_up(upto, d);
        upto += lane >= d ? y : 0;
    }
    upto -= __popcll(word);
#pragma unroll
    for (int k = 0; k < kPagesPerBlock / kWide; ++k) {
        const int at = k * (kWide / 64) + wave;
        const uint64_t w = __shfl(word, at);
        const int64_t p = (int64_t)block * kPagesPerBlock + 64 * at + lane;
        const int32_t rank = before + __shfl(upto, at) + __popcll(w & (((uint64_t)1 << lane) - 1));
        if (p < pages) f((int32_t)p, (bool)(w >> lane & 1), rank);
    }
}

// What sequence i of the next batch has of the present one.
struct Branch {
    int32_t parent;         // -1: nothing
    int32_t kept, wanted;   // rows; wanted -1: wrong
};

__device__ __forceinline__ int32_t fork_length(const ForkArgs &a, int32_t b)
{
    const int32_t n = a.length[b];
    return n < 0 || n > (int64_t)a.columns << a.page_shift || n > kMaxKeys ? -1 : n;
}

__device__ __forceinline__ Branch branch_of(const ForkArgs &a, int32_t i)
{
    Branch r = {a.parent[i], 0, -1};
    if (r.parent < -1 || r.parent >= a.batch) return r;
    const int32_t n = r.parent < 0 ? 0 : fork_length(a, r.parent);
    const int32_t wanted = a.wanted ? a.wanted[i] : n;
    if (n < 0 || wanted < 0 || wanted > (int64_t)a.columns << a.page_shift || wanted > kMaxKeys) return r;
    r.wanted = wanted;
    r.kept = n < wanted ? n : wanted;
    return r;
}

__device__ __forceinline__ int32_t columns_of(int32_t rows, int32_t shift) { return rows <= 0 ? 0 : ((rows - 1) >> shift) + 1; }

// Whether a sequence that keeps `kept` rows keeps its column c: not a page that is wholly behind the window of the next row, and of the last one.
__device__ __forceinline__ bool column_kept(const ForkArgs &a, int32_t c, int32_t kept)
{
    const int64_t first = (int64_t)c << a.page_shift;
    return first < kept && (a.window == 0 || first < a.sinks || first + (1 << a.page_shift) > (int64_t)kept - a.window);
}

// Page of an entry, -1 for a number that is none.
__device__ __forceinline__ int32_t entry_of(const ForkArgs &a, int32_t b, int32_t c)
{
    const int32_t p = a.page[b * a.page_ld + c];
    return (uint32_t)p < (uint32_t)a.pages ? p : -1;
}

// The page that sequence i is going to write to, which it keeps in part; -1: none.
__device__ __forceinline__ int32_t page_in_part(const ForkArgs &a, const Branch &r)
{
    if (r.wanted < 0 || r.parent < 0 || (r.kept & ((1 << a.page_shift) - 1)) == 0) return -1;
    return entry_of(a, r.parent, r.kept >> a.page_shift);
}

// First step, page by page.
__device__ __forceinline__ void fork_begin(const ForkArgs &a, int64_t p)
{
    a.holders_out[p] = a.holders[p];
    a.keeper[p] = kNone;
}

// Second step, entry by entry: those of the present batch (rows 0 .. batch - 1) hold their pages no more, whole ones of the next do.  Sums and minima of whole numbers: their
// order does not matter.
__device__ __forceinline__ void fork_hold(const ForkArgs &a, int32_t row, int32_t c0, int32_t step)
{
    if (row < a.batch) {
        const int32_t columns = columns_of(fork_length(a, row), a.page_shift);
        for (int32_t c = c0; c < columns; c += step) {
            const int32_t p = entry_of(a, row, c);
            if (p >= 0) atomicAdd(a.holders_out + p, -1);
        }
        return;
    }
    const int32_t i = row - a.batch;
    const Branch r = branch_of(a, i);
    for (int32_t c = c0; c < a.columns; c += step) {
        int32_t entry = -1;
        if (r.wanted >= 0 && r.parent >= 0 && column_kept(a, c, r.kept)) {
            entry = entry_of(a, r.parent, c);
            if (entry >= 0) {
                if (c == r.kept >> a.page_shift) atomicMin(a.keeper + entry, i);
                else atomicAdd(a.holders_out + entry, 1);
            }
        }
        a.page_out[i * a.page_out_ld + c] = entry;
    }
}

// Third step: free pages, and the pages that the sequences before each take.  A sequence is left with the page that it keeps in part if it is the first of those and none holds
// it whole.
__device__ __forceinline__ void fork_count(const ForkArgs &a, int32_t block)
{
    count_block(block, a.pages, a.free_bits, a.free_before, [&](int32_t p) { return a.holders_out[p] == 0 && a.keeper[p] == kNone; });
}

__device__ __forceinline__ void fork_need(const ForkArgs &a)
{
    int64_t before = 0, all;
    for (int32_t i0 = 0; i0 < a.new_batch; i0 += kWide) {
        const int32_t i = i0 + (int32_t)threadIdx.x;
        int64_t mine = 0;
        if (i < a.new_batch) {
            const Branch r = branch_of(a, i);
            const int32_t part = page_in_part(a, r);
            const bool copied = part >= 0 && !(a.keeper[part] == i && a.holders_out[part] == 0);
            if (r.wanted >= 0) mine = (copied ? 1 : 0) + columns_of(r.wanted, a.page_shift) - columns_of(r.kept, a.page_shift);
        }
        const int64_t mine_before = sum_before(mine, all);
        if (i < a.new_batch) a.needed[i] = before + mine_before;
        before += all;
    }
    if (threadIdx.x == 0) a.needed[a.new_batch] = before;
}

__device__ __forceinline__ bool served(const ForkArgs &a, int32_t i, int32_t free_all)
{
    const int64_t upto = a.needed[i + 1];
    return upto == a.needed[i] || upto <= free_all;
}

// Fourth step, for kWide sequences from i0 on: lengths, moves, and holders of pages that are kept in part.
__device__ __forceinline__ void fork_finish(const ForkArgs &a, int32_t i0, int32_t free_all)
{
    __shared__ int32_t dropped_s[kWide];
    const int32_t i = i0 + (int32_t)threadIdx.x;
    bool dropped = false;
    if (i < a.new_batch) {
        const Branch r = branch_of(a, i);
        const bool is = r.wanted >= 0 && served(a, i, free_all);
        const int32_t part = page_in_part(a, r);
        const bool copied = is && part >= 0 && a.needed[i + 1] - a.needed[i] > columns_of(r.wanted, a.page_shift) - columns_of(r.kept, a.page_shift);
        a.length_out[i] = is ? r.wanted : -1;
        a.moves[3 * (int64_t)i] = copied ? part : -1;
        if (!copied) a.moves[3 * (int64_t)i + 1] = -1;
        a.moves[3 * (int64_t)i + 2] = copied ? r.kept & ((1 << a.page_shift) - 1) : 0;
        if (is && part >= 0 && !copied) a.holders_out[part] = 1;
        dropped = r.wanted >= 0 && !is;
    }
    dropped_s[threadIdx.x] = dropped;
    if (!__syncthreads_or(dropped)) return;
    // those that found no room hold nothing
    for (int k = 0; k < kWide; ++k) {
        if (!dropped_s[k]) continue;
        const int32_t part = branch_of(a, i0 + k).kept >> a.page_shift;   // of a page kept in part the holder was not counted
        for (int32_t c = threadIdx.x; c < a.columns; c += kWide) {
            int32_t &entry = a.page_out[(i0 + k) * a.page_out_ld + c];
            if (entry >= 0 && c != part) atomicAdd(a.holders_out + entry, -1);
            entry = -1;
        }
    }
}

// And for the pages of a block: the n-th free page goes to the sequence that takes it.
__device__ __forceinline__ void fork_take(const ForkArgs &a, int32_t block, int32_t before, int32_t free_all)
{
    const int64_t taken_all = a.needed[a.new_batch];
    if (before >= taken_all) return;
    each_page(block, a.pages, a.free_bits, before, [&](int32_t p, bool is, int32_t rank) {
        if (!is || rank >= taken_all) return;
        // the last sequence that begins at this page or before, which takes some
        int32_t lo = 0, hi = a.new_batch;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) / 2;
            if (a.needed[mid] <= rank) lo = mid; else hi = mid;
        }
        if (!served(a, lo, free_all)) return;
        const Branch r = branch_of(a, lo);
        const int32_t first = columns_of(r.kept, a.page_shift), grown = columns_of(r.wanted, a.page_shift) - first;
        const int64_t mine = a.needed[lo];
        const int32_t copied = (int32_t)(a.needed[lo + 1] - mine) - grown, n = (int32_t)(rank - mine);
        if (n < copied) a.moves[3 * (int64_t)lo + 1] = p;
        a.page_out[lo * a.page_out_ld + (n < copied ? r.kept >> a.page_shift : first + n - copied)] = p;
        a.holders_out[p] = 1;
    });
}

__global__ void __launch_bounds__(kThreads) fork_begin_kernel(ForkArgs a)
{
    const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (p < a.pages) fork_begin(a, p);
}

__global__ void __launch_bounds__(kThreads) fork_hold_kernel(ForkArgs a) { fork_hold(a, blockIdx.x, blockIdx.y * kThreads + threadIdx.x, gridDim.y * kThreads); }

__global__ void __launch_bounds__(kWide) fork_count_kernel(ForkArgs a, int32_t blocks)
{
    if ((int32_t)blockIdx.x < blocks) fork_count(a, blockIdx.x);
    else fork_need(a);
}

__global__ void __launch_bounds__(kWide) fork_take_kernel(ForkArgs a, int32_t blocks)
{
    int32_t before, free_all;
    sum_counts(a.free_before, blocks, blockIdx.x, before, free_all);
    if ((int32_t)blockIdx.x < blocks) fork_take(a, blockIdx.x, before, free_all);
    else fork_finish(a, (blockIdx.x - blocks) * kWide, free_all);
}

// All of it by one workgroup, tables of numbers of sequences and pages in LDS: few of the steps wait for memory.
constexpr int32_t kSmallEntries = 32768, kSmallPages = 8192;   // of sequences kWide at most

__global__ void __launch_bounds__(kWide) fork_kernel(ForkArgs a, int32_t blocks)
{
    __shared__ int32_t holders_s[kSmallPages], keeper_s[kSmallPages], length_s[kWide], parent_s[kWide], wanted_s[kWide], free_s[kSmallPages / kPagesPerBlock];
    __shared__ int64_t needed_s[kWide + 1];
    __shared__ uint64_t bits_s[kSmallPages / 64];
    int32_t *const holders_out = a.holders_out;
    const int32_t t = threadIdx.x;
    if (t < a.batch) length_s[t] = a.length[t];
    if (t < a.new_batch) parent_s[t] = a.parent[t];
    if (t < a.new_batch && a.wanted) wanted_s[t] = a.wanted[t];
    a.length = length_s;
    a.parent = parent_s;
    a.wanted = a.wanted ? wanted_s : nullptr;
    a.holders_out = holders_s;
    a.keeper = keeper_s;
    a.free_bits = bits_s;
    a.free_before = free_s;
    a.needed = needed_s;
#pragma unroll
    for (int32_t k = 0; k < kSmallPages; k += kWide)
        if (k + t < a.pages) fork_begin(a, k + t);
    __syncthreads();
    // a wavefront for each row
    for (int32_t row = t / 64; row < a.batch + a.new_batch; row += kWide / 64) fork_hold(a, row, t % 64, 64);
    __syncthreads();
    for (int32_t block = 0; block < blocks; ++block) fork_count(a, block);
    fork_need(a);
    __syncthreads();
    int32_t free_all = 0;
    for (int32_t block = 0; block < blocks; ++block) free_all += free_s[block];
    fork_finish(a, 0, free_all);
    __syncthreads();   // entries of pages that are copied were written in the second step, by others
    int32_t before = 0;
    for (int32_t block = 0; block < blocks; ++block) {
        fork_take(a, block, before, free_all);
        before += free_s[block];
    }
    __syncthreads();
    for (int32_t p = t; p < a.pages; p += kWide) holders_out[p] = holders_s[p];
}

// -- pages to the lowest numbers ---------------------------------------------------------------------------------------------------
__device__ __forceinline__ void compact_count(const CompactArgs &a, int32_t block)
{
    count_block(block, a.pages, a.used_bits, a.used_before, [&](int32_t p) { return a.holders[p] != 0; });
}

// Pages in use below number `count`, that of all of them.
__device__ __forceinline__ int32_t used_below(const CompactArgs &a, int32_t count)
{
    const int32_t edge = count / kPagesPerBlock, words = count / 64, rest = count % 64;
    int32_t n = 0, all;
    for (int32_t k = threadIdx.x; k < edge; k += kWide) n += a.used_before[k];
    for (int32_t w = edge * 64 + (int32_t)threadIdx.x; w <= words && w * 64 < count; w += kWide) {
        const uint64_t word = a.used_bits[w];
        n += __popcll(w < words ? word : word & (((uint64_t)1 << rest) - 1));
    }
    sum_before(n, all);
    return all;
}

// The k-th page in use from number `count` on goes to the k-th free one below it: sources and targets of the moves, each by its own thread.  holders_out may be holders.
__device__ __forceinline__ void compact_moves(const CompactArgs &a, int32_t block, int32_t before, int32_t count, int32_t below_count)
{
    const int32_t moved = count - below_count;   // as many are free below `count`
    each_page(block, a.pages, a.used_bits, before, [&](int32_t p, bool used, int32_t used_before) {
        if (used && p >= count) a.moves[3 * (int64_t)(used_before - below_count)] = p;
        if (!used && p < count) a.moves[3 * (int64_t)(p - used_before) + 1] = p;
        if (p < a.pages / 2) {
            const int64_t at = 3 * (int64_t)p;
            if (p >= moved) a.moves[at] = a.moves[at + 1] = -1;
            a.moves[at + 2] = p < moved ? 1 << a.page_shift : 0;
        }
        a.to[p] = p;
        a.holders_out[p] = a.holders[p];
    });
}

// Where page number k of the moves went, and its holders.
__device__ __forceinline__ void compact_to(const CompactArgs &a, int64_t k)
{
    const int32_t from = a.moves[3 * k], to = a.moves[3 * k + 1];
    if (from < 0) return;
    a.to[from] = to;
    a.holders_out[to] = a.holders_out[from];
    a.holders_out[from] = 0;
}

__device__ __forceinline__ void compact_table(const CompactArgs &a, int32_t b, int32_t c0, int32_t step)
{
    const int32_t n = a.length[b], used = n > (int64_t)a.columns << a.page_shift ? 0 : columns_of(n, a.page_shift);
    for (int32_t c = c0; c < a.columns; c += step) {
        const int32_t p = a.page[b * a.page_ld + c];
        a.page_out[b * a.page_out_ld + c] = c < used && (uint32_t)p < (uint32_t)a.pages ? a.to[p] : p;
    }
}

__global__ void __launch_bounds__(kWide) compact_count_kernel(CompactArgs a) { compact_count(a, blockIdx.x); }

__global__ void __launch_bounds__(kWide) compact_moves_kernel(CompactArgs a, int32_t blocks)
{
    int32_t before, count;
    sum_counts(a.used_before, blocks, blockIdx.x, before, count);
    compact_moves(a, blockIdx.x, before, count, used_below(a, count));
}

__global__ void __launch_bounds__(kThreads) compact_to_kernel(CompactArgs a)
{
    const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k < a.pages / 2) compact_to(a, k);
}

__global__ void __launch_bounds__(kThreads) compact_tables_kernel(CompactArgs a) { compact_table(a, blockIdx.x, blockIdx.y * kThreads + threadIdx.x, gridDim.y * kThreads); }

// All of it by one workgroup, pages and moves in LDS.
__global__ void __launch_bounds__(kWide) compact_kernel(CompactArgs a, int32_t blocks)
{
    __shared__ int32_t holders_s[kSmallPages], to_s[kSmallPages], moves_s[kSmallPages / 2 * 3], used_s[kSmallPages / kPagesPerBlock];
    __shared__ uint64_t bits_s[kSmallPages / 64];
    int32_t *const holders_out = a.holders_out, *const moves = a.moves;
    const int32_t t = threadIdx.x;
#pragma unroll
    for (int32_t k = 0; k < kSmallPages; k += kWide)
        if (k + t < a.pages) holders_s[k + t] = a.holders[k + t];
    a.holders = a.holders_out = holders_s;
    a.to = to_s;
    a.moves = moves_s;
    a.used_bits = bits_s;
    a.used_before = used_s;
    __syncthreads();
    for (int32_t block = 0; block < blocks; ++block) compact_count(a, block);
    __syncthreads();
    int32_t count = 0, before = 0;
    for (int32_t block = 0; block < blocks; ++block) count += used_s[block];
    const int32_t below_count = used_below(a, count);
    for (int32_t block = 0; block < blocks; ++block) {
        compact_moves(a, block, before, count, below_count);
        before += used_s[block];
    }
    __syncthreads();
    for (int32_t k = t; k < a.pages / 2; k += kWide) compact_to(a, k);
    __syncthreads();
    for (int32_t b = t / 64; b < a.batch; b += kWide / 64) compact_table(a, b, t % 64, 64);
    for (int32_t p = t; p < a.pages; p += kWide) holders_out[p] = holders_s[p];
    for (int32_t k = t; k < a.pages / 2 * 3; k += kWide) moves[k] = moves_s[k];
}

}  // namespace

hipError_t launch_accept(const AcceptArgs &a, sc_dtype dtype, hipStream_t stream)
{
    const int32_t bytes = dtype == SC_F32 ? 4 : 2;
    const int32_t pieces = 2 * a.kv_heads * (a.head_dim * bytes / 16);
    accept_kernel<<<dim3(a.s.batch, (pieces + kThreads - 1) / kThreads), kThreads, 0, stream>>>(a, bytes);
    return hipGetLastError();
}

namespace {

uint32_t column_blocks(int32_t columns) { return (uint32_t)((columns + kThreads - 1) / kThreads < 64 ? (columns + kThreads - 1) / kThreads : 64); }
uint32_t page_blocks(int32_t pages) { return (uint32_t)(((int64_t)pages + kThreads - 1) / kThreads); }

}  // namespace

hipError_t launch_fork(const ForkArgs &a, hipStream_t stream)
{
    const int32_t blocks = blocks_of_pages(a.pages), rows = a.batch + a.new_batch;
    if ((int64_t)rows * a.columns <= kSmallEntries && a.batch <= kWide && a.new_batch <= kWide && a.pages <= kSmallPages) {
        fork_kernel<<<1, kWide, 0, stream>>>(a, blocks);
        return hipGetLastError();
    }
    fork_begin_kernel<<<page_blocks(a.pages), kThreads, 0, stream>>>(a);
    if (a.columns > 0 && rows > 0) fork_hold_kernel<<<dim3(rows, column_blocks(a.columns)), kThreads, 0, stream>>>(a);
    fork_count_kernel<<<blocks + 1, kWide, 0, stream>>>(a, blocks);
    fork_take_kernel<<<blocks + (a.new_batch + kWide - 1) / kWide, kWide, 0, stream>>>(a, blocks);
    return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs &a, hipStream_t stream)
{
    const int32_t blocks = blocks_of_pages(a.pages);
    if ((int64_t)a.batch * a.columns <= kSmallEntries && a.batch <= kWide && a.pages <= kSmallPages) {
        compact_kernel<<<1, kWide, 0, stream>>>(a, blocks);
        return hipGetLastError();
    }
    compact_count_kernel<<<blocks, kWide, 0, stream>>>(a);
    compact_moves_kernel<<<blocks, kWide, 0, stream>>>(a, blocks);
    if (a.pages > 1) compact_to_kernel<<<page_blocks(a.pages / 2), kThreads, 0, stream>>>(a);
    if (a.batch > 0 && a.columns > 0) compact_tables_kernel<<<dim3(a.batch, column_blocks(a.columns)), kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

hipError_t launch_copy(const CopyArgs &a, sc_dtype dtype, hipStream_t stream)
{
    const int32_t bytes = dtype == SC_F32 ? 4 : 2;
    const int64_t page = 2 * (((int64_t)a.kv_heads * a.head_dim * bytes) << a.page_shift);
    const int64_t parts = (page / 16 + 4 * kThreads - 1) / (4 * kThreads);
    constexpr int64_t kEach = 1 << 23;   // a grid has fewer than 2^32 threads
    for (CopyArgs x = a; x.count > 0; x.count -= kEach, x.moves += 3 * kEach)
        copy_kernel<<<dim3((uint32_t)(x.count < kEach ? x.count : kEach), (uint32_t)(parts < 64 ? parts : 64)), kThreads, 0, stream>>>(x, bytes);
    return hipGetLastError();
}

}  // namespace sck
