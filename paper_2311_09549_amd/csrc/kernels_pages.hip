// Pages of a cache: the accepted rows of trees, the next batch of sequences from the present one, pages moved to the lowest numbers, and copies of pages.
//
// Tables are integers by the thousand and rows are moved as they are: bound by launches and chains of reads, and by memory where pages move.
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

// Whether it is left with that page: the first of those that keep it in part, if none holds it whole.  `holders`: of whole pages.
__device__ __forceinline__ bool keeps_part(const ForkArgs &a, int32_t i, int32_t page) { return a.keeper[page] == i && a.holders_out[page] == 0; }

__global__ void __launch_bounds__(kThreads) fork_begin_kernel(ForkArgs a)
{
    const int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (p >= a.pages) return;
    a.holders_out[p] = a.holders[p];
    a.keeper[p] = kNone;
}

// Entries of the present batch hold their pages no more, whole ones of the next do.  Sums of whole numbers: their order does not matter.
__global__ void __launch_bounds__(kThreads) fork_hold_kernel(ForkArgs a)
{
    const int32_t b = blockIdx.x, c0 = blockIdx.y * kThreads + threadIdx.x, step = gridDim.y * kThreads;
    if (b < a.batch) {
        const int32_t columns = columns_of(fork_length(a, b), a.page_shift);
        for (int32_t c = c0; c < columns; c += step) {
            const int32_t p = entry_of(a, b, c);
            if (p >= 0) atomicAdd(a.holders_out + p, -1);
        }
        return;
    }
    const int32_t i = b - a.batch;
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

// Sum over the threads of a workgroup, and of those before each.
template <typename T>
__device__ __forceinline__ T sum_before(T x, T &all)
{
    __shared__ T wave_s[kThreads / 64];
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
    for (int k = 0; k < kThreads / 64; ++k) {
        before += k < wave ? wave_s[k] : 0;
        all += wave_s[k];
    }
    return before + upto - x;
}

// Pages that a sequence of the next batch takes.
__device__ __forceinline__ int32_t pages_needed(const ForkArgs &a, int32_t i)
{
    const Branch r = branch_of(a, i);
    if (r.wanted < 0) return 0;
    const int32_t part = page_in_part(a, r);
    return (part >= 0 && !keeps_part(a, i, part) ? 1 : 0) + columns_of(r.wanted, a.page_shift) - columns_of(r.kept, a.page_shift);
}

// Free pages, a bit each and their number in each block of them, and, by the last workgroup, the pages that the sequences before each take.
__global__ void __launch_bounds__(kThreads) fork_count_kernel(ForkArgs a)
{
    if (blockIdx.x + 1 == gridDim.x) {
        int64_t before = 0, all;
        for (int32_t i0 = 0; i0 < a.new_batch; i0 += kThreads) {
            const int32_t i = i0 + threadIdx.x;
            const int64_t mine = sum_before<int64_t>(i < a.new_batch ? pages_needed(a, i) : 0, all);
            if (i < a.new_batch) a.needed[i] = before + mine;
            before += all;
        }
        if (threadIdx.x == 0) a.needed[a.new_batch] = before;
        return;
    }
    int32_t n = 0, all;
    for (int32_t k = threadIdx.x; k < kPagesPerBlock; k += kThreads) {
        const int64_t p = (int64_t)blockIdx.x * kPagesPerBlock + k;
        const bool is = p < a.pages && a.holders_out[p] == 0 && a.keeper[p] == kNone;
        const uint64_t bits = __ballot(is);
        if (k % 64 == 0) a.free_bits[p / 64] = bits;
        n += is;
    }
    sum_before(n, all);
    if (threadIdx.x == 0) a.free_before[blockIdx.x] = all;
}

// The n-th free page goes to the sequence that takes it; lengths, moves, and holders of pages that are taken or kept in part.
__global__ void __launch_bounds__(kThreads) fork_take_kernel(ForkArgs a, int32_t blocks)
{
    // free pages before this block of them, and of all
    int32_t before = 0, free_all = 0, all;
    for (int32_t k0 = 0; k0 < blocks; k0 += kThreads) {
        const int32_t k = k0 + threadIdx.x, n = k < blocks ? a.free_before[k] : 0;
        sum_before(k < (int32_t)blockIdx.x ? n : 0, all);
        before += all;
        sum_before(n, all);
        free_all += all;
    }
    const int64_t taken_all = a.needed[a.new_batch];
    const auto served = [&](int32_t i) { return a.needed[i + 1] == a.needed[i] || a.needed[i + 1] <= free_all; };
    if ((int32_t)blockIdx.x >= blocks) {
        // sequences, 256 a workgroup
        __shared__ int32_t dropped_s[kThreads];
        const int32_t i0 = (blockIdx.x - blocks) * kThreads, i = i0 + threadIdx.x;
        dropped_s[threadIdx.x] = 0;
        if (i < a.new_batch) {
            const Branch r = branch_of(a, i);
            const bool is = r.wanted >= 0 && served(i);
            const int32_t part = page_in_part(a, r);
            const bool copied = is && part >= 0 && a.needed[i + 1] - a.needed[i] > columns_of(r.wanted, a.page_shift) - columns_of(r.kept, a.page_shift);
            a.length_out[i] = is ? r.wanted : -1;
            a.moves[3 * i] = copied ? part : -1;
            if (!copied) a.moves[3 * i + 1] = -1;
            a.moves[3 * i + 2] = copied ? r.kept & ((1 << a.page_shift) - 1) : 0;
            if (is && part >= 0 && !copied) a.holders_out[part] = 1;
            dropped_s[threadIdx.x] = r.wanted >= 0 && !is;
        }
        __syncthreads();
        // those that found no room hold nothing
        for (int k = 0; k < kThreads; ++k) {
            if (!dropped_s[k]) continue;
            const int32_t part = branch_of(a, i0 + k).kept >> a.page_shift;   // of a page kept in part the holder was not counted
            for (int32_t c = threadIdx.x; c < a.columns; c += kThreads) {
                int32_t &entry = a.page_out[(i0 + k) * a.page_out_ld + c];
                if (entry >= 0 && c != part) atomicAdd(a.holders_out + entry, -1);
                entry = -1;
            }
        }
        return;
    }
    for (int32_t k0 = 0; k0 < kPagesPerBlock && before < taken_all; k0 += kThreads) {
        const int64_t p = (int64_t)blockIdx.x * kPagesPerBlock + k0 + threadIdx.x;
        const bool mine = a.free_bits[p / 64] >> (threadIdx.x % 64) & 1;
        const int32_t rank = before + sum_before<int32_t>(mine, all);
        before += all;
        if (!mine || rank >= taken_all) continue;
        // the sequence: the last one that begins at this page or before, which takes some
        int32_t lo = 0, hi = a.new_batch;
        while (hi - lo > 1) {
            const int32_t mid = (lo + hi) / 2;
            if (a.needed[mid] <= rank) lo = mid; else hi = mid;
        }
        if (!served(lo)) continue;
        const Branch r = branch_of(a, lo);
        const int32_t first = columns_of(r.kept, a.page_shift), grown = columns_of(r.wanted, a.page_shift) - first;
        const int32_t copied = (int32_t)(a.needed[lo + 1] - a.needed[lo]) - grown, n = (int32_t)(rank - a.needed[lo]);
        if (n < copied) a.moves[3 * lo + 1] = (int32_t)p;
        a.page_out[lo * a.page_out_ld + (n < copied ? r.kept >> a.page_shift : first + n - copied)] = (int32_t)p;
        a.holders_out[p] = 1;
    }
}

// -- pages to the lowest numbers ---------------------------------------------------------------------------------------------------
__global__ void __launch_bounds__(kThreads) compact_count_kernel(CompactArgs a)
{
    int32_t n = 0, all;
    for (int32_t k = threadIdx.x; k < kPagesPerBlock; k += kThreads) {
        const int32_t p = blockIdx.x * kPagesPerBlock + k;
        n += p < a.pages && a.holders[p] != 0;
    }
    sum_before(n, all);
    if (threadIdx.x == 0) a.used_before[blockIdx.x] = all;
}

// The k-th page in use from number `count` on goes to the k-th free one below it: sources and targets of the moves, each by its own thread.  holders_out may be holders.
__global__ void __launch_bounds__(kThreads) compact_moves_kernel(CompactArgs a, int32_t blocks)
{
    // pages in use before this block of them, in all, and below `count`: in the blocks before the one that has number `count`, and some of that one
    int32_t before = 0, count = 0, below_count = 0, n = 0, all;
    for (int32_t k0 = 0; k0 < blocks; k0 += kThreads) {
        const int32_t k = k0 + threadIdx.x, used = k < blocks ? a.used_before[k] : 0;
        sum_before(k < (int32_t)blockIdx.x ? used : 0, all);
        before += all;
        sum_before(used, all);
        count += all;
    }
    const int32_t edge = count / kPagesPerBlock;
    for (int32_t k = threadIdx.x; k < edge; k += kThreads) n += a.used_before[k];
    for (int32_t p = edge * kPagesPerBlock + threadIdx.x; p < count; p += kThreads) n += a.holders[p] != 0;
    sum_before(n, below_count);
    const int32_t moved = count - below_count;   // as many are free below `count`
    for (int32_t k0 = 0; k0 < kPagesPerBlock; k0 += kThreads) {
        const int64_t at = (int64_t)blockIdx.x * kPagesPerBlock + k0 + threadIdx.x;
        const int32_t p = (int32_t)at;
        const bool used = at < a.pages && a.holders[p] != 0;
        const int32_t used_before = before + sum_before<int32_t>(used, all);
        before += all;
        if (at >= a.pages) continue;
        if (used && p >= count) a.moves[3 * (int64_t)(used_before - below_count)] = p;
        if (!used && p < count) a.moves[3 * (int64_t)(p - used_before) + 1] = p;
        if (p < a.pages / 2) {
            if (p >= moved) a.moves[3 * at] = a.moves[3 * at + 1] = -1;
            a.moves[3 * at + 2] = p < moved ? 1 << a.page_shift : 0;
        }
        a.to[p] = p;
        a.holders_out[p] = a.holders[p];
    }
}

// Where pages went, and their holders.
__global__ void __launch_bounds__(kThreads) compact_to_kernel(CompactArgs a)
{
    const int64_t k = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    if (k >= a.pages / 2 || a.moves[3 * k] < 0) return;
    const int32_t from = a.moves[3 * k], to = a.moves[3 * k + 1];
    a.to[from] = to;
    a.holders_out[to] = a.holders_out[from];
    a.holders_out[from] = 0;
}

__global__ void __launch_bounds__(kThreads) compact_tables_kernel(CompactArgs a)
{
    const int32_t b = blockIdx.x, n = a.length[b], used = n > (int64_t)a.columns << a.page_shift ? 0 : columns_of(n, a.page_shift);
    for (int32_t c = blockIdx.y * kThreads + threadIdx.x; c < a.columns; c += gridDim.y * kThreads) {
        const int32_t p = a.page[b * a.page_ld + c];
        a.page_out[b * a.page_out_ld + c] = c < used && (uint32_t)p < (uint32_t)a.pages ? a.to[p] : p;
    }
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
    const int32_t blocks = blocks_of_pages(a.pages);
    fork_begin_kernel<<<page_blocks(a.pages), kThreads, 0, stream>>>(a);
    if (a.columns > 0 && a.batch + a.new_batch > 0) fork_hold_kernel<<<dim3(a.batch + a.new_batch, column_blocks(a.columns)), kThreads, 0, stream>>>(a);
    fork_count_kernel<<<blocks + 1, kThreads, 0, stream>>>(a);
    fork_take_kernel<<<blocks + (a.new_batch + kThreads - 1) / kThreads, kThreads, 0, stream>>>(a, blocks);
    return hipGetLastError();
}

hipError_t launch_compact(const CompactArgs &a, hipStream_t stream)
{
    const int32_t blocks = blocks_of_pages(a.pages);
    compact_count_kernel<<<blocks, kThreads, 0, stream>>>(a);
    compact_moves_kernel<<<blocks, kThreads, 0, stream>>>(a, blocks);
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
