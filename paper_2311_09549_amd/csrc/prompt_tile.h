// Prompt attention of 16-bit types: tiles of keys and values in LDS, shared by the wavefronts of a workgroup.
//
// A wavefront has 32 query rows of one head; a workgroup NW of them, which share the keys of one key head: as many of the
// heads of that key head as there are (1, 2, 4 or 8), and rows of them one behind the other.  Both products are transposed as in
// attention_device.h, on v_mfma 32x32x16: S^T = K Q^T, O^T = V^T P^T.  A lane (q = lane % 32, half = lane / 32) holds of query q the scores
// with keys 8 (r / 4) + 4 half + r % 4 of each 32, r = 0..15, and eight of them in a row, as they are, are its operand of a step of the
// second product, whose 16 keys are then taken in the order 4 half + 0..3, 8 + 4 half + 0..3.  Values are read from LDS in that order by
// transposing reads (ds_read_b64_tr_b16: 16 lanes read 4 rows of 16 elements and get 4 rows of one element each).
//
// Rows of a tile are whole rows of the head; their 16-byte pieces are exchanged within a row (exclusive or with bits of the
// row number), so that the 32 rows that a read of keys touches, and the 4 of a transposing read, lie in different banks.
//
// The maximum that weights are taken against is raised only where a score passes it by more than 2^8: sums are rescaled a few times a row instead of at
// every new maximum, and weights lose nothing: they are lowered by as much in bf16, which has the exponents of fp32.
//
// Eight wavefronts of 256 registers fill a compute unit; tiles of 128 keys halve the barriers of tiles of 64 (1,095 -> 1,045 us in the first case below).  bf16, heads of
// 128: 16,384 rows, 16 heads on 4 key heads in 1,070 us, 1.03 PFLOP/s, where a large product of the library reaches 1.36: matrix pipes busy 0.50 of the time,
// vector ALUs 0.49 (a maximum, a power of two, a sum and a conversion per score), and LDS reads, 256 rows' worth for every 32 that use them,
// about as long again.  Twelve packed prompts up to 2,048 rows, 32 heads on 8: 146 us, 0.59 PFLOP/s, matrix pipes 0.34: the start and end
// of blocks, with nothing beside them on the compute unit.
//
// Windows and trees: tiles of 32 KB for keys and values go straight to LDS (global_load_lds), in the order of the exchange, three ahead of the one that is worked on, and page
// numbers come a tile ahead of those; the registers that this frees keep queries from being spilled.  The waits are by counts of loads, so nothing else of a
// wavefront may load in the main loop.  bf16, heads of 128: 16,384 rows through a window of 4,096 and four first keys, 16 heads on 4, in 590 us (0.81 PFLOP/s; its 66 tiles of 64 keys a block take 2.2 us each,
// products, powers and LDS reads as above); chunks of four sequences up to 509 rows through a window of 1,000 in 53 us, 16 of them before the first and behind the last of 18 tiles; 24 trees of up to 63 rows behind 8,191 keys in 112 us and
// 18 for the join, 170 with tiles through registers.
#pragma once

#include "attention_device.h"

namespace sck {

template <typename TR, int DP, int NW, int KT>
struct PromptTile {
    static constexpr int THREADS = 64 * NW, CHUNKS = DP / 8, DT = DP / 32, NT = KT / 32;   // pieces of a row, tiles of the head, tiles of keys
    static constexpr int LOADS = KT * CHUNKS / THREADS, ROWS_PER_LOAD = THREADS / CHUNKS;
    static constexpr int ROW_BYTES = DP * 2, TILE_BYTES = KT * ROW_BYTES;
    static constexpr float kRaise = 8.0f;
    // A weight's exponent is s scale_log2 - m scale_log2 in one operation, off by roundings of the second product: less than 2^-14 of the weight where that
    // is at most 2^8.  Beyond it, up to products that pass fp32, the difference of the scores is taken first, which is exact where it matters.
    static constexpr float kFar = 256.0f;
    // Weights up to 2^15 in fp16; up to 1 in bf16, as without the lag, so that sums of values near the largest stay in fp32.
    static constexpr float kLift = TR::kLift > 0.0f ? TR::kLift - kRaise + 1.0f : -kRaise;
    static_assert(KT * CHUNKS % THREADS == 0 && ROWS_PER_LOAD * CHUNKS == THREADS, "whole rows per load");

    // Place of piece c of row r.
    static __device__ __forceinline__ int key_piece(int r, int c)
    {
        if constexpr (CHUNKS >= 16) return c ^ (r & 15);
        else return c ^ ((r & 7) ^ (r >> 3 & 1));
    }
    static __device__ __forceinline__ int value_piece(int r, int c)
    {
        if constexpr (CHUNKS >= 16) return c ^ ((r & 1) << 1 | (r & 2) << 1 | (r & 1) << 3);
        else return c ^ ((r & 2) << 1 | (r & 1) << 1);
    }
};

// What a piece of a wavefront's 32 rows takes in the workspace: per lane its sums, its maximum and its sum of weights.
template <int DP>
constexpr int kPromptPiece = 64 * (DP / 2 + 2);   // floats

template <int R>
__device__ __forceinline__ RowBlock row_block_of(const Sequences &s, int32_t number, int heads_log2)
{
    return heads_log2 == 0 ? row_block<R>(s, number) : heads_log2 == 1 ? row_block<R / 2>(s, number) : heads_log2 == 2 ? row_block<R / 4>(s, number) : row_block<R / 8>(s, number);
}

// Block number k of those that have rows, of `rows` (a power of two) each: 64 sequences at a time, a lane each.  Numbers without rows in between would leave compute units idle:
// workgroups go to the shader engines in turn, and of 24 sequences of 63 rows every other number has rows, on every other engine (530 us instead of 290 behind 8,192 keys).
constexpr int32_t kCountedBatch = 1024;   // more sequences take as many reads one after the other as that is 64s

__device__ __forceinline__ RowBlock row_block_at(const Sequences &s, int32_t k, int32_t rows_log2)
{
    for (int32_t c = 0; 64 * c < s.batch; ++c) {
        const int32_t b = 64 * c + (int32_t)(threadIdx.x % 64);
        const int32_t begin = b < s.batch ? row_begin(s, b) : 0, end = b < s.batch ? row_begin(s, b + 1) : 0;
        const int32_t n = end > begin ? ((end - begin - 1) >> rows_log2) + 1 : 0;
        int32_t upto = n;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t y = __shfl_up(upto, d);
            upto += (int32_t)(threadIdx.x % 64) >= d ? y : 0;
        }
        const int32_t all = __builtin_amdgcn_readlane(upto, 63);
        if (k < all) {
            const int at = __ffsll((unsigned long long)__ballot(upto > k)) - 1;
            RowBlock r;
            r.sequence = 64 * c + at;
            r.begin = __builtin_amdgcn_readlane(begin, at);
            const int32_t last = __builtin_amdgcn_readlane(end, at);
            r.count = last - r.begin;
            r.first = r.begin + ((k - __builtin_amdgcn_readlane(upto, at) + __builtin_amdgcn_readlane(n, at)) << rows_log2);
            r.end = r.first + (1 << rows_log2) < last ? r.first + (1 << rows_log2) : last;
            return r;
        }
        k -= all;
    }
    return {-1, 0, 0, 0, 0};
}

// Keys that row r of a block sees: none but those up to its own position.
__device__ __forceinline__ int32_t keys_seen(const AttendArgs &a, const RowBlock &blk, int32_t length, int32_t r)
{
    const int32_t n = a.causal ? length - blk.count - blk.begin + 1 + r : length;
    return n < 0 ? 0 : n;
}

// The tiles of keys that a block of rows sees, as one line: those of the first keys, up to key `first`, then those from first + skip on (whole tiles both).  `length`: keys that
// its last row sees, without the skipped ones.  `low` and `last_low`: the first key that its first and its last row see through the window.
struct BlockKeys {
    int32_t first, skip, length, low, last_low;
};

// What rows see: every key before them; of those the ones in a window, and the first ones; what is before their tree, their ancestors and themselves (attention.h).
enum Sees { kEverything, kWindow, kTree };

template <Sees SEES>
__device__ __forceinline__ BlockKeys block_keys(const AttendArgs &a, const RowBlock &blk, int32_t length, int32_t tile)
{
    const int32_t n = keys_seen(a, blk, length, blk.end - 1);
    BlockKeys k = {0, 0, n, 0, 0};
    if (SEES != kWindow) return k;
    k.low = window_low(a.window, keys_seen(a, blk, length, blk.first) - 1);
    k.last_low = window_low(a.window, n - 1);
    const int32_t from = k.low / tile * tile, first = a.sinks < from ? (a.sinks + tile - 1) / tile * tile : from;
    if (first < from) k = {first, from - first, n - (from - first), k.low, k.last_low};
    return k;
}

// Length of a sequence whose rows are trees, -1 for a wrong one.
__device__ __forceinline__ int32_t tree_length(const AttendArgs &a, int32_t b, int32_t count)
{
    const int32_t n = paged_length(a.s, b);
    return n < count || (a.parent && count > kMaxNodes) ? -1 : n;
}

// kTree: a lane finds the ancestors of its row among the keys of a tile by going up from it, parents in LDS; all lanes of a wavefront go as long as one has any.
// SPLIT: as in decode, the tiles of keys of all blocks are put in one line, block after block, one group of heads after the other, and every workgroup takes an
// equal share of it; blocks that shares cut leave pieces, which prompt_join_kernel joins.  Without it a workgroup has one block, and a call takes as long as
// the longest of them, or as the compute unit that was given most.  Chunks of four prompts behind up to 8,191 keys, 32 heads of 128: 262 to 274 us with, 320
// without; L2 misses are six times as many, since workgroups begin at different keys, and the join is 18 us.
template <typename TR, int DP, bool PAGED, bool SPLIT, Sees SEES, int NW, int KT>
__global__ void __launch_bounds__(64 * NW, NW / 4) prompt_tile_kernel(AttendArgs a, int heads_log2)
{
    using P = PromptTile<TR, DP, NW, KT>;
    constexpr int CHUNKS = P::CHUNKS, DT = P::DT, NT = P::NT, LOADS = P::LOADS, R = 32 * NW;
    constexpr bool WINDOW = SEES == kWindow, TREE = SEES == kTree;
    // Windows and trees: keys and values go straight to LDS, three tiles ahead, in four buffers.
    constexpr bool DIRECT = SEES != kEverything;
    constexpr int BUFFERS = DIRECT ? 4 : 2;
    __shared__ __attribute__((aligned(16))) char tile_s[BUFFERS * 2 * P::TILE_BYTES];   // [buffer][keys, values]
    __shared__ int32_t parent_s[TREE ? kMaxNodes : 1];
    const int32_t head_groups = a.heads >> heads_log2;
    const auto length_of = [&](const RowBlock &blk) { return TREE ? tree_length(a, blk.sequence, blk.count) : PAGED ? paged_length(a.s, blk.sequence) : blk.count; };

    // Keys of tiles first_tile .. last_tile - 1 for a block of rows and a group of heads; sums: where the sums go if those are not all tiles that it sees.
    const auto work = [&](const RowBlock &blk, int32_t head_group, int32_t first_tile, int32_t last_tile, float *sums) __attribute__((always_inline)) {
        uint32_t thread = threadIdx.x;
        asm volatile("" : "+v"(thread));   // what follows from it is made again for each block, instead of taking the registers of the main loop
        const int lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64), q = lane % 32, half = lane / 32;
        const int32_t head0 = head_group << heads_log2, kv = head0 / a.group;
        const int32_t length = length_of(blk);
        const int32_t head = head0 + (wave & ((1 << heads_log2) - 1)), first = blk.first + 32 * (wave >> heads_log2), row = first + q;
        const bool mine = row < blk.end;
        char *out = static_cast<char *>(a.out.data) + (row * a.out.row + head * a.out.head) * 2;
        if (length < 0) {
            if (mine)
                for (int d = 8 * half; d < a.head_dim; d += 16) *reinterpret_cast<u32x4 *>(out + 2 * d) = u32x4{0, 0, 0, 0} + TR::kExponent * 0x10001u + 0x00010001u;
            return;
        }

        const auto sees = [&](int32_t r) { return keys_seen(a, blk, length, r); };
        const BlockKeys line = block_keys<SEES>(a, blk, length, KT);
        int32_t block_most = line.length;
        if (SPLIT && last_tile < (block_most + KT - 1) / KT) block_most = last_tile * KT;
        const auto key_of = [&](int32_t place) { return WINDOW && place >= line.first ? place + line.skip : place; };
        const int32_t visible = mine && !TREE ? sees(row) : 0;
        const int32_t most = first < blk.end ? sees((first + 32 < blk.end ? first + 32 : blk.end) - 1) : 0;
        // the first key that the lane's row, and any row of the wavefront, sees through the window
        const int32_t low = WINDOW ? window_low(a.window, visible - 1) : 0, least = WINDOW && first < blk.end ? window_low(a.window, sees(first) - 1) : 0;

        // keys before the tree; the lane's node; whether its chain has a wrong number.  Chains are needed where the tiles have nodes.
        const int32_t before = length - blk.count;
        const bool chains = TREE && a.parent && block_most > before;
        constexpr int32_t kWrong = -2;
        int32_t node = mine ? row - blk.begin : -1;
        if (chains) {
            for (int32_t i = thread; i < blk.count; i += P::THREADS) parent_s[i] = a.parent[blk.begin + i];
            __syncthreads();
            for (int32_t i = node; __any(i >= 0);) {
                const int32_t p = parent_s[i < 0 ? 0 : i];
                const bool ok = i < 0 || parent_ok(i, p);
                node = ok ? node : kWrong;
                i = i < 0 || !ok ? -1 : p;
            }
        }

        u32x4 qf[DP / 16];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) {
            qf[c] = u32x4{0, 0, 0, 0};
            const int e = (2 * c + half) * 8;
            if (mine && e < a.head_dim) qf[c] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(a.q.data) + (row * a.q.row + head * a.q.head + e) * 2);
        }
        f32x16 o[DT];
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
            for (int r = 0; r < 16; ++r) o[d][r] = 0.0f;
        float m = kMinusInf, l = 0.0f;
        bool far = false;   // of any query of the wavefront

        // this thread's pieces of a tile
        const int piece = thread % CHUNKS, row0 = thread / CHUNKS;
        const bool held = piece * 8 < a.head_dim;
        const int64_t k_row = (PAGED ? a.cache.row : a.k.row) * 2, v_row = (PAGED ? a.cache.row : a.v.row) * 2;
        const char *k0 = PAGED ? static_cast<const char *>(a.cache.keys) + (kv * a.cache.head + piece * 8) * 2
                               : static_cast<const char *>(a.k.data) + (blk.begin * a.k.row + kv * a.k.head + piece * 8) * 2;
        const char *v0 = PAGED ? static_cast<const char *>(a.cache.values) + (kv * a.cache.head + piece * 8) * 2
                               : static_cast<const char *>(a.v.data) + (blk.begin * a.v.row + kv * a.v.head + piece * 8) * 2;
        bool bad = false;
        u32x4 ks[LOADS], vs[LOADS];
        // In pages a row's keys and values wait for its page number, within every tile: chunks of four prompts behind up to 8,191 keys take 5.0 us a tile
        // without a split, packed keys 4.1.
        const auto fetch = [&](int32_t base) {
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                int32_t key = base + row0 + n * P::ROWS_PER_LOAD;
                key = key < length ? key : length - 1;   // rows behind the last key are seen by none: any that are there
                int64_t k_at = key * k_row, v_at = key * v_row;
                if (PAGED) {
                    int32_t page = page_of(a.s, blk.sequence, key);
                    bad |= page < 0;
                    if (page < 0) page = 0;
                    k_at = v_at = (page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row) * 2;
                }
                ks[n] = vs[n] = u32x4{0, 0, 0, 0};
                if (held) {
                    ks[n] = *reinterpret_cast<const u32x4 *>(k0 + k_at);
                    vs[n] = *reinterpret_cast<const u32x4 *>(v0 + v_at);
                }
            }
        };
        // Tiles that some rows see in part are stored without infinities and NaN among the values, which the product would spread to rows that do not see them
        // (0 times infinity); the answer is whether there were any.
        const auto put = [&](char *buffer, bool part) {
            uint32_t any = 0;
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                const int r = row0 + n * P::ROWS_PER_LOAD;
                if (part) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        any |= Special<TR>::infinite_or_nan(vs[n][i]);
                        vs[n][i] = Special<TR>::without(vs[n][i]);
                    }
                }
                *reinterpret_cast<u32x4 *>(buffer + r * P::ROW_BYTES + 16 * P::key_piece(r, piece)) = ks[n];
                *reinterpret_cast<u32x4 *>(buffer + P::TILE_BYTES + r * P::ROW_BYTES + 16 * P::value_piece(r, piece)) = vs[n];
            }
            return any != 0;
        };
        // Straight to LDS: a load of a wavefront fills 64 pieces in a row, whole rows, and its lanes ask for the pieces that belong there.  The rows of a load are in one page, whose
        // number is read by the scalar unit a tile ahead.  Pieces behind the head are 0 from the start and stay so.
        constexpr int LOAD_ROWS = 64 / CHUNKS;
        static_assert(LOAD_ROWS <= 16, "in one page");
        const uint32_t tile_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)tile_s;
        int32_t page_next[LOADS];
        const auto find_pages = [&](int32_t base) {
            if constexpr (PAGED && DIRECT) {
#pragma unroll
                for (int n = 0; n < LOADS; ++n) {
                    const int32_t key = base + wave * LOAD_ROWS + n * P::ROWS_PER_LOAD;
                    page_next[n] = page_of_all(a.s, blk.sequence, key < length ? key : length - 1);
                }
            }
        };
        const auto to_lds = [](uint32_t at, const char *p) {
            // m0 is no register that the compiler gives away, which it warns of; it writes it itself before each instruction of its own that reads it
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
            asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(at), "v"(p) : "memory", "m0");
#pragma clang diagnostic pop
        };
        const auto load_tile = [&](int32_t base, int buffer) {
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                const int r = wave * LOAD_ROWS + n * P::ROWS_PER_LOAD + lane / CHUNKS;
                const int32_t key = base + r < length ? base + r : length - 1;   // rows behind the last key are seen by none: any that are there
                const char *k, *v;
                if constexpr (PAGED) {
                    const int32_t page = page_next[n] < 0 ? 0 : page_next[n];
                    bad |= page_next[n] < 0 && (!WINDOW || key >= line.low || key < a.sinks);   // pages behind every row's window may be gone
                    const int64_t at = (page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row + kv * a.cache.head) * 2;
                    k = static_cast<const char *>(a.cache.keys) + at;
                    v = static_cast<const char *>(a.cache.values) + at;
                } else {
                    k = static_cast<const char *>(a.k.data) + ((blk.begin + key) * a.k.row + kv * a.k.head) * 2;
                    v = static_cast<const char *>(a.v.data) + ((blk.begin + key) * a.v.row + kv * a.v.head) * 2;
                }
                const uint32_t at = tile_at + buffer * 2 * P::TILE_BYTES + (wave * LOAD_ROWS + n * P::ROWS_PER_LOAD) * P::ROW_BYTES;
                const int kc = P::key_piece(r, lane % CHUNKS), vc = P::value_piece(r, lane % CHUNKS);   // exchanges are their own inverse
                if (kc * 8 < a.head_dim) to_lds(at, k + 16 * kc);
                if (vc * 8 < a.head_dim) to_lds(at + P::TILE_BYTES, v + 16 * vc);
            }
        };
        // Of a tile that some rows see in part: infinities and NaN among the values that this lane has loaded become 0; whether there were any.
        const auto clean = [&](int buffer) {
            uint32_t any = 0;
#pragma unroll
            for (int n = 0; n < LOADS; ++n) {
                u32x4 *p = reinterpret_cast<u32x4 *>(tile_s + (2 * buffer + 1) * P::TILE_BYTES + (wave * LOAD_ROWS + n * P::ROWS_PER_LOAD) * P::ROW_BYTES + 16 * lane);
                u32x4 x = *p;
                uint32_t here = 0;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    here |= Special<TR>::infinite_or_nan(x[i]);
                    x[i] = Special<TR>::without(x[i]);
                }
                if (here) *p = x;
                any |= here;
            }
            return any != 0;
        };
        // They are added to the rows that see them, from memory.
        const auto add_special = [&](int32_t base, const uint32_t (&seen)[NT]) {
#pragma unroll 1
            for (int32_t key = base; key < base + KT && key < most; ++key) {
                const char *p = static_cast<const char *>(PAGED ? a.cache.values : a.v.data);
                if (PAGED) {
                    const int32_t page = page_of(a.s, blk.sequence, key);
                    p += ((page < 0 ? 0 : page) * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row + kv * a.cache.head) * 2;
                } else {
                    p += ((blk.begin + key) * a.v.row + kv * a.v.head) * 2;
                }
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) {
                        const int e = 32 * d + 8 * (r / 4) + 4 * half + r % 4;
                        if ((!TREE && key >= visible) || e >= a.head_dim || (WINDOW && key < low && key >= a.sinks)) continue;
                        if (TREE) {
                            uint32_t word = seen[0];
#pragma unroll
                            for (int t = 1; t < NT; ++t) word = (key - base) / 32 == t ? seen[t] : word;
                            if (!(word >> (key - base) % 32 & 1)) continue;
                        }
                        const typename TR::elem x = reinterpret_cast<const typename TR::elem *>(p)[e];
                        if ((__builtin_bit_cast(uint16_t, x) & TR::kExponent) == TR::kExponent) o[d][r] += (float)x;
                    }
            }
        };

        // Where the lane reads, of the first buffer: pieces of the keys of its query's number, and its part of a transposing read.  The other rows of a tile are
        // at constant distances, which are multiples of what the exchange of pieces goes by.
        int k_at[DP / 16], v_at[DT];
#pragma unroll
        for (int c = 0; c < DP / 16; ++c) k_at[c] = q * P::ROW_BYTES + 16 * P::key_piece(q, 2 * c + half);
#pragma unroll
        for (int d = 0; d < DT; ++d) {
            const int r = 4 * half + lane % 16 / 4, c = 4 * d + 2 * (lane / 16 % 2) + lane % 4 / 2;
            v_at[d] = P::TILE_BYTES + r * P::ROW_BYTES + 16 * P::value_piece(r, c) + lane % 2 * 8;
        }
        typedef __attribute__((address_space(3))) char *Lds;
        const auto tile = [&](Lds buffer, int32_t base, auto masked, const uint32_t (&seen)[NT]) {
            constexpr bool MASK = decltype(masked)::value;
            f32x16 s[NT];
#pragma unroll
            for (int t = 0; t < NT; ++t) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[t][r] = 0.0f;
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) {
                    s[t] = TR::mfma32(*(__attribute__((address_space(3))) u32x4 *)(buffer + k_at[c] + 32 * t * P::ROW_BYTES), qf[c], s[t]);
                }
            }
            float top = kMinusInf;
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const int n = 32 * t + 8 * (r / 4) + 4 * half + r % 4;   // number of the key in the tile
                    if (MASK && TREE) s[t][r] = seen[t] >> (8 * (r / 4) + r % 4) & 1 ? s[t][r] : kMinusInf;   // (shifted by the lane's 4 half)
                    if (MASK && SEES == kEverything) s[t][r] = n < visible - base ? s[t][r] : kMinusInf;
                    if (MASK && WINDOW) s[t][r] = n < visible - base && (n >= low - base || n < a.sinks - base) ? s[t][r] : kMinusInf;
                    top = fmaxf(top, s[t][r]);
                }
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any((top - m) * a.scale_log2 > P::kRaise)) {
                const float next = fmaxf(m, top), base_next = finite_max(next);
                const float shrink = __builtin_amdgcn_exp2f((m - base_next) * a.scale_log2);
                m = next;
                far = __any(fabsf(base_next * a.scale_log2) > P::kFar);
                l *= shrink;
#pragma unroll
                for (int d = 0; d < DT; ++d)
#pragma unroll
                    for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
            }
            const float from = finite_max(m), minus = far ? P::kLift : P::kLift - from * a.scale_log2;
            if (far) {
#pragma unroll
                for (int t = 0; t < NT; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[t][r] -= from;
            }
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    s[t][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[t][r], a.scale_log2, minus));
            u32x4 w[NT][2];
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    l += s[t][r] + s[t][r + 1];   // in fp32; weights are rounded once, to the type of the values, for the product that takes both in it
                    w[t][r / 8][r / 2 % 4] = TR::pack(s[t][r], s[t][r + 1]);
                }

            // operand of tile d of the head and keys 32 t + 16 n + ..
            const auto values = [&](int d, int t, int n) {
                u32x4 y;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const Lds p = buffer + v_at[d] + (32 * t + 16 * n + 8 * h) * P::ROW_BYTES;
                    const u32x2 z = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)p));
                    y[2 * h] = z.x;
                    y[2 * h + 1] = z.y;
                }
                return y;
            };
#pragma unroll
            for (int t = 0; t < NT; ++t)
#pragma unroll
                for (int n = 0; n < 2; ++n)
#pragma unroll
                    for (int d = 0; d < DT; ++d) o[d] = TR::mfma32(values(d, t, n), w[t][n], o[d]);
        };

        if (block_most > 0) {
            const int32_t block_all = TREE && a.parent ? before : sees(blk.first);   // keys that every row of the block sees
            // whether every row of the block sees the whole tile of keys from `key` on
            const auto whole = [&](int32_t key) { return key + KT <= block_all && (!WINDOW || key >= line.last_low || key + KT <= a.sinks); };
            int32_t place = SPLIT ? first_tile * KT : 0;
            // Keys of the row's chain among those of a tile: bits of the keys before the tree (or, of rows in order, up to the row), then of nodes.
            const auto chain = [&](int32_t base, uint32_t (&seen)[NT]) {
                const int32_t n = (a.parent ? before : before + node + 1) - base;
#pragma unroll
                for (int t = 0; t < NT; ++t) seen[t] = node < 0 || n <= 32 * t ? 0u : n >= 32 * t + 32 ? ~0u : (1u << (n - 32 * t)) - 1;
                const int32_t first_node = base - before;
                for (int32_t i = chains ? node : -1; __any(i >= 0 && i >= first_node);) {
                    const int32_t bit = i - first_node, p = parent_s[i < 0 ? 0 : i];
                    const uint32_t one = i >= 0 && bit >= 0 && bit < KT ? 1u << (bit & 31) : 0u;
#pragma unroll
                    for (int t = 0; t < NT; ++t) seen[t] |= bit >> 5 == t ? one : 0u;
                    i = i < 0 ? -1 : p;
                }
            };
            if constexpr (DIRECT) {
                constexpr int PER = 2 * LOADS;   // loads of a wavefront for a tile
                int32_t ahead = place;           // what has been asked for
                int buffer = 0;
                // queries have arrived: a wait for them within the loop would be one for the loads on their way
#pragma unroll
                for (int c = 0; c < DP / 16; ++c) asm volatile("" : "+v"(qf[c]));
                __syncthreads();   // the buffers are done with
                find_pages(key_of(ahead));
                const auto more = [&](int to) {
                    if (ahead >= block_most) return;
                    load_tile(key_of(ahead), to);
                    ahead += KT;
                    find_pages(key_of(ahead));
                };
#pragma unroll
                for (int n = 0; n < BUFFERS - 1; ++n) more(n);
                const auto pass = [&](auto masked) {
                    constexpr bool MASK = decltype(masked)::value;
                    const int32_t base = key_of(place);
                    // this tile has arrived, the two behind it may be on their way
                    if (ahead - place > 2 * KT) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(2 * PER) : "memory");
                    else if (ahead - place > KT) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(PER) : "memory");
                    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
                    bool special = false;
                    if (MASK) special = __syncthreads_or(clean(buffer));
                    else __syncthreads();
                    more((buffer + BUFFERS - 1) % BUFFERS);   // every wavefront is done with the tile before this one
                    if ((!MASK && (!TREE || first < blk.end)) || (MASK && base < most && (!WINDOW || base + KT > least || base < a.sinks))) {
                        uint32_t seen[NT] = {}, mine_of[NT];
                        if constexpr (MASK && TREE) {
                            chain(base, seen);
#pragma unroll
                            for (int t = 0; t < NT; ++t) mine_of[t] = seen[t] >> 4 * half;
                        }
                        tile((Lds)tile_s + buffer * 2 * P::TILE_BYTES, base, masked, mine_of);
                        if (MASK && special) add_special(base, seen);
                    }
                    buffer = (buffer + 1) % BUFFERS;
                    place += KT;
                };
                // edges of windows and first keys, and what every row of the block sees whole, in turn; of trees first what is before them
                if constexpr (WINDOW) {
                    while (place < block_most) {
                        while (place < block_most && !whole(key_of(place))) pass(std::true_type());
                        while (place < block_most && whole(key_of(place))) pass(std::false_type());
                    }
                } else {
                    while (place < block_most && whole(place)) pass(std::false_type());
                    while (place < block_most) pass(std::true_type());
                }
            } else {
                fetch(place);
                bool special = __syncthreads_or(put(tile_s, place + KT > block_all));
                int buffer = 0;
                const auto pass = [&](auto masked) {
                    constexpr bool MASK = decltype(masked)::value;
                    const bool more = place + KT < block_most, part = MASK || place + 2 * KT > block_all;
                    if (more) fetch(place + KT);
                    if (!MASK || place < most) {
                        const uint32_t seen[NT] = {};
                        tile((Lds)tile_s + buffer * 2 * P::TILE_BYTES, place, masked, seen);
                        if (MASK && special) add_special(place, seen);
                    }
                    buffer ^= 1;
                    bool any = false;
                    if (more) any = put(tile_s + buffer * 2 * P::TILE_BYTES, part);
                    if (part) special = __syncthreads_or(any);
                    else __syncthreads();
                    place += KT;
                };
                // tiles that every row of the block sees whole, then the others
                while (place + KT <= block_all && (!SPLIT || place < block_most)) pass(std::false_type());
                while (place < block_most) pass(std::true_type());
            }
        }
        if (PAGED) bad = __syncthreads_or(bad);
        l += __shfl_xor(l, 32);
        if (TREE && node == kWrong) l = __builtin_nanf("");
        if (SPLIT && sums) {
            if (first >= blk.end) return;   // nobody joins it
            float *p = sums + wave * kPromptPiece<DP>;
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 4; ++r) reinterpret_cast<f32x4 *>(p)[(4 * d + r) * 64 + lane] = f32x4{o[d][4 * r], o[d][4 * r + 1], o[d][4 * r + 2], o[d][4 * r + 3]};
            p[32 * DP + lane] = m;
            p[32 * DP + 64 + lane] = PAGED && bad ? __builtin_nanf("") : l;
            return;
        }
        const float factor = PAGED && bad ? __builtin_nanf("") : l == 0.0f ? 0.0f : 1.0f / l;
        if (mine) {
#pragma unroll
            for (int d = 0; d < DT; ++d)
#pragma unroll
                for (int r = 0; r < 16; r += 4) {
                    const int e = 32 * d + 2 * r + 4 * half;
                    if (e < a.head_dim)
                        *reinterpret_cast<u32x2 *>(out + 2 * e) = u32x2{TR::pack(o[d][r] * factor, o[d][r + 1] * factor), TR::pack(o[d][r + 2] * factor, o[d][r + 3] * factor)};
                }
        }
    };

    if (DIRECT && a.head_dim < DP)
        for (int x = threadIdx.x; x < (int)sizeof(tile_s) / 16; x += P::THREADS) reinterpret_cast<u32x4 *>(tile_s)[x] = u32x4{0, 0, 0, 0};

    if constexpr (!SPLIT) {
        // Blocks of a key head follow each other at a distance that is a multiple of the number of its XCD, where that is one, and share that
        // one's L2; the last rows of a sequence, which see most keys, come first.
        const int32_t number = a.blocks - 1 - (int32_t)(blockIdx.x / head_groups);
        RowBlock blk;
        if (DIRECT && a.s.batch <= kCountedBatch) blk = row_block_at(a.s, number, (R == 256 ? 8 : 7) - heads_log2);
        else blk = row_block_of<R>(a.s, number, heads_log2);
        if (blk.sequence >= 0) work(blk, blockIdx.x % head_groups, 0, 0, nullptr);
    } else {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        // tiles of a block of rows; one that sees nothing has one too, since its rows are written
        const auto tiles_of = [&](const RowBlock &blk) {
            if (blk.sequence < 0) return 0;
            const int32_t n = block_keys<SEES>(a, blk, length_of(blk), KT).length;
            return n <= KT ? 1 : (n - 1) / KT + 1;
        };
        // In the line a block's tiles lie behind kBegin places that stand for its start and end, which cost about as much as they.
        constexpr int kBegin = DP == 128 && DIRECT ? 4 : 2;
        __shared__ int64_t upto_s[kSplitBlocks + 1], wave_s[NW];
        constexpr int EACH = kSplitBlocks / (64 * NW);
        int32_t places[EACH];
        int64_t sum = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            const int32_t number = threadIdx.x * EACH + i;
            places[i] = number < a.blocks ? tiles_of(row_block_of<R>(a.s, number, heads_log2)) : 0;
            if (places[i]) places[i] += kBegin;
            sum += places[i];
        }
        int64_t upto = sum;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t y = __shfl_up(upto, d);
            upto += lane >= d ? y : 0;
        }
        if (lane == 63) wave_s[wave] = upto;
        __syncthreads();
        upto -= sum;
        for (int i = 0; i < wave; ++i) upto += wave_s[i];
        if (threadIdx.x == 0) upto_s[0] = 0;
#pragma unroll
        for (int i = 0; i < EACH; ++i) {
            upto += places[i];
            upto_s[threadIdx.x * EACH + i + 1] = upto;
        }
        __syncthreads();
        const int64_t all = upto_s[kSplitBlocks];
        // shares of a key head one after the other on one XCD, which workgroups go to in turn
        const int32_t w = gridDim.x % 8 == 0 ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x;
        const int64_t units = all * head_groups, size = units <= 4 * (int64_t)gridDim.x ? 4 : (units - 1) / gridDim.x + 1;
        const int64_t share1 = (w + 1) * size < units ? (w + 1) * size : units;
        int64_t at = w * size;
        int32_t begun_in = -1, ends_in = -1;   // blocks that this share has a piece of: one that began before it, one that goes on behind it
        if (at < share1) {
            int32_t head_group = __builtin_amdgcn_readfirstlane((int32_t)(at / all)), number = 0;
            const int64_t place = at - head_group * all;
            for (int32_t hi = kSplitBlocks; hi - number > 1;) {   // the last block that begins at `place` or before, which has it
                const int32_t mid = (number + hi) / 2;
                if (upto_s[mid] <= place) number = mid; else hi = mid;
            }
            number = __builtin_amdgcn_readfirstlane(number);
            int32_t from = __builtin_amdgcn_readfirstlane((int32_t)(place - upto_s[number]));
            while (true) {
                const int32_t n = __builtin_amdgcn_readfirstlane((int32_t)(upto_s[number + 1] - upto_s[number]));
                const int32_t to = share1 - at < n - from ? from + (int32_t)(share1 - at) : n, id = head_group * a.blocks + number;
                const int32_t first = from < kBegin ? 0 : from - kBegin, last = to < kBegin ? 0 : to - kBegin;
                if (first < last) {
                    if (first > 0) begun_in = id;
                    if (to < n) ends_in = id;
                    float *sums = first > 0 || to < n ? a.pieces + (2 * (int64_t)w + (first > 0 ? 0 : 1)) * NW * kPromptPiece<DP> : nullptr;
                    work(row_block_of<R>(a.s, number, heads_log2), head_group, first, last, sums);
                }
                at += to - from;
                if (at >= share1) break;
                from = 0;
                do {
                    if (++number == a.blocks) {
                        number = 0;
                        ++head_group;
                    }
                } while (upto_s[number + 1] == upto_s[number]);
            }
        }
        if (threadIdx.x == 0) {
            a.cut[2 * w] = begun_in;
            a.cut[2 * w + 1] = ends_in;
        }
    }
}

// Joins the pieces of the block that begins in share blockIdx.x and goes on behind it, in the order of the shares; a wavefront has the 32 rows of one of the first kernel's, and DT tiles
// of 32 elements of their head: one of them, where one long sequence has many pieces (33 of them 80 us with four, 35 with one).
template <typename TR, int DP, int NW, int DT>
__global__ void __launch_bounds__(64) prompt_join_kernel(AttendArgs a, int heads_log2, int32_t shares)
{
    constexpr int UNROLL = DT == 1 ? 4 : 1;
    const int32_t w = blockIdx.x, wave = blockIdx.y, tile0 = blockIdx.z * DT;
    const int lane = threadIdx.x;
    const int32_t id = a.cut[2 * w + 1];
    if (id < 0 || a.cut[2 * w] == id) return;
    // shares behind w that begin in the block: as many in a row as there are
    int32_t more = 0;
    while (true) {
        const int32_t n = w + 1 + more + lane;
        const uint64_t bits = __ballot(n < shares && a.cut[2 * (n < shares ? n : w)] == id);
        const int run = ~bits == 0 ? 64 : __builtin_ctzll(~bits);
        more += run;
        if (run < 64) break;
    }
    const RowBlock blk = row_block_of<32 * NW>(a.s, id % a.blocks, heads_log2);
    const int32_t head = (id / a.blocks << heads_log2) + (wave & ((1 << heads_log2) - 1)), row = blk.first + 32 * (wave >> heads_log2) + lane % 32;
    if (blk.sequence < 0 || blk.first + 32 * (wave >> heads_log2) >= blk.end) return;
    const auto piece = [&](int32_t n) { return a.pieces + (n == 0 ? 2 * (int64_t)w + 1 : 2 * ((int64_t)w + n)) * NW * kPromptPiece<DP> + wave * kPromptPiece<DP>; };
    float top = kMinusInf;
    for (int32_t n = 0; n <= more; ++n) top = fmaxf(top, piece(n)[32 * DP + lane]);
    top = finite_max(top);
    f32x4 o[4 * DT];
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) o[i] = f32x4{0, 0, 0, 0};
#pragma unroll UNROLL
    for (int32_t n = 0; n <= more; ++n) {
        const float *p = piece(n);
        const float m = p[32 * DP + lane], part = p[32 * DP + 64 + lane];
        const float factor = __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
        l += part * factor;
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) o[i] += reinterpret_cast<const f32x4 *>(p)[(4 * tile0 + i) * 64 + lane] * factor;
    }
    const float factor = l == 0.0f ? 0.0f : 1.0f / l;
    if (row >= blk.end) return;
    char *out = static_cast<char *>(a.out.data) + (row * a.out.row + head * a.out.head) * 2;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
        const int e = 32 * tile0 + 8 * i + 4 * (lane / 32);
        if (e < a.head_dim) *reinterpret_cast<u32x2 *>(out + 2 * e) = u32x2{TR::pack(o[i].x * factor, o[i].y * factor), TR::pack(o[i].z * factor, o[i].w * factor)};
    }
}

}  // namespace sck
