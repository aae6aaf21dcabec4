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
#pragma once

#include "attention_device.h"

namespace sck {

template <typename TR, int DP, int NW, int KT>
struct PromptTile {
    static constexpr int THREADS = 64 * NW, CHUNKS = DP / 8, DT = DP / 32, NT = KT / 32;   // pieces of a row, tiles of the head, tiles of keys
    static constexpr int LOADS = KT * CHUNKS / THREADS, ROWS_PER_LOAD = THREADS / CHUNKS;
    static constexpr int ROW_BYTES = DP * 2, TILE_BYTES = KT * ROW_BYTES, LDS_BYTES = 4 * TILE_BYTES;
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

// Keys that row r of a block sees: none but those up to its own position.
__device__ __forceinline__ int32_t keys_seen(const AttendArgs &a, const RowBlock &blk, int32_t length, int32_t r)
{
    const int32_t n = a.causal ? length - blk.count - blk.begin + 1 + r : length;
    return n < 0 ? 0 : n;
}

// SPLIT: as in decode, the tiles of keys of all blocks are put in one line, block after block, one group of heads after the other, and every workgroup takes an
// equal share of it; blocks that shares cut leave pieces, which prompt_join_kernel joins.  Without it a workgroup has one block, and a call takes as long as
// the longest of them, or as the compute unit that was given most.  Chunks of four prompts behind up to 8,191 keys, 32 heads of 128: 262 to 274 us with, 320
// without; L2 misses are six times as many, since workgroups begin at different keys, and the join is 18 us.
template <typename TR, int DP, bool PAGED, bool SPLIT, int NW, int KT>
__global__ void __launch_bounds__(64 * NW, NW / 4) prompt_tile_kernel(AttendArgs a, int heads_log2)
{
    using P = PromptTile<TR, DP, NW, KT>;
    constexpr int CHUNKS = P::CHUNKS, DT = P::DT, NT = P::NT, LOADS = P::LOADS, R = 32 * NW;
    __shared__ __attribute__((aligned(16))) char tile_s[P::LDS_BYTES];   // [buffer][keys, values]
    const int32_t head_groups = a.heads >> heads_log2;

    // Keys of tiles first_tile .. last_tile - 1 for a block of rows and a group of heads; sums: where the sums go if those are not all tiles that it sees.
    const auto work = [&](const RowBlock &blk, int32_t head_group, int32_t first_tile, int32_t last_tile, float *sums) __attribute__((always_inline)) {
        uint32_t thread = threadIdx.x;
        asm volatile("" : "+v"(thread));   // what follows from it is made again for each block, instead of taking the registers of the main loop
        const int lane = thread % 64, wave = __builtin_amdgcn_readfirstlane(thread / 64), q = lane % 32, half = lane / 32;
        const int32_t head0 = head_group << heads_log2, kv = head0 / a.group;
        const int32_t length = PAGED ? paged_length(a.s, blk.sequence) : blk.count;
        const int32_t head = head0 + (wave & ((1 << heads_log2) - 1)), first = blk.first + 32 * (wave >> heads_log2), row = first + q;
        const bool mine = row < blk.end;
        char *out = static_cast<char *>(a.out.data) + (row * a.out.row + head * a.out.head) * 2;
        if (length < 0) {
            if (mine)
                for (int d = 8 * half; d < a.head_dim; d += 16) *reinterpret_cast<u32x4 *>(out + 2 * d) = u32x4{0, 0, 0, 0} + TR::kExponent * 0x10001u + 0x00010001u;
            return;
        }

        const auto sees = [&](int32_t r) { return keys_seen(a, blk, length, r); };
        int32_t block_most = sees(blk.end - 1);
        if (SPLIT && last_tile < (block_most + KT - 1) / KT) block_most = last_tile * KT;
        const int32_t visible = mine ? sees(row) : 0;
        const int32_t most = first < blk.end ? sees((first + 32 < blk.end ? first + 32 : blk.end) - 1) : 0;

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
        // They are added to the rows that see them, from memory.
        const auto add_special = [&](int32_t base) {
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
                        if (key >= visible || e >= a.head_dim) continue;
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
        const auto tile = [&](Lds buffer, int32_t base, auto masked) {
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
                    if (MASK) s[t][r] = 32 * t + 8 * (r / 4) + 4 * half + r % 4 < visible - base ? s[t][r] : kMinusInf;
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
                    l += s[t][r] + s[t][r + 1];
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
            const int32_t block_all = sees(blk.first);   // keys that every row of the block sees
            int32_t base = SPLIT ? first_tile * KT : 0;
            fetch(base);
            bool special = __syncthreads_or(put(tile_s, base + KT > block_all));
            int buffer = 0;
            const auto pass = [&](auto masked) {
                constexpr bool MASK = decltype(masked)::value;
                const bool more = base + KT < block_most, part = MASK || base + 2 * KT > block_all;
                if (more) fetch(base + KT);
                if (!MASK || base < most) {
                    tile((Lds)tile_s + buffer * 2 * P::TILE_BYTES, base, masked);
                    if (MASK && special) add_special(base);
                }
                buffer ^= 1;
                bool any = false;
                if (more) any = put(tile_s + buffer * 2 * P::TILE_BYTES, part);
                if (part) special = __syncthreads_or(any);
                else __syncthreads();
                base += KT;
            };
            // tiles that every row of the block sees whole, then the others
            while (base + KT <= block_all && (!SPLIT || base < block_most)) pass(std::false_type());
            while (base < block_most) pass(std::true_type());
        }
        if (PAGED) bad = __syncthreads_or(bad);
        l += __shfl_xor(l, 32);
        if (SPLIT && sums) {
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

    if constexpr (!SPLIT) {
        // Blocks of a key head follow each other at a distance that is a multiple of the number of its XCD, where that is one, and share that
        // one's L2; the last rows of a sequence, which see most keys, come first.
        const RowBlock blk = row_block_of<R>(a.s, a.blocks - 1 - (int32_t)(blockIdx.x / head_groups), heads_log2);
        if (blk.sequence >= 0) work(blk, blockIdx.x % head_groups, 0, 0, nullptr);
    } else {
        const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
        // tiles of a block of rows; one that sees nothing has one too, since its rows are written
        const auto tiles_of = [&](const RowBlock &blk) {
            if (blk.sequence < 0) return 0;
            const int32_t n = keys_seen(a, blk, PAGED ? paged_length(a.s, blk.sequence) : blk.count, blk.end - 1);
            return n <= KT ? 1 : (n - 1) / KT + 1;
        };
        // In the line a block's tiles lie behind kBegin places that stand for its start and end, which cost about as much as they.
        constexpr int kBegin = 2;
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

// Joins the pieces of the block that begins in share blockIdx.x and goes on behind it, in the order of the shares; a wavefront has the 32 rows of one of the first kernel's.
template <typename TR, int DP, int NW>
__global__ void __launch_bounds__(64) prompt_join_kernel(AttendArgs a, int heads_log2, int32_t shares)
{
    constexpr int DT = DP / 32;
    const int32_t w = blockIdx.x, wave = blockIdx.y;
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
    const auto piece = [&](int32_t n) { return a.pieces + (n == 0 ? 2 * (int64_t)w + 1 : 2 * ((int64_t)w + n)) * NW * kPromptPiece<DP> + wave * kPromptPiece<DP>; };
    float top = kMinusInf;
    for (int32_t n = 0; n <= more; ++n) top = fmaxf(top, piece(n)[32 * DP + lane]);
    top = finite_max(top);
    f32x4 o[4 * DT];
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) o[i] = f32x4{0, 0, 0, 0};
    for (int32_t n = 0; n <= more; ++n) {
        const float *p = piece(n);
        const float m = p[32 * DP + lane], part = p[32 * DP + 64 + lane];
        const float factor = __builtin_amdgcn_exp2f((m - top) * a.scale_log2);
        l += part * factor;
#pragma unroll
        for (int i = 0; i < 4 * DT; ++i) o[i] += reinterpret_cast<const f32x4 *>(p)[i * 64 + lane] * factor;
    }
    const float factor = l == 0.0f ? 0.0f : 1.0f / l;
    if (blk.sequence < 0 || row >= blk.end) return;
    char *out = static_cast<char *>(a.out.data) + (row * a.out.row + head * a.out.head) * 2;
#pragma unroll
    for (int i = 0; i < 4 * DT; ++i) {
        const int e = 8 * i + 4 * (lane / 32);
        if (e < a.head_dim) *reinterpret_cast<u32x2 *>(out + 2 * e) = u32x2{TR::pack(o[i].x * factor, o[i].y * factor), TR::pack(o[i].z * factor, o[i].w * factor)};
    }
}

}  // namespace sck
