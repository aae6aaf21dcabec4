// Prompt: attention of the rows of packed sequences over their keys, packed as well or in the pages of a cache.  One pass over the keys with the running
// maximum and sum of each row; scores and weights stay in registers.
//
// 16-bit types: prompt_tile.h.  fp32, here: the matrix cores have a sixteenth of the rate for it, so that keys and values straight from L2, for 16 rows of a
// wavefront, keep up with them.  SPLIT: the four wavefronts of a workgroup have the same 16 rows and every fourth step of their keys; otherwise 16 rows
// each and all keys.
//
// Five prompts up to 777 rows, 8 heads of 96 on 2: 37 us (30 TFLOP/s; a large product of the library reaches 153), 48 with the blocks in the order of their rows.  Matrix pipes are busy a third of
// the time, padding to 128 included: the 728 workgroups have 4.2 steps a wavefront on average, beside the search for their block, its rank among the others, the first
// keys and a join, and the heads of a key head read its keys each for itself.
#include <type_traits>

#include "prompt_tile.h"

namespace sck {

namespace {

// fp32: below so many workgroups of 64 rows (four for each compute unit) the keys are split too: the five prompts above take 50 us with and 114 without.
constexpr int64_t kSplitBlocks32 = 1024;

template <typename TR, int DP, bool EXACT, bool PAGED, bool SPLIT>
__global__ void __launch_bounds__(256, DP == 256 ? 1 : 2) prompt_kernel(AttendArgs a)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, STEP = SPLIT ? 4 * W::KEYS : W::KEYS;
    __shared__ typename std::conditional<SPLIT, typename Join<W>::Space, char>::type join_s;
    const int32_t head = blockIdx.x % a.heads, kv = head / a.group, place = blockIdx.x / a.heads;
    RowBlock blk;
    if (SPLIT && a.blocks <= 256 && a.s.batch > 1) {
        // The block with the place-th most keys: each thread has one and counts those before it.
        __shared__ int32_t keys_s[256];
        __shared__ RowBlock blk_s;
        blk = (int32_t)threadIdx.x < a.blocks ? row_block<16>(a.s, threadIdx.x) : RowBlock{-1, 0, 0, 0, 0};
        const int32_t mine = blk.sequence < 0 ? -1 : keys_seen(a, blk, PAGED ? paged_length(a.s, blk.sequence) : blk.count, blk.end - 1);
        keys_s[threadIdx.x] = mine;
        __syncthreads();
        int32_t ahead = 0;
#pragma unroll 8
        for (int32_t n = 0; n < a.blocks; ++n) ahead += keys_s[n] > mine || (keys_s[n] == mine && n < (int32_t)threadIdx.x);
        if (ahead == place && (int32_t)threadIdx.x < a.blocks) blk_s = blk;
        __syncthreads();
        const auto same = [](int32_t x) { return __builtin_amdgcn_readfirstlane(x); };
        blk = {same(blk_s.sequence), same(blk_s.first), same(blk_s.end), same(blk_s.begin), same(blk_s.count)};
    } else {
        blk = row_block<SPLIT ? 16 : 64>(a.s, a.blocks - 1 - place);
    }
    if (blk.sequence < 0) return;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int32_t first = SPLIT ? blk.first : blk.first + wave * 16, end = blk.end < first + 16 ? blk.end : first + 16;   // rows of the wavefront
    if (first >= end) return;   // never with SPLIT, whose wavefronts meet
    const int32_t length = PAGED ? paged_length(a.s, blk.sequence) : blk.count;

    W w;
    w.init(lane, a.head_dim);
    const int32_t row = first + w.col;
    char *out = static_cast<char *>(a.out.data) + (row * a.out.row + head * a.out.head) * B;
    if (length < 0) {
        if (row < end) w.store(out, __builtin_nanf(""));   // no sums yet: 0 * NaN
        return;
    }
    w.load_q(static_cast<const char *>(a.q.data) + ((row < end ? row : first) * a.q.row + head * a.q.head) * B, row < end);

    // keys that a row sees: none but those up to its own position
    const int32_t before = length - blk.count - blk.begin + 1;
    const auto sees = [&](int32_t r) {
        const int32_t n = a.causal ? before + r : length;
        return n < 0 ? 0 : n;
    };
    const int32_t visible = row < end ? sees(row) : 0, all = sees(first), most = sees(end - 1);
    const int64_t k_row = (PAGED ? a.cache.row : a.k.row) * B, v_row = (PAGED ? a.cache.row : a.v.row) * B;
    const char *k0 = PAGED ? static_cast<const char *>(a.cache.keys) + kv * a.cache.head * B
                           : static_cast<const char *>(a.k.data) + (blk.begin * a.k.row + kv * a.k.head) * B;
    const char *v0 = PAGED ? static_cast<const char *>(a.cache.values) + kv * a.cache.head * B
                           : static_cast<const char *>(a.v.data) + (blk.begin * a.v.row + kv * a.v.head) * B;
    bool bad = false;
    typename W::Keys keys;
    typename W::Values values;
    KeyTile t[TILES];
    const auto find = [&](int32_t base) __attribute__((always_inline)) {
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            int32_t at = base + 16 * n;
            if (at >= length) at = base;   // nothing of it is seen: any rows that are there
            t[n].last = length - 1 - at;
            if (PAGED) {
                int32_t page = page_of(a.s, blk.sequence, at);
                bad |= page < 0;
                if (page < 0) page = 0;
                const int64_t off = (page * a.cache.page + (at & ((1 << a.s.page_shift) - 1)) * a.cache.row) * B;
                t[n].k = k0 + off;
                t[n].v = v0 + off;
            } else {
                t[n].k = k0 + at * k_row;
                t[n].v = v0 + at * v_row;
            }
        }
    };
    // keys of the next step are asked for when the scores have used this step's, values when the second product has
    int32_t base = SPLIT ? wave * W::KEYS : 0;
    if (base < most) {
        find(base);
        w.load_keys(keys, t, k_row);
        w.load_values(values, t, v_row);
    }
    for (; base < most; base += STEP) {
        const bool more = base + STEP < most;
        typename W::Scores scores;
        w.scores(scores, keys);
        if (more) {
            find(base + STEP);
            w.load_keys(keys, t, k_row);
        }
        if (base + W::KEYS <= all) w.template add<false>(scores, values, a.scale_log2, 0);
        else w.template add<true>(scores, values, a.scale_log2, visible - base);
        if (more) w.load_values(values, t, v_row);
    }
    const float l = bad ? __builtin_nanf("") : over_groups_sum(w.l);
    if constexpr (SPLIT) {
        float r[W::EPL], top, sum;
        Join<W>::run(w, join_s, wave, lane, l, a.scale_log2, r, top, sum);
        if (row < end) Join<W>::template store<TR, EXACT>(w, r, wave, out, sum == 0.0f ? 0.0f : 1.0f / sum);
    } else {
        if (row < end) w.store(out, l == 0.0f ? 0.0f : 1.0f / l);
    }
}

// 16-bit types: wavefronts of a workgroup, and what a split costs besides.
template <int DP>
constexpr int kPromptWaves = DP == 256 ? 4 : 8;
template <int DP>
constexpr int64_t kSplitTiles = DP == 128 ? 7 : 12;

template <typename TR, int DP, bool PAGED>
void launch_padded(AttendArgs a, hipStream_t stream)
{
    if constexpr (TR::kBytes == 2) {
        constexpr int NW = kPromptWaves<DP>, KT = DP == 256 ? 32 : 128;
        int heads_log2 = 0;
        while (heads_log2 < 3 && a.group % (2 << heads_log2) == 0 && (2 << heads_log2) <= NW) ++heads_log2;
        const int64_t blocks = a.s.rows / (32 * NW >> heads_log2) + a.s.batch, groups = a.heads >> heads_log2;
        // Keys are split where the longest block alone would take longer than everything in equal shares.  The host knows neither lengths nor their sum: the longest
        // is taken as all that the table has room for, or twice the mean of packed sequences, the mean as half of that.  (A table for many more keys than there are
        // is split for nothing: 32, 8, 128, 4 sequences of 16 rows behind 100 keys 27 us with a table for 8,192, 10 with a view of the columns in use.)  Measured in tiles, the start and
        // the join of a split cost kSplitTiles, and its tiles 1.3 times as much (workgroups that begin at different keys do not meet in L2).  bf16, heads and key heads
        // of d, with and without a split: 8, 1, 128, 4,096 rows 80 and 118 us; 4, 4, 256, 2,000 rows 69 and 128; 8, 8, 64, 2,000 rows 38 and 46; chunks
        // behind up to 8,191 keys, 32, 8, 128: 264 and 320; but 32, 8, 128, 2,048 rows 90 and 73, 4,000 rows 196 and 172, 600 rows 50 and 29.
        const int64_t longest = PAGED ? table_room(a.s) : a.s.batch > 1 ? 2 * (int64_t)a.s.rows / a.s.batch : a.s.rows;
        const int64_t tiles = (longest < kMaxKeys ? longest : kMaxKeys) / KT;
        const int shares = prompt_shares(a.n_cu);
        if (a.pieces && blocks <= kSplitBlocks && tiles > 4 && tiles * shares > kSplitTiles<DP> * shares + 13 * blocks * groups * tiles / 20) {
            a.blocks = (int32_t)blocks;
            prompt_tile_kernel<TR, DP, PAGED, true, NW, KT><<<shares, 64 * NW, 0, stream>>>(a, heads_log2);
            prompt_join_kernel<TR, DP, NW><<<dim3(shares, NW), 64, 0, stream>>>(a, heads_log2, shares);
            return;
        }
        const auto kernel = prompt_tile_kernel<TR, DP, PAGED, false, NW, KT>;
        // a grid has fewer than 2^32 threads
        const int64_t each = (((int64_t)1 << 32) / (64 * NW) - 1) / groups;
        for (int64_t end = blocks; end > 0; end -= each) {
            a.blocks = (int32_t)end;
            kernel<<<(uint32_t)((end < each ? end : each) * groups), 64 * NW, 0, stream>>>(a, heads_log2);
        }
    } else {
        const bool split = (int64_t)row_blocks<64>(a.s.rows, a.s.batch) * a.heads < kSplitBlocks32;
        a.blocks = split ? row_blocks<16>(a.s.rows, a.s.batch) : row_blocks<64>(a.s.rows, a.s.batch);
        const auto kernel = a.head_dim == DP ? (split ? prompt_kernel<TR, DP, true, PAGED, true> : prompt_kernel<TR, DP, true, PAGED, false>)
                                             : (split ? prompt_kernel<TR, DP, false, PAGED, true> : prompt_kernel<TR, DP, false, PAGED, false>);
        // a grid has fewer than 2^32 threads
        const int32_t each = (int32_t)(((int64_t)1 << 24) - 1) / a.heads;
        for (int32_t end = a.blocks; end > 0; end -= each) {
            a.blocks = end;
            kernel<<<(end < each ? end : each) * a.heads, 256, 0, stream>>>(a);
        }
    }
}

template <typename TR, bool PAGED>
void launch_typed(const AttendArgs &a, hipStream_t stream)
{
    const int dp = padded_dim(a.head_dim);
    if (dp == 64) launch_padded<TR, 64, PAGED>(a, stream);
    else if (dp == 128) launch_padded<TR, 128, PAGED>(a, stream);
    else launch_padded<TR, 256, PAGED>(a, stream);
}

template <typename TR>
void launch_typed(const AttendArgs &a, bool paged, hipStream_t stream)
{
    if (paged) launch_typed<TR, true>(a, stream);
    else launch_typed<TR, false>(a, stream);
}

}  // namespace

int prompt_shares(int n_cu) { return n_cu; }   // the registers of a workgroup are a compute unit's

size_t prompt_workspace(sc_dtype dtype, int head_dim, int n_cu)
{
    if (dtype == SC_F32) return 0;
    const int dp = padded_dim(head_dim), n = prompt_shares(n_cu);
    const size_t piece = dp == 64 ? kPromptWaves<64> * kPromptPiece<64> : dp == 128 ? kPromptWaves<128> * kPromptPiece<128> : kPromptWaves<256> * kPromptPiece<256>;
    return 2 * n * (piece * sizeof(float) + sizeof(int32_t));
}

hipError_t launch_prompt(const AttendArgs &a, sc_dtype dtype, bool paged, hipStream_t stream)
{
    if (dtype == SC_BF16) launch_typed<Bf16>(a, paged, stream);
    else if (dtype == SC_F16) launch_typed<F16>(a, paged, stream);
    else launch_typed<F32>(a, paged, stream);
    return hipGetLastError();
}

}  // namespace sck
