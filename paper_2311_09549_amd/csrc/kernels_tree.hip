// Trees: attention of a few rows per sequence over a paged cache, of which each sees what is before the tree, its ancestors and itself; and of single rows through a window.
//
// Rows of a sequence and the heads that share a key head are one list of pairs (row, head), and tiles of 16 RT of them take the keys as decode's heads do: the keys that a
// sequence's rows see (span_of: with a window, a line without the gap), tile after tile and key head after key head, are one line of units of 128, and every
// workgroup takes an equal share of it.  A step's keys and values are read into registers once for RT products of 16 pairs each: with few pairs everything is bound by memory.
// Steps that all rows see whole are taken without a mask; the others by bits, one for each key and row, from chains of parents that are gone up once, in LDS.
//
// Single rows, 64 sequences up to 32,767 keys through a window of 4,096, bf16, 32 heads of 128 on 8: 154 us a call, 5.0 TB/s (a large copy reaches 4.7), of which the join is 5.  Trees
// behind 24 sequences of 8,192 keys: of 4 rows 171 us (4.7 TB/s), of 16 rows, 64 pairs, 186 (4.3).  fp32, 16 heads of 80 with keys of their own, trees of up to 21 rows behind
// 12 sequences up to 1,500: 28 us (29 with the products of pieces behind the head) and 7 for the join, matrix pipes (with pairs padded to 16 or 32) busy a quarter of the time, 2.9 TB/s, waits 0.4: what a step of keys
// ahead does not cover; two tiles of pairs at a time, with one workgroup on a compute unit instead of two, take 50.  Behind few keys, tree_whole_kernel: 8 sequences of 320 keys and 8 rows 10.6 us, a chain of reads.
#include "attention_device.h"

namespace sck {

namespace {

constexpr int kWaves = 4;   // that Join takes
constexpr int64_t kWholeKeys = 512;

// Registers of a wavefront: queries and sums of RT tiles, keys and values of a step.
template <typename W, int RT>
constexpr int kTreeGroups = RT * 4 * (W::QC + W::EPL) + W::TILES * 4 * (W::QC + W::VW) + 60 <= 256 ? 2 : 1;   // workgroups on a compute unit

// Most tiles of pairs that a workgroup takes.
template <typename TR, int DP>
constexpr int kTreeTiles = DP == 256 ? 1 : TR::kBytes == 4 ? (DP == 64 ? 2 : 1) : 4;

__device__ __forceinline__ int32_t same(int32_t x) { return __builtin_amdgcn_readfirstlane(x); }

// What a sequence has: rows, keys (-1: a wrong length), their line.
struct TreeSequence {
    int32_t begin, count, length;
    Span span;
};

__device__ __forceinline__ TreeSequence tree_sequence(const AttendArgs &a, int32_t b)
{
    TreeSequence q;
    q.begin = row_begin(a.s, b);
    q.count = row_begin(a.s, b + 1) - q.begin;
    q.length = paged_length(a.s, b);
    if (a.tree && (q.length < q.count || (a.parent && q.count > kMaxNodes))) q.length = -1;
    q.span = span_of(q.length, a.window, a.sinks, q.length - q.count);
    return q;
}

// Units of a segment (one at least: its rows are written), and tiles of a key head.
__device__ __forceinline__ int32_t tree_units(const TreeSequence &q) { return q.span.length <= kDecodeUnit ? 1 : units_of(q.span.length); }
template <int PAIRS>
__device__ __forceinline__ int32_t tree_tiles(const AttendArgs &a, int32_t count) { return count <= 0 ? 0 : (int32_t)(((int64_t)count * a.group - 1) / PAIRS) + 1; }

// The line of units, 64 sequences at a time, a lane each.
template <int PAIRS>
struct TreeLine {
    const AttendArgs &a;
    int lane;
    int64_t mine, upto;    // units of sequence 64 chunk + lane, of it and those before it in the chunk
    int32_t chunk;
    int64_t before;        // units of the chunks before

    static __device__ __forceinline__ int64_t lane_value(int64_t x, int at)
    {
        return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((uint32_t)(x >> 32), at) << 32 | (uint32_t)__builtin_amdgcn_readlane((uint32_t)x, at));
    }
    __device__ __forceinline__ void load(int32_t c)
    {
        chunk = c;
        const int32_t b = 64 * c + lane;
        mine = 0;
        if (b < a.s.batch) {
            const TreeSequence q = tree_sequence(a, b);
            mine = (int64_t)tree_units(q) * tree_tiles<PAIRS>(a, q.count) * a.kv_heads;
        }
        upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t y = __shfl_up(upto, d);
            upto += lane >= d ? y : 0;
        }
    }
    __device__ __forceinline__ int64_t chunk_units() const { return lane_value(upto, 63); }
    // Units of all sequences.  One chunk stays loaded.
    __device__ __forceinline__ int64_t all()
    {
        int64_t n = 0;
        for (int32_t c = 0; 64 * c < a.s.batch; ++c) {
            load(c);
            n += chunk_units();
        }
        before = 0;
        if (a.s.batch > 64) load(0);
        return n;
    }
    // The sequence that has unit u (below all()), and the units before it.
    __device__ __forceinline__ int32_t find(int64_t u, int64_t &ahead)
    {
        while (before + chunk_units() <= u) {
            before += chunk_units();
            load(chunk + 1);
        }
        const int at = __ffsll((unsigned long long)__ballot(before + upto > u)) - 1;
        ahead = before + lane_value(upto, at) - lane_value(mine, at);
        return 64 * chunk + at;
    }
};

// What the rows of a tile of pairs see, in LDS: chains of their parents, and per row the nodes that it sees and its depth.
template <int PAIRS>
struct TreeSeen {
    struct Space {
        int32_t parent[kMaxNodes];
        uint32_t seen[PAIRS][kMaxNodes / 32 + 1];
        int32_t depth[PAIRS];
    };
    const AttendArgs &a;
    Space &space;
    bool chains;                  // whether `space` is needed, and filled
    int32_t before;               // keys before the rows
    int32_t row_first, row_last;  // of the tile
    int32_t all, low;             // keys that all rows of the tile see: below `all`, and from `low` on or below `sinks`

    // `tile`: of pairs; `end`: of the keys of the line that it takes here.
    __device__ __forceinline__ TreeSeen(const AttendArgs &args, Space &s, const TreeSequence &q, int32_t tile, int32_t end) : a(args), space(s)
    {
        before = q.length - q.count;
        row_first = same(tile * PAIRS / a.group);
        row_last = same((tile * PAIRS + PAIRS - 1) / a.group);
        row_last = row_last < q.count ? row_last : q.count - 1;
        // chains, where keys are nodes or a window goes by depths
        chains = a.parent && q.length >= 0 && (a.window || key_at(q.span, end - 1) >= before);
        all = a.parent ? before : before + row_first + 1;
        low = window_low(a.window, before + row_last);
    }
    // By all threads of a workgroup, which meet twice.
    __device__ __forceinline__ void fill(const TreeSequence &q)
    {
        if (!chains) return;
        for (int32_t i = threadIdx.x; i < q.count; i += blockDim.x) space.parent[i] = a.parent[q.begin + i];
        __syncthreads();
        const int32_t i = row_first + (int32_t)threadIdx.x;
        if (i <= row_last) {
            const int32_t depth = depth_of(space.parent, i);
            uint32_t(&seen)[kMaxNodes / 32 + 1] = space.seen[threadIdx.x];
            space.depth[threadIdx.x] = depth;
            int32_t node = depth < 0 ? -1 : i, up = 0;
            seen[(q.count + 31) / 32] = 0;
            for (int32_t word = (q.count - 1) / 32; word >= 0; --word) {
                uint32_t bits = 0;
                for (; node >= 32 * word && node >= 0; node = space.parent[node], ++up)
                    if (!a.window || up < a.window || before + depth - up < a.sinks) bits |= 1u << (node & 31);
                seen[word] = bits;
            }
        }
        __syncthreads();
    }
    __device__ __forceinline__ bool whole(int32_t key) const { return key + 16 <= all && (key >= low || key + 16 <= a.sinks); }
    // Of the 16 keys from `key` on, bits of those that row i sees.
    __device__ __forceinline__ uint32_t of(int32_t key, int32_t i) const
    {
        const int32_t at = i - row_first, place = a.parent ? (chains ? before + space.depth[at] : 0) : before + i;
        uint32_t bits = below((a.parent ? before : place + 1) - key);
        if (a.window) bits &= ~below(window_low(a.window, place) - key) | below(a.sinks - key);
        if (a.parent && key + 16 > before) {
            const int32_t node = key - before;   // the first of them; nodes behind the last have no bits
            const uint32_t *seen = space.seen[at];
            if (node < 0) bits |= seen[0] << -node;
            else bits |= (uint32_t)(((uint64_t)seen[node / 32 + 1] << 32 | seen[node / 32]) >> (node & 31));
        }
        return bits & 0xffffu;
    }
    __device__ __forceinline__ bool wrong(int32_t i) const { return chains && i >= 0 && space.depth[i - row_first] < 0; }
};

template <typename TR, int DP, bool EXACT, int RT>
__global__ void __launch_bounds__(64 * kWaves, (kTreeGroups<Wave<TR, DP, EXACT>, RT>)) tree_kernel(AttendArgs a, int32_t groups_log2)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, EPL = W::EPL, PAIRS = 16 * RT;
    __shared__ typename Join<W>::Space join_s;
    __shared__ typename TreeSeen<PAIRS>::Space seen_s;
    const int lane = threadIdx.x % 64, wave = same(threadIdx.x / 64);
    TreeLine<PAIRS> line = {a, lane};
    const int64_t units = line.all();   // in scalar registers, as what follows from it
    const int64_t share0 = share_begin(units, blockIdx.x, groups_log2), share1 = share_begin(units, blockIdx.x + 1, groups_log2);
    TreeCut cut = {0, 0, 0, 0, 0, 0};
    if (share0 < share1) {
        // Units [u0, u1) of a segment (a tile of pairs and a key head): what is worked on at a time.
        struct Part {
            int64_t before;   // place in the line of the first unit of sequence b
            int32_t b, kv, tile, tiles, n_units, u0, u1;
            TreeSequence q;
        };
        int64_t at = share0;
        Part part;
        const auto load = [&]() {
            const TreeSequence q = tree_sequence(a, part.b);
            part.q = {same(q.begin), same(q.count), same(q.length), {same(q.span.first), same(q.span.skip), same(q.span.length)}};
            part.n_units = tree_units(part.q);
            part.tiles = same(tree_tiles<PAIRS>(a, part.q.count));
        };
        const auto upto = [&]() { part.u1 = (int32_t)(share1 - at < part.n_units - part.u0 ? part.u0 + (share1 - at) : part.n_units); };
        part.b = line.find(at, part.before);
        load();
        const int64_t segment = quotient(at - part.before, part.n_units);
        part.u0 = same((int32_t)(at - part.before - segment * part.n_units));
        part.kv = same((int32_t)quotient(segment, part.tiles));
        part.tile = same((int32_t)(segment - (int64_t)part.kv * part.tiles));
        upto();

        W w[RT];
        int32_t row[RT];   // of the lane's pairs, from the first row of the sequence; -1: no pair
        const int64_t row_bytes = a.cache.row * B;
        constexpr int32_t STEP = kWaves * W::KEYS;
        typename W::Keys keys;
        typename W::Values values;
        KeyTile t[TILES];
        bool bad = false;
        const auto find = [&](int32_t base) __attribute__((always_inline)) {
#pragma unroll
            for (int n = 0; n < TILES; ++n) {
                const int32_t v = base + 16 * n, key = key_at(part.q.span, v < part.q.span.length ? v : base);   // behind the last key nothing is seen: any rows that are there
                t[n].last = part.q.length - 1 - key;
                int32_t page = page_of_all(a.s, part.b, key);
                bad |= page < 0;
                if (page < 0) page = 0;
                const int64_t off = (page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row + part.kv * a.cache.head) * B;
                t[n].k = static_cast<const char *>(a.cache.keys) + off;
                t[n].v = static_cast<const char *>(a.cache.values) + off;
            }
        };
        const auto head_of = [&](int32_t pair, int32_t i) { return part.kv * a.group + (pair - i * a.group); };
        while (true) {
            const int32_t end = part.u1 == part.n_units ? part.q.span.length : part.u1 * kDecodeUnit, base0 = part.u0 * kDecodeUnit + wave * W::KEYS;
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                w[r].init(lane, a.head_dim);
                const int32_t pair = part.tile * PAIRS + 16 * r + w[r].col, i = pair / a.group;
                const bool there = i < part.q.count;
                row[r] = there ? i : -1;
                w[r].load_q(static_cast<const char *>(a.q.data) + ((int64_t)(part.q.begin + (there ? i : 0)) * a.q.row + (there ? head_of(pair, i) : 0) * a.q.head) * B, there);
            }
            if (base0 < end) {
                find(base0);
                w[0].load_keys(keys, t, row_bytes);
                w[0].load_values(values, t, row_bytes);
            }
            TreeSeen<PAIRS> rows(a, seen_s, part.q, part.tile, end);
            rows.fill(part.q);
            for (int32_t base = base0; base < end; base += STEP) {
                const bool more = base + STEP < end;
                typename W::Scores scores[RT];
#pragma unroll
                for (int r = 0; r < RT; ++r) w[r].template scores<B == 4>(scores[r], keys);
                if (more) {
                    find(base + STEP);
                    w[0].load_keys(keys, t, row_bytes);
                }
                bool whole = true, special = false;
                int32_t key[TILES];
                uint32_t seen[RT];
#pragma unroll
                for (int n = 0; n < TILES; ++n) {
                    key[n] = key_at(part.q.span, base + 16 * n);
                    whole &= base + 16 * n < part.q.span.length && rows.whole(key[n]);
                }
                if (!whole) {
#pragma unroll
                    for (int r = 0; r < RT; ++r) {
                        // of lanes without a pair as of the first row: no part of the wavefront has a branch of its own here, where all registers hold operands of products
                        // (the compiler moves some of them about behind such a branch, before it has all lanes back)
                        seen[r] = 0;
#pragma unroll
                        for (int n = 0; n < TILES; ++n)
                            if (base + 16 * n < part.q.span.length) seen[r] |= rows.of(key[n], row[r] < 0 ? rows.row_first : row[r]) << 16 * n;
                        W::mask(scores[r], seen[r] >> 4 * w[0].g);
                    }
                    special = W::any_special(values);
                    if (special) W::without_infinities(values);
                }
#pragma unroll
                for (int r = 0; r < RT; ++r) w[r].add_seen(scores[r], values, a.scale_log2);
                if (more) w[0].load_values(values, t, row_bytes);
                if (special) {
                    // infinities and NaN that the products would have spread to rows that do not see them (0 times infinity) are added to those that do, from memory
#pragma unroll 1
                    for (int n = 0; n < W::KEYS; ++n) {
                        const int32_t place = base + (n & ~15), j = key_at(part.q.span, place) + (n & 15);
                        if (place >= part.q.span.length || j >= part.q.length) continue;
                        const int32_t page = page_of(a.s, part.b, j);
                        const char *p = static_cast<const char *>(a.cache.values) +
                                        ((page < 0 ? 0 : page) * a.cache.page + (j & ((1 << a.s.page_shift) - 1)) * a.cache.row + part.kv * a.cache.head) * B;
#pragma unroll
                        for (int r = 0; r < RT; ++r)
                            if (seen[r] >> n & 1) w[r].add_special(p);
                    }
                }
            }
            bad |= part.q.length < 0;
            const bool whole_segment = part.u0 == 0 && part.u1 == part.n_units;
            const int64_t first = part.before + ((int64_t)part.kv * part.tiles + part.tile) * part.n_units;
            float *piece = a.pieces + (int64_t)piece_slot(first, share0, blockIdx.x) * RT * piece_floats(DP);
#pragma unroll
            for (int r = 0; r < RT; ++r) {
                const bool wrong = bad || rows.wrong(row[r]);
                const float l = over_groups_sum(w[r].l);
                float x[EPL], top, sum;
                Join<W>::run(w[r], join_s, wave, lane, wrong ? __builtin_nanf("") : l, a.scale_log2, x, top, sum);
                if (row[r] < 0) continue;
                const int32_t pair = part.tile * PAIRS + 16 * r + w[0].col;
                if (whole_segment) {
                    char *out = static_cast<char *>(a.out.data) + ((int64_t)(part.q.begin + row[r]) * a.out.row + head_of(pair, row[r]) * a.out.head) * B;
                    Join<W>::template store<TR, EXACT>(w[r], x, wave, out, sum == 0.0f ? 0.0f : 1.0f / sum);
                } else {
                    float *p = piece + r * piece_floats(DP);
                    const int e0 = (4 * w[0].g + wave) * EPL;
#pragma unroll
                    for (int u = 0; u < EPL; u += 4) *reinterpret_cast<f32x4 *>(p + w[0].col * DP + e0 + u) = f32x4{x[u], x[u + 1], x[u + 2], x[u + 3]};
                    if (wave == 0 && w[0].g == 0) {
                        p[kHeadTile * DP + w[0].col] = top;
                        p[kHeadTile * (DP + 1) + w[0].col] = sum;
                    }
                }
            }
            if (part.u0 == 0 && part.u1 < part.n_units) cut = {first, units, part.n_units, part.b, part.kv, part.tile};
            // the next part
            at += part.u1 - part.u0;
            if (at >= share1) break;
            bad = false;
            part.u0 = 0;
            if (++part.tile == part.tiles) {
                part.tile = 0;
                if (++part.kv == a.kv_heads) {
                    part.kv = 0;
                    part.before = at;
                    do {
                        ++part.b;   // share1 is not behind the last unit
                        load();
                    } while (part.tiles == 0);
                }
            }
            upto();
        }
    }
    if (threadIdx.x == 0) a.tree_cut[blockIdx.x] = cut;
}

// Joins the pieces of the segment that workgroup blockIdx.x of the first kernel began and left to others, in the order of the line; a wavefront has one pair.
template <typename TR, int DP, int RT>
__global__ void __launch_bounds__(256) tree_join_kernel(AttendArgs a, int32_t groups_log2)
{
    constexpr int B = TR::kBytes, LANES = DP / 4, PARTS = 64 / LANES, PAIRS = 16 * RT;
    const TreeCut cut = a.tree_cut[blockIdx.x];
    if (cut.units == 0) return;
    const int lane = threadIdx.x % 64, at = blockIdx.y * 4 + threadIdx.x / 64;   // pair of the tile
    const int32_t begin = row_begin(a.s, cut.b), count = row_begin(a.s, cut.b + 1) - begin;
    const int32_t pair = cut.tile * PAIRS + at, i = pair / a.group;
    if (i >= count) return;
    const int32_t w0 = blockIdx.x, w1 = share_of(cut.all, cut.first + cut.units - 1, groups_log2);
    const auto piece = [&](int32_t w) {
        return a.pieces + ((int64_t)piece_slot(cut.first, share_begin(cut.all, w, groups_log2), w) * RT + at / 16) * piece_floats(DP);
    };
    // workgroups between them may have no units, where there are fewer of those: they have no piece either
    const auto none = [&](int32_t w) { return share_begin(cut.all, w, groups_log2) == share_begin(cut.all, w + 1, groups_log2); };
    float top = kMinusInf;
    for (int32_t w = w0 + lane; w <= w1; w += 64)
        if (!none(w)) top = fmaxf(top, piece(w)[kHeadTile * DP + at % 16]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    top = finite_max(top);
    f32x4 sum = {0, 0, 0, 0};
    float weight = 0.0f;
    const int part = lane / LANES, e = lane % LANES * 4;
    for (int32_t base = w0; base <= w1; base += 64) {
        const int32_t w = base + lane;
        const bool is = w <= w1 && !none(w);
        float factor = 0.0f;
        if (is) {
            const float *p = piece(w);
            factor = __builtin_amdgcn_exp2f((p[kHeadTile * DP + at % 16] - top) * a.scale_log2);
            weight += p[kHeadTile * (DP + 1) + at % 16] * factor;
        }
        const uint64_t there = __ballot(is);
        const int n = w1 - base < 63 ? w1 - base + 1 : 64;
        for (int k0 = 0; k0 < n; k0 += PARTS) {
            const int k = k0 + part;
            const float f = __shfl(factor, k % 64);
            if (k < n && (there >> k & 1)) sum += *reinterpret_cast<const f32x4 *>(piece(base + k) + at % 16 * DP + e) * f;
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) weight += __shfl_xor(weight, d);
#pragma unroll
    for (int d = LANES; d < 64; d *= 2)
#pragma unroll
        for (int k = 0; k < 4; ++k) sum[k] += __shfl_xor(sum[k], d);
    if (part != 0 || e >= a.head_dim) return;
    sum *= weight == 0.0f ? 0.0f : 1.0f / weight;
    char *out = static_cast<char *>(a.out.data) + ((int64_t)(begin + i) * a.out.row + (cut.kv * a.group + pair - i * a.group) * a.out.head + e) * B;
    if constexpr (B == 2) *reinterpret_cast<u32x2 *>(out) = u32x2{TR::pack(sum.x, sum.y), TR::pack(sum.z, sum.w)};
    else *reinterpret_cast<f32x4 *>(out) = sum;
}

// Few keys: a workgroup for each tile of 16 pairs, whose wavefronts take a few steps each; no shares to find, no pieces to join.
template <int DP>
constexpr int kWholeWaves = DP == 256 ? 4 : 8;

// Tiles of pairs of all sequences, without a table of them: sequence b has the numbers from row_begin(b) * group / 16 + b up to that of b + 1, never fewer than it has tiles;
// numbers left over have no pairs.
__device__ __forceinline__ int32_t first_tile_of(const AttendArgs &a, int32_t b) { return (int32_t)((int64_t)row_begin(a.s, b) * a.group / kHeadTile) + b; }

template <typename TR, int DP, bool EXACT>
__global__ void __launch_bounds__(64 * kWholeWaves<DP>, kWholeWaves<DP> / 4) tree_whole_kernel(AttendArgs a)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, EPL = W::EPL, WAVES = kWholeWaves<DP>, LD = DP + 4, PAIRS = kHeadTile;   // rows of sums begin in different banks
    // chains are done with before sums are stored
    __shared__ union {
        typename TreeSeen<PAIRS>::Space seen;
        __attribute__((aligned(16))) float sum[WAVES][PAIRS][LD];
    } space_s;
    __shared__ float top_s[WAVES][PAIRS], weight_s[WAVES][PAIRS];
    const int lane = threadIdx.x % 64, wave = same(threadIdx.x / 64);
    const int32_t kv = blockIdx.x % a.kv_heads, number = blockIdx.x / a.kv_heads;
    // the last sequence that begins at this number or before, 64 at a time
    int32_t b = 0;
    for (int32_t end = a.s.batch;;) {
        const int32_t step = (end - b + 63) / 64;
        const int64_t at = b + (int64_t)lane * step;
        const uint64_t bits = __ballot(at < end && first_tile_of(a, (int32_t)at) <= number);
        if (bits == 0) return;
        b += (63 - __builtin_clzll(bits)) * step;
        if (step == 1) break;
        end = end - b < step ? end : b + step;
    }
    TreeSequence q = tree_sequence(a, b);
    q = {same(q.begin), same(q.count), same(q.length), {same(q.span.first), same(q.span.skip), same(q.span.length)}};
    const int32_t tile = same(number - first_tile_of(a, b));
    if (q.count <= 0 || (int64_t)tile * PAIRS >= (int64_t)q.count * a.group) return;
    constexpr int32_t STEP = WAVES * W::KEYS;
    W w;
    w.init(lane, a.head_dim);
    const int32_t pair = tile * PAIRS + w.col, i = pair / a.group, row = i < q.count ? i : -1;
    const int32_t head = row < 0 ? 0 : kv * a.group + (pair - i * a.group);
    w.load_q(static_cast<const char *>(a.q.data) + ((int64_t)(q.begin + (row < 0 ? 0 : row)) * a.q.row + head * a.q.head) * B, row >= 0);
    const char *k0 = static_cast<const char *>(a.cache.keys) + kv * a.cache.head * B, *v0 = static_cast<const char *>(a.cache.values) + kv * a.cache.head * B;
    const int64_t row_bytes = a.cache.row * B;
    const int32_t end = q.span.length;
    bool bad = q.length < 0;
    TreeSeen<PAIRS> rows(a, space_s.seen, q, tile, end);
    bool filled = false;
    for (int32_t base0 = 0; base0 < end || !filled; base0 += STEP) {
        const int32_t base = base0 + wave * W::KEYS;
        typename W::Keys keys;
        typename W::Values values;
        typename W::Scores scores;
        KeyTile t[TILES];
        int32_t key[TILES];
        if (base < end) {
#pragma unroll
            for (int n = 0; n < TILES; ++n) {
                key[n] = key_at(q.span, base + 16 * n < end ? base + 16 * n : base);   // behind the last key nothing is seen: any rows that are there
                t[n].last = q.length - 1 - key[n];
                int32_t page = page_of_all(a.s, b, key[n]);
                bad |= page < 0;
                if (page < 0) page = 0;
                const int64_t off = (page * a.cache.page + (key[n] & ((1 << a.s.page_shift) - 1)) * a.cache.row) * B;
                t[n].k = k0 + off;
                t[n].v = v0 + off;
            }
            w.load_keys(keys, t, row_bytes);
            w.load_values(values, t, row_bytes);
        }
        if (!filled) rows.fill(q);   // keys and values are on their way
        filled = true;
        if (base < end) {
            w.template scores<B == 4>(scores, keys);
            uint32_t seen = 0;
#pragma unroll
            for (int n = 0; n < TILES; ++n)
                if (base + 16 * n < end) seen |= rows.of(key[n], row < 0 ? rows.row_first : row) << 16 * n;
            W::mask(scores, seen >> 4 * w.g);
            const bool special = W::any_special(values);
            if (special) W::without_infinities(values);
            w.add_seen(scores, values, a.scale_log2);
            if (special) {
                // infinities and NaN that the product would have spread to rows that do not see them are added to those that do, from memory
#pragma unroll 1
                for (int n = 0; n < W::KEYS; ++n) {
                    const KeyTile &x = n < 16 ? t[0] : t[TILES - 1];
                    if (n % 16 <= x.last && (seen >> n & 1)) w.add_special(x.v + n % 16 * row_bytes);
                }
            }
        }
    }
    const int parts = end <= 0 ? 0 : end > STEP - W::KEYS ? WAVES : (end - 1) / W::KEYS + 1;   // wavefronts that have had keys
    const float l = bad || rows.wrong(row) ? __builtin_nanf("") : over_groups_sum(w.l);
    __syncthreads();
    if (wave < parts) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int u = 0; u < EPL; u += 4)
                *reinterpret_cast<f32x4 *>(&space_s.sum[wave][w.col][(4 * w.g + k) * EPL + u]) = f32x4{w.o[u][k], w.o[u + 1][k], w.o[u + 2][k], w.o[u + 3][k]};
        if (w.g == 0) {
            top_s[wave][w.col] = w.m;
            weight_s[wave][w.col] = l;
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < PAIRS * (DP / 4); x += 64 * WAVES) {
        const int c = x / (DP / 4), e = x % (DP / 4) * 4;
        const int32_t p = tile * PAIRS + c, r = p / a.group;
        if (r >= q.count || (!EXACT && e >= a.head_dim)) continue;
        float m[WAVES], top = kMinusInf, weight = 0.0f;
        f32x4 sum = {0, 0, 0, 0};
#pragma unroll
        for (int n = 0; n < WAVES; ++n) {
            m[n] = n < parts ? top_s[n][c] : kMinusInf;
            top = fmaxf(top, m[n]);
        }
#pragma unroll
        for (int n = 0; n < WAVES; ++n) {
            if (n >= parts) continue;
            const float factor = __builtin_amdgcn_exp2f((m[n] - finite_max(top)) * a.scale_log2);
            sum += *reinterpret_cast<const f32x4 *>(&space_s.sum[n][c][e]) * factor;
            weight += weight_s[n][c] * factor;
        }
        sum *= q.length < 0 ? __builtin_nanf("") : weight == 0.0f ? 0.0f : 1.0f / weight;
        char *out = static_cast<char *>(a.out.data) + ((int64_t)(q.begin + r) * a.out.row + (kv * a.group + p - r * a.group) * a.out.head + e) * B;
        if constexpr (B == 2) *reinterpret_cast<u32x2 *>(out) = u32x2{TR::pack(sum.x, sum.y), TR::pack(sum.z, sum.w)};
        else *reinterpret_cast<f32x4 *>(out) = sum;
    }
}

template <typename TR, int DP, bool EXACT, int RT>
void launch_pairs(const AttendArgs &a, hipStream_t stream)
{
    const int32_t groups_log2 = a.groups_log2 - (kTreeGroups<Wave<TR, DP, EXACT>, RT> == 1 ? 1 : 0);   // what is on the GPU at once
    tree_kernel<TR, DP, EXACT, RT><<<1 << groups_log2, 64 * kWaves, 0, stream>>>(a, groups_log2);
    tree_join_kernel<TR, DP, RT><<<dim3(1 << groups_log2, 4 * RT), 256, 0, stream>>>(a, groups_log2);
}

// Keys that a sequence may have to read: all that the table has room for, or that a window has, where every row of the call counts as a key.  What the first kernel reads once for all pairs of a sequence,
// tree_whole_kernel reads for each 16, which pays where few rows leave the GPU to them.  bf16, 32 heads of 128 on 8, window of 256 and four first keys, us there and here: single rows of 256 sequences 79 and 56, of 384
// 123 and 91, 24 trees of 63 rows 137 and 74, 64 of 8 rows 48 and 26, 24 of 20 rows 50 and 51 (of heads of 64, 24 and 43; 16 heads of 256 on 2, 38 and 46); fp32, 16 heads of 128 on 4, 384 single rows 103 and 86.
int64_t room_of(const AttendArgs &a)
{
    const int64_t room = table_room(a.s), through = (int64_t)a.window + a.sinks + 32 + a.s.rows;
    return a.window && through < room ? through : room;
}

int64_t whole_tiles(const AttendArgs &a) { return (int64_t)a.s.rows * a.group / kHeadTile + a.s.batch; }

// Whether the keys of a tile are shared by the wavefronts of a workgroup, through LDS (prompt_tile.h), by the pairs of a sequence and a key head on average.  bf16, 32 heads of 128 on 8,
// us there and here: 24 sequences of 640 keys, 4 rows 24 and 26, 8 rows 24 and 38, 16 rows 25 and 46; of 2,560 keys 64, 64 and 66 beside 51, 62 and 77; of 8,192
// keys, 8 rows 209 and 181, 16 rows 210 and 180, 24 rows 211 and 320, 63 rows 295 and 596.  One sequence of 32,768 keys, 16 rows 82 and 61, 24 rows 82 and 73, 63 rows 113 and 109.  320 keys, by tree_whole_kernel: 8 sequences
// of 16 rows 16 and 13, 24 of 8 rows 16 and 21.  Heads of 64 and 256 go by the same numbers, which suit them less: of 64, 24 sequences of 8 rows behind 320 keys 23 and 12, behind 640 27 and 28, 16 rows behind 2,560
// 52 and 55, behind 8,192 144 and 114, 24 rows 144 and 172; of 256, 8 rows behind 320 keys 34 and 38, behind 640 55 and 53, 16 rows behind 2,560 190 and 300, behind 8,192 494 and 929, 63 rows 947 and 3,759.
bool through_lds(const AttendArgs &a, sc_dtype dtype)
{
    if (!a.tree || a.window || dtype == SC_F32) return false;
    const int64_t pairs = (int64_t)a.s.rows * a.group / a.s.batch, room = room_of(a);
    if (room <= kWholeKeys) return pairs >= 16 && whole_tiles(a) * a.kv_heads > a.n_cu;
    return pairs >= 96 || (pairs > 16 && room <= 4096 && (int64_t)a.s.batch * a.kv_heads >= a.n_cu / 2);
}

template <typename TR, int DP, bool EXACT>
void launch_exact(const AttendArgs &a, hipStream_t stream)
{
    const int64_t tiles = whole_tiles(a);
    if (room_of(a) <= kWholeKeys && tiles * a.kv_heads < 1 << 22) {
        tree_whole_kernel<TR, DP, EXACT><<<(uint32_t)(tiles * a.kv_heads), 64 * kWholeWaves<DP>, 0, stream>>>(a);
        return;
    }
    // Tiles of a workgroup: as many as a sequence has pairs for on average, and as its registers hold.
    constexpr int kMost = kTreeTiles<TR, DP>;
    const int64_t pairs = a.tree ? (int64_t)a.s.rows * a.group / a.s.batch : 1;
    if constexpr (kMost >= 4) {
        if (pairs > 32) return launch_pairs<TR, DP, EXACT, 4>(a, stream);
    }
    if constexpr (kMost >= 2) {
        if (pairs > 16) return launch_pairs<TR, DP, EXACT, 2>(a, stream);
    }
    launch_pairs<TR, DP, EXACT, 1>(a, stream);
}

template <typename TR, int DP>
void launch_padded(const AttendArgs &a, hipStream_t stream)
{
    if (a.head_dim == DP) launch_exact<TR, DP, true>(a, stream);
    else launch_exact<TR, DP, false>(a, stream);
}

template <typename TR>
void launch_typed(const AttendArgs &a, hipStream_t stream)
{
    const int dp = padded_dim(a.head_dim);
    if (dp == 64) launch_padded<TR, 64>(a, stream);
    else if (dp == 128) launch_padded<TR, 128>(a, stream);
    else launch_padded<TR, 256>(a, stream);
}

}  // namespace

size_t row_pieces(int head_dim, int groups_log2) { return sizeof(float) * 2 * ((size_t)1 << groups_log2) * piece_floats(padded_dim(head_dim)); }

// Four tiles of pairs: of heads of 128 for half as many workgroups.
size_t tree_pieces(int head_dim, int groups_log2)
{
    const int dp = padded_dim(head_dim);
    return row_pieces(head_dim, groups_log2) * (dp == 256 ? 1 : dp == 128 ? 2 : 4);
}

hipError_t launch_tree(const AttendArgs &a, sc_dtype dtype, hipStream_t stream)
{
    if (through_lds(a, dtype)) return launch_prompt_tree(a, dtype, stream);
    if (dtype == SC_BF16) launch_typed<Bf16>(a, stream);
    else if (dtype == SC_F16) launch_typed<F16>(a, stream);
    else launch_typed<F32>(a, stream);
    return hipGetLastError();
}

}  // namespace sck
