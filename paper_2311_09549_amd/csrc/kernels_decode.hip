// Decode: attention of one row per sequence over a paged cache.
//
// Every key and value is read once, for all the heads that share it, and little is computed on it: bound by memory, as long as the whole GPU
// reads.  Few sequences of very different lengths must not leave compute units idle, so the keys of all sequences and key heads are put in
// one line of units of 128 keys, and every workgroup takes an equal share of the line, by arithmetic on the lengths that are in device memory
// (nobody on the host knows them).  A share that ends inside a segment (one sequence, one tile of 16 heads of a key head) leaves its
// sums with their maximum and weight in the workspace, and a second kernel joins the pieces in order.
//
// 32 heads of 128 on 8: 64 sequences up to 8,191 keys, fp16, in 104 us (4.75 TB/s); 64 heads on 8, one sequence of 131,071 keys, bf16, in 100 us (5.4 TB/s; a large copy reaches
// 4.8).  The join is 7.5 us of either.  16 heads of 80 with keys of their own, 24 sequences up to 1,500, fp32: 35 us (2.6 TB/s).  Segments have 372 keys
// there and a workgroup two or three units, so that the largest share has 384 keys beside a mean of 279; the matrix pipes, with one column in
// sixteen of use, are busy a third of the time.
#include "attention_device.h"

namespace sck {

namespace {

constexpr int kWaves = 4;   // that join() takes
constexpr int64_t kWholeKeys = 512;

// A value that all lanes hold alike, in scalar registers: what follows from it is scalar too.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

// The line of units of the sequences, as a wavefront finds it: 64 sequences at a time, a lane each.  Units of 64 sequences are less than 2^31.
struct Line {
    const Sequences &s;
    int lane;
    int32_t mine, upto;    // units of sequence 64 chunk + lane, of it and those before it in the chunk
    int32_t chunk;
    int64_t before;        // units of the chunks before

    __device__ __forceinline__ void load(int32_t c)
    {
        chunk = c;
        const int32_t b = 64 * c + lane;
        mine = b < s.batch ? units_of(paged_length(s, b)) : 0;
        upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int32_t y = __shfl_up(upto, d);
            upto += lane >= d ? y : 0;
        }
    }
    __device__ __forceinline__ int32_t chunk_units() const { return __builtin_amdgcn_readlane(upto, 63); }
    // Units of all sequences.  One chunk stays loaded.
    __device__ __forceinline__ int64_t all()
    {
        int64_t n = 0;
        for (int32_t c = 0; 64 * c < s.batch; ++c) {
            load(c);
            n += chunk_units();
        }
        before = 0;
        if (s.batch > 64) load(0);
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
        ahead = before + __builtin_amdgcn_readlane(upto, at) - __builtin_amdgcn_readlane(mine, at);
        return 64 * chunk + at;
    }
    // Units of the sequences before b.
    __device__ __forceinline__ int64_t until(int32_t b)
    {
        while (chunk < b / 64) {
            before += chunk_units();
            load(chunk + 1);
        }
        return before + __builtin_amdgcn_readlane(upto, b % 64) - __builtin_amdgcn_readlane(mine, b % 64);
    }
};

template <typename TR, int DP, bool EXACT>
__global__ void __launch_bounds__(64 * kWaves, DP == 256 ? 1 : 2) decode_kernel(AttendArgs a)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, EPL = W::EPL;
    __shared__ typename Join<W>::Space join_s;
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int32_t segments = a.kv_heads * a.head_tiles;   // of a sequence
    Line line = {a.s, lane};
    const int64_t units = line.all() * segments;
    const int64_t share0 = share_begin(units, blockIdx.x, a.groups_log2), share1 = share_begin(units, blockIdx.x + 1, a.groups_log2);
    if (share0 >= share1) return;
    W w;
    // Units [u0, u1) of a segment: what is worked on at a time.
    struct Part {
        int64_t before;   // place in the line of the first unit of sequence b
        int32_t b, segment, length, n_units, u0, u1;
    };
    const auto upto = [&](Part &p, int64_t at) { p.u1 = (int32_t)(share1 - at < p.n_units - p.u0 ? p.u0 + (share1 - at) : p.n_units); };
    int64_t at = share0;
    Part part;
    part.b = line.find(quotient(at, segments), part.before);
    part.before *= segments;
    part.length = __builtin_amdgcn_readfirstlane(paged_length(a.s, part.b));
    part.n_units = units_of(part.length);
    part.segment = (int32_t)quotient(at - part.before, part.n_units);
    part.u0 = (int32_t)(at - part.before - (int64_t)part.segment * part.n_units);
    upto(part, at);

    const int64_t row_bytes = a.cache.row * B;
    constexpr int32_t STEP = kWaves * W::KEYS;
    const auto heads_of = [&](const Part &p) { const int32_t n = a.group - p.segment % a.head_tiles * kHeadTile; return n < kHeadTile ? n : kHeadTile; };
    const auto head_of = [&](const Part &p, int32_t heads) { return p.segment / a.head_tiles * a.group + p.segment % a.head_tiles * kHeadTile + (w.col < heads ? w.col : 0); };
    const auto end_of = [&](const Part &p) { return p.u1 == p.n_units ? p.length : p.u1 * kDecodeUnit; };
    // Keys of the next step are asked for when the scores have used this step's, values when the second product has: one of the two is always on its way.
    // Every step masks: the vector ALUs have time, and a second form of it would be as much code again, which a short call waits for.
    typename W::Keys keys;
    typename W::Values values;
    KeyTile t[TILES];
    bool bad = false;
    const auto find = [&](const Part &p, int32_t base) __attribute__((always_inline)) {
        const int32_t kv = p.segment / a.head_tiles;
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            int32_t key = base + 16 * n;
            if (key >= p.length) key = base;   // nothing of it is seen: any rows that are there
            t[n].last = p.length - 1 - key;
            int32_t page = page_of(a.s, p.b, key);
            bad |= page < 0;
            if (page < 0) page = 0;
            const int64_t off = (page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row + kv * a.cache.head) * B;
            t[n].k = static_cast<const char *>(a.cache.keys) + off;
            t[n].v = static_cast<const char *>(a.cache.values) + off;
        }
    };
    // Queries and the first step of a part.
    const auto ask = [&](const Part &p) __attribute__((always_inline)) {
        const int32_t heads = heads_of(p), base = p.u0 * kDecodeUnit + wave * W::KEYS;
        w.load_q(static_cast<const char *>(a.q.data) + (p.b * a.q.row + head_of(p, heads) * a.q.head) * B, w.col < heads);
        if (base < end_of(p)) {
            find(p, base);
            w.load_keys(keys, t, row_bytes);
            w.load_values(values, t, row_bytes);
        }
    };
    w.init(lane, a.head_dim);
    ask(part);
    while (true) {
        // the next part is known, and its queries and first keys asked for, before this one's wavefronts are joined
        const int64_t next_at = at + (part.u1 - part.u0);
        const bool again = next_at < share1;
        Part next = part;
        if (again) {
            next.u0 = 0;
            if (++next.segment == segments) {
                next.segment = 0;
                next.before = next_at;
                do next.length = __builtin_amdgcn_readfirstlane(paged_length(a.s, ++next.b)); while (units_of(next.length) == 0);   // share1 is not behind the last unit
                next.n_units = units_of(next.length);
            }
            upto(next, next_at);
        }
        const int32_t end = end_of(part);
        for (int32_t base = part.u0 * kDecodeUnit + wave * W::KEYS; base < end; base += STEP) {
            const bool more = base + STEP < end;
            typename W::Scores scores;
            w.scores(scores, keys);
            if (more) {
                find(part, base + STEP);
                w.load_keys(keys, t, row_bytes);
            }
            w.template add<true, true>(scores, values, a.scale_log2, part.length - base);
            if (more) w.load_values(values, t, row_bytes);
        }
        const float l = bad ? __builtin_nanf("") : over_groups_sum(w.l);
        bad = false;
        if (again) ask(next);
        float r[EPL], top, sum;
        Join<W>::run(w, join_s, wave, lane, l, a.scale_log2, r, top, sum);
        const int32_t heads = heads_of(part);
        if (part.u0 == 0 && part.u1 == part.n_units) {
            const float factor = sum == 0.0f ? 0.0f : 1.0f / sum;
            if (w.col < heads)
                Join<W>::template store<TR, EXACT>(w, r, wave, static_cast<char *>(a.out.data) + (part.b * a.out.row + head_of(part, heads) * a.out.head) * B, factor);
        } else {
            float *piece = a.pieces + (int64_t)piece_slot(part.before + (int64_t)part.segment * part.n_units, share0, blockIdx.x) * piece_floats(DP);
            if (w.col < heads) {
                const int e0 = (4 * w.g + wave) * EPL;
#pragma unroll
                for (int u = 0; u < EPL; u += 4) *reinterpret_cast<f32x4 *>(piece + w.col * DP + e0 + u) = f32x4{r[u], r[u + 1], r[u + 2], r[u + 3]};
                if (wave == 0 && w.g == 0) {
                    piece[kHeadTile * DP + w.col] = top;
                    piece[kHeadTile * (DP + 1) + w.col] = sum;
                }
            }
        }
        if (!again) break;
        w.init(lane, a.head_dim);
        part = next;
        at = next_at;
    }
}

// Few keys: a workgroup for each segment with as many wavefronts as LDS holds the sums of, so that most take one step.  What such a call waits for
// is a chain of reads, length and page number, then keys and values, and the page numbers of a wavefront's first step do not wait for the length.
template <int DP>
constexpr int kWholeWaves = DP == 256 ? 8 : 16;

template <typename TR, int DP, bool EXACT>
__global__ void __launch_bounds__(64 * kWholeWaves<DP>, kWholeWaves<DP> / 4) decode_whole_kernel(AttendArgs a)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, EPL = W::EPL, WAVES = kWholeWaves<DP>, LD = DP + 4;   // rows of sums begin in different banks
    __shared__ __attribute__((aligned(16))) float sum_s[WAVES][kHeadTile][LD];
    __shared__ float top_s[WAVES][kHeadTile], weight_s[WAVES][kHeadTile];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int32_t segments = a.kv_heads * a.head_tiles, b = blockIdx.x / segments, segment = blockIdx.x % segments;
    const int32_t kv = segment / a.head_tiles, head0 = segment % a.head_tiles * kHeadTile, heads = a.group - head0 < kHeadTile ? a.group - head0 : kHeadTile;
    const int64_t room = table_room(a.s);   // at most kWholeKeys
    constexpr int32_t STEP = WAVES * W::KEYS;
    int32_t base = wave * W::KEYS, page[TILES];
#pragma unroll
    for (int n = 0; n < TILES; ++n) page[n] = base + 16 * n < room ? page_of(a.s, b, base + 16 * n) : -1;
    const int32_t length = __builtin_amdgcn_readfirstlane(paged_length(a.s, b));
    W w;
    w.init(lane, a.head_dim);
    const int32_t head = kv * a.group + head0 + (w.col < heads ? w.col : 0);
    w.load_q(static_cast<const char *>(a.q.data) + (b * a.q.row + head * a.q.head) * B, w.col < heads);
    const char *k0 = static_cast<const char *>(a.cache.keys) + kv * a.cache.head * B, *v0 = static_cast<const char *>(a.cache.values) + kv * a.cache.head * B;
    const int64_t row_bytes = a.cache.row * B;
    bool bad = false;
    for (; base < length; base += STEP) {
        typename W::Keys keys;
        typename W::Values values;
        typename W::Scores scores;
        KeyTile t[TILES];
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            int32_t key = base + 16 * n, p = page[n];
            if (key >= length) {   // nothing of it is seen: any rows that are there
                key = base;
                p = page[0];
            }
            t[n].last = length - 1 - key;
            bad |= p < 0;
            if (p < 0) p = 0;
            const int64_t off = (p * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row) * B;
            t[n].k = k0 + off;
            t[n].v = v0 + off;
        }
        w.load_keys(keys, t, row_bytes);
        w.load_values(values, t, row_bytes);
#pragma unroll
        for (int n = 0; n < TILES; ++n) page[n] = base + STEP + 16 * n < length ? page_of(a.s, b, base + STEP + 16 * n) : -1;
        w.scores(scores, keys);
        w.template add<true, true>(scores, values, a.scale_log2, length - base);
    }
    const int parts = length <= 0 ? 0 : length > STEP - W::KEYS ? WAVES : (length - 1) / W::KEYS + 1;   // wavefronts that have had keys
    const float l = bad ? __builtin_nanf("") : over_groups_sum(w.l);
    if (wave < parts && w.col < heads) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int u = 0; u < EPL; u += 4)
                *reinterpret_cast<f32x4 *>(&sum_s[wave][w.col][(4 * w.g + i) * EPL + u]) = f32x4{w.o[u][i], w.o[u + 1][i], w.o[u + 2][i], w.o[u + 3][i]};
        if (w.g == 0) {
            top_s[wave][w.col] = w.m;
            weight_s[wave][w.col] = l;
        }
    }
    __syncthreads();
    for (int x = threadIdx.x; x < heads * (DP / 4); x += 64 * WAVES) {
        const int c = x / (DP / 4), e = x % (DP / 4) * 4;
        if (!EXACT && e >= a.head_dim) continue;
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
            sum += *reinterpret_cast<const f32x4 *>(&sum_s[n][c][e]) * factor;
            weight += weight_s[n][c] * factor;
        }
        sum *= length < 0 ? __builtin_nanf("") : weight == 0.0f ? 0.0f : 1.0f / weight;
        char *out = static_cast<char *>(a.out.data) + (b * a.out.row + (kv * a.group + head0 + c) * a.out.head + e) * B;
        if constexpr (B == 2) *reinterpret_cast<u32x2 *>(out) = u32x2{TR::pack(sum.x, sum.y), TR::pack(sum.z, sum.w)};
        else *reinterpret_cast<f32x4 *>(out) = sum;
    }
}

// Joins the pieces of one row, in the order of the line, and gives rows that no workgroup had (no keys, or a wrong length) their value.
template <typename TR, int DP>
__global__ void __launch_bounds__(256) decode_join_kernel(AttendArgs a)
{
    constexpr int B = TR::kBytes, LANES = DP / 4, PARTS = 256 / LANES;
    __shared__ f32x4 sum_s[PARTS][LANES];
    __shared__ float weight_s[PARTS], top_s[4], factor_s[1 << kMaxGroupsLog2], total_s[1 << kMaxGroupsLog2];
    constexpr float kNoPiece = -1.0f;   // no sum of weights.  Pieces of weights 0 are added: infinite values reach their row from them as well
    const int32_t b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x % 64;
    const int part = threadIdx.x / LANES, e = threadIdx.x % LANES * 4;
    const int32_t length = paged_length(a.s, b), n_units = units_of(length);
    char *out = static_cast<char *>(a.out.data) + (b * a.out.row + head * a.out.head + e) * B;
    f32x4 sum = {0, 0, 0, 0};
    float weight = 0.0f;
    if (n_units) {
        const int32_t segments = a.kv_heads * a.head_tiles, tile = head % a.group / kHeadTile, col = head % a.group % kHeadTile;
        const int32_t segment = head / a.group * a.head_tiles + tile;
        Line line = {a.s, lane};
        const int64_t units = line.all() * segments, first = line.until(b) * segments + (int64_t)segment * n_units;
        const int32_t w0 = share_of(units, first, a.groups_log2), w1 = share_of(units, first + n_units - 1, a.groups_log2);
        if (w0 == w1) return;   // whole in one workgroup, which has stored it
        float top = kMinusInf;
        // several workgroups have no units where there are fewer of those: they have no piece either
        for (int32_t w = w0 + threadIdx.x; w <= w1; w += 256) {
            const int64_t share0 = share_begin(units, w, a.groups_log2);
            const bool none = share0 == share_begin(units, w + 1, a.groups_log2);
            const int64_t at = (int64_t)piece_slot(first, share0, w) * piece_floats(DP) + kHeadTile * DP + col;
            const float m = none ? kMinusInf : a.pieces[at];
            factor_s[w - w0] = m;
            total_s[w - w0] = none ? kNoPiece : a.pieces[at + kHeadTile];
            top = fmaxf(top, m);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        if (lane == 0) top_s[threadIdx.x / 64] = top;
        __syncthreads();
        top = finite_max(fmaxf(fmaxf(top_s[0], top_s[1]), fmaxf(top_s[2], top_s[3])));
#pragma unroll 4
        for (int32_t w = w0 + part; w <= w1; w += PARTS) {
            const float factor = __builtin_amdgcn_exp2f((factor_s[w - w0] - top) * a.scale_log2), total = total_s[w - w0];
            if (total == kNoPiece) continue;
            const float *piece = a.pieces + (int64_t)piece_slot(first, share_begin(units, w, a.groups_log2), w) * piece_floats(DP);
            sum += *reinterpret_cast<const f32x4 *>(piece + col * DP + e) * factor;
            weight += total * factor;
        }
        sum_s[part][threadIdx.x % LANES] = sum;
        if (e == 0) weight_s[part] = weight;
        __syncthreads();
        if (part != 0) return;
#pragma unroll
        for (int n = 1; n < PARTS; ++n) {
            sum += sum_s[n][threadIdx.x];
            weight += weight_s[n];
        }
    } else if (part != 0) {
        return;
    }
    const float factor = length < 0 ? __builtin_nanf("") : weight == 0.0f ? 0.0f : 1.0f / weight;
    sum *= factor;
    if (e < a.head_dim) {
        if constexpr (B == 2) *reinterpret_cast<u32x2 *>(out) = u32x2{TR::pack(sum.x, sum.y), TR::pack(sum.z, sum.w)};
        else *reinterpret_cast<f32x4 *>(out) = sum;
    }
}

template <typename TR, int DP, bool EXACT>
void launch_exact(const AttendArgs &a, hipStream_t stream)
{
    // Few keys: a workgroup for each segment does with them before shares are found and pieces joined.  bf16, 32 heads of 128 on 8, us here and with shares: one sequence
    // of 64 keys 4.3 and 8.1, of 333 7.2 and 11.6, of 512 8.7 and 12.5; 64 sequences of 512 25.9 and 28.2.  Lengths are in device memory: the most that the
    // table has room for decides, and a table for many more keys takes the longer way.
    if (table_room(a.s) <= kWholeKeys && (int64_t)a.s.batch * a.kv_heads * a.head_tiles < 1 << 22) {
        decode_whole_kernel<TR, DP, EXACT><<<a.s.batch * a.kv_heads * a.head_tiles, 64 * kWholeWaves<DP>, 0, stream>>>(a);
        return;
    }
    decode_kernel<TR, DP, EXACT><<<1 << a.groups_log2, 64 * kWaves, 0, stream>>>(a);
    decode_join_kernel<TR, DP><<<dim3(a.s.batch, a.heads), 256, 0, stream>>>(a);
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

hipError_t launch_decode(const AttendArgs &a, sc_dtype dtype, hipStream_t stream)
{
    if (dtype == SC_BF16) launch_typed<Bf16>(a, stream);
    else if (dtype == SC_F16) launch_typed<F16>(a, stream);
    else launch_typed<F32>(a, stream);
    return hipGetLastError();
}

}  // namespace sck
