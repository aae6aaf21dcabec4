// Decode: attention of one row per sequence over a paged cache.
//
// Every key and value is read once, for all the heads that share it, and little is computed on it: bound by memory, as long as the whole GPU
// reads.  Few sequences of very different lengths must not leave compute units idle, so the keys of all sequences and key heads are put in
// one line of units of 128 keys, and every workgroup takes an equal share of the line, by arithmetic on the lengths that are in device memory
// (nobody on the host knows them).  A share that ends inside a segment (one sequence, one tile of 16 heads of a key head) leaves its
// sums with their maximum and weight in the workspace, and a second kernel joins the pieces in order.
#include "attention_device.h"

namespace sck {

namespace {

constexpr int kWaves = 4;

// Sums over the wavefront's lanes of per-lane values, and places in the line; wave-uniform results.
__device__ __forceinline__ int64_t wave_sum(int64_t x)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) x += __shfl_xor(x, d);
    return x;
}

// A value that all lanes hold alike, in scalar registers: what follows from it is scalar too.
__device__ __forceinline__ int64_t uniform(int64_t x)
{
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), hi = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));
    return (int64_t)((uint64_t)hi << 32 | lo);
}

__device__ __forceinline__ int64_t units_in_all(const Sequences &s, int lane)
{
    int64_t n = 0;
    for (int32_t b = lane; b < s.batch; b += 64) n += units_of(paged_length(s, b));
    return uniform(wave_sum(n));
}

// Units of the sequences before b.
__device__ __forceinline__ int64_t units_before(const Sequences &s, int32_t b, int lane)
{
    int64_t n = 0;
    for (int32_t x = lane; x < b; x += 64) n += units_of(paged_length(s, x));
    return uniform(wave_sum(n));
}

// The sequence that has unit u of the line of sequences (0 <= u < all of them), and the units before it.
__device__ __forceinline__ int32_t sequence_at(const Sequences &s, int64_t u, int lane, int64_t &before)
{
    before = 0;
    for (int32_t b0 = 0; b0 < s.batch; b0 += 64) {
        const int64_t mine = b0 + lane < s.batch ? units_of(paged_length(s, b0 + lane)) : 0;
        int64_t upto = mine;
#pragma unroll
        for (int d = 1; d < 64; d *= 2) {
            const int64_t y = __shfl_up(upto, d);
            if (lane >= d) upto += y;
        }
        const uint64_t past = __ballot(before + upto > u);
        if (past) {
            const int at = __ffsll((unsigned long long)past) - 1;
            before += uniform(__shfl(upto - mine, at));
            return b0 + __builtin_amdgcn_readfirstlane(at);
        }
        before += uniform(__shfl(upto, 63));
    }
    return s.batch;
}

template <typename TR, int DP, bool EXACT>
__global__ void __launch_bounds__(64 * kWaves) decode_kernel(AttendArgs a)
{
    using W = Wave<TR, DP, EXACT>;
    constexpr int B = TR::kBytes, TILES = W::TILES, EPL = W::EPL;
    __shared__ float part_s[kWaves][kWaves - 1][64][EPL];   // [quarter of the rows][other wavefronts][lane]
    __shared__ float top_s[kWaves][16], sum_s[kWaves][16];
    const int lane = threadIdx.x % 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int32_t segments = a.kv_heads * a.head_tiles;   // of a sequence
    const int64_t units = units_in_all(a.s, lane) * segments;
    const int64_t share0 = share_begin(units, blockIdx.x, a.groups), share1 = share_begin(units, blockIdx.x + 1, a.groups);
    if (share0 >= share1) return;
    int64_t before;
    int32_t b = sequence_at(a.s, share0 / segments, lane, before);
    int64_t at = share0;   // place in the line
    before *= segments;    // of the first unit of sequence b
    W w;
    while (at < share1 && b < a.s.batch) {
        const int32_t length = paged_length(a.s, b), n_units = units_of(length);
        if (n_units == 0) {
            ++b;
            continue;
        }
        const int32_t segment = (int32_t)((at - before) / n_units), u0 = (int32_t)((at - before) % n_units);
        const int32_t u1 = (int32_t)(share1 - at < n_units - u0 ? u0 + (share1 - at) : n_units);
        const int32_t kv = segment / a.head_tiles, head0 = segment % a.head_tiles * kHeadTile, heads = a.group - head0 < kHeadTile ? a.group - head0 : kHeadTile;
        w.init(lane, a.head_dim);
        const int32_t head = kv * a.group + head0 + (w.col < heads ? w.col : 0);
        w.load_q(static_cast<const char *>(a.q.data) + (b * a.q.row + head * a.q.head) * B, w.col < heads);
        const char *k0 = static_cast<const char *>(a.cache.keys) + kv * a.cache.head * B, *v0 = static_cast<const char *>(a.cache.values) + kv * a.cache.head * B;
        const int64_t row_bytes = a.cache.row * B;
        const int32_t end = u1 * kDecodeUnit < length ? u1 * kDecodeUnit : length;
        bool bad = false;
        for (int32_t base = u0 * kDecodeUnit + wave * W::KEYS; base < end; base += kWaves * W::KEYS) {
            KeyTile t[TILES];
#pragma unroll
            for (int n = 0; n < TILES; ++n) {
                int32_t key = base + 16 * n;
                if (key >= length) key = base;   // nothing of it is seen: any rows that are there
                t[n].last = length - 1 - key;
                int32_t page = page_of(a.s, b, key);
                bad |= page < 0;
                if (page < 0) page = 0;
                const int64_t off = (page * a.cache.page + (key & ((1 << a.s.page_shift) - 1)) * a.cache.row) * B;
                t[n].k = k0 + off;
                t[n].v = v0 + off;
            }
            typename W::Keys keys;
            typename W::Values values;
            w.load_keys(keys, t, row_bytes);
            w.load_values(values, t, row_bytes);
            if (base + W::KEYS <= length) w.template step<false>(keys, values, a.scale_log2, 0);
            else w.template step<true>(keys, values, a.scale_log2, length - base);
        }

        // join the wavefronts: each sums the elements (4 g + wave) EPL + [0, EPL) of every row
        const float l = bad ? __builtin_nanf("") : over_groups_sum(w.l);
        if (w.g == 0) {
            top_s[wave][w.col] = w.m;
            sum_s[wave][w.col] = l;
        }
        __syncthreads();
        float top = kMinusInf, sum = 0.0f;
#pragma unroll
        for (int n = 0; n < kWaves; ++n) top = fmaxf(top, top_s[n][w.col]);
#pragma unroll
        for (int n = 0; n < kWaves; ++n) sum += sum_s[n][w.col] * __builtin_amdgcn_exp2f((top_s[n][w.col] - finite_max(top)) * a.scale_log2);
        const float mine = __builtin_amdgcn_exp2f((w.m - finite_max(top)) * a.scale_log2);
        float r[EPL];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i == wave) {
#pragma unroll
                for (int u = 0; u < EPL; ++u) r[u] = w.o[u][i] * mine;
            } else {
#pragma unroll
                for (int u = 0; u < EPL; ++u) part_s[i][wave - (wave > i)][lane][u] = w.o[u][i] * mine;
            }
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < kWaves - 1; ++n)
#pragma unroll
            for (int u = 0; u < EPL; ++u) r[u] += part_s[wave][n][lane][u];
        const int e0 = (4 * w.g + wave) * EPL;
        if (u0 == 0 && u1 == n_units) {
            const float factor = sum == 0.0f ? 0.0f : 1.0f / sum;
            char *out = static_cast<char *>(a.out.data) + (b * a.out.row + head * a.out.head + e0) * B;
            if (w.col < heads) {
#pragma unroll
                for (int u = 0; u < EPL; u += 4) {
                    if (!EXACT && e0 + u >= a.head_dim) break;
                    if constexpr (B == 2) *reinterpret_cast<u32x2 *>(out + u * B) = u32x2{TR::pack(r[u] * factor, r[u + 1] * factor), TR::pack(r[u + 2] * factor, r[u + 3] * factor)};
                    else *reinterpret_cast<f32x4 *>(out + u * B) = f32x4{r[u], r[u + 1], r[u + 2], r[u + 3]} * factor;
                }
            }
        } else {
            float *piece = a.pieces + (int64_t)piece_slot(before + (int64_t)segment * n_units, share0, blockIdx.x) * piece_floats(DP);
            if (w.col < heads) {
#pragma unroll
                for (int u = 0; u < EPL; u += 4) *reinterpret_cast<f32x4 *>(piece + w.col * DP + e0 + u) = f32x4{r[u], r[u + 1], r[u + 2], r[u + 3]};
                if (wave == 0 && w.g == 0) {
                    piece[kHeadTile * DP + w.col] = top;
                    piece[kHeadTile * (DP + 1) + w.col] = sum;
                }
            }
        }
        at += u1 - u0;
        if (segment == segments - 1 && u1 == n_units) {
            before += (int64_t)segments * n_units;
            ++b;
        }
    }
}

// Joins the pieces of one row, in the order of the line, and gives rows that no workgroup had (no keys, or a wrong length) their value.
template <typename TR, int DP>
__global__ void __launch_bounds__(256) decode_join_kernel(AttendArgs a)
{
    constexpr int B = TR::kBytes, LANES = DP / 4, PARTS = 256 / LANES;
    __shared__ f32x4 sum_s[PARTS][LANES];
    __shared__ float weight_s[PARTS];
    const int32_t b = blockIdx.x, head = blockIdx.y, lane = threadIdx.x % 64;
    const int part = threadIdx.x / LANES, e = threadIdx.x % LANES * 4;
    const int32_t length = paged_length(a.s, b), n_units = units_of(length);
    char *out = static_cast<char *>(a.out.data) + (b * a.out.row + head * a.out.head + e) * B;
    f32x4 sum = {0, 0, 0, 0};
    float weight = 0.0f;
    if (n_units) {
        const int32_t segments = a.kv_heads * a.head_tiles, tile = head % a.group / kHeadTile, col = head % a.group % kHeadTile;
        const int32_t segment = head / a.group * a.head_tiles + tile;
        const int64_t units = units_in_all(a.s, lane) * segments, first = units_before(a.s, b, lane) * segments + (int64_t)segment * n_units;
        const int32_t w0 = share_of(units, first, a.groups), w1 = share_of(units, first + n_units - 1, a.groups);
        if (w0 == w1) return;   // whole in one workgroup, which has stored it
        float top = kMinusInf;
        for (int32_t w = w0 + lane; w <= w1; w += 64) {
            // a workgroup that has no units has no piece
            if (share_begin(units, w, a.groups) == share_begin(units, w + 1, a.groups)) continue;
            top = fmaxf(top, a.pieces[(int64_t)piece_slot(first, share_begin(units, w, a.groups), w) * piece_floats(DP) + kHeadTile * DP + col]);
        }
#pragma unroll
        for (int d = 1; d < 64; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
        for (int32_t w = w0 + part; w <= w1; w += PARTS) {
            if (share_begin(units, w, a.groups) == share_begin(units, w + 1, a.groups)) continue;
            const float *piece = a.pieces + (int64_t)piece_slot(first, share_begin(units, w, a.groups), w) * piece_floats(DP);
            const float factor = __builtin_amdgcn_exp2f((piece[kHeadTile * DP + col] - finite_max(top)) * a.scale_log2);
            sum += *reinterpret_cast<const f32x4 *>(piece + col * DP + e) * factor;
            weight += piece[kHeadTile * (DP + 1) + col] * factor;
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

template <typename TR, int DP>
void launch_padded(const AttendArgs &a, hipStream_t stream)
{
    if (a.head_dim == DP) decode_kernel<TR, DP, true><<<a.groups, 64 * kWaves, 0, stream>>>(a);
    else decode_kernel<TR, DP, false><<<a.groups, 64 * kWaves, 0, stream>>>(a);
    decode_join_kernel<TR, DP><<<dim3(a.s.batch, a.heads), 256, 0, stream>>>(a);
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
