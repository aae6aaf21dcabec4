// Device side of attention shared by its kernels: types, and one step of a wavefront, 16 query rows against 32 (16-bit types) or 16
// (fp32) keys, without LDS.
//
// Both products are taken transposed, on v_mfma 16x16: scores S^T = K Q^T (rows keys, columns queries) and O^T = V^T P^T (rows
// elements of a head, columns queries).  A lane (col = lane % 16, g = lane / 16) then holds the scores of query `col` with keys
// 16 t + 4 g + i, and sums of the same query: its maximum, sum and rescaling are one register each, and the scores it holds are,
// in the order it holds them, its operand of the second product.  The sum over keys may be taken in any order, so
// the values are put in that order too: a lane reads, of each of those keys, elements col * EPL .. + EPL - 1 of the row of
// values, 16 lanes a whole row.  Element u of what it read belongs to product number u, whose row m stands for
// element m * EPL + u of the head; pairs of keys are brought into one register by v_perm.  The sum over the elements of a head
// may be taken in any order as well, so 16-byte pieces of query and key rows are operands as they are read.
#pragma once

#include "attention.h"

namespace sck {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));

constexpr float kMinusInf = -__builtin_inff();

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
    using elem = __bf16;
    static constexpr int kBytes = 2, kTiles = 2;
    static constexpr uint32_t kExponent = 0x7f80u, kMantissa = 0x007fu, kOne = 0x3f80u;
    // Weights are 2^((score - maximum) * scale / ln 2 + kLift): no lift, bf16 has the exponents of fp32.
    static constexpr float kLift = 0.0f;
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const f32x2 f = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
    }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    }
};

struct F16 {
    using elem = _Float16;
    static constexpr int kBytes = 2, kTiles = 2;
    static constexpr uint32_t kExponent = 0x7c00u, kMantissa = 0x03ffu, kOne = 0x3c00u;
    // fp16 loses weights below 2^-24, which add up over a long row: with the largest weight at 2^14 they reach 2^-38 of it.
    static constexpr float kLift = 14.0f;
    static __device__ __forceinline__ uint32_t pack(float a, float b)
    {
        const f32x2 f = {a, b};
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, f16x2));
    }
    static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(u32x4 a, u32x4 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    }
};

struct F32 {
    using elem = float;
    static constexpr int kBytes = 4, kTiles = 1;
    static constexpr uint32_t kExponent = 0x7f800000u, kMantissa = 0x007fffffu, kOne = 0x3f800000u;
    static constexpr float kLift = 0.0f;
    static __device__ __forceinline__ f32x4 mfma(uint32_t a, uint32_t b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b), c, 0, 0, 0);
    }
};

// Maximum / sum over the four lanes that hold one query.
__device__ __forceinline__ float over_groups_max(float x)
{
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float over_groups_sum(float x)
{
    x += __shfl_xor(x, 16);
    return x + __shfl_xor(x, 32);
}

// A maximum of -infinity (no key yet, or scores of -infinity alone) is taken as 0 in differences: weights 0 instead of NaN.
__device__ __forceinline__ float finite_max(float m) { return m == kMinusInf ? 0.0f : m; }

// Of 16 bits those below x.
__device__ __forceinline__ uint32_t below(int32_t x) { return x <= 0 ? 0u : x >= 16 ? 0xffffu : (1u << x) - 1; }

// Page of key j of sequence b, as page_of, for a sequence and a key that all lanes have alike: read by the scalar unit, whose wait is not one for the vector loads on
// their way.
__device__ __forceinline__ int32_t page_of_all(const Sequences &s, int32_t b, int32_t j)
{
    const int64_t at = (int64_t)__builtin_amdgcn_readfirstlane(b) * s.page_ld + (__builtin_amdgcn_readfirstlane(j) >> s.page_shift);
    const int32_t p = ((const __attribute__((address_space(4))) int32_t *)(uintptr_t)s.page)[at];
    return (uint32_t)p < (uint32_t)s.pages ? p : -1;
}

// Where 16 keys lie (wave-uniform): first rows of keys and values for the lane's head, and the last key of the tile that may be read (0..15).
struct KeyTile {
    const char *k, *v;
    int last;
};

// Infinities and NaN among the elements of a word, both halves of it (16-bit types) at a time.
template <typename TR>
struct Special {
    static constexpr int B = TR::kBytes;
    static constexpr uint32_t both(uint32_t x) { return B == 2 ? x * 0x10001u : x; }
    static constexpr int kTop = 8 * B - 1;   // sign bit of an element
    static __device__ __forceinline__ uint32_t infinite_or_nan(uint32_t x)   // 1 in each element that is
    {
        constexpr uint32_t lowest = TR::kMantissa + 1;   // of the exponent's bits: all of them set carry into the sign's
        return ((x & both(TR::kExponent)) + both(lowest)) >> kTop & both(1);
    }
    static __device__ __forceinline__ uint32_t indicator(uint32_t x, int kind)   // 1.0 in each element of that kind
    {
        const uint32_t out = infinite_or_nan(x), negative = x >> kTop & both(1);
        uint32_t nan = ((x & both(TR::kMantissa)) + both(TR::kMantissa)) & both(TR::kMantissa + 1);   // a mantissa that is not 0 carries
        nan = nan >> (__builtin_ctz(TR::kMantissa + 1)) & out;
        return (kind == 0 ? out & ~nan & ~negative : kind == 1 ? out & ~nan & negative : nan) * TR::kOne;
    }
    static __device__ __forceinline__ uint32_t without(uint32_t x) { return x & ~(infinite_or_nan(x) * (B == 2 ? 0xffffu : 0xffffffffu)); }   // 0 in their place
};

// Wave's state for 16 query rows.  DP: head_dim padded (64, 128, 256); EXACT: head_dim == DP.
template <typename TR, int DP, bool EXACT>
struct Wave {
    static constexpr int B = TR::kBytes, TILES = TR::kTiles, KEYS = 16 * TILES;
    static constexpr int EPL = DP / 16;               // elements of a row of values that a lane reads
    static constexpr int QC = DP * B / 64;            // 16-byte pieces of a query or key row that a lane reads
    static constexpr int VW = EPL * B / 4;            // words of a row of values that a lane reads

    u32x4 q[QC];
    f32x4 o[EPL];
    float m, l;      // maximum (of the scores before the scale) and sum of weights of the lane's query; l of this lane's keys alone

    int col, g, head_dim;

    __device__ __forceinline__ void init(int lane, int hd)
    {
        col = lane % 16;
        g = lane / 16;
        head_dim = hd;
        m = kMinusInf;
        l = 0.0f;
#pragma unroll
        for (int u = 0; u < EPL; ++u) o[u] = f32x4{0, 0, 0, 0};
    }

    // First element of the lane's piece c of a query or key row.
    __device__ __forceinline__ int piece(int c) const { return (c * 4 + g) * (16 / B); }

    __device__ __forceinline__ void load_q(const void *row, bool valid)
    {
#pragma unroll
        for (int c = 0; c < QC; ++c) {
            q[c] = u32x4{0, 0, 0, 0};
            if (valid && (EXACT || piece(c) < head_dim)) q[c] = *reinterpret_cast<const u32x4 *>(static_cast<const char *>(row) + piece(c) * B);
        }
    }

    struct Keys { u32x4 k[TILES][QC]; };
    struct Values { uint32_t v[TILES * 4][VW]; };

    // Piece rows of keys 16 t + col.
    __device__ __forceinline__ void load_keys(Keys &x, const KeyTile (&t)[TILES], int64_t row_bytes) const
    {
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            const char *p = t[n].k + (col < t[n].last ? col : t[n].last) * row_bytes;
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                x.k[n][c] = u32x4{0, 0, 0, 0};
                if (EXACT || piece(c) < head_dim) x.k[n][c] = *reinterpret_cast<const u32x4 *>(p + piece(c) * B);
            }
        }
    }

    __device__ __forceinline__ void load_values(Values &x, const KeyTile (&t)[TILES], int64_t row_bytes) const
    {
#pragma unroll
        for (int n = 0; n < TILES; ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 4 * g + i;
                const char *p = t[n].v + (r < t[n].last ? r : t[n].last) * row_bytes + col * EPL * B;
                uint32_t(&w)[VW] = x.v[n * 4 + i];
                if constexpr (VW == 2) {
                    u32x2 y = {0, 0};
                    if (EXACT || col * EPL < head_dim) y = *reinterpret_cast<const u32x2 *>(p);
                    w[0] = y.x;
                    w[1] = y.y;
                } else {
#pragma unroll
                    for (int b = 0; b < VW / 4; ++b) {
                        u32x4 y = {0, 0, 0, 0};
                        if (EXACT || col * EPL + b * (16 / B) < head_dim) y = *reinterpret_cast<const u32x4 *>(p + 16 * b);
                        w[4 * b] = y.x;
                        w[4 * b + 1] = y.y;
                        w[4 * b + 2] = y.z;
                        w[4 * b + 3] = y.w;
                    }
                }
            }
    }

    // The lane's operand of product u from rows of values (16-bit types: 8 keys).
    static __device__ __forceinline__ u32x4 operand(const Values &x, int u)
    {
        const uint32_t sel = u % 2 ? 0x07060302u : 0x05040100u;
        u32x4 a;
#pragma unroll
        for (int p = 0; p < 4; ++p) a[p] = __builtin_amdgcn_perm(x.v[2 * p + 1][u / 2], x.v[2 * p][u / 2], sel);
        return a;
    }

    // o += V^T P^T for the weights p of the lane's keys.  16-bit types: the product takes both operands in the type of the values, so weights are rounded to it here, by half a step of
    // each at most; their sums are of the fp32 ones.
    __device__ __forceinline__ void add_values(const Values &x, const float (&p)[TILES * 4])
    {
        if constexpr (B == 2) {
            const u32x4 w = {TR::pack(p[0], p[1]), TR::pack(p[2], p[3]), TR::pack(p[4], p[5]), TR::pack(p[6], p[7])};
#pragma unroll
            for (int u = 0; u < EPL; ++u) o[u] = TR::mfma(operand(x, u), w, o[u]);
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int u = 0; u < EPL; ++u) o[u] = TR::mfma(x.v[i][u], __builtin_bit_cast(uint32_t, p[i]), o[u]);
        }
    }

    static __device__ __forceinline__ bool any_special(const Values &x)
    {
        uint32_t any = 0;
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j)
#pragma unroll
            for (int w = 0; w < VW; ++w) any |= Special<TR>::infinite_or_nan(x.v[j][w]);
        return __any(any != 0);
    }

    // Infinities and NaN among values that some query of the step does not see: the product would spread them to it (0 times infinity).
    // They are taken out of x; queries that see one get it from a product of indicators, one for each of +infinity, -infinity, NaN.
    __device__ __forceinline__ void part_infinities(Values &x, int visible)
    {
        if (!any_special(x)) return;
        const f32x4 none = {0, 0, 0, 0};
        uint32_t one[TILES * 4];
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) one[j] = j / 4 * 16 + 4 * g + j % 4 < visible ? TR::kOne : 0u;
        fresh(x);
#pragma unroll
        for (int u = 0; u < EPL; ++u) {
            u32x4 y = {0, 0, 0, 0};
            if constexpr (B == 2) {
                y = operand(x, u);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = x.v[j][u];
            }
#pragma unroll
            for (int kind = 0; kind < 3; ++kind) {
                f32x4 n = none;
                u32x4 is;
#pragma unroll
                for (int h = 0; h < 4; ++h) is[h] = Special<TR>::indicator(y[h], kind);
                if constexpr (B == 2) {
                    n = TR::mfma(is, u32x4{one[0] | one[1] << 16, one[2] | one[3] << 16, one[4] | one[5] << 16, one[6] | one[7] << 16}, none);
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j) n = TR::mfma(is[j], one[j], n);
                }
                const float give = kind == 0 ? -kMinusInf : kind == 1 ? kMinusInf : __builtin_nanf("");
#pragma unroll
                for (int i = 0; i < 4; ++i) o[u][i] += n[i] > 0.0f ? give : 0.0f;
            }
            __builtin_amdgcn_sched_barrier(0);   // one at a time: side by side they would take the registers of the main loop
        }
        fresh(x);
        without_infinities(x);
    }
    static __device__ __forceinline__ void without_infinities(Values &x)
    {
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j)
#pragma unroll
            for (int w = 0; w < VW; ++w) x.v[j][w] = Special<TR>::without(x.v[j][w]);
    }
    // What was computed from x before is not kept for later.
    static __device__ __forceinline__ void fresh(Values &x)
    {
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j)
#pragma unroll
            for (int w = 0; w < VW; ++w) asm volatile("" : "+v"(x.v[j][w]));
    }

    // Values of keys that no query of the step sees, all of which see the first `visible`, become 0.
    __device__ __forceinline__ void hide(Values &x, int visible) const
    {
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j)
#pragma unroll
            for (int w = 0; w < VW; ++w) x.v[j][w] = j / 4 * 16 + 4 * g + j % 4 < visible ? x.v[j][w] : 0u;
    }

    struct Scores { f32x4 s[TILES]; };

    // TRIM: without the products of pieces behind the head, by a branch that all lanes take alike.
    template <bool TRIM = false>
    __device__ __forceinline__ void scores(Scores &x, const Keys &k) const
    {
#pragma unroll
        for (int n = 0; n < TILES; ++n) {
            x.s[n] = f32x4{0, 0, 0, 0};
#pragma unroll
            for (int c = 0; c < QC; ++c) {
                if (TRIM && !EXACT && c >= QC / 2 && c * (64 / B) >= head_dim) continue;   // more than half of DP is head
                if constexpr (B == 2) {
                    x.s[n] = TR::mfma(k.k[n][c], q[c], x.s[n]);
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) x.s[n] = TR::mfma(k.k[n][c][e], q[c][e], x.s[n]);
                }
            }
        }
    }

    // The rest of a step: scores of keys of which the lane's query sees the first `visible` (MASK; ALIKE: as every query does), running maximum and sum,
    // second product.
    template <bool MASK, bool ALIKE = false>
    __device__ __forceinline__ void add(const Scores &x, Values &v, float scale_log2, int visible)
    {
        const f32x4(&s)[TILES] = x.s;
        float p[TILES * 4], top = kMinusInf;
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) {
            p[j] = s[j / 4][j % 4];
            if (MASK) p[j] = j / 4 * 16 + 4 * g + j % 4 < visible ? p[j] : kMinusInf;
            top = fmaxf(top, p[j]);
        }
        const float next = fmaxf(m, over_groups_max(top));
        // the difference first: no score times the scale is beyond fp32, and close scores lose nothing
        const float from = finite_max(next), shrink = __builtin_amdgcn_exp2f((m - from) * scale_log2);
        m = next;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) {
            p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[j] - from, scale_log2, TR::kLift));
            sum += p[j];
        }
        l = l * shrink + sum;
#pragma unroll
        for (int u = 0; u < EPL; ++u) o[u] *= shrink;
        if (MASK && ALIKE) hide(v, visible);
        else if (MASK) part_infinities(v, visible);
        add_values(v, p);
    }

    // Adds the infinities and NaN of a row of values that the lane's query sees.
    __device__ __forceinline__ void add_special(const char *row)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int u = 0; u < EPL; ++u) {
                const int e = (4 * g + i) * EPL + u;
                if (!EXACT && e >= head_dim) continue;
                const typename TR::elem x = reinterpret_cast<const typename TR::elem *>(row)[e];
                if (!(__builtin_fabsf((float)x) < -kMinusInf)) o[u][i] += (float)x;
            }
    }

    // Bit of the lane's j-th key among bits of the step's keys, shifted by 4 g.
    static constexpr int seen_bit(int j) { return j / 4 * 16 + j % 4; }

    // Scores of keys whose bits are not set become -infinity.
    static __device__ __forceinline__ void mask(Scores &x, uint32_t seen)
    {
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) x.s[j / 4][j % 4] = seen >> seen_bit(j) & 1 ? x.s[j / 4][j % 4] : kMinusInf;
    }

    // The rest of a step for scores that have been masked, if they had to be, and values of which those that a query does not see are finite.
    __device__ __forceinline__ void add_seen(const Scores &x, const Values &v, float scale_log2)
    {
        float p[TILES * 4], top = kMinusInf;
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) {
            p[j] = x.s[j / 4][j % 4];
            top = fmaxf(top, p[j]);
        }
        const float next = fmaxf(m, over_groups_max(top));
        const float from = finite_max(next), shrink = __builtin_amdgcn_exp2f((m - from) * scale_log2);
        m = next;
        float sum = 0.0f;
#pragma unroll
        for (int j = 0; j < TILES * 4; ++j) {
            p[j] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[j] - from, scale_log2, TR::kLift));
            sum += p[j];
        }
        l = l * shrink + sum;
#pragma unroll
        for (int u = 0; u < EPL; ++u) o[u] *= shrink;
        add_values(v, p);
    }

    // The lane's sums are elements 4 g EPL + [0, 4 EPL) of query `col`, in the order o[0][0], o[1][0], .., o[0][1], ..
    __device__ __forceinline__ float sum_at(int e) const { return o[e % EPL][e / EPL]; }

    // Stores the row of query `col`, sums times `factor`.
    __device__ __forceinline__ void store(void *row, float factor) const
    {
#pragma unroll
        for (int e = 0; e < 4 * EPL; e += 16 / B) {
            const int at = 4 * g * EPL + e;
            u32x4 y;
            if constexpr (B == 2) {
#pragma unroll
                for (int w = 0; w < 4; ++w) y[w] = TR::pack(sum_at(e + 2 * w) * factor, sum_at(e + 2 * w + 1) * factor);
            } else {
#pragma unroll
                for (int w = 0; w < 4; ++w) y[w] = __builtin_bit_cast(uint32_t, sum_at(e + w) * factor);
            }
            if (EXACT || at < head_dim) *reinterpret_cast<u32x4 *>(static_cast<char *>(row) + at * B) = y;
        }
    }
};

// Join of four wavefronts that have had different keys of the same queries: each is left with the sums of a quarter of every row, elements
// (4 g + wave) EPL + [0, EPL) of query `col`, and with the maximum and sum of weights of the whole.
template <typename W>
struct Join {
    static constexpr int WAVES = 4, EPL = W::EPL;
    struct Space {
        alignas(16) float part[WAVES][WAVES - 1][64][EPL];   // [quarter][other wavefronts][lane]
        float top[WAVES][16], sum[WAVES][16];
    };

    // l: sum of weights of the wavefront, over its lanes.  Space may be used again after the next barrier.
    static __device__ __forceinline__ void run(const W &w, Space &space, int wave, int lane, float l, float scale_log2, float (&r)[EPL], float &top, float &sum)
    {
        if (w.g == 0) {
            space.top[wave][w.col] = w.m;
            space.sum[wave][w.col] = l;
        }
        __syncthreads();
        top = kMinusInf;
        sum = 0.0f;
#pragma unroll
        for (int n = 0; n < WAVES; ++n) top = fmaxf(top, space.top[n][w.col]);
#pragma unroll
        for (int n = 0; n < WAVES; ++n) sum += space.sum[n][w.col] * __builtin_amdgcn_exp2f((space.top[n][w.col] - finite_max(top)) * scale_log2);
        const float mine = __builtin_amdgcn_exp2f((w.m - finite_max(top)) * scale_log2);
        // (r apart from the stores: one store to either place would keep it out of registers)
#pragma unroll
        for (int u = 0; u < EPL; ++u) r[u] = (wave == 0 ? w.o[u][0] : wave == 1 ? w.o[u][1] : wave == 2 ? w.o[u][2] : w.o[u][3]) * mine;
#pragma unroll
        for (int i = 0; i < WAVES; ++i)
            if (i != wave) {
#pragma unroll
                for (int u = 0; u < EPL; u += 4)
                    *reinterpret_cast<f32x4 *>(&space.part[i][wave - (wave > i)][lane][u]) = f32x4{w.o[u][i], w.o[u + 1][i], w.o[u + 2][i], w.o[u + 3][i]} * mine;
            }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < WAVES - 1; ++n)
#pragma unroll
            for (int u = 0; u < EPL; ++u) r[u] += space.part[wave][n][lane][u];
    }

    // Stores the quarter in the row `out`, times `factor`.
    template <typename TR, bool EXACT>
    static __device__ __forceinline__ void store(const W &w, const float (&r)[EPL], int wave, char *out, float factor)
    {
        const int e0 = (4 * w.g + wave) * EPL;
#pragma unroll
        for (int u = 0; u < EPL; u += 4) {
            if (!EXACT && e0 + u >= w.head_dim) break;
            char *at = out + (e0 + u) * TR::kBytes;
            if constexpr (TR::kBytes == 2) *reinterpret_cast<u32x2 *>(at) = u32x2{TR::pack(r[u] * factor, r[u + 1] * factor), TR::pack(r[u + 2] * factor, r[u + 3] * factor)};
            else *reinterpret_cast<f32x4 *>(at) = f32x4{r[u], r[u + 1], r[u + 2], r[u + 3]} * factor;
        }
    }
};

}  // namespace sck
