// Append: new rows of keys and values into the pages of their sequences, queries and keys rotated by their positions on the way.
//
// A row is moved once, heads + 2 kv_heads heads in and as many out, and pairs / head_dim of it turned: nothing but memory traffic, or,
// for the few rows of a decoding step, the latency of a launch and of three dependent reads (row start, length, page number).  A workgroup
// takes one row: all its heads turn by the same angles, so it takes their sines and cosines once, into LDS.
//
// 4,623 rows of 32 + 2 * 8 heads of 128, bf16, 64 elements rotated: 25 us, 4.5 TB/s, where a large copy reaches 4.8; 33 us with the row asked for after its place
// is known.  One row: 3.5 us, launch and chain of reads.
#include "attention.h"

namespace sck {

namespace {

constexpr int kAppendThreads = 256;
constexpr int kAhead = 3;   // pieces of a thread that are on their way before the row's place is known: the whole of 32 + 2 * 8 heads of 128, 16 bits

template <typename E, int N>
struct alignas(sizeof(E) * N < 16 ? sizeof(E) * N : 16) Vec {
    E v[N];
};

template <typename E, int N>
__device__ __forceinline__ Vec<E, N> load(const E *p) { return *reinterpret_cast<const Vec<E, N> *>(p); }
template <typename E, int N>
__device__ __forceinline__ void store(E *p, const Vec<E, N> &x) { *reinterpret_cast<Vec<E, N> *>(p) = x; }

// A thread's share of a row: a vector, or two of them half a rotation apart, on its way from the rows to queries or cache.
template <typename E, int N, bool INTERLEAVED>
struct Piece {
    Vec<E, N> v, w;
    int head, e;      // of queries, then keys, then values; first element (of the first vector)
    bool turned;

    // Piece x of a row: those of rotated heads first, with what is not rotated of them behind the pairs.
    __device__ __forceinline__ void read(const AppendArgs &a, int32_t row, int x, int n_rotated, int per_head, int whole, int pairs_of_vectors)
    {
        if (x >= n_rotated) {
            const int y = x - n_rotated, h = y / whole;
            head = a.heads + a.kv_heads + h;
            e = (y - h * whole) * N;
            turned = false;
            v = load<E, N>(static_cast<const E *>(a.v.data) + row * a.v.row + h * a.v.head + e);
            return;
        }
        head = x / per_head;
        const int y = x - head * per_head, h = head - a.heads;
        const E *src = head < a.heads ? static_cast<const E *>(a.q.data) + row * a.q.row + head * a.q.head : static_cast<const E *>(a.k.data) + row * a.k.row + h * a.k.head;
        if (INTERLEAVED) {
            e = y * N;
            turned = true;
        } else {
            turned = y < pairs_of_vectors;
            e = turned ? y * N : 2 * a.pairs + (y - pairs_of_vectors) * N;
            if (turned) w = load<E, N>(src + a.pairs + e);
        }
        v = load<E, N>(src + e);
    }

    // at: of the row in the cache, or negative for one that has no place.
    __device__ __forceinline__ void write(const AppendArgs &a, int32_t row, int64_t at, const float *cos_s, const float *sin_s)
    {
        if (INTERLEAVED && turned) {
#pragma unroll
            for (int i = 0; i < N; i += 2) {
                const int t = e / 2 + i / 2;
                if (t >= a.pairs) continue;
                const float c = cos_s[t], s = sin_s[t], p = (float)v.v[i], q = (float)v.v[i + 1];
                v.v[i] = (E)(p * c - q * s);
                v.v[i + 1] = (E)(q * c + p * s);
            }
        } else if (turned) {
#pragma unroll
            for (int i = 0; i < N; ++i) {
                const float c = cos_s[e + i], s = sin_s[e + i], p = (float)v.v[i], q = (float)w.v[i];
                v.v[i] = (E)(p * c - q * s);
                w.v[i] = (E)(q * c + p * s);
            }
        }
        if (head >= a.heads && at < 0) return;
        E *dst = head < a.heads ? static_cast<E *>(a.q_out.data) + row * a.q_out.row + head * a.q_out.head
                 : head < a.heads + a.kv_heads ? static_cast<E *>(a.cache.keys) + at + (head - a.heads) * a.cache.head
                                               : static_cast<E *>(a.cache.values) + at + (head - a.heads - a.kv_heads) * a.cache.head;
        store(dst + e, v);
        if (!INTERLEAVED && turned) store(dst + a.pairs + e, w);
    }
};

// E: element, N: elements of a vector; N divides the pairs of a row where its pairs are half a rotation apart, and whatever is not rotated.
template <typename E, int N, bool INTERLEAVED>
__global__ void __launch_bounds__(kAppendThreads) append_kernel(AppendArgs a)
{
    __shared__ float cos_s[kMaxPairs], sin_s[kMaxPairs];
    const int32_t row = blockIdx.x;
    // vectors of a rotated head: pairs of vectors half a rotation apart (or vectors of pairs), then the rest of the row
    const int turned = INTERLEAVED ? a.head_dim / N : a.pairs / N, plain = INTERLEAVED ? 0 : (a.head_dim - 2 * a.pairs) / N, per_head = turned + plain;
    const int whole = a.head_dim / N;
    const int n_rotated = (a.heads + a.kv_heads) * per_head, n = n_rotated + a.kv_heads * whole;

    // The row does not wait for its place: the first pieces are asked for before the tables are read.
    Piece<E, N, INTERLEAVED> piece[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
        const int x = threadIdx.x + i * kAppendThreads;
        if (x < n) piece[i].read(a, row, x, n_rotated, per_head, whole, turned);
    }
    const int32_t b = sequence_of(a.s, row);
    if (b < 0) return;
    const int32_t begin = row_begin(a.s, b), count = row_begin(a.s, b + 1) - begin;
    const int64_t position = (int64_t)a.s.length[b] - count + (row - begin);
    // row of the cache, or none
    int32_t page = -1;
    if (position >= 0 && position < table_room(a.s)) page = page_of(a.s, b, (int32_t)position);
    for (int t = threadIdx.x; t < a.pairs; t += kAppendThreads) {
        const double x = (double)position * a.turns[t];
        float c, s;
        sincospif(2.0f * (float)(x - rint(x)), &s, &c);
        cos_s[t] = c;
        sin_s[t] = s;
    }
    const int64_t at = page < 0 ? -1 : page * a.cache.page + ((int32_t)position & ((1 << a.s.page_shift) - 1)) * a.cache.row;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kAhead; ++i)
        if (threadIdx.x + i * kAppendThreads < n) piece[i].write(a, row, at, cos_s, sin_s);
    for (int x = threadIdx.x + kAhead * kAppendThreads; x < n; x += kAppendThreads) {
        piece[0].read(a, row, x, n_rotated, per_head, whole, turned);
        piece[0].write(a, row, at, cos_s, sin_s);
    }
}

template <typename E>
void launch_typed(const AppendArgs &a, hipStream_t stream)
{
    const int blocks = a.s.rows;
    // the widest vector that halves of a rotation and the rest of a row are whole numbers of
    if (a.interleaved) append_kernel<E, 8, true><<<blocks, kAppendThreads, 0, stream>>>(a);
    else if (a.pairs % 8 == 0) append_kernel<E, 8, false><<<blocks, kAppendThreads, 0, stream>>>(a);
    else if (a.pairs % 4 == 0) append_kernel<E, 4, false><<<blocks, kAppendThreads, 0, stream>>>(a);
    else if (a.pairs % 2 == 0) append_kernel<E, 2, false><<<blocks, kAppendThreads, 0, stream>>>(a);
    else append_kernel<E, 1, false><<<blocks, kAppendThreads, 0, stream>>>(a);
}

}  // namespace

hipError_t launch_append(const AppendArgs &a, sc_dtype dtype, hipStream_t stream)
{
    if (dtype == SC_BF16) launch_typed<__bf16>(a, stream);
    else if (dtype == SC_F16) launch_typed<_Float16>(a, stream);
    else launch_typed<float>(a, stream);
    return hipGetLastError();
}

}  // namespace sck
