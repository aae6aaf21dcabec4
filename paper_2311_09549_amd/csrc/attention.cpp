// Entry points of attention: checks of the arguments, then launches.  The kernels are in kernels_append.hip, kernels_prompt.hip and
// kernels_decode.hip.
#include "attention.h"

#include <algorithm>
#include <array>
#include <climits>
#include <cmath>
#include <cstdio>
#include <new>
#include <utility>

using namespace sck;

namespace {

int elem_size(sc_dtype t) { return t == SC_F32 ? 4 : 2; }

bool aligned(const sc_attention *at, const void *p, int64_t s0, int64_t s1, int64_t s2 = 0)
{
    const int64_t per16 = 16 / elem_size(at->dtype);
    return (uintptr_t)p % 16 == 0 && s0 % per16 == 0 && s1 % per16 == 0 && s2 % per16 == 0;
}

// Strides and counts are bounded so that no element's offset overflows 64 bits.
constexpr int64_t kMaxStride = (int64_t)1 << 36;
bool stride_ok(int64_t s) { return s >= 0 && s <= kMaxStride; }

sc_status check_rows(const sc_attention *at, const sc_rows_view *v, Rows &out)
{
    if (!v->data) return SC_ERR_NULL;
    if (!stride_ok(v->row_stride) || !stride_ok(v->head_stride)) return SC_ERR_BAD_DIMS;
    if (!aligned(at, v->data, v->row_stride, v->head_stride)) return SC_ERR_SHAPE_MISMATCH;
    out = {v->data, v->row_stride, v->head_stride};
    return SC_OK;
}

// Whether no two elements of a written view coincide: axis by axis from the smallest stride on, a stride has to pass what the axes
// before it reach.
bool disjoint(int64_t head_dim, std::array<std::pair<int64_t, int64_t>, 3> axes)   // {stride, count}
{
    std::sort(axes.begin(), axes.end());
    int64_t reach = head_dim;
    for (const auto &[stride, count] : axes) {
        if (count <= 1) continue;
        if (stride < reach || count - 1 > (INT64_MAX / 4 - reach) / stride) return false;
        reach += (count - 1) * stride;
    }
    return true;
}

bool written_ok(const Rows &r, int64_t rows, int32_t heads, int32_t head_dim) { return disjoint(head_dim, {{{r.row, rows}, {r.head, heads}, {0, 1}}}); }

sc_status check_cache(const sc_attention *at, const sc_cache_view *c, Sequences &s, Cache &out)
{
    if (!c->keys || !c->values) return SC_ERR_NULL;
    if (c->pages < 1 || c->pages > INT32_MAX) return SC_ERR_BAD_DIMS;
    if (!stride_ok(c->page_stride) || !stride_ok(c->row_stride) || !stride_ok(c->head_stride)) return SC_ERR_BAD_DIMS;
    if (!aligned(at, c->keys, c->page_stride, c->row_stride, c->head_stride) || (uintptr_t)c->values % 16) return SC_ERR_SHAPE_MISMATCH;
    if (!disjoint(at->head_dim, {{{c->page_stride, c->pages}, {c->row_stride, at->page_rows}, {c->head_stride, at->kv_heads}}})) return SC_ERR_SHAPE_MISMATCH;
    s.pages = (int32_t)c->pages;
    s.page_shift = at->page_shift;
    out = {c->keys, c->values, c->page_stride, c->row_stride, c->head_stride};
    return SC_OK;
}

sc_status check_sequences(const sc_sequence_view *v, bool paged, Sequences &s)
{
    s = {};
    if (v->batch < 0 || v->batch > kMaxBatch || v->rows < 0 || v->rows > kMaxRows) return SC_ERR_BAD_DIMS;
    if (!v->row_start && v->rows != v->batch) return SC_ERR_SHAPE_MISMATCH;
    if (paged) {
        if (v->batch > 0 && (!v->length || (!v->page && v->page_count != 0))) return SC_ERR_NULL;
        if (v->page_ld < 0 || v->page_ld > INT32_MAX || v->page_count < 0 || v->page_count > INT32_MAX) return SC_ERR_BAD_DIMS;
    } else if (v->length) {
        return SC_ERR_SHAPE_MISMATCH;   // packed keys: a sequence has as many as it has rows
    }
    s.batch = v->batch;
    s.rows = (int32_t)v->rows;
    s.row_start = v->row_start;
    s.length = v->length;
    s.page = v->page;
    s.page_ld = paged ? v->page_ld : 0;
    s.page_count = paged ? v->page_count : 0;
    return SC_OK;
}

#define SC_TRY(x)                          \
    do {                                   \
        const sc_status st_ = (x);         \
        if (st_ != SC_OK) return st_;      \
    } while (0)

sc_status launched(hipError_t e) { return e == hipSuccess ? SC_OK : SC_ERR_DEVICE; }

AttendArgs attend_args(const sc_attention *at)
{
    AttendArgs a = {};
    a.heads = at->heads;
    a.kv_heads = at->kv_heads;
    a.group = at->heads / at->kv_heads;
    a.head_dim = at->head_dim;
    a.causal = at->causal;
    a.scale_log2 = at->scale_log2;
    return a;
}

sc_status prompt_workspace_of(const sc_attention *at, void *workspace, size_t bytes, AttendArgs &a)
{
    a.n_cu = at->n_cu;
    if (!workspace || !at->prompt_ws_bytes) return SC_OK;
    if (bytes < at->prompt_ws_bytes) return SC_ERR_WORKSPACE_SMALL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    a.pieces = static_cast<float *>(workspace);
    a.cut = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + at->prompt_ws_bytes - 2 * prompt_shares(at->n_cu) * sizeof(int32_t));
    return SC_OK;
}

}  // namespace

extern "C" sc_status sc_attention_create(sc_attention **out, const sc_attention_desc *d)
{
    if (!out || !d) return SC_ERR_NULL;
    *out = nullptr;
    if (d->dtype != SC_BF16 && d->dtype != SC_F16 && d->dtype != SC_F32) return SC_ERR_BAD_DTYPE;
    if (d->heads < 1 || d->kv_heads < 1 || d->heads > 4096 || d->heads % d->kv_heads) return SC_ERR_BAD_DIMS;
    if (d->head_dim < 8 || d->head_dim > kMaxHeadDim || d->head_dim % 8) return SC_ERR_BAD_DIMS;
    if (d->page_rows < 16 || d->page_rows > 4096 || (d->page_rows & (d->page_rows - 1))) return SC_ERR_BAD_DIMS;
    const double scale = d->scale == 0.0f ? 1.0 / std::sqrt((double)d->head_dim) : (double)d->scale;
    const float scale_log2 = (float)(scale * 1.4426950408889634);   // 1 / ln 2
    if (!(scale > 0.0) || !std::isnormal(scale_log2)) return SC_ERR_BAD_DIMS;
    if (d->rotary_dim < 0 || d->rotary_dim > d->head_dim || d->rotary_dim % 2) return SC_ERR_BAD_DIMS;
    if (d->rotary_dim && !d->rotary_freq) return SC_ERR_NULL;
    for (int t = 0; t < d->rotary_dim / 2; ++t)
        if (!std::isfinite(d->rotary_freq[t])) return SC_ERR_BAD_DIMS;
    sc_attention *at = new (std::nothrow) sc_attention();
    if (!at) return SC_ERR_ALLOC;
    at->dtype = d->dtype;
    at->heads = d->heads;
    at->kv_heads = d->kv_heads;
    at->head_dim = d->head_dim;
    at->page_rows = d->page_rows;
    while ((1 << at->page_shift) < d->page_rows) ++at->page_shift;
    at->causal = d->causal != 0;
    at->scale_log2 = scale_log2;
    at->pairs = d->rotary_dim / 2;
    at->interleaved = d->rotary_interleaved != 0;
    for (int t = 0; t < at->pairs; ++t) at->turns[t] = d->rotary_freq[t] * 0.15915494309189535;   // 1 / (2 pi)
    at->n_cu = 256;
    int ndev = 0, dev = 0, cus = 0;
    if (hipGetDeviceCount(&ndev) == hipSuccess && ndev > 0 && hipGetDevice(&dev) == hipSuccess &&
        hipDeviceGetAttribute(&cus, hipDeviceAttributeMultiprocessorCount, dev) == hipSuccess && cus > 0) {
        at->n_cu = cus;
        at->has_device = true;
    } else {
        (void)hipGetLastError();
    }
    // workgroups of decode: the power of two from two a compute unit on (two wavefronts a SIMD are what its registers allow)
    while (at->groups_log2 < kMaxGroupsLog2 && (1 << at->groups_log2) < 2 * at->n_cu) ++at->groups_log2;
    at->ws_bytes = sizeof(float) * 2 * ((size_t)1 << at->groups_log2) * piece_floats(padded_dim(at->head_dim));
    at->prompt_ws_bytes = prompt_workspace(at->dtype, at->head_dim, at->n_cu);
    *out = at;
    return SC_OK;
}

extern "C" sc_status sc_attention_workspace_bytes(const sc_attention *at, size_t *bytes)
{
    if (!at || !bytes) return SC_ERR_NULL;
    *bytes = at->ws_bytes;
    return SC_OK;
}

extern "C" sc_status sc_attention_prompt_workspace_bytes(const sc_attention *at, size_t *bytes)
{
    if (!at || !bytes) return SC_ERR_NULL;
    *bytes = at->prompt_ws_bytes;
    return SC_OK;
}

extern "C" sc_status sc_attention_describe(const sc_attention *at, char *buf, size_t n)
{
    if (!at || !buf) return SC_ERR_NULL;
    if (n == 0) return SC_ERR_BAD_DIMS;
    const int e = elem_size(at->dtype), d = at->head_dim;
    snprintf(buf, n,
             "attention %s: heads %d, key heads %d, head_dim %d (kernels padded to %d), pages of %d rows, %s\n"
             "  A(i,l) = sum_j softmax_j(%g * sum_k X(i,k) Y(j,k)) Z(j,l)\n"
             "  append: rotates %d of %d elements (%s), moves %d bytes a row\n"
             "  prompt: %d flops per row and key, reads and writes %d bytes a row and %d bytes a key, %zu bytes of workspace\n"
             "  decode: %d flops and %d bytes a key, %d workgroups, %zu bytes of workspace\n",
             at->dtype == SC_F32 ? "f32" : at->dtype == SC_F16 ? "f16" : "bf16", at->heads, at->kv_heads, d, padded_dim(d), at->page_rows,
             at->causal ? "causal" : "not causal", at->scale_log2 * 0.6931471805599453, 2 * at->pairs, d,
             at->interleaved ? "adjacent pairs" : "pairs of halves", 2 * (at->heads + 2 * at->kv_heads) * d * e, 4 * at->heads * d, 2 * at->heads * d * e,
             2 * at->kv_heads * d * e, at->prompt_ws_bytes, 4 * at->heads * d, 2 * at->kv_heads * d * e, 1 << at->groups_log2, at->ws_bytes);
    return SC_OK;
}

extern "C" sc_status sc_attention_append(const sc_attention *at, const sc_sequence_view *sequences, const sc_rows_view *q, const sc_rows_view *k,
                                         const sc_rows_view *v, const sc_rows_view *q_out, const sc_cache_view *cache, void *hip_stream)
{
    if (!at || !sequences || !k || !v || !cache || !q != !q_out) return SC_ERR_NULL;
    AppendArgs a = {};
    SC_TRY(check_sequences(sequences, true, a.s));
    SC_TRY(check_cache(at, cache, a.s, a.cache));
    if (a.s.rows == 0 || a.s.batch == 0) return SC_OK;
    SC_TRY(check_rows(at, k, a.k));
    SC_TRY(check_rows(at, v, a.v));
    if (q) {
        SC_TRY(check_rows(at, q, a.q));
        SC_TRY(check_rows(at, q_out, a.q_out));
        if (!written_ok(a.q_out, a.s.rows, at->heads, at->head_dim)) return SC_ERR_SHAPE_MISMATCH;
        if (a.q.data == a.q_out.data && (a.q.row != a.q_out.row || a.q.head != a.q_out.head)) return SC_ERR_SHAPE_MISMATCH;
    }
    if (!at->has_device) return SC_ERR_DEVICE;
    a.heads = q ? at->heads : 0;
    a.kv_heads = at->kv_heads;
    a.head_dim = at->head_dim;
    a.pairs = at->pairs;
    a.interleaved = at->interleaved;
    for (int t = 0; t < at->pairs; ++t) a.turns[t] = at->turns[t];
    return launched(launch_append(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_prompt(const sc_attention *at, const sc_sequence_view *sequences, const sc_rows_view *q, const sc_rows_view *k,
                                         const sc_rows_view *v, const sc_rows_view *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!at || !sequences || !q || !k || !v || !out) return SC_ERR_NULL;
    AttendArgs a = attend_args(at);
    SC_TRY(check_sequences(sequences, false, a.s));
    if (a.s.rows == 0 || a.s.batch == 0) return SC_OK;
    SC_TRY(check_rows(at, q, a.q));
    SC_TRY(check_rows(at, k, a.k));
    SC_TRY(check_rows(at, v, a.v));
    SC_TRY(check_rows(at, out, a.out));
    if (!written_ok(a.out, a.s.rows, at->heads, at->head_dim)) return SC_ERR_SHAPE_MISMATCH;
    SC_TRY(prompt_workspace_of(at, workspace, workspace_bytes, a));
    if (!at->has_device) return SC_ERR_DEVICE;
    return launched(launch_prompt(a, at->dtype, false, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_prompt_paged(const sc_attention *at, const sc_sequence_view *sequences, const sc_rows_view *q,
                                               const sc_cache_view *cache, const sc_rows_view *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!at || !sequences || !q || !cache || !out) return SC_ERR_NULL;
    AttendArgs a = attend_args(at);
    SC_TRY(check_sequences(sequences, true, a.s));
    SC_TRY(check_cache(at, cache, a.s, a.cache));
    if (a.s.rows == 0 || a.s.batch == 0) return SC_OK;
    SC_TRY(check_rows(at, q, a.q));
    SC_TRY(check_rows(at, out, a.out));
    if (!written_ok(a.out, a.s.rows, at->heads, at->head_dim)) return SC_ERR_SHAPE_MISMATCH;
    SC_TRY(prompt_workspace_of(at, workspace, workspace_bytes, a));
    if (!at->has_device) return SC_ERR_DEVICE;
    return launched(launch_prompt(a, at->dtype, true, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_decode(const sc_attention *at, const sc_sequence_view *sequences, const sc_rows_view *q, const sc_cache_view *cache,
                                         const sc_rows_view *out, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!at || !sequences || !q || !cache || !out) return SC_ERR_NULL;
    AttendArgs a = attend_args(at);
    SC_TRY(check_sequences(sequences, true, a.s));
    if (sequences->row_start) return SC_ERR_SHAPE_MISMATCH;   // one row per sequence
    SC_TRY(check_cache(at, cache, a.s, a.cache));
    if (a.s.batch == 0) return SC_OK;
    SC_TRY(check_rows(at, q, a.q));
    SC_TRY(check_rows(at, out, a.out));
    if (!written_ok(a.out, a.s.rows, at->heads, at->head_dim)) return SC_ERR_SHAPE_MISMATCH;
    if (workspace_bytes < at->ws_bytes) return SC_ERR_WORKSPACE_SMALL;
    if (!workspace) return SC_ERR_NULL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    if (!at->has_device) return SC_ERR_DEVICE;
    a.groups_log2 = at->groups_log2;
    a.head_tiles = (a.group + kHeadTile - 1) / kHeadTile;
    if (units_of((int32_t)std::min<int64_t>(table_room(a.s), INT32_MAX)) * (int64_t)a.s.batch >= kMaxUnits / ((int64_t)a.kv_heads * a.head_tiles)) return SC_ERR_BAD_DIMS;
    a.pieces = static_cast<float *>(workspace);
    return launched(launch_decode(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_destroy(sc_attention *at)
{
    delete at;
    return SC_OK;
}
