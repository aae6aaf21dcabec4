// Entry points of attention: checks of the arguments, then launches.  The kernels are in kernels_append.hip, kernels_prompt.hip,
// kernels_decode.hip, kernels_tree.hip (trees, and single rows through a window) and kernels_pages.hip.
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
    a.groups_log2 = at->groups_log2;
    a.n_cu = at->n_cu;
    a.window = at->window;
    a.sinks = at->sinks;
    return a;
}

sc_status prompt_workspace_of(const sc_attention *at, void *workspace, size_t bytes, AttendArgs &a)
{
    if (!workspace || !at->prompt_ws_bytes) return SC_OK;
    if (bytes < at->prompt_ws_bytes) return SC_ERR_WORKSPACE_SMALL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    a.pieces = static_cast<float *>(workspace);
    a.cut = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + at->prompt_ws_bytes - 2 * prompt_shares(at->n_cu) * sizeof(int32_t));
    return SC_OK;
}

// Whether the line of units of trees stays below what its arithmetic takes, whatever the lengths and row starts: as many units as the table has room for, and tiles of one
// sequence as for all rows.
bool tree_line_ok(const AttendArgs &a)
{
    if (a.tree && a.s.rows * (int64_t)a.group > (int64_t)1 << 30) return false;   // pairs of a sequence are numbered in 32 bits
    const double units = 1.0 + (double)units_of((int32_t)std::min<int64_t>(table_room(a.s), kMaxKeys));
    const double tiles = 1.0 + (double)(a.tree ? a.s.rows : 1) * a.group / kHeadTile;
    return units * tiles * a.kv_heads * a.s.batch < (double)kMaxUnits;
}

// Ranges of 32-bit numbers.
bool overlap(const int32_t *p, int64_t n, const int32_t *q, int64_t m) { return p && q && n > 0 && m > 0 && (uintptr_t)p < (uintptr_t)(q + m) && (uintptr_t)q < (uintptr_t)(p + n); }

int64_t table_numbers(int32_t batch, int64_t ld, int64_t columns) { return batch > 0 && columns > 0 ? (batch - 1) * ld + columns : 0; }

// What fork and compact share.
sc_status check_pages(const sc_attention *at, const sc_pages_view *v, int32_t new_batch, int64_t moves)
{
    if (v->batch < 0 || v->batch > kMaxBatch || new_batch < 0 || new_batch > kMaxBatch) return SC_ERR_BAD_DIMS;
    if (v->pages < 1 || v->pages > kMaxPages || v->page_count < 0 || v->page_count > kMaxKeys / 16) return SC_ERR_BAD_DIMS;
    if (v->page_ld < 0 || v->page_ld > INT32_MAX || v->page_out_ld < 0 || v->page_out_ld > INT32_MAX) return SC_ERR_BAD_DIMS;
    if (new_batch > 1 && v->page_out_ld < v->page_count) return SC_ERR_SHAPE_MISMATCH;   // rows that are written do not coincide
    if (!v->holders || !v->holders_out || (moves > 0 && !v->moves)) return SC_ERR_NULL;
    if (v->batch > 0 && (!v->length || (v->page_count > 0 && !v->page))) return SC_ERR_NULL;
    if (new_batch > 0 && v->page_count > 0 && !v->page_out) return SC_ERR_NULL;
    const int64_t in = table_numbers(v->batch, v->page_ld, v->page_count), out = table_numbers(new_batch, v->page_out_ld, v->page_count);
    // what is written is apart from what is read and from the rest that is written, but for holders, and the table of compact, which may be changed in place
    const std::array<std::pair<const int32_t *, int64_t>, 6> reads = {{{v->page, in}, {v->length, v->batch}, {v->holders, v->pages}, {v->parent, new_batch}, {v->wanted, new_batch}, {nullptr, 0}}};
    const std::array<std::pair<const int32_t *, int64_t>, 4> writes = {{{v->page_out, out}, {v->length_out, new_batch}, {v->holders_out, v->pages}, {v->moves, moves * 3}}};
    for (size_t i = 0; i < writes.size(); ++i) {
        for (const auto &r : reads) {
            const bool in_place = (r.first == v->holders && i == 2 && r.first == writes[i].first) ||
                                  (r.first == v->page && i == 0 && !v->parent && r.first == writes[i].first && v->page_ld == v->page_out_ld);
            if (!in_place && overlap(r.first, r.second, writes[i].first, writes[i].second)) return SC_ERR_SHAPE_MISMATCH;
        }
        for (size_t j = 0; j < i; ++j)
            if (overlap(writes[j].first, writes[j].second, writes[i].first, writes[i].second)) return SC_ERR_SHAPE_MISMATCH;
    }
    return SC_OK;
}

size_t up_to(size_t n, size_t to) { return (n + to - 1) / to * to; }

// Workspace of fork, and of compact, which needs less: numbers of pages first.
struct PagesSpace {
    size_t bits, needed, before, bytes;
    PagesSpace(int64_t pages, int64_t new_batch)
    {
        const size_t blocks = (size_t)(pages + kPagesPerBlock - 1) / kPagesPerBlock;
        bits = up_to(4 * (size_t)pages, 256);
        needed = bits + blocks * (kPagesPerBlock / 8);
        before = needed + up_to(8 * ((size_t)new_batch + 1), 256);
        bytes = before + up_to(4 * blocks, 256);
    }
};

sc_status create(sc_attention **out, const sc_attention_desc *d, int32_t window, int32_t sinks)
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
    at->window = window;
    at->sinks = sinks;
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
    at->ws_bytes = row_pieces(at->head_dim, at->groups_log2) + (window ? cut_bytes(at->groups_log2) : 0);
    at->prompt_ws_bytes = prompt_workspace(at->dtype, at->head_dim, at->n_cu);
    at->tree_ws_bytes = std::max(tree_pieces(at->head_dim, at->groups_log2), up_to(at->prompt_ws_bytes, 256)) + cut_bytes(at->groups_log2);
    *out = at;
    return SC_OK;
}

}  // namespace

extern "C" sc_status sc_attention_create(sc_attention **out, const sc_attention_desc *d) { return create(out, d, 0, 0); }

extern "C" sc_status sc_attention_create_window(sc_attention **out, const sc_attention_desc *d, int32_t window, int32_t sinks)
{
    if (!out || !d) return SC_ERR_NULL;
    *out = nullptr;
    if (window < 1 || window > kMaxKeys || sinks < 0 || sinks > kMaxKeys || !d->causal) return SC_ERR_BAD_DIMS;
    return create(out, d, window, sinks);
}

extern "C" sc_status sc_attention_tree_workspace_bytes(const sc_attention *at, size_t *bytes)
{
    if (!at || !bytes) return SC_ERR_NULL;
    *bytes = at->tree_ws_bytes;
    return SC_OK;
}

extern "C" sc_status sc_attention_pages_workspace_bytes(int64_t pages, int32_t new_batch, size_t *bytes)
{
    if (!bytes) return SC_ERR_NULL;
    if (pages < 1 || pages > kMaxPages || new_batch < 0 || new_batch > kMaxBatch) return SC_ERR_BAD_DIMS;
    *bytes = PagesSpace(pages, new_batch).bytes;
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
    char window[96] = "";
    if (at->window) snprintf(window, sizeof window, ", a window of %d and the first %d", at->window, at->sinks);
    snprintf(buf, n,
             "attention %s: heads %d, key heads %d, head_dim %d (kernels padded to %d), pages of %d rows, %s%s\n"
             "  A(i,l) = sum_j softmax_j(%g * sum_k X(i,k) Y(j,k)) Z(j,l)\n"
             "  append: rotates %d of %d elements (%s), moves %d bytes a row\n"
             "  prompt: %d flops per row and key, reads and writes %d bytes a row and %d bytes a key, %zu bytes of workspace\n"
             "  decode: %d flops and %d bytes a key, %d workgroups, %zu bytes of workspace\n"
             "  tree: %d flops per row and key that it sees, %d bytes a key for all rows of a sequence, %zu bytes of workspace\n",
             at->dtype == SC_F32 ? "f32" : at->dtype == SC_F16 ? "f16" : "bf16", at->heads, at->kv_heads, d, padded_dim(d), at->page_rows,
             at->causal ? "causal" : "not causal", window, at->scale_log2 * 0.6931471805599453, 2 * at->pairs, d,
             at->interleaved ? "adjacent pairs" : "pairs of halves", 2 * (at->heads + 2 * at->kv_heads) * d * e, 4 * at->heads * d, 2 * at->heads * d * e,
             2 * at->kv_heads * d * e, at->prompt_ws_bytes, 4 * at->heads * d, 2 * at->kv_heads * d * e, 1 << at->groups_log2, at->ws_bytes,
             4 * at->heads * d, 2 * at->kv_heads * d * e, at->tree_ws_bytes);
    return SC_OK;
}

namespace {

sc_status append(const sc_attention *at, const sc_sequence_view *sequences, const int32_t *parent, const sc_rows_view *q, const sc_rows_view *k,
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
    a.parent = parent;
    for (int t = 0; t < at->pairs; ++t) a.turns[t] = at->turns[t];
    return launched(launch_append(a, at->dtype, (hipStream_t)hip_stream));
}

}  // namespace

extern "C" sc_status sc_attention_append(const sc_attention *at, const sc_sequence_view *sequences, const sc_rows_view *q, const sc_rows_view *k,
                                         const sc_rows_view *v, const sc_rows_view *q_out, const sc_cache_view *cache, void *hip_stream)
{
    return append(at, sequences, nullptr, q, k, v, q_out, cache, hip_stream);
}

extern "C" sc_status sc_attention_append_tree(const sc_attention *at, const sc_sequence_view *sequences, const int32_t *parent, const sc_rows_view *q,
                                              const sc_rows_view *k, const sc_rows_view *v, const sc_rows_view *q_out, const sc_cache_view *cache, void *hip_stream)
{
    if (!parent && !(sequences && sequences->rows == 0)) return SC_ERR_NULL;
    return append(at, sequences, parent, q, k, v, q_out, cache, hip_stream);
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
    a.head_tiles = (a.group + kHeadTile - 1) / kHeadTile;
    if (units_of((int32_t)std::min<int64_t>(table_room(a.s), INT32_MAX)) * (int64_t)a.s.batch >= kMaxUnits / ((int64_t)a.kv_heads * a.head_tiles)) return SC_ERR_BAD_DIMS;
    a.pieces = static_cast<float *>(workspace);
    if (at->window) {
        a.tree_cut = reinterpret_cast<TreeCut *>(static_cast<char *>(workspace) + at->ws_bytes - cut_bytes(at->groups_log2));
        return launched(launch_tree(a, at->dtype, (hipStream_t)hip_stream));
    }
    return launched(launch_decode(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_tree(const sc_attention *at, const sc_sequence_view *sequences, const int32_t *parent, const sc_rows_view *q,
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
    if (workspace_bytes < at->tree_ws_bytes) return SC_ERR_WORKSPACE_SMALL;
    if (!workspace) return SC_ERR_NULL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    a.tree = 1;
    a.parent = parent;
    a.causal = 1;
    if (!tree_line_ok(a)) return SC_ERR_BAD_DIMS;
    if (!at->has_device) return SC_ERR_DEVICE;
    a.pieces = static_cast<float *>(workspace);
    a.tree_cut = reinterpret_cast<TreeCut *>(static_cast<char *>(workspace) + at->tree_ws_bytes - cut_bytes(at->groups_log2));
    a.cut = reinterpret_cast<int32_t *>(static_cast<char *>(workspace) + at->prompt_ws_bytes - 2 * prompt_shares(at->n_cu) * sizeof(int32_t));   // of the other kernels
    return launched(launch_tree(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_accept(const sc_attention *at, const sc_sequence_view *sequences, const int32_t *parent, const int32_t *last,
                                         const sc_cache_view *cache, int32_t *length_out, void *hip_stream)
{
    if (!at || !sequences || !cache) return SC_ERR_NULL;
    AcceptArgs a = {};
    SC_TRY(check_sequences(sequences, true, a.s));
    SC_TRY(check_cache(at, cache, a.s, a.cache));
    if (a.s.batch == 0) return SC_OK;
    if ((!parent && a.s.rows) || !last) return SC_ERR_NULL;
    // not in place: several workgroups read the length of a sequence, one of which writes the new one
    for (const auto &[p, n] : {std::pair<const int32_t *, int64_t>{a.s.length, a.s.batch}, {a.s.row_start, a.s.batch + (int64_t)1}, {parent, a.s.rows}, {last, a.s.batch},
                               {a.s.page, table_numbers(a.s.batch, a.s.page_ld, a.s.page_count)}})
        if (overlap(p, n, length_out, a.s.batch)) return SC_ERR_SHAPE_MISMATCH;
    if (!at->has_device) return SC_ERR_DEVICE;
    a.kv_heads = at->kv_heads;
    a.head_dim = at->head_dim;
    a.parent = parent;
    a.last = last;
    a.length_out = length_out;
    return launched(launch_accept(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_fork(const sc_attention *at, const sc_pages_view *v, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!at || !v) return SC_ERR_NULL;
    if (v->new_batch > 0 && (!v->parent || !v->length_out)) return SC_ERR_NULL;
    SC_TRY(check_pages(at, v, v->new_batch, v->new_batch));
    const PagesSpace space(v->pages, v->new_batch);
    if (workspace_bytes < space.bytes) return SC_ERR_WORKSPACE_SMALL;
    if (!workspace) return SC_ERR_NULL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    if (!at->has_device) return SC_ERR_DEVICE;
    char *w = static_cast<char *>(workspace);
    const ForkArgs a = {v->batch, v->new_batch, (int32_t)v->page_count, (int32_t)v->pages, at->page_shift, at->window, at->sinks, v->page, v->length, v->holders, v->page_ld,
                        v->parent, v->wanted, v->page_out, v->length_out, v->holders_out, v->moves, v->page_out_ld, reinterpret_cast<int32_t *>(w),
                        reinterpret_cast<uint64_t *>(w + space.bits), reinterpret_cast<int32_t *>(w + space.before), reinterpret_cast<int64_t *>(w + space.needed)};
    return launched(launch_fork(a, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_compact(const sc_attention *at, const sc_pages_view *v, void *workspace, size_t workspace_bytes, void *hip_stream)
{
    if (!at || !v) return SC_ERR_NULL;
    if (v->new_batch != 0 || v->parent || v->wanted || v->length_out) return SC_ERR_SHAPE_MISMATCH;   // fork's
    SC_TRY(check_pages(at, v, v->batch, v->pages / 2));
    const PagesSpace space(v->pages, 0);
    if (workspace_bytes < space.bytes) return SC_ERR_WORKSPACE_SMALL;
    if (!workspace) return SC_ERR_NULL;
    if ((uintptr_t)workspace % 256) return SC_ERR_SHAPE_MISMATCH;
    if (!at->has_device) return SC_ERR_DEVICE;
    char *w = static_cast<char *>(workspace);
    const CompactArgs a = {v->batch, (int32_t)v->page_count, (int32_t)v->pages, at->page_shift, v->page, v->length, v->holders, v->page_ld, v->page_out, v->holders_out, v->moves,
                           v->page_out_ld, reinterpret_cast<int32_t *>(w), reinterpret_cast<uint64_t *>(w + space.bits), reinterpret_cast<int32_t *>(w + space.before)};
    return launched(launch_compact(a, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_copy(const sc_attention *at, const sc_cache_view *cache, const int32_t *moves, int64_t count, void *hip_stream)
{
    if (!at || !cache) return SC_ERR_NULL;
    if (count < 0 || count > kMaxPages) return SC_ERR_BAD_DIMS;
    CopyArgs a = {};
    Sequences s = {};
    SC_TRY(check_cache(at, cache, s, a.cache));
    if (count == 0) return SC_OK;
    if (!moves) return SC_ERR_NULL;
    if (!at->has_device) return SC_ERR_DEVICE;
    a.kv_heads = at->kv_heads;
    a.head_dim = at->head_dim;
    a.page_shift = at->page_shift;
    a.pages = s.pages;
    a.moves = moves;
    a.count = count;
    return launched(launch_copy(a, at->dtype, (hipStream_t)hip_stream));
}

extern "C" sc_status sc_attention_destroy(sc_attention *at)
{
    delete at;
    return SC_OK;
}
