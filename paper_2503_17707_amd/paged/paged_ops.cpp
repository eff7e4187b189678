// Entry points of the paged cache and beam selection (include/pipeboost_ops.h):
// argument checks, then the launch.
#include <hip/hip_runtime.h>

#include <cstdarg>
#include <cstdio>

#include "../../include/pipeboost.h"
#include "../../include/pipeboost_ops.h"
#include "paged.h"

__attribute__((visibility("hidden"))) int pb_fail_status(int code, const char* msg);  // model.cpp

namespace {

int refuse(const char* fmt, ...) {
    char buf[256];
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(buf, sizeof(buf), fmt, ap);
    va_end(ap);
    return pb_fail_status(PB_EINVAL, buf);
}

int launched(const char* op, hipError_t e) {
    if (e == hipSuccess) return PB_OK;
    char buf[256];
    snprintf(buf, sizeof(buf), "%s: launch failed: %s", op, hipGetErrorString(e));
    return pb_fail_status(PB_EHIP, buf);
}

bool aligned(const void* p, uintptr_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

bool sizes_ok(const pb_kv_pool* c) {
    return c && c->n_pages >= 1 && c->n_pages <= (1 << 30) && c->page_size >= 1 && c->page_size <= 4096 && c->n_kv_heads >= 1 &&
           c->n_kv_heads <= 65535 && (c->head_dim == 64 || c->head_dim == 128);
}

// A stride is used (and checked) only if its dimension has more than one place.
bool stride_ok(int64_t stride, int64_t places, int hd) {
    return places <= 1 || (stride >= hd && stride % 8 == 0 && stride < ((int64_t)1 << 44));
}

int make_pool(const char* op, int32_t dtype, const pb_kv_pool* c, pb::PagePool* out) {
    if (dtype != PB_BF16 && dtype != PB_F16) return refuse("%s: bad dtype %d", op, dtype);
    if (!c) return refuse("%s: pool is NULL", op);
    if (!sizes_ok(c))
        return refuse("%s: pool of %d pages of %d tokens, %d heads of %d (page_size 1..4096, head_dim 64 or 128)", op,
                      c->n_pages, c->page_size, c->n_kv_heads, c->head_dim);
    if ((int64_t)c->page_size * c->n_kv_heads * (c->head_dim / 4) > 0x7fffffff) return refuse("%s: a page of 2^35 bytes or more", op);
    if (!c->base || !aligned(c->base, 16)) return refuse("%s: pool base must be non-NULL and 16-byte aligned", op);
    if (!stride_ok(c->page_stride, c->n_pages, c->head_dim) || !stride_ok(c->v_offset, 2, c->head_dim) ||
        !stride_ok(c->head_stride, c->n_kv_heads, c->head_dim) || !stride_ok(c->token_stride, c->page_size, c->head_dim) ||
        (c->page_size > 1 && c->token_stride > 0x7fffffff))
        return refuse("%s: pool strides %lld, %lld, %lld, %lld must be multiples of 8 and at least head_dim "
                      "(token_stride < 2^31)", op,
                      (long long)c->page_stride, (long long)c->v_offset, (long long)c->head_stride,
                      (long long)c->token_stride);
    out->base = (uint16_t*)c->base;
    out->page_stride = c->page_stride;
    out->v_offset = c->v_offset;
    out->head_stride = c->head_stride;
    out->token_stride = c->token_stride;
    out->n_pages = c->n_pages;
    out->page_size = c->page_size;
    out->n_kv_heads = c->n_kv_heads;
    out->head_dim = c->head_dim;
    out->div = pb::FastDiv((uint32_t)c->page_size);
    return PB_OK;
}

int check_tables(const char* op, const int32_t* tables, int32_t width, int64_t ld, int32_t rows) {
    if (rows < 0 || rows > 65535) return refuse("%s: %d rows (0..65535)", op, rows);
    if (width < 1 || ld < width) return refuse("%s: tables of width %d with row stride %lld", op, width, (long long)ld);
    if (rows > 0 && !tables) return refuse("%s: tables is NULL", op);
    return PB_OK;
}

bool rows_ok(const void* p, int64_t ld, int64_t rows, int64_t cols) {
    return p && aligned(p, 16) && (rows <= 1 || (ld >= cols && ld % 8 == 0));
}

bool overlap(const void* a, size_t na, const void* b, size_t nb) {
    return a && b && na && nb && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}

}  // namespace

extern "C" int pb_op_kv_append(int32_t dtype, const void* k, int64_t ld_k, const void* v, int64_t ld_v, int32_t n_rows,
                               const pb_kv_pool* pool, const int32_t* tables, int32_t width, int64_t ld_tables,
                               const int32_t* start, const int32_t* lens, const int32_t* row0, int32_t n_seqs,
                               int32_t max_rows, void* stream) {
    const char* op = "pb_op_kv_append";
    pb::AppendParams p{};
    if (int rc = make_pool(op, dtype, pool, &p.pool)) return rc;
    if (int rc = check_tables(op, tables, width, ld_tables, n_seqs)) return rc;
    if (n_rows < 0 || max_rows < 0) return refuse("%s: n_rows=%d max_rows=%d", op, n_rows, max_rows);
    if (n_seqs == 0 || n_rows == 0 || max_rows == 0) return PB_OK;
    const int64_t cols = (int64_t)pool->n_kv_heads * pool->head_dim;
    if (!rows_ok(k, ld_k, n_rows, cols) || !rows_ok(v, ld_v, n_rows, cols))
        return refuse("%s: k and v must be 16-byte aligned, row strides (%lld, %lld) multiples of 8 and at least %lld", op,
                      (long long)ld_k, (long long)ld_v, (long long)cols);
    if (!start || !lens) return refuse("%s: NULL operand", op);
    p.k = (const uint16_t*)k; p.ld_k = ld_k; p.v = (const uint16_t*)v; p.ld_v = ld_v; p.n_rows = n_rows;
    p.tab = {tables, ld_tables, width, n_seqs};
    p.start = start; p.lens = lens; p.row0 = row0; p.max_rows = max_rows;
    return launched(op, pb::launch_kv_append(p, (hipStream_t)stream));
}

extern "C" size_t pb_op_paged_attention_workspace(int32_t n_seqs, int32_t n_heads, const pb_kv_pool* pool, int32_t width) {
    if (!sizes_ok(pool) || n_seqs < 0 || n_seqs > 65535 || width < 1 || n_heads < 1 || n_heads > 65535 ||
        n_heads % pool->n_kv_heads || (int64_t)width * pool->page_size > (1 << 30))
        return 0;
    return pb::paged_attention_workspace(n_seqs, n_heads, pool->n_kv_heads, pool->head_dim, width, pool->page_size);
}

extern "C" int pb_op_paged_attention(int32_t dtype, const void* q, int64_t ld_q, const pb_kv_pool* pool,
                                     const int32_t* tables, int32_t width, int64_t ld_tables, const int32_t* lens,
                                     int32_t n_seqs, int32_t n_heads, float scale, int32_t window, int32_t shared,
                                     void* out, int64_t ld_out, void* workspace, size_t workspace_bytes, void* stream) {
    const char* op = "pb_op_paged_attention";
    pb::PagedAttentionParams p{};
    if (int rc = make_pool(op, dtype, pool, &p.pool)) return rc;
    if (int rc = check_tables(op, tables, width, ld_tables, n_seqs)) return rc;
    if (n_heads < 1 || n_heads > 65535 || n_heads % pool->n_kv_heads)
        return refuse("%s: %d heads are no multiple of %d key and value heads", op, n_heads, pool->n_kv_heads);
    if (window < 0 || !(scale - scale == 0.f)) return refuse("%s: window=%d scale=%g", op, window, (double)scale);
    if ((int64_t)width * pool->page_size > (1 << 30)) return refuse("%s: tables of more than 2^30 tokens a row", op);
    if (n_seqs == 0) return PB_OK;
    if (!pb::paged_attention_fits(n_seqs, n_heads, pool->n_kv_heads))
        return refuse("%s: %d sequences of %d heads on %d: more blocks than a launch takes", op, n_seqs, n_heads, pool->n_kv_heads);
    const int64_t cols = (int64_t)n_heads * pool->head_dim;
    if (!rows_ok(q, ld_q, n_seqs, cols) || !rows_ok(out, ld_out, n_seqs, cols))
        return refuse("%s: q and out must be 16-byte aligned, row strides (%lld, %lld) multiples of 8 and at least %lld",
                      op, (long long)ld_q, (long long)ld_out, (long long)cols);
    if (!lens) return refuse("%s: lens is NULL", op);
    if (workspace && !aligned(workspace, 16)) return refuse("%s: workspace must be 16-byte aligned", op);
    const size_t rows = (size_t)n_seqs - 1;
    if (overlap(workspace, workspace_bytes, q, (rows * ld_q + cols) * 2) ||
        overlap(workspace, workspace_bytes, out, (rows * ld_out + cols) * 2) ||
        overlap(workspace, workspace_bytes, lens, (size_t)n_seqs * 4) ||
        overlap(workspace, workspace_bytes, tables, (rows * ld_tables + width) * 4))
        return refuse("%s: the workspace overlaps an operand", op);
    p.q = (const uint16_t*)q; p.ld_q = ld_q; p.out = (uint16_t*)out; p.ld_out = ld_out;
    p.tab = {tables, ld_tables, width, n_seqs};
    p.lens = lens; p.n_heads = n_heads; p.scale = scale; p.window = window; p.shared = shared != 0;
    p.ws = workspace; p.ws_bytes = workspace ? workspace_bytes : 0;
    return launched(op, pb::launch_paged_attention(dtype, p, (hipStream_t)stream));
}

static bool beam_ok(int32_t B, int32_t W, int32_t V) {
    return B >= 0 && B <= 65535 && W >= 1 && W <= pb::BEAM_MAX_WIDTH && V >= 1 && V <= pb::BEAM_MAX_VOCAB;
}

extern "C" size_t pb_op_beam_select_workspace(int32_t B, int32_t W, int32_t V) {
    return beam_ok(B, W, V) ? pb::beam_select_workspace(B, W, V) : 0;
}

extern "C" int pb_op_beam_select(const float* logits, int64_t ld_logits, const float* scores, const int32_t* alive,
                                 int32_t B, int32_t W, int32_t V, int32_t eos, int32_t pad, float* out_scores,
                                 int32_t* out_tokens, int32_t* out_parents, int32_t* out_alive, void* workspace,
                                 size_t workspace_bytes, void* stream) {
    const char* op = "pb_op_beam_select";
    if (!beam_ok(B, W, V)) return refuse("%s: B=%d W=%d V=%d (W 1..%d, V 1..2^20)", op, B, W, V, pb::BEAM_MAX_WIDTH);
    if (eos < -1 || eos >= V || pad < 0 || pad >= V) return refuse("%s: eos=%d pad=%d outside the vocabulary", op, eos, pad);
    if (B == 0) return PB_OK;
    if (!logits || !aligned(logits, 4) || ((int64_t)B * W > 1 && ld_logits < V))
        return refuse("%s: logits NULL, unaligned or with rows of %lld < V", op, (long long)ld_logits);
    if (!scores || !alive || !out_scores || !out_tokens || !out_parents || !out_alive) return refuse("%s: NULL operand", op);
    const size_t need = pb::beam_select_workspace(B, W, V);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
        return refuse("%s: workspace of %zu bytes, 16-byte aligned, is needed (%zu given)", op, need, workspace ? workspace_bytes : 0);
    pb::BeamParams p{};
    p.logits = logits; p.ld = ld_logits; p.scores = scores; p.alive = alive;
    p.B = B; p.W = W; p.V = V; p.eos = eos; p.pad = pad;
    p.out_scores = out_scores; p.out_tokens = out_tokens; p.out_parents = out_parents; p.out_alive = out_alive;
    p.ws = workspace;
    return launched(op, pb::launch_beam_select(p, (hipStream_t)stream));
}

extern "C" size_t pb_op_page_fork_workspace(int32_t out_rows, int32_t n_pages) {
    if (out_rows < 0 || out_rows > 65535 || n_pages < 1 || n_pages > (1 << 30)) return 0;
    return pb::page_fork_workspace(out_rows, n_pages);
}

extern "C" int pb_op_page_fork(int32_t dtype, const pb_kv_pool* pool, int32_t n_layers, int64_t layer_stride,
                               const int32_t* parents, int32_t out_rows, const int32_t* tables, int32_t width,
                               const int32_t* lens, int32_t in_rows, const int32_t* refs, const int32_t* grow,
                               int32_t* out_tables, int32_t* out_start, int32_t* out_lens, int32_t* out_refs,
                               int32_t* short_of, void* workspace, size_t workspace_bytes, void* stream) {
    const char* op = "pb_op_page_fork";
    pb::ForkParams p{};
    if (int rc = make_pool(op, dtype, pool, &p.pool)) return rc;
    if (int rc = check_tables(op, tables, width, width, in_rows)) return rc;
    if (out_rows < 0 || out_rows > 65535) return refuse("%s: %d rows (0..65535)", op, out_rows);
    if (n_layers < 1 || n_layers > 65535 || !stride_ok(layer_stride, n_layers, pool->head_dim))
        return refuse("%s: %d layers with stride %lld", op, n_layers, (long long)layer_stride);
    if ((out_rows && (!parents || !grow || !out_tables || !out_start || !out_lens)) || (in_rows && !lens) || !refs ||
        !out_refs || !short_of)
        return refuse("%s: NULL operand", op);
    const size_t need = pb::page_fork_workspace(out_rows, pool->n_pages);
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < need)
        return refuse("%s: workspace of %zu bytes, 16-byte aligned, is needed (%zu given)", op, need, workspace ? workspace_bytes : 0);
    const struct { const void* p; size_t n; } ins[] = {{parents, (size_t)out_rows * 4}, {tables, (size_t)in_rows * width * 4},
                                                       {lens, (size_t)in_rows * 4}, {refs, (size_t)pool->n_pages * 4},
                                                       {grow, (size_t)out_rows * 4}},
        outs[] = {{out_tables, (size_t)out_rows * width * 4}, {out_start, (size_t)out_rows * 4},
                  {out_lens, (size_t)out_rows * 4}, {out_refs, (size_t)pool->n_pages * 4}, {short_of, 8}, {workspace, need}};
    for (const auto& i : ins)
        for (const auto& o : outs)
            if (overlap(i.p, i.n, o.p, o.n)) return refuse("%s: an output overlaps an input", op);
    for (const auto& o : outs)  // (some are read again: places in the tables come from out_start)
        for (const auto* other = &o + 1; other < outs + sizeof(outs) / sizeof(outs[0]); ++other)
            if (overlap(o.p, o.n, other->p, other->n)) return refuse("%s: two outputs overlap, or one the workspace", op);
    p.n_layers = n_layers; p.layer_stride = layer_stride; p.parents = parents; p.out_rows = out_rows;
    p.tables = tables; p.width = width; p.lens = lens; p.in_rows = in_rows; p.refs = refs; p.grow = grow;
    p.out_tables = out_tables; p.out_start = out_start; p.out_lens = out_lens; p.out_refs = out_refs;
    p.short_of = short_of; p.ws = workspace;
    if (pb::page_fork_copies(p) > 0x7fffffff)
        return refuse("%s: %d rows in %d layers of pages of %lld bytes: 2^31 pieces of 32 KB to copy or more", op, out_rows, n_layers,
                      (long long)pool->page_size * 4 * pool->n_kv_heads * pool->head_dim);
    return launched(op, pb::launch_page_fork(p, (hipStream_t)stream));
}
