// Launch wrappers of the paged cache's kernels and beam selection
// (paged_attention.hip, paged_cache.hip, beam.hip; entry points in paged_ops.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "fastdiv.h"

namespace pb {

// One layer's pages.  Element (page, c, h, t, j) (c = 0 keys, 1 values) is at
// base + page page_stride + c v_offset + h head_stride + t token_stride + j;
// strides in elements of the 16-bit storage type, multiples of 8, 64-bit: a
// pool may be larger than 2^31 elements.
struct PagePool {
    uint16_t* base;
    int64_t page_stride, v_offset, head_stride, token_stride;
    int n_pages, page_size, n_kv_heads, head_dim;
    FastDiv div;  // by page_size
};

// Rows of one call's sequences: page table row s at tables + s * ld, `width` entries.
struct PageTables {
    const int32_t* ids;
    int64_t ld;
    int width, rows;
};

struct AppendParams {
    const uint16_t *k, *v;
    int64_t ld_k, ld_v;
    int n_rows;
    PagePool pool;
    PageTables tab;
    const int32_t *start, *lens, *row0;
    int max_rows;
};
hipError_t launch_kv_append(const AppendParams& p, hipStream_t s);

struct PagedAttentionParams {
    const uint16_t* q; int64_t ld_q;
    uint16_t* out; int64_t ld_out;
    PagePool pool;
    PageTables tab;
    const int32_t* lens;
    int n_heads;
    float scale;
    int window;
    bool shared;  // rows next to each other share pages
    void* ws; size_t ws_bytes;
};
size_t paged_attention_workspace(int n_seqs, int n_heads, int n_kv_heads, int hd, int width, int page_size);
bool paged_attention_fits(int n_seqs, int n_heads, int n_kv_heads);  // a launch holds its blocks
hipError_t launch_paged_attention(int dtype, const PagedAttentionParams& p, hipStream_t s);

struct BeamParams {
    const float* logits; int64_t ld;
    const float* scores;
    const int32_t* alive;
    int B, W, V, eos, pad;
    float* out_scores;
    int32_t *out_tokens, *out_parents, *out_alive;
    void* ws;
};
constexpr int BEAM_MAX_WIDTH = 32, BEAM_MAX_VOCAB = 1 << 20;
size_t beam_select_workspace(int B, int W, int V);
hipError_t launch_beam_select(const BeamParams& p, hipStream_t s);

struct ForkParams {
    PagePool pool;
    int n_layers; int64_t layer_stride;
    const int32_t* parents; int out_rows;
    const int32_t* tables; int width;
    const int32_t* lens; int in_rows;
    const int32_t *refs, *grow;
    int32_t *out_tables, *out_start, *out_lens, *out_refs, *short_of;
    void* ws;
};
size_t page_fork_workspace(int out_rows, int n_pages);
// Pieces of pages that the rows' copies can be, at most; launches need them below 2^31.
int64_t page_fork_copies(const ForkParams& p);
hipError_t launch_page_fork(const ForkParams& p, hipStream_t s);

}  // namespace pb
