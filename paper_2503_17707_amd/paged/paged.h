// Launch wrappers of the paged cache's kernels and beam selection
// (paged_attention.hip, paged_cache.hip, beam.hip; entry points in paged_ops.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pb {

// Quotients by a divisor fixed at launch, exact for 0 <= n < 2^31: with
// s = ceil(log2 d) and m = floor(2^(31 + s) / d) + 1, n / d = (2 n m) >> (32 + s)
// (m d - 2^(31 + s) <= d <= 2^s, so the error n (m d - 2^(31+s)) / (d 2^(31+s)) is
// below 1 / d; m < 2^32 because d > 2^(s-1)).
struct FastDiv {
    uint32_t m, s, d;
    FastDiv(uint32_t div = 1) : d(div) {
        s = 0;
        while ((1u << s) < div) ++s;
        m = (uint32_t)((((uint64_t)1 << (31 + s)) / div) + 1);
    }
    __host__ __device__ inline uint32_t quot(uint32_t n) const {
#if defined(__HIP_DEVICE_COMPILE__)
        return __umulhi(n << 1, m) >> s;
#else
        return (uint32_t)(((uint64_t)(n << 1) * m) >> 32) >> s;
#endif
    }
};

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
    void* ws; size_t ws_bytes;
};
size_t paged_attention_workspace(int n_seqs, int n_heads, int n_kv_heads, int hd, int width, int page_size);
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
hipError_t launch_page_fork(const ForkParams& p, hipStream_t s);

}  // namespace pb
