// A cache of pages: new rows of keys and values written into it, and its pages
// shared, copied on write, handed out and freed as rows are reordered.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {

// ---- append -----------------------------------------------------------------
// Row i of sequence s (i < lens[s] - start[s]) goes to token start[s] + i of its
// pages, 16 bytes per thread and step.  Nothing but the rows' bytes in and out
// bounds it.  Block (x, s) takes `rpb` rows of sequence s: one for a decode
// step, enough for 16 KB for prompts, so a ragged batch leaves only blocks that
// end at once.  A row outside [0, n_rows), past the table's width or on a page
// id outside the pool is skipped.
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p, int rpb) {
    const int s = blockIdx.y;
    const int start = p.start[s];
    const int n = min(p.lens[s] - start, p.max_rows);
    const int i0 = blockIdx.x * rpb;
    if (start < 0 || i0 >= n) return;
    const int i1 = min(i0 + rpb, n);
    const int row0 = p.row0 ? p.row0[s] : s * p.max_rows;
    const int cph = p.pool.head_dim / 8;             // 16-byte chunks of a head
    const int half = p.pool.n_kv_heads * cph;        // ... of a row of K
    const int32_t* ids = p.tab.ids + s * p.tab.ld;
    for (int c = threadIdx.x; c < (i1 - i0) * 2 * half; c += 256) {
        const int i = i0 + c / (2 * half);
        int e = c % (2 * half);
        const bool isv = e >= half;
        e -= isv ? half : 0;
        const int h = e / cph, j = (e % cph) * 8;
        const int64_t row = (int64_t)row0 + i;
        const int x = start + i;
        const int col = p.pool.div.quot(x);
        if (row < 0 || row >= p.n_rows || col >= p.tab.width) continue;
        const int page = ids[col];
        if (page < 0 || page >= p.pool.n_pages) continue;
        const int t = x - col * p.pool.page_size;
        const u32x4 val = *(const u32x4*)((isv ? p.v + row * p.ld_v : p.k + row * p.ld_k) + e * 8);
        *(u32x4*)(p.pool.base + page * p.pool.page_stride + (isv ? p.pool.v_offset : 0) + h * p.pool.head_stride +
                  t * p.pool.token_stride + j) = val;
    }
}

// ---- fork ---------------------------------------------------------------------
// Four launches, each ordered after the one before by the stream:
//  1 counts: out_refs = refs, per-page scratch cleared
//  2 tables: the old rows' references leave the counts, the new rows' join them
//    (integer atomics: the order does not matter), and every row that will be
//    written to inside a page names itself at that page
//  3 places: one block decides who copies, ranks the free pages and hands them out
//  4 copies: the tokens of every page copied, in every layer

struct ForkScratch {  // in the workspace
    int32_t *movers, *first;            // [n_pages] growing rows whose last page it is, the lowest of them
    int32_t *offset, *src, *dst, *tok;  // [out_rows] (offset: one more)
};

__host__ __device__ inline ForkScratch fork_scratch(void* ws, int out_rows, int n_pages) {
    int32_t* w = (int32_t*)ws;
    ForkScratch f;
    f.movers = w;
    f.first = w + n_pages;
    f.offset = f.first + n_pages;
    f.src = f.offset + out_rows + 1;
    f.dst = f.src + out_rows;
    f.tok = f.dst + out_rows;
    return f;
}

struct ForkRow {
    int parent, start, n, grow;  // start tokens on n pages; grow > 0: tokens to make room for
    bool there, wide;
};

__device__ inline int row_len(const ForkParams& p, int r) {
    const int64_t most = min((int64_t)p.width * p.pool.page_size, (int64_t)0x7fffffff);
    return (int)min((int64_t)max(p.lens[r], 0), most);
}

__device__ inline int pages_of(const ForkParams& p, int64_t tokens) {
    return tokens <= 0 ? 0 : (int)p.pool.div.quot((uint32_t)(tokens - 1)) + 1;
}

// What out row r is: a function of the inputs alone, the same in every launch.
__device__ inline ForkRow fork_row(const ForkParams& p, int r) {
    ForkRow f;
    f.parent = p.parents[r];
    f.there = f.parent >= 0 && f.parent < p.in_rows;
    f.start = f.there ? row_len(p, f.parent) : 0;
    f.n = pages_of(p, f.start);
    const int g = f.there ? max(p.grow[r], 0) : 0;
    const int64_t total = (int64_t)f.start + g;
    f.wide = total > (int64_t)p.width * p.pool.page_size || total > 0x7fffffff;
    f.grow = f.wide ? 0 : g;
    return f;
}

__device__ inline int good_page(const ForkParams& p, int id) { return id >= 0 && id < p.pool.n_pages ? id : -1; }

// the last page of a row that will be written to inside it (-1: none)
__device__ inline int moving_page(const ForkParams& p, const ForkRow& f) {
    if (f.grow <= 0 || f.start - pages_of(p, f.start) * p.pool.page_size == 0) return -1;
    return good_page(p, p.tables[(int64_t)f.parent * p.width + f.n - 1]);
}

__global__ __launch_bounds__(256) void fork_counts_kernel(ForkParams p) {
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    for (int i = blockIdx.x * 256 + threadIdx.x; i < p.pool.n_pages; i += gridDim.x * 256) {
        p.out_refs[i] = p.refs[i];
        f.movers[i] = 0;
        f.first[i] = 0x7fffffff;
    }
    if (blockIdx.x == 0 && threadIdx.x < 2) p.short_of[threadIdx.x] = 0;
}

__global__ __launch_bounds__(256) void fork_tables_kernel(ForkParams p) {
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    const int r = blockIdx.y;
    if (r < p.in_rows) {
        const int n = pages_of(p, row_len(p, r));
        for (int i = blockIdx.x * 256 + threadIdx.x; i < n; i += gridDim.x * 256) {
            const int id = good_page(p, p.tables[(int64_t)r * p.width + i]);
            if (id >= 0) atomicSub(&p.out_refs[id], 1);
        }
    }
    if (r < p.out_rows) {
        const ForkRow w = fork_row(p, r);
        for (int i = blockIdx.x * 256 + threadIdx.x; i < p.width; i += gridDim.x * 256) {
            const int id = i < w.n ? good_page(p, p.tables[(int64_t)w.parent * p.width + i]) : -1;
            p.out_tables[(int64_t)r * p.width + i] = id;
            if (id >= 0) atomicAdd(&p.out_refs[id], 1);
        }
        if (blockIdx.x == 0 && threadIdx.x == 0) {
            p.out_start[r] = w.start;
            if (w.wide) atomicAdd(&p.short_of[1], 1);
            const int id = moving_page(p, w);
            if (id >= 0) {
                atomicAdd(&f.movers[id], 1);
                atomicMin(&f.first[id], r);
            }
        }
    }
}

// Exclusive prefix sum over the block's 1024 threads; *total gets the sum.
__device__ inline int block_scan(int v, int* lds, int* total) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int x = v;
    for (int o = 1; o < 64; o <<= 1) {
        const int y = __shfl_up(x, o, 64);
        if (lane >= o) x += y;
    }
    __syncthreads();  // the last use of lds has ended
    if (lane == 63) lds[wave] = x;
    __syncthreads();
    int before = 0, all = 0;
    for (int w = 0; w < 16; ++w) {
        if (w < wave) before += lds[w];
        all += lds[w];
    }
    *total = all;
    return before + x - v;
}

__global__ __launch_bounds__(1024) void fork_places_kernel(ForkParams p) {
    __shared__ int lds[16];
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    const int tid = threadIdx.x, R = p.out_rows, P = p.pool.n_pages;
    // who copies, and how many pages each row asks for
    int64_t asked = 0;
    for (int r0 = 0; r0 < R; r0 += 1024) {
        const int r = r0 + tid;
        int need = 0, src = -1, tok = 0;
        if (r < R) {
            const ForkRow w = fork_row(p, r);
            const int id = moving_page(p, w);
            if (id >= 0 && (p.out_refs[id] > f.movers[id] || f.first[id] != r)) {
                src = id;
                tok = w.start - (w.n - 1) * p.pool.page_size;
            }
            need = pages_of(p, (int64_t)w.start + w.grow) - w.n + (src >= 0);
        }
        int total;
        const int before = block_scan(need, lds, &total);
        if (r < R) {
            f.offset[r] = (int)min(asked + before, (int64_t)0x7fffffff);
            f.src[r] = src;
            f.dst[r] = -1;
            f.tok[r] = tok;
        }
        asked += total;
    }
    // are there as many free pages
    int64_t found = 0;
    for (int i0 = 0; i0 < P && found < asked; i0 += 1024) {
        int total;
        block_scan(i0 + tid < P && p.out_refs[i0 + tid] == 0, lds, &total);
        found += total;
    }
    const bool enough = found >= asked;
    if (tid == 0) {
        f.offset[R] = (int)min(asked, (int64_t)0x7fffffff);
        if (!enough) p.short_of[0] = (int)min(asked - found, (int64_t)0x7fffffff);
    }
    for (int r = tid; r < R; r += 1024) {
        const ForkRow w = fork_row(p, r);
        p.out_lens[r] = w.start + (enough ? w.grow : 0);
        if (!enough) f.src[r] = -1;
    }
    __syncthreads();  // offset is whole
    if (!enough) return;
    // free page of rank k to the row whose [offset, next offset) holds k
    int64_t rank0 = 0;
    for (int i0 = 0; i0 < P && rank0 < asked; i0 += 1024) {
        const int page = i0 + tid;
        const bool free = page < P && p.out_refs[page] == 0;
        int total;
        const int64_t k = rank0 + block_scan(free, lds, &total);
        rank0 += total;
        if (free && k < asked) {
            int lo = 0, hi = R - 1;  // the last row with offset <= k
            while (lo < hi) {
                const int mid = (lo + hi + 1) / 2;
                if (f.offset[mid] <= k) lo = mid; else hi = mid - 1;
            }
            const int j = (int)(k - f.offset[lo]);
            const bool copies = f.src[lo] >= 0;
            const int n = pages_of(p, p.out_start[lo]);
            p.out_tables[(int64_t)lo * p.width + n - copies + j] = page;
            p.out_refs[page] = 1;
            if (copies && j == 0) f.dst[lo] = page;
        }
    }
    __syncthreads();  // every free page was looked at before counts move again
    for (int r = tid; r < R; r += 1024)
        if (f.src[r] >= 0) atomicSub(&p.out_refs[f.src[r]], 1);
}

__global__ __launch_bounds__(256) void fork_copy_kernel(ForkParams p) {
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    const int r = blockIdx.x;
    const int src = f.src[r], dst = f.dst[r], tok = f.tok[r];
    if (src < 0 || dst < 0) return;
    const int cph = p.pool.head_dim / 8;
    uint16_t* base = p.pool.base + blockIdx.y * p.layer_stride;
    const uint16_t* from = base + src * p.pool.page_stride;
    uint16_t* to = base + dst * p.pool.page_stride;
    const int n = tok * 2 * p.pool.n_kv_heads * cph;
    for (int i = threadIdx.x; i < n; i += 256) {
        const int j = i % cph, a = i / cph;
        const int h = a % p.pool.n_kv_heads, b = a / p.pool.n_kv_heads;
        const int64_t o = (b & 1) * p.pool.v_offset + h * p.pool.head_stride + (b >> 1) * p.pool.token_stride + j * 8;
        *(u32x4*)(to + o) = *(const u32x4*)(from + o);
    }
}

}  // namespace

hipError_t launch_kv_append(const AppendParams& p, hipStream_t s) {
    if (p.tab.rows <= 0 || p.max_rows <= 0 || p.n_rows <= 0) return hipSuccess;
    const int row_bytes = 2 * p.pool.n_kv_heads * p.pool.head_dim * 2;
    const int rpb = p.max_rows == 1 ? 1 : (16384 + row_bytes - 1) / row_bytes;
    PB_LAUNCH(kv_append_kernel, dim3((p.max_rows + rpb - 1) / rpb, p.tab.rows), dim3(256), 0, s, p, rpb);
    return hipGetLastError();
}

size_t page_fork_workspace(int out_rows, int n_pages) { return ((size_t)2 * n_pages + 4 * (size_t)out_rows + 1) * 4; }

hipError_t launch_page_fork(const ForkParams& p, hipStream_t s) {
    const int P = p.pool.n_pages;
    PB_LAUNCH(fork_counts_kernel, dim3((P + 1023) / 1024), dim3(256), 0, s, p);
    const int rows = p.in_rows > p.out_rows ? p.in_rows : p.out_rows;
    if (rows > 0)
        PB_LAUNCH(fork_tables_kernel, dim3((p.width + 1023) / 1024, rows), dim3(256), 0, s, p);
    if (p.out_rows > 0) {
        PB_LAUNCH(fork_places_kernel, dim3(1), dim3(1024), 0, s, p);
        PB_LAUNCH(fork_copy_kernel, dim3(p.out_rows, p.n_layers), dim3(256), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace pb
