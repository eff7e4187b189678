// A cache of pages: new rows of keys and values written into it, and its pages
// shared, copied on write, handed out and freed as rows are reordered.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {


// ---- append -----------------------------------------------------------------
// Row i of sequence s (i < lens[s] - start[s]) goes to token start[s] + i of its
// pages, 16 bytes per thread and step.  Nothing but the rows' bytes in and out
// bounds it.  Block (x, s) takes `rpb` rows of sequence s: one for
// a decode step, about 16 KB for prompts, so a ragged batch leaves only blocks that
// end at once.  A row outside [0, n_rows), past the table's width or on a page
// id outside the pool is skipped.  A decode step's tokens are read next and stay in
// cache; prompts' are not (streaming stores: 16 ragged prompts of 40 heads of 128, 221
// MB, 48.0 us against 52.0).
template <bool PROMPTS>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendParams p, int rpb, FastDiv per_row) {
    const int s = blockIdx.y;
    const int start = p.start[s];
    const int n = (int)min((int64_t)p.lens[s] - start, (int64_t)p.max_rows);
    if (start < 0) return;
    const int64_t row0 = p.row0 ? p.row0[s] : (int64_t)s * p.max_rows;
    const int lc = p.pool.head_dim == 128 ? 4 : 3;          // log2 of a head's 16-byte chunks
    const int half = p.pool.n_kv_heads << lc;               // chunks of a row of K
    const int32_t* ids = p.tab.ids + s * p.tab.ld;
    for (int64_t i0 = (int64_t)blockIdx.x * rpb; i0 < n; i0 += (int64_t)gridDim.x * rpb) {
        const int rows = min((int64_t)rpb, n - i0);
        for (int c = threadIdx.x; c < rows * 2 * half; c += 256) {
            const int r = per_row.quot(c), i = (int)i0 + r;
            int e = c - r * 2 * half;
            const bool isv = e >= half;
            e -= isv ? half : 0;
            const int h = e >> lc, j = (e & ((1 << lc) - 1)) * 8;
            const int64_t row = row0 + i;
            const int col = p.pool.div.quot(start + i);
            if (row < 0 || row >= p.n_rows || col >= p.tab.width) continue;
            const int page = ids[col];
            if (page < 0 || page >= p.pool.n_pages) continue;
            const u32x4 val = *(const u32x4*)((isv ? p.v + row * p.ld_v : p.k + row * p.ld_k) + e * 8);
            u32x4* to = (u32x4*)(p.pool.base + page * p.pool.page_stride + (isv ? p.pool.v_offset : 0) +
                                 h * p.pool.head_stride + (start + i - col * p.pool.page_size) * p.pool.token_stride + j);
            if (PROMPTS) __builtin_nontemporal_store(val, to);
            else *to = val;
        }
    }
}

// ---- fork ---------------------------------------------------------------------
// Steps, each ordered after the one before:
//  1 counts: out_refs = refs, per-page scratch cleared
//  2 tables: the old rows' references leave the counts, the new rows' join them
//    (integer atomics: the order does not matter), and every row that will be
//    written to inside a page names itself at that page
//  3 places: one block decides who copies, ranks the free pages and hands them out
//  4 copies: the tokens of every page copied, in every layer
// Copying bounds large calls, the chain of launches and dependent reads small ones:
// up to SMALL_PAGES pages and SMALL_ENTRIES table entries one block takes steps 1
// to 3 with the counts in LDS (256 rows of 22 pages in 1300: 53 us with the copies,
// 57 the other way; 256 rows of 96: 17.4 against 16.1).

constexpr int SMALL_PAGES = 8192, SMALL_ROWS = 512, SMALL_ENTRIES = 16384;

struct ForkScratch {  // in the workspace
    int32_t *movers, *first;            // [n_pages] growing rows whose last page it is, the lowest of them
    int32_t *offset, *slot;             // [out_rows] rank of a row's first new page; its place in the copy list or -1
    int32_t *src, *dst, *tok;           // [out_rows] copy list: pages, tokens
    int32_t *count;                     // its length
};

__host__ __device__ inline ForkScratch fork_scratch(void* ws, int out_rows, int n_pages) {
    int32_t* w = (int32_t*)ws;
    ForkScratch f;
    f.movers = w;
    f.first = w + n_pages;
    f.offset = f.first + n_pages;
    f.slot = f.offset + out_rows;
    f.src = f.slot + out_rows;
    f.dst = f.src + out_rows;
    f.tok = f.dst + out_rows;
    f.count = f.tok + out_rows;
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

// Steps 1 to 3 (SMALL; out_rows and in_rows up to SMALL_ROWS) or step 3.
template <bool SMALL>
__global__ __launch_bounds__(1024) void fork_places_kernel(ForkParams p, FastDiv width) {
    extern __shared__ int32_t small[];  // SMALL: counts, movers, first by page
    __shared__ int lds[16];
    __shared__ int copies;  // length of the copy list
    // SMALL: per row its first new page's rank, its pages, its place in the copy list
    __shared__ int32_t offsets[SMALL ? SMALL_ROWS : 1], n_of[SMALL ? SMALL_ROWS : 1], slots[SMALL ? SMALL_ROWS : 1];
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    const int tid = threadIdx.x, R = p.out_rows, P = p.pool.n_pages;
    int32_t* refs = SMALL ? small : p.out_refs;
    int32_t* movers = SMALL ? small + P : f.movers;
    int32_t* first = SMALL ? small + 2 * P : f.first;
    int32_t* offset = SMALL ? offsets : f.offset;
    int32_t* slot = SMALL ? slots : f.slot;
    if (tid == 0) copies = 0;
    __syncthreads();
    ForkRow mine{};  // SMALL: row tid
    int my_page = -1;
    if (SMALL) {
        __shared__ int32_t held[SMALL_ROWS], parent_of[SMALL_ROWS];
        for (int i = tid; i < P; i += 1024) {
            refs[i] = p.refs[i];
            movers[i] = 0;
            first[i] = 0x7fffffff;
        }
        if (tid < p.in_rows) held[tid] = pages_of(p, row_len(p, tid));
        if (tid < R) {
            mine = fork_row(p, tid);
            my_page = moving_page(p, mine);
            n_of[tid] = mine.n;
            parent_of[tid] = mine.parent;
            p.out_start[tid] = mine.start;
        }
        const int wide = __syncthreads_count(mine.wide);
        if (tid < 2) p.short_of[tid] = tid ? wide : 0;
        if (my_page >= 0) {
            atomicAdd(&movers[my_page], 1);
            atomicMin(&first[my_page], tid);
        }
        // four entries of a thread in flight
        const int32_t* __restrict__ tables = p.tables;
        int32_t* __restrict__ out_tables = p.out_tables;
        const int n_in = p.in_rows * p.width, n_out = R * p.width;
        for (int i0 = tid; i0 < max(n_in, n_out); i0 += 4 * 1024) {
            int was[4], is[4];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * 1024, r = width.quot(i), c = i - r * p.width;
                was[u] = i < n_in && c < held[r] ? tables[i] : -1;
                is[u] = i < n_out && c < n_of[r] ? tables[parent_of[r] * p.width + c] : -1;
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int i = i0 + u * 1024;
                was[u] = good_page(p, was[u]);
                is[u] = good_page(p, is[u]);
                if (was[u] >= 0) atomicSub(&refs[was[u]], 1);
                if (is[u] >= 0) atomicAdd(&refs[is[u]], 1);
                if (i < n_out) out_tables[i] = is[u];
            }
        }
        __syncthreads();
    }
    // who copies, and how many pages each row asks for
    int64_t asked = 0;
    int my_src = -1;
    for (int r0 = 0; r0 < R; r0 += 1024) {
        const int r = r0 + tid;
        int need = 0, src = -1, tok = 0;
        if (r < R) {
            const ForkRow w = SMALL ? mine : fork_row(p, r);
            const int id = SMALL ? my_page : moving_page(p, w);
            if (id >= 0 && (refs[id] > movers[id] || first[id] != r)) {
                src = id;
                tok = w.start - (w.n - 1) * p.pool.page_size;
            }
            need = pages_of(p, (int64_t)w.start + w.grow) - w.n + (src >= 0);
        }
        int total;
        const int before = block_scan(need, lds, &total);
        if (r < R) {
            offset[r] = (int)min(asked + before, (int64_t)0x7fffffff);
            const int at = src >= 0 ? atomicAdd(&copies, 1) : -1;  // in any order: copies do not meet
            slot[r] = at;
            if (at >= 0) {
                f.src[at] = my_src = src;
                f.tok[at] = tok;
            }
        }
        asked += total;
    }
    __syncthreads();  // `first` was read: from here on it lists the free pages
    // the free pages in ascending order, as many as are asked for
    constexpr int PER = 4;  // pages of a thread at a time
    int32_t* list = first;
    int64_t found = 0;
    for (int i0 = 0; i0 < P && found < asked; i0 += 1024 * PER) {
        const int page = i0 + tid * PER;
        bool free[PER];
        int n = 0, total;
#pragma unroll
        for (int j = 0; j < PER; ++j) {
            free[j] = page + j < P && refs[min(page + j, P - 1)] == 0;
            n += free[j];
        }
        int64_t k = found + block_scan(n, lds, &total);
        found += total;
#pragma unroll
        for (int j = 0; j < PER; ++j)
            if (free[j] && k < asked) list[k++] = page + j;
    }
    const bool enough = found >= asked;
    if (tid == 0) {
        *f.count = enough ? copies : 0;
        if (!enough) p.short_of[0] = (int)min(asked - found, (int64_t)0x7fffffff);
    }
    for (int r = tid; r < R; r += 1024) {
        const ForkRow w = SMALL ? mine : fork_row(p, r);
        p.out_lens[r] = w.start + (enough ? w.grow : 0);
    }
    __syncthreads();  // offset and list are whole
    // the page of rank k to the row whose [offset, next offset) holds k
    for (int k = tid; enough && k < asked; k += 1024) {
        int lo = 0, hi = R - 1;  // the last row with offset <= k
        while (lo < hi) {
            const int mid = (lo + hi + 1) / 2;
            if (offset[mid] <= k) lo = mid; else hi = mid - 1;
        }
        const int page = list[k], at = k - offset[lo];
        const int copy = slot[lo], last = SMALL ? n_of[lo] : pages_of(p, p.out_start[lo]);
        p.out_tables[(int64_t)lo * p.width + last - (copy >= 0) + at] = page;
        refs[page] = 1;
        if (copy >= 0 && at == 0) f.dst[copy] = page;
    }
    if (SMALL) {
        // (a page that is copied is in use: nobody counts it free)
        if (enough && my_src >= 0) atomicSub(&refs[my_src], 1);
        __syncthreads();
        for (int i = tid; i < P; i += 1024) p.out_refs[i] = refs[i];
    } else if (enough) {
        for (int i = tid; i < copies; i += 1024) atomicSub(&refs[f.src[i]], 1);
    }
}

// The copies' tokens (not their pages), PIECE 16-byte chunks of one in one layer to
// a block at a time, eight steps of a thread in flight; as many blocks as the chip
// holds take the pieces in turn, since how many copies there are is not known here.
// Some 80 copies of 6 tokens in 24 layers of 32 heads of 64 (rows of one parent copy the
// same page, which is read from memory once: 75 MB in, 100 out): 45 to 46 us, 3.8 TB/s;
// the call 53, with ordinary stores 62.
constexpr int PIECE = 8 * 256, COPY_BLOCKS = 1024;
__global__ __launch_bounds__(256) void fork_copy_kernel(ForkParams p, FastDiv heads, FastDiv layers, FastDiv pieces,
                                                        bool by_token) {
    const ForkScratch f = fork_scratch(p.ws, p.out_rows, p.pool.n_pages);
    const int lc = p.pool.head_dim == 128 ? 4 : 3;
    const int64_t items = (int64_t)*f.count * p.n_layers * pieces.d;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const uint32_t cl = pieces.quot((uint32_t)item), copy = layers.quot(cl);
        const int i0 = ((uint32_t)item - cl * pieces.d) * PIECE, tok = f.tok[copy];
        const int n = (tok * 2 * p.pool.n_kv_heads) << lc;
        if (i0 >= n) continue;
        uint16_t* base = p.pool.base + (cl - copy * p.n_layers) * p.layer_stride;
        const uint16_t* from = base + f.src[copy] * p.pool.page_stride;
        uint16_t* to = base + f.dst[copy] * p.pool.page_stride;
        int64_t o[8];
        u32x4 v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            // token by token, or head by head: whichever a page holds together
            const int i = min(i0 + u * 256 + (int)threadIdx.x, n - 1), a = i >> lc, j = i & ((1 << lc) - 1);
            int h, t, c;
            if (by_token) {
                const int row = heads.quot(a);
                h = a - row * p.pool.n_kv_heads, c = row & 1, t = row >> 1;
            } else {
                const int row = a / tok;
                t = a - row * tok, c = row >= p.pool.n_kv_heads, h = row - (c ? p.pool.n_kv_heads : 0);
            }
            o[u] = c * p.pool.v_offset + h * p.pool.head_stride + t * p.pool.token_stride + j * 8;
            v[u] = *(const u32x4*)(from + o[u]);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
            if (i0 + u * 256 + (int)threadIdx.x < n) __builtin_nontemporal_store(v[u], (u32x4*)(to + o[u]));
    }
}

}  // namespace

hipError_t launch_kv_append(const AppendParams& p, hipStream_t s) {
    if (p.tab.rows <= 0 || p.max_rows <= 0 || p.n_rows <= 0) return hipSuccess;
    const int row_bytes = 2 * p.pool.n_kv_heads * p.pool.head_dim * 2;
    const int rpb = p.max_rows == 1 ? 1 : (16384 + row_bytes - 1) / row_bytes;
    const FastDiv per_row(2 * p.pool.n_kv_heads * p.pool.head_dim / 8);
    // (max_rows may be far more than any sequence has: blocks take rows in turn then)
    const int blocks = (p.max_rows - 1) / rpb + 1, most = 32768 / p.tab.rows + 1;
    const dim3 grid(blocks < most ? blocks : most, p.tab.rows);
    if (p.max_rows == 1) PB_LAUNCH(kv_append_kernel<false>, grid, dim3(256), 0, s, p, rpb, per_row);
    else PB_LAUNCH(kv_append_kernel<true>, grid, dim3(256), 0, s, p, rpb, per_row);
    return hipGetLastError();
}

size_t page_fork_workspace(int out_rows, int n_pages) { return ((size_t)2 * n_pages + 5 * (size_t)out_rows + 1) * 4; }

static int64_t copy_pieces(const PagePool& c) {
    const int64_t chunks = (int64_t)c.page_size * 2 * c.n_kv_heads * c.head_dim / 8;
    return (chunks + PIECE - 1) / PIECE;
}

int64_t page_fork_copies(const ForkParams& p) { return p.out_rows * (int64_t)p.n_layers * copy_pieces(p.pool); }

hipError_t launch_page_fork(const ForkParams& p, hipStream_t s) {
    const int P = p.pool.n_pages;
    const int rows = p.in_rows > p.out_rows ? p.in_rows : p.out_rows;
    if (P <= SMALL_PAGES && rows <= SMALL_ROWS && (int64_t)rows * p.width <= SMALL_ENTRIES) {
        const int lds = 3 * P * 4;
        if (lds > 32 << 10) {  // with the static part more than 64 KB has to be asked for
            const hipError_t e = hipFuncSetAttribute((const void*)fork_places_kernel<true>,
                                                     hipFuncAttributeMaxDynamicSharedMemorySize, lds);
            if (e != hipSuccess) return e;
        }
        PB_LAUNCH(fork_places_kernel<true>, dim3(1), dim3(1024), lds, s, p, FastDiv(p.width));
    } else {
        PB_LAUNCH(fork_counts_kernel, dim3((P + 1023) / 1024), dim3(256), 0, s, p);
        if (rows > 0) PB_LAUNCH(fork_tables_kernel, dim3((p.width + 1023) / 1024, rows), dim3(256), 0, s, p);
        if (p.out_rows > 0) PB_LAUNCH(fork_places_kernel<false>, dim3(1), dim3(1024), 0, s, p, FastDiv(p.width));
    }
    const int64_t most = page_fork_copies(p), pieces = copy_pieces(p.pool);
    if (most > 0)
        PB_LAUNCH(fork_copy_kernel, dim3((unsigned)(most < COPY_BLOCKS ? most : COPY_BLOCKS)), dim3(256), 0, s, p,
                  FastDiv(p.pool.n_kv_heads), FastDiv(p.n_layers), FastDiv((uint32_t)pieces),
                  p.pool.token_stride > p.pool.head_stride);
    return hipGetLastError();
}

}  // namespace pb
