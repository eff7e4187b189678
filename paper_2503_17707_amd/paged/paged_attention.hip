// Attention of one new token per sequence over a paged cache, flash-style: one
// pass over a sequence's keys and values with a running maximum and sum (fp32).
//
// What bounds it is reading the keys and values once: per token and key/value
// head 2 HD elements against 4 HD flops per query head, and with up to 16 query
// heads to a key/value head the matrix units take them all at the price of one.
// So everything here serves loads in flight and an even share of them:
//
//  - A wave takes tiles of 16 or 32 tokens.  Keys go from memory straight into the
//    A operand of v_mfma_f32_16x16x32 (a lane holds 8 consecutive dimensions of one
//    token), S^T[token, query] = K Q^T with the group's queries as the 16 columns.
//    Values are contracted over tokens, which memory does not hold consecutively:
//    they pass through LDS (written by rows, read with the transposing
//    ds_read_b64_tr_b16), O^T[dimension, query] += V^T P^T.  As soon as a tile's
//    registers are free the next tile's loads are issued.  (Two tiles ahead: no
//    faster for few blocks, 10% slower for many, which then hold fewer waves.)
//    Values are read once and by whole lines, so they bypass what caches may keep
//    (131071 tokens: 97 us against 104); a line of keys is read in two halves.
//    Where rows share pages, as beams do, caches serve most reads and are used (4
//    prompts of 1000 with 8 beams each, 32 heads of 64: 28.1 us against 32.7; the same
//    rows on pages of their own: 62.6 against 57.6).
//  - Sequences are cut into pieces, at most as long as a length chosen on the device
//    from the call's lengths (which may change between replays of a recorded launch),
//    so that about PIECES blocks of like work cover a ragged batch as well as one long
//    sequence.  A second launch joins the pieces of sequences that have several; of many
//    sequences one ahead lists the pieces.
//
// Measured, the join with it: 131071 tokens, 32 heads on 8 of 128 (537 MB) 97 us, 5.5
// TB/s; 48 ragged sequences up to 16384, 64 heads on 8 (368 MB) 74 us, 5.0 TB/s; 32 ragged
// up to 2048, 40 heads (198 MB) 45.7 us, 4.3 TB/s; a 4 GiB copy reaches 4.7 TB/s on this card.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
// Tokens per tile: with one operand of queries 16, half the registers and so
// three waves per SIMD instead of two at the same bytes in flight; with more, 32.
template <int NQ> constexpr int tile_of() { return NQ == 1 ? 16 : 32; }
constexpr int IDS = 512;      // pages whose places are held in LDS at a time
// Pieces (us for 48 ragged sequences up to 16384, 64 heads on 8 of 128 | one of 131071,
// 32 on 8 | 8 of 2048, 40 heads of 128): for 1024 blocks 77.0 | 99.5 | 67.9, for 2048
// 73.8 | 96.9 | 68.0.
constexpr int PIECES = 2048;  // blocks aimed at
// No piece is shorter than SHORTEST tokens, nor than LEAST once the blocks of such
// pieces number more than 512: what a block does before its first tile costs as much
// as some 100 tokens.  5 sequences of 1714, 64 heads on 8 of 128: 128 tokens 15.7 us,
// 256 16.2; 32 of 303, 40 heads of 128 in tables of 2080: 256 49.9 us, 512 42.4.
constexpr int SHORTEST = 128, LEAST = 512, FEW_BLOCKS = 512;

// How a call is cut: written to the workspace by the first block, or by a launch before
// (LISTED), and read by the join.
struct Cut {
    int on;        // 0: one piece per sequence, no join
    int qb;        // blocks of 16 NQ query heads per key/value head
    int32_t* at;   // [rows][2] first piece of each sequence, how many
    int most;      // pieces there can be
    int4* list;    // [most] each piece's sequence (-1: none), first token, end and how many
                   // pieces the sequence has (-1: one that is past its table); NULL: not listed
    float* ml;     // [pieces][n_heads][2] maximum (log2 units) and sum
    float* acc;    // [pieces][n_heads][HD] unnormalised output
};

// D[16x16] += A[16x16] B[16x16]: lane l holds A row l % 16, k = 4 (l / 16) .. + 3, and
// B column l % 16 likewise; D as the 16x16x32 product's.
template <typename T> __device__ __forceinline__ f32x4 mma16(u32x2 a, u32x2 b, f32x4 c);
template <> __device__ __forceinline__ f32x4 mma16<_Float16>(u32x2 a, u32x2 b, f32x4 c) {
    typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16f16(__builtin_bit_cast(f16x4, a), __builtin_bit_cast(f16x4, b), c, 0, 0, 0);
}
template <> __device__ __forceinline__ f32x4 mma16<__bf16>(u32x2 a, u32x2 b, f32x4 c) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(s16x4, a), __builtin_bit_cast(s16x4, b), c, 0, 0, 0);
}

template <typename T> __device__ constexpr uint32_t ones2();
template <> __device__ constexpr uint32_t ones2<_Float16>() { return 0x3C003C00u; }
template <> __device__ constexpr uint32_t ones2<__bf16>() { return 0x3F803F80u; }

// A probability enters the products with V as two numbers of the storage type, cut off
// after its first bits and what that leaves: within 2^-21 of it in fp16 and 2^-15 in
// bf16, far below the output's own rounding (rounded to the type alone it showed: up to
// half a step more).  The second product costs 0.4 us on 513 tokens of 32 heads of 64 (6.8),
// nothing where memory is the bound.  No part of a probability that is not 0 is 0
// or negative (the second one is TINY at least), so an infinite value comes through.
// Probabilities are kept times UNIT: an fp16 part vanishes below 2^-25, which then is 2^-40
// of the largest probability, and a hundred thousand of the small ones can matter.
template <typename T> struct Parts;
template <> struct Parts<_Float16> {
    static constexpr float UNIT = 32768.f, TINY = 5.9604644775390625e-8f;  // 2^15, 2^-24
    __device__ static __forceinline__ uint32_t cut2(float a, float b) {
        return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_pkrtz(a, b));
    }
};
template <> struct Parts<__bf16> {
    static constexpr float UNIT = 1.f, TINY = 1.17549435e-38f;  // 2^-126
    __device__ static __forceinline__ uint32_t cut2(float a, float b) {
        return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    }
};
template <typename T>
__device__ __forceinline__ void two_parts(const float (&w)[4], u32x2& first, u32x2& rest) {
    first = u32x2{Parts<T>::cut2(w[0], w[1]), Parts<T>::cut2(w[2], w[3])};
    T f[4];
    __builtin_memcpy(f, &first, 8);
    float d[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) d[r] = fmaxf(w[r] - (float)f[r], fminf(w[r], Parts<T>::TINY));
    rest = pack4<T>(d[0], d[1], d[2], d[3]);
}

// 16-byte chunk of row `row` in a tile of values: the 16 lanes of a transposing
// read address four rows at two neighbouring chunks; (row & 3) and bit 2 of the row
// keep them, and the rows of the next lane group, in different banks.
template <int HD> __device__ __forceinline__ int vswz(int row, int ch) {
    if (HD == 128) return ch ^ ((row & 3) << 1) ^ (((row >> 2) & 1) << 3);
    return ch ^ (((row & 3) ^ ((row >> 2) & 1)) << 1);
}

// Transposing LDS read: within 16 lanes, lane i receives element i % 4 of the
// 8-byte segments addressed by lanes 4 j + i / 4, j = 0..3.
__device__ __forceinline__ u32x2 read_tr16(const uint8_t* p) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(p)));
}

// Maximum over the four lanes that hold a query's scores (l, l ^ 16, l ^ 32, l ^ 48).
__device__ __forceinline__ float group4_max(float v) {
    const auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
    const auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

// Sum over the wave in every lane, and sum over the lanes up to this one: in
// registers (a lane exchange through LDS takes a hundred cycles, and the cut of a
// call needs a dozen of them before the first load).
__device__ __forceinline__ int wave_sum_dpp(int v) {
    v += __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, false);   // quad_perm 1 0 3 2
    v += __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, false);   // quad_perm 2 3 0 1
    v += __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, false);  // row_half_mirror
    v += __builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, false);  // row_mirror
    const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = (int)(a[0] + a[1]);
    const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    return (int)(b[0] + b[1]);
}

__device__ __forceinline__ int wave_scan_dpp(int v) {
    v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr 1
    v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr 2
    v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr 4
    v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr 8
    v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // lane 15 of a row to rows 1, 3
    v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // lane 31 to rows 2, 3
    return v;
}

// LDS written and read by the same wave: its LDS instructions run in order, the
// compiler has to keep them so.
__device__ __forceinline__ void wave_lds_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
    __builtin_amdgcn_wave_barrier();
}

// Tokens of sequence s that its query attends to: [lo, lo + n).  A length past the
// table's width counts as none here and is found out where ids are read.
struct Span {
    int lo, n;
    bool wide;
};
__device__ __forceinline__ Span span_of(const PagedAttentionParams& p, int s) {
    Span r;
    const int len = max(p.lens[s], 0);
    r.wide = len > (int64_t)p.tab.width * p.pool.page_size;
    r.n = r.wide ? 0 : p.window > 0 ? min(len, p.window) : len;
    r.lo = len - r.n;
    return r;
}

// Pieces of this call are at most so long.
__device__ __forceinline__ int piece_length(int64_t tokens, int blocks_per_piece) {
    const int64_t c = (tokens * blocks_per_piece + PIECES - 1) / PIECES;
    const int64_t least = min(max(tokens * blocks_per_piece / FEW_BLOCKS, (int64_t)SHORTEST), (int64_t)LEAST);
    const int64_t m = min(max(c, least), (int64_t)1 << 30);  // no sequence is longer
    return (int)((m + 31) / 32 * 32);
}

__device__ __forceinline__ int pieces_of(int n, int len_c) { return max(1, (n + len_c - 1) / len_c); }

// A sequence's pieces are equally long, whole tiles but for the last.
__device__ __forceinline__ int piece_tokens(int n, int pieces) {
    return pieces == 1 ? n : (n + pieces * 32 - 1) / (pieces * 32) * 32;
}

// Long pieces come first, so that the short ones fill the end.
__device__ __forceinline__ bool is_long(int n, int k, int len_c) { return n >= (int64_t)k * (len_c / 2); }

// The cut of more sequences than LISTED, by one block.  Up to there every wave of the
// attention works it out for itself, which spares 3 us of a launch, but takes lengths
// times blocks, and blocks grow with the lengths (32 heads on 8 of 128 in tables of 16384
// tokens, listed and each wave for itself: 96 sequences up to 2000 80 us and 76, 192 163 and
// 162, 1024 up to 600 241 and 402, 4096 up to 200 416 and 3146; 192 up to 200, 32 heads of
// 64: 39 and 53).
constexpr int LISTED = 128;
__global__ __launch_bounds__(1024) void paged_cut_kernel(PagedAttentionParams p, Cut cut, int hb) {
    __shared__ int64_t tokens_of[16];
    __shared__ int longs_of[16], shorts_of[16];
    const int S = p.tab.rows, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const Span own = tid < S ? span_of(p, tid) : Span{};
    auto span = [&](int i) { return i == tid ? own : span_of(p, i); };
    int low = 0, high = 0;  // (a wave's sums fit: 4096 lengths of up to 2^30)
    for (int i = tid; i < S; i += 1024) {
        const int n = span(i).n;
        low += n & 0x7fff;
        high += n >> 15;
    }
    low = wave_sum_dpp(low);
    high = wave_sum_dpp(high);
    if (lane == 0) tokens_of[wave] = ((int64_t)high << 15) + low;
    __syncthreads();
    int64_t tokens = 0;
    for (int w = 0; w < 16; ++w) tokens += tokens_of[w];
    const int len_c = piece_length(tokens, hb);
    int longs = 0;
    for (int i = tid; i < S; i += 1024) {
        const int n = span(i).n, k = pieces_of(n, len_c);
        longs += is_long(n, k, len_c) ? k : 0;
    }
    longs = wave_sum_dpp(longs);
    if (lane == 0) longs_of[wave] = longs;
    __syncthreads();
    int at_long = 0, at_short = 0;  // of the next 1024 sequences
    for (int w = 0; w < 16; ++w) at_short += longs_of[w];
    for (int i0 = 0; i0 < S; i0 += 1024) {
        const int i = i0 + tid;
        const Span x = i < S ? span(i) : Span{};
        const int k = i < S ? pieces_of(x.n, len_c) : 0;
        const bool lng = is_long(x.n, k, len_c);
        const int l = wave_scan_dpp(lng ? k : 0), s = wave_scan_dpp(lng ? 0 : k);
        __syncthreads();  // what was there was read
        if (lane == 63) {
            longs_of[wave] = l;
            shorts_of[wave] = s;
        }
        __syncthreads();
        int at = (lng ? at_long + l : at_short + s) - k;
        for (int w = 0; w < 16; ++w) {
            if (w < wave) at += lng ? longs_of[w] : shorts_of[w];
            at_long += longs_of[w];
            at_short += shorts_of[w];
        }
        if (i < S) {
            cut.at[2 * i] = at;
            cut.at[2 * i + 1] = k;
        }
        const int len = k > 0 ? piece_tokens(x.n, k) : 0;
        constexpr int OWN = 8;  // pieces that a lane lists by itself, more by the whole wave
        for (int j = 0; j < OWN && j < k; ++j)
            cut.list[at + j] = make_int4(i, x.lo + min(j * len, x.n), x.lo + min(j * len + len, x.n), x.wide ? -1 : k);
        for (uint64_t many = __ballot(k > OWN); many; many &= many - 1) {
            const int who = __ffsll((unsigned long long)many) - 1;
            const int first = __builtin_amdgcn_readlane(at, who), pieces = __builtin_amdgcn_readlane(k, who);
            const int lo = __builtin_amdgcn_readlane(x.lo, who), n = __builtin_amdgcn_readlane(x.n, who);
            const int l = __builtin_amdgcn_readlane(len, who);
            for (int j = OWN + lane; j < pieces; j += 64)
                cut.list[first + j] = make_int4(i - lane + who, lo + min(j * l, n), lo + min(j * l + l, n), pieces);
        }
    }
    for (int j = at_short + tid; j < cut.most; j += 1024) cut.list[j] = make_int4(-1, 0, 0, 0);
}

template <typename T, int HD, int NQ, int NW, bool SHARED>
__global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2)))
void paged_attention_kernel(PagedAttentionParams p, Cut cut) {
    typedef typename Mfma<T>::vec8 vec8;
    constexpr int KT = tile_of<NQ>();
    constexpr int RT = KT / 16;          // 16-token tiles of S^T
    constexpr int CS = HD / 32;          // 32-wide steps over the head
    constexpr int CT = HD / 16;          // 16-row tiles of O^T
    constexpr int CPR = HD / 8;          // 16-byte chunks per token
    constexpr int RPI = 64 / CPR;        // tokens per load instruction of values
    constexpr int NV = KT / RPI;         // ... instructions
    constexpr int VB = KT * HD * 2;      // bytes of a wave's values in LDS
    constexpr int WB = 16 * HD * 4;      // bytes of 16 query heads' fp32 output
    static_assert(WB >= VB, "LDS of a wave");
    __shared__ __attribute__((aligned(16))) uint8_t sv[NW * WB];  // each wave's values, later its output
    __shared__ int64_t places[IDS];      // elements from the pool's base to each page
    __shared__ float wm[NW][16 * NQ], wl[NW][16 * NQ];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int group = p.n_heads / p.pool.n_kv_heads;
    const int hb = p.pool.n_kv_heads * cut.qb;
    // blocks that share keys and values run on one XCD, and its L2 holds them: every
    // eighth block does (4 sequences of 30000, 71 heads on one: 36.4 us; neighbouring blocks: 43.6)
    const int unit = blockIdx.x / (8 * cut.qb) * 8 + blockIdx.x % 8;  // (piece, key/value head)
    const int kvh = unit % p.pool.n_kv_heads, q0 = (int)(blockIdx.x / 8 % cut.qb) * 16 * NQ;
    const int item = unit / p.pool.n_kv_heads;
    int s = item, pieces = 1, slot = 0;
    int ka, kb;         // tokens of this block
    bool wide = false;  // the sequence is past its table
    if (!cut.on && s >= p.tab.rows) return;

    if (cut.list) {
        if (item >= cut.most) return;
        const int4 mine = cut.list[item];
        s = __builtin_amdgcn_readfirstlane(mine.x);
        if (s < 0) return;  // the grid is sized for the most pieces there can be
        ka = __builtin_amdgcn_readfirstlane(mine.y);
        kb = __builtin_amdgcn_readfirstlane(mine.z);
        pieces = __builtin_amdgcn_readfirstlane(mine.w);
        wide = pieces < 0;
        slot = item;
    } else if (cut.on) {
        // Which piece of which sequence: every wave works the cut out for itself from
        // the lengths (a scan over them, without a barrier).
        const int S = p.tab.rows, per = (S + 63) / 64;
        const int s0 = min(lane * per, S), s1 = min(s0 + per, S);
        // tokens in two parts whose sums over 65535 sequences of 2^30 fit 32 bits
        const Span own = s0 < s1 ? span_of(p, s0) : Span{};
        int low = 0, high = 0;
        for (int i = s0; i < s1; ++i) {
            const int n = i == s0 ? own.n : span_of(p, i).n;
            low += n & 0x7fff;
            high += n >> 15;
        }
        const int len_c = piece_length(((int64_t)wave_sum_dpp(high) << 15) + wave_sum_dpp(low), hb);
        int n_long = 0, n_short = 0;  // pieces of this lane's sequences
        for (int i = s0; i < s1; ++i) {
            const int n = i == s0 ? own.n : span_of(p, i).n, k = pieces_of(n, len_c);
            if (is_long(n, k, len_c)) n_long += k; else n_short += k;
        }
        int at_long = wave_scan_dpp(n_long), at_short = wave_scan_dpp(n_short);
        at_short += __builtin_amdgcn_readlane(at_long, 63) - n_short;
        at_long -= n_long;
        int mine = -1, piece = 0;
        Span found{};
        for (int i = s0; i < s1; ++i) {
            const Span x = i == s0 ? own : span_of(p, i);
            const int n = x.n, k = pieces_of(n, len_c);
            int& at = is_long(n, k, len_c) ? at_long : at_short;
            if (item >= at && item < at + k) {
                mine = i;
                found = x;
                piece = item - at;
                pieces = k;
            }
            if (blockIdx.x == 0 && wave == 0) {
                cut.at[2 * i] = at;
                cut.at[2 * i + 1] = k;
            }
            at += k;
        }
        const uint64_t who = __ballot(mine >= 0);
        if (!who) return;
        const int l = __ffsll((unsigned long long)who) - 1;
        s = __builtin_amdgcn_readlane(mine, l);
        piece = __builtin_amdgcn_readlane(piece, l);
        pieces = __builtin_amdgcn_readlane(pieces, l);
        found.lo = __builtin_amdgcn_readlane(found.lo, l);
        found.n = __builtin_amdgcn_readlane(found.n, l);
        wide = __builtin_amdgcn_readlane(found.wide, l);
        const int len = piece_tokens(found.n, pieces);
        ka = found.lo + min(piece * len, found.n);
        kb = found.lo + min(piece * len + len, found.n);
        slot = item;
    } else {
        const Span sp = span_of(p, s);
        wide = sp.wide;
        ka = sp.lo;
        kb = sp.lo + sp.n;
    }
    const int nq = min(group - q0, 16 * NQ);  // query heads of this block
    const int h0 = kvh * group + q0;

    vec8 qf[NQ][CS];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        const uint16_t* qr = p.q + s * p.ld_q + (int64_t)(h0 + min(16 * t + lr, nq - 1)) * HD;
#pragma unroll
        for (int c = 0; c < CS; ++c) qf[t][c] = as_vec8<T>(*(const u32x4*)(qr + c * 32 + lg * 8));
    }
    f32x4 o[NQ][CT], ol[NQ];
    float m[NQ];
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        m[t] = -INFINITY;
        ol[t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < CT; ++c) o[t][c] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const float fold = p.scale * LOG2E;
    const uint16_t* base = p.pool.base + kvh * p.pool.head_stride;
    uint8_t* myv = sv + wave * WB;
    bool bad = wide;

    // IDS pages at a time
    for (int seg = ka; seg < kb && !bad;) {
        const int col0 = (int)p.pool.div.quot(seg);
        const int64_t end = (int64_t)(col0 + IDS) * p.pool.page_size;
        const int seg_end = end < kb ? (int)end : kb;
        const int cols = (int)p.pool.div.quot(seg_end - 1) + 1 - col0;
        const int32_t* row = p.tab.ids + s * p.tab.ld + col0;
        bool wrong = false;
        __syncthreads();
        for (int i = tid; i < cols; i += 64 * NW) {
            const int id = row[i];
            wrong |= id < 0 || id >= p.pool.n_pages;
            places[i] = id * p.pool.page_stride;
        }
        bad = __syncthreads_or(wrong);
        if (bad) break;

        // Address of a token's keys (this head).  The products are what a load costs
        // most in instructions: three of 32 bits here.
        auto token = [&](int key) {
            const uint32_t col = p.pool.div.quot(key), t = key - col * p.pool.page_size;
            return base + (places[col - col0] + (int64_t)((uint64_t)t * (uint32_t)p.pool.token_stride));
        };
        u32x4 kr[RT][CS], vr[NV];
        auto load = [&](int k0) {  // tokens past the end: the last one again
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                const uint16_t* a = token(min(k0 + 16 * i + lr, seg_end - 1)) + lg * 8;
#pragma unroll
                for (int c = 0; c < CS; ++c) kr[i][c] = *(const u32x4*)(a + c * 32);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const u32x4* a = (const u32x4*)(token(min(k0 + i * RPI + lane / CPR, seg_end - 1)) + p.pool.v_offset +
                                                lane % CPR * 8);
                vr[i] = SHARED ? *a : __builtin_nontemporal_load(a);
            }
        };
        int k0 = seg + wave * KT;
        if (k0 < seg_end) load(k0);
        for (; k0 < seg_end; k0 += KT * NW) {
            f32x4 sc[NQ][RT];
#pragma unroll
            for (int t = 0; t < NQ; ++t)
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    sc[t][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int c = 0; c < CS; ++c) sc[t][i] = Mfma<T>::mma(as_vec8<T>(kr[i][c]), qf[t][c], sc[t][i]);
                }
            const bool edge = k0 + KT > seg_end;
            wave_lds_order();
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int r = i * RPI + lane / CPR;
                // no weight reaches tokens past the end, but zero times what is read
                // in their place need not be zero
                if (edge && k0 + r >= seg_end) vr[i] = u32x4{0, 0, 0, 0};
                *(u32x4*)(myv + r * HD * 2 + (vswz<HD>(r, lane % CPR) << 4)) = vr[i];
            }
            wave_lds_order();
            if (k0 + KT * NW < seg_end) load(k0 + KT * NW);

            u32x2 pf[NQ][RT], pr[NQ][RT];  // P^T in its two parts, 4 tokens of a query in each
#pragma unroll
            for (int t = 0; t < NQ; ++t) {
                float mx = -INFINITY;
#pragma unroll
                for (int i = 0; i < RT; ++i)
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        float x = sc[t][i][r] * fold;
                        if (edge && k0 + 16 * i + 4 * lg + r >= seg_end) x = -INFINITY;
                        sc[t][i][r] = x;
                        mx = fmaxf(mx, x);
                    }
                const float m_new = fmaxf(m[t], group4_max(mx));
                const float mb = m_new == -INFINITY ? 0.f : m_new;  // nothing but -inf so far: all weights 0
                const float alpha = __builtin_amdgcn_exp2f(m[t] - mb);
                m[t] = m_new;
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    float w[4];
#pragma unroll
                    // (UNIT comes in last: far from zero mb - 15 would be rounded, and a weight of
                    // 2^16 is fp16's infinity)
                    for (int r = 0; r < 4; ++r) w[r] = __builtin_amdgcn_exp2f(sc[t][i][r] - mb) * Parts<T>::UNIT;
                    two_parts<T>(w, pf[t][i], pr[t][i]);
                }
                if (__any(alpha != 1.f)) {
#pragma unroll
                    for (int c = 0; c < CT; ++c)
#pragma unroll
                        for (int r = 0; r < 4; ++r) o[t][c][r] *= alpha;
#pragma unroll
                    for (int r = 0; r < 4; ++r) ol[t][r] *= alpha;
                }
            }
            // V^T operand, row c: tokens 16 i + 4 lg + j, in the order in which a lane
            // holds its probabilities
            const uint32_t one = ones2<T>();
#pragma unroll
            for (int c = 0; c <= CT; ++c) {
                u32x2 v[RT];
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    if (c < CT) {
                        const int r = 16 * i + 4 * lg + (lr >> 2);
                        const int col = 16 * c + 4 * (lr & 3);
                        v[i] = read_tr16(myv + r * HD * 2 + (vswz<HD>(r, col >> 3) << 4) + (col & 7) * 2);
                    } else {
                        // the sum of the probabilities as they enter the products
                        v[i] = u32x2{one, one};
                    }
                }
#pragma unroll
                for (int t = 0; t < NQ; ++t) {
                    f32x4& d = c < CT ? o[t][c < CT ? c : 0] : ol[t];
                    if constexpr (RT == 2) {
                        const auto vv = as_vec8<T>(u32x4{v[0][0], v[0][1], v[1][0], v[1][1]});
                        d = Mfma<T>::mma(vv, as_vec8<T>(u32x4{pf[t][0][0], pf[t][0][1], pf[t][1][0], pf[t][1][1]}), d);
                        d = Mfma<T>::mma(vv, as_vec8<T>(u32x4{pr[t][0][0], pr[t][0][1], pr[t][1][0], pr[t][1][1]}), d);
                    } else {
                        d = mma16<T>(v[0], pf[t][0], d);
                        d = mma16<T>(v[0], pr[t][0], d);
                    }
                }
            }
        }
        seg = seg_end;
    }

    // join the waves, 16 query heads at a time
    if (lg == 0)
#pragma unroll
        for (int t = 0; t < NQ; ++t) {
            wm[wave][16 * t + lr] = m[t];
            wl[wave][16 * t + lr] = ol[t][0];
        }
    const int q = tid / (4 * NW);       // 4 NW threads to a query head
#pragma unroll
    for (int t = 0; t < NQ; ++t) {
        if (16 * t >= nq) break;
        __syncthreads();
#pragma unroll
        for (int c = 0; c < CT; ++c)
            *(f32x4*)(sv + wave * WB + lr * HD * 4 + (((4 * c + lg) ^ lr) << 4)) = o[t][c];
        __syncthreads();
        if (16 * t + q >= nq) continue;
        float M = -INFINITY, L = 0.f, f[NW];
#pragma unroll
        for (int w = 0; w < NW; ++w) M = fmaxf(M, wm[w][16 * t + q]);
        const float Mb = M == -INFINITY ? 0.f : M;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            f[w] = __builtin_amdgcn_exp2f(wm[w][16 * t + q] - Mb);
            L += f[w] * wl[w][16 * t + q];
        }
        if (bad) L = NAN;
        const int h = h0 + 16 * t + q;
        const bool empty = ka == kb && !bad;  // (of a sequence in one piece)
#pragma unroll
        for (int j = 0; j < (HD + 16 * NW - 1) / (16 * NW); ++j) {
            const int ch = j * 4 * NW + tid % (4 * NW);  // 4 dimensions
            if (4 * ch >= HD) break;
            f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int w = 0; w < NW; ++w) {
                const f32x4 x = *(const f32x4*)(sv + w * WB + q * HD * 4 + ((ch ^ q) << 4));
#pragma unroll
                for (int r = 0; r < 4; ++r) a[r] += f[w] * x[r];
            }
            if (pieces > 1) {
                *(f32x4*)(cut.acc + ((int64_t)slot * p.n_heads + h) * HD + 4 * ch) = a;
            } else {
                const float inv = empty ? 0.f : 1.f / L;
                *(u32x2*)(p.out + s * p.ld_out + (int64_t)h * HD + 4 * ch) =
                    pack4<T>(a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
            }
        }
        if (pieces > 1 && tid % (4 * NW) == 0) {
            cut.ml[((int64_t)slot * p.n_heads + h) * 2] = M;
            cut.ml[((int64_t)slot * p.n_heads + h) * 2 + 1] = L;
        }
    }
}

// Joins the pieces of sequences with several: 4 TX dimensions of the heads' row per
// block, TX threads across them, the 256 / TX others taking pieces in turn.
template <typename T, int HD, int TX>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedAttentionParams p, Cut cut) {
    constexpr int TY = 256 / TX;
    __shared__ f32x4 sa[TY][TX];
    __shared__ float sm[TY][TX];
    const int s = blockIdx.y;
    const int i0 = cut.at[2 * s], n = cut.at[2 * s + 1];
    if (n <= 1) return;
    const int x = threadIdx.x % TX, y = threadIdx.x / TX;
    const int d = (blockIdx.x * TX + x) * 4, h = d / HD;
    const int64_t rows = p.n_heads;
    const float2* ml = (const float2*)cut.ml + i0 * rows + h;
    const float* acc = cut.acc + i0 * rows * HD + d;
    // the first HOLD pieces of a thread are on their way before the maximum is known
    constexpr int HOLD = 4;
    float2 w[HOLD];
    f32x4 v[HOLD];
    float M = -INFINITY;
#pragma unroll
    for (int j = 0; j < HOLD; ++j) {
        const int i = min(y + j * TY, n - 1);
        w[j] = ml[i * rows];
        v[j] = *(const f32x4*)(acc + i * rows * HD);
        M = fmaxf(M, w[j].x);
    }
    for (int i = y + HOLD * TY; i < n; i += TY) M = fmaxf(M, ml[i * rows].x);
    sm[y][x] = M;
    __syncthreads();
#pragma unroll
    for (int j = 0; j < TY; ++j) M = fmaxf(M, sm[j][x]);
    f32x4 a = f32x4{0.f, 0.f, 0.f, 0.f};
    float L = 0.f;
    auto add = [&](float2 u, f32x4 o) {
        const float f = __builtin_amdgcn_exp2f(u.x - M);
        L += f * u.y;
#pragma unroll
        for (int r = 0; r < 4; ++r) a[r] += f * o[r];
    };
#pragma unroll
    for (int j = 0; j < HOLD; ++j)
        if (y + j * TY < n) add(w[j], v[j]);
#pragma unroll 4
    for (int i = y + HOLD * TY; i < n; i += TY) add(ml[i * rows], *(const f32x4*)(acc + i * rows * HD));
    __syncthreads();  // the maxima were read
    sa[y][x] = a;
    sm[y][x] = L;
    __syncthreads();
    if (y == 0) {
#pragma unroll
        for (int j = 1; j < TY; ++j) {
            L += sm[j][x];
#pragma unroll
            for (int r = 0; r < 4; ++r) a[r] += sa[j][x][r];
        }
        const float inv = 1.f / L;
        *(u32x2*)(p.out + s * p.ld_out + d) = pack4<T>(a[0] * inv, a[1] * inv, a[2] * inv, a[3] * inv);
    }
}

template <typename T, int HD>
void launch_join(const PagedAttentionParams& p, const Cut& cut, hipStream_t s) {
    // as wide as leaves 512 blocks; the widest one (64) keeps a batch's launch small
    const int quads = p.n_heads * HD / 4;
    const dim3 block(256);
    if ((int64_t)(quads / 16) * p.tab.rows < 512 || quads % 16)
        PB_LAUNCH((paged_join_kernel<T, HD, 8>), dim3(quads / 8, p.tab.rows), block, 0, s, p, cut);
    else if ((int64_t)(quads / 64) * p.tab.rows < 512 || quads % 64)
        PB_LAUNCH((paged_join_kernel<T, HD, 16>), dim3(quads / 16, p.tab.rows), block, 0, s, p, cut);
    else
        PB_LAUNCH((paged_join_kernel<T, HD, 64>), dim3(quads / 64, p.tab.rows), block, 0, s, p, cut);
}

// Most pieces a call can have: PIECES blocks' worth and the remainder of each
// sequence, or every sequence at its `longest` cut into shortest pieces.
int64_t most_pieces(int rows, int hb, int64_t longest) {
    const int64_t each = (longest + SHORTEST - 1) / SHORTEST;
    const int64_t a = PIECES / hb + rows, b = rows * each;
    return a < b ? a : b;
}

// Blocks of a launch; its threads are counted in 32 bits, 256 to a block.
constexpr int64_t MOST_BLOCKS = 1 << 24;
int64_t grid_blocks(int64_t items, int n_kv_heads, int qb) { return (items * n_kv_heads + 7) / 8 * 8 * qb; }

// The cut and the list of pieces (multiples of 16 bytes), their partial results.
size_t at_bytes(int rows) { return ((size_t)rows * 8 + 15) / 16 * 16; }
size_t list_bytes(int rows, int64_t pieces) { return rows > LISTED ? (size_t)pieces * 16 : 0; }
size_t cut_bytes(int rows, int64_t pieces, int n_heads, int hd) {
    return at_bytes(rows) + list_bytes(rows, pieces) + (size_t)pieces * n_heads * (hd + 2) * 4;
}

template <typename T, int HD, bool SHARED>
hipError_t launch(const PagedAttentionParams& p, hipStream_t s) {
    const int group = p.n_heads / p.pool.n_kv_heads;
    int nq = group <= 16 ? 1 : 2;
    Cut cut{};
    cut.qb = (group + 16 * nq - 1) / (16 * nq);
    int hb = p.pool.n_kv_heads * cut.qb;
    int64_t items = p.tab.rows;
    const int64_t held = (int64_t)p.tab.width * p.pool.page_size;
    const int64_t longest = p.window > 0 && p.window < held ? p.window : held;  // that is attended to
    const int64_t most = most_pieces(p.tab.rows, hb, longest);
    // Short sequences stay whole: the join costs 4 us (one of 513, 32 heads of 64: 6.8
    // us, cut 9.3), and so do longer ones that fill the chip as they are (8 of 1000: 14.2,
    // cut 18.6; one of 2000: 11.7 cut, 18.1 whole).  With heads of 128 a few blocks take longer
    // (32 blocks of 600: 10.5, of 1000 16.5; cut 10.6 and 12.2; 128 of 1000: 18.4, cut 19.8).
    const int64_t whole = (int64_t)p.tab.rows * hb;
    const int uncut = HD == 64 ? (whole >= 256 ? 2048 : 1024) : (whole >= 64 ? 1024 : 640);
    if (longest > uncut && most > p.tab.rows && grid_blocks(most, p.pool.n_kv_heads, cut.qb) < MOST_BLOCKS && p.ws &&
        p.ws_bytes >= cut_bytes(p.tab.rows, most, p.n_heads, HD)) {
        cut.on = 1;
        cut.most = (int)most;
        cut.at = (int32_t*)p.ws;
        const size_t list = list_bytes(p.tab.rows, most);
        if (list) cut.list = (int4*)((char*)p.ws + at_bytes(p.tab.rows));
        cut.acc = (float*)((char*)p.ws + at_bytes(p.tab.rows) + list);
        cut.ml = cut.acc + (size_t)most * p.n_heads * HD;
        items = most;
    }
    // Whole sequences of more than 16 heads to a key/value head that leave the chip mostly
    // idle: more blocks of 16 heads, on the caches (12 ragged of 662, 71 heads on one of
    // 128: 11.1 us, 15.7 with 32; 100 of 500 would be 500 blocks: 26.7 us against 20.8).
    const int qb1 = (group + 15) / 16;
    if (nq == 2 && !cut.on && items * p.pool.n_kv_heads * qb1 <= 256) {
        nq = 1;
        cut.qb = qb1;
        hb = p.pool.n_kv_heads * qb1;
    }
    const dim3 grid((unsigned)grid_blocks(items, p.pool.n_kv_heads, cut.qb));
    if (cut.list) PB_LAUNCH(paged_cut_kernel, dim3(1), dim3(1024), 0, s, p, cut, hb);
    // Few uncut blocks: eight waves each (8 sequences of 1000, 32 heads of 64: 14.2 us,
    // four 17.0); cut ones have little to share out.
    if (nq == 1 && !cut.on && items * hb < 512)
        PB_LAUNCH((paged_attention_kernel<T, HD, 1, 8, SHARED>), grid, dim3(512), 0, s, p, cut);
    else if (nq == 1) PB_LAUNCH((paged_attention_kernel<T, HD, 1, 4, SHARED>), grid, dim3(256), 0, s, p, cut);
    else PB_LAUNCH((paged_attention_kernel<T, HD, 2, 4, SHARED>), grid, dim3(256), 0, s, p, cut);
    if (cut.on) launch_join<T, HD>(p, cut, s);
    return hipGetLastError();
}

template <typename T, int HD>
hipError_t launch_shared(const PagedAttentionParams& p, hipStream_t s) {
    // more than 32 heads to a key/value head: several blocks read the same values too
    // (4 sequences of 30000, 71 heads on one: 36.4 us against 39.9)
    const bool shared = p.shared || p.n_heads / p.pool.n_kv_heads > 32;
    return shared ? launch<T, HD, true>(p, s) : launch<T, HD, false>(p, s);
}

}  // namespace

size_t paged_attention_workspace(int n_seqs, int n_heads, int n_kv_heads, int hd, int width, int page_size) {
    const int group = n_heads / n_kv_heads, nq = group <= 16 ? 1 : 2;
    const int64_t most = most_pieces(n_seqs, n_kv_heads * ((group + 16 * nq - 1) / (16 * nq)), (int64_t)width * page_size);
    return most > n_seqs ? cut_bytes(n_seqs, most, n_heads, hd) : 0;
}

bool paged_attention_fits(int n_seqs, int n_heads, int n_kv_heads) {
    const int group = n_heads / n_kv_heads, nq = group <= 16 ? 1 : 2;
    return grid_blocks(n_seqs, n_kv_heads, (group + 16 * nq - 1) / (16 * nq)) < MOST_BLOCKS;
}

hipError_t launch_paged_attention(int dtype, const PagedAttentionParams& p, hipStream_t s) {
    if (p.tab.rows <= 0) return hipSuccess;
    if (p.pool.head_dim == 64) return dtype == 1 ? launch_shared<_Float16, 64>(p, s) : launch_shared<__bf16, 64>(p, s);
    return dtype == 1 ? launch_shared<_Float16, 128>(p, s) : launch_shared<__bf16, 128>(p, s);
}

}  // namespace pb
