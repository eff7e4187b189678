// Products of 8-bit rows: out[M, N] from X[M, K] W[N, K]^T, exact in 32-bit integers
// (v_mfma_i32_16x16x64_i8), times the scales of token m and channel n, with the
// epilogues of the decoder's projections.
//
// As in the 16-bit products the MFMA's A operand is the weight rows (output features
// n) and its B operand the tokens m: a lane ends up with four consecutive features of
// one token.  Lane l gives 16 bytes of row l % 16, the 16 at K offset 16 (l / 16) of
// the step's 64; which of the 64 a lane holds does not matter as long as both operands
// agree, and sums of integers do not depend on their order: every kernel and split gives
// the same bits, so a rule of predicted times chooses freely among them (gemm_q8_plan.h).
//
// What bounds them: one to some sixty tokens, reading the weights once; thousands, the
// matrix units (2 M N K operations, twice those of 16 bits a cycle) about as much as the
// copies that feed them; between, the copies alone (see the wide tiles).
#include <type_traits>

#include "../csrc/common.h"
#include "gemm_q8_plan.h"

namespace pb {

using namespace q8;

namespace {

typedef int32_t i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ i32x4 mma8(i32x4 a, i32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
}

template <typename T>
__device__ __forceinline__ void store4(T* p, int left, const float (&y)[4]) {
    T t[4] = {(T)y[0], (T)y[1], (T)y[2], (T)y[3]};
    if (left >= 4) {
        __builtin_memcpy(p, t, sizeof(t));
    } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < left) p[r] = t[r];
    }
}

template <typename T>
__device__ __forceinline__ void load4(const T* p, int left, T (&t)[4]) {
    if (left >= 4) {
        __builtin_memcpy(t, p, sizeof(t));
    } else {
#pragma unroll
        for (int r = 0; r < 4; ++r) t[r] = r < 3 && r < left ? p[r] : T();
    }
}

// What the epilogue knows of features n .. n+3: loaded first, made ready when the loads of
// a wave's features, scales and old values are all on their way.
struct Features {
    float sw[4], b[4];
    uint16_t bias[4];
    int left;  // of them inside N: 4 or more, or fewer
};

__device__ __forceinline__ Features load_features(const GemmQ8Params& p, int n) {
    Features f;
    f.left = p.N - n;
    load4(p.sw + n, f.left, f.sw);
#pragma unroll
    for (int r = 0; r < 4; ++r) f.bias[r] = 0;  // (zero in both types)
    if (p.bias) load4((const uint16_t*)p.bias + n, f.left, f.bias);
    return f;
}

__device__ __forceinline__ void ready(const GemmQ8Params& p, Features& f) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float wide = __uint_as_float((uint32_t)f.bias[r] << 16);
        f.b[r] = p.bf16 ? wide : (float)__builtin_bit_cast(_Float16, f.bias[r]);
    }
}

// What the residual stream holds there (asked for before the sums are at hand; a load after
// another feature's store would wait for it).
__device__ __forceinline__ void load_old(const GemmQ8Params& p, int m, int n, int left, float (&old)[4]) {
    if (p.epi == Q8_RESID) load4((const float*)p.out + (int64_t)m * p.ldo + n, left, old);
}

// (the sum rounded to fp32, times sx) times sw plus bias, the second product and the sum
// rounded once; then ReLU or the scale of the first qcols features.
__device__ __forceinline__ void values(const GemmQ8Params& p, int epi, int n, float sx, const Features& f, i32x4 acc,
                                       float (&y)[4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        y[r] = fmaf((float)acc[r] * sx, f.sw[r], f.b[r]);
        if (epi == Q8_RELU) y[r] = y[r] < 0.f ? 0.f : y[r];  // (NaN stays)
        if (epi == Q8_QKV) y[r] *= n + r < p.qcols ? p.qscale : 1.f;
        // the 16-bit rounding apart from the product before it, in every kernel
        asm volatile("" : "+v"(y[r]));
    }
}

// Features n .. n+3 of token m.  Rows of the output may start at any element (N odd): vectors
// go there as they come.
__device__ __forceinline__ void epilogue8(const GemmQ8Params& p, int m, int n, float sx, const Features& f, i32x4 acc,
                                          const float (&old)[4]) {
    float y[4];
    values(p, p.epi, n, sx, f, acc, y);
    const int64_t at = (int64_t)m * p.ldo + n;
    if (p.epi >= Q8_RESID) {
        if (p.epi == Q8_RESID) {
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] += old[r];
        }
        store4((float*)p.out + at, f.left, y);
    } else if (p.bf16) {
        store4((__bf16*)p.out + at, f.left, y);
    } else {
        store4((_Float16*)p.out + at, f.left, y);
    }
}

// ---- which block does what ----------------------------------------------------------

// The hardware deals consecutive blocks round-robin to the 8 XCDs: piece i of n such that
// each XCD gets a contiguous run of pieces.
__device__ __forceinline__ int of_xcd(int i, int n) {
    const int x = i & 7, each = n >> 3, rest = n & 7;
    return x * each + min(x, rest) + (i >> 3);
}

struct Job {
    int m0, n0, t0, nk;  // corner; first K tile and how many
    int phase;           // the one of them that a ring begins with
    bool last, partial;  // takes what lies past the last whole K tile; leaves sums
    int32_t* sums;       // [BM][BN]
};

// Tiles are walked in groups of 8 tile-rows: blocks that share an XCD's L2 share rows of
// X and of W.
constexpr int GROUP_M = 8;

template <int BM, int BN>
__device__ __forceinline__ void tile_corner(const GemmQ8Params& p, int tile, int& m0, int& n0) {
    const int tiles_m = (p.M + BM - 1) / BM, tiles_n = (p.N + BN - 1) / BN;
    const int per_group = GROUP_M * tiles_n;
    const int first_m = (tile / per_group) * GROUP_M;
    const int rows = min(tiles_m - first_m, GROUP_M);
    m0 = (first_m + (tile % per_group) % rows) * BM;
    n0 = ((tile % per_group) / rows) * BN;
}

template <int BM, int BN, int BK>
__device__ __forceinline__ Job tile_job(const GemmQ8Params& p, const Split& sp) {
    const int bid = (int)blockIdx.x, nblk = (int)gridDim.x;
    const int whole = p.K / BK;
    Job j;
    int tile;
    if (bid < sp.full) {
        tile = of_xcd(bid, sp.full);
        j.t0 = 0;
        j.nk = whole;
        j.last = true;
        j.partial = false;
        j.sums = nullptr;
    } else {
        const int r = of_xcd(bid - sp.full, nblk - sp.full);
        const int i = r % sp.tail, s = r / sp.tail;
        tile = sp.full + i;
        j.t0 = s * sp.kt;
        j.last = s == sp.splits - 1;
        j.nk = j.last ? whole - j.t0 : sp.kt;
        j.partial = true;
        j.sums = p.ws + ((int64_t)s * sp.tail + i) * (BM * BN);
    }
    tile_corner<BM, BN>(p, tile, j.m0, j.n0);
    j.phase = (int)((uint32_t)(j.n0 / BN) % (uint32_t)sp.phases) * j.nk / sp.phases;
    return j;
}

// A wave's sums as they are stored where all of its features are inside N.  No branch but for
// the last token, the next row's old values asked for before this one's stores (with branches on
// kind, type and edge about every four features and loads between the stores: 1633 x 16384 x
// 4096 onto the stream 169 us, now 144, in fp16 136, now 110; 4096 x 16384 x 4096 in fp16 277
// and 235).
template <typename T, int EPI, int MF, int NF>
__device__ __forceinline__ void store_inside(const GemmQ8Params& p, int mb, int nb, int lr, int lg, const float (&sx)[MF],
                                             Features (&f)[NF], const i32x4 (&acc)[NF][MF]) {
    constexpr bool ADD = EPI == Q8_RESID;
    T* out = (T*)p.out + (int64_t)(mb + lr) * p.ldo + (nb + 4 * lg);
    const T* next = out;
    float old[2][NF][4];
    auto load_row = [&](int j) {
        if (mb + 16 * j + lr < p.M) {
#pragma unroll
            for (int i = 0; i < NF; ++i) __builtin_memcpy(old[j & 1][i], next + 16 * i, sizeof(old[0][0]));
        }
        next += 16 * p.ldo;
    };
    if (ADD) load_row(0);
#pragma unroll
    for (int i = 0; i < NF; ++i) ready(p, f[i]);
#pragma unroll
    for (int j = 0; j < MF; ++j, out += 16 * p.ldo) {
        asm volatile("" : "+v"(out));  // (one row's address at a time)
        if (ADD && j + 1 < MF) load_row(j + 1);
        if (mb + 16 * j + lr >= p.M) continue;
        T t[NF][4];
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            float y[4];
            values(p, EPI, nb + 16 * i + 4 * lg, sx[j], f[i], acc[i][j], y);
#pragma unroll
            for (int r = 0; r < 4; ++r) t[i][r] = (T)(ADD ? y[r] + old[j & 1][i][r] : y[r]);
        }
        if constexpr (sizeof(T) == 2 && NF % 2 == 0) {
            // two fragments' features 4 lg .. + 3 become one's 8 (lg / 2) .. + 7, a whole 16 bytes
#pragma unroll
            for (int i = 0; i < NF; i += 2) {
                uint32_t a[2], b[2];
                __builtin_memcpy(a, t[i], sizeof(a));
                __builtin_memcpy(b, t[i + 1], sizeof(b));
                const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
                const auto hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
                const uint32_t w[4] = {lo[0], hi[0], lo[1], hi[1]};
                __builtin_memcpy(out + 16 * i + 12 * (lg & 1), w, sizeof(w));
            }
        } else {
#pragma unroll
            for (int i = 0; i < NF; ++i) __builtin_memcpy(out + 16 * i, t[i], sizeof(t[i]));
        }
    }
}

// A wave's sums: acc[i][j] holds features nb + 16 i + 4 lg + r of token mb + 16 j + lr.
template <int BN, int MF, int NF>
__device__ __forceinline__ void store_tile(const GemmQ8Params& p, const Job& jb, int mb, int nb, int lr, int lg,
                                           const i32x4 (&acc)[NF][MF]) {
    if (jb.partial) {
#pragma unroll
        for (int j = 0; j < MF; ++j) {
            const int m = mb + 16 * j + lr;
            if (m >= p.M) continue;
#pragma unroll
            for (int i = 0; i < NF; ++i)
                *(i32x4*)(jb.sums + (int64_t)(m - jb.m0) * BN + (nb + 16 * i + 4 * lg - jb.n0)) = acc[i][j];
        }
        return;
    }
    Features f[NF];
#pragma unroll
    for (int i = 0; i < NF; ++i) f[i] = load_features(p, nb + 16 * i + 4 * lg);
    float sx[MF];
#pragma unroll
    for (int j = 0; j < MF; ++j) sx[j] = p.sx[min(mb + 16 * j + lr, p.M - 1)];
    const bool inside = nb + 16 * NF <= p.N;
    if (inside) {
        auto store = [&](auto kind, auto type) {
            store_inside<decltype(type), decltype(kind)::value>(p, mb, nb, lr, lg, sx, f, acc);
        };
        if (p.epi == Q8_RESID) store(std::integral_constant<int, Q8_RESID>(), 0.f);
        else if (p.epi == Q8_LOGITS) store(std::integral_constant<int, Q8_LOGITS>(), 0.f);
        else if (p.epi == Q8_RELU && p.bf16) store(std::integral_constant<int, Q8_RELU>(), (__bf16)0);
        else if (p.epi == Q8_RELU) store(std::integral_constant<int, Q8_RELU>(), (_Float16)0);
        else if (p.bf16) store(std::integral_constant<int, Q8_QKV>(), (__bf16)0);
        else store(std::integral_constant<int, Q8_QKV>(), (_Float16)0);
        return;
    }
#pragma unroll
    for (int i = 0; i < NF; ++i) ready(p, f[i]);
#pragma unroll
    for (int j = 0; j < MF; ++j) {
        const int m = mb + 16 * j + lr;
        if (m >= p.M) continue;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            const int n = nb + 16 * i + 4 * lg;
            float old[4] = {};
            if (f[i].left > 0) load_old(p, m, n, f[i].left, old);
            if (f[i].left > 0) epilogue8(p, m, n, sx[j], f[i], acc[i][j], old);
        }
    }
}

// What lies past the last whole K tile (K is a multiple of 16, a lane's 16 bytes are in
// or out as a whole), straight from memory.
template <int MF, int NF>
__device__ __forceinline__ void add_rest(const GemmQ8Params& p, int k0, int mb, int nb, int lr, int lg,
                                         i32x4 (&acc)[NF][MF]) {
    for (int k = k0 + 16 * lg; k - 16 * lg < p.K; k += 64) {
        i32x4 a[NF], b[MF];
        const bool in = k < p.K;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            a[i] = i32x4{0, 0, 0, 0};
            if (in) a[i] = *(const i32x4*)(p.W + (int64_t)min(nb + 16 * i + lr, p.N - 1) * p.ldw + k);
        }
#pragma unroll
        for (int j = 0; j < MF; ++j) {
            b[j] = i32x4{0, 0, 0, 0};
            if (in) b[j] = *(const i32x4*)(p.X + (int64_t)min(mb + 16 * j + lr, p.M - 1) * p.ldx + k);
        }
#pragma unroll
        for (int i = 0; i < NF; ++i)
#pragma unroll
            for (int j = 0; j < MF; ++j) acc[i][j] = mma8(a[i], b[j], acc[i][j]);
    }
}

// 16-byte chunks of a row past the start of a line of 128 bytes (rows are a multiple of 16 bytes
// apart, so rows 8 apart have the same).
__device__ __forceinline__ uint32_t turn_of(const int8_t* base, int64_t ld, uint32_t row) {
    return ((uint32_t)((uintptr_t)base >> 4) + row * (uint32_t)(ld >> 4)) & 7;
}

// ---- 256-feature tiles: two wave groups in ping-pong ----------------------------------
// 64 XF tokens x 256 features, eight waves (2 x 4) of 32 XF x 64, K tiles of 128 bytes in
// two LDS stages, filled by LDS-DMA.  A K tile is four phases, one per quadrant of the
// wave tile, and a phase has two slots, each closed by a barrier: a memory slot (operand
// reads of the quadrant into registers, one or two copies) and a product slot (4 XF
// products at raised wave priority).  Waves 4-7 run one slot behind waves 0-3 and share
// their SIMDs: one of the two is always in its product slot while the other reads LDS.
//
// A stage is four regions in order of need: Wa (32 of each wave's 64 features), X0 (half
// of its tokens), Wb, X1.  Quadrants go (Wa, X0), (Wb, X0), (Wb, X1), (Wa, X1); Wa of the
// next tile is read in the last phase, into the registers of this tile's Wb, so even
// tiles start with feature half 0 and odd ones with half 1.  A region is free once both
// groups have read it, one slot later, and is then refilled with tile t + 2: a copy has
// seven phases to land, and every wait is for all but the youngest one and a half tiles
// of a wave's copies.  Past the last tile the copies re-read it (nobody reads them).
// LDS rows are 128 bytes, 16-byte chunks XOR-permuted by row & 7: operand reads of 16
// rows are free of bank conflicts.
//
// 4096 x 36864 x 9216: 980-1016 us, 2.7-2.8 POP/s (the vendor library's 8-bit product 1212 us).  All
// tile heights copy 42-46 GB/s a CU (11 TB/s in all) into LDS, and that is the bound: one
// round of 240 blocks (M 1511, N 4992, K 5120) takes 46.8 us with cold weights, 45 with a
// sixteenth of its products, 36.7 if every copy finds its lines in the L2, 32.4 without
// copies; of the large tile of 4096 tokens products and copies alone take 0.87 of the time
// each.  So a block takes as many tokens as fill tiles.  Two phases a tile, three stages, stages
// of uneven depth for tokens and weights and K ranges that start apart took as long, weights
// from memory into registers 1.7 times as long.
//
// SKEW: rows off 128 bytes in three stages, pieces as in the ring below (1511 x 4999 x 5104 67 ->
// 54 us; three stages of taller tiles do not fit).  Piece t + 3 goes where piece t was, in the
// same order and slots: it is asked for three tiles ahead and first read two tiles ahead.
template <int XF, bool SKEW>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2))) void q8_wide_kernel(GemmQ8Params p, Split sp) {
    constexpr int BM = 64 * XF, BN = 256, RB = 128;
    constexpr int XH = 16 * XF;                // tokens of a wave's X half
    constexpr int XC = BM / 2 / 8;             // copies of an X region
    constexpr int XQ = (XC + 7) / 8;           // ... per wave (XF = 3: four waves repeat the last one)
    constexpr int LAG = (4 + 2 * XQ) * 3 / 2;  // copies younger than the one a slot needs
    constexpr int STAGE = (BM + BN) * RB;
    constexpr int S = SKEW ? 3 : 2;
    __shared__ __attribute__((aligned(16))) uint8_t smem[S * STAGE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave & 1, wn = wave >> 1;
    const Job jb = tile_job<BM, BN, RB>(p, sp);
    const int m0 = jb.m0, n0 = jb.n0, nk = jb.nk;

    // copies: region X h is token rows (2 g + h) XH .. + XH - 1 (g = 0, 1), region W h
    // feature rows 64 g + 32 h .. + 31 (g = 0 .. 3), 8 rows per copy; copy q of this wave
    // is number wave + 8 q of its region.  Lane i writes row i / 8, physical chunk i % 8.
    // Rows past the edge re-read the last one.
    const int lrow = lane >> 3, chk = ((lane & 7) ^ lrow) * 16;
    const int lr = lane & 15, lg = lane >> 4;
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int8_t* Xb = p.X + (int64_t)m0 * p.ldx + (int64_t)jb.t0 * RB;
    const int8_t* Wb = p.W + (int64_t)n0 * p.ldw + (int64_t)jb.t0 * RB;
    // SKEW: rows 8 apart have the same turn, so a lane's chunks are late in all copies of X or W
    // or in none (rows past the edge too: only where they start, not what is in range, goes by it)
    const uint32_t begin_x = SKEW && chk / 16 + turn_of(Xb, p.ldx, lrow) < 8 ? RB : 0;
    const uint32_t begin_w = SKEW && chk / 16 + turn_of(Wb, p.ldw, lrow) < 8 ? RB : 0;
    int xrow[2 * XQ], wrow[4];  // first row of copy q of region h: [XQ h + q], [2 h + q]
    uint32_t xoff[2 * XQ], woff[4];
#pragma unroll
    for (int i = 0; i < 2 * XQ; ++i) {
        const int h = i / XQ, c = min(wave + 8 * (i % XQ), XC - 1);
        xrow[i] = (2 * (c / (XC / 2)) + h) * XH + (c % (XC / 2)) * 8;
        xoff[i] = (uint32_t)min(xrow[i] + lrow, p.M - 1 - m0) * (uint32_t)p.ldx + chk + begin_x;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int h = i >> 1, c = wave + 8 * (i & 1);
        wrow[i] = (c >> 2) * 64 + h * 32 + (c & 3) * 8;
        woff[i] = (uint32_t)min(wrow[i] + lrow, p.N - 1 - n0) * (uint32_t)p.ldw + chk + begin_w;
    }
    // piece t; SKEW: counted from a tile before, of the first and last what is inside the range
    const int last = SKEW ? nk : nk - 1;  // (a launch has a K tile for every block)
    auto place = [&](uint32_t off, int t, uint32_t begin) -> uint32_t {
        if constexpr (!SKEW) return off;
        if (t == 0 && begin == 0) return off - chk + RB;
        return t == last ? off - begin : off;
    };
    auto copy_x = [&](int t, uint32_t stage, int h) {
        const int8_t* b = Xb + (int64_t)(SKEW ? t - 1 : t) * RB;
#pragma unroll
        for (int i = XQ * h; i < XQ * h + XQ; ++i) dma16s(b, place(xoff[i], t, begin_x), lds0 + stage + xrow[i] * RB);
    };
    auto copy_w = [&](int t, uint32_t stage, int h) {
        const int8_t* b = Wb + (int64_t)(SKEW ? t - 1 : t) * RB;
#pragma unroll
        for (int i = 2 * h; i < 2 * h + 2; ++i) dma16s(b, place(woff[i], t, begin_w), lds0 + stage + (BM + wrow[i]) * RB);
    };

    i32x4 acc[4][2 * XF] = {};
    i32x4 w0[2][2], w1[2][2], x[XF][2];  // [fragment][k half]
    const uint32_t lk[2] = {(uint32_t)(lr * RB + ((lg ^ (lr & 7)) << 4)), (uint32_t)(lr * RB + (((4 + lg) ^ (lr & 7)) << 4))};
    bool late_x[2], late_w[2];
#pragma unroll
    for (int kk = 0; kk < 2; ++kk) {
        late_x[kk] = SKEW && kk * 4 + lg + turn_of(Xb, p.ldx, lr) >= 8;
        late_w[kk] = SKEW && kk * 4 + lg + turn_of(Wb, p.ldw, lr) >= 8;
    }
    auto read_w = [&](i32x4(&w)[2][2], uint32_t stage, uint32_t next, int h) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint8_t* s = smem + (late_w[kk] ? next : stage) + (BM + wn * 64 + h * 32) * RB;
#pragma unroll
            for (int i = 0; i < 2; ++i) w[i][kk] = *(const i32x4*)(s + i * 16 * RB + lk[kk]);
        }
    };
    auto read_x = [&](uint32_t stage, uint32_t next, int h) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const uint8_t* s = smem + (late_x[kk] ? next : stage) + (2 * wm + h) * XH * RB;
#pragma unroll
            for (int j = 0; j < XF; ++j) x[j][kk] = *(const i32x4*)(s + j * 16 * RB + lk[kk]);
        }
    };
    // nothing moves across the end of a slot
    auto barrier = [] { asm volatile("s_barrier" ::: "memory"); };
    auto end_memory = [&] {
        __builtin_amdgcn_sched_barrier(0);
        asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    auto products = [&](const i32x4(&w)[2][2], int fi, int fj) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < XF; ++j) acc[fi + i][fj + j] = mma8(w[i][kk], x[j][kk], acc[fi + i][fj + j]);
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
        barrier();
        __builtin_amdgcn_sched_barrier(0);
    };

    auto fill = [&](int t, int stage, int first) {  // a whole stage, in order of need
        copy_w(t, stage * STAGE, first);
        copy_x(t, stage * STAGE, 0);
        copy_w(t, stage * STAGE, 1 - first);
        copy_x(t, stage * STAGE, 1);
    };
    fill(0, 0, 0);
    fill(min(1, last), 1, SKEW ? 0 : 1);
    if (SKEW) fill(min(2, last), 2, 1);
    wait_vmcnt<LAG>();
    barrier();
    read_w(w0, 0, STAGE, 0);
    end_memory();              // both groups hold Wa of tile 0: its region may be refilled
    if (wave >= 4) barrier();  // one slot behind from here on
    uint32_t s0 = 0, s1 = STAGE, s2 = 2 * STAGE;  // the stages of pieces t, t + 1, t + 2
    auto tile = [&](int t, auto parity) {
        constexpr int P = decltype(parity)::value;  // t % 2: the feature half of Wa, without SKEW the stage
        auto& wa = P ? w1 : w0;
        auto& wb = P ? w0 : w1;
        const uint32_t here = SKEW ? s0 : P * STAGE, next = SKEW ? s1 : (1 - P) * STAGE;
        const int tn = min(t + S, last);
        read_x(here, next, 0);
        copy_w(tn, here, P);
        wait_vmcnt<LAG>();  // Wb landed
        end_memory();
        products(wa, 2 * P, 0);
        read_w(wb, here, next, 1 - P);
        copy_x(tn, here, 0);
        wait_vmcnt<LAG>();  // X1 landed
        end_memory();
        products(wb, 2 - 2 * P, 0);
        read_x(here, next, 1);
        copy_w(tn, here, 1 - P);
        wait_vmcnt<LAG>();  // Wa of t + 1 landed
        end_memory();
        products(wb, 2 - 2 * P, XF);
        read_w(wb, next, s2, 1 - P);  // Wa of t + 1
        copy_x(tn, here, 1);
        wait_vmcnt<LAG>();  // X0 of t + 1 landed
        end_memory();
        products(wa, 2 * P, XF);
        if (SKEW) {
            s0 = s1;
            s1 = s2;
            s2 = here;
        }
    };
    const std::integral_constant<int, 0> even;
    const std::integral_constant<int, 1> odd;
    int t = 0;
    for (; t + 1 < nk; t += 2) {
        tile(t, even);
        tile(t + 1, odd);
    }
    if (t < nk) tile(t, even);
    if (wave < 4) barrier();  // as many barriers in both groups
    const int mb = m0 + wm * 2 * XH, nb = n0 + wn * 64;
    if (jb.last) add_rest<2 * XF, 4>(p, p.K / RB * RB, mb, nb, lr, lg, acc);
    store_tile<BN, 2 * XF, 4>(p, jb, mb, nb, lr, lg, acc);
    wait_vmcnt<0>();  // the last copies have landed before the block's LDS is given back
}

// ---- smaller tiles: a ring of wide rows ------------------------------------------------
// BM tokens x BN features, the waves WGM x WGN; a ring stage holds BK bytes of the BM token
// rows and BN weight rows, so a copy fetches row pieces of 128 or 256 bytes; S - 1 stages are
// in flight while one is multiplied.  Bound by the weights' stream: 24 x 16384 x 4096 16.2 us
// from memory (4.2 TB/s; 12.9 from the last-level cache), 64 x 36864 x 9216 70 us (4.9 TB/s).
// 16-byte chunks are XOR-permuted by the low row bits.
//
// SKEW: for rows that do not start on 128 bytes.  BK bytes of such a row from a K tile's first
// on would touch a line more.  So a row's pieces start where its lines do, `turn` chunks
// before its K tiles: piece t holds, in the places of a tile's chunks, those of tile t whose
// place + turn is below CPR and the others (`late`) of tile t - 1.  A tile is read from two
// stages; a ring of one more has as many copies in flight.  A step of 128 bytes took 1.5 and
// 1.4 times as long (64 x 128 and 128 x 128), now 1.13 and 1.12; of 256 bytes 1.47 (32 x 64), now
// 1.33, and 1.2, now as long (32 x 32, 64 x 64: not kept).  300 x 4096 x 4112 22.7 -> 18.8 us.
template <int BM, int BN, int WGM, int WGN, int BK, int S, bool SKEW>
__global__ __launch_bounds__(64 * WGM * WGN) void q8_ring_kernel(GemmQ8Params p, Split sp) {
    constexpr int NW = WGM * WGN;
    constexpr int WM = BM / WGM, WN = BN / WGN;
    constexpr int MF = WM / 16, NF = WN / 16;
    constexpr int CPR = BK / 16;              // chunks per row
    constexpr int MASK = (CPR < 16 ? CPR : 16) - 1;
    constexpr int RPI = 1024 / BK;            // rows per copy
    constexpr int NL = (BM + BN) / RPI / NW;  // copies per wave and stage
    constexpr int STAGE = (BM + BN) * BK;
    static_assert(BM % (RPI * NW) == 0 && BN % (RPI * NW) == 0, "copies split into X and W");
    static_assert(S >= 2 && (S - 2) * NL < 64, "pipeline depth");
    __shared__ __attribute__((aligned(16))) uint8_t smem[S * STAGE];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WGM, wn = wave / WGM;
    const int lr = lane & 15, lg = lane >> 4;
    const Job jb = tile_job<BM, BN, BK>(p, sp);
    const int m0 = jb.m0, n0 = jb.n0, nk = jb.nk;

    const int8_t* Xb = p.X + (int64_t)m0 * p.ldx + (int64_t)jb.t0 * BK;
    const int8_t* Wb = p.W + (int64_t)n0 * p.ldw + (int64_t)jb.t0 * BK;
    auto chunk = [&](int j) { return (uint32_t)((lane % CPR) ^ (((wave + NW * j) * RPI + lane / CPR) & MASK)); };
    uint32_t off[NL], late = 0;  // SKEW: off from a tile before, where the late ones are
#pragma unroll
    for (int j = 0; j < NL; ++j) {
        const int row = (wave + NW * j) * RPI + lane / CPR;
        const bool is_x = (wave + NW * j) * RPI < BM;
        const uint32_t r = is_x ? min(row, p.M - 1 - m0) : min(row - BM, p.N - 1 - n0);
        off[j] = r * (uint32_t)(is_x ? p.ldx : p.ldw) + chunk(j) * 16;
        if constexpr (SKEW) {
            if (chunk(j) + (is_x ? turn_of(Xb, p.ldx, r) : turn_of(Wb, p.ldw, r)) >= CPR) late |= 1u << j;
            else off[j] += BK;
        }
    }
    const uint32_t lds0 = (uint32_t)(uintptr_t)smem;
    const int pieces = SKEW && nk > 0 ? nk + 1 : nk;
    auto issue = [&](int t, int stage) {
        if constexpr (!SKEW) {
            t += jb.phase;
            t = t >= nk ? t - nk : t;
        }
        const int64_t at = (int64_t)(SKEW ? t - 1 : t) * BK;
        const int8_t *xk = Xb + at, *wk = Wb + at;
#pragma unroll
        for (int j = 0; j < NL; ++j) {
            uint32_t o = off[j];
            if constexpr (SKEW) {  // nothing is read before a row's tiles, nor past them: what is there again
                const bool l = late >> j & 1;
                if (t == 0 && l) o += BK - chunk(j) * 16;
                if (t == nk && !l) o -= BK;
            }
            dma16s((wave + NW * j) * RPI < BM ? xk : wk, o, lds0 + stage * STAGE + (wave + NW * j) * 1024);
        }
    };
    bool late_x[BK / 64], late_w[BK / 64];  // of this lane's chunks of a tile
#pragma unroll
    for (int kk = 0; kk < BK / 64; ++kk) {
        late_x[kk] = SKEW && kk * 4 + lg + turn_of(Xb, p.ldx, lr) >= CPR;
        late_w[kk] = SKEW && kk * 4 + lg + turn_of(Wb, p.ldw, lr) >= CPR;
    }
    i32x4 acc[NF][MF] = {};
    auto compute = [&](int stage) {
        const uint8_t* s = smem + stage * STAGE;
        const int next = SKEW ? (stage == S - 1 ? -(S - 1) * STAGE : STAGE) : 0;
#pragma unroll
        for (int kk = 0; kk < BK / 64; ++kk) {
            const int ch = kk * 4 + lg;
            const uint8_t *sx = s + (late_x[kk] ? next : 0), *sw = s + (late_w[kk] ? next : 0);
            i32x4 b[MF];
#pragma unroll
            for (int j = 0; j < MF; ++j) {
                const int row = wm * WM + j * 16 + lr;
                b[j] = *(const i32x4*)(sx + row * BK + ((ch ^ (row & MASK)) << 4));
            }
#pragma unroll
            for (int i = 0; i < NF; ++i) {
                const int row = BM + wn * WN + i * 16 + lr;
                const i32x4 a = *(const i32x4*)(sw + row * BK + ((ch ^ (row & MASK)) << 4));
#pragma unroll
                for (int j = 0; j < MF; ++j) acc[i][j] = mma8(a, b[j], acc[i][j]);
            }
        }
    };
    // tile t is whole once pieces up to t (SKEW: t + 1) have landed
    constexpr int BEHIND = SKEW ? S - 3 : S - 2;
    static_assert(BEHIND >= 1, "copies in flight");
#pragma unroll
    for (int q = 0; q < S - 1; ++q)
        if (q < pieces) issue(q, q);
    int t = 0, st = 0;
    for (; t + S - 1 < pieces; ++t) {
        wait_vmcnt<BEHIND * NL>();
        __syncthreads();  // tile t visible to all waves; the stage before it free
        issue(t + S - 1, st == 0 ? S - 1 : st - 1);
        compute(st);
        st = st == S - 1 ? 0 : st + 1;
    }
    for (; t < nk; ++t) {
        wait_vmcnt<0>();
        __syncthreads();
        compute(st);
        st = st == S - 1 ? 0 : st + 1;
    }
    const int mb = m0 + wm * WM, nb = n0 + wn * WN;
    if (jb.last) add_rest<MF, NF>(p, p.K / BK * BK, mb, nb, lr, lg, acc);
    store_tile<BN, MF, NF>(p, jb, mb, nb, lr, lg, acc);
}

// ---- up to 16 tokens: weights from memory into the matrix operands ----------------------
// 16 features a block; its KW waves take pieces of 256 bytes of K in turn and add their
// sums through LDS.  Nothing is shared between waves, so weights need no LDS: a wave has
// the next piece's loads in flight while it multiplies one.  Lanes of tokens that do not
// exist load nothing and multiply zeros.  Bound by launch and load latency up to some 20 MB
// of weights (one token, N 6144, K 2048: 5.8 us in a recorded graph), by memory above.
template <int KW>
__global__ __launch_bounds__(64 * KW) void q8_few_kernel(GemmQ8Params p) {
    __shared__ i32x4 part[KW][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int n0 = (int)blockIdx.x * 16;
    const int8_t* w = p.W + (int64_t)min(n0 + lr, p.N - 1) * p.ldw + 16 * lg;
    const int8_t* x = p.X + (int64_t)min(lr, p.M - 1) * p.ldx + 16 * lg;
    const bool here = lr < p.M;
    struct Piece {
        i32x4 a[4], b[4];
    };
    auto load = [&](Piece& c, int k) {
#pragma unroll
        for (int q = 0; q < 4; ++q) c.a[q] = __builtin_nontemporal_load((const i32x4*)(w + k + 64 * q));
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            c.b[q] = i32x4{0, 0, 0, 0};
            if (here) c.b[q] = *(const i32x4*)(x + k + 64 * q);
        }
    };
    i32x4 acc = {0, 0, 0, 0};
    auto multiply = [&](const Piece& c) {
#pragma unroll
        for (int q = 0; q < 4; ++q) acc = mma8(c.a[q], c.b[q], acc);
    };
    const int pieces = p.K / 256;
    Piece c0, c1;
    int t = wave;
    if (t < pieces) load(c0, t * 256);
    for (; t < pieces; t += 2 * KW) {
        if (t + KW < pieces) load(c1, (t + KW) * 256);
        multiply(c0);
        if (t + 2 * KW < pieces) load(c0, (t + 2 * KW) * 256);
        if (t + KW < pieces) multiply(c1);
    }
    if (pieces * 256 < p.K && wave == pieces % KW) {  // the rest, to the wave whose turn it is
        for (int k = pieces * 256; k < p.K; k += 64) {
            const bool in = k + 16 * lg < p.K;
            i32x4 a = {0, 0, 0, 0}, b = {0, 0, 0, 0};
            if (in) a = *(const i32x4*)(w + k);
            if (in && here) b = *(const i32x4*)(x + k);
            acc = mma8(a, b, acc);
        }
    }
    part[wave][lane] = acc;
    __syncthreads();
    if (wave > 0) return;
    const int n = n0 + 4 * lg;
    float old[4] = {};
    if (here && n < p.N) load_old(p, lr, n, p.N - n, old);
#pragma unroll
    for (int k = 1; k < KW; ++k) acc += part[k][lane];
    if (here && n < p.N) {
        Features f = load_features(p, n);
        ready(p, f);
        epilogue8(p, lr, n, p.sx[lr], f, acc, old);
    }
}

// ---- the sums of split tiles -------------------------------------------------------------
// A thread adds the ranges' sums of four features of one token.  Bound by memory (40 tiles of
// 192 x 256 in six ranges 12 us, 4.6 TB/s); splits are worth it where tiles leave CUs idle.
template <int BM, int BN>
__global__ __launch_bounds__(256) void q8_join_kernel(GemmQ8Params p, Split sp) {
    constexpr int GROUPS = BM * BN / 4 / 256;  // blocks per tile
    const int i = (int)blockIdx.x / GROUPS;
    const int at = ((int)blockIdx.x % GROUPS * 256 + (int)threadIdx.x) * 4;
    int m0, n0;
    tile_corner<BM, BN>(p, sp.full + i, m0, n0);
    const int m = m0 + at / BN, n = n0 + at % BN;
    if (m >= p.M || n >= p.N) return;
    const int64_t stride = (int64_t)sp.tail * (BM * BN);
    const int32_t* src = p.ws + (int64_t)i * (BM * BN) + at;
    Features f = load_features(p, n);
    const float sx = p.sx[m];
    float old[4] = {};
    load_old(p, m, n, f.left, old);
    i32x4 v = {0, 0, 0, 0};
    for (int s = 0; s < sp.splits; s += 8) {  // eight ranges' loads in flight together
        i32x4 o[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
            o[q] = i32x4{0, 0, 0, 0};
            if (s + q < sp.splits) o[q] = __builtin_nontemporal_load((const i32x4*)(src + (s + q) * stride));
        }
#pragma unroll
        for (int q = 0; q < 8; ++q) v += o[q];
    }
    ready(p, f);
    epilogue8(p, m, n, sx, f, v, old);
}

// ---- launches ----------------------------------------------------------------------------

template <int BM, int BN, typename F>
void launch_tiles(F kernel, const GemmQ8Params& p, const Plan& c, hipStream_t s) {
    const Split sp = split_of(p, c);
    PB_LAUNCH(kernel, sp.full + sp.tail * sp.splits, SHAPES[c.shape].threads, 0, s, p, sp);
    if (sp.tail) PB_LAUNCH((q8_join_kernel<BM, BN>), sp.tail * (BM * BN / 4 / 256), 256, 0, s, p, sp);
}

// S_SKEW: stages for rows off 128 bytes (0: the same kernel, which lost little by them).
template <int BM, int BN, int WGM, int WGN, int BK, int S, int S_SKEW>
void launch_ring(const GemmQ8Params& p, const Plan& c, hipStream_t s) {
    if constexpr (S_SKEW > 0) {
        if (skewed(p)) return launch_tiles<BM, BN>(q8_ring_kernel<BM, BN, WGM, WGN, BK, S_SKEW, true>, p, c, s);
    }
    launch_tiles<BM, BN>(q8_ring_kernel<BM, BN, WGM, WGN, BK, S, false>, p, c, s);
}

template <int KW>
void launch_few(const GemmQ8Params& p, hipStream_t s) {
    PB_LAUNCH((q8_few_kernel<KW>), (p.N + 15) / 16, 64 * KW, 0, s, p);
}

void launch_plan(const GemmQ8Params& p, const Plan& c, hipStream_t s) {
    switch (c.shape) {
        case 0: launch_few<4>(p, s); break;
        case 1: launch_few<8>(p, s); break;
        case 2: launch_ring<32, 32, 1, 2, 256, 4, 0>(p, c, s); break;
        case 3: launch_ring<32, 64, 1, 4, 256, 4, 5>(p, c, s); break;
        case 4: launch_ring<64, 64, 1, 4, 256, 4, 0>(p, c, s); break;
        case 5: launch_ring<64, 128, 2, 4, 128, 4, 6>(p, c, s); break;
        case 6: launch_ring<128, 64, 2, 2, 256, 3, 0>(p, c, s); break;
        case 7: launch_ring<128, 128, 2, 4, 128, 4, 5>(p, c, s); break;
        case 8:
            if (skewed(p)) launch_tiles<128, 256>(q8_wide_kernel<2, true>, p, c, s);
            else launch_tiles<128, 256>(q8_wide_kernel<2, false>, p, c, s);
            break;
        case 9: launch_tiles<192, 256>(q8_wide_kernel<3, false>, p, c, s); break;
        case 10: launch_tiles<256, 256>(q8_wide_kernel<4, false>, p, c, s); break;
    }
}

}  // namespace

bool gemm_q8_fits(int M, int N) {
    return M <= (1 << 24) && N <= (1 << 24) && (((int64_t)M + 63) / 64) * (((int64_t)N + 63) / 64) < (1 << 23);
}

size_t gemm_q8_workspace(int M, int N, int K) {
    GemmQ8Params p{};
    p.M = M; p.N = N; p.K = K;
    return workspace_of(p);
}

hipError_t launch_gemm_q8(const GemmQ8Params& p, hipStream_t s) {
    launch_plan(p, plan_of(p, p.ws_bytes), s);
    return hipGetLastError();
}

}  // namespace pb
