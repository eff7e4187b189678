// Beam search's selection: of every live hypothesis's continuations, the W best
// of each prompt.
//
// log softmax(l)[v] = l[v] - m - log sum exp(l - m): a row's order is its logits'
// order, so a row offers its W largest logits and its log sum, and only those are
// compared across rows.  What bounds it is reading the logits once, if the
// arithmetic on them (four instructions a logit, one of them exp2 at a quarter of
// the rate) hides behind it; the two launches then cost their latency:
//
//  chunks  One block per (row, chunk of 256 R logits), the chunk in registers.  The
//          W-th largest of the 256 threads' maxima is a value that at least W
//          logits reach and that only W threads (and ties) hold any above: found by
//          bisection on the bits, with ballots, it leaves a handful of candidates,
//          each placed by counting those before it.  The chunk's maximum and sum of
//          exponentials come from the same registers, as the logits arrive:
//          2^(x log2 e - c) with c the rounded maximum in the base of two, one
//          multiply-add and exact in c.  (256 rows of 50272 logits take 11.6 us, 128 of
//          128256 15.1; loading alone takes 8.4 and 10.3, and with the sum after the
//          selection and every logit cleaned first it was 14.2 and 18.5: the vector
//          units were the bound.)
//  join    One block per prompt over the sorted lists of its rows' chunks: the same
//          idea, the W-th largest list head keeps all but W lists (and ties) out.
//          One block's chain of dependent steps: 4.9 us for 8 x 7 lists, 6.0 for 32 x 16.
//
// Sums of exponentials run in fp32 within a chunk and are joined in 64 bits, their
// weights and the logarithm's fraction to fp32, as near as the sums are; a
// candidate's score, score + ((l - m) - log sum), is formed and compared in 64 bits,
// because candidates of different rows can lie closer than fp32 tells apart at
// scores of tens.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {

constexpr float LOG2E = 1.4426950408889634f;
constexpr float HUGE_LOGIT = 4194304.f;  // 2^22: below it a rounded maximum is exact, in base two also
constexpr int NT = 256;       // threads of a chunk's block
constexpr int MOST = 1024;    // candidates of a chunk: 32 threads' 32 logits
// More candidates than CROWD are looked at again before they are placed: equal ones, as a
// rule (4 beams that all offer 50272 equal logits: 19 us, placed as they are 238).
constexpr int CROWD = 192;
constexpr int LISTS = 4096;   // lists of a prompt: 32 rows of 2^20 logits in 128 chunks

// What a logit counts as: NaN is no candidate, +inf the largest float.
__device__ inline float clean(float x) {
    return __builtin_amdgcn_fmed3f(x == x ? x : -INFINITY, -INFINITY, 3.402823466e38f);
}

// Unsigned keys in the order of the floats (-0 and +0 alike).
__device__ inline uint32_t key_of(float x) {
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
constexpr uint32_t KEY_NONE = 0x007fffffu;  // of -inf
__device__ inline float float_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key); }

// A logit and its token as one key: of equal logits the lower token is the larger key.
__device__ inline uint64_t entry_of(float x, int v) { return (uint64_t)key_of(x) << 32 | (uint32_t)~v; }

template <int N> struct Words { uint32_t w[N]; };

// The value of the lane that the DPP control names.
template <int CONTROL, typename T>
__device__ inline T moved(T v) {
    auto b = __builtin_bit_cast(Words<sizeof(T) / 4>, v);
    for (uint32_t& w : b.w) w = (uint32_t)__builtin_amdgcn_mov_dpp((int)w, CONTROL, 0xf, 0xf, false);
    return __builtin_bit_cast(T, b);
}

// op over groups of g lanes (4 to 64), in every lane, without LDS: quads, rows of 16,
// then the rows.
template <typename T, typename Op>
__device__ inline T over_lanes(T v, int g, Op op) {
    using B = Words<sizeof(T) / 4>;
    v = op(v, moved<0xB1>(v));                // quad_perm 1 0 3 2
    v = op(v, moved<0x4E>(v));                // quad_perm 2 3 0 1
    if (g >= 8) v = op(v, moved<0x141>(v));   // row_half_mirror
    if (g >= 16) v = op(v, moved<0x140>(v));  // row_mirror
    auto halves = [&](auto swap) {
        B a = __builtin_bit_cast(B, v), b = a;
        for (int i = 0; i < (int)(sizeof(T) / 4); ++i) {
            const auto s = swap(a.w[i]);
            a.w[i] = s[0];
            b.w[i] = s[1];
        }
        v = op(__builtin_bit_cast(T, a), __builtin_bit_cast(T, b));
    };
    if (g >= 32) halves([](uint32_t w) { return __builtin_amdgcn_permlane16_swap(w, w, false, false); });
    if (g >= 64) halves([](uint32_t w) { return __builtin_amdgcn_permlane32_swap(w, w, false, false); });
    return v;
}
constexpr auto add = [](auto a, auto b) { return a + b; };
constexpr auto larger = [](float a, float b) { return fmaxf(a, b); };

// How many of n keys in LDS are larger, counted by the four lanes that share `mine`.
__device__ inline int rank_of(const uint64_t* keys, int n, uint64_t mine) {
    int rank = 0;
#pragma unroll 4
    for (int j = threadIdx.x % 4; j < n; j += 4) rank += keys[j] > mine;
    return over_lanes(rank, 4, add);
}

struct ChunkBest {
    float2* ms;    // [rows][chunks] maximum and sum of exponentials
    float* val;    // [rows][chunks][W], descending; -inf: none left
    int32_t* idx;  // [rows][chunks][W]
};

__host__ __device__ inline ChunkBest chunk_best(void* ws, size_t lists, int W) {
    ChunkBest r;
    r.ms = (float2*)ws;
    r.val = (float*)(r.ms + lists);
    r.idx = (int32_t*)(r.val + lists * W);
    return r;
}

// (a, i) comes before (b, j)
template <typename K> __device__ inline bool before(K a, int i, K b, int j) { return a > b || (a == b && i < j); }

// Maximum of G values.
template <int G>
__device__ inline float max_of(const float* x) {
    // v_max3 itself: fmaxf would first quiet each operand.  With a NaN among them the
    // result is any of them.
    float v = x[0];
#pragma unroll
    for (int i = 1; i < G; i += 2) asm("v_max3_f32 %0, %0, %1, %2" : "+v"(v) : "v"(x[i]), "v"(x[i + 1 < G ? i + 1 : i]));
    return v;
}

// Zero, which the compiler cannot know to be the same in all lanes.
__device__ inline int zero_of_lane() {
    int z = 0;
    asm volatile("" : "+v"(z));
    return z;
}

// A value t that at least `want` of `keys` keys reach, and at most `most` of them
// unless more are equal (then t is the want-th largest itself; 0 if there are no
// `want` keys).  hi: the largest key; count(t): how many reach t, the same in every
// lane.  The want-th largest of a few hundred shares the largest one's leading bits:
// the common part is found first, upwards from 14 of them, then bits are added until
// few enough keys are left.  (Two bits a step, with three counts, take 5% longer.)
template <typename Count>
__device__ inline uint32_t reach(Count count, int keys, uint32_t hi, int want, int most) {
    hi = __builtin_amdgcn_readfirstlane(hi);  // (all steps on the scalar unit)
    int b = 18, n = 0;
    uint32_t t = 0;
    for (; b < 32; b += 2) {
        t = hi >> b << b;
        n = count(t);
        if (n >= want) break;
    }
    if (b >= 32) {
        b = 32;
        t = 0;
        n = keys;
    }
    while (n > most && b > 0) {
        --b;
        const uint32_t trial = t | (1u << b);
        const int c = count(trial);
        if (c >= want) {
            t = trial;
            n = c;
        }
    }
    return t;
}

template <int R>
__global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(5))) void beam_chunks_kernel(BeamParams p, int chunks) {
    __shared__ __attribute__((aligned(16))) float smax[NT];
    __shared__ float ssum[NT / 64];
    __shared__ uint64_t cand[MOST];
    __shared__ int cn, eq[NT / 64];
    __shared__ uint32_t reached;
    constexpr int G = R < 8 ? R : 8;
    const int row = blockIdx.x / chunks, chunk = blockIdx.x % chunks;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int W = p.W, v0 = chunk * NT * R + tid;
    const ChunkBest out = chunk_best(p.ws, (size_t)p.B * W * chunks, W);
    const size_t list = (size_t)row * chunks + chunk;
    const float* l = p.logits + row * p.ld + chunk * NT * R;
    const int left = p.V - chunk * NT * R;
    float x[R], top[R / G];  // the logits, the largest of every G
    if (left >= NT * R) {
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = l[i * NT + (unsigned)tid];
    } else {
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = l[min(i * NT + tid, left - 1)];
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = i * NT + tid < left ? x[i] : -INFINITY;
    }
    // Sum of 2^(x log2 e - ref), ref a whole number near the largest so far.  NaN or
    // +inf make it NaN.
    float ref = -2 * HUGE_LOGIT, sum = 0.f;
#pragma unroll
    for (int g = 0; g < R / G; ++g) {
        top[g] = max_of<G>(x + g * G);
        const float next = fmaxf(ref, __builtin_rintf(top[g] * LOG2E));
        sum *= __builtin_amdgcn_exp2f(ref - next);
#pragma unroll
        for (int i = 0; i < G; ++i) sum += __builtin_amdgcn_exp2f(__builtin_fmaf(x[g * G + i], LOG2E, -next));
        ref = next;
    }
    // (the sum is used before the barrier, so it is formed while loads are under way)
    const bool odd = __any(!(sum < INFINITY));
    if (odd) {
        asm volatile("");  // a branch: rarely taken
#pragma unroll
        for (int i = 0; i < R; ++i) x[i] = clean(x[i]);
#pragma unroll
        for (int g = 0; g < R / G; ++g) top[g] = max_of<G>(x + g * G);
    }
    float mx = top[0];
#pragma unroll
    for (int g = 1; g < R / G; ++g) mx = fmaxf(mx, top[g]);
    smax[tid] = mx;
    if (tid == 0) cn = 0;
    __syncthreads();
    // the W-th largest of the maxima of every four threads is a little lower than
    // that of all, and found with one ballot a step, by one wave
    const f32x4 four = *(const f32x4*)&smax[4 * lane];
    const float of4 = fmaxf(fmaxf(four[0], four[1]), fmaxf(four[2], four[3]));
    const float m = over_lanes(of4, 64, larger);
    if (wave == (blockIdx.x & 3)) {
        const uint32_t key4 = key_of(of4);
        const uint32_t r = reach([&](uint32_t least) { return __popcll(__ballot(key4 >= least)); }, 64, key_of(m), W, W);
        if (lane == 0) reached = r;
    }
    __syncthreads();
    uint32_t t = max(reached, KEY_NONE + 1);
    if (m > -INFINITY) {
        if (odd || !(fabsf(m) < HUGE_LOGIT)) {
            sum = 0.f;  // logits cleaned since, or too large for a whole number between them
#pragma unroll
            for (int i = 0; i < R; ++i) sum += __builtin_amdgcn_exp2f((x[i] - m) * LOG2E);
        } else {
            sum *= __builtin_amdgcn_exp2f(__builtin_fmaf(-m, LOG2E, ref));
        }
        float least = float_of(t);
        // one counter, at an address that may differ between lanes: a single LDS add
        int* const count = &cn + zero_of_lane();
#pragma unroll
        for (int g = 0; g < R / G; ++g)
            if (top[g] >= least)
#pragma unroll
                for (int i = g * G; i < g * G + G; ++i)
                    if (x[i] >= least) {
                        const int at = atomicAdd(count, 1);
                        if (at < CROWD) cand[at] = entry_of(x[i], v0 + i * NT);
                        else least = INFINITY;  // looked at again anyway
                    }
    } else {
        sum = 0.f;
    }
    sum = over_lanes(sum, 64, add);
    if (lane == 0) ssum[wave] = sum;
    __syncthreads();
    int n = cn;
    if (n > CROWD) {
        // Many equal ones, or the best side by side in few groups of four threads.  By
        // all the threads' maxima: W threads reach t, and hold those above it and those at
        // it, MOST at most; or more do, then t is the W-th largest maximum, those above it
        // are in W - 1 threads, and of those at t the W lowest are enough, taken in
        // ascending order: MOST at most again.
        auto count = [&](uint32_t least) {
            int c = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) c += __popcll(__ballot(key_of(four[i]) >= least));
            return c;
        };
        t = max(reach(count, NT, key_of(m), W, W), KEY_NONE + 1);
        __syncthreads();
        if (tid == 0) cn = 0;
        __syncthreads();
        const float best = float_of(t);
#pragma unroll
        for (int i = 0; i < R; ++i)
            if (x[i] > best) cand[atomicAdd(&cn + zero_of_lane(), 1)] = entry_of(x[i], v0 + i * NT);
        __syncthreads();
        n = cn;
        int taken = 0;
        for (int i = 0; i < R && taken < W; ++i) {
            float v = 0.f;
#pragma unroll
            for (int j = 0; j < R; ++j) v = j == i ? x[j] : v;
            const bool mine = v == best;
            const uint64_t b = __ballot(mine);
            if (lane == 0) eq[wave] = __popcll(b);
            __syncthreads();
            int at = taken + __popcll(b & (((uint64_t)1 << lane) - 1)), all = 0;
            for (int w = 0; w < NT / 64; ++w) {
                if (w < wave) at += eq[w];
                all += eq[w];
            }
            if (mine && at < W) cand[n + at] = entry_of(v, v0 + i * NT);
            taken += all;
            __syncthreads();
        }
        n += min(taken, W);
    }
    __syncthreads();
    for (int c0 = wave * 16; c0 < n; c0 += NT / 4) {
        const int c = c0 + lane / 4;
        const uint64_t e = cand[min(c, n - 1)];
        const int rank = rank_of(cand, n, e);
        if (c < n && tid % 4 == 0 && rank < W) {
            out.val[list * W + rank] = float_of((uint32_t)(e >> 32));
            out.idx[list * W + rank] = ~(uint32_t)e;
        }
    }
    for (int c = n + tid; c < W; c += NT) {
        out.val[list * W + c] = -INFINITY;
        out.idx[list * W + c] = 0;
    }
    if (tid == 0) out.ms[list] = make_float2(m, (ssum[0] + ssum[1]) + (ssum[2] + ssum[3]));
}

static_assert(BEAM_MAX_VOCAB <= 1 << 20 && BEAM_MAX_WIDTH <= 1 << 11, "a place's 20 and 11 bits");
constexpr int HELD = 8;  // heads that a lane holds in registers: 512 lists, more are read again
constexpr int TIED = 64;  // lists whose heads may pass the bisection: the W and ties
// More entries than MANY go through a bisection of their own before they are placed, down
// to FEW (20 prompts of 32 beams and 6245 logits, 32 lists each: the call 23 us, 112 without
// it; 10 of 12 beams and 954 logits, some 140 entries: 11.4, with it 14.7).
constexpr int FEW = 128, MANY = 256;

// Which of n candidates, K to a thread, are the `want` that come first, by score and then
// place: a bit for each of this thread's.  None is -inf.  By all threads, bit by bit: 8 us
// with 256 of them and 45 with 1024, for candidates too much alike for anything else.
constexpr int K = 4;
template <int JT>
__device__ __forceinline__ uint32_t first_of(const double (&score)[K], const int (&place)[K], int n, int want) {
    uint64_t key[K];  // in the order of the doubles (-0 and +0 alike), 0: none
#pragma unroll
    for (int k = 0; k < K; ++k) {
        const uint64_t b = __builtin_bit_cast(uint64_t, score[k] + 0.0);
        key[k] = score[k] == -INFINITY ? 0 : b >> 63 ? ~b : b | (uint64_t)1 << 63;
    }
    // (three counters in turn, one barrier a count)
    __shared__ int counter[3];
    int turn = 0;
    if (threadIdx.x == 0) counter[0] = 0;
    __syncthreads();
    auto count = [&](auto passed) {
        int c = 0;
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (k * JT < n) c += __popcll(__ballot(passed(k)));
        const int next = turn == 2 ? 0 : turn + 1;
        if (threadIdx.x == 0) counter[next] = 0;
        if (threadIdx.x % 64 == 0) atomicAdd(&counter[turn], c);
        __syncthreads();
        c = counter[turn];
        turn = next;
        return c;
    };
    uint64_t t = 0;  // the want-th largest
#pragma unroll 1
    for (uint64_t bit = (uint64_t)1 << 63; bit; bit >>= 1)
        if (count([&](int k) { return key[k] >= (t | bit); }) >= want) t |= bit;
    want -= count([&](int k) { return key[k] > t; });
    uint32_t low = 0;  // and the want-th lowest place of those equal to it, inverted
#pragma unroll 1
    for (uint32_t bit = 1u << 31; bit && t; bit >>= 1)
        if (count([&](int k) { return key[k] == t && ~(uint32_t)place[k] >= (low | bit); }) >= want) low |= bit;
    uint32_t kept = 0;
#pragma unroll
    for (int k = 0; k < K; ++k)
        if (key[k] > t || (t && key[k] == t && ~(uint32_t)place[k] >= low)) kept |= 1u << k;
    return kept;
}

// log of 1 <= x < 2^21: the exponent's part in 64 bits, the rest within 2^-23.
__device__ inline double log_of(double x) {
    const float v = (float)x;
    const uint32_t b = __float_as_uint(v);
    const int e = (int)((b + 0x00400000u) >> 23) - 127;  // v / 2^e in [3/4, 3/2)
    const float f = __uint_as_float(b - ((uint32_t)e << 23));
    return e * 0.6931471805599453 + (double)(__builtin_amdgcn_logf(f) * 0.6931471805599453f);
}

template <int JT>
__global__ __launch_bounds__(JT) void beam_join_kernel(BeamParams p, int chunks, FastDiv by_chunks, FastDiv by_width) {
    __shared__ double lse[BEAM_MAX_WIDTH];
    __shared__ float row_max[BEAM_MAX_WIDTH], own[BEAM_MAX_WIDTH];
    __shared__ uint32_t key[LISTS], threshold;
    __shared__ int live[BEAM_MAX_WIDTH], pick[TIED], picks;
    __shared__ double sc[TIED * BEAM_MAX_WIDTH];
    __shared__ int id[TIED * BEAM_MAX_WIDTH], cn;
    __shared__ double few_sc[FEW];
    __shared__ int few_id[FEW];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, W = p.W;
    const int lists = W * chunks;
    const ChunkBest in = chunk_best(p.ws, (size_t)p.B * lists, W);
    const size_t first = (size_t)b * lists;
    if (tid == 0) picks = cn = 0;
    if (tid < W) {
        own[tid] = p.scores[b * W + tid];
        live[tid] = p.alive[b * W + tid];
    }
    // the heads of this thread's first list are on their way meanwhile
    const float head_val = tid < lists ? in.val[(first + tid) * W] : 0.f;
    const int head_idx = tid < lists ? in.idx[(first + tid) * W] : 0;
    // the rows' log sums, g lanes to a row
    int g = 4;
    while (g < 64 && g < chunks) g *= 2;
    for (int w = tid / g; w < (W + 64 / g - 1) / (64 / g) * (64 / g); w += JT / g) {  // whole waves
        const float2* ms = in.ms + first + min(w, W - 1) * chunks;
        const float2 mine = tid % g < chunks ? ms[tid % g] : make_float2(-INFINITY, 0.f);
        float m = mine.x;
        for (int c = tid % g + g; c < chunks; c += g) m = fmaxf(m, ms[c].x);
        m = over_lanes(m, g, larger);
        auto term = [&](float2 v) { return v.x == -INFINITY ? 0.0 : (double)v.y * __builtin_amdgcn_exp2f((v.x - m) * LOG2E); };
        double sum = term(mine);
        for (int c = tid % g + g; c < chunks; c += g) sum += term(ms[c]);
        sum = over_lanes(sum, g, add);
        if (tid % g == 0 && w < W) {
            row_max[w] = m;
            lse[w] = log_of(sum);
        }
    }
    __syncthreads();
    // score of a list's k-th entry and its place (w, v); an ended hypothesis stands
    // at the head of its first list, as token pad
    auto score_as = [&](int i, int k, int& place, float v, int v_idx) -> double {
        const int w = by_chunks.quot(i);
        place = w << 20 | p.pad;
        if (!(own[w] - own[w] == 0.f)) return -INFINITY;
        if (live[w] == 0) return i == w * chunks && k == 0 ? (double)own[w] : -INFINITY;
        if (v == -INFINITY) return -INFINITY;
        place = w << 20 | v_idx;
        return (double)own[w] + (((double)v - (double)row_max[w]) - lse[w]);
    };
    auto score_of = [&](int i, int k, int& place) {
        return score_as(i, k, place, in.val[(first + i) * W + k], in.idx[(first + i) * W + k]);
    };
    for (int i = tid; i < lists; i += JT) {
        int place;
        key[i] = key_of((float)(i == tid ? score_as(i, 0, place, head_val, head_idx) : score_of(i, 0, place)));
    }
    __syncthreads();
    // the W-th largest head, about, to fp32 (rounding keeps the order)
    if (wave == 0) {
        // from the lanes' maxima of every 64th head: at least W heads reach it
        uint32_t held[HELD], top = 0;
#pragma unroll
        for (int j = 0; j < HELD; ++j) {
            held[j] = j * 64 + lane < lists ? key[j * 64 + lane] : 0;
            top = max(top, held[j]);
        }
        for (int i = HELD * 64 + lane; i < lists; i += 64) top = max(top, key[i]);
        const uint32_t hi = key_of(over_lanes(top ? float_of(top) : -INFINITY, 64, larger));
        uint32_t v = reach([&](uint32_t least) { return __popcll(__ballot(top >= least)); }, 64, hi, W, W);
        auto count = [&](uint32_t least) {
            int n = 0;
#pragma unroll
            for (int j = 0; j < HELD; ++j) n += __popcll(__ballot(held[j] >= least));
            for (int i = HELD * 64; i < lists; i += 64) n += __popcll(__ballot(i + lane < lists && key[i + lane] >= least));
            return n;
        };
        if (lists > 64 && count(v) > TIED) v = reach(count, lists, hi, W, TIED);
        if (lane == 0) threshold = v;
    }
    __syncthreads();
    const uint32_t t = max(threshold, KEY_NONE + 1);
    for (int i = tid; i < lists; i += JT)
        if (key[i] >= t) {
            const int at = atomicAdd(&picks, 1);
            if (at < TIED) pick[at] = i;
        }
    __syncthreads();
    int n = picks;
    if (n > TIED) {
        // Many heads alike to fp32: the W that come first in 64 bits.
        double s[K];
        int at[K];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int i = k * JT + tid;
            s[k] = i < lists && key[min(i, lists - 1)] >= t ? score_of(i, 0, at[k]) : -INFINITY;
        }
        const uint32_t kept = first_of<JT>(s, at, lists, W);
        if (tid == 0) picks = 0;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < K; ++k)
            if (kept >> k & 1) pick[atomicAdd(&picks, 1)] = k * JT + tid;
        __syncthreads();
        n = picks;
    }
    // their entries that reach the W-th head too
    for (int i = tid; i < n * W; i += JT) {
        int place;
        const int nth = by_width.quot(i);
        const double s = score_of(pick[nth], i - nth * W, place);
        if (s > -INFINITY && key_of((float)s) >= t) {
            const int at = atomicAdd(&cn, 1);
            sc[at] = s;
            id[at] = place;
        }
    }
    __syncthreads();
    n = cn;
    const double* score = sc;
    const int* place = id;
    if (n > MANY) {
        // Few lists, so most of their entries reach the W-th head: the same once more over
        // all entries.
        if (wave == 0) {
            constexpr int E = TIED * BEAM_MAX_WIDTH / 64;
            uint32_t held[E], top = 0;
#pragma unroll
            for (int j = 0; j < E; ++j) {
                held[j] = 0;
                if (j * 64 < n) held[j] = j * 64 + lane < n ? key_of((float)sc[min(j * 64 + lane, n - 1)]) : 0;
                top = max(top, held[j]);
            }
            const uint32_t hi = key_of(over_lanes(top ? float_of(top) : -INFINITY, 64, larger));
            const uint32_t v = reach([&](uint32_t least) {
                int c = 0;
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (j * 64 < n) c += __popcll(__ballot(held[j] >= least));
                return c;
            }, n, hi, W, FEW);
            if (lane == 0) {
                threshold = v;
                picks = 0;
            }
        }
        __syncthreads();
        for (int c = tid; c < n; c += JT)
            if (key_of((float)sc[c]) >= threshold) {
                const int at = atomicAdd(&picks, 1);
                if (at < FEW) {
                    few_sc[at] = sc[c];
                    few_id[at] = id[c];
                }
            }
        __syncthreads();
        if (picks > FEW) {  // equal ones
            double s[K];
            int at[K];
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int c = k * JT + tid;
                s[k] = c < n ? sc[min(c, n - 1)] : -INFINITY;
                at[k] = id[min(c, n - 1)];
            }
            const uint32_t kept = first_of<JT>(s, at, n, W);
            if (tid == 0) picks = 0;
            __syncthreads();
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (kept >> k & 1) {
                    const int to = atomicAdd(&picks, 1);
                    few_sc[to] = s[k];
                    few_id[to] = at[k];
                }
            __syncthreads();
        }
        n = picks;
        score = few_sc;
        place = few_id;
    }
    // (scores and alive are in LDS: the outputs may be the same arrays)
    constexpr int G = 8;  // lanes that share a candidate's count
    for (int c0 = 0; c0 < n; c0 += JT / G) {
        const int c = min(c0 + tid / G, n - 1);
        const double s = score[c];
        const int own_place = place[c];
        int rank = 0;
#pragma unroll 4
        for (int j = tid % G; j < n; j += G) {
            const bool lower = place[j] < own_place;
            rank += (score[j] > s) | ((score[j] == s) & lower);
        }
        rank = over_lanes(rank, G, add);
        if (rank >= W || c0 + tid / G >= n || tid % G) continue;
        const int o = b * W + rank, w = own_place >> 20, token = own_place & 0xfffff;
        p.out_scores[o] = (float)score[c];
        p.out_tokens[o] = token;
        p.out_parents[o] = b * W + w;
        p.out_alive[o] = live[w] != 0 && token != p.eos;
    }
    for (int i = n + tid; i < W; i += JT) {  // places that no candidate takes
        const int o = b * W + i;
        p.out_scores[o] = -INFINITY;
        p.out_tokens[o] = p.pad;
        p.out_parents[o] = -1;
        p.out_alive[o] = 0;
    }
}

constexpr int BLOCKS = 512;
// Logits per thread: the most (fewest lists to join) that leave BLOCKS blocks,
// and enough that a row has at most 64 lists (128 of 2^20 logits).
int logits_per_thread(int64_t rows, int V) {
    int r = 32;
    while (r > 4 && rows * ((V + NT * r - 1) / (NT * r)) < BLOCKS) r /= 2;
    while (r < 32 && (V + NT * r - 1) / (NT * r) > 64) r *= 2;
    return r;
}

}  // namespace

size_t beam_select_workspace(int B, int W, int V) {
    const int r = logits_per_thread((int64_t)B * W, V);
    return (size_t)B * W * ((V + NT * r - 1) / (NT * r)) * (8 + (size_t)W * 8);
}

hipError_t launch_beam_select(const BeamParams& p, hipStream_t s) {
    if (p.B <= 0) return hipSuccess;
    const int r = logits_per_thread((int64_t)p.B * p.W, p.V), chunks = (p.V + NT * r - 1) / (NT * r);
    if ((int64_t)p.B * p.W * chunks > 0x7fffffff) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(p.B * p.W * chunks));
    if (r == 32) PB_LAUNCH(beam_chunks_kernel<32>, grid, dim3(NT), 0, s, p, chunks);
    else if (r == 16) PB_LAUNCH(beam_chunks_kernel<16>, grid, dim3(NT), 0, s, p, chunks);
    else if (r == 8) PB_LAUNCH(beam_chunks_kernel<8>, grid, dim3(NT), 0, s, p, chunks);
    else PB_LAUNCH(beam_chunks_kernel<4>, grid, dim3(NT), 0, s, p, chunks);
    const FastDiv by_chunks(chunks), by_width(p.W);
    // (wide beams have up to W entries a list: 8 prompts of 20 beams and 900 logits 13.5 us,
    // with 256 threads 15.3)
    if (p.W * chunks <= 256 && p.W <= 11) PB_LAUNCH(beam_join_kernel<256>, dim3(p.B), dim3(256), 0, s, p, chunks, by_chunks, by_width);
    else PB_LAUNCH(beam_join_kernel<1024>, dim3(p.B), dim3(1024), 0, s, p, chunks, by_chunks, by_width);
    return hipGetLastError();
}

}  // namespace pb
