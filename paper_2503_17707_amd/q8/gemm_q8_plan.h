// Which kernel an 8-bit product takes and how its K is split: host code, apart from the
// kernels (gemm_q8.hip) so that it can be asked without a GPU.
#pragma once

#include <cmath>
#include <utility>

#include "q8.h"

namespace pb::q8 {

// Tiles 0 .. full-1 run over the whole of K; the others' K tiles are cut into `splits` ranges
// of kt, the last one taking the rest and what lies past the last whole K tile.  Range s of
// tile full + i leaves its sums at ws + (s tail + i) BM BN.  Columns of tiles start at
// `phases` places of their range, and go round.
struct Split {
    int full, tail, splits, kt, phases;
};

enum Kind { FEW, RING, WIDE };

// A kernel and what its launches cost, in us: `start`; a K step (bk bytes of it) of all
// blocks that run at once, and the share by which it grows with each token; the weights'
// bytes at tbs TB/s; the share of the shorter of steps and weights that shows; `skew`: the
// share by which a step grows where rows do not start on 128 bytes; a further round of
// blocks; a join and its bytes; `channels`: the share by which weights slow down where
// ranges of K start a multiple of 4 KB apart and read the same memory channels.
struct Shape {
    Kind kind;
    int bm, bn, bk, threads, slots;  // slots: blocks that run at once on 256 CUs
    float start, step, token, tbs, both, skew, round, join, join_tbs, channels;
};

// Fitted to 16 000 launches of 580 products (M 1 .. 4096, N 64 .. 50272, K 16 .. 36864, cold
// weights, in recorded graphs; mean error 4-10% a kernel).  The chosen kernel and split was 1.6%
// above the fastest in up to 16 splits in the mean, 6% at the 90th percentile.  Kernels that
// gained less than 0.2% beside these are not kept (16 waves or 32 features for few tokens,
// 512-byte rows).
constexpr Shape SHAPES[] = {
    {FEW, 16, 16, 256, 256, 2048, 2.62f, 0.106f, 0.211f, 4.99f, 0.91f, 0.67f, 0.0f, 0, 0, 0},
    {FEW, 16, 16, 256, 512, 256, 2.54f, 0.175f, 0.027f, 6.88f, 0.37f, 0.03f, 0, 0, 0, 0},
    {RING, 32, 32, 256, 128, 512, 3.16f, 0.273f, 0, 7.72f, 0.79f, 0.17f, 1.9f, 2.4f, 4.5f, 0.01f},
    {RING, 32, 64, 256, 256, 256, 3.32f, 0.304f, 0, 8.67f, 0.78f, 0.33f, 2.1f, 2.6f, 8.7f, 0.02f},
    {RING, 64, 64, 256, 256, 256, 3.85f, 0.473f, 0, 7.70f, 0.37f, 0.23f, 2.7f, 2.4f, 10.6f, 0.03f},
    {RING, 64, 128, 128, 512, 256, 3.53f, 0.335f, 0, 9.57f, 0.72f, 0.13f, 2.4f, 2.2f, 9.0f, 0.32f},
    {RING, 128, 64, 256, 256, 256, 4.42f, 0.718f, 0, 5.45f, 0.19f, 0.12f, 2.7f, 2.3f, 8.9f, 0.10f},
    {RING, 128, 128, 128, 512, 256, 4.30f, 0.492f, 0, 7.09f, 0.34f, 0.12f, 3.0f, 2.8f, 8.3f, 0.28f},
    {WIDE, 128, 256, 128, 512, 256, 5.84f, 0.706f, 0, 8.68f, 0.70f, 0.28f, 3.6f, 3.0f, 8.0f, 0.32f},
    {WIDE, 192, 256, 128, 512, 256, 7.24f, 0.874f, 0, 6.91f, 0.41f, 0.41f, 5.4f, 2.9f, 8.2f, 0.31f},
    {WIDE, 256, 256, 128, 512, 256, 8.99f, 1.040f, 0, 6.90f, 0.29f, 0.46f, 6.9f, 2.4f, 8.5f, 0.83f},
};
constexpr int N_SHAPES = sizeof(SHAPES) / sizeof(SHAPES[0]);

// splits > 1: the K steps of the last `tail` tiles in that many ranges.
struct Plan {
    int shape, splits, tail;
};

inline int tiles_of(const GemmQ8Params& p, const Shape& c) { return ((p.M + c.bm - 1) / c.bm) * ((p.N + c.bn - 1) / c.bn); }

inline size_t bytes_of(const Plan& c) {
    return c.splits > 1 ? (size_t)c.tail * c.splits * SHAPES[c.shape].bm * SHAPES[c.shape].bn * 4 : 0;
}

// Whether some row starts inside 128 bytes.
inline bool skewed(const GemmQ8Params& p) {
    return (((uintptr_t)p.W | (uintptr_t)p.X | (uintptr_t)p.ldw | (uintptr_t)p.ldx) & 127) != 0;
}

// The numbers of tokens that a kernel is considered for (tall tiles of few tokens would be idle).
constexpr int fewest_tokens(const Shape& c) { return c.kind == WIDE ? 65 : c.kind == RING && c.bm == 128 ? 33 : 1; }
constexpr int most_tokens(const Shape& c) { return c.kind == FEW ? 16 : c.bm == 32 ? 64 : c.bm == 64 ? 512 : 1 << 24; }

// Ranges of K that tiles are cut into, if a range has two steps and the ranges fit the chip at once:
// of all tiles (fewer than slots), or of a last round's (256 blocks).
constexpr int ALL_SPLITS[] = {16, 12, 8, 6, 5, 4, 3, 2}, TAIL_SPLITS[] = {8, 6, 5, 4, 3, 2};

// Weight rows a multiple of 4 KB apart have the same K on the same memory channels, so blocks
// in step ask few of them at a time: where copies fetch 256 bytes of a row, columns of tiles
// start at 16 places of K (cold weights: 7 x 36864 x 8192 65 -> 58 us, 24 x 16384 x 4096 18.1 ->
// 16.2, 48 x 16384 x 8192 34.5 -> 29.3).  Copies of 128 bytes lose by it (69 -> 90 us in tiles of
// 64 x 128), as do more tokens, whose rows would come from beyond the L2 several times.
inline int phases_of(const GemmQ8Params& p, const Shape& c) { return c.kind == RING && c.bk == 256 && p.M <= 128 && p.ldw % 4096 == 0 && !skewed(p) ? 16 : 1; }

// Predicted time of a launch: whole rounds of tiles, then what is left of them, then the
// ranges of split tiles, each round as long as its K steps; beside it the weights, of the
// shorter one the share `both`.  (Shapes as constants: a choice takes 0.04 to 0.23 us of a call,
// 0.1 to 0.5 as data.)
template <int I>
float time_of(const GemmQ8Params& p, bool skew, int split, int tail, int tiles, int whole) {
    constexpr Shape c = SHAPES[I];
    int kt = whole, splits = 1;
    if (split > 1) {
        kt = (whole + split - 1) / split;
        splits = (whole + kt - 1) / kt;
        if (splits == 1) tail = 0;
    }
    const int rounds = (tiles - tail + c.slots - 1) / c.slots, cut = (tail * splits + c.slots - 1) / c.slots;
    float work = (float)(rounds * whole + cut * kt) * c.step, weights = (float)p.N * (float)p.K * (1e-6f / c.tbs);
    if (skew) work *= 1.f + c.skew;
    work *= 1.f + c.token * (float)p.M;
    if (tail && kt * c.bk % 4096 == 0) weights *= 1.f + c.channels;
    float t = c.start + fmaxf(work, weights) + c.both * fminf(work, weights) + (float)(rounds + cut - 1) * c.round;
    if (p.K % c.bk) t += 0.6f;
    // (0.5: the join's launch where no graph replays it)
    if constexpr (c.kind != FEW)
        if (tail) t += c.join + 0.5f + (float)(tail * splits) * ((float)(c.bm * c.bn) * 8e-6f / c.join_tbs);
    return t;
}

struct Choice {
    Plan plan;
    float t;
};

template <int I>
void consider(const GemmQ8Params& p, bool skew, size_t room, Choice& best) {
    constexpr Shape c = SHAPES[I];
    // 4 waves for few tokens from 12288 features on, where blocks are many (measured side by side)
    if (p.M < fewest_tokens(c) || p.M > most_tokens(c) || (c.kind == WIDE && p.K < 128)) return;
    if (c.kind == FEW && (c.threads == 256) != (p.N >= 12288)) return;
    const int tiles = tiles_of(p, c), whole = p.K / c.bk;
    auto take = [&](int split, int tail) {
        if (split > 1 && bytes_of({I, split, tail}) > room) return;
        const float t = time_of<I>(p, skew, split, tail, tiles, whole);
        if (best.plan.shape < 0 || t < best.t) best = {{I, split, tail}, t};
    };
    take(1, 0);
    if (c.kind == FEW) return;
    // the splits that come next to filling the chip: of all tiles, or of a last round's
    int tried = 0;
    if (tiles < c.slots) {
        for (const int s : ALL_SPLITS)
            if (tried < 3 && s * tiles <= c.slots && whole >= 2 * s) {
                take(s, tiles);
                ++tried;
            }
    } else if (const int tail = tiles % 256) {
        for (const int s : TAIL_SPLITS)
            if (tried < 2 && s * tail <= 256 && whole >= 2 * s) {
                take(s, tail);
                ++tried;
            }
    }
}

template <int... I>
Plan best_of(const GemmQ8Params& p, size_t room, std::integer_sequence<int, I...>) {
    Choice best{{-1, 1, 0}, 0.f};
    const bool skew = skewed(p);
    (consider<I>(p, skew, room, best), ...);
    return best.plan;
}

inline Plan plan_of(const GemmQ8Params& p, size_t room) { return best_of(p, room, std::make_integer_sequence<int, N_SHAPES>()); }

// How a plan's tiles and ranges lie.
inline Split split_of(const GemmQ8Params& p, const Plan& c) {
    const Shape& shape = SHAPES[c.shape];
    const int tiles = tiles_of(p, shape), whole = p.K / shape.bk;
    Split sp{tiles, 0, 1, whole, phases_of(p, shape)};
    if (c.splits > 1) {
        sp.kt = (whole + c.splits - 1) / c.splits;
        sp.splits = (whole + sp.kt - 1) / sp.kt;
        if (sp.splits > 1) {
            sp.tail = c.tail;
            sp.full = tiles - c.tail;
        }
    }
    return sp;
}

// Bytes that hold the sums of every plan for up to p.M tokens, whatever the rows' strides: a
// kernel's ranges are at most the largest split's of all its tiles, and at most its slots.
inline size_t workspace_of(const GemmQ8Params& p) {
    size_t most = 0;
    for (const Shape& c : SHAPES) {
        if (c.kind == FEW || p.M < fewest_tokens(c) || (c.kind == WIDE && p.K < 128)) continue;
        GemmQ8Params q = p;
        q.M = p.M < most_tokens(c) ? p.M : most_tokens(c);
        for (const int s : ALL_SPLITS) {
            if (p.K / c.bk < 2 * s) continue;
            const int64_t ranges = (int64_t)tiles_of(q, c) * s;
            const size_t bytes = (size_t)(ranges < c.slots ? ranges : c.slots) * c.bm * c.bn * 4;
            most = bytes > most ? bytes : most;
            break;
        }
    }
    return most;
}

}  // namespace pb::q8
