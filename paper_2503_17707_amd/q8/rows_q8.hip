// Rows in 8 bits: norm_q8 (residual addition, RMS or layer norm, quantization) and
// quant_q8 (quantization alone).
//
// A row's scale is max|y| / 127 as fp32, its numbers rint(y / scale).  The whole of it
// is formed in fp64 from the stored row: sums, the norm, the largest magnitude and the
// quotient, so the numbers are those of the formula but where y / scale lies within
// about 2^-45 of the border of two integers, and neither the order of a sum nor the
// split of a row over lanes shows in them.  (In fp32 one number in some 50 000 would
// be off by one step.)  CDNA4 does fp64 outside the matrix units at half the rate of
// fp32.  A layer norm with a bias takes some fourteen such operations an element and, of rows
// of several pieces a thread, eight or nine conversions (an element is widened again for each
// use).  With a delta to read and a sum to write that keeps the vector units busy for two thirds
// of the time; without, it is the bound: 4096 rows of 9216 in fp32 62 us, 3.1 TB/s, the vector
// units 0.78 busy (RMS without a bias, nine operations: 44 us, 4.3 TB/s).
//
// Both read a row once into registers (fp32) and write it once: 4096 rows of 9216, fp32
// stream and fp16 delta, 82-89 us (4.7-5.1 TB/s, a large copy 4.76); 4096 of 36864 in fp16
// 83-88 us (5.1-5.5); 1001 of 4091 in bf16, one round of blocks, 11-13 us (2.9-3.4).  Few
// rows are bound by the latency of one load, the reductions and one store (one of 2048: 2.6 us).
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "../csrc/common.h"
#include "q8.h"

namespace pb {

namespace {

// VEC elements at any address of their own type: rows of odd widths start anywhere, and
// global memory serves vectors there too.
template <typename T, int VEC>
struct Pack {
    T v[VEC];
};

template <int VEC, typename T>
__device__ __forceinline__ Pack<T, VEC> load_pack(const T* p) {
    Pack<T, VEC> a;
    __builtin_memcpy(&a, p, sizeof(a));
    return a;
}

template <typename T, typename F, int VEC>
__device__ __forceinline__ void store_pack(T* p, const F (&f)[VEC]) {
    Pack<T, VEC> a;
#pragma unroll
    for (int e = 0; e < VEC; ++e) a.v[e] = (T)f[e];
    __builtin_memcpy(p, &a, sizeof(a));
}

// Piece i of a lane: VEC elements of a row of d >= VEC.  The last one, where it is cut
// short, is moved back to end with the row, over `over` elements of the piece before it
// (as all pieces past the end are: over >= VEC).  So every lane loads whole vectors, with
// no branch between one load and the next, and an element taken twice gives the same
// result twice; only sums have to leave it out.  Only a lane's last piece can be so: the
// launches give a row as many pieces as it needs and no more.
template <int VEC>
struct Place {
    uint32_t at;
    int over;
    __device__ Place(int i, bool last, int threads, int lane, int d) {
        const int c = (i * threads + lane) * VEC;
        at = last ? min(c, d - VEC) : c;
        over = c - (int)at;
    }
};

// Element `at` of a row (rows of a block share a scalar base: a lane's part is 32 bits).
template <typename T>
__device__ __forceinline__ const T* element(const T* row, uint32_t at) {
    return (const T*)((const char*)row + (uint32_t)(at * (uint32_t)sizeof(T)));
}

template <typename T>
__device__ __forceinline__ T* element(T* row, uint32_t at) {
    return (T*)((char*)row + (uint32_t)(at * (uint32_t)sizeof(T)));
}

// Other lanes' values without a way through LDS: within rows of 16 by DPP (quad_perm 1 0
// 3 2, quad_perm 2 3 0 1, row_half_mirror, row_mirror), across rows by permlane swaps.
template <int STEP>
__device__ __forceinline__ uint32_t from_lane(uint32_t v) {
    if constexpr (STEP == 0) return __builtin_amdgcn_mov_dpp(v, 0xB1, 0xf, 0xf, false);
    if constexpr (STEP == 1) return __builtin_amdgcn_mov_dpp(v, 0x4E, 0xf, 0xf, false);
    if constexpr (STEP == 2) return __builtin_amdgcn_mov_dpp(v, 0x141, 0xf, 0xf, false);
    return __builtin_amdgcn_mov_dpp(v, 0x140, 0xf, 0xf, false);
}

// One value over groups of 16, 32 or 64 lanes.
template <int LANES, typename F>
__device__ __forceinline__ double lanes_fold(double v, F f) {
    auto word = [&](int k) { return (uint32_t)(__builtin_bit_cast(uint64_t, v) >> (32 * k)); };
    auto value = [](uint32_t lo, uint32_t hi) { return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo); };
    v = f(v, value(from_lane<0>(word(0)), from_lane<0>(word(1))));
    v = f(v, value(from_lane<1>(word(0)), from_lane<1>(word(1))));
    v = f(v, value(from_lane<2>(word(0)), from_lane<2>(word(1))));
    v = f(v, value(from_lane<3>(word(0)), from_lane<3>(word(1))));
    if constexpr (LANES > 16) {
        const auto lo = __builtin_amdgcn_permlane16_swap(word(0), word(0), false, false);
        const auto hi = __builtin_amdgcn_permlane16_swap(word(1), word(1), false, false);
        v = f(value(lo[0], hi[0]), value(lo[1], hi[1]));
    }
    if constexpr (LANES > 32) {
        const auto lo = __builtin_amdgcn_permlane32_swap(word(0), word(0), false, false);
        const auto hi = __builtin_amdgcn_permlane32_swap(word(1), word(1), false, false);
        v = f(value(lo[0], hi[0]), value(lo[1], hi[1]));
    }
    return v;
}

// One value over a row's threads: LANES of a wave, or (LANES = 0) a block of any number of
// waves, by one use of `lds`.
template <int LANES, typename F>
__device__ __forceinline__ double row_fold(double v, double* lds, F f) {
    v = lanes_fold<(LANES ? LANES : 64)>(v, f);
    if constexpr (LANES == 0) {  // (folds of zero and more than 16 waves there are none)
        const int lane = threadIdx.x & 63;
        if (lane == 0) lds[threadIdx.x >> 6] = v;
        lds_barrier();
        v = (lane & 15) < (int)blockDim.x / 64 ? lds[lane & 15] : 0.0;
        v = lanes_fold<16>(v, f);
    }
    return v;
}

// Two at once.
template <int LANES, typename F, typename G>
__device__ __forceinline__ void row_fold2(double& a, double& b, double (*lds)[2], F f, G g) {
    a = lanes_fold<(LANES ? LANES : 64)>(a, f);
    b = lanes_fold<(LANES ? LANES : 64)>(b, g);
    if constexpr (LANES == 0) {
        if ((threadIdx.x & 63) == 0) {
            lds[threadIdx.x >> 6][0] = a;
            lds[threadIdx.x >> 6][1] = b;
        }
        lds_barrier();
        const int lane = threadIdx.x & 63;
        const bool in = (lane & 15) < (int)blockDim.x / 64;
        a = lanes_fold<16>(in ? lds[lane & 15][0] : 0.0, f);
        b = lanes_fold<16>(in ? lds[lane & 15][1] : 0.0, g);
    }
}

struct Plus {
    __device__ double operator()(double a, double b) const { return a + b; }
};
struct Larger {
    __device__ double operator()(double a, double b) const { return fmax(a, b); }
};

// max(top, |y|) in one instruction (fmax() quiets both operands first; a NaN is left out here).
__device__ __forceinline__ double max_abs(double top, double y) {
    asm("v_max_f64 %0, %0, |%1|" : "+v"(top) : "v"(y));
    return top;
}

// Whether one of VEC gains or biases is a NaN or an infinity: all bits of its exponent set.
template <typename T, int VEC>
__device__ __forceinline__ bool not_finite(const Pack<T, VEC>& x) {
    constexpr uint16_t BITS = std::is_same_v<T, __bf16> ? 0x7f80 : 0x7c00;
    if constexpr (VEC == 1) return (__builtin_bit_cast(uint16_t, x.v[0]) & BITS) == BITS;
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    u16x2 w[VEC / 2 + VEC % 2], top = {0, 0};
    __builtin_memcpy(w, &x, sizeof(x));
#pragma unroll
    for (int k = 0; k < VEC / 2; ++k) top = __builtin_elementwise_max(top, w[k] & u16x2{0x7fff, 0x7fff});
    return top[0] >= BITS || top[1] >= BITS;
}

// A value that all lanes hold, in scalar registers: it leaves vector registers for more waves
// or loads (10000 rows of 3000 in fp32 82 -> 77 us, 1831 of 16384 in fp16 66 -> 65).
template <bool SCALAR>
__device__ __forceinline__ double of_row(double v) {
    if constexpr (!SCALAR) return v;
    const uint64_t w = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)w), hi = __builtin_amdgcn_readfirstlane((uint32_t)(w >> 32));
    return __builtin_bit_cast(double, (uint64_t)hi << 32 | lo);
}

// Keeps the compiler from holding a conversion made before this point: kept as fp64, a
// row's elements would take the registers of half the waves.
template <typename T, int VEC>
__device__ __forceinline__ void again(Pack<T, VEC>& x) {
    if constexpr (sizeof(x) % 4 == 0) {
        uint32_t w[sizeof(x) / 4];
        __builtin_memcpy(w, &x, sizeof(x));
#pragma unroll
        for (uint32_t& k : w) asm volatile("" : "+v"(k));
        __builtin_memcpy(&x, w, sizeof(x));
    }
}

template <int VEC>
__device__ __forceinline__ void again(float (&x)[VEC]) {
#pragma unroll
    for (float& k : x) asm volatile("" : "+v"(k));
}

// 1 / sqrt(x) and 1 / x from the hardware's approximations and two steps of Newton, a few units
// of the last place off (the library's are 30 operations and more, of every wave of a row).
__device__ __forceinline__ double rsqrt64(double x) {
    double r = __builtin_amdgcn_rsq(x);
    if (x > 0.0 && x < INFINITY) {
        r = fma(r * 0.5, fma(-x * r, r, 1.0), r);
        r = fma(r * 0.5, fma(-x * r, r, 1.0), r);
    }
    return r;
}

__device__ __forceinline__ double reciprocal64(float x) {  // (of a scale; 0 for none)
    if (!(x > 0.f)) return 0.0;
    double r = __builtin_amdgcn_rcp((double)x);
    r = fma(fma(-(double)x, r, 1.0), r, r);
    return fma(fma(-(double)x, r, 1.0), r, r);
}

// The scale of a row whose largest magnitude is `top` (NaN: some value is no number).
__device__ __forceinline__ float row_scale(double top) {
    const float s = (float)(top * (1.0 / 127.0));
    if (!(s <= 3.402823466e38f)) return __builtin_nanf("");
    return s < 1.17549435e-38f ? 0.f : s;  // rows below it are zeros: a subnormal scale holds too few bits
}

// rint(y / scale), at most 127: a product with the reciprocal and one correction, exact where
// the quotient is a number of 53 bits, so that ties are ties.  Added to 1.5 2^52, which has no
// bits below 1, it is rounded to the nearest integer, ties to even, in the low word.
__device__ __forceinline__ int quotient(double y, double scale, double inv) {
    const double t = y * inv;
    return (int)(uint32_t)__builtin_bit_cast(uint64_t, fma(fma(-scale, t, y), inv, t) + 6755399441055744.0);
}

// (a scale that is zero or no number: zeros)
template <int VEC>
__device__ __forceinline__ void store_q(int8_t* p, const double (&y)[VEC], float scale, double inv) {
    int r[VEC] = {};
    if (scale > 0.f) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) r[e] = quotient(y[e], (double)scale, inv);
    }
    store_pack<int8_t, int, VEC>(p, r);
}

// (12 fp32 or 16 16-bit elements a thread; 16 fp32 ones leave no registers for more)
constexpr bool loads_ahead(int vec, int nv, int lanes) { return lanes == 0 && (vec == 4 ? nv == 3 : nv == 2); }

// S: type of the stream, T: storage type.  LANES threads (0: a block) take a row of d >= VEC
// in NV pieces of VEC elements each; BIAS: b is given (without it the largest magnitude is
// known with the sum of squares).
template <typename T, typename S, int VEC, int NV, int LANES, bool BIAS>
__global__ __launch_bounds__(LANES ? 256 : 1024) __attribute__((amdgpu_waves_per_eu(4))) void norm_q8_kernel(NormQ8Params p) {
    constexpr int RPB = LANES ? 256 / LANES : 1;
    __shared__ double lds1[16], lds3[16], lds2[16][2];
    const int lane = LANES ? threadIdx.x % LANES : threadIdx.x;
    const int threads = LANES ? LANES : blockDim.x;
    const int first = LANES ? (int)blockIdx.x * RPB + (int)threadIdx.x / LANES : blockIdx.x;
    const int step = (int)gridDim.x * RPB;
    // Long rows are walked over, the next one loaded while one is worked on; gains and biases
    // stay (4096 x 9216 in fp32: 114 -> 96 us).
    constexpr bool AHEAD = loads_ahead(VEC, NV, LANES);
    // (not with a thread's one piece of eight elements: past 80 scalar registers a SIMD holds
    // seven waves, not eight, and a CU one block of 1024; 3662 rows of 8192 in fp16 61 -> 83 us)
    constexpr bool SCALAR = LANES == 0 && (VEC == 4 || NV > 1);
    const double width = SCALAR ? p.width : (double)p.d;
    Pack<S, VEC> x[NV];
    Pack<T, VEC> t[NV], g[NV], b[NV];
    auto place = [&](int i) { return Place<VEC>(i, i == NV - 1, threads, lane, p.d); };
    auto load_row = [&](int row) {
#pragma unroll
        for (int i = 0; i < NV; ++i) x[i] = load_pack<VEC>(element((const S*)p.x + (int64_t)row * p.ld_x, place(i).at));
        if (p.delta) {
#pragma unroll
            for (int i = 0; i < NV; ++i) t[i] = load_pack<VEC>(element((const T*)p.delta + (int64_t)row * p.ld_delta, place(i).at));
        }
    };
    auto load_gains = [&] {
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            g[i] = load_pack<VEC>(element((const T*)p.g, place(i).at));
            if constexpr (BIAS) b[i] = load_pack<VEC>(element((const T*)p.b, place(i).at));
        }
    };
    bool bad = false;  // a gain or bias that is no finite number: no y of its column is
    auto check_gains = [&] {
        bad = false;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            bad |= not_finite(g[i]);
            if constexpr (BIAS) bad |= not_finite(b[i]);
        }
    };
    // total and the terms of piece i's own elements
    auto add_piece = [&](int i, double total, auto term) {
        double all = total;
#pragma unroll
        for (int e = 0; e < VEC; ++e) all = term(e, all);
        if (i < NV - 1) return all;
        const int over = place(i).over;
        if (over) {  // (lanes of few waves)
            all = total;
#pragma unroll
            for (int e = 0; e < VEC; ++e) all = e >= over ? term(e, all) : all;
        }
        return all;
    };
    if (AHEAD) {
        load_row(min(first, p.rows - 1));
        load_gains();
        check_gains();
    }
    for (int row = first; row < p.rows; row += step) {
        if (!AHEAD) {
            load_row(row);
            load_gains();
        }
        float s[NV][VEC];
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[i][e] = (float)x[i].v[e];
        if (p.delta) {  // the norm is taken of the sum as the stream keeps it
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[i][e] = (float)(S)(s[i][e] + (float)t[i].v[e]);
        }
        if (AHEAD && row + step < p.rows) load_row(row + step);
        // s - mean, then y, are kept in fp64 where a thread has one piece; of more they are formed
        // again for each use (kept, they would cost a long row half of its waves)
        constexpr bool KEPT = NV == 1;
        double kept[VEC];
        if (KEPT) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) kept[e] = (double)s[0][e];
        }
        double mean = 0.0;
        if (p.layer) {
            double sum = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                sum = add_piece(i, sum, [&](int e, double a) { return a + (KEPT ? kept[e] : (double)s[i][e]); });
            sum = row_fold<LANES>(sum, lds1, Plus());
            mean = sum * p.inv_d;  // and one step of division: rows of one value have it as their mean
            mean = of_row<SCALAR>(fma(fma(-width, mean, sum), p.inv_d, mean));
            if (KEPT) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) kept[e] -= mean;
            }
        }
        auto centred = [&](int i, int e) { return KEPT ? kept[e] : (double)s[i][e] - mean; };
        double square = 0.0, top = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            if (!KEPT) again(s[i]);
            square = add_piece(i, square, [&](int e, double a) {
                const double v = centred(i, e);
                return fma(v, v, a);
            });
            if (!BIAS) {
#pragma unroll
                for (int e = 0; e < VEC; ++e) top = max_abs(top, centred(i, e) * (double)(float)g[i].v[e]);
            }
        }
        if (!AHEAD && !BIAS) check_gains();
        if (BIAS) {
            square = row_fold<LANES>(square, &lds2[0][0], Plus());
        } else {
            if (bad) top = INFINITY;
            row_fold2<LANES>(square, top, lds2, Plus(), Larger());
        }
        // (fp64 products of fp32 numbers do not overflow: where the variance is a positive number
        // and gains and biases are finite, so is every y)
        const double var = fma(square, p.inv_d, (double)p.eps);
        const double rstd = of_row<SCALAR>(rsqrt64(var));
        const bool none = !(var > 0.0 && var < INFINITY);
        // every lane has read its row: the sum may take its place
        if (p.sum) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const Place<VEC> at = place(i);
                if (at.over < VEC) store_pack<S, float, VEC>(element((S*)p.sum + (int64_t)row * p.ld_sum, at.at), s[i]);
            }
        }
        auto normed = [&](int i, double (&y)[VEC]) {
            if (!KEPT) again(s[i]);
            again(g[i]);
            if (BIAS) again(b[i]);
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double v = centred(i, e) * rstd, gain = (double)(float)g[i].v[e];
                if constexpr (BIAS) y[e] = fma(v, gain, (double)(float)b[i].v[e]);
                else y[e] = v * gain;
            }
        };
        double y[VEC];
        if (KEPT) normed(0, y);
        if (BIAS || p.out) {
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const Place<VEC> at = place(i);
                if (!KEPT) normed(i, y);
                if (BIAS) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) top = max_abs(top, y[e]);
                    asm volatile("" : "+v"(top));  // (y is used up here)
                }
                if (p.out) {
                    float f[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e) f[e] = (float)y[e];
                    if (at.over < VEC) store_pack<T, float, VEC>(element((T*)p.out + (int64_t)row * p.ld_out, at.at), f);
                }
            }
        }
        if (!p.q) {
            if (LANES == 0) lds_barrier();
            continue;
        }
        if (BIAS) {
            if (!AHEAD) check_gains();
            if (bad) top = INFINITY;
            top = row_fold<LANES>(top, lds3, Larger());
        } else {
            top *= rstd;
        }
        if (none) top = INFINITY;
        const float scale = row_scale(top);
        const double inv = reciprocal64(scale);
        if (lane == 0) p.scale[row] = scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const Place<VEC> at = place(i);
            if (!KEPT) normed(i, y);
            if (at.over < VEC) store_q<VEC>(element(p.q + (int64_t)row * p.ld_q, at.at), y, scale, inv);
        }
        if (LANES == 0) lds_barrier();  // the places in LDS are free for the next row
    }
}

// The largest magnitude of some values as bits of fp32 (NaN above infinity above numbers).
template <typename S, int VEC>
__device__ __forceinline__ uint32_t largest_bits(uint32_t top, const Pack<S, VEC>& x) {
#pragma unroll
    for (int e = 0; e < VEC; ++e) top = max(top, __float_as_uint((float)x.v[e]) & 0x7fffffffu);
    return top;
}

template <int TPR>
__device__ __forceinline__ uint32_t row_largest(uint32_t v, uint32_t* lds) {
    v = max(v, from_lane<0>(v));
    v = max(v, from_lane<1>(v));
    v = max(v, from_lane<2>(v));
    v = max(v, from_lane<3>(v));
    if constexpr (TPR > 16) {
        const auto a = __builtin_amdgcn_permlane16_swap(v, v, false, false);
        v = max(a[0], a[1]);
    }
    if constexpr (TPR > 32) {
        const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
        v = max(b[0], b[1]);
    }
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
        lds_barrier();
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) v = max(v, lds[w]);
        lds_barrier();
    }
    return v;
}

// NV pieces a thread; NV = 0: rows of any length, read twice (the second time from the
// caches).
template <typename S, int VEC, int NV, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void quant_q8_kernel(QuantQ8Params p) {
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    static_assert(TPR <= 64 || RPB == 1, "rows of several waves have a block each");
    __shared__ uint32_t lds[TPR < 64 ? 1 : TPR / 64];
    const int lane = threadIdx.x % TPR;
    const int pieces = (p.cols + VEC * TPR - 1) / (VEC * TPR);
    const int first = RPB == 1 ? blockIdx.x : (int)blockIdx.x * RPB + (int)threadIdx.x / TPR;
    for (int row = first; row < p.rows; row += (int)gridDim.x * RPB) {
        const S* src = (const S*)p.x + (int64_t)row * p.ld_x;
        int8_t* dst = p.q + (int64_t)row * p.ld_q;
        Pack<S, VEC> x[NV ? NV : 1];
        uint32_t top = 0;
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) x[i] = load_pack<VEC>(src + Place<VEC>(i, NV == 0 || i == NV - 1, TPR, lane, p.cols).at);
#pragma unroll
            for (int i = 0; i < NV; ++i) top = largest_bits<S, VEC>(top, x[i]);
        } else {
            for (int i = 0; i < pieces; ++i)
                top = largest_bits<S, VEC>(top, load_pack<VEC>(src + Place<VEC>(i, NV == 0 || i == NV - 1, TPR, lane, p.cols).at));
        }
        const float scale = row_scale((double)__uint_as_float(row_largest<TPR>(top, lds)));
        const double inv = reciprocal64(scale);
        if (lane == 0) p.scale[row] = scale;
        auto store = [&](const Place<VEC>& at, const Pack<S, VEC>& v) {
            double y[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = (double)(float)v.v[e];
            if (at.over < VEC) store_q<VEC>(dst + at.at, y, scale, inv);
        };
        if constexpr (NV > 0) {
#pragma unroll
            for (int i = 0; i < NV; ++i) store(Place<VEC>(i, NV == 0 || i == NV - 1, TPR, lane, p.cols), x[i]);
        } else {
            for (int i = 0; i < pieces; ++i) {
                const Place<VEC> at(i, true, TPR, lane, p.cols);
                store(at, load_pack<VEC>(src + at.at));
            }
        }
    }
}

// Blocks walk over rows where a launch would hold too many (row numbers plus a step stay
// below 2^31).
int row_blocks(int rows, int per_block) {
    const int n = rows / per_block + (rows % per_block != 0);
    return n < (1 << 18) ? n : 1 << 18;
}

template <typename T, typename S, int VEC, int NV, int LANES>
void norm_nv(const NormQ8Params& p, int threads, hipStream_t s) {
    int blocks = row_blocks(p.rows, LANES ? 256 / LANES : 1);
    if (loads_ahead(VEC, NV, LANES)) blocks = std::min(blocks, 256 * (1024 / threads));  // whole blocks of 16 waves a CU
    if (p.b) PB_LAUNCH((norm_q8_kernel<T, S, VEC, NV, LANES, true>), blocks, threads, 0, s, p);
    else PB_LAUNCH((norm_q8_kernel<T, S, VEC, NV, LANES, false>), blocks, threads, 0, s, p);
}

template <typename S, int VEC, int NV, int TPR>
void quant_nv(const QuantQ8Params& p, hipStream_t s) {
    PB_LAUNCH((quant_q8_kernel<S, VEC, NV, TPR>), row_blocks(p.rows, TPR < 256 ? 256 / TPR : 1), TPR < 256 ? 256 : TPR, 0, s, p);
}

// Rows of up to 128 pieces share waves.  Longer ones have a block each, of a piece (16 bits) or
// two (fp32) a thread, as many waves as may be; from there on rows are walked over with the
// next one's loads in flight, 12 fp32 or 16 16-bit elements a thread
// (30 M elements in fp32, two pieces a thread without loads ahead -> three with: rows of 4104
// 90 -> 78 us, 6144 72 -> 69, 8192 95 -> 76, but 3600 71 -> 83; in fp16, one piece -> two: 8192
// 58 -> 53, 6656 64 -> 60, 6144 59 -> 62).  16 fp32 elements leave no registers to load ahead.
// A CU gets the whole blocks that 16 waves hold: 9 waves to 16, fewest just past 512 threads (layer norm
// of 30 M elements with a delta, fp32: 6144 67 us, 6148 81, 7168 76, 8192 73; fp16: 8192 50, 8200 66, 9216
// 61, 10240 58).
template <typename T, typename S>
void norm_type(const NormQ8Params& p, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S), MOST = 1024;
    const int n = (p.d + VEC - 1) / VEC;  // pieces
    auto waves = [&](int pieces) { return ((n + pieces - 1) / pieces + 63) / 64 * 64; };
    if (p.d < VEC) norm_nv<T, S, 1, 1, 16>(p, 256, s);
    else if (n <= 16) norm_nv<T, S, VEC, 1, 16>(p, 256, s);
    else if (n <= 32) norm_nv<T, S, VEC, 1, 32>(p, 256, s);
    else if (n <= 64) norm_nv<T, S, VEC, 1, 64>(p, 256, s);
    else if constexpr (VEC == 8) {
        if (n <= 768) norm_nv<T, S, VEC, 1, 0>(p, waves(1), s);
        else norm_nv<T, S, VEC, 2, 0>(p, waves(2), s);
    } else {
        if (n <= 128) norm_nv<T, S, VEC, 2, 64>(p, 256, s);
        else if (n <= MOST) norm_nv<T, S, VEC, 2, 0>(p, waves(2), s);
        else if (n <= 3 * MOST) norm_nv<T, S, VEC, 3, 0>(p, waves(3), s);
        else norm_nv<T, S, VEC, 4, 0>(p, waves(4), s);
    }
}

// A row of n pieces on TPR threads with NV pieces each, where they hold it.
template <typename S, int VEC, int NV, int TPR>
bool quant_on(const QuantQ8Params& p, int n, hipStream_t s) {
    if (n > NV * TPR) return false;
    quant_nv<S, VEC, NV, TPR>(p, s);
    return true;
}

// The smallest number of registers that holds a row; longer rows than 1024 threads hold in
// eight pieces are read twice (NV 0).
template <typename S>
void quant_type(const QuantQ8Params& p, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    const int n = (int)(((int64_t)p.cols + VEC - 1) / VEC);
    if (p.cols < VEC) {
        quant_nv<S, 1, 1, 16>(p, s);
        return;
    }
    const bool held = quant_on<S, VEC, 1, 16>(p, n, s) || quant_on<S, VEC, 1, 32>(p, n, s) || quant_on<S, VEC, 1, 64>(p, n, s) ||
                      quant_on<S, VEC, 2, 64>(p, n, s) || quant_on<S, VEC, 1, 256>(p, n, s) || quant_on<S, VEC, 2, 256>(p, n, s) ||
                      quant_on<S, VEC, 3, 256>(p, n, s) || quant_on<S, VEC, 4, 256>(p, n, s) || quant_on<S, VEC, 3, 512>(p, n, s) ||
                      quant_on<S, VEC, 4, 512>(p, n, s) || quant_on<S, VEC, 5, 512>(p, n, s) || quant_on<S, VEC, 3, 1024>(p, n, s) ||
                      quant_on<S, VEC, 4, 1024>(p, n, s) || quant_on<S, VEC, 5, 1024>(p, n, s) || quant_on<S, VEC, 6, 1024>(p, n, s) ||
                      quant_on<S, VEC, 7, 1024>(p, n, s) || quant_on<S, VEC, 8, 1024>(p, n, s);
    if (!held) quant_nv<S, VEC, 0, 1024>(p, s);
}

}  // namespace

hipError_t launch_norm_q8(int dtype, bool f32, const NormQ8Params& p, hipStream_t s) {
    if (dtype == 1) {
        if (f32) norm_type<_Float16, float>(p, s);
        else norm_type<_Float16, _Float16>(p, s);
    } else {
        if (f32) norm_type<__bf16, float>(p, s);
        else norm_type<__bf16, __bf16>(p, s);
    }
    return hipGetLastError();
}

hipError_t launch_quant_q8(int dtype, bool f32, const QuantQ8Params& p, hipStream_t s) {
    if (f32) quant_type<float>(p, s);
    else if (dtype == 1) quant_type<_Float16>(p, s);
    else quant_type<__bf16>(p, s);
    return hipGetLastError();
}

}  // namespace pb
