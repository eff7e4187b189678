// Rows in 8 bits: norm_q8 (residual addition, RMS or layer norm, quantization) and
// quant_q8 (quantization alone).
//
// A row's scale is max|y| / 127 as fp32, its numbers rint(y / scale).  The whole of it
// is formed in fp64 from the stored row: sums, the norm, the largest magnitude and the
// quotient, so the numbers are those of the formula but where y / scale lies within
// about 2^-45 of the border of two integers, and neither the order of a sum nor the
// split of a row over lanes shows in them.  (In fp32 one number in some 50 000 would
// be off by one step.)  CDNA4 does fp64 at the rate of fp32 outside the matrix units:
// some ten operations an element are a tenth of the time the memory takes.
//
// Both read a row once into registers (fp32) and write it once: bound by memory, for
// few rows by the latency of one load, the reductions and one store.
#include <cmath>
#include <type_traits>

#include "../csrc/common.h"
#include "q8.h"

namespace pb {

namespace {

// Elements at any address of their own type: rows of odd widths start anywhere, and
// global memory serves vectors there too.
template <typename T, int N>
struct Vec {
    T v[N];
};

template <typename T, int N>
__device__ __forceinline__ void load_some(const T* p, int left, float (&f)[N]) {
    if (left >= N) {
        Vec<T, N> a;
        __builtin_memcpy(&a, p, sizeof(a));
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = (float)a.v[e];
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e) f[e] = e < left ? (float)p[e] : 0.f;
    }
}

template <typename T, typename F, int N>
__device__ __forceinline__ void store_some(T* p, int left, const F (&f)[N]) {
    if (left >= N) {
        Vec<T, N> a;
#pragma unroll
        for (int e = 0; e < N; ++e) a.v[e] = (T)f[e];
        __builtin_memcpy(p, &a, sizeof(a));
    } else {
#pragma unroll
        for (int e = 0; e < N; ++e)
            if (e < left) p[e] = (T)f[e];
    }
}

// Two values over the TPR threads of a row: the sum of a, the larger of m.
template <int TPR>
__device__ __forceinline__ void row_reduce(double& a, double& m, double* lds) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        a += __shfl_xor(a, o, 64);
        m = fmax(m, __shfl_xor(m, o, 64));
    }
    if (TPR > 64) {
        constexpr int NW = TPR / 64;
        const int wave = threadIdx.x >> 6;
        if ((threadIdx.x & 63) == 0) {
            lds[wave] = a;
            lds[NW + wave] = m;
        }
        lds_barrier();
        a = lds[0];
        m = lds[NW];
#pragma unroll
        for (int w = 1; w < NW; ++w) {
            a += lds[w];
            m = fmax(m, lds[NW + w]);
        }
        lds_barrier();
    }
}

// The scale of a row whose largest magnitude is `top` (NaN where a value is no number).
__device__ __forceinline__ float row_scale(double top) {
    const float s = (float)(top / 127.0);
    if (!(s <= 3.402823466e38f)) return __builtin_nanf("");
    return s < 1.17549435e-38f ? 0.f : s;  // rows below it are zeros: a subnormal scale holds too few bits
}

// rint(y / scale): the quotient correctly rounded (a product with the rounded
// reciprocal and one correction), so that ties are ties.
__device__ __forceinline__ int quotient(double y, double scale, double inv) {
    const double t = y * inv;
    return (int)rint(fma(fma(-scale, t, y), inv, t));
}

template <int N>
__device__ __forceinline__ void store_q(int8_t* p, int left, const double (&y)[N], float scale, double inv) {
    int r[N];
#pragma unroll
    for (int e = 0; e < N; ++e) r[e] = scale > 0.f ? quotient(y[e], (double)scale, inv) : 0;
    store_some<int8_t, int, N>(p, left, r);
}

// S: type of the stream, T: storage type.  TPR threads take a row in NV pieces of VEC
// elements each.
template <typename T, typename S, int NV, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void norm_q8_kernel(NormQ8Params p) {
    constexpr int VEC = 16 / sizeof(S);
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    __shared__ double lds[2 * (TPR / 64)];
    const int lane = threadIdx.x % TPR;
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        float s[NV][VEC];
        double sum = 0.0, top = 0.0, square = 0.0, check = 0.0;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * VEC, left = p.d - c;
#pragma unroll
            for (int e = 0; e < VEC; ++e) s[i][e] = 0.f;
            if (left <= 0) continue;
            load_some<S, VEC>((const S*)p.x + row * p.ld_x + c, left, s[i]);
            if (p.delta) {
                float t[VEC];
                load_some<T, VEC>((const T*)p.delta + row * p.ld_delta + c, left, t);
                // the norm is taken of the sum as the stream keeps it
#pragma unroll
                for (int e = 0; e < VEC; ++e) s[i][e] = (float)(S)(s[i][e] + t[e]);
                if (p.sum) store_some<S, float, VEC>((S*)p.sum + row * p.ld_sum + c, left, s[i]);
            }
        }
        double mean = 0.0;
        if (p.layer) {
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < VEC; ++e) sum += (double)s[i][e];
            row_reduce<TPR>(sum, top, lds);
            mean = sum / p.d;
        }
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int left = p.d - (i * TPR + lane) * VEC;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const double v = (double)s[i][e] - mean;
                if (e < left) square = fma(v, v, square);
            }
        }
        row_reduce<TPR>(square, top, lds);
        const double rstd = 1.0 / sqrt(square / p.d + (double)p.eps);
        auto normed = [&](int i, double (&y)[VEC]) {
            const int c = (i * TPR + lane) * VEC, left = p.d - c;
            float g[VEC], b[VEC];
            load_some<T, VEC>((const T*)p.g + c, left, g);
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = ((double)s[i][e] - mean) * rstd * (double)g[e];
            if (p.b) {
                load_some<T, VEC>((const T*)p.b + c, left, b);
#pragma unroll
                for (int e = 0; e < VEC; ++e) y[e] += (double)b[e];
            }
        };
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * VEC, left = p.d - c;
            if (left <= 0) continue;
            double y[VEC];
            normed(i, y);
#pragma unroll
            for (int e = 0; e < VEC; ++e)
                if (e < left) {
                    top = fmax(top, fabs(y[e]));
                    check = fma(y[e], 0.0, check);  // NaN for what is no finite number
                }
            if (p.out) {
                float f[VEC];
#pragma unroll
                for (int e = 0; e < VEC; ++e) f[e] = (float)y[e];
                store_some<T, float, VEC>((T*)p.out + row * p.ld_out + c, left, f);
            }
        }
        if (!p.q) continue;
        row_reduce<TPR>(check, top, lds);
        const float scale = row_scale(top + check);
        const double inv = scale > 0.f ? 1.0 / (double)scale : 0.0;
        if (lane == 0) p.scale[row] = scale;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int c = (i * TPR + lane) * VEC, left = p.d - c;
            if (left <= 0) continue;
            double y[VEC];
            normed(i, y);
            store_q<VEC>(p.q + row * p.ld_q + c, left, y, scale, inv);
        }
    }
}

// NV pieces a thread; NV = 0: rows of any length, read twice (the second time from the
// caches).
template <typename S, int NV, int TPR>
__global__ __launch_bounds__(TPR < 256 ? 256 : TPR) void quant_q8_kernel(QuantQ8Params p) {
    constexpr int VEC = 16 / sizeof(S);
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    constexpr int KEPT = NV ? NV : 1;
    __shared__ double lds[2 * (TPR / 64)];
    const int lane = threadIdx.x % TPR;
    const int pieces = NV ? NV : (p.cols + VEC * TPR - 1) / (VEC * TPR);
    for (int64_t row = (int64_t)blockIdx.x * RPB + threadIdx.x / TPR; row < p.rows; row += (int64_t)gridDim.x * RPB) {
        float s[KEPT][VEC];
        float top = 0.f, check = 0.f;
        auto load = [&](int i) {
            const int c = (i * TPR + lane) * VEC, left = p.cols - c;
            float(&f)[VEC] = s[NV ? i : 0];
#pragma unroll
            for (int e = 0; e < VEC; ++e) f[e] = 0.f;
            if (left > 0) load_some<S, VEC>((const S*)p.x + row * p.ld_x + c, left, f);
        };
        auto look = [&](int i) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                top = fmaxf(top, fabsf(s[NV ? i : 0][e]));
                check = fmaf(s[NV ? i : 0][e], 0.f, check);
            }
        };
        if (NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) load(i);
#pragma unroll
            for (int i = 0; i < NV; ++i) look(i);
        } else {
            for (int i = 0; i < pieces; ++i) {
                load(i);
                look(i);
            }
        }
        double most = top, bad = check;
        row_reduce<TPR>(bad, most, lds);
        const float scale = row_scale(most + bad);
        const double inv = scale > 0.f ? 1.0 / (double)scale : 0.0;
        if (lane == 0) p.scale[row] = scale;
        auto store = [&](int i) {
            const int c = (i * TPR + lane) * VEC, left = p.cols - c;
            if (left <= 0) return;
            double y[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = s[NV ? i : 0][e];
            store_q<VEC>(p.q + row * p.ld_q + c, left, y, scale, inv);
        };
        if (NV) {
#pragma unroll
            for (int i = 0; i < NV; ++i) store(i);
        } else {
            for (int i = 0; i < pieces; ++i) {
                load(i);
                store(i);
            }
        }
    }
}

// Blocks walk over rows where a launch would hold too many.
template <int TPR>
int row_blocks(int rows) {
    constexpr int RPB = TPR < 256 ? 256 / TPR : 1;
    const int64_t n = ((int64_t)rows + RPB - 1) / RPB;
    return (int)(n < (1 << 20) ? n : (1 << 20));
}

template <typename T, typename S, int NV, int TPR>
void norm_nv(const NormQ8Params& p, hipStream_t s) {
    PB_LAUNCH((norm_q8_kernel<T, S, NV, TPR>), row_blocks<TPR>(p.rows), TPR < 256 ? 256 : TPR, 0, s, p);
}

template <typename S, int NV, int TPR>
void quant_nv(const QuantQ8Params& p, hipStream_t s) {
    PB_LAUNCH((quant_q8_kernel<S, NV, TPR>), row_blocks<TPR>(p.rows), TPR < 256 ? 256 : TPR, 0, s, p);
}

template <typename T, typename S>
void norm_type(const NormQ8Params& p, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    const int n = (p.d + VEC - 1) / VEC;  // pieces
    if (n <= 64) norm_nv<T, S, 1, 64>(p, s);
    else if (n <= 128) norm_nv<T, S, 2, 64>(p, s);
    else if (n <= 256) norm_nv<T, S, 1, 256>(p, s);
    else if (n <= 512) norm_nv<T, S, 2, 256>(p, s);
    else if (n <= 1024) norm_nv<T, S, 4, 256>(p, s);
    else if (n <= 1536) norm_nv<T, S, 6, 256>(p, s);
    else if (n <= 2048) norm_nv<T, S, 8, 256>(p, s);
    else if constexpr (VEC == 4) {
        if (n <= 2560) norm_nv<T, S, 10, 256>(p, s);
        else if (n <= 3328) norm_nv<T, S, 13, 256>(p, s);
        else norm_nv<T, S, 16, 256>(p, s);
    }
}

template <typename S>
void quant_type(const QuantQ8Params& p, hipStream_t s) {
    constexpr int VEC = 16 / sizeof(S);
    const int n = (int)(((int64_t)p.cols + VEC - 1) / VEC);
    if (n <= 64) quant_nv<S, 1, 64>(p, s);
    else if (n <= 128) quant_nv<S, 2, 64>(p, s);
    else if (n <= 256) quant_nv<S, 1, 256>(p, s);
    else if (n <= 512) quant_nv<S, 2, 256>(p, s);
    else if (n <= 1024) quant_nv<S, 4, 256>(p, s);
    else if (n <= 2048) quant_nv<S, 8, 256>(p, s);
    else if (n <= 3 * 1024) quant_nv<S, 3, 1024>(p, s);
    else if (n <= 5120) quant_nv<S, 5, 1024>(p, s);
    else if (n <= 8192) quant_nv<S, 8, 1024>(p, s);
    else quant_nv<S, 0, 1024>(p, s);
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
