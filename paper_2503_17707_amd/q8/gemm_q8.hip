// Products of 8-bit rows: out[M, N] from X[M, K] W[N, K]^T, exact in 32-bit integers
// (v_mfma_i32_16x16x64_i8), times the scales of token m and channel n, with the
// epilogues of the decoder's projections.
//
// As in the 16-bit products the MFMA's A operand is the weight rows (output features
// n) and its B operand the tokens m: a lane ends up with four consecutive features of
// one token.  Lane l gives 16 bytes of row l % 16, the 16 at K offset 16 (l / 16) of
// the step's 64; which of the 64 a lane holds does not matter as long as both operands
// agree, and sums of integers do not depend on their order: every variant gives the
// same bits.
#include "../csrc/common.h"
#include "q8.h"

namespace pb {

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
__device__ __forceinline__ void load4(const T* p, int left, float (&f)[4]) {
    T t[4] = {};
    if (left >= 4) {
        __builtin_memcpy(t, p, sizeof(t));
    } else {
#pragma unroll
        for (int r = 0; r < 3; ++r)
            if (r < left) t[r] = p[r];
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) f[r] = (float)t[r];
}

// Features n .. n+3 of token m: (sum rounded to fp32, times sx) times sw plus bias,
// the second product and the sum rounded once; then the epilogue.  Rows of the output
// may start at any element (N odd): vectors go there as they come.
__device__ __forceinline__ void epilogue8(const GemmQ8Params& p, int m, int n, i32x4 acc) {
    const int left = p.N - n;
    const float sx = p.sx[m];
    float sw[4], b[4] = {0.f, 0.f, 0.f, 0.f}, y[4];
    load4(p.sw + n, left, sw);
    if (p.bias) {
        if (p.bf16) load4((const __bf16*)p.bias + n, left, b);
        else load4((const _Float16*)p.bias + n, left, b);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        y[r] = fmaf((float)acc[r] * sx, sw[r], b[r]);
        if (p.epi == Q8_RELU) y[r] = y[r] < 0.f ? 0.f : y[r];  // (NaN stays)
        if (p.epi == Q8_QKV && n + r < p.qcols) y[r] *= p.qscale;
    }
    const int64_t at = (int64_t)m * p.ldo + n;
    if (p.epi >= Q8_RESID) {
        float* out = (float*)p.out + at;
        if (p.epi == Q8_RESID) {
            float old[4];
            load4(out, left, old);
#pragma unroll
            for (int r = 0; r < 4; ++r) y[r] += old[r];
        }
        store4(out, left, y);
    } else if (p.bf16) {
        store4((__bf16*)p.out + at, left, y);
    } else {
        store4((_Float16*)p.out + at, left, y);
    }
}

// 64 tokens x 64 features a block, four waves of 32 x 32, operands straight from memory.
__global__ __launch_bounds__(256) void q8_plain_kernel(GemmQ8Params p, int tiles_n) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int lr = lane & 15, lg = lane >> 4;
    const int m0 = ((int)blockIdx.x / tiles_n) * 64 + (wave & 1) * 32;
    const int n0 = ((int)blockIdx.x % tiles_n) * 64 + (wave >> 1) * 32;
    const int8_t *x[2], *w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {  // rows past the edge re-read the last one
        x[i] = p.X + (int64_t)min(m0 + 16 * i + lr, p.M - 1) * p.ldx;
        w[i] = p.W + (int64_t)min(n0 + 16 * i + lr, p.N - 1) * p.ldw;
    }
    i32x4 acc[2][2] = {};
    for (int k = 16 * lg; k - 16 * lg < p.K; k += 64) {
        const i32x4 zero = {0, 0, 0, 0};
        const bool in = k < p.K;  // K is a multiple of 16
        i32x4 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            a[i] = in ? *(const i32x4*)(w[i] + k) : zero;
            b[i] = in ? *(const i32x4*)(x[i] + k) : zero;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = mma8(a[i], b[j], acc[i][j]);
    }
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int m = m0 + 16 * j + lr, n = n0 + 16 * i + 4 * lg;
            if (m < p.M && n < p.N) epilogue8(p, m, n, acc[i][j]);
        }
}

}  // namespace

bool gemm_q8_fits(int M, int N) { return (((int64_t)M + 63) / 64) * (((int64_t)N + 63) / 64) < (1 << 23); }

size_t gemm_q8_workspace(int, int, int) { return 0; }

hipError_t launch_gemm_q8(const GemmQ8Params& p, hipStream_t s) {
    const int tm = (p.M + 63) / 64, tn = (p.N + 63) / 64;
    PB_LAUNCH(q8_plain_kernel, tm * tn, 256, 0, s, p, tn);
    return hipGetLastError();
}

}  // namespace pb
