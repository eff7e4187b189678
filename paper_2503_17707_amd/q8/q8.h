// Launch wrappers of the 8-bit linear layers' kernels (rows_q8.hip, gemm_q8.hip;
// entry points in q8_ops.cpp).
#pragma once

#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace pb {

// Rows of a stream (fp32 or the 16-bit storage type), normalized and quantized.
struct NormQ8Params {
    const void* x; int64_t ld_x;
    const void* delta; int64_t ld_delta;  // NULL: nothing is added
    void* sum; int64_t ld_sum;            // x + delta, of x's type; NULL: not kept
    const void *g, *b;                    // b may be NULL
    void* out; int64_t ld_out;            // the norm in the storage type; NULL: not wanted
    int8_t* q; int64_t ld_q;              // NULL: not wanted (scale then too)
    float* scale;
    int rows, d;
    double width, inv_d;  // d, 1 / d
    float eps;
    bool layer;
};
constexpr int NORM_Q8_MAX = 16384;
hipError_t launch_norm_q8(int dtype, bool f32, const NormQ8Params& p, hipStream_t s);

struct QuantQ8Params {
    const void* x; int64_t ld_x;
    int8_t* q; int64_t ld_q;
    float* scale;
    int rows, cols;
};
hipError_t launch_quant_q8(int dtype, bool f32, const QuantQ8Params& p, hipStream_t s);

enum { Q8_QKV = 0, Q8_RELU = 1, Q8_RESID = 2, Q8_LOGITS = 3 };

struct GemmQ8Params {
    const int8_t* X; int64_t ldx;
    const float* sx;
    const int8_t* W; int64_t ldw;
    const float* sw;
    const void* bias;             // NULL: none
    void* out; int64_t ldo;       // C (storage type) or R (fp32)
    int M, N, K;
    float qscale;
    int qcols;
    int epi;
    bool bf16;
    int32_t* ws; size_t ws_bytes;
};
// Integer products of K terms stay inside 32 bits: 128 * 128 * K < 2^31.
constexpr int GEMM_Q8_MAX_K = 131056;
size_t gemm_q8_workspace(int M, int N, int K);
bool gemm_q8_fits(int M, int N);  // a launch holds its blocks
hipError_t launch_gemm_q8(const GemmQ8Params& p, hipStream_t s);

}  // namespace pb
