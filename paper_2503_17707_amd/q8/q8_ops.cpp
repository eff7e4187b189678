// Entry points of the 8-bit linear layers (include/pipeboost_ops.h): argument checks,
// then the launch.
#include "../../include/pipeboost_ops.h"
#include "../op_checks.h"
#include "q8.h"

using pb::aligned;
using pb::launched;
using pb::overlap;
using pb::refuse;

namespace {

// Rows of `cols` elements of `size` bytes at stride ld: non-NULL, on whole elements,
// not over one another, their extent inside 64 bits.  (The stride of a single row is not used.)
bool rows_ok(const void* p, int64_t ld, int64_t rows, int64_t cols, int size) {
    return p && aligned(p, (uintptr_t)size) && (rows <= 1 || (ld >= cols && ld < ((int64_t)1 << 40) && ld <= ((int64_t)1 << 56) / rows));
}

size_t span(int64_t ld, int64_t rows, int64_t cols, int size) {
    return (size_t)((rows > 1 ? (rows - 1) * ld : 0) + cols) * (size_t)size;
}

struct Operand {
    const void* p;
    size_t n;
};

// An output over an input or over another output.
bool any_overlap(const Operand* in, int n_in, const Operand* out, int n_out) {
    for (int o = 0; o < n_out; ++o) {
        for (int i = 0; i < n_in; ++i)
            if (overlap(in[i].p, in[i].n, out[o].p, out[o].n)) return true;
        for (int i = 0; i < o; ++i)
            if (overlap(out[i].p, out[i].n, out[o].p, out[o].n)) return true;
    }
    return false;
}

}  // namespace

extern "C" int pb_op_norm_q8(int32_t dtype, int32_t layer, const void* x, int64_t ld_x, int32_t x_f32, const void* delta,
                             int64_t ld_delta, void* sum, int64_t ld_sum, const void* g, const void* b, float eps,
                             void* out, int64_t ld_out, int8_t* q, int64_t ld_q, float* scale, int32_t rows, int32_t d,
                             void* stream) {
    const char* op = "pb_op_norm_q8";
    if (dtype != PB_BF16 && dtype != PB_F16) return refuse("%s: bad dtype %d", op, dtype);
    if (rows < 0 || rows > (1 << 30) || d < 1 || d > pb::NORM_Q8_MAX)
        return refuse("%s: %d rows (up to 2^30) of %d (1..%d)", op, rows, d, pb::NORM_Q8_MAX);
    if (!(eps >= 0.f) || !(eps - eps == 0.f)) return refuse("%s: eps=%g", op, (double)eps);
    if (rows == 0) return PB_OK;
    const int xs = x_f32 ? 4 : 2;
    if (!rows_ok(x, ld_x, rows, d, xs)) return refuse("%s: x NULL, unaligned or with rows of %lld < d", op, (long long)ld_x);
    if (!g || !aligned(g, 2) || !aligned(b, 2)) return refuse("%s: g NULL, or g or b unaligned", op);
    if (sum && !delta) return refuse("%s: a sum without anything to add", op);
    if ((delta && !rows_ok(delta, ld_delta, rows, d, 2)) || (sum && !rows_ok(sum, ld_sum, rows, d, xs)) ||
        (out && !rows_ok(out, ld_out, rows, d, 2)) || (q && !rows_ok(q, ld_q, rows, d, 1)))
        return refuse("%s: rows unaligned or shorter than d (strides %lld, %lld, %lld, %lld)", op, (long long)ld_delta,
                      (long long)ld_sum, (long long)ld_out, (long long)ld_q);
    if (!out && !q) return refuse("%s: neither out nor q", op);
    if ((q != nullptr) != (scale != nullptr) || !aligned(scale, 4)) return refuse("%s: q and scale go together, scale 4-byte aligned", op);
    const bool in_place = sum == x && (rows == 1 || ld_sum == ld_x);
    const Operand in[] = {{in_place ? nullptr : x, span(ld_x, rows, d, xs)}, {delta, span(ld_delta, rows, d, 2)},
                          {g, (size_t)d * 2}, {b, (size_t)d * 2}},
                  outs[] = {{sum, span(ld_sum, rows, d, xs)}, {out, span(ld_out, rows, d, 2)},
                            {q, span(ld_q, rows, d, 1)}, {scale, (size_t)rows * 4}};
    if (any_overlap(in, 4, outs, 4)) return refuse("%s: an output overlaps an input or another output", op);
    pb::NormQ8Params p{};
    p.x = x; p.ld_x = ld_x; p.delta = delta; p.ld_delta = ld_delta; p.sum = sum; p.ld_sum = ld_sum;
    p.g = g; p.b = b; p.out = out; p.ld_out = ld_out; p.q = q; p.ld_q = ld_q; p.scale = scale;
    p.rows = rows; p.d = d; p.width = d; p.inv_d = 1.0 / d; p.eps = eps; p.layer = layer != 0;
    return launched(op, pb::launch_norm_q8(dtype, x_f32 != 0, p, (hipStream_t)stream));
}

extern "C" int pb_op_quant_q8(int32_t dtype, const void* x, int64_t ld_x, int32_t x_f32, int8_t* q, int64_t ld_q,
                              float* scale, int32_t rows, int32_t cols, void* stream) {
    const char* op = "pb_op_quant_q8";
    if (dtype != PB_BF16 && dtype != PB_F16) return refuse("%s: bad dtype %d", op, dtype);
    if (rows < 0 || rows > (1 << 30) || cols < 1 || cols > (1 << 24)) return refuse("%s: %d rows (up to 2^30) of %d (1..2^24)", op, rows, cols);
    if (rows == 0) return PB_OK;
    const int xs = x_f32 ? 4 : 2;
    if (!rows_ok(x, ld_x, rows, cols, xs) || !rows_ok(q, ld_q, rows, cols, 1))
        return refuse("%s: x or q NULL, unaligned or with rows (%lld, %lld) shorter than %d", op, (long long)ld_x,
                      (long long)ld_q, cols);
    if (!scale || !aligned(scale, 4)) return refuse("%s: scale NULL or unaligned", op);
    const Operand in[] = {{x, span(ld_x, rows, cols, xs)}},
                  outs[] = {{q, span(ld_q, rows, cols, 1)}, {scale, (size_t)rows * 4}};
    if (any_overlap(in, 1, outs, 2)) return refuse("%s: an output overlaps an input or another output", op);
    pb::QuantQ8Params p{};
    p.x = x; p.ld_x = ld_x; p.q = q; p.ld_q = ld_q; p.scale = scale; p.rows = rows; p.cols = cols;
    return launched(op, pb::launch_quant_q8(dtype, x_f32 != 0, p, (hipStream_t)stream));
}

extern "C" size_t pb_op_gemm_q8_workspace(int32_t M, int32_t N, int32_t K) {
    if (M < 1 || N < 1 || K < 16 || K > pb::GEMM_Q8_MAX_K || K % 16 || !pb::gemm_q8_fits(M, N)) return 0;
    return pb::gemm_q8_workspace(M, N, K);
}

extern "C" int pb_op_gemm_q8(int32_t dtype, int32_t epi, const int8_t* X, int64_t ldx, const float* sx, const int8_t* W,
                             int64_t ldw, const float* sw, const void* bias, void* C, float* R, int64_t ldo, int32_t M,
                             int32_t N, int32_t K, float qscale, int32_t qcols, void* workspace, size_t workspace_bytes,
                             void* stream) {
    const char* op = "pb_op_gemm_q8";
    if (dtype != PB_BF16 && dtype != PB_F16) return refuse("%s: bad dtype %d", op, dtype);
    if (epi < pb::Q8_QKV || epi > pb::Q8_LOGITS) return refuse("%s: bad epilogue %d", op, epi);
    if (M < 0 || N < 1 || K < 16 || K % 16 || K > pb::GEMM_Q8_MAX_K)
        return refuse("%s: M=%d N=%d K=%d (K a multiple of 16 up to %d)", op, M, N, K, pb::GEMM_Q8_MAX_K);
    if (M == 0) return PB_OK;
    if (!pb::gemm_q8_fits(M, N)) return refuse("%s: M=%d N=%d: more tiles than a launch takes", op, M, N);
    const bool wide = epi >= pb::Q8_RESID;
    void* out = wide ? (void*)R : C;
    const int os = wide ? 4 : 2;
    const int64_t most = 1 << 23;  // a tile's offsets fit 32 bits
    if (!rows_ok(X, ldx, M, K, 16) || !rows_ok(W, ldw, N, K, 16) || (M > 1 && (ldx % 16 || ldx > most)) ||
        (N > 1 && (ldw % 16 || ldw > most)))
        return refuse("%s: X and W must be 16-byte aligned, row strides (%lld, %lld) multiples of 16, at least K and at most 2^23",
                      op, (long long)ldx, (long long)ldw);
    if (!rows_ok(out, ldo, M, N, os))
        return refuse("%s: %s NULL, unaligned or with rows of %lld < N", op, wide ? "R" : "C", (long long)ldo);
    if (!sx || !sw || !aligned(sx, 4) || !aligned(sw, 4) || !aligned(bias, 2)) return refuse("%s: scales NULL or unaligned, or bias unaligned", op);
    if (workspace && !aligned(workspace, 16)) return refuse("%s: workspace must be 16-byte aligned", op);
    const Operand in[] = {{X, span(ldx, M, K, 1)}, {sx, (size_t)M * 4}, {W, span(ldw, N, K, 1)}, {sw, (size_t)N * 4},
                          {bias, (size_t)N * 2}},
                  outs[] = {{out, span(ldo, M, N, os)}, {workspace, workspace_bytes}};
    if (any_overlap(in, 5, outs, 2)) return refuse("%s: the output or the workspace overlaps an operand", op);
    pb::GemmQ8Params p{};
    p.X = X; p.ldx = ldx; p.sx = sx; p.W = W; p.ldw = ldw; p.sw = sw; p.bias = bias; p.out = out; p.ldo = ldo;
    p.M = M; p.N = N; p.K = K; p.qscale = qscale; p.qcols = epi == pb::Q8_QKV ? qcols : 0; p.epi = epi;
    p.bf16 = dtype == PB_BF16;
    p.ws = (int32_t*)workspace; p.ws_bytes = workspace ? workspace_bytes : 0;
    return launched(op, pb::launch_gemm_q8(p, (hipStream_t)stream));
}
