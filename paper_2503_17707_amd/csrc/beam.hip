// Beam search's selection: of every live hypothesis's continuations, the W best
// of each prompt.
//
// log softmax(l)[v] = l[v] - m - log sum exp(l - m): a row's order is its logits'
// order, so a row offers its W largest logits and its log sum, and only those are
// compared across rows.  The sum of exponentials runs in fp32 per thread and is
// joined in 64 bits; a candidate's score, score + (l - m) - log sum, is formed and
// compared in 64 bits, because candidates of different rows can lie closer than
// fp32 tells apart at scores of tens.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// What a logit counts as: NaN is no candidate, +inf the largest float.
__device__ inline float clean(float x) { return x == x ? fminf(x, 3.402823466e38f) : -INFINITY; }

struct RowBest {
    float* val;    // [rows][W], descending; -inf: none left
    int32_t* idx;  // [rows][W]
    double* lse;   // [rows], log sum exp(l - largest)
};

__host__ __device__ inline RowBest row_best(void* ws, int rows, int W) {
    RowBest r;
    r.lse = (double*)ws;
    r.val = (float*)(r.lse + rows);
    r.idx = (int32_t*)(r.val + (size_t)rows * W);
    return r;
}

// (a, i) comes before (b, j)
__device__ inline bool before(float a, int i, float b, int j) { return a > b || (a == b && i < j); }

__global__ __launch_bounds__(1024) void beam_rows_kernel(BeamParams p) {
    __shared__ float sv[16];
    __shared__ int si[16];
    __shared__ double ss[16];
    const int row = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float* x = p.logits + row * p.ld;
    const RowBest out = row_best(p.ws, p.B * p.W, p.W);
    float last = INFINITY;
    int last_i = -1;
    float m = 0.f;
    for (int r = 0; r < p.W; ++r) {
        float bv = -INFINITY;
        int bi = 0x7fffffff;
        for (int v = tid; v < p.V; v += 1024) {
            const float a = clean(x[v]);
            if (before(last, last_i, a, v) && before(a, v, bv, bi)) bv = a, bi = v;
        }
        for (int o = 32; o > 0; o >>= 1) {
            const float ov = __shfl_xor(bv, o, 64);
            const int oi = __shfl_xor(bi, o, 64);
            if (before(ov, oi, bv, bi)) bv = ov, bi = oi;
        }
        __syncthreads();
        if (lane == 0) sv[wave] = bv, si[wave] = bi;
        __syncthreads();
        bv = sv[0], bi = si[0];
        for (int w = 1; w < 16; ++w)
            if (before(sv[w], si[w], bv, bi)) bv = sv[w], bi = si[w];
        if (r == 0) m = bv;
        if (tid == 0) {
            out.val[(size_t)row * p.W + r] = bv;
            out.idx[(size_t)row * p.W + r] = bi;
        }
        last = bv, last_i = bi;
    }
    float sum = 0.f;
    for (int v = tid; v < p.V; v += 1024) {
        const float a = clean(x[v]);
        if (a > -INFINITY) sum += __builtin_amdgcn_exp2f((a - m) * LOG2E);
    }
    double d = sum;
    for (int o = 32; o > 0; o >>= 1) d += __shfl_xor(d, o, 64);
    if (lane == 0) ss[wave] = d;
    __syncthreads();
    if (tid == 0) {
        d = 0;
        for (int w = 0; w < 16; ++w) d += ss[w];
        out.lse[row] = log(d);
    }
}

// One block per prompt: its at most W W candidates, one per thread, each placed
// by how many come before it.
__global__ __launch_bounds__(1024) void beam_join_kernel(BeamParams p) {
    __shared__ double sc[1024];
    __shared__ int id[1024];
    const int b = blockIdx.x, tid = threadIdx.x, W = p.W, n = W * W;
    const RowBest in = row_best(p.ws, p.B * W, W);
    const int w = tid / W, k = tid % W;
    double score = -INFINITY;
    int token = p.pad;
    bool grows = false;
    if (tid < n) {
        const int row = b * W + w;
        const float own = p.scores[row];
        if (own - own == 0.f) {  // finite
            if (p.alive[row] == 0) {
                if (k == 0) score = own;
            } else {
                const float v = in.val[(size_t)row * W + k];
                if (v > -INFINITY) {
                    token = in.idx[(size_t)row * W + k];
                    score = (double)own + (((double)v - (double)in.val[(size_t)row * W]) - in.lse[row]);
                    grows = token != p.eos;
                }
            }
        }
    }
    const int flat = w * p.V + token;  // W V < 2^31 (checked by the entry point)
    sc[tid] = score;
    id[tid] = flat;
    __syncthreads();
    int rank = 0;
    if (score > -INFINITY)
        for (int i = 0; i < n; ++i) rank += sc[i] > score || (sc[i] == score && id[i] < flat);
    int found = __syncthreads_count(score > -INFINITY);
    if (score > -INFINITY && rank < W) {
        const int o = b * W + rank;
        p.out_scores[o] = (float)score;
        p.out_tokens[o] = token;
        p.out_parents[o] = b * W + w;
        p.out_alive[o] = grows;
    }
    if (tid >= found && tid < W) {
        const int o = b * W + tid;
        p.out_scores[o] = -INFINITY;
        p.out_tokens[o] = p.pad;
        p.out_parents[o] = -1;
        p.out_alive[o] = 0;
    }
}

}  // namespace

size_t beam_select_workspace(int B, int W, int) { return (size_t)B * W * (8 + (size_t)W * 8); }

hipError_t launch_beam_select(const BeamParams& p, hipStream_t s) {
    if (p.B <= 0) return hipSuccess;
    PB_LAUNCH(beam_rows_kernel, dim3(p.B * p.W), dim3(1024), 0, s, p);
    PB_LAUNCH(beam_join_kernel, dim3(p.B), dim3(1024), 0, s, p);
    return hipGetLastError();
}

}  // namespace pb
