// Attention of one new token per sequence over a paged cache.
#include "common.h"
#include "paged.h"

namespace pb {

namespace {

constexpr float LOG2E = 1.4426950408889634f;

// One block per (head, sequence), its waves taking 64-key chunks in turn with a
// running max and sum (fp32), joined at the end.
template <typename T, int HD, int NW>
__global__ __launch_bounds__(64 * NW) void paged_attention_kernel(PagedAttentionParams p) {
    constexpr int G = HD / 8;     // lanes per key row
    constexpr int KPI = 64 / G;   // keys per load instruction
    constexpr int NI = 64 / KPI;  // load instructions per 64-key chunk
    __shared__ float wm[NW], wl[NW], wo[NW][HD];
    __shared__ int bad;
    const int h = blockIdx.x, s = blockIdx.y;
    const int kvh = h / (p.n_heads / p.pool.n_kv_heads);
    const int len = max(p.lens[s], 0);
    const int lo = p.window > 0 ? max(0, len - p.window) : 0;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int sub = lane % G, grp = lane / G;
    const int32_t* ids = p.tab.ids + s * p.tab.ld;
    uint16_t* orow = p.out + s * p.ld_out + h * HD;
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    const int c0 = (int)p.pool.div.quot(lo), c1 = len ? (int)p.pool.div.quot(len - 1) + 1 : 0;
    for (int c = c0 + threadIdx.x; c < c1; c += 64 * NW)
        if (c >= p.tab.width || ids[c] < 0 || ids[c] >= p.pool.n_pages) bad = 1;
    __syncthreads();
    if (bad || len == 0) {
        for (int j = threadIdx.x; j < HD; j += 64 * NW) ((T*)orow)[j] = (T)(bad ? NAN : 0.f);
        return;
    }
    float q[8];
    {
        const u32x4 raw = *(const u32x4*)(p.q + s * p.ld_q + h * HD + sub * 8);
        T e[8];
        __builtin_memcpy(e, &raw, 16);
        for (int j = 0; j < 8; ++j) q[j] = (float)e[j] * p.scale;
    }
    const uint16_t* base = p.pool.base + kvh * p.pool.head_stride + sub * 8;
    float m_run = -INFINITY, l = 0.f, o[8];
    for (int j = 0; j < 8; ++j) o[j] = 0.f;
    for (int k0 = lo + wave * 64; k0 < len; k0 += NW * 64) {
        u32x4 kr[NI], vr[NI];
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const int key = min(k0 + i * KPI + grp, len - 1);
            const int col = p.pool.div.quot(key);
            const uint16_t* a = base + ids[col] * p.pool.page_stride + (key - col * p.pool.page_size) * p.pool.token_stride;
            kr[i] = *(const u32x4*)a;
            vr[i] = *(const u32x4*)(a + p.pool.v_offset);
        }
        float sc[NI], mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            T e[8];
            __builtin_memcpy(e, &kr[i], 16);
            float a = 0.f;
            for (int j = 0; j < 8; ++j) a += q[j] * (float)e[j];
            for (int sh = 1; sh < G; sh <<= 1) a += __shfl_xor(a, sh, 64);
            sc[i] = k0 + i * KPI + grp < len ? a : -INFINITY;
            mx = fmaxf(mx, sc[i]);
        }
        const float m_new = fmaxf(m_run, wave_max(mx));
        const float alpha = __builtin_amdgcn_exp2f((m_run - m_new) * LOG2E);
        l *= alpha;
        for (int j = 0; j < 8; ++j) o[j] *= alpha;
#pragma unroll
        for (int i = 0; i < NI; ++i) {
            const float e = k0 + i * KPI + grp < len ? __builtin_amdgcn_exp2f((sc[i] - m_new) * LOG2E) : 0.f;
            l += e;
            T x[8];
            // past the end the last token was read: its value may be infinite
            if (k0 + i * KPI + grp >= len) vr[i] = u32x4{0, 0, 0, 0};
            __builtin_memcpy(x, &vr[i], 16);
            for (int j = 0; j < 8; ++j) o[j] += e * (float)x[j];
        }
        m_run = m_new;
    }
    for (int sh = G; sh < 64; sh <<= 1) {
        l += __shfl_xor(l, sh, 64);
        for (int j = 0; j < 8; ++j) o[j] += __shfl_xor(o[j], sh, 64);
    }
    if (lane == 0) {
        wm[wave] = m_run;
        wl[wave] = l;
    }
    if (grp == 0)
        for (int j = 0; j < 8; ++j) wo[wave][sub * 8 + j] = o[j];
    __syncthreads();
    if (threadIdx.x < HD) {
        float M = -INFINITY, acc = 0.f, L = 0.f;
        for (int w = 0; w < NW; ++w) M = fmaxf(M, wm[w]);
        for (int w = 0; w < NW; ++w) {
            if (lo + w * 64 >= len) continue;  // a wave with no key
            const float f = __builtin_amdgcn_exp2f((wm[w] - M) * LOG2E);
            acc += f * wo[w][threadIdx.x];
            L += f * wl[w];
        }
        ((T*)orow)[threadIdx.x] = (T)(acc / L);
    }
}

}  // namespace

size_t paged_attention_workspace(int, int, int, int, int, int) { return 0; }

hipError_t launch_paged_attention(int dtype, const PagedAttentionParams& p, hipStream_t s) {
    const dim3 grid(p.n_heads, p.tab.rows);
    if (p.tab.rows <= 0) return hipSuccess;
    if (p.pool.head_dim == 64) {
        if (dtype == 1) PB_LAUNCH((paged_attention_kernel<_Float16, 64, 8>), grid, dim3(512), 0, s, p);
        else PB_LAUNCH((paged_attention_kernel<__bf16, 64, 8>), grid, dim3(512), 0, s, p);
    } else {
        if (dtype == 1) PB_LAUNCH((paged_attention_kernel<_Float16, 128, 8>), grid, dim3(512), 0, s, p);
        else PB_LAUNCH((paged_attention_kernel<__bf16, 128, 8>), grid, dim3(512), 0, s, p);
    }
    return hipGetLastError();
}

}  // namespace pb
