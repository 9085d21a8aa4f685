// Attention of a block of drafted nodes over a paged cache and the block itself: plain first form, a warp per
// (node, query head) that walks the keys one by one with a running maximum and sum.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <algorithm>

#include "cache.cuh"

namespace ngs {

template <int D, bool QUANT>
__global__ void __launch_bounds__(128) tree_attention_plain_kernel(TreeAttnArgs a) {
    constexpr int E = D / 32;
    const int lane = threadIdx.x & 31;
    const long long row = (long long)blockIdx.x * 4 + (threadIdx.x >> 5);  // (s, node, query head)
    grid_dependency_wait();
    grid_launch_dependents();
    if (row >= (long long)a.S * a.N * a.Hq) return;
    const CacheArgs& c = a.cache;
    const int hq = (int)(row % a.Hq), h = hq / (a.Hq / c.heads);
    const long long sn = row / a.Hq;
    const int s = (int)(sn / a.N), node = (int)(sn - (long long)s * a.N);
    const int live = a.n_nodes ? min(a.n_nodes[s], a.N) : a.N;
    int len = a.len[s];
    if (len < 0 || len > (c.max_pages << c.page_shift)) {
        if (lane == 0) atomicOr(a.status, SPEC_STATUS_CAPACITY);
        len = -1;
    }
    float q[E], o[E], m = -INFINITY, l = 0.0f;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        q[j] = __bfloat162float(((const __nv_bfloat16*)a.q)[sn * a.q_tok + hq * a.q_head + lane * E + j]);
        o[j] = 0.0f;
    }
    auto key = [&](const float (&k)[E], const float (&v)[E]) {
        float t = 0.0f;
#pragma unroll
        for (int j = 0; j < E; ++j) t += q[j] * k[j];
#pragma unroll
        for (int x = 16; x > 0; x >>= 1) t += __shfl_xor_sync(0xffffffffu, t, x);
        t *= a.scale;
        const float mn = fmaxf(m, t), f = m == -INFINITY ? 0.0f : expf(m - mn), p = expf(t - mn);
        l = l * f + p;
#pragma unroll
        for (int j = 0; j < E; ++j) o[j] = o[j] * f + p * v[j];
        m = mn;
    };
    if (node < live && len >= 0) {
        for (int pos = 0; pos < len; ++pos) {
            const int page = c.table[(long long)s * c.max_pages + (pos >> c.page_shift)];
            if ((unsigned)page >= (unsigned)c.n_pages) {
                if (lane == 0) atomicOr(a.status, SPEC_STATUS_CAPACITY);
                continue;
            }
            const long long at = (((long long)page * c.heads + h) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
            float k[E], v[E];
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const long long i = at * D + lane * E + j;
                if (QUANT) {
                    uint32_t x;
                    asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(x) : "h"((uint16_t)(((const uint8_t*)c.k)[i] | (((const uint8_t*)c.v)[i] << 8))));
                    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&x));
                    k[j] = f.x * (c.k_exp[at] == 255 ? NAN : ldexpf(1.0f, c.k_exp[at] - 127));
                    v[j] = f.y * (c.v_exp[at] == 255 ? NAN : ldexpf(1.0f, c.v_exp[at] - 127));
                } else {
                    k[j] = __bfloat162float(((const __nv_bfloat16*)c.k)[i]);
                    v[j] = __bfloat162float(((const __nv_bfloat16*)c.v)[i]);
                }
            }
            key(k, v);
        }
        const int words = (a.N + 31) / 32;
        for (int j = 0; j < live; ++j) {
            if (!((a.mask[sn * words + (j >> 5)] >> (j & 31)) & 1)) continue;
            const long long b = (long long)s * a.N + j;
            float k[E], v[E];
#pragma unroll
            for (int i = 0; i < E; ++i) {
                k[i] = __bfloat162float(((const __nv_bfloat16*)a.k)[b * a.k_tok + h * a.k_head + lane * E + i]);
                v[i] = __bfloat162float(((const __nv_bfloat16*)a.v)[b * a.v_tok + h * a.v_head + lane * E + i]);
            }
            key(k, v);
        }
    }
#pragma unroll
    for (int j = 0; j < E; ++j) ((__nv_bfloat16*)a.out)[row * D + lane * E + j] = __float2bfloat16_rn(l == 0.0f ? 0.0f : o[j] / l);
    if (a.lse && lane == 0) a.lse[row] = m + logf(l);
}

size_t tree_attention_bytes(int num_sms, int S, int N, int Hq, int heads, int head_dim) { return 16; }

int launch_tree_attention(spec_ctx* ctx, const TreeAttnArgs& a, cudaStream_t st) {
    const long long rows = (long long)a.S * a.N * a.Hq;
    const dim3 grid((unsigned)((rows + 3) / 4));
    auto go = [&](auto kernel) { return launch_pdl(kernel, grid, dim3(128), 0, st, a); };
    cudaError_t e;
    if (a.cache.quantised) e = a.cache.head_dim == 64 ? go(tree_attention_plain_kernel<64, true>) : go(tree_attention_plain_kernel<128, true>);
    else e = a.cache.head_dim == 64 ? go(tree_attention_plain_kernel<64, false>) : go(tree_attention_plain_kernel<128, false>);
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_tree_attention launch");
}

}  // namespace ngs
