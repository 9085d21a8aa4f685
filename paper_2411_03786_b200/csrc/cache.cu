// What surrounds the attention of a verification call: rotary positions of the block's queries and keys, the paged
// key/value cache (bfloat16, or E4M3 codes with a power-of-two scale per vector) and the bit masks of draft trees.
//
// All four kernels move each byte once and compute next to nothing on it, so HBM (or, for a decode step's few
// tokens, the launch) bounds them; a thread handles 16 bytes of a head at a time.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>

#include "cache.cuh"

namespace ngs {

constexpr int CACHE_THREADS = 256;

__device__ __forceinline__ void unpack_bf16x8(const uint4& v, float (&x)[8]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        x[2 * j] = __uint_as_float(w[j] << 16);
        x[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
    }
}
__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&p);
}
__device__ __forceinline__ uint4 pack_bf16x8(const float (&x)[8]) {
    return make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
}

// cos and sin of pos * freq, times the factor.  The angle is taken in turns and reduced in 64 bits: in 32 bits a
// position of 131072 would leave an error of 4e-3 radian, as much as half a step of a bf16 result.
__device__ __forceinline__ float2 rope_cos_sin(int pos, float freq, float factor) {
    const double turns = (double)pos * ((double)freq * 0.15915494309189535);  // 1 / (2 pi)
    const float r = (float)(turns - rint(turns));
    float sn, cs;
    sincospif(2.0f * r, &sn, &cs);
    return make_float2(cs * factor, sn * factor);
}

// Rotates the chunk of 8 elements that starts at element e of a head.  `table` holds (cos, sin) of the pairs; `other`
// is the chunk that the pairs of a half layout have their other elements in.
__device__ __forceinline__ void rope_chunk(float (&x)[8], const float (&other)[8], const float2* table, int e, int half, bool interleaved) {
    if (interleaved) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 cs = table[e / 2 + j];
            const float a = x[2 * j], b = x[2 * j + 1];
            x[2 * j] = a * cs.x - b * cs.y;
            x[2 * j + 1] = a * cs.y + b * cs.x;
        }
    } else {
        const bool first = e < half;
        const int p = first ? e : e - half;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 cs = table[p + j];
            x[j] = first ? x[j] * cs.x - other[j] * cs.y : other[j] * cs.y + x[j] * cs.x;
        }
    }
}

// ------------------------------------------------------------------------------------------ rotary positions
struct RopeRows {
    const __nv_bfloat16* x;
    __nv_bfloat16* y;
    long long tok, head;  // strides of x in elements; y is [T, heads, D]
    int heads;
};
// One CTA per token (and slice of its heads): the (cos, sin) table of the token is made once and serves all heads of
// q and k.  A thread owns both chunks that a pair lies in, so that y may be x.
__global__ void __launch_bounds__(CACHE_THREADS) rope_rows_kernel(RopeRows q, RopeRows k, int D, RopeArgs rope, const int32_t* __restrict__ pos) {
    extern __shared__ float2 table[];
    grid_dependency_wait();
    grid_launch_dependents();
    const long long t = blockIdx.x;
    const int half = rope.rot / 2;
    const int p = pos[t];
    for (int i = threadIdx.x; i < half; i += blockDim.x) table[i] = rope_cos_sin(p, rope.freq[i], rope.factor);
    __syncthreads();
    const int per_head = D / 16;  // a work item is 16 elements: two chunks that pair up, or two neighbours
    const int rot_items = rope.rot / 16;
    const int items = (q.heads + k.heads) * per_head;
    for (int it = blockIdx.y * blockDim.x + threadIdx.x; it < items; it += gridDim.y * blockDim.x) {
        const int h = it / per_head, i = it - h * per_head;
        const bool is_q = h < q.heads;
        const RopeRows& r = is_q ? q : k;
        const int hh = is_q ? h : h - q.heads;
        const bool rotated = i < rot_items;
        const bool split = rotated && !rope.interleaved;
        const int e0 = split ? i * 8 : i * 16, e1 = split ? e0 + half : e0 + 8;
        const __nv_bfloat16* x = r.x + t * r.tok + hh * r.head;
        __nv_bfloat16* y = r.y + (t * r.heads + hh) * D;
        uint4 a = *reinterpret_cast<const uint4*>(x + e0), b = *reinterpret_cast<const uint4*>(x + e1);
        if (rotated) {
            float fa[8], fb[8], ga[8];
            unpack_bf16x8(a, fa);
            unpack_bf16x8(b, fb);
#pragma unroll
            for (int j = 0; j < 8; ++j) ga[j] = fa[j];
            rope_chunk(fa, fb, table, e0, half, rope.interleaved);
            rope_chunk(fb, ga, table, e1, half, rope.interleaved);
            a = pack_bf16x8(fa);
            b = pack_bf16x8(fb);
        }
        *reinterpret_cast<uint4*>(y + e0) = a;
        *reinterpret_cast<uint4*>(y + e1) = b;
    }
}

int launch_rope_rows(spec_ctx* ctx, const RopeArgs& rope, const void* d_q, int Hq, long long q_tok, long long q_head, void* d_q_out,
                     const void* d_k, int Hkv, long long k_tok, long long k_head, void* d_k_out, int D, const int32_t* d_pos, int T,
                     cudaStream_t st) {
    const RopeRows q{(const __nv_bfloat16*)d_q, (__nv_bfloat16*)d_q_out, q_tok, q_head, Hq};
    const RopeRows k{(const __nv_bfloat16*)d_k, (__nv_bfloat16*)d_k_out, k_tok, k_head, Hkv};
    const int items = (Hq + Hkv) * (D / 16);
    const int threads = std::min(CACHE_THREADS, (items + 31) / 32 * 32);
    const int slices = std::max(1, std::min((items + threads - 1) / threads, ctx->num_sms * 4 / T));
    cudaError_t e = launch_pdl(rope_rows_kernel, dim3(T, slices), dim3(threads), sizeof(float2) * (rope.rot / 2), st, q, k, D, rope, d_pos);
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_rope_rows launch");
}

// ------------------------------------------------------------------------------------------ cache
// Where position `pos` of sequence s lies: index of its vector of head 0 counted in vectors of D elements, or -1.
__device__ __forceinline__ long long cache_slot(const CacheArgs& c, int s, int pos, int* status) {
    if (pos < 0 || (pos >> c.page_shift) >= c.max_pages) {
        atomicOr(status, SPEC_STATUS_CAPACITY);
        return -1;
    }
    const int page = c.table[(long long)s * c.max_pages + (pos >> c.page_shift)];
    if ((unsigned)page >= (unsigned)c.n_pages) {
        atomicOr(status, SPEC_STATUS_CAPACITY);
        return -1;
    }
    return (((long long)page * c.heads) << c.page_shift) + (pos & ((1 << c.page_shift) - 1));
}

// Quantises a vector that LANES neighbouring lanes hold 8 elements each of.  The scale is the smallest power of two
// that brings the largest magnitude to at most 448: E4M3 keeps three mantissa bits at every exponent, so a power of
// two loses nothing against a finer scale, dividing by it rounds nothing, and a reader gets code * scale exactly in
// bfloat16.  Its exponent stays in [-120, 7]: magnitudes above 448 * 2^7 (infinities too) are held as that.  A vector
// with a NaN is held as the scale byte 255 and reads as NaN throughout.
template <int LANES>
__device__ __forceinline__ uint2 quantise_vector(const float (&x)[8], uint8_t& scale) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
    int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);  // 448 = 1.75 * 2^8
    e = top == 0u ? 0 : min(max(e, E8_MIN), E8_MAX);
    const bool nan = top > 0x7F800000u;
    scale = nan ? 255 : (uint8_t)(e + 127);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint16_t r;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(x[2 * j + 1] * inv), "f"(x[2 * j] * inv));
        w[j] = nan ? 0x7F7Fu : r;
    }
    return make_uint2(w[0] | (w[1] << 16), w[2] | (w[3] << 16));
}

// A CTA writes TOK tokens of one sequence, all heads of K and V: the rotation table is made once per token.
constexpr int WRITE_TOK = 8;
template <int D, bool QUANT>
__global__ void __launch_bounds__(CACHE_THREADS) cache_write_kernel(CacheArgs c, const __nv_bfloat16* __restrict__ k, long long k_tok,
                                                                    long long k_head, const __nv_bfloat16* __restrict__ v, long long v_tok,
                                                                    long long v_head, int N, int n, const int32_t* __restrict__ nodes,
                                                                    const int32_t* __restrict__ start, const int32_t* __restrict__ count,
                                                                    RopeArgs rope, int* status) {
    constexpr int LANES = D / 8;
    extern __shared__ float2 table[];  // [WRITE_TOK, rot / 2]
    __shared__ long long src[WRITE_TOK], dst[WRITE_TOK];
    grid_dependency_wait();
    grid_launch_dependents();
    const int s = blockIdx.y, i0 = blockIdx.x * WRITE_TOK;
    const int n_here = min(count ? min(count[s], n) : n, i0 + WRITE_TOK) - i0;
    if (n_here <= 0) return;
    const int pos0 = start[s] + i0;
    if (threadIdx.x < n_here) {
        const int i = i0 + threadIdx.x;
        const int node = nodes ? nodes[(long long)s * n + i] : i;
        const bool ok = node >= 0 && node < N;
        src[threadIdx.x] = (long long)s * N + node;
        dst[threadIdx.x] = ok ? cache_slot(c, s, pos0 + (int)threadIdx.x, status) : -1;
    }
    const int half = rope.rot / 2;
    for (int i = threadIdx.x; i < n_here * half; i += CACHE_THREADS)
        table[i] = rope_cos_sin(pos0 + i / half, rope.freq[i % half], rope.factor);
    __syncthreads();
    const int vectors = n_here * c.heads, lane = threadIdx.x % LANES;
    // (the loop count is the same for all threads of a warp, whose lanes exchange maxima)
    for (int base = 0; base < vectors; base += CACHE_THREADS / LANES) {
        const int w = base + threadIdx.x / LANES;
        const bool on = w < vectors && dst[min(w, vectors - 1) / c.heads] >= 0;
        const int t = min(w, vectors - 1) / c.heads, h = min(w, vectors - 1) - t * c.heads;
        uint4 kv = make_uint4(0, 0, 0, 0), vv = kv;
        const __nv_bfloat16* kp = k + src[t] * k_tok + h * k_head;
        if (on) {
            kv = *reinterpret_cast<const uint4*>(kp + lane * 8);
            vv = *reinterpret_cast<const uint4*>(v + src[t] * v_tok + h * v_head + lane * 8);
        }
        const int e = lane * 8;
        float x[8];
        if (on && e < rope.rot) {
            float other[8];
            unpack_bf16x8(kv, x);
            if (!rope.interleaved) {
                const uint4 o = *reinterpret_cast<const uint4*>(kp + (e < half ? e + half : e - half));
                unpack_bf16x8(o, other);
            }
            rope_chunk(x, other, table + t * half, e, half, rope.interleaved);
            kv = pack_bf16x8(x);  // a key is bfloat16 before it is quantised, as it is for the block's own attention
        }
        const long long at = on ? dst[t] + ((long long)h << c.page_shift) : 0;
        if (QUANT) {
            uint8_t ks, vs;
            unpack_bf16x8(kv, x);
            const uint2 kq = quantise_vector<LANES>(x, ks);
            unpack_bf16x8(vv, x);
            const uint2 vq = quantise_vector<LANES>(x, vs);
            if (on) {
                *reinterpret_cast<uint2*>((uint8_t*)c.k + at * D + e) = kq;
                *reinterpret_cast<uint2*>((uint8_t*)c.v + at * D + e) = vq;
                if (lane == 0) {
                    c.k_exp[at] = ks;
                    c.v_exp[at] = vs;
                }
            }
        } else if (on) {
            *reinterpret_cast<uint4*>((__nv_bfloat16*)c.k + at * D + e) = kv;
            *reinterpret_cast<uint4*>((__nv_bfloat16*)c.v + at * D + e) = vv;
        }
    }
}

// 8 E4M3 codes times a power of two, as bfloat16 (exact).
__device__ __forceinline__ uint4 dequantise8(uint2 codes, uint8_t scale) {
    const float f = scale == 255 ? __uint_as_float(0x7FC00000u) : ldexpf(1.0f, (int)scale - 127);
    const uint32_t w[4] = {codes.x & 0xFFFFu, codes.x >> 16, codes.y & 0xFFFFu, codes.y >> 16};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t h2;
        asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((uint16_t)w[j]));
        const float2 x = __half22float2(*reinterpret_cast<const __half2*>(&h2));
        r[j] = pack_bf16x2(x.x * f, x.y * f);
    }
    return make_uint4(r[0], r[1], r[2], r[3]);
}

template <int D, bool QUANT>
__global__ void __launch_bounds__(CACHE_THREADS) cache_read_kernel(CacheArgs c, int n, const int32_t* __restrict__ start,
                                                                   const int32_t* __restrict__ count, __nv_bfloat16* __restrict__ k_out,
                                                                   __nv_bfloat16* __restrict__ v_out, int* status) {
    constexpr int LANES = D / 8;
    grid_dependency_wait();
    grid_launch_dependents();
    const int s = blockIdx.y;
    const int n_here = count ? min(count[s], n) : n;
    const int pos0 = start[s];
    const long long vectors = (long long)n * c.heads;
    const int lane = threadIdx.x % LANES;
    for (long long w = (long long)blockIdx.x * (CACHE_THREADS / LANES) + threadIdx.x / LANES; w < vectors;
         w += (long long)gridDim.x * (CACHE_THREADS / LANES)) {
        const int t = (int)(w / c.heads), h = (int)(w - (long long)t * c.heads);
        uint4 kv = make_uint4(0, 0, 0, 0), vv = kv;
        const long long slot = t < n_here ? cache_slot(c, s, pos0 + t, status) : -1;
        if (slot >= 0) {
            const long long at = slot + ((long long)h << c.page_shift);
            if (QUANT) {
                kv = dequantise8(*reinterpret_cast<const uint2*>((const uint8_t*)c.k + at * D + lane * 8), c.k_exp[at]);
                vv = dequantise8(*reinterpret_cast<const uint2*>((const uint8_t*)c.v + at * D + lane * 8), c.v_exp[at]);
            } else {
                kv = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)c.k + at * D + lane * 8);
                vv = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)c.v + at * D + lane * 8);
            }
        }
        const long long o = (((long long)s * n + t) * c.heads + h) * D + lane * 8;
        *reinterpret_cast<uint4*>(k_out + o) = kv;
        *reinterpret_cast<uint4*>(v_out + o) = vv;
    }
}

int launch_cache_write(spec_ctx* ctx, const CacheArgs& c, const void* d_k, long long k_tok, long long k_head, const void* d_v,
                       long long v_tok, long long v_head, int S, int N, int n, const int32_t* d_nodes, const int32_t* d_start,
                       const int32_t* d_count, const RopeArgs& rope, cudaStream_t st) {
    const dim3 grid((n + WRITE_TOK - 1) / WRITE_TOK, S);
    const size_t smem = sizeof(float2) * WRITE_TOK * (rope.rot / 2);
    auto go = [&](auto kernel) {
        return launch_pdl(kernel, grid, dim3(CACHE_THREADS), smem, st, c, (const __nv_bfloat16*)d_k, k_tok, k_head,
                          (const __nv_bfloat16*)d_v, v_tok, v_head, N, n, d_nodes, d_start, d_count, rope, ctx->d_status);
    };
    cudaError_t e;
    if (c.quantised) e = c.head_dim == 64 ? go(cache_write_kernel<64, true>) : go(cache_write_kernel<128, true>);
    else e = c.head_dim == 64 ? go(cache_write_kernel<64, false>) : go(cache_write_kernel<128, false>);
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_cache_write launch");
}

int launch_cache_read(spec_ctx* ctx, const CacheArgs& c, int S, int n, const int32_t* d_start, const int32_t* d_count, void* d_k_out,
                      void* d_v_out, cudaStream_t st) {
    const long long per_cta = CACHE_THREADS / (c.head_dim / 8);
    const dim3 grid((unsigned)std::min<long long>(((long long)n * c.heads + per_cta - 1) / per_cta, 1 << 20), S);
    auto go = [&](auto kernel) {
        return launch_pdl(kernel, grid, dim3(CACHE_THREADS), 0, st, c, n, d_start, d_count, (__nv_bfloat16*)d_k_out, (__nv_bfloat16*)d_v_out,
                          ctx->d_status);
    };
    cudaError_t e;
    if (c.quantised) e = c.head_dim == 64 ? go(cache_read_kernel<64, true>) : go(cache_read_kernel<128, true>);
    else e = c.head_dim == 64 ? go(cache_read_kernel<64, false>) : go(cache_read_kernel<128, false>);
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_cache_read launch");
}

// ------------------------------------------------------------------------------------------ masks of draft trees
// A thread walks from its node to the root.  Parents come before their children, so the walk meets the words of the
// node's mask in descending order and each is stored once.  A node whose walk leaves that order has no mask.
__global__ void __launch_bounds__(128) tree_mask_kernel(const int32_t* __restrict__ parent, int N, int words, const int32_t* __restrict__ n_nodes,
                                                        int32_t* __restrict__ mask, int32_t* __restrict__ depth) {
    extern __shared__ int32_t par[];
    grid_dependency_wait();
    grid_launch_dependents();
    const int s = blockIdx.y, node = blockIdx.x * blockDim.x + threadIdx.x;
    const int live = n_nodes ? min(n_nodes[s], N) : N;
    for (int i = threadIdx.x; i < N; i += blockDim.x) par[i] = parent[(long long)s * N + i];
    __syncthreads();
    if (node >= N) return;
    int steps = -1, at = node;
    bool ok = node < live;
    while (ok && at >= 0) {  // ends: `at` falls with every step
        const int up = par[at];
        ok = up >= -1 && up < at;
        at = up;
        ++steps;
    }
    int32_t* row = mask + ((long long)s * N + node) * words;
    at = ok ? node : -1;
    for (int w = words - 1; w >= 0; --w) {
        uint32_t bits = 0;
        while (at >= 0 && (at >> 5) == w) {
            bits |= 1u << (at & 31);
            at = par[at];
        }
        row[w] = (int32_t)bits;
    }
    if (depth) depth[(long long)s * N + node] = ok ? steps : -1;
}

int launch_tree_mask(spec_ctx* ctx, const int32_t* d_parent, int S, int N, const int32_t* d_n_nodes, int32_t* d_mask, int32_t* d_depth,
                     cudaStream_t st) {
    cudaError_t e = launch_pdl(tree_mask_kernel, dim3((N + 127) / 128, S), dim3(128), sizeof(int32_t) * N, st, d_parent, N, (N + 31) / 32,
                               d_n_nodes, d_mask, d_depth);
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_tree_mask launch");
}

}  // namespace ngs
