// What surrounds the attention of a verification call: rotary positions of the block's queries and keys, the paged
// key/value cache (bfloat16, or E4M3 codes with a power-of-two scale per vector) and the bit masks of draft trees.
//
// All four kernels move each byte once and compute little on it; a thread handles 16 bytes of a head at a time.  A prompt
// is bound by its bytes, a decode step's few tokens by the launch, rotary rows of few heads by what is done once per token,
// and a mask by the walk to the root, a step of which waits for the one before.
//
//   rotary positions        y0 = (x0 cos a - x1 sin a) f, y1 = (x0 sin a + x1 cos a) f, a = pos * freq, in fp32, rounded once
//   E4M3 vector             scale = the smallest 2^e with max |x| <= 448 * 2^e, code = E4M3 nearest to x / scale
//
// On a B200 (copies 6.5 TB/s), 8 prompts of 4001 tokens, 8 heads of 128, keys rotated on the way: written to an E4M3 cache
// in 57 us (197 MB, 3.5 TB/s; 44 without rotation, and 44 rotated into a bfloat16 cache: only the sine and cosine of each
// token and the conversions together are more than the loads hide), read back in 44 us (197 MB, 4.5 TB/s).  Rotation of 32001 tokens,
// 32 + 8 heads of 128, half of each: 122 us (656 MB, 5.4 TB/s); of 32000 tokens with 3 + 1 heads of 64 or 1 + 1 of 128: 34 us
// (33 MB, 1 TB/s: a CTA of one or two warps for each token's table).  A decode step's 48 tokens: 2 to 4 us, the launch.  Masks of 64 x 144
// nodes: 10 us; of one chain of 4096: 242 us.
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include <algorithm>
#include <type_traits>

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

// The (cos, sin) table of one token, in the order in which lanes read it: pair p of a run of G pairs that one lane has
// lies at (p % G) * (half / G) + p / G, so that neighbouring lanes read neighbouring words (in the order of the pairs all
// lanes of a warp would meet in two banks).
__device__ __forceinline__ int table_at(int p, int g, int half) { return (p % g) * (half / g) + p / g; }

// Rotates the chunk of 8 elements that starts at element e of a head; `other` is the chunk that the pairs of a half layout
// have their other elements in.  G: pairs that one lane has, 8 in a half layout, and 8 or 4 if interleaved.
template <bool INTERLEAVED, int G>
__device__ __forceinline__ uint4 rope_chunk(const uint4& chunk, uint4 other, const float2* table, int e, int half) {
    float x[8], y[8];
    unpack_bf16x8(chunk, x);
    if (INTERLEAVED) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const float2 cs = table[table_at(e / 2 + j, G, half)];
            y[2 * j] = x[2 * j] * cs.x - x[2 * j + 1] * cs.y;
            y[2 * j + 1] = x[2 * j] * cs.y + x[2 * j + 1] * cs.x;
        }
    } else {
        const bool first = e < half;
        const uint32_t sign = first ? 0x80008000u : 0u;  // the first of a pair takes the other's product off
        other.x ^= sign;
        other.y ^= sign;
        other.z ^= sign;
        other.w ^= sign;
        float o[8];
        unpack_bf16x8(other, o);
        const float2* row = table + (first ? e : e - half) / 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float2 cs = row[j * (half / 8)];
            y[j] = x[j] * cs.x + o[j] * cs.y;
        }
    }
    return pack_bf16x8(y);
}

// ------------------------------------------------------------------------------------------ rotary positions
struct RopeRows {
    const __nv_bfloat16* x;
    __nv_bfloat16* y;
    long long tok, head;  // strides of x in elements; y is [T, heads, D]
    int heads;
};
// One CTA per token (and slice of its heads): the (cos, sin) table of the token is made once and serves all heads of
// q and k.  A thread owns both chunks that a pair lies in, so that y may be x, and has them on their way before the
// table is made: loading them after it left the kernel waiting twice (32001 tokens, 40 heads of 128: 166 us, so 123).
constexpr int ROPE_THREADS = 512;
template <bool INTERLEAVED>
__global__ void __launch_bounds__(ROPE_THREADS) rope_rows_kernel(RopeRows q, RopeRows k, int D, RopeArgs rope, const int32_t* __restrict__ pos) {
    extern __shared__ float2 table[];
    grid_dependency_wait();
    grid_launch_dependents();
    const long long t = blockIdx.x;
    const int half = rope.rot / 2;
    const int per_head = D / 16;  // a work item is 16 elements: two chunks that pair up, or two neighbours
    const int rot_items = rope.rot / 16;
    const int items = (q.heads + k.heads) * per_head;
    const int it = blockIdx.y * blockDim.x + threadIdx.x;
    const int h = it / per_head, i = it - h * per_head;
    const bool is_q = h < q.heads;
    const RopeRows& r = is_q ? q : k;
    const int hh = is_q ? h : h - q.heads;
    const bool rotated = i < rot_items;
    const bool split = rotated && !INTERLEAVED;
    const int e0 = split ? i * 8 : i * 16, e1 = split ? e0 + half : e0 + 8;
    uint4 a = make_uint4(0, 0, 0, 0), b = a;
    if (it < items) {
        const __nv_bfloat16* x = r.x + t * r.tok + hh * r.head;
        a = *reinterpret_cast<const uint4*>(x + e0);
        b = *reinterpret_cast<const uint4*>(x + e1);
    }
    for (int j = threadIdx.x; j < half; j += blockDim.x) table[table_at(j, 8, half)] = rope_cos_sin(pos[t], rope.freq[j], rope.factor);
    __syncthreads();
    if (it >= items) return;
    if (rotated) {
        const uint4 a0 = a;
        a = rope_chunk<INTERLEAVED, 8>(a0, b, table, e0, half);
        b = rope_chunk<INTERLEAVED, 8>(b, a0, table, e1, half);
    }
    __nv_bfloat16* y = r.y + (t * r.heads + hh) * D;
    *reinterpret_cast<uint4*>(y + e0) = a;
    *reinterpret_cast<uint4*>(y + e1) = b;
}

int launch_rope_rows(spec_ctx* ctx, const RopeArgs& rope, const void* d_q, int Hq, long long q_tok, long long q_head, void* d_q_out,
                     const void* d_k, int Hkv, long long k_tok, long long k_head, void* d_k_out, int D, const int32_t* d_pos, int T,
                     cudaStream_t st) {
    const RopeRows q{(const __nv_bfloat16*)d_q, (__nv_bfloat16*)d_q_out, q_tok, q_head, Hq};
    const RopeRows k{(const __nv_bfloat16*)d_k, (__nv_bfloat16*)d_k_out, k_tok, k_head, Hkv};
    const int items = (Hq + Hkv) * (D / 16);
    // as few threads as hold all items of a token in equal slices; few tokens: smaller slices, for more of the SMs
    int slices = (items + ROPE_THREADS - 1) / ROPE_THREADS;
    slices = std::max(slices, std::min((items + 63) / 64, ctx->num_sms / T));
    const int threads = ((items + slices - 1) / slices + 31) / 32 * 32;
    auto go = [&](auto kernel) { return launch_pdl(kernel, dim3(T, slices), dim3(threads), sizeof(float2) * (rope.rot / 2), st, q, k, D, rope, d_pos); };
    cudaError_t e = rope.interleaved ? go(rope_rows_kernel<true>) : go(rope_rows_kernel<false>);
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

// The largest magnitude of 8 bfloat16, as its bits: they order like the magnitudes, NaN above all.
__device__ __forceinline__ uint32_t top16(const uint4& v) {
    const uint32_t m = __vmaxu2(__vmaxu2(v.x & 0x7FFF7FFFu, v.y & 0x7FFF7FFFu), __vmaxu2(v.z & 0x7FFF7FFFu, v.w & 0x7FFF7FFFu));
    return max(m & 0xFFFFu, m >> 16);
}

// Quantises a vector that LANES neighbouring lanes hold 8 elements each of.  The scale is the smallest power of two
// that brings the largest magnitude to at most 448: E4M3 keeps three mantissa bits at every exponent, so a power of
// two loses nothing against a finer scale, dividing by it rounds nothing, and a reader gets code * scale exactly in
// bfloat16.  Its exponent stays in [-120, 7]: magnitudes above 448 * 2^7 (infinities too) are held as that.  A vector
// with a NaN is held as the scale byte 255 and reads as NaN throughout.
__device__ __forceinline__ uint2 quantise_to(const uint4& v, uint32_t top, uint32_t& scale) {
    int e = (int)(top >> 7) - 127 - 8 + ((top & 0x7Fu) > 0x60u ? 1 : 0);  // 448 = 1.75 * 2^8
    e = top == 0u ? 0 : min(max(e, E8_MIN), E8_MAX);
    const bool nan = top > 0x7F80u;
    scale = nan ? 255u : (uint32_t)(e + 127);
    const float inv = __uint_as_float((uint32_t)(127 - e) << 23);
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t r[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint16_t q;
        asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(q) : "f"(__uint_as_float(w[j] & 0xFFFF0000u) * inv), "f"(__uint_as_float(w[j] << 16) * inv));
        r[j] = q;
    }
    return nan ? make_uint2(0x7F7F7F7Fu, 0x7F7F7F7Fu) : make_uint2(__byte_perm(r[0], r[1], 0x5410), __byte_perm(r[2], r[3], 0x5410));
}
// Both vectors of a slot: their two maxima travel in one word.
template <int LANES>
__device__ __forceinline__ void quantise_vectors(const uint4& k, const uint4& v, uint2& kq, uint2& vq, uint32_t& ks, uint32_t& vs) {
    uint32_t m = top16(k) | (top16(v) << 16);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) m = __vmaxu2(m, __shfl_xor_sync(0xffffffffu, m, o));
    kq = quantise_to(k, m & 0xFFFFu, ks);
    vq = quantise_to(v, m >> 16, vs);
}

// A CTA writes `n_tok` tokens of one sequence, all heads of K and V: the rotation table is made once per token.  A thread
// has CACHE_DEPTH vectors' chunks of K and V on their way before it makes its part of the table and looks up the slots.
constexpr int CACHE_DEPTH = 4, WRITE_MAX_TOK = 32;
enum { ROPE_NONE, ROPE_HALF, ROPE_PAIRS };
template <int D, bool QUANT, int ROPE>
__global__ void __launch_bounds__(CACHE_THREADS, 4) cache_write_kernel(CacheArgs c, const __nv_bfloat16* __restrict__ k, long long k_tok,
                                                                    long long k_head, const __nv_bfloat16* __restrict__ v, long long v_tok,
                                                                    long long v_head, int N, int n, int n_tok, const int32_t* __restrict__ nodes,
                                                                    const int32_t* __restrict__ start, const int32_t* __restrict__ count,
                                                                    RopeArgs rope, int* status) {
    constexpr int LANES = D / 8, PASS = CACHE_THREADS / LANES;  // vectors that the CTA handles side by side
    extern __shared__ float2 table[];  // [n_tok, rot / 2]
    __shared__ long long dst[WRITE_MAX_TOK];
    grid_dependency_wait();
    grid_launch_dependents();
    const int s = blockIdx.y, i0 = blockIdx.x * n_tok;
    const int n_here = min(count ? min(count[s], n) : n, i0 + n_tok) - i0;
    if (n_here <= 0) return;
    const int pos0 = start[s] + i0;
    const int vectors = n_here * c.heads, lane = threadIdx.x % LANES, e = lane * 8;
    const int half = rope.rot / 2;
    for (int base = 0; base < vectors; base += CACHE_DEPTH * PASS) {  // (once, unless there are very many heads)
        uint4 kv[CACHE_DEPTH], vv[CACHE_DEPTH];
        int tok[CACHE_DEPTH], head[CACHE_DEPTH];
#pragma unroll
        for (int j = 0; j < CACHE_DEPTH; ++j) {
            const int w = base + j * PASS + threadIdx.x / LANES;
            kv[j] = vv[j] = make_uint4(0, 0, 0, 0);
            tok[j] = -1;
            if (w < vectors) {
                const int t = w / c.heads, h = w - t * c.heads;
                tok[j] = t;
                head[j] = h;
                const int node = nodes ? nodes[(long long)s * n + i0 + t] : i0 + t;
                if (node >= 0 && node < N) {
                    const long long src = (long long)s * N + node;
                    kv[j] = *reinterpret_cast<const uint4*>(k + src * k_tok + h * k_head + e);
                    vv[j] = *reinterpret_cast<const uint4*>(v + src * v_tok + h * v_head + e);
                }
            }
        }
        if (base == 0) {
            if (threadIdx.x < n_here) {
                const int node = nodes ? nodes[(long long)s * n + i0 + threadIdx.x] : i0 + (int)threadIdx.x;
                dst[threadIdx.x] = node >= 0 && node < N ? cache_slot(c, s, pos0 + (int)threadIdx.x, status) : -1;
            }
            for (int i = threadIdx.x; ROPE != ROPE_NONE && i < n_here * half; i += CACHE_THREADS) {
                const int t = i / half, p = i - t * half;
                table[t * half + table_at(p, ROPE == ROPE_PAIRS ? 4 : 8, half)] = rope_cos_sin(pos0 + t, rope.freq[p], rope.factor);
            }
            __syncthreads();
        }
#pragma unroll
        for (int j = 0; j < CACHE_DEPTH; ++j) {  // (lanes exchange chunks and maxima: all of a warp come here)
            const int t = max(tok[j], 0);
            const long long slot = dst[t];
            const bool on = tok[j] >= 0 && slot >= 0;
            if (ROPE != ROPE_NONE) {  // a key is bfloat16 before it is quantised, as it is for the block's own attention
                const bool rotated = e < rope.rot;
                uint4 o = kv[j];
                if (ROPE == ROPE_HALF) {  // the pairs' other elements are `half` elements away, in another lane
                    const int from = (threadIdx.x & 31) + (!rotated ? 0 : (e < half ? half / 8 : -(half / 8)));
                    o.x = __shfl_sync(0xffffffffu, kv[j].x, from);
                    o.y = __shfl_sync(0xffffffffu, kv[j].y, from);
                    o.z = __shfl_sync(0xffffffffu, kv[j].z, from);
                    o.w = __shfl_sync(0xffffffffu, kv[j].w, from);
                }
                if (rotated) kv[j] = rope_chunk<ROPE == ROPE_PAIRS, ROPE == ROPE_PAIRS ? 4 : 8>(kv[j], o, table + t * half, e, half);
            }
            const long long at = on ? slot + ((long long)head[j] << c.page_shift) : 0;
            if (QUANT) {
                uint2 kq, vq;
                uint32_t ks, vs;
                quantise_vectors<LANES>(kv[j], vv[j], kq, vq, ks, vs);
                if (on) {
                    *reinterpret_cast<uint2*>((uint8_t*)c.k + at * D + e) = kq;
                    *reinterpret_cast<uint2*>((uint8_t*)c.v + at * D + e) = vq;
                    if (lane == 0) {
                        c.k_exp[at] = (uint8_t)ks;
                        c.v_exp[at] = (uint8_t)vs;
                    }
                }
            } else if (on) {
                *reinterpret_cast<uint4*>((__nv_bfloat16*)c.k + at * D + e) = kv[j];
                *reinterpret_cast<uint4*>((__nv_bfloat16*)c.v + at * D + e) = vv[j];
            }
        }
    }
}

// 8 E4M3 codes times a power of two, as bfloat16 (exact).  Scales beyond the format's largest read as NaN.
__device__ __forceinline__ uint4 dequantise8(uint2 codes, uint8_t scale) {
    const float f = (int)scale > 127 + E8_MAX ? __uint_as_float(0x7FC00000u) : ldexpf(1.0f, (int)scale - 127);
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
    constexpr int LANES = D / 8, PASS = CACHE_THREADS / LANES;
    grid_dependency_wait();
    grid_launch_dependents();
    const int s = blockIdx.y;
    const int n_here = count ? min(count[s], n) : n;
    const int pos0 = start[s];
    const long long vectors = (long long)n * c.heads;
    const int lane = threadIdx.x % LANES;
    const long long first = (long long)blockIdx.x * (CACHE_DEPTH * PASS) + threadIdx.x / LANES;
    uint4 kv[CACHE_DEPTH], vv[CACHE_DEPTH];  // QUANT: codes in x, y and the scale byte in z
#pragma unroll
    for (int j = 0; j < CACHE_DEPTH; ++j) {
        const long long w = first + j * PASS;
        kv[j] = vv[j] = make_uint4(0, 0, 127, 0);
        if (!QUANT) kv[j].z = vv[j].z = 0;
        if (w >= vectors) continue;
        const int t = (int)(w / c.heads), h = (int)(w - (long long)t * c.heads);
        const long long slot = t < n_here ? cache_slot(c, s, pos0 + t, status) : -1;
        if (slot < 0) continue;
        const long long at = slot + ((long long)h << c.page_shift);
        if (QUANT) {
            const uint2 kq = *reinterpret_cast<const uint2*>((const uint8_t*)c.k + at * D + lane * 8);
            const uint2 vq = *reinterpret_cast<const uint2*>((const uint8_t*)c.v + at * D + lane * 8);
            kv[j] = make_uint4(kq.x, kq.y, c.k_exp[at], 0);
            vv[j] = make_uint4(vq.x, vq.y, c.v_exp[at], 0);
        } else {
            kv[j] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)c.k + at * D + lane * 8);
            vv[j] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)c.v + at * D + lane * 8);
        }
    }
#pragma unroll
    for (int j = 0; j < CACHE_DEPTH; ++j) {
        const long long w = first + j * PASS;
        if (w >= vectors) continue;
        if (QUANT) {
            kv[j] = dequantise8(make_uint2(kv[j].x, kv[j].y), (uint8_t)kv[j].z);
            vv[j] = dequantise8(make_uint2(vv[j].x, vv[j].y), (uint8_t)vv[j].z);
        }
        const long long o = ((long long)s * vectors + w) * D + lane * 8;
        *reinterpret_cast<uint4*>(k_out + o) = kv[j];
        *reinterpret_cast<uint4*>(v_out + o) = vv[j];
    }
}

int launch_cache_write(spec_ctx* ctx, const CacheArgs& c, const void* d_k, long long k_tok, long long k_head, const void* d_v,
                       long long v_tok, long long v_head, int S, int N, int n, const int32_t* d_nodes, const int32_t* d_start,
                       const int32_t* d_count, const RopeArgs& rope, cudaStream_t st) {
    // tokens of a CTA: CACHE_DEPTH vectors per thread, fewer where that would leave SMs without work
    const int pass = CACHE_THREADS / (c.head_dim / 8);
    const long long vectors = (long long)S * n * c.heads;
    const int depth = (int)std::min<long long>(CACHE_DEPTH, std::max<long long>(1, vectors / ((long long)pass * 2 * ctx->num_sms)));
    const int n_tok = std::min(std::min(WRITE_MAX_TOK, n), std::max(1, depth * pass / c.heads));
    const dim3 grid((n + n_tok - 1) / n_tok, S);
    const size_t smem = sizeof(float2) * n_tok * (rope.rot / 2);
    auto go = [&](auto kernel) {
        return launch_pdl(kernel, grid, dim3(CACHE_THREADS), smem, st, c, (const __nv_bfloat16*)d_k, k_tok, k_head,
                          (const __nv_bfloat16*)d_v, v_tok, v_head, N, n, n_tok, d_nodes, d_start, d_count, rope, ctx->d_status);
    };
    auto by_rope = [&](auto dim, auto quant) {
        constexpr int D = decltype(dim)::value;
        constexpr bool Q = decltype(quant)::value;
        return rope.rot == 0 ? go(cache_write_kernel<D, Q, ROPE_NONE>) : (rope.interleaved ? go(cache_write_kernel<D, Q, ROPE_PAIRS>) : go(cache_write_kernel<D, Q, ROPE_HALF>));
    };
    using D64 = std::integral_constant<int, 64>;
    using D128 = std::integral_constant<int, 128>;
    cudaError_t e;
    if (c.quantised) e = c.head_dim == 64 ? by_rope(D64(), std::true_type()) : by_rope(D128(), std::true_type());
    else e = c.head_dim == 64 ? by_rope(D64(), std::false_type()) : by_rope(D128(), std::false_type());
    ctx->launches += 1;
    return check_cuda(ctx, e, "spec_cache_write launch");
}

int launch_cache_read(spec_ctx* ctx, const CacheArgs& c, int S, int n, const int32_t* d_start, const int32_t* d_count, void* d_k_out,
                      void* d_v_out, cudaStream_t st) {
    const long long per_cta = CACHE_DEPTH * (CACHE_THREADS / (c.head_dim / 8));
    const dim3 grid((unsigned)(((long long)n * c.heads + per_cta - 1) / per_cta), S);
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
