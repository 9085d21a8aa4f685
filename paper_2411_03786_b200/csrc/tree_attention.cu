// Attention of a block of drafted nodes over a paged cache and the block itself (spec_tree_attention).
//
// For a sequence s and key head h the queries of all nodes and of the G = Hq / heads query heads that share h form the
// rows of one matrix Q, row r = node * G + g; keys and values are the cache's `len` positions followed by the block's
// nodes, cut into tiles of 128.  Per tile
//     S = Q K^T,   m' = max(m, rowmax S),   P = exp(c S - c m'),   l = l exp(c m - c m') + rowsum P,   O = O exp(..) + P V
// and o = O / l at the end.  Both products run on the tensor cores (tcgen05, bf16 x bf16 -> fp32): S and O live in tensor
// memory, P goes back into tensor memory as bfloat16 (over S, which has been read by then) and is the A operand of
// P V from there, so that no intermediate touches shared memory.  P is at most 2^8 and keeps 8 bits (the products take
// nothing wider; it is what the error against exact arithmetic, 2e-3 of the outputs' rms, comes from); its row sum is
// taken in fp32 before the rounding.  m need not be the maximum itself: it is a score of the row that stays the
// reference until weights grow beyond 2^8, so that the read-modify-write of O that a new reference costs happens in
// the first tiles and hardly ever after.
//
// Two streams per CTA hide the softmax of one tile behind the products of another.  With more than 128 rows they are
// two row tiles against the same keys; with at most 128 they are the even and the odd tiles of keys against the same
// rows, joined at the end (O of both streams lies in the same lanes).  One warp issues the products of both in turn,
// which keeps them out of step: in step, both would wait for the exponentials and then both for the products.
//
// Work: the tiles of all (s, h) in a row are cut into equal consecutive ranges, one per CTA (with several row-tile pairs:
// per group of CTAs, one for each, which walk the same keys in step and so share them in L2).  A range that ends inside
// an (s, h) leaves fp32 partial rows and their (m, l), which a second kernel joins in a fixed order.  Any mixture of
// lengths thus occupies all SMs to within a tile, and nothing about the lengths is needed on the host.
//
// Warps (896 threads, which share the registers unevenly): 0-7 and 8-15 softmax of stream 0 and 1 (a row's 128 scores
// belong to two threads, of warps w and w + 4: a single warp per scheduler leaves the special function unit waiting);
// 16-23 turn an E4M3 cache's tiles into bfloat16 (code * scale, which is exact) and mend value tiles (zeros after the
// end of a context, and in place of what is not finite in the block); 24 TMA; 25 issues the products; 26 walks the CTA's
// range and tells the others; 27 writes the rows of nodes that are not live.
//
// What bounds it, on a B200 (copies 6.5 TB/s, products 1650 TFLOP/s in a burst, 1400 under the power cap):
//   few rows, bfloat16 cache    the bytes: 64 sequences of one token, 32 / 8 heads of 128, 2048 keys: 99-102 us, 5.3 TB/s
//   few rows, E4M3 cache        the loader warps, which are at one tile together: wait, loads, conversion, stores, fence, 1500
//                               cycles for 128 vectors of 128, of which integer instructions alone would take 430 (but 11
//                               more of them for 16 codes made 102 us 123): 16 x 8192 keys, 102 us, 2.6 TB/s of codes, no
//                               faster than a bfloat16 cache (92 us) yet
//   many rows, long contexts    a stream's chain scores -> weights -> outputs, of which two overlap (a key tile per 4100
//                               cycles), and the power cap: 4 x 704 nodes, 16384 keys, 690-820 us, 0.92-1.09 PFLOP/s
//   prompts                     the same, with masks in every tile of the block: a chain of 4096 nodes, 32 / 8 heads, 508 us,
//                               0.27 PFLOP/s of what is visible; 32 / 32 heads, 618 us (hidden tiles are not left out there)
//   short contexts              a segment's beginning and end, 6-10 us where a tile takes 2: 64 x 144 nodes, 2048 keys,
//                               bfloat16 470 us, E4M3 550-575 us
//   one short call              two launches and a segment: 10-15 us
#include <cuda_bf16.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "cache.cuh"
#include "tc100.cuh"

namespace ngs {

constexpr int SOFTMAX_WARPS = 16, LOADER_WARPS = 8, LOADERS = 32 * LOADER_WARPS, TMA_WARP = 24, MMA_WARP = 25, PLAN_WARP = 26, BLANK_WARP = 27;
constexpr int TILE = 128;  // keys of a tile and rows of a row tile
constexpr int ATT_SMEM = 227 * 1024;
constexpr int ATT_THREADS = 896;  // whole warpgroups, which is what registers are moved between
constexpr int LAUNCH_REGS = 72;   // per thread at launch: 65536 / 896, rounded down to a multiple of 8
constexpr int REGS_SOFTMAX = 88, REGS_LOADER = 40, REGS_CONTROL = 72;
constexpr int SEGMENTS = 4;  // segments that the planning warp is ahead
static_assert(128 * (4 * REGS_SOFTMAX + 2 * REGS_LOADER + REGS_CONTROL) <= ATT_THREADS * LAUNCH_REGS, "the warpgroups' shares exceed the launch's registers");
constexpr int START = 4;  // tiles that the beginning and end of a segment take as long as (2 or 8 instead: no better)
constexpr float RESCALE = 256.0f;  // what 32 weights may add up to before their reference is moved

struct AttParams {
    TreeAttnArgs a;
    int G, n_qtiles, side, n_groups, passes;  // side: row-tile pairs that run side by side
    int rows_cap;                             // rows of a partial result
    float c;                                  // scale * log2(e)
    struct JoinTask* tasks;                   // [grid]
    float2* part_ml;                          // [grid * 2, rows_cap]
    float* part_o;                            // [grid * 2, D / 4, rows_cap, 4]
    unsigned long long wait_limit_ns;
};

// A run of key tiles [t0, t1) of one (s, h) against one row-tile pair.
struct Segment {
    int s, h, qt, t0, t1, n_prefix, len, live, rows;
    int whole;  // all key tiles of the (s, h)
    int split;  // the streams take the even and the odd key tiles; else a row tile each
    int slot;   // partial result: 0 = the CTA's range starts here, 1 = it ends here
    int more;   // 0: there was none left
    int first;  // tile t >= n_prefix is the block's tile t - first
};
// An (s, h) and row-tile pair that several CTAs walked: its partial rows are joined.  Recorded by the second of them.
struct __align__(16) JoinTask {
    int s, h, qt, rows;
    int n;      // parts; 0: nothing to join
    int first;  // slot of the first CTA's part
    int pad[2];
};
struct AttShared {
    uint64_t full[8], empty[8], go[8], stg_full[6], stg_empty[6], s_full[2], p_full[2], o_full, q_full, xch, seg_full[SEGMENTS], seg_empty[SEGMENTS];
    Segment segment[SEGMENTS];
    int nonfinite[16], bad_pages[16];  // by segment: its number + 1 if a value of the block is not finite, a page is not one of the pool's
    uint32_t tmem;
    int abort_flag;
};

// What is read in place of a page that is not there: its keys as NaN (and the scales of its keys, 255), the scales of its
// values as 1.
template <int N, int BYTE>
struct __align__(16) Filled {
    uint8_t byte[N];
    constexpr Filled() : byte() {
        for (int i = 0; i < N; ++i) byte[i] = BYTE;
    }
};
__device__ const Filled<TILE * 128, 255> nan_page;
__device__ const Filled<TILE, 127> unit_scales;

template <int D, bool Q8>
struct Geometry {
    static constexpr int HALVES = D / 64;  // 128-byte swizzle rows per vector
    static constexpr int TILE_BYTES = TILE * D * 2;
    static constexpr int SLOTS = Q8 ? (D == 128 ? 3 : 6) : (D == 128 ? 5 : 8);  // bf16 tiles in flight
    static constexpr int STAGES = Q8 ? (D == 128 ? 4 : 6) : 0;                  // E4M3 tiles in flight
    static constexpr int STAGE_BYTES = TILE * D;
    static constexpr int EXP_AT = 2 * TILE_BYTES + SLOTS * TILE_BYTES + STAGES * STAGE_BYTES;
    static constexpr int MISC_AT = EXP_AT + STAGES * TILE;
    static constexpr int SMEM = MISC_AT + (int)sizeof(AttShared);
    static_assert(SMEM <= ATT_SMEM, "shared memory");
};


// Key tiles of sequence s; 0 if it has no live node (or a length that its pages cannot hold).
__device__ __forceinline__ int sequence_tiles(const TreeAttnArgs& a, int s, int& len, int& live, int& n_prefix) {
    len = a.len[s];
    live = a.n_nodes ? min(max(a.n_nodes[s], 0), a.N) : a.N;
    if (len < 0 || (long long)len > ((long long)a.cache.max_pages << a.cache.page_shift)) {
        len = 0;
        live = 0;
    }
    n_prefix = (len + TILE - 1) / TILE;
    return live == 0 ? 0 : n_prefix + (live + TILE - 1) / TILE;
}

__device__ __forceinline__ int places(int n_tiles) { return n_tiles ? n_tiles + START : 0; }

// Quotient of numbers that nearly always fit in 32 bits (a 64-bit division is a long subroutine).
__device__ __forceinline__ long long quotient(long long a, long long b) {
    return ((a | b) >> 32) == 0 ? (long long)((uint32_t)a / (uint32_t)b) : a / b;
}
// The work is cut where it costs the same: every (s, h) counts as START places more than it has tiles, for what it takes to
// begin and end a segment (its places first), and the places [0, total) are cut into equal consecutive ranges: the first
// `rem` groups have base + 1 places, the others base.  With fewer places than groups, as many groups as places have one.
struct Ranges {
    long long total, n, base, rem;
    __device__ __forceinline__ Ranges(const AttParams& p, long long total_) : total(total_), n(min((long long)p.n_groups, total_)), base(0), rem(0) {
        if (n) {
            base = quotient(total, n);
            rem = total - base * n;
        }
    }
    __device__ __forceinline__ long long begin(long long g) const { return g * base + min(g, rem); }
    __device__ __forceinline__ long long group_of(long long x) const {
        return x < rem * (base + 1) ? quotient(x, base + 1) : rem + quotient(x - rem * (base + 1), base);
    }
};

// The planning warp's place in the CTA's range.
struct Walk {
    int s, h, t, pass, slot;
    long long pos, hi;
};
template <bool Q8>
__device__ __forceinline__ void advance(const AttParams& p, Walk& w, Segment& g) {
    int rows = 0;
    while (w.pos < w.hi && rows <= 0) {
        int len, live, n_prefix;
        const int n_tiles = sequence_tiles(p.a, w.s, len, live, n_prefix), n = places(n_tiles);
        if (w.t < n) {
            const int take = (int)min((long long)(n - w.t), w.hi - w.pos), qt = w.pass * p.side + (int)(blockIdx.x % p.side);
            g.t0 = max(w.t - START, 0);
            g.t1 = w.t + take - START;
            if (g.t1 > g.t0) {
                rows = qt < p.n_qtiles ? min(2 * TILE, live * p.G - qt * 2 * TILE) : 0;
                g.s = w.s;
                g.h = w.h;
                g.qt = qt;
                g.n_prefix = g.first = n_prefix;
                g.len = len;
                g.live = live;
                g.whole = g.t1 - g.t0 == n_tiles;
                // (a last single row tile beside pairs of the same keys: an E4M3 cache's tiles are converted for it alone, and
                // two at a time take longer than one
                // for both streams; 64 sequences of 144 nodes, 4 heads to a key head, 2048 keys: 657 us so, 761 us split)
                g.split = rows <= TILE && (!Q8 || qt == 0);
                g.slot = w.slot;
                w.slot = 1;
            }
            w.pos += take;
            w.t += take;
        }
        if (w.t >= n) {  // on to the next key head
            w.t = 0;
            if (n_tiles == 0 || ++w.h == p.a.cache.heads) {
                w.h = 0;
                if (++w.s == p.a.S) {
                    w.s = 0;
                    ++w.pass;
                }
            }
        }
    }
    g.rows = rows;
    g.more = rows > 0;
}

// Tiles of the block that the rows of a segment attend to, by a warp: the bits of their nodes lie one after another.
// Rows of drafts attend to their own few nodes, so that of a wide block's tiles most are empty for most rows.  Beyond
// MASK_WORDS looking would take longer than a tile or two, and all tiles count as attended to.  A segment takes those
// from the first to the last of them (8-bit cache: 64 sequences of 144 nodes in rows of 9, 2048 keys: 644 -> 561 us; one
// of 666 nodes, 14 / 2 heads of 64, 873 keys: 40 -> 30 us; one token: 14.4 -> 14.8 us).
constexpr int MASK_WORDS = 8192;
__device__ __forceinline__ uint32_t block_tiles(const AttParams& p, const Segment& g, int lane) {
    const int W = (p.a.N + 31) / 32, n0 = g.qt * 2 * TILE / p.G, n1 = (g.qt * 2 * TILE + g.rows - 1) / p.G + 1, words = (n1 - n0) * W;
    if (words > MASK_WORDS) return 0xFFFFFFFFu;
    const int32_t* bits = p.a.mask + ((long long)g.s * p.a.N + n0) * W;
    const int turn = 32 % W;
    uint32_t tiles = 0;
    int w = lane % W;  // the word's place in its node's mask
#pragma unroll 1
    for (int i0 = lane; i0 < words; i0 += 32 * 16) {
        int32_t x[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = i0 + 32 * j < words ? bits[i0 + 32 * j] : 0;
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            if (x[j]) tiles |= 1u << (w >> 2);
            w += turn;
            if (w >= W) w -= W;
        }
    }
    return __reduce_or_sync(0xffffffffu, tiles);
}

// Calls f(is_v, tile) for the key and value tiles of a segment in the order in which the products consume them;
// `lead`: streams that start side by side on different tiles (2 if they split the keys).
template <typename F>
__device__ __forceinline__ bool for_each_tile(const Segment& g, F&& f) {
    const int lead = g.split ? 2 : 1;
    const int t1 = g.t1;
    int k = g.t0, v = k;
    while (v < t1) {  // (one call of f: it is inlined)
        const bool is_v = k == t1 || k >= v + lead;
        if (!f(is_v, is_v ? v : k)) return false;
        if (is_v) ++v;
        else ++k;
    }
    return true;
}

__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
    const __nv_bfloat162 r = __hmul2(*reinterpret_cast<const __nv_bfloat162*>(&a), *reinterpret_cast<const __nv_bfloat162*>(&b));
    return *reinterpret_cast<const uint32_t*>(&r);
}
// Four E4M3 codes times a power of two as bfloat16, two to a word: a code's sign, exponent and mantissa moved into a
// bfloat16's fields read as its value times 2^-120 (subnormals as subnormals), and `f` holds scale * 2^120.  (The integer
// pipe is what converting is bound by: it has the shift to the right, the masks and the two joins, 6 instructions; the
// shift to the left is a multiplication.  Codes 0x7F and 0xFF, which the cache has in vectors of scale NaN only, would be
// 480: looking for them takes 11 more for 16 codes, one token of 16 sequences over 8192 keys 102 -> 123 us.)
__device__ __forceinline__ void e4m3x4_bf16x4(uint32_t w, uint32_t f, uint32_t& lo, uint32_t& hi) {
    uint32_t left;
    asm("mul.lo.u32 %0, %1, 16;" : "=r"(left) : "r"(w));
    const uint32_t low = left & 0xF0F0F0F0u, high = ((w >> 4) & 0x07070707u) | (w & 0x80808080u);  // the bytes of the results
    lo = mul_bf16x2(__byte_perm(low, high, 0x5140), f);
    hi = mul_bf16x2(__byte_perm(low, high, 0x7362), f);
}
__device__ __forceinline__ uint32_t scale_bf16x2(uint32_t exp) {
    return exp > 127u + E8_MAX ? 0x7FC07FC0u : (exp + 120u) * 0x00800080u;  // beyond the largest: NaN
}
__device__ __forceinline__ void st_shared16(uint32_t addr, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared16(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
// Where 16-byte chunk `c` of row r lies in a tile: blocks of 64 elements, rows of 128 bytes, chunks swizzled by the row.
__device__ __forceinline__ uint32_t tile_at(int r, int c) { return (uint32_t)((c >> 3) * (TILE * 128) + r * 128 + (((c & 7) ^ (r & 7)) << 4)); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// Weights 2^(c s - mc) of 32 scores, as bfloat16, and their sum.
__device__ __forceinline__ float weights32(const uint32_t (&s)[32], float c, float mc, uint32_t (&w)[16]) {
    float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < 16; ++j) {
        const float x = exp2_approx(fmaf(__uint_as_float(s[2 * j]), c, -mc)), y = exp2_approx(fmaf(__uint_as_float(s[2 * j + 1]), c, -mc));
        sum[(2 * j) & 3] += x;
        sum[(2 * j + 1) & 3] += y;
        w[j] = pack2(x, y);
    }
    return (sum[0] + sum[1]) + (sum[2] + sum[3]);
}
__device__ __forceinline__ float max32(const uint32_t (&s)[32]) {
    float m[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m[j] = fmaxf(__uint_as_float(s[j]), __uint_as_float(s[j + 4]));
#pragma unroll
        for (int i = j + 8; i < 32; i += 8) m[j] = fmaxf(m[j], fmaxf(__uint_as_float(s[i]), __uint_as_float(s[i + 4])));
    }
    return fmaxf(fmaxf(m[0], m[1]), fmaxf(m[2], m[3]));
}
__device__ __forceinline__ void hide(uint32_t (&s)[32], uint32_t seen) {  // scores without their bit become -inf
#pragma unroll
    for (int j = 0; j < 32; ++j)
        if (!((seen >> j) & 1u)) s[j] = 0xFF800000u;
}

// Positions [at, at + 32) of sequence s that lie in pages of the pool, as bits; `at` is one of the sequence's positions.
__device__ __forceinline__ uint32_t paged(const CacheArgs& c, int s, int at, int len) {
    const int32_t* table = c.table + (long long)s * c.max_pages + (at >> c.page_shift);
    auto bits = [&](int page) { return (unsigned)page < (unsigned)c.n_pages ? 0xFFFFFFFFu : 0u; };
    const uint32_t first = bits(table[0]);
    if (c.page_shift > 4) return first;
    return (first & 0xFFFFu) | (at + 16 < len ? bits(table[1]) << 16 : 0u);
}

__device__ __forceinline__ uint32_t nonfinite_to_zero(uint32_t v, bool& found) {
    if ((v & 0x7F80u) == 0x7F80u) {
        v &= 0xFFFF0000u;
        found = true;
    }
    if ((v & 0x7F800000u) == 0x7F800000u) {
        v &= 0x0000FFFFu;
        found = true;
    }
    return v;
}

template <int D, bool Q8>
__global__ void __launch_bounds__(ATT_THREADS, 1)
tree_attention_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ CUtensorMap tm_bk,
                      const __grid_constant__ CUtensorMap tm_bv, const __grid_constant__ AttParams p) {
    using Geo = Geometry<D, Q8>;
    extern __shared__ __align__(1024) unsigned char smem[];
    const uint32_t base = smem_u32(smem);
    if (base & 1023u) {  // (never: the swizzled tiles need it)
        if (threadIdx.x == 0) atomicOr(p.a.status, SPEC_STATUS_TIMEOUT);
        return;
    }
    const uint32_t q_at = base, ring_at = base + 2 * Geo::TILE_BYTES, stg_at = ring_at + Geo::SLOTS * Geo::TILE_BYTES;
    const uint32_t exp_at = base + Geo::EXP_AT;
    AttShared& sh = *reinterpret_cast<AttShared*>(smem + Geo::MISC_AT);
    volatile int* abort_flag = &sh.abort_flag;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const TreeAttnArgs& a = p.a;
    const CacheArgs& cache = a.cache;

    if (threadIdx.x == 0) {
        for (int i = 0; i < Geo::SLOTS; ++i) {
            mbar_init(smem_u32(&sh.full[i]), LOADERS);
            mbar_init(smem_u32(&sh.empty[i]), 1);
            mbar_init(smem_u32(&sh.go[i]), 1);
        }
        for (int i = 0; i < Geo::STAGES; ++i) {
            mbar_init(smem_u32(&sh.stg_full[i]), 1);
            mbar_init(smem_u32(&sh.stg_empty[i]), LOADERS);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&sh.s_full[i]), 1);
            mbar_init(smem_u32(&sh.p_full[i]), 8);
        }
        mbar_init(smem_u32(&sh.o_full), 1);
        mbar_init(smem_u32(&sh.q_full), SOFTMAX_WARPS);
        mbar_init(smem_u32(&sh.xch), SOFTMAX_WARPS / 2);
        for (int i = 0; i < SEGMENTS; ++i) {
            mbar_init(smem_u32(&sh.seg_full[i]), 1);
            mbar_init(smem_u32(&sh.seg_empty[i]), SOFTMAX_WARPS + LOADERS + 2);
        }
        for (int i = 0; i < 16; ++i) sh.nonfinite[i] = sh.bad_pages[i] = 0;
        sh.abort_flag = p.wait_limit_ns == 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == MMA_WARP) {
        tmem_alloc(smem_u32(&sh.tmem), 512);
        tmem_relinquish();
    }
    if (warp == TMA_WARP && lane < (Q8 ? 2 : 4))
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(lane == 0 ? &tm_k : (lane == 1 ? &tm_v : (lane == 2 ? &tm_bk : &tm_bv)))) : "memory");
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    grid_dependency_wait();
    const uint32_t tmem = sh.tmem;
    const uint32_t full = smem_u32(&sh.full[0]), empty = smem_u32(&sh.empty[0]), go = smem_u32(&sh.go[0]), stg_full = smem_u32(&sh.stg_full[0]), stg_empty = smem_u32(&sh.stg_empty[0]);
    const uint32_t s_full = smem_u32(&sh.s_full[0]), p_full = smem_u32(&sh.p_full[0]), o_full = smem_u32(&sh.o_full), q_full = smem_u32(&sh.q_full);
    const uint32_t xch_bar = smem_u32(&sh.xch), seg_full = smem_u32(&sh.seg_full[0]), seg_empty = smem_u32(&sh.seg_empty[0]);
    auto wait = [&](uint32_t bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, p.wait_limit_ns); };
    uint32_t n_seg = 0;  // segments that this warp has been through
    auto segment = [&]() -> const Segment& { return sh.segment[n_seg % SEGMENTS]; };
    auto segment_there = [&]() { return wait(seg_full + 8 * (n_seg % SEGMENTS), (n_seg / SEGMENTS) & 1u); };
    auto segment_done = [&]() {  // after the last look at it: by one lane for its warp, or by each of the loaders
        mbar_arrive(seg_empty + 8 * (n_seg % SEGMENTS));
    };

    if (warp < SOFTMAX_WARPS) {
        // ------------------------------------------------------------------------------------ softmax
        set_regs_up<REGS_SOFTMAX>();
        const int stream = warp >> 3, half = (warp >> 2) & 1, wq = warp & 3;
        const uint32_t lanes = tmem + ((uint32_t)(wq * 32) << 16);
        const uint32_t s_tm = lanes + stream * TILE, o_tm = lanes + 2 * TILE + stream * TILE;
        // The two warps of the same rows meet at a barrier of their own, with a vote.  They go through the same number of
        // meetings whatever happens: a wait that has expired is passed over, and the end is decided together.
        auto meet = [&](bool vote) {
            int r;
            asm volatile("{\n .reg .pred p, q;\n setp.ne.b32 p, %2, 0;\n bar.red.or.pred q, %1, 64, p;\n selp.b32 %0, 1, 0, q;\n}\n" : "=r"(r) : "r"(1 + stream * 4 + wq), "r"((int)vote) : "memory");
            return r != 0;
        };
        uint32_t n_s = 0, n_xch = 0;  // tiles of this stream, exchanges so far
        for (;; ++n_seg) {
            const bool there = __all_sync(0xffffffffu, segment_there());
            const Segment& g = segment();
            if (meet(!there || !g.more)) break;
            const bool split = g.split;
            const int tile_row = (split ? 0 : stream * TILE) + wq * 32 + lane;
            const bool valid = tile_row < g.rows;
            const bool warp_on = (split ? 0 : stream * TILE) + wq * 32 < g.rows;
            // ---- queries into shared memory (once: by stream 0 if both read the same rows), 16 rows by each warp
            if (!split || stream == 0) {
                constexpr int LPR = D / 8, RPI = 32 / LPR;  // lanes per row, rows per instruction
                const int R = g.qt * 2 * TILE + tile_row, node = R / p.G, gq = R - node * p.G;
                const long long off = valid ? ((long long)g.s * a.N + node) * a.q_tok + (long long)(g.h * p.G + gq) * a.q_head : -1;
                const uint32_t dst = q_at + stream * Geo::TILE_BYTES;
                const int c = lane % LPR;
                uint4 v[16 / RPI];
#pragma unroll
                for (int i = 0; i < 16 / RPI; ++i) {
                    const long long o = __shfl_sync(0xffffffffu, off, half * 16 + i * RPI + lane / LPR);
                    v[i] = make_uint4(0, 0, 0, 0);
                    if (o >= 0) v[i] = *reinterpret_cast<const uint4*>((const __nv_bfloat16*)a.q + o + c * 8);
                }
#pragma unroll
                for (int i = 0; i < 16 / RPI; ++i) st_shared16(dst + tile_at(wq * 32 + half * 16 + i * RPI + lane / LPR, c), v[i]);
                fence_async_smem();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
            // ---- key tiles
            float m = -INFINITY, l = 0.0f;  // m: the same in both threads of a row; l: this thread's columns
            const int step = split ? 2 : 1;
            for (int t = g.t0 + (split ? stream : 0); t < g.t1; t += step) {
                wait(s_full + 8 * stream, n_s & 1u);
                ++n_s;
                __syncwarp();
                tc_fence_after();
                if (warp_on) {
                    const int valid_keys = t < g.n_prefix ? g.len - t * TILE : g.live - (t - g.first) * TILE;
                    const bool masked = t >= g.n_prefix || valid_keys < TILE;
                    auto load = [&](int i, uint32_t(&x)[32]) {  // scores [32 i, 32 i + 32) of the row, -inf where it has none
                        tmem_ld32(s_tm + 32 * i, x);
                        tmem_wait_ld();
                        if (masked) {
                            const int left = valid_keys - 32 * i;
                            uint32_t seen = left >= 32 ? 0xFFFFFFFFu : (left <= 0 ? 0u : (1u << left) - 1u);
                            if (t >= g.n_prefix) {
                                const int words = (a.N + 31) / 32, at = (t - g.first) * 4 + i, node = (g.qt * 2 * TILE + tile_row) / p.G;
                                seen &= (valid && at < words) ? (uint32_t)a.mask[((long long)g.s * a.N + node) * words + at] : 0u;
                            }
                            hide(x, seen);
                        }
                    };
                    // The reference m is a score of the row that was the largest when it was taken: in the first tile, and
                    // again whenever some 32 weights add up to more than RESCALE (or to no number).  Only then is the
                    // maximum looked for, by both threads over the whole row.
                    uint32_t w[2][16];
                    float sum[2];
                    bool look = t < g.t0 + step;
#pragma unroll 1
                    for (;;) {
                        if (look) {
                            if (t < g.n_prefix && __any_sync(0xffffffffu, sh.bad_pages[n_seg & 15u] == (int)n_seg + 1)) {
                                // keys of missing pages: their NaN (which a maximum passes over) become -inf in this warp's half
#pragma unroll 1
                                for (int i = 2 * half; i < 2 * half + 2; ++i) {
                                    const int at = t * TILE + 32 * i;
                                    if (at >= g.len) break;
                                    uint32_t x[32], (&lo)[16] = *reinterpret_cast<uint32_t(*)[16]>(&x[0]), (&hi)[16] = *reinterpret_cast<uint32_t(*)[16]>(&x[16]);
                                    tmem_ld32(s_tm + 32 * i, x);
                                    tmem_wait_ld();
                                    hide(x, paged(cache, g.s, at, g.len));
                                    tmem_st16(s_tm + 32 * i, lo);
                                    tmem_st16(s_tm + 32 * i + 16, hi);
                                    tmem_wait_st();
                                }
                            }
                            float top = -INFINITY;
#pragma unroll 1
                            for (int i = 0; i < 4; ++i) {
                                uint32_t x[32];
                                load(i, x);
                                top = fmaxf(top, max32(x));
                            }
                            const bool move = top > m && !((top - m) * p.c <= 1.0f);
                            const float f = move ? exp2_approx((m - top) * p.c) : 1.0f;
                            if (move) m = top;
                            l *= f;
                            if (t >= g.t0 + step && __any_sync(0xffffffffu, move)) {  // this warp's half of O's columns
#pragma unroll 1
                                for (int i = half * (D / 2); i < (half + 1) * (D / 2); i += 16) {
                                    uint32_t o[16];
                                    tmem_ld16(o_tm + i, o);
                                    tmem_wait_ld();
#pragma unroll
                                    for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
                                    tmem_st16(o_tm + i, o);
                                }
                            }
                        }
                        // (no reference: all of the row's keys so far are hidden, and any number will do for their weights, 0)
                        const float mc = m == -INFINITY ? 0.0f : m * p.c;
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            uint32_t x[32];
                            load(2 * half + i, x);
                            sum[i] = weights32(x, p.c, mc, w[i]);
                        }
                        if (!meet(!look && (m == -INFINITY || !(sum[0] <= RESCALE && sum[1] <= RESCALE)))) break;
                        look = true;
                    }
                    // (the other warp has read its scores, which these weights overwrite in part)
                    l += sum[0] + sum[1];
                    tmem_st16(s_tm + 32 * half, w[0]);
                    tmem_st16(s_tm + 32 * half + 16, w[1]);
                    tmem_wait_st();
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * stream);
            }
            // ---- results
            wait(o_full, n_seg & 1u);
            __syncwarp();
            tc_fence_after();
            // sums and references change hands through the lanes' own columns of the scores, which are done with
            float f0 = 1.0f, f1 = 0.0f;
            const bool both = split && g.t1 - g.t0 > 1;  // stream 1 had a tile
            if (warp_on && (stream == 0 || !split || both)) {
                tmem_st1(s_tm + half, __float_as_uint(l));
                tmem_st1(s_tm + 2, __float_as_uint(m));
                tmem_wait_st();
                tc_fence_before();
                meet(false);
                tc_fence_after();
                const uint32_t other = tmem_ld1(s_tm + 1 - half);
                tmem_wait_ld();
                l += __uint_as_float(other);
            }
            if (both) {
                if (stream == 1) {
                    __syncwarp();
                    if (lane == 0) mbar_arrive(xch_bar);
                } else {
                    wait(xch_bar, n_xch & 1u);
                    __syncwarp();
                    tc_fence_after();
                    if (warp_on) {
                        const uint32_t la = tmem_ld1(s_tm + TILE), lb = tmem_ld1(s_tm + TILE + 1), m1 = tmem_ld1(s_tm + TILE + 2);
                        tmem_wait_ld();
                        const float other = __uint_as_float(m1), top = fmaxf(m, other);
                        f0 = m == -INFINITY ? 0.0f : exp2_approx((m - top) * p.c);
                        f1 = other == -INFINITY ? 0.0f : exp2_approx((other - top) * p.c);
                        l = l * f0 + (__uint_as_float(la) + __uint_as_float(lb)) * f1;
                        m = top;
                    }
                }
                ++n_xch;
            }
            if ((!split || stream == 0) && warp_on) {
                const int R = g.qt * 2 * TILE + tile_row, node = R / p.G, gq = R - node * p.G;
                const bool poisoned = sh.nonfinite[n_seg & 15u] == (int)n_seg + 1;
                const float inv = g.whole ? (l == 0.0f ? 0.0f : 1.0f / l) : 1.0f;
                const long long out_row = ((long long)g.s * a.N + node) * a.Hq + g.h * p.G + gq;
                const long long part = (long long)blockIdx.x * 2 + g.slot;
#pragma unroll 1
                for (int i = half * (D / 64); i < (half + 1) * (D / 64); ++i) {  // this warp's half of the columns
                    uint32_t o[32];
                    float x[32];
                    tmem_ld32(o_tm + 32 * i, o);
                    tmem_wait_ld();
#pragma unroll
                    for (int j = 0; j < 32; ++j) x[j] = __uint_as_float(o[j]) * f0;
                    if (both) {
                        tmem_ld32(o_tm + TILE + 32 * i, o);
                        tmem_wait_ld();
#pragma unroll
                        for (int j = 0; j < 32; ++j) x[j] += __uint_as_float(o[j]) * f1;
                    }
                    if (poisoned && valid) {
                        // values of the block that are not finite were taken as 0 in the products, where a weight of 0
                        // would have made them NaN; rows that do attend to them get them here
                        const int words = (a.N + 31) / 32;
                        const int from = (max(g.t0, g.n_prefix) - g.first) * TILE, to = min((g.t1 - g.first) * TILE, g.live);
                        for (int n = from; n < to; ++n) {
                            if (!((a.mask[((long long)g.s * a.N + node) * words + (n >> 5)] >> (n & 31)) & 1)) continue;
                            const __nv_bfloat16* v = (const __nv_bfloat16*)a.v + ((long long)g.s * a.N + n) * a.v_tok + (long long)g.h * a.v_head + 32 * i;
#pragma unroll
                            for (int j = 0; j < 32; ++j) {
                                const float y = __bfloat162float(v[j]);
                                if (!isfinite(y)) x[j] += y;
                            }
                        }
                    }
                    if (g.whole) {  // into the row's place in the query tile, which is done with
                        const uint32_t dst = q_at + stream * Geo::TILE_BYTES;
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            st_shared16(dst + tile_at(wq * 32 + lane, 4 * i + j),
                                        make_uint4(pack2(x[8 * j] * inv, x[8 * j + 1] * inv), pack2(x[8 * j + 2] * inv, x[8 * j + 3] * inv),
                                                   pack2(x[8 * j + 4] * inv, x[8 * j + 5] * inv), pack2(x[8 * j + 6] * inv, x[8 * j + 7] * inv)));
                    } else if (valid) {  // four columns of neighbouring rows side by side
                        float4* dst = reinterpret_cast<float4*>(p.part_o) + (part * (D / 4) + 8 * i) * p.rows_cap + tile_row;
#pragma unroll
                        for (int j = 0; j < 8; ++j) dst[(long long)j * p.rows_cap] = make_float4(x[4 * j], x[4 * j + 1], x[4 * j + 2], x[4 * j + 3]);
                    }
                }
                if (g.whole) {  // rows of the output from there, a 128-byte line (D = 64: half of one) by neighbouring lanes
                    constexpr int LPR = D / 16, RPI = 32 / LPR;  // lanes that share a row of this warp's columns, rows per instruction
                    const long long off = valid ? out_row * D : -1;
                    const uint32_t src = q_at + stream * Geo::TILE_BYTES;
                    const int c = half * LPR + lane % LPR;
                    __syncwarp();
#pragma unroll
                    for (int r0 = 0; r0 < 32; r0 += RPI) {
                        const int r = r0 + lane / LPR;
                        const long long o = __shfl_sync(0xffffffffu, off, r);
                        const uint4 v = ld_shared16(src + tile_at(wq * 32 + r, c));
                        if (o >= 0) *reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + o + c * 8) = v;
                    }
                }
                if (valid && half == 0) {
                    if (!g.whole) p.part_ml[part * p.rows_cap + tile_row] = make_float2(m, l);
                    else if (a.lse) a.lse[out_row] = l == 0.0f ? -INFINITY : (m * p.c + log2f(l)) * LN2;
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) segment_done();
        }
    } else if (warp < SOFTMAX_WARPS + LOADER_WARPS) {
        // ------------------------------------------------------------------------------------ tiles written by threads
        // (A wait that has expired is noticed by a warp's lanes at different times.  The other roles vote; here a lane leaves
        // by itself, so that nothing between this and the end of the role may wait for the warp's other lanes: they would be
        // waited for without a limit.  A vote at every wait: one token of 16 sequences over 8192 keys, E4M3: 102 -> 105 us.)
        set_regs_down<REGS_LOADER>();
        const int tid = threadIdx.x - 32 * SOFTMAX_WARPS;
        constexpr int CH = D / 8;  // 16-byte chunks of a bf16 vector
        uint32_t slot = 0, phase = 0, stg = 0, stg_phase = 0;
        uint32_t go_phase = 0;  // bit per slot
        for (;; ++n_seg) {
            if (!segment_there()) break;
            const Segment g = segment();  // (in registers: shared memory is looked at again after every barrier)
            if (!g.more) break;
            const bool ok = for_each_tile(g, [&](bool is_v, int t) {
                const bool block = t >= g.n_prefix;
                const uint32_t dst = ring_at + slot * Geo::TILE_BYTES, bar_full = full + 8 * slot, bar_empty = empty + 8 * slot;
                const uint32_t my_phase = phase, my_slot = slot;
                if (++slot == Geo::SLOTS) {
                    slot = 0;
                    phase ^= 1u;
                }
                const int rows = block ? g.live - (t - g.first) * TILE : g.len - t * TILE;  // may exceed the tile
                if (!Q8 && !(is_v && (block || rows < TILE))) return true;  // all TMA's
                if (Q8 && !block) {
                    if (!wait(stg_full + 8 * stg, stg_phase)) return false;
                    if (!wait(bar_empty, my_phase ^ 1u)) return false;
                    const uint32_t src = stg_at + stg * Geo::STAGE_BYTES, ex = exp_at + stg * TILE;
                    // A thread has 16 codes of rows 32 (D = 64: 64) apart, a staging row's pieces dealt out so that the 8 lanes
                    // that load or store together meet in no bank: lanes 0-3 the front of row r, 4-7 the back of row r + 1,
                    // the next 8 the other two (the swizzle turns even pieces of one row into odd ones of the next).
                    constexpr int LPR = D / 16, PER = TILE * LPR / LOADERS, STEP = LOADERS / LPR;
                    const int r = D == 64 ? tid / LPR : (tid / 16) * 2 + (((tid >> 3) ^ (tid >> 2)) & 1), c = D == 64 ? tid % LPR : (tid & 7);
                    const uint32_t from = src + r * D + c * 16, to = dst + tile_at(r, 2 * c);
                    uint4 v[PER];
                    uint32_t e[PER];
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        v[i] = ld_shared16(from + i * STEP * D);
                        asm volatile("ld.shared.u8 %0, [%1];" : "=r"(e[i]) : "r"(ex + r + i * STEP) : "memory");
                    }
                    if (rows < TILE) {  // (whatever the staging tile held)
#pragma unroll
                        for (int i = 0; i < PER; ++i)
                            if (r + i * STEP >= rows) {
                                v[i] = make_uint4(0, 0, 0, 0);
                                e[i] = 127;
                            }
                    }
#pragma unroll
                    for (int i = 0; i < PER; ++i) {
                        const uint32_t f = scale_bf16x2(e[i]);
                        uint4 lo, hi;
                        e4m3x4_bf16x4(v[i].x, f, lo.x, lo.y);
                        e4m3x4_bf16x4(v[i].y, f, lo.z, lo.w);
                        e4m3x4_bf16x4(v[i].z, f, hi.x, hi.y);
                        e4m3x4_bf16x4(v[i].w, f, hi.z, hi.w);
                        st_shared16(to + i * STEP * 128, lo);
                        st_shared16((to ^ 16u) + i * STEP * 128, hi);
                    }
                    mbar_arrive(stg_empty + 8 * stg);
                    if (++stg == Geo::STAGES) {
                        stg = 0;
                        stg_phase ^= 1u;
                    }
                } else {
                    if (!Q8) {
                        // TMA's as well, but what lies beyond the end must be 0 (a weight of 0 would not keep a NaN out of the
                        // products), and so must values of the block that are not finite.  (A barrier's parity tells one use
                        // of a slot from the next, not from the one after, so these threads, which skip slots, do not wait for
                        // empty ones: the TMA warp waits for every slot, and a barrier of the slot's own says it has landed.)
                        if (!wait(go + 8 * my_slot, (go_phase >> my_slot) & 1u)) return false;
                        go_phase ^= 1u << my_slot;
                        bool found = false;
#pragma unroll 2
                        for (int i = 0; i < TILE * CH / LOADERS; ++i) {
                            const int r = i * (LOADERS / CH) + tid / CH, c = tid % CH;
                            if (r >= rows) {
                                st_shared16(dst + tile_at(r, c), make_uint4(0, 0, 0, 0));
                            } else if (block) {
                                uint4 v = ld_shared16(dst + tile_at(r, c));
                                bool bad = false;
                                v.x = nonfinite_to_zero(v.x, bad);
                                v.y = nonfinite_to_zero(v.y, bad);
                                v.z = nonfinite_to_zero(v.z, bad);
                                v.w = nonfinite_to_zero(v.w, bad);
                                if (bad) st_shared16(dst + tile_at(r, c), v);
                                found |= bad;
                            }
                        }
                        if (found) sh.nonfinite[n_seg & 15u] = (int)n_seg + 1;
                        fence_async_smem();
                        mbar_arrive(bar_full);
                        return true;
                    }
                    bool found = false;  // a tile of the block
                    constexpr int PER = TILE * CH / LOADERS;
                    {
                        uint4 v[PER];
#pragma unroll
                        for (int i = 0; i < PER; ++i) {
                            const int r = i * (LOADERS / CH) + tid / CH, c = tid % CH;
                            v[i] = make_uint4(0, 0, 0, 0);
                            if (r >= rows) continue;
                            const long long tok = (long long)g.s * a.N + (t - g.first) * TILE + r;
                            const __nv_bfloat16* src = is_v ? (const __nv_bfloat16*)a.v + tok * a.v_tok + (long long)g.h * a.v_head
                                                            : (const __nv_bfloat16*)a.k + tok * a.k_tok + (long long)g.h * a.k_head;
                            v[i] = *reinterpret_cast<const uint4*>(src + c * 8);
                        }
                        if (!wait(bar_empty, my_phase ^ 1u)) return false;
#pragma unroll
                        for (int i = 0; i < PER; ++i) {
                            const int r = i * (LOADERS / CH) + tid / CH, c = tid % CH;
                            if (is_v) {
                                v[i].x = nonfinite_to_zero(v[i].x, found);
                                v[i].y = nonfinite_to_zero(v[i].y, found);
                                v[i].z = nonfinite_to_zero(v[i].z, found);
                                v[i].w = nonfinite_to_zero(v[i].w, found);
                            }
                            st_shared16(dst + tile_at(r, c), v[i]);
                        }
                    }
                    if (found) sh.nonfinite[n_seg & 15u] = (int)n_seg + 1;
                }
                fence_async_smem();
                mbar_arrive(bar_full);
                return true;
            });
            if (!ok) break;
            segment_done();
        }
    } else {
        set_regs_down<REGS_CONTROL>();
        if (warp == TMA_WARP) {
            // -------------------------------------------------------------------------------- TMA
            // A lane fetches one page's part of a tile.  Page numbers are read 32 at a time, a window ahead of their use (two
            // registers, by the window's parity: a load is never waited for where it is issued).
            uint32_t slot = 0, phase = 0;
            constexpr uint32_t RING = Q8 ? Geo::STAGES : Geo::SLOTS;
            const int page = 1 << cache.page_shift, per_tile = TILE >> cache.page_shift;
            const int all_rows = (cache.n_pages * cache.heads) << cache.page_shift;  // a coordinate beyond the cache: reads as 0
            for (;; ++n_seg) {
                if (!__all_sync(0xffffffffu, segment_there())) break;
                const Segment g = segment();
                if (!g.more) break;
                const int32_t* table = cache.table + (long long)g.s * cache.max_pages;
                const int n_pages = (g.len + page - 1) >> cache.page_shift;
                const int wsh = cache.page_shift - 2, in_window = (1 << wsh) - 1;  // tiles of a window: 4 to 32
                auto fetch = [&](int window) { return window * 32 + lane < n_pages ? table[window * 32 + lane] : 0; };
                const int w0 = g.t0 >> wsh;
                int even = fetch(w0 + (w0 & 1)), odd = fetch(w0 + 1 - (w0 & 1));
                const bool ok = for_each_tile(g, [&](bool is_v, int t) {
                    const bool block = t >= g.n_prefix;
                    const int rows = block ? TILE : min(g.len - t * TILE, TILE);
                    const bool mended = !Q8 && is_v && (block || rows < TILE);  // goes through the other threads' hands
                    const uint32_t bar_full = (Q8 ? stg_full : full) + 8 * slot, bar_empty = (Q8 ? stg_empty : empty) + 8 * slot;
                    const uint32_t dst = Q8 ? stg_at + slot * Geo::STAGE_BYTES : ring_at + slot * Geo::TILE_BYTES;
                    const uint32_t ex = exp_at + slot * TILE, bar_go = go + 8 * slot;
                    const uint32_t my_phase = phase;
                    if (!Q8 || !block) {
                        if (++slot == RING) {
                            slot = 0;
                            phase ^= 1u;
                        }
                    }
                    const int window = t >> wsh;
                    const int pid = __shfl_sync(0xffffffffu, (window & 1) ? odd : even, ((t & in_window) << (7 - cache.page_shift)) + (lane & (per_tile - 1)));
                    if (is_v && t > g.t0 && (t & in_window) == 0) {  // values, which come last, have left the window before
                        if (window & 1) even = fetch(window + 1);
                        else odd = fetch(window + 1);
                    }
                    if (Q8 && block) return true;
                    const int pages = block ? 0 : (rows + page - 1) >> cache.page_shift;
                    // A page that is not one of the pool's: its keys are made NaN, so that no weights come of the tile before
                    // the softmax warps have looked for its maximum, which is when they hide the positions of missing pages
                    // (masks in every tile instead, for the case that there are any: 64 x 144 nodes, E4M3: 563 -> 573 us); its values
                    // are 0.
                    const bool good = lane >= pages || (unsigned)pid < (unsigned)cache.n_pages;
                    if (!good) {
                        atomicOr(a.status, SPEC_STATUS_CAPACITY);
                        sh.bad_pages[n_seg & 15u] = (int)n_seg + 1;
                    }
                    const bool got = wait(bar_empty, my_phase ^ 1u);
                    if (!__all_sync(0xffffffffu, got)) return false;
                    __syncwarp();  // (what lane 0's arrival publishes includes the line above)
                    const uint32_t bar = mended ? bar_go : bar_full;
                    if (lane == 0) {
                        mbar_expect_tx(bar, (uint32_t)(block ? TILE : pages * page) * (Q8 ? D + 1 : 2 * D));
                        if (!Q8 && !mended) mbar_arrive_n(bar_full, LOADERS - 1);
                    }
                    __syncwarp();
                    if (block) {
                        if (lane < Geo::HALVES) tma_load_3d(dst + lane * (TILE * 128), is_v ? &tm_bv : &tm_bk, 64 * lane, g.h, g.s * a.N + (t - g.first) * TILE, bar);
                    } else if (lane < pages) {
                        const int row = good ? (pid * cache.heads + g.h) << cache.page_shift : all_rows;
                        const CUtensorMap* tm = is_v ? &tm_v : &tm_k;
                        if (Q8) {
                            tma_load_2d(dst + lane * page * D, tm, 0, row, bar);
                            bulk_load(ex + lane * page, good ? (is_v ? cache.v_exp : cache.k_exp) + row : (is_v ? unit_scales.byte : nan_page.byte), page, bar);
                        } else {
#pragma unroll
                            for (int i = 0; i < Geo::HALVES; ++i) {
                                const uint32_t to = dst + i * (TILE * 128) + lane * page * 128;
                                if (good || is_v) tma_load_2d(to, tm, 64 * i, row, bar);
                                else bulk_load(to, nan_page.byte, page * 128, bar);
                            }
                        }
                    }
                    return true;
                });
                if (!ok) break;
                __syncwarp();
                if (lane == 0) segment_done();
            }
        } else if (warp == MMA_WARP && lane == 0) {
            // -------------------------------------------------------------------------------- products
            const uint32_t id_qk = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(TILE >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
            const uint32_t id_pv = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(TILE >> 4) << 24);
            uint32_t slot = 0, phase = 0, n_p[2] = {0, 0};
            bool ok = true;
            auto take = [&](uint32_t& at, uint32_t& index) {  // the next tile of the ring, once it is there
                index = slot;
                at = ring_at + slot * Geo::TILE_BYTES;
                const bool got = wait(full + 8 * slot, phase);
                if (++slot == Geo::SLOTS) {
                    slot = 0;
                    phase ^= 1u;
                }
                tc_fence_after();
                return got;
            };
            auto ready = [&]() { return mbar_test_wait(full + 8 * slot, phase); };
            // (descriptors of the first k-slice; the others are a constant further in their address field)
            const uint64_t q_desc = make_kmajor_sw128_desc(q_at), k_desc = make_kmajor_sw128_desc(0), v_desc = make_mnmajor_sw128_desc(0, TILE * 128);
            auto qk = [&](int stream, int q_tile, uint32_t k_at) {
                const uint64_t qd = q_desc + (uint64_t)(q_tile * (Geo::TILE_BYTES >> 4)), kd = k_desc + (k_at >> 4);
                const uint32_t d = tmem + stream * TILE;
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    constexpr uint32_t half = TILE * 128 >> 4;
                    tc_mma_bf16(d, qd + ((k >> 2) * half + (k & 3) * 2), kd + ((k >> 2) * half + (k & 3) * 2), id_qk, k != 0);
                }
                tc_commit(s_full + 8 * stream);
            };
            auto pv = [&](int stream, uint32_t v_at, bool add) {
                const uint64_t vd = v_desc + (v_at >> 4);
                const uint32_t w = tmem + stream * TILE, d = tmem + 2 * TILE + stream * TILE;
#pragma unroll
                for (int k = 0; k < TILE / 16; ++k) tc_mma_bf16_ts(d, w + 8 * k, vd + k * (2048 >> 4), id_pv, (add || k != 0) ? 1u : 0u);
            };
            for (;; ++n_seg) {
                if (!segment_there()) break;
                const Segment& g = segment();
                if (!g.more) break;
                const int n = g.t1 - g.t0;
                uint32_t k_at, v_at, ki, vi;
                if (!(ok = wait(q_full, n_seg & 1u))) break;
                tc_fence_after();
                if (!g.split) {  // two row tiles, the same keys
                    if (!(ok = take(k_at, ki))) break;
                    qk(0, 0, k_at);
                    qk(1, 1, k_at);
                    tc_commit(empty + 8 * ki);
                    // (what can be done before the weights are there, or after the scores are on their way, is: the chain
                    // from a stream's weights to its next scores is what the pace depends on)
                    for (int t = 0; t < n && ok; ++t) {
                        const bool more = t + 1 < n;
                        if (!(ok = take(v_at, vi))) break;
                        const bool early = more && ready();  // the next keys: looked at once before, waited for only after
                        if (early) take(k_at, ki);
                        if (!(ok = wait(p_full, n_p[0]++ & 1u))) break;
                        tc_fence_after();
                        pv(0, v_at, t > 0);
                        if (more) {
                            if (!early && !(ok = take(k_at, ki))) break;
                            qk(0, 0, k_at);
                        }
                        if (!(ok = wait(p_full + 8, n_p[1]++ & 1u))) break;
                        tc_fence_after();
                        pv(1, v_at, t > 0);
                        if (more) qk(1, 1, k_at);
                        tc_commit(empty + 8 * vi);
                        if (more) tc_commit(empty + 8 * ki);
                    }
                } else {  // one row tile, alternate keys
                    for (int t = 0; t < 2 && t < n && ok; ++t) {
                        if (!(ok = take(k_at, ki))) break;
                        qk(t, 0, k_at);
                        tc_commit(empty + 8 * ki);
                    }
                    for (int t = 0; t < n && ok; ++t) {
                        const int i = t & 1;
                        const bool more = t + 2 < n;
                        if (!(ok = take(v_at, vi))) break;
                        const bool early = more && ready();
                        if (early) take(k_at, ki);
                        if (!(ok = wait(p_full + 8 * i, n_p[i]++ & 1u))) break;
                        tc_fence_after();
                        pv(i, v_at, t > 1);
                        if (more) {
                            if (!early && !(ok = take(k_at, ki))) break;
                            qk(i, 0, k_at);
                        }
                        tc_commit(empty + 8 * vi);
                        if (more) tc_commit(empty + 8 * ki);
                    }
                }
                if (!ok) break;
                tc_commit(o_full);
                segment_done();
            }
        } else if (warp == PLAN_WARP) {
            // -------------------------------------------------------------------------------- this CTA's range of key tiles
            int len, live, np;
            const int n_first = lane < a.S ? places(sequence_tiles(a, lane, len, live, np)) : 0;
            auto scan = [&](int n) {  // inclusive
                long long upto = n;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) {
                    const long long other = __shfl_up_sync(0xffffffffu, upto, o);
                    if (lane >= o) upto += other;
                }
                return upto;
            };
            const long long first_upto = scan(n_first);
            long long sum = 0;
            if (a.S > 32) {
                for (int s = lane + 32; s < a.S; s += 32) sum += places(sequence_tiles(a, s, len, live, np));
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
            }
            const long long per_pass = (sum + __shfl_sync(0xffffffffu, first_upto, 31)) * cache.heads, total = per_pass * p.passes;
            const Ranges ranges(p, total);
            const long long group = min((long long)(blockIdx.x / p.side), ranges.n);
            Walk w;
            w.pos = ranges.begin(group);
            w.hi = group < ranges.n ? ranges.begin(group + 1) : w.pos;
            w.pass = p.passes > 1 && per_pass ? (int)quotient(w.pos, per_pass) : 0;
            w.slot = 0;
            const long long x = w.pos - w.pass * per_pass;  // < per_pass
            int mine = 0;  // the lane whose sequence the range starts in has its place
            long long before = 0;
            for (int s0 = 0; s0 < a.S; s0 += 32) {
                const int s = s0 + lane;
                const int n = s0 == 0 ? n_first : (s < a.S ? places(sequence_tiles(a, s, len, live, np)) : 0);
                const long long upto = before + (s0 == 0 ? first_upto : scan(n));
                const long long from = (upto - n) * cache.heads;
                if (n > 0 && x >= from && x < upto * cache.heads) {
                    mine = 1;
                    w.s = s;
                    w.h = (int)quotient(x - from, n);
                    w.t = (int)(x - from - (long long)w.h * n);
                }
                before = __shfl_sync(0xffffffffu, upto, 31);
                if (before * cache.heads > x) break;
            }
            const unsigned who = __ballot_sync(0xffffffffu, mine);
            const int src = who ? __ffs(who) - 1 : 0;
            const int first_pass = w.pass;
            w.s = __shfl_sync(0xffffffffu, w.s, src);
            w.h = __shfl_sync(0xffffffffu, w.h, src);
            w.t = __shfl_sync(0xffffffffu, w.t, src);
            const int s = w.s, h = w.h, t = w.t;
            const long long u0 = w.pos - t;  // the first place of the (s, h)
            const bool inside = w.pos < w.hi && t > START;  // an (s, h) has tiles before this range
            int known_s = -1, known_qt = -1;
            uint32_t known = 0;  // tiles of the block that some node of the known rows attends to
            for (uint32_t k = 0;; ++k) {
                if (!__all_sync(0xffffffffu, wait(seg_empty + 8 * (k % SEGMENTS), ((k / SEGMENTS) & 1u) ^ 1u))) break;
                Segment& g = sh.segment[k % SEGMENTS];
                if (lane == 0) advance<Q8>(p, w, g);
                __syncwarp();
                const int n_pre = g.n_prefix, from = max(g.t0 - n_pre, 0), to = g.t1 - n_pre;
                if (g.more && to > 0) {
                    if (a.N > TILE && (g.s != known_s || g.qt != known_qt)) {  // (consecutive key heads see the same bits)
                        known_s = g.s;
                        known_qt = g.qt;
                        known = block_tiles(p, g, lane);
                    }
                    uint32_t live_tiles = (a.N > TILE ? known : 1u) & (0xFFFFFFFFu << from);
                    if (to < 32) live_tiles &= (1u << to) - 1u;
                    if (live_tiles == 0 && g.t0 >= n_pre) live_tiles = 1u << from;  // one tile there has to be
                    __syncwarp();
                    if (lane == 0) {  // from the first to the last of them
                        const int first = live_tiles ? __ffs(live_tiles) - 1 : from;
                        g.first = n_pre + from - first;
                        g.t1 = max(g.t0, n_pre) + (live_tiles ? 32 - __clz(live_tiles) - first : 0);
                    }
                }
                const int more = g.more;
                __syncwarp();
                if (lane == 0) mbar_arrive(seg_full + 8 * (k % SEGMENTS));
                if (!more) break;
            }
            if (lane == 0) {
                JoinTask task = {s, h, first_pass * p.side + (int)(blockIdx.x % p.side), 0, 0, 0, {0, 0}};
                if (inside && u0 + START >= ranges.begin(group - 1) && task.qt < p.n_qtiles) {
                    const int n = places(sequence_tiles(a, s, len, live, np));
                    task.rows = min(2 * TILE, live * p.G - task.qt * 2 * TILE);
                    task.n = task.rows > 0 ? (int)(ranges.group_of(u0 + n - 1) - group) + 2 : 0;
                    task.first = u0 > ranges.begin(group - 1);  // that range begins with another (s, h)
                }
                p.tasks[blockIdx.x] = task;
            }
        } else if (warp == BLANK_WARP) {
            // -------------------------------------------------------------------------------- nodes that are not live
            const long long n_nodes = (long long)a.S * a.N;
            for (long long i0 = 32ll * blockIdx.x; i0 < n_nodes; i0 += 32ll * gridDim.x) {
                const long long i = i0 + lane;
                bool blank = false;
                if (i < n_nodes) {
                    const int s = (int)quotient(i, a.N), node = (int)(i - (long long)s * a.N);
                    int len, live, np;
                    sequence_tiles(a, s, len, live, np);
                    blank = node >= live;
                    if (node == 0 && (a.len[s] < 0 || (long long)a.len[s] > ((long long)cache.max_pages << cache.page_shift)))
                        atomicOr(a.status, SPEC_STATUS_CAPACITY);
                }
                for (unsigned left = __ballot_sync(0xffffffffu, blank); left; left &= left - 1) {
                    const long long at = (i0 + __ffs(left) - 1) * a.Hq;
                    uint4* out = reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + at * D);
                    for (int j = lane; j < a.Hq * (D / 8); j += 32) out[j] = make_uint4(0, 0, 0, 0);
                    if (a.lse)
                        for (int j = lane; j < a.Hq; j += 32) a.lse[at + j] = -INFINITY;
                }
            }
        }
    }
    tc_fence_before();
    __syncthreads();
    if (*abort_flag) {
        if (threadIdx.x == 0) atomicOr(a.status, SPEC_STATUS_TIMEOUT);
        let_copies_land();
    }
    if (warp == MMA_WARP) tmem_dealloc(tmem, 512);
}

// Joins the partial rows of every (s, h, row-tile pair) whose key tiles were spread over several CTAs, in an order that
// only their number decides.  16 columns per warp; a lane per row, and with 16 rows or fewer several lanes per row, which
// share the parts (one token of 32 heads, 4095 keys: 18 parts for each of 8 key heads; the call 17.4 -> 14.3 us).  It is
// a chain of memory latencies (the record, a round of parts, the output): the loads of 4 parts are in flight (8: fewer
// warps to an SM, slower).
constexpr int JOIN_DEPTH = 4;
template <int D>
__global__ void __launch_bounds__(2 * D) join_kernel(const __grid_constant__ AttParams p) {
    const TreeAttnArgs& a = p.a;
    const int lane = threadIdx.x & 31, cols = threadIdx.x >> 5;  // columns [16 cols, 16 cols + 16)
    grid_launch_dependents();
    grid_dependency_wait();
    const int cta = p.side + blockIdx.x, r0 = blockIdx.y * 32;
    const JoinTask task = p.tasks[cta];
    const int n = task.n, rows = min(task.rows - r0, 32);
    if (n == 0 || rows <= 0) return;
    const int bits = rows > 16 ? 5 : (rows > 8 ? 4 : (rows > 4 ? 3 : 2)), lanes = 1 << bits, sharers = 32 >> bits;  // lanes: for distinct rows
    const int r = r0 + min(lane & (lanes - 1), rows - 1), mine = lane >> bits;
    const int R = task.qt * 2 * TILE + r, node = R / p.G, gq = R - node * p.G;
    const long long out_row = ((long long)task.s * a.N + node) * a.Hq + task.h * p.G + gq;
    uint4* out = reinterpret_cast<uint4*>((__nv_bfloat16*)a.out + out_row * D + 16 * cols);
    const long long at0 = 2ll * (cta - p.side) + task.first, at1 = 2ll * cta;
    auto part = [&](int i) { return i == 0 ? at0 : at1 + (long long)(i - 1) * p.side * 2; };
    float m = -INFINITY, l = 0.0f, x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = 0.0f;
    for (int i0 = mine; i0 < n; i0 += JOIN_DEPTH * sharers) {
        float2 ml[JOIN_DEPTH];
        float4 o[JOIN_DEPTH][4];
#pragma unroll
        for (int i = 0; i < JOIN_DEPTH; ++i) {
            if (i0 + i * sharers >= n) continue;
            const long long at = part(i0 + i * sharers);
            ml[i] = p.part_ml[at * p.rows_cap + r];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[i][j] = reinterpret_cast<const float4*>(p.part_o)[(at * (D / 4) + 4 * cols + j) * p.rows_cap + r];
        }
#pragma unroll
        for (int i = 0; i < JOIN_DEPTH; ++i) {
            if (i0 + i * sharers >= n) continue;
            const float top = fmaxf(m, ml[i].x), f0 = m == -INFINITY ? 0.0f : exp2f((m - top) * p.c), f = ml[i].x == -INFINITY ? 0.0f : exp2f((ml[i].x - top) * p.c);
            m = top;
            l = l * f0 + ml[i].y * f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                x[4 * j] = x[4 * j] * f0 + o[i][j].x * f;
                x[4 * j + 1] = x[4 * j + 1] * f0 + o[i][j].y * f;
                x[4 * j + 2] = x[4 * j + 2] * f0 + o[i][j].z * f;
                x[4 * j + 3] = x[4 * j + 3] * f0 + o[i][j].w * f;
            }
        }
    }
    __syncwarp();
    for (int d = lanes; d < 32; d <<= 1) {
        const float m1 = __shfl_xor_sync(0xffffffffu, m, d), top = fmaxf(m, m1);
        const float f0 = m == -INFINITY ? 0.0f : exp2f((m - top) * p.c), f1 = m1 == -INFINITY ? 0.0f : exp2f((m1 - top) * p.c);
        m = top;
        l = l * f0 + __shfl_xor_sync(0xffffffffu, l, d) * f1;
#pragma unroll
        for (int j = 0; j < 16; ++j) x[j] = x[j] * f0 + __shfl_xor_sync(0xffffffffu, x[j], d) * f1;
    }
    if (lane >= rows) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int j = 0; j < 2; ++j)
        out[j] = make_uint4(pack2(x[8 * j] * inv, x[8 * j + 1] * inv), pack2(x[8 * j + 2] * inv, x[8 * j + 3] * inv),
                            pack2(x[8 * j + 4] * inv, x[8 * j + 5] * inv), pack2(x[8 * j + 6] * inv, x[8 * j + 7] * inv));
    if (a.lse && cols == 0) a.lse[out_row] = l == 0.0f ? -INFINITY : (m * p.c + log2f(l)) * LN2;
}

// ------------------------------------------------------------------------------------------ host
static void plan(int num_sms, int S, int N, int Hq, int heads, int head_dim, AttParams& p, size_t& bytes) {
    p.G = Hq / heads;
    const int rows = N * p.G;
    p.n_qtiles = (rows + 2 * TILE - 1) / (2 * TILE);
    p.side = std::min(p.n_qtiles, num_sms);
    p.n_groups = num_sms / p.side;
    p.passes = (p.n_qtiles + p.side - 1) / p.side;
    p.rows_cap = std::min(2 * TILE, rows);
    const size_t parts = (size_t)p.n_groups * p.side * 2 * p.rows_cap;
    const size_t tasks = (size_t)p.n_groups * p.side * sizeof(JoinTask);
    p.tasks = nullptr;
    p.part_o = reinterpret_cast<float*>(tasks);
    p.part_ml = reinterpret_cast<float2*>(tasks + parts * head_dim * 4);
    bytes = tasks + parts * (head_dim * 4 + 8);
}

size_t tree_attention_bytes(int num_sms, int S, int N, int Hq, int heads, int head_dim) {
    AttParams p;
    size_t bytes;
    plan(num_sms, S, N, Hq, heads, head_dim, p, bytes);
    return bytes;
}

// The cache as rows of one vector: [n_pages * heads * page, D], a page and 128 bytes (E4M3: a whole vector) at a time.
static int cache_map(spec_ctx* ctx, CUtensorMap* tm, const void* base, const CacheArgs& c) {
    const int elem = c.quantised ? 1 : 2;
    cuuint64_t dims[2] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.n_pages * c.heads << c.page_shift};
    cuuint64_t strides[1] = {(cuuint64_t)c.head_dim * elem};
    cuuint32_t box[2] = {(cuuint32_t)(c.quantised ? c.head_dim : 64), 1u << c.page_shift};
    cuuint32_t estr[2] = {1u, 1u};
    CUresult r = ctx->encode(tm, c.quantised ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(base), dims,
                             strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, c.quantised ? CU_TENSOR_MAP_SWIZZLE_NONE : CU_TENSOR_MAP_SWIZZLE_128B,
                             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(ctx, SPEC_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return SPEC_OK;
}

// Keys or values of the block, [S * N, heads, D] strided, 128 nodes of a head and 128 bytes at a time.
static int block_map(spec_ctx* ctx, CUtensorMap* tm, const void* base, long long tok, long long head, const TreeAttnArgs& a) {
    const CacheArgs& c = a.cache;
    cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.heads, (cuuint64_t)a.S * a.N};
    // (the stride of a dimension of one is never used, but has to be a valid one)
    cuuint64_t strides[2] = {(cuuint64_t)(c.heads > 1 ? head : c.head_dim) * 2, (cuuint64_t)((long long)a.S * a.N > 1 ? tok : (long long)c.heads * c.head_dim) * 2};
    cuuint32_t box[3] = {64u, 1u, (cuuint32_t)TILE};
    cuuint32_t estr[3] = {1u, 1u, 1u};
    CUresult r = ctx->encode(tm, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
                             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    if (r != CUDA_SUCCESS) return fail(ctx, SPEC_ERR_CUDA, "cuTensorMapEncodeTiled failed with code %d", (int)r);
    return SPEC_OK;
}

template <int D, bool Q8>
static int launch(spec_ctx* ctx, const AttParams& p, cudaStream_t st) {
    auto kernel = tree_attention_kernel<D, Q8>;
    {
        static bool done[64] = {false};
        std::lock_guard<std::mutex> lock(host_mutex());
        bool& d = done[ctx->device & 63];
        if (!d) {
            cudaFuncAttributes attr;
            int rc = check_cuda(ctx, cudaFuncGetAttributes(&attr, kernel), "spec_tree_attention: cudaFuncGetAttributes");
            if (rc) return rc;
            if (attr.numRegs < LAUNCH_REGS)  // the warpgroups would wait for registers for ever
                return fail(ctx, SPEC_ERR_UNSUPPORTED, "spec_tree_attention: built with %d registers per thread", attr.numRegs);
            if ((rc = check_cuda(ctx, cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, Geometry<D, Q8>::SMEM),
                                 "spec_tree_attention: cudaFuncSetAttribute")))
                return rc;
            d = true;
        }
    }
    CUtensorMap tm_k, tm_v, tm_bk, tm_bv;
    int rc = cache_map(ctx, &tm_k, p.a.cache.k, p.a.cache);
    if (rc || (rc = cache_map(ctx, &tm_v, p.a.cache.v, p.a.cache)) || (rc = block_map(ctx, &tm_bk, p.a.k, p.a.k_tok, p.a.k_head, p.a)) ||
        (rc = block_map(ctx, &tm_bv, p.a.v, p.a.v_tok, p.a.v_head, p.a)))
        return rc;
    cudaError_t e = launch_pdl(kernel, dim3(p.n_groups * p.side), dim3(ATT_THREADS), (size_t)Geometry<D, Q8>::SMEM, st, tm_k, tm_v, tm_bk, tm_bv, p);
    if ((rc = check_cuda(ctx, e, "spec_tree_attention launch"))) return rc;
    ++ctx->launches;
    if (p.n_groups == 1) return SPEC_OK;  // nothing is spread
    e = launch_pdl(join_kernel<D>, dim3((p.n_groups - 1) * p.side, (p.rows_cap + 31) / 32), dim3(2 * D), 0, st, p);
    ++ctx->launches;
    return check_cuda(ctx, e, "spec_tree_attention join launch");
}

int launch_tree_attention(spec_ctx* ctx, const TreeAttnArgs& a, cudaStream_t st) {
    AttParams p;
    size_t bytes;
    plan(ctx->num_sms, a.S, a.N, a.Hq, a.cache.heads, a.cache.head_dim, p, bytes);
    p.a = a;
    p.c = a.scale * LOG2E;
    p.tasks = reinterpret_cast<JoinTask*>(a.work);
    p.part_o = reinterpret_cast<float*>((char*)a.work + (size_t)p.part_o);
    p.part_ml = reinterpret_cast<float2*>((char*)a.work + (size_t)p.part_ml);
    p.wait_limit_ns = ctx->wait_limit_ns;
    if (a.cache.quantised) return a.cache.head_dim == 64 ? launch<64, true>(ctx, p, st) : launch<128, true>(ctx, p, st);
    return a.cache.head_dim == 64 ? launch<64, false>(ctx, p, st) : launch<128, false>(ctx, p, st);
}

}  // namespace ngs
