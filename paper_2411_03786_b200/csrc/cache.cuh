// The paged key/value cache and rotary positions as the kernels see them.
#pragma once
#include "common.cuh"

namespace ngs {

constexpr int E8_MIN = -120, E8_MAX = 7;  // exponents of a vector's scale
constexpr int kMaxNodes = 4096;           // nodes of a sequence's draft block

struct CacheArgs {
    void *k, *v;             // [n_pages, heads, page, D] bf16 or E4M3 codes
    uint8_t *k_exp, *v_exp;  // [n_pages, heads, page] exponent + 127 of the vector's scale
    const int32_t* table;    // [S, max_pages]
    int n_pages, max_pages, page_shift, heads, head_dim, quantised;
};

struct RopeArgs {
    const float* freq;  // [rot / 2] radians per position
    int rot, interleaved;
    float factor;
};

int launch_rope_rows(spec_ctx* ctx, const RopeArgs& rope, const void* d_q, int Hq, long long q_tok, long long q_head, void* d_q_out,
                     const void* d_k, int Hkv, long long k_tok, long long k_head, void* d_k_out, int D, const int32_t* d_pos, int T,
                     cudaStream_t st);
int launch_cache_write(spec_ctx* ctx, const CacheArgs& c, const void* d_k, long long k_tok, long long k_head, const void* d_v,
                       long long v_tok, long long v_head, int S, int N, int n, const int32_t* d_nodes, const int32_t* d_start,
                       const int32_t* d_count, const RopeArgs& rope, cudaStream_t st);
int launch_cache_read(spec_ctx* ctx, const CacheArgs& c, int S, int n, const int32_t* d_start, const int32_t* d_count, void* d_k_out,
                      void* d_v_out, cudaStream_t st);
int launch_tree_mask(spec_ctx* ctx, const int32_t* d_parent, int S, int N, const int32_t* d_n_nodes, int32_t* d_mask, int32_t* d_depth,
                     cudaStream_t st);

// tree_attention.cu
struct TreeAttnArgs {
    CacheArgs cache;
    const void *q, *k, *v;  // block of drafted nodes, bf16
    long long q_tok, q_head, k_tok, k_head, v_tok, v_head;
    int S, N, Hq;
    const int32_t* mask;     // [S, N, ceil(N / 32)]
    const int32_t* len;      // [S]
    const int32_t* n_nodes;  // [S] or null
    float scale;
    void* out;   // [S, N, Hq, D] bf16
    float* lse;  // [S, N, Hq] or null
    void* work;
    int* status;
};
size_t tree_attention_bytes(int num_sms, int S, int N, int Hq, int heads, int head_dim);
int launch_tree_attention(spec_ctx* ctx, const TreeAttnArgs& a, cudaStream_t st);

}  // namespace ngs
