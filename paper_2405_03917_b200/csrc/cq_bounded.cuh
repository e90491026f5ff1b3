// Operators that keep a coded cache within bounds (sm_100a): attention with a sliding window, attention over pages,
// masses of cached tokens.  What their kernels share: where a sequence's codes and queries are, and which tokens a query sees.
#pragma once

#include "cq_common.cuh"

namespace cq {

// Division of block numbers by the blocks of a page: floor(x / d) = floor(x ceil(2^64 / d) / 2^64) for x d < 2^64.
struct PageDiv {
    uint64_t inverse = 0;             // 0: d = 1
    void set(int d) { inverse = d > 1 ? ~(uint64_t)0 / (uint64_t)d + 1 : 0; }
#ifdef __CUDACC__
    __device__ __forceinline__ int quotient(int x) const { return inverse ? (int)__umul64hi((uint64_t)x, inverse) : x; }
#endif
};

// One call.  sh.max_tokens is the capacity of a sequence, sh.n_blocks its code blocks.  The codes of a contiguous cache are
// read as pages of the whole capacity, page s being sequence s (page_table null).
struct BoundedArgs {
    Shape sh;
    const __half* q;                  // [n_rows][n_q_heads][head_dim]
    const uint8_t *kc, *vc;
    const __half *kcb, *vcb;          // [n_kv_heads][G][2^b][c]
    const int32_t* seq_lens;
    const int32_t* q_offsets;         // null: max_q rows per sequence
    const int32_t* page_table;        // [n_seq][pages_per_seq]
    int64_t n_pages;
    int pages_per_seq, page_blocks;
    PageDiv page_div;
    int n_rows, max_q;
    int window, sinks;                // window 0: every token up to the query's
    float scale_log2e;
    __half* out;                      // [n_rows][n_q_heads][head_dim]
    int least_rows, most_rows;        // sequences with rows (new tokens x R) outside of this range belong to another kernel
};

#ifdef __CUDACC__
namespace {

// Sequence s: its context length, its first row of q and its new tokens.
struct SeqView {
    int n, row0, m;
};
__device__ __forceinline__ SeqView seq_view(const BoundedArgs& a, int s)
{
    SeqView v;
    const int64_t n = a.seq_lens[s];
    v.n = (int)(n < 0 ? 0 : (n > a.sh.max_tokens ? a.sh.max_tokens : n));
    if (a.q_offsets) {
        int lo = a.q_offsets[s], hi = a.q_offsets[s + 1];
        lo = lo < 0 ? 0 : (lo > a.n_rows ? a.n_rows : lo);
        hi = hi < lo ? lo : (hi > a.n_rows ? a.n_rows : hi);
        v.row0 = lo;
        v.m = hi - lo > a.max_q ? a.max_q : hi - lo;
    } else {
        v.row0 = s * a.max_q;
        v.m = a.max_q;
    }
    return v;
}

// Page that block blk of sequence s lies in (contiguous caches: s itself); -1 where the page table names none.
__device__ __forceinline__ int page_index(const BoundedArgs& a, int s, int blk)
{
    if (!a.page_table) return s;
    const int page = a.page_table[(int64_t)s * a.pages_per_seq + a.page_div.quotient(blk)];
    return page >= 0 && page < a.n_pages ? page : -1;
}
// Byte offset of block blk of head h, which lies in this page.
__device__ __forceinline__ int64_t page_block_offset(const BoundedArgs& a, int page, int h, int blk)
{
    if (a.page_table) blk -= a.page_div.quotient(blk) * a.page_blocks;
    return (((int64_t)page * a.sh.n_kv_heads + h) * a.page_blocks + blk) * (int64_t)a.sh.block_bytes;
}
// The two in one; -1 without a page.
__device__ __forceinline__ int64_t block_offset(const BoundedArgs& a, int s, int h, int blk)
{
    const int page = page_index(a, s, blk);
    return page < 0 ? -1 : page_block_offset(a, page, h, blk);
}

__device__ __forceinline__ bool token_visible(int t, int pos, int window, int sinks)
{
    return t <= pos && (window == 0 || t < sinks || t > pos - window);
}
// What queries are multiplied by ahead of the products, so that the scores' factor can be positive: the sign of the scale (1 and -1 are exact), zero
// for a scale of zero (a query that is no number, or infinite, stays visible: NaN).
__device__ __forceinline__ __half2 query_sign(float scale) { return __float2half2_rn(scale < 0.f ? -1.f : scale == 0.f ? 0.f : 1.f); }
__device__ __forceinline__ uint32_t signed_query(uint32_t two, __half2 sign)
{
    const __half2 x = __hmul2(*reinterpret_cast<const __half2*>(&two), sign);
    return *reinterpret_cast<const uint32_t*>(&x);
}
// First token of the window of a query at pos (0 without a window).
__device__ __forceinline__ int window_first(int pos, int window) { return window == 0 || pos < window ? 0 : pos - window + 1; }

}  // namespace
#endif

// plain kernels, any shape (cq_bounded_plain.cu)
cudaError_t launch_bounded_plain(const BoundedArgs& a, cudaStream_t st);
cudaError_t launch_mass_plain(const BoundedArgs& a, const float* mass_in, float* mass_out, float* lse, cudaStream_t st);
// codes of n_rows new tokens, laid out as one sequence of n_rows tokens, to the pages of their sequences
cudaError_t launch_codes_to_pages(const BoundedArgs& a, const uint8_t* k_staged, const uint8_t* v_staged, uint8_t* k_pages, uint8_t* v_pages,
                                  cudaStream_t st);

// few rows per sequence (cq_gather_attn.cu): head_dim 128, one byte per code, c = 2, 4 or 8
bool gather_attn_supported(const Shape& sh);
size_t gather_attn_workspace_bytes();
cudaError_t launch_gather_attn(const BoundedArgs& a, void* workspace, cudaStream_t st);
// the masses with the same scores (uniform rows, a contiguous cache, no window); the same shapes
size_t gather_mass_workspace_bytes(const BoundedArgs& a);
size_t gather_mass_least_bytes(const BoundedArgs& a);      // what it cannot do without
cudaError_t launch_gather_mass(const BoundedArgs& a, const float* mass_in, float* mass_out, void* workspace, size_t workspace_bytes, cudaStream_t st);

// many rows per sequence (cq_chunk_attn.cu): the tensor-core kernel of the prefill attention in its bounded form
bool chunk_attn_supported(const Shape& sh);
size_t chunk_attn_workspace_bytes(const BoundedArgs& a);        // (goes by least_rows as well: ask for the arguments of the launch)
cudaError_t launch_chunk_attn(const BoundedArgs& a, void* workspace, size_t workspace_bytes, cudaStream_t st);
// the masses that they give (uniform rows, a contiguous cache, no window)
size_t chunk_mass_workspace_bytes(const BoundedArgs& a);
cudaError_t launch_chunk_mass(const BoundedArgs& a, const float* mass_in, float* mass_out, void* workspace, cudaStream_t st);

// the heaviest tokens of a cache to the front of another (cq_evict.cu)
struct EvictArgs {
    Shape sh;                          // the cache that is read; n_q_heads == n_kv_heads
    const float* mass;
    const uint8_t *kc, *vc;
    const int32_t* seq_lens;
    int n_keep, n_sinks, n_recent;
    int64_t out_tokens;                // capacity of the cache that is written
    uint8_t *k_out, *v_out;
    float* mass_out;
    int32_t *kept, *lens_out;
};
cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st);

}  // namespace cq
