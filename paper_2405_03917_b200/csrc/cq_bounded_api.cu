// extern "C" entry points of the operators on bounded caches (window, pages, masses, eviction): host-side validation and
// dispatch only.
#include <limits.h>

#include "cq_bounded.cuh"

using namespace cq;

namespace {

constexpr int64_t kMostTokens = (int64_t)1 << 30;        // positions are 32-bit in these kernels
constexpr int64_t kMostRows = (int64_t)1 << 30;          // rows x query heads of a call

constexpr int kFewRows = 16;                             // rows (new tokens x R) of a sequence up to which it takes the gather kernel

// What a call shares: the quantiser, the cache, and how many new tokens a sequence may have.
int bounded_shape(int64_t n_seq, int64_t n_rows, int max_q, int64_t max_tokens, int n_q_heads, int n_kv_heads, int head_dim, int c, int b,
                  int64_t window, int64_t n_sinks, BoundedArgs* a)
{
    *a = BoundedArgs();
    const int st = make_shape(n_seq, max_tokens, n_q_heads, n_kv_heads, head_dim, c, b, &a->sh);
    if (st != CQ_OK) return st;
    if (max_q <= 0 || max_q > max_tokens || n_rows < 0 || window < 0 || n_sinks < 0) return CQ_ERR_SHAPE;
    if (max_tokens > kMostTokens || n_rows * n_q_heads > kMostRows || n_rows > INT_MAX || n_seq * (int64_t)max_q * n_q_heads > kMostRows)
        return CQ_ERR_UNSUPPORTED;
    a->n_rows = (int)n_rows;
    a->max_q = max_q;
    a->window = window >= max_tokens ? 0 : (int)window;                      // (no query is further on than the capacity)
    a->sinks = a->window == 0 ? 0 : (int)(n_sinks < max_tokens ? n_sinks : max_tokens);
    a->n_pages = n_seq;
    a->pages_per_seq = 1;
    a->page_blocks = (int)a->sh.n_blocks;
    a->least_rows = 0;
    a->most_rows = INT_MAX;
    return CQ_OK;
}

int paged_shape(int64_t n_seq, int64_t n_rows, int max_q, int n_q_heads, int n_kv_heads, int head_dim, int c, int b, int64_t n_pages,
                int64_t page_tokens, int64_t pages_per_seq, int64_t window, int64_t n_sinks, BoundedArgs* a)
{
    if (n_pages <= 0 || page_tokens <= 0 || pages_per_seq <= 0 || page_tokens % kTokenBlock != 0) return CQ_ERR_SHAPE;
    if (page_tokens > kMostTokens || pages_per_seq > kMostTokens || n_pages > INT_MAX) return CQ_ERR_UNSUPPORTED;
    const int st = bounded_shape(n_seq, n_rows, max_q, page_tokens * pages_per_seq, n_q_heads, n_kv_heads, head_dim, c, b, window, n_sinks, a);
    if (st != CQ_OK) return st;
    a->n_pages = n_pages;
    a->pages_per_seq = (int)pages_per_seq;
    a->page_blocks = (int)(page_tokens / kTokenBlock);
    a->page_div.set(a->page_blocks);
    return CQ_OK;
}

struct Extent {
    const void* first;
    size_t bytes;
};
bool overlap(const Extent& a, const Extent& b)
{
    const uintptr_t x = reinterpret_cast<uintptr_t>(a.first), y = reinterpret_cast<uintptr_t>(b.first);
    return x < y + b.bytes && y < x + a.bytes;
}

bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
int status(cudaError_t e) { return e == cudaSuccess ? CQ_OK : CQ_ERR_CUDA; }

// What of a ragged batch is the tensor-core kernel's beside the gather kernel: the sequences with more rows than that takes.  Its plan goes by
// this (fewer row tiles leave more CTAs for each), so the workspace is asked for, checked and laid out for the same arguments.
BoundedArgs many_rows(BoundedArgs a)
{
    a.least_rows = kFewRows + 1;
    return a;
}

int run_attn(BoundedArgs a, int variant, void* workspace, size_t workspace_bytes, cudaStream_t st)
{
    if (variant < 0 || variant > 3) return CQ_ERR_SHAPE;
    const bool gather = gather_attn_supported(a.sh), chunk = chunk_attn_supported(a.sh);
    if ((variant == 2 && !gather) || (variant == 3 && !chunk)) return CQ_ERR_UNSUPPORTED;
    if (a.n_rows == 0) return CQ_OK;
    if (variant == 2) return status(launch_gather_attn(a, workspace, st));
    if (variant == 3) return status(launch_chunk_attn(a, workspace, workspace_bytes, st));
    if (variant == 1 || !gather || !chunk) return status(launch_bounded_plain(a, st));
    // every sequence takes the kernel of its number of rows; without ragged rows that is the same one for all
    if ((int64_t)a.max_q * a.sh.R <= kFewRows) return status(launch_gather_attn(a, workspace, st));
    if (a.q_offsets) {
        BoundedArgs few = a;
        few.most_rows = kFewRows;
        const cudaError_t e = launch_gather_attn(few, workspace, st);
        if (e != cudaSuccess) return CQ_ERR_CUDA;
        a = many_rows(a);
    }
    return status(launch_chunk_attn(a, workspace, workspace_bytes, st));
}
size_t attn_workspace(const BoundedArgs& a, bool ragged)
{
    size_t bytes = 256;                                                        // enough for every kernel that the shape has
    auto room_for = [&](size_t need) { bytes = need > bytes ? need : bytes; };
    if (gather_attn_supported(a.sh)) room_for(gather_attn_workspace_bytes());
    if (chunk_attn_supported(a.sh)) {
        room_for(chunk_attn_workspace_bytes(a));
        if (ragged) room_for(chunk_attn_workspace_bytes(many_rows(a)));
    }
    return bytes;
}

}  // namespace

extern "C" {

size_t cq_window_attn_workspace_bytes(int n_seq, int n_q_tokens, int n_q_heads, int n_kv_heads, int head_dim, int c, int b,
                                      int64_t max_tokens, int64_t window, int64_t n_sinks)
{
    BoundedArgs a;
    if (bounded_shape(n_seq, (int64_t)n_seq * n_q_tokens, n_q_tokens, max_tokens, n_q_heads, n_kv_heads, head_dim, c, b, window, n_sinks, &a) != CQ_OK)
        return 0;
    return attn_workspace(a, false);
}

int cq_window_attn_variant(const void* q_fp16, const void* k_codes, const void* v_codes, const void* k_cb_fp16, const void* v_cb_fp16,
                           const int32_t* seq_lens, float scale, int64_t window, int64_t n_sinks, int n_seq, int n_q_tokens, int n_q_heads,
                           int n_kv_heads, int head_dim, int c, int b, int64_t max_tokens, void* out_fp16, void* workspace,
                           size_t workspace_bytes, int variant, void* stream)
{
    if (!q_fp16 || !k_codes || !v_codes || !k_cb_fp16 || !v_cb_fp16 || !seq_lens || !out_fp16 || !workspace) return CQ_ERR_NULL;
    BoundedArgs a;
    const int st = bounded_shape(n_seq, (int64_t)n_seq * n_q_tokens, n_q_tokens, max_tokens, n_q_heads, n_kv_heads, head_dim, c, b, window, n_sinks, &a);
    if (st != CQ_OK) return st;
    if (!aligned16(q_fp16) || !aligned16(k_codes) || !aligned16(v_codes) || !aligned16(k_cb_fp16) || !aligned16(v_cb_fp16) ||
        !aligned16(out_fp16) || !aligned16(workspace) || !aligned4(seq_lens))
        return CQ_ERR_ALIGN;
    if (workspace_bytes < attn_workspace(a, false)) return CQ_ERR_WORKSPACE;
    a.q = static_cast<const __half*>(q_fp16);
    a.kc = static_cast<const uint8_t*>(k_codes);
    a.vc = static_cast<const uint8_t*>(v_codes);
    a.kcb = static_cast<const __half*>(k_cb_fp16);
    a.vcb = static_cast<const __half*>(v_cb_fp16);
    a.seq_lens = seq_lens;
    a.scale_log2e = scale * kLog2e;
    a.out = static_cast<__half*>(out_fp16);
    return run_attn(a, variant, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int cq_window_attn(const void* q_fp16, const void* k_codes, const void* v_codes, const void* k_cb_fp16, const void* v_cb_fp16,
                   const int32_t* seq_lens, float scale, int64_t window, int64_t n_sinks, int n_seq, int n_q_tokens, int n_q_heads,
                   int n_kv_heads, int head_dim, int c, int b, int64_t max_tokens, void* out_fp16, void* workspace, size_t workspace_bytes,
                   void* stream)
{
    return cq_window_attn_variant(q_fp16, k_codes, v_codes, k_cb_fp16, v_cb_fp16, seq_lens, scale, window, n_sinks, n_seq, n_q_tokens, n_q_heads,
                                  n_kv_heads, head_dim, c, b, max_tokens, out_fp16, workspace, workspace_bytes, 0, stream);
}

size_t cq_paged_attn_workspace_bytes(int n_seq, int64_t n_rows, int max_q, int n_q_heads, int n_kv_heads, int head_dim, int c, int b,
                                     int64_t page_tokens, int64_t pages_per_seq, int64_t window, int64_t n_sinks)
{
    BoundedArgs a;
    if (paged_shape(n_seq, n_rows, max_q, n_q_heads, n_kv_heads, head_dim, c, b, 1, page_tokens, pages_per_seq, window, n_sinks, &a) != CQ_OK) return 0;
    return attn_workspace(a, true);
}

int cq_paged_attn_variant(const void* q_fp16, const int32_t* q_offsets, const void* k_pages, const void* v_pages, const void* k_cb_fp16,
                          const void* v_cb_fp16, const int32_t* page_table, const int32_t* seq_lens, float scale, int64_t window,
                          int64_t n_sinks, int n_seq, int64_t n_rows, int max_q, int n_q_heads, int n_kv_heads, int head_dim, int c, int b,
                          int64_t n_pages, int64_t page_tokens, int64_t pages_per_seq, void* out_fp16, void* workspace,
                          size_t workspace_bytes, int variant, void* stream)
{
    if (!q_fp16 || !q_offsets || !k_pages || !v_pages || !k_cb_fp16 || !v_cb_fp16 || !page_table || !seq_lens || !out_fp16 || !workspace)
        return CQ_ERR_NULL;
    BoundedArgs a;
    const int st = paged_shape(n_seq, n_rows, max_q, n_q_heads, n_kv_heads, head_dim, c, b, n_pages, page_tokens, pages_per_seq, window, n_sinks, &a);
    if (st != CQ_OK) return st;
    if (!aligned16(q_fp16) || !aligned16(k_pages) || !aligned16(v_pages) || !aligned16(k_cb_fp16) || !aligned16(v_cb_fp16) ||
        !aligned16(out_fp16) || !aligned16(workspace) || !aligned4(seq_lens) || !aligned4(q_offsets) || !aligned4(page_table))
        return CQ_ERR_ALIGN;
    if (workspace_bytes < attn_workspace(a, true)) return CQ_ERR_WORKSPACE;
    a.q = static_cast<const __half*>(q_fp16);
    a.kc = static_cast<const uint8_t*>(k_pages);
    a.vc = static_cast<const uint8_t*>(v_pages);
    a.kcb = static_cast<const __half*>(k_cb_fp16);
    a.vcb = static_cast<const __half*>(v_cb_fp16);
    a.seq_lens = seq_lens;
    a.q_offsets = q_offsets;
    a.page_table = page_table;
    a.scale_log2e = scale * kLog2e;
    a.out = static_cast<__half*>(out_fp16);
    return run_attn(a, variant, workspace, workspace_bytes, static_cast<cudaStream_t>(stream));
}

int cq_paged_attn(const void* q_fp16, const int32_t* q_offsets, const void* k_pages, const void* v_pages, const void* k_cb_fp16,
                  const void* v_cb_fp16, const int32_t* page_table, const int32_t* seq_lens, float scale, int64_t window, int64_t n_sinks,
                  int n_seq, int64_t n_rows, int max_q, int n_q_heads, int n_kv_heads, int head_dim, int c, int b, int64_t n_pages,
                  int64_t page_tokens, int64_t pages_per_seq, void* out_fp16, void* workspace, size_t workspace_bytes, void* stream)
{
    return cq_paged_attn_variant(q_fp16, q_offsets, k_pages, v_pages, k_cb_fp16, v_cb_fp16, page_table, seq_lens, scale, window, n_sinks, n_seq, n_rows,
                                 max_q, n_q_heads, n_kv_heads, head_dim, c, b, n_pages, page_tokens, pages_per_seq, out_fp16, workspace,
                                 workspace_bytes, 0, stream);
}

size_t cq_paged_append_workspace_bytes(int64_t n_rows, int n_heads, int head_dim, int c, int b)
{
    return 2 * round_up(cq_codes_bytes(1, n_rows, n_heads, head_dim, c, b), 256);
}

int cq_paged_append(const void* k_fp16, const void* v_fp16, const int32_t* q_offsets, const float* k_cb, const float* v_cb,
                    const int32_t* page_table, const int32_t* seq_lens, int n_seq, int64_t n_rows, int max_q, int n_heads, int head_dim,
                    int c, int b, int64_t n_pages, int64_t page_tokens, int64_t pages_per_seq, void* k_pages, void* v_pages, void* workspace,
                    size_t workspace_bytes, void* stream)
{
    if (!k_fp16 || !v_fp16 || !q_offsets || !k_cb || !v_cb || !page_table || !seq_lens || !k_pages || !v_pages || !workspace) return CQ_ERR_NULL;
    if (k_pages == v_pages) return CQ_ERR_SHAPE;
    BoundedArgs a;
    int st = paged_shape(n_seq, n_rows, max_q, n_heads, n_heads, head_dim, c, b, n_pages, page_tokens, pages_per_seq, 0, 0, &a);
    if (st != CQ_OK) return st;
    if (!aligned16(k_fp16) || !aligned16(v_fp16) || !aligned16(k_cb) || !aligned16(v_cb) || !aligned16(k_pages) || !aligned16(v_pages) ||
        !aligned16(workspace) || !aligned4(q_offsets) || !aligned4(page_table) || !aligned4(seq_lens))
        return CQ_ERR_ALIGN;
    if (n_rows == 0) return CQ_OK;
    if (workspace_bytes < cq_paged_append_workspace_bytes(n_rows, n_heads, head_dim, c, b)) return CQ_ERR_WORKSPACE;
    uint8_t* k_staged = static_cast<uint8_t*>(workspace);
    uint8_t* v_staged = k_staged + round_up(cq_codes_bytes(1, n_rows, n_heads, head_dim, c, b), 256);
    st = cq_encode_kv(k_fp16, v_fp16, k_cb, v_cb, nullptr, 1, n_rows, 0, n_rows, n_heads, head_dim, c, b, k_staged, v_staged, stream);
    if (st != CQ_OK) return st;
    a.seq_lens = seq_lens;
    a.q_offsets = q_offsets;
    a.page_table = page_table;
    return status(launch_codes_to_pages(a, k_staged, v_staged, static_cast<uint8_t*>(k_pages), static_cast<uint8_t*>(v_pages),
                                        static_cast<cudaStream_t>(stream)));
}

namespace {
// Kernel of a call: 1 plain, 2 gather, 3 tensor cores (where the variant leaves it open: by the rows of a sequence).
int mass_kernel(const BoundedArgs& a, int variant)
{
    if (variant != 0) return variant;
    if (!gather_attn_supported(a.sh) || !chunk_attn_supported(a.sh)) return 1;
    return (int64_t)a.max_q * a.sh.R <= kFewRows ? 2 : 3;
}
size_t mass_workspace(const BoundedArgs& a, int kernel, bool least)
{
    if (kernel == 2) return least ? gather_mass_least_bytes(a) : gather_mass_workspace_bytes(a);
    if (kernel == 3) return chunk_mass_workspace_bytes(a);
    return round_up((size_t)a.n_rows * a.sh.n_q_heads * sizeof(float), 256);
}
}  // namespace

size_t cq_attn_mass_workspace_bytes(int n_seq, int n_q_tokens, int n_q_heads, int n_kv_heads, int head_dim, int c, int b, int64_t max_tokens)
{
    BoundedArgs a;
    if (bounded_shape(n_seq, (int64_t)n_seq * n_q_tokens, n_q_tokens, max_tokens, n_q_heads, n_kv_heads, head_dim, c, b, 0, 0, &a) != CQ_OK) return 0;
    size_t bytes = mass_workspace(a, 1, false);                                // enough for every kernel that the shape has
    if (gather_attn_supported(a.sh) && mass_workspace(a, 2, false) > bytes) bytes = mass_workspace(a, 2, false);
    if (chunk_attn_supported(a.sh) && mass_workspace(a, 3, false) > bytes) bytes = mass_workspace(a, 3, false);
    return bytes;
}

int cq_attn_mass_variant(const void* q_fp16, const void* k_codes, const void* k_cb_fp16, const int32_t* seq_lens, float scale,
                         const float* mass_in, int n_seq, int n_q_tokens, int n_q_heads, int n_kv_heads, int head_dim, int c, int b,
                         int64_t max_tokens, float* mass_out, void* workspace, size_t workspace_bytes, int variant, void* stream)
{
    if (!q_fp16 || !k_codes || !k_cb_fp16 || !seq_lens || !mass_out || !workspace) return CQ_ERR_NULL;
    BoundedArgs a;
    const int st = bounded_shape(n_seq, (int64_t)n_seq * n_q_tokens, n_q_tokens, max_tokens, n_q_heads, n_kv_heads, head_dim, c, b, 0, 0, &a);
    if (st != CQ_OK) return st;
    if (!aligned16(q_fp16) || !aligned16(k_codes) || !aligned16(k_cb_fp16) || !aligned16(workspace) || !aligned4(seq_lens) || !aligned4(mass_in) ||
        !aligned4(mass_out))
        return CQ_ERR_ALIGN;
    if (variant < 0 || variant > 3) return CQ_ERR_SHAPE;
    if ((variant == 2 && !gather_attn_supported(a.sh)) || (variant == 3 && !chunk_attn_supported(a.sh))) return CQ_ERR_UNSUPPORTED;
    const int kernel = mass_kernel(a, variant);
    if (workspace_bytes < mass_workspace(a, kernel, true)) return CQ_ERR_WORKSPACE;
    a.q = static_cast<const __half*>(q_fp16);
    a.kc = static_cast<const uint8_t*>(k_codes);
    a.kcb = static_cast<const __half*>(k_cb_fp16);
    a.seq_lens = seq_lens;
    a.scale_log2e = scale * kLog2e;
    if (kernel == 2) return status(launch_gather_mass(a, mass_in, mass_out, workspace, workspace_bytes, static_cast<cudaStream_t>(stream)));
    if (kernel == 3) return status(launch_chunk_mass(a, mass_in, mass_out, workspace, static_cast<cudaStream_t>(stream)));
    return status(launch_mass_plain(a, mass_in, mass_out, static_cast<float*>(workspace), static_cast<cudaStream_t>(stream)));
}

int cq_attn_mass(const void* q_fp16, const void* k_codes, const void* k_cb_fp16, const int32_t* seq_lens, float scale, const float* mass_in,
                 int n_seq, int n_q_tokens, int n_q_heads, int n_kv_heads, int head_dim, int c, int b, int64_t max_tokens, float* mass_out,
                 void* workspace, size_t workspace_bytes, void* stream)
{
    return cq_attn_mass_variant(q_fp16, k_codes, k_cb_fp16, seq_lens, scale, mass_in, n_seq, n_q_tokens, n_q_heads, n_kv_heads, head_dim, c, b,
                                max_tokens, mass_out, workspace, workspace_bytes, 0, stream);
}

int cq_evict(const float* mass, const void* k_codes, const void* v_codes, const int32_t* seq_lens, int n_seq, int n_heads, int head_dim, int c,
             int b, int64_t max_tokens, int64_t n_keep, int64_t n_sinks, int64_t n_recent, int64_t out_max_tokens, float* mass_out,
             void* k_codes_out, void* v_codes_out, int32_t* kept_out, int32_t* seq_lens_out, void* stream)
{
    if (!mass || !k_codes || !v_codes || !seq_lens || !mass_out || !k_codes_out || !v_codes_out || !kept_out || !seq_lens_out) return CQ_ERR_NULL;
    EvictArgs a;
    const int st = make_shape(n_seq, max_tokens, n_heads, n_heads, head_dim, c, b, &a.sh);
    if (st != CQ_OK) return st;
    if (n_keep <= 0 || n_keep > out_max_tokens || n_sinks < 0 || n_recent < 0 || n_sinks > n_keep || n_recent > n_keep - n_sinks) return CQ_ERR_SHAPE;
    if (max_tokens > kMostTokens || out_max_tokens > kMostTokens) return CQ_ERR_UNSUPPORTED;
    // in place: all three, at the same capacity; otherwise none of them
    const int same = (k_codes_out == k_codes) + (v_codes_out == v_codes) + (mass_out == mass);
    if (same != 0 && (same != 3 || out_max_tokens != max_tokens)) return CQ_ERR_SHAPE;
    if (k_codes_out == v_codes_out || k_codes_out == v_codes || v_codes_out == k_codes || seq_lens_out == seq_lens) return CQ_ERR_SHAPE;
    if (!aligned16(k_codes) || !aligned16(v_codes) || !aligned16(k_codes_out) || !aligned16(v_codes_out) || !aligned4(mass) || !aligned4(mass_out) ||
        !aligned4(seq_lens) || !aligned4(kept_out) || !aligned4(seq_lens_out))
        return CQ_ERR_ALIGN;
    // what is written overlaps nothing else, apart from the buffers that are moved in place
    const size_t rows = (size_t)n_seq * n_heads, out_blocks = (size_t)((out_max_tokens + kTokenBlock - 1) / kTokenBlock);
    const size_t codes = rows * a.sh.n_blocks * a.sh.block_bytes, codes_out = rows * out_blocks * a.sh.block_bytes;
    const Extent in[] = {{k_codes, codes}, {v_codes, codes}, {mass, rows * max_tokens * sizeof(float)}, {seq_lens, n_seq * sizeof(int32_t)}};
    const Extent out[] = {{k_codes_out, codes_out}, {v_codes_out, codes_out}, {mass_out, rows * out_max_tokens * sizeof(float)},
                          {kept_out, rows * n_keep * sizeof(int32_t)}, {seq_lens_out, n_seq * sizeof(int32_t)}};
    for (int i = 0; i < 5; ++i) {
        for (int j = 0; j < 4; ++j)
            if (overlap(out[i], in[j]) && !(same == 3 && i == j)) return CQ_ERR_SHAPE;
        for (int j = 0; j < i; ++j)
            if (overlap(out[i], out[j])) return CQ_ERR_SHAPE;
    }
    a.mass = mass;
    a.kc = static_cast<const uint8_t*>(k_codes);
    a.vc = static_cast<const uint8_t*>(v_codes);
    a.seq_lens = seq_lens;
    a.n_keep = (int)n_keep;
    a.n_sinks = (int)n_sinks;
    a.n_recent = (int)n_recent;
    a.out_tokens = out_max_tokens;
    a.k_out = static_cast<uint8_t*>(k_codes_out);
    a.v_out = static_cast<uint8_t*>(v_codes_out);
    a.mass_out = mass_out;
    a.kept = kept_out;
    a.lens_out = seq_lens_out;
    return status(launch_evict(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
