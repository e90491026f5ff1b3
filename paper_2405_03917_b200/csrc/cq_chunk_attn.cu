// Attention of many query rows over a bounded cache (window, sinks, pages, ragged rows), and the masses that they give to cached tokens:
// the bounded forms of the tensor-core kernel in cq_prefill_tc.cu, and what joins the parts of a context or the row tiles.
//
// Attention.  What bounds it: per 64 tokens and 256 rows the MMAs take 1024 cycles of about 2160.  The rest is a chain: scores of a row tile
// (tensor memory has room for one tile of them beside the outputs, queries and weights), their way into registers, the other row tile's
// scores, at some 300 cycles for a hand-over: 4 x 2048 queries over 8192 tokens, 32 heads on 8, CQ-8c8b, 1.07 ... 1.16 ms in pages of
// 64, 0.99 ... 1.04 without (the plain prefill attention: 0.98 ... 1.03; side by side the look-up of pages costs 6 %).  Two
// threads share a row (3 x 333 queries with a window of 511, 32 heads of CQ-4c8b: 79 us with one, 55 ... 61 with two; the prompts above are as
// fast with one).  Half of the exponentials on the FMA pipe (1060 ... 1138 against 1046 us for those prompts), scores and weights in the same
// columns (1186 against 978) and scores in halves (1152 against 988) were slower.  A context is shared by several CTAs where the row
// tiles leave SMs idle.
// Masses, from 17 rows of a sequence on.  A first pass leaves every row's log-sum-exp, a second one works the scores out again and adds up,
// per token, the weights of a row tile: over the 32 rows of a warp by exchanges that halve the columns (lane i is left with column i), over the
// warps through shared memory, over row tiles in a kernel of its own; every sum has one order.  What bounds it: the exponentials (two
// passes, 16 per clock and SM) and the waits behind them: 1190 and 1660 cycles per 64 tokens of 128 rows.  A second tile of scores in the
// outputs' columns changed nothing.  4 x 32 queries over 5001 ... 8192 tokens, 32 heads on 8, CQ-8c8b: 65 us, 227 us with the gather kernel.
#include "cq_prefill_tc.cu"

namespace cq {

namespace {

constexpr int kMergeWarps = 8;

// A warp per row of a row tile: log-sum-exp merge of the parts' accumulators.
__global__ void __launch_bounds__(kMergeWarps * 32) chunk_merge_kernel(PfBounded<kPfAttn> b)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const BoundedArgs& a = b.a;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, R = a.sh.R, q_per_tile = PfCfgB::kRows / R;
    constexpr int kPerTile = PfCfgB::kRows / kMergeWarps;                    // CTAs of a row tile
    const int item = blockIdx.x / kPerTile, rho = blockIdx.x % kPerTile * kMergeWarps + warp;
    int number = 0;
    const int s = pf_find_tile(a, item / a.sh.n_kv_heads, q_per_tile, number);
    if (s < 0) return;
    const SeqView sv = seq_view(a, s);
    const int qi = (pf_tiles_of(a, sv, q_per_tile) - 1 - number) * q_per_tile + rho / R;
    if (rho >= q_per_tile * R || qi >= sv.m) return;
    const float* first = b.partials + ((int64_t)item * b.parts * PfCfgB::kRows + rho) * partial_stride(128);
    auto part = [&](int i) { return first + (int64_t)i * PfCfgB::kRows * partial_stride(128); };
    float M = -INFINITY;
#pragma unroll 4
    for (int i = 0; i < b.parts; ++i) M = fmaxf(M, part(i)[0]);
    float L = 0.f, x[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < b.parts; ++i) {
        const float m = part(i)[0], f = m == -INFINITY ? 0.f : exp2f(m - M);
        const float2 u = *reinterpret_cast<const float2*>(part(i) + 2 + 4 * lane), v = *reinterpret_cast<const float2*>(part(i) + 4 + 4 * lane);
        L = fmaf(f, part(i)[1], L);
        x[0] = fmaf(f, u.x, x[0]);
        x[1] = fmaf(f, u.y, x[1]);
        x[2] = fmaf(f, v.x, x[2]);
        x[3] = fmaf(f, v.y, x[3]);
    }
    const float inv = L == 0.f ? 1.f : 1.f / L;                             // (nothing seen: the sums are zero; a wait gave up: NaN)
    *reinterpret_cast<uint2*>(a.out + (((int64_t)sv.row0 + qi) * a.sh.n_q_heads + item % a.sh.n_kv_heads * R + rho % R) * 128 + 4 * lane) =
        make_uint2(pack_half2(x[0] * inv, x[1] * inv), pack_half2(x[2] * inv, x[3] * inv));
}

// Row tiles of all sequences (a bound, where the counts are known to the device only) and the CTAs that share one's context: where
// the tiles alone leave most SMs idle.
struct Plan {
    int64_t tiles;
    int parts;
};
Plan plan_of(const BoundedArgs& a)
{
    const int q_per_tile = PfCfgB::kRows / a.sh.R;
    Plan p;
    p.tiles = a.sh.n_seq * ((a.max_q + q_per_tile - 1) / q_per_tile);
    const int64_t least_new = a.least_rows / a.sh.R > 0 ? a.least_rows / a.sh.R : 1;      // new tokens of a sequence that takes this kernel
    const int64_t sequences = a.sh.n_seq < a.n_rows / least_new ? a.sh.n_seq : a.n_rows / least_new;
    const int64_t ragged = a.n_rows / q_per_tile + sequences;
    if (ragged < p.tiles) p.tiles = ragged;
    if (p.tiles < 1) p.tiles = 1;
    const int64_t ctas = p.tiles * a.sh.n_kv_heads, sms = device_sm_count();
    const int64_t most = (a.sh.max_tokens + PfCfgB::kTile * kPfLeastShare - 1) / (PfCfgB::kTile * kPfLeastShare);
    p.parts = 2 * ctas <= sms ? (int)(sms / ctas) : 1;
    if (p.parts > most) p.parts = (int)most;
    return p;
}

}  // namespace

bool chunk_attn_supported(const Shape& sh)
{
    return sh.head_dim == 128 && sh.b <= 8 && sh.K * sh.c >= 8 && (sh.c == 2 || sh.c == 4 || sh.c == 8) && sh.R <= PfCfgB::kRows;
}

size_t chunk_attn_workspace_bytes(const BoundedArgs& a)
{
    const Plan p = plan_of(a);
    return p.parts == 1 ? 0 : (size_t)(p.tiles * a.sh.n_kv_heads * p.parts) * PfCfgB::kRows * partial_stride(128) * sizeof(float);
}

namespace {

template <int kWhat>
cudaError_t launch_kernel(const PfBounded<kWhat>& b, int64_t items, int slot, cudaStream_t st)
{
    const BoundedArgs& a = b.a;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)(items * b.parts), PfCfgB::kThreads, PfCfgB::kSmemBytes, st, &attr);
    auto go = [&](auto kernel, int at) {
        const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), PfCfgB::kSmemBytes, at);
        if (e != cudaSuccess) return e;
        return cudaLaunchKernelEx(&cfg, kernel, a.q, a.kc, a.vc, (const float*)nullptr, (const float*)nullptr, a.seq_lens, a.scale_log2e, a.sh, a.max_q, 0,
                                  (float*)nullptr, b);
    };
    return a.sh.c == 8 ? go(prefill_tc_kernel<8, PfBounded<kWhat>>, slot) : a.sh.c == 4 ? go(prefill_tc_kernel<4, PfBounded<kWhat>>, slot + 1)
                                                                                        : go(prefill_tc_kernel<2, PfBounded<kWhat>>, slot + 2);
}

// Masses of several row tiles: a thread per token adds those of the tiles that see it, the earliest queries' first.
__global__ void __launch_bounds__(256) mass_sum_kernel(BoundedArgs a, const float* __restrict__ sums, int row_tiles, int chunks, const float* mass_in,
                                                       float* mass_out)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t item = blockIdx.x / chunks;
    const int t = (int)(blockIdx.x % chunks) * 256 + (int)threadIdx.x;
    const SeqView sv = seq_view(a, (int)(item / a.sh.n_kv_heads));
    if (t >= sv.n) return;
    const int q_per_tile = PfCfgB::kRows / a.sh.R;
    const int64_t at = item * a.sh.max_tokens + t, stride = a.sh.n_seq * a.sh.n_kv_heads * a.sh.max_tokens;
    float sum = 0.f;
    for (int i = 0; i < row_tiles; ++i) {
        const int last = (i + 1) * q_per_tile < sv.m ? (i + 1) * q_per_tile - 1 : sv.m - 1;       // the tile's last query; it wrote whole tiles of tokens
        if ((sv.n - sv.m + last) / PfCfgB::kTile >= t / PfCfgB::kTile && sv.n - sv.m + last >= 0) sum += sums[i * stride + at];
    }
    mass_out[at] = (mass_in ? mass_in[at] : 0.f) + sum;
}

size_t lse_bytes(const BoundedArgs& a, const Plan& p) { return round_up((size_t)(p.tiles * a.sh.n_kv_heads * p.parts) * PfCfgB::kRows * 2 * sizeof(float), 256); }
int row_tiles_of(const BoundedArgs& a) { const int q_per_tile = PfCfgB::kRows / a.sh.R; return (a.max_q + q_per_tile - 1) / q_per_tile; }

}  // namespace

cudaError_t launch_chunk_attn(const BoundedArgs& a, void* workspace, size_t workspace_bytes, cudaStream_t st)
{
    if (workspace_bytes < chunk_attn_workspace_bytes(a)) return cudaErrorInvalidValue;       // (the caller has asked for another plan)
    const Plan p = plan_of(a);
    const int64_t items = p.tiles * a.sh.n_kv_heads;
    if (items * p.parts > 0x7fffffff || items * (PfCfgB::kRows / kMergeWarps) > 0x7fffffff) return cudaErrorInvalidConfiguration;
    PfBounded<kPfAttn> b = {};
    b.a = a;
    b.tiles = (int)p.tiles;
    b.parts = p.parts;
    b.partials = static_cast<float*>(workspace);
    const cudaError_t e = launch_kernel(b, items, 146, st);
    if (e != cudaSuccess || p.parts == 1) return e;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)(items * (PfCfgB::kRows / kMergeWarps)), kMergeWarps * 32, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, chunk_merge_kernel, b);
}

size_t chunk_mass_workspace_bytes(const BoundedArgs& a)
{
    const int row_tiles = row_tiles_of(a);
    return lse_bytes(a, plan_of(a)) + (row_tiles > 1 ? (size_t)row_tiles * a.sh.n_seq * a.sh.n_kv_heads * a.sh.max_tokens * sizeof(float) : 0);
}

cudaError_t launch_chunk_mass(const BoundedArgs& a, const float* mass_in, float* mass_out, void* workspace, cudaStream_t st)
{
    const Plan p = plan_of(a);
    const int64_t items = p.tiles * a.sh.n_kv_heads, chunks = (a.sh.max_tokens + 255) / 256, sum_grid = a.sh.n_seq * a.sh.n_kv_heads * chunks;
    if (items * p.parts > 0x7fffffff || sum_grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    PfBounded<kPfLse> b = {};
    b.a = a;
    b.tiles = (int)p.tiles;
    b.parts = p.parts;
    b.partials = static_cast<float*>(workspace);
    b.row_tiles = row_tiles_of(a);
    cudaError_t e = launch_kernel(b, items, 149, st);
    if (e != cudaSuccess) return e;
    PfBounded<kPfMass> c = {};
    c.a = a;
    c.tiles = b.tiles;
    c.parts = b.parts;
    c.partials = b.partials;
    c.row_tiles = b.row_tiles;
    c.mass_in = mass_in;
    float* sums = reinterpret_cast<float*>(static_cast<char*>(workspace) + lse_bytes(a, p));
    c.mass_out = c.row_tiles > 1 ? sums : mass_out;
    e = launch_kernel(c, items, 152, st);
    if (e != cudaSuccess || c.row_tiles == 1) return e;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)sum_grid, 256, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, mass_sum_kernel, a, (const float*)sums, c.row_tiles, (int)chunks, mass_in, mass_out);
}

}  // namespace cq
