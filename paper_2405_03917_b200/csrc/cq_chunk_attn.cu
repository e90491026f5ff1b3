// Attention of many query rows over a bounded cache (window, sinks, pages, ragged rows): the bounded form of the tensor-core kernel in
// cq_prefill_tc.cuh, and the merge of contexts that several CTAs share.
#include "cq_prefill_tc.cuh"

namespace cq {

namespace {

constexpr int kMergeWarps = 8;

// A warp per row of a row tile: log-sum-exp merge of the parts' accumulators.
__global__ void __launch_bounds__(kMergeWarps * 32) chunk_merge_kernel(PfBounded b)
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
    const float inv = L > 0.f ? 1.f / L : 1.f;                              // (nothing seen: the sums are zero; a wait gave up: NaN)
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

cudaError_t launch_chunk_attn(const BoundedArgs& a, void* workspace, cudaStream_t st)
{
    const Plan p = plan_of(a);
    const int64_t items = p.tiles * a.sh.n_kv_heads;
    if (items * p.parts > 0x7fffffff || items * (PfCfgB::kRows / kMergeWarps) > 0x7fffffff) return cudaErrorInvalidConfiguration;
    PfBounded b;
    b.a = a;
    b.tiles = (int)p.tiles;
    b.parts = p.parts;
    b.partials = static_cast<float*>(workspace);
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = overlapped_config((unsigned)(items * p.parts), PfCfgB::kThreads, PfCfgB::kSmemBytes, st, &attr);
    auto go = [&](auto kernel, int slot) {
        const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), PfCfgB::kSmemBytes, slot);
        if (e != cudaSuccess) return e;
        return cudaLaunchKernelEx(&cfg, kernel, a.q, a.kc, a.vc, (const float*)nullptr, (const float*)nullptr, a.seq_lens, a.scale_log2e, a.sh, a.max_q, 0,
                                  (float*)nullptr, b);
    };
    cudaError_t e = a.sh.c == 8 ? go(prefill_tc_kernel<8, PfBounded>, 106) : a.sh.c == 4 ? go(prefill_tc_kernel<4, PfBounded>, 107)
                                                                                         : go(prefill_tc_kernel<2, PfBounded>, 108);
    if (e != cudaSuccess || p.parts == 1) return e;
    cfg = overlapped_config((unsigned)(items * (PfCfgB::kRows / kMergeWarps)), kMergeWarps * 32, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, chunk_merge_kernel, b);
}

}  // namespace cq
