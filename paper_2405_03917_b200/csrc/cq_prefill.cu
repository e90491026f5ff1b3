// Causal attention of a run of new tokens over the CQ-coded cache (a prompt, or a chunk of one).
//
// Section 2.1 of the paper: Eq. 1 gives the output of "the current token" from the keys and values
// of all tokens up to and including it; here it is applied to each of the n_q newest cached tokens,
// with K and V replaced by their CQ reconstructions (Section 3.2).  Query i of sequence s sits at
// position seq_lens[s] - n_q + i and attends the cached tokens 0 ... that position.
//
// With many queries per cached token the per-query lookup tables of the decode kernels no longer
// pay (one table per query); the codes are turned back into vectors instead and the two
// contractions run on the tensor cores:
//   prefill_tc_kernel (cq_prefill_tc.cu; head_dim 128, one byte per code, c = 2, 4 or 8): one CTA per (sequence, KV
//     head, 256 (query, head of the KV head's group) rows), as two row tiles of 128, one row per lane
//     of tensor memory.  Both codebooks are kept in shared memory as fp16, code-major, so that the
//     lanes of a gather (one group each) meet in no bank whatever the codes are.  Four producer warps
//     gather the codes of 64 cached tokens into swizzled fp16 tiles (three stages); S = Q Khat^T and
//     O += P Vhat are tcgen05 MMAs with fp32 accumulators, Q and P read from tensor memory, issued by
//     a warp each; eight softmax warps take a row per thread (running maximum, log2 domain).
//     What bounds it: per 64 tokens and 256 rows the MMAs take 1024 cycles and the exponentials 1024
//     (two per clock and SM quarter); each waits for the other in turn through the two row tiles.
//     4 x 2048 queries over 8192 tokens, 32 heads on 8, CQ-8c8b: 3.20 ms with m16n8k16 MMAs and the
//     tiles' fragments in registers, 1.36 ms with one MMA-issuing thread that did scores and sums in
//     turn, 0.95 ms now, 0.57 ms being the contractions at the measured GEMM rate.
//   prefill_generic_kernel: any supported shape, one CTA per (sequence, query, head), plain loops.
#include "cq_prefill_tc.cu"

namespace cq {

namespace {

// ------------------------------------------------------------------------------------------
// generic kernel
// ------------------------------------------------------------------------------------------
constexpr int kGenWarps = 4;
constexpr int kMaxLaneCh = 8;          // head_dim <= 256: up to 8 channels per lane

__global__ void __launch_bounds__(kGenWarps * 32)
prefill_generic_kernel(const __half* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                       const float* __restrict__ kcb, const float* __restrict__ vcb,
                       const int32_t* __restrict__ seq_lens, float scale_log2e, Shape sh, int n_q, float* __restrict__ out)
{
    __shared__ float red_m[kGenWarps], red_l[kGenWarps];
    __shared__ float red_acc[kGenWarps][256];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int hq = blockIdx.x % sh.n_q_heads;
    const int qi = (blockIdx.x / sh.n_q_heads) % n_q;
    const int64_t s = blockIdx.x / ((int64_t)sh.n_q_heads * n_q);
    const int hkv = hq / sh.R;
    int64_t n = seq_lens[s];
    n = n < 0 ? 0 : (n > sh.max_tokens ? sh.max_tokens : n);
    const int64_t n_att = n - n_q + qi + 1;                              // tokens 0 .. position of the query
    const int64_t row = (s * n_q + qi) * sh.n_q_heads + hq;
    float* o = out + row * sh.head_dim;
    if (n_att <= 0) {
        for (int d = threadIdx.x; d < sh.head_dim; d += blockDim.x) o[d] = 0.f;
        return;
    }
    float qd[kMaxLaneCh], acc[kMaxLaneCh];
#pragma unroll
    for (int j = 0; j < kMaxLaneCh; ++j) {
        const int d = lane + 32 * j;
        qd[j] = d < sh.head_dim ? __half2float(q[row * sh.head_dim + d]) * scale_log2e : 0.f;
        acc[j] = 0.f;
    }
    float m = -INFINITY, l = 0.f;
    for (int64_t t = warp; t < n_att; t += kGenWarps) {
        const uint8_t* kblk = kc + code_word_offset(sh, sh.n_kv_heads, s, hkv, t / kTokenBlock, 0);
        const uint8_t* vblk = vc + code_word_offset(sh, sh.n_kv_heads, s, hkv, t / kTokenBlock, 0);
        const int k = (int)(t % kTokenBlock);
        float dot = 0.f, vv[kMaxLaneCh];
#pragma unroll
        for (int j = 0; j < kMaxLaneCh; ++j) {
            const int d = lane + 32 * j;
            vv[j] = 0.f;
            if (d < sh.head_dim) {
                const int g = d / sh.c, i = d % sh.c;
                dot = fmaf(qd[j], kcb[(((int64_t)hkv * sh.G + g) * sh.K + read_code(kblk, sh, g, k)) * sh.c + i], dot);
                vv[j] = vcb[(((int64_t)hkv * sh.G + g) * sh.K + read_code(vblk, sh, g, k)) * sh.c + i];
            }
        }
#pragma unroll
        for (int off = 16; off > 0; off >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, off);
        const float m_new = fmaxf(m, dot);
        const float corr = exp2f(m - m_new), p = exp2f(dot - m_new);
        l = l * corr + p;
#pragma unroll
        for (int j = 0; j < kMaxLaneCh; ++j) acc[j] = fmaf(p, vv[j], acc[j] * corr);
        m = m_new;
    }
    if (lane == 0) { red_m[warp] = m; red_l[warp] = l; }
#pragma unroll
    for (int j = 0; j < kMaxLaneCh; ++j) red_acc[warp][lane + 32 * j] = acc[j];
    __syncthreads();
    float M = -INFINITY;
    for (int w = 0; w < kGenWarps; ++w) M = fmaxf(M, red_m[w]);
    float L = 0.f;
    for (int w = 0; w < kGenWarps; ++w) L += red_m[w] == -INFINITY ? 0.f : exp2f(red_m[w] - M) * red_l[w];
    for (int d = threadIdx.x; d < sh.head_dim; d += blockDim.x) {
        float a = 0.f;
        for (int w = 0; w < kGenWarps; ++w)
            if (red_m[w] != -INFINITY) a = fmaf(exp2f(red_m[w] - M), red_acc[w][d], a);
        o[d] = a / L;
    }
}

}  // namespace

bool prefill_mma_supported(const Shape& sh)
{
    return sh.head_dim == 128 && sh.b == 8 && (sh.c == 2 || sh.c == 4 || sh.c == 8) && sh.R <= 64 && PfCfg::kRows % sh.R == 0;
}

cudaError_t launch_prefill(const __half* q, const uint8_t* kc, const uint8_t* vc, const float* kcb, const float* vcb,
                           const int32_t* seq_lens, float scale, const Shape& sh, int n_q, float* out, bool generic,
                           cudaStream_t st)
{
    if (!generic && prefill_mma_supported(sh)) {
        using C = PfCfg;
        const int q_per_tile = C::kRows / sh.R;
        const int row_tiles = (n_q + q_per_tile - 1) / q_per_tile;
        const int64_t grid = sh.n_seq * sh.n_kv_heads * row_tiles;
        if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = overlapped_config((unsigned)grid, C::kThreads, C::kSmemBytes, st, &attr);
        auto go = [&](auto kernel, int slot) {
            const cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(kernel), C::kSmemBytes, slot);
            if (e != cudaSuccess) return e;
            return cudaLaunchKernelEx(&cfg, kernel, q, kc, vc, kcb, vcb, seq_lens, scale * kLog2e, sh, n_q, row_tiles, out, PfNone());
        };
        return sh.c == 8 ? go(prefill_tc_kernel<8>, 40) : sh.c == 4 ? go(prefill_tc_kernel<4>, 41) : go(prefill_tc_kernel<2>, 42);
    }
    const int64_t grid = sh.n_seq * (int64_t)n_q * sh.n_q_heads;
    if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    prefill_generic_kernel<<<(unsigned)grid, kGenWarps * 32, 0, st>>>(q, kc, vc, kcb, vcb, seq_lens, scale * kLog2e, sh, n_q, out);
    return cudaGetLastError();
}

}  // namespace cq
