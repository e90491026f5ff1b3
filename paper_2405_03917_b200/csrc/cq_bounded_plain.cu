// Plain kernels of the operators on bounded caches: every supported shape, no tensor cores.
//
//   bounded_plain_kernel   out_i = sum_t p_t Vhat_t, p = softmax over the tokens that query i sees (window, sinks, pages)
//   mass_lse_kernel, mass_plain_kernel   mass[t] += sum over queries and query heads of p_t
//   codes_to_pages_kernel  codes of new tokens into the pages of their sequences
//
// One CTA per (row, query head), a token per warp and turn: the lanes hold the channels.  They stand in for the tuned kernels
// at shapes that have none, and the tests compare both.  What bounds them: a chain of dependent loads per token; one query each over
// 16 x 4096 tokens, 32 heads on 8, takes 2.3 ms with CQ-8c10b and 1.3 ms with head_dim 64, masses 2.8 and 1.5 ms.
// The way into the pages is the library's encode and one more launch: 64 x 1 tokens of 8 heads, CQ-8c8b, 9.0 us (5.8 of them the encode),
// 4 x 2048 tokens 94 us (90).
#include "cq_bounded.cuh"

namespace cq {

namespace {

constexpr int kWarps = 4;
constexpr int kLaneCh = 8;          // head_dim <= 256: up to 8 channels per lane

// The r-th of the tokens that a query at pos sees, in order: first the sinks before its window, then the window.
struct Visible {
    int n_first, from, count;
};
__device__ __forceinline__ Visible visible_tokens(int pos, int window, int sinks)
{
    Visible v;
    v.from = window_first(pos, window);
    v.n_first = sinks < v.from ? sinks : v.from;
    v.count = pos < 0 ? 0 : v.n_first + pos - v.from + 1;
    return v;
}

__global__ void __launch_bounds__(kWarps * 32) bounded_plain_kernel(BoundedArgs a)
{
    __shared__ float red_m[kWarps], red_l[kWarps];
    __shared__ float red_acc[kWarps][32 * kLaneCh];
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int hq = blockIdx.x % sh.n_q_heads, hkv = hq / sh.R;
    const int i = (blockIdx.x / sh.n_q_heads) % a.max_q;
    const int s = (int)(blockIdx.x / ((int64_t)sh.n_q_heads * a.max_q));
    const SeqView sv = seq_view(a, s);
    if (i >= sv.m || sv.m * sh.R < a.least_rows || sv.m * sh.R > a.most_rows) return;
    const int64_t row = ((int64_t)sv.row0 + i) * sh.n_q_heads + hq;
    const int pos = sv.n - sv.m + i;
    const Visible vis = visible_tokens(pos, a.window, a.sinks);
    float qd[kLaneCh], acc[kLaneCh];
#pragma unroll
    for (int j = 0; j < kLaneCh; ++j) {
        const int d = lane + 32 * j;
        qd[j] = d < sh.head_dim ? __half2float(a.q[row * sh.head_dim + d]) : 0.f;
        acc[j] = 0.f;
    }
    const __half* kcb = a.kcb + (int64_t)hkv * sh.G * sh.K * sh.c;
    const __half* vcb = a.vcb + (int64_t)hkv * sh.G * sh.K * sh.c;
    float m = -INFINITY, l = 0.f;
    for (int r = warp; r < vis.count; r += kWarps) {
        const int t = r < vis.n_first ? r : r - vis.n_first + vis.from;
        const int64_t off = block_offset(a, s, hkv, t / kTokenBlock);
        if (off < 0) continue;
        const int k = t % kTokenBlock;
        float dot = 0.f, vv[kLaneCh];
#pragma unroll
        for (int j = 0; j < kLaneCh; ++j) {
            const int d = lane + 32 * j;
            vv[j] = 0.f;
            if (d < sh.head_dim) {
                const int g = d / sh.c, e = d % sh.c;
                dot = fmaf(qd[j], __half2float(kcb[((int64_t)g * sh.K + read_code(a.kc + off, sh, g, k)) * sh.c + e]), dot);
                vv[j] = __half2float(vcb[((int64_t)g * sh.K + read_code(a.vc + off, sh, g, k)) * sh.c + e]);
            }
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
        dot *= a.scale_log2e;
        const float m_new = fmaxf(m, dot), ref = m_new == -INFINITY ? 0.f : m_new;      // (a score that is no number moves no reference)
        const float corr = exp2f(m - ref), p = exp2f(dot - ref);
        l = l * corr + p;
#pragma unroll
        for (int j = 0; j < kLaneCh; ++j) acc[j] = fmaf(p, vv[j], acc[j] * corr);
        m = m_new;
    }
    if (lane == 0) { red_m[warp] = m; red_l[warp] = l; }
#pragma unroll
    for (int j = 0; j < kLaneCh; ++j) red_acc[warp][lane + 32 * j] = acc[j];
    __syncthreads();
    float M = -INFINITY, L = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w]);
    auto bring = [&](int w) { return red_m[w] == -INFINITY ? 1.f : exp2f(red_m[w] - M); };      // (no reference: the sums are zero, or no numbers)
    for (int w = 0; w < kWarps; ++w) L += bring(w) * red_l[w];
    for (int d = threadIdx.x; d < sh.head_dim; d += blockDim.x) {
        float x = 0.f;
        for (int w = 0; w < kWarps; ++w) x = fmaf(bring(w), red_acc[w][d], x);
        a.out[row * sh.head_dim + d] = __float2half_rn(L == 0.f ? 0.f : x / L);      // nothing seen: a zero row
    }
}

// Score of a token (log2 domain), the lanes sharing its channels; the same in every lane.
__device__ __forceinline__ float plain_score(const BoundedArgs& a, const __half* kcb, const uint8_t* blk, const float (&qd)[kLaneCh], int k)
{
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31;
    float dot = 0.f;
#pragma unroll
    for (int j = 0; j < kLaneCh; ++j) {
        const int d = lane + 32 * j;
        if (d < sh.head_dim) {
            const int g = d / sh.c;
            dot = fmaf(qd[j], __half2float(kcb[((int64_t)g * sh.K + read_code(blk, sh, g, k)) * sh.c + d % sh.c]), dot);
        }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    return dot * a.scale_log2e;
}

// lse[(sequence, query), query head]: log2 of the sum of 2^score over the tokens that the query sees (-inf: none)
__global__ void __launch_bounds__(kWarps * 32) mass_lse_kernel(BoundedArgs a, float* __restrict__ lse)
{
    __shared__ float red_m[kWarps], red_l[kWarps];
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int hq = blockIdx.x % sh.n_q_heads, hkv = hq / sh.R;
    const int i = (blockIdx.x / sh.n_q_heads) % a.max_q;
    const int s = (int)(blockIdx.x / ((int64_t)sh.n_q_heads * a.max_q));
    const SeqView sv = seq_view(a, s);
    const int pos = sv.n - sv.m + i;
    const int64_t row = blockIdx.x;
    float qd[kLaneCh];
#pragma unroll
    for (int j = 0; j < kLaneCh; ++j) qd[j] = lane + 32 * j < sh.head_dim ? __half2float(a.q[row * sh.head_dim + lane + 32 * j]) : 0.f;
    const __half* kcb = a.kcb + (int64_t)hkv * sh.G * sh.K * sh.c;
    float m = -INFINITY, l = 0.f;
    for (int t = warp; t <= pos; t += kWarps) {
        const float x = plain_score(a, kcb, a.kc + block_offset(a, s, hkv, t / kTokenBlock), qd, t % kTokenBlock);
        const float m_new = fmaxf(m, x), ref = m_new == -INFINITY ? 0.f : m_new;
        l = l * exp2f(m - ref) + exp2f(x - ref);
        m = m_new;
    }
    if (lane == 0) { red_m[warp] = m; red_l[warp] = l; }
    __syncthreads();
    if (threadIdx.x == 0) {
        float M = -INFINITY, L = 0.f;
        for (int w = 0; w < kWarps; ++w) M = fmaxf(M, red_m[w]);
        for (int w = 0; w < kWarps; ++w) L += (red_m[w] == -INFINITY ? 1.f : exp2f(red_m[w] - M)) * red_l[w];
        lse[row] = L == 0.f ? -INFINITY : M + log2f(L);
    }
}

// A CTA per (sequence, KV head, 16-token block): its tokens' masses from every (query, query head), in a fixed order
__global__ void __launch_bounds__(kWarps * 32) mass_plain_kernel(BoundedArgs a, const float* __restrict__ lse, const float* mass_in, float* mass_out)
{
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int blk = (int)(blockIdx.x % sh.n_blocks);
    const int hkv = (int)((blockIdx.x / sh.n_blocks) % sh.n_kv_heads);
    const int s = (int)(blockIdx.x / (sh.n_blocks * sh.n_kv_heads));
    const SeqView sv = seq_view(a, s);
    if (blk * kTokenBlock >= sv.n) return;
    const __half* kcb = a.kcb + (int64_t)hkv * sh.G * sh.K * sh.c;
    const uint8_t* codes = a.kc + block_offset(a, s, hkv, blk);
    for (int k = warp; k < kTokenBlock && blk * kTokenBlock + k < sv.n; k += kWarps) {
        const int t = blk * kTokenBlock + k;
        float sum = 0.f;
        for (int i = 0; i < sv.m; ++i) {
            if (t > sv.n - sv.m + i) continue;
            for (int r = 0; r < sh.R; ++r) {
                const int64_t row = ((int64_t)sv.row0 + i) * sh.n_q_heads + hkv * sh.R + r;
                float qd[kLaneCh];
#pragma unroll
                for (int j = 0; j < kLaneCh; ++j) qd[j] = lane + 32 * j < sh.head_dim ? __half2float(a.q[row * sh.head_dim + lane + 32 * j]) : 0.f;
                sum += exp2f(plain_score(a, kcb, codes, qd, k) - lse[row]);
            }
        }
        const int64_t at = ((int64_t)s * sh.n_kv_heads + hkv) * sh.max_tokens + t;
        if (lane == 0) mass_out[at] = (mass_in ? mass_in[at] : 0.f) + sum;
    }
}

// A thread per (sequence, block that new tokens fall into, head, group); a warp walks the groups.  It alone writes the block's
// words of the group, so that the packed upper bits of neighbouring tokens (b > 8) meet in no race.
__global__ void codes_to_pages_kernel(BoundedArgs a, const uint8_t* __restrict__ ks, const uint8_t* __restrict__ vs, uint8_t* __restrict__ kp,
                                      uint8_t* __restrict__ vp, int blocks_per_seq, int64_t total)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Shape& sh = a.sh;
    const int64_t id = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
    if (id >= total) return;
    const int g = (int)(id % sh.G);
    const int h = (int)((id / sh.G) % sh.n_kv_heads);
    const int bi = (int)((id / sh.G / sh.n_kv_heads) % blocks_per_seq);
    const int s = (int)(id / sh.G / sh.n_kv_heads / blocks_per_seq);
    const SeqView sv = seq_view(a, s);
    const int64_t first = (int64_t)a.seq_lens[s] - sv.m;                       // position of the first new token (may lie outside)
    const int64_t blk = (first < 0 ? 0 : first) / kTokenBlock + bi;
    if (sv.m == 0 || blk >= sh.n_blocks || blk * kTokenBlock >= first + sv.m) return;
    const int64_t off = block_offset(a, s, h, (int)blk);
    if (off < 0) return;
    const int64_t lo = first > blk * kTokenBlock ? first : blk * kTokenBlock;  // new positions of this block: lo ... hi - 1
    int64_t hi = first + sv.m < (blk + 1) * kTokenBlock ? first + sv.m : (blk + 1) * kTokenBlock;
    hi = hi < sh.max_tokens ? hi : sh.max_tokens;
    const int64_t staged_blocks = ((int64_t)a.n_rows + kTokenBlock - 1) / kTokenBlock;
#pragma unroll 1
    for (int tensor = 0; tensor < 2; ++tensor) {
        const uint8_t* src = tensor ? vs : ks;
        uint8_t* dst = (tensor ? vp : kp) + off;
        if (sh.hb == 0 && hi - lo == kTokenBlock) {
            uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < kTokenBlock; ++k) {
                const int64_t row = sv.row0 + (lo - first) + k;
                w[k >> 2] |= (uint32_t)src[((int64_t)h * staged_blocks + row / kTokenBlock) * sh.block_bytes + g * kTokenBlock + row % kTokenBlock] << (8 * (k & 3));
            }
            *reinterpret_cast<uint4*>(dst + g * kTokenBlock) = make_uint4(w[0], w[1], w[2], w[3]);
            continue;
        }
        for (int64_t t = lo; t < hi; ++t) {
            const int64_t row = sv.row0 + (t - first);
            const int code = read_code(src + ((int64_t)h * staged_blocks + row / kTokenBlock) * sh.block_bytes, sh, g, (int)(row % kTokenBlock));
            const int k = (int)(t % kTokenBlock);
            dst[g * kTokenBlock + k] = (uint8_t)code;
            if (sh.hb) {
                const int bit = k * sh.hb;
                uint8_t* high = dst + sh.G * kTokenBlock + g * 2 * sh.hb + (bit >> 3);
                const uint32_t mask = ((1u << sh.hb) - 1u) << (bit & 7);
                *high = (uint8_t)((*high & ~mask) | (((uint32_t)code >> 8) << (bit & 7) & mask));
            }
        }
    }
}

}  // namespace

cudaError_t launch_bounded_plain(const BoundedArgs& a, cudaStream_t st)
{
    const int64_t grid = a.sh.n_seq * (int64_t)a.max_q * a.sh.n_q_heads;
    if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    bounded_plain_kernel<<<(unsigned)grid, kWarps * 32, 0, st>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_mass_plain(const BoundedArgs& a, const float* mass_in, float* mass_out, float* lse, cudaStream_t st)
{
    const int64_t rows = a.sh.n_seq * (int64_t)a.max_q * a.sh.n_q_heads, grid = a.sh.n_seq * a.sh.n_kv_heads * a.sh.n_blocks;
    if (rows > 0x7fffffff || grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    mass_lse_kernel<<<(unsigned)rows, kWarps * 32, 0, st>>>(a, lse);
    mass_plain_kernel<<<(unsigned)grid, kWarps * 32, 0, st>>>(a, lse, mass_in, mass_out);
    return cudaGetLastError();
}

cudaError_t launch_codes_to_pages(const BoundedArgs& a, const uint8_t* k_staged, const uint8_t* v_staged, uint8_t* k_pages, uint8_t* v_pages,
                                  cudaStream_t st)
{
    const int blocks_per_seq = (a.max_q + kTokenBlock - 1) / kTokenBlock + 1;
    const int64_t total = a.sh.n_seq * a.sh.n_kv_heads * a.sh.G * blocks_per_seq;
    if ((total + 255) / 256 > 0x7fffffff) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)((total + 255) / 256), 256, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, codes_to_pages_kernel, a, k_staged, v_staged, k_pages, v_pages, blocks_per_seq, total);
}

}  // namespace cq
