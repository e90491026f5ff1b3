// Eviction from a coded cache by accumulated attention weight.
//
// Per (sequence, head): of n cached tokens stay the n_sinks first, the n_recent last and, of the others, those of largest mass
// (equal masses: the lower position), n_keep in all; codes and masses move to positions 0, 1, ... in their old order.
//
//   evict_select_kernel  one CTA per (sequence, head): the masses become whole numbers of the same order, the n-th largest is
//       found by three histograms of 11, 11 and 10 bits in shared memory, and the positions that stay are listed in order
//       (ballots in a warp, one scan over the warps).
//   evict_move_kernel    a warp per 16 tokens that stay: a lane takes one (tensor, group) of them, a byte load per token (the
//       lanes of a load read one token's codes: whole 16-token blocks pass through L1), and writes one 16-byte word.
//       In place a CTA goes through its (sequence, head) in order: positions only ever move down, and all reads of a turn are done
//       before its writes.
#include "cq_bounded.cuh"

namespace cq {

namespace {

constexpr int kSelectThreads = 1024, kSelectWarps = kSelectThreads / 32;
constexpr int kBins = 2048;

// Whole number of the same order as the mass: any NaN above all numbers, the two zeros alike.
__device__ __forceinline__ uint32_t mass_key(float m)
{
    if (m != m) return 0xffffffffu;
    const uint32_t u = __float_as_uint(m + 0.f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// kEach: masses a thread keeps in registers (0: they are read again from memory at every pass)
template <int kEach>
__global__ void __launch_bounds__(kSelectThreads) evict_select_kernel(EvictArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ uint32_t hist[kBins];
    __shared__ uint32_t warp_sum[kSelectWarps];
    __shared__ uint32_t found[2];                    // bin of the n-th largest, tokens above it
    __shared__ uint32_t warp_above[kSelectWarps], warp_equal[kSelectWarps];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int s = blockIdx.x / a.sh.n_kv_heads;
    const int64_t n64 = a.seq_lens[s];
    const int n = (int)(n64 < 0 ? 0 : (n64 > a.sh.max_tokens ? a.sh.max_tokens : n64));
    const float* mass = a.mass + (int64_t)blockIdx.x * a.sh.max_tokens;
    int32_t* kept = a.kept + (int64_t)blockIdx.x * a.n_keep;
    if (n <= a.n_keep) {
        for (int j = threadIdx.x; j < a.n_keep; j += kSelectThreads) kept[j] = j < n ? j : -1;
        return;
    }
    const int c_lo = a.n_sinks, c_hi = n - a.n_recent;                        // the tokens that compete
    uint32_t need = (uint32_t)(a.n_keep - a.n_sinks - a.n_recent);            // how many of them stay (fewer than there are)
    // warp w holds per_warp tokens from w * per_warp, register (or turn) j of lane l token j * 32 + l of them
    const int turns = kEach ? kEach : (n + kSelectThreads - 1) / kSelectThreads;
    const int base = warp * turns * 32 + lane;
    uint32_t key[kEach ? kEach : 1];
    if (kEach) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) key[j] = base + 32 * j < n ? mass_key(mass[base + 32 * j]) : 0u;
    }
    auto key_at = [&](int j) { return kEach ? key[kEach ? j : 0] : (base + 32 * j < n ? mass_key(mass[base + 32 * j]) : 0u); };
    uint32_t prefix = 0u, mask = 0u;
    if (need > 0) {
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bins = pass == 2 ? 1024 : kBins;
            for (int i = threadIdx.x; i < kBins; i += kSelectThreads) hist[i] = 0u;
            __syncthreads();
            auto count = [&](int j) {
                const int t = base + 32 * j;
                const uint32_t k = key_at(j);
                if (t >= c_lo && t < c_hi && (k & mask) == prefix) atomicAdd(&hist[(k >> shift) & (bins - 1)], 1u);
            };
            if (kEach) {
#pragma unroll
                for (int j = 0; j < kEach; ++j) count(j);
            } else {
                for (int j = 0; j < turns; ++j) count(j);
            }
            __syncthreads();
            // thread i owns bins 2 i and 2 i + 1, counted from the top
            const int top = kBins - 1 - 2 * (int)threadIdx.x;
            const uint32_t h0 = hist[top], h1 = hist[top - 1];
            uint32_t incl = h0 + h1;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += x;
            }
            if (lane == 31) warp_sum[warp] = incl;
            __syncthreads();
            uint32_t before = 0u;
            for (int w = 0; w < warp; ++w) before += warp_sum[w];
            before += incl - h0 - h1;
            if (before < need && need <= before + h0) { found[0] = (uint32_t)top; found[1] = before; }
            else if (before + h0 < need && need <= before + h0 + h1) { found[0] = (uint32_t)top - 1u; found[1] = before + h0; }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= (uint32_t)(bins - 1) << shift;
            need -= found[1];
            __syncthreads();
        }
    }
    // the keys above `prefix` stay, and the first `need` that equal it (need 0 and prefix 0 with nothing to choose: none)
    const bool choose = a.n_keep > a.n_sinks + a.n_recent;
    auto rank = [&](int j, bool& above, bool& equal) {
        const int t = base + 32 * j;
        const uint32_t k = key_at(j);
        const bool forced = t < c_lo || (t >= c_hi && t < n);
        above = forced || (choose && t < c_hi && k > prefix);
        equal = choose && !forced && t < c_hi && k == prefix;
    };
    uint32_t n_above = 0u, n_equal = 0u;
    auto tally = [&](int j) {
        bool above, equal;
        rank(j, above, equal);
        n_above += __popc(__ballot_sync(0xffffffffu, above));
        n_equal += __popc(__ballot_sync(0xffffffffu, equal));
    };
    if (kEach) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) tally(j);
    } else {
        for (int j = 0; j < turns; ++j) tally(j);
    }
    if (lane == 0) { warp_above[warp] = n_above; warp_equal[warp] = n_equal; }
    __syncthreads();
    uint32_t above_before = 0u, equal_before = 0u;
    for (int w = 0; w < warp; ++w) { above_before += warp_above[w]; equal_before += warp_equal[w]; }
    const uint32_t below = (1u << lane) - 1u;
    auto list = [&](int j) {
        bool above, equal;
        rank(j, above, equal);
        const uint32_t eq = __ballot_sync(0xffffffffu, equal), ab = __ballot_sync(0xffffffffu, above);
        const uint32_t e = equal_before + __popc(eq & below);
        const uint32_t at = above_before + __popc(ab & below) + (e < need ? e : need);
        if (above || (equal && e < need)) kept[at] = base + 32 * j;
        above_before += __popc(ab);
        equal_before += __popc(eq);
    };
    if (kEach) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) list(j);
    } else {
        for (int j = 0; j < turns; ++j) list(j);
    }
}

constexpr int kMoveWarps = 8;

// One CTA: out blocks blockIdx.y * per_cta ... of (sequence, head) blockIdx.x; in place one CTA takes them all.
__global__ void __launch_bounds__(kMoveWarps * 32) evict_move_kernel(EvictArgs a, int per_cta, int in_place)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int s = blockIdx.x / sh.n_kv_heads;
    const int64_t n64 = a.seq_lens[s];
    const int n = (int)(n64 < 0 ? 0 : (n64 > sh.max_tokens ? sh.max_tokens : n64));
    const int left = n < a.n_keep ? n : a.n_keep;
    if (threadIdx.x == 0 && blockIdx.y == 0 && blockIdx.x % sh.n_kv_heads == 0) a.lens_out[s] = left;
    const int n_out = (left + kTokenBlock - 1) / kTokenBlock, first = blockIdx.y * per_cta;
    const int last = first + per_cta < n_out ? first + per_cta : n_out;
    const int64_t out_blocks = (a.out_tokens + kTokenBlock - 1) / kTokenBlock;
    const int32_t* kept = a.kept + (int64_t)blockIdx.x * a.n_keep;
    const float* mass = a.mass + (int64_t)blockIdx.x * sh.max_tokens;
    float* mass_out = a.mass_out + (int64_t)blockIdx.x * a.out_tokens;
    const int64_t from = (int64_t)blockIdx.x * sh.n_blocks * sh.block_bytes, to = (int64_t)blockIdx.x * out_blocks * sh.block_bytes;
    const int words = 2 * sh.G;                                               // (tensor, group) of a block
    for (int b0 = first; b0 < last; b0 += kMoveWarps) {
        const int ob = b0 + warp;
        const int j = ob * kTokenBlock + (lane & 15);
        const int idx = ob < last && j < left ? kept[j] : -1;                 // lane k and k + 16: source of token k
        const float m = idx >= 0 ? mass[idx] : 0.f;
        for (int w0 = 0; w0 < words; w0 += 32) {
            const int w = w0 + lane, tensor = w >= sh.G, g = tensor ? w - sh.G : w;
            const bool live = ob < last && w < words;
            const uint8_t* src = (tensor ? a.vc : a.kc) + from;
            uint32_t lo[4] = {0u, 0u, 0u, 0u}, hi[4] = {0u, 0u, 0u, 0u};
#pragma unroll
            for (int k = 0; k < kTokenBlock; ++k) {
                const int t = __shfl_sync(0xffffffffu, idx, k);
                if (live && t >= 0) {
                    const uint8_t* blk = src + (int64_t)(t / kTokenBlock) * sh.block_bytes;
                    lo[k >> 2] |= (uint32_t)blk[g * kTokenBlock + t % kTokenBlock] << (8 * (k & 3));
                    if (sh.hb) {
                        const uint32_t high = (uint32_t)read_code(blk, sh, g, t % kTokenBlock) >> 8;
                        const int bit = k * sh.hb;
#pragma unroll
                        for (int e = 0; e < 4; ++e)                           // (token k's bits never straddle a byte)
                            if (e == bit >> 5) hi[e] |= high << (bit & 31);
                    }
                }
            }
            if (in_place) __syncthreads();
            if (live) {
                uint8_t* dst = (tensor ? a.v_out : a.k_out) + to + (int64_t)ob * sh.block_bytes;
                if (sh.hb == 0) {
                    *reinterpret_cast<uint4*>(dst + g * kTokenBlock) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
                } else {                                                      // blocks of wide codes start at even bytes
#pragma unroll
                    for (int e = 0; e < kTokenBlock; e += 2) {
                        *reinterpret_cast<uint16_t*>(dst + g * kTokenBlock + e) = (uint16_t)(lo[e >> 2] >> (8 * (e & 2)));
                        if (e < 2 * sh.hb)
                            *reinterpret_cast<uint16_t*>(dst + sh.G * kTokenBlock + g * 2 * sh.hb + e) = (uint16_t)(hi[e >> 2] >> (8 * (e & 2)));
                    }
                }
            }
        }
        if (lane < kTokenBlock && idx >= 0) mass_out[j] = m;
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st)
{
    const int64_t items = a.sh.n_seq * a.sh.n_kv_heads;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)items, kSelectThreads, 0, st, &attr);
    cudaError_t e;
    if (a.sh.max_tokens <= 4 * kSelectThreads) e = cudaLaunchKernelEx(&cfg, evict_select_kernel<4>, a);
    else if (a.sh.max_tokens <= 16 * kSelectThreads) e = cudaLaunchKernelEx(&cfg, evict_select_kernel<16>, a);
    else if (a.sh.max_tokens <= 32 * kSelectThreads) e = cudaLaunchKernelEx(&cfg, evict_select_kernel<32>, a);
    else e = cudaLaunchKernelEx(&cfg, evict_select_kernel<0>, a);
    if (e != cudaSuccess) return e;
    const int in_place = a.k_out == a.kc;
    const int64_t most = a.n_keep < a.sh.max_tokens ? a.n_keep : a.sh.max_tokens;
    const int n_out = (int)((most + kTokenBlock - 1) / kTokenBlock);
    int per_cta = in_place ? n_out : 4 * kMoveWarps;
    while ((n_out + per_cta - 1) / per_cta > 65535) per_cta *= 2;
    cudaLaunchAttribute attr2;
    cudaLaunchConfig_t move = overlapped_config((unsigned)items, kMoveWarps * 32, 0, st, &attr2);
    move.gridDim = dim3((unsigned)items, (unsigned)((n_out + per_cta - 1) / per_cta));
    return cudaLaunchKernelEx(&move, evict_move_kernel, a, per_cta, in_place);
}

}  // namespace cq
