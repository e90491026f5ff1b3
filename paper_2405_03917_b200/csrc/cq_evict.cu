// Eviction from a coded cache by accumulated attention weight.
//
// Per (sequence, head): of n cached tokens stay the n_sinks first, the n_recent last and, of the others, those of largest mass
// (equal masses: the lower position), n_keep in all; codes and masses move to positions 0, 1, ... in their old order.
//
//   evict_select_kernel  one CTA per (sequence, head): the masses become whole numbers of the same order, kept in registers.  The
//       last one that stays is found by two histograms of 8 bits in shared memory; the few tokens that share these 16 bits with it are
//       then ranked against each other, and the positions that stay are listed in order (ballots in a warp, one scan over the warps).
//       Masses crowd in few bins: every lane counts in a column of its own, so that the lanes of a warp never meet.  What bounds it is
//       the number of instructions per token: 32 sequences x 40 heads of 8192 ... 32768 tokens: 345 us with a shared column per bin
//       and all 32 bits by histograms, 280 us with columns of their own and masses read again for every pass, 161 us with masses in
//       registers, room for the longest, 117 us with a loop for each of three lengths (105 MB of masses: 16 us).  Capacities above 32768
//       do not fit the registers: 16 x 40 heads of 32768 tokens 208 us at that capacity, 317 us at 32784, move included.
//   evict_move_kernel    a warp per 16 tokens that stay: a lane takes one (tensor, group) of them, a byte load per token (the
//       lanes of a load read one token's codes: whole 16-token blocks pass through L1), and writes one 16-byte word.
//       186 us for the same call: it keeps 4096 of some 20000 tokens, and of ten 16-token blocks nine hold one that stays, so that
//       nearly all codes are read (176 us with what is written, at the copy rate).
//       (16-byte words of the source blocks instead, their bytes shifted in one by one: 268 us.)
//       In place a CTA goes through its (sequence, head) in order: positions only ever move down, and all reads of a turn are done
//       before its writes: the same call takes 322 us in place, 303 into another cache (8 heads of 4097 tokens 29 and 11).
#include "cq_bounded.cuh"

namespace cq {

namespace {

constexpr int kBins = 256;

// Whole number of the same order as the mass, never zero: any NaN above all numbers (a sum with a NaN is the canonical one, which is
// positive), the two zeros alike.
__device__ __forceinline__ uint32_t mass_key(float m)
{
    const uint32_t u = __float_as_uint(__fadd_rn(m, 0.f));
    return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}

// Shared memory of a selecting CTA.
template <int kThreads>
struct SelectShared {
    static constexpr int kFewMost = kThreads;        // tokens that are ranked against each other
    uint32_t hist[kBins][32];                        // later: the keys that are ranked
    uint32_t count[kBins];
    uint32_t found[3];                               // the digit of the last one that stays, tokens above it, tokens with it
    uint32_t few;
    uint32_t warp_above[32], warp_equal[32];
};

// Of the tokens c_lo ... c_hi - 1, the `need` that stay (fewer than there are), to `kept`.
template <int kThreads, int kEach>
__device__ __forceinline__ void select_tokens(const float* mass, int c_lo, int c_hi, uint32_t need, int32_t* kept, SelectShared<kThreads>& sm)
{
    constexpr int kWarps = kThreads / 32;
    auto& hist = sm.hist;
    auto& count = sm.count;
    auto& found = sm.found;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    // warp w goes through the tokens from c_lo + w * turns * 32 on, turn j of lane l takes token j * 32 + l of them
    const int turns = (c_hi - c_lo + kThreads - 1) / kThreads;
    const int base = c_lo + warp * turns * 32 + lane;
    auto load = [&](int j) {                                                  // 0: no token (no mass has that key)
        const int t = base + 32 * j;
        return j < turns && t < c_hi ? mass_key(mass[t]) : 0u;
    };
    uint32_t key[kEach ? kEach : 1];
    if (kEach) {
#pragma unroll
        for (int j = 0; j < kEach; ++j) key[j] = load(j);
    }
    auto each = [&](auto&& use) {                                             // use(turn, key) for the warp's tokens, in order
        if (kEach) {
#pragma unroll
            for (int j = 0; j < kEach; ++j)
                if (j < turns) use(j, key[kEach ? j : 0]);
        } else {
            for (int j = 0; j < turns; ++j) use(j, load(j));
        }
    };
    // Keys above `least` stay, and of those that equal it the first `need`; or (all) every key from `least` on.
    bool all = false;
    uint32_t least = 0u, mask = 0u;
    auto digit = [&](int shift) {                                             // finds the next eight bits
        for (int i = threadIdx.x; i < kBins * 32; i += kThreads) (&hist[0][0])[i] = 0u;
        __syncthreads();
        each([&](int, uint32_t k) {
            if (k != 0u && (k & mask) == least) atomicAdd(&hist[(k >> shift) & (kBins - 1)][lane], 1u);
        });
        __syncthreads();
        for (int bin = warp; bin < kBins; bin += kWarps) {
            const uint32_t sum = __reduce_add_sync(0xffffffffu, hist[bin][lane]);
            if (lane == 0) count[bin] = sum;
        }
        __syncthreads();
        if (warp == 0) {                                                      // lane l: bins 8 l ... 8 l + 7, counted from the top
            uint32_t c[8], mine = 0u;
#pragma unroll
            for (int i = 0; i < 8; ++i) { c[i] = count[kBins - 1 - (8 * lane + i)]; mine += c[i]; }
            uint32_t before = mine;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const uint32_t x = __shfl_up_sync(0xffffffffu, before, o);
                if (lane >= o) before += x;
            }
            before -= mine;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if (before < need && need <= before + c[i]) {
                    found[0] = (uint32_t)(kBins - 1 - (8 * lane + i));
                    found[1] = before;
                    found[2] = c[i];
                }
                before += c[i];
            }
        }
        __syncthreads();
        least |= found[0] << shift;
        mask |= 0xffu << shift;
        need -= found[1];
        all = need == found[2];                                               // the digits so far tell those that stay from the others
        __syncthreads();
    };
    // (one copy of the unrolled loop for all digits: the instructions of four came late, 307 against 303 us and 24.6 against 22.0)
#pragma unroll 1
    for (int shift = 24;; shift -= 8) {
        digit(shift);
        if (all || shift == 0 || (shift <= 16 && found[2] <= SelectShared<kThreads>::kFewMost)) break;
    }
    if (!all && mask != 0xffffffffu) {
        // few share the digits: each is ranked against the others
        uint32_t* keys = &hist[0][0];
        if (threadIdx.x == 0) sm.few = 0u;
        __syncthreads();
        each([&](int, uint32_t k) {
            if ((k & mask) == least) keys[atomicAdd(&sm.few, 1u)] = k;           // (not 0: `least` has its highest digits)
        });
        __syncthreads();
        const uint32_t total = sm.few;
        if (threadIdx.x < total) {
            const uint32_t k = keys[threadIdx.x];
            uint32_t above = 0u, equal = 0u;
            for (uint32_t i = 0; i < total; ++i) {
                const uint32_t other = keys[i];
                above += other > k;
                equal += other == k;
            }
            if (above < need && need <= above + equal) {                      // (all that write here hold the same key)
                found[0] = k;
                found[1] = above;
                found[2] = equal;
            }
        }
        __syncthreads();
        least = found[0];
        need -= found[1];
        all = need == found[2];
    }
    if (all) --least;                                                         // those from `least` on are those above the number before it
    uint32_t n_above = 0u, n_equal = 0u;
    each([&](int, uint32_t k) {
        n_above += k > least;
        if (!all) n_equal += k == least;
    });
    n_above = __reduce_add_sync(0xffffffffu, n_above);
    n_equal = __reduce_add_sync(0xffffffffu, n_equal);
    if (lane == 0) { sm.warp_above[warp] = n_above; sm.warp_equal[warp] = n_equal; }
    __syncthreads();
    uint32_t above_before = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_above[lane] : 0u);
    uint32_t equal_before = __reduce_add_sync(0xffffffffu, lane < warp ? sm.warp_equal[lane] : 0u);
    const uint32_t below = (1u << lane) - 1u;
    if (all) {
        each([&](int j, uint32_t k) {
            const bool above = k > least;
            const uint32_t ab = __ballot_sync(0xffffffffu, above);
            if (above) kept[above_before + __popc(ab & below)] = base + 32 * j;
            above_before += __popc(ab);
        });
    } else {
        each([&](int j, uint32_t k) {
            const bool above = k > least, equal = k == least;
            const uint32_t eq = __ballot_sync(0xffffffffu, equal), ab = __ballot_sync(0xffffffffu, above);
            const uint32_t e = equal_before + __popc(eq & below);
            if (above || (equal && e < need)) kept[above_before + __popc(ab & below) + (e < need ? e : need)] = base + 32 * j;
            above_before += __popc(ab);
            equal_before += __popc(eq);
        });
    }
}

// kEach: masses a thread keeps in registers (0: they are read again from memory for every pass), kCtas: CTAs of an SM.  The unrolled loops are
// those of the smallest of three numbers of turns that the sequence needs: 32 x 40 heads of 8192 ... 32768 tokens, move included, 347 us
// with 32 turns for all, 303 with 16, 24 and 32 (two or four more: slower by 1 %, the code grows); 8 heads of 4097 tokens 13.9 and 10.8 us.
// (Upper halves of the keys in shared memory and two CTAs on an SM: 388 us.  One kernel that selects and moves: 408 us.)
template <int kThreads, int kEach, int kCtas>
__global__ void __launch_bounds__(kThreads, kCtas) evict_select_kernel(EvictArgs a)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    __shared__ SelectShared<kThreads> sm;
    const int s = blockIdx.x / a.sh.n_kv_heads;
    const int64_t n64 = a.seq_lens[s];
    const int n = (int)(n64 < 0 ? 0 : (n64 > a.sh.max_tokens ? a.sh.max_tokens : n64));
    const float* mass = a.mass + (int64_t)blockIdx.x * a.sh.max_tokens;
    int32_t* kept = a.kept + (int64_t)blockIdx.x * a.n_keep;
    if (n <= a.n_keep) {
        for (int j = threadIdx.x; j < a.n_keep; j += kThreads) kept[j] = j < n ? j : -1;
        return;
    }
    const int c_lo = a.n_sinks, c_hi = n - a.n_recent;                        // the tokens that compete
    for (int j = threadIdx.x; j < a.n_sinks; j += kThreads) kept[j] = j;
    for (int j = threadIdx.x; j < a.n_recent; j += kThreads) kept[a.n_keep - a.n_recent + j] = c_hi + j;
    kept += a.n_sinks;
    const uint32_t need = (uint32_t)(a.n_keep - a.n_sinks - a.n_recent);
    if (need == 0u) return;
    const int turns = (c_hi - c_lo + kThreads - 1) / kThreads;
    if constexpr (kEach > 4) {
        constexpr int kLow = kEach == 32 ? 16 : kEach / 4, kMid = kEach == 32 ? 24 : kEach / 2;
        if (turns <= kLow) return select_tokens<kThreads, kLow>(mass, c_lo, c_hi, need, kept, sm);
        if (turns <= kMid) return select_tokens<kThreads, kMid>(mass, c_lo, c_hi, need, kept, sm);
    }
    select_tokens<kThreads, kEach>(mass, c_lo, c_hi, need, kept, sm);
}

constexpr int kMoveWarps = 8;

// One CTA: out blocks blockIdx.y * per_cta ... of (sequence, head) blockIdx.x; in place one CTA takes them all.
// kHigh: codes wider than a byte; kInPlace.
template <bool kHigh, bool kInPlace>
__global__ void __launch_bounds__(kMoveWarps * 32) evict_move_kernel(EvictArgs a, int per_cta)
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
        const bool there = ob < last && j < left;
        const int idx = there ? kept[j] : 0;                                  // lanes k and k + 16: the source of token k (none: any)
        const int64_t at = (int64_t)(idx / kTokenBlock) * sh.block_bytes + idx % kTokenBlock;
        const uint32_t none = __ballot_sync(0xffffffffu, !there) & 0xffffu;
        const float m = there ? mass[idx] : 0.f;
        for (int w0 = 0; w0 < words; w0 += 32) {
            const int w = w0 + lane, tensor = w >= sh.G, g = tensor ? w - sh.G : w;
            const bool live = ob < last && w < words;
            const uint8_t* src = (tensor ? a.vc : a.kc) + from + (live ? g * kTokenBlock : 0);
            uint32_t lo[4] = {0u, 0u, 0u, 0u}, hi[4] = {0u, 0u, 0u, 0u};
            if (ob < last) {
                uint32_t byte[kTokenBlock];
#pragma unroll
                for (int k = 0; k < kTokenBlock; ++k) byte[k] = src[__shfl_sync(0xffffffffu, at, k)];
#pragma unroll
                for (int k = 0; k < kTokenBlock; k += 4)
                    lo[k >> 2] = __byte_perm(__byte_perm(byte[k], byte[k + 1], 0x0040), __byte_perm(byte[k + 2], byte[k + 3], 0x0040), 0x5410);
                if (none) {                                                   // behind the last token: zeros
#pragma unroll
                    for (int k = 0; k < kTokenBlock; ++k)
                        if ((none >> k) & 1u) lo[k >> 2] &= ~(0xffu << (8 * (k & 3)));
                }
                if (kHigh) {
#pragma unroll
                    for (int k = 0; k < kTokenBlock; ++k) {
                        const int t = __shfl_sync(0xffffffffu, idx, k);
                        if (!live || ((none >> k) & 1u)) continue;
                        const uint8_t* blk = (tensor ? a.vc : a.kc) + from + (int64_t)(t / kTokenBlock) * sh.block_bytes;
                        const uint32_t high = (uint32_t)read_code(blk, sh, g, t % kTokenBlock) >> 8;
                        const int bit = k * sh.hb;
#pragma unroll
                        for (int e = 0; e < 4; ++e)                           // (token k's bits never straddle a byte)
                            if (e == bit >> 5) hi[e] |= high << (bit & 31);
                    }
                }
            }
            if (kInPlace) __syncthreads();
            if (live) {
                uint8_t* dst = (tensor ? a.v_out : a.k_out) + to + (int64_t)ob * sh.block_bytes;
                if (!kHigh) {
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
        if (lane < kTokenBlock && there) mass_out[j] = m;
    }
}

}  // namespace

cudaError_t launch_evict(const EvictArgs& a, cudaStream_t st)
{
    const int64_t items = a.sh.n_seq * a.sh.n_kv_heads;
    auto go = [&](auto kernel, int threads) {
        cudaLaunchAttribute attr;
        const cudaLaunchConfig_t cfg = overlapped_config((unsigned)items, threads, 0, st, &attr);
        return cudaLaunchKernelEx(&cfg, kernel, a);
    };
    // By capacity; where short ones are many, smaller CTAs, four on an SM: 32 x 32 heads of 500 ... 1000 tokens 22.0 us (one CTA 39.5, two of
    // 1024 threads 32.1), 64 x 32 heads 40.2 (76, 61), move included.
    const int64_t cap = a.sh.max_tokens;
    const cudaError_t e = cap <= 4096 ? (items >= 2 * device_sm_count() ? go(evict_select_kernel<512, 8, 4>, 512) : go(evict_select_kernel<1024, 4, 1>, 1024))
                          : cap <= 16384 ? go(evict_select_kernel<1024, 16, 1>, 1024)
                          : cap <= 32768 ? go(evict_select_kernel<1024, 32, 1>, 1024) : go(evict_select_kernel<1024, 0, 1>, 1024);
    if (e != cudaSuccess) return e;
    const bool in_place = a.k_out == a.kc;
    const int64_t most = a.n_keep < a.sh.max_tokens ? a.n_keep : a.sh.max_tokens;
    const int n_out = (int)((most + kTokenBlock - 1) / kTokenBlock);
    int per_cta = in_place ? n_out : 4 * kMoveWarps;
    while ((n_out + per_cta - 1) / per_cta > 65535) per_cta *= 2;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = overlapped_config((unsigned)items, kMoveWarps * 32, 0, st, &attr);
    cfg.gridDim = dim3((unsigned)items, (unsigned)((n_out + per_cta - 1) / per_cta));
    if (a.sh.hb) return in_place ? cudaLaunchKernelEx(&cfg, evict_move_kernel<true, true>, a, per_cta) : cudaLaunchKernelEx(&cfg, evict_move_kernel<true, false>, a, per_cta);
    return in_place ? cudaLaunchKernelEx(&cfg, evict_move_kernel<false, true>, a, per_cta) : cudaLaunchKernelEx(&cfg, evict_move_kernel<false, false>, a, per_cta);
}

}  // namespace cq
