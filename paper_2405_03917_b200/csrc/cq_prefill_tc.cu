// Tensor-core kernel of the attention of many query rows over a coded cache (head_dim 128, one byte per code): device code shared
// by the causal attention over a contiguous cache (cq_prefill.cu) and by the operators on bounded caches (cq_chunk_attn.cu), which include
// this file; it is not compiled by itself.
#pragma once

#include <type_traits>

#include "cq_bounded.cuh"

namespace cq {

namespace {

// kParts: softmax threads of a row, each with as many of its columns.
template <int kParts>
struct PfCfgT {
    static constexpr int kRows = 256;             // (query, head) rows per CTA: two tiles of 128, one tensor-memory lane each
    static constexpr int kSoftWarps = 8 * kParts; // softmax: four per row tile and part, a thread per row (and part)
    static constexpr int kMmaWarp = kSoftWarps;   // one thread issues the MMAs
    static constexpr int kProducerWarp0 = kMmaWarp + 1, kProducerWarps = 4;       // dequantise the tiles
    static constexpr int kSumWarp = kProducerWarp0 + kProducerWarps;
    static constexpr int kThreads = (kSumWarp + 1) * 32;
    static constexpr int kTile = 64;              // cached tokens per step
    static constexpr int kStages = 3;
    static constexpr int kCbBytes = 128 * 256 * 2;                     // one codebook as fp16, code-major
    static constexpr int kKcbOffset = 0, kVcbOffset = kCbBytes;
    static constexpr int kHalfBytes = kTile * 128;                     // 64 channels of a tile: rows of 128 bytes, one per token
    static constexpr int kTileBytes = 2 * kHalfBytes;
    static constexpr int kVtOffset = 2 * kCbBytes;                     // [stages]
    static constexpr int kKtOffset = kVtOffset + kStages * kTileBytes; // [stages]
    static constexpr int kCtlOffset = kKtOffset + kStages * kTileBytes;
    static constexpr int kExchangeOffset = kCtlOffset + 256;           // two parts: [part][row] what the threads of a row tell each other
    static constexpr int kSmemBytes = kExchangeOffset + (kParts > 1 ? kParts * kRows * 4 : 0);      // 224.25 KiB, 226.25 with two parts
    // tensor-memory columns: output accumulators (fp32) and queries (fp16, two per column) of both row tiles, ONE tile of
    // scores (fp32) that the row tiles use in turn, weights (fp16) of both row tiles
    static constexpr int kOCol = 0, kQCol = 256, kSCol = 384, kPCol = 448;
    // where the set-up leaves the queries: behind stage 0, which the producers fill while they are read
    static constexpr int kOutStride = 144;        // bytes between the rows of a warp's 32 x 32 block of results (in the codebooks' place)
    __host__ __device__ static constexpr int q_offset(int rho) { return (rho < 128 ? kVtOffset : kKtOffset) + kTileBytes + (rho & 127) * 256; }
    static_assert(kStages >= 3 && kSoftWarps * 32 * kOutStride <= 2 * kCbBytes, "room");
    static_assert(kKtOffset % 1024 == 0 && kTileBytes % 1024 == 0, "swizzled tiles");
    static_assert(kSmemBytes <= 227 * 1024, "shared memory");
};

using PfCfg = PfCfgT<1>;
using PfCfgB = PfCfgT<2>;                 // the bounded form

constexpr int kPfLeastShare = 4;          // tiles of a CTA's part of a context, at least

struct PfCtl {
    uint64_t full[PfCfg::kStages];        // K and V tile of the stage are written (one arrival per producer warp)
    uint64_t empty[PfCfg::kStages];       // the MMAs that read the stage are done
    uint64_t s_full[2];                   // scores of the row tile are in tensor memory
    uint64_t s_free[2];                   // they have been read (one arrival per warp): their columns take the other row tile's
    uint64_t q_full[2];                   // queries of the row tile are in tensor memory (one arrival per warp)
    uint64_t p_full[2];                   // its weights are (one arrival per warp)
    uint64_t pv_done[2];                  // the sums with those weights are done
    uint64_t drained[2];                  // every MMA of the warp that issues the scores / the sums is done
    uint32_t tmem_base;
    int failed;                           // a wait gave up
    alignas(4) uint8_t hole[PfCfg::kStages][4];      // bounded: the 16-token block of the stage lies in no page
    int found, number;                    // bounded: this CTA's sequence and row tile
};
static_assert(sizeof(PfCtl) <= 256, "control block");

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// 2^x by the special-function unit (two units in the last place; P is rounded to fp16 afterwards)
__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}

__device__ __forceinline__ void pf_init(uint64_t* bar, int arrivals)
{
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(bar)), "r"(arrivals) : "memory");
}
__device__ __forceinline__ void pf_arrive(uint64_t* bar)
{
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Waits for the phase with the given parity; gives up after a bounded number of polls, or when another wait has, and then
// returns false: the other roles leave their loops (by a vote: the lanes of a warp can come out of it with different
// answers), the softmax warps run through theirs, in step and for nothing, and their rows become NaN.
#ifndef CQ_PREFILL_POLLS
#define CQ_PREFILL_POLLS (1 << 17)
#endif
__device__ __forceinline__ bool pf_wait(PfCtl* ctl, uint64_t* bar, uint32_t parity)
{
    for (int poll = 0; poll < CQ_PREFILL_POLLS; ++poll) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
        if (done) return true;
        if ((poll & 63) == 63 && *reinterpret_cast<volatile int*>(&ctl->failed)) return false;
    }
    ctl->failed = 1;
    return false;
}
// Whether a wait of the CTA has given up.  Who has not waited arrives too early: from then on a barrier says nothing about the other threads' data
// either.  (The word is written before such an arrival, so whoever reads on because of one finds it.)
__device__ __forceinline__ bool pf_failed(const PfCtl* ctl) { return *reinterpret_cast<const volatile int*>(&ctl->failed) != 0; }

// Shared-memory matrix descriptor of a tile of 128-byte rows with the 128-byte swizzle (16-byte chunk index XOR row mod 8).
// Rows = tokens.  As keys (contraction along the row) eight rows are one core matrix group of 1024 bytes; as values (the
// row is the N dimension) the next 64 channels are kHalfBytes on and the next eight tokens 1024 bytes.  Low word: start
// address and leading offset in 16-byte units; high word: stride offset, descriptor version of sm_100, swizzle.
__device__ __forceinline__ uint32_t pf_desc_lo(uint32_t saddr, uint32_t leading_bytes) { return (saddr >> 4) | ((leading_bytes >> 4) << 16); }
constexpr uint32_t kPfDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);
// D[128 x N] (+)= A[128 x 16] * B, A (fp16) from tensor memory, B (fp16) from shared memory, fp32 accumulator
__device__ __forceinline__ void pf_mma(uint32_t d_tmem, uint32_t a_tmem, uint32_t b_lo, uint32_t idesc, bool accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\t.reg .b64 d;\n\tsetp.ne.b32 p, %5, 0;\n\tmov.b64 d, {%2, %3};\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], d, %4, p;\n\t}"
                 ::"r"(d_tmem), "r"(a_tmem), "r"(b_lo), "r"(kPfDescHi), "r"(idesc), "r"(accumulate ? 1u : 0u) : "memory");
}
// One lane of the warp, the same one every time.  (A branch on this, unlike one on the lane number, lets the compiler keep
// the operands of the MMAs in uniform registers: an issue costs some ten cycles instead of seventy.)
__device__ __forceinline__ bool pf_elect()
{
    uint32_t is;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(is));
    return is != 0;
}
__device__ __forceinline__ void pf_commit(uint64_t* bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// Waits, also after another wait has given up, until the MMAs that this warp has issued are done with shared memory and
// tensor memory: the CTA gives both back next.
__device__ __forceinline__ void pf_drain(uint64_t* bar)
{
    if (pf_elect()) pf_commit(bar);
    for (int poll = 0; poll < (1 << 20); ++poll) {
        uint32_t done;
        asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], 0;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                     : "=r"(done) : "r"(smem_u32(bar)) : "memory");
        if (done) break;
    }
    __syncwarp();
}

#define CQ_R32(u) "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]), "=r"(u[4]), "=r"(u[5]), "=r"(u[6]), "=r"(u[7]), "=r"(u[8]), "=r"(u[9]), "=r"(u[10]), "=r"(u[11]), "=r"(u[12]), "=r"(u[13]), "=r"(u[14]), "=r"(u[15]), "=r"(u[16]), "=r"(u[17]), "=r"(u[18]), "=r"(u[19]), "=r"(u[20]), "=r"(u[21]), "=r"(u[22]), "=r"(u[23]), "=r"(u[24]), "=r"(u[25]), "=r"(u[26]), "=r"(u[27]), "=r"(u[28]), "=r"(u[29]), "=r"(u[30]), "=r"(u[31])
#define CQ_RW32(u) "+r"(u[0]), "+r"(u[1]), "+r"(u[2]), "+r"(u[3]), "+r"(u[4]), "+r"(u[5]), "+r"(u[6]), "+r"(u[7]), "+r"(u[8]), "+r"(u[9]), "+r"(u[10]), "+r"(u[11]), "+r"(u[12]), "+r"(u[13]), "+r"(u[14]), "+r"(u[15]), "+r"(u[16]), "+r"(u[17]), "+r"(u[18]), "+r"(u[19]), "+r"(u[20]), "+r"(u[21]), "+r"(u[22]), "+r"(u[23]), "+r"(u[24]), "+r"(u[25]), "+r"(u[26]), "+r"(u[27]), "+r"(u[28]), "+r"(u[29]), "+r"(u[30]), "+r"(u[31])
#define CQ_IN32(u) "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]), "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]), "r"(u[16]), "r"(u[17]), "r"(u[18]), "r"(u[19]), "r"(u[20]), "r"(u[21]), "r"(u[22]), "r"(u[23]), "r"(u[24]), "r"(u[25]), "r"(u[26]), "r"(u[27]), "r"(u[28]), "r"(u[29]), "r"(u[30]), "r"(u[31])
// 32 consecutive columns of this thread's row (the values are there after pf_ld_wait, whose registers pass through it)
__device__ __forceinline__ void pf_ld32(uint32_t (&u)[32], uint32_t taddr)
{
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : CQ_R32(u) : "r"(taddr) : "memory");
}
__device__ __forceinline__ void pf_ld_wait(uint32_t (&u)[32]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : CQ_RW32(u)::"memory"); }
__device__ __forceinline__ void pf_st32(uint32_t taddr, const uint32_t (&u)[32])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
                 ::"r"(taddr), CQ_IN32(u) : "memory");
}
__device__ __forceinline__ void pf_st16(uint32_t taddr, const uint32_t (&u)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(taddr), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]), "r"(u[4]), "r"(u[5]), "r"(u[6]), "r"(u[7]), "r"(u[8]), "r"(u[9]), "r"(u[10]),
                 "r"(u[11]), "r"(u[12]), "r"(u[13]), "r"(u[14]), "r"(u[15]) : "memory");
}
__device__ __forceinline__ void pf_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void pf_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void pf_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// The bounded form: windows, sinks, pages, ragged rows, fp16 codebooks and results, contexts split over CTAs.  kPfLse and kPfMass do the
// scores alone: the first leaves the log-sum-exp of every row, as (reference, sum) of every part of its context; the second adds up,
// per token, the weights of a row tile's rows.
enum PfWhat { kPfNone, kPfAttn, kPfLse, kPfMass };
struct PfNone {
    static constexpr int kWhat = kPfNone;
};
template <int kWhatFor>
struct PfBounded {
    static constexpr int kWhat = kWhatFor;
    BoundedArgs a;
    int tiles;                 // bound on the row tiles of all sequences
    int parts;                 // CTAs that share a row tile's context
    float* partials;           // attention, parts > 1: [CTA][256 rows][partial_stride(128)] (reference, sum, accumulators);
                               // log-sum-exps: [CTA][256 rows][2] (reference NaN: a wait gave up)
    const float* mass_in;      // masses: of one row tile per sequence, on top of these (may be null)
    float* mass_out;           // [sequence][KV head][max_tokens]; of several row tiles, [row tile][sequence][KV head][max_tokens]
    int row_tiles;
};
// Row tiles of a sequence.
__device__ __forceinline__ int pf_tiles_of(const BoundedArgs& a, const SeqView& v, int q_per_tile)
{
    const int rows = v.m * a.sh.R;
    return rows < a.least_rows || rows > a.most_rows ? 0 : (v.m + q_per_tile - 1) / q_per_tile;
}
// The sequence that row tile `index` of all belongs to (-1: none) and its number there.  Entered by whole warps; the same in all lanes.
// With as many new tokens in every sequence: a division.  Otherwise up to kPfSorted sequences are taken in the order of their lengths,
// the longest first (a row tile of a long one started last would keep its SM busy alone: 24 sequences of 600 to 9001 tokens with 1 to
// 512 new ones, 306 ... 355 us; side by side 307, and 395 in their own order); of more than that, whose row tiles fill the GPU many times over, the counts alone are
// looked at, for the comparison takes a CTA some ten cycles per sequence (2 us at 64).
constexpr int kPfSorted = 64;
__device__ __forceinline__ int pf_find_tile(const BoundedArgs& a, int index, int q_per_tile, int& tile)
{
    const int lane = threadIdx.x & 31, n_seq = (int)a.sh.n_seq;
    if (!a.q_offsets) {
        const int each = (a.max_q + q_per_tile - 1) / q_per_tile;
        tile = index % each;
        return index / each < n_seq ? index / each : -1;
    }
    if (n_seq <= kPfSorted) {
        int len[2], tiles[2], before[2] = {0, 0};
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const SeqView v = seq_view(a, lane + 32 * k < n_seq ? lane + 32 * k : 0);
            len[k] = v.n;
            tiles[k] = lane + 32 * k < n_seq ? pf_tiles_of(a, v, q_per_tile) : 0;
        }
        for (int j = 0; j < n_seq; ++j) {
            const int len_j = __shfl_sync(0xffffffffu, j < 32 ? len[0] : len[1], j & 31);
            const int tiles_j = __shfl_sync(0xffffffffu, j < 32 ? tiles[0] : tiles[1], j & 31);
#pragma unroll
            for (int k = 0; k < 2; ++k) before[k] += len_j > len[k] || (len_j == len[k] && j < lane + 32 * k) ? tiles_j : 0;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            const uint32_t hit = __ballot_sync(0xffffffffu, index >= before[k] && index < before[k] + tiles[k]);
            if (hit) {
                tile = index - __shfl_sync(0xffffffffu, before[k], __ffs(hit) - 1);
                return 32 * k + __ffs(hit) - 1;
            }
        }
        return -1;
    }
    for (int s0 = 0; s0 < n_seq; s0 += 32) {
        const int mine = s0 + lane < n_seq ? pf_tiles_of(a, seq_view(a, s0 + lane), q_per_tile) : 0;
        int incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int x = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += x;
        }
        const uint32_t hit = __ballot_sync(0xffffffffu, index >= incl - mine && index < incl);
        if (hit) {
            const int l = __ffs(hit) - 1;
            tile = index - __shfl_sync(0xffffffffu, incl - mine, l);
            return s0 + l;
        }
        index -= __shfl_sync(0xffffffffu, incl, 31);
    }
    return -1;
}

// Of the threads of a warp pair (barrier `id`): whether any says so.
__device__ __forceinline__ bool pf_pair_any(int id, bool q)
{
    uint32_t any;
    asm volatile("{\n\t.reg .pred p, r;\n\tsetp.ne.b32 p, %1, 0;\n\tbarrier.cta.red.or.pred r, %2, 64, p;\n\tselp.u32 %0, 1, 0, r;\n\t}"
                 : "=r"(any) : "r"((uint32_t)q), "r"(id) : "memory");
    return any != 0;
}
__device__ __forceinline__ void pf_pair_sync(int id) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(id) : "memory"); }

template <int kC, class Bounded = PfNone>
__global__ void __launch_bounds__(Bounded::kWhat == kPfNone ? PfCfg::kThreads : PfCfgB::kThreads, 1)
prefill_tc_kernel(const __half* __restrict__ q, const uint8_t* __restrict__ kc, const uint8_t* __restrict__ vc,
                  const float* __restrict__ kcb, const float* __restrict__ vcb,
                  const int32_t* __restrict__ seq_lens, float scale_log2e, Shape sh, int n_q, int row_tiles,
                  float* __restrict__ out, Bounded bounded)
{
    constexpr int kWhat = Bounded::kWhat;
    constexpr bool kBounded = kWhat != kPfNone, kSums = kWhat == kPfNone || kWhat == kPfAttn;      // kSums: values and their sums
    asm volatile("griddepcontrol.wait;" ::: "memory");      // launched ahead of the end of the kernel before it, and
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");       // the kernel behind it ahead of its own
    using C = typename std::conditional<kBounded, PfCfgB, PfCfg>::type;
    constexpr int G = 128 / kC;
    extern __shared__ __align__(1024) uint8_t smem[];
    PfCtl* ctl = reinterpret_cast<PfCtl*>(smem + C::kCtlOffset);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int R = sh.R;
    const int q_per_tile = C::kRows / R;                                   // query tokens of one row tile

    int tile, hkv;
    int64_t s, n, q_first;                                                 // q_first: row of q that holds the sequence's first new token
    if constexpr (kBounded) {
        const int item = blockIdx.x / bounded.parts;
        hkv = item % sh.n_kv_heads;
        if (warp == 0) {
            int number = 0;
            ctl->found = pf_find_tile(bounded.a, item / sh.n_kv_heads, q_per_tile, number);      // (all lanes the same)
            ctl->number = number;
        }
        __syncthreads();
        const int found = ctl->found, number = ctl->number;
        if (found < 0) return;
        const SeqView sv = seq_view(bounded.a, found);
        s = found;
        n = sv.n;
        n_q = sv.m;
        q_first = sv.row0;
        tile = pf_tiles_of(bounded.a, sv, q_per_tile) - 1 - number;
    } else {
        tile = row_tiles - 1 - blockIdx.x % row_tiles;                     // later queries attend more tokens: they start first
        hkv = (blockIdx.x / row_tiles) % sh.n_kv_heads;
        s = blockIdx.x / ((int64_t)row_tiles * sh.n_kv_heads);
        n = seq_lens[s];
        n = n < 0 ? 0 : (n > sh.max_tokens ? sh.max_tokens : n);
        q_first = s * n_q;
    }
    const int qi0 = tile * q_per_tile;
    // row rho of the CTA: query qi0 + rho / R, head hkv * R + rho % R, position n - n_q + query
    const int64_t pos0 = n - n_q + qi0;                                    // position of the tile's first query (may be negative)
    int q_last = qi0 + q_per_tile - 1;
    if (q_last > n_q - 1) q_last = n_q - 1;
    const int64_t pos_last = n - n_q + q_last;                             // largest position of the tile
    int n_tiles = pos_last < 0 ? 0 : (int)(pos_last / C::kTile + 1);
    // bounded: the tiles that some row sees are those of the sinks, then from the first window on; this CTA's part of them
    int first_tile = 0, sink_tiles = 0, window_tile = 0;
    if constexpr (kBounded) {
        window_tile = window_first((int)pos0, bounded.a.window) / C::kTile;
        sink_tiles = bounded.a.window ? (bounded.a.sinks + C::kTile - 1) / C::kTile : 0;
        sink_tiles = sink_tiles < window_tile ? sink_tiles : window_tile;
        n_tiles = n_tiles ? sink_tiles + n_tiles - window_tile : 0;
        if (bounded.parts > 1) {
            int share = (n_tiles + bounded.parts - 1) / bounded.parts;
            share = share < kPfLeastShare ? kPfLeastShare : share;
            first_tile = share * (int)(blockIdx.x % bounded.parts);
            n_tiles = n_tiles - first_tile < share ? n_tiles - first_tile : share;
            n_tiles = n_tiles < 0 ? 0 : n_tiles;
        }
    }
    auto tile_at = [&](int jt) {                                            // the jt-th tile of this CTA
        if constexpr (!kBounded) return jt;
        const int i = first_tile + jt;
        return i < sink_tiles ? i : i - sink_tiles + window_tile;
    };
    const int n_halves = (q_last - qi0 + 1) * R > 128 ? 2 : 1;             // row tiles of 128 in use
    // (a negative scale: the queries change sign instead; a zero one: they become zero; both are exact)
    const uint32_t q_sign = scale_log2e < 0.f ? 0x80008000u : 0u, q_keep = scale_log2e == 0.f ? 0u : 0xffffffffu;
    const float scale = scale_log2e == 0.f ? 1.f : fabsf(scale_log2e);

    const int rows_used = q_per_tile * R;                                  // (bounded: R need not divide 256)

    // ---- barriers, tensor memory
    if (threadIdx.x == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            pf_init(&ctl->full[i], C::kProducerWarps);
            pf_init(&ctl->empty[i], 1);
        }
        for (int t = 0; t < 2; ++t) {
            pf_init(&ctl->s_full[t], 1);
            pf_init(&ctl->s_free[t], C::kSoftWarps / 2);
            pf_init(&ctl->q_full[t], C::kSoftWarps / 2);
            pf_init(&ctl->p_full[t], C::kSoftWarps / 2);
            pf_init(&ctl->pv_done[t], 1);
            pf_init(&ctl->drained[t], 1);
        }
        ctl->failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == C::kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(&ctl->tmem_base)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    // ---- queries, coalesced, into the tile buffers of stages 1 and 2 (row tile 0: the values', 1: the keys'); 16-byte chunk
    // i of row rho goes to chunk i XOR (rho mod 8) of its 256 bytes, so that a thread per row can read them without conflicts
#pragma unroll 4
    for (int i = threadIdx.x; i < n_halves * 128 * 16; i += C::kThreads) {
        const int rho = i >> 4, qi = qi0 + rho / R;
        uint4 x = make_uint4(0u, 0u, 0u, 0u);
        if (qi < n_q && (!kBounded || rho < rows_used))
            x = reinterpret_cast<const uint4*>(q + ((q_first + qi) * sh.n_q_heads + hkv * R + rho % R) * 128)[i & 15];
        *reinterpret_cast<uint4*>(smem + C::q_offset(rho) + (((i & 15) ^ (rho & 7)) << 4)) = x;
    }
    // ---- codebooks as fp16, code-major ([code][group][channel]): the lanes of a gather take different groups, so they
    // meet in no bank whatever the codes are.  For c = 2 (one word per centroid) group g sits in column
    // 16 (g mod 4) + g / 4.  A warp takes 64 bytes of eight groups at a time, a quarter of it two groups: two lines of
    // memory per quarter of a load, and at most four lanes that meet in a bank of a store.  (Straight copies, whose stores
    // met eight at a time, took 12.7 thousand cycles per CTA; 4 thousand are what the L2 takes to deliver 256 KB.)
    if constexpr (kBounded) {
        // fp16 as they come: a warp takes four centroids' 64 bytes (c = 8) of eight groups, a quarter of it two groups
        constexpr int kHalves = (G / 8) * (64 * kC / 8), kTasks = kSums ? 2 * kHalves : kHalves, kBatch = 6, kWarps = C::kThreads / 32;
        const int gl = lane >> 2, j = lane & 3, pieces = sh.K * kC / 8;     // 16-byte pieces of a group's codebook
#pragma unroll 1
        for (int i0 = warp; i0 < kTasks; i0 += kBatch * kWarps) {
            uint4 x[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u * kWarps, o = (i % kHalves) % (G / 8), piece = (i % kHalves) / (G / 8) * 4 + j;
                const int g = kC == 2 ? 4 * (8 * (o >> 2) + gl) + (o & 3) : 8 * o + gl;
                x[u] = make_uint4(0u, 0u, 0u, 0u);
                if (i < kTasks && piece < pieces)
                    x[u] = reinterpret_cast<const uint4*>((i < kHalves ? bounded.a.kcb : bounded.a.vcb) + ((int64_t)hkv * G + g) * sh.K * kC)[piece];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u * kWarps, o = (i % kHalves) % (G / 8), piece = (i % kHalves) / (G / 8) * 4 + j;
                if (i >= kTasks) break;
                uint8_t* book = smem + (i < kHalves ? C::kKcbOffset : C::kVcbOffset);
                if (kC == 8) *reinterpret_cast<uint4*>(book + piece * 256 + (8 * o + gl) * 16) = x[u];
                if (kC == 4) {
                    *reinterpret_cast<uint2*>(book + 2 * piece * 256 + (8 * o + gl) * 8) = make_uint2(x[u].x, x[u].y);
                    *reinterpret_cast<uint2*>(book + (2 * piece + 1) * 256 + (8 * o + gl) * 8) = make_uint2(x[u].z, x[u].w);
                }
                if (kC == 2) {
                    uint8_t* dst = book + 4 * piece * 256 + (16 * (o & 3) + 8 * (o >> 2) + gl) * 4;
                    *reinterpret_cast<uint32_t*>(dst) = x[u].x;
                    *reinterpret_cast<uint32_t*>(dst + 256) = x[u].y;
                    *reinterpret_cast<uint32_t*>(dst + 512) = x[u].z;
                    *reinterpret_cast<uint32_t*>(dst + 768) = x[u].w;
                }
            }
        }
    } else {
        constexpr int kTasks = 2 * 256, kBatch = 6, kWarps = C::kThreads / 32;
        const int gl = lane >> 2, j = lane & 3;
#pragma unroll 1
        for (int i0 = warp; i0 < kTasks; i0 += kBatch * kWarps) {
            float4 x[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u * kWarps, o = (i & 255) % (G / 8), seg = (i & 255) / (G / 8);
                const int g = kC == 2 ? 4 * (8 * (o >> 2) + gl) + (o & 3) : 8 * o + gl;
                if (i < kTasks)
                    x[u] = reinterpret_cast<const float4*>((i < 256 ? kcb : vcb) + (int64_t)hkv * 128 * 256)[(g * 16 * kC + seg) * 4 + j];
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const int i = i0 + u * kWarps, o = (i & 255) % (G / 8), seg = (i & 255) / (G / 8);
                if (i >= kTasks) break;
                uint8_t* book = smem + (i < 256 ? C::kKcbOffset : C::kVcbOffset);
                const uint32_t lo = pack_half2(x[u].x, x[u].y), hi = pack_half2(x[u].z, x[u].w);
                if (kC == 8) *reinterpret_cast<uint2*>(book + (seg * 2 + (j >> 1)) * 256 + (8 * o + gl) * 16 + (j & 1) * 8) = make_uint2(lo, hi);
                if (kC == 4) *reinterpret_cast<uint2*>(book + (seg * 4 + j) * 256 + (8 * o + gl) * 8) = make_uint2(lo, hi);
                if (kC == 2) {
                    uint8_t* dst = book + (seg * 8 + 2 * j) * 256 + (16 * (o & 3) + 8 * (o >> 2) + gl) * 4;
                    *reinterpret_cast<uint32_t*>(dst) = lo;
                    *reinterpret_cast<uint32_t*>(dst + 256) = hi;
                }
            }
        }
    }
    // bounded: whether any page that this CTA may attend is missing (then the softmax warps look for holes, tile by tile)
    bool missing = false;
    if constexpr (kBounded) {
        const BoundedArgs& a = bounded.a;
        if (a.page_table && pos_last >= 0)
            for (int i = threadIdx.x; i <= a.page_div.quotient((int)(pos_last / kTokenBlock)); i += C::kThreads) {
                const int page = a.page_table[s * a.pages_per_seq + i];
                missing |= page < 0 || page >= a.n_pages;
            }
    }
    pf_fence_before();
    if constexpr (kBounded) missing = __syncthreads_or(missing);
    else __syncthreads();
    pf_fence_after();
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&ctl->tmem_base);

    if (warp >= C::kProducerWarp0 && warp < C::kSumWarp) {
        // ---------------------------------------------------------------- producers: codes -> fp16 tiles of 64 tokens
        // A warp takes one 16-token block of the tile.  16-byte chunk `ch` (channels 8 ch ... + 7) of token t goes to byte
        // (ch / 8) * kHalfBytes + t * 128 + ((ch % 8) ^ (t % 8)) * 16: eight lanes of a store hold the chunks of one token,
        // so they meet in no bank either.
        const int pw = warp - C::kProducerWarp0;
        const uint8_t* kbase = kc + (kBounded ? 0 : code_word_offset(sh, sh.n_kv_heads, s, hkv, 0, 0));
        const uint8_t* vbase = vc + (kBounded ? 0 : code_word_offset(sh, sh.n_kv_heads, s, hkv, 0, 0));
        int64_t block_at = -1;                          // bounded: where the block of the tile after the next lies (-1: nowhere)
        auto look_up = [&](int jt) {
            if constexpr (kBounded) {
                const int64_t blk = (int64_t)tile_at(jt) * (C::kTile / kTokenBlock) + pw;
                block_at = jt < n_tiles && blk < sh.n_blocks ? block_offset(bounded.a, (int)s, hkv, (int)blk) : -1;
            }
        };
        bool hole = false, hole_next = false;           // bounded: the tile's block lies nowhere
        constexpr int kW = kC == 8 ? 2 : kC == 4 ? 4 : 8;                   // code words a lane takes of a block, per tensor
        uint32_t kw[kW], vw[kW], kn[kW], vn[kW];        // this tile's and the next one's, loaded a whole tile ahead of their use
        auto load_codes = [&](int jt, uint32_t (&kw)[kW], uint32_t (&vw)[kW]) {
            const int64_t blk = (int64_t)jt * (C::kTile / kTokenBlock) + pw;
#pragma unroll
            for (int i = 0; i < kW; ++i) kw[i] = vw[i] = 0u;
            int64_t at = blk * (G * kTokenBlock);
            if constexpr (kBounded) {
                at = block_at;
                hole_next = at < 0;
                look_up(jt + 1);
                if (at < 0) return;
            } else if (jt >= n_tiles || blk >= sh.n_blocks) {
                return;
            }
            const uint8_t* kp = kbase + at;
            const uint8_t* vp = vbase + at;
            if (kC == 8) {                              // lane = (token half, group)
                const int off = (lane & 15) * kTokenBlock + 8 * (lane >> 4);
                const uint2 a = *reinterpret_cast<const uint2*>(kp + off);
                kw[0] = a.x; kw[1] = a.y;
                if (kSums) {
                    const uint2 b = *reinterpret_cast<const uint2*>(vp + off);
                    vw[0] = b.x; vw[1] = b.y;
                }
            } else if (kC == 4) {                       // lane = group
                const uint4 a = *reinterpret_cast<const uint4*>(kp + lane * kTokenBlock);
                kw[0] = a.x; kw[1] = a.y; kw[2 % kW] = a.z; kw[3 % kW] = a.w;
                if (kSums) {
                    const uint4 b = *reinterpret_cast<const uint4*>(vp + lane * kTokenBlock);
                    vw[0] = b.x; vw[1] = b.y; vw[2 % kW] = b.z; vw[3 % kW] = b.w;
                }
            } else {                                    // lane = (token half, chunk of four groups, taken in another order by the other half)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int off = (4 * (lane & 15) + (i ^ (lane >> 4))) * kTokenBlock + 8 * (lane >> 4);
                    const uint2 a = *reinterpret_cast<const uint2*>(kp + off);
                    kw[(2 * i) % kW] = a.x; kw[(2 * i + 1) % kW] = a.y;
                    if (kSums) {
                        const uint2 b = *reinterpret_cast<const uint2*>(vp + off);
                        vw[(2 * i) % kW] = b.x; vw[(2 * i + 1) % kW] = b.y;
                    }
                }
            }
        };
        auto fill = [&](const uint32_t (&w)[kW], int book, int tile_off) {
            if (kC == 4) {
#pragma unroll
                for (int k = 0; k < 16; ++k) {
                    const uint32_t code = (w[(k >> 2) % kW] >> (8 * (k & 3))) & 0xffu;
                    const int tok = 16 * pw + k;
                    const uint32_t dst = (uint32_t)((lane >> 4) * C::kHalfBytes + tok * 128 + ((((lane >> 1) & 7) ^ (k & 7)) << 4) + 8 * (lane & 1));
                    *reinterpret_cast<uint2*>(smem + tile_off + dst) = *reinterpret_cast<const uint2*>(smem + book + (code * G + lane) * 8);
                }
            } else {
                const int ch = lane & 15;
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int tok = 16 * pw + 8 * (lane >> 4) + k;
                    const uint32_t dst = (uint32_t)((ch >> 3) * C::kHalfBytes + tok * 128 + (((ch & 7) ^ k) << 4));
                    uint4 v;
                    if (kC == 8) {
                        const uint32_t code = (w[(k >> 2) % kW] >> (8 * (k & 3))) & 0xffu;
                        v = *reinterpret_cast<const uint4*>(smem + book + (code * G + ch) * 16);
                    } else {
                        // (the halves' gathers fall into different halves of the banks)
                        const int hb = lane >> 4;
                        uint32_t e[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const uint32_t code = (w[(2 * i + (k >> 2)) % kW] >> (8 * (k & 3))) & 0xffu;
                            e[i] = *reinterpret_cast<const uint32_t*>(smem + book + (code * G + 16 * (i ^ hb) + ch) * 4);
                        }
                        v = hb ? make_uint4(e[1], e[0], e[3], e[2]) : make_uint4(e[0], e[1], e[2], e[3]);
                    }
                    *reinterpret_cast<uint4*>(smem + tile_off + dst) = v;
                }
            }
        };
        look_up(0);
        load_codes(0, kn, vn);
        for (int jt = 0; jt < n_tiles; ++jt) {
            hole = hole_next;
            const int stage = jt % C::kStages;
#pragma unroll
            for (int i = 0; i < kW; ++i) { kw[i] = kn[i]; vw[i] = vn[i]; }
            load_codes(jt + 1, kn, vn);
            bool ok = jt < C::kStages || pf_wait(ctl, &ctl->empty[stage], (uint32_t)(jt / C::kStages - 1) & 1u);
            if (jt == 1) ok = ok && pf_wait(ctl, &ctl->q_full[lane % n_halves], 0u);      // the queries lay there
            if (!__all_sync(0xffffffffu, ok)) break;
            if (kBounded && lane == 0) ctl->hole[stage][pw] = hole;
            fill(kw, C::kKcbOffset, C::kKtOffset + stage * C::kTileBytes);
            if (kSums) fill(vw, C::kVcbOffset, C::kVtOffset + stage * C::kTileBytes);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) pf_arrive(&ctl->full[stage]);
        }
    } else if (warp == C::kMmaWarp) {
        // ---------------------------------------------------------------- scores: Q Khat^T of (tile, row tile) 0, 1, 2, ...
        // (All lanes of the warp go round the loop, a turn of which goes once round the stages, and different lanes wait for
        // different barriers: with everything in a one-thread branch an MMA took some 60 cycles to issue and a wait, behind
        // the exponentials in the queue that it shares with them, 200.)
        constexpr uint32_t kScores = (1u << 4) | ((64u >> 3) << 17) | ((128u >> 4) << 24);       // D fp32, A and B fp16, M = 128, N = 64
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), kdesc = pf_desc_lo(smem_u32(smem + C::kKtOffset), 16);
        const int n_work = __shfl_sync(0xffffffffu, n_tiles * n_halves, 0);
        auto go = [&](auto halves_in_use) {
            constexpr int kHalves = decltype(halves_in_use)::value, kTurn = kHalves * C::kStages;
            if (!__all_sync(0xffffffffu, pf_wait(ctl, &ctl->q_full[lane % kHalves], 0u))) return;                // the queries
            for (int o = 0; o * kTurn < n_work; ++o) {
#pragma unroll
                for (int u = 0; u < kTurn; ++u) {
                    if (o * kTurn + u >= n_work) break;
                    const int t = u % kHalves, stage = u / kHalves, jt = o * C::kStages + stage;
                    // even lanes: the scores of the work before have been read; odd lanes: the tile is there
                    const bool first = o == 0 && u == 0;
                    uint64_t* bar = (lane & 1) || first ? &ctl->full[stage] : &ctl->s_free[t == 0 ? kHalves - 1 : 0];
                    const uint32_t parity = (lane & 1) || first ? (uint32_t)o & 1u : (uint32_t)(t == 0 ? jt - 1 : jt) & 1u;
                    if (!__all_sync(0xffffffffu, pf_wait(ctl, bar, parity))) return;
                    pf_fence_after();
                    if (pf_elect()) {
#pragma unroll
                        for (int ks = 0; ks < 8; ++ks)               // 16 channels = 32 bytes of the 128-byte rows
                            pf_mma(tm + C::kSCol, tm + C::kQCol + 64 * t + 8 * ks,
                                   kdesc + (stage * C::kTileBytes + (ks >> 2) * C::kHalfBytes + (ks & 3) * 32) / 16, kScores, ks > 0);
                        pf_commit(&ctl->s_full[t]);
                        if (!kSums && t == kHalves - 1) pf_commit(&ctl->empty[stage]);
                    }
                }
            }
        };
        if (n_work > 0) {
            if (n_halves == 2) go(std::integral_constant<int, 2>());
            else go(std::integral_constant<int, 1>());
            __syncwarp();
            pf_drain(&ctl->drained[0]);
        }
    } else if (!kSums && warp == C::kSumWarp) {
        // ---------------------------------------------------------------- masses: the row tiles' and warps' sums to one, two tokens per lane
        if constexpr (kWhat == kPfMass) {
            const volatile float* sums = reinterpret_cast<const float*>(smem + C::kVtOffset);
            const int64_t row_tile = bounded.row_tiles > 1 ? tile : 0;
            const int64_t base = ((row_tile * sh.n_seq + s) * sh.n_kv_heads + hkv) * sh.max_tokens;
            const bool old = bounded.mass_in && bounded.row_tiles == 1;
            bool there = true;                                              // (a wait gave up: NaN for the tokens of this and all further tiles)
            for (int jt = 0; jt < n_tiles; ++jt) {
                const int64_t t0 = (int64_t)tile_at(jt) * C::kTile + lane;
                float sum[2];
#pragma unroll
                for (int k = 0; k < 2; ++k) sum[k] = old && t0 + 32 * k < n ? bounded.mass_in[base + t0 + 32 * k] : 0.f;
                if (there) there = __all_sync(0xffffffffu, pf_wait(ctl, &ctl->p_full[lane % n_halves], (uint32_t)jt & 1u) && !pf_failed(ctl));
                float add[2] = {0.f, 0.f};
                for (int i = 0; i < 4 * n_halves; ++i)
#pragma unroll
                    for (int k = 0; k < 2; ++k) add[k] += sums[((jt & 1) * 8 + i) * C::kTile + 32 * k + lane];
                __syncwarp();
                if (lane == 0) pf_arrive(&ctl->pv_done[0]);                 // the next ones may come
#pragma unroll
                for (int k = 0; k < 2; ++k)
                    if (t0 + 32 * k < n) bounded.mass_out[base + t0 + 32 * k] = there ? sum[k] + add[k] : __int_as_float(0x7fffffff);
            }
        }
    } else if (kSums && warp == C::kSumWarp) {
        // ---------------------------------------------------------------- sums: P Vhat, in the same order
        constexpr uint32_t kSums = (1u << 4) | (1u << 16) | ((128u >> 3) << 17) | ((128u >> 4) << 24);   // N = 128, B's rows along N
        const uint32_t tm = __shfl_sync(0xffffffffu, tmem, 0), vdesc = pf_desc_lo(smem_u32(smem + C::kVtOffset), C::kHalfBytes);
        const int n_work = __shfl_sync(0xffffffffu, n_tiles * n_halves, 0);
        auto go = [&](auto halves_in_use) {
            constexpr int kHalves = decltype(halves_in_use)::value, kTurn = kHalves * C::kStages;
            for (int o = 0; o * kTurn < n_work; ++o) {
#pragma unroll
                for (int u = 0; u < kTurn; ++u) {
                    if (o * kTurn + u >= n_work) break;
                    const int t = u % kHalves, stage = u / kHalves, jt = o * C::kStages + stage;
                    uint64_t* bar = lane & 1 ? &ctl->full[stage] : &ctl->p_full[t];
                    const uint32_t parity = lane & 1 ? (uint32_t)o & 1u : (uint32_t)jt & 1u;
                    if (!__all_sync(0xffffffffu, pf_wait(ctl, bar, parity))) return;
                    pf_fence_after();
                    const bool more = jt > 0;
                    if (pf_elect()) {
#pragma unroll
                        for (int ks = 0; ks < 4; ++ks)               // 16 tokens = 2048 bytes
                            pf_mma(tm + C::kOCol + 128 * t, tm + C::kPCol + 32 * t + 8 * ks,
                                   vdesc + (stage * C::kTileBytes + ks * 2048) / 16, kSums, more || ks > 0);
                        pf_commit(&ctl->pv_done[t]);
                        if (t == kHalves - 1) pf_commit(&ctl->empty[stage]);
                    }
                }
            }
        };
        if (n_work > 0) {
            if (n_halves == 2) go(std::integral_constant<int, 2>());
            else go(std::integral_constant<int, 1>());
            __syncwarp();
            pf_drain(&ctl->drained[1]);
        }
    } else if constexpr (kBounded) {
        // ---------------------------------------------------------------- softmax: two threads per row, 32 columns each.  (A thread per row
        // took some 2000 cycles for its 64 columns, as long as everything else in two tiles; half the exponentials on the FMA pipe instead
        // of the special-function unit made that longer still: it is latencies that a single thread cannot hide.)  The threads of a
        // row are in two warps, which agree on the reference of the weights; only when it moves do they exchange maxima.
        const int part = warp >> 3, t = (warp >> 2) & 1;
        if (warp < C::kSoftWarps && t < n_halves) {
            const int row0 = t * 128 + (warp & 3) * 32, rho = row0 + lane, pair = 1 + (warp & 7);
            const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
            const uint32_t s_addr = lanes + C::kSCol + 32 * part, p_addr = lanes + C::kPCol + 32 * t + 16 * part, o_addr = lanes + C::kOCol + 128 * t + 64 * part;
            volatile float* exchange = reinterpret_cast<float*>(smem + C::kExchangeOffset);
            const int qi = qi0 + rho / R, window = bounded.a.window;
            const int pos = qi < n_q && rho < rows_used ? (int)pos0 + rho / R : -1;
            // a tile part that starts at j0 is seen whole by all rows of the warp up to seen_to, and from behind seen_from or up to seen_sinks
            const int seen_to = (int)pos0 + row0 / R - 31, seen_from = window ? (int)pos0 + (row0 + 31) / R - window : -1, seen_sinks = bounded.a.sinks - 32;
            {
                const __half2 sign = query_sign(scale_log2e);
                uint32_t u[32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 v = *reinterpret_cast<const uint4*>(smem + C::q_offset(rho) + (((8 * part + i) ^ (rho & 7)) << 4));
                    u[4 * i] = signed_query(v.x, sign); u[4 * i + 1] = signed_query(v.y, sign);
                    u[4 * i + 2] = signed_query(v.z, sign); u[4 * i + 3] = signed_query(v.w, sign);
                }
                pf_st32(lanes + C::kQCol + 64 * t + 32 * part, u);
                pf_st_wait();
                pf_fence_before();
                __syncwarp();
                if (lane == 0) pf_arrive(&ctl->q_full[t]);
            }
            float m = -INFINITY, l = 0.f;                                   // reference of the weights (log2 domain), the sum of this thread's
            bool ok = true;
            if constexpr (kWhat == kPfMass) {                               // the row's log-sum-exp, from the parts of its context
                const float* of = bounded.partials + ((int64_t)(blockIdx.x / bounded.parts) * bounded.parts * C::kRows + rho) * 2;
                bool gave_up = false;
                for (int i = 0; i < bounded.parts; ++i) {
                    const float mi = of[(int64_t)i * C::kRows * 2];
                    gave_up |= mi != mi;
                    m = fmaxf(m, mi);
                }
                for (int i = 0; i < bounded.parts; ++i) {
                    const float mi = of[(int64_t)i * C::kRows * 2];
                    l += (mi == -INFINITY ? 1.f : exp2f(mi - m)) * of[(int64_t)i * C::kRows * 2 + 1];      // (no reference: zero, or no number)
                }
                // (a row that sees nothing: no weight; a row that is none: none of its scores, which are zero, counts; a sum that is no number comes from
                // scores that are none, or infinite: they give NaN by themselves, and what the row does not see gets no weight)
                m = !(qi < n_q && rho < rows_used) ? INFINITY : gave_up ? __int_as_float(0x7fffffff) : l == 0.f ? 0.f : l == l ? m + log2f(l) : m == -INFINITY ? 0.f : m;
            }
#pragma unroll 1
            for (int jt = 0; jt < n_tiles; ++jt) {
                ok &= pf_wait(ctl, &ctl->s_full[t], (uint32_t)jt & 1u);
                pf_fence_after();
                uint32_t a[32];
                pf_ld32(a, s_addr);
                pf_ld_wait(a);
                pf_fence_before();
                __syncwarp();
                if (lane == 0) pf_arrive(&ctl->s_free[t]);
                float* sa = reinterpret_cast<float*>(a);
                const int j0 = tile_at(jt) * C::kTile + 32 * part;
                if (j0 > seen_to || (j0 <= seen_from && j0 > seen_sinks) || missing) {
                    // bit i: this row sees column i
                    const int left = pos - j0, sinks = bounded.a.sinks - j0;
                    uint32_t sees = left < 0 ? 0u : left >= 31 ? ~0u : (2u << left) - 1u;
                    if (window && left - window >= 0) {                     // columns 0 ... left - window are behind the window, sinks apart
                        const uint32_t behind = left - window >= 31 ? ~0u : (2u << (left - window)) - 1u;
                        const uint32_t first = sinks <= 0 ? 0u : sinks >= 32 ? ~0u : (1u << sinks) - 1u;
                        sees &= ~behind | first;
                    }
                    if (missing) {
                        const int stage = jt % C::kStages;
                        ok &= pf_wait(ctl, &ctl->full[stage], (uint32_t)(jt / C::kStages) & 1u);      // (long since: it orders the read)
                        const volatile uint8_t* holes = &ctl->hole[stage][2 * part];
                        if (holes[0]) sees &= 0xffff0000u;
                        if (holes[1]) sees &= 0x0000ffffu;
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (!((sees >> i) & 1u)) sa[i] = -INFINITY;
                }
                if constexpr (kWhat == kPfMass) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) sa[i] = ex2_approx(fmaf(sa[i], scale, -m));
                    // lane i ends up with the sum of column i over the rows of the warp: with every step half of the columns changes hands
#pragma unroll
                    for (int o = 16; o > 0; o >>= 1)
#pragma unroll
                        for (int i = 0; i < o; ++i) {
                            const float keep = lane & o ? sa[i + o] : sa[i], give = lane & o ? sa[i] : sa[i + o];
                            sa[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                        }
                    // (two places in turn: what lay here was taken before the last tile's sums were handed over)
                    reinterpret_cast<volatile float*>(smem + C::kVtOffset)[((jt & 1) * 8 + t * 4 + (warp & 3)) * C::kTile + 32 * part + lane] =
                        ok ? sa[0] : __int_as_float(0x7fffffff);
                    if (jt > 0) ok &= pf_wait(ctl, &ctl->pv_done[0], (uint32_t)(jt - 1) & 1u);      // the last tile's have been taken
                    __syncwarp();
                    if (lane == 0) pf_arrive(&ctl->p_full[t]);
                } else {
                    float mx[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = max3(sa[k], sa[k + 4], sa[k + 8]);
#pragma unroll
                    for (int i = 12; i < 28; i += 8)
#pragma unroll
                        for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], sa[i + k], sa[i + 4 + k]);
#pragma unroll
                    for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], sa[28 + k]);
                    const float m_tile = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * scale;      // (-inf: the row sees nothing of this part)
                    if constexpr (kWhat == kPfLse) {
                        const float m_new = fmaxf(m, m_tile), mm = m_new == -INFINITY ? 0.f : m_new;
                        l *= m == -INFINITY ? 0.f : exp2f(m - mm);
                        m = m_new;
                        float l0 = 0.f, l1 = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            l0 += ex2_approx(fmaf(sa[2 * i], scale, -mm));
                            l1 += ex2_approx(fmaf(sa[2 * i + 1], scale, -mm));
                        }
                        l += l0 + l1;
                    } else {
                        // The reference follows the maximum only when it is more than 8 (a factor of 256) behind: the sums rarely have to be
                        // rescaled, and fp16 weights up to 256 are as precise as weights up to 1.
                        const bool rescale = pf_pair_any(pair, m_tile > m + 8.f || (m == -INFINITY && m_tile > -INFINITY));
                        float f = 1.f;
                        if (rescale) {
                            exchange[part * C::kRows + rho] = m_tile;
                            pf_pair_sync(pair);
                            const float m_new = max3(m, m_tile, exchange[(part ^ 1) * C::kRows + rho]);
                            pf_pair_sync(pair);
                            f = m == -INFINITY ? 0.f : exp2f(m - m_new);
                            m = m_new;
                            l *= f;
                        }
                        const float mm = m == -INFINITY ? 0.f : m;
                        // The products take weights in fp16, the normaliser sums them as they are.  (Summed as rounded, the largest calls
                        // take 675 and 1154 us, not 666 and 1141; the error of 3 x 333 queries against 64 bits is 2.10e-4 and 2.12e-4, of
                        // which the outputs' own rounding makes 2.07e-4.)
                        uint32_t p[16];
                        float l0 = 0.f, l1 = 0.f;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const float x0 = ex2_approx(fmaf(sa[2 * i], scale, -mm)), x1 = ex2_approx(fmaf(sa[2 * i + 1], scale, -mm));
                            l0 += x0;
                            l1 += x1;
                            p[i] = pack_half2(x0, x1);
                        }
                        l += l0 + l1;
                        if (jt > 0) {                                               // the last sums are done with the weights' columns
                            ok &= pf_wait(ctl, &ctl->pv_done[t], (uint32_t)(jt - 1) & 1u);
                            pf_fence_after();
                            if (rescale) {
#pragma unroll 1
                                for (int c0 = 0; c0 < 64; c0 += 32) {
                                    uint32_t o[32];
                                    pf_ld32(o, o_addr + c0);
                                    pf_ld_wait(o);
#pragma unroll
                                    for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                                    pf_st32(o_addr + c0, o);
                                }
                            }
                        }
                        pf_st16(p_addr, p);
                        pf_st_wait();
                        pf_fence_before();
                        __syncwarp();
                        if (lane == 0) pf_arrive(&ctl->p_full[t]);
                    }
                }
            }
            if constexpr (kWhat == kPfLse) {                                // the two threads of a row to one
                ok = !pf_pair_any(pair, !ok || pf_failed(ctl));
                exchange[part * C::kRows + rho] = m;
                pf_pair_sync(pair);
                const float other = exchange[(part ^ 1) * C::kRows + rho], top = fmaxf(m, other);
                pf_pair_sync(pair);
                exchange[part * C::kRows + rho] = l = m == -INFINITY ? l : l * exp2f(m - top);
                pf_pair_sync(pair);
                if (part == 0) {
                    float* of = bounded.partials + ((int64_t)blockIdx.x * C::kRows + rho) * 2;
                    of[0] = ok ? top : __int_as_float(0x7fffffff);          // (a wait gave up: no reference is a number)
                    of[1] = l + exchange[C::kRows + rho];
                }
                pf_fence_before();
            }
            if constexpr (kWhat == kPfMass) pf_fence_before();
            if constexpr (kWhat == kPfAttn) {
                exchange[part * C::kRows + rho] = l;
                pf_pair_sync(pair);
                l += exchange[(part ^ 1) * C::kRows + rho];
                // ---- normalise and write, through shared memory (the codebooks are done with when the last sums are), in whole lines
                if (n_tiles > 0) ok &= pf_wait(ctl, &ctl->pv_done[t], (uint32_t)(n_tiles - 1) & 1u);
                ok = !pf_pair_any(pair, !ok || pf_failed(ctl));                 // (the rows' both halves)
                pf_fence_after();
                const bool partial = bounded.parts > 1;                         // (partials: the accumulators as they are)
                // nothing seen: a zero row; a wait gave up: NaN rows, so that nothing takes them for a result
                const float inv = !ok ? __int_as_float(0x7fffffff) : partial ? 1.f : l == 0.f ? 0.f : 1.f / l;
                float* to_part = nullptr;
                if (partial) {
                    to_part = bounded.partials + ((int64_t)blockIdx.x * C::kRows + row0) * partial_stride(128);
                    if (part == 0) {
                        to_part[lane * partial_stride(128)] = m;
                        to_part[lane * partial_stride(128) + 1] = l;
                    }
                }
                uint8_t* block = smem + warp * 32 * C::kOutStride;
#pragma unroll 1
                for (int c0 = 0; c0 < 64; c0 += 32) {
                    uint32_t o[32];
                    if (n_tiles > 0) {
                        pf_ld32(o, o_addr + c0);
                        pf_ld_wait(o);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(block + lane * C::kOutStride + 16 * i) =
                            inv == 0.f || n_tiles == 0 ? make_float4(0.f, 0.f, 0.f, 0.f)
                                                       : make_float4(__uint_as_float(o[4 * i]) * inv, __uint_as_float(o[4 * i + 1]) * inv,
                                                                     __uint_as_float(o[4 * i + 2]) * inv, __uint_as_float(o[4 * i + 3]) * inv);
                    __syncwarp();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const int rw = 4 * i + (lane >> 3), rr = row0 + rw, qr = qi0 + rr / R, column = 64 * part + c0 + 4 * (lane & 7);
                        const float4 v = *reinterpret_cast<const float4*>(block + rw * C::kOutStride + 16 * (lane & 7));
                        if (partial) {
                            float* to = to_part + rw * partial_stride(128) + 2 + column;
                            *reinterpret_cast<float2*>(to) = make_float2(v.x, v.y);
                            *reinterpret_cast<float2*>(to + 2) = make_float2(v.z, v.w);
                        } else if (qr < n_q && rr < rows_used) {
                            *reinterpret_cast<uint2*>(bounded.a.out + ((q_first + qr) * sh.n_q_heads + hkv * R + rr % R) * 128 + column) =
                                make_uint2(pack_half2(v.x, v.y), pack_half2(v.z, v.w));
                        }
                    }
                    __syncwarp();
                }
                pf_fence_before();
            }
        }
    } else if (warp < 4 * n_halves) {
        // ---------------------------------------------------------------- softmax: a thread per row
        const int t = warp >> 2, rho = threadIdx.x;
        const uint32_t lanes = tmem + ((uint32_t)((warp & 3) * 32) << 16);
        const uint32_t s_addr = lanes + C::kSCol, p_addr = lanes + C::kPCol + 32 * t, o_addr = lanes + C::kOCol + 128 * t;
        const int qi = qi0 + rho / R;
        const bool live = qi < n_q;
        const int64_t pos = live ? pos0 + rho / R : -1;
        const int64_t pos_warp = pos0 + (warp * 32) / R;                   // smallest position among the warp's rows
        {
            uint32_t u[32];
#pragma unroll
            for (int half = 0; half < 2; ++half) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint4 v = *reinterpret_cast<const uint4*>(smem + C::q_offset(rho) + (((8 * half + i) ^ (rho & 7)) << 4));
                    u[4 * i] = (v.x ^ q_sign) & q_keep; u[4 * i + 1] = (v.y ^ q_sign) & q_keep;
                    u[4 * i + 2] = (v.z ^ q_sign) & q_keep; u[4 * i + 3] = (v.w ^ q_sign) & q_keep;
                }
                pf_st32(lanes + C::kQCol + 64 * t + 32 * half, u);
            }
            pf_st_wait();
            pf_fence_before();
            __syncwarp();
            if (lane == 0) pf_arrive(&ctl->q_full[t]);
        }
        float m = -INFINITY, l = 0.f;                                       // reference of the weights (log2 domain), their sum
        bool ok = true;
        for (int jt = 0; jt < n_tiles; ++jt) {
            ok &= pf_wait(ctl, &ctl->s_full[t], (uint32_t)jt & 1u);
            pf_fence_after();
            uint32_t a[32], b[32];
            pf_ld32(a, s_addr);
            pf_ld32(b, s_addr + 32);
            pf_ld_wait(a);
            pf_ld_wait(b);
            pf_fence_before();
            __syncwarp();
            if (lane == 0) pf_arrive(&ctl->s_free[t]);
            float* sa = reinterpret_cast<float*>(a);
            float* sb = reinterpret_cast<float*>(b);
            const int64_t j0 = (int64_t)jt * C::kTile;
            if (j0 + C::kTile - 1 > pos_warp) {                             // some row's causal limit lies in the tile
                const int64_t left = pos - j0;                              // columns 0 ... left are attended
#pragma unroll
                for (int i = 0; i < 32; ++i) {
                    if (i > left) sa[i] = -INFINITY;
                    if (i + 32 > left) sb[i] = -INFINITY;
                }
            }
            float mx[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) mx[i] = max3(sa[i], sb[i], sa[i + 4]);
#pragma unroll
            for (int i = 8; i < 32; i += 8)
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], sa[i + k], sa[i + 4 + k]);
#pragma unroll
            for (int i = 4; i < 28; i += 8)
#pragma unroll
                for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], sb[i + k], sb[i + 4 + k]);
#pragma unroll
            for (int k = 0; k < 4; ++k) mx[k] = fmaxf(mx[k], sb[28 + k]);
            const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]);
            const float m_tile = top * scale;                               // (-inf: the row attends nothing of the tile)
            // The weights' reference follows the maximum only when it is more than 8 (a factor of 256) behind: the sums
            // rarely have to be rescaled, and fp16 weights up to 256 are as precise as weights up to 1.
            const bool move = m_tile > m + 8.f || (m == -INFINITY && m_tile > -INFINITY);
            const bool rescale = __any_sync(0xffffffffu, move);
            float f = 1.f;
            if (rescale) {
                const float m_new = fmaxf(m, m_tile);
                f = m == -INFINITY ? 0.f : exp2f(m - m_new);
                m = m_new;
                l *= f;
            }
            const float mm = m == -INFINITY ? 0.f : m;
            uint32_t p[32];
            float l0 = 0.f, l1 = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x0 = ex2_approx(fmaf(sa[2 * i], scale, -mm)), x1 = ex2_approx(fmaf(sa[2 * i + 1], scale, -mm));
                l0 += x0;
                l1 += x1;
                p[i] = pack_half2(x0, x1);
            }
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float x0 = ex2_approx(fmaf(sb[2 * i], scale, -mm)), x1 = ex2_approx(fmaf(sb[2 * i + 1], scale, -mm));
                l0 += x0;
                l1 += x1;
                p[16 + i] = pack_half2(x0, x1);
            }
            l += l0 + l1;
            if (jt > 0) {                                                   // the last sums are done with the weights' columns
                ok &= pf_wait(ctl, &ctl->pv_done[t], (uint32_t)(jt - 1) & 1u);
                pf_fence_after();
                if (rescale) {
#pragma unroll 1
                    for (int c0 = 0; c0 < 128; c0 += 32) {
                        uint32_t o[32];
                        pf_ld32(o, o_addr + c0);
                        pf_ld_wait(o);
#pragma unroll
                        for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                        pf_st32(o_addr + c0, o);
                    }
                }
            }
            pf_st32(p_addr, p);
            pf_st_wait();
            pf_fence_before();
            __syncwarp();
            if (lane == 0) pf_arrive(&ctl->p_full[t]);
        }
        // ---- normalise and write: through shared memory (the codebooks are done with when the last sums are), so that the
        // stores take whole lines; a thread per row wrote 32 lines at a time (10.8 thousand cycles per CTA)
        if (n_tiles > 0) ok &= pf_wait(ctl, &ctl->pv_done[t], (uint32_t)(n_tiles - 1) & 1u);
        ok = __all_sync(0xffffffffu, ok && !pf_failed(ctl));
        pf_fence_after();
        // no position: zero row; a wait gave up: NaN rows, so that nothing takes them for a result
        const float inv = !ok ? __int_as_float(0x7fffffff) : l > 0.f ? 1.f / l : 0.f;
        uint8_t* block = smem + warp * 32 * C::kOutStride;
#pragma unroll 1
        for (int c0 = 0; c0 < 128; c0 += 32) {
            uint32_t o[32];
            if (n_tiles > 0) {
                pf_ld32(o, o_addr + c0);
                pf_ld_wait(o);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i)
                *reinterpret_cast<float4*>(block + lane * C::kOutStride + 16 * i) =
                    inv == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f)
                               : make_float4(__uint_as_float(o[4 * i]) * inv, __uint_as_float(o[4 * i + 1]) * inv,
                                             __uint_as_float(o[4 * i + 2]) * inv, __uint_as_float(o[4 * i + 3]) * inv);
            __syncwarp();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int rw = 4 * i + (lane >> 3), rr = warp * 32 + rw, qr = qi0 + rr / R;
                if (qr < n_q)
                    *reinterpret_cast<float4*>(out + ((q_first + qr) * sh.n_q_heads + hkv * R + rr % R) * 128 + c0 + 4 * (lane & 7)) =
                        *reinterpret_cast<const float4*>(block + rw * C::kOutStride + 16 * (lane & 7));
            }
            __syncwarp();
        }
        pf_fence_before();
    }
    // every MMA that was issued has been waited for; hand the tensor memory back
    __syncthreads();
    if (warp == C::kMmaWarp) {
        pf_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
    }
}

}  // namespace

}  // namespace cq
