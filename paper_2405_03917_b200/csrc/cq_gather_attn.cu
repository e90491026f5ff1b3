// Attention of few query rows over a coded cache: window, sinks, pages; and the masses of cached tokens (head_dim 128, one byte per
// code, c = 2, 4 or 8).
//
//   out_r = sum_t p_rt Vhat_t / sum_t p_rt,  p_rt = 2^(scale log2e <q_r, Khat_t> - m_r)      r: (query token, head) of a KV head
//
// Both codebooks lie in shared memory as fp16, code-major: row j holds the centroids j of all groups (256 bytes).  A warp takes blocks
// of 16 tokens; its lanes load centroids as they lie there into the fragments of m16n8k16 MMAs, so no tile of keys or values is
// ever written.  What makes that possible without bank conflicts is the choice of what a fragment's rows and columns mean:
//   scores: a row (four query rows) or a column (eight) of keys is (token, half of the groups): the eight lanes that load one token
//       together take eight different groups.  The other operand holds every query twice, with the channels of one half and with
//       those of the other, and the accumulators where the halves agree are added up.
//   sums:   a loaded word holds two neighbouring channels of ONE token, but the contraction runs over tokens.  So the k pair
//       (2i, 2i + 1) of an MMA is one token, A's rows r hold (p, 0) there and rows r + 8 (0, p): they sum the even and the odd
//       channels.  Lanes of a quad hold different tokens of the same column; in the kernel for four rows the rows of A that are left
//       over select lanes of a quad, so that a column stands for two groups, and a second copy of the value centroids, half a line
//       further on, parts the rest: no conflict.  With eight rows two lanes meet.
// Shared memory: 64 KiB + 2 x 64 KiB of centroids, one CTA of eight warps per SM; the codes of a warp's next blocks
// travel by asynchronous copies.
//
// What bounds it: shared memory.  A token costs 4 wavefronts of centroids (of 5 in all) and 3 cycles of MMAs; a block of 16 tokens
// takes about 110 cycles, 82 of them wavefronts.  64 sequences, 32 heads on 8, CQ-8c8b: window of 4096 82 us, contexts of
// 4096 ... 16384 in pages 165 us = 1.0 TB/s; of 16384 without a window 239 us, as long as the table kernels of the plain decode
// attention take (238; 64 heads on 8 by eight rows: 256 and 433).  With a KV head to every query head a whole centroid is gathered where
// those read one table entry: 16 x 4096, 32 heads of CQ-4c8b 91 us (60 there), 40 heads of CQ-8c8b 96 us (52).
//
// Masses take two passes: kLse leaves every row's log-sum-exp and, for up to four rows, the scores; mass_of_scores_kernel turns these into
// weights and adds up, per token, those of all rows.  Where scores are not kept, kMass works them out again.  (Row after row tile goes
// over the same blocks in the same CTA: every sum has one writer and one order.)  Keys alone leave room for two CTAs on an SM (one:
// 450 against 291 us; ten or twelve warps instead of eight spill: 175 and 179 against 160 us).  64 sequences of 16384 tokens, 32 heads
// on 8, CQ-8c8b: 291 us without stored scores, 160 us with them.
//
// Work is dealt evenly: the blocks that all (KV head, sequence, row tile) items attend lie on one line, every CTA takes an equal
// stretch of it (a stretch that crosses into another KV head loads that head's centroids), and what a cut item leaves behind
// is merged by a second, small kernel.
#include <limits.h>

#include "cq_bounded.cuh"
#include "cq_bulk_copy.cuh"

namespace cq {

namespace {

enum Mode { kAttn, kLse, kMass };

constexpr int kBookBytes = 256 * 256;
// Eight warps (12 were as fast: 81 and 82 us for 64 sequences with a window of 4096, 32 heads on 8), and their share of the rest of
// shared memory: codes on their way (2 blocks' for c = 2, 4 for c = 4, 8 for c = 8), then accumulators.
constexpr int kKOffset = 0, kVOffset = kBookBytes;
template <int kMode>
struct Cfg {
    static constexpr int kCtas = kMode == kAttn ? 1 : 2;                      // of an SM
    static constexpr int kWarps = 8, kThreads = kWarps * 32;
    static constexpr int kWarpBytes = kMode == kAttn ? 4096 : 2048;
    static constexpr int kStageOffset = kMode == kAttn ? 3 * kBookBytes : kBookBytes;
    static constexpr int kStatOffset = kStageOffset + kWarps * kWarpBytes;    // [warp][8] references, [warp][8] sums, what the scans need
    static constexpr int kQOffset = kStatOffset + 2 * kWarps * 8 * 4 + 256;   // queries of the item, and (kMass) their log-sum-exps
    static constexpr int kSmemBytes = kQOffset + 8 * 256 + (kMode == kMass ? 32 : 0);
    static_assert(kSmemBytes <= 227 * 1024 / kCtas - (kCtas > 1 ? 1024 : 0), "shared memory");
};
constexpr int kLeastShare = 16;                                           // blocks that a CTA takes at least

__host__ __device__ constexpr int partial_floats(int rows, int mode) { return 2 * rows + (mode == kAttn ? (rows == 4 ? 16 : 32) * 32 : 0); }

// The masses' part of a call.
struct MassArgs {
    const float* mass_in;                                                 // may be null
    float* mass_out;
    float* lse;                                                           // [sequence][KV head][row_stride]: log2 of the sum of 2^score
    int row_stride;
    float* scores;                                                        // null, or the scores (log2 domain) of four rows: [sequence][KV head][block][row][16]
};

// What a CTA leaves of the items that its stretch cuts: [0] the end or the middle of one, [1] the beginning of one.
struct Cut {
    int head, seq, tile, state;                                           // state 0: none, 1: goes on in the next CTA, 2: ends here
};

__device__ __forceinline__ float ex2f(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ void mma16816_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// prmt with all four selector bits: bit 3 of a nibble puts the sign of the byte it names (zero for a weight's upper byte) into all eight bits
__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel)
{
    uint32_t d;
    asm("prmt.b32 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(b), "r"(sel));
    return d;
}
// a centroid's words, as they lie in a code-major codebook
template <int E>
__device__ __forceinline__ void load_words(uint32_t* w, const uint8_t* at)
{
    if (E == 4) {
        const uint4 v = *reinterpret_cast<const uint4*>(at);
        w[0] = v.x; w[1 % E] = v.y; w[2 % E] = v.z; w[3 % E] = v.w;
    } else if (E == 2) {
        const uint2 v = *reinterpret_cast<const uint2*>(at);
        w[0] = v.x; w[1 % E] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t*>(at);
    }
}

__device__ __forceinline__ void copy16(uint32_t dst, const void* src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void copies_issued() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kPending>
__device__ __forceinline__ void copies_wait()      // all but the newest kPending groups
{
    asm volatile("cp.async.wait_group %0;" ::"n"(kPending) : "memory");
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }


// Row tiles of a sequence and the blocks that one of them attends at most (at least one: rows that see nothing are written too).
struct Cost {
    int tiles, blocks;
};
template <int kRows, int kMode>
__device__ __forceinline__ Cost cost_of(const BoundedArgs& a, const SeqView& v)
{
    Cost c;
    const int rows = v.m * a.sh.R;
    c.tiles = rows < a.least_rows || rows > a.most_rows ? 0 : (rows + kRows - 1) / kRows;
    c.blocks = (v.n + kTokenBlock - 1) / kTokenBlock;
    if (a.window) {
        const int64_t span = (int64_t)a.window + (kRows + a.sh.R - 2) / a.sh.R;   // tokens from the first of a tile's windows to its last row
        const int64_t most = (span + 2 * kTokenBlock - 2) / kTokenBlock + (a.sinks + kTokenBlock - 1) / kTokenBlock;
        c.blocks = c.blocks < most ? c.blocks : (int)most;
    }
    c.blocks = c.blocks < 1 ? 1 : c.blocks;
    if (kMode == kMass) {                                                   // a CTA goes through all row tiles of its blocks
        c.blocks = (v.n + kTokenBlock - 1) / kTokenBlock;
        c.tiles = c.blocks ? 1 : 0;
    }
    return c;
}

// Where register `reg` of `lane` belongs: row of the tile and channel.
template <int kC, int kRows>
__device__ __forceinline__ void place_of(int reg, int lane, int& row, int& channel)
{
    constexpr int E = kC / 2, kLow = 8 / E;                                 // words of a centroid; columns that share a block of groups
    const int r = lane >> 2, p = lane & 3, nt = reg >> 2, n = 2 * p + (reg & 1), par = (reg >> 1) & 1;
    const int m = nt / E, w = nt % E;
    int group;
    if (kRows == 4) {
        row = r & 3;
        group = (n % kLow) * 2 + (r >> 2) + 2 * kLow * (n / kLow + E * m);
    } else {
        row = r;
        group = n % kLow + kLow * (n / kLow + E * m);
    }
    channel = group * kC + 2 * w + par;
}

// Sum of `v` over the threads before this one, and over all; every thread takes part.
template <int kWarps>
__device__ __forceinline__ int64_t block_prefix(int64_t v, int64_t* scratch, int64_t& total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    int64_t incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t x = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += x;
    }
    if (lane == 31) scratch[warp] = incl;
    __syncthreads();
    int64_t before = 0;
    total = 0;
    for (int w = 0; w < kWarps; ++w) {
        if (w < warp) before += scratch[w];
        total += scratch[w];
    }
    __syncthreads();
    return before + incl - v;
}

template <int kC, int kRows, int kMode>
__global__ void __launch_bounds__(Cfg<kMode>::kThreads, Cfg<kMode>::kCtas)
gather_kernel(BoundedArgs a, MassArgs mass, float* __restrict__ partials, Cut* __restrict__ cuts)
{
    using C = Cfg<kMode>;
    constexpr int kWarps = C::kWarps, kThreads = C::kThreads, kWarpBytes = C::kWarpBytes;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int G = 128 / kC, E = kC / 2;
    constexpr int kLow = 8 / E;
    constexpr int kKWords = G / 8;                                          // key code words (four tokens each) of a lane
    constexpr int kVGroups = kRows == 4 ? 4 / E : 8 / E;                    // groups of a lane's values
    constexpr int kVWords = kRows == 4 ? 2 * kVGroups : kVGroups;           // their code words (eight or four tokens)
    constexpr int kNT = kRows == 4 ? 4 : 8;                                 // accumulator tiles
    constexpr int kBlockBytes = (kMode == kAttn ? 2 : 1) * G * kTokenBlock; // key and value codes of a block
    constexpr int kStages = kWarpBytes / kBlockBytes;                       // blocks of a warp whose codes have room
    static_assert(kStages >= 2 && (kMode != kAttn || kNT * 4 * 128 <= kWarpBytes), "room");
    extern __shared__ __align__(1024) uint8_t smem[];
    float* wm = reinterpret_cast<float*>(smem + C::kStatOffset);            // [warp][8]: reference and sum of the weights
    float* wl = wm + kWarps * 8;
    int64_t* scratch = reinterpret_cast<int64_t*>(wl + kWarps * 8);
    uint64_t* book_bar = reinterpret_cast<uint64_t*>(scratch + kWarps);
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = lane >> 2, p = lane & 3, R = sh.R, n_seq = (int)sh.n_seq;

    // ---- this CTA's stretch of the line
    int64_t per_head = 0, mine = 0, before = 0;
    auto blocks_of = [&](int s) {
        if (s >= n_seq) return (int64_t)0;
        const Cost c = cost_of<kRows, kMode>(a, seq_view(a, s));
        return (int64_t)c.tiles * c.blocks;
    };
    for (int s0 = 0; s0 < n_seq; s0 += kThreads) {
        int64_t all;
        mine = blocks_of(s0 + (int)threadIdx.x);
        before = block_prefix<kWarps>(mine, scratch, all);
        per_head += all;
    }
    const int64_t total = per_head * sh.n_kv_heads;
    int64_t share = (total + gridDim.x - 1) / gridDim.x;
    share = share < kLeastShare ? kLeastShare : share;
    int64_t x = share * blockIdx.x;
    const int64_t x_end = x + share < total ? x + share : total;
    if (threadIdx.x < 2) cuts[2 * blockIdx.x + threadIdx.x].state = 0;
    if (x >= x_end) return;
    int head = (int)(x / per_head), seq = 0;
    int64_t rest = x - head * per_head;                                     // blocks of the sequence before x
    for (int s0 = 0; s0 < n_seq; s0 += kThreads) {
        int64_t all = per_head;
        if (n_seq > kThreads) {                                             // (otherwise the first scan's results are still there)
            mine = blocks_of(s0 + (int)threadIdx.x);
            before = block_prefix<kWarps>(mine, scratch, all);
        }
        if (rest >= all) { rest -= all; continue; }
        if (before <= rest && rest < before + mine) { scratch[0] = s0 + (int)threadIdx.x; scratch[1] = rest - before; }
        __syncthreads();
        seq = (int)scratch[0];
        rest = scratch[1];
        break;
    }
    // (before the next writer of scratch and of the cut records, the CTA has met again)

    const __half2 q_sign = query_sign(a.scale_log2e);
    const float scale = a.scale_log2e == 0.f ? 1.f : fabsf(a.scale_log2e);

    // ---- lane constants
    const int tq = lane >> 3, hp = lane & 7;                                // scores: token quad of a block, group in its eight
    const int flip = E == 4 ? 0 : E == 2 ? tq & 1 : tq;                     // order of the eights, so that the quads of a load meet in no bank
    uint32_t koff[kKWords];                                                 // byte of the lane's i-th centroid in a row
#pragma unroll
    for (int i = 0; i < kKWords; ++i) koff[i] = (uint32_t)((8 * (i ^ flip) + hp) * 2 * kC);
    uint32_t voff[kVGroups];                                                // the same for values; byte 2: the copy
    const int vg0 = kRows == 4 ? (r % kLow) * 2 + (p & 1) + 2 * kLow * (r / kLow) : r % kLow + kLow * (r / kLow);       // the first of its groups
#pragma unroll
    for (int m = 0; m < kVGroups; ++m) {
        const int g = vg0 + m * (kRows == 4 ? 2 : 1) * kLow * E;
        voff[m] = (uint32_t)((g * 2 * kC) ^ ((p >> 1) * 64)) | ((uint32_t)(p >> 1) << 16);
    }
    uint8_t* stage0 = smem + C::kStageOffset + warp * kWarpBytes;              // [stage][block of the turn][key codes, value codes]
    const uint32_t stage_addr = (uint32_t)__cvta_generic_to_shared(stage0) + 16 * lane;
    const uint8_t* k_codes = stage0 + hp * kTokenBlock + 4 * tq;            // the lane's codes in a block
    const uint8_t* v_codes = stage0 + G * kTokenBlock + vg0 * kTokenBlock + (kRows == 4 ? 8 * (p >> 1) : 4 * p);
    const int64_t from_v = (int64_t)(reinterpret_cast<uintptr_t>(a.vc) - reinterpret_cast<uintptr_t>(a.kc));
    const uint8_t* src_lane = a.kc + (kMode == kAttn && G == 16 && lane >= 16 ? from_v - 256 : 0) + 16 * lane;      // 16 groups: half a warp per tensor
    // Weights (packed in twos) to the fragments of the sums: (p, 0), (0, p) of a word's low and of its high half; four rows: in the rows
    // that select the lane
    uint32_t sel0 = 0x9910u, sel1 = 0x1099u, sel2 = 0xBB32u, sel3 = 0x32BBu;
    if (kRows == 4 && (p & 1) != (r >> 2)) sel0 = sel1 = sel2 = sel3 = 0x9999u;

    // (kept in registers: worked out anew at every use, these cost as much as the rest of the loop)
#pragma unroll
    for (int i = 0; i < kKWords; ++i) asm volatile("" : "+r"(koff[i]));
#pragma unroll
    for (int m = 0; m < kVGroups; ++m) asm volatile("" : "+r"(voff[m]));
    asm volatile("" : "+r"(sel0), "+r"(sel1), "+r"(sel2), "+r"(sel3), "+l"(src_lane));

    // ---- the items of the stretch
    struct Item {
        int head, seq, tile, tiles, row0, rows;                                  // rows row0 ... of the sequence's (query token, head) rows
        int q_first, before_q;                                              // the sequence's first row of q; its tokens before the new ones
        int pos_lo, pos_hi;                                                 // positions of the first and the last row
        int n, sb, wb0, xa, xb, v_end;                                      // tokens; blocks of sinks, first block of a window, the part of the blocks
        bool begins, ends;                                                  // whether that part is the item's first, its last
    };
    auto place_tile = [&](Item& it) {                                       // what follows from the number of its row tile
        it.row0 = it.tile * kRows;
        it.rows = it.n - it.before_q;                                       // (new tokens)
        it.rows = it.rows * R - it.row0 < kRows ? it.rows * R - it.row0 : kRows;
        it.pos_lo = it.before_q + it.row0 / R;
        it.pos_hi = it.before_q + (it.row0 + it.rows - 1) / R;
        // the blocks that some row sees: those of the sinks, then from the first window on
        it.wb0 = window_first(it.pos_lo, a.window) / kTokenBlock;
        it.sb = a.window ? (a.sinks + kTokenBlock - 1) / kTokenBlock : 0;
        it.sb = it.sb < it.wb0 ? it.sb : it.wb0;
        const int last = kMode == kMass && it.tile == 0 ? it.n - 1 : it.pos_hi;      // (masses: the first tile takes what was there along)
        const int n_blocks = last < 0 ? 0 : it.sb + last / kTokenBlock + 1 - it.wb0;
        it.v_end = it.xb < n_blocks ? it.xb : n_blocks;
    };
    SeqView here = seq_view(a, seq), ahead = here;                          // of the sequence at x, and of the next one
    auto look_ahead = [&]() { ahead = seq_view(a, seq + 1 == n_seq ? 0 : seq + 1); };
    auto take = [&](Item& it) {                                             // the item at x; the same in all threads
        while (x < x_end && head < sh.n_kv_heads) {
            const SeqView sv = here;
            const Cost cost = cost_of<kRows, kMode>(a, sv);
            if ((int64_t)cost.tiles * cost.blocks <= rest) {                // the sequence is done (or belongs to another kernel)
                rest -= (int64_t)cost.tiles * cost.blocks;
                if (++seq == n_seq) { seq = 0; ++head; }
                here = ahead;
                look_ahead();
                continue;
            }
            it.head = head;
            it.seq = seq;
            it.tile = (int)(rest / cost.blocks);
            it.tiles = (sv.m * R + kRows - 1) / kRows;
            it.xa = (int)(rest - (int64_t)it.tile * cost.blocks);
            const int xb = cost.blocks - it.xa < x_end - x ? cost.blocks : it.xa + (int)(x_end - x);
            it.begins = it.xa == 0;
            it.ends = xb == cost.blocks;
            it.q_first = sv.row0;
            it.before_q = sv.n - sv.m;
            it.n = sv.n;
            it.xb = xb;
            place_tile(it);
            x += xb - it.xa;
            rest += xb - it.xa;
            return true;
        }
        return false;
    };
    // The warp's i-th block of an item (-1: none), and where it lies (bit 0: some row does not see all of it; -1: nowhere).
    auto block_of = [&](const Item& it, int i) {
        const int v = it.xa + warp + i * kWarps;
        return v >= it.v_end ? -1 : v < it.sb ? v : v - it.sb + it.wb0;
    };
    auto look_up = [&](const Item& it, int i) -> int64_t {
        const int blk = block_of(it, i), t0 = blk * kTokenBlock;
        if (blk < 0) return -1;
        const bool all_seen = t0 + kTokenBlock - 1 <= it.pos_lo && (a.window == 0 || t0 > it.pos_hi - a.window || t0 + kTokenBlock <= a.sinks);
        const int64_t at = block_offset(a, it.seq, it.head, blk);
        return at < 0 ? -1 : at | (all_seen ? 0 : 1);
    };
    auto copy_queries = [&](const Item& it) {                               // (rows beyond the tile's: its last one)
        if (threadIdx.x < kRows * 16) {
            const int i = (int)threadIdx.x >> 4, row = it.row0 + (i < it.rows ? i : it.rows - 1);
            copy16((uint32_t)__cvta_generic_to_shared(smem + C::kQOffset) + 16 * threadIdx.x,
                           a.q + (((int64_t)it.q_first + row / R) * sh.n_q_heads + it.head * R + row % R) * 128 + 8 * (threadIdx.x & 15));
        }
        if (kMode == kMass && threadIdx.x < kRows / 4)
            copy16((uint32_t)__cvta_generic_to_shared(smem + C::kQOffset) + 2048 + 16 * threadIdx.x,
                   mass.lse + ((int64_t)it.seq * sh.n_kv_heads + it.head) * mass.row_stride + it.row0 + 4 * threadIdx.x);
    };
    // Centroids of a head: two bulk copies bring them as they lie in memory ([group][code]) into the places of the two value copies;
    // `lay_out` turns them code-major, the values twice, the second time with the halves of a 128-byte line exchanged.  It goes along
    // diagonals: the lanes that access shared memory together take different codes of different groups, so that neither side of
    // the transposition has conflicts.  (Loads that scatter into place cost a tag per 16 bytes: 12 thousand cycles.)
    // (Without values the keys are turned in place.)
    constexpr int kKRaw = kMode == kAttn ? kVOffset : kKOffset, kVRaw = kVOffset + kBookBytes;
    uint32_t book_phase = 0u;
    auto copy_books = [&](int of) {
        if (threadIdx.x == 0) {
            const uint32_t bytes = (uint32_t)(G * sh.K * kC) * 2u;
            fence_async_smem();
            mbar_expect_tx(book_bar, kMode == kAttn ? 2 * bytes : bytes);
            bulk_copy_g2s(smem + kKRaw, a.kcb + (int64_t)of * G * sh.K * kC, bytes, book_bar);
            if (kMode == kAttn) bulk_copy_g2s(smem + kVRaw, a.vcb + (int64_t)of * G * sh.K * kC, bytes, book_bar);
        }
    };
    auto lay_out = [&]() -> bool {
        const bool there = mbar_wait(book_bar, book_phase);
        if (__syncthreads_or(!there)) {                                     // (a copy that never came: the caller gives up)
            mbar_wait(book_bar, book_phase);
            return false;
        }
        book_phase ^= 1u;
        constexpr int kWide = kC == 8 ? 8 : kC == 4 ? 16 : 32;              // lanes that access shared memory together
        constexpr int kTasks = (G / kWide) * (256 * kWide / 32);            // of a warp: 32 / kWide codes of kWide groups
        constexpr int kMine = (kTasks + kWarps - 1) / kWarps;
        auto place = [&](int task, int& from, int& to) {                    // bytes in the raw and in the laid out book; whether there is such a code
            const int g = (task % (G / kWide)) * kWide + lane % kWide;
            const int step = (task / (G / kWide)) * (32 / kWide) + lane / kWide;       // of the kWide steps of a square of codes and groups
            const int j = step / kWide * kWide + (step + lane) % kWide;
            from = (g * sh.K + j) * 2 * kC;
            to = j * 256 + g * 2 * kC;
            return j < sh.K;
        };
        auto put = [&](uint8_t* dst, const uint32_t (&w)[E]) {
            if (E == 4) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1 % E], w[2 % E], w[3 % E]);
            else if (E == 2) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1 % E]);
            else *reinterpret_cast<uint32_t*>(dst) = w[0];
        };
        uint32_t v[kMine][E];
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int task = warp + i * kWarps;
            if (task >= kTasks) break;
            int from, to;
            const bool is = place(task, from, to);
            uint32_t k[E];
#pragma unroll
            for (int e = 0; e < E; ++e) k[e] = v[i][e] = 0u;                // (codes of tokens that nobody sees may name these)
            if (is && kMode == kAttn) load_words<E>(k, smem + kKRaw + from);
            if (is) load_words<E>(v[i], smem + (kMode == kAttn ? kVRaw : kKRaw) + from);
            if (kMode == kAttn) put(smem + kKOffset + to, k);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
            const int task = warp + i * kWarps;
            if (task >= kTasks) break;
            int from, to;
            place(task, from, to);
            put(smem + (kMode == kAttn ? kVOffset : kKOffset) + to, v[i]);
            if (kMode == kAttn) put(smem + kVOffset + kBookBytes + (to ^ 64), v[i]);
        }
        __syncthreads();
        return true;
    };

    int loaded = head < sh.n_kv_heads ? head : -1;
    if (threadIdx.x == 0) {
        mbar_init(book_bar, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        copy_books(head);
    }
    __syncthreads();
    look_ahead();
    Item it, next;
    bool more = take(it), laid_out = false, broken = false;
    int64_t where = more ? look_up(it, lane) : -1;                          // lane i: where the i-th of the warp's next 32 blocks lies
    if (more) copy_queries(it);
    while (more) {
        if (loaded != it.head) {
            loaded = it.head;
            laid_out = false;
            copy_books(loaded);
        }
        copies_issued();
        uint32_t partial_now = 0u;                                          // bits of the blocks on their way that need a mask, the oldest lowest
        auto fetch = [&](int turn) {                                        // starts the copies of a block
            const int64_t off = __shfl_sync(0xffffffffu, where, turn & 31);
            const uint32_t dst = stage_addr + (turn % kStages) * kBlockBytes;
            if (off >= 0) {
                const uint8_t* src = src_lane + (off & ~(int64_t)1);
                if (kMode != kAttn && G == 16) {
                    if (lane < 16) copy16(dst, src);
                } else {
#pragma unroll
                    for (int i = 0; i < kBlockBytes / 512; ++i)
                        copy16(dst + 512 * i, G == 16 ? src : src + (i < G / 32 ? 512 * i : from_v + 512 * (i - G / 32)));
                }
            }
            partial_now |= (uint32_t)(off & 1) << (kStages - 1);
            copies_issued();
            if ((turn & 31) == 31) where = look_up(it, turn + 1 + lane);
        };
        const int left = it.v_end - it.xa - warp, turns = left <= 0 ? 0 : (left + kWarps - 1) / kWarps;
#pragma unroll
        for (int i = 0; i < kStages; ++i) {
            fetch(i);
            if (i < kStages - 1) partial_now >>= 1;
        }
        if (!laid_out) {
            copies_wait<kStages>();                                         // the first item's queries
            broken |= !lay_out();
            laid_out = true;
        }
        // the lane's row of scores: p of four, r of eight (rows beyond the tile's: its last one)
        constexpr int kQF = kRows == 4 ? 2 : 4;
        const int my_row = kRows == 4 ? p : r;
        const int pos = it.before_q + (it.row0 + (my_row < it.rows ? my_row : it.rows - 1)) / R;
        uint32_t qf[4][kQF];
        {
            const uint32_t* qr = reinterpret_cast<const uint32_t*>(smem + C::kQOffset) + (kRows == 4 ? r >> 1 : r) * 64;
            auto word = [&](int w, int h) { return signed_query(qr[(8 * (w / E) + 4 * h + p) * E + w % E], q_sign); };       // w of half h
#pragma unroll
            for (int w = 0; w < 8; ++w) {
                if (kRows == 4) {
                    qf[w >> 1][w & 1] = word(w, r & 1);
                } else {
                    qf[w >> 1][(2 * (w & 1)) % kQF] = word(w, 0);
                    qf[w >> 1][(2 * (w & 1) + 1) % kQF] = word(w, 1);
                }
            }
        }
        float acc[kNT][4];
#pragma unroll
        for (int i = 0; i < kNT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
        float m_ref = -INFINITY, l = 0.f;                                   // kMass: m_ref is the row's log-sum-exp
        float* sums = nullptr;
        float was[kRows == 4 ? 2 : 4];                                      // sums so far of the tokens that are weighed next
        auto look_back = [&](int turn) {
            if constexpr (kMode == kMass) {
                const int blk = block_of(it, turn), t0 = blk * kTokenBlock + (kRows == 4 ? 2 * r : 4 * p);
#pragma unroll
                for (int j = 0; j < (kRows == 4 ? 2 : 4); ++j) {
                    was[j] = 0.f;
                    if (blk >= 0 && (kRows == 4 ? p : r) == 0 && t0 + j < it.n && (it.tile > 0 || mass.mass_in))
                        was[j] = it.tile > 0 ? sums[t0 + j] : mass.mass_in[(sums - mass.mass_out) + t0 + j];
                }
            }
        };
        float* scores = nullptr;                                            // the lane's place in a block's
        if (kMode == kLse && kRows == 4 && mass.scores)
            scores = mass.scores + ((int64_t)it.seq * sh.n_kv_heads + it.head) * sh.n_blocks * 64 + p * 16 + 2 * r;
        if constexpr (kMode == kMass) {
            m_ref = reinterpret_cast<const float*>(smem + C::kQOffset + 2048)[my_row];
            sums = mass.mass_out + ((int64_t)it.seq * sh.n_kv_heads + it.head) * sh.max_tokens;
        }

        // Scores run one turn ahead of the sums: the two share no register, so that one's loads and products fill the other's waits.
        auto score = [&](float* sc, const uint8_t* codes) {
            uint32_t kcur[kKWords];
#pragma unroll
            for (int i = 0; i < kKWords; ++i) kcur[i] = *reinterpret_cast<const uint32_t*>(codes + 8 * (i ^ flip) * kTokenBlock);
            auto keys = [&](uint32_t (&w)[8], int j) {                      // words of token 4 tq + j, this lane's groups
#pragma unroll
                for (int i = 0; i < kKWords; ++i) load_words<E>(w + i * E, smem + kKOffset + prmt(kcur[i], koff[i], 0x7704u | ((uint32_t)j << 4)));
                if (E == 2) {                                               // the eights were loaded in the order of i XOR flip
#pragma unroll
                    for (int i = 0; i < 4; i += 2)
#pragma unroll
                        for (int k = 0; k < 2; ++k) {
                            const uint32_t lo = w[2 * i + k], hi = w[2 * i + 2 + k];
                            w[2 * i + k] = flip ? hi : lo;
                            w[2 * i + 2 + k] = flip ? lo : hi;
                        }
                }
                if (E == 1) {
#pragma unroll
                    for (int bit = 1; bit <= 2; bit <<= 1)
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (!(i & bit)) {
                                const uint32_t lo = w[i], hi = w[i | bit];
                                w[i] = flip & bit ? hi : lo;
                                w[i | bit] = flip & bit ? lo : hi;
                            }
                }
            };
            if constexpr (kRows == 4) {
                float part[4];                                              // over the lane's half of the groups, tokens 4 tq + j
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    uint32_t w0[8], w1[8];
                    keys(w0, 2 * t);
                    keys(w1, 2 * t + 1);
                    float d[4];
                    mma16816_first(d, w0[0], w1[0], w0[1], w1[1], qf[0][0], qf[0][1]);
#pragma unroll
                    for (int ks = 1; ks < 4; ++ks) mma16816(d, w0[2 * ks], w1[2 * ks], w0[2 * ks + 1], w1[2 * ks + 1], qf[ks][0], qf[ks][1]);
                    part[2 * t] = r & 1 ? d[1] : d[0];
                    part[2 * t + 1] = r & 1 ? d[3] : d[2];
                }
                // the lane of the other half (r ^ 1) keeps the other two tokens
                const float give0 = r & 1 ? part[0] : part[2], give1 = r & 1 ? part[1] : part[3];
                sc[0] = (r & 1 ? part[2] : part[0]) + __shfl_xor_sync(0xffffffffu, give0, 4);
                sc[1] = (r & 1 ? part[3] : part[1]) + __shfl_xor_sync(0xffffffffu, give1, 4);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    uint32_t w[8];
                    keys(w, j);
                    float d[4];
                    mma16816_first(d, qf[0][0], qf[0][1], qf[0][2 % kQF], qf[0][3 % kQF], w[0], w[1]);
#pragma unroll
                    for (int ks = 1; ks < 4; ++ks) mma16816(d, qf[ks][0], qf[ks][1], qf[ks][2 % kQF], qf[ks][3 % kQF], w[2 * ks], w[2 * ks + 1]);
                    sc[j] = d[0] + d[3];
                }
            }
        };
        // Four rows: a lane has the scores of row p, tokens 2 r + {0, 1}; eight: of row r, tokens 4 p + {0 ... 3}.
        constexpr int kSc = kRows == 4 ? 2 : 4, kX = kRows == 4 ? 4 : 2;
        uint32_t x[kX];                                                     // weights, in twos, as `sum` takes them
        auto weigh = [&](float (&sc)[kSc], int turn, uint32_t partial) {
            if (partial) {
                // (a block that is not there, or lies in no page: no token)
                const int blk = block_of(it, turn);
                const int t0 = blk < 0 || page_index(a, it.seq, blk) < 0 ? INT_MAX - 16 : blk * kTokenBlock + (kRows == 4 ? 2 * r : 4 * p);
#pragma unroll
                for (int j = 0; j < kSc; ++j)
                    if (!token_visible(t0 + j, pos, a.window, a.sinks)) sc[j] = -INFINITY;
            }
            // ---- weights.  Their reference follows the row's maximum only when it is more than 8 (a factor of 256) behind: fp16
            // weights up to 256 are as precise as weights up to 1, and the sums are rarely rescaled.
            if constexpr (kMode == kMass) {
                // the rows' weights of a token add up across the lanes that hold them; one lane of them has the sum so far
                float w[kSc];
#pragma unroll
                for (int j = 0; j < kSc; ++j) {
                    w[j] = my_row < it.rows && sc[j] != -INFINITY ? ex2f(fmaf(sc[j], scale, -m_ref)) : 0.f;      // (a row that sees nothing: -inf)
#pragma unroll
                    for (int o = kRows == 4 ? 1 : 4; o <= (kRows == 4 ? 2 : 16); o <<= 1) w[j] += __shfl_xor_sync(0xffffffffu, w[j], o);
                }
                const int blk = block_of(it, turn), t0 = blk * kTokenBlock + (kRows == 4 ? 2 * r : 4 * p);
                if (blk >= 0 && (kRows == 4 ? p : r) == 0)
#pragma unroll
                    for (int j = 0; j < kSc; ++j)
                        if (t0 + j < it.n) sums[t0 + j] = was[j] + (broken ? __int_as_float(0x7fffffff) : w[j]);
            } else {
                float top = fmaxf(sc[0], sc[1]);
                if (kSc == 4) top = fmaxf(top, fmaxf(sc[2 % kSc], sc[3 % kSc]));
                top *= scale;
                if (__any_sync(0xffffffffu, top > m_ref + 8.f)) {
#pragma unroll
                    for (int o = kRows == 4 ? 4 : 1; o <= (kRows == 4 ? 16 : 2); o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
                    const float m_new = fmaxf(m_ref, top);
                    float f = m_ref == -INFINITY ? 0.f : ex2f(m_ref - m_new);
                    m_ref = m_new;
                    l *= f;
                    if constexpr (kMode == kAttn) {
                        if (kRows == 4) f = __shfl_sync(0xffffffffu, f, r & 3); // (the accumulators are row r & 3's)
#pragma unroll
                        for (int i = 0; i < kNT; ++i)
#pragma unroll
                            for (int k = 0; k < 4; ++k) acc[i][k] *= f;
                    }
                }
                const float ref = m_ref == -INFINITY ? 0.f : m_ref;
                if constexpr (kMode == kLse) {
#pragma unroll
                    for (int j = 0; j < kSc; ++j) l += ex2f(fmaf(sc[j], scale, -ref));
                    const int blk = block_of(it, turn);
                    if (kRows == 4 && scores && blk >= 0)
                        *reinterpret_cast<float2*>(scores + (int64_t)blk * 64) = make_float2(sc[0] * scale, sc[1] * scale);
                } else {
                    uint32_t y[kSc / 2];
#pragma unroll
                    for (int j = 0; j < kSc / 2; ++j) {
                        const __half2 h = __floats2half2_rn(ex2f(fmaf(sc[2 * j], scale, -ref)), ex2f(fmaf(sc[2 * j + 1], scale, -ref)));
                        const float2 f = __half22float2(h);                         // (the normaliser sums the weights as they are used)
                        l += f.x + f.y;
                        y[j] = *reinterpret_cast<const uint32_t*>(&h);
                    }
#pragma unroll
                    for (int i = 0; i < kX; ++i) x[i] = kRows == 4 ? __shfl_sync(0xffffffffu, y[0], (2 * (p & 2) + i) * 4 + (r & 3)) : y[i % (kSc / 2)];
                }
            }
        };
        // Four rows: row r & 3, tokens 8 (p / 2) + {0 ... 7}; eight: row r, tokens 4 p + {0 ... 3}
        auto sum = [&](const uint8_t* codes) {
            uint32_t vcur[kVWords];
#pragma unroll
            for (int m = 0; m < kVGroups; ++m) {
                const uint8_t* at = codes + m * ((kRows == 4 ? 2 : 1) * kLow * E * kTokenBlock);
                if (kRows == 4) {
                    const uint2 two = *reinterpret_cast<const uint2*>(at);
                    vcur[(2 * m) % kVWords] = two.x;
                    vcur[(2 * m + 1) % kVWords] = two.y;
                } else {
                    vcur[m % kVWords] = *reinterpret_cast<const uint32_t*>(at);
                }
            }
#pragma unroll
            for (int i = 0; i < kX; ++i) {
                const uint32_t a0 = prmt(x[i], x[i], sel0), a1 = prmt(x[i], x[i], sel1), a2 = prmt(x[i], x[i], sel2), a3 = prmt(x[i], x[i], sel3);
#pragma unroll
                for (int m = 0; m < kVGroups; ++m) {
                    uint32_t b[2][E];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int at = 2 * i + e;                           // of the lane's four or eight
                        const uint32_t word = vcur[kRows == 4 ? (2 * m + (at >> 2)) % kVWords : m % kVWords];
                        load_words<E>(b[e], smem + kVOffset + prmt(word, voff[m], 0x7604u | ((uint32_t)(at & 3) << 4)));
                    }
#pragma unroll
                    for (int w = 0; w < E; ++w) mma16816(acc[(m * E + w) % kNT], a0, a1, a2, a3, b[0][w], b[1][w]);
                }
            }
        };
        if (turns > 0) {
            // Turn i: sums of block i, scores of block i + 1, and the copies of block i + kStages start when its place is free.
            float sc[kSc];
            copies_wait<kStages - 1>();
            __syncwarp();
            look_back(0);
            score(sc, k_codes);
            weigh(sc, 0, partial_now & 1u);
            partial_now >>= 1;
#pragma unroll 1
            for (int turn = 0; turn < turns; ++turn) {
                copies_wait<kStages - 2>();                                 // those of block turn + 1 are there
                __syncwarp();
                look_back(turn + 1);
                score(sc, k_codes + ((turn + 1) % kStages) * kBlockBytes);
                if constexpr (kMode == kAttn) sum(v_codes + (turn % kStages) * kBlockBytes);
                weigh(sc, turn + 1, partial_now & 1u);
                __syncwarp();
                fetch(turn + kStages);
                partial_now >>= 1;
            }
        }
        copies_wait_all();
        bool more_next = true;
        if (kMode == kMass && it.tile + 1 < it.tiles) {
            next = it;
            ++next.tile;
            place_tile(next);
        } else {
            more_next = take(next);
        }
        const int64_t where_next = more_next ? look_up(next, lane) : -1;    // (needed when the sums are done)

        if constexpr (kMode == kMass) {
            __syncthreads();
            if (more_next) copy_queries(next);                              // (this item's have been read)
            copies_wait_all();
            __syncthreads();
        } else {
            // ---- the warps' sums to one
            // Every warp brings its accumulators to the largest reference; then they are plain sums.
#pragma unroll
            for (int o = kRows == 4 ? 4 : 1; o <= (kRows == 4 ? 16 : 2); o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
            const bool speaks = kRows == 4 ? r == 0 : p == 0;                   // for its row
            if (speaks) wm[warp * 8 + my_row] = m_ref;
            __syncthreads();
            if (more_next) copy_queries(next);                                  // (this item's have been read)
            float M = -INFINITY;
#pragma unroll
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w * 8 + my_row]);
            float bring = m_ref == -INFINITY ? 0.f : ex2f(m_ref - M);
            if (speaks) wl[warp * 8 + my_row] = l * bring;
            if (kRows == 4) bring = __shfl_sync(0xffffffffu, bring, r & 3);
            const bool whole = it.begins && it.ends;
            float* part = partials + (int64_t)(2 * blockIdx.x + (it.begins ? 1 : 0)) * partial_floats(kRows, kMode);
            if constexpr (kMode == kLse) {
                __syncthreads();
                if (threadIdx.x < kRows) {                                      // (the first lane of a row's lanes holds the largest reference)
                    float L = 0.f, top = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        L += wl[w * 8 + threadIdx.x];
                        top = fmaxf(top, wm[w * 8 + threadIdx.x]);
                    }
                    if (broken) L = __int_as_float(0x7fffffff);
                    if (!whole) {
                        part[threadIdx.x] = top;
                        part[kRows + threadIdx.x] = L;
                    } else if ((int)threadIdx.x < it.rows) {
                        mass.lse[((int64_t)it.seq * sh.n_kv_heads + it.head) * mass.row_stride + it.row0 + threadIdx.x] = top + log2f(L);
                    }
                }
            }
            if constexpr (kMode == kAttn) {
                float* mine = reinterpret_cast<float*>(stage0);
#pragma unroll
                for (int i = 0; i < kNT * 4; ++i) mine[i * 32 + lane] = acc[i >> 2][i & 3] * bring;
                __syncthreads();
#pragma unroll 2
                for (int reg = warp; reg < kNT * 4; reg += kWarps) {                // this warp sums one register of all warps, lane by lane
                    int row, channel;
                    place_of<kC, kRows>(reg, lane, row, channel);
                    float L = 0.f, sum_of = 0.f;
#pragma unroll
                    for (int w = 0; w < kWarps; ++w) {
                        L += wl[w * 8 + row];
                        sum_of += reinterpret_cast<const float*>(smem + C::kStageOffset + w * kWarpBytes)[reg * 32 + lane];
                    }
                    if (broken) sum_of = __int_as_float(0x7fffffff);                // (nothing that could be taken for a result)
                    if (whole) {
                        if (row < it.rows) {
                            const int at = it.row0 + row;
                            a.out[(((int64_t)it.q_first + at / R) * sh.n_q_heads + it.head * R + at % R) * 128 + channel] = __float2half_rn(L == 0.f ? sum_of : sum_of / L);
                        }
                    } else {
                        part[2 * kRows + reg * 32 + lane] = sum_of;
                        if (reg == 0 && p == 0 && r < kRows) part[kRows + row] = L;
                    }
                }
                if (!whole && warp == 0 && speaks) part[my_row] = M;
            }
            copies_wait_all();
            __syncthreads();
            if (!whole && threadIdx.x == 0) {
                Cut c;
                c.head = it.head; c.seq = it.seq; c.tile = it.tile; c.state = it.ends ? 2 : 1;
                cuts[2 * blockIdx.x + (it.begins ? 1 : 0)] = c;
            }
        }
        it = next;
        where = where_next;
        more = more_next;
    }
    if (!laid_out) mbar_wait(book_bar, book_phase);                         // (no copy may outlive the CTA)
}

// CTA k merges the item that begins in CTA k's stretch and goes on in the next ones'.
template <int kC, int kRows, int kMode>
__global__ void __launch_bounds__(kMode == kAttn ? 512 : 32)
gather_merge_kernel(BoundedArgs a, MassArgs mass, const float* __restrict__ partials, const Cut* __restrict__ cuts, int n_ctas)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int k = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Cut first = cuts[2 * k + 1];
    if (first.state == 0) return;
    int last = k + 1;                                                       // the CTA in whose stretch the item ends
    for (int j0 = k + 1;; j0 += 32) {
        const int j = j0 + lane;
        const uint32_t stop = __ballot_sync(0xffffffffu, j >= n_ctas - 1 || cuts[2 * j].state != 1);
        if (stop) { last = j0 + __ffs(stop) - 1; break; }
    }
    last = last < n_ctas - 1 ? last : n_ctas - 1;
    const SeqView sv = seq_view(a, first.seq);
    const int R = a.sh.R, row0 = first.tile * kRows;
    if constexpr (kMode == kLse) {
        if (lane >= kRows || row0 + lane >= sv.m * R) return;
        auto part = [&](int j) { return partials + (int64_t)(2 * j + (j == k)) * partial_floats(kRows, kMode) + lane; };
        float M = -INFINITY, L = 0.f;
#pragma unroll 4
        for (int j = k; j <= last; ++j) M = fmaxf(M, part(j)[0]);
#pragma unroll 4
        for (int j = k; j <= last; ++j) L = fmaf(part(j)[0] == -INFINITY ? 0.f : ex2f(part(j)[0] - M), part(j)[kRows], L);
        mass.lse[((int64_t)first.seq * a.sh.n_kv_heads + first.head) * mass.row_stride + row0 + lane] = M + log2f(L);
    } else {
        for (int reg = warp; reg < (kRows == 4 ? 16 : 32); reg += 16) {
            int row, channel;
            place_of<kC, kRows>(reg, lane, row, channel);
            auto part = [&](int j) { return partials + (int64_t)(2 * j + (j == k)) * partial_floats(kRows, kMode); };
            float M = -INFINITY, L = 0.f, sum = 0.f;
#pragma unroll 4
            for (int j = k; j <= last; ++j) M = fmaxf(M, part(j)[row]);
#pragma unroll 4
            for (int j = k; j <= last; ++j) {
                const float mj = part(j)[row], f = mj == -INFINITY ? 0.f : ex2f(mj - M);
                L = fmaf(f, part(j)[kRows + row], L);
                sum = fmaf(f, part(j)[2 * kRows + reg * 32 + lane], sum);
            }
            const int at = row0 + row;
            if (at < sv.m * R)
                a.out[(((int64_t)sv.row0 + at / R) * a.sh.n_q_heads + first.head * R + at % R) * 128 + channel] = __float2half_rn(L == 0.f ? sum : sum / L);
        }
    }
}

constexpr int kStreamThreads = 256, kStreamEach = 4;                        // tokens of a thread

// Masses from stored scores of up to four rows: a thread per token, the rows' weights in the order of the rows.
__global__ void __launch_bounds__(kStreamThreads) mass_of_scores_kernel(BoundedArgs a, MassArgs mass, int chunks)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int64_t item = blockIdx.x / chunks;                               // (sequence, KV head)
    const int64_t n64 = a.seq_lens[item / a.sh.n_kv_heads];
    const int n = (int)(n64 < 0 ? 0 : (n64 > a.sh.max_tokens ? a.sh.max_tokens : n64));
    const int t0 = (int)(blockIdx.x % chunks) * (kStreamThreads * kStreamEach) + (int)threadIdx.x;
    if (t0 - (int)threadIdx.x >= n) return;
    const int rows = a.max_q * a.sh.R;
    float lse[4], x[kStreamEach][4], was[kStreamEach];
#pragma unroll
    for (int r = 0; r < 4; ++r) lse[r] = r < rows ? mass.lse[item * mass.row_stride + r] : 0.f;
    const float* scores = mass.scores + item * a.sh.n_blocks * 64;
#pragma unroll
    for (int u = 0; u < kStreamEach; ++u) {
        const int t = t0 + u * kStreamThreads;
#pragma unroll
        for (int r = 0; r < 4; ++r) x[u][r] = t < n && r < rows ? scores[(int64_t)(t / kTokenBlock) * 64 + r * 16 + t % kTokenBlock] : -INFINITY;
        was[u] = t < n && mass.mass_in ? mass.mass_in[item * a.sh.max_tokens + t] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < kStreamEach; ++u) {
        const int t = t0 + u * kStreamThreads;
        float w = 0.f;
#pragma unroll
        for (int r = 0; r < 4; ++r) w += x[u][r] == -INFINITY ? 0.f : ex2f(x[u][r] - lse[r]);
        if (t < n) mass.mass_out[item * a.sh.max_tokens + t] = was[u] + w;
    }
}

template <int kC, int kRows, int kMode>
cudaError_t launch(const BoundedArgs& a, const MassArgs& mass, void* workspace, int slot, cudaStream_t st)
{
    using C = Cfg<kMode>;
    const int grid = device_sm_count() * C::kCtas;
    Cut* cuts = static_cast<Cut*>(workspace);
    float* partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up(2 * grid * sizeof(Cut), 256));
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(gather_kernel<kC, kRows, kMode>), C::kSmemBytes, slot);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = overlapped_config((unsigned)grid, C::kThreads, C::kSmemBytes, st, &attr);
    e = cudaLaunchKernelEx(&cfg, gather_kernel<kC, kRows, kMode>, a, mass, partials, cuts);
    if (e != cudaSuccess || kMode == kMass) return e;
    cfg.dynamicSmemBytes = 0;
    cfg.blockDim = dim3(kMode == kAttn ? 512 : 32);
    cfg.gridDim = dim3((unsigned)(grid - 1 > 0 ? grid - 1 : 1));
    return cudaLaunchKernelEx(&cfg, gather_merge_kernel<kC, kRows, kMode>, a, mass, (const float*)partials, (const Cut*)cuts, grid);
}

size_t cuts_bytes(int mode) { return round_up(2 * (size_t)device_sm_count() * (mode == kAttn ? 1 : 2) * sizeof(Cut), 256); }
size_t gather_bytes(int mode)
{
    return cuts_bytes(mode) + round_up(2 * (size_t)device_sm_count() * (mode == kAttn ? 1 : 2) * partial_floats(8, mode) * sizeof(float), 256);
}
int mass_row_stride(const BoundedArgs& a) { return (a.max_q * a.sh.R + 7) / 8 * 8; }

template <int kMode>
cudaError_t launch_mode(const BoundedArgs& a, const MassArgs& mass, void* workspace, int slot, cudaStream_t st)      // call-site slots from `slot` on: six
{
    // Tiles of four rows where a query token has that few heads, otherwise of eight: with four rows no two lanes meet in a bank.
    // (Masses of many rows go over the keys once per tile: eight rows at a time from 16 rows on.)
    const bool four = kMode == kAttn ? a.sh.R <= 4 : a.max_q * a.sh.R <= 4;
    if (a.sh.c == 8) return four ? launch<8, 4, kMode>(a, mass, workspace, slot, st) : launch<8, 8, kMode>(a, mass, workspace, slot + 1, st);
    if (a.sh.c == 4) return four ? launch<4, 4, kMode>(a, mass, workspace, slot + 2, st) : launch<4, 8, kMode>(a, mass, workspace, slot + 3, st);
    return four ? launch<2, 4, kMode>(a, mass, workspace, slot + 4, st) : launch<2, 8, kMode>(a, mass, workspace, slot + 5, st);
}

}  // namespace

bool gather_attn_supported(const Shape& sh) { return sh.head_dim == 128 && sh.b <= 8 && (sh.c == 2 || sh.c == 4 || sh.c == 8); }

size_t gather_attn_workspace_bytes() { return gather_bytes(kAttn); }
cudaError_t launch_gather_attn(const BoundedArgs& a, void* workspace, cudaStream_t st) { return launch_mode<kAttn>(a, MassArgs(), workspace, 128, st); }

namespace {
size_t lse_bytes(const BoundedArgs& a) { return gather_bytes(kLse) + round_up((size_t)a.sh.n_seq * a.sh.n_kv_heads * mass_row_stride(a) * sizeof(float), 256); }
// Bytes of the scores of one step's rows, where they are few: 16 bytes per cached token and KV head, as many as the key codes of c = 8.
size_t score_bytes(const BoundedArgs& a) { return a.max_q * a.sh.R <= 4 ? (size_t)a.sh.n_seq * a.sh.n_kv_heads * a.sh.n_blocks * 64 * sizeof(float) : 0; }
}  // namespace

size_t gather_mass_workspace_bytes(const BoundedArgs& a) { return lse_bytes(a) + score_bytes(a); }
size_t gather_mass_least_bytes(const BoundedArgs& a) { return lse_bytes(a); }
// With room for the scores the second pass reads them; otherwise it works them out again.
cudaError_t launch_gather_mass(const BoundedArgs& a, const float* mass_in, float* mass_out, void* workspace, size_t workspace_bytes, cudaStream_t st)
{
    MassArgs mass;
    mass.mass_in = mass_in;
    mass.mass_out = mass_out;
    mass.lse = reinterpret_cast<float*>(static_cast<char*>(workspace) + gather_bytes(kLse));
    mass.row_stride = mass_row_stride(a);
    const bool store = score_bytes(a) && workspace_bytes >= gather_mass_workspace_bytes(a);
    mass.scores = store ? reinterpret_cast<float*>(static_cast<char*>(workspace) + lse_bytes(a)) : nullptr;
    const cudaError_t e = launch_mode<kLse>(a, mass, workspace, 134, st);
    if (e != cudaSuccess) return e;
    if (!store) return launch_mode<kMass>(a, mass, workspace, 140, st);
    const int64_t chunks = (a.sh.max_tokens + kStreamThreads * kStreamEach - 1) / (kStreamThreads * kStreamEach), grid = a.sh.n_seq * a.sh.n_kv_heads * chunks;
    if (grid > 0x7fffffff) return cudaErrorInvalidConfiguration;
    cudaLaunchAttribute attr;
    const cudaLaunchConfig_t cfg = overlapped_config((unsigned)grid, kStreamThreads, 0, st, &attr);
    return cudaLaunchKernelEx(&cfg, mass_of_scores_kernel, a, mass, (int)chunks);
}

}  // namespace cq
