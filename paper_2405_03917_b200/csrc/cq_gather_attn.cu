// Attention of few query rows over a coded cache: window, sinks, pages (head_dim 128, one byte per code, c = 2, 4 or 8).
//
//   out_r = sum_t p_rt Vhat_t / sum_t p_rt,  p_rt = 2^(scale log2e <q_r, Khat_t> - m_r)      r: (query token, head) of a KV head
//
// Both codebooks lie in shared memory as fp16, code-major: row j holds the centroids j of all groups (256 bytes).  A warp takes blocks
// of 16 tokens; its lanes load centroids as they lie there into the fragments of m16n8k16 MMAs, so no tile of keys or values is
// ever written.  What makes that possible without bank conflicts is the choice of what a fragment's rows and columns mean:
//   scores: a column of B is (token, half of the groups): the eight lanes that load one token together take eight different groups.
//       The rows of A hold every query twice, rows r with the channels of one half and rows r + 8 with those of the other, so
//       that a token's score is the sum of two accumulators of one lane.
//   sums:   a loaded word holds two neighbouring channels of ONE token, but the contraction runs over tokens.  So the k pair
//       (2i, 2i + 1) of an MMA is one token, A's rows r hold (p, 0) there and rows r + 8 (0, p): they sum the even and the odd
//       channels.  Lanes of a quad hold different tokens of the same column; in the kernel for four rows the rows of A that are left
//       over select lanes of a quad, so that a column stands for two groups, and a second copy of the value centroids, half a line
//       further on, parts the rest: no conflict.  With eight rows two lanes meet.
// Shared memory: 64 KiB + 2 x 64 KiB of centroids, one CTA of 16 warps per SM.
//
// Work is dealt evenly: the blocks that all (KV head, sequence, row tile) items attend lie on one line, every CTA takes an equal
// stretch of it (a stretch that crosses into another KV head loads that head's centroids), and what a cut item leaves behind
// is merged by a second, small kernel.
#include "cq_bounded.cuh"

namespace cq {

namespace {

constexpr int kWarps = 16, kThreads = kWarps * 32;
constexpr int kBookBytes = 256 * 256;
constexpr int kKOffset = 0, kVOffset = kBookBytes, kRedOffset = 3 * kBookBytes;
constexpr int kRedRegs = 16;                                              // accumulator registers that are reduced at a time
constexpr int kStatOffset = kRedOffset + kWarps * kRedRegs * 32 * 4;
constexpr int kSmemBytes = kStatOffset + 2 * kWarps * 8 * 4 + 256;
static_assert(kSmemBytes <= 227 * 1024, "shared memory");
constexpr int kLeastShare = 16;                                           // blocks that a CTA takes at least: one per warp

__host__ __device__ constexpr int partial_floats(int rows) { return 2 * rows + (rows == 4 ? 16 : 32) * 32; }

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
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// Row tiles of a sequence and the blocks that one of them attends at most (at least one: rows that see nothing are written too).
struct Cost {
    int tiles, blocks;
};
template <int kRows>
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

template <int kC, int kRows>
__global__ void __launch_bounds__(kThreads, 1) gather_attn_kernel(BoundedArgs a, float* __restrict__ partials, Cut* __restrict__ cuts)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    constexpr int G = 128 / kC, E = kC / 2;
    constexpr int kLow = 8 / E;
    constexpr int kKWords = G / 8;                                          // key code words (four tokens each) of a lane
    constexpr int kVGroups = kRows == 4 ? 4 / E : 8 / E;                    // groups of a lane's values
    constexpr int kVWords = kRows == 4 ? 2 * kVGroups : kVGroups;           // their code words (eight or four tokens)
    constexpr int kNT = kRows == 4 ? 4 : 8;                                 // accumulator tiles
    extern __shared__ __align__(1024) uint8_t smem[];
    float* red = reinterpret_cast<float*>(smem + kRedOffset);
    float* wm = reinterpret_cast<float*>(smem + kStatOffset);               // [warp][8]: reference and sum of the weights
    float* wl = wm + kWarps * 8;
    int64_t* scratch = reinterpret_cast<int64_t*>(wl + kWarps * 8);
    const Shape& sh = a.sh;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int r = lane >> 2, p = lane & 3, R = sh.R, n_seq = (int)sh.n_seq;

    // ---- this CTA's stretch of the line
    int64_t per_head = 0;
    for (int s0 = 0; s0 < n_seq; s0 += kThreads) {
        const int s = s0 + (int)threadIdx.x;
        int64_t mine = 0, all;
        if (s < n_seq) {
            const Cost c = cost_of<kRows>(a, seq_view(a, s));
            mine = (int64_t)c.tiles * c.blocks;
        }
        block_prefix(mine, scratch, all);
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
    int64_t rest = x % per_head;                                            // blocks of the sequence before x
    for (int s0 = 0; s0 < n_seq; s0 += kThreads) {
        const int s = s0 + (int)threadIdx.x;
        int64_t mine = 0, all;
        if (s < n_seq) {
            const Cost c = cost_of<kRows>(a, seq_view(a, s));
            mine = (int64_t)c.tiles * c.blocks;
        }
        const int64_t before = block_prefix(mine, scratch, all);
        if (rest >= all) { rest -= all; continue; }
        if (before <= rest && rest < before + mine) { scratch[0] = s; scratch[1] = rest - before; }
        __syncthreads();
        seq = (int)scratch[0];
        rest = scratch[1];
        break;
    }
    __syncthreads();                                                        // (scratch, and the cut records before their next writers)

    // a negative scale: the queries change sign instead; a zero one: they become zero; both are exact
    const uint32_t q_sign = a.scale_log2e < 0.f ? 0x80008000u : 0u, q_keep = a.scale_log2e == 0.f ? 0u : 0xffffffffu;
    const float scale = a.scale_log2e == 0.f ? 1.f : fabsf(a.scale_log2e);

    // ---- lane constants
    const int tq = lane >> 3, hp = lane & 7;                                // scores: token quad of a block, group in its eight
    const int flip = E == 4 ? 0 : E == 2 ? tq & 1 : tq;                     // order of the eights, so that the quads of a load meet in no bank
    uint32_t koff[kKWords];                                                 // byte of the lane's i-th centroid in a row
#pragma unroll
    for (int i = 0; i < kKWords; ++i) koff[i] = (uint32_t)((8 * (i ^ flip) + hp) * 2 * kC);
    uint32_t voff[kVGroups];                                                // the same for values; byte 2: the copy
    int vgroup[kVGroups];
#pragma unroll
    for (int m = 0; m < kVGroups; ++m) {
        vgroup[m] = kRows == 4 ? (r % kLow) * 2 + (p & 1) + 2 * kLow * (r / kLow + E * m) : r % kLow + kLow * (r / kLow + E * m);
        voff[m] = (uint32_t)((vgroup[m] * 2 * kC) ^ ((p >> 1) * 64)) | ((uint32_t)(p >> 1) << 16);
    }
    const uint32_t smem_base = (uint32_t)__cvta_generic_to_shared(smem);

    int loaded = -1;
    while (x < x_end) {
        if (loaded != head) {
            // centroids of the head, code-major; the values twice, the second time with the halves of a 128-byte line exchanged
            loaded = head;
            constexpr int kPer = 8 / kC;                                    // centroids of a 16-byte piece
            constexpr int kSide = 32 / (kC == 8 ? 8 : kC == 4 ? 16 : 32);   // pieces of a group that a warp takes at a time
            constexpr int kWide = 32 / kSide;                               // groups that it takes at a time
            const int pieces = sh.K / kPer > 0 ? sh.K / kPer : 1;           // pieces of a group's codebook
#pragma unroll 1
            for (int tensor = 0; tensor < 2; ++tensor) {
                const __half* book = (tensor ? a.vcb : a.kcb) + (int64_t)head * G * sh.K * kC;
                constexpr int kTasks = (G / kWide) * (256 / kPer / kSide);  // of a warp
                constexpr int kAhead = 8;
#pragma unroll 1
                for (int t0 = warp; t0 < kTasks; t0 += kAhead * kWarps) {
                    uint4 v[kAhead];
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int task = t0 + u * kWarps;
                        const int g = (task % (G / kWide)) * kWide + lane % kWide, piece = (task / (G / kWide)) * kSide + lane / kWide;
                        v[u] = make_uint4(0u, 0u, 0u, 0u);
                        if (task < kTasks && piece < pieces) {
                            if (sh.K >= kPer) {
                                v[u] = reinterpret_cast<const uint4*>(book + (int64_t)g * sh.K * kC)[piece];
                            } else {                                        // two centroids of two channels
                                const uint2 two = *reinterpret_cast<const uint2*>(book + (int64_t)g * sh.K * kC);
                                v[u].x = two.x; v[u].y = two.y;
                            }
                        }
                    }
#pragma unroll
                    for (int u = 0; u < kAhead; ++u) {
                        const int task = t0 + u * kWarps;
                        if (task >= kTasks) break;
                        const int g = (task % (G / kWide)) * kWide + lane % kWide, piece = (task / (G / kWide)) * kSide + lane / kWide;
                        const int at = piece * kPer * 256 + g * 2 * kC;
                        auto put = [&](uint8_t* dst) {
                            if (kC == 8) *reinterpret_cast<uint4*>(dst) = v[u];
                            if (kC == 4) {
                                *reinterpret_cast<uint2*>(dst) = make_uint2(v[u].x, v[u].y);
                                *reinterpret_cast<uint2*>(dst + 256) = make_uint2(v[u].z, v[u].w);
                            }
                            if (kC == 2) {
                                *reinterpret_cast<uint32_t*>(dst) = v[u].x;
                                *reinterpret_cast<uint32_t*>(dst + 256) = v[u].y;
                                *reinterpret_cast<uint32_t*>(dst + 512) = v[u].z;
                                *reinterpret_cast<uint32_t*>(dst + 768) = v[u].w;
                            }
                        };
                        if (tensor == 0) put(smem + kKOffset + at);
                        else { put(smem + kVOffset + at); put(smem + kVOffset + kBookBytes + (at ^ 64)); }
                    }
                }
            }
            __syncthreads();
        }

        // ---- the item, and the part of it that lies in the stretch
        const SeqView sv = seq_view(a, seq);
        const Cost cost = cost_of<kRows>(a, sv);
        if ((int64_t)cost.tiles * cost.blocks <= rest) {                    // the sequence is done (or belongs to another kernel)
            rest -= (int64_t)cost.tiles * cost.blocks;
            if (++seq == n_seq) { seq = 0; ++head; }
            if (head >= sh.n_kv_heads) break;
            continue;
        }
        const int tile = (int)(rest / cost.blocks), xa = (int)(rest % cost.blocks);
        const int xb = cost.blocks - xa < x_end - x ? cost.blocks : xa + (int)(x_end - x);
        const int row0 = tile * kRows, rows = sv.m * R - row0 < kRows ? sv.m * R - row0 : kRows;
        const int pos_lo = sv.n - sv.m + row0 / R, pos_hi = sv.n - sv.m + (row0 + rows - 1) / R;      // positions of its first and last row
        // the blocks that some row sees: those of the sinks, then from the first window on
        const int wb0 = window_first(pos_lo, a.window) / kTokenBlock;
        int sb = a.window ? (a.sinks + kTokenBlock - 1) / kTokenBlock : 0;
        sb = sb < wb0 ? sb : wb0;
        const int n_blocks = pos_hi < 0 ? 0 : sb + pos_hi / kTokenBlock + 1 - wb0;
        const int v_end = xb < n_blocks ? xb : n_blocks;

        // this lane's row; rows beyond the tile's do as its last one
        const int rho = row0 + (kRows == 4 ? r & 3 : r), my_row = rho < row0 + rows ? rho : row0 + rows - 1;
        const int pos = sv.n - sv.m + my_row / R;
        uint32_t qa[4][4];
        {
            const uint32_t* qr = reinterpret_cast<const uint32_t*>(a.q + (((int64_t)sv.row0 + my_row / R) * sh.n_q_heads + head * R + my_row % R) * 128);
#pragma unroll
            for (int w = 0; w < 8; ++w)
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    qa[w >> 1][2 * (w & 1) + h] = (qr[(8 * (w / E) + 4 * h + p) * E + w % E] ^ q_sign) & q_keep;
        }
        float acc[kNT][4];
#pragma unroll
        for (int i = 0; i < kNT; ++i)
#pragma unroll
            for (int k = 0; k < 4; ++k) acc[i][k] = 0.f;
        float m_ref = -INFINITY, l = 0.f;

        uint32_t kw[kKWords], vw[kVWords];
        int64_t off = -1;
        auto block_of = [&](int v) { return v < sb ? v : v - sb + wb0; };
        auto load = [&](int v) {
            off = v < v_end ? block_offset(a, seq, head, block_of(v)) : -1;
            const uint8_t *kp = a.kc + off, *vp = a.vc + off;
#pragma unroll
            for (int i = 0; i < kKWords; ++i)
                kw[i] = off >= 0 ? *reinterpret_cast<const uint32_t*>(kp + (8 * (i ^ flip) + hp) * kTokenBlock + 4 * tq) : 0u;
#pragma unroll
            for (int m = 0; m < kVGroups; ++m) {
                if (kRows == 4) {
                    uint2 two = make_uint2(0u, 0u);
                    if (off >= 0) two = *reinterpret_cast<const uint2*>(vp + vgroup[m] * kTokenBlock + 8 * (p >> 1));
                    vw[(2 * m) % kVWords] = two.x;
                    vw[(2 * m + 1) % kVWords] = two.y;
                } else {
                    vw[m % kVWords] = off >= 0 ? *reinterpret_cast<const uint32_t*>(vp + vgroup[m] * kTokenBlock + 4 * p) : 0u;
                }
            }
        };
        load(xa + warp);
#pragma unroll 1
        for (int v = xa + warp; v < v_end; v += kWarps) {
            uint32_t kcur[kKWords], vcur[kVWords];
#pragma unroll
            for (int i = 0; i < kKWords; ++i) kcur[i] = kw[i];
#pragma unroll
            for (int i = 0; i < kVWords; ++i) vcur[i] = vw[i];
            const bool here = off >= 0;
            load(v + kWarps);
            if (!here) continue;                                            // (the same in all lanes)
            // ---- scores: this lane's row, tokens 4 p + j of the block
            float sc[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t w[8];
#pragma unroll
                for (int i = 0; i < kKWords; ++i) {
                    const uint32_t at = smem_base + kKOffset + __byte_perm(kcur[i], koff[i], 0x7504u | ((uint32_t)j << 4) | 0x0600u);
                    if (E == 4)
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w[4 * (i % 2)]), "=r"(w[4 * (i % 2) + 1]), "=r"(w[4 * (i % 2) + 2]), "=r"(w[4 * (i % 2) + 3]) : "r"(at));
                    else if (E == 2)
                        asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(w[2 * (i % 4)]), "=r"(w[2 * (i % 4) + 1]) : "r"(at));
                    else
                        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[i % 8]) : "r"(at));
                }
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
                float d[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int ks = 0; ks < 4; ++ks) mma16816(d, qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3], w[2 * ks], w[2 * ks + 1]);
                sc[j] = d[0] + d[3];
            }
            const int t0 = block_of(v) * kTokenBlock;
            const bool all_seen = t0 + kTokenBlock - 1 <= pos_lo && (a.window == 0 || t0 > pos_hi - a.window || t0 + kTokenBlock <= a.sinks);
            if (!all_seen) {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (!token_visible(t0 + 4 * p + j, pos, a.window, a.sinks)) sc[j] = -INFINITY;
            }
            // ---- weights.  Their reference follows the row's maximum only when it is more than 8 (a factor of 256) behind: fp16
            // weights up to 256 are as precise as weights up to 1, and the sums are rarely rescaled.
            const float top = fmaxf(fmaxf(sc[0], sc[1]), fmaxf(sc[2], sc[3])) * scale;
            if (__any_sync(0xffffffffu, top > m_ref + 8.f)) {
                float row_top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
                row_top = fmaxf(row_top, __shfl_xor_sync(0xffffffffu, row_top, 2));
                if (row_top > m_ref) {
                    const float f = m_ref == -INFINITY ? 0.f : ex2f(m_ref - row_top);
                    m_ref = row_top;
                    l *= f;
#pragma unroll
                    for (int i = 0; i < kNT; ++i)
#pragma unroll
                        for (int k = 0; k < 4; ++k) acc[i][k] *= f;
                }
            }
            const float ref = m_ref == -INFINITY ? 0.f : m_ref;
            uint32_t y[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const __half2 h = __floats2half2_rn(ex2f(fmaf(sc[2 * j], scale, -ref)), ex2f(fmaf(sc[2 * j + 1], scale, -ref)));
                const float2 f = __half22float2(h);                         // (the normaliser sums the weights as they are used)
                l += f.x + f.y;
                y[j] = *reinterpret_cast<const uint32_t*>(&h);
            }
            // ---- sums
            constexpr int kSteps = kRows == 4 ? 4 : 2;                      // a step takes two tokens per lane
            uint32_t pw[kSteps];
            if (kRows == 4) {
                // lanes p and p ^ 1 hold the weights of eight tokens; rows 0-3 use the lanes with even p, rows 4-7 the others
                const uint32_t z0 = __shfl_xor_sync(0xffffffffu, y[0], 1), z1 = __shfl_xor_sync(0xffffffffu, y[1], 1);
                const bool active = (p & 1) == (r >> 2), odd = r >> 2;
                pw[0] = active ? (odd ? z0 : y[0]) : 0u;
                pw[1] = active ? (odd ? z1 : y[1]) : 0u;
                pw[2 % kSteps] = active ? (odd ? y[0] : z0) : 0u;
                pw[3 % kSteps] = active ? (odd ? y[1] : z1) : 0u;
            } else {
                pw[0] = y[0];
                pw[1] = y[1];
            }
#pragma unroll
            for (int i = 0; i < kSteps; ++i) {
                const uint32_t a0 = pw[i] & 0xffffu, a1 = pw[i] << 16, a2 = pw[i] >> 16, a3 = pw[i] & 0xffff0000u;
#pragma unroll
                for (int m = 0; m < kVGroups; ++m) {
                    uint32_t b[2][4];
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int tok = 2 * i + e;                          // of the lane's four or eight
                        const uint32_t word = vcur[kRows == 4 ? (2 * m + (tok >> 2)) % kVWords : m % kVWords];
                        const uint32_t at = smem_base + kVOffset + __byte_perm(word, voff[m], 0x7604u | ((uint32_t)(tok & 3) << 4));
                        if (E == 4)
                            asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(b[e][0]), "=r"(b[e][1]), "=r"(b[e][2]), "=r"(b[e][3]) : "r"(at));
                        else if (E == 2)
                            asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(b[e][0]), "=r"(b[e][1]) : "r"(at));
                        else
                            asm volatile("ld.shared.u32 %0, [%1];" : "=r"(b[e][0]) : "r"(at));
                    }
#pragma unroll
                    for (int w = 0; w < E; ++w) mma16816(acc[(m * E + w) % kNT], a0, a1, a2, a3, b[0][w], b[1][w]);
                }
            }
        }

        // ---- the warps' sums to one
        l += __shfl_xor_sync(0xffffffffu, l, 1);
        l += __shfl_xor_sync(0xffffffffu, l, 2);
        if (p == 0 && (kRows == 8 || r < 4)) {
            wm[warp * 8 + r] = m_ref;
            wl[warp * 8 + r] = l;
        }
        const bool whole = xa == 0 && xb == cost.blocks;
        const int slot = xa == 0;
        float* part = partials + (int64_t)(2 * blockIdx.x + slot) * partial_floats(kRows);
#pragma unroll
        for (int round = 0; round < kNT * 4 / kRedRegs; ++round) {
#pragma unroll
            for (int i = 0; i < kRedRegs; ++i) red[(warp * kRedRegs + i) * 32 + lane] = acc[(round * kRedRegs + i) >> 2][i & 3];
            __syncthreads();
            const int reg = round * kRedRegs + warp;                        // thread (warp, lane) sums register `reg` of lane `lane`
            int row, channel;
            place_of<kC, kRows>(reg, lane, row, channel);
            float M = -INFINITY, L = 0.f, sum = 0.f;
            for (int w = 0; w < kWarps; ++w) M = fmaxf(M, wm[w * 8 + row]);
            for (int w = 0; w < kWarps; ++w) {
                const float mw = wm[w * 8 + row], f = mw == -INFINITY ? 0.f : ex2f(mw - M);
                L = fmaf(f, wl[w * 8 + row], L);
                sum = fmaf(f, red[(w * kRedRegs + warp) * 32 + lane], sum);
            }
            if (whole) {
                if (row < rows) {
                    const int at = row0 + row;
                    a.out[(((int64_t)sv.row0 + at / R) * sh.n_q_heads + head * R + at % R) * 128 + channel] = __float2half_rn(L > 0.f ? sum / L : 0.f);
                }
            } else {
                part[2 * kRows + reg * 32 + lane] = sum;
                if (round == 0 && threadIdx.x < 32 && p == 0 && (kRows == 8 || r < 4)) { part[row] = M; part[kRows + row] = L; }
            }
            __syncthreads();
        }
        if (!whole && threadIdx.x == 0) {
            Cut c;
            c.head = head; c.seq = seq; c.tile = tile; c.state = xb == cost.blocks ? 2 : 1;
            cuts[2 * blockIdx.x + slot] = c;
        }
        x += xb - xa;
        rest += xb - xa;
    }
}

// CTA k merges the item that begins in CTA k's stretch and goes on in the next ones'.
template <int kC, int kRows>
__global__ void __launch_bounds__(kThreads) gather_merge_kernel(BoundedArgs a, const float* __restrict__ partials, const Cut* __restrict__ cuts, int n_ctas)
{
    asm volatile("griddepcontrol.wait;" ::: "memory");
    const int k = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const Cut first = cuts[2 * k + 1];
    if (first.state == 0) return;
    int last = k + 1;
    while (last < n_ctas - 1 && cuts[2 * last].state == 1) ++last;
    const SeqView sv = seq_view(a, first.seq);
    const int R = a.sh.R, row0 = first.tile * kRows;
    for (int reg = warp; reg < (kRows == 4 ? 16 : 32); reg += kWarps) {
        int row, channel;
        place_of<kC, kRows>(reg, lane, row, channel);
        float M = -INFINITY, L = 0.f, sum = 0.f;
        for (int j = k; j <= last; ++j) {
            const float* part = partials + (int64_t)(2 * j + (j == k)) * partial_floats(kRows);
            const float mj = part[row], lj = part[kRows + row], xj = part[2 * kRows + reg * 32 + lane];
            const float m_new = fmaxf(M, mj);
            if (m_new == -INFINITY) continue;
            const float fo = ex2f(M - m_new), fj = ex2f(mj - m_new);
            L = fmaf(L, fo, lj * fj);
            sum = fmaf(sum, fo, xj * fj);
            M = m_new;
        }
        const int at = row0 + row;
        if (at < sv.m * R)
            a.out[(((int64_t)sv.row0 + at / R) * a.sh.n_q_heads + first.head * R + at % R) * 128 + channel] = __float2half_rn(L > 0.f ? sum / L : 0.f);
    }
}

template <int kC, int kRows>
cudaError_t launch(const BoundedArgs& a, void* workspace, int slot, cudaStream_t st)
{
    const int grid = device_sm_count();
    Cut* cuts = static_cast<Cut*>(workspace);
    float* partials = reinterpret_cast<float*>(static_cast<char*>(workspace) + round_up(2 * grid * sizeof(Cut), 256));
    cudaError_t e = ensure_dynamic_smem(reinterpret_cast<const void*>(gather_attn_kernel<kC, kRows>), kSmemBytes, slot);
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr;
    cudaLaunchConfig_t cfg = overlapped_config((unsigned)grid, kThreads, kSmemBytes, st, &attr);
    e = cudaLaunchKernelEx(&cfg, gather_attn_kernel<kC, kRows>, a, partials, cuts);
    if (e != cudaSuccess) return e;
    cfg.dynamicSmemBytes = 0;
    cfg.gridDim = dim3((unsigned)(grid - 1 > 0 ? grid - 1 : 1));
    return cudaLaunchKernelEx(&cfg, gather_merge_kernel<kC, kRows>, a, (const float*)partials, (const Cut*)cuts, grid);
}

}  // namespace

bool gather_attn_supported(const Shape& sh) { return sh.head_dim == 128 && sh.b <= 8 && (sh.c == 2 || sh.c == 4 || sh.c == 8); }

size_t gather_attn_workspace_bytes()
{
    const size_t grid = (size_t)device_sm_count();
    return round_up(2 * grid * sizeof(Cut), 256) + round_up(2 * grid * partial_floats(8) * sizeof(float), 256);
}

// Tiles of four rows where a query token has that few heads, otherwise of eight: with four rows no two lanes meet in a bank.
cudaError_t launch_gather_attn(const BoundedArgs& a, void* workspace, cudaStream_t st)
{
    const bool four = a.sh.R <= 4;
    if (a.sh.c == 8) return four ? launch<8, 4>(a, workspace, 100, st) : launch<8, 8>(a, workspace, 101, st);
    if (a.sh.c == 4) return four ? launch<4, 4>(a, workspace, 102, st) : launch<4, 8>(a, workspace, 103, st);
    return four ? launch<2, 4>(a, workspace, 104, st) : launch<2, 8>(a, workspace, 105, st);
}

}  // namespace cq
