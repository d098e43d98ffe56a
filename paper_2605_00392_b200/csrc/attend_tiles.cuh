// Attention of many query rows per kv head (prefill) over the 8-bit paged cache, on the tcgen05 tensor cores.
//
// A CTA takes two tiles of rows of a request and kv head, each as many tokens as fit 128 rows with all their heads of that kv
// head (a row per token and head, a token's heads beside each other), against blocks of 128 cached tokens:
//   S = Q K^T   bf16 operands in shared memory (queries as they are, codes exact), fp32 sums in TMEM
//   P           fp16 weights, written over S in TMEM by the thread that owns the row
//   O += P V    P from TMEM, V from shared memory, fp32 sums in TMEM
// One CTA per SM takes items (two tiles) blockIdx.x, + gridDim.x, ...; what its warps do:
//   0-3, 4-7  a row per thread of the first and second tile: softmax, output
//   8-11      codes to bf16 (keys) and fp16 (values) in the swizzled operand layout (tiles of (token, 64 elements), K-major for the
//             keys, MN-major for the values)
//   12, 13    issue the MMAs of the first and second tile, in turns (one warp for both was the pace of the kernel)
//   14        bulk copies of codes        15        finds the items and fetches their queries, by TMA
// S of a tile's next block is issued behind the PV of this one, whose P it overwrites.  The tiles take turns: one's PV and S, then the
// other's, so that one's softmax runs beside the other's MMAs (left to themselves they fell into step, both softmaxes, then
// both MMAs: 4850 cycles a block).  One item's output leaves while the next one's scores are computed.
// Everything large comes by bulk copies: with 227 KB of shared memory there are some 20 KB of L1 left, and ordinary loads of
// 64 KB of queries, which need a line of it each while they are on their way, took 10,000 cycles.
// A row's sums are rescaled only where 16 of its weights add up to more than 2^12 by the maximum so far: no weight has then left fp16's
// range, and the sums, which are needed anyway, show it with less work than a maximum (4 % of the time of 37 requests of 512 rows that
// see 8512 tokens).  Blocks seen in part, and an item's blocks from the first whose scales want a reference of their own for l, are gone
// through with more care, in two passes.  A tile's rows behind the request's last (the next request's queries, or whatever shared
// memory held where a token's heads do not divide 128) are computed like the others, but have no voice in how a warp goes on: a
// row's bits do not hang on them.
// Every wait is bounded, and the lanes of a warp take its result together.  Where one gives up its warp leaves; those that wait for it give
// up too, and the softmax's warps write NaN to the rows of the item in work and of all that the CTA would have taken behind it.
// Bound by the tensor cores and, about as much, by the exponentials: 128 x 128 scores take 1024 cycles of either (16 exponentials a
// cycle and SM; two products of 128^3 at 4096 multiply-adds).  It takes 2250: 1.05 PFLOP/s at 512 rows over 8512 tokens, 218 us for 8 causal
// requests of 2783 tokens and 97 us for 64 of 300 to 375, 10 heads.  Keys that need no conversion would make that 15 % less, a softmax
// without arithmetic as much: both want the issue slots and the shared memory that the products read at its full rate.
#pragma once
#include "attend.cuh"

namespace rtp {

constexpr int kTlRows = 128;                         // rows of a tile
constexpr int kTlTiles = 2;
constexpr int kTlBlock = 128;                        // tokens of a block
constexpr int kTlSoft = kTlTiles * kTlRows;
constexpr int kTlThreads = kTlSoft + 128 + 128;     // (the last warp only makes it 128 registers a thread)
constexpr int kTlSoftRegs = 200, kTlCodeRegs = 40, kTlOtherRegs = 72;    // registers of a thread: 2, 1, 1 of four warpgroups
static_assert(2 * kTlSoftRegs + kTlCodeRegs + kTlOtherRegs <= 4 * 128, "what the block was launched with");
constexpr int kTlGroups = kTlBlock / 16;             // a page holds at least 16 tokens: scales are per 16

constexpr float kTlSlack = 4096.f;                   // what 16 weights may add up to (fp16 ends at 2^16)
constexpr float kTlLarge = 1048576.f;                // scores under this are rounded by less than 2^-4

template <int D> struct TlShape {
    static constexpr int kSlabs = D / 64;
    static constexpr int kSlab = 128 * 128;          // 128 rows (tokens) of 64 fp16
    static constexpr int kOperand = kSlabs * kSlab;  // queries of a tile; keys or values of a block
    static constexpr int kSlot = kTlBlock * D;       // codes of a block
    static constexpr int kSlots = D == 128 ? 2 : 4;
    static constexpr int kSmem = (kTlTiles + 4) * kOperand + kSlots * kSlot + 1024 /*alignment*/;
};

// A CTA's piece of work.
struct TlItem {
    int i, head, j0, row0, n, len;                   // i < 0: no more; j0: first of its tokens, in the request
    int after;                                       // where the CTA's numbers go on
    int blocks[kTlTiles];                            // blocks of tokens that each tile sees any of
};
constexpr int kTlItems = 4;                          // pieces that the scheduler may be ahead by, about
constexpr int kTlReaders = 15;                       // warps that read them
constexpr int kTlGroupRing = 8;

struct TlShared {
    // ks, log2 vs, 1 / vs of each 16 tokens of the line's n-th block at n mod kTlGroupRing; w: infinity if any of the block's scales wants
    // a reference of its own for l, else 0
    float4 group[kTlGroupRing][kTlGroups];
    TlItem item[kTlItems];
    uint64_t item_full[kTlItems], item_empty[kTlItems];
    uint64_t code_full[4], code_empty[4];            // keys of block 0, values of block 0, keys of block 1, ...
    uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
    uint64_t q_full[kTlTiles], q_empty[kTlTiles], s_full[kTlTiles], p_full[kTlTiles], o_full[kTlTiles], o_empty[kTlTiles];
    uint64_t turn[kTlTiles], done;
    uint32_t tmem;
    volatile int gave_up, after[kTlSoft / 32];       // after: of the item that a warp of the softmax has in work
};

// The k-th item, for a whole warp.  false: a wait gave up, and t is nothing.
__device__ inline bool tl_take(const AttendArgs &a, TlShared *sh, uint32_t k, TlItem &t)
{
    if (!attend_wait(a, &sh->item_full[k % kTlItems], k / kTlItems & 1)) return false;
    t = sh->item[k % kTlItems];
    __syncwarp();
    if ((threadIdx.x & 31) == 0) ptx::mbar_arrive(&sh->item_empty[k % kTlItems]);
    return true;
}

// The CTA's next item that has rows, from its `at`-th number on, for a whole warp; i < 0: there is none.
__device__ inline void tl_next(const AttendArgs &a, int row_blocks, int tile_tokens, int at, TlItem &t)
{
    const int lane = threadIdx.x & 31, per = a.batch * a.c.kv_heads, all = row_blocks * per;
    auto number = [&](int round) { return round * (int)gridDim.x + (int)(round & 1 ? gridDim.x - 1 - blockIdx.x : blockIdx.x); };
    const int rounds = (all + (int)gridDim.x - 1) / (int)gridDim.x;
    // 32 of the numbers at a time, one per lane (bounds that are far above the requests' lengths leave most of them empty)
#pragma unroll 1
    for (; at < rounds; at += 32) {
        const int mine = number(at + lane);
        bool has = false;
        if (at + lane < rounds && mine < all) {
            // the last rows of every request first: with a causal mask they have the most to do
            const int rest = mine % per;
            t.i = rest / a.c.kv_heads;
            t.head = rest - t.i * a.c.kv_heads;
            t.j0 = (row_blocks - 1 - mine / per) * kTlTiles * tile_tokens;
            has = attend_request(a, t.i, t.row0, t.n, t.len) && t.j0 < t.n;
        }
        const uint32_t found = __ballot_sync(0xffffffffu, has);
        if (found) {
            const int from = __ffs(found) - 1;
            t.after = at + from + 1;
            t.i = __shfl_sync(0xffffffffu, t.i, from);
            t.head = __shfl_sync(0xffffffffu, t.head, from);
            t.j0 = __shfl_sync(0xffffffffu, t.j0, from);
            t.row0 = __shfl_sync(0xffffffffu, t.row0, from);
            t.n = __shfl_sync(0xffffffffu, t.n, from);
            t.len = __shfl_sync(0xffffffffu, t.len, from);
#pragma unroll
            for (int x = 0; x < kTlTiles; ++x) {
                const int first = t.j0 + x * tile_tokens, last = min(first + tile_tokens, t.n) - 1;
                const int end = first >= t.n || t.len < 0 ? 0 : a.causal ? t.len - t.n + 1 + last : t.len;
                t.blocks[x] = (max(end, 0) + kTlBlock - 1) / kTlBlock;
            }
            return;
        }
    }
    t.i = -1;
    t.after = at;
}

__device__ inline void umma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
        "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ inline void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
        "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
// One lane of a full warp, the same each time.
__device__ inline bool elect_one()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Instruction descriptor of kind::f16 with fp16 operands (see ptx::idesc_bf16).
__device__ inline uint32_t idesc_f16(int M, int N, bool b_mn_major)
{
    return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

template <int N> __device__ inline void regs_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ inline void regs_fewer() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }
// 32 bytes, a whole sector of one lane's row (32-byte aligned).
__device__ inline void st_global_v8(void *p, const uint32_t *v)
{
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(p), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]),
                 "r"(v[5]), "r"(v[6]), "r"(v[7])
                 : "memory");
}
__device__ inline uint4 ld_shared_u4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
// Four codes of a word, in order, as two pairs of bf16: 128 + the low seven bits is the bf16 number with those as its last bits, and 128
// + 128 for the sign bit the one with that bit; their difference is the code.  (low, sign: 0x7f.., 0x80..; the other way round its negative.)
__device__ inline void codes_to_bf16(uint32_t x, uint32_t low, uint32_t sign, uint32_t &lo, uint32_t &hi)
{
    constexpr uint32_t k128 = 0x43434343u;
    const uint32_t a = x & low, b = x & sign;
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(lo) : "r"(__byte_perm(a, k128, 0x4140)), "r"(__byte_perm(b, k128, 0x4140)));
    asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(hi) : "r"(__byte_perm(a, k128, 0x4342)), "r"(__byte_perm(b, k128, 0x4342)));
}
// A thread's pieces of a block's codes, to the operand: 16 codes of token 8 q + r, piece pc of each slab, odd tokens the slabs in the other
// order: eight neighbouring lanes read and write eight different places of 128 bytes.
template <int D, bool kValues>
__device__ inline void tile_codes(uint32_t from, uint32_t to, int r, int pc, uint32_t low)
{
    constexpr int kSlabs = D / 64;
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int b = 0; b < kSlabs; ++b) {
            const int slab = b ^ (kSlabs > 1 ? r & 1 : 0);
            const uint4 c = ld_shared_u4(from + 8 * q * D + (slab * 4 + pc) * 16);
            uint4 lo, hi;
            if (kValues) {
                codes_to_half(c.x ^ 0x80808080u, lo.x, lo.y);
                codes_to_half(c.y ^ 0x80808080u, lo.z, lo.w);
                codes_to_half(c.z ^ 0x80808080u, hi.x, hi.y);
                codes_to_half(c.w ^ 0x80808080u, hi.z, hi.w);
            } else {
                codes_to_bf16(c.x, low, ~low, lo.x, lo.y);
                codes_to_bf16(c.y, low, ~low, lo.z, lo.w);
                codes_to_bf16(c.z, low, ~low, hi.x, hi.y);
                codes_to_bf16(c.w, low, ~low, hi.z, hi.w);
            }
            const uint32_t line = to + slab * 16384 + 8 * q * 128;
            ptx::st_shared_v4(line + (((2 * pc) ^ r) << 4), lo);          // (32 w + 8 q + r) & 7 = r
            ptx::st_shared_v4(line + (((2 * pc + 1) ^ r) << 4), hi);
        }
}
// Two fp32 at a time.
__device__ inline uint64_t pack2(float a, float b)
{
    uint64_t r;
    asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
    return r;
}
__device__ inline void unpack2(uint64_t x, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ inline uint64_t fma2(uint64_t a, uint64_t b, uint64_t c)
{
    uint64_t r;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
    return r;
}
__device__ inline uint64_t add2(uint64_t a, uint64_t b)
{
    uint64_t r;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}

__device__ inline float max3(float a, float b, float c) { return fmaxf(fmaxf(a, b), c); }    // (one instruction)
__device__ inline float max16(const float (&s)[16])
{
    const float a = max3(s[0], s[1], s[2]), b = max3(s[3], s[4], s[5]), c = max3(s[6], s[7], s[8]), d = max3(s[9], s[10], s[11]);
    return max3(max3(a, b, c), max3(d, s[12], s[13]), fmaxf(s[14], s[15]));
}

// The largest s' of 32 of a row's scores (two groups), and their weights p, the sum of these (without the values' scale) into l, the largest
// sum of 16 into `most`.  The scores come from TMEM 32 at a time: a thread that keeps its 128 spills whatever else it has, and what is
// spilled comes back from L2 (shared memory has left L1 next to nothing).
__device__ inline float tile_top(const uint32_t (&v)[32], const float4 *group, float factor, float now)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        float s[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) s[e] = __uint_as_float(v[16 * h + e]);
        const float4 g = group[h];
        now = fmaxf(now, fmaf(max16(s), factor * g.x, g.y));
    }
    return now;
}
__device__ inline void tile_weights(const uint32_t (&v)[32], const float4 *group, float factor, float top, uint32_t *p, float &most, float &l)
{
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        const float4 g = group[h];
        const float k = factor * g.x, b = g.y - top;
        const uint64_t k2 = pack2(k, k), b2 = pack2(b, b);
        uint64_t sum2 = 0;
        float w[16];
#pragma unroll
        for (int e = 0; e < 16; e += 2)
            unpack2(fma2(pack2(__uint_as_float(v[16 * h + e]), __uint_as_float(v[16 * h + e + 1])), k2, b2), w[e], w[e + 1]);
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            w[e] = ex2(w[e]);
            w[e + 1] = ex2(w[e + 1]);
            sum2 = add2(sum2, pack2(w[e], w[e + 1]));
            p[8 * h + e / 2] = pack_half(w[e], w[e + 1]);
        }
        float s0, s1;
        unpack2(sum2, s0, s1);
        s0 += s1;
        most = fmaxf(most, s0);
        l = fmaf(s0, g.z, l);
    }
}
// The same where tokens from `left` on are not seen, or scores are so large that their own rounding matters: it is what the maximum
// went through, so they go through it too before the maximum is taken off; or where l has a reference of its own (now_s: the largest s;
// gap = top - ref, 0 where it has not).  Loops of few instructions, from TMEM again.
__device__ inline float careful_top(const float4 *group, float factor, int left, int seen, uint32_t t_s, float &now_s)
{
    float now = kAtNothing;
    now_s = kAtNothing;
#pragma unroll 1
    for (int c = 0; 32 * c < seen; ++c, left -= 32) {
        uint32_t v[32];
        ptx::tmem_ld32(t_s + c * 32, v);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float s[16];
#pragma unroll
            for (int e = 0; e < 16; ++e) s[e] = 16 * h + e < left ? __uint_as_float(v[16 * h + e]) : -INFINITY;
            const float4 g = group[2 * c + h];
            const float most = max16(s), k = factor * g.x;
            now = fmaxf(now, fmaf(most, k, g.y));
            now_s = fmaxf(now_s, most * k);
        }
    }
    return now;
}
__device__ inline void careful_weights(const float4 *group, float factor, float top, float gap, int left, int seen, uint32_t t_s, float &l)
{
#pragma unroll 1
    for (int c = 0; c < kTlBlock / 32; ++c, left -= 32) {
        uint32_t v[32], p[16];
        if (32 * c < seen) {
            ptx::tmem_ld32(t_s + c * 32, v);
            ptx::tmem_ld_wait();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 g = group[2 * c + h];
                const float k = factor * g.x, lv = weight_log(g.y, gap);
                float w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = ex2(fmaf(__uint_as_float(v[16 * h + e]), k, lv) - top);
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = 16 * h + e < left ? w[e] : 0.f;
                const float sum = ((w[0] + w[1]) + (w[2] + w[3])) + ((w[4] + w[5]) + (w[6] + w[7])) + (((w[8] + w[9]) + (w[10] + w[11])) + ((w[12] + w[13]) + (w[14] + w[15])));
#pragma unroll
                for (int e = 0; e < 8; ++e) p[8 * h + e] = pack_half(w[2 * e], w[2 * e + 1]);
                // weights of 0 add nothing, whatever the block's scale is (of a page that the row does not see)
                if (sum != 0.f) l = fmaf(sum, ex2(gap - lv), l);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 16; ++e) p[e] = 0u;
        }
        tmem_st16(t_s + c * 16, p);
    }
}

template <int D>
__global__ void __launch_bounds__(kTlThreads, 1)
attend_tiles_kernel(const __grid_constant__ AttendArgs a, const __grid_constant__ CUtensorMap map_q, int row_blocks, int tile_tokens)
{
    using S = TlShape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ TlShared shared;
    TlShared *const sh = &shared;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < kTlItems; ++s) {
            ptx::mbar_init(&sh->item_full[s], 1);
            ptx::mbar_init(&sh->item_empty[s], kTlReaders);
        }
        for (int s = 0; s < S::kSlots; ++s) {
            ptx::mbar_init(&sh->code_full[s], 1);
            ptx::mbar_init(&sh->code_empty[s], 128);
        }
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(&sh->k_full[s], 128);
            ptx::mbar_init(&sh->k_empty[s], kTlTiles);
            ptx::mbar_init(&sh->v_full[s], 128);
            ptx::mbar_init(&sh->v_empty[s], kTlTiles);
        }
        for (int x = 0; x < kTlTiles; ++x) {
            ptx::mbar_init(&sh->q_full[x], 1);
            ptx::mbar_init(&sh->q_empty[x], 1);
            ptx::mbar_init(&sh->s_full[x], 1);
            ptx::mbar_init(&sh->p_full[x], kTlRows);
            ptx::mbar_init(&sh->o_full[x], 1);
            ptx::mbar_init(&sh->o_empty[x], kTlRows);
            ptx::mbar_init(&sh->turn[x], 1);
        }
        ptx::mbar_init(&sh->done, kTlTiles);
        sh->gave_up = 0;
        ptx::fence_mbar_init();
    }
    ptx::grid_dep_wait();                            // (before TMEM is taken: a kernel ahead may be waiting for it)
    if (warp == 12) {
        ptx::tmem_alloc(&sh->tmem, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, sh->tmem, 0), s_u32 = ptx::smem_u32(smem);
    const uint32_t k_u32 = s_u32 + kTlTiles * S::kOperand, v_u32 = k_u32 + 2 * S::kOperand, code_u32 = v_u32 + 2 * S::kOperand;
    // TMEM: scores (and weights over them) of the tiles at columns 0 and 128, outputs at 256 and 256 + D
    // (not earlier: a kernel behind this one that takes TMEM before it waits could otherwise have it first)
    ptx::grid_dep_launch();

    // (registers: one instruction for each warpgroup, ahead of all that the warpgroup does)
    if (warp >= 12) {
        regs_fewer<kTlOtherRegs>();
        if (warp == 15) {
            // ---------------- the work: items blockIdx.x, + gridDim.x, ... that have rows; their queries, as they are, in the operand's
            // layout already
            int at = 0;
            bool ok = true;
            uint32_t uses[kTlTiles] = {0, 0};
    #pragma unroll 1
            for (uint32_t k = 0; ok; ++k) {
                TlItem t;
                tl_next(a, row_blocks, tile_tokens, at, t);
                at = t.after;
                if (k >= kTlItems) ok = attend_wait(a, &sh->item_empty[k % kTlItems], (k / kTlItems - 1) & 1);
                if (ok && lane == 0) {
                    sh->item[k % kTlItems] = t;
                    ptx::mbar_arrive(&sh->item_full[k % kTlItems]);
                }
                if (t.i < 0) break;
    #pragma unroll
                for (int x = 0; x < kTlTiles; ++x) {
                    if (!ok || t.blocks[x] == 0) continue;
                    if (uses[x] > 0) ok = attend_wait(a, &sh->q_empty[x], (uses[x] - 1) & 1);
                    if (ok && lane == 0) {
                        ptx::mbar_arrive_expect_tx(&sh->q_full[x], (uint32_t)(S::kSlabs * tile_tokens * a.group * 128));
                        for (int b = 0; b < S::kSlabs; ++b)
                            ptx::tma_load_3d(s_u32 + x * S::kOperand + b * S::kSlab, &map_q, &sh->q_full[x], b * 64, t.head * a.group,
                                             t.row0 + t.j0 + x * tile_tokens);
                    }
                    __syncwarp();
                    if (ok) ++uses[x];
                }
            }
            if (!ok) sh->gave_up = 1;
            // no copy is left on its way into memory that this CTA gives back
    #pragma unroll
            for (int x = 0; x < kTlTiles; ++x)
                if (uses[x] > 0) ptx::mbar_wait(&sh->q_full[x], (uses[x] - 1) & 1);
        } else if (warp == 14) {
            // ---------------- codes of the items' blocks, and their scales ----------------------------------------
            const int per_page = min(a.c.page_size, kTlBlock), copies = kTlBlock / per_page;   // a page of a head is one piece of memory
            TlItem t;
            bool ok = true;
            uint32_t n = 0, copy = 0;                    // blocks, slots so far
    #pragma unroll 1
            for (uint32_t item = 0; ok && (ok = tl_take(a, sh, item, t)) && t.i >= 0; ++item) {
                const int most = max(t.blocks[0], t.blocks[1]);
    #pragma unroll 1
                for (int j = 0; ok && j < most; ++j, ++n) {
                    // lane: a copy's page, and (lane < 8) the page of its 16 tokens.  Tokens behind the end are not fetched: what lies in
                    // the slot are codes too, and nobody sees them
                    const int t0 = j * kTlBlock, t_copy = t0 + lane * per_page, t_group = t0 + lane * 16;
                    const int page = lane < copies && t_copy < t.len ? attend_page(a, t.i, t_copy) : -1;
                    const int page_g = lane < kTlGroups && t_group < t.len ? attend_page(a, t.i, t_group) : -1;
                    if (lane < kTlGroups) {
                        const int64_t block = (int64_t)max(page_g, 0) * a.c.kv_heads + t.head;
                        const float nan = __uint_as_float(0x7fc00000u);
                        float lv, inv;
                        const bool wide = value_scale(page_g < 0 ? nan : __ldg(a.c.v_scale + block), lv, inv);
                        const bool any = __any_sync((1u << kTlGroups) - 1u, wide);
                        sh->group[n % kTlGroupRing][lane] = make_float4(page_g < 0 ? nan : __ldg(a.c.k_scale + block), lv, inv, any ? INFINITY : 0.f);
                    }
                    const uint32_t bytes = (uint32_t)(__popc(__ballot_sync(0xffffffffu, page >= 0)) * per_page * D);
                    const int64_t from = ((int64_t)max(page, 0) * a.c.kv_heads + t.head) * a.c.page_size * D;
    #pragma unroll 1
                    for (int v = 0; ok && v < 2; ++v, ++copy) {
                        const uint32_t slot = copy % S::kSlots, turn = copy / S::kSlots;
                        if (turn > 0) ok = attend_wait(a, &sh->code_empty[slot], (turn - 1) & 1);
                        if (!ok) break;
                        if (lane == 0) ptx::mbar_arrive_expect_tx(&sh->code_full[slot], bytes);
                        __syncwarp();
                        if (page >= 0)
                            ptx::bulk_load(code_u32 + slot * S::kSlot + lane * per_page * D, (v ? a.c.v : a.c.k) + from, (uint32_t)(per_page * D), &sh->code_full[slot]);
                    }
                }
            }
            if (!ok) sh->gave_up = 1;
            // no copy is left on its way into memory that this CTA gives back
            for (uint32_t c = copy > S::kSlots ? copy - S::kSlots : 0; c < copy; ++c)
                ptx::mbar_wait(&sh->code_full[c % S::kSlots], c / S::kSlots & 1);
        } else {
            // ---------------- the MMAs of tile x ----------------------------------------------------------------
            // the whole warp walks the blocks, one elected lane issues
            const int x = warp - 12;
            const bool issuer = elect_one();
            const uint32_t id_s = ptx::idesc_bf16(kTlRows, kTlBlock, false, false), id_o = idesc_f16(kTlRows, D, true);
            const uint32_t t_s = tmem + x * 128, t_o = tmem + 256 + x * D;
            // descriptors differ from these by multiples of 16 bytes in the address (their low 14 bits, which never carry)
            const uint64_t d_q = ptx::smem_desc_sw128(s_u32 + x * S::kOperand, 16, 1024), d_k = ptx::smem_desc_sw128(k_u32, 16, 1024);
            const uint64_t d_v = ptx::smem_desc_sw128(v_u32, S::kSlab, 1024);
            auto wait = [&](uint64_t *bar, uint32_t parity) { return ptx::mbar_wait(bar, parity, a.polls); };
            bool ok = true;
            uint32_t n = 0, step = 0, items = 0, turns = 0;      // blocks and steps; this tile's items and blocks so far
            TlItem t;
    #pragma unroll 1
            for (uint32_t item = 0; ok && (ok = tl_take(a, sh, item, t)) && t.i >= 0; ++item) {
                const int most = max(t.blocks[0], t.blocks[1]), mine = x ? t.blocks[1] : t.blocks[0];
                // step j: products of block j - 1, scores of block j; n is block j's number.  A block that this tile sees nothing of is passed on
                // once it is there (not before: its buffer's turns would be mixed up)
    #pragma unroll 1
                for (int j = 0; j <= most && most > 0; ++j, ++n, ++step) {
                    const uint32_t s = n & 1, s_before = s ^ 1;
                    const bool products = j > 0 && j <= mine, scores = j < mine;
                    // what is there early is waited for first, the weights last: their way to the next scores is the kernel's longest
                    if (j > 0) ok = wait(&sh->v_full[s_before], ((n - 1) >> 1) & 1);
                    if (j < most) ok = ok && wait(&sh->k_full[s], (n >> 1) & 1);
                    if (j == 0 && mine > 0) ok = ok && wait(&sh->q_full[x], items & 1);
                    if (j == 1 && mine > 0 && items > 0) ok = ok && wait(&sh->o_empty[x], (items - 1) & 1);   // (the last item's output is out of TMEM)
                    // the other tile's turn before this
                    if (x > 0 || step > 0) ok = ok && wait(&sh->turn[x ^ 1], (x ? step : step - 1) & 1);
                    if (products) {
                        ok = ok && wait(&sh->p_full[x], turns & 1);
                        ++turns;
                    }
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    ptx::tc_fence_after();
                    if (products && issuer) {
                        const uint64_t v0 = d_v + s_before * (S::kOperand >> 4);
    #pragma unroll
                        for (int k = 0; k < kTlBlock / 16; ++k) umma_f16_ts(t_o, t_s + k * 8, v0 + k * (2048 >> 4), id_o, j - 1 + k > 0);
                        ptx::umma_commit(&sh->v_empty[s_before]);
                        if (j == mine) ptx::umma_commit(&sh->o_full[x]);
                    } else if (j > 0 && issuer) {
                        ptx::mbar_arrive(&sh->v_empty[s_before]);
                    }
                    if (j < most) {
                        if (scores && issuer) {
                            const uint64_t k0 = d_k + s * (S::kOperand >> 4);
    #pragma unroll
                            for (int k = 0; k < D / 16; ++k) {
                                const int at = ((k >> 2) * S::kSlab + (k & 3) * 32) >> 4;
                                ptx::umma_bf16(t_s, d_q + at, k0 + at, id_s, k > 0);
                            }
                            ptx::umma_commit(&sh->s_full[x]);
                            ptx::umma_commit(&sh->k_empty[s]);
                            if (j + 1 == mine) ptx::umma_commit(&sh->q_empty[x]);
                        } else if (issuer) {
                            ptx::mbar_arrive(&sh->k_empty[s]);
                        }
                    }
                    if (issuer) ptx::mbar_arrive(&sh->turn[x]);
                    __syncwarp();
                }
                if (most > 0) --n;                       // (the next item's first block has the number of the step without scores)
                items += mine > 0;
            }
            if (!ok) sh->gave_up = 1;
            // all MMAs done (also after a wait that gave up: the memory they use is about to be freed)
            if (issuer) ptx::umma_commit(&sh->done);
            __syncwarp();
            if (!ptx::mbar_wait(&sh->done, 0)) sh->gave_up = 1;
        }
    } else if (warp >= 8) {
        regs_fewer<kTlCodeRegs>();
        // ---------------- codes to bf16 and fp16 ---------------------------------------------------------------------
        const int w = warp - 8, r = lane >> 2, pc = lane & 3;
        const uint32_t low = a.scale_log2 < 0.f ? 0x80808080u : 0x7f7f7f7fu;       // (a negative scale: negative keys)
        TlItem t;
        bool ok = true;
        uint32_t n = 0, copy = 0;
#pragma unroll 1
        for (uint32_t item = 0; ok && (ok = tl_take(a, sh, item, t)) && t.i >= 0; ++item) {
            const int most = max(t.blocks[0], t.blocks[1]);
#pragma unroll 1
            for (int j = 0; ok && j < 2 * most; ++j, ++copy) {
                const bool values = j & 1;           // keys of a block, then its values
                const uint32_t slot = copy % S::kSlots, s = n & 1;
                ok = ptx::mbar_wait(&sh->code_full[slot], copy / S::kSlots & 1, a.polls);
                if (ok && n >= 2) ok = ptx::mbar_wait(values ? &sh->v_empty[s] : &sh->k_empty[s], ((n >> 1) - 1) & 1, a.polls);
                ok = __all_sync(0xffffffffu, ok);
                if (!ok) break;
                const uint32_t from = code_u32 + slot * S::kSlot + (32 * w + r) * D, to = (values ? v_u32 : k_u32) + s * S::kOperand + (32 * w + r) * 128;
                if (values) tile_codes<D, true>(from, to, r, pc, low);
                else tile_codes<D, false>(from, to, r, pc, low);
                ptx::mbar_arrive(&sh->code_empty[slot]);
                ptx::fence_proxy_async_smem();
                ptx::mbar_arrive(values ? &sh->v_full[s] : &sh->k_full[s]);
                n += values;
            }
        }
        if (!ok) sh->gave_up = 1;
    } else {
        regs_more<kTlSoftRegs>();
        // ---------------- a row per thread -------------------------------------------------------------------
        const int x = warp >> 2, r = tid & 127, jj = r / a.group, r_head = r - jj * a.group;   // a row's token of the tile, and its head
        const uint32_t lanes = (uint32_t)(warp & 3) << 21;
        const uint32_t t_s = tmem + lanes + x * 128, t_o = tmem + lanes + 256 + x * D;
        bool ok = true;
        uint32_t n = 0, turns = 0, items = 0;        // blocks; this tile's blocks and items so far
        // the item in work: what of it outlives the look at the next one
        int mine = -1, end = 0, blocks = 0, most = 0;
        const float factor = fabsf(a.scale_log2);    // (a negative scale is in the keys: the largest sum is the largest score)
        bool has = false, bad = false;
        // the row's place among (row, query head) of the item, -1: it is none of the request's
        auto place = [&](const TlItem &t) {
            const int j_row = t.j0 + x * tile_tokens + jj;
            return jj < tile_tokens && j_row < t.n ? (t.row0 + j_row) * a.q_heads + t.head * a.group + r_head : -1;
        };
#pragma unroll 1
        for (uint32_t item = 0;; ++item) {
            float top = kAtNothing, ref = kAtNothing, l = 0.f;   // m', r (what l is relative to: m' until a block is wide)
            bool wide = false;
            const int warp_most = __shfl_sync(0xffffffffu, end, 31), warp_end = __shfl_sync(0xffffffffu, end, 0);   // (the first row sees the fewest tokens)
#pragma unroll 1
            for (int j = 0; ok && j < blocks; ++j, ++turns) {
                if (!(ok = attend_wait(a, &sh->s_full[x], turns & 1))) break;
                ptx::tc_fence_after();
                const float4 *group = sh->group[(n + j) % kTlGroupRing];
                const int left = end - j * kTlBlock; // tokens of the block that the row sees
                const bool masked = (j + 1) * kTlBlock > warp_end;
                const int seen = min(warp_most - j * kTlBlock, kTlBlock);
                bool careful = masked || wide;
                // Weights against the maximum so far, in one pass; only where a row has one that is too large for fp16 by it (or nothing
                // yet: the first block) its maximum is looked for first
                for (bool first = j == 0 || careful;; first = true) {
                    if (first) {
                        if (group[0].w != 0.f) wide = careful = true;    // from here on, for the item
                        float now = kAtNothing, now_s = kAtNothing;      // the row's maximum (of s', with the values' scale), and that of s
                        if (careful) {
                            now = careful_top(group, factor, left, seen, t_s, now_s);
                        } else {
#pragma unroll 1
                            for (int c = 0; c < 4; c += 2) {
                                uint32_t va[32], vb[32];
                                ptx::tmem_ld32(t_s + 32 * c, va);
                                ptx::tmem_ld32(t_s + 32 * c + 32, vb);
                                ptx::tmem_ld_wait();
                                now = tile_top(va, group + 2 * c, factor, now);
                                now = tile_top(vb, group + 2 * c + 2, factor, now);
                            }
                        }
                        const float to = fmaxf(top, now), k = ex2(top - to);
                        top = to;
                        const float r = wide ? fmaxf(ref, now_s) : to;
                        l *= ex2(ref - r);
                        ref = r;
                        if (j > 0 && __any_sync(0xffffffffu, mine >= 0 && k < 1.f)) {
#pragma unroll 1
                            for (int c = 0; c < D / 16; ++c) {
                                uint32_t o[16];
                                ptx::tmem_ld16(t_o + c * 16, o);
                                ptx::tmem_ld_wait();
#pragma unroll
                                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * k);
                                tmem_st16(t_o + c * 16, o);
                            }
                        }
                        careful = careful || __any_sync(0xffffffffu, mine >= 0 && fabsf(top) > kTlLarge);
                    }
                    if (careful) {
                        careful_weights(group, factor, top, top - ref, left, seen, t_s, l);
                        break;
                    }
                    uint32_t va[32], vb[32], p[64];
                    float most = group[0].w, more = 0.f;         // (a wide block: infinity)
                    ptx::tmem_ld32(t_s, va);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld32(t_s + 32, vb);
                    tile_weights(va, group, factor, top, p, most, more);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld32(t_s + 64, va);
                    tile_weights(vb, group + 2, factor, top, p + 16, most, more);
                    ptx::tmem_ld_wait();
                    ptx::tmem_ld32(t_s + 96, vb);
                    tile_weights(va, group + 4, factor, top, p + 32, most, more);
                    ptx::tmem_ld_wait();
                    tile_weights(vb, group + 6, factor, top, p + 48, most, more);
                    if (!first && __any_sync(0xffffffffu, mine >= 0 && most > kTlSlack)) continue;
                    l += more;
#pragma unroll
                    for (int c = 0; c < 4; ++c) tmem_st16(t_s + 16 * c, *reinterpret_cast<uint32_t (*)[16]>(p + 16 * c));
                    break;
                }
                tmem_st_wait();
                ptx::tc_fence_before();
                ptx::mbar_arrive(&sh->p_full[x]);
            }
            n += most;
            TlItem next;
            next.i = -1;
            if (ok) ok = tl_take(a, sh, item, next);
            int mine_next = -1, end_next = 0;
            if (ok && next.i >= 0) {
                mine_next = place(next);
                end_next = a.causal ? next.len - next.n + 1 + min(next.j0 + x * tile_tokens + jj, next.n - 1) : next.len;
            }
            const int blocks_next = next.i < 0 ? 0 : x ? next.blocks[1] : next.blocks[0];
            // ---- out
            if (ok && has) {
                const bool any = blocks > 0;
                if (any) ok = attend_wait(a, &sh->o_full[x], items++ & 1);
                ptx::tc_fence_after();
                const bool nan = bad || sh->gave_up;
                const float half = half_gap(top, ref), k = nan ? __uint_as_float(0x7fc00000u) : l == 0.f ? 0.f : 1.f / l * half;
                __nv_bfloat16 *to = a.out + (int64_t)max(mine, 0) * D;
#pragma unroll 1
                for (int b = 0; b < D / 32; ++b) {
                    uint32_t v[32];
                    ptx::tmem_ld32(t_o + b * 32, v);
                    ptx::tmem_ld_wait();
                    if (b == D / 32 - 1 && any) {
                        ptx::tc_fence_before();
                        ptx::mbar_arrive(&sh->o_empty[x]);
                    }
                    uint32_t o[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(v[2 * e]) * k * half, __uint_as_float(v[2 * e + 1]) * k * half);
                        o[e] = any || nan ? *reinterpret_cast<const uint32_t *>(&h) : 0u;      // a tile that saw no block has no sums
                    }
                    if (mine >= 0) {
                        st_global_v8(to + b * 32, o);
                        st_global_v8(to + b * 32 + 16, o + 8);
                    }
                }
                if (mine >= 0 && a.lse) a.lse[mine] = nan ? k : l == 0.f ? -INFINITY : (ref + log2f(l)) * kAtLn2;
            }
            if (!ok) {
                // a wait gave up: the rows of this item and of all that the CTA would have taken behind it
                sh->gave_up = 1;
                int after = has ? sh->after[warp] : 0;
                for (next.i = 0; next.i >= 0; mine = next.i < 0 ? -1 : place(next)) {
                    if (mine >= 0) {
                        for (int e = 0; e < D; ++e) a.out[(int64_t)mine * D + e] = __float2bfloat16(__uint_as_float(0x7fc00000u));
                        if (a.lse) a.lse[mine] = __uint_as_float(0x7fc00000u);
                    }
                    tl_next(a, row_blocks, tile_tokens, after, next);
                    after = next.after;
                }
                break;
            }
            if (next.i < 0) break;
            has = true;
            bad = next.len < 0;
            mine = mine_next;
            end = end_next;
            blocks = blocks_next;
            most = max(next.blocks[0], next.blocks[1]);
            sh->after[warp] = next.after;            // (kept for a wait that gives up alone)
        }
        ptx::tc_fence_before();
    }
    __syncthreads();
    if (warp == 12) {
        ptx::tc_fence_after();
        ptx::tmem_dealloc(tmem, 512);
    }
}

}  // namespace rtp
