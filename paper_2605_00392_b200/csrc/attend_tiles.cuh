// Attention of many query rows per kv head (prefill) over the 8-bit paged cache, on the tcgen05 tensor cores.
//
// A CTA takes 256 rows (token by token, a token's heads of one kv head beside each other) of a request and kv head as two tiles of
// 128, against blocks of 128 tokens:
//   S = Q K^T   fp16 operands in shared memory, fp32 sums in TMEM
//   P           fp16 weights, written over S in TMEM by the thread that owns the row
//   O += P V    P from TMEM, V from shared memory, fp32 sums in TMEM
// Warps 0-3 and 4-7: a row per thread of the first and second tile (queries in, softmax, output).  Warps 8-11 take the codes of a block
// from global memory to fp16 in the swizzled operand layout; both operands are tiles of (token, 64 elements), K-major for the keys,
// MN-major for the values.  Warp 12 issues the MMAs.  While one tile's softmax runs, the other's MMAs do; S of a tile's next block is
// issued behind the PV of this one, whose P it overwrites.
// A row's sums are rescaled only when its maximum has grown by more than 2^8 (the weights have that room in fp16).
// Bound by the tensor cores and, about as much, by the exponentials: 128 x 128 scores take 1024 cycles of either (16 exponentials a
// cycle and SM; two products of 128^3 at 4096 multiply-adds).
#pragma once
#include "attend.cuh"

namespace rtp {

constexpr int kTlRows = 128;                         // rows of a tile
constexpr int kTlTiles = 2;
constexpr int kTlBlock = 128;                        // tokens of a block
constexpr int kTlSoft = kTlTiles * kTlRows;
constexpr int kTlThreads = kTlSoft + 128 + 128;     // (three of the last four warps only give up their registers)
constexpr int kTlSoftRegs = 176, kTlCodeRegs = 112, kTlMmaRegs = 48;   // registers of a thread by role: 2, 1, 1 of four warpgroups at 128
static_assert(2 * kTlSoftRegs + kTlCodeRegs + kTlMmaRegs <= 4 * 128, "what the block was launched with");
constexpr int kTlGroups = kTlBlock / 16;             // a page holds at least 16 tokens: scales are per 16

constexpr float kTlLarge = 1048576.f;                // scores under this are rounded by less than 2^-4

template <int D> struct TlShape {
    static constexpr int kSlabs = D / 64;
    static constexpr int kSlab = 128 * 128;          // 128 rows (tokens) of 64 fp16
    static constexpr int kOperand = kSlabs * kSlab;
    static constexpr int kSmem = (kTlTiles + 4) * kOperand + 1024 /*alignment*/ + 1024 /*scales, barriers*/;
};

struct TlShared {
    float4 group[4][kTlGroups];                      // ks, log2 vs, 1 / vs of each 16 tokens of block j at j mod 4
    uint64_t q_full, k_full[2], v_full[2], k_empty[2], v_empty[2], s_full[kTlTiles], p_full[kTlTiles], o_full;
    uint32_t tmem;
    volatile int gave_up;
};

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
__device__ inline void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// Instruction descriptor of kind::f16 with fp16 operands (see ptx::idesc_bf16).
__device__ inline uint32_t idesc_f16(int M, int N, bool b_mn_major)
{
    return (1u << 4) | ((b_mn_major ? 1u : 0u) << 16) | ((uint32_t)(N >> 3) << 17) | ((uint32_t)(M >> 4) << 24);
}

template <int N> __device__ inline void regs_more() { asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N)); }
template <int N> __device__ inline void regs_fewer() { asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N)); }

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

// Weights of a row's 128 scores `v` in its place in TMEM, their sum (without the values' scale) into l.  kCare: tokens from `left` on are not
// seen, and scores may be so large that their own rounding matters, which the maximum went through: they go through it too before
// the maximum is taken off.
template <bool kCare>
__device__ inline void tile_weights(const uint32_t (&v)[kTlBlock], const float4 *group, float factor, float top, int left, uint32_t t_s, float &l)
{
#pragma unroll
    for (int c = 0; c < kTlBlock / 32; ++c) {
        uint32_t p[16];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float4 g = group[2 * c + h];
            const float k = factor * g.x, b = kCare ? g.y : g.y - top;
            const uint64_t k2 = pack2(k, k), b2 = pack2(b, b);
            uint64_t sum2 = 0;
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                const int at = 32 * c + 16 * h + e;
                float w0, w1;
                unpack2(fma2(pack2(__uint_as_float(v[at]), __uint_as_float(v[at + 1])), k2, b2), w0, w1);
                if (kCare) {
                    w0 -= top;
                    w1 -= top;
                }
                w0 = ex2(w0);
                w1 = ex2(w1);
                if (kCare) {
                    if (at >= left) w0 = 0.f;
                    if (at + 1 >= left) w1 = 0.f;
                }
                sum2 = add2(sum2, pack2(w0, w1));
                p[8 * h + e / 2] = pack_half(w0, w1);
            }
            float s0, s1;
            unpack2(sum2, s0, s1);
            // weights of 0 add nothing, whatever the block's scale is (of a page that the row does not see)
            if (!kCare || s0 + s1 != 0.f) l = fmaf(s0 + s1, g.z, l);
        }
        tmem_st16(t_s + c * 16, p);
    }
}

template <int D>
__global__ void __launch_bounds__(kTlThreads, 1)
attend_tiles_kernel(const __grid_constant__ AttendArgs a, int row_blocks)
{
    using S = TlShape<D>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    TlShared *sh = reinterpret_cast<TlShared *>(smem + (kTlTiles + 4) * S::kOperand);
    static_assert(sizeof(TlShared) <= 1024, "");
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    // the last rows of every request first: with a causal mask they have the most to do
    const int per = a.batch * a.c.kv_heads, rb = row_blocks - 1 - (int)blockIdx.x / per, rest = (int)blockIdx.x % per;
    const int i = rest / a.c.kv_heads, head = rest % a.c.kv_heads;
    int row0, n, len;
    if (!attend_request(a, i, row0, n, len)) return;
    const int rows = n * a.group, m0 = rb * kTlSoft;
    if (m0 >= rows) return;
    // blocks of tokens that each tile sees any of
    int blocks[kTlTiles];
#pragma unroll
    for (int x = 0; x < kTlTiles; ++x) {
        const int first = m0 + x * kTlRows, last = min(first + kTlRows, rows) - 1;
        const int end = first >= rows || len < 0 ? 0 : a.causal ? min(len, len - n + 1 + last / a.group) : len;
        blocks[x] = (max(end, 0) + kTlBlock - 1) / kTlBlock;
    }
    const int most = max(blocks[0], blocks[1]);

    if (tid == 0) {
        ptx::mbar_init(&sh->q_full, kTlSoft);
        for (int s = 0; s < 2; ++s) {
            ptx::mbar_init(&sh->k_full[s], 128);
            ptx::mbar_init(&sh->v_full[s], 128);
            ptx::mbar_init(&sh->k_empty[s], 1);
            ptx::mbar_init(&sh->v_empty[s], 1);
        }
        for (int x = 0; x < kTlTiles; ++x) {
            ptx::mbar_init(&sh->s_full[x], 1);
            ptx::mbar_init(&sh->p_full[x], kTlRows);
        }
        ptx::mbar_init(&sh->o_full, 1);
        sh->gave_up = 0;
        ptx::fence_mbar_init();
    }
    if (warp == 12) {
        ptx::tmem_alloc(&sh->tmem, 512);
        ptx::tmem_relinquish();
    }
    ptx::tc_fence_before();
    __syncthreads();
    ptx::tc_fence_after();
    const uint32_t tmem = sh->tmem, s_u32 = ptx::smem_u32(smem);
    const uint32_t k_u32 = s_u32 + kTlTiles * S::kOperand, v_u32 = k_u32 + 2 * S::kOperand;
    // TMEM: scores (and weights over them) of the tiles at columns 0 and 128, outputs at 256 and 256 + D

    if (warp >= 12) {
        // ---------------- the MMAs ------------------------------------------------------------------------
        regs_fewer<kTlMmaRegs>();
        if (warp == 12 && lane == 0 && most > 0) {
            const uint32_t id_s = idesc_f16(kTlRows, kTlBlock, false), id_o = idesc_f16(kTlRows, D, true);
            bool ok = ptx::mbar_wait(&sh->q_full, 0) && ptx::mbar_wait(&sh->k_full[0], 0);
            ptx::tc_fence_after();
            auto scores = [&](int x, int s) {
#pragma unroll
                for (int k = 0; k < D / 16; ++k) {
                    const uint32_t at = (k >> 2) * S::kSlab + (k & 3) * 32;
                    ptx::umma_bf16(tmem + x * 128, ptx::smem_desc_sw128(s_u32 + x * S::kOperand + at, 16, 1024),
                                   ptx::smem_desc_sw128(k_u32 + s * S::kOperand + at, 16, 1024), id_s, k > 0);
                }
                ptx::umma_commit(&sh->s_full[x]);
            };
            if (ok) {
                for (int x = 0; x < kTlTiles; ++x)
                    if (blocks[x] > 0) scores(x, 0);
                ptx::umma_commit(&sh->k_empty[0]);
            }
            for (int j = 0; ok && j < most; ++j) {
                const int s = j & 1;
                bool have_k = false, have_v = false;
                for (int x = 0; ok && x < kTlTiles; ++x) {
                    if (j >= blocks[x]) continue;
                    ok = ptx::mbar_wait(&sh->p_full[x], s);
                    if (ok && !have_v) ok = have_v = ptx::mbar_wait(&sh->v_full[s], (j >> 1) & 1);
                    if (!ok) break;
                    ptx::tc_fence_after();
#pragma unroll
                    for (int k = 0; k < kTlBlock / 16; ++k)
                        umma_f16_ts(tmem + 256 + x * D, tmem + x * 128 + k * 8,
                                    ptx::smem_desc_sw128(v_u32 + s * S::kOperand + k * 2048, S::kSlab, 1024), id_o, j > 0 || k > 0);
                    if (j + 1 < blocks[x]) {
                        if (!have_k) ok = have_k = ptx::mbar_wait(&sh->k_full[s ^ 1], ((j + 1) >> 1) & 1);
                        if (!ok) break;
                        ptx::tc_fence_after();
                        scores(x, s ^ 1);
                    }
                }
                if (ok) {
                    ptx::umma_commit(&sh->v_empty[s]);
                    if (j + 1 < most) ptx::umma_commit(&sh->k_empty[s ^ 1]);
                }
            }
            if (!ok) sh->gave_up = 1;
            // all MMAs done (also after a wait that gave up: the memory they use is about to be freed)
            ptx::umma_commit(&sh->o_full);
            if (!ptx::mbar_wait(&sh->o_full, 0)) sh->gave_up = 1;
        }
    } else if (warp >= 8) {
        // ---------------- codes to fp16 ---------------------------------------------------------------------
        // a thread's pieces: 16 codes of token 32 w + 8 q + lane / 4, piece lane % 4 of each slab: eight neighbouring lanes then
        // store to eight different places of a 128-byte line
        regs_fewer<kTlCodeRegs>();
        const int w = warp - 8, ct = tid - kTlSoft, r = lane >> 2, pc = lane & 3;
        constexpr int kPieces = 4 * S::kSlabs;
        auto page_of = [&](int j, int half) { return attend_page(a, i, min(j * kTlBlock + 32 * w + 16 * half, max(len - 1, 0))); };
        auto load = [&](const int8_t *codes, int j, const int (&page)[2], uint4 (&x)[kPieces]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int t = j * kTlBlock + 32 * w + 8 * q + r;
                const int8_t *from = codes + (((int64_t)max(page[q >> 1], 0) * a.c.kv_heads + head) * a.c.page_size + (t & (a.c.page_size - 1))) * D;
#pragma unroll
                for (int b = 0; b < S::kSlabs; ++b) x[q * S::kSlabs + b] = __ldg(reinterpret_cast<const uint4 *>(from) + b * 4 + pc);
            }
        };
        auto store = [&](uint32_t to, const uint4 (&x)[kPieces]) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int t = 32 * w + 8 * q + r;
#pragma unroll
                for (int b = 0; b < S::kSlabs; ++b) {
                    const uint4 c = x[q * S::kSlabs + b];
                    uint4 lo, hi;
                    codes_to_half(c.x ^ 0x80808080u, lo.x, lo.y);
                    codes_to_half(c.y ^ 0x80808080u, lo.z, lo.w);
                    codes_to_half(c.z ^ 0x80808080u, hi.x, hi.y);
                    codes_to_half(c.w ^ 0x80808080u, hi.z, hi.w);
                    const uint32_t line = to + b * S::kSlab + t * 128;
                    ptx::st_shared_v4(line + (((2 * pc) ^ (t & 7)) << 4), lo);
                    ptx::st_shared_v4(line + (((2 * pc + 1) ^ (t & 7)) << 4), hi);
                }
            }
        };
        // scales of the 16 tokens that thread ct < 8 looks after
        auto scales = [&](int j) {
            const int page = attend_page(a, i, min(j * kTlBlock + 16 * ct, max(len - 1, 0)));
            const int64_t block = (int64_t)max(page, 0) * a.c.kv_heads + head;
            const float nan = __uint_as_float(0x7fc00000u);
            return make_float2(page < 0 ? nan : __ldg(a.c.k_scale + block), page < 0 ? nan : __ldg(a.c.v_scale + block));
        };
        uint4 xk[kPieces], xv[kPieces];
        int page[2];
        float2 sc = make_float2(0.f, 0.f);
        if (most > 0) {
            page[0] = page_of(0, 0);
            page[1] = page_of(0, 1);
            load(a.c.k, 0, page, xk);
            load(a.c.v, 0, page, xv);
            if (ct < kTlGroups) sc = scales(0);
        }
        bool ok = true;
        for (int j = 0; j < most; ++j) {
            const int s = j & 1, more = j + 1 < most;
            if (more) {
                page[0] = page_of(j + 1, 0);
                page[1] = page_of(j + 1, 1);
            }
            if (j >= 2 && !(ok = ptx::mbar_wait(&sh->k_empty[s], ((j >> 1) - 1) & 1))) break;
            store(k_u32 + s * S::kOperand, xk);
            if (ct < kTlGroups) {
                float lv, inv;
                value_scale(sc.y, lv, inv);
                sh->group[j & 3][ct] = make_float4(sc.x, lv, inv, 0.f);
            }
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(&sh->k_full[s]);
            if (more) {
                load(a.c.k, j + 1, page, xk);
                if (ct < kTlGroups) sc = scales(j + 1);
            }
            if (j >= 2 && !(ok = ptx::mbar_wait(&sh->v_empty[s], ((j >> 1) - 1) & 1))) break;
            store(v_u32 + s * S::kOperand, xv);
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(&sh->v_full[s]);
            if (more) load(a.c.v, j + 1, page, xv);
        }
        if (!ok) sh->gave_up = 1;
    } else {
        // ---------------- a row per thread -------------------------------------------------------------------
        regs_more<kTlSoftRegs>();
        const int x = warp >> 2, r = tid & 127, m = m0 + x * kTlRows + r, j_row = m / a.group;
        const bool real = m < rows;
        const uint32_t q_row = s_u32 + x * S::kOperand + r * 128;
        const int64_t o_row = (int64_t)(row0 + j_row) * a.q_heads + head * a.group + (m - j_row * a.group);
        float factor = 0.f;
        {
            uint4 raw[D / 8];
            float top = 0.f;
            const uint4 *p = reinterpret_cast<const uint4 *>(a.q + (int64_t)(row0 + j_row) * a.q_stride +
                                                             (int64_t)(head * a.group + (m - j_row * a.group)) * D);
#pragma unroll
            for (int e = 0; e < D / 8; ++e) raw[e] = real ? __ldg(p + e) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                float f[8];
                Elem<__nv_bfloat16>::unpack(raw[e], f);
#pragma unroll
                for (int z = 0; z < 8; ++z) top = max_nan(top, fabsf(f[z]));
            }
            float unit = query_scale(top, a.scale_log2, factor);
            if (factor < 0.f) {                      // the scores' factor is positive: the largest sum is the largest score
                factor = -factor;
                unit = -unit;
            }
#pragma unroll
            for (int e = 0; e < D / 8; ++e) {
                float f[8];
                Elem<__nv_bfloat16>::unpack(raw[e], f);
                uint4 h = make_uint4(pack_half(f[0] * unit, f[1] * unit), pack_half(f[2] * unit, f[3] * unit),
                                     pack_half(f[4] * unit, f[5] * unit), pack_half(f[6] * unit, f[7] * unit));
                ptx::st_shared_v4(q_row + (e >> 3) * S::kSlab + (((e & 7) ^ (r & 7)) << 4), h);
            }
            ptx::fence_proxy_async_smem();
            ptx::mbar_arrive(&sh->q_full);
        }
        const int end = a.causal ? min(len, len - n + 1 + min(m, rows - 1) / a.group) : len;
        // the first row of the warp sees the fewest tokens
        const int warp_end = a.causal ? min(len, len - n + 1 + min(m - lane, rows - 1) / a.group) : len;
        const uint32_t lanes = (uint32_t)(warp & 3) << 21, t_s = tmem + lanes + x * 128, t_o = tmem + lanes + 256 + x * D;
        float top = kAtNothing, l = 0.f;
        bool ok = true;
        for (int j = 0; j < blocks[x]; ++j) {
            if (!(ok = ptx::mbar_wait(&sh->s_full[x], j & 1))) break;
            ptx::tc_fence_after();
            const float4 *group = sh->group[j & 3];
            const int left = end - j * kTlBlock;     // tokens of the block that the row sees
            const bool masked = (j + 1) * kTlBlock > warp_end;
            // ---- the row's maximum (of s', with the values' scale)
            uint32_t v[kTlBlock];
#pragma unroll
            for (int c = 0; c < kTlBlock / 32; ++c) ptx::tmem_ld32(t_s + c * 32, *reinterpret_cast<uint32_t (*)[32]>(v + c * 32));
            ptx::tmem_ld_wait();
            float now = kAtNothing;
#pragma unroll
            for (int c = 0; c < kTlGroups; ++c) {
                float most_s = -INFINITY;
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) most_s = fmaxf(most_s, 16 * c + e < left ? __uint_as_float(v[16 * c + e]) : -INFINITY);
                } else {
#pragma unroll
                    for (int e = 0; e < 16; ++e) most_s = fmaxf(most_s, __uint_as_float(v[16 * c + e]));
                }
                const float4 g = group[c];
                now = fmaxf(now, fmaf(most_s, factor * g.x, g.y));
            }
            if (__any_sync(0xffffffffu, now - top > kAtSlack)) {
                const float next = fmaxf(top, now), k = ex2(top - next);
                top = next;
                l *= k;
                if (j > 0) {
#pragma unroll
                    for (int c = 0; c < D / 16; ++c) {
                        uint32_t v[16];
                        ptx::tmem_ld16(t_o + c * 16, v);
                        ptx::tmem_ld_wait();
#pragma unroll
                        for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * k);
                        tmem_st16(t_o + c * 16, v);
                    }
                }
            }
            // ---- weights
            if (masked || __any_sync(0xffffffffu, fabsf(top) > kTlLarge)) tile_weights<true>(v, group, factor, top, left, t_s, l);
            else tile_weights<false>(v, group, factor, top, left, t_s, l);
            tmem_st_wait();
            ptx::tc_fence_before();
            ptx::mbar_arrive(&sh->p_full[x]);
        }
        if (!ok) sh->gave_up = 1;
        // ---- out
        if (most > 0 && !ptx::mbar_wait(&sh->o_full, 0)) sh->gave_up = 1;
        ptx::tc_fence_after();
        const bool nan = len < 0 || sh->gave_up;
        const float k = nan ? __uint_as_float(0x7fc00000u) : l == 0.f ? 0.f : 1.f / l;
#pragma unroll
        for (int c = 0; c < D / 16; ++c) {
            uint32_t v[16];
            ptx::tmem_ld16(t_o + c * 16, v);
            ptx::tmem_ld_wait();
            uint4 o[2];
            __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(o);
#pragma unroll
            for (int e = 0; e < 8; ++e)              // (a tile that saw no block has no sums: what TMEM holds is not used)
                h[e] = blocks[x] > 0 || nan ? __floats2bfloat162_rn(__uint_as_float(v[2 * e]) * k, __uint_as_float(v[2 * e + 1]) * k)
                                            : __floats2bfloat162_rn(0.f, 0.f);
            // over the queries (all MMAs are done), swizzled alike
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const int ch = 2 * c + e;
                ptx::st_shared_v4(q_row + (ch >> 3) * S::kSlab + (((ch & 7) ^ (r & 7)) << 4), o[e]);
            }
        }
        if (real && a.lse) a.lse[o_row] = nan ? k : l == 0.f ? -INFINITY : (top + log2f(l)) * kAtLn2;
        __syncwarp();
        // whole rows, 16 bytes a lane
        constexpr int kLanes = D / 8;                // lanes of a row
        const int first = m0 + x * kTlRows + (r & ~31);
#pragma unroll 4
        for (int y = lane / kLanes; y < 32; y += 32 / kLanes) {
            const int mm = first + y, ch = lane % kLanes, rr = (r & ~31) + y;
            if (mm < rows) {
                const int jj = mm / a.group;
                const int64_t row = (int64_t)(row0 + jj) * a.q_heads + head * a.group + (mm - jj * a.group);
                const float4 o = ptx::ld_shared_v4(s_u32 + x * S::kOperand + rr * 128 + (ch >> 3) * S::kSlab + (((ch & 7) ^ (rr & 7)) << 4));
                *reinterpret_cast<float4 *>(a.out + row * D + ch * 8) = o;
            }
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
