// Attention of few query rows per kv head (single tokens, a few drafted ones) over the 8-bit paged cache: bound by reading
// the codes once.
//
// A tile of rows (a token's heads of one kv head, token by token) against 64 tokens a step, a warp 16 of them, on mma.sync m16n8k16: at one
// or a few rows the tensor cores are idle either way (a step of 16 KB has 0.7 us of HBM time per SM and 0.02 of mma), and its fragments come
// straight out of 16-byte pieces because both contractions may run in any order:
//   scores  a lane takes 32 (D = 64: 16) neighbouring elements of a token's key; the queries' fragments are laid out to match
//   values  a lane takes 16 (8) neighbouring columns of four tokens
// Tiles of 16 rows have the rows as the mma's 16 and tokens or columns as its 8.  Calls of at most 8 rows a kv head have tiles of 8, the other way round:
// half the mma, half the accumulators, half the softmax; the weights change sides by movmatrix.
// Codes come by 16-byte cp.async into a ring of steps in shared memory, the pieces swizzled by row so that both ways of reading find them in
// different banks; a fifth warp fetches them, with the scales of their blocks, and walks the tables: the four others have nothing but
// the arithmetic, about 300 instructions for 16 tokens, and that is what HBM is kept waiting by (with the fetching in the same warps it
// was 540, and 4.7 TB/s).
//
// The work, all (request, kv head, tile of rows) with their blocks of 64 tokens, is one line that is cut into equal runs, one per CTA
// (two or three to an SM), whatever the requests' lengths: each CTA sums up the batch for itself and finds its place.  A tile that a cut goes through is
// left in parts (fp32 sums, m', l) that attend_join_kernel puts together in the order of the line, so results do not depend on timing.
// Where every tile has a CTA of its own and few blocks, each CTA takes its tile whole, and there is nothing to join.
// The ring runs across tiles: the next one's codes are on their way while this one's warps are added up.
// Steps with tokens that a row does not see, and all behind one whose scales want a reference of their own for l, take the largest s and s'
// anew; the others only where a weight would pass 2^8.
// 16 requests of 8000 to 32000 tokens, 32 heads on 8: 122 us, 5.3 TB/s; 64 of 350 to 1500, 10 heads: 38 us, 4.1 TB/s
// (of 4096 in a batch of which the others have no rows 49 us).
#pragma once
#include "attend.cuh"

namespace rtp {

constexpr int kArWarps = 4;                          // that compute; one more fetches
constexpr int kArThreads = 32 * (kArWarps + 1);
constexpr int kArBlock = 16 * kArWarps;              // tokens of a step
constexpr int kArMostCtas = 3 * 160;                 // what the workspace is sized for (a B200 has 148 SMs)
constexpr int kArRows = 16;
constexpr int kArLeast = 4;                          // blocks of a run at least
constexpr int kArWhole = 8;                          // blocks of the longest tile up to which tiles are taken whole

template <int D, int R> struct ArShape {
    // CTAs of an SM (with 16 rows three would leave a thread 128 registers, which spill: no kernel here may have a stack frame)
    static constexpr int kPerSm = R == 8 ? 3 : 2;
    static constexpr int kStages = (R == 8 ? 4 : 5) * (D == 128 ? 1 : 2);
    static constexpr int kBytes = kArBlock * D;      // keys (or values) of a step
    static constexpr int kSteps = D / 16;            // mma steps of a score
    static constexpr int kNt = R == 8 ? D / 16 : D / 8;            // mma tiles of the output
    static constexpr int kRing = kStages * 2 * kBytes;
    static constexpr int kFrag = R == 8 ? 0 : kSteps * 32 * 16;    // the queries' fragments
    static constexpr int kJoin = (kArWarps / 2) * 32 * kNt * 16;   // accumulators of half the warps
    static constexpr int kSmem = kRing + kFrag + kJoin + 1024 /*alignment*/;
};

// A place in the line of work.
struct ArPlace {
    int i, head, tile, block;                        // request, kv head, tile of rows, block of tokens
    int row0, n, len, blocks, tiles;                 // of the request

    template <int R> __device__ void request(const AttendArgs &a, int at)
    {
        i = at;
        head = tile = block = 0;
        tiles = 0;
        if (i < a.batch && attend_request(a, i, row0, n, len)) {
            tiles = (n * a.group + R - 1) / R;
            blocks = max(1, (len + kArBlock - 1) / kArBlock);
        }
    }
    // `steps` blocks on, within the tile or to the next one's first, for a whole warp (the line ends before the batch does: the caller
    // counts, and does not ask for what is behind the line's end).  Requests without rows are passed over 32 at a time.
    template <int R> __device__ void next(const AttendArgs &a, int steps)
    {
        block += steps;
        if (block < blocks) return;
        block = 0;
        if (++tile < tiles) return;
        tile = 0;
        if (++head < a.c.kv_heads) return;
        head = tiles = 0;
        uint32_t found = 0;
        for (++i; i < a.batch; i += 32) {
            const int mine = i + (int)(threadIdx.x & 31);
            found = __ballot_sync(0xffffffffu, mine < a.batch && attend_request(a, mine, row0, n, len));
            if (found) break;
        }
        if (!found) return;
        const int from = __ffs(found) - 1;
        i += from;
        row0 = __shfl_sync(0xffffffffu, row0, from);
        n = __shfl_sync(0xffffffffu, n, from);
        len = __shfl_sync(0xffffffffu, len, from);
        tiles = (n * a.group + R - 1) / R;
        blocks = max(1, (len + kArBlock - 1) / kArBlock);
    }
};

template <int R> __device__ inline int64_t ar_units(const AttendArgs &a, int i, bool whole)
{
    int row0, n, len;
    if (!attend_request(a, i, row0, n, len)) return 0;
    return (int64_t)((n * a.group + R - 1) / R) * a.c.kv_heads * (whole ? 1 : max(1, (len + kArBlock - 1) / kArBlock));
}

// Where CTA `blockIdx.x` of the line begins, and how many blocks it takes (0: none).  whole: it takes the tile of that number.
template <int R> __device__ inline int ar_find(const AttendArgs &a, bool whole, ArPlace &at, int &chunk)
{
    __shared__ int64_t warp_units[kArWarps + 1], found_before;
    __shared__ int found;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int per = (a.batch + kArThreads - 1) / kArThreads, i0 = min(tid * per, a.batch), i1 = min(i0 + per, a.batch);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += ar_units<R>(a, i, whole);
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
    }
    if (lane == 31) warp_units[warp] = upto;
    __syncthreads();
    int64_t total = 0, before = upto - mine;
#pragma unroll
    for (int w = 0; w <= kArWarps; ++w) {
        if (w < warp) before += warp_units[w];
        total += warp_units[w];
    }
    const int64_t run = whole ? 1 : max((total + gridDim.x - 1) / gridDim.x, (int64_t)kArLeast);
    const int64_t start = run * blockIdx.x;
    chunk = (int)run;
    if (start >= total) return 0;
    if (start >= before && start < before + mine) {
        int i = i0;
        for (int64_t u; (u = ar_units<R>(a, i, whole)) <= start - before; ++i) before += u;
        found = i;
        found_before = before;
    }
    __syncthreads();
    at.request<R>(a, found);
    const int64_t rel = start - found_before;
    if (whole) {
        at.tile = (int)(rel % at.tiles);
        at.head = (int)(rel / at.tiles);
        return at.blocks;
    }
    at.block = (int)(rel % at.blocks);
    at.tile = (int)(rel / at.blocks % at.tiles);
    at.head = (int)(rel / at.blocks / at.tiles);
    return (int)min(run, total - start);
}

__device__ inline void mma_f16(float (&d)[4], const uint4 &a, uint32_t b0, uint32_t b1)
{
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a.x), "r"(a.y), "r"(a.z), "r"(a.w), "r"(b0), "r"(b1));
}
__device__ inline uint4 lds_v4(uint32_t at)
{
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ inline uint2 lds_v2(uint32_t at)
{
    uint2 v;
    asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(at));
    return v;
}
__device__ inline float2 lds_f2(uint32_t at)
{
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(at));
    return v;
}
__device__ inline float4 lds_f4(uint32_t at)
{
    float4 v;
    asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at));
    return v;
}
// The four warps that compute, among themselves.
__device__ inline void ar_sync() { asm volatile("bar.sync 1, %0;" ::"n"(32 * kArWarps) : "memory"); }

// Place of 16-byte piece `ch` of row t of a step (rows of a warp's 16 tokens are 16 neighbouring rows).
template <int D> __device__ inline uint32_t ar_piece(int t, int ch)
{
    if (D == 128) return (uint32_t)(t * 128 + ((ch ^ (t & 7)) << 4));
    const int line = t >> 1;
    return (uint32_t)(line * 128 + ((((t & 1) * 4 + ch) ^ ((line & 3) << 1)) << 4));
}

// An 8 x 8 matrix of fp16, a row's two neighbouring elements a lane, to its transpose.
__device__ inline uint32_t mat_trans(uint32_t x)
{
    uint32_t r;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(x));
    return r;
}

// Parts of a tile that a cut goes through: `part` [2 per CTA][16][D] sums, `part_ml` [2 per CTA][16] (m', l, r).  A part that holds its
// tile's first block is the CTA's second, any other its first.  join[CTA]: the tile that begins in the CTA and does not end in it:
// (first row of the request, kv head, the tile's first row | its rows << 26, CTAs that it goes through; 0: there is none).
template <int D, int R>
__global__ void __launch_bounds__(kArThreads, ArShape<D, R>::kPerSm)
attend_rows_kernel(const __grid_constant__ AttendArgs a, int whole_tiles, float *__restrict__ part, float4 *__restrict__ part_ml, int4 *__restrict__ join)
{
    using S = ArShape<D, R>;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *sm = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ float row_factor[kArRows];
    __shared__ float2 row_ml[kArWarps][R];
    __shared__ float row_ref[kArWarps][R];           // r of a warp's rows once they have one; infinity before (it is m' then)
    __shared__ float4 scales[S::kStages][kArWarps];  // ks, log2 vs, 1 / vs of each warp's 16 tokens; w: infinity from the tile's first wide one on, else 0
    __shared__ uint64_t full[S::kStages], empty[S::kStages];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
    const uint32_t ring = ptx::smem_u32(sm), frag = ring + S::kRing, scales_u32 = ptx::smem_u32(scales);
    const uint32_t joined = frag + S::kFrag + lane * 16;
    if (tid == 0) {
        for (int s = 0; s < S::kStages; ++s) {
            ptx::mbar_init(&full[s], 33);            // every lane's copies, and the scales
            ptx::mbar_init(&empty[s], kArWarps);
        }
        ptx::fence_mbar_init();
    }
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    ArPlace at;
    int chunk;
    const int todo = ar_find<R>(a, whole_tiles, at, chunk);          // (its barriers order the initialisation too)
    if (todo == 0) {
        if (tid == 0 && !whole_tiles) join[blockIdx.x] = make_int4(0, 0, 0, 0);
        return;
    }

    if (warp == kArWarps) {
        // ---------------- codes and scales: a step ahead with the tables ---------------------------------------
        const float nan = __uint_as_float(0x7fc00000u);
        uint32_t n = 0;
        // of the step that is fetched, for the 16 tokens of warp lane / 8: their block (-1: none), and the codes' place in it
        int block = -1, slot = 0;
        bool fresh = false, wide = false;            // a tile's first step (of this CTA); a scale so far wants a reference of its own for l
#pragma unroll 1
        for (int look = 0; look <= todo; ++look) {
            int next_block = -1, next_slot = 0;
            bool next_fresh = false;
            if (look < todo) {
                next_fresh = at.block == 0;
                const int t = at.block * kArBlock + (lane >> 3) * 16;
                const int page = t < at.len ? attend_page(a, at.i, t) : -1;
                next_block = page < 0 ? -1 : page * a.c.kv_heads + at.head;
                next_slot = t & (a.c.page_size - 1);
                if (look + 1 < todo) at.next<R>(a, 1);
            }
            if (look > 0) {
                const uint32_t s = n % S::kStages, turn = n / S::kStages, to = ring + s * 2 * S::kBytes;
                const float ks = block < 0 ? nan : __ldg(a.c.k_scale + block), vs = block < 0 ? nan : __ldg(a.c.v_scale + block);
                bool ok = true;
                if (turn > 0) ok = ptx::mbar_wait(&empty[s], (turn - 1) & 1, a.polls);
                if (!__all_sync(0xffffffffu, ok)) break;
                const int64_t from = ((int64_t)max(block, 0) * a.c.page_size + slot) * D;
#pragma unroll
                for (int w = 0; w < kArWarps; ++w) {
                    if (__shfl_sync(0xffffffffu, block, 8 * w) < 0) continue;
                    const int64_t base = __shfl_sync(0xffffffffu, from, 8 * w);
#pragma unroll
                    for (int p = 0; p < D / 32; ++p) {
                        const int piece = lane + 32 * p, t = piece / (D / 16), ch = piece % (D / 16);
                        const uint32_t place = to + ar_piece<D>(16 * w + t, ch);
                        ptx::cp_async_16(place, a.c.k + base + piece * 16, 16);
                        ptx::cp_async_16(place + S::kBytes, a.c.v + base + piece * 16, 16);
                    }
                }
                ptx::cp_async_arrive(&full[s]);
                float lv, inv;
                wide = value_scale(vs, lv, inv) || (wide && !fresh);
                if ((lane & 7) == 0) scales[s][lane >> 3] = make_float4(ks, lv, inv, wide ? INFINITY : 0.f);
                __syncwarp();
                if (lane == 0) ptx::mbar_arrive(&full[s]);
                ++n;
            }
            block = next_block;
            slot = next_slot;
            fresh = next_fresh;
        }
        // no copy, nor its arrival, is left on its way into memory that this CTA gives back
        for (uint32_t c = n > S::kStages ? n - S::kStages : 0; c < n; ++c) ptx::mbar_wait(&full[c % S::kStages], c / S::kStages & 1);
        return;
    }

    uint32_t n = 0;                                  // steps so far
    bool dead = false;                               // a wait gave up: what is left comes out NaN
#pragma unroll 1
    for (int left = todo; left > 0;) {
        // ---- a tile of rows: its queries as fragments
        const int first = at.block, steps = min(left, at.blocks - at.block), rows = at.n * a.group;
        float f0, f1;                                // factors of this lane's two rows
        uint32_t qf[R == 8 ? S::kSteps * 2 : 1];     // 8 rows: this lane's fragments
        if constexpr (R == 8) {
            // row g, elements D / 4 * c ..
            const int m = at.tile * R + g, j = min(m, rows - 1) / a.group, h = at.head * a.group + (min(m, rows - 1) - j * a.group);
            const uint4 *p = reinterpret_cast<const uint4 *>(a.q + (int64_t)(at.row0 + j) * a.q_stride + (int64_t)h * D + c * (D / 4));
            uint4 raw[D / 32];
#pragma unroll
            for (int e = 0; e < D / 32; ++e) {
                raw[e] = make_uint4(0u, 0u, 0u, 0u);
                if (m < rows) raw[e] = __ldg(p + e);
            }
            float top = 0.f;
#pragma unroll
            for (int e = 0; e < D / 32; ++e) {
                float t8[8];
                Elem<__nv_bfloat16>::unpack(raw[e], t8);
#pragma unroll
                for (int x = 0; x < 8; ++x) top = max_nan(top, fabsf(t8[x]));
            }
            top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 1));
            top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 2));
            float factor;
            const float unit = query_scale(top, a.scale_log2, factor);
#pragma unroll
            for (int e = 0; e < D / 32; ++e) {
                float t8[8];
                Elem<__nv_bfloat16>::unpack(raw[e], t8);
#pragma unroll
                for (int x = 0; x < 4; ++x) qf[4 * e + x] = pack_half(t8[2 * x] * unit, t8[2 * x + 1] * unit);
            }
            f0 = __shfl_sync(0xffffffffu, factor, 8 * c);
            f1 = __shfl_sync(0xffffffffu, factor, 8 * c + 4);
        } else {
            ar_sync();                                   // the last tile's fragments and sums have been read
            {
                constexpr int kPer = D / 8;              // elements of a thread: 8 threads a row
                const int r = tid >> 3, k = tid & 7, m = at.tile * R + r;
                uint4 raw[kPer / 8];
#pragma unroll
                for (int e = 0; e < kPer / 8; ++e) raw[e] = make_uint4(0u, 0u, 0u, 0u);
                if (m < rows) {
                    const int j = m / a.group, h = at.head * a.group + (m - j * a.group);
                    const uint4 *p = reinterpret_cast<const uint4 *>(a.q + (int64_t)(at.row0 + j) * a.q_stride + (int64_t)h * D + k * kPer);
#pragma unroll
                    for (int e = 0; e < kPer / 8; ++e) raw[e] = __ldg(p + e);
                }
                float f[kPer], top = 0.f;
#pragma unroll
                for (int e = 0; e < kPer / 8; ++e) {
                    float t8[8];
                    Elem<__nv_bfloat16>::unpack(raw[e], t8);
#pragma unroll
                    for (int x = 0; x < 8; ++x) {
                        f[8 * e + x] = t8[x];
                        top = max_nan(top, fabsf(t8[x]));
                    }
                }
#pragma unroll
                for (int o = 1; o < 8; o <<= 1) top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, o));
                float factor;
                const float unit = query_scale(top, a.scale_log2, factor);
                if (k == 0) row_factor[r] = factor;
                // element d: lane (r & 7) * 4 + d / (D / 4), step (d mod D / 4) / 4, register (d & 2) + (r >= 8)
#pragma unroll
                for (int e = 0; e < kPer; e += 2) {
                    const int d = k * kPer + e, lane_to = (r & 7) * 4 + d / (D / 4), step = d % (D / 4) / 4;
                    const uint32_t to = frag + (uint32_t)((step * 32 + lane_to) * 16 + ((d & 2) + (r >> 3)) * 4);
                    asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(pack_half(f[e] * unit, f[e + 1] * unit)) : "memory");
                }
            }
            ar_sync();
            f0 = row_factor[g];
            f1 = row_factor[g + 8];
        }
        // this lane's two rows: 2c, 2c + 1 of 8, or g, g + 8 of 16
        const int mine[2] = {R == 8 ? 2 * c : g, R == 8 ? 2 * c + 1 : g + 8};
        // ends of this lane's two rows, of the tile's first and last one
        int end[2], lo_end, hi_end;
        {
            const int m0 = at.tile * R, last = min(m0 + R, rows) - 1, len = max(at.len, 0), past = len - at.n + 1;
            end[0] = a.causal ? min(len, past + min(m0 + mine[0], last) / a.group) : len;
            end[1] = a.causal ? min(len, past + min(m0 + mine[1], last) / a.group) : len;
            lo_end = a.causal ? min(len, past + m0 / a.group) : len;
            hi_end = a.causal ? min(len, past + last / a.group) : len;
        }
        float acc[S::kNt][4], m[2] = {kAtNothing, kAtNothing}, l[2] = {0.f, 0.f};
#pragma unroll
        for (int j = 0; j < S::kNt; ++j) acc[j][0] = acc[j][1] = acc[j][2] = acc[j][3] = 0.f;

        if (R == 8 ? g == 0 : c == 0) row_ref[warp][mine[0]] = row_ref[warp][mine[1]] = INFINITY;
        __syncwarp();
        int t0 = first * kArBlock + warp * 16;
        uint32_t stage = n % S::kStages, parity = n / S::kStages & 1;
#pragma unroll 1
        for (int b = 0; b < steps; ++b, t0 += kArBlock) {
            // (lane by lane: nothing below branches on it, and what a lane reads of a step that is not there are codes and scales all the same)
            if (!dead && !ptx::mbar_wait(&full[stage], parity, a.polls)) dead = true;
            __syncwarp();
            const uint32_t kt = ring + stage * 2 * S::kBytes + warp * 16 * D, vt = kt + S::kBytes;
            if (t0 < hi_end) {
                const float4 sc = lds_f4(scales_u32 + (stage * kArWarps + warp) * 16);
                if constexpr (R == 8) {
                    // ---- scores of tokens t0 + g (s[0], s[1]) and 8 more (s[2], s[3]) for rows 2c, 2c + 1
                    float s[4] = {};
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        const uint4 k0 = lds_v4(kt + ar_piece<D>(g, D == 128 ? 2 * c + h : c)), k1 = lds_v4(kt + ar_piece<D>(g + 8, D == 128 ? 2 * c + h : c));
                        const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            uint4 ka;
                            codes_to_half(w0[e] ^ 0x80808080u, ka.x, ka.z);
                            codes_to_half(w1[e] ^ 0x80808080u, ka.y, ka.w);
                            mma_f16(s, ka, qf[2 * (h * 4 + e)], qf[2 * (h * 4 + e) + 1]);
                        }
                    }
                    // ---- weights
                    const float k0 = f0 * sc.x, k1 = f1 * sc.x;
                    float w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) w[e] = fmaf(s[e], e & 1 ? k1 : k0, sc.y);
                    const float top0 = fmaxf(w[0], w[2]), top1 = fmaxf(w[1], w[3]);
                    bool careful = t0 + 16 > lo_end;
                    if (__any_sync(0xffffffffu, careful || fmaxf(fmaxf(top0 - m[0], top1 - m[1]), sc.w) > kAtSlack)) {
                        careful = careful || __any_sync(0xffffffffu, sc.w != 0.f);
                        if (careful) {
                            // tokens that a row does not see, or a reference of its own for l, from here to the tile's end: the largest s and
                            // s' are taken every time
                            bool seen[4];
                            float top_s[2], top[2], r[2];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                s[e] *= e & 1 ? k1 : k0;
                                seen[e] = t0 + g + 8 * (e >> 1) < end[e & 1];
                            }
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                top_s[x] = fmaxf(seen[x] ? s[x] : -INFINITY, seen[2 + x] ? s[2 + x] : -INFINITY);
#pragma unroll
                                for (int o = 4; o < 32; o <<= 1) top_s[x] = fmaxf(top_s[x], __shfl_xor_sync(0xffffffffu, top_s[x], o));
                                r[x] = row_ref[warp][mine[x]];
                                if (r[x] == INFINITY) r[x] = m[x];
                                top[x] = fmaxf(m[x], top_s[x] + sc.y);
                                const float to = fmaxf(r[x], top_s[x]), k = ex2(m[x] - top[x]);
                                l[x] *= ex2(r[x] - to);
                                m[x] = top[x];
                                r[x] = to;
#pragma unroll
                                for (int j = 0; j < S::kNt; ++j) {
                                    acc[j][x] *= k;
                                    acc[j][x + 2] *= k;
                                }
                            }
                            __syncwarp();
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                if (g == 0) row_ref[warp][mine[x]] = r[x];
                                const float gap = m[x] - r[x], lv = weight_log(sc.y, gap);
                                s[x] = seen[x] ? ex2(s[x] + lv - m[x]) : 0.f;
                                s[2 + x] = seen[2 + x] ? ex2(s[2 + x] + lv - m[x]) : 0.f;
                                if (seen[x] || seen[2 + x]) l[x] = fmaf(s[x] + s[2 + x], ex2(gap - lv), l[x]);
                            }
                            __syncwarp();
                        } else {
                            float n0 = top0, n1 = top1;
#pragma unroll
                            for (int o = 4; o < 32; o <<= 1) {
                                n0 = fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, o));
                                n1 = fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, o));
                            }
                            n0 = fmaxf(m[0], n0);
                            n1 = fmaxf(m[1], n1);
                            const float c0 = ex2(m[0] - n0), c1 = ex2(m[1] - n1);
                            m[0] = n0;
                            m[1] = n1;
                            l[0] *= c0;
                            l[1] *= c1;
#pragma unroll
                            for (int j = 0; j < S::kNt; ++j) {
                                acc[j][0] *= c0;
                                acc[j][1] *= c1;
                                acc[j][2] *= c0;
                                acc[j][3] *= c1;
                            }
                        }
                    }
                    if (!careful) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) s[e] = ex2(w[e] - m[e & 1]);
                        l[0] = fmaf(s[0] + s[2], sc.z, l[0]);
                        l[1] = fmaf(s[1] + s[3], sc.z, l[1]);
                    }
                    const uint32_t b0 = mat_trans(pack_half(s[0], s[1])), b1 = mat_trans(pack_half(s[2], s[3]));
                    // ---- values: tokens 2c, 2c + 1, 2c + 8, 2c + 9, columns D / 8 * g ..: mma tile j has columns 2j and 2j + 1 of these
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) {
                        uint32_t v[4][2];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int t = 2 * c + (x & 1) + 8 * (x >> 1);
                            const uint2 r = D == 128 ? lds_v2(vt + ar_piece<D>(t, g) + half * 8) : lds_v2(vt + ar_piece<D>(t, g >> 1) + (g & 1) * 8);
                            v[x][0] = r.x ^ 0x80808080u;
                            v[x][1] = r.y ^ 0x80808080u;
                        }
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            uint4 va, vb;
                            codes_to_half(__byte_perm(v[0][w], v[1][w], 0x5140), va.x, va.y);
                            codes_to_half(__byte_perm(v[2][w], v[3][w], 0x5140), va.z, va.w);
                            codes_to_half(__byte_perm(v[0][w], v[1][w], 0x7362), vb.x, vb.y);
                            codes_to_half(__byte_perm(v[2][w], v[3][w], 0x7362), vb.z, vb.w);
                            mma_f16(acc[2 * (2 * half + w)], va, b0, b1);
                            mma_f16(acc[2 * (2 * half + w) + 1], vb, b0, b1);
                        }
                    }
                } else {
                    // ---- scores of tokens t0 + 2c, 2c + 1 (s[0]) and 8 more (s[1]) for rows g, g + 8
                    float s[2][4] = {};
#pragma unroll
                    for (int h = 0; h < D / 64; ++h) {
                        uint32_t w[2][4];
#pragma unroll
                        for (int x = 0; x < 2; ++x) {
                            const uint4 v = lds_v4(kt + ar_piece<D>(g + 8 * x, D == 128 ? 2 * c + h : c));
                            w[x][0] = v.x ^ 0x80808080u;
                            w[x][1] = v.y ^ 0x80808080u;
                            w[x][2] = v.z ^ 0x80808080u;
                            w[x][3] = v.w ^ 0x80808080u;
                        }
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const uint4 qf = lds_v4(frag + (uint32_t)(((h * 4 + e) * 32 + lane) * 16));
#pragma unroll
                            for (int x = 0; x < 2; ++x) {
                                uint32_t b0, b1;
                                codes_to_half(w[x][e], b0, b1);
                                mma_f16(s[x], qf, b0, b1);
                            }
                        }
                    }
                    // ---- weights
                    const float k0 = f0 * sc.x, k1 = f1 * sc.x;
                    float w[2][4];
#pragma unroll
                    for (int x = 0; x < 2; ++x)
#pragma unroll
                        for (int e = 0; e < 4; ++e) w[x][e] = fmaf(s[x][e], e < 2 ? k0 : k1, sc.y);
                    const float top0 = fmaxf(fmaxf(w[0][0], w[0][1]), fmaxf(w[1][0], w[1][1]));
                    const float top1 = fmaxf(fmaxf(w[0][2], w[0][3]), fmaxf(w[1][2], w[1][3]));
                    bool careful = t0 + 16 > lo_end;
                    if (__any_sync(0xffffffffu, careful || fmaxf(fmaxf(top0 - m[0], top1 - m[1]), sc.w) > kAtSlack)) {
                        careful = careful || __any_sync(0xffffffffu, sc.w != 0.f);
                        if (careful) {
                            // (as with 8 rows)
#pragma unroll
                            for (int h = 0; h < 2; ++h) {        // row g + 8 h: its scores are s[0][2h], s[0][2h + 1], s[1][2h], s[1][2h + 1]
                                float top_s = -INFINITY;
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    float &x = s[e >> 1][2 * h + (e & 1)];
                                    x *= h ? k1 : k0;
                                    if (t0 + 8 * (e >> 1) + 2 * c + (e & 1) < end[h]) top_s = fmaxf(top_s, x);
                                }
                                top_s = fmaxf(top_s, __shfl_xor_sync(0xffffffffu, top_s, 1));
                                top_s = fmaxf(top_s, __shfl_xor_sync(0xffffffffu, top_s, 2));
                                float r = row_ref[warp][mine[h]];
                                if (r == INFINITY) r = m[h];
                                const float top = fmaxf(m[h], top_s + sc.y), to = fmaxf(r, top_s), k = ex2(m[h] - top);
                                l[h] *= ex2(r - to);
                                m[h] = top;
#pragma unroll
                                for (int j = 0; j < S::kNt; ++j) {
                                    acc[j][2 * h] *= k;
                                    acc[j][2 * h + 1] *= k;
                                }
                                __syncwarp();
                                if (c == 0) row_ref[warp][mine[h]] = to;
                                __syncwarp();
                                const float gap = top - to, lv = weight_log(sc.y, gap), z = ex2(gap - lv);
#pragma unroll
                                for (int e = 0; e < 4; ++e) {
                                    float &x = s[e >> 1][2 * h + (e & 1)];
                                    const bool seen = t0 + 8 * (e >> 1) + 2 * c + (e & 1) < end[h];
                                    x = seen ? ex2(x + lv - top) : 0.f;
                                    if (seen) l[h] = fmaf(x, z, l[h]);
                                }
                            }
                        } else {
                            float n0 = fmaxf(top0, __shfl_xor_sync(0xffffffffu, top0, 1)), n1 = fmaxf(top1, __shfl_xor_sync(0xffffffffu, top1, 1));
                            n0 = fmaxf(m[0], fmaxf(n0, __shfl_xor_sync(0xffffffffu, n0, 2)));
                            n1 = fmaxf(m[1], fmaxf(n1, __shfl_xor_sync(0xffffffffu, n1, 2)));
                            const float c0 = ex2(m[0] - n0), c1 = ex2(m[1] - n1);
                            m[0] = n0;
                            m[1] = n1;
                            l[0] *= c0;
                            l[1] *= c1;
#pragma unroll
                            for (int j = 0; j < S::kNt; ++j) {
                                acc[j][0] *= c0;
                                acc[j][1] *= c0;
                                acc[j][2] *= c1;
                                acc[j][3] *= c1;
                            }
                        }
                    }
                    if (!careful) {
#pragma unroll
                        for (int x = 0; x < 2; ++x)
#pragma unroll
                            for (int e = 0; e < 4; ++e) s[x][e] = ex2(w[x][e] - m[e >> 1]);
                        l[0] = fmaf((s[0][0] + s[0][1]) + (s[1][0] + s[1][1]), sc.z, l[0]);
                        l[1] = fmaf((s[0][2] + s[0][3]) + (s[1][2] + s[1][3]), sc.z, l[1]);
                    }
                    const uint4 pf = make_uint4(pack_half(s[0][0], s[0][1]), pack_half(s[0][2], s[0][3]), pack_half(s[1][0], s[1][1]),
                                                pack_half(s[1][2], s[1][3]));
                    // ---- values: tokens 2c, 2c + 1, 2c + 8, 2c + 9, columns D / 8 * g ..
                    // (8 bytes at a time: 16 would be four more registers a token than there are)
#pragma unroll
                    for (int half = 0; half < D / 64; ++half) {
                        uint32_t v[4][2];
#pragma unroll
                        for (int x = 0; x < 4; ++x) {
                            const int t = 2 * c + (x & 1) + 8 * (x >> 1);
                            const uint2 r = D == 128 ? lds_v2(vt + ar_piece<D>(t, g) + half * 8) : lds_v2(vt + ar_piece<D>(t, g >> 1) + (g & 1) * 8);
                            v[x][0] = r.x ^ 0x80808080u;
                            v[x][1] = r.y ^ 0x80808080u;
                        }
#pragma unroll
                        for (int w = 0; w < 2; ++w) {
                            uint32_t b0[4], b1[4];
                            codes_to_half(__byte_perm(v[0][w], v[1][w], 0x5140), b0[0], b0[1]);
                            codes_to_half(__byte_perm(v[0][w], v[1][w], 0x7362), b0[2], b0[3]);
                            codes_to_half(__byte_perm(v[2][w], v[3][w], 0x5140), b1[0], b1[1]);
                            codes_to_half(__byte_perm(v[2][w], v[3][w], 0x7362), b1[2], b1[3]);
#pragma unroll
                            for (int j = 0; j < 4; ++j) mma_f16(acc[4 * (2 * half + w) + j], pf, b0[j], b1[j]);
                        }
                    }
                }
            }
            __syncwarp();
            if (lane == 0) ptx::mbar_arrive(&empty[stage]);
            if (++stage == S::kStages) {
                stage = 0;
                parity ^= 1u;
            }
        }
        n += steps;
        if (__any_sync(0xffffffffu, dead)) l[0] = l[1] = __uint_as_float(0x7fc00000u);

        // ---- the warps' sums, put together in their order: to a common m', then 2 + 2, then 1 + 1
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            // over the lanes of a row: the four of a g, or the eight of a c
#pragma unroll
            for (int o = R == 8 ? 4 : 1; o < (R == 8 ? 32 : 4); o <<= 1) l[x] += __shfl_xor_sync(0xffffffffu, l[x], o);
            if (R == 8 ? g == 0 : c == 0) {
                row_ml[warp][mine[x]] = make_float2(m[x], l[x]);
                if (row_ref[warp][mine[x]] == INFINITY) row_ref[warp][mine[x]] = m[x];
            }
        }
        ar_sync();
        float sum_l[2], ref[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            float top = kAtNothing;
            ref[x] = kAtNothing;
#pragma unroll
            for (int w = 0; w < kArWarps; ++w) {
                top = fmaxf(top, row_ml[w][mine[x]].x);
                ref[x] = fmaxf(ref[x], row_ref[w][mine[x]]);
            }
            sum_l[x] = 0.f;
#pragma unroll
            for (int w = 0; w < kArWarps; ++w) sum_l[x] += row_ml[w][mine[x]].y * ex2(row_ref[w][mine[x]] - ref[x]);
            const float k = ex2(m[x] - top);
            m[x] = top;
#pragma unroll
            for (int j = 0; j < S::kNt; ++j) {
                acc[j][R == 8 ? x : 2 * x] *= k;
                acc[j][R == 8 ? x + 2 : 2 * x + 1] *= k;
            }
        }
#pragma unroll
        for (int half = kArWarps / 2; half > 0; half >>= 1) {
            if (warp >= half && warp < 2 * half) {
#pragma unroll
                for (int j = 0; j < S::kNt; ++j)
                    ptx::st_shared_v4(joined + ((warp - half) * S::kNt + j) * 512,
                                      make_uint4(__float_as_uint(acc[j][0]), __float_as_uint(acc[j][1]), __float_as_uint(acc[j][2]), __float_as_uint(acc[j][3])));
            }
            ar_sync();
            if (warp < half) {
#pragma unroll
                for (int j = 0; j < S::kNt; ++j) {
                    const float4 o = ptx::ld_shared_v4(joined + (warp * S::kNt + j) * 512);
                    acc[j][0] += o.x;
                    acc[j][1] += o.y;
                    acc[j][2] += o.z;
                    acc[j][3] += o.w;
                }
            }
            if (half > 1) ar_sync();
        }
        const bool whole = first == 0 && steps == at.blocks;
        if (warp == 0) {
            // 16 rows: lane (g, c) has columns D / 4 * c .. of rows g, g + 8: column n-tile j, c0 / c1 = j / j + D / 8
            // 8 rows: columns D / 8 * g .. of rows 2c, 2c + 1: column 2j (+ 1) in c0, c1 (c2, c3) of tile j
            constexpr int kCols = R == 8 ? D / 8 : D / 4;
            auto value = [&](int x, int e) {
                if constexpr (R == 8) return acc[e / 2][2 * (e & 1) + x];
                else return acc[e % (D / 8)][2 * x + e / (D / 8)];
            };
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int r = mine[x], mr = at.tile * R + r, col = (R == 8 ? g : c) * kCols;
                if (mr >= rows) continue;
                const bool lead = R == 8 ? g == 0 : c == 0;
                if (whole) {
                    const bool nan = at.len < 0;
                    const float half = half_gap(m[x], ref[x]);
                    const float k = nan ? __uint_as_float(0x7fc00000u) : sum_l[x] == 0.f ? 0.f : 1.f / sum_l[x] * half;
                    const int j = mr / a.group;
                    const int64_t o = (int64_t)(at.row0 + j) * a.q_heads + at.head * a.group + (mr - j * a.group);
                    __nv_bfloat16 *to = a.out + o * D + col;
#pragma unroll
                    for (int e = 0; e < kCols; e += 8) {
                        uint4 w;
                        __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&w);
#pragma unroll
                        for (int z = 0; z < 4; ++z) h[z] = __floats2bfloat162_rn(value(x, e + 2 * z) * k * half, value(x, e + 2 * z + 1) * k * half);
                        *reinterpret_cast<uint4 *>(to + e) = w;
                    }
                    if (a.lse && lead) a.lse[o] = nan ? k : sum_l[x] == 0.f ? -INFINITY : (ref[x] + log2f(sum_l[x])) * kAtLn2;
                } else {
                    const int slot = 2 * blockIdx.x + (first == 0 ? 1 : 0);
                    float *to = part + ((int64_t)slot * kArRows + r) * D + col;
#pragma unroll
                    for (int e = 0; e < kCols; e += 4)
                        *reinterpret_cast<float4 *>(to + e) = make_float4(value(x, e), value(x, e + 1), value(x, e + 2), value(x, e + 3));
                    if (lead) part_ml[(int64_t)slot * kArRows + r] = make_float4(m[x], sum_l[x], ref[x], 0.f);
                }
            }
        }
        left -= steps;
        if (left == 0 && tid == 0 && !whole_tiles) {
            // a tile that begins here and goes on: the CTAs behind that have the rest of its blocks
            const int rest = at.blocks - steps;
            const bool goes_on = first == 0 && rest > 0;
            join[blockIdx.x] = goes_on ? make_int4(at.row0, at.head, at.tile * R | min(rows - at.tile * R, R) << 26,
                                                   1 + (rest + chunk - 1) / chunk)
                                       : make_int4(0, 0, 0, 0);
        }
        if (left > 0) at.next<R>(a, steps);
    }
}

// Puts the parts of tile (CTA blockIdx.x of the kernel above) together: a thread per row and four columns.
template <int D>
__global__ void __launch_bounds__(kArRows * D / 4)
attend_join_kernel(const __grid_constant__ AttendArgs a, const float *part, const float4 *part_ml, const int4 *join)
{
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    const int4 what = join[blockIdx.x];
    const int r = threadIdx.x / (D / 4), col = threadIdx.x % (D / 4) * 4;
    // the first two parts, which most joined tiles have and no more, are read beside the record that tells whether there are any: one trip to
    // L2 instead of three (what is read of a tile that has none is not used)
    const int next = min((int)blockIdx.x + 1, (int)gridDim.x - 1);
    const int64_t at0 = (int64_t)(2 * blockIdx.x + 1) * kArRows + r, at1 = (int64_t)(2 * next) * kArRows + r;
    const float4 ml0 = part_ml[at0], ml1 = part_ml[at1];
    const float4 x0 = *reinterpret_cast<const float4 *>(part + at0 * D + col), x1 = *reinterpret_cast<const float4 *>(part + at1 * D + col);
    if (what.w == 0 || r >= (int)((uint32_t)what.z >> 26)) return;
    // (nothing that the workspace says leads out of it, or below out of the outputs, whoever else should write there meanwhile)
    const int parts = min(what.w, (int)(gridDim.x - blockIdx.x));
    float top = fmaxf(ml0.x, ml1.x), ref = fmaxf(ml0.z, ml1.z);
    for (int p = 2; p < parts; ++p) {
        const float4 ml = part_ml[(int64_t)(2 * (blockIdx.x + p)) * kArRows + r];
        top = fmaxf(top, ml.x);
        ref = fmaxf(ref, ml.z);
    }
    const float k0 = ex2(ml0.x - top), k1 = ex2(ml1.x - top);
    float4 o = make_float4(fmaf(x1.x, k1, x0.x * k0), fmaf(x1.y, k1, x0.y * k0), fmaf(x1.z, k1, x0.z * k0), fmaf(x1.w, k1, x0.w * k0));
    float l = fmaf(ml1.y, ex2(ml1.z - ref), ml0.y * ex2(ml0.z - ref));
    for (int p = 2; p < parts; ++p) {
        const int64_t at = (int64_t)(2 * (blockIdx.x + p)) * kArRows + r;
        const float4 ml = part_ml[at];
        const float4 x = *reinterpret_cast<const float4 *>(part + at * D + col);
        const float k = ex2(ml.x - top);
        l = fmaf(ml.y, ex2(ml.z - ref), l);
        o.x = fmaf(x.x, k, o.x);
        o.y = fmaf(x.y, k, o.y);
        o.z = fmaf(x.z, k, o.z);
        o.w = fmaf(x.w, k, o.w);
    }
    const int m = (what.z & 0x3ffffff) + r, j = m / a.group;
    if (what.x < 0 || what.x >= a.rows - j || (uint32_t)what.y >= (uint32_t)a.c.kv_heads) return;
    const int64_t row = (int64_t)(what.x + j) * a.q_heads + what.y * a.group + (m - j * a.group);
    const float half = half_gap(top, ref), k = l == 0.f ? 0.f : 1.f / l * half;
    uint2 w;
    __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&w);
    h[0] = __floats2bfloat162_rn(o.x * k * half, o.y * k * half);
    h[1] = __floats2bfloat162_rn(o.z * k * half, o.w * k * half);
    *reinterpret_cast<uint2 *>(a.out + row * D + col) = w;
    if (a.lse && col == 0) a.lse[row] = l == 0.f ? -INFINITY : (ref + log2f(l)) * kAtLn2;
}

}  // namespace rtp
