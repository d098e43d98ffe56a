// The pages of the 8-bit cache: which page each new token goes to (rtprune_page_map), and the codes and scales that
// are written there (rtprune_cache_write).
#include <algorithm>
#include <atomic>

#include "serve.cuh"

namespace rtp {

// ---- page tables, slots, positions ----------------------------------------------------------------------------------
//
// Request i has c_i tokens in pages already and n_i = offsets[i+1] - offsets[i] new ones; it needs
// ceil((c_i + n_i) / ps) - ceil(c_i / ps) more pages, which come from the free list in the order of the requests: an
// exclusive prefix sum over the batch.  Every CTA takes that sum for itself (the lengths are 8 bytes a request, read
// from L2; a kernel of its own for the sum, or a look-back between CTAs, would cost another launch's latency), then maps
// its rows: a binary search in shared memory for the request of a thread's first row, its others follow.  What is
// written is a few bytes a row: the call is bound by a launch and three trips to L2 (lengths, table or list, stores):
// 4.3 us for a token each of 64 requests, 8.8 us for 1024 requests of 300 to 400 rows.
constexpr int kPmThreads = 256;
constexpr int kPmRows = 4;                   // rows of a thread, neighbours: 16-byte stores
constexpr int kPmMaxBatch = 16384;           // two words a request in shared memory

__global__ void __launch_bounds__(kPmThreads)
page_map_kernel(const int32_t *__restrict__ offsets, const int32_t *__restrict__ context_lens, int batch, int total_rows,
                const int32_t *__restrict__ token_index, const int32_t *__restrict__ position_base,
                const int32_t *__restrict__ free_pages, const int32_t *__restrict__ free_head, int n_free, int page_shift,
                int32_t *__restrict__ tables, int64_t table_stride, int max_pages, int32_t *__restrict__ slots,
                int32_t *__restrict__ positions, int32_t *__restrict__ seq_lens, int32_t *__restrict__ state)
{
    extern __shared__ int32_t sm[];
    int32_t *off = sm;                        // [batch + 1]
    int32_t *first = sm + batch + 1;          // [batch]: pages handed out before the request's first
    __shared__ int64_t warp_sum64[kPmThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int ps_1 = (1 << page_shift) - 1;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    const int head = __ldg(free_head);
    bool bad = false, wide = false;           // lengths outside the contract; a table row too short
    for (int i = tid; i < batch; i += kPmThreads) {
        const int lo = __ldg(offsets + i), hi = __ldg(offsets + i + 1), c = context_lens ? __ldg(context_lens + i) : 0;
        const int64_t end = (int64_t)c + hi - lo;
        const bool ok = lo >= 0 && hi >= lo && hi <= total_rows && c >= 0 && end <= INT32_MAX - ps_1;
        bad |= !ok;
        const int has = ok ? (c + ps_1) >> page_shift : 0, all = ok ? (int)((end + ps_1) >> page_shift) : 0;
        wide |= all > max_pages;
        off[i] = lo;
        if (i == batch - 1) off[batch] = hi;
        first[i] = all - has;
        if (blockIdx.x == 0) seq_lens[i] = ok ? (int)end : 0;
    }
    __syncthreads();
    // exclusive prefix sum: a run of neighbouring requests per thread, then the warps, then the CTA
    const int per = (batch + kPmThreads - 1) / kPmThreads, i0 = min(tid * per, batch), i1 = min(i0 + per, batch);
    int64_t mine = 0;
    for (int i = i0; i < i1; ++i) mine += first[i];
    int64_t upto = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int64_t t = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += t;
    }
    if (lane == 31) warp_sum64[warp] = upto;
    const int any_bad = __syncthreads_or(bad), any_wide = __syncthreads_or(wide);
    int64_t run = (int64_t)head + upto - mine, all_pages = 0;
#pragma unroll
    for (int w = 0; w < kPmThreads / 32; ++w) {
        if (w < warp) run += warp_sum64[w];
        all_pages += warp_sum64[w];
    }
    for (int i = i0; i < i1; ++i) {
        const int need = first[i];
        first[i] = (int)min(run, (int64_t)INT32_MAX);   // past the free list's end either way
        run += need;
    }
    if (blockIdx.x == 0 && tid == 0) {
        const int64_t next = (int64_t)head + all_pages;
        const bool short_list = head < 0 || next > n_free;
        state[0] = (int32_t)min(next, (int64_t)max(n_free, head));
        state[1] = (any_bad ? (int)RTPRUNE_DEV_BAD_OFFSETS : 0) | (any_wide || short_list ? (int)RTPRUNE_DEV_NO_PAGES : 0);
    }
    __syncthreads();
    const int row0 = ((int)blockIdx.x * kPmThreads + tid) * kPmRows;
    if (row0 >= total_rows) return;
    // the last request whose rows begin at or before row0 (its offset counts, an empty one's too: the walk below passes those)
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (off[mid] <= row0) lo = mid;
        else hi = mid;
    }
    int slot[kPmRows], pos[kPmRows], i = lo, ctx = 0, seen = -1;
#pragma unroll
    for (int r = 0; r < kPmRows; ++r) {
        const int row = row0 + r;
        while (i < batch - 1 && row >= off[i + 1]) ++i;
        slot[r] = pos[r] = -1;
        const int j = row - off[i];
        if (row >= total_rows || j < 0 || row >= off[i + 1] || off[i] < 0 || off[i + 1] > total_rows) continue;
        if (seen != i) ctx = context_lens ? __ldg(context_lens + i) : 0, seen = i;
        if (ctx < 0 || (int64_t)ctx + off[i + 1] - off[i] > INT32_MAX - ps_1) continue;
        const int x = ctx + j, p = x >> page_shift, has = (ctx + ps_1) >> page_shift;
        const int at = p < has ? -1 : min(first[i], INT32_MAX - p) + p - has;
        int page = -1;
        if (p < max_pages) {
            int32_t *entry = tables + (int64_t)i * table_stride + p;
            if (p < has) page = *entry;
            else if (at >= 0 && at < n_free) page = __ldg(free_pages + at);
            // a new page begins with a new token, which writes the table's entry
            if (p >= has && (x & ps_1) == 0) *entry = page;
        }
        const int64_t s = ((int64_t)page << page_shift) + (x & ps_1);
        if (page >= 0 && s <= INT32_MAX) slot[r] = (int)s;
        pos[r] = token_index ? (position_base ? __ldg(position_base + i) : ctx) + __ldg(token_index + row)
                             : position_base ? __ldg(position_base + i) + j : x;
    }
    if (row0 + kPmRows <= total_rows && (((uintptr_t)slots | (uintptr_t)positions) & 15u) == 0) {
        *reinterpret_cast<int4 *>(slots + row0) = make_int4(slot[0], slot[1], slot[2], slot[3]);
        if (positions) *reinterpret_cast<int4 *>(positions + row0) = make_int4(pos[0], pos[1], pos[2], pos[3]);
    } else {
#pragma unroll
        for (int r = 0; r < kPmRows; ++r)
            if (row0 + r < total_rows) {
                slots[row0 + r] = slot[r];
                if (positions) positions[row0 + r] = pos[r];
            }
    }
}

// Words of memory that a call reads or writes: `rows` runs of `words`, `stride` apart.
struct Words {
    const int32_t *p;
    int64_t words, rows = 1, stride = 0;
};
// Whether two pieces of memory share a byte (b: one run).
static bool overlap(const Words &a, const Words &b)
{
    if (!a.p || !b.p || a.words <= 0 || b.words <= 0 || a.rows <= 0) return false;
    const int64_t from = (int64_t)((intptr_t)b.p - (intptr_t)a.p), to = from + b.words * 4;      // b, in bytes from a's first
    const int64_t pitch = a.stride * 4, len = a.words * 4;
    if (to <= 0 || from >= (a.rows - 1) * pitch + len) return false;
    if (a.rows == 1) return true;
    // the run that b begins in (or the first), and the next
    const int64_t row = std::max<int64_t>(0, from / pitch);
    return from < row * pitch + len || (row + 1 < a.rows && to > (row + 1) * pitch);
}

// ---- codes and scales -----------------------------------------------------------------------------------------------
//
// A page is one block of tokens: each kv head of it has one scale for its keys and one for its values, the smallest
// power of two s with 127 s >= the largest |x| among the page's tokens, and codes rint(x / s).  A token appended to a
// page whose scale is too small makes it grow, and the page's earlier codes are taken to the new scale (a shift, rounded
// once).  Powers of two because a cache grows token by token: with s = max / 127 every new maximum of a page would round
// all its earlier codes again (about ln 64 = 4 times while 64 tokens arrive), with powers of two only a doubling does, the
// shift itself is exact, and no code hangs on how a division rounds.  The price is 64 to 127 levels instead of 127.
//
// A unit is (run, head, keys or values): the run are rows whose slots follow one another in one page, found from the
// slots alone (a row leads a run if it starts a page, or the row ahead is not its page's token before it).  A CTA
// takes the runs that begin in its window of rows, which it finds in one look at the slots (a bit per row that begins or ends
// something); its threads hold the run in registers between the maximum and the codes, so that it is read once.
// Bound by HBM: 2 or 4 bytes read and 1 written an element.  64 requests of 300 to 375 tokens, 10 heads of 128 in bf16: 33 us, 5.0 TB/s
// (several heads to a CTA, one after the other, 53.7 us; codes by conversion instructions 44.7).  In fp32, or with pages of 128, a run is longer than what
// its threads keep and is read twice: 64 x 337 tokens in fp32 68 us and, in pages of 128, 83; in bf16 33 and 44.
constexpr int kCwThreads = 128;
constexpr int kCwKeep = 8;                   // 16-byte vectors of a run that a thread keeps; longer runs are read twice
constexpr int kCwMaxWindow = 64;

// Smallest power of two s >= 2^-126 with 127 s >= top; 0 for 0, NaN for what is not finite.
__device__ inline float block_scale(float top)
{
    if (top == 0.f) return 0.f;
    const uint32_t b = __float_as_uint(top);
    const int e = (int)(b >> 23) - 127;                          // top = 2^e (1 + f), 127 / 128 = 2^-1 (1 + 126 / 128)
    if (!(top <= 3.4028235e38f)) return __uint_as_float(0x7fc00000u);
    const int up = e - 6 + ((b & 0x7fffffu) > 0x7e0000u ? 1 : 0);
    return __uint_as_float((uint32_t)(max(up, -126) + 127) << 23);
}

template <typename T> struct CodesOf;        // a 16-byte vector's codes
template <> struct CodesOf<__nv_bfloat16> {
    using Out = uint2;
};
template <> struct CodesOf<float> {
    using Out = uint32_t;
};

// Codes of four values of at most 127 s: x / s (inv = 1 / s, a power of two) added to 1.5 2^23 leaves the nearest whole number, ties to
// even, in the sum's last bits, in two's complement.
__device__ inline uint32_t codes4(float a, float b, float c, float d, float inv)
{
    constexpr float kRound = 12582912.f;
    const uint32_t i0 = __float_as_uint(fmaf(a, inv, kRound)), i1 = __float_as_uint(fmaf(b, inv, kRound));
    const uint32_t i2 = __float_as_uint(fmaf(c, inv, kRound)), i3 = __float_as_uint(fmaf(d, inv, kRound));
    return __byte_perm(__byte_perm(i0, i1, 0x0040), __byte_perm(i2, i3, 0x0040), 0x5410);
}
// Four codes at a scale, to another.
__device__ inline uint32_t shift4(uint32_t x, float shrink)
{
    return codes4((float)(int8_t)x, (float)(int8_t)(x >> 8), (float)(int8_t)(x >> 16), (float)(int8_t)(x >> 24), shrink);
}
// The largest |x| of a 16-byte vector, with what there was (NaN if there is one): in bf16 two at a time, on the bits.
template <typename T> struct Largest;
template <> struct Largest<__nv_bfloat16> {
    uint32_t m = 0u;
    __device__ static inline uint32_t max2(uint32_t a, uint32_t b)
    {
        uint32_t r;
        asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
        return r;
    }
    __device__ inline void take(const uint4 &v)
    {
        m = max2(m, max2(max2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), max2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
    }
    __device__ inline float value() const { return max_nan(__uint_as_float(m << 16), __uint_as_float(m & 0xffff0000u)); }
};
template <> struct Largest<float> {
    float m = 0.f;
    __device__ inline void take(const uint4 &v)
    {
        m = max_nan(m, max_nan(max_nan(fabsf(__uint_as_float(v.x)), fabsf(__uint_as_float(v.y))), max_nan(fabsf(__uint_as_float(v.z)), fabsf(__uint_as_float(v.w)))));
    }
    __device__ inline float value() const { return m; }
};

template <typename T>
__global__ void __launch_bounds__(kCwThreads, 8)
cache_write_kernel(const T *__restrict__ k, int64_t k_stride, const T *__restrict__ v, int64_t v_stride, int rows, int window,
                   const int32_t *__restrict__ slots, const __grid_constant__ CacheView c)
{
    constexpr int kVec = Elem<T>::kPerVec, kLook = (kCwMaxWindow + 128) / kCwThreads + 1;
    using Out = typename CodesOf<T>::Out;
    __shared__ uint32_t breaks[kLook * kCwThreads / 32], leads[kCwMaxWindow / 32];    // rows that do not follow the one ahead; those that lead a run
    __shared__ int32_t slot_of[kCwMaxWindow];
    __shared__ float red[2][kCwThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    // the heads of a window beside each other: what runs at a time reads whole rows
    const int units = 2 * c.kv_heads, unit = (int)(blockIdx.x % units);
    const int row0 = (int)(blockIdx.x / units) * window, ps = c.page_size;
    const int64_t n_slots = (int64_t)c.num_pages << c.page_shift;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    // a run that begins in the window ends, at the latest, a page behind it
    for (int i = tid; i < (window + ps + 31) / 32 * 32; i += kCwThreads) {
        const int r = row0 + i;
        const int s = r < rows ? __ldg(slots + r) : -1, ahead = r > 0 && r < rows ? __ldg(slots + r - 1) : -1;
        const bool valid = s >= 0 && s < n_slots, follows = valid && (s & (ps - 1)) != 0 && ahead == s - 1;
        const uint32_t brk = __ballot_sync(0xffffffffu, !follows), led = __ballot_sync(0xffffffffu, !follows && valid && i < window);
        if (lane == 0) breaks[i >> 5] = brk;
        if (lane == 0 && i < kCwMaxWindow) leads[i >> 5] = led;
        if (i < kCwMaxWindow) slot_of[i] = s;
    }
    __syncthreads();
    const int per_row = c.dim / kVec, row_step = kCwThreads / per_row;      // threads of a row; rows at a time
    const int my_row = tid / per_row, my_vec = tid - my_row * per_row;
    int turn = 0;
    const bool values = unit >= c.kv_heads;
    const int head = values ? unit - c.kv_heads : unit;
    const T *src = (values ? v : k) + (int64_t)head * c.dim;
    const int64_t stride = values ? v_stride : k_stride;
    int8_t *codes = values ? c.v : c.k;
    float *scales = values ? c.v_scale : c.k_scale;
#pragma unroll 1
    for (int word = 0; word * 32 < window; ++word)
#pragma unroll 1
        for (uint32_t left = leads[word]; left; left &= left - 1, turn ^= 1) {
            const int i = word * 32 + __ffs(left) - 1, slot0 = slot_of[i], at = slot0 & (ps - 1), page = slot0 >> c.page_shift;
            int next = (i + 1) >> 5;
            uint32_t bits = breaks[next] & (0xffffffffu << ((i + 1) & 31));
            while (!bits) bits = breaks[++next];                 // (there is one: where the page ends)
            const int len = next * 32 + __ffs(bits) - 1 - i;
            const T *from = src + (int64_t)(row0 + i + my_row) * stride + my_vec * kVec;
            const int64_t step = row_step * stride;
            float *scale = scales + (int64_t)page * c.kv_heads + head;
            uint4 held[kCwKeep];
#pragma unroll
            for (int t = 0; t < kCwKeep; ++t) {
                held[t] = make_uint4(0u, 0u, 0u, 0u);
                if (t * row_step + my_row < len) held[t] = __ldg(reinterpret_cast<const uint4 *>(from + t * step));
            }
            const float old = at ? *scale : 0.f;
            Largest<T> largest;
#pragma unroll
            for (int t = 0; t < kCwKeep; ++t) largest.take(held[t]);
            for (int r = kCwKeep * row_step + my_row; r < len; r += row_step)
                largest.take(__ldg(reinterpret_cast<const uint4 *>(from + (r - my_row) * stride)));
            float top = largest.value();
            top = warp_max_redux(top);
            if (lane == 0) red[turn][warp] = top;
            __syncthreads();
            top = max_nan(max_nan(red[turn][0], red[turn][1]), max_nan(red[turn][2], red[turn][3]));
            const float s = max_nan(block_scale(top), old);
            const float inv = s > 0.f ? 1.f / s : 0.f;            // (NaN: codes 0)
            int8_t *block = codes + ((int64_t)page * c.kv_heads + head) * ps * c.dim;
            if (at && s != old && s == s) {
                // the page's earlier codes, to the new scale
                const float shrink = old * inv;
                uint4 *p = reinterpret_cast<uint4 *>(block);
                for (int j = tid; j < at * c.dim / 16; j += kCwThreads) {
                    uint4 w = p[j];
                    w.x = shift4(w.x, shrink);
                    w.y = shift4(w.y, shrink);
                    w.z = shift4(w.z, shrink);
                    w.w = shift4(w.w, shrink);
                    p[j] = w;
                }
            }
            int8_t *to = block + (int64_t)(at + my_row) * c.dim + my_vec * kVec;
            auto put = [&](int r, const uint4 &x) {
                float f[kVec];
                Elem<T>::unpack(x, f);
                Out o;
                uint32_t *w = reinterpret_cast<uint32_t *>(&o);
#pragma unroll
                for (int e = 0; e < kVec; e += 4) w[e / 4] = inv > 0.f ? codes4(f[e], f[e + 1], f[e + 2], f[e + 3], inv) : 0u;
                *reinterpret_cast<Out *>(to + r * c.dim) = o;
            };
#pragma unroll
            for (int t = 0; t < kCwKeep; ++t)
                if (t * row_step + my_row < len) put(t * row_step, held[t]);
            for (int r = kCwKeep * row_step; r + my_row < len; r += row_step) put(r, __ldg(reinterpret_cast<const uint4 *>(from + (int64_t)r * stride)));
            // (every thread has its `old`: the barrier above lies between that and this; the next run has another page, and its maxima the other half
            // of `red`)
            if (tid == 0) *scale = s;
        }
}

template <typename T>
static cudaError_t launch_write(cudaStream_t st, const void *k, int64_t k_stride, const void *v, int64_t v_stride, int rows,
                                const int32_t *slots, const CacheView &c, int sms)
{
    // rows of a window: about twelve CTAs to an SM (eight run at a time), so that single tokens, each a run of its own, go side by
    // side, and long runs, of which a window of 64 rows starts one or two, do not launch CTAs that find none.  Windows of 1 row and of 64
    // against this rule, 10 heads of 128, in us: a token of 64 requests 4.8 / 60.2 / 4.8, of 256 13.4 / 58.7 / 12.0, five tokens of 64
    // 9.4 / 15.1 / 6.1, 300 tokens of 1 request 7.7 / 3.7 / 3.7, of 4 26.4 / 5.4 / 5.1, of 64 398 / 30.5 / 30.3
    const int64_t want = (int64_t)rows * 2 * c.kv_heads / ((int64_t)sms * 12);
    int window = 1;
    while (window < kCwMaxWindow && window < want) window *= 2;
    const int64_t ctas = (int64_t)((rows + window - 1) / window) * 2 * c.kv_heads;
    if (ctas > INT32_MAX) return cudaErrorInvalidConfiguration;
    const dim3 grid((unsigned)ctas);
    return launch_chained(cache_write_kernel<T>, grid, dim3(kCwThreads), (size_t)0, st, (const T *)k, k_stride, (const T *)v, v_stride,
                          rows, window, slots, c);
}

}  // namespace rtp

extern "C" rtprune_status_t rtprune_page_map(void *cuda_stream, const int32_t *offsets, const int32_t *context_lens, int32_t batch,
                                             int64_t total_rows, const int32_t *token_index, const int32_t *position_base,
                                             const int32_t *free_pages, const int32_t *free_head, int32_t n_free,
                                             int32_t page_size, int32_t *block_tables, int64_t table_stride, int32_t max_pages,
                                             int32_t *slot_map, int32_t *positions, int32_t *seq_lens, int32_t *state)
{
    using namespace rtp;
    if (batch < 0 || total_rows < 0 || n_free < 0 || max_pages < 0 || table_stride < max_pages) return RTPRUNE_ERR_INVALID_ARG;
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) return RTPRUNE_ERR_UNSUPPORTED;
    if (batch > kPmMaxBatch || total_rows > INT32_MAX - kPmThreads * kPmRows) return RTPRUNE_ERR_UNSUPPORTED;
    if (batch == 0) return total_rows == 0 ? RTPRUNE_OK : RTPRUNE_ERR_INVALID_ARG;
    if (!offsets || !free_head || !seq_lens || !state || (!free_pages && n_free) || (!block_tables && max_pages) ||
        (!slot_map && total_rows))
        return RTPRUNE_ERR_INVALID_ARG;
    // every CTA reads the lengths, the lists and the head, whichever wrote its part of the outputs before
    const Words in[] = {{offsets, batch + 1}, {context_lens, batch}, {position_base, batch}, {token_index, total_rows}, {free_pages, n_free}, {free_head, 1}};
    const Words out[] = {{block_tables, max_pages, batch, table_stride}, {slot_map, total_rows}, {positions, total_rows}, {seq_lens, batch}, {state, 2}};
    for (int o = 0; o < 5; ++o) {
        for (const Words &i : in)
            if (overlap(out[o], i)) return RTPRUNE_ERR_INVALID_ARG;
        for (int other = o + 1; other < 5; ++other)
            if (overlap(out[o], out[other])) return RTPRUNE_ERR_INVALID_ARG;
    }
    int shift = 4;
    while ((1 << shift) < page_size) ++shift;
    const int64_t per_cta = kPmThreads * kPmRows;
    const size_t smem = (size_t)(2 * batch + 1) * 4;
    if (smem > 40 * 1024) {                  // (the kernel's own few bytes count towards the 48 KB too)
        if (cudaFuncSetAttribute(page_map_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (2 * kPmMaxBatch + 1) * 4) != cudaSuccess)
            return RTPRUNE_ERR_CUDA;
    }
    const dim3 grid((unsigned)std::max<int64_t>(1, (total_rows + per_cta - 1) / per_cta));
    if (launch_chained(page_map_kernel, grid, dim3(kPmThreads), smem, (cudaStream_t)cuda_stream, offsets, context_lens, batch,
                       (int)total_rows, token_index, position_base, free_pages, free_head, n_free, shift, block_tables, table_stride,
                       max_pages, slot_map, positions, seq_lens, state) != cudaSuccess)
        return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}

extern "C" rtprune_status_t rtprune_cache_write(void *cuda_stream, rtprune_dtype_t dtype, const void *k, int64_t k_stride,
                                                const void *v, int64_t v_stride, int64_t rows, const int32_t *slot_map,
                                                const rtprune_cache_t *cache)
{
    using namespace rtp;
    CacheView c;
    rtprune_status_t status;
    if (rows < 0 || (dtype != RTPRUNE_BF16 && dtype != RTPRUNE_FP32)) return RTPRUNE_ERR_INVALID_ARG;
    if (!cache_view(cache, c, status)) return status;
    const int64_t width = (int64_t)c.kv_heads * c.dim, vec = dtype == RTPRUNE_BF16 ? 8 : 4;
    if (rows == 0) return RTPRUNE_OK;
    if (!k || !v || !slot_map || k_stride < width || v_stride < width || k_stride % vec || v_stride % vec ||
        ((uintptr_t)k | (uintptr_t)v) & 15u)
        return RTPRUNE_ERR_INVALID_ARG;
    if (rows > INT32_MAX - 4 * kCwMaxWindow) return RTPRUNE_ERR_UNSUPPORTED;     // (a CTA looks a window and a page ahead)
    const int sms = device_sms();
    if (!sms) return RTPRUNE_ERR_CUDA;
    cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = dtype == RTPRUNE_BF16 ? launch_write<__nv_bfloat16>(st, k, k_stride, v, v_stride, (int)rows, slot_map, c, sms)
                                                : launch_write<float>(st, k, k_stride, v, v_stride, (int)rows, slot_map, c, sms);
    if (e != cudaSuccess) return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}
