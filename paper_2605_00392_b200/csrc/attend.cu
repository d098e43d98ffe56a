// Attention over the 8-bit paged cache (rtprune_cache_attend).
#include <algorithm>
#include <atomic>
#include <cmath>

#include "attend.cuh"
#include "attend_rows.cuh"
#include "attend_tiles.cuh"

namespace rtp {

constexpr int kAtFewRows = 32, kAtFewTiles = 296;

// Whether attend_rows_kernel takes the call: few rows of a kv head, so few tiles of 16 rows in the whole call that it has them all in one
// go, two to an SM, where attend_tiles_kernel's of 256 rows leave most SMs without any, or more heads of a kv head than a tile has rows.
// Rows against tiles, heads of 128, in us.  64 requests behind 1000 tokens, 10 heads: of 16 rows 54 / 97, 32 rows 95 / 97, 48 rows
// 132 / 98, 128 rows 329 / 108; 16 requests behind 16000, 8 heads of 4: 32 rows 257 / 234, 64 rows 500 / 239.  Few tiles, 10 heads:
// 220 (one image of 337 tokens) 11.1 / 13.2, 440 (two) 19.6 / 12.8, 320 (8 x 64 rows behind 1000) 33 / 26, 160 (2 x 128 behind 4000)
// 50 / 70, 80 (128 behind 16000) 85 / 236.
static bool few_rows(int64_t batch, int64_t max_q_len, int64_t kv_heads, int group)
{
    const int64_t rows = max_q_len * group;
    return rows <= kAtFewRows || batch * kv_heads * ((rows + 15) / 16) <= kAtFewTiles || group > kTlRows;
}

// Workspace of attend_rows_kernel with `ctas` CTAs.
struct RowsLayout {
    size_t part, part_ml, join, total;
};
static RowsLayout rows_layout(int ctas, int dim)
{
    RowsLayout w;
    w.part = 0;
    w.part_ml = w.part + (size_t)2 * ctas * kArRows * dim * 4;
    w.join = w.part_ml + (size_t)2 * ctas * kArRows * 16;
    w.total = w.join + (size_t)ctas * 16;
    return w;
}

// The kernel's dynamic shared memory, set once on each device (a bit of the mask).
template <typename K> static cudaError_t allow_smem(K kernel, int bytes, std::atomic<unsigned long long> &ready)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess || (dev < 64 && (ready.load(std::memory_order_relaxed) >> dev & 1))) return e;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && dev < 64) ready.fetch_or(1ull << dev, std::memory_order_relaxed);
    return e;
}

// A tensor of rows of `dims` elements for TMA, boxes of `box`; at most three dimensions.
static bool tensor_map(CUtensorMap *map, CUtensorMapDataType type, const void *base, int rank, const cuuint64_t *dims, const cuuint64_t *strides,
                       const cuuint32_t *box, CUtensorMapSwizzle swizzle)
{
    typedef CUresult (*EncodeTiledFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *,
                                      const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                                      CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
    static std::atomic<void *> encode{nullptr};       // the driver's entry point, looked up once
    void *fn = encode.load(std::memory_order_relaxed);
    if (!fn) {
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &fn, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return false;
        encode.store(fn, std::memory_order_relaxed);
    }
    const cuuint32_t unit[3] = {1, 1, 1};
    return ((EncodeTiledFn)fn)(map, type, (cuuint32_t)rank, const_cast<void *>(base), dims, strides, box, unit, CU_TENSOR_MAP_INTERLEAVE_NONE,
                               swizzle, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// The queries (element, head, row); boxes of 64 elements of `heads` heads of `tokens` rows.
static bool queries_map(CUtensorMap *map, const AttendArgs &a, int heads, int tokens)
{
    const cuuint64_t dims[3] = {(cuuint64_t)a.c.dim, (cuuint64_t)a.q_heads, (cuuint64_t)a.rows};
    const cuuint64_t strides[2] = {(cuuint64_t)a.c.dim * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)heads, (cuuint32_t)tokens};
    return tensor_map(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.q, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int D, int R>
static cudaError_t launch_rows(const AttendArgs &a, uint8_t *ws, cudaStream_t st)
{
    const int ctas = std::min(ArShape<D, R>::kPerSm * device_sms(), kArMostCtas);
    if (!ctas) return cudaErrorInvalidDevice;
    const RowsLayout w = rows_layout(ctas, D);
    // every tile a CTA of its own, and a second kernel saved, where there are CTAs enough for as many as there can be and the longest is short.
    // 10 heads, one token for one request of 256 tokens 7.2 us against 8.7 cut and joined, for one of 500 10.8 against 9.1 on the GPU but 13.8
    // against 16.1 a call from the host, for 44 of 101 to 500 13.6 against 16.9; for one of 1001 17.9 against 10.2.
    const int64_t tiles = (int64_t)a.batch * a.c.kv_heads * (((int64_t)std::min(a.max_q_len, a.rows) * a.group + R - 1) / R);
    const bool whole = tiles <= ctas && a.max_len <= kArWhole * kArBlock;
    static std::atomic<unsigned long long> ready{0};             // devices that know the kernel's shared memory
    cudaError_t e = allow_smem(attend_rows_kernel<D, R>, ArShape<D, R>::kSmem, ready);
    if (e != cudaSuccess) return e;
    e = launch_chained(attend_rows_kernel<D, R>, dim3(whole ? (unsigned)tiles : (unsigned)ctas), dim3(kArThreads), (size_t)ArShape<D, R>::kSmem, st, a,
                       whole ? 1 : 0, (float *)(ws + w.part),
                       (float4 *)(ws + w.part_ml), (int4 *)(ws + w.join));
    if (e != cudaSuccess || whole) return e;
    return launch_chained(attend_join_kernel<D>, dim3(ctas), dim3(kArRows * D / 4), (size_t)0, st, a, (const float *)(ws + w.part),
                          (const float4 *)(ws + w.part_ml), (const int4 *)(ws + w.join));
}

// Items of the longest request that the call can have (it has no more rows than there are).
static int64_t tile_row_blocks(const AttendArgs &a)
{
    const int tokens = kTlTiles * (kTlRows / a.group);
    return (std::min(a.max_q_len, a.rows) + tokens - 1) / tokens;
}

template <int D>
static cudaError_t launch_tiles(const AttendArgs &a, cudaStream_t st)
{
    static std::atomic<unsigned long long> ready{0};
    const cudaError_t e = allow_smem(attend_tiles_kernel<D>, TlShape<D>::kSmem, ready);
    if (e != cudaSuccess) return e;
    const int sms = device_sms(), tokens = kTlRows / a.group;
    CUtensorMap map;
    if (!sms || !queries_map(&map, a, a.group, tokens)) return cudaErrorUnknown;
    const int64_t blocks = tile_row_blocks(a), items = blocks * a.batch * a.c.kv_heads;
    return launch_chained(attend_tiles_kernel<D>, dim3((unsigned)std::min<int64_t>(items, sms)), dim3(kTlThreads), (size_t)TlShape<D>::kSmem, st,
                          a, map, (int)blocks, tokens);
}

}  // namespace rtp

extern "C" rtprune_status_t rtprune_cache_attend_workspace(int32_t batch, int32_t max_q_len, int64_t max_seq_len, int32_t q_heads,
                                                           int32_t kv_heads, int32_t head_dim, size_t *workspace_bytes)
{
    if (!workspace_bytes || batch < 0 || max_q_len < 0 || max_seq_len < 0 || q_heads <= 0 || kv_heads <= 0 || head_dim <= 0)
        return RTPRUNE_ERR_INVALID_ARG;
    *workspace_bytes = 256;
    if (rtp::few_rows(batch, max_q_len, kv_heads, q_heads / kv_heads))
        *workspace_bytes = rtp::rows_layout(rtp::kArMostCtas, head_dim).total;
    return RTPRUNE_OK;
}

namespace rtp {

// rtprune_cache_attend; polls: after which its waits give up, -1: as many as the call's sizes ask.
static rtprune_status_t cache_attend(void *cuda_stream, const void *q, int64_t q_stride, int64_t rows, int32_t q_heads, const int32_t *offsets,
                                     const int32_t *seq_lens, int32_t batch, int32_t max_q_len, int64_t max_seq_len,
                                     const int32_t *block_tables, int64_t table_stride, int32_t max_pages, const rtprune_cache_t *cache,
                                     float scale, int32_t causal, void *out, float *lse, void *workspace, size_t workspace_bytes, int32_t polls)
{
    CacheView c;
    rtprune_status_t status;
    if (rows < 0 || batch < 0 || max_q_len < 0 || max_seq_len < 0 || q_heads <= 0 || max_pages < 0 || table_stride < max_pages ||
        !std::isfinite(scale))
        return RTPRUNE_ERR_INVALID_ARG;
    if (!cache_view(cache, c, status)) return status;
    if (q_heads % c.kv_heads || max_seq_len > (int64_t)max_pages * c.page_size) return RTPRUNE_ERR_INVALID_ARG;
    if (rows > INT32_MAX / 2 || max_seq_len > INT32_MAX / 2 || batch > 65535 || q_heads > 4096 ||
        rows * q_heads > INT32_MAX)
        return RTPRUNE_ERR_UNSUPPORTED;
    if (rows == 0 || batch == 0 || max_q_len == 0) return RTPRUNE_OK;
    if (!q || !offsets || !seq_lens || (!block_tables && max_pages) || !out || q_stride < (int64_t)q_heads * c.dim || q_stride % 8 ||
        ((uintptr_t)q & 15u) || ((uintptr_t)out & 31u))
        return RTPRUNE_ERR_INVALID_ARG;
    size_t need = 0;
    status = rtprune_cache_attend_workspace(batch, max_q_len, max_seq_len, q_heads, c.kv_heads, c.dim, &need);
    if (status != RTPRUNE_OK) return status;
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)) return RTPRUNE_ERR_WORKSPACE;
    AttendArgs a = {(const __nv_bfloat16 *)q, q_stride, offsets, seq_lens, block_tables, table_stride, batch, (int)rows, q_heads,
                    q_heads / c.kv_heads, max_q_len, (int)max_seq_len, max_pages, c, scale * 1.4426950408889634f, causal ? 1 : 0,
                    (__nv_bfloat16 *)out, lse, 0};
    if (few_rows(batch, max_q_len, c.kv_heads, a.group)) {
        // a tile's first row has 26 bits of a word, and a CTA's blocks (of half a 148th of the line, and fewer) an int
        const int64_t most = std::min<int64_t>(max_q_len, rows) * a.group, tiles = (most + 7) / 8 * batch * c.kv_heads;
        if (most >= 1 << 26 || tiles * (max_seq_len / kArBlock + 1) / 64 > INT32_MAX) return RTPRUNE_ERR_UNSUPPORTED;
        // a wait lasts as long as the fetching warp looks for the next request that has rows, at most (a thousand cycles for 32 of them)
        a.polls = polls >= 0 ? (uint32_t)polls : ptx::kSpinLimit + 32u * (uint32_t)batch;
        uint8_t *ws = (uint8_t *)workspace;
        cudaStream_t st = (cudaStream_t)cuda_stream;
        // tiles of 8 rows where a request has no more: 64 steps 37 us against 52 with 16, 16 long ones of 4 heads 122 against 162 (at 32 rows of
        // a kv head, 16 requests behind 16000 tokens, 360 against 257)
        const bool eight = (int64_t)max_q_len * a.group <= 8;
        const cudaError_t e = c.dim == 128 ? eight ? launch_rows<128, 8>(a, ws, st) : launch_rows<128, 16>(a, ws, st)
                                           : eight ? launch_rows<64, 8>(a, ws, st) : launch_rows<64, 16>(a, ws, st);
        if (e != cudaSuccess) return RTPRUNE_ERR_CUDA;
        return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
    }
    if (tile_row_blocks(a) * batch * c.kv_heads > INT32_MAX / 2) return RTPRUNE_ERR_UNSUPPORTED;
    // waits last as long as the items that are ahead, at most (five of them, some 7000 cycles a block each), and the search for the next one (a
    // thousand cycles for 32 numbers); a poll is 20 cycles or more
    a.polls = (uint32_t)polls;
    if (polls < 0)
        a.polls = ptx::kSpinLimit + 4096u * (uint32_t)std::min<int64_t>(max_seq_len / kTlBlock + 1, 1 << 19) +
                  16u * (uint32_t)(tile_row_blocks(a) * batch * c.kv_heads / std::max(device_sms(), 1) + 1);
    const cudaError_t e = c.dim == 128 ? launch_tiles<128>(a, (cudaStream_t)cuda_stream) : launch_tiles<64>(a, (cudaStream_t)cuda_stream);
    if (e != cudaSuccess)
        return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}

}  // namespace rtp

extern "C" rtprune_status_t rtprune_cache_attend(void *cuda_stream, const void *q, int64_t q_stride, int64_t rows, int32_t q_heads,
                                                 const int32_t *offsets, const int32_t *seq_lens, int32_t batch, int32_t max_q_len,
                                                 int64_t max_seq_len, const int32_t *block_tables, int64_t table_stride,
                                                 int32_t max_pages, const rtprune_cache_t *cache, float scale, int32_t causal,
                                                 void *out, float *lse, void *workspace, size_t workspace_bytes)
{
    return rtp::cache_attend(cuda_stream, q, q_stride, rows, q_heads, offsets, seq_lens, batch, max_q_len, max_seq_len, block_tables, table_stride,
                             max_pages, cache, scale, causal, out, lse, workspace, workspace_bytes, -1);
}

extern "C" rtprune_status_t rtprune_test_cache_attend_expired(void *cuda_stream, const void *q, int64_t q_stride, int64_t rows, int32_t q_heads,
                                                              const int32_t *offsets, const int32_t *seq_lens, int32_t batch,
                                                              int32_t max_q_len, int64_t max_seq_len, const int32_t *block_tables,
                                                              int64_t table_stride, int32_t max_pages, const rtprune_cache_t *cache,
                                                              float scale, int32_t causal, void *out, float *lse, void *workspace,
                                                              size_t workspace_bytes, int32_t polls)
{
    return rtp::cache_attend(cuda_stream, q, q_stride, rows, q_heads, offsets, seq_lens, batch, max_q_len, max_seq_len, block_tables, table_stride,
                             max_pages, cache, scale, causal, out, lse, workspace, workspace_bytes, std::max(polls, 0));
}
