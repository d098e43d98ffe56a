// Attention over the 8-bit paged cache (rtprune_cache_attend).
#include <algorithm>
#include <cmath>

#include "serve.cuh"

namespace rtp {

// Row r of request i, its j-th of n_i, sees the cached tokens t < end: L_i, or L_i - n_i + j + 1 when causal.
//   s_t = scale * ks * (q . kc_t),  out = sum_t softmax(s)_t vs vc_t,  lse = log sum_t exp s_t
// with kc, vc the codes of token t and ks, vs the scales of its page and head.
struct AttendArgs {
    const __nv_bfloat16 *q;
    int64_t q_stride;
    const int32_t *offsets, *seq_lens, *tables;
    int64_t table_stride;
    int32_t batch, rows, q_heads, group, max_q_len, max_len, max_pages;
    CacheView c;
    float scale_log2;                        // scale * log2(e): the softmax runs in powers of two
    int32_t causal;
    __nv_bfloat16 *out;
    float *lse;
};

// A request's rows and lengths, checked.  false: no rows of it can be written.  `len` < 0: outside the contract, its rows come out NaN.
__device__ inline bool attend_request(const AttendArgs &a, int i, int &row0, int &n, int &len)
{
    row0 = __ldg(a.offsets + i);
    const int hi = __ldg(a.offsets + i + 1);
    n = hi - row0;
    len = __ldg(a.seq_lens + i);
    if (row0 < 0 || n <= 0 || hi > a.rows || n > a.max_q_len) return false;
    if (len < 0 || len > a.max_len) len = -1;
    return true;
}

// The page of token t, or -1.
__device__ inline int attend_page(const AttendArgs &a, int i, int t)
{
    const int p = t >> a.c.page_shift;
    const int page = p < a.max_pages ? __ldg(a.tables + (int64_t)i * a.table_stride + p) : -1;
    return page < a.c.num_pages ? page : -1;
}

constexpr int kAtWarps = 4;

// A warp per (row, head), one token after the other.
__global__ void __launch_bounds__(32 * kAtWarps)
attend_simple_kernel(const __grid_constant__ AttendArgs a)
{
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, per = a.c.dim / 32;
    const int i = blockIdx.z, head = blockIdx.y, j = (int)blockIdx.x * kAtWarps + warp;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    int row0, n, len;
    if (!attend_request(a, i, row0, n, len) || j >= n) return;
    const int64_t row = row0 + j;
    const __nv_bfloat16 *qp = a.q + row * a.q_stride + (int64_t)head * a.c.dim + lane * per;
    float q[4] = {}, acc[4] = {}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < per; ++e) q[e] = __bfloat162float(qp[e]) * a.scale_log2;
    const int end = len < 0 ? 0 : a.causal ? min(len, len - n + j + 1) : len;
    const int kvh = head / a.group;
    bool nan = len < 0;
    for (int t = 0; t < end; ++t) {
        const int page = attend_page(a, i, t);
        if (page < 0) {
            nan = true;
            break;
        }
        const int64_t block = (int64_t)page * a.c.kv_heads + kvh;
        const int64_t at = (block * a.c.page_size + (t & (a.c.page_size - 1))) * a.c.dim + lane * per;
        float s = 0.f;
        for (int e = 0; e < per; ++e) s += q[e] * (float)a.c.k[at + e];
        s = warp_sum(s) * __ldg(a.c.k_scale + block);
        const float top = max_nan(m, s), keep = exp2f(m - top), p = exp2f(s - top);
        l = l * keep + p;
        const float pv = p * __ldg(a.c.v_scale + block);
        for (int e = 0; e < per; ++e) acc[e] = acc[e] * keep + pv * (float)a.c.v[at + e];
        m = top;
    }
    const float inv = nan ? __uint_as_float(0x7fc00000u) : end > 0 ? 1.f / l : 0.f;
    __nv_bfloat16 *o = a.out + (row * a.q_heads + head) * a.c.dim + lane * per;
    for (int e = 0; e < per; ++e) o[e] = __float2bfloat16_rn(acc[e] * inv);
    if (a.lse && lane == 0)
        a.lse[row * a.q_heads + head] = nan ? inv : end > 0 ? (m + log2f(l)) * 0.69314718055994531f : -INFINITY;
}

}  // namespace rtp

extern "C" rtprune_status_t rtprune_cache_attend_workspace(int32_t batch, int32_t max_q_len, int64_t max_seq_len, int32_t q_heads,
                                                           int32_t kv_heads, int32_t head_dim, size_t *workspace_bytes)
{
    if (!workspace_bytes || batch < 0 || max_q_len < 0 || max_seq_len < 0 || q_heads <= 0 || kv_heads <= 0 || head_dim <= 0)
        return RTPRUNE_ERR_INVALID_ARG;
    *workspace_bytes = 256;
    return RTPRUNE_OK;
}

extern "C" rtprune_status_t rtprune_cache_attend(void *cuda_stream, const void *q, int64_t q_stride, int64_t rows, int32_t q_heads,
                                                 const int32_t *offsets, const int32_t *seq_lens, int32_t batch, int32_t max_q_len,
                                                 int64_t max_seq_len, const int32_t *block_tables, int64_t table_stride,
                                                 int32_t max_pages, const rtprune_cache_t *cache, float scale, int32_t causal,
                                                 void *out, float *lse, void *workspace, size_t workspace_bytes)
{
    using namespace rtp;
    CacheView c;
    rtprune_status_t status;
    if (rows < 0 || batch < 0 || max_q_len < 0 || max_seq_len < 0 || q_heads <= 0 || max_pages < 0 || table_stride < max_pages ||
        !std::isfinite(scale))
        return RTPRUNE_ERR_INVALID_ARG;
    if (!cache_view(cache, c, status)) return status;
    if (q_heads % c.kv_heads || max_seq_len > (int64_t)max_pages * c.page_size) return RTPRUNE_ERR_INVALID_ARG;
    if (rows > INT32_MAX || max_seq_len > INT32_MAX / 2 || batch > 65535 || q_heads > 4096) return RTPRUNE_ERR_UNSUPPORTED;
    if (rows == 0 || batch == 0 || max_q_len == 0) return RTPRUNE_OK;
    if (!q || !offsets || !seq_lens || (!block_tables && max_pages) || !out || q_stride < (int64_t)q_heads * c.dim || q_stride % 8 ||
        (((uintptr_t)q | (uintptr_t)out) & 15u))
        return RTPRUNE_ERR_INVALID_ARG;
    size_t need = 0;
    status = rtprune_cache_attend_workspace(batch, max_q_len, max_seq_len, q_heads, c.kv_heads, c.dim, &need);
    if (status != RTPRUNE_OK) return status;
    if (!workspace || workspace_bytes < need || ((uintptr_t)workspace & 255u)) return RTPRUNE_ERR_WORKSPACE;
    AttendArgs a = {(const __nv_bfloat16 *)q, q_stride, offsets, seq_lens, block_tables, table_stride, batch, (int)rows, q_heads,
                    q_heads / c.kv_heads, max_q_len, (int)max_seq_len, max_pages, c, scale * 1.4426950408889634f, causal ? 1 : 0,
                    (__nv_bfloat16 *)out, lse};
    const dim3 grid((unsigned)((max_q_len + kAtWarps - 1) / kAtWarps), (unsigned)q_heads, (unsigned)batch);
    if (launch_chained(attend_simple_kernel, grid, dim3(32 * kAtWarps), (size_t)0, (cudaStream_t)cuda_stream, a) != cudaSuccess)
        return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}
