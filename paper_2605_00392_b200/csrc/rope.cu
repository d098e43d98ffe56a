// Norms of queries and keys per head and the rotation by position, in one pass (rtprune_qk_norm_rope).
#include <algorithm>

#include "serve.cuh"

namespace rtp {

// y = x w / sqrt(mean x^2 + eps) over a head's elements (no weights: y = x), then the first `rotary` of them in pairs
// (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin) by the angle pos f_p.
//
// A thread holds the two elements of each of its pairs: 16 bytes of first and 16 of second elements (half-split pairs:
// half a rotated part apart; adjacent pairs: 32 bytes in a row), so that the rotation needs no exchange and the norm one
// sum over the D / 16 (fp32: D / 8) threads of a head.  A CTA takes a few rows with all their heads: their angles' cosines and sines are
// computed once, into shared memory.  Angles in 64 bits, taken modulo a turn before they are rounded to 32: at position 10^6 an fp32
// angle would be off by 0.03.  Everything else in fp32, rounded once, at the store.
// Bound by HBM: each element read and written once.
constexpr int kRpThreads = 256;
constexpr int kRpMaxRows = 8;                // rows of a CTA
constexpr int kRpAhead = 4;                  // units of a thread whose loads are in flight together

template <typename T> __device__ inline uint4 pack_vec(const float (&f)[Elem<T>::kPerVec]);
template <> __device__ inline uint4 pack_vec<__nv_bfloat16>(const float (&f)[8])
{
    uint4 v;
    __nv_bfloat162 *h = reinterpret_cast<__nv_bfloat162 *>(&v);
#pragma unroll
    for (int i = 0; i < 4; ++i) h[i] = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
    return v;
}
template <> __device__ inline uint4 pack_vec<float>(const float (&f)[4])
{
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

struct RopeArgs {
    const void *q, *k, *q_weight, *k_weight;
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int32_t *positions;
    const double *inv_freq;
    int rows, rows_per_cta, q_heads, heads, dim, rotary, interleaved, group_shift;   // a head: 1 << group_shift threads
    float eps;
};

template <typename T>
__global__ void __launch_bounds__(kRpThreads)
qk_norm_rope_kernel(const __grid_constant__ RopeArgs a)
{
    constexpr int kVec = Elem<T>::kPerVec;
    __shared__ float2 turn[kRpMaxRows * 128];                    // cos, sin of each row's angles (rotary <= 256)
    __shared__ int pos[kRpMaxRows];
    const int tid = threadIdx.x, half = a.rotary / 2;
    const int row0 = (int)blockIdx.x * a.rows_per_cta, n = min(a.rows_per_cta, a.rows - row0);
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    if (tid < n) pos[tid] = __ldg(a.positions + row0 + tid);
    for (int i = tid; i < n * half; i += kRpThreads) {
        const int r = i / half, f = i - r * half;
        const double turns = (double)__ldg(a.positions + row0 + r) * __ldg(a.inv_freq + f) * 0.15915494309189533577;
        float s, c;
        sincospif(2.f * (float)(turns - rint(turns)), &s, &c);
        turn[i] = make_float2(c, s);
    }
    __syncthreads();
    // unit = (row, head, thread of the head); heads are queries' first, then keys'
    const int per_head = a.dim / (2 * kVec);                     // threads of a head that hold something
    const int group = 1 << a.group_shift, units = n * a.heads << a.group_shift;
    const int at = tid & (group - 1);                            // the same for all units of a thread
    // first and second elements of this thread's pairs: rotated ones, then those that pass through, in the same way
    int lo, hi;
    const int p0 = at * kVec;
    const bool turned = p0 < half;
    if (a.interleaved) lo = 2 * p0, hi = lo + kVec;
    else if (turned) lo = p0, hi = lo + half;
    else lo = half + p0, hi = lo + (a.dim - a.rotary) / 2;
    const bool holds = at < per_head;
    for (int base = 0; base < units; base += kRpThreads * kRpAhead) {
        const int u0 = base + tid;
        uint4 x[kRpAhead], y[kRpAhead];
#pragma unroll
        for (int t = 0; t < kRpAhead; ++t) {
            const int h = (u0 + t * kRpThreads) >> a.group_shift, r = h / a.heads, hd = h - r * a.heads;
            x[t] = y[t] = make_uint4(0u, 0u, 0u, 0u);
            if (u0 + t * kRpThreads < units && holds && pos[r] >= 0) {
                const T *p = hd < a.q_heads ? (const T *)a.q + (row0 + r) * a.q_stride + hd * a.dim
                                            : (const T *)a.k + (row0 + r) * a.k_stride + (hd - a.q_heads) * a.dim;
                x[t] = *reinterpret_cast<const uint4 *>(p + lo);
                y[t] = *reinterpret_cast<const uint4 *>(p + hi);
            }
        }
#pragma unroll
        for (int t = 0; t < kRpAhead; ++t) {
            if (base + t * kRpThreads >= units) break;           // the same for the whole CTA
            const int u = u0 + t * kRpThreads, h = u >> a.group_shift, r = h / a.heads, hd = h - r * a.heads;
            float f[kVec], g[kVec];
            Elem<T>::unpack(x[t], f);
            Elem<T>::unpack(y[t], g);
            const T *w = (const T *)(hd < a.q_heads ? a.q_weight : a.k_weight);
            if (a.q_weight || a.k_weight) {
                float sum = 0.f;
#pragma unroll
                for (int e = 0; e < kVec; ++e) sum += f[e] * f[e] + g[e] * g[e];
                for (int o = group >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                if (w && holds) {
                    const float norm = 1.f / sqrtf(sum / (float)a.dim + a.eps);
                    float wf[kVec], wg[kVec];
                    Elem<T>::unpack(ldg_vec(w + lo), wf);
                    Elem<T>::unpack(ldg_vec(w + hi), wg);
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        f[e] *= norm * wf[e];
                        g[e] *= norm * wg[e];
                    }
                }
            }
            if (u >= units || !holds || pos[r] < 0) continue;
            if (turned) {
                const float2 *cs = turn + r * half + p0;
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < kVec; e += 2) {
                        const float2 c0 = cs[e / 2], c1 = cs[kVec / 2 + e / 2];
                        const float a0 = f[e], b0 = f[e + 1], a1 = g[e], b1 = g[e + 1];
                        f[e] = a0 * c0.x - b0 * c0.y;
                        f[e + 1] = b0 * c0.x + a0 * c0.y;
                        g[e] = a1 * c1.x - b1 * c1.y;
                        g[e + 1] = b1 * c1.x + a1 * c1.y;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        const float2 c = cs[e];
                        const float p = f[e], q = g[e];
                        f[e] = p * c.x - q * c.y;
                        g[e] = q * c.x + p * c.y;
                    }
                }
            }
            T *o = hd < a.q_heads ? (T *)a.q_out + (row0 + r) * a.q_out_stride + hd * a.dim
                                  : (T *)a.k_out + (row0 + r) * a.k_out_stride + (hd - a.q_heads) * a.dim;
            *reinterpret_cast<uint4 *>(o + lo) = pack_vec<T>(f);
            *reinterpret_cast<uint4 *>(o + hi) = pack_vec<T>(g);
        }
    }
}

}  // namespace rtp

extern "C" rtprune_status_t rtprune_qk_norm_rope(void *cuda_stream, rtprune_dtype_t dtype, const void *q, int64_t q_stride,
                                                 const void *k, int64_t k_stride, int64_t rows, int32_t q_heads, int32_t kv_heads,
                                                 int32_t head_dim, const void *q_weight, const void *k_weight, float eps,
                                                 const int32_t *positions, const double *inv_freq, int32_t rotary_dim,
                                                 int32_t interleaved, void *q_out, int64_t q_out_stride, void *k_out,
                                                 int64_t k_out_stride)
{
    using namespace rtp;
    if (rows < 0 || q_heads < 0 || kv_heads < 0 || q_heads + kv_heads == 0 || head_dim <= 0 || rotary_dim < 0 || rotary_dim > head_dim ||
        !(eps >= 0.f) || (dtype != RTPRUNE_BF16 && dtype != RTPRUNE_FP32))
        return RTPRUNE_ERR_INVALID_ARG;
    if (head_dim % 16 || rotary_dim % 16 || head_dim > 256 || q_heads > 4096 || kv_heads > 4096) return RTPRUNE_ERR_UNSUPPORTED;
    if (rows > INT32_MAX - kRpMaxRows) return RTPRUNE_ERR_UNSUPPORTED;
    if (rows == 0) return RTPRUNE_OK;
    const int64_t vec = dtype == RTPRUNE_BF16 ? 8 : 4;
    auto bad = [&](const void *p, int64_t stride, int64_t heads) {
        return !p || ((uintptr_t)p & 15u) || stride < heads * head_dim || stride % vec;
    };
    if (q_heads && (bad(q, q_stride, q_heads) || bad(q_out, q_out_stride, q_heads))) return RTPRUNE_ERR_INVALID_ARG;
    if (kv_heads && (bad(k, k_stride, kv_heads) || bad(k_out, k_out_stride, kv_heads))) return RTPRUNE_ERR_INVALID_ARG;
    if (!positions || (rotary_dim && !inv_freq) || ((uintptr_t)inv_freq & 7u) || (((uintptr_t)q_weight | (uintptr_t)k_weight) & 15u))
        return RTPRUNE_ERR_INVALID_ARG;
    int dev = 0, sms = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess)
        return RTPRUNE_ERR_CUDA;
    RopeArgs a = {q, k, q_weight, k_weight, q_out, k_out, q_stride, k_stride, q_out_stride, k_out_stride, positions, inv_freq,
                  (int)rows, 1, q_heads, q_heads + kv_heads, head_dim, rotary_dim, interleaved ? 1 : 0, 0, eps};
    while ((2 * vec << a.group_shift) < head_dim) ++a.group_shift;
    // rows of a CTA: one while that fills the device, up to kRpMaxRows so that a thread has several loads in flight
    a.rows_per_cta = (int)std::min<int64_t>(kRpMaxRows, std::max<int64_t>(1, rows / (sms * 8)));
    const dim3 grid((unsigned)((rows + a.rows_per_cta - 1) / a.rows_per_cta));
    const cudaError_t e = dtype == RTPRUNE_BF16
                              ? launch_chained(qk_norm_rope_kernel<__nv_bfloat16>, grid, dim3(kRpThreads), (size_t)0, (cudaStream_t)cuda_stream, a)
                              : launch_chained(qk_norm_rope_kernel<float>, grid, dim3(kRpThreads), (size_t)0, (cudaStream_t)cuda_stream, a);
    if (e != cudaSuccess) return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}
