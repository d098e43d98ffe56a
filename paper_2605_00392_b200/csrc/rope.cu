// Norms of queries and keys per head and the rotation by position, in one pass (rtprune_qk_norm_rope).
#include <algorithm>

#include "serve.cuh"

namespace rtp {

// y = x w / sqrt(mean x^2 + eps) over a head's elements (no weights: y = x), then the first `rotary` of them in pairs
// (y_i, y_j) -> (y_i cos - y_j sin, y_j cos + y_i sin) by the angle pos f_p.
//
// A warp takes a row with all its heads, or, where there are few rows, some of them, then the next that is its own, whose position it
// has read by then.  A lane holds the two elements of each of its pairs: 16 bytes of first and 16 of second elements
// (half-split pairs: half a rotated part apart; adjacent pairs: 32 bytes in a row), so that the rotation needs no exchange and the norm one
// sum over the D / 16 (fp32: D / 8) lanes of a head, and its pairs are the same ones in every head.  The row's angles are computed
// once, shared out over the lanes, while the first heads are on their way.  Angles in 64 bits, taken modulo a turn before they are rounded to
// 32: at position 10^6 an fp32 angle would be off by 0.03.  Everything else in fp32, rounded once, at the store.
// Each element is read and written once.  4999 rows of 40 heads in fp32: 41 us, 5.0 TB/s.  21568 rows of 20 heads in bf16: 54 us, 4.1 TB/s
// (57 with a CTA for every four rows); there it is latency and issue slots (58 % of them) more than HBM: without the norm it takes 47, without
// the turning or the angles 53.  Other numbers of heads in flight and CTAs to an SM (5 at 4, 1 at 7) are as fast, and slower in fp32 (47, 53);
// packed fp32 arithmetic is slower (64).
constexpr int kRpWarps = 4;
constexpr int kRpPerSm = 5;                  // CTAs of an SM; no more are launched
constexpr int kRpAhead = 3;                  // heads' pieces of a lane whose loads are in flight together

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

// (by value: a choice between two registers, not between two addresses)
__device__ inline uint4 pick(bool second, uint4 b, uint4 a)
{
    return make_uint4(second ? b.x : a.x, second ? b.y : a.y, second ? b.z : a.z, second ? b.w : a.w);
}

struct RopeArgs {
    const void *q, *k, *q_weight, *k_weight;
    void *q_out, *k_out;
    int64_t q_stride, k_stride, q_out_stride, k_out_stride;
    const int32_t *positions;
    const double *inv_freq;
    int rows, parts, part_units, q_heads, heads, dim, rotary, interleaved, group_shift;      // a head: 1 << group_shift lanes
    float eps;
};

template <typename T>
__global__ void __launch_bounds__(32 * kRpWarps, kRpPerSm)
qk_norm_rope_kernel(const __grid_constant__ RopeArgs a)
{
    constexpr int kVec = Elem<T>::kPerVec;
    __shared__ __align__(16) float2 turns[kRpWarps][128];        // cos, sin of a row's angles (rotary <= 256)
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = a.rotary / 2;
    const int64_t items = (int64_t)a.rows * a.parts, stride = (int64_t)gridDim.x * kRpWarps;
    int64_t item = (int64_t)blockIdx.x * kRpWarps + warp;
    ptx::grid_dep_launch();
    ptx::grid_dep_wait();
    if (item >= items) return;
    const int group = 1 << a.group_shift, at = lane & (group - 1);
    // first and second elements of this lane's pairs: rotated ones, then those that pass through, in the same way
    int lo, hi;
    const int p0 = at * kVec;
    const bool turned = p0 < half;
    if (a.interleaved) lo = 2 * p0, hi = lo + kVec;
    else if (turned) lo = p0, hi = lo + half;
    else lo = half + p0, hi = lo + (a.dim - a.rotary) / 2;
    const bool holds = at < a.dim / (2 * kVec);
    const uint4 none = make_uint4(0u, 0u, 0u, 0u);
    // weights of this lane's elements
    const uint4 q_lo = a.q_weight && holds ? ldg_vec((const T *)a.q_weight + lo) : none, q_hi = a.q_weight && holds ? ldg_vec((const T *)a.q_weight + hi) : none;
    const uint4 k_lo = a.k_weight && holds ? ldg_vec((const T *)a.k_weight + lo) : none, k_hi = a.k_weight && holds ? ldg_vec((const T *)a.k_weight + hi) : none;
    float c[kVec], s[kVec];                                      // of this lane's pairs
    const float inv_dim = 1.f / (float)a.dim;
    int next = __ldg(a.positions + (a.parts == 1 ? item : item / a.parts));
#pragma unroll 1
    while (item < items) {
        const int64_t row = a.parts == 1 ? item : item / a.parts;
        const int pos = next;
        // unit = (head, lane of the head); heads are queries' first, then keys'
        const int first = (int)(item - row * a.parts) * a.part_units;
        const int units = pos < 0 ? first : min(a.heads << a.group_shift, first + a.part_units);
        item += stride;
        if (item < items) next = __ldg(a.positions + (a.parts == 1 ? item : item / a.parts));      // while this row is turned
#pragma unroll 1
        for (int u0 = first + lane; u0 - lane < units; u0 += 32 * kRpAhead) {
            uint4 x[kRpAhead], y[kRpAhead];
#pragma unroll
            for (int t = 0; t < kRpAhead; ++t) {
                const int u = u0 + 32 * t, hd = u >> a.group_shift;
                x[t] = y[t] = none;
                if (u < units && holds) {
                    const T *p = hd < a.q_heads ? (const T *)a.q + row * a.q_stride + hd * a.dim : (const T *)a.k + row * a.k_stride + (hd - a.q_heads) * a.dim;
                    x[t] = *reinterpret_cast<const uint4 *>(p + lo);
                    y[t] = *reinterpret_cast<const uint4 *>(p + hi);
                }
            }
            if (u0 == first + lane) {
                __syncwarp();                                        // (the row before has been turned)
                for (int f = lane; f < half; f += 32) {
                    const double turn = (double)pos * __ldg(a.inv_freq + f) * 0.15915494309189533577;
                    float2 t;
                    sincospif(2.f * (float)(turn - rint(turn)), &t.y, &t.x);
                    turns[warp][f] = t;
                }
                __syncwarp();
#pragma unroll
                for (int e = 0; e < kVec; ++e) {
                    const float2 t = turned ? turns[warp][p0 + e] : make_float2(1.f, 0.f);   // (no turn: as it is)
                    c[e] = t.x;
                    s[e] = t.y;
                }
            }
#pragma unroll
            for (int t = 0; t < kRpAhead; ++t) {
                if (u0 - lane + 32 * t >= units) break;              // the same for the whole warp
                const int u = u0 + 32 * t, hd = u >> a.group_shift;
                const bool is_k = hd >= a.q_heads;
                float f[kVec], g[kVec];
                Elem<T>::unpack(x[t], f);
                Elem<T>::unpack(y[t], g);
                if (a.q_weight || a.k_weight) {
                    float sum = 0.f;
#pragma unroll
                    for (int e = 0; e < kVec; ++e) sum += f[e] * f[e] + g[e] * g[e];
                    for (int o = group >> 1; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
                    if (is_k ? a.k_weight != nullptr : a.q_weight != nullptr) {
                        const float norm = rsqrtf(fmaf(sum, inv_dim, a.eps));
                        float wf[kVec], wg[kVec];
                        Elem<T>::unpack(pick(is_k, k_lo, q_lo), wf);
                        Elem<T>::unpack(pick(is_k, k_hi, q_hi), wg);
#pragma unroll
                        for (int e = 0; e < kVec; ++e) {
                            f[e] *= norm * wf[e];
                            g[e] *= norm * wg[e];
                        }
                    }
                }
                if (u >= units || !holds) continue;
                if (a.interleaved) {
#pragma unroll
                    for (int e = 0; e < kVec; e += 2) {
                        const float a0 = f[e], b0 = f[e + 1], a1 = g[e], b1 = g[e + 1];
                        const float c0 = c[e / 2], s0 = s[e / 2], c1 = c[kVec / 2 + e / 2], s1 = s[kVec / 2 + e / 2];
                        f[e] = a0 * c0 - b0 * s0;
                        f[e + 1] = b0 * c0 + a0 * s0;
                        g[e] = a1 * c1 - b1 * s1;
                        g[e + 1] = b1 * c1 + a1 * s1;
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < kVec; ++e) {
                        const float p = f[e], q = g[e];
                        f[e] = p * c[e] - q * s[e];
                        g[e] = q * c[e] + p * s[e];
                    }
                }
                T *o = is_k ? (T *)a.k_out + row * a.k_out_stride + (hd - a.q_heads) * a.dim : (T *)a.q_out + row * a.q_out_stride + hd * a.dim;
                *reinterpret_cast<uint4 *>(o + lo) = pack_vec<T>(f);
                *reinterpret_cast<uint4 *>(o + hi) = pack_vec<T>(g);
            }
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
    if (rows > INT32_MAX - kRpWarps) return RTPRUNE_ERR_UNSUPPORTED;
    if (rows == 0) return RTPRUNE_OK;
    const int64_t vec = dtype == RTPRUNE_BF16 ? 8 : 4;
    auto bad = [&](const void *p, int64_t stride, int64_t heads) {
        return !p || ((uintptr_t)p & 15u) || stride < heads * head_dim || stride % vec;
    };
    if (q_heads && (bad(q, q_stride, q_heads) || bad(q_out, q_out_stride, q_heads))) return RTPRUNE_ERR_INVALID_ARG;
    if (kv_heads && (bad(k, k_stride, kv_heads) || bad(k_out, k_out_stride, kv_heads))) return RTPRUNE_ERR_INVALID_ARG;
    if (!positions || (rotary_dim && !inv_freq) || ((uintptr_t)inv_freq & 7u) || (((uintptr_t)q_weight | (uintptr_t)k_weight) & 15u))
        return RTPRUNE_ERR_INVALID_ARG;
    RopeArgs a = {q, k, q_weight, k_weight, q_out, k_out, q_stride, k_stride, q_out_stride, k_out_stride, positions, inv_freq,
                  (int)rows, 1, 0, q_heads, q_heads + kv_heads, head_dim, rotary_dim, interleaved ? 1 : 0, 0, eps};
    while ((2 * vec << a.group_shift) < head_dim) ++a.group_shift;
    // few rows: their heads shared out over warps, down to one piece of each lane (a warp for a row against this, 20 heads in bf16, in us:
    // 1 row 4.8 / 2.8, 64 5.0 / 2.9, 512 5.6 / 4.0, 1000 6.2 / 6.8, 2000 7.9 / 11.4; 40 heads, 256 rows 7.9 / 3.9, in fp32 1000 rows 15.5 / 15.0)
    const int units = a.heads << a.group_shift;
    if (rows < 1024) a.parts = (units + 31) / 32;
    a.part_units = ((units + a.parts - 1) / a.parts + 31) / 32 * 32;
    const int sms = device_sms();
    if (!sms) return RTPRUNE_ERR_CUDA;
    const int64_t ctas = std::min<int64_t>((rows * a.parts + kRpWarps - 1) / kRpWarps, (int64_t)sms * kRpPerSm);
    const dim3 grid((unsigned)ctas), block(32 * kRpWarps);
    const cudaError_t e = dtype == RTPRUNE_BF16
                              ? launch_chained(qk_norm_rope_kernel<__nv_bfloat16>, grid, block, (size_t)0, (cudaStream_t)cuda_stream, a)
                              : launch_chained(qk_norm_rope_kernel<float>, grid, block, (size_t)0, (cudaStream_t)cuda_stream, a);
    if (e != cudaSuccess) return RTPRUNE_ERR_CUDA;
    return cudaGetLastError() == cudaSuccess ? RTPRUNE_OK : RTPRUNE_ERR_CUDA;
}
