// What the attention kernels over the 8-bit paged cache share: the call's arguments, the checks of a request, and the
// steps from codes to fp16.
//
// Row r of request i, its j-th of n_i, sees the cached tokens t < end: L_i, or L_i - n_i + j + 1 when causal.
//   s_t = scale * ks * (q . kc_t),  out = sum_t softmax(s)_t vs vc_t,  lse = log sum_t exp s_t
// with kc, vc the codes of token t and ks, vs the scales of its page and head.
//
// Codes are whole numbers up to 127, exact in fp16 and in bf16.  Scores of many rows are products of bf16, queries as they are; those of
// few rows products of fp16, where a query's elements are exact too once its row has been taken to a largest value between 1 and 2 by a
// power of two (an element under 2^-14 of that is off by 2^-25 at most).  Weights and values are fp16 in both.  The softmax runs in powers
// of two on
//   s'_t = s_t log2(e) + log2(vs),  p'_t = 2^(s'_t - m'),  m' about the largest s' so far,
// so that the values' scale is inside the weight (p' is what fp16 has to hold, and it is largest where the products are) and the
// products are with bare codes; the sum of the softmax is that of p'_t / vs = 2^(s_t - m'), l.
//
// That holds while the scales that a row sees are within 2^80 of one another: from 2^-60 to 2^20.  Where a block's is outside (scales
// may be anything from 2^-126 to 2^121), or is 0, a row goes on, to the end of its tile, with a second reference r about the largest s,
//   l = sum_t 2^(s_t - r),  out = sum p' vc / l * 2^(m' - r),
// because 2^(s_t - m') may pass fp32's range, and with a block's log2(vs) raised to m' - r - 80 in its weights: their p' are then 2^-80
// and less, nothing in fp16, as what they stand for is, but still numbers of which p' / vs can be taken for l.  A block of zeros has no
// log2(vs); one far below all others has it lead m' only where a row sees nothing else.
#pragma once
#include "serve.cuh"

namespace rtp {

struct AttendArgs {
    const __nv_bfloat16 *q;
    int64_t q_stride;
    const int32_t *offsets, *seq_lens, *tables;
    int64_t table_stride;
    int32_t batch, rows, q_heads, group, max_q_len, max_len, max_pages;
    CacheView c;
    float scale_log2;                        // scale * log2(e)
    int32_t causal;
    __nv_bfloat16 *out;
    float *lse;
    uint32_t polls;                          // after which a wait gives up: the rows that hang on it, and those of the CTA's later work, come out NaN
};

// Bounded wait of a whole warp: no lane goes on as if what the others gave up on were there.
__device__ inline bool attend_wait(const AttendArgs &a, uint64_t *bar, uint32_t parity)
{
    return __all_sync(0xffffffffu, ptx::mbar_wait(bar, parity, a.polls));
}

constexpr float kAtNothing = -3.4028235e38f; // m' of a row that has seen nothing yet: no score is less (finite: -inf minus it is still -inf)
constexpr float kAtSlack = 8.f;              // m' follows the maximum only where a weight would pass 2^8 (fp16 ends at 2^16)
constexpr float kAtLowLog = -60.f, kAtHighLog = 20.f;      // log2(vs) for which l may have m' as its reference
constexpr float kAtZeroLog = -200.f;         // log2(vs) of a block of scale 0
constexpr float kAtLogGap = 80.f;
constexpr float kAtLn2 = 0.69314718055994531f;

// A request's rows and lengths.  false: it has no rows, or none that may be written.  len = -1: outside the contract, its rows
// come out NaN.
__device__ inline bool attend_request(const AttendArgs &a, int i, int &row0, int &n, int &len)
{
    row0 = __ldg(a.offsets + i);
    const int hi = __ldg(a.offsets + i + 1);
    n = hi - row0;
    len = __ldg(a.seq_lens + i);
    if (len < 0 || len > a.max_len) len = -1;
    return row0 >= 0 && hi > row0 && hi <= a.rows && n <= a.max_q_len;
}

// The page of token t, or -1.
__device__ inline int attend_page(const AttendArgs &a, int i, int t)
{
    const int p = t >> a.c.page_shift;
    const int page = p < a.max_pages ? __ldg(a.tables + (int64_t)i * a.table_stride + p) : -1;
    return page < a.c.num_pages ? page : -1;
}

__device__ inline float ex2(float x)
{
    float r;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// log2(vs) and 1 / vs of a block's scale; true: one that m' does not do for as the reference of l.
__device__ inline bool value_scale(float vs, float &lv, float &inv)
{
    lv = vs == 0.f ? kAtZeroLog : __log2f(vs);
    inv = __frcp_rn(vs);
    return lv < kAtLowLog || lv > kAtHighLog;
}
// log2(vs) for the weights of a block, gap = m' - r.  (NaN stays.)
__device__ inline float weight_log(float lv, float gap) { return lv < gap - kAtLogGap ? gap - kAtLogGap : lv; }
// What a row's sums are multiplied by, twice: the root of 2^(m' - r), which may be as little as 2^-134.
__device__ inline float half_gap(float m, float ref) { return ex2(0.5f * (m - ref)); }
// Power of two that takes a row's largest |q| to [1, 4), and the factor of the row's scores that makes up for it (NaN where
// the row is not finite).
__device__ inline float query_scale(float top, float scale_log2, float &factor)
{
    const int e = max(min((int)(__float_as_uint(top) >> 23) - 127, 126), -126);
    factor = top <= 3.4e38f ? scale_log2 * __uint_as_float((uint32_t)(e + 127) << 23) : __uint_as_float(0x7fc00000u);
    return __uint_as_float((uint32_t)(127 - e) << 23);
}

// 1024 + (code + 128) is the fp16 number with the biased code as its last bits: bytes beside 0x64, minus 1152.
constexpr uint32_t kAtMagic = 0x64646464u, kAtBias = 0x64806480u;
__device__ inline uint32_t half_sub(uint32_t a, uint32_t b)
{
    uint32_t r;
    asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
// Four codes of a word, in order, as two pairs of fp16 (x: the word with its codes biased by 128).
__device__ inline void codes_to_half(uint32_t x, uint32_t &lo, uint32_t &hi)
{
    lo = half_sub(__byte_perm(x, kAtMagic, 0x4140), kAtBias);
    hi = half_sub(__byte_perm(x, kAtMagic, 0x4342), kAtBias);
}
__device__ inline uint32_t pack_half(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

}  // namespace rtp
