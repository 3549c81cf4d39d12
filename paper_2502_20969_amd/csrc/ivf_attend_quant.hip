// Attention over a quantised cache: the formula as it stands, one wavefront per new token and query head, one key after the
// other with a running maximum and sum in 32 bits.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <math.h>
#include <type_traits>

namespace ivf {
using namespace dev;

template <typename T>
__global__ __launch_bounds__(64) void attend_quant_kernel(CacheView cache, QuantView quant, StepView step, ivf_rows q, ivf_rows out, float* lse,
                                                          float scale_log2, int hq, int group, int d, int window, int sinks) {
    const int t = blockIdx.x / hq, head = blockIdx.x % hq, lane = lane_id();
    int lo = 0, hi = step.n_seq;                            // the last sequence that begins at or before t
    if (token_of(step, 0) > t || token_of(step, step.n_seq) <= t) return;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (step.q_off[mid] <= t) lo = mid; else hi = mid;
    }
    const int g = group_of(step, lo), plen = prefix_of(step, g), keys = plen + own_len(step, lo);
    const int pos = keys - (token_of(step, lo + 1) - t);
    const T* src = (const T*)q.data + t * q.token_stride + head * q.head_stride;
    const int64_t at_head = head / group * cache.head_stride, at_scale = head / group * quant.head_stride;
    float x[4], o[4] = {0.f, 0.f, 0.f, 0.f}, m = -INFINITY, l = 0.f;
    for (int e = 0; e < 4; ++e) x[e] = e * 64 + lane < d ? (float)src[e * 64 + lane] : 0.f;
    for (int j = 0; j <= pos && j < keys; ++j) {
        if (window > 0 && pos - j >= window && j >= sinks) continue;
        const int64_t slot = slot_of_key(step, lo, g, plen, j);
        const int64_t at = slot_offset(cache, slot) + at_head, sc = scale_offset(cache, quant, slot) + at_scale;
        const float kp = power_of(quant, quant.k[sc]), vp = power_of(quant, quant.v[sc]);
        float dot = 0.f;
        for (int e = 0; e < 4; ++e)
            if (e * 64 + lane < d) dot += x[e] * (__builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)cache.k)[at + e * 64 + lane], 0) * kp);
        dot = group_sum<64>(dot) * scale_log2;
        const float m2 = fmaxf(m, dot), f = m == -INFINITY ? 0.f : exp2f(m - m2), w = m2 == -INFINITY && dot == dot ? 0.f : exp2f(dot - m2);
        m = m2;
        l = l * f + w;
        for (int e = 0; e < 4; ++e)
            if (e * 64 + lane < d) o[e] = o[e] * f + w * (__builtin_amdgcn_cvt_f32_fp8(((const uint8_t*)cache.v)[at + e * 64 + lane], 0) * vp);
    }
    const float f = l > 0.f || l != l ? 1.f / l : 0.f;
    T* dst = (T*)out.data + t * out.token_stride + head * out.head_stride;
    for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < d) dst[e * 64 + lane] = (T)(o[e] * f);
    if (lse && lane == 0) lse[(int64_t)t * hq + head] = l > 0.f || l != l ? (m + log2f(l)) * 0.6931471805599453f : -INFINITY;
}

hipError_t launch_attend_quant(const CacheView& cache, const QuantView& quant, const StepView& step, int row_dtype, const ivf_rows& q, const ivf_rows& out,
                               float* lse, float scale_log2, int hq, int group, int d, int window, int sinks, hipStream_t s) {
    const int64_t grid = (int64_t)step.n_tokens * hq;
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    if (row_dtype == IVF_F16)
        hipLaunchKernelGGL(attend_quant_kernel<_Float16>, dim3((unsigned)grid), dim3(64), 0, s, cache, quant, step, q, out, lse, scale_log2, hq, group, d, window, sinks);
    else
        hipLaunchKernelGGL(attend_quant_kernel<__bf16>, dim3((unsigned)grid), dim3(64), 0, s, cache, quant, step, q, out, lse, scale_log2, hq, group, d, window, sinks);
    return hipGetLastError();
}

}  // namespace ivf
