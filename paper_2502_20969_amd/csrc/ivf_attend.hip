// Attention of a step's new tokens over the paged cache.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <algorithm>

namespace ivf {
using namespace dev;

struct AttendArgs {
    CacheView cache;
    StepView step;
    ivf_rows q, out;
    float* lse;
    float scale;
    int hq, group, window, sinks;        // group: query heads per key head
};

// One wavefront per token and query head, 64 keys at a time: a lane takes the product with one key, then the lanes
// take the elements of the values.
template <typename T, int D>
__global__ __launch_bounds__(64) void attend_rows_kernel(AttendArgs a) {
    constexpr int kPer = (D + 63) / 64;
    const int lane = threadIdx.x, h = blockIdx.y, kvh = h / a.group;
    __shared__ float s_q[D];
    for (int t = blockIdx.x; t < a.step.n_tokens; t += gridDim.x) {
        int lo = 0, hi = a.step.n_seq;                     // the last sequence that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.step.q_off[mid] <= t) lo = mid; else hi = mid;
        }
        const int s = lo, g = group_of(a.step, s), plen = prefix_of(a.step, g);
        const int n = own_len(a.step, s);
        const int pos = plen + n - (a.step.q_off[s + 1] - t);
        const T* q = (const T*)a.q.data + t * a.q.token_stride + h * a.q.head_stride;
        __syncthreads();
        for (int e = lane; e < D; e += 64) s_q[e] = (float)q[e] * a.scale;
        __syncthreads();
        float m = -INFINITY, l = 0.f, o[kPer] = {};
        const int end = min(pos + 1, plen + n);
        const int low = a.window > 0 ? max(0, pos - a.window + 1) : 0;
        for (int j0 = 0; j0 < end; j0 += 64) {
            if (j0 + 64 <= low && j0 >= a.sinks) continue;
            const int j = j0 + lane;
            const bool sees = j < end && (j >= low || j < a.sinks);
            int64_t off = 0;
            float x = -INFINITY;
            if (sees) {
                const int64_t slot = j < plen ? slot_in(a.step.prefix_table + g * a.step.prefix_stride, a.step.prefix_entries, a.step.prefix_shift, j)
                                              : slot_in(a.step.table + s * a.step.table_stride, a.step.own_entries, a.step.shift, j - plen);
                off = slot_offset(a.cache, slot) + kvh * a.cache.head_stride;
                const T* k = (const T*)a.cache.k + off;
                x = 0.f;
                for (int e = 0; e < D; ++e) x += s_q[e] * (float)k[e];
            }
            float top = x;
            for (int w = 32; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
            if (__ballot(sees) == 0) continue;
            const float m2 = fmaxf(m, top);
            const float keep = m2 == -INFINITY ? 1.f : expf(m - m2);
            const float p = sees ? expf(x - m2) : 0.f;
            float sum = p;
            for (int w = 32; w >= 1; w >>= 1) sum += __shfl_xor(sum, w);
            l = l * keep + sum;
            m = m2;
            for (int i = 0; i < kPer; ++i) o[i] *= keep;
            for (uint64_t left = __ballot(sees); left; left &= left - 1) {
                const int from = __builtin_ctzll(left);
                const float pj = __shfl(p, from);
                const T* v = (const T*)a.cache.v + __shfl((long long)off, from);
                for (int i = 0; i < kPer; ++i)
                    if (i * 64 + lane < D) o[i] += pj * (float)v[i * 64 + lane];
            }
        }
        T* out = (T*)a.out.data + t * a.out.token_stride + h * a.out.head_stride;
        for (int i = 0; i < kPer; ++i)
            if (i * 64 + lane < D) out[i * 64 + lane] = (T)(l == 0.f ? 0.f : o[i] / l);
        if (a.lse && lane == 0) a.lse[(int64_t)t * a.hq + h] = l == 0.f ? -INFINITY : m + logf(l);
    }
}

static int check_heads(const ivf_kv_cache* cache, int n_q_heads, int window, int sinks) {
    if (cache->d != 64 && cache->d != 96 && cache->d != 128 && cache->d != 256)
        return fail(IVF_ELIMIT, "d must be 64, 96, 128 or 256 (got %d)", cache->d);
    if (n_q_heads < 1 || n_q_heads % cache->n_heads != 0)
        return fail(IVF_EINVAL, "n_q_heads (%d) must be a multiple of the cache's heads (%d)", n_q_heads, cache->n_heads);
    if (window < 0 || sinks < 0) return fail(IVF_EINVAL, "window and sinks must not be negative");
    return IVF_OK;
}

template <typename T>
static hipError_t launch_attend(const AttendArgs& a, int d, hipStream_t s) {
    const dim3 grid(std::min(a.step.n_tokens, 1 << 20), a.hq), block(64);
    switch (d) {
    case 64: hipLaunchKernelGGL((attend_rows_kernel<T, 64>), grid, block, 0, s, a); break;
    case 96: hipLaunchKernelGGL((attend_rows_kernel<T, 96>), grid, block, 0, s, a); break;
    case 128: hipLaunchKernelGGL((attend_rows_kernel<T, 128>), grid, block, 0, s, a); break;
    default: hipLaunchKernelGGL((attend_rows_kernel<T, 256>), grid, block, 0, s, a); break;
    }
    return hipGetLastError();
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_attend_workspace(const ivf_kv_step* step, const ivf_kv_cache* cache, int32_t n_q_heads, int32_t window,
                                    int32_t sinks, size_t* bytes) {
    CacheView cv; StepView sv;
    int rc = make_views(step, cache, &cv, &sv);
    if (rc) return rc;
    if ((rc = check_heads(cache, n_q_heads, window, sinks))) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    *bytes = 0;
    return IVF_OK;
}

extern "C" int ivf_attend(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* q, int32_t n_q_heads,
                          const ivf_rows* out, float* lse, float scale, int32_t window, int32_t sinks, void* workspace,
                          size_t workspace_bytes, void* stream) {
    size_t need = 0;
    int rc = ivf_attend_workspace(step, cache, n_q_heads, window, sinks, &need);
    if (rc) return rc;
    AttendArgs a{};
    if ((rc = make_views(step, cache, &a.cache, &a.step))) return rc;
    if ((rc = check_rows(q, "q")) || (rc = check_rows(out, "out"))) return rc;
    if (!(scale > 0.f) || scale > 1e30f) return fail(IVF_EINVAL, "scale must be positive");
    if (((uintptr_t)workspace & 15u) != 0) return fail(IVF_EINVAL, "workspace must be 16-byte aligned");
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(IVF_EINVAL, "this call needs %zu bytes of workspace (got %zu)", need, workspace ? workspace_bytes : (size_t)0);
    a.q = *q; a.out = *out; a.lse = lse; a.scale = scale;
    a.hq = n_q_heads; a.group = n_q_heads / cache->n_heads; a.window = window; a.sinks = sinks;
    HIP_TRY(cache->dtype == IVF_F16 ? launch_attend<_Float16>(a, cache->d, (hipStream_t)stream)
                                    : launch_attend<__bf16>(a, cache->d, (hipStream_t)stream));
    return IVF_OK;
}
