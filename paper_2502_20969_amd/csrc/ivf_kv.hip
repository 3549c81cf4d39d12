// Appending to the paged cache: the new tokens' keys and values go to the slots of their places, keys and queries
// are rotated by position on the way.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <algorithm>

namespace ivf {
using namespace dev;

int check_rows(const ivf_rows* r, const char* what) {
    if (!r || !r->data) return fail(IVF_EINVAL, "%s is NULL", what);
    if (((uintptr_t)r->data & 15u) != 0) return fail(IVF_EINVAL, "%s must be 16-byte aligned", what);
    if (r->token_stride % 8 != 0 || r->head_stride % 8 != 0)
        return fail(IVF_EINVAL, "strides of %s must be multiples of 8 elements", what);
    return IVF_OK;
}

static int shift_of(int32_t page) {
    if (page < 1 || (page & (page - 1)) != 0) return -1;
    return __builtin_ctz((unsigned)page);
}

int make_views(const ivf_kv_step* step, const ivf_kv_cache* cache, CacheView* cv, StepView* sv) {
    if (!step || !cache) return fail(IVF_EINVAL, "step or cache is NULL");
    if (!cache->k || !cache->v) return fail(IVF_EINVAL, "cache k or v is NULL");
    if ((((uintptr_t)cache->k | (uintptr_t)cache->v) & 15u) != 0) return fail(IVF_EINVAL, "cache k and v must be 16-byte aligned");
    if (cache->dtype != IVF_F16 && cache->dtype != IVF_BF16) return fail(IVF_EINVAL, "cache type %d: f16 or bf16 only", cache->dtype);
    if (cache->n_pages < 1 || cache->n_heads < 1 || cache->d < 1) return fail(IVF_EINVAL, "cache n_pages, n_heads and d must be at least 1");
    if (cache->page_stride % 8 != 0 || cache->token_stride % 8 != 0 || cache->head_stride % 8 != 0)
        return fail(IVF_EINVAL, "cache strides must be multiples of 8 elements");
    for (int64_t stride : {cache->page_stride, cache->token_stride})
        if (stride > (1 << 30) - 1 || stride < -(1 << 30)) return fail(IVF_ELIMIT, "cache stride of %lld elements", (long long)stride);
    const int cs = shift_of(cache->page);
    if (cs < 0) return fail(IVF_EINVAL, "cache page (%d) must be a power of two", cache->page);
    if (cache->n_pages > INT64_MAX >> 32) return fail(IVF_ELIMIT, "cache of %lld pages", (long long)cache->n_pages);
    if (!step->q_off || !step->len || !step->table) return fail(IVF_EINVAL, "q_off, len or table is NULL");
    if (step->n_seq < 1 || step->n_tokens < 1 || step->table_stride < 1)
        return fail(IVF_EINVAL, "n_seq, n_tokens and table_stride must be at least 1");
    if (step->max_q < 0 || step->max_len < 0 || step->max_prefix < 0) return fail(IVF_EINVAL, "max_q, max_len and max_prefix must not be negative");
    const int ss = shift_of(step->page);
    if (ss < 0 || ss > cs) return fail(IVF_EINVAL, "step page (%d) must be a power of two of at most the cache's (%d)", step->page, cache->page);
    if (step->n_groups < 0) return fail(IVF_EINVAL, "n_groups must not be negative");
    int ps = 0;
    if (step->n_groups > 0) {
        if (!step->group_off || !step->prefix_len || !step->prefix_table) return fail(IVF_EINVAL, "group_off, prefix_len or prefix_table is NULL");
        if (step->prefix_stride < 1) return fail(IVF_EINVAL, "prefix_stride must be at least 1");
        ps = shift_of(step->prefix_page);
        if (ps < 0 || ps > cs)
            return fail(IVF_EINVAL, "step prefix_page (%d) must be a power of two of at most the cache's (%d)", step->prefix_page, cache->page);
    }
    const int64_t slots = cache->n_pages << cs;
    // a prefix and the own keys together, and the tile behind them, stay below 2^31
    auto cap = [](int64_t stride, int shift) { return std::min<int64_t>(std::min<int64_t>(stride, (int64_t)1 << 30 >> shift) << shift, ((int64_t)1 << 30) - 1024); };
    *cv = CacheView{cache->k, cache->v, cache->page_stride, cache->token_stride, cache->head_stride, cs,
                    (int)(cache->page_stride * 2), (int)(cache->token_stride * 2)};
    *sv = StepView{step->q_off, step->len, step->table, step->group_off, step->prefix_len, step->prefix_table,
                   step->table_stride, step->prefix_stride, cap(step->table_stride, ss), cap(step->prefix_stride, ps),
                   slots >> ss, step->n_seq, step->n_tokens, step->n_groups, ss, ps,
                   (int)std::min<int64_t>((slots >> ss) - 1, INT32_MAX), (int)std::min<int64_t>((slots >> ps) - 1, INT32_MAX)};
    return IVF_OK;
}

struct AppendArgs {
    CacheView cache;
    StepView step;
    ivf_rows k, v, q, q_out;
    const float* rotary;
    const int32_t* positions;
    int n_positions, rot, hq, hkv, d;
};

template <typename T> __device__ __forceinline__ float to_float(uint32_t bits);
template <> __device__ __forceinline__ float to_float<_Float16>(uint32_t bits) { return (float)__builtin_bit_cast(_Float16, (uint16_t)bits); }
template <> __device__ __forceinline__ float to_float<__bf16>(uint32_t bits) { return __uint_as_float(bits << 16); }
template <typename T> __device__ __forceinline__ uint32_t to_bits(float x) { return __builtin_bit_cast(uint16_t, (T)x); }

// Rotates eight pairs: `a` and `b` hold eight elements each, c and s their cosines and sines.  INTERLEAVED: a and b are
// sixteen elements in a row, pairs side by side.
template <typename T, bool INTERLEAVED>
__device__ __forceinline__ void rotate(uint4& a, uint4& b, const float (&c)[8], const float (&s)[8]) {
    uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    if (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = to_float<T>(w[i] & 0xFFFFu), y = to_float<T>(w[i] >> 16);
            w[i] = to_bits<T>(x * c[i] - y * s[i]) | to_bits<T>(y * c[i] + x * s[i]) << 16;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float x0 = to_float<T>(w[i] & 0xFFFFu), x1 = to_float<T>(w[i] >> 16);
            const float y0 = to_float<T>(w[i + 4] & 0xFFFFu), y1 = to_float<T>(w[i + 4] >> 16);
            w[i] = to_bits<T>(x0 * c[2 * i] - y0 * s[2 * i]) | to_bits<T>(x1 * c[2 * i + 1] - y1 * s[2 * i + 1]) << 16;
            w[i + 4] = to_bits<T>(y0 * c[2 * i] + x0 * s[2 * i]) | to_bits<T>(y1 * c[2 * i + 1] + x1 * s[2 * i + 1]) << 16;
        }
    }
    a = make_uint4(w[0], w[1], w[2], w[3]);
    b = make_uint4(w[4], w[5], w[6], w[7]);
}

// One workgroup per new token.  A unit is sixteen elements of a head: in the rotated part eight pairs (two chunks of
// eight that lie rot / 2 apart, or sixteen in a row), behind it sixteen in a row.  A thread keeps its unit's cosines and
// sines and takes that unit of one head after the other.  Rotated in 32 bits, rounded once.
// Bound by memory: 17,000 tokens of 64 query and 8 key heads of 128 in 131 us, 5.4 TB/s read and written.  One token per
// sequence is a chain of loads (sequence, place, table, cosines): 3.8 us for one, 6.6 for 200.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
    const int t = blockIdx.x, tid = threadIdx.x;
    // the sequence: how many of them begin at or before t
    int below = 0;
    for (int i = tid; i < a.step.n_seq; i += 256) below += a.step.q_off[i] <= t;
    __shared__ int s_count;
    if (tid == 0) s_count = 0;
    __syncthreads();
    if (below) atomicAdd(&s_count, below);
    __syncthreads();
    const int seq = s_count - 1;
    int64_t slot = -1;
    int pos = 0;
    if (seq >= 0) {
        const int place = a.step.len[seq] - (a.step.q_off[seq + 1] - t);
        pos = place + prefix_of(a.step, group_of(a.step, seq));
        if (place >= 0 && place < a.step.own_cap) {
            const int64_t e = a.step.table[seq * a.step.table_stride + (place >> a.step.shift)];
            if (e >= 0 && e < a.step.own_entries) slot = (e << a.step.shift) + (place & ((1 << a.step.shift) - 1));
        }
    }
    if (a.positions) pos = a.positions[t];
    const int upr = a.d / 16;                               // units of a head
    const int heads = a.hq + 2 * a.hkv;
    const int64_t base = slot < 0 ? 0 : slot_offset(a.cache, slot);
    const int per = 256 / upr, u = tid % upr;               // heads at a time
    if (tid >= per * upr) return;
    const bool turns = u * 16 < a.rot;
    int lo = u * 16, hi = lo + 8;                           // where the unit's two chunks begin
    float c[8], s[8];
    if (turns) {
        if (!INTERLEAVED) { lo = u * 8; hi = lo + a.rot / 2; }
        const float* row = a.rotary + (int64_t)min(max(pos, 0), a.n_positions - 1) * a.rot + u * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = row[i]; s[i] = row[i + a.rot / 2]; }
    }
    for (int h = tid / upr; h < heads; h += per) {
        const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
        const int hh = is_q ? h : is_v ? h - a.hq - a.hkv : h - a.hq;
        const ivf_rows& r = is_q ? a.q : is_v ? a.v : a.k;
        if (!is_q && slot < 0) continue;
        const T* src = (const T*)r.data + t * r.token_stride + hh * r.head_stride;
        uint4 x = *(const uint4*)(src + lo), y = *(const uint4*)(src + hi);
        if (turns && !is_v) rotate<T, INTERLEAVED>(x, y, c, s);
        T* dst = is_q ? (T*)a.q_out.data + t * a.q_out.token_stride + hh * a.q_out.head_stride
                      : (T*)(is_v ? a.cache.v : a.cache.k) + base + hh * a.cache.head_stride;
        *(uint4*)(dst + lo) = x;
        *(uint4*)(dst + hi) = y;
    }
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_kv_append(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* k, const ivf_rows* v,
                             const float* rotary, int32_t n_positions, int32_t rot, int32_t interleaved, const int32_t* positions,
                             const ivf_rows* q, const ivf_rows* q_out, int32_t n_q_heads, void* stream) {
    AppendArgs a{};
    int rc = make_views(step, cache, &a.cache, &a.step);
    if (rc) return rc;
    if ((rc = check_rows(k, "k")) || (rc = check_rows(v, "v"))) return rc;
    if (n_q_heads < 0 || (n_q_heads == 0) != (q == nullptr) || (q == nullptr) != (q_out == nullptr))
        return fail(IVF_EINVAL, "q, q_out and n_q_heads go together");
    if (q && ((rc = check_rows(q, "q")) || (rc = check_rows(q_out, "q_out")))) return rc;
    if (cache->d % 16 != 0) return fail(IVF_EINVAL, "d must be a multiple of 16 (got %d)", cache->d);
    if (cache->d > 1024) return fail(IVF_ELIMIT, "d = %d is above 1024", cache->d);
    if (rot < 0 || rot % 16 != 0 || rot > cache->d) return fail(IVF_EINVAL, "rot must be a multiple of 16 of at most d (got %d)", rot);
    if ((rot > 0) != (rotary != nullptr)) return fail(IVF_EINVAL, "rotary and rot go together");
    if (rot > 0 && n_positions < 1) return fail(IVF_EINVAL, "n_positions must be at least 1");
    a.k = *k; a.v = *v;
    if (q) { a.q = *q; a.q_out = *q_out; }
    a.rotary = rotary; a.positions = positions; a.n_positions = n_positions; a.rot = rot;
    a.hq = n_q_heads; a.hkv = cache->n_heads; a.d = cache->d;
    const dim3 grid(step->n_tokens), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (cache->dtype == IVF_F16) {
        if (interleaved) hipLaunchKernelGGL((kv_append_kernel<_Float16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_append_kernel<_Float16, false>), grid, block, 0, s, a);
    } else {
        if (interleaved) hipLaunchKernelGGL((kv_append_kernel<__bf16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_append_kernel<__bf16, false>), grid, block, 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
