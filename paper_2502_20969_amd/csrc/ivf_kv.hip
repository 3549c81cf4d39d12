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

int make_views(const ivf_kv_step* step, const ivf_kv_cache* cache, CacheView* cv, StepView* sv, QuantView* qv) {
    if (!step || !cache) return fail(IVF_EINVAL, "step or cache is NULL");
    if (!cache->k || !cache->v) return fail(IVF_EINVAL, "cache k or v is NULL");
    if ((((uintptr_t)cache->k | (uintptr_t)cache->v) & 15u) != 0) return fail(IVF_EINVAL, "cache k and v must be 16-byte aligned");
    const bool quant = cache->dtype == IVF_E4M3;
    if (!quant && cache->dtype != IVF_F16 && cache->dtype != IVF_BF16) return fail(IVF_EINVAL, "cache type %d: f16, bf16 or e4m3 only", cache->dtype);
    if (cache->n_pages < 1 || cache->n_heads < 1 || cache->d < 1) return fail(IVF_EINVAL, "cache n_pages, n_heads and d must be at least 1");
    const int lot = quant ? 16 : 8;
    if (cache->page_stride % lot != 0 || cache->token_stride % lot != 0 || cache->head_stride % lot != 0)
        return fail(IVF_EINVAL, "cache strides must be multiples of %d elements", lot);
    for (int64_t stride : {cache->page_stride, cache->token_stride})
        if (stride > (1 << 30) - 1 || stride < -(1 << 30)) return fail(IVF_ELIMIT, "cache stride of %lld elements", (long long)stride);
    if (quant) {
        if (!cache->k_scale || !cache->v_scale) return fail(IVF_EINVAL, "cache k_scale or v_scale is NULL");
        const bool half = cache->row_dtype == IVF_F16;
        if (!half && cache->row_dtype != IVF_BF16) return fail(IVF_EINVAL, "row_dtype %d: f16 or bf16 only", cache->row_dtype);
        for (int64_t stride : {cache->scale_page_stride, cache->scale_token_stride})
            if (stride > (1 << 30) - 1 || stride < -(1 << 30)) return fail(IVF_ELIMIT, "scale stride of %lld bytes", (long long)stride);
        *qv = QuantView{cache->k_scale, cache->v_scale, cache->scale_page_stride, cache->scale_token_stride, cache->scale_head_stride,
                        127 + (half ? -15 : -117), 127 + (half ? 8 : 120)};
    }
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
                    (int)(cache->page_stride * (quant ? 1 : 2)), (int)(cache->token_stride * (quant ? 1 : 2))};
    *sv = StepView{step->q_off, step->len, step->table, step->group_off, step->prefix_len, step->prefix_table,
                   step->table_stride, step->prefix_stride, cap(step->table_stride, ss), cap(step->prefix_stride, ps),
                   slots >> ss, step->n_seq, step->n_tokens, step->n_groups, ss, ps,
                   (int)std::min<int64_t>((slots >> ss) - 1, INT32_MAX), (int)std::min<int64_t>((slots >> ps) - 1, INT32_MAX)};
    return IVF_OK;
}

struct AppendArgs {
    CacheView cache;
    QuantView quant;
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

// Slot and position of a new token, by a workgroup of 256; -1: no slot.
__device__ __forceinline__ int64_t place_token(const AppendArgs& a, int t, int& pos) {
    // the sequence: how many of them begin at or before t
    int below = 0;
    for (int i = threadIdx.x; i < a.step.n_seq; i += 256) below += a.step.q_off[i] <= t;
    __shared__ int s_count;
    if (threadIdx.x == 0) s_count = 0;
    __syncthreads();
    if (below) atomicAdd(&s_count, below);
    __syncthreads();
    const int seq = s_count - 1;
    int64_t slot = -1;
    pos = 0;
    if (seq >= 0) {
        const int place = a.step.len[seq] - (a.step.q_off[seq + 1] - t);
        pos = place + prefix_of(a.step, group_of(a.step, seq));
        if (place >= 0 && place < a.step.own_cap) {
            const int64_t e = a.step.table[seq * a.step.table_stride + (place >> a.step.shift)];
            if (e >= 0 && e < a.step.own_entries) slot = (e << a.step.shift) + (place & ((1 << a.step.shift) - 1));
        }
    }
    if (a.positions) pos = a.positions[t];
    return slot;
}

// One workgroup per new token.  A unit is sixteen elements of a head: in the rotated part eight pairs (two chunks of
// eight that lie rot / 2 apart, or sixteen in a row), behind it sixteen in a row.  A thread keeps its unit's cosines and
// sines and takes that unit of one head after the other.  Rotated in 32 bits, rounded once.
// Bound by memory: 17,000 tokens of 64 query and 8 key heads of 128 in 131 us, 5.4 TB/s read and written.  One token per
// sequence is a chain of loads (sequence, place, table, cosines): 3.8 us for one, 6.6 for 200.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
    const int t = blockIdx.x, tid = threadIdx.x;
    int pos;
    const int64_t slot = place_token(a, t, pos);
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

// Eight pairs of numbers rotated as 32-bit numbers, products and sum rounded one by one: what is quantised does not depend
// on which of them a compiler joins.  INTERLEAVED: x are sixteen in a row, pairs side by side; else x[i] and x[8 + i] are a pair.
template <bool INTERLEAVED>
__device__ __forceinline__ void rotate_exact(float (&x)[16], const float (&c)[8], const float (&s)[8]) {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        float& xa = x[INTERLEAVED ? 2 * i : i];
        float& xb = x[INTERLEAVED ? 2 * i + 1 : 8 + i];
        const float a = xa, b = xb;
        xa = a * c[i] - b * s[i];
        xb = b * c[i] + a * s[i];
    }
}

// Four numbers of at most 448 as e4m3, ties to even
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// The same into a quantised cache: x becomes the e4m3 number nearest to x 2^-e, e the least with max |x| <= 448 2^e.  448 is 1.75 * 2^8, so e
// comes from the exponent and fraction of the largest number's bits, and 2^-e is exact.  The units of a head go to the lanes of a group of
// `width`, a power of two, which find the largest by exchanging it.
// Bound by memory, of which it moves 0.7 of what the 16-bit kernel does: 17,000 tokens of 64 query and 8 key heads of 128 in 125 us, 5.4 TB/s; vector
// instructions take 57 % of the SIMDs' cycles.  One token: 4.7 us, 200 of as many sequences 7.8.
template <typename T, bool INTERLEAVED>
__global__ __launch_bounds__(256) void kv_append_quant_kernel(AppendArgs a) {
    const int t = blockIdx.x, tid = threadIdx.x;
    int pos;
    const int64_t slot = place_token(a, t, pos);
    const int upr = a.d / 16, width = upr <= 1 ? 1 : 1 << (32 - __builtin_clz(upr - 1));
    const int heads = a.hq + 2 * a.hkv, per = 256 / width, u = tid & (width - 1);
    const bool unit = u < upr, turns = u * 16 < a.rot;
    const int64_t base = slot < 0 ? 0 : slot_offset(a.cache, slot), scales = slot < 0 ? 0 : scale_offset(a.cache, a.quant, slot);
    int lo = u * 16, hi = lo + 8;                           // where the unit's two chunks begin
    float c[8], s[8];
    if (turns) {
        if (!INTERLEAVED) { lo = u * 8; hi = lo + a.rot / 2; }
        const float* row = a.rotary + (int64_t)min(max(pos, 0), a.n_positions - 1) * a.rot + u * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i) { c[i] = row[i]; s[i] = row[i + a.rot / 2]; }
    }
    const float most = __uint_as_float((uint32_t)a.quant.most << 23) * 240.f;
    for (int h = tid / width; h < heads; h += per) {
        const bool is_q = h < a.hq, is_v = h >= a.hq + a.hkv;
        const int hh = is_q ? h : is_v ? h - a.hq - a.hkv : h - a.hq;
        const ivf_rows& r = is_q ? a.q : is_v ? a.v : a.k;
        if (!is_q && slot < 0) continue;
        const T* src = (const T*)r.data + t * r.token_stride + hh * r.head_stride;
        uint4 x = make_uint4(0, 0, 0, 0), y = x;
        if (unit) { x = *(const uint4*)(src + lo); y = *(const uint4*)(src + hi); }
        if (is_q) {
            if (turns) rotate<T, INTERLEAVED>(x, y, c, s);
            T* dst = (T*)a.q_out.data + t * a.q_out.token_stride + hh * a.q_out.head_stride;
            if (unit) { *(uint4*)(dst + lo) = x; *(uint4*)(dst + hi) = y; }
            continue;
        }
        float f[16];
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 8; ++i) { f[2 * i] = to_float<T>(w[i] & 0xFFFFu); f[2 * i + 1] = to_float<T>(w[i] >> 16); }
        if (turns && !is_v) rotate_exact<INTERLEAVED>(f, c, s);
        uint32_t top = 0;                                   // the largest, as bits
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const bool finite = (__float_as_uint(f[i]) & 0x7F800000u) != 0x7F800000u;
            f[i] = finite ? fminf(fmaxf(f[i], -most), most) : NAN;
            top = max(top, finite ? __float_as_uint(f[i]) & 0x7FFFFFFFu : 0u);
        }
        for (int step = 1; step < width; step <<= 1) top = max(top, (uint32_t)__shfl_xor((int)top, step));
        // 448 = 1.75 * 2^8
        const int byte = max((int)(top >> 23) - 8 + ((top & 0x7FFFFFu) > 0x600000u), a.quant.least);
        const float by = __uint_as_float((uint32_t)(254 - byte) << 23);
        uint32_t code[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) code[i] = to_e4m3(f[4 * i] * by, f[4 * i + 1] * by, f[4 * i + 2] * by, f[4 * i + 3] * by);
        if (!unit) continue;
        uint8_t* dst = (uint8_t*)(is_v ? a.cache.v : a.cache.k) + base + hh * a.cache.head_stride;
        *(uint2*)(dst + lo) = make_uint2(code[0], code[1]);
        *(uint2*)(dst + hi) = make_uint2(code[2], code[3]);
        if (u == 0) (is_v ? a.quant.v : a.quant.k)[scales + hh * a.quant.head_stride] = (uint8_t)byte;
    }
}

struct ReadArgs {
    CacheView cache;
    QuantView quant;
    StepView step;
    ivf_rows k, v;
    const int32_t *out_off, *first;
    int64_t n_rows;
    int hkv, d, rows_wg;
};

// A workgroup reads a.rows_wg rows: its first lanes find their slots, then a thread takes a piece of 8 elements of a head, of one row after the
// other, kReadAtOnce of them at a time: a wavefront's stores are 1 KB in a row (with 16 elements a thread, whose stores are two halves, 64,900 rows
// of 8 heads of 128 took 89 us instead of 60: 5.5 TB/s; out of a 16-bit cache 81: 5.1).  Sixteen rows a workgroup where that fills the chip, else four (1391 rows: 5.4 and 4.0 us).
constexpr int kReadRows = 16, kReadAtOnce = 4;
template <typename T, bool QUANT>
__global__ __launch_bounds__(256) void kv_read_kernel(ReadArgs a) {
    __shared__ int64_t s_at[kReadRows], s_scale[kReadRows];             // where the rows' slots begin in codes and powers; -1: no such key
    const int64_t row0 = (int64_t)blockIdx.x * a.rows_wg;
    if ((int)threadIdx.x < a.rows_wg) {
        const int64_t r = row0 + threadIdx.x;
        int64_t slot = -1;
        if (r < a.n_rows && r >= a.out_off[0] && r < a.out_off[a.step.n_seq]) {
            int lo = 0, hi = a.step.n_seq;                  // out_off[lo] <= r < out_off[hi]
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (a.out_off[mid] <= r) lo = mid; else hi = mid;
            }
            const int g = group_of(a.step, lo), plen = prefix_of(a.step, g);
            const int64_t j = r - a.out_off[lo] + (a.first ? a.first[lo] : 0);
            if (j >= 0 && j < plen + own_len(a.step, lo)) slot = slot_of_key(a.step, lo, g, plen, (int)j);
        }
        s_at[threadIdx.x] = slot < 0 ? INT64_MIN : slot_offset(a.cache, slot);
        if (QUANT) s_scale[threadIdx.x] = slot < 0 ? 0 : scale_offset(a.cache, a.quant, slot);
    }
    __syncthreads();
    // units of a row: of keys, then of values; `wide` threads take one each, the others those of further rows
    const int upr = a.d / 8, units = 2 * a.hkv * upr, wide = min(units, 256), rows = 256 / wide;
    const int first = threadIdx.x / wide;
    if (first >= rows) return;
    for (int i = threadIdx.x % wide; i < units; i += wide) {
        const bool is_v = i >= a.hkv * upr;
        const int h = (is_v ? i - a.hkv * upr : i) / upr, at_unit = i % upr * 8;
        const ivf_rows& to = is_v ? a.v : a.k;
        T* out = (T*)to.data + row0 * to.token_stride + h * to.head_stride + at_unit;
        const int64_t at = h * a.cache.head_stride + at_unit, at_scale = h * a.quant.head_stride;
        const uint8_t* pool = (const uint8_t*)(is_v ? a.cache.v : a.cache.k);
        const uint8_t* scales = is_v ? a.quant.v : a.quant.k;
        for (int r0 = first; r0 < a.rows_wg; r0 += rows * kReadAtOnce) {
            u4_t x[kReadAtOnce];
            int byte[kReadAtOnce];
#pragma unroll
            for (int u = 0; u < kReadAtOnce; ++u) {
                const int r = min(r0 + u * rows, a.rows_wg - 1);
                if (s_at[r] == INT64_MIN) continue;
                if (QUANT) {
                    const uint2 c = *(const uint2*)(pool + s_at[r] + at);
                    x[u][0] = c.x;
                    x[u][1] = c.y;
                    byte[u] = scales[s_scale[r] + at_scale];
                } else {
                    x[u] = *(const u4_t*)(pool + (s_at[r] + at) * 2);
                }
            }
#pragma unroll
            for (int u = 0; u < kReadAtOnce; ++u) {
                const int r = r0 + u * rows;
                if (r >= a.rows_wg || s_at[r] == INT64_MIN) continue;
                if (QUANT) {
                    const float p = power_of(a.quant, byte[u]);
                    const uint32_t lo = x[u][0], hi = x[u][1];
                    x[u] = u4_t{from_e4m3<T, false>(lo, p), from_e4m3<T, true>(lo, p), from_e4m3<T, false>(hi, p), from_e4m3<T, true>(hi, p)};
                }
                __builtin_nontemporal_store(x[u], (u4_t*)(out + r * to.token_stride));
            }
        }
    }
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_kv_append(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* k, const ivf_rows* v,
                             const float* rotary, int32_t n_positions, int32_t rot, int32_t interleaved, const int32_t* positions,
                             const ivf_rows* q, const ivf_rows* q_out, int32_t n_q_heads, void* stream) {
    AppendArgs a{};
    int rc = make_views(step, cache, &a.cache, &a.step, &a.quant);
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
    if (too_many_threads(step->n_tokens, 256)) return fail(IVF_ELIMIT, "%d tokens", step->n_tokens);
    a.k = *k; a.v = *v;
    if (q) { a.q = *q; a.q_out = *q_out; }
    a.rotary = rotary; a.positions = positions; a.n_positions = n_positions; a.rot = rot;
    a.hq = n_q_heads; a.hkv = cache->n_heads; a.d = cache->d;
    const dim3 grid(step->n_tokens), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (cache->dtype == IVF_E4M3) {
        const bool half = cache->row_dtype == IVF_F16;
        if (half && interleaved) hipLaunchKernelGGL((kv_append_quant_kernel<_Float16, true>), grid, block, 0, s, a);
        else if (half) hipLaunchKernelGGL((kv_append_quant_kernel<_Float16, false>), grid, block, 0, s, a);
        else if (interleaved) hipLaunchKernelGGL((kv_append_quant_kernel<__bf16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_append_quant_kernel<__bf16, false>), grid, block, 0, s, a);
    } else if (cache->dtype == IVF_F16) {
        if (interleaved) hipLaunchKernelGGL((kv_append_kernel<_Float16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_append_kernel<_Float16, false>), grid, block, 0, s, a);
    } else {
        if (interleaved) hipLaunchKernelGGL((kv_append_kernel<__bf16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_append_kernel<__bf16, false>), grid, block, 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}

extern "C" int ivf_kv_read(const ivf_kv_step* step, const ivf_kv_cache* cache, const int32_t* out_off, const int32_t* first, int64_t n_rows,
                           const ivf_rows* k, const ivf_rows* v, void* stream) {
    ReadArgs a{};
    int rc = make_views(step, cache, &a.cache, &a.step, &a.quant);
    if (rc) return rc;
    if (!out_off) return fail(IVF_EINVAL, "out_off is NULL");
    if ((rc = check_rows(k, "k")) || (rc = check_rows(v, "v"))) return rc;
    if (cache->d % 16 != 0) return fail(IVF_EINVAL, "d must be a multiple of 16 (got %d)", cache->d);
    if (n_rows < 1) return fail(IVF_EINVAL, "n_rows must be at least 1");
    if (too_many_threads((n_rows - 1) / kReadRows + 1, 256)) return fail(IVF_ELIMIT, "%lld rows", (long long)n_rows);
    if ((int64_t)2 * cache->n_heads * (cache->d / 8) > 1 << 30) return fail(IVF_ELIMIT, "%d heads of %d", cache->n_heads, cache->d);
    a.k = *k; a.v = *v; a.out_off = out_off; a.first = first; a.n_rows = n_rows; a.hkv = cache->n_heads; a.d = cache->d;
    a.rows_wg = n_rows >= kReadRows * 1024 ? kReadRows : 4;
    const dim3 grid((unsigned)((n_rows + a.rows_wg - 1) / a.rows_wg)), block(256);
    hipStream_t s = (hipStream_t)stream;
    if (cache->dtype == IVF_E4M3) {
        if (cache->row_dtype == IVF_F16) hipLaunchKernelGGL((kv_read_kernel<_Float16, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((kv_read_kernel<__bf16, true>), grid, block, 0, s, a);
    } else {
        hipLaunchKernelGGL((kv_read_kernel<_Float16, false>), grid, block, 0, s, a);
    }
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
