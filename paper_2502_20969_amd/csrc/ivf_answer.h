// Shared by the operators of answering from retrieved passages (ivf_kv.hip, ivf_attend.hip, ivf_beam.hip): the
// paged cache and the sequences of a step as the kernels see them.
#pragma once
#include "../../include/ivf.h"
#include "ivf_internal.h"
#include <type_traits>

namespace ivf {

// The cache: slot t is place t & (page - 1) of page t >> page_shift.  Offsets count elements.
struct CacheView {
    void* k;
    void* v;
    int64_t page_stride, token_stride, head_stride;
    int page_shift, page_bytes, token_bytes;
};

struct StepView {
    const int32_t *q_off, *len, *table, *group_off, *prefix_len, *prefix_table;
    int64_t table_stride, prefix_stride;
    int64_t own_cap, prefix_cap;         // keys that a row of the tables can name, at most 2^30 - 1024
    int64_t own_entries;                 // entries that lie in the cache
    int n_seq, n_tokens, n_groups, shift, prefix_shift;
    int own_last, prefix_last;           // the last own entry, and the last prefix entry, that lies in the cache
};

// The powers of two of a quantised cache.  Strides count bytes.
struct QuantView {
    uint8_t* k;
    uint8_t* v;
    int64_t page_stride, token_stride, head_stride;
    int least, most;                     // bytes that stand for powers of the rows' type
};

// Checks the caller's structures and fills the views; a status, with the error text set.  `qv`: filled for a quantised cache.
int make_views(const ivf_kv_step* step, const ivf_kv_cache* cache, CacheView* cv, StepView* sv, QuantView* qv);
// Checks the rows of `what`: pointer, alignment and strides.
int check_rows(const ivf_rows* r, const char* what);
// A launch has fewer than 2^32 threads.
inline bool too_many_threads(int64_t workgroups, int threads) { return workgroups > (int64_t)UINT32_MAX / threads; }

namespace dev {

__device__ __forceinline__ int clamp_len(int n, int64_t cap) { return n < 0 ? 0 : (int64_t)n > cap ? (int)cap : n; }

// First token of sequence s; q_off is taken into 0 .. n_tokens.
__device__ __forceinline__ int token_of(const StepView& st, int s) { return min(max(st.q_off[s], 0), st.n_tokens); }
__device__ __forceinline__ int own_len(const StepView& st, int s) { return clamp_len(st.len[s], st.own_cap); }

// Group of sequence s, -1 where it is in none: the last group that starts at or before it.
__device__ __forceinline__ int group_of(const StepView& st, int s) {
    if (st.n_groups == 0 || s < st.group_off[0] || s >= st.group_off[st.n_groups]) return -1;
    int lo = 0, hi = st.n_groups;              // group_off[lo] <= s < group_off[hi]
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (st.group_off[mid] <= s) lo = mid; else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ int prefix_of(const StepView& st, int g) {
    return g < 0 ? 0 : clamp_len(st.prefix_len[g], st.prefix_cap);
}

__device__ __forceinline__ int64_t slot_offset(const CacheView& c, int64_t slot) {
    return (slot >> c.page_shift) * c.page_stride + (slot & ((1ll << c.page_shift) - 1)) * c.token_stride;
}

__device__ __forceinline__ int64_t scale_offset(const CacheView& c, const QuantView& q, int64_t slot) {
    return (slot >> c.page_shift) * q.page_stride + (slot & ((1ll << c.page_shift) - 1)) * q.token_stride;
}
// 2^e of a byte e + 127
__device__ __forceinline__ float power_of(const QuantView& q, int byte) {
    return __uint_as_float((uint32_t)min(max(byte, q.least), q.most) << 23);
}

// Two e4m3 numbers times a power of two, in T
template <typename T, bool HIGH> __device__ __forceinline__ uint32_t from_e4m3(uint32_t code, float power) {
    if constexpr (std::is_same<T, _Float16>::value) return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(code, power, HIGH));
    else return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(code, power, HIGH));
}

// Slot of key j of sequence s, group g, whose prefix has plen keys: taken into the cache
__device__ __forceinline__ int64_t slot_of_key(const StepView& st, int s, int g, int plen, int j) {
    if (j < plen) {
        const int e = st.prefix_table[g * st.prefix_stride + (j >> st.prefix_shift)];
        return ((int64_t)min(max(e, 0), st.prefix_last) << st.prefix_shift) + (j & ((1 << st.prefix_shift) - 1));
    }
    j -= plen;
    const int e = st.table[s * st.table_stride + (j >> st.shift)];
    return ((int64_t)min(max(e, 0), st.own_last) << st.shift) + (j & ((1 << st.shift) - 1));
}

}  // namespace dev
}  // namespace ivf
