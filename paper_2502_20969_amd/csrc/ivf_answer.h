// Shared by the operators of answering from retrieved passages (ivf_kv.hip, ivf_attend.hip, ivf_beam.hip): the
// paged cache and the sequences of a step as the kernels see them.
#pragma once
#include "../../include/ivf.h"
#include "ivf_internal.h"

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

// Checks the caller's structures and fills the views; a status, with the error text set.
int make_views(const ivf_kv_step* step, const ivf_kv_cache* cache, CacheView* cv, StepView* sv);
// Checks the rows of `what`: pointer, alignment and strides.
int check_rows(const ivf_rows* r, const char* what);

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

}  // namespace dev
}  // namespace ivf
