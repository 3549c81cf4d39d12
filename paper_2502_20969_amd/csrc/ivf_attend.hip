// Attention of a step's new tokens over the paged cache: how a call is cut into passes, and its entry points.  The kernels are in
// ivf_attend.h; those of quantised caches are built in ivf_attend_quant.hip.
#include "ivf_attend.h"

namespace ivf {

static int check_heads(const ivf_kv_cache* cache, int n_q_heads, int window, int sinks) {
    if (cache->d != 64 && cache->d != 96 && cache->d != 128 && cache->d != 256)
        return fail(IVF_ELIMIT, "d must be 64, 96, 128 or 256 (got %d)", cache->d);
    if (n_q_heads < 1 || n_q_heads % cache->n_heads != 0)
        return fail(IVF_EINVAL, "n_q_heads (%d) must be a multiple of the cache's heads (%d)", n_q_heads, cache->n_heads);
    if (window < 0 || sinks < 0) return fail(IVF_EINVAL, "window and sinks must not be negative");
    return IVF_OK;
}

static AttendPlan plan_attend(const ivf_kv_step* st, const StepView& sv, int hkv, int group, int d, int window, int sinks) {
    AttendPlan p{};
    const int64_t rows = (int64_t)sv.n_tokens * group;
    auto known = [](int hint, int64_t cap) { return hint > 0 ? std::min<int64_t>(hint, cap) : cap; };
    const int64_t len = known(st->max_len, sv.own_cap), pre = sv.n_groups > 0 ? known(st->max_prefix, sv.prefix_cap) : 0;
    const int64_t most_q = std::max<int64_t>(known(st->max_q, sv.n_tokens), (sv.n_tokens + sv.n_seq - 1) / sv.n_seq);
    // a pass of its own for the prefix costs a launch and partial sums, and saves the prefix's keys of all sequences but one: worth it
    // from some hundred keys on (16 groups of 4, 8 key heads of 128: prefixes of 128 keys 39.7 us with it, 31.6 without; of 500 44.8 and
    // 43.5; of 2000 55 and 73)
    p.shared = pre >= 512 && sv.n_seq > sv.n_groups && rows < (int64_t)sv.n_seq * kWideRows;
    const int64_t keys_all = p.shared ? len : len + pre;
    // keys that a row reads: of a window a tile more
    auto read_keys = [&](int64_t keys) { return window > 0 ? std::min<int64_t>(keys, (int64_t)window + std::min<int64_t>(sinks, keys) + most_q + 64) : keys; };
    const int64_t keys = read_keys(keys_all);
    p.wide = sv.n_seq == 1 ? rows > kNarrowRows : most_q * group > kNarrowRows;
    // where the sequences have about as many tokens each, none or few have few rows: not worth a launch of their own and the joining
    // that its split brings (34 prompts of 361 to 1085 tokens: 103 us with it, 69 without)
    p.narrow = !p.wide || rows < (int64_t)sv.n_seq * most_q * group / 2;
    auto split = [](int64_t units, int64_t want, int64_t keys, int64_t least) {
        const int64_t most = (keys + least - 1) / least;
        return (int)std::max<int64_t>(1, std::min<int64_t>({(want + units - 1) / units, most, 64}));
    };
    // few rows: pieces of 1024 keys and more for several workgroups a place on the chip (two fit a compute unit), smaller ones
    // only while places are free (64 windows of 4096: pieces of 512 keys 214 us, of 1024 204; one token over 700 keys needs the small ones)
    auto split_few = [&](int64_t units, int64_t keys) { return std::max(split(units, 4096, keys, 1024), split(units, 512, keys, 128)); };
    // many rows: only as far as places are free, since every piece more is 2 x 4 d bytes a row written and read, and in pieces that
    // outweigh the joining (6 prompts, 1840 keys, 2 key heads: one piece 50 us, two 36; 18 prompts, 1061 keys: 36 and 42)
    auto split_many = [](int64_t units, int64_t keys) { return (int)std::max<int64_t>(1, std::min<int64_t>({512 / units, keys / 768, 64})); };
    p.tiles_narrow = 1;
    // (unknown: twice what sequences of equal lengths would need)
    const int64_t tile_rows = st->max_q > 0 || sv.n_seq == 1 ? most_q * group : std::min(rows, 2 * rows / sv.n_seq);
    p.tiles_wide = (int)std::max<int64_t>(1, (tile_rows + kWideRows - 1) / kWideRows);
    // where most of these would find no rows, the sequences' tiles are counted out one behind the other instead (a prompt of 8000 tokens
    // among 63 single ones: 126,000 workgroups that only end, 897 us; counted out 738.  Prompts of 361 to 1085 tokens: 67.7 and 68.9)
    if (sv.n_seq * (int64_t)p.tiles_wide > 2 * (rows / kWideRows + sv.n_seq)) p.tiles_wide = 0;
    if (p.narrow) p.split_narrow = split_few((int64_t)sv.n_seq * hkv, keys);
    if (p.wide) p.split_wide = split_many(hkv * ((rows + kWideRows - 1) / kWideRows + sv.n_seq / 2), keys);
    p.n_own = p.wide ? p.split_wide : p.split_narrow;
    if (p.shared) {
        const int64_t group_rows = rows / sv.n_groups;
        p.prefix_narrow = group_rows <= kNarrowRows;
        const int tile = p.prefix_narrow ? kNarrowRows : kWideRows;
        p.tiles_prefix = (int)std::max<int64_t>(1, (group_rows + tile - 1) / tile);
        const int64_t units = (int64_t)sv.n_groups * hkv * p.tiles_prefix;
        p.split_prefix = p.prefix_narrow ? split_few(units, read_keys(pre)) : split(units, 512, read_keys(pre), 256);
        p.part_own = p.split_prefix;
    }
    // A workgroup of one wavefront where many have little to do, or where two wavefronts' tiles leave no room for another workgroup:
    // the start of one then hides behind the work of others (204 sequences of 1 to 5 tokens, a window of 10, 16 heads of 128: 58 us by
    // two wavefronts, 44 by one; 180 of up to 114 keys, heads of 256: 73 and 51).  Else two share the start and the end (24 sequences
    // of up to 60,000: 543 and 574)
    const int64_t piece = std::max(keys / std::max(1, p.split_narrow), p.shared && p.prefix_narrow ? read_keys(pre) / p.split_prefix : 0);
    p.one_wave = d > 64 && p.narrow && (int64_t)sv.n_seq * hkv * p.split_narrow >= 512 && (d > 128 || piece <= 256);
    p.parts = p.shared || p.n_own > 1 ? p.part_own + p.n_own : 0;
    // (with them among the others, a prompt of 16,000 tokens beside two single ones of 60,000 keys took 16 GB of workspace for the
    // pieces of the two; apart 24 MB)
    if (p.narrow && p.wide && (p.shared || p.split_narrow > 1)) p.few_tokens = std::max(1, kNarrowRows / group);
    return p;
}

// partial sums of the tokens, and of the few's places
static int64_t plan_sums(const AttendPlan& p, int64_t n_tokens, int hq) { return n_tokens * hq * p.parts; }
static int64_t plan_few_sums(const AttendPlan& p, int64_t n_seq, int hq) { return n_seq * p.few_tokens * hq * p.split_narrow; }
static size_t plan_bytes(const AttendPlan& p, const StepView& sv, int hq, int d) {
    return (size_t)(plan_sums(p, sv.n_tokens, hq) + plan_few_sums(p, sv.n_seq, hq)) * ((size_t)d * 4 + 8);
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_attend_workspace(const ivf_kv_step* step, const ivf_kv_cache* cache, int32_t n_q_heads, int32_t window,
                                    int32_t sinks, size_t* bytes) {
    CacheView cv; StepView sv; QuantView qv;
    int rc = make_views(step, cache, &cv, &sv, &qv);
    if (rc) return rc;
    if ((rc = check_heads(cache, n_q_heads, window, sinks))) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    const AttendPlan p = plan_attend(step, sv, cache->n_heads, n_q_heads / cache->n_heads, cache->d, window, sinks);
    *bytes = plan_bytes(p, sv, n_q_heads, cache->d);
    return IVF_OK;
}

extern "C" int ivf_attend(const ivf_kv_step* step, const ivf_kv_cache* cache, const ivf_rows* q, int32_t n_q_heads,
                          const ivf_rows* out, float* lse, float scale, int32_t window, int32_t sinks, void* workspace,
                          size_t workspace_bytes, void* stream) {
    AttendArgs a{};
    int rc = make_views(step, cache, &a.cache, &a.step, &a.quant);
    if (rc) return rc;
    if ((rc = check_heads(cache, n_q_heads, window, sinks))) return rc;
    if ((rc = check_rows(q, "q")) || (rc = check_rows(out, "out"))) return rc;
    if (!(scale > 0.f) || scale > 1e30f) return fail(IVF_EINVAL, "scale must be positive");
    if (((uintptr_t)workspace & 15u) != 0) return fail(IVF_EINVAL, "workspace must be 16-byte aligned");
    a.q = *q; a.out = *out; a.lse = lse; a.scale_log2 = scale * 1.4426950408889634f;
    a.hq = n_q_heads; a.hkv = cache->n_heads; a.group = n_q_heads / cache->n_heads; a.window = window; a.sinks = sinks;
    const AttendPlan p = plan_attend(step, a.step, a.hkv, a.group, cache->d, window, sinks);
    const size_t need = plan_bytes(p, a.step, n_q_heads, cache->d);
    if (workspace_bytes < need || (need > 0 && !workspace))
        return fail(IVF_EINVAL, "this call needs %zu bytes of workspace (got %zu)", need, workspace ? workspace_bytes : (size_t)0);
    a.part_o = (float*)workspace;
    const int64_t sums = plan_sums(p, a.step.n_tokens, n_q_heads), few = plan_few_sums(p, a.step.n_seq, n_q_heads);
    a.few_o = a.part_o + sums * cache->d;
    a.part_ml = (float2*)(a.few_o + few * cache->d);
    a.few_ml = a.part_ml + sums;
    const hipStream_t s = (hipStream_t)stream;
    const hipError_t e = cache->dtype == IVF_E4M3  ? launch_attend_quant(a, p, cache->row_dtype, cache->d, s)
                         : cache->dtype == IVF_F16 ? launch_attend<_Float16, false>(a, p, cache->d, s)
                                                   : launch_attend<__bf16, false>(a, p, cache->d, s);
    HIP_TRY(e);
    return IVF_OK;
}
