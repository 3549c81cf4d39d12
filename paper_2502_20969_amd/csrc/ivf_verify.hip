// Verification of drafted tokens against the target's probabilities, and the token that follows the accepted ones.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <math.h>

namespace ivf {
using namespace dev;

struct VerifyArgs {
    StepView step;               // q_off, len, n_seq and n_tokens
    const void* logits;
    int64_t row_stride, draft_stride;
    const int32_t* tokens;
    const float *uniform, *draft;
    int32_t *accepted, *follows, *len_out;
    int vocab;
    float scale;                 // 0: the largest entry alone counts
    struct Row { double sum; float top; int32_t best; };
    Row* rows;                   // [n_tokens] largest entry, its token (-1: none), and sum of exp(scale (x - top))
};

constexpr int kVerifyThreads = 256;

template <typename T> __device__ __forceinline__ float entry_of(const void* logits, int64_t at) {
    const float x = (float)((const T*)logits)[at];
    return x == x ? x : -INFINITY;
}
// The weight of an entry of a row whose largest is `top`: probabilities are weights over their sum
__device__ __forceinline__ double weight_of(float x, float top, float scale) {
    if (x == -INFINITY) return 0.0;
    if (top == INFINITY) return x == INFINITY ? 1.0 : 0.0;
    return exp((double)scale * ((double)x - (double)top));
}

__device__ __forceinline__ double block_sum(double x, double* s_part) {
    for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
    __syncthreads();
    if (lane_id() == 0) s_part[wave_id()] = x;
    __syncthreads();
    double all = 0.0;
    for (int w = 0; w < kVerifyThreads / 64; ++w) all += s_part[w];
    return all;
}

// One workgroup per row: its largest entry and the sum of the weights.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_rows_kernel(VerifyArgs a) {
    __shared__ double s_part[kVerifyThreads / 64];
    __shared__ unsigned long long s_best;
    const int t = blockIdx.x;
    const int64_t at = t * a.row_stride;
    unsigned long long best = 0;                            // larger entries first, then lower tokens; 0: none
    for (int i = threadIdx.x; i < a.vocab; i += kVerifyThreads) {
        const float x = entry_of<T>(a.logits, at + i) + 0.f;
        const uint32_t u = __float_as_uint(x);
        if (x > -INFINITY) best = max(best, (unsigned long long)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~(uint32_t)i);
    }
    if (threadIdx.x == 0) s_best = 0;
    __syncthreads();
    atomicMax(&s_best, best);
    __syncthreads();
    best = s_best;
    const uint32_t u = (uint32_t)(best >> 32);
    const float top = best ? __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u) : -INFINITY;
    double sum = 0.0;
    if (a.scale > 0.f)
        for (int i = threadIdx.x; i < a.vocab; i += kVerifyThreads) sum += weight_of(entry_of<T>(a.logits, at + i), top, a.scale);
    sum = block_sum(sum, s_part);
    if (threadIdx.x == 0) a.rows[t] = VerifyArgs::Row{sum, top, best ? (int32_t)~(uint32_t)best : -1};
}

// One workgroup per sequence: the accepted drafts, and the token that follows.
template <typename T>
__global__ __launch_bounds__(kVerifyThreads) void verify_pick_kernel(VerifyArgs a) {
    __shared__ double s_part[kVerifyThreads / 64], s_all[kVerifyThreads];
    __shared__ int s_accepted;
    const int s = blockIdx.x, t0 = token_of(a.step, s), count = max(0, token_of(a.step, s + 1) - t0);
    if (threadIdx.x == 0) {
        int n = 0;
        for (; n + 1 < count; ++n) {
            const int t = t0 + n + 1, token = a.tokens[t];
            if (token < 0 || token >= a.vocab) break;
            const VerifyArgs::Row row = a.rows[t - 1];
            if (a.scale == 0.f) {
                if (token != row.best) break;
                continue;
            }
            const float d = a.draft ? a.draft[t * a.draft_stride + token] : 1.f;
            const double w = weight_of(entry_of<T>(a.logits, (t - 1) * a.row_stride + token), row.top, a.scale);
            if (!((double)a.uniform[t] * (double)(d > 0.f ? d : 0.f) * row.sum < w)) break;
        }
        s_accepted = n;
        a.accepted[s] = n;
        a.len_out[s] = a.step.len[s] - max(0, count - 1 - n);
    }
    __syncthreads();
    const int n = s_accepted, t = t0 + n;
    if (count == 0 || a.scale == 0.f) {
        if (threadIdx.x == 0) a.follows[s] = count == 0 ? -1 : a.rows[t].best;
        return;
    }
    const VerifyArgs::Row row = a.rows[t];
    const bool refused = n + 1 < count;
    const int not_this = refused && !a.draft ? a.tokens[t + 1] : -1;
    bool less = refused;
    auto left = [&](int i) {
        const double w = weight_of(entry_of<T>(a.logits, t * a.row_stride + i), row.top, a.scale);
        if (!less) return w;
        if (!a.draft) return i == not_this ? 0.0 : w;
        const float d = a.draft[(t + 1) * a.draft_stride + i];
        return fmax(w - row.sum * (double)(d > 0.f ? d : 0.f), 0.0);
    };
    // a thread takes a run of tokens
    const int per = (a.vocab + kVerifyThreads - 1) / kVerifyThreads, i0 = min(a.vocab, (int)threadIdx.x * per), i1 = min(a.vocab, i0 + per);
    double mine = 0.0, all;
    for (int tries = 0; tries < 2; ++tries) {
        mine = 0.0;
        for (int i = i0; i < i1; ++i) mine += left(i);
        all = block_sum(mine, s_part);
        if (all > 0.0) break;
        less = false;
    }
    s_all[threadIdx.x] = mine;
    __syncthreads();
    if (threadIdx.x != 0) return;
    double run = 0.0;
    int token = -1;
    const double reach = (double)a.uniform[t0] * all;
    for (int p = 0; p < kVerifyThreads && token < 0; ++p) {
        if (!(run + s_all[p] > reach) && !(s_all[p] > 0.0)) continue;
        // the run that holds it; where rounding lets none be above, the last token of any weight
        bool last = true;
        for (int q = p + 1; q < kVerifyThreads; ++q) last = last && !(s_all[q] > 0.0);
        if (run + s_all[p] > reach || last) {
            double at = run;
            for (int i = p * per; i < min(a.vocab, (p + 1) * per); ++i) {
                const double w = left(i);
                if (!(w > 0.0)) continue;
                token = i;
                at += w;
                if (at > reach) break;
            }
        }
        run += s_all[p];
    }
    a.follows[s] = token;
}

static int check_verify(int n_seq, int n_tokens, int vocab) {
    if (n_seq < 1 || n_tokens < 1 || vocab < 1) return fail(IVF_EINVAL, "n_seq, n_tokens and vocab must be at least 1");
    if (vocab > 1 << 30) return fail(IVF_ELIMIT, "vocab = %d is above 2^30", vocab);
    if (n_seq > 1 << 24 || n_tokens > 1 << 24) return fail(IVF_ELIMIT, "%d sequences, %d tokens: at most 2^24", n_seq, n_tokens);
    return IVF_OK;
}

template <typename T> static void launch_verify(const VerifyArgs& a, hipStream_t s) {
    hipLaunchKernelGGL(verify_rows_kernel<T>, dim3(a.step.n_tokens), dim3(kVerifyThreads), 0, s, a);
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3(a.step.n_seq), dim3(kVerifyThreads), 0, s, a);
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_verify_workspace(int32_t n_seq, int32_t n_tokens, int32_t vocab, size_t* bytes) {
    int rc = check_verify(n_seq, n_tokens, vocab);
    if (rc) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    *bytes = (size_t)n_tokens * sizeof(VerifyArgs::Row);
    return IVF_OK;
}

extern "C" int ivf_verify_draft(const ivf_kv_step* step, const void* logits, int64_t row_stride, int dtype, int32_t vocab, float scale,
                                const int32_t* tokens, const float* uniform, const float* draft, int64_t draft_stride, int32_t* accepted,
                                int32_t* follows, int32_t* len_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!step) return fail(IVF_EINVAL, "step is NULL");
    if (!step->q_off || !step->len) return fail(IVF_EINVAL, "q_off or len is NULL");
    size_t need = 0;
    int rc = ivf_verify_workspace(step->n_seq, step->n_tokens, vocab, &need);
    if (rc) return rc;
    if (!logits || !tokens || !accepted || !follows || !len_out) return fail(IVF_EINVAL, "logits, tokens or an output is NULL");
    if (dtype != IVF_F32 && dtype != IVF_F16 && dtype != IVF_BF16) return fail(IVF_EINVAL, "unknown dtype %d", dtype);
    if (!(scale >= 0.f) || scale > 1e30f) return fail(IVF_EINVAL, "scale must not be negative");
    if (scale > 0.f && !uniform) return fail(IVF_EINVAL, "uniform is NULL");
    if (row_stride < vocab) return fail(IVF_EINVAL, "row_stride (%lld) is below vocab (%d)", (long long)row_stride, vocab);
    if (draft && draft_stride < vocab) return fail(IVF_EINVAL, "draft_stride (%lld) is below vocab (%d)", (long long)draft_stride, vocab);
    if (((uintptr_t)logits & (dtype == IVF_F32 ? 3u : 1u)) != 0 || ((uintptr_t)draft & 3u) != 0)
        return fail(IVF_EINVAL, "logits and draft must be aligned to their elements");
    if (accepted == follows || accepted == len_out || follows == len_out) return fail(IVF_EINVAL, "outputs must not be the same array");
    for (const void* in : {(const void*)step->q_off, (const void*)tokens, (const void*)uniform})
        if (in && (in == accepted || in == follows || in == len_out)) return fail(IVF_EINVAL, "an output is an input");
    if (accepted == step->len || follows == step->len) return fail(IVF_EINVAL, "an output is an input");
    if (!workspace || ((uintptr_t)workspace & 15u) != 0) return fail(IVF_EINVAL, "workspace must be given and 16-byte aligned");
    if (workspace_bytes < need) return fail(IVF_EINVAL, "this call needs %zu bytes of workspace (got %zu)", need, workspace_bytes);
    VerifyArgs a{};
    a.step.q_off = step->q_off; a.step.len = step->len; a.step.n_seq = step->n_seq; a.step.n_tokens = step->n_tokens;
    a.logits = logits; a.row_stride = row_stride; a.draft = draft; a.draft_stride = draft_stride; a.tokens = tokens; a.uniform = uniform;
    a.accepted = accepted; a.follows = follows; a.len_out = len_out; a.vocab = vocab; a.scale = scale;
    a.rows = (VerifyArgs::Row*)workspace;
    hipStream_t s = (hipStream_t)stream;
    if (dtype == IVF_F32) launch_verify<float>(a, s);
    else if (dtype == IVF_F16) launch_verify<_Float16>(a, s);
    else launch_verify<__bf16>(a, s);
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
