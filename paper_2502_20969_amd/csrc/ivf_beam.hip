// A step of a beam search: the best continuations over beams and vocabulary, and the beams' states in their new order.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <algorithm>

namespace ivf {
using namespace dev;

struct BeamArgs {
    const void* logits;
    int64_t row_stride;
    const float* scores_in;
    const uint8_t* done_in;
    float* scores_out;
    int32_t *parent, *token;
    uint8_t* done_out;
    unsigned long long* keys;     // [rows][k] the row's best logits, best first, packed with their tokens; 0 = none
    float* lse;                   // [rows][2] maximum, and logarithm of the sum
    int prompts, beams, vocab, k, eos;
};

// A logit and its token as one word: larger is better, equal logits by lower token.  No continuation: 0.
__device__ __forceinline__ unsigned long long pack_logit(float x, uint32_t token) {
    if (!(x > -INFINITY)) return 0;                       // -inf and NaN
    x += 0.f;                                             // -0 is 0
    const uint32_t u = __float_as_uint(x);
    return (unsigned long long)(u & 0x80000000u ? ~u : u | 0x80000000u) << 32 | ~token;
}
__device__ __forceinline__ float logit_of(unsigned long long key) {
    const uint32_t u = (uint32_t)(key >> 32);
    return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}

__device__ __forceinline__ unsigned long long block_max(unsigned long long x, unsigned long long* s) {
    for (int w = 32; w >= 1; w >>= 1) x = max(x, (unsigned long long)__shfl_xor((long long)x, w));
    __syncthreads();
    if (lane_id() == 0) s[wave_id()] = x;
    __syncthreads();
    for (int i = 0; i < 4; ++i) x = max(x, s[i]);
    return x;
}

// One workgroup per row: the maximum, the sum, then the k best, one pass over the row each.
template <typename T>
__global__ __launch_bounds__(256) void beam_rows_kernel(BeamArgs a) {
    __shared__ unsigned long long s_best[4];
    __shared__ float s_sum[4];
    const int row = blockIdx.x, tid = threadIdx.x;
    const T* x = (const T*)a.logits + row * a.row_stride;
    unsigned long long last = ~0ull;
    float top = 0.f;
    for (int i = 0; i < a.k; ++i) {
        unsigned long long best = 0;
        for (int t = tid; t < a.vocab; t += 256) {
            const unsigned long long key = pack_logit((float)x[t], t);
            if (key < last) best = max(best, key);
        }
        last = block_max(best, s_best);
        if (i == 0) top = logit_of(last);
        if (tid == 0) a.keys[(int64_t)row * a.k + i] = last;
        if (last == 0) {
            for (int j = i + 1 + tid; j < a.k; j += 256) a.keys[(int64_t)row * a.k + j] = 0;
            break;
        }
    }
    float sum = 0.f;
    for (int t = tid; t < a.vocab; t += 256) {
        const float v = (float)x[t];
        if (v > -INFINITY) sum += v == top ? 1.f : expf(v - top);
    }
    sum = group_sum<64>(sum);
    if (lane_id() == 0) s_sum[wave_id()] = sum;
    __syncthreads();
    if (tid == 0) {
        a.lse[row * 2] = top;
        a.lse[row * 2 + 1] = logf(s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3]);
    }
}

// One wavefront per prompt: k times the best candidate of the rows' lists, a lane per row.
__global__ __launch_bounds__(64) void beam_pick_kernel(BeamArgs a) {
    const int prompt = blockIdx.x, b = threadIdx.x, row0 = prompt * a.beams, row = row0 + b;
    const bool mine = b < a.beams;
    const bool done = mine && a.done_in && a.done_in[row];
    const float run = mine ? a.scores_in[row] : -INFINITY;
    int at = 0;
    for (int i = 0; i < a.k; ++i) {
        float score = -INFINITY;
        int token = -1;
        if (mine && at < a.k) {
            if (done) {
                if (at == 0) { score = run; token = a.eos; }
            } else {
                const unsigned long long key = a.keys[(int64_t)row * a.k + at];
                const float v = logit_of(key), top = a.lse[row * 2];
                if (key) { score = run + ((v == top ? 0.f : v - top) - a.lse[row * 2 + 1]); token = (int)~(uint32_t)key; }
            }
        }
        if (!(score > -INFINITY)) token = -1;
        float best = token >= 0 || (done && at == 0 && score > -INFINITY) ? score : -INFINITY;
        float top = best;
        for (int w = 32; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
        const uint64_t at_top = __ballot(best == top && best > -INFINITY);
        const int from = at_top ? __builtin_ctzll(at_top) : 0;
        const int o = prompt * a.k + i;
        if (b == from) {
            a.scores_out[o] = at_top ? score : -INFINITY;
            a.parent[o] = row0 + from;
            a.token[o] = at_top ? token : -1;
            a.done_out[o] = !at_top || done || token == a.eos;
            ++at;
        }
    }
}

struct BeamMove {
    const uint8_t* from;
    uint8_t* to;
    int64_t row_bytes, from_stride, to_stride;
};
struct BeamMoves { BeamMove m[IVF_MAX_BEAM_STATES]; };

// Rows of the states to their new places, one workgroup per row and state.
__global__ __launch_bounds__(256) void beam_move_kernel(BeamMoves moves, const int32_t* parent) {
    const BeamMove& m = moves.m[blockIdx.y];
    const uint8_t* from = m.from + parent[blockIdx.x] * m.from_stride;
    uint8_t* to = m.to + (int64_t)blockIdx.x * m.to_stride;
    const bool wide = (((uintptr_t)from | (uintptr_t)to) & 15u) == 0;
    const int64_t n = wide ? m.row_bytes / 16 : 0;
    for (int64_t i = threadIdx.x; i < n; i += 256) ((uint4*)to)[i] = ((const uint4*)from)[i];
    for (int64_t i = n * 16 + threadIdx.x; i < m.row_bytes; i += 256) to[i] = from[i];
}

static int check_beams(int n_prompts, int beams_in, int vocab, int beams_out) {
    if (n_prompts < 1 || beams_in < 1 || vocab < 1 || beams_out < 1)
        return fail(IVF_EINVAL, "n_prompts, beams_in, vocab and beams_out must be at least 1");
    if (beams_in > IVF_MAX_BEAMS || beams_out > IVF_MAX_BEAMS)
        return fail(IVF_ELIMIT, "%d beams in, %d out: at most %d", beams_in, beams_out, IVF_MAX_BEAMS);
    if ((int64_t)n_prompts * std::max(beams_in, beams_out) > (1 << 24)) return fail(IVF_ELIMIT, "%d prompts of %d beams", n_prompts, beams_in);
    return IVF_OK;
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_beam_workspace(int32_t n_prompts, int32_t beams_in, int32_t vocab, int32_t beams_out, size_t* bytes) {
    int rc = check_beams(n_prompts, beams_in, vocab, beams_out);
    if (rc) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    const size_t rows = (size_t)n_prompts * beams_in;
    *bytes = rows * beams_out * 8 + rows * 8;
    return IVF_OK;
}

extern "C" int ivf_beam_step(const void* logits, int64_t row_stride, int dtype, int32_t n_prompts, int32_t beams_in, int32_t vocab,
                             const float* scores_in, const uint8_t* done_in, int32_t eos, int32_t beams_out, float* scores_out,
                             int32_t* parent, int32_t* token, uint8_t* done_out, const ivf_beam_state* states, int32_t n_states,
                             void* workspace, size_t workspace_bytes, void* stream) {
    size_t need = 0;
    int rc = ivf_beam_workspace(n_prompts, beams_in, vocab, beams_out, &need);
    if (rc) return rc;
    if (!logits || !scores_in || !scores_out || !parent || !token || !done_out) return fail(IVF_EINVAL, "logits, scores or an output is NULL");
    if (dtype != IVF_F32 && dtype != IVF_F16 && dtype != IVF_BF16) return fail(IVF_EINVAL, "unknown dtype %d", dtype);
    if (row_stride < vocab) return fail(IVF_EINVAL, "row_stride (%lld) is below vocab (%d)", (long long)row_stride, vocab);
    if (((uintptr_t)logits & (dtype == IVF_F32 ? 3u : 1u)) != 0) return fail(IVF_EINVAL, "logits must be aligned to their elements");
    if (n_states < 0 || (n_states > 0 && !states)) return fail(IVF_EINVAL, "states is NULL or n_states negative");
    if (n_states > IVF_MAX_BEAM_STATES) return fail(IVF_ELIMIT, "%d states: at most %d", n_states, IVF_MAX_BEAM_STATES);
    BeamMoves moves{};
    for (int i = 0; i < n_states; ++i) {
        const ivf_beam_state& s = states[i];
        if (!s.from || !s.to) return fail(IVF_EINVAL, "state %d: NULL", i);
        if (s.row_bytes < 1 || s.from_stride < 0 || s.to_stride < s.row_bytes) return fail(IVF_EINVAL, "state %d: row_bytes or strides", i);
        moves.m[i] = BeamMove{(const uint8_t*)s.from, (uint8_t*)s.to, s.row_bytes, s.from_stride, s.to_stride};
    }
    if (!workspace || ((uintptr_t)workspace & 15u) != 0) return fail(IVF_EINVAL, "workspace must be given and 16-byte aligned");
    if (workspace_bytes < need) return fail(IVF_EINVAL, "this call needs %zu bytes of workspace (got %zu)", need, workspace_bytes);
    const int rows = n_prompts * beams_in;
    BeamArgs a{logits, row_stride, scores_in, done_in, scores_out, parent, token, done_out, (unsigned long long*)workspace,
               (float*)((unsigned long long*)workspace + (size_t)rows * beams_out), n_prompts, beams_in, vocab, beams_out, eos};
    hipStream_t s = (hipStream_t)stream;
    if (dtype == IVF_F32) hipLaunchKernelGGL(beam_rows_kernel<float>, dim3(rows), dim3(256), 0, s, a);
    else if (dtype == IVF_F16) hipLaunchKernelGGL(beam_rows_kernel<_Float16>, dim3(rows), dim3(256), 0, s, a);
    else hipLaunchKernelGGL(beam_rows_kernel<__bf16>, dim3(rows), dim3(256), 0, s, a);
    hipLaunchKernelGGL(beam_pick_kernel, dim3(n_prompts), dim3(64), 0, s, a);
    if (n_states > 0) hipLaunchKernelGGL(beam_move_kernel, dim3(n_prompts * beams_out, n_states), dim3(256), 0, s, moves, parent);
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
