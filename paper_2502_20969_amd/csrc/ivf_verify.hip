// Verification of drafted tokens against the target's probabilities, and the token that follows the accepted ones.
//
//   p = w / W,  w_i = 2^(c (x_i - top)),  c = scale log2(e),  W = sum_i w_i
//
// in 64 bits: the token that follows is where a running sum over the vocabulary passes u times its whole, and with 131,072 steps such a sum
// of 32-bit terms would put one draw in a hundred on another token.  The logits are read once, a tile to a wavefront, which leaves
// the tile's largest entry and its sum of weights relative to that; a row's (top, W) are those of its tiles joined.  A draw looks for the
// tile, the run of entries inside it, and the entry in turn.  Only a refused draft that was drawn from probabilities needs a second pass
// over its row, for the sums of max(w - W d, 0).
#include "ivf_answer.h"
#include "ivf_device.h"
#include <math.h>

namespace ivf {
using namespace dev;

// Of a tile: its largest entry (-inf: none), and the sum of its weights relative to that, or the largest's token where scale is 0
struct VerifyTile {
    double sum;
    float top;
    int32_t best;
};
struct VerifyArgs {
    StepView step;               // q_off, len, n_seq and n_tokens
    const void* logits;
    int64_t row_stride, draft_stride;
    const int32_t* tokens;
    const float *uniform, *draft;
    int32_t *accepted, *follows, *len_out;
    VerifyTile* tiles;           // [n_tokens][n_tile]
    double* left;                // [n_seq][n_tile] sums of max(w - W d, 0)
    uint32_t* ticket;            // [n_seq] workgroups that have left theirs
    double rise;                 // scale * log2(e); 0: the largest entry alone counts
    int vocab, n_tile;
};

constexpr int kVerifyWaves = 4;
constexpr int kVerifyRun = 32;                            // entries of a lane
constexpr int kVerifyTile = 64 * kVerifyRun;
constexpr int kVerifyRows = 32;                           // rows of a sequence whose (top, W) are kept in LDS

// 2^y in 64 bits, 0 below the smallest number: the series of exp(f ln 2) around the nearest whole number, f within 1/2, off by (0.35)^12 /
// 12! = 6e-15 at most
__device__ __forceinline__ double exp2_64(double y) {
    y = fmax(y, -2000.0);
    const double n = rint(y), f = y - n;
    constexpr double kLn2 = 0.693147180559945309417;
    constexpr double c1 = kLn2, c2 = c1 * kLn2 / 2, c3 = c2 * kLn2 / 3, c4 = c3 * kLn2 / 4, c5 = c4 * kLn2 / 5, c6 = c5 * kLn2 / 6, c7 = c6 * kLn2 / 7,
                     c8 = c7 * kLn2 / 8, c9 = c8 * kLn2 / 9, c10 = c9 * kLn2 / 10, c11 = c10 * kLn2 / 11;
    double p = __builtin_fma(c11, f, c10);
    p = __builtin_fma(p, f, c9);
    p = __builtin_fma(p, f, c8);
    p = __builtin_fma(p, f, c7);
    p = __builtin_fma(p, f, c6);
    p = __builtin_fma(p, f, c5);
    p = __builtin_fma(p, f, c4);
    p = __builtin_fma(p, f, c3);
    p = __builtin_fma(p, f, c2);
    p = __builtin_fma(p, f, c1);
    p = __builtin_fma(p, f, 1.0);
    return __builtin_amdgcn_ldexp(p, (int)n);
}

template <typename T> __device__ __forceinline__ float entry_of(const void* logits, int64_t at) {
    const float x = (float)((const T*)logits)[at];
    return x == x ? x : -INFINITY;
}
// The weight of an entry relative to `top`, a finite number or +inf (then the entries that are, alone)
__device__ __forceinline__ double weight_of(float x, float top, double rise) {
    if (top == INFINITY) return x == INFINITY ? 1.0 : 0.0;
    return exp2_64(rise * ((double)x - (double)top));     // 0 for -inf, and NaN
}

template <typename V> __device__ __forceinline__ V lanes_sum(V x) {
    for (int w = 32; w >= 1; w >>= 1) x += __shfl_xor(x, w);
    return x;
}
__device__ __forceinline__ float lanes_max(float x) {
    for (int w = 32; w >= 1; w >>= 1) x = fmaxf(x, __shfl_xor(x, w));
    return x;
}
// sums over the lanes up to this one
__device__ __forceinline__ double lanes_prefix(double x) {
    const int lane = lane_id();
    for (int w = 1; w < 64; w <<= 1) {
        const double y = __shfl_up(x, w);
        if (lane >= w) x += y;
    }
    return x;
}

// 16 bytes of entries from any element
typedef u4_t u4_any_t __attribute__((aligned(2)));
template <typename T> constexpr int kPerLoad = 16 / (int)sizeof(T);
template <typename T> __device__ __forceinline__ float unpack(const u4_t& v, int e) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[e]);
    else if constexpr (std::is_same<T, _Float16>::value) return (float)__builtin_bit_cast(_Float16, (uint16_t)(v[e / 2] >> (16 * (e & 1))));
    else return __uint_as_float(e & 1 ? v[e / 2] & 0xFFFF0000u : v[e / 2] << 16);
}

// A wavefront per tile: its largest entry, then its weights, from registers.  Entry e of load i of a lane is entry (i * 64 + lane) * kPerLoad + e.
template <typename T>
__global__ __launch_bounds__(kVerifyWaves * 64) void verify_tiles_kernel(VerifyArgs a) {
    constexpr int kPer = kPerLoad<T>, kLoads = kVerifyRun / kPer;
    for (int64_t i = (int64_t)blockIdx.x * (kVerifyWaves * 64) + threadIdx.x; i < a.step.n_seq; i += (int64_t)gridDim.x * (kVerifyWaves * 64)) a.ticket[i] = 0;
    const int lane = lane_id(), per_row = (a.n_tile + kVerifyWaves - 1) / kVerifyWaves;
    const int row = blockIdx.x / per_row, tile = blockIdx.x % per_row * kVerifyWaves + wave_id();
    if (tile >= a.n_tile) return;
    const T* x = (const T*)a.logits + row * a.row_stride;
    const int i0 = tile * kVerifyTile + lane * kPer;
    float v[kVerifyRun], top = -INFINITY;
    u4_t raw[kLoads];
    if ((tile + 1) * kVerifyTile <= a.vocab) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) raw[i] = *(const u4_any_t*)(x + i0 + i * 64 * kPer);
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) v[i] = unpack<T>(raw[i / kPer], i % kPer);
    } else {
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) {
            const int at = i0 + i / kPer * 64 * kPer + i % kPer;
            v[i] = at < a.vocab ? (float)x[at] : -INFINITY;
        }
    }
#pragma unroll
    for (int i = 0; i < kVerifyRun; ++i) top = fmaxf(top, v[i]);          // NaN counts for nothing
    top = lanes_max(top);
    VerifyTile out = {0.0, top, -1};
    if (a.rise == 0.0) {
        int best = 0x7FFFFFFF;
#pragma unroll
        for (int i = kVerifyRun - 1; i >= 0; --i)
            if (v[i] == top) best = i0 + i / kPer * 64 * kPer + i % kPer;
        for (int w = 32; w >= 1; w >>= 1) best = min(best, __shfl_xor(best, w));
        if (top > -INFINITY) out.best = best;
    } else if (top > -INFINITY) {
        double sum = 0.0;
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) sum += weight_of(v[i], top, a.rise);
        out.sum = lanes_sum(sum);
    }
    if (lane == 0) a.tiles[(int64_t)row * a.n_tile + tile] = out;
}

// A row's tiles joined, by a wavefront
__device__ __forceinline__ VerifyTile join_tiles(const VerifyArgs& a, int64_t row) {
    VerifyTile all = {0.0, -INFINITY, -1};
    const VerifyTile* tiles = a.tiles + row * a.n_tile;
    for (int i0 = 0; i0 < a.n_tile; i0 += 64) {
        const VerifyTile t = i0 + lane_id() < a.n_tile ? tiles[i0 + lane_id()] : VerifyTile{0.0, -INFINITY, -1};
        const float top = fmaxf(all.top, lanes_max(t.top));
        if (a.rise == 0.0) {
            if (top > all.top) all.best = __shfl(t.best, __builtin_ctzll(__ballot(t.top == top)));
        } else if (top > -INFINITY) {
            all.sum = all.sum * (all.top == -INFINITY ? 0.0 : weight_of(all.top, top, a.rise)) +
                      lanes_sum(t.top == -INFINITY ? 0.0 : t.sum * weight_of(t.top, top, a.rise));
        }
        all.top = top;
    }
    return all;
}

// The weights that a sequence's next token is drawn from
template <typename T> struct Weights {
    const VerifyArgs& a;
    int64_t logits, draft;                                // where the rows begin; draft -1: none
    int without;                                          // a token that is left out
    float top;
    double whole;
    __device__ __forceinline__ double operator()(int i) const {
        const double w = i == without ? 0.0 : weight_of(entry_of<T>(a.logits, logits + i), top, a.rise);
        if (draft < 0) return w;
        const float d = a.draft[draft + i];
        return fmax(w - whole * (double)(d > 0.f ? d : 0.f), 0.0);
    }
};

// By a wavefront: the first of n entries from i0 on at which the running sum, `run` before them, is above `reach`; the last of any weight where
// rounding lets none be; -1: no weight at all.
template <typename W> __device__ __forceinline__ int draw_in_tile(const W& weights, int i0, int n, double run, double reach) {
    const int lane = lane_id();
    double mine = 0.0;
    for (int i = lane * kVerifyRun; i < min(n, (lane + 1) * kVerifyRun); ++i) mine += weights(i0 + i);
    const double upto = run + lanes_prefix(mine);
    const uint64_t some = __ballot(mine > 0.0);
    if (!some) return -1;
    const uint64_t above = __ballot(mine > 0.0 && upto > reach);
    const int l = above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
    run = __shfl(upto - mine, l);
    // the lane's run, an entry a lane
    const int i = l * kVerifyRun + lane;
    const double w = lane < kVerifyRun && i < n ? weights(i0 + i) : 0.0;
    const double to = run + lanes_prefix(w);
    const uint64_t any = __ballot(w > 0.0), over = __ballot(w > 0.0 && to > reach);
    return i0 + l * kVerifyRun + (over ? __builtin_ctzll(over) : 63 - __builtin_clzll(any));
}

// The accepted drafts of a sequence, and the token that follows.  One workgroup, or, where a second pass over a row may be needed, one for every
// kVerifyWaves tiles, all of which find the same; the last one to leave its sums draws.
template <typename T>
__global__ __launch_bounds__(kVerifyWaves * 64) void verify_pick_kernel(VerifyArgs a, int parts) {
    __shared__ int s_refused;
    __shared__ uint32_t s_ticket;
    __shared__ VerifyTile s_row[kVerifyRows];
    const int s = blockIdx.x / parts, part = blockIdx.x % parts, lane = lane_id(), wave = wave_id();
    const int t0 = token_of(a.step, s), count = max(0, token_of(a.step, s + 1) - t0);
    if (threadIdx.x == 0) s_refused = max(1, count);
    __syncthreads();
    for (int i = wave; i < count; i += kVerifyWaves) {
        const VerifyTile row = join_tiles(a, t0 + i);
        if (i < kVerifyRows && lane == 0) s_row[i] = row;
        const int t = t0 + i + 1;
        if (i + 1 == count) break;
        const int token = a.tokens[t];
        bool ok = token >= 0 && token < a.vocab && row.top > -INFINITY;
        if (a.rise == 0.0) {
            ok = ok && token == row.best;
        } else if (ok) {
            const float d = a.draft ? a.draft[t * a.draft_stride + token] : 1.f;
            const double w = weight_of(entry_of<T>(a.logits, (t - 1) * a.row_stride + token), row.top, a.rise);
            ok = (double)a.uniform[t] * (double)(d > 0.f ? d : 0.f) * row.sum < w;
        }
        if (!ok && lane == 0) atomicMin(&s_refused, i + 1);
    }
    __syncthreads();
    const int n = s_refused - 1, t = t0 + n;
    const bool refused = n + 1 < count;
    if (part == 0 && threadIdx.x == 0) {
        a.accepted[s] = n;
        a.len_out[s] = a.step.len[s] - max(0, count - 1 - n);
    }
    const VerifyTile row = count == 0 ? VerifyTile{0.0, -INFINITY, -1} : n < kVerifyRows ? s_row[n] : join_tiles(a, t);
    const bool second = refused && a.draft && a.rise != 0.0 && row.top > -INFINITY;
    if (!second && part > 0) return;
    Weights<T> weights = {a, t * a.row_stride, -1, -1, row.top, row.sum};
    double* left = a.left + (int64_t)s * a.n_tile;
    if (second) {
        weights.draft = (t + 1) * a.draft_stride;
        const int tile = part * kVerifyWaves + wave;
        if (tile < a.n_tile) {
            double sum = 0.0;
            for (int i = tile * kVerifyTile + lane; i < min(a.vocab, (tile + 1) * kVerifyTile); i += 64) sum += weights(i);
            sum = lanes_sum(sum);
            if (lane == 0) left[tile] = sum;
        }
        if (parts > 1) {
            __threadfence();
            __syncthreads();
            if (threadIdx.x == 0) s_ticket = atomicAdd(&a.ticket[s], 1u);
            __syncthreads();
            if (s_ticket != (uint32_t)parts - 1) return;
            __threadfence();
        } else {
            __syncthreads();
        }
    }
    if (wave > 0) return;
    int token = -1;
    if (a.rise == 0.0) {
        token = row.best;
    } else if (row.top > -INFINITY) {
        const VerifyTile* tiles = a.tiles + (int64_t)t * a.n_tile;
        if (refused && !second) weights.without = a.tokens[t + 1];
        if (weights.without >= a.vocab) weights.without = -1;
        for (int tries = 0; tries < 2 && token < 0; ++tries) {           // where nothing is left, from p itself
            const bool from_left = second && tries == 0;
            if (tries == 1) { weights.draft = -1; weights.without = -1; }
            // the sum of the tile of the token that is left out, anew: less its weight it may lose what is left
            double anew = 0.0;
            const int at = weights.without < 0 ? -1 : weights.without / kVerifyTile;
            if (at >= 0) {
                for (int i = at * kVerifyTile + lane; i < min(a.vocab, (at + 1) * kVerifyTile); i += 64) anew += weights(i);
                anew = lanes_sum(anew);
            }
            auto sum_of = [&](int i) {
                if (i >= a.n_tile) return 0.0;
                if (from_left) return left[i];
                const VerifyTile x = tiles[i];
                return i == at ? anew : x.top == -INFINITY ? 0.0 : x.sum * weight_of(x.top, row.top, a.rise);
            };
            double whole = 0.0;
            for (int i0 = 0; i0 < a.n_tile; i0 += 64) whole += __shfl(lanes_prefix(sum_of(i0 + lane)), 63);
            if (!(whole > 0.0)) continue;
            const double reach = (double)a.uniform[t0] * whole;
            double run = 0.0, before = 0.0;
            int tile = -1;
            for (int i0 = 0; i0 < a.n_tile; i0 += 64) {
                const double mine = sum_of(i0 + lane), upto = run + lanes_prefix(mine);
                const uint64_t some = __ballot(mine > 0.0), above = __ballot(mine > 0.0 && upto > reach);
                if (some) {
                    const int l = above ? __builtin_ctzll(above) : 63 - __builtin_clzll(some);
                    tile = i0 + l;
                    before = __shfl(upto - mine, l);
                }
                if (above) break;
                run = __shfl(upto, 63);
            }
            token = draw_in_tile(weights, tile * kVerifyTile, min(kVerifyTile, a.vocab - tile * kVerifyTile), before, reach);
        }
    }
    if (lane == 0) a.follows[s] = token;
}

static int check_verify(int n_seq, int n_tokens, int vocab) {
    if (n_seq < 1 || n_tokens < 1 || vocab < 1) return fail(IVF_EINVAL, "n_seq, n_tokens and vocab must be at least 1");
    if (vocab > 1 << 30) return fail(IVF_ELIMIT, "vocab = %d is above 2^30", vocab);
    if (n_seq > 1 << 24 || n_tokens > 1 << 24) return fail(IVF_ELIMIT, "%d sequences, %d tokens: at most 2^24", n_seq, n_tokens);
    const int64_t blocks = (vocab + (int64_t)kVerifyTile * kVerifyWaves - 1) / (kVerifyTile * kVerifyWaves);
    if (blocks * n_seq > INT32_MAX || blocks * n_tokens > INT32_MAX)
        return fail(IVF_ELIMIT, "%d sequences, %d tokens over %d entries", n_seq, n_tokens, vocab);
    return IVF_OK;
}

template <typename T> static void launch_verify(const VerifyArgs& a, hipStream_t s) {
    const int per_row = (a.n_tile + kVerifyWaves - 1) / kVerifyWaves, parts = a.draft && a.rise != 0.0 ? per_row : 1;
    hipLaunchKernelGGL(verify_tiles_kernel<T>, dim3((unsigned)((int64_t)a.step.n_tokens * per_row)), dim3(kVerifyWaves * 64), 0, s, a);
    hipLaunchKernelGGL(verify_pick_kernel<T>, dim3((unsigned)((int64_t)a.step.n_seq * parts)), dim3(kVerifyWaves * 64), 0, s, a, parts);
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_verify_workspace(int32_t n_seq, int32_t n_tokens, int32_t vocab, size_t* bytes) {
    int rc = check_verify(n_seq, n_tokens, vocab);
    if (rc) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    const size_t n_tile = ((size_t)vocab + kVerifyTile - 1) / kVerifyTile;
    *bytes = (size_t)n_tokens * n_tile * sizeof(VerifyTile) + (size_t)n_seq * (n_tile * 8 + 4);
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
    a.accepted = accepted; a.follows = follows; a.len_out = len_out; a.vocab = vocab;
    a.n_tile = (vocab + kVerifyTile - 1) / kVerifyTile;
    a.rise = (double)scale * 1.44269504088896340736;
    a.tiles = (VerifyTile*)workspace;
    a.left = (double*)(a.tiles + (size_t)a.step.n_tokens * a.n_tile);
    a.ticket = (uint32_t*)(a.left + (size_t)a.step.n_seq * a.n_tile);
    hipStream_t s = (hipStream_t)stream;
    if (dtype == IVF_F32) launch_verify<float>(a, s);
    else if (dtype == IVF_F16) launch_verify<_Float16>(a, s);
    else launch_verify<__bf16>(a, s);
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
