// A step of a beam search: the best continuations over beams and vocabulary, and the beams' states in their new order.
#include "ivf_answer.h"
#include "ivf_device.h"
#include <algorithm>

namespace ivf {
using namespace dev;

// Workgroup `part` of a row goes over a share of its vocabulary, tile by tile, and leaves its k best logits, sorted, and
// (maximum, sum); the workgroup of a prompt joins the parts of its rows, picks, and moves the states' rows.
struct BeamMove {
    const uint8_t* from;
    uint8_t* to;
    int64_t row_bytes, from_stride, to_stride;
};
struct BeamArgs {
    const void* logits;
    int64_t row_stride;
    const float* scores_in;
    const uint8_t* done_in;
    float* scores_out;
    int32_t *parent, *token;
    uint8_t* done_out;
    unsigned long long* keys;     // [rows][parts][k] best logits, best first, packed with their tokens; 0 = none
    float2* sums;                 // [rows][parts] R, and sum of exp(x - R); R +inf: number of infinite logits
    int prompts, beams, vocab, k, eos, parts, share;     // share: tokens of a part
    BeamMove moves[IVF_MAX_BEAM_STATES];
    int n_moves;
};

constexpr int kBeamThreads = 256;
constexpr int kBeamElems = 32;                           // logits of a lane's part of a tile
constexpr int kBeamTile = 64 * kBeamElems;                // of a wavefront
constexpr int kBeamPool = 256;                           // candidates ranked at once
constexpr float kBeamSlack = 40.f;                       // terms of up to exp(40) are summed before the reference rises
constexpr float kLog2e = 1.4426950408889634f;

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

// The largest value of a wavefront, in every lane, by moves between registers
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t x) {
    x = max(x, xor_lane_u32<1>(x));
    x = max(x, xor_lane_u32<2>(x));
    x = max(x, xor_lane_u32<4>(x));
    x = max(x, xor_lane_u32<8>(x));
    x = max(x, xor_lane_u32<16>(x));
    return max(x, xor_lane_u32<32>(x));
}
__device__ __forceinline__ float wave_max(float x) {
    const uint32_t u = __float_as_uint(x), m = wave_max_u32(u & 0x80000000u ? ~u : u | 0x80000000u);
    return __uint_as_float(m & 0x80000000u ? m ^ 0x80000000u : ~m);
}
__device__ __forceinline__ unsigned long long wave_max(unsigned long long x) {
    const uint32_t hi = (uint32_t)(x >> 32), top = wave_max_u32(hi);
    return (unsigned long long)top << 32 | wave_max_u32(hi == top ? (uint32_t)x : 0u);
}

// 16 bytes of logits from any element
template <typename T> struct Logits;
template <> struct Logits<float> {
    static constexpr int kPer = 4;
    static constexpr uint32_t kNone = 0xFF800000u;         // -inf
    static __device__ __forceinline__ float get(const uint4& v, int e) { return __uint_as_float((&v.x)[e]); }
};
template <> struct Logits<_Float16> {
    static constexpr int kPer = 8;
    static constexpr uint32_t kNone = 0xFC00FC00u;
    static __device__ __forceinline__ float get(const uint4& v, int e) {
        return (float)__builtin_bit_cast(_Float16, (uint16_t)((&v.x)[e / 2] >> (16 * (e & 1))));
    }
};
template <> struct Logits<__bf16> {
    static constexpr int kPer = 8;
    static constexpr uint32_t kNone = 0xFF80FF80u;
    static __device__ __forceinline__ float get(const uint4& v, int e) {
        const uint32_t w = (&v.x)[e / 2];
        return __uint_as_float(e & 1 ? w & 0xFFFF0000u : w << 16);
    }
};
typedef u4_t u4_half_t __attribute__((aligned(2)));

// The k best words of pool[0 .. n) to best[0 .. k), best first, by counting, by the 64 lanes of a wavefront (threads =
// 64) or all of a workgroup; best past n is 0.
__device__ __forceinline__ void rank_pool(const unsigned long long* pool, int n, unsigned long long* best, int k, int first, int threads) {
    for (int i = n + first; i < k; i += threads) best[i] = 0;
    for (int i = first; i < n; i += threads) {
        const unsigned long long mine = pool[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += pool[j] > mine;
        if (rank < k) best[rank] = mine;
    }
}

// The same for the lists of a workgroup's wavefronts, in which 0 marks no entry: those go last.
__device__ __forceinline__ void rank_parts(const unsigned long long* pool, int n, unsigned long long* best, int k) {
    for (int i = threadIdx.x; i < n; i += kBeamThreads) {
        const unsigned long long mine = pool[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += pool[j] > mine || (pool[j] == mine && j < i);
        if (rank < k) best[rank] = mine;
    }
}

// Sums of exp(x - R) of two sets, (R, sum), as one
__device__ __forceinline__ float2 join_sums(float2 x, float2 y) {
    const float2 hi = x.x >= y.x ? x : y, lo = x.x >= y.x ? y : x;
    if (lo.x == hi.x) return make_float2(hi.x, hi.y + lo.y);
    if (lo.x == -INFINITY || hi.x == INFINITY) return hi;
    return make_float2(hi.x, hi.y + lo.y * __builtin_amdgcn_exp2f((lo.x - hi.x) * kLog2e));
}

// Reads the logits once.  Wavefronts work for themselves: each takes every fourth tile of 32 logits a lane, the next one
// requested before one is worked on, and sums exp(x - R) with an R that hardly ever has to rise.  What may belong to the k
// best is rare: in the first tile what reaches a value that k of the lanes' maxima reach, later what is better than the
// k-th best so far; it goes to a pool in LDS and is ranked by counting.
// Its vector instructions take 69 % of the SIMDs' cycles, a third of them those of first tiles: 512 rows of 131,072 bf16 logits, a tenth of
// them done and not read, in 37 us, 3.3 TB/s.
template <typename T>
__global__ __launch_bounds__(kBeamThreads) void beam_part_kernel(BeamArgs a) {
    constexpr int kPer = Logits<T>::kPer, kLoads = kBeamElems / kPer, kWaves = kBeamThreads / 64;
    __shared__ unsigned long long s_pool[kWaves][kBeamPool];
    __shared__ unsigned long long s_best[kWaves][IVF_MAX_BEAMS];
    __shared__ float2 s_sum[kWaves];
    const int row = blockIdx.x / a.parts, part = blockIdx.x % a.parts, lane = lane_id(), wave = wave_id(), k = a.k;
    if (a.done_in && a.done_in[row]) return;               // its only continuation needs no logits
    const int begin = part * a.share, end = min(a.vocab, begin + a.share);
    const T* x = (const T*)a.logits + row * a.row_stride;
    const int tiles = (end - begin + kBeamTile - 1) / kBeamTile;
    unsigned long long *pool = s_pool[wave], *best = s_best[wave];
    auto request = [&](int tile, uint4 (&raw)[kLoads]) __attribute__((always_inline)) {
        const int t0 = begin + tile * kBeamTile + lane * kPer;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const int t = t0 + i * 64 * kPer;
            if (t + kPer <= end) {
                const u4_t v = *(const u4_half_t*)(x + t);
                raw[i] = make_uint4(v.x, v.y, v.z, v.w);
            } else {                                       // the last few, one by one, with -inf behind them
                uint32_t w[4];
                for (int e = 0; e < 4; ++e) w[e] = Logits<T>::kNone;
                for (int e = 0; e < kPer; ++e) {
                    if (t + e >= end) break;
                    if (kPer == 4) w[e] = __float_as_uint((float)x[t + e]);
                    else if (e & 1) w[e / 2] = (w[e / 2] & 0xFFFFu) | (uint32_t)((const uint16_t*)x)[t + e] << 16;
                    else w[e / 2] = (w[e / 2] & 0xFFFF0000u) | ((const uint16_t*)x)[t + e];
                }
                raw[i] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
    };
    float R = -INFINITY, sum = 0.f;                        // sum of exp(x - R); R +inf: number of infinite logits
    unsigned long long least = 0;                          // the k-th best so far; 0: fewer
    int have = 0;
    uint4 next[kLoads];
    if (wave < tiles) request(wave, next);
    for (int tile = wave; tile < tiles; tile += kWaves) {
        uint4 raw[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) raw[i] = next[i];
        if (tile + kWaves < tiles) request(tile + kWaves, next);
        const int t0 = begin + tile * kBeamTile + lane * kPer;
        auto token = [&](int i, int e) { return t0 + i * 64 * kPer + e; };
        auto value = [&](int i, int e) __attribute__((always_inline)) { return Logits<T>::get(raw[i], e); };
        float top = -INFINITY;                             // NaN counts for nothing
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) top = fmaxf(top, value(i, e));
        // the sum, relative to a logit that no other is far above
        if (__ballot(top > R + kBeamSlack)) {              // -inf at first
            const float r2 = wave_max(fmaxf(top, R));
            sum = R == -INFINITY || r2 == INFINITY ? 0.f : sum * __builtin_amdgcn_exp2f((R - r2) * kLog2e);
            R = r2;
        }
        if (R > -INFINITY) {
            float add[2] = {0.f, 0.f};
#pragma unroll
            for (int i = 0; i < kLoads; ++i)
#pragma unroll
                for (int e = 0; e < kPer; ++e) add[e & 1] += __builtin_amdgcn_exp2f((value(i, e) - R) * kLog2e);
            float more = add[0] + add[1];
            if (__ballot(more != more)) {                  // NaN, or the largest is infinite: those share the probability
                more = 0.f;
#pragma unroll
                for (int i = 0; i < kLoads; ++i)
#pragma unroll
                    for (int e = 0; e < kPer; ++e) {
                        const float v = fmaxf(value(i, e), -INFINITY);
                        more += R == INFINITY ? (v == INFINITY ? 1.f : 0.f) : __builtin_amdgcn_exp2f((v - R) * kLog2e);
                    }
            }
            sum += more;
        }
        // what has to be reached: above `least`, or in the first tile at least `edge`, which k of the lanes' maxima reach if so
        // many lanes have any
        float edge = -INFINITY;
        if (tile == wave) {
            float left = top;
            for (int i = 0; i < k; ++i) {
                edge = wave_max(left);
                const uint64_t at = __ballot(left == edge);
                if (lane == __builtin_ctzll(at)) left = -INFINITY;
            }
        }
        // they go in by ballots; when the pool is full (masses of equal values) it is ranked in between
        float reach = fmaxf(edge, least ? logit_of(least) : -INFINITY);
        if (!__ballot(top >= reach && top > -INFINITY)) continue;
        int n = have;
        auto settle = [&]() {
            __builtin_amdgcn_wave_barrier();
            rank_pool(pool, n, best, k, lane, 64);
            __builtin_amdgcn_wave_barrier();
            have = n = min(n, k);
            least = have == k ? best[k - 1] : 0;
            if (least) reach = fmaxf(edge, logit_of(least));
            if (lane < have) pool[lane] = best[lane];
            __builtin_amdgcn_wave_barrier();
        };
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
#pragma unroll
            for (int e = 0; e < kPer; ++e) {
                const float v = value(i, e);
                if (!__ballot(v >= reach)) continue;
                const unsigned long long word = pack_logit(v, token(i, e));
                const bool in = v >= reach && word > least;
                const uint64_t who = __ballot(in);
                if (in) pool[n + __popcll(who & ((1ull << lane) - 1ull))] = word;
                n += __popcll(who);
                if (n > kBeamPool - 64) settle();
            }
        if (n > have) settle();
    }
    // join the lanes, then the wavefronts
    const float ws = group_sum<64>(sum);
    if (lane == 0) s_sum[wave] = make_float2(R, ws);
    if (lane < k) pool[lane] = lane < have ? pool[lane] : 0;
    __syncthreads();
    // the lists of the four wavefronts, one behind the other
    unsigned long long* both = s_pool[0];
    if (wave > 0 && lane < k) both[wave * k + lane] = pool[lane];
    __syncthreads();
    rank_parts(both, kWaves * k, a.keys + (int64_t)blockIdx.x * k, k);
    if (threadIdx.x == 0) {
        float2 all = s_sum[0];
        for (int w = 1; w < kWaves; ++w) all = join_sums(all, s_sum[w]);
        a.sums[blockIdx.x] = all;
    }
}

__device__ __forceinline__ void move_row(const BeamMove& m, int64_t from_row, int64_t to_row, int i0, int step) {
    const uint8_t* from = m.from + from_row * m.from_stride;
    uint8_t* to = m.to + to_row * m.to_stride;
    const bool wide = (((uintptr_t)from | (uintptr_t)to) & 15u) == 0, words = (((uintptr_t)from | (uintptr_t)to) & 3u) == 0;
    int64_t done = 0;
    if (wide) {
        const int64_t n = m.row_bytes / 16;
        for (int64_t i = i0; i < n; i += step) ((uint4*)to)[i] = ((const uint4*)from)[i];
        done = n * 16;
    } else if (words) {
        const int64_t n = m.row_bytes / 4;
        for (int64_t i = i0; i < n; i += step) ((uint32_t*)to)[i] = ((const uint32_t*)from)[i];
        done = n * 4;
    }
    for (int64_t i = done + i0; i < m.row_bytes; i += step) to[i] = from[i];
}

// One workgroup per prompt.  A wavefront joins the parts of a row, then the rows' continuations are joined, and at last
// all move the states' rows, where they are small.  Latency bounds it (7.3 us for 64 prompts of 8 beams): few candidates
// are ranked by counting, which has no chain of dependent steps, more by taking k times the best of the sorted lists' heads, a
// lane per list (9.4 us for those 64 prompts).
constexpr int kPickThreads = 512;
__global__ __launch_bounds__(kPickThreads) void beam_pick_kernel(BeamArgs a) {
    __shared__ float s_score[IVF_MAX_BEAMS * IVF_MAX_BEAMS];
    __shared__ int32_t s_token[IVF_MAX_BEAMS * IVF_MAX_BEAMS];
    __shared__ int32_t s_parent[IVF_MAX_BEAMS];
    extern __shared__ __align__(16) unsigned char s_raw[];
    const int prompt = blockIdx.x, lane = lane_id(), wave = wave_id(), k = a.k, row0 = prompt * a.beams;
    unsigned long long* lists = (unsigned long long*)s_raw + (size_t)wave * a.parts * k;
    for (int b = wave; b < a.beams; b += kPickThreads / 64) {
        const int64_t row = row0 + b;
        const float run = a.scores_in[row];
        const bool done = a.done_in && a.done_in[row];
        float* score = s_score + b * k;
        int32_t* token = s_token + b * k;
        if (done || !(run > -INFINITY)) {
            if (lane < k) { score[lane] = done && lane == 0 && run > -INFINITY ? run : -INFINITY; token[lane] = a.eos; }
            continue;
        }
        const int n = a.parts * k;
        const unsigned long long* keys = a.keys + row * n;
        const float2 ps = lane < a.parts ? a.sums[row * a.parts + lane] : make_float2(-INFINITY, 0.f);
        unsigned long long mine = 0;                       // the lane's result: the best of rank `lane`
        if (n <= 64) {                                     // by counting
            const unsigned long long word = lane < n ? keys[lane] : 0;
            const int lo = (int)word, hi = (int)(word >> 32);
            int rank = 0;
            for (int j = 0; j < n; ++j) {
                const unsigned long long other = (unsigned long long)(uint32_t)__builtin_amdgcn_readlane(hi, j) << 32 | (uint32_t)__builtin_amdgcn_readlane(lo, j);
                rank += other > word;
            }
            if (lane < k) lists[lane] = 0;
            __builtin_amdgcn_wave_barrier();
            if (word && rank < k) lists[rank] = word;
            __builtin_amdgcn_wave_barrier();
            if (lane < k) mine = lists[lane];
            __builtin_amdgcn_wave_barrier();
        } else {                                           // k times the best of the lists' heads
            for (int i = lane; i < n; i += 64) lists[i] = keys[i];
            __builtin_amdgcn_wave_barrier();
            int at = 0;
            unsigned long long head = lane < a.parts ? lists[lane * k] : 0;
            for (int i = 0; i < k; ++i) {
                const unsigned long long best = wave_max(head);
                if (lane == i) mine = best;
                if (best == 0) break;
                if (head == best) { ++at; head = at < k ? lists[lane * k + at] : 0; }
            }
            __builtin_amdgcn_wave_barrier();
        }
        const float R = wave_max(ps.x);
        const float sum = group_sum<64>(ps.x == R ? ps.y : ps.x == -INFINITY || R == INFINITY ? 0.f : ps.y * __builtin_amdgcn_exp2f((ps.x - R) * kLog2e));
        // the logarithm of the sum of exp(x - top), top the largest logit: the factor between R and it in 64 bits
        const float top = logit_of(__shfl((long long)mine, 0));
        const float lse = logf(R == top ? sum : (float)((double)sum * exp((double)R - (double)top)));
        if (lane < k) {
            const float v = logit_of(mine);
            const float y = run + ((v == top ? 0.f : v - top) - lse);
            score[lane] = mine && y > -INFINITY ? y : -INFINITY;
            token[lane] = (int32_t)~(uint32_t)mine;
        }
    }
    __syncthreads();
    const int n = a.beams * k;
    auto put = [&](int i, float top, int from, int token) {      // continuation i: of row `from`, none if top is -inf
        const bool reach = top > -INFINITY;
        const int64_t o = (int64_t)prompt * k + i, row = row0 + (reach ? from : 0);
        a.scores_out[o] = top;
        a.parent[o] = (int32_t)row;
        a.token[o] = reach ? token : -1;
        a.done_out[o] = !reach || (a.done_in && a.done_in[row]) || token == a.eos;
        s_parent[i] = (int32_t)row;
    };
    if (n <= kPickThreads) {                               // by counting, a thread per continuation
        if (wave * 64 < n) {
            const int c = min((int)threadIdx.x, n - 1);
            const float mine = s_score[c];
            int rank = 0;
#pragma unroll 8
            for (int j = 0; j < n; ++j) rank += s_score[j] > mine || (s_score[j] == mine && j < c);
            if ((int)threadIdx.x < n && rank < k) put(rank, mine, c / k, s_token[c]);
        }
    } else if (wave == 0) {                                // k times the best of the rows' heads
        int at = 0;
        float head = lane < a.beams ? s_score[lane * k] : -INFINITY;
        for (int i = 0; i < k; ++i) {
            const float top = wave_max(head);
            const uint64_t reach = __ballot(head == top && top > -INFINITY);
            if (lane == (reach ? __builtin_ctzll(reach) : 0)) {
                put(i, top, lane, s_token[lane * k + at]);
                if (reach) { ++at; head = at < k ? s_score[lane * k + at] : -INFINITY; }
            }
        }
    }
    __syncthreads();
    for (int j = wave; j < k * a.n_moves; j += kPickThreads / 64)
        move_row(a.moves[j % a.n_moves], s_parent[j / a.n_moves], (int64_t)prompt * k + j / a.n_moves, lane, 64);
}

// Large states: a workgroup per row and state.
__global__ __launch_bounds__(256) void beam_move_kernel(BeamArgs a) {
    move_row(a.moves[blockIdx.y], a.parent[blockIdx.x], blockIdx.x, threadIdx.x, 256);
}

struct BeamPlan { int parts, share; };

// Parts of a row: four workgroups a compute unit (a wavefront's first tile, in which it finds what has to be reached, costs several
// others: 64 prompts of 8 beams over 131,072 logits 49 us with 2048 workgroups, 43 with 1024, 52 with 512), tiles of their own, few
// enough for a wavefront to join, whose lists (448 entries) fit LDS.
static BeamPlan plan_beams(int64_t rows, int vocab, int k) {
    constexpr int kShare = 4 * kBeamTile;                  // a tile for each of the wavefronts
    const int tiles = (vocab + kShare - 1) / kShare;
    const int64_t want = std::max<int64_t>(1, 1024 / rows);
    const int parts = (int)std::min<int64_t>({want, tiles, 64, std::max(1, 448 / k)});
    const int per = (tiles + parts - 1) / parts;
    return BeamPlan{(tiles + per - 1) / per, per * kShare};
}

static int check_beams(int n_prompts, int beams_in, int vocab, int beams_out) {
    if (n_prompts < 1 || beams_in < 1 || vocab < 1 || beams_out < 1)
        return fail(IVF_EINVAL, "n_prompts, beams_in, vocab and beams_out must be at least 1");
    if (beams_in > IVF_MAX_BEAMS || beams_out > IVF_MAX_BEAMS)
        return fail(IVF_ELIMIT, "%d beams in, %d out: at most %d", beams_in, beams_out, IVF_MAX_BEAMS);
    if (vocab > 1 << 30) return fail(IVF_ELIMIT, "vocab = %d is above 2^30", vocab);      // tokens are counted in int, up to a tile past the last
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
    const BeamPlan p = plan_beams((int64_t)rows, vocab, beams_out);
    *bytes = rows * p.parts * ((size_t)beams_out * 8 + 8);
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
    BeamArgs a{};
    int64_t moved = 0;
    for (int i = 0; i < n_states; ++i) {
        const ivf_beam_state& s = states[i];
        if (!s.from || !s.to) return fail(IVF_EINVAL, "state %d: NULL", i);
        if (s.from == s.to) return fail(IVF_EINVAL, "state %d: to is from", i);
        if (s.row_bytes < 1 || s.from_stride < 0 || s.to_stride < s.row_bytes) return fail(IVF_EINVAL, "state %d: row_bytes or strides", i);
        a.moves[i] = BeamMove{(const uint8_t*)s.from, (uint8_t*)s.to, s.row_bytes, s.from_stride, s.to_stride};
        moved += s.row_bytes * beams_out;
    }
    if (scores_out == scores_in) return fail(IVF_EINVAL, "scores_out is scores_in");
    if (done_out == done_in) return fail(IVF_EINVAL, "done_out is done_in");
    if (!workspace || ((uintptr_t)workspace & 15u) != 0) return fail(IVF_EINVAL, "workspace must be given and 16-byte aligned");
    if (workspace_bytes < need) return fail(IVF_EINVAL, "this call needs %zu bytes of workspace (got %zu)", need, workspace_bytes);
    const int64_t rows = (int64_t)n_prompts * beams_in;
    const BeamPlan p = plan_beams(rows, vocab, beams_out);
    a.logits = logits; a.row_stride = row_stride; a.scores_in = scores_in; a.done_in = done_in; a.scores_out = scores_out;
    a.parent = parent; a.token = token; a.done_out = done_out;
    a.keys = (unsigned long long*)workspace;
    a.sums = (float2*)(a.keys + rows * p.parts * beams_out);
    a.prompts = n_prompts; a.beams = beams_in; a.vocab = vocab; a.k = beams_out; a.eos = eos; a.parts = p.parts; a.share = p.share;
    // states above 64 KB a prompt are moved by workgroups of their own
    const bool apart = moved > 65536;
    a.n_moves = apart ? 0 : n_states;
    hipStream_t s = (hipStream_t)stream;
    const dim3 grid((unsigned)(rows * p.parts)), block(kBeamThreads);
    if (dtype == IVF_F32) hipLaunchKernelGGL(beam_part_kernel<float>, grid, block, 0, s, a);
    else if (dtype == IVF_F16) hipLaunchKernelGGL(beam_part_kernel<_Float16>, grid, block, 0, s, a);
    else hipLaunchKernelGGL(beam_part_kernel<__bf16>, grid, block, 0, s, a);
    const size_t lds = (size_t)kPickThreads / 64 * p.parts * beams_out * 8;
    hipLaunchKernelGGL(beam_pick_kernel, dim3(n_prompts), dim3(kPickThreads), lds, s, a);
    if (apart) hipLaunchKernelGGL(beam_move_kernel, dim3(n_prompts * beams_out, n_states), dim3(256), 0, s, a);
    HIP_TRY(hipGetLastError());
    return IVF_OK;
}
