// Verification of drafted tokens against the target's probabilities, and the token that follows the accepted ones.
//
//   p = w / W,  w_i = 2^(c (x_i - top)),  c = scale log2(e),  W = sum_i w_i
//
// in 64 bits: the token that follows is where a running sum over the vocabulary passes u times its whole, and with 131,072 steps such a sum
// of 32-bit terms would put one draw in a hundred on another token.  The logits are read once, a tile to a wavefront, which leaves
// the tile's largest entry and its sum of weights relative to that; a row's (top, W) are those of its tiles joined.  A draw looks for the
// tile, the run of entries inside it, and the entry in turn.  Only a refused draft that was drawn from probabilities needs a second pass
// over its row, for the sums of max(w - W d, 0).
//
// What bounds it: half of a call the weights' 64-bit vector instructions (86 % of the SIMDs' cycles in the tiles), half kernels of few workgroups that
// wait for each other.  225 rows of 131,072 bf16 logits: tiles 23 us, the decision 7.5 (a chain of loads: tokens, entries, tiles), what the drafts leave
// of 64 rows 10.4, the draw 6.1 (again a chain: sums, a tile); by the largest entry alone 12 and 4.  Five rows of 50,001: 5.3 and 7.1.
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
    VerifyTile* chosen;          // [n_seq] the row that such a sum is formed of, joined, its number in `best`; -1: none
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

// 2^(t / 256) for t = v by - less, `less` a whole number below 2^40 in size, t from -330,000 on, from a table of 2^(i / 256) in LDS: the series
// around the nearest whole number is off by (0.00136)^4 / 4! = 1.4e-13.  The weights of all entries are formed by it, in 17 instructions
// each with what is around it (225 rows of 131,072 entries, by exp2_64 37 us, so 23).
constexpr int kPowers = 256;
__device__ __forceinline__ double exp2_by(const double* table, double v, double by, double less) {
    const double whole = 0x1.8p52 - less, shifted = __builtin_fma(v, by, whole);     // the whole number is in the low bits
    const int n = (int)__builtin_bit_cast(long long, shifted);
    const double f = __builtin_fma(v, by, whole - shifted);
    constexpr double c1 = 0.693147180559945309417 / kPowers, c2 = c1 * c1 / 2, c3 = c2 * c1 / 3;
    const double p = __builtin_fma(__builtin_fma(c3, f, c2), f, c1), b = table[n & (kPowers - 1)];
    return __builtin_amdgcn_ldexp(__builtin_fma(b * f, p, b), n >> 8);
}

// Whether a row's weights are formed by it, and the entry that whatever lies below it (-inf and NaN among that) counts as: 990 / rise below the
// largest.  rise |top| is below 2^32 then, and the entry's rounding to 32 bits below 2^8 / rise, so that its weight is below 2^-730 of the largest.  With
// rise at 2^-90 or below it could lie under the lowest number of 32 bits, which may have any weight.
__device__ __forceinline__ bool by_table(double rise, double less) { return fabs(less) < 0x1p40 && rise > 0x1p-90; }
__device__ __forceinline__ float least_entry(double rise, float top) { return (float)((double)top - 990.0 / rise); }

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

// A lane's kVerifyRun entries of a tile that begins at entry i0 of x, spread so that the lanes' loads lie side by side; `fill` behind the row's end.
template <typename T> __device__ __forceinline__ int place_in_tile(int i) {
    constexpr int kPer = kPerLoad<T>;
    return (i / kPer * 64 + lane_id()) * kPer + i % kPer;
}
template <typename T> __device__ __forceinline__ void load_tile(const T* x, int i0, int vocab, float fill, float (&v)[kVerifyRun]) {
    constexpr int kPer = kPerLoad<T>, kLoads = kVerifyRun / kPer;
    if (i0 + kVerifyTile <= vocab) {
        u4_t raw[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) raw[i] = *(const u4_any_t*)(x + i0 + place_in_tile<T>(i * kPer));
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) v[i] = unpack<T>(raw[i / kPer], i % kPer);
    } else {
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) {
            const int at = i0 + place_in_tile<T>(i);
            v[i] = at < vocab ? (float)x[at] : fill;
        }
    }
}

// A wavefront per tile: its largest entry, then its weights, from registers.  (Two tiles a wavefront, the second on its way meanwhile: 26 us against 23, for the registers leave
// four wavefronts a SIMD.)
template <typename T>
__global__ __launch_bounds__(kVerifyWaves * 64, 6) void verify_tiles_kernel(VerifyArgs a) {
    const int per_row = (a.n_tile + kVerifyWaves - 1) / kVerifyWaves;
    const int row = blockIdx.x / per_row, tile = blockIdx.x % per_row * kVerifyWaves + wave_id();
    float v[kVerifyRun], top = -INFINITY;
    load_tile((const T*)a.logits + row * a.row_stride, tile * kVerifyTile, a.vocab, -INFINITY, v);
#pragma unroll
    for (int i = 0; i < kVerifyRun; ++i) top = fmaxf(top, v[i]);          // NaN counts for nothing
    top = lanes_max(top);
    VerifyTile out = {0.0, top, -1};
    __shared__ double s_powers[kPowers];
    static_assert(kPowers == kVerifyWaves * 64, "a power a thread");
    s_powers[threadIdx.x] = exp2_64(threadIdx.x / (double)kPowers);
    __syncthreads();
    if (a.rise == 0.0) {
        int best = 0x7FFFFFFF;
#pragma unroll
        for (int i = kVerifyRun - 1; i >= 0; --i)
            if (v[i] == top) best = min(best, tile * kVerifyTile + place_in_tile<T>(i));
        for (int w = 32; w >= 1; w >>= 1) best = min(best, __shfl_xor(best, w));
        if (top > -INFINITY) out.best = best;
    } else if (top > -INFINITY) {
        double sum = 0.0;
        if (top == INFINITY) {
#pragma unroll
            for (int i = 0; i < kVerifyRun; ++i) sum += v[i] == INFINITY ? 1.0 : 0.0;
        } else {
            const double by = a.rise * kPowers, less = rint(by * (double)top);
            if (by_table(a.rise, less)) {
                const float least = least_entry(a.rise, top);
#pragma unroll
                for (int i = 0; i < kVerifyRun; ++i) sum += exp2_by(s_powers, (double)fmaxf(v[i], least), by, less);
                sum *= exp2_64(__builtin_fma((double)top, by, -less) * (-1.0 / kPowers));
            } else {
#pragma unroll 1
                for (int i = 0; i < kVerifyRun; ++i) {
                    float x = v[0];
#pragma unroll
                    for (int j = 1; j < kVerifyRun; ++j) x = i == j ? v[j] : x;
                    sum += weight_of(x, top, a.rise);
                }
            }
        }
        out.sum = lanes_sum(sum);
    }
    if (lane_id() == 0 && tile < a.n_tile) a.tiles[(int64_t)row * a.n_tile + tile] = out;
}

// A row's tiles joined, by a wavefront; `t`: the lane's of the first 64, which the caller has requested
__device__ __forceinline__ VerifyTile tile_of(const VerifyArgs& a, int64_t row, int i) {
    return i < a.n_tile ? a.tiles[row * a.n_tile + i] : VerifyTile{0.0, -INFINITY, -1};
}
__device__ __forceinline__ VerifyTile join_tiles(const VerifyArgs& a, int64_t row, VerifyTile t) {
    VerifyTile all = {0.0, -INFINITY, -1};
    for (int i0 = 0; i0 < a.n_tile; i0 += 64) {
        if (i0 > 0) t = tile_of(a, row, i0 + lane_id());
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

// What a draft's probability d leaves of a weight w, max(w - W d, 0).  w and W are off by 1.5e-13 of themselves: where target and draft say the same,
// what their difference comes out as is of either sign.  Less than 2^-40 of w is therefore nothing.
__device__ __forceinline__ double left_of(double w, double whole, float d) {
    const double x = __builtin_fma(-whole, (double)fmaxf(d, 0.f), w);
    return x > w * 0x1p-40 ? x : 0.0;
}
// The same of the entries of one row, whose tiles' sums and entries are formed by this alone: a tile has a sum above zero exactly where one of its
// entries has.  In units of 2^(less / kPowers) by the table of powers, else of the largest entry's weight.
struct Left {
    const double* table;
    double rise, by, less, whole;
    float top, least;
    bool tabled;
    __device__ __forceinline__ Left(const double* powers, double rise_, float top_, double sum) : table(powers), rise(rise_), top(top_) {
        by = rise * kPowers;
        less = rint(by * (double)top);
        tabled = by_table(rise, less);
        least = least_entry(rise, top);
        whole = tabled ? sum / exp2_64(__builtin_fma((double)top, by, -less) * (-1.0 / kPowers)) : sum;
    }
    template <bool TABLE> __device__ __forceinline__ double of(float x, float d) const {
        if (!TABLE) return left_of(weight_of(x, top, rise), whole, d);
        // an entry that has no weight must leave nothing
        return x > least ? left_of(exp2_by(table, (double)x, by, less), whole, d) : 0.0;
    }
};

// The weights that a sequence's next token is drawn from
template <typename T> struct Weights {
    const T* logits;                                      // the row
    const float* draft;                                   // its draft's, or NULL
    const Left* left;                                     // with `draft`
    int vocab, without;                                   // a token that is left out, or -1
    float top;
    double rise;
    // of N entries from i0 on; 0 behind the row's end
    template <int N> __device__ __forceinline__ void operator()(int i0, double (&w)[N]) const {
        float x[N], d[N];
#pragma unroll
        for (int i = 0; i < N; ++i) {
            x[i] = i0 + i < vocab ? (float)logits[i0 + i] : -INFINITY;
            d[i] = draft && i0 + i < vocab ? draft[i0 + i] : 0.f;
        }
#pragma unroll
        for (int i = 0; i < N; ++i)
            w[i] = i0 + i == without ? 0.0 : !draft ? weight_of(x[i], top, rise) : left->tabled ? left->of<true>(x[i], d[i]) : left->of<false>(x[i], d[i]);
    }
};

// A draw by a workgroup of kDrawWaves: sums up to every thread, and the first thread whose sum is above what is to be reached.
constexpr int kDrawWaves = 8, kDrawThreads = kDrawWaves * 64, kDrawRun = kVerifyTile / kDrawThreads;
struct DrawShared {
    double part[kDrawWaves], before;
    int first, last, token;
};
__device__ __forceinline__ double draw_prefix(DrawShared& sh, double x, double& whole) {
    double upto = lanes_prefix(x), before = 0.0;
    __syncthreads();
    if (lane_id() == 63) sh.part[wave_id()] = upto;
    if (threadIdx.x == 0) { sh.first = 0x7FFFFFFF; sh.last = -1; }
    __syncthreads();
    whole = 0.0;
#pragma unroll
    for (int w = 0; w < kDrawWaves; ++w) {
        if (w == wave_id()) before = whole;
        whole += sh.part[w];
    }
    return before + upto;
}
// The thread whose `mine` takes the sum above `reach`; the last of any weight where rounding lets none be (none: -1); behind draw_prefix
__device__ __forceinline__ int draw_thread(DrawShared& sh, double mine, double upto, double reach, double& before) {
    const uint64_t some = __ballot(mine > 0.0), above = __ballot(mine > 0.0 && upto > reach);
    if (lane_id() == 0) {
        if (above) atomicMin(&sh.first, wave_id() * 64 + __builtin_ctzll(above));
        if (some) atomicMax(&sh.last, wave_id() * 64 + 63 - __builtin_clzll(some));
    }
    __syncthreads();
    const int at = sh.first != 0x7FFFFFFF ? sh.first : sh.last;
    if ((int)threadIdx.x == at) sh.before = upto - mine;
    __syncthreads();
    before = sh.before;
    return at;
}
// The token that follows; left: the tiles' sums where a draft's probabilities are subtracted; row: that of the weights
template <typename T> __device__ __forceinline__ int draw(const VerifyArgs& a, DrawShared& sh, Weights<T> weights, int64_t row, const double* left, float uniform) {
    for (int tries = 0; tries < 2; ++tries) {
        // the tile of a token that is left out is summed anew: less that token's weight its sum may lose all that is left
        const int at = weights.without < 0 ? -1 : weights.without / kVerifyTile;
        auto sum_of = [&](int i) {
            if (weights.draft) return i < a.n_tile ? left[i] : 0.0;
            const VerifyTile x = tile_of(a, row, i);
            return x.top == -INFINITY ? 0.0 : x.sum * weight_of(x.top, weights.top, a.rise);
        };
        double mine = sum_of(threadIdx.x), anew = 0.0, w[kDrawRun], whole, part;
        if (at >= 0) {
            weights(at * kVerifyTile + threadIdx.x * kDrawRun, w);
            double x = 0.0;
#pragma unroll
            for (int i = 0; i < kDrawRun; ++i) x += w[i];
            draw_prefix(sh, x, anew);
            if ((int)threadIdx.x == at) mine = anew;
        }
        double upto = draw_prefix(sh, mine, whole);
        for (int i0 = kDrawThreads; i0 < a.n_tile; i0 += kDrawThreads) {
            const int i = i0 + threadIdx.x;
            draw_prefix(sh, i == at ? anew : sum_of(i), part);
            whole += part;
        }
        if (whole > 0.0) {
            const double reach = (double)uniform * whole;
            double run = 0.0, before = 0.0;
            int tile = -1;
            for (int i0 = 0; i0 < a.n_tile; i0 += kDrawThreads) {
                const int i = i0 + threadIdx.x;
                if (a.n_tile > kDrawThreads) {
                    mine = i == at ? anew : sum_of(i);
                    upto = run + draw_prefix(sh, mine, part);
                }
                double from;
                const int here = draw_thread(sh, mine, upto, reach, from);
                if (here >= 0) { tile = i0 + here; before = from; }
                if (sh.first != 0x7FFFFFFF) break;
                run += part;
            }
            weights(tile * kVerifyTile + threadIdx.x * kDrawRun, w);
            mine = 0.0;
#pragma unroll
            for (int i = 0; i < kDrawRun; ++i) mine += w[i];
            upto = before + draw_prefix(sh, mine, part);
            double at_run;
            const int here = draw_thread(sh, mine, upto, reach, at_run);
            if ((int)threadIdx.x == here) {
                int found = 0;
                bool over = false;
#pragma unroll
                for (int i = 0; i < kDrawRun; ++i) {
                    at_run += w[i];
                    if (!over && w[i] > 0.0) { found = i; over = at_run > reach; }
                }
                sh.token = tile * kVerifyTile + here * kDrawRun + found;
            }
            __syncthreads();
            if (here >= 0) return sh.token;
        }
        weights.draft = nullptr;                          // nothing is left: from p itself
        weights.without = -1;
    }
    return -1;
}

// A workgroup per sequence: the accepted drafts, by a wavefront a row, and the token that follows where no draft's probabilities are to be
// subtracted; else the row and what is known of it, for the two kernels below.
template <typename T>
__global__ __launch_bounds__(kDrawThreads) void verify_decide_kernel(VerifyArgs a) {
    __shared__ int s_refused;
    __shared__ VerifyTile s_row[kVerifyRows];
    __shared__ DrawShared s_draw;
    const int s = blockIdx.x, lane = lane_id(), wave = wave_id();
    const int t0 = token_of(a.step, s), count = max(0, token_of(a.step, s + 1) - t0);
    if (threadIdx.x == 0) s_refused = max(1, count);
    __syncthreads();
    for (int i = wave; i < count; i += kDrawWaves) {
        const int t = t0 + i + 1;
        const bool drafted = i + 1 < count;
        const VerifyTile first = tile_of(a, t - 1, lane);
        const int token = drafted ? a.tokens[t] : -1;
        const bool known = token >= 0 && token < a.vocab;
        float x = 0.f, d = 1.f, u = 0.f;
        if (known && a.rise != 0.0) {
            x = entry_of<T>(a.logits, (t - 1) * a.row_stride + token);
            if (a.draft) d = a.draft[t * a.draft_stride + token];
            u = a.uniform[t];
        }
        const VerifyTile row = join_tiles(a, t - 1, first);
        if (i < kVerifyRows && lane == 0) s_row[i] = row;
        bool ok = known && row.top > -INFINITY;
        if (a.rise == 0.0) ok = ok && token == row.best;
        else ok = ok && (double)u * (double)fmaxf(d, 0.f) * row.sum < weight_of(x, row.top, a.rise);
        if (drafted && !ok && lane == 0) atomicMin(&s_refused, i + 1);
    }
    __syncthreads();
    const int n = s_refused - 1, t = t0 + n;
    const bool refused = n + 1 < count;
    const VerifyTile row = count == 0 ? VerifyTile{0.0, -INFINITY, -1} : n < kVerifyRows ? s_row[n] : join_tiles(a, t, tile_of(a, t, lane));
    const bool later = refused && a.draft && a.rise != 0.0 && row.top > -INFINITY;
    if (threadIdx.x == 0) {
        a.accepted[s] = n;
        a.len_out[s] = a.step.len[s] - max(0, count - 1 - n);
        if (a.draft && a.rise != 0.0) a.chosen[s] = VerifyTile{row.sum, row.top, later ? t : -1};
    }
    if (later) return;
    int token = -1;
    if (a.rise == 0.0) {
        token = row.best;
    } else if (row.top > -INFINITY) {
        int without = refused ? a.tokens[t + 1] : -1;
        if (without >= a.vocab) without = -1;
        const Weights<T> weights = {(const T*)a.logits + t * a.row_stride, nullptr, nullptr, a.vocab, without, row.top, a.rise};
        token = draw(a, s_draw, weights, t, nullptr, a.uniform[t0]);
    }
    if (threadIdx.x == 0) a.follows[s] = token;
}

// A wavefront per tile of the rows whose draft's probabilities are subtracted
template <typename T>
__global__ __launch_bounds__(kVerifyWaves * 64) void verify_left_kernel(VerifyArgs a) {
    const int per_row = (a.n_tile + kVerifyWaves - 1) / kVerifyWaves;
    const int s = blockIdx.x / per_row, tile = blockIdx.x % per_row * kVerifyWaves + wave_id(), i0 = tile * kVerifyTile;
    const VerifyTile chosen = a.chosen[s];
    if (chosen.best < 0) return;                          // all wavefronts
    const int64_t t = chosen.best;
    const float* draft = a.draft + (t + 1) * a.draft_stride;
    float x[kVerifyRun], d[kVerifyRun];
    if (tile < a.n_tile) {
        load_tile((const T*)a.logits + t * a.row_stride, i0, a.vocab, -INFINITY, x);
        // the draft's entries in the places of the logits'
#pragma unroll
        for (int i = 0; i < kVerifyRun; i += 4) {
            const int at = i0 + place_in_tile<T>(i);
            if (i0 + kVerifyTile <= a.vocab) {
                const u4_t y = *(const u4_any_t*)(draft + at);
#pragma unroll
                for (int e = 0; e < 4; ++e) d[i + e] = __uint_as_float(y[e]);
            } else {
#pragma unroll
                for (int e = 0; e < 4; ++e) d[i + e] = at + e < a.vocab ? draft[at + e] : 0.f;
            }
        }
    }
    __shared__ double s_powers[kPowers];
    s_powers[threadIdx.x] = exp2_64(threadIdx.x / (double)kPowers);
    __syncthreads();
    if (tile >= a.n_tile) return;
    const Left left(s_powers, a.rise, chosen.top, chosen.sum);
    double sum = 0.0;
    if (left.tabled) {
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) sum += left.of<true>(x[i], d[i]);
    } else {
#pragma unroll
        for (int i = 0; i < kVerifyRun; ++i) sum += left.of<false>(x[i], d[i]);
    }
    sum = lanes_sum(sum);
    if (lane_id() == 0) a.left[(int64_t)s * a.n_tile + tile] = sum;
}

template <typename T>
__global__ __launch_bounds__(kDrawThreads) void verify_draw_kernel(VerifyArgs a) {
    __shared__ DrawShared s_draw;
    __shared__ double s_powers[kPowers];
    const int s = blockIdx.x;
    const VerifyTile chosen = a.chosen[s];
    if (chosen.best < 0) return;
    if (threadIdx.x < kPowers) s_powers[threadIdx.x] = exp2_64(threadIdx.x / (double)kPowers);
    __syncthreads();
    const int64_t t = chosen.best;
    const Left left(s_powers, a.rise, chosen.top, chosen.sum);
    const Weights<T> weights = {(const T*)a.logits + t * a.row_stride, a.draft + (t + 1) * a.draft_stride, &left, a.vocab, -1, chosen.top, a.rise};
    const int token = draw(a, s_draw, weights, t, a.left + (int64_t)s * a.n_tile, a.uniform[token_of(a.step, s)]);
    if (threadIdx.x == 0) a.follows[s] = token;
}

static int check_verify(int n_seq, int n_tokens, int vocab) {
    if (n_seq < 1 || n_tokens < 1 || vocab < 1) return fail(IVF_EINVAL, "n_seq, n_tokens and vocab must be at least 1");
    if (vocab > 1 << 30) return fail(IVF_ELIMIT, "vocab = %d is above 2^30", vocab);
    // launches of kDrawThreads a sequence, and kVerifyWaves * 64 for as many tiles of a row
    const int64_t blocks = (vocab + (int64_t)kVerifyTile * kVerifyWaves - 1) / (kVerifyTile * kVerifyWaves);
    if (too_many_threads(n_seq, kDrawThreads) || too_many_threads(blocks * n_seq, kVerifyWaves * 64) || too_many_threads(blocks * n_tokens, kVerifyWaves * 64))
        return fail(IVF_ELIMIT, "%d sequences, %d tokens over %d entries", n_seq, n_tokens, vocab);
    return IVF_OK;
}

// (a kernel that is not launched leaves to the next ones what its workspace held before)
template <typename T> static hipError_t launch_verify(const VerifyArgs& a, hipStream_t s) {
    const int64_t per_row = (a.n_tile + kVerifyWaves - 1) / kVerifyWaves;
    const dim3 block(kVerifyWaves * 64);
    hipError_t e;
    hipLaunchKernelGGL(verify_tiles_kernel<T>, dim3((unsigned)(a.step.n_tokens * per_row)), block, 0, s, a);
    if ((e = hipGetLastError())) return e;
    hipLaunchKernelGGL(verify_decide_kernel<T>, dim3(a.step.n_seq), dim3(kDrawThreads), 0, s, a);
    if ((e = hipGetLastError()) || !a.draft || a.rise == 0.0) return e;
    hipLaunchKernelGGL(verify_left_kernel<T>, dim3((unsigned)(a.step.n_seq * per_row)), block, 0, s, a);
    if ((e = hipGetLastError())) return e;
    hipLaunchKernelGGL(verify_draw_kernel<T>, dim3(a.step.n_seq), dim3(kDrawThreads), 0, s, a);
    return hipGetLastError();
}

}  // namespace ivf

using namespace ivf;

extern "C" int ivf_verify_workspace(int32_t n_seq, int32_t n_tokens, int32_t vocab, size_t* bytes) {
    int rc = check_verify(n_seq, n_tokens, vocab);
    if (rc) return rc;
    if (!bytes) return fail(IVF_EINVAL, "bytes is NULL");
    const size_t n_tile = ((size_t)vocab + kVerifyTile - 1) / kVerifyTile;
    *bytes = (size_t)n_tokens * n_tile * sizeof(VerifyTile) + (size_t)n_seq * (n_tile * 8 + sizeof(VerifyTile));
    return IVF_OK;
}

extern "C" int ivf_verify_draft(const ivf_kv_step* step, const void* logits, int64_t row_stride, int dtype, int32_t vocab, double scale,
                                const int32_t* tokens, const float* uniform, const float* draft, int64_t draft_stride, int32_t* accepted,
                                int32_t* follows, int32_t* len_out, void* workspace, size_t workspace_bytes, void* stream) {
    if (!step) return fail(IVF_EINVAL, "step is NULL");
    if (!step->q_off || !step->len) return fail(IVF_EINVAL, "q_off or len is NULL");
    size_t need = 0;
    int rc = ivf_verify_workspace(step->n_seq, step->n_tokens, vocab, &need);
    if (rc) return rc;
    if (!logits || !tokens || !accepted || !follows || !len_out) return fail(IVF_EINVAL, "logits, tokens or an output is NULL");
    if (dtype != IVF_F32 && dtype != IVF_F16 && dtype != IVF_BF16) return fail(IVF_EINVAL, "unknown dtype %d", dtype);
    if (!(scale >= 0.0) || scale > 1e30) return fail(IVF_EINVAL, "scale must be from 0 to 1e30");
    if (scale > 0.0 && !uniform) return fail(IVF_EINVAL, "uniform is NULL");
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
    a.rise = scale * 1.44269504088896340736;
    a.tiles = (VerifyTile*)workspace;
    a.chosen = a.tiles + (size_t)a.step.n_tokens * a.n_tile;
    a.left = (double*)(a.chosen + a.step.n_seq);
    hipStream_t s = (hipStream_t)stream;
    HIP_TRY(dtype == IVF_F32 ? launch_verify<float>(a, s) : dtype == IVF_F16 ? launch_verify<_Float16>(a, s) : launch_verify<__bf16>(a, s));
    return IVF_OK;
}
