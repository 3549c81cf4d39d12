// Attention of a step's new tokens over the paged cache.
//
//   out = sum_j w_j v_j / sum_j w_j,  w_j = exp(scale q . k_j) over the keys j that the token sees
//
// in one pass over the keys with a running maximum m: w_j is taken as 2^(x_j - m), x_j = q . k_j scale log2(e), and what
// was summed is scaled by 2^(m - m') when m rises to m'.  Sums over disjoint sets of keys are joined by the same rule, so
// the keys of a long sequence are split over workgroups and those of a prefix are read for all tokens of its group at
// once, whose sequences then add their own keys.
//
// Rows.  The new tokens of a sequence (of a group, for its prefix) times the query heads that share a key head are the
// rows of one product, row r = token r / G, head r % G: 32 of them to a wavefront.  Scores are formed transposed,
// S^T = K Q^T by 32 x 32 x 16 MFMAs (lane l holds 16 of 32 keys of row l % 32), so that a row's maximum and sum stay
// inside a lane but for one exchange with lane l ^ 32, and the weights are already where O^T += V^T P^T wants them: the
// order of keys inside a product is free, and V is read from LDS transposed in the order in which S^T came out.
//
// Keys and values go from memory to LDS directly, without passing registers, 16 bytes a lane; the chunks of a row are
// permuted on the way so that both kinds of LDS reads are spread over the banks.  The tables' entries are fetched into
// LDS in the same way ahead of the tiles they name.
//
// What bounds it.  Few rows: memory, if the keys are long (24 sequences of up to 60,000 keys, 8 key heads of 128, bf16: 533 us, 5.6
// TB/s of reads, no byte twice), else the chain of lengths, table, keys and joins (one token over 700 keys: 9 us and 3 for the joining).
// Many rows: the matrix and the vector instructions of a SIMD's two wavefronts, which seldom run side by side: of a prompt of 16,000
// tokens, 32 query and 8 key heads of 128, in 2.04 ms, 1030 TFLOP/s, the matrix units are busy for 52 % of the SIMDs' cycles, vector
// instructions (those that start products among them) for 47 %; LDS for 26 % of a compute unit's, without bank conflicts.  Heads of 64: 35 % and 56 %, LDS
// 35 %, half of that by bank conflicts (three prompts, 4250 tokens, behind 6000 keys: 375 us, 650 TFLOP/s).
//
// Quantised caches (Q8).  What a key or value stands for, an e4m3 number times the power of two of its token and head, is exact in T, so nothing
// else changes.  Few rows: tiles are codes in LDS.  A lane reads sixteen codes of a key, which serve two products (the order of elements inside a product is
// free too), and converts them with the key's power; eight codes of one element of eight values, read transposed, it converts as they are, and the
// weights (bf16) or the numbers (f16) are multiplied by the values' powers.  LDS carries a third of what it does with tiles of T, and memory bounds it: 24 sequences of
// up to 60,000 keys as above in 291 us, 5.0 TB/s, the loads alone in 286.  Many rows: every wavefront converts its share of a tile once and writes it
// into LDS, a tile ahead: 8000 tokens behind 2001, 32 query and 8 key heads of 128, in 870 to 985 us where 16-bit keys and values take 800 to 865: the
// conversions are 10 % more vector instructions, the writes double what LDS does, and the clock falls with the power of both.
#pragma once
#include "ivf_answer.h"
#include "ivf_device.h"
#include <algorithm>
#include <atomic>
#include <math.h>
#include <type_traits>

namespace ivf {
using namespace dev;

enum { kConcat, kOwn, kPrefix };     // keys of a pass: prefix and own, own only, prefix only
constexpr int kNarrowRows = 32, kWideRows = 128, kAllRows = 0x7FFFFFFF;

struct AttendArgs {
    CacheView cache;
    StepView step;
    ivf_rows q, out;
    float* lse;
    float scale_log2;                // scale * log2(e)
    int hq, hkv, group, window, sinks;       // group: query heads per key head
    // partial sums [token][query head][parts]: O [d] unnormalised, and (m, l); m of the first own one NaN: the row's result is
    // complete, or its own sums are among the few
    float* part_o;
    float2* part_ml;
    int parts, part_own;             // 0: no partial sums; those of the prefix, which come first
    // where sequences of few and of many rows meet, the own sums of the few's [sequence][few_tokens][query head][few_parts]: their keys
    // may be cut into many pieces, and the many rows of the others need no room for as many
    float* few_o;
    float2* few_ml;
    int few_tokens, few_parts;       // 0: all are among the others
    // one launch makes one pass or two, which read different keys
    struct Pass {
        int mode, part0, n_part;     // its range of partial sums
        int n_split, n_tile;         // workgroups that share a row's keys; that share a unit's rows (0: one per tile of each sequence)
        int rows_lo, rows_hi;        // units with more than rows_lo and at most rows_hi rows
    } pass[2];
    int first_blocks;                // workgroups of the first pass
    QuantView quant;
};

// ---- memory to LDS ------------------------------------------------------------------------------
// The loads are written as assembly so that the compiler, which cannot know which of them a read from LDS depends on,
// does not wait for all of them; they have no register outputs.  (m0 is the compiler's own, set where it
// needs it and not carried across statements: naming it as changed changes no instruction.)
extern __shared__ __align__(1024) unsigned char s_mem[];

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// lane l's 16 (4) bytes at g go to LDS address `to` + 16 l (4 l); `to` is the same in all lanes
__device__ __forceinline__ void fetch16(const void* g, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" :: "v"(g), "s"(to) : "memory");
}
__device__ __forceinline__ void fetch4(const void* g, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off" :: "v"(g), "s"(to) : "memory");
}
// the same from `off` bytes behind a place that all lanes share
__device__ __forceinline__ void fetch16(const void* base, uint32_t off, uint32_t to) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" :: "v"(off), "s"(base), "s"(to) : "memory");
}
// lane l's byte at g as a word to `to` + 4 l
__device__ __forceinline__ void fetch_byte(const void* g, uint32_t to) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %0, off" :: "v"(g), "s"(to) : "memory");
}
__device__ __forceinline__ void wait_loads() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory"); }
__device__ __forceinline__ void barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// ---- types ------------------------------------------------------------------------------------------
typedef short s4_t __attribute__((ext_vector_type(4)));
typedef short s8_t __attribute__((ext_vector_type(8)));
typedef float f16v_t __attribute__((ext_vector_type(16)));
typedef _Float16 h8_t __attribute__((ext_vector_type(8)));
typedef __bf16 b8_t __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s4_t* lds_s4;
typedef __attribute__((address_space(3))) const s8_t* lds_s8;
typedef __attribute__((address_space(3))) u4_t* lds_u4;
typedef int i2_t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) i2_t* lds_i2;
typedef _Float16 h2_t __attribute__((ext_vector_type(2)));
typedef float f4_t __attribute__((ext_vector_type(4)));
template <typename V> using lds_ptr = __attribute__((address_space(3))) V*;

template <typename T> struct Half;
template <> struct Half<_Float16> {
    static constexpr uint32_t kExponent = 0x7C00u;
    // weights reach from 2^-22 of the largest down to f16's smallest numbers only if the largest lies high
    static constexpr float kLift = 7.f;
    static __device__ __forceinline__ f16v_t mfma(s8_t a, s8_t b, f16v_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(h8_t, a), __builtin_bit_cast(h8_t, b), c, 0, 0, 0);
    }
};
template <> struct Half<__bf16> {
    static constexpr uint32_t kExponent = 0x7F80u;
    static constexpr float kLift = 0.f;
    static __device__ __forceinline__ f16v_t mfma(s8_t a, s8_t b, f16v_t c) {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(b8_t, a), __builtin_bit_cast(b8_t, b), c, 0, 0, 0);
    }
};

// the value of lane (l & ~3) + u
__device__ __forceinline__ int quad_lane(int x, int u) {
    switch (u) {
    case 0: return __builtin_amdgcn_mov_dpp(x, 0x00, 0xF, 0xF, true);
    case 1: return __builtin_amdgcn_mov_dpp(x, 0x55, 0xF, 0xF, true);
    case 2: return __builtin_amdgcn_mov_dpp(x, 0xAA, 0xF, 0xF, true);
    default: return __builtin_amdgcn_mov_dpp(x, 0xFF, 0xF, 0xF, true);
    }
}
__device__ __forceinline__ int64_t quad_lane(int64_t x, int u) {
    const int lo = (int)x, hi = (int)(x >> 32);
    int a, b;
    switch (u) {
    case 0: a = __builtin_amdgcn_mov_dpp(lo, 0x00, 0xF, 0xF, true); b = __builtin_amdgcn_mov_dpp(hi, 0x00, 0xF, 0xF, true); break;
    case 1: a = __builtin_amdgcn_mov_dpp(lo, 0x55, 0xF, 0xF, true); b = __builtin_amdgcn_mov_dpp(hi, 0x55, 0xF, 0xF, true); break;
    case 2: a = __builtin_amdgcn_mov_dpp(lo, 0xAA, 0xF, 0xF, true); b = __builtin_amdgcn_mov_dpp(hi, 0xAA, 0xF, 0xF, true); break;
    default: a = __builtin_amdgcn_mov_dpp(lo, 0xFF, 0xF, 0xF, true); b = __builtin_amdgcn_mov_dpp(hi, 0xFF, 0xF, 0xF, true); break;
    }
    return (int64_t)((uint64_t)(uint32_t)b << 32 | (uint32_t)a);
}
__device__ __forceinline__ float other_half(float x) { return __uint_as_float(xor_lane_u32<32>(__float_as_uint(x))); }

// A maximum rises only when the new one is 2^kSlack above it: until then weights of up to 2^kSlack are summed, which
// costs no precision, and the sums need not be scaled for every small rise.
constexpr float kSlack = 8.f;

// NARROW: the workgroup has one tile of 32 rows, its NARROW wavefronts take the tiles of keys in turn, each with LDS of its own.
// 0: every one of four wavefronts has 32 rows of its own and all share the tiles.
template <int D, int NARROW, bool Q8>
struct Shape {
    static constexpr int kChunks = D <= 64 ? 8 : D <= 128 ? 16 : 32;       // 16-byte chunks of a staged row
    // Q8 with few rows: tiles stay codes in LDS and are converted where the products take them; with many rows they are converted on the way
    static constexpr bool kDirect = Q8 && NARROW;
    static constexpr int kLanes = Q8 ? kChunks / 2 : kChunks;              // lanes that load a row, 16 bytes each
    static constexpr int kPitch = (kDirect ? kLanes : kChunks) * 16;
    static constexpr int kKeys = NARROW || D > 128 ? 32 : 64;              // keys of a tile
    static constexpr int kWaves = NARROW ? NARROW : 4;
    static constexpr int kStages = 2;                                      // one tile is on its way while one is worked on
    static constexpr int kTileBytes = kKeys * kPitch * 2 + (kDirect ? 256 : 0);      // keys, then values; the bytes of their powers, a word each
    static constexpr int kPowerBytes = kDirect ? 256 : 0;                  // the values' powers of the tile that is worked on
    static constexpr int kRowsPerLoad = 64 / kLanes;
    static constexpr int kWaveRows = NARROW ? kKeys : kKeys / kWaves;      // rows of a tile that a wavefront fetches
    static constexpr int kLoads = kWaveRows / kRowsPerLoad;                // loads for its keys, and as many for its values
    static constexpr int kRows = NARROW ? 32 : 32 * kWaves;                // rows of a workgroup
    static constexpr int kSets = (kLoads + 3) / 4;
    static constexpr int kEntrySlots = 4;                                  // tiles whose table entries are kept: an entry comes three tiles ahead
    static constexpr int kJoinBytes = NARROW ? kWaves * 32 * (D * 4 + 8) : 0;    // to join the wavefronts, in the same place
    static constexpr int kStageBytes = std::max((NARROW ? kWaves : 1) * (kStages * kTileBytes + kPowerBytes), kJoinBytes);
    static constexpr int kLds = kStageBytes + kWaves * kEntrySlots * kSets * 256;
};

// x as if it were new: what follows from it is computed where it is used, not kept from before a loop.  With heads of 256 such values
// would be kept in scratch memory, and a reload waits for every tile on its way (narrow, 24 sequences of up to 20,000 keys: 809 us
// against 452)
__device__ __forceinline__ int again(int x) { asm volatile("" : "+v"(x)); return x; }

// chunk c of row r of a tile lies at place c ^ place_swap(r)
template <int CHUNKS> __device__ __forceinline__ int place_swap(int row) {
    return CHUNKS == 8 ? row & 7 : (row & 3) << 2 | (row >> 2 & 3);
}

// The same of rows of codes, 4, 8 or 16 chunks, so that eight rows 0 - 3 and 8 - 11, and eight in a row, are spread over the banks
template <int CHUNKS> __device__ __forceinline__ int code_swap(int row) {
    return CHUNKS == 4 ? (row >> 1 & 1) | ((row >> 2 ^ row >> 3) & 1) << 1 : (row & 3) | ((row >> 2 ^ row >> 3) & 1) << 2;
}
// Q8 with few rows: the key whose scores register r of the lanes' lower half has, and the one that lane l % 32 gives the product
__device__ __forceinline__ constexpr int direct_key(int r) { return 16 * (r >> 3) + (r & 7); }
__device__ __forceinline__ int direct_row(int l) { return (l & 16) | (l >> 2 & 1) << 3 | (l & 3) | (l >> 3 & 1) << 2; }

// Registers: two workgroups a compute unit, but of heads of 256 one, whose sums and queries alone take 192 (eight wavefronts: a prompt
// of 8000 tokens 890 us against 803).  What the edge tiles need where a value is not finite decides how many: without it the kernel of many
// rows would take 189 of heads of 128 and 133 of heads of 64, with it 256 and some 200 in scratch memory, and 202.  The loop over inner tiles
// uses no scratch memory, an edge tile stores and reloads about ten values and waits for the tile on its way each time.
// Q8 with few rows: two wavefronts a SIMD, of heads of 64 three (40 windows of 4096 keys: 58 us by two with three tiles in LDS, 48 by three with two), else one.
template <typename T, int D, int NARROW, bool Q8>
__global__ __launch_bounds__((Shape<D, NARROW, Q8>::kWaves * 64), (D > 128 || (NARROW && !Q8) ? 1 : NARROW && D == 64 ? 3 : 2)) void attend_kernel(AttendArgs a) {
    using S = Shape<D, NARROW, Q8>;
    using H = Half<T>;
    constexpr int kKeySteps = D / 16, kBlocks = D / 32, kKeyTiles = S::kKeys / 32;
    constexpr int kBatch = D == 96 ? 3 : 4;
    const int lane = lane_id(), wave = wave_id(), half = lane >> 5;
    const int G = a.group;
    int at = blockIdx.x;
    const bool second = at >= a.first_blocks;
    const AttendArgs::Pass& pass = a.pass[second];
    if (second) at -= a.first_blocks;
    int kvh;
    if constexpr (S::kDirect) {
        // The key heads of a unit's piece to one XCD, to which every eighth workgroup goes: a row of codes of one head, or its powers, may be less
        // than a line of the L2 cache (heads of 64, tokens one after the other: every line was fetched twice, 40 windows of 4096 keys 67 us, now 55).
        // Many rows read their keys again and again: there an XCD that has one head of eight keeps it in its cache (a prompt of 8000 tokens: 858 us, by
        // this 900)
        const int pieces = (second ? (int)gridDim.x - a.first_blocks : a.first_blocks) / a.hkv, whole = pieces & ~7;
        if (at < whole * a.hkv) {
            const int x = at & 7, i = at >> 3;
            kvh = i % a.hkv;
            at = i / a.hkv * 8 + x;
        } else {
            at -= whole * a.hkv;
            kvh = at % a.hkv;
            at = whole + at / a.hkv;
        }
    } else {
        kvh = at % a.hkv; at /= a.hkv;
    }
    int tile0 = 0, split, unit;
    if (pass.n_tile > 0) {
        tile0 = pass.n_tile - 1 - at % pass.n_tile; at /= pass.n_tile;     // the rows that see most first
        split = at % pass.n_split; unit = at / pass.n_split;
    } else {
        // the sequences' tiles one behind the other: which one this is, by looking at 64 sequences at a time
        split = at % pass.n_split; at /= pass.n_split;
        unit = -1;
        for (int s = 0; s < a.step.n_seq && unit < 0; s += 64) {
            const int i = min(s + lane, a.step.n_seq - 1);
            const int n = s + lane < a.step.n_seq ? (max(0, token_of(a.step, i + 1) - token_of(a.step, i)) * G + S::kRows - 1) / S::kRows : 0;
            int upto = n;
            for (int w = 1; w < 64; w <<= 1) { const int x = __shfl_up(upto, w); upto += lane >= w ? x : 0; }
            const uint64_t behind = __ballot(upto > at);
            if (behind) {
                const int l = __builtin_ctzll(behind);
                unit = s + l;
                tile0 = __builtin_amdgcn_readlane(upto, l) - 1 - at;
            } else {
                at -= __builtin_amdgcn_readlane(upto, 63);
            }
        }
        if (unit < 0) return;
    }

    // The unit: its tokens and keys.  Keys, positions, window and sinks are counted from the begin of what the pass reads: own
    // keys alone do not wait for the prefix's length
    const bool by_group = pass.mode == kPrefix;
    int s0 = unit, s1 = unit + 1, g = -1;
    if (by_group) {
        g = unit;
        s0 = min(max(a.step.group_off[g], 0), a.step.n_seq);
        s1 = min(max(a.step.group_off[g + 1], s0), a.step.n_seq);
    } else if (a.step.n_groups > 0) {
        g = group_of(a.step, unit);
    }
    const int t0 = token_of(a.step, s0), t1 = token_of(a.step, s1), own = by_group ? 0 : own_len(a.step, unit);
    const int rows = (t1 - t0) * G;
    if (rows <= pass.rows_lo || rows > pass.rows_hi) return;
    const int before = prefix_of(a.step, g);                               // keys of the prefix, which
    const int plen = pass.mode == kOwn ? 0 : before;                          // this pass reads or not
    if (by_group && plen == 0) return;
    const int sinks = pass.mode == kOwn ? (a.window > 0 ? max(0, a.sinks - before) : 0) : a.sinks;
    const int ke = plen + own;
    const int32_t* ptab = a.step.prefix_table + (int64_t)max(g, 0) * a.step.prefix_stride;
    const int32_t* otab = a.step.table + (int64_t)s0 * a.step.table_stride;

    // position of a token: where its sequence's keys end, less the tokens behind it
    auto position = [&](int t) {
        if (!by_group) return plen + own - (t1 - t);
        int lo = s0, hi = s1;                       // the last sequence that begins at or before t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (a.step.q_off[mid] <= t) lo = mid; else hi = mid;
        }
        return plen + own_len(a.step, lo) - (token_of(a.step, lo + 1) - t);
    };
    // the window's first key, of a position that may be below 0
    auto first_of = [&](int p) { return max(0, max(p, 0) - (a.window - 1)); };

    unsigned char* stage = s_mem + (NARROW ? wave * (S::kStages * S::kTileBytes + S::kPowerBytes) : 0);
    const uint32_t stage_at = __builtin_amdgcn_readfirstlane(lds_address(stage));
    const int32_t* entries = (const int32_t*)(s_mem + S::kStageBytes + wave * S::kEntrySlots * S::kSets * 256);
    const uint32_t entries_at = __builtin_amdgcn_readfirstlane(lds_address(entries));

    // Where a lane's pieces of a tile lie: of keys row l % 32, chunk 2 s + l / 32; of values (see `value`) row 8 u + 4 (l / 32) +
    // (l % 16) / 4, chunk 4 b + 2 (l / 16 % 2) + l % 4 / 2.  Rows begin at multiples of the pitch, so that s, b and u change single
    // bits of the first place
    const int key_place = (lane & 31) * S::kPitch + ((half ^ place_swap<S::kChunks>(lane & 31)) << 4);
    const int value_row = 4 * half + (lane & 15) / 4;
    const int value_place = (S::kKeys + value_row) * S::kPitch + (((2 * (lane >> 4 & 1) + (lane & 3) / 2) ^ place_swap<S::kChunks>(value_row)) << 4) + (lane & 1) * 8;
    constexpr int kRowBit = S::kChunks == 8 ? 0 : 32;
    // Q8 with few rows: 16 codes of key direct_row(l % 32), chunk 2 j + l / 32; and of values, which are read transposed, eight rows 16 s + 8 (l / 32) and on by
    // sixteen lanes, chunk 2 b + l / 16 % 2
    const int direct_place = S::kDirect ? direct_row(lane & 31) * S::kPitch + ((half ^ code_swap<S::kLanes>(direct_row(lane & 31))) << 4) : 0;
    const int direct_value = S::kDirect ? (S::kKeys + 8 * half + (lane & 15) / 2) * S::kPitch + (((lane >> 4 & 1) ^ code_swap<S::kLanes>(8 * half + (lane & 15) / 2)) << 4) + (lane & 1) * 8 : 0;

    // the chunk of a row that a lane fetches by load 0, in bytes; another load's rows change single bits of it
    const int chunk_place = S::kDirect ? ((lane % S::kLanes) ^ code_swap<S::kLanes>(lane / S::kLanes)) * 16 : Q8 ? lane % S::kLanes * 16 : ((lane % S::kChunks) ^ place_swap<S::kChunks>((NARROW ? 0 : wave * S::kWaveRows) + lane / S::kChunks)) * 16;
    auto chunk_bytes = [&](int u) {
        if (S::kDirect) return (uint32_t)(chunk_place ^ (S::kLanes == 4 ? 0 : S::kLanes == 8 ? (u & 1) << 6 : ((u ^ u >> 1) & 1) << 6));
        return Q8 ? (uint32_t)chunk_place : (uint32_t)(chunk_place ^ (S::kChunks == 8 ? 0 : S::kChunks == 16 ? (u & 3) << 4 : (u & 1) << 7 | (u >> 1 & 3) << 4));
    };
    // in registers: a choice between two of the arguments would otherwise be a load, which waits for the tiles on their way
    const int pre_shift = __builtin_amdgcn_readfirstlane(a.step.prefix_shift), own_shift = __builtin_amdgcn_readfirstlane(a.step.shift);
    const int pre_last = __builtin_amdgcn_readfirstlane(a.step.prefix_last), own_last = __builtin_amdgcn_readfirstlane(a.step.own_last);
    const int page_shift = a.cache.page_shift;
    const char* kbase = (const char*)a.cache.k + kvh * a.cache.head_stride * (Q8 ? 1 : 2);
    const char* vbase = (const char*)a.cache.v + kvh * a.cache.head_stride * (Q8 ? 1 : 2);
    const uint8_t* kscales = Q8 ? a.quant.k + kvh * a.quant.head_stride : nullptr;
    const uint8_t* vscales = Q8 ? a.quant.v + kvh * a.quant.head_stride : nullptr;
    // Where a wavefront's rows of every tile lie in one page each, which then is found by scalar instructions alone: pages of at
    // least so many tokens, and a prefix of whole groups of them.  Without this the vector units spend part of their time on places
    // (three prompts, 4250 tokens, heads of 64, behind 6001 keys or with slots for table entries 407 us, behind 6000 in pages 373).
    const bool paged = !NARROW && (plen == 0 || (1 << pre_shift >= S::kWaveRows && plen % S::kWaveRows == 0)) &&
                       1 << own_shift >= S::kWaveRows && a.cache.token_bytes >= 0 && a.cache.token_bytes < 1 << 26;
    uint32_t page_place[NARROW ? 1 : S::kLoads];
#pragma unroll
    for (int u = 0; u < (NARROW ? 1 : S::kLoads); ++u)
        page_place[u] = (uint32_t)((u * S::kRowsPerLoad + lane / S::kLanes) * a.cache.token_bytes) + chunk_bytes(u);
    const int64_t page_scale = Q8 && !NARROW ? (int64_t)((S::kLoads < 4 ? lane & (S::kLoads - 1) : lane & 3) * S::kRowsPerLoad + lane / S::kLanes) * a.quant.token_stride : 0;

    const int tile_step = pass.n_tile > 0 ? pass.n_tile : rows / S::kRows + 1;
    for (int tile = tile0; tile * S::kRows < rows; tile += tile_step) {
        // rows of the workgroup and of this lane
        const int row_first = tile * S::kRows, row_last = min(rows, row_first + S::kRows) - 1;
        const int row = row_first + (NARROW ? 0 : wave * 32) + (lane & 31);
        const bool mine = row < rows;
        const int tok = t0 + (mine ? row : rows - 1) / G, head = kvh * G + (mine ? row : rows - 1) % G;
        const int pos = mine ? position(tok) : -1;
        const int lim = min(pos, ke - 1);                                  // sees keys up to lim that are at or above low, or sinks
        const int low = a.window > 0 ? first_of(pos) : 0;
        // over the workgroup's rows (positions rise inside a sequence; over a group, all rows are looked at)
        int most = -1, least = 0x7FFFFFFF;
        if (by_group) {
            for (int r = row_first + lane; r <= row_last; r += 64) {
                const int p = position(t0 + r / G);
                most = max(most, p);
                least = min(least, p);
            }
            for (int w = 32; w >= 1; w >>= 1) { most = max(most, __shfl_xor(most, w)); least = min(least, __shfl_xor(least, w)); }
        } else {
            most = position(t0 + row_last / G);
            least = position(t0 + row_first / G);
        }
        most = __builtin_amdgcn_readfirstlane(most);
        least = __builtin_amdgcn_readfirstlane(least);
        // the tiles of keys that some row sees: [0, n_sink) and [n_low, n_end) of the grid
        const int end = min(ke, most + 1);
        const int n_end = max(0, end + S::kKeys - 1) / S::kKeys;
        int n_low = 0, n_sink = 0;
        if (a.window > 0) {
            n_low = min(n_end, first_of(least) / S::kKeys);
            n_sink = min(n_low, sinks > 0 ? (min(sinks, end) + S::kKeys - 1) / S::kKeys : 0);
        }
        const int seen = n_sink + n_end - n_low;
        const int per = (seen + pass.n_split - 1) / pass.n_split;
        const int v0 = min(seen, split * per), v1 = min(seen, v0 + per);
        // those whose keys all rows see come first: [inner0, inner1) of them
        const int all_low = a.window > 0 ? first_of(most) : 0;
        const int inner_to = (min(least, ke - 1) + 1) / S::kKeys, inner_from = (all_low + S::kKeys - 1) / S::kKeys;
        const int inner0 = min(v1, max(v0, n_sink + max(inner_from - n_low, 0)));
        const int inner1 = min(v1, max(inner0, n_sink + inner_to - n_low)), inner = inner1 - inner0;
        // of these tiles the wavefront takes n, the first n_full of them inner ones
        auto mine_of = [&](int count) { return NARROW ? (count - wave + S::kWaves - 1) / S::kWaves : count; };
        const int n = mine_of(v1 - v0), n_full = mine_of(inner);
        auto first_key = [&](int i) {
            const int c = NARROW ? wave + i * S::kWaves : i;
            const int v = c < inner ? inner0 + c : v0 + c - inner < inner0 ? v0 + c - inner : v0 + c;
            return (v < n_sink ? v : v - n_sink + n_low) * S::kKeys;
        };

        // the rows of Q as the second operand: lane l, row l % 32, elements 16 s + 8 (l / 32) and on
        s8_t q[kKeySteps];
        {
            const T* src = (const T*)a.q.data + tok * a.q.token_stride + head * a.q.head_stride + half * 8;
#pragma unroll
            for (int s = 0; s < kKeySteps; ++s) {
                // (Q8 with few rows: a lane's sixteen codes in a row serve two steps)
                if constexpr (S::kDirect) q[s] = mine ? *(const s8_t*)(src + (s >> 1) * 32 + half * 8 + (s & 1) * 8) : s8_t{};
                else q[s] = mine ? *(const s8_t*)(src + s * 16) : s8_t{};
            }
            // waited for here: in the loops below, a wait for them would be one for the tiles on their way
#pragma unroll
            for (int s = 0; s < kKeySteps; ++s) asm volatile("" : "+v"(q[s]));
        }

        // Fetching.  Load u of a wavefront brings rows u * kRowsPerLoad + lane / kChunks; four loads make a set, and lane l keeps
        // the place of the row that load l % 4 of the set brings to its group, so that a load finds its lanes' places in the
        // lanes' own quads
        auto row_of = [&](int set) {
            const int lane = D > 128 ? again(lane_id()) : lane_id();
            return (NARROW ? 0 : wave * S::kWaveRows) + (S::kLoads < 4 ? lane & (S::kLoads - 1) : set * 4 + (lane & 3)) * S::kRowsPerLoad + lane / S::kLanes;
        };
        auto key_of = [&](int i, int set) { return min(first_key(i) + row_of(set), ke - 1); };
        auto fetch_entries = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int set = 0; set < S::kSets; ++set) {
                const int key = key_of(i, set);
                const bool pre = key < plen;
                fetch4((pre ? ptab : otab) + ((pre ? key : key - plen) >> (pre ? pre_shift : own_shift)), entries_at + ((i & (S::kEntrySlots - 1)) * S::kSets + set) * 256);
            }
        };
        // the first key of the wavefront's rows of a tile, where they lie in one page; its entry is read by a scalar load
        auto page_key = [&](int i) { return min(first_key(i) + wave * S::kWaveRows, (ke - 1) & -S::kWaveRows); };
        auto page_entry = [&](int i) {
            const int key = page_key(i);
            typedef const __attribute__((address_space(4))) int32_t* scalar_t;
            return key < plen ? *(scalar_t)(uintptr_t)(ptab + (key >> pre_shift)) : *(scalar_t)(uintptr_t)(otab + ((key - plen) >> own_shift));
        };
        int entry = 0;                     // of the next tile to be fetched
        // Q8: the codes of a tile on its way, of the rows that a lane's loads bring, and the powers' bytes of the row whose place it keeps
        uint4 kcode[Q8 ? S::kLoads : 1], vcode[Q8 ? S::kLoads : 1];
        int kbyte[Q8 ? S::kSets : 1], vbyte[Q8 ? S::kSets : 1];
        // bytes from the cache's begin (and from that of the powers), of the wavefront's rows of a tile
        auto page_at = [&](int i, int64_t* scale) __attribute__((always_inline)) {
            const int key = page_key(i);
            const bool pre = key < plen;
            const int shift = pre ? pre_shift : own_shift, up = page_shift - shift, j = pre ? key : key - plen;
            const int e = min(max(entry, 0), pre ? pre_last : own_last);
            const int in_page = (e & ((1 << up) - 1)) << shift | (j & ((1 << shift) - 1));
            if (Q8) *scale = (int64_t)(e >> up) * (int)a.quant.page_stride + (int64_t)in_page * (int)a.quant.token_stride;
            return (int64_t)(e >> up) * a.cache.page_bytes + (int64_t)in_page * a.cache.token_bytes;
        };
        auto fetch_paged = [&](int i) __attribute__((always_inline)) {
            const int64_t at = page_at(i, nullptr);
            const uint32_t to = stage_at + (i % S::kStages) * S::kTileBytes + wave * S::kWaveRows * S::kPitch;
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u)
                if (D % 64 == 0 || chunk_bytes(u) < D * 2) {
                    fetch16(kbase + at, page_place[u], to + u * 1024);
                    fetch16(vbase + at, page_place[u], to + S::kKeys * S::kPitch + u * 1024);
                }
        };
        int64_t place[S::kSets];           // bytes from the cache's begin, of the next tile to be fetched
        int64_t scale_place[Q8 ? S::kSets : 1];
        auto locate = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int set = 0; set < S::kSets; ++set) {
                const int key = key_of(i, set);
                const bool pre = key < plen;
                const int shift = pre ? pre_shift : own_shift, up = page_shift - shift;
                const int e = min(max(entries[((i & (S::kEntrySlots - 1)) * S::kSets + set) * 64 + lane], 0), pre ? pre_last : own_last);
                const int j = pre ? key : key - plen;
                const int in_page = (e & ((1 << up) - 1)) << shift | (j & ((1 << shift) - 1));
                place[set] = (int64_t)(e >> up) * a.cache.page_bytes + (int64_t)in_page * a.cache.token_bytes;
                if constexpr (Q8 && !S::kDirect) scale_place[set] = (int64_t)(e >> up) * (int)a.quant.page_stride + (int64_t)in_page * (int)a.quant.token_stride;
            }
            if constexpr (S::kDirect) {
                // of key l % 32, whose entry another lane has fetched
                const int r = lane & 31, from = r / (4 * S::kRowsPerLoad) * 64 + r % S::kRowsPerLoad * S::kLanes + r / S::kRowsPerLoad % 4;
                const int key = min(first_key(i) + r, ke - 1);
                const bool pre = key < plen;
                const int shift = pre ? pre_shift : own_shift, up = page_shift - shift;
                const int e = min(max(entries[(i & (S::kEntrySlots - 1)) * S::kSets * 64 + from], 0), pre ? pre_last : own_last);
                const int in_page = (e & ((1 << up) - 1)) << shift | ((pre ? key : key - plen) & ((1 << shift) - 1));
                scale_place[0] = (int64_t)(e >> up) * (int)a.quant.page_stride + (int64_t)in_page * (int)a.quant.token_stride;
            }
        };
        auto fetch_tile = [&](int i) __attribute__((always_inline)) {
            if constexpr (Q8) {
                const uint32_t to = stage_at + (i % S::kStages) * S::kTileBytes;
#pragma unroll
                for (int u = 0; u < S::kLoads; ++u) {
                    const int64_t at = quad_lane(place[u / 4], u & 3) + chunk_bytes(u);        // by all lanes
                    if (D % 64 == 0 || chunk_bytes(u) < D) {
                        fetch16(kbase + at, to + u * 1024);
                        fetch16(vbase + at, to + S::kKeys * S::kPitch + u * 1024);
                    }
                }
                fetch_byte((half ? vscales : kscales) + scale_place[0], to + 2 * S::kKeys * S::kPitch);
                return;
            }
            const uint32_t to = stage_at + (i % S::kStages) * S::kTileBytes + (NARROW ? 0 : wave * S::kWaveRows * S::kPitch);
            const int swap = D > 128 ? again(chunk_place) : chunk_place;
            auto chunk_bytes = [&](int u) {
                return (uint32_t)(swap ^ (S::kChunks == 8 ? 0 : S::kChunks == 16 ? (u & 3) << 4 : (u & 1) << 7 | (u >> 1 & 3) << 4));
            };
#pragma unroll
            for (int u = 0; u < S::kLoads; ++u) {
                const int64_t at = quad_lane(place[u / 4], u & 3) + chunk_bytes(u);
                if (D % 64 == 0 || chunk_bytes(u) < D * 2) {
                    fetch16(kbase + at, to + u * 1024);
                    fetch16(vbase + at, to + S::kKeys * S::kPitch + u * 1024);
                }
            }
        };

        // Q8 with many rows: a tile's codes on their way to registers.  (One place for both ways to find them: two would each load into registers of their
        // own, and wait, to copy them)
        auto fetch_codes = [&](int i) __attribute__((always_inline)) {
            if constexpr (Q8 && !S::kDirect) {
                static_assert(S::kSets == 1, "one set of loads");
                int64_t at[S::kLoads], scale;
                if (paged) {
                    const int64_t first = page_at(i, &scale);
                    scale += page_scale;
#pragma unroll
                    for (int u = 0; u < S::kLoads; ++u) at[u] = first + page_place[u];
                } else {
                    scale = scale_place[0];
#pragma unroll
                    for (int u = 0; u < S::kLoads; ++u) at[u] = quad_lane(place[0], u & 3) + chunk_place;       // by all lanes
                }
                kbyte[0] = kscales[scale];
                vbyte[0] = vscales[scale];
#pragma unroll
                for (int u = 0; u < S::kLoads; ++u)
                    if (D % 64 == 0 || chunk_place < D) {
                        kcode[u] = *(const uint4*)(kbase + at[u]);
                        vcode[u] = *(const uint4*)(vbase + at[u]);
                    }
            }
        };
        // Q8 with many rows: the codes that arrived by load c (of keys, then of values), as numbers of the rows' type, to the place that the tile's
        // products read them from.  A lane's 16 codes are two chunks of a row there
        auto put_codes = [&](int i, int c) __attribute__((always_inline)) {
            if constexpr (Q8 && !S::kDirect) {
                const int u = c % S::kLoads, r = wave * S::kWaveRows + u * S::kRowsPerLoad + lane / S::kLanes;
                const uint32_t at = stage_at + (i % S::kStages) * S::kTileBytes + (c < S::kLoads ? 0 : S::kKeys * S::kPitch) + r * S::kPitch +
                                    ((lane % S::kLanes * 2 ^ place_swap<S::kChunks>(r)) << 4);
                const float p = __int_as_float(quad_lane(__float_as_int(power_of(a.quant, c < S::kLoads ? kbyte[0] : vbyte[0])), u & 3));      // by all lanes
                const uint4 x = c < S::kLoads ? kcode[u] : vcode[u];
                if (D % 64 == 0 || chunk_place < D) {
                    *(lds_u4)(uintptr_t)at = u4_t{from_e4m3<T, false>(x.x, p), from_e4m3<T, true>(x.x, p), from_e4m3<T, false>(x.y, p), from_e4m3<T, true>(x.y, p)};
                    *(lds_u4)(uintptr_t)(at ^ 16) = u4_t{from_e4m3<T, false>(x.z, p), from_e4m3<T, true>(x.z, p), from_e4m3<T, false>(x.w, p), from_e4m3<T, true>(x.w, p)};
                }
            }
        };
        constexpr int kPuts = Q8 && !S::kDirect ? 2 * S::kLoads : 0;
        auto put_tile = [&](int i) __attribute__((always_inline)) {
#pragma unroll
            for (int c = 0; c < kPuts; ++c) put_codes(i, c);
        };

        f16v_t o[kBlocks] = {};
        float m = -INFINITY, l = 0.f;

        // The sums of heads of 256 stay in accumulation registers but where they are scaled; else all 128 change sides twice a tile (a
        // prompt of 8000 tokens: 803 us against 659)
        auto keep_sums = [&]() __attribute__((always_inline)) {
            if constexpr (!NARROW && D > 128) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) asm volatile("" : "+a"(o[b]));
            }
        };

        // Q8 with few rows, bf16: the weights are multiplied by the values' powers
        constexpr bool kByPower = S::kDirect && !std::is_same<T, _Float16>::value;
        // one tile: scores, weights, products; `full`: every row sees all its keys.  False: nothing is done, it is one for the other
        // kind, which is right for all
        auto compute = [&](int i, auto full_tag) __attribute__((always_inline)) {
            constexpr bool full = decltype(full_tag)::value;
            const int j0 = first_key(i);
            const uint32_t tile_at = stage_at + (i % S::kStages) * S::kTileBytes;
            keep_sums();
            const uint32_t key_at = tile_at + key_place, value_at = tile_at + value_place;
            f16v_t x[kKeyTiles];
#pragma unroll
            for (int t = 0; t < kKeyTiles; ++t) x[t] = f16v_t{};
            // what register r of tile t's scores is, less what all of a lane have in common
            auto key_index = [](int t, int r) { return S::kDirect ? direct_key(r) : t * 32 + (r & 3) + 8 * (r >> 2); };
            const int lane_key = (S::kDirect ? 8 : 4) * half;
            // Q8 with few rows: the powers of the values, in the order of their keys: of f16 the two that a product of two takes; of bf16, which has no such
            // products, those that the weights are multiplied by.  That changes nothing but exponents unless a power is near the ends of what bf16 holds: weights
            // are up to 2^8, and times 2^119 below 2^128; what rounding takes from w 2^-60 because it is below 2^-126 is below 2^-66 of the largest weight.
            // From a tile with other powers on, and in edge tiles, every value is converted by its own: two at a time by the first's power and by the
            // second's.  (All tiles so: 24 sequences of up to 60,000 keys as above 373 us, not 297.  24 of up to 20,000 of which many heads are all zeros,
            // under 2^-117: 122 us, not 117)
            constexpr int kEndLow = 127 - 60, kEndHigh = 127 + 119;
            u4_t half_powers[2];
            f4_t powers[4];
            const uint32_t direct_at = tile_at + direct_value;
            if constexpr (S::kDirect) {
                const lds_ptr<const int> bytes = (lds_ptr<const int>)(uintptr_t)(tile_at + 2 * S::kKeys * S::kPitch);
                const uint32_t table = stage_at + S::kStages * S::kTileBytes;
                u4_t c[D / 32];
#pragma unroll
                for (int j = 0; j < D / 32; ++j) c[j] = *(lds_ptr<const u4_t>)(uintptr_t)((tile_at + direct_place) ^ (uint32_t)(j << 5));
                const int vbyte = bytes[32 + (lane & 31)];
                const float kp = power_of(a.quant, bytes[direct_row(lane & 31)]), vp = power_of(a.quant, vbyte);
                if constexpr (kByPower) ((lds_ptr<float>)(uintptr_t)table)[lane & 31] = vp;
                else ((lds_ptr<_Float16>)(uintptr_t)table)[lane & 31] = (_Float16)vp;
#pragma unroll
                for (int j = 0; j < D / 32; ++j)
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const u4_t k = {from_e4m3<T, false>(c[j][2 * u], kp), from_e4m3<T, true>(c[j][2 * u], kp), from_e4m3<T, false>(c[j][2 * u + 1], kp),
                                        from_e4m3<T, true>(c[j][2 * u + 1], kp)};
                        x[0] = H::mfma(__builtin_bit_cast(s8_t, k), q[2 * j + u], x[0]);
                    }
#pragma unroll
                for (int u = 0; u < (kByPower ? full ? 4 : 0 : 2); ++u) {
                    if constexpr (!kByPower) half_powers[u] = *(lds_ptr<const u4_t>)(uintptr_t)(table + (16 * u + 8 * half) * 2);
                    else powers[u] = *(lds_ptr<const f4_t>)(uintptr_t)(table + (16 * (u / 2) + 8 * half + 4 * (u & 1)) * 4);
                }
                if (kByPower && full && __ballot((uint32_t)(vbyte - kEndLow) > kEndHigh - kEndLow) != 0) return false;
            } else {
            // reads of LDS run kBatch products ahead: one wavefront's products then hide their latency
            constexpr int kScores = kKeySteps * kKeyTiles;
            auto key = [&](int c) __attribute__((always_inline)) {
                return *(lds_s8)(uintptr_t)((key_at ^ (uint32_t)(c / kKeyTiles << 5)) + c % kKeyTiles * 32 * S::kPitch);
            };
            s8_t k[2][kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) k[0][u] = key(u);
#pragma unroll
            for (int c = 0; c < kScores; c += kBatch) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    if (c + kBatch + u < kScores) k[(c / kBatch + 1) & 1][u] = key(c + kBatch + u);
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    x[(c + u) % kKeyTiles] = H::mfma(k[c / kBatch & 1][u], q[(c + u) / kKeyTiles], x[(c + u) % kKeyTiles]);
            }
            __builtin_amdgcn_sched_barrier(0);
            }
            auto sees = [&](int j) { return j <= lim && (j >= low || j < sinks); };
            if (!full) {
                const int to = lim - j0 - lane_key, from = low - j0 - lane_key, sunk = sinks - j0 - lane_key;
#pragma unroll
                for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
                    for (int r = 0; r < 16; ++r) x[t][r] = key_index(t, r) <= to ? x[t][r] : -INFINITY;
                if (a.window > 0) {
#pragma unroll
                    for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int j = key_index(t, r);
                            x[t][r] = j >= from || j < sunk ? x[t][r] : -INFINITY;
                        }
                }
            }
            float top = x[0][0];
#pragma unroll
            for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; ++r) top = fmaxf(top, x[t][r]);
            top = fmaxf(top, other_half(top)) * a.scale_log2;
            if (__ballot(top > m + kSlack) != 0) {
                const float m2 = fmaxf(m, top);
                const float f = m2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - m2);
                m = m2;
                l *= f;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) o[b] *= f;
            }
            keep_sums();
            // The weights are summed as they are and rounded to the cache's type for the product, whose operands are 16 bits wide: a term is
            // off by at most 2^-8 (bf16) or 2^-11 (f16) of itself, as the result's own rounding is.  Against 64 bits the results are
            // then off by 1.2 to 1.4 times what 32-bit weights leave (bf16 0.0022 of their size and 0.0017, f16 0.00028 and 0.00021)
            const float minus = (m == -INFINITY ? 0.f : -m) + H::kLift;
            s8_t p[kKeyTiles * 2];
            float sum[2] = {0.f, 0.f};
#pragma unroll
            for (int t = 0; t < kKeyTiles; ++t)
#pragma unroll
                for (int r = 0; r < 16; r += 2) {
                    const float w0 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][r], a.scale_log2, minus));
                    const float w1 = __builtin_amdgcn_exp2f(__builtin_fmaf(x[t][r + 1], a.scale_log2, minus));
                    sum[0] += w0;
                    sum[1] += w1;
                    p[t * 2 + r / 8][r % 8] = __builtin_bit_cast(short, (T)(kByPower && full ? w0 * powers[r / 4][r % 4] : w0));
                    p[t * 2 + r / 8][r % 8 + 1] = __builtin_bit_cast(short, (T)(kByPower && full ? w1 * powers[r / 4][r % 4 + 1] : w1));
                }
            l += sum[0] + sum[1];
            // V transposed, the keys in the order of p: lane l, element l % 32 of a block of 32, keys 16 s + 4 (l / 32) .. + 4 and
            // eight behind those
            auto codes = [&](int s, int b) __attribute__((always_inline)) {
                return __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i2)(uintptr_t)((direct_at ^ (uint32_t)(b << 5)) + s * 16 * S::kPitch));
            };
            auto of_codes = [&](i2_t c, int s) __attribute__((always_inline)) {
                u4_t v = {from_e4m3<T, false>(c[0], 1.f), from_e4m3<T, true>(c[0], 1.f), from_e4m3<T, false>(c[1], 1.f), from_e4m3<T, true>(c[1], 1.f)};
                if constexpr (!kByPower) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] = __builtin_bit_cast(uint32_t, __builtin_bit_cast(h2_t, (uint32_t)v[e]) * __builtin_bit_cast(h2_t, (uint32_t)half_powers[s][e]));
                }
                return __builtin_bit_cast(s8_t, v);
            };
            // bf16, each by its own power
            auto by_powers = [&](i2_t c, f4_t first, f4_t second) __attribute__((always_inline)) {
                u4_t v;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const f4_t power = e < 2 ? first : second;
                    const uint32_t low = e & 1 ? from_e4m3<T, true>(c[e / 2], power[2]) : from_e4m3<T, false>(c[e / 2], power[0]);
                    const uint32_t high = e & 1 ? from_e4m3<T, true>(c[e / 2], power[3]) : from_e4m3<T, false>(c[e / 2], power[1]);
                    v[e] = __builtin_amdgcn_perm(high, low, 0x07060100u);
                }
                return __builtin_bit_cast(s8_t, v);
            };
            auto value = [&](int s, int b) __attribute__((always_inline)) {
                if constexpr (kByPower) {
                    const uint32_t at = stage_at + S::kStages * S::kTileBytes + (16 * s + 8 * half) * 4;
                    return by_powers(codes(s, b), *(lds_ptr<const f4_t>)(uintptr_t)at, *(lds_ptr<const f4_t>)(uintptr_t)(at + 16));
                }
                if constexpr (S::kDirect) return of_codes(codes(s, b), s);
                s8_t v;
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const s4_t y = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                        (lds_s4)(uintptr_t)((value_at ^ (uint32_t)(b << 6 | u * kRowBit)) + (u * 8 + s * 16) * S::kPitch));
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[u * 4 + e] = y[e];
                }
                return v;
            };
            if (!full) {
                // A value that is not finite, times the weight zero of a row that does not see it, is NaN.  So a block of the tile's
                // sums is formed by itself, and added if it is finite (the check that costs least: reading all values for it
                // beforehand took longer than the products).  If not, such values are left out of the product, and counted
                // instead for the rows that see them, the three kinds in one number
#pragma unroll
                for (int b = 0; b < kBlocks; ++b) {
                    f16v_t y{};
#pragma unroll
                    for (int s = 0; s < kKeyTiles * 2; ++s) y = H::mfma(value(s, b), p[s], y);
                    float odd = 0.f;                                   // NaN where one is not finite
#pragma unroll
                    for (int r = 0; r < 16; ++r) odd = __builtin_fmaf(y[r], 0.f, odd);
                    if (__builtin_expect(__ballot(odd != odd) != 0, 0)) {
                        auto of = [](float x) { return __builtin_bit_cast(short, (T)x); };
                        f16v_t n{};
                        y = f16v_t{};
#pragma unroll
                        for (int s = 0; s < kKeyTiles * 2; ++s) {
                            s8_t v = value(s, b), kind, seen;
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                const int j = j0 + 16 * s + (S::kDirect ? e : (e & 3) + 8 * (e >> 2)) + lane_key;
                                const uint32_t bits = (uint16_t)v[e];
                                const bool finite = (bits & H::kExponent) != H::kExponent;
                                kind[e] = finite ? (short)0 : (bits & 0x7FFFu) != H::kExponent ? of(16384.f) : bits >> 15 ? of(128.f) : of(1.f);
                                v[e] = finite ? v[e] : (short)0;
                                seen[e] = sees(j) ? of(1.f) : (short)0;
                            }
                            y = H::mfma(v, p[s], y);
                            n = H::mfma(kind, seen, n);
                        }
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int c = (int)n[r];           // NaN, -inf and +inf by digits of 128
                            if (c != 0) y[r] += c >= 16384 || ((c & 127) && c >= 128) ? NAN : c >= 128 ? -INFINITY : INFINITY;
                        }
                    }
                    o[b] += y;
                }
                return true;
            }
            constexpr int kSums = kKeyTiles * 2 * kBlocks;
            if constexpr (S::kDirect) {
                i2_t v[2][kBatch];
#pragma unroll
                for (int u = 0; u < kBatch; ++u) v[0][u] = codes(u / kBlocks, u % kBlocks);
#pragma unroll
                for (int c = 0; c < kSums; c += kBatch) {
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        if (c + kBatch + u < kSums) v[(c / kBatch + 1) & 1][u] = codes((c + kBatch + u) / kBlocks, (c + kBatch + u) % kBlocks);
#pragma unroll
                    for (int u = 0; u < kBatch; ++u)
                        o[(c + u) % kBlocks] = H::mfma(of_codes(v[c / kBatch & 1][u], (c + u) / kBlocks), p[(c + u) / kBlocks], o[(c + u) % kBlocks]);
                }
                __builtin_amdgcn_sched_barrier(0);
                return true;
            }
            s8_t v[2][kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) v[0][u] = value(u / kBlocks, u % kBlocks);
#pragma unroll
            for (int c = 0; c < kSums; c += kBatch) {
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int u = 0; u < kBatch; ++u)
                    if (c + kBatch + u < kSums) v[(c / kBatch + 1) & 1][u] = value((c + kBatch + u) / kBlocks, (c + kBatch + u) % kBlocks);
#pragma unroll
                for (int u = 0; u < kBatch; ++u) o[(c + u) % kBlocks] = H::mfma(v[c / kBatch & 1][u], p[(c + u) / kBlocks], o[(c + u) % kBlocks]);
            }
            __builtin_amdgcn_sched_barrier(0);
            return true;
        };

        // Q8 with many rows: a tile is fetched into registers two tiles ahead, and put into LDS one ahead.  (Put piece by piece between the products of
        // scores a prompt of 8000 tokens took 962 us against 985, but what the edge tiles then stored in scratch memory cost more: windows of 1024 284 against
        // 239, a prompt of 4000 tokens with heads of 256 481 against 235)
        constexpr bool kConvert = Q8 && !S::kDirect;
        constexpr int kLocate = S::kDirect ? S::kStages : kConvert ? 3 : 2;
        if constexpr (S::kDirect) {
            // the entries of a tile come before the tile that is as many stages behind it, so that they are there when that one is
            if (n > 0) {
#pragma unroll
                for (int i = 0; i < S::kStages; ++i)
                    if (i < n) fetch_entries(i);
                wait_loads();
#pragma unroll
                for (int i = 0; i + 1 < S::kStages; ++i)
                    if (i < n) {
                        locate(i);
                        if (i + S::kStages < n) fetch_entries(i + S::kStages);
                        fetch_tile(i);
                    }
                if (S::kStages - 1 < n) locate(S::kStages - 1);
            }
        } else if constexpr (kConvert) {
            if (n > 0) {
                if (paged) {
                    entry = page_entry(0);
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (i < n) fetch_entries(i);
                    wait_loads();
                    locate(0);
                }
                fetch_codes(0);
                if (paged) {
                    if (n > 1) entry = page_entry(1);
                } else if (n > 1) {
                    locate(1);
                }
                put_tile(0);
                if (n > 1) fetch_codes(1);
                if (paged) {
                    if (n > 2) entry = page_entry(2);
                } else if (n > 2) {
                    locate(2);
                }
            }
        } else if (paged) {
            if (n > 0) { entry = page_entry(0); fetch_paged(0); }
            if (n > 1) entry = page_entry(1);
        } else if (n > 0) {
#pragma unroll
            for (int i = 0; i < 3; ++i)
                if (i < n) fetch_entries(i);
            wait_loads();
            locate(0);
            fetch_tile(0);
            if (n > 1) locate(1);
        }
        auto arrive = [&](int i) __attribute__((always_inline)) {
            if constexpr (S::kDirect) {
                wait_loads();
                if (i + 2 * S::kStages - 1 < n) fetch_entries(i + 2 * S::kStages - 1);
                if (i + S::kStages - 1 < n) fetch_tile(i + S::kStages - 1);
                return;
            }
            if constexpr (kConvert) {
                wait_loads();            // the codes of tile i + 1 have arrived, and the entries that the next places come from
                barrier();               // for every wavefront: tile i is in LDS, and the tile before has been read
                if (i + 1 < n) put_tile(i + 1);
                if (!paged && i + 4 < n) fetch_entries(i + 4);
                if (i + 2 < n) fetch_codes(i + 2);
                if (paged && i + 3 < n) entry = page_entry(i + 3);
                return;
            }
            wait_loads();                // tile i has arrived
            if (!NARROW) barrier();      // for every wavefront, and the tile before has been read
            if (paged) {
                if (i + 1 < n) fetch_paged(i + 1);
                if (i + 2 < n) entry = page_entry(i + 2);
                return;
            }
            if (i + 1 < n) fetch_tile(i + 1);
            if (i + 3 < n) fetch_entries(i + 3);
        };
        const bool idle = !NARROW && row_first + wave * 32 >= rows;        // no rows: this wavefront only fetches
        // the keys that some row of the wavefront sees: [0, wave_sinks) and [wave_low, wave_lim]
        int wave_lim = lim, wave_low = mine ? low : 0x7FFFFFFF;
        for (int w = 16; w >= 1; w >>= 1) { wave_lim = max(wave_lim, __shfl_xor(wave_lim, w)); wave_low = min(wave_low, __shfl_xor(wave_low, w)); }
        wave_lim = __builtin_amdgcn_readfirstlane(wave_lim);
        wave_low = __builtin_amdgcn_readfirstlane(wave_low);
        auto unseen = [&](int i) {
            const int j = first_key(i);
            return j > wave_lim || (j + S::kKeys <= wave_low && j >= sinks);
        };
        // two loops, so that what the tiles at the edges need takes no registers from the others
        if constexpr (kByPower) {
            int i = 0;
            bool here = false;             // tile i has arrived
            for (; i < n_full; ++i) {
                arrive(i);
                if (!idle && !compute(i, std::true_type{})) { here = true; break; }
                if (!paged && i + kLocate < n) locate(i + kLocate);
            }
            for (; i < n; ++i) {
                if (!here) arrive(i);
                here = false;
                if (!idle && !unseen(i)) compute(i, std::false_type{});
                if (!paged && i + kLocate < n) locate(i + kLocate);
            }
        } else {
            for (int i = 0; i < n_full; ++i) {
                arrive(i);
                if (!idle) compute(i, std::true_type{});
                if (!paged && i + kLocate < n) locate(i + kLocate);
            }
            for (int i = n_full; i < n; ++i) {
                arrive(i);
                if (!idle && !unseen(i)) compute(i, std::false_type{});
                if (!paged && i + kLocate < n) locate(i + kLocate);
            }
        }
        l += other_half(l);

        // what is left to do with the sums
        const bool last = pass.mode == kConcat && pass.n_split == 1;             // they are complete
        const bool few = NARROW && !by_group && a.few_tokens > 0;
        auto piece = [&](int t, int h) {                                   // its place among the partial sums
            return few ? (((int64_t)unit * a.few_tokens + (t - t0)) * a.hq + h) * a.few_parts + split : ((int64_t)t * a.hq + h) * a.parts + pass.part0 + split;
        };
        auto finish = [&](int t, int h, float mm, float ll) {              // by one lane per row
            if (a.lse && last) a.lse[(int64_t)t * a.hq + h] = ll > 0.f || ll != ll ? (mm + __builtin_amdgcn_logf(ll) - H::kLift) * 0.6931471805599453f : -INFINITY;
            if (few) a.few_ml[piece(t, h)] = make_float2(mm, ll);
            if (a.parts == 0) return;
            float2* ml = a.part_ml + ((int64_t)t * a.hq + h) * a.parts;
            if (!few) ml[pass.part0 + split] = make_float2(last ? NAN : mm, ll);
            else if (split == 0) ml[pass.part0].x = NAN;
            if (split == 0) {
                for (int i = pass.n_split; i < pass.n_part && !few; ++i) ml[pass.part0 + i] = make_float2(-INFINITY, 0.f);
                if (pass.mode == kOwn && before == 0)                           // no prefix pass comes by here
                    for (int i = 0; i < pass.part0; ++i) ml[i] = make_float2(-INFINITY, 0.f);
            }
        };
        if (!NARROW) {
            if (mine) {
                if (half == 0) finish(tok, head, m, l);
                const float f = last ? (l > 0.f || l != l ? 1.f / l : 0.f) : 1.f;
                T* out = (T*)a.out.data + tok * a.out.token_stride + head * a.out.head_stride;
                float* part = last ? nullptr : a.part_o + piece(tok, head) * D;
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int r = 0; r < 16; r += 4) {
                        const int d = 32 * b + 2 * r + 4 * half;
                        if (last) {
                            s4_t y;
#pragma unroll
                            for (int e = 0; e < 4; ++e) y[e] = __builtin_bit_cast(short, (T)(o[b][r + e] * f));
                            *(s4_t*)(out + d) = y;
                        } else if (v1 > v0) {
                            *(float4*)(part + d) = make_float4(o[b][r], o[b][r + 1], o[b][r + 2], o[b][r + 3]);
                        }
                    }
            }
            barrier();                   // the tiles have been read before the next rows' are fetched
        } else {
            // the wavefronts' sums are joined through LDS: [wavefront][row][D], and [wavefront][row] (m, l)
            __syncthreads();
            float* so = (float*)s_mem;
            float2* sm = (float2*)(s_mem + (size_t)S::kWaves * 32 * D * 4);
            if (half == 0) sm[wave * 32 + (lane & 31)] = make_float2(m, l);
            __syncthreads();
            float mm = -INFINITY;
#pragma unroll
            for (int w = 0; w < S::kWaves; ++w) mm = fmaxf(mm, sm[w * 32 + (lane & 31)].x);
            const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
            if (mine) {
#pragma unroll
                for (int b = 0; b < kBlocks; ++b)
#pragma unroll
                    for (int r = 0; r < 16; r += 4)
                        *(float4*)(so + ((size_t)wave * 32 + (lane & 31)) * D + 32 * b + 2 * r + 4 * half) =
                            make_float4(o[b][r] * f, o[b][r + 1] * f, o[b][r + 2] * f, o[b][r + 3] * f);
            }
            __syncthreads();
            const int count = row_last - row_first + 1;
            for (int c = threadIdx.x; c < count * (D / 4); c += S::kWaves * 64) {
                const int r = c / (D / 4), d = c % (D / 4) * 4;
                const int t = t0 + (row_first + r) / G, h = kvh * G + (row_first + r) % G;
                float top = -INFINITY, sum = 0.f;
                float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                for (int w = 0; w < S::kWaves; ++w) top = fmaxf(top, sm[w * 32 + r].x);
#pragma unroll
                for (int w = 0; w < S::kWaves; ++w) {
                    const float2 p = sm[w * 32 + r];
                    sum += p.x == -INFINITY ? p.y : p.y * __builtin_amdgcn_exp2f(p.x - top);
                    const float4 z = *(const float4*)(so + ((size_t)w * 32 + r) * D + d);
                    y.x += z.x; y.y += z.y; y.z += z.z; y.w += z.w;
                }
                if (d == 0) finish(t, h, top, sum);
                if (last) {
                    const float g1 = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
                    s4_t z = {__builtin_bit_cast(short, (T)(y.x * g1)), __builtin_bit_cast(short, (T)(y.y * g1)),
                              __builtin_bit_cast(short, (T)(y.z * g1)), __builtin_bit_cast(short, (T)(y.w * g1))};
                    *(s4_t*)((T*)a.out.data + t * a.out.token_stride + h * a.out.head_stride + d) = z;
                } else if (v1 > v0) {
                    *(float4*)((few ? a.few_o : a.part_o) + piece(t, h) * D + d) = y;
                }
            }
            __syncthreads();
        }
    }
}

// Joins a row's partial sums: one wavefront per token and query head, bound by latency (1536 rows of 34 parts of 128: 7 us).  Lane i weighs part i; then D / 4 lanes take a part's
// elements, and several parts at a time are on their way.  FEW: the own ones are those of place `few`.
template <typename T, int D, bool FEW>
__device__ __forceinline__ void join_row(const AttendArgs& a, int64_t row, int64_t few, int lane) {
    constexpr int kLanes = D / 4, kAtOnce = 64 / kLanes;             // lanes of a part; parts of one load
    constexpr int kUnroll = 4;
    const int parts = FEW ? a.part_own + a.few_parts : a.parts;
    auto ml = [&](int i) { return FEW && i >= a.part_own ? a.few_ml[few * a.few_parts + i - a.part_own] : a.part_ml[row * a.parts + i]; };
    auto po = [&](int i) { return FEW && i >= a.part_own ? a.few_o + (few * a.few_parts + i - a.part_own) * D : a.part_o + (row * a.parts + i) * D; };
    float m = -INFINITY, sum = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
    const int group = min(lane / kLanes, kAtOnce - 1), d = lane % kLanes * 4;
    for (int p0 = 0; p0 < parts; p0 += 64) {                         // 64 parts at a time
        const float2 p = p0 + lane < parts ? ml(p0 + lane) : make_float2(-INFINITY, 0.f);
        if (__ballot(p.x != p.x)) return;                            // complete already
        float top = p.x;
        for (int w = 32; w >= 1; w >>= 1) top = fmaxf(top, __shfl_xor(top, w));
        const float m2 = fmaxf(m, top);
        if (m2 == -INFINITY) {                                       // nothing seen, or no score is a number: then the sums are NaN
            sum += group_sum<64>(p.y);
            continue;
        }
        const float keep = __builtin_amdgcn_exp2f(m - m2);
        const float f = p.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(p.x - m2);
        m = m2;
        sum = sum * keep + group_sum<64>(p.y * f);
        o.x *= keep; o.y *= keep; o.z *= keep; o.w *= keep;
        const int n = min(64, parts - p0);
        for (int i0 = 0; i0 < n; i0 += kAtOnce * kUnroll) {
            float4 y[kUnroll];
            float w[kUnroll];
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) {
                const int i = i0 + u * kAtOnce + group;
                const float weight = __shfl(f, i & 63), at = __shfl(p.x, i & 63);      // by all lanes
                const bool has = i < n && at > -INFINITY && lane < kLanes * kAtOnce;
                y[u] = has ? *(const float4*)(po(p0 + i) + d) : make_float4(0.f, 0.f, 0.f, 0.f);
                w[u] = has ? weight : 0.f;
            }
#pragma unroll
            for (int u = 0; u < kUnroll; ++u) { o.x += y[u].x * w[u]; o.y += y[u].y * w[u]; o.z += y[u].z * w[u]; o.w += y[u].w * w[u]; }
        }
    }
    // the groups of lanes
    auto add = [&](int from) { o.x += __shfl(o.x, from); o.y += __shfl(o.y, from); o.z += __shfl(o.z, from); o.w += __shfl(o.w, from); };
    if (kLanes == 16) { add(lane ^ 32); add(lane ^ 16); }
    if (kLanes == 24) add((lane + 24) & 63);
    if (kLanes == 32) add(lane ^ 32);
    const int t = (int)(row / a.hq), h = (int)(row % a.hq);
    const float f = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    if (lane < kLanes) {
        const s4_t y = {__builtin_bit_cast(short, (T)(o.x * f)), __builtin_bit_cast(short, (T)(o.y * f)), __builtin_bit_cast(short, (T)(o.z * f)),
                        __builtin_bit_cast(short, (T)(o.w * f))};
        *(s4_t*)((T*)a.out.data + t * a.out.token_stride + h * a.out.head_stride + d) = y;
    }
    if (a.lse && lane == 0)
        a.lse[row] = sum > 0.f || sum != sum ? (m + __builtin_amdgcn_logf(sum) - Half<T>::kLift) * 0.6931471805599453f : -INFINITY;
}

template <typename T, int D, bool FEW>
__global__ __launch_bounds__(256) void attend_join_kernel(AttendArgs a) {
    const int lane = lane_id();
    const int64_t rows = !FEW || a.parts > 0 ? (int64_t)a.step.n_tokens * a.hq : 0, stride = (int64_t)gridDim.x * 4, first = (int64_t)blockIdx.x * 4 + wave_id();
    if (rows <= stride) {
        if (first < rows) join_row<T, D, false>(a, first, 0, lane);
    } else {
        // several rows a wavefront, most of them complete already where there are prompts: asked for 64 at a time
        for (int64_t row0 = first; row0 < rows; row0 += 64 * stride) {
            const int64_t mine = row0 + lane * stride;
            const float m = mine < rows ? a.part_ml[mine * a.parts + a.part_own].x : NAN;
            for (uint64_t left = __ballot(m == m); left; left &= left - 1) join_row<T, D, false>(a, row0 + __builtin_ctzll(left) * stride, 0, lane);
        }
    }
    if (!FEW) return;
    // the sequences of few rows: of their places, those that hold a token
    const int64_t few = (int64_t)a.step.n_seq * a.few_tokens * a.hq;
    for (int64_t at0 = first; at0 < few; at0 += 64 * stride) {
        const int64_t mine = at0 + lane * stride;
        int64_t row = -1;
        if (mine < few) {
            const int64_t place = mine / a.hq;
            const int s = (int)(place / a.few_tokens), i = (int)(place % a.few_tokens), t0 = token_of(a.step, s), n = token_of(a.step, s + 1) - t0;
            if (i < n && n * a.group <= kNarrowRows) row = (int64_t)(t0 + i) * a.hq + mine % a.hq;
        }
        for (uint64_t left = __ballot(row >= 0); left; left &= left - 1) {
            const int l = __builtin_ctzll(left);
            join_row<T, D, true>(a, __shfl(row, l), at0 + l * stride, lane);
        }
    }
}

// How a call is cut into passes.
struct AttendPlan {
    bool shared;                     // the prefix in a pass of its own
    bool narrow, wide;               // kernels that the own (or all) keys need
    bool prefix_narrow;
    bool one_wave;                   // narrow workgroups of one wavefront
    int split_narrow, split_wide, split_prefix;
    int tiles_narrow, tiles_wide, tiles_prefix;      // workgroups along a unit's rows
    int parts, part_own, n_own;      // partial sums of a row, of them the prefix's and its own
    int few_tokens;                  // those of sequences of few rows apart: so many tokens each
};

// One launch for one pass or two: units of the first and of the second.
template <typename T, int D, int NARROW, bool Q8>
static hipError_t launch_passes(AttendArgs a, int64_t units0, int64_t units1, hipStream_t s) {
    using S = Shape<D, NARROW, Q8>;
    const int64_t packed = (int64_t)a.step.n_tokens * a.group / S::kRows + a.step.n_seq;         // at least the sequences' tiles
    auto blocks = [&](int64_t units, const AttendArgs::Pass& p) { return (p.n_tile > 0 ? units * p.n_tile : units ? packed : 0) * p.n_split * a.hkv; };
    const int64_t first = blocks(units0, a.pass[0]), grid = first + blocks(units1, a.pass[1]);
    if (grid > 0x7FFFFFFF) return hipErrorInvalidValue;
    static std::atomic<uint64_t> allowed{0};            // the devices that know of the kernel's LDS
    int device;
    if (hipError_t e = hipGetDevice(&device)) return e;
    if (const uint64_t bit = 1ull << (device & 63); !(allowed.load() & bit)) {
        if (hipError_t e = hipFuncSetAttribute((const void*)attend_kernel<T, D, NARROW, Q8>, hipFuncAttributeMaxDynamicSharedMemorySize, S::kLds)) return e;
        allowed |= bit;
    }
    a.first_blocks = (int)first;
    hipLaunchKernelGGL((attend_kernel<T, D, NARROW, Q8>), dim3((unsigned)grid), dim3(S::kWaves * 64), S::kLds, s, a);
    return hipGetLastError();
}

template <typename T, int D, bool Q8>
static hipError_t launch_attend(AttendArgs a, const AttendPlan& p, hipStream_t s) {
    const int64_t rows = (int64_t)a.step.n_tokens * a.hq, units = a.step.n_seq, groups = p.shared ? a.step.n_groups : 0;
    hipError_t e;
    a.parts = p.parts;
    a.part_own = p.part_own;
    a.few_tokens = p.few_tokens;
    a.few_parts = p.split_narrow;
    const int mode = p.shared ? kOwn : kConcat;
    // the prefix goes first, with those of the other keys' passes that the same kernel makes
    const AttendArgs::Pass prefix = {kPrefix, 0, p.split_prefix, p.split_prefix, p.tiles_prefix, 0, kAllRows};
    const AttendArgs::Pass wide = {mode, p.part_own, p.n_own, p.split_wide, p.tiles_wide, p.narrow ? kNarrowRows : 0, kAllRows};
    const AttendArgs::Pass narrow = {mode, p.part_own, p.n_own, p.split_narrow, p.tiles_narrow, 0, p.wide ? kNarrowRows : kAllRows};
    const int64_t groups_wide = p.prefix_narrow ? 0 : groups, groups_narrow = groups - groups_wide;
    a.pass[0] = prefix;
    if (groups_wide || p.wide) {
        a.pass[1] = wide;
        if ((e = launch_passes<T, D, 0, Q8>(a, groups_wide, p.wide ? units : 0, s))) return e;
    }
    if (groups_narrow || p.narrow) {
        a.pass[1] = narrow;
        const int64_t n = p.narrow ? units : 0;
        if constexpr (D > 64) e = p.one_wave ? launch_passes<T, D, 1, Q8>(a, groups_narrow, n, s) : launch_passes<T, D, 2, Q8>(a, groups_narrow, n, s);
        else e = launch_passes<T, D, 2, Q8>(a, groups_narrow, n, s);
        if (e) return e;
    }
    const int64_t joins = std::max(p.parts > 0 ? rows : 0, units * p.few_tokens * a.hq);
    if (joins > 0) {
        const dim3 grid((unsigned)std::min<int64_t>((joins + 3) / 4, 8192)), block(256);
        if (p.few_tokens > 0) hipLaunchKernelGGL((attend_join_kernel<T, D, true>), grid, block, 0, s, a);
        else hipLaunchKernelGGL((attend_join_kernel<T, D, false>), grid, block, 0, s, a);
        return hipGetLastError();
    }
    return hipSuccess;
}

template <typename T, bool Q8>
static hipError_t launch_attend(const AttendArgs& a, const AttendPlan& p, int d, hipStream_t s) {
    switch (d) {
    case 64: return launch_attend<T, 64, Q8>(a, p, s);
    case 96: return launch_attend<T, 96, Q8>(a, p, s);
    case 128: return launch_attend<T, 128, Q8>(a, p, s);
    default: return launch_attend<T, 256, Q8>(a, p, s);
    }
}

// The same over quantised caches (ivf_attend_quant.hip)
hipError_t launch_attend_quant(const AttendArgs& a, const AttendPlan& p, int row_dtype, int d, hipStream_t s);

}  // namespace ivf
