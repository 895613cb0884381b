// The k best scores of a segment by a workgroup, shared by select.hip and
// logprob.hip.
//
// One workgroup per problem segment.  Scores are mapped to 64-bit keys
// (order-preserving score bits << 32 | inverted local index), which makes
// every key unique: "score descending, index ascending" becomes "key
// descending" and the answer is unique.
//
// A segment is read once, kTile rows at a time, the next tile's scores on their
// way while one is worked on.  Of a tile only the keys above a bound are looked
// at further: the k-th best key so far, or, while fewer than k are kept (or too
// many pass), a bound from the tile itself.  Each wave takes the j-th largest of
// its lanes' maxima; if r waves have j lanes each above a value, r j >= k keys
// are, so the r-th largest of those is at most the k-th best.  About k keys pass;
// they meet the kept ones in LDS and every key finds its rank by counting the
// larger ones.  A tile whose keys still do not fit the list gives its best in k
// rounds of a block-wide maximum.
// Bound by latency for one short segment (a load, four barriers) and by the
// score reads for long ones.  Measured against k rounds over all keys (256
// threads): 256 segments of 65,536 rows, k = 16,
// 172 -> 20 us; one of 8,192 rows, k = 10, 19 -> 6 us.
#pragma once

#include "internal.hpp"

namespace hwsel {

// rows of a tile: 32 keys per thread of a small workgroup, 8 of a large one
constexpr int kTile = 8192;

// Larger key = better score.  NaN ranks lowest, -0 equals +0 (the sum makes it that).
__device__ __forceinline__ uint32_t desc_bits(float s) { return s != s ? 0u : order_key(s + 0.0f); }

// The score that has these bits (a NaN for 0).
__device__ __forceinline__ float desc_value(uint32_t b) { return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b); }

template <int CTRL, int ROW_MASK, bool ZERO_FILL>
__device__ __forceinline__ uint32_t dpp_max_u32(uint32_t v)
{
    const uint32_t w = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, ZERO_FILL);
    return w > v ? w : v;
}

// Maximum over the wave of an unsigned 32-bit value (0 is the identity), in
// every lane: scan within rows, row broadcasts to lane 63, then readlane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v)
{
    v = dpp_max_u32<0x111, 0xf, true>(v);
    v = dpp_max_u32<0x112, 0xf, true>(v);
    v = dpp_max_u32<0x114, 0xf, true>(v);
    v = dpp_max_u32<0x118, 0xf, true>(v);
    v = dpp_max_u32<0x142, 0xa, false>(v);
    v = dpp_max_u32<0x143, 0xc, false>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

// Maximum over the wave of 64-bit keys: the largest high word, then the
// largest low word among the lanes holding it.
__device__ __forceinline__ uint64_t wave_max_key(uint64_t v)
{
    const uint32_t hi = wave_max_u32((uint32_t)(v >> 32));
    const uint32_t lo = wave_max_u32((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return ((uint64_t)hi << 32) | lo;
}

// Block maximum with one barrier: the waves' maxima go to sh (a buffer the
// caller alternates between rounds, so no round overwrites one still read).
template <int NT>
__device__ __forceinline__ uint64_t block_max_key(uint64_t v, uint64_t *sh)
{
    v = wave_max_key(v);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    uint64_t r = sh[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) r = sh[w] > r ? sh[w] : r;
    return r;
}

__device__ __forceinline__ int64_t seg_len(const int64_t *seg, int32_t p)
{
    int64_t n = seg[p + 1] - seg[p];
    n = n < 0 ? 0 : n;
    return n > 0x7fffffff ? 0x7fffffff : n;
}

__device__ __forceinline__ uint64_t lane_value(uint64_t v, int l)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), l);
    return ((uint64_t)hi << 32) | lo;
}

constexpr int kList = 512;            // keys of one tile that are ranked at once

template <int NT>
struct TopkLds {
    uint64_t top[2][64], cand[kList];                       // kept keys, descending; the tile's
    uint64_t per_wave[2][NT / 64];
    // Keys listed of tiles 0, 3, 6, ..., of tiles 1, 4, ... and of tiles 2, 5, ...
    // Every wave has to read the same count of a tile, and nothing but barriers
    // keeps waves together.  Tile i's count is complete at the barrier after
    // its appends and read before the next tile's; the counter of tile i + 2
    // (tile i - 1's) is cleared between the two: its last reads came before
    // the first, and tile i + 2 appends after the second.
    int32_t n_cand[3];
};

// The k best of one segment by NT threads, TILE rows at a time (lds: for at
// least as many threads).  emit(j, key): the j-th best, by one thread (0: there
// is none).
template <int NT, int TILE, class Lds, class Emit>
__device__ __forceinline__ void topk_tiles(const float *__restrict__ s, int32_t n, int32_t k, Lds &lds, Emit &&emit)
{
    constexpr int kWaves = NT / 64, kPer = TILE / NT;       // keys per thread and tile
    auto &top = lds.top;
    auto &cand = lds.cand;
    auto &per_wave = lds.per_wave;
    auto &n_cand = lds.n_cand;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    // r waves with j lanes each: r at most half the waves
    const int32_t j_of = (k + kWaves / 2 - 1) / (kWaves / 2), r_of = (k + j_of - 1) / j_of;

    float next[kPer];
    auto fetch = [&](int32_t t0) {
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
            const uint32_t i = (uint32_t)t0 + threadIdx.x + q * NT;
            next[q] = i < (uint32_t)n ? s[i] : __builtin_nanf("");
        }
    };
    fetch(0);
    if (threadIdx.x < 3) n_cand[threadIdx.x] = 0;           // (the first bound's barrier follows)
    int32_t kept = 0, cur = 0, turn = 0;                    // block-uniform; turn: the tile's counter
    uint64_t floor = 0;                                     // keys at or below it are out (0: none)
    for (uint32_t t0 = 0; t0 < (uint32_t)n; t0 += TILE) {
        uint32_t hi[kPer];                                  // score bits of the thread's keys
        auto key = [&](int q) -> uint64_t {                 // 0: no row (every real key is > 0)
            const uint32_t i = t0 + threadIdx.x + q * NT;
            return i < (uint32_t)n ? ((uint64_t)hi[q] << 32) | (0xffffffffu - i) : 0ull;
        };
#pragma unroll
        for (int q = 0; q < kPer; ++q) hi[q] = desc_bits(next[q]);
        if (t0 + TILE < (uint32_t)n) fetch(t0 + TILE);
        uint32_t most_hi = 0;                               // of the lane's largest key
#pragma unroll
        for (int q = 0; q < kPer; ++q) most_hi = hi[q] > most_hi ? hi[q] : most_hi;

        // A key that is at most the k-th best of the tile and of the kept ones.
        auto bound = [&]() -> uint64_t {
            uint64_t m = 0, v = 0;                          // m: the lane's largest key
#pragma unroll
            for (int q = 0; q < kPer; ++q) m = key(q) > m ? key(q) : m;
            for (int32_t j = 0; j < j_of; ++j) {
                v = wave_max_key(m);
                m = m == v ? 0ull : m;
            }
            if (lane == 0) per_wave[0][wave] = v;
            __syncthreads();
            const uint64_t mine = lane < kWaves ? per_wave[0][lane] : 0ull;
            int32_t above = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const uint64_t o = lane_value(mine, w);
                above += o > mine || (o == mine && w < lane);
            }
            return lane_value(mine, __builtin_ctzll(__ballot(lane < kWaves && above == r_of - 1)));
        };
        auto append = [&](uint64_t limit) {                 // keys above limit to cand; counted beyond its end too
            if (__ballot(most_hi >= (uint32_t)(limit >> 32)) == 0) return;
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                const uint64_t v = key(q);
                const uint64_t take = __ballot(v > limit);
                if (take == 0) continue;
                int32_t at = 0;
                if (lane == 0) at = atomicAdd(&n_cand[turn], __popcll(take));
                at = __builtin_amdgcn_readfirstlane(at) +
                     (int32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(take >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)take, 0u));
                if (v > limit && at < kList) cand[at] = v;
            }
        };
        auto raised = [&](uint64_t b) { return b != 0 && b - 1 > floor ? b - 1 : floor; };
        const bool bounded = kept < k;
        if (bounded) append(raised(bound()));
        else append(floor);
        __syncthreads();
        if (threadIdx.x == 0) n_cand[turn == 0 ? 2 : turn - 1] = 0;
        int32_t m = n_cand[turn];
        if (m > kList && !bounded) {                        // far more than k above the floor: bound them
            __syncthreads();                                // all have read the count
            if (threadIdx.x == 0) n_cand[turn] = 0;
            append(raised(bound()));                        // (the bound's barrier comes before)
            __syncthreads();
            m = n_cand[turn];
        }
        turn = turn == 2 ? 0 : turn + 1;
        if (m > kList) {                                    // the tile's best in rounds
            uint64_t prev = ~0ull;
            __syncthreads();
            for (m = 0; m < k; ++m) {                       // block-uniform trip count
                uint64_t best = 0;
#pragma unroll
                for (int q = 0; q < kPer; ++q) {
                    const uint64_t v = key(q);
                    best = (v < prev && v > floor && v > best) ? v : best;
                }
                best = block_max_key<NT>(best, per_wave[m & 1]);
                if (best == 0) break;
                if (threadIdx.x == 0) cand[m] = best;
                prev = best;
            }
            __syncthreads();
        }
        if (m > 0) {
            // the rank of every kept and every new key among both
            for (int32_t e = threadIdx.x; e < kept + m; e += NT) {
                const uint64_t v = e < kept ? top[cur][e] : cand[e - kept];
                int32_t rank = e < kept ? e : 0;
                if (e >= kept)
                    for (int32_t q = 0; q < kept; ++q) rank += top[cur][q] > v;
                // eight reads in flight (one at a time, 450 keys took 20 us)
#pragma unroll 8
                for (int32_t q = 0; q < m; ++q) rank += cand[q] > v;
                if (rank < k) top[cur ^ 1][rank] = v;
            }
            cur ^= 1;
            kept = kept + m < k ? kept + m : k;
            __syncthreads();
            if (kept == k) floor = top[cur][k - 1];
        }
    }
    for (int32_t j = threadIdx.x; j < k; j += NT) emit(j, j < kept ? top[cur][j] : 0ull);
}

}  // namespace hwsel
