// Per-problem selection (top-k by score, see topk.hpp) and selection regret.
#include "topk.hpp"

namespace hwsel {
namespace {

// Smaller key = faster runtime.  NaN ranks above +inf, -0 equals +0.
__device__ __forceinline__ uint32_t asc_bits(float t)
{
    if (t != t) return 0xffffffffu;
    uint32_t b = __float_as_uint(t);
    if ((b << 1) == 0u) b = 0u;
    return (b & 0x80000000u) ? ~b : (b | 0x80000000u);
}

// By length: up to 64 rows are one wave's, a row per lane, each key's rank by
// counting the larger ones; up to 1,024 are 256 threads' with four keys each
// (the other waves are gone before the first barrier); longer ones take
// tiles.  Going through a whole tile's keys costs a wave over 1,000
// instructions however few the rows: 100,000 segments of 16 rows, k = 4,
// 800 us so and 96 us by length, 3,000 of 300, k = 5, 28 and 12 us.
// Three waves a SIMD, 155 registers: with the 170 that it would take, two,
// 600 of 8,192, k = 10, took 14.2 us in place of 9.9, 100,000 of 16 132.
constexpr int kShort = 1024, kShortThreads = 256;

template <int NT>
__global__ __launch_bounds__(NT, 3) void k_topk(const float *__restrict__ scores, const int64_t *__restrict__ seg, int32_t k,
                                             int32_t *__restrict__ idx, float *__restrict__ vals)
{
    __shared__ TopkLds<NT> lds;
    const int32_t p = blockIdx.x;
    const int32_t n = (int32_t)seg_len(seg, p);
    const float *s = scores + seg[p];
    idx += (int64_t)p * k;
    if (vals) vals += (int64_t)p * k;
    auto emit = [&](int32_t j, uint64_t key) {
        const int32_t li = key ? (int32_t)(0xffffffffu - (uint32_t)key) : -1;
        idx[j] = li;
        if (vals) vals[j] = li < 0 ? -__builtin_inff() : s[li];
    };
    if (n <= 64) {
        const int32_t lane = threadIdx.x;
        if (lane >= 64) return;
        const float v = lane < n ? s[lane] : 0.0f;
        const uint64_t own = lane < n ? ((uint64_t)desc_bits(v) << 32) | (0xffffffffu - (uint32_t)lane) : 0ull;
        int32_t rank = 0;
        for (int32_t l = 0; l < n; ++l) rank += lane_value(own, l) > own;
        const int32_t j = lane < n ? rank : lane;           // past the rows: no pick
        if (j < k) {
            idx[j] = lane < n ? lane : -1;
            if (vals) vals[j] = lane < n ? v : -__builtin_inff();
        }
    } else if (n <= kShort) {
        if (threadIdx.x >= kShortThreads) return;
        topk_tiles<kShortThreads, kShort>(s, n, k, lds, emit);
    } else {
        topk_tiles<NT, kTile>(s, n, k, lds, emit);
    }
}

// 1 - t_star / t_pick in binary64; equal runtimes (inf included) give 0 and a
// NaN runtime (a kernel that never finishes) gives 1.
__device__ __forceinline__ float regret_value(float t_star, float t_pick)
{
    if (t_pick == t_star) return 0.0f;
    if (t_pick != t_pick) return 1.0f;
    return (float)(1.0 - (double)t_star / (double)t_pick);
}

// The runtime whose asc_bits are b (0 for -0).
__device__ __forceinline__ float asc_value(uint32_t b)
{
    return __uint_as_float((b & 0x80000000u) ? b ^ 0x80000000u : ~b);
}

// The fastest row by a block-wide minimum, all of a step's loads in flight;
// up to 512 rows are the first wave's alone, a load per 64 rows that are there.
// The picks' runtimes are fetched by the first wave's lanes meanwhile.
// Bound by the reads (long segments) and latency: 256 segments of
// 65,536 rows 83 -> 14 us (from 128 loads of one row each, one after another);
// 100,000 of 16 rows 66 us then, 91 with eight loads for every lane, now 52.
template <int NT>
__global__ __launch_bounds__(NT) void k_regret(const float *__restrict__ rt, const int64_t *__restrict__ seg,
                                               const int32_t *__restrict__ idx, int32_t k, float *__restrict__ r1,
                                               float *__restrict__ rk, int32_t *__restrict__ best)
{
    __shared__ uint64_t sh[NT / 64];
    const int32_t p = blockIdx.x;
    const int64_t base = seg[p];
    const int64_t n = seg_len(seg, p);
    const float *t = rt + base;
    const int lane = threadIdx.x;
    // lane j < k of the first wave: pick j
    float t_pick = 0.0f;
    uint64_t pick_key = ~0ull;
    bool counted = false;
    if (lane < k) {
        const int32_t c = idx[(int64_t)p * k + lane];
        counted = c >= 0 && c < n;
        if (counted) {
            t_pick = t[c];
            pick_key = ((uint64_t)asc_bits(t_pick) << 32) | (uint64_t)(uint32_t)c;
        }
    }
    constexpr int kIn = NT >= 512 ? 16 : 8;
    constexpr int kFew = 8;
    uint64_t m = ~0ull;
    const bool few = n <= 64 * kFew;                        // the first wave's alone
    if (few) {
        if (threadIdx.x >= 64) return;
#pragma unroll
        for (int q = 0; q < kFew; ++q) {
            if (64 * q >= n) break;                         // (uniform)
            const uint32_t i = lane + 64 * q < n ? lane + 64 * q : lane < n ? lane : 0;
            const uint64_t key = ((uint64_t)asc_bits(t[i]) << 32) | i;
            m = key < m ? key : m;
        }
        m = ~wave_max_key(~m);
    }
    for (int64_t i0 = threadIdx.x; i0 < n && !few; i0 += kIn * NT) {
        float v[kIn];
#pragma unroll
        for (int q = 0; q < kIn; ++q) v[q] = t[i0 + q * NT < n ? i0 + q * NT : i0];
#pragma unroll
        for (int q = 0; q < kIn; ++q) {
            const int64_t i = i0 + q * NT < n ? i0 + q * NT : i0;
            const uint64_t key = ((uint64_t)asc_bits(v[q]) << 32) | (uint64_t)(uint32_t)i;
            m = key < m ? key : m;
        }
    }
    if (!few) m = ~block_max_key<NT>(~m, sh);               // block minimum of the unique keys
    if (threadIdx.x >= 64) return;
    const uint64_t bk = ~wave_max_key(~pick_key);
    // its runtime as it stands (a key does not tell -0 from +0)
    const float t_k = __shfl(t_pick, __builtin_ctzll(__ballot(pick_key == bk)));
    if (threadIdx.x != 0) return;
    if (n == 0) {
        r1[p] = __builtin_nanf("");
        if (rk) rk[p] = __builtin_nanf("");
        if (best) best[p] = -1;
        return;
    }
    const float t_star = (uint32_t)(m >> 32) == 0xffffffffu ? __builtin_nanf("") : asc_value((uint32_t)(m >> 32));
    r1[p] = counted ? regret_value(t_star, t_pick) : __builtin_nanf("");
    if (rk) rk[p] = bk == ~0ull ? __builtin_nanf("") : regret_value(t_star, t_k);
    if (best) best[p] = (int32_t)(uint32_t)m;
}

}  // namespace

// Segment lengths are not known here.  While every problem has a CU to itself,
// a large workgroup has the most loads in flight; beyond that, small ones
// share the CUs better and waste less on short segments.  Top-16 and regret:
// 256 problems of 65,536 rows 39 us large, 67 small; 300 of 50,000 59 and 61;
// 600 of 25,000 50 and 43.  The regret's large ones have 512 threads of twice
// the loads: as fast on long segments as 1,024, and half the waves to start on
// short ones (60 of 8,192 rows 3.7 us, 4.4 with 1,024).
hipError_t launch_topk(const float *scores, const int64_t *seg, int32_t P, int32_t k, int32_t *idx,
                       float *vals, hipStream_t s)
{
    if (P <= compute_units())
        hipLaunchKernelGGL(k_topk<1024>, dim3(P), dim3(1024), 0, s, scores, seg, k, idx, vals);
    else
        each_span(P, [&](int32_t p0, int32_t n) {
            const int64_t o = (int64_t)p0 * k;
            hipLaunchKernelGGL(k_topk<256>, dim3(n), dim3(256), 0, s, scores, seg + p0, k, idx + o, vals ? vals + o : nullptr);
        });
    return hipGetLastError();
}

hipError_t launch_regret(const float *rt, const int64_t *seg, int32_t P, const int32_t *idx,
                         int32_t k, float *r1, float *rk, int32_t *best, hipStream_t s)
{
    if (P <= compute_units())
        hipLaunchKernelGGL(k_regret<512>, dim3(P), dim3(512), 0, s, rt, seg, idx, k, r1, rk, best);
    else
        each_span(P, [&](int32_t p0, int32_t n) {
            hipLaunchKernelGGL(k_regret<256>, dim3(n), dim3(256), 0, s, rt, seg + p0, idx + (int64_t)p0 * k, k, r1 + p0,
                               rk ? rk + p0 : nullptr, best ? best + p0 : nullptr);
        });
    return hipGetLastError();
}

}  // namespace hwsel
