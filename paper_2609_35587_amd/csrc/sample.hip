// Drawing candidates from a problem's scores: softmax at a temperature, limited
// by top-k, top-p and min-p, by given random numbers.
//
// Weights are whole numbers, so sums do not depend on their order and every
// comparison is exact.  The kept set is a prefix of the order (score
// descending, index ascending), found without sorting: a histogram of count
// and mass over the exponents t = (score - best) rate, which fall as scores
// fall, names the bin in which the prefix ends, and the few scores of that bin
// are ranked.  A draw is the first candidate at which the running sum of kept
// weights passes a point: sums of 256 candidates are kept, and the 256 that a
// draw falls into are weighed again.
//
// A workgroup takes a problem (a wave one of up to 1,024 candidates); a wave has
// consecutive candidates of it, 256 a step.  Scores are read once from HBM; as
// many as LDS has room for stay there, first as scores, then as weights, the
// others are read and weighed again.
// (Kept in registers instead, 64 a thread, the unrolled passes were 24,000
// instructions with spills: 121 us for 256 problems of 65,536.)
// Bound by latency: counters show the vector units busy 24 % of the time for 600
// problems of up to 8,192 and 56 % for 256 of 65,536 (92 vector instructions a
// candidate: those past LDS are weighed twice), waves waiting 57 % of theirs.
// The paths for cuts among very many scores are inlined; k_sample<1024> keeps 14
// vector registers in scratch for them, k_sample<512> of six waves 18 and
// k_sample_waves 24.
#include "internal.hpp"

namespace hwsel {
namespace {

struct Settings {
    hwsel_sampling_t how;
    int32_t n_draws;
};

typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));   // four scores from any segment's start

// What is known of a problem once its scores have been read.
struct Problem {
    const float *s;
    int32_t n;
    float best, rate;
};

// t = (s - best) * rate of a score, by stated steps (compiled without
// multiply-add contraction: every product and sum rounds).  NaN, as of a NaN
// score, and -inf end at -60, where weights are 0; the best score is at 0 also
// where it or the rate is infinite.
__device__ __forceinline__ float exponent_of(const Problem &q, float s)
{
    const float t = fmaxf((s - q.best) * q.rate, -60.0f);
    return s == q.best ? 0.0f : t;
}

// floor(2^32 2^t) for t in [-60, 0], 2^32 itself as 2^32 - 1 (no other weight
// is: above 2^31 they are multiples of 2^8).
__device__ __forceinline__ uint32_t weight32(float t)
{
    // 1.5 2^23 + 32: the sum is rounded to a whole number, n + 32 in its low bits
    const float shifted = t + 12582944.0f, f = t - (shifted - 12582944.0f);
    float p = 1.5403530e-04f;                               // ln(2)^i / i!, i = 6 .. 0
    p = p * f + 1.3333558e-03f;
    p = p * f + 9.6181291e-03f;
    p = p * f + 5.5504109e-02f;
    p = p * f + 2.4022651e-01f;
    p = p * f + 6.9314718e-01f;
    p = p * f + 1.0f;
    const float v = __uint_as_float((__float_as_uint(shifted) << 23) + __float_as_uint(p));  // p 2^(n + 32)
    uint32_t w;
    asm("v_cvt_u32_f32 %0, %1" : "=v"(w) : "v"(v));         // (saturates; in C++ 2^32 would be undefined)
    return w;
}

__device__ __forceinline__ uint64_t whole(uint32_t w) { return (uint64_t)w + (w == 0xffffffffu); }

// Neither NaN nor -inf.  (Not s > -inf: of a ballot over that the compiler makes
// "not equal to -inf", which a NaN passes.)
__device__ __forceinline__ bool takes_part(float s) { return s >= -3.402823466e+38f; }

// Key of a score that takes part (larger is better), 0 for NaN and -inf.
__device__ __forceinline__ uint32_t key_of(float s) { return takes_part(s) ? order_key(s + 0.0f) : 0u; }

__device__ __forceinline__ float score_of(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

// Sums and maxima over a wave by lane moves: scans within rows of 16, then row
// broadcasts (through LDS, as shuffles go, each of their six steps waits for a
// round trip).
template <int CTRL, int ROW_MASK, bool ZERO_FILL>
__device__ __forceinline__ uint32_t dpp_plus(uint32_t v)
{
    return v + (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, ZERO_FILL);
}

__device__ __forceinline__ uint32_t wave_scan(uint32_t v)  // inclusive
{
    v = dpp_plus<0x111, 0xf, true>(v);
    v = dpp_plus<0x112, 0xf, true>(v);
    v = dpp_plus<0x114, 0xf, true>(v);
    v = dpp_plus<0x118, 0xf, true>(v);
    v = dpp_plus<0x142, 0xa, false>(v);
    return dpp_plus<0x143, 0xc, false>(v);
}

__device__ __forceinline__ uint32_t wave_sum(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_scan(v), 63); }

// Of values below 2^58, as numbers of 26 bits.
__device__ __forceinline__ uint64_t wave_scan(uint64_t v)
{
    const uint32_t a = wave_scan((uint32_t)v & 0x3ffffffu), b = wave_scan((uint32_t)(v >> 26) & 0x3ffffffu),
                   c = wave_scan((uint32_t)(v >> 52));
    return ((uint64_t)c << 52) + ((uint64_t)b << 26) + a;
}

// Of values below 2^52.
__device__ __forceinline__ uint64_t wave_scan52(uint64_t v)
{
    const uint32_t a = wave_scan((uint32_t)v & 0x3ffffffu), b = wave_scan((uint32_t)(v >> 26));
    return ((uint64_t)b << 26) + a;
}

__device__ __forceinline__ uint64_t lane_u64(uint64_t v, int l)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, l);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), l);
    return ((uint64_t)hi << 32) | lo;
}

__device__ __forceinline__ uint64_t wave_sum(uint64_t v) { return lane_u64(wave_scan(v), 63); }

template <int CTRL, int ROW_MASK, bool ZERO_FILL>
__device__ __forceinline__ uint32_t dpp_most(uint32_t v)
{
    const uint32_t w = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROW_MASK, 0xf, ZERO_FILL);
    return w > v ? w : v;
}

__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = dpp_most<0x111, 0xf, true>(v);
    v = dpp_most<0x112, 0xf, true>(v);
    v = dpp_most<0x114, 0xf, true>(v);
    v = dpp_most<0x118, 0xf, true>(v);
    v = dpp_most<0x142, 0xa, false>(v);
    v = dpp_most<0x143, 0xc, false>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}

constexpr int kParts = 256;                                 // sums of consecutive candidates, at most

template <int NT, int BINS, int CACHED>
struct Lds {
    static constexpr int kList = BINS * 3 / 8;              // scores around a bin that are ranked at once
    // Running sums after each lane's four candidates of a step, once the bins are done with.
    static constexpr int kFine = (BINS * 12 + kList * 16) / 8 / 64 * 64;
    uint32_t cache[CACHED];
    union {
        struct {
            uint64_t mass[BINS + 1], list[kList], sorted[kList];
            uint32_t count[BINS + 1];
        };
        uint64_t fine[kFine];
    };
    union {                                                 // (the cut is found before parts are summed)
        uint64_t part[kParts + 1];
        uint32_t near[kList];
    };
    uint64_t wave_mass[NT / 64], cut, found_mass;
    uint32_t wave_count[NT / 64], found_count, found_bin, n_near;
    float wave_best[NT / 64], wave_least[NT / 64];
};

// The end of the kept prefix: a candidate is in it if its score's key is
// greater, or equal and its index is at most `last`.
struct Cut {
    uint32_t key;
    int32_t last;
};

__device__ __forceinline__ bool within(const Cut &c, uint32_t key, int32_t i)
{
    return key > c.key || (key == c.key && key != 0 && i <= c.last);
}

struct Limits {
    uint32_t k;
    float top_p;
    uint64_t least;
};

// A problem's settings, as the header defines their odd values.
__device__ __forceinline__ void read_settings(const Settings &set, int32_t p, float best, Problem &q, Limits &lim)
{
    const float T = set.how.temperature_of ? set.how.temperature_of[p] : set.how.temperature;
    const int32_t k = set.how.top_k_of ? set.how.top_k_of[p] : set.how.top_k;
    const float min_p = set.how.min_p_of ? set.how.min_p_of[p] : set.how.min_p;
    const bool cold = !(T > 0.0f);
    lim.k = cold ? 1u : k > 0 ? (uint32_t)k : 0xffffffffu;
    lim.top_p = set.how.top_p_of ? set.how.top_p_of[p] : set.how.top_p;
    lim.least = (uint64_t)ceil(min_p > 0.0f ? (min_p < 1.0f ? (double)min_p : 1.0) * 4294967296.0 : 0.0);
    lim.least = lim.least < 1 ? 1 : lim.least;
    q.best = best + 0.0f;
    q.rate = cold ? 1.0f : (float)(1.4426950408889634 / (double)T);
}

// The mass before which top_p keeps.
__device__ __forceinline__ uint64_t share_of(const Limits &lim, uint64_t mass)
{
    const uint64_t need = (uint64_t)ceil((double)mass * (double)(lim.top_p > 0.0f ? lim.top_p : 0.0f));
    return need < 1 ? 1 : need;
}

// Problem p's candidates, its best score not known yet.
__device__ __forceinline__ Problem problem_of(const float *scores, int64_t R, const int64_t *seg, int32_t p)
{
    int64_t lo = seg[p], hi = seg[p + 1];
    lo = lo < 0 ? 0 : lo > R ? R : lo;
    hi = hi < lo ? lo : hi > R ? R : hi;
    return {scores + lo, (int32_t)(hi - lo), 0.0f, 1.0f};
}

// The lowest index of the best score among four from index i on, or the one known.
__device__ __forceinline__ uint32_t first_best(const Problem &q, const f32x4u_t &t, int32_t i, uint32_t known)
{
#pragma unroll
    for (int c = 3; c >= 0; --c) known = t[c] == q.best && (uint32_t)(i + c) < known ? (uint32_t)(i + c) : known;
    return known;
}

// The draws of a problem with one candidate left, by N threads.  (Loops over draws
// count without a sign, here and below: up to 2^31 - 1 draws and a step more.)
template <int N>
__device__ __forceinline__ void write_one(int32_t at, int thread, int32_t n_draws, int32_t *idx, float *prob)
{
    for (uint32_t j = thread; j < (uint32_t)n_draws; j += N) {
        idx[j] = at;
        if (prob) prob[j] = 1.0f;
    }
}

// How a workgroup of NT threads goes through n candidates: a wave has `steps`
// steps of 256, from `base` on; `each` steps are one part.
struct Walk {
    int32_t n, steps, base, each, per_wave;                 // per_wave: parts of a wave
};

template <int NT>
__device__ __forceinline__ Walk walk_of(int32_t n, int wave)
{
    constexpr int kWaves = NT / 64, kMost = kParts / kWaves;
    Walk w;
    w.n = n;
    w.steps = (int32_t)(((int64_t)n + 256 * kWaves - 1) / (256 * kWaves));
    w.base = (int32_t)((int64_t)wave * w.steps * 256 < n ? wave * w.steps * 256 : n);
    w.each = (w.steps + kMost - 1) / kMost;
    w.per_wave = w.each > 0 ? (w.steps + w.each - 1) / w.each : 0;
    return w;
}

// body(step, the lane's four scores, -inf past the end): AHEAD steps' loads at a
// time while they are whole.
template <int AHEAD = 4, class F>
__device__ __forceinline__ void each_step(const float *__restrict__ s, const Walk &w, int32_t first, int32_t last, F &&body)
{
    const int lane = threadIdx.x & 63;
    int32_t i = first;
    if constexpr (AHEAD > 1)
        for (; i + AHEAD <= last && (int64_t)w.base + (i + AHEAD) * 256 <= w.n; i += AHEAD) {
            f32x4u_t t[AHEAD];
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) t[j] = *reinterpret_cast<const f32x4u_t *>(s + w.base + (i + j) * 256 + lane * 4);
#pragma unroll
            for (int j = 0; j < AHEAD; ++j) body(i + j, t[j]);
        }
#pragma unroll 1
    for (; i < last; ++i) {
        const int64_t at = (int64_t)w.base + i * 256 + lane * 4;
        f32x4u_t t;
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = at + c < w.n ? s[at + c] : -__builtin_inff();
        body(i, t);
    }
}

// Sums to sums before: part[e] becomes the sum of part[0 .. e), part[n] the whole.
__device__ __forceinline__ void sums_before(uint64_t *part, int n)
{
    if (threadIdx.x < 64) {
        uint64_t run = 0;
        for (int e0 = 0; e0 < n; e0 += 64) {
            const int e = e0 + (int)threadIdx.x;
            const uint64_t v = e < n ? part[e] : 0, scan = wave_scan(v);
            if (e < n) part[e] = run + scan - v;
            run += lane_u64(scan, 63);
        }
        if (threadIdx.x == 0) part[n] = run;
    }
}

// Which bin, from the best one down, takes the running count (by_mass: mass)
// to `want`; count and mass of the bins before it.
template <int NT, int BINS, class L>
__device__ __forceinline__ void find_bin(L &lds, bool by_mass, uint64_t want, uint32_t &bin, uint32_t &before_count,
                                         uint64_t &before_mass)
{
    constexpr int kEach = BINS / NT;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint64_t m[kEach], m_sum = 0;
    uint32_t c[kEach], c_sum = 0;
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        m[j] = lds.mass[threadIdx.x * kEach + j];
        c[j] = lds.count[threadIdx.x * kEach + j];
        m_sum += m[j];
        c_sum += c[j];
    }
    const uint64_t m_scan = wave_scan(m_sum);
    const uint32_t c_scan = wave_scan(c_sum);
    if (lane == 63) {
        lds.wave_mass[wave] = m_scan;
        lds.wave_count[wave] = c_scan;
    }
    __syncthreads();
    uint64_t m_at = m_scan - m_sum;
    uint32_t c_at = c_scan - c_sum;
    for (int w = 0; w < wave; ++w) {
        m_at += lds.wave_mass[w];
        c_at += lds.wave_count[w];
    }
#pragma unroll
    for (int j = 0; j < kEach; ++j) {
        const uint64_t at = by_mass ? m_at : (uint64_t)c_at, with = at + (by_mass ? m[j] : (uint64_t)c[j]);
        if (at < want && with >= want) {
            lds.found_bin = threadIdx.x * kEach + j;
            lds.found_mass = m_at;
            lds.found_count = c_at;
        }
        m_at += m[j];
        c_at += c[j];
    }
    __syncthreads();
    bin = lds.found_bin;
    before_mass = lds.found_mass;
    before_count = lds.found_count;
    __syncthreads();
}

// A key that many of a bin's candidates share (a model of few leaves gives many
// equal scores): they are counted instead of listed.  0: none.
struct Tied {
    uint32_t key, count;
};

// The key that most lanes hold (0: a lane without one).
__device__ __forceinline__ uint32_t commonest(uint32_t key)
{
    uint32_t same = 0;
#pragma unroll 8
    for (int l = 0; l < 64; ++l) same += key != 0 && key == (uint32_t)__builtin_amdgcn_readlane((int)key, l);
    const uint32_t most = wave_max((same << 6) | (threadIdx.x & 63));
    return (uint32_t)__builtin_amdgcn_readlane((int)key, (int)(most & 63));
}

// The index of the left-th candidate with this key in a wave's steps (it is there).
template <int AHEAD>
__device__ __forceinline__ int32_t tied_at(const Problem &q, const Walk &walk, int32_t first, int32_t last, uint32_t key, uint32_t left)
{
    int32_t at = 0;
    bool found = false;
    each_step<AHEAD>(q.s, walk, first, last, [&](int32_t i, const f32x4u_t &t) {
        uint32_t tied = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) tied += key_of(t[c]) == key;
        const uint32_t scan = wave_scan(tied), here = (uint32_t)__builtin_amdgcn_readlane((int)scan, 63);
        if (found) return;
        if (left > here) {
            left -= here;
            return;
        }
        found = true;
        const int lane = __builtin_ctzll(__ballot(scan >= left));
        uint32_t run = scan - tied;
        int c_at = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            run += key_of(t[c]) == key;
            c_at += run < left;
        }
        at = walk.base + i * 256 + lane * 4 + __builtin_amdgcn_readlane(c_at, lane);
    });
    return at;
}

// The cut by digits, where a bin holds too many to rank: the largest key K at
// which the count (by_mass: mass) of scores with keys >= K reaches `want`, by 11
// or 10 bits at a time over all scores, then the last of those tied with it
// that is needed; the mass up to there.
template <int NT, int BINS, class L>
__device__ __forceinline__ Cut cut_by_digits(const Problem &q, const Walk &walk, bool by_mass, uint64_t want, uint64_t &mass,
                                             L &lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    uint32_t prefix = 0, above_count = 0;
    uint64_t above_mass = 0;
    constexpr int kBits = BINS == 4096 ? 12 : BINS == 2048 ? 11 : 10;
#pragma unroll 1
    for (int left = 32; left > 0;) {
        const int bits = left < kBits ? left : kBits, shift = left - bits;
        for (int b = threadIdx.x; b < BINS; b += NT) {
            lds.mass[b] = 0;
            lds.count[b] = 0;
        }
        __syncthreads();
        each_step<1>(q.s, walk, 0, walk.steps, [&](int32_t, const f32x4u_t &t) {
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                const float v = c == 0 ? t[0] : c == 1 ? t[1] : c == 2 ? t[2] : t[3];
                const uint32_t key = key_of(v);
                const bool in = key != 0 && (left == 32 || key >> left == prefix);
                const uint64_t lanes = __ballot(in);
                if (lanes == 0) continue;
                const uint32_t bin = (1u << bits) - 1 - ((key >> shift) & ((1u << bits) - 1));     // best first
                const uint64_t w = whole(weight32(exponent_of(q, v)));
                // one add for the lanes that agree with the first (equal scores)
                const int first = __builtin_ctzll(lanes);
                const bool same = in && key == (uint32_t)__builtin_amdgcn_readlane((int)key, first);
                const uint64_t agree = __ballot(same);
                if (same && lane == first) {
                    atomicAdd(&lds.count[bin], (uint32_t)__popcll(agree));
                    atomicAdd((unsigned long long *)&lds.mass[bin], (unsigned long long)(w * __popcll(agree)));
                } else if (in && !same) {
                    atomicAdd(&lds.count[bin], 1u);
                    atomicAdd((unsigned long long *)&lds.mass[bin], (unsigned long long)w);
                }
            }
        });
        __syncthreads();
        uint32_t bin, c;
        uint64_t m;
        find_bin<NT, BINS>(lds, by_mass, want - (by_mass ? above_mass : (uint64_t)above_count), bin, c, m);
        above_count += c;
        above_mass += m;
        prefix = (prefix << bits) | ((1u << bits) - 1 - bin);
        left = shift;
    }
    const uint64_t w = whole(weight32(exponent_of(q, score_of(prefix))));
    const uint64_t ties = by_mass ? (want - above_mass + w - 1) / w : want - above_count;
    mass = above_mass + ties * w;
    // index of the ties-th candidate with this key: its part, then its place there
    const int n_parts = NT / 64 * walk.per_wave;
#pragma unroll 1
    for (int e = 0; e < walk.per_wave; ++e) {
        const int32_t b = e * walk.each, end = b + walk.each < walk.steps ? b + walk.each : walk.steps;
        uint32_t n = 0;
        each_step<1>(q.s, walk, b, end, [&](int32_t, const f32x4u_t &t) {
#pragma unroll
            for (int c = 0; c < 4; ++c) n += key_of(t[c]) == prefix;
        });
        n = wave_sum(n);
        if (lane == 0) lds.part[wave * walk.per_wave + e] = n;
    }
    __syncthreads();
    sums_before(lds.part, n_parts);
    __syncthreads();
#pragma unroll 1
    for (int e = 0; e < walk.per_wave; ++e) {
        const int part = wave * walk.per_wave + e;
        if (!(lds.part[part] < ties && lds.part[part + 1] >= ties)) continue;
        const int32_t b = e * walk.each, end = b + walk.each < walk.steps ? b + walk.each : walk.steps;
        const int32_t at = tied_at<1>(q, walk, b, end, prefix, (uint32_t)(ties - lds.part[part]));
        if (lane == 0) lds.found_bin = (uint32_t)at;
    }
    __syncthreads();
    const int32_t last = (int32_t)lds.found_bin;
    __syncthreads();
    return {prefix, last};
}

// Weights of scores around one whose weight is w: a smaller score never weighs
// more by over 2^-23 of it.
__device__ __forceinline__ void near_weights(uint32_t w, uint32_t &lo, uint32_t &hi)
{
    const uint32_t slack = (w >> 19) + 1;
    lo = w > slack ? w - slack : 1u;
    hi = w < 0xffffffffu - slack ? w + slack : 0xffffffffu;
}

// A candidate as it is ranked: the larger, the better.
__device__ __forceinline__ uint64_t rank_of(float s, uint32_t i) { return ((uint64_t)key_of(s) << 32) | (0xffffffffu - i); }

// The m candidates of lds.near to lds.list, 0 for those that are not of the bin,
// and how many of each wave's are.
template <int NT, class L>
__device__ __forceinline__ void list_bin(const Problem &q, float bin_scale, uint32_t bin, uint32_t m, L &lds)
{
    uint32_t in_bin = 0;
    for (uint32_t e = threadIdx.x; e < m; e += NT) {
        const uint32_t i = lds.near[e];
        const float v = q.s[i];
        const bool in = (uint32_t)(-exponent_of(q, v) * bin_scale) == bin;
        lds.list[e] = in ? rank_of(v, i) : 0;
        in_bin += in;
    }
    in_bin = wave_sum(in_bin);
    if ((threadIdx.x & 63) == 0) lds.wave_count[threadIdx.x >> 6] = in_bin;
}

// The cut among the m candidates of lds.list and the tied ones: they are ranked.
// The count (by_mass: mass) before the bin is given.  If the cut is among the
// tied ones its index is left open: ties says the how-manieth of them it is (else 0).
template <int NT, class L>
__device__ __forceinline__ Cut rank_bin(const Problem &q, uint32_t m, const Tied &tied, bool by_mass,
                                        uint32_t before_count, uint64_t before_mass, uint64_t want, uint64_t &mass, uint32_t &ties,
                                        L &lds)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    if (tied.key != 0) {                                    // one entry for all of them
        if (threadIdx.x == 0) lds.list[m] = (uint64_t)tied.key << 32;
        ++m;
    }
    __syncthreads();
    uint32_t in_bin = tied.key != 0;
#pragma unroll
    for (int o = 0; o < NT / 64; ++o) in_bin += lds.wave_count[o];
    for (uint32_t e = threadIdx.x; e < m; e += NT) {
        const uint64_t v = lds.list[e];
        uint32_t rank = 0;
#pragma unroll 8
        for (uint32_t o = 0; o < m; ++o) rank += lds.list[o] > v;
        if (v != 0) lds.sorted[rank] = v;
    }
    __syncthreads();
    uint64_t run = before_mass;
    uint32_t run_count = before_count;
    for (uint32_t e0 = 0; e0 < in_bin; e0 += NT) {          // (block-uniform)
        const uint32_t e = e0 + threadIdx.x;
        const uint64_t v = e < in_bin ? lds.sorted[e] : 0;
        const uint32_t key = (uint32_t)(v >> 32), n = e >= in_bin ? 0 : key == tied.key ? tied.count : 1;
        const uint64_t each = e < in_bin ? whole(weight32(exponent_of(q, score_of(key)))) : 0, w = each * n;
        const uint64_t scan = wave_scan(w);
        const uint32_t scan_n = wave_scan(n);
        if (lane == 63) {
            lds.wave_mass[wave] = scan;
            lds.wave_count[wave] = scan_n;
        }
        __syncthreads();
        uint64_t upto = run + scan;
        uint32_t upto_n = run_count + scan_n;
        for (int o = 0; o < NT / 64; ++o) {
            if (o < wave) {
                upto += lds.wave_mass[o];
                upto_n += lds.wave_count[o];
            }
            run += lds.wave_mass[o];
            run_count += lds.wave_count[o];
        }
        if (e < in_bin && (by_mass ? upto - w < want && upto >= want : upto_n - n < want && upto_n >= want)) {
            uint32_t of = 0;
            if (key == tied.key) {
                of = (uint32_t)(by_mass ? (want - (upto - w) + each - 1) / each : want - (upto_n - n));
                upto -= (n - of) * each;
            }
            lds.cut = v;
            lds.found_mass = upto;
            lds.found_count = of;
        }
        __syncthreads();
    }
    const uint64_t cut = lds.cut;
    mass = lds.found_mass;
    ties = lds.found_count;
    __syncthreads();
    return {(uint32_t)(cut >> 32), (int32_t)(0xffffffffu - (uint32_t)cut)};
}

// A draw's point in the running sum.
__device__ __forceinline__ uint64_t point_of(float u, uint64_t total)
{
    const float v = floorf(u * 16777216.0f);
    const uint32_t u24 = v > 0.0f ? (v < 16777215.0f ? (uint32_t)v : 16777215u) : 0u;
    return (total >> 24) * u24 + (((total & 0xffffffull) * u24) >> 24);
}

// Kept weights of four consecutive candidates from i on.
__device__ __forceinline__ void kept_weights(const Problem &q, const Cut &cut, uint64_t least, const f32x4u_t &t, int32_t i,
                                             uint64_t (&w)[4])
{
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        const uint64_t v = within(cut, key_of(t[c]), i + c) ? whole(weight32(exponent_of(q, t[c]))) : 0;
        w[c] = v >= least ? v : 0;
    }
}

// Draw j in the part of steps [first, last) of a walk, r into its running sum.
__device__ __forceinline__ void draw_in(const Problem &q, const Cut &cut, uint64_t least, const Walk &walk, int32_t first,
                                        int32_t last, uint64_t r, uint64_t total, int32_t *idx, float *prob)
{
    const int lane = threadIdx.x & 63;
    for (int32_t i = first; i < last; ++i) {
        const int64_t at = (int64_t)walk.base + i * 256 + lane * 4;
        f32x4u_t t;
#pragma unroll
        for (int c = 0; c < 4; ++c) t[c] = at + c < walk.n ? q.s[at + c] : -__builtin_inff();
        uint64_t w[4];
        kept_weights(q, cut, least, t, (int32_t)at, w);
        const uint64_t sum = w[0] + w[1] + w[2] + w[3], scan = wave_scan52(sum), over = __ballot(scan > r);
        if (over) {
            if (lane == __builtin_ctzll(over)) {
                uint64_t run = scan - sum;
                int c = 0;
                while (c < 3 && run + w[c] <= r) run += w[c++];
                *idx = (int32_t)at + c;
                if (prob) *prob = (float)((double)w[c] / (double)total);
            }
            return;
        }
        r -= lane_u64(scan, 63);
    }
}

// A workgroup's work on problem p.
template <int NT, int BINS, int CACHED>
__device__ __forceinline__ void sample_problem(Lds<NT, BINS, CACHED> &lds, int32_t p, const float *__restrict__ scores, int64_t R,
                                               const int64_t *__restrict__ seg, const Settings &set,
                                               const float *__restrict__ u, int32_t *__restrict__ idx,
                                               float *__restrict__ prob, int32_t *__restrict__ kept_out)
{
    constexpr int kWaves = NT / 64;
    constexpr uint32_t kList = Lds<NT, BINS, CACHED>::kList;
    const int32_t lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Problem q = problem_of(scores, R, seg, p);
    u += (int64_t)p * set.n_draws;
    idx += (int64_t)p * set.n_draws;
    if (prob) prob += (int64_t)p * set.n_draws;
    const Walk walk = walk_of<NT>(q.n, wave);
    const int32_t cached = walk.steps < CACHED / (NT * 4) ? walk.steps : CACHED / (NT * 4);    // steps in LDS
    auto slot = [&](int32_t i) { return reinterpret_cast<u32x4_t *>(lds.cache + (i * NT + (int)threadIdx.x) * 4); };

    // the best score, the least that takes part, and how many do
    for (int b = threadIdx.x; b < BINS; b += NT) {
        lds.mass[b] = 0;
        lds.count[b] = 0;
    }
    if (threadIdx.x == 0) lds.n_near = 0;
    float most = -__builtin_inff(), least_score = __builtin_inff();
    uint32_t alive = 0;
    each_step(q.s, walk, 0, walk.steps, [&](int32_t i, const f32x4u_t &t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool in = takes_part(t[c]);
            alive += in;
            most = fmaxf(most, t[c]);
            least_score = fminf(least_score, in ? t[c] : __builtin_inff());
        }
        if (i < cached) *slot(i) = __builtin_bit_cast(u32x4_t, t);
    });
    most = score_of(wave_max(order_key(most + 0.0f)));
    least_score = -score_of(wave_max(order_key(0.0f - least_score)));
    alive = wave_sum(alive);
    if (lane == 0) {
        lds.wave_best[wave] = most;
        lds.wave_least[wave] = least_score;
        lds.wave_count[wave] = alive;
    }
    __syncthreads();
    alive = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        most = fmaxf(most, lds.wave_best[w]);
        least_score = fminf(least_score, lds.wave_least[w]);
        alive += lds.wave_count[w];
    }
    __syncthreads();
    if (alive == 0) {
        for (uint32_t j = threadIdx.x; j < (uint32_t)set.n_draws; j += NT) {
            idx[j] = -1;
            if (prob) prob[j] = 0.0f;
        }
        if (threadIdx.x == 0 && kept_out) kept_out[p] = 0;
        return;
    }
    Limits lim;
    read_settings(set, p, most, q, lim);
    // every draw is the best one, and its index is all there is to find: 600 problems of 8,192 with 64 draws 5.4 us (27)
    if (lim.k == 1) {
        uint32_t first = 0xffffffffu;
        for (int32_t i = 0; i < cached; ++i) first = first_best(q, __builtin_bit_cast(f32x4u_t, *slot(i)), walk.base + i * 256 + lane * 4, first);
        each_step(q.s, walk, cached, walk.steps, [&](int32_t i, const f32x4u_t &t) { first = first_best(q, t, walk.base + i * 256 + lane * 4, first); });
        first = ~wave_max(~first);
        if (lane == 0) lds.wave_count[wave] = first;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWaves; ++w) first = lds.wave_count[w] < first ? lds.wave_count[w] : first;
        write_one<NT>((int32_t)first, threadIdx.x, set.n_draws, idx, prob);
        if (threadIdx.x == 0 && kept_out) kept_out[p] = 1;
        return;
    }

    // weights, and count and mass of each bin if a prefix is wanted
    const bool by_count = lim.k < alive, by_mass = lim.top_p < 1.0f;
    const float t_least = -exponent_of(q, least_score), span = t_least < 34.0f ? t_least : 34.0f;
    const float bin_scale = span > 0.0f ? fminf((float)(BINS - 1) / span, 1e30f) : 1.0f;
    Cut cut{0, 0x7fffffff};
    if (by_count || by_mass) {
        auto weigh = [&](const f32x4u_t &t) -> u32x4_t {
            u32x4_t w;
            uint32_t bin[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const float e = exponent_of(q, t[c]);
                w[c] = weight32(e);
                bin[c] = w[c] != 0 ? (uint32_t)(-e * bin_scale) : BINS;   // (a place for those of no bin)
            }
            if (by_mass) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (w[c] != 0) atomicAdd((unsigned long long *)&lds.mass[bin[c]], (unsigned long long)whole(w[c]));
            }
            if (by_count) {
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (w[c] != 0) atomicAdd(&lds.count[bin[c]], 1u);
            }
            return w;
        };
        for (int32_t i = 0; i < cached; ++i) *slot(i) = weigh(__builtin_bit_cast(f32x4u_t, *slot(i)));
        each_step(q.s, walk, cached, walk.steps, [&](int32_t, const f32x4u_t &t) { weigh(t); });
        __syncthreads();
        // (scores that weigh nothing are in no bin: there may be fewer in the bins than k)
        uint64_t mass = 0, upto;
        uint32_t in_bins = 0;
        for (int b = threadIdx.x; b < BINS; b += NT) {
            in_bins += lds.count[b];
            mass += lds.mass[b];
        }
        in_bins = wave_sum(in_bins);
        mass = wave_sum(mass);
        if (lane == 0) {
            lds.wave_count[wave] = in_bins;
            lds.wave_mass[wave] = mass;
        }
        __syncthreads();
        in_bins = 0;
        mass = 0;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
            in_bins += lds.wave_count[w];
            mass += lds.wave_mass[w];
        }
        __syncthreads();
        bool bins_left = true;
        // first the k best, then the share of their mass
#pragma unroll 1
        for (int turn = by_count && lim.k < in_bins ? 0 : 1; turn < (by_mass ? 2 : 1); ++turn) {
            const uint64_t want = turn ? share_of(lim, mass) : lim.k;
            uint32_t bin, c, m = kList + 1, tied_here = 0, tied_before = 0;      // of this wave, of the waves before it
            uint64_t before;
            Tied tied{0, 0};
            if (bins_left) {
                find_bin<NT, BINS>(lds, turn, want, bin, c, before);
                // the candidates whose weights lie around the bin's, with room for the rounding of either side
                const float top = exp2f(-(float)bin / bin_scale + 32.0f) * (1.0f + 4e-6f) + 1.0f,
                            low = exp2f(-(float)(bin + 1) / bin_scale + 32.0f) * (1.0f - 4e-6f) - 1.0f;
                const uint32_t w_hi = top < 4294967040.0f ? (uint32_t)top : 0xffffffffu,
                               w_lo = low > 1.0f ? (uint32_t)low : 1u;
                auto list = [&](int32_t i) {
                    const uint32_t at = atomicAdd(&lds.n_near, 1u);
                    if (at < kList) lds.near[at] = (uint32_t)i;
                };
                auto in_bin = [&](float v) { return takes_part(v) && (uint32_t)(-exponent_of(q, v) * bin_scale) == bin; };
                for (int32_t i = 0; i < cached; ++i) {
                    const u32x4_t w = *slot(i);
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (w[e] >= w_lo && w[e] <= w_hi) list(walk.base + i * 256 + lane * 4 + e);
                }
                each_step(q.s, walk, cached, walk.steps, [&](int32_t i, const f32x4u_t &t) {
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (in_bin(t[e])) list(walk.base + i * 256 + lane * 4 + e);
                });
                __syncthreads();
                m = lds.n_near;
                if (m > kList) {                            // again without those of the commonest score
                    tied.key = commonest(key_of(q.s[lds.near[lane * (kList / 64)]]));
                    __syncthreads();
                    if (threadIdx.x == 0) lds.n_near = 0;
                    __syncthreads();
                    auto sort_out = [&](int32_t i, float v) {
                        if (!in_bin(v)) return;
                        if (key_of(v) == tied.key) ++tied_here;
                        else list(i);
                    };
                    for (int32_t i = 0; i < cached; ++i) {
                        const u32x4_t w = *slot(i);
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int32_t at = walk.base + i * 256 + lane * 4 + e;
                            if (w[e] >= w_lo && w[e] <= w_hi) sort_out(at, q.s[at]);
                        }
                    }
                    each_step(q.s, walk, cached, walk.steps, [&](int32_t i, const f32x4u_t &t) {
#pragma unroll
                        for (int e = 0; e < 4; ++e) sort_out(walk.base + i * 256 + lane * 4 + e, t[e]);
                    });
                    tied_here = wave_sum(tied_here);
                    if (lane == 0) lds.wave_count[wave] = tied_here;
                    __syncthreads();
                    m = lds.n_near;
                    for (int w = 0; w < kWaves; ++w) {
                        tied.count += lds.wave_count[w];
                        tied_before += w < wave ? lds.wave_count[w] : 0;
                    }
                    if (tied.count == 0) tied.key = 0;      // (of a weight near the bin's, but outside it)
                }
                __syncthreads();
                if (threadIdx.x == 0) lds.n_near = 0;
            }
            if (m + (tied.key != 0) <= kList) {
                uint32_t ties;
                list_bin<NT>(q, bin_scale, bin, m, lds);
                cut = rank_bin<NT>(q, m, tied, turn, c, before, want, upto, ties, lds);
                if (ties != 0) {
                    if (ties > tied_before && ties <= tied_before + tied_here) {
                        const int32_t at = tied_at<4>(q, walk, 0, walk.steps, cut.key, ties - tied_before);
                        if (lane == 0) lds.found_bin = (uint32_t)at;
                    }
                    __syncthreads();
                    cut.last = (int32_t)lds.found_bin;
                    __syncthreads();
                }
            } else {
                cut = cut_by_digits<NT, BINS>(q, walk, turn, want, upto, lds);
                bins_left = false;                          // (it used their place)
            }
            mass = upto;
        }
    } else {
        for (int32_t i = 0; i < cached; ++i) {
            const f32x4u_t t = __builtin_bit_cast(f32x4u_t, *slot(i));
            u32x4_t w;
#pragma unroll
            for (int c = 0; c < 4; ++c) w[c] = weight32(exponent_of(q, t[c]));
            *slot(i) = w;
        }
    }

    // Sums of what is kept, a part's at a time.  A weight tells whether its
    // candidate is, but for those around the cut's.
    const uint32_t floor32 = lim.least < 0xffffffffull ? (uint32_t)lim.least : 0xffffffffu;
    uint32_t near_lo = 0, near_hi = 0, kept = 0;
    if (cut.key != 0) near_weights(weight32(exponent_of(q, score_of(cut.key))), near_lo, near_hi);
    // many draws of a problem that is all in LDS: running sums for every lane and step
    const bool fine = set.n_draws > kWaves && walk.steps <= cached && walk.steps * NT <= Lds<NT, BINS, CACHED>::kFine;
    __syncthreads();                                        // (the bins are read)
    uint64_t sum = 0;
    int32_t part = wave * walk.per_wave, left = walk.each;  // the part that is summed, its steps to come
    auto stepped = [&](int32_t i) {
        if (--left > 0 && i + 1 < walk.steps) return;
        sum = wave_sum(sum);
        if (lane == 0) lds.part[part] = sum;
        ++part;
        left = walk.each;
        sum = 0;
    };
#pragma unroll 1
    for (int32_t i = 0; i < cached; ++i) {
        u32x4_t w = *slot(i);
        uint64_t four = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            bool in = w[c] >= floor32 && w[c] >= near_lo;
            if (w[c] >= near_lo && w[c] <= near_hi) {
                const int32_t at = walk.base + i * 256 + lane * 4 + c;
                in = in && at < q.n && within(cut, key_of(q.s[at < q.n ? at : 0]), at);
            }
            w[c] = in ? w[c] : 0;
            four += whole(w[c]);
            kept += in;
        }
        sum += four;
        if (fine) {                                         // (a part is a step: at most kParts of them fit)
            *slot(i) = w;
            lds.fine[i * NT + threadIdx.x] = wave_scan52(four);
        }
        stepped(i);
    }
    each_step(q.s, walk, cached, walk.steps, [&](int32_t i, const f32x4u_t &t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const uint32_t w = weight32(exponent_of(q, t[c]));
            bool in = w >= floor32 && w >= near_lo;
            if (w >= near_lo && w <= near_hi) in = in && within(cut, key_of(t[c]), walk.base + i * 256 + lane * 4 + c);
            sum += in ? whole(w) : 0;
            kept += in;
        }
        stepped(i);
    });
    kept = wave_sum(kept);
    if (lane == 0) lds.wave_count[wave] = kept;
    __syncthreads();
    const int n_parts = kWaves * walk.per_wave;
    sums_before(lds.part, n_parts);
    if (threadIdx.x == 0 && kept_out) {
        kept = 0;
        for (int w = 0; w < kWaves; ++w) kept += lds.wave_count[w];
        kept_out[p] = (int32_t)kept;
    }
    __syncthreads();
    const uint64_t total = lds.part[n_parts];
    if (fine) {                                             // a thread a draw
        for (uint32_t j = threadIdx.x; j < (uint32_t)set.n_draws; j += NT) {
            uint64_t r = point_of(u[j], total);
            int part = 0, four = 0;
            for (int step = kParts; step > 0; step >>= 1)   // parts that end at or before the point
                if (part + step < n_parts && lds.part[part + step] <= r) part += step;
            r -= lds.part[part];
            const int of = part / walk.steps, i = part % walk.steps, first = i * NT + of * 64;
            for (int step = 32; step > 0; step >>= 1)
                if (lds.fine[first + four + step - 1] <= r) four += step;
            r -= four ? lds.fine[first + four - 1] : 0;
            const u32x4_t w = *reinterpret_cast<const u32x4_t *>(lds.cache + (first + four) * 4);
            int c = 0;
#pragma unroll
            for (int e = 0; e < 3; ++e)
                if (c == e && whole(w[e]) <= r) {
                    r -= whole(w[e]);
                    ++c;
                }
            idx[j] = (of * walk.steps + i) * 256 + four * 4 + c;
            if (prob) prob[j] = (float)((double)whole(w[c]) / (double)total);
        }
        return;
    }
    for (uint32_t j = wave; j < (uint32_t)set.n_draws; j += kWaves) {
        uint64_t r = point_of(u[j], total);
        int part = 0;                                       // parts that end at or before the point
        for (int e = lane; e < ((n_parts + 63) & ~63); e += 64) part += __popcll(__ballot(e < n_parts && lds.part[e + 1] <= r));
        r -= lds.part[part];
        const Walk of = walk_of<NT>(q.n, part / walk.per_wave);
        const int32_t first = part % walk.per_wave * walk.each;
        draw_in(q, cut, lim.least, of, first, first + walk.each < walk.steps ? first + walk.each : walk.steps, r, total, idx + j,
                prob ? prob + j : nullptr);
    }
}

// WAVES: of a SIMD.
template <int NT, int BINS, int CACHED, int WAVES>
__global__ __launch_bounds__(NT, WAVES) void k_sample(const float *__restrict__ scores, int64_t R,
                                                      const int64_t *__restrict__ seg, Settings set,
                                                      const float *__restrict__ u, int32_t *__restrict__ idx,
                                                      float *__restrict__ prob, int32_t *__restrict__ kept_out)
{
    __shared__ Lds<NT, BINS, CACHED> lds;
    sample_problem<NT, BINS, CACHED>(lds, blockIdx.x, scores, R, seg, set, u, idx, prob, kept_out);
}

// Up to 1,024 candidates: a wave has a problem to itself, its scores and
// weights in registers, and waits for no other.  The steps are those above, the
// histogram one of 256 bins; the candidates of a bin are compared all with all.
constexpr int kSmall = 1024, kSmallBins = 256, kSmallList = 64;

union SmallLds {                                            // a wave's
    struct {
        uint64_t mass[kSmallBins], list[kSmallList];
        uint32_t count[kSmallBins];
    };
    struct {
        uint64_t run[kSmall / 4];                           // running sums after each four candidates
        uint32_t w[kSmall];
    };
};

// What this wave has written to LDS is there for all its lanes.
__device__ __forceinline__ void wave_sync()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// The index of a lane's candidate e.
__device__ __forceinline__ int32_t small_index(int lane, int e) { return (e >> 2) * 256 + lane * 4 + (e & 3); }

// The candidate at which the count (by_mass: mass), best first, reaches `want`,
// 1 <= want <= all of it; the mass up to there.
template <int EACH>
__device__ __forceinline__ Cut small_cut(const Problem &q, const float (&s)[EACH], const uint32_t (&w)[EACH],
                                         float bin_scale, bool by_mass, uint64_t want, uint64_t &mass, SmallLds &lds)
{
    const int lane = threadIdx.x & 63;
    uint64_t m[4], m_sum = 0;
    uint32_t c[4], c_sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        m[j] = lds.mass[lane * 4 + j];
        c[j] = lds.count[lane * 4 + j];
        m_sum += m[j];
        c_sum += c[j];
    }
    const uint64_t m_scan = wave_scan52(m_sum);
    const uint32_t c_scan = wave_scan(c_sum);
    uint64_t m_at = m_scan - m_sum;
    uint32_t c_at = c_scan - c_sum;
    const uint64_t from = by_mass ? m_at : (uint64_t)c_at, to = by_mass ? m_scan : (uint64_t)c_scan;
    const int owner = __builtin_ctzll(__ballot(from < want && to >= want));
    int j_at = 0;
#pragma unroll
    for (int j = 0; j < 3; ++j)
        if (j_at == j && (by_mass ? m_at + m[j] : (uint64_t)(c_at + c[j])) < want) {
            m_at += m[j];
            c_at += c[j];
            ++j_at;
        }
    const uint32_t bin = 4 * owner + (uint32_t)__builtin_amdgcn_readlane(j_at, owner);
    const uint64_t before_mass = lane_u64(m_at, owner);
    const uint32_t before_count = (uint32_t)__builtin_amdgcn_readlane((int)c_at, owner);

    uint32_t in_bin = 0, members = 0;                       // members: bit e, this lane's candidate e
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const bool in = w[e] != 0 && (uint32_t)(-exponent_of(q, s[e]) * bin_scale) == bin;
        const uint64_t lanes = __ballot(in);
        const uint32_t at = in_bin + __builtin_amdgcn_mbcnt_hi((uint32_t)(lanes >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)lanes, 0));
        if (in && at < kSmallList) lds.list[at] = ((uint64_t)key_of(s[e]) << 32) | (0xffffffffu - (uint32_t)small_index(lane, e));
        in_bin += (uint32_t)__popcll(lanes);
        members |= (uint32_t)in << e;
    }
    if (in_bin <= kSmallList) {                             // a lane each
        wave_sync();
        const bool own = (uint32_t)lane < in_bin;
        const uint64_t v = own ? lds.list[lane] : 0;
        const uint64_t v_w = own ? whole(weight32(exponent_of(q, score_of((uint32_t)(v >> 32))))) : 0;
        uint64_t mass_at = before_mass;
        uint32_t count_at = before_count;
        for (uint32_t o = 0; o < in_bin; ++o) {
            const uint64_t other = lane_u64(v, (int)o), other_w = lane_u64(v_w, (int)o);
            mass_at += other > v ? other_w : 0;
            count_at += other > v;
        }
        const uint64_t at = by_mass ? mass_at : (uint64_t)count_at, with = by_mass ? mass_at + v_w : (uint64_t)count_at + 1;
        const int at_lane = __builtin_ctzll(__ballot(own && at < want && with >= want));
        const uint64_t cut = lane_u64(v, at_lane);
        mass = lane_u64(mass_at + v_w, at_lane);
        return {(uint32_t)(cut >> 32), (int32_t)(0xffffffffu - (uint32_t)cut)};
    }
    // Many in a bin (equal scores): the largest key from which on `want` is reached, by halving.
    uint32_t hi = 0, lo = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const uint32_t key = members >> e & 1 ? key_of(s[e]) : 0;
        hi = key > hi ? key : hi;
        lo = key != 0 && ~key > lo ? ~key : lo;
    }
    hi = wave_max(hi);
    lo = ~wave_max(lo);
    auto from_key = [&](uint32_t key, uint64_t &n, uint64_t &sum) {        // of the bin, and of those before it
        uint64_t lane_n = 0, lane_sum = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const bool in = (members >> e & 1) && key_of(s[e]) >= key;
            lane_n += in;
            lane_sum += in ? whole(w[e]) : 0;
        }
        n = before_count + wave_sum((uint32_t)lane_n);
        sum = before_mass + lane_u64(wave_scan52(lane_sum), 63);
    };
    uint64_t n, sum;
#pragma unroll 1
    while (lo < hi) {
        const uint32_t mid = hi - (hi - lo) / 2;            // above lo
        from_key(mid, n, sum);
        if ((by_mass ? sum : n) >= want) lo = mid;
        else hi = mid - 1;
    }
    from_key(lo + 1, n, sum);                               // (no key is 2^32 - 1: it would be a NaN's)
    const uint64_t each = whole(weight32(exponent_of(q, score_of(lo))));
    uint32_t left = (uint32_t)(by_mass ? (want - sum + each - 1) / each : want - n);       // of those with this key
    mass = sum + left * each;
    int32_t last = 0;
    bool found = false;
#pragma unroll
    for (int i = 0; i < EACH / 4; ++i) {
        uint32_t tied = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) tied += key_of(s[4 * i + e]) == lo;
        const uint32_t scan = wave_scan(tied), here = (uint32_t)__builtin_amdgcn_readlane((int)scan, 63);
        if (!found && left <= here) {
            const int at_lane = __builtin_ctzll(__ballot(scan >= left));
            uint32_t run = scan - tied;
            int at = 0;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                run += key_of(s[4 * i + e]) == lo;
                at += run < left;
            }
            last = i * 256 + at_lane * 4 + __builtin_amdgcn_readlane(at, at_lane);
            found = true;
        }
        left -= found ? 0 : here;
    }
    return {lo, last};
}

// EACH: candidates a lane.
template <int EACH>
__device__ __forceinline__ void sample_small(Problem q, int32_t p, const Settings &set, const float *__restrict__ u,
                                             int32_t *__restrict__ idx, float *__restrict__ prob, int32_t *__restrict__ kept_out,
                                             SmallLds &lds)
{
    const int lane = threadIdx.x & 63;
    u += (int64_t)p * set.n_draws;
    idx += (int64_t)p * set.n_draws;
    if (prob) prob += (int64_t)p * set.n_draws;
    float s[EACH];
#pragma unroll
    for (int i = 0; i < EACH / 4; ++i) {
        const int32_t at = i * 256 + lane * 4;
        if (i * 256 + 256 <= q.n) {
            const f32x4u_t t = *reinterpret_cast<const f32x4u_t *>(q.s + at);
#pragma unroll
            for (int c = 0; c < 4; ++c) s[4 * i + c] = t[c];
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c) s[4 * i + c] = at + c < q.n ? q.s[at + c] : -__builtin_inff();
        }
    }
    const float u_first = lane < set.n_draws ? u[lane] : 0.0f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        lds.mass[lane * 4 + j] = 0;
        lds.count[lane * 4 + j] = 0;
    }
    float most = -__builtin_inff(), least_score = __builtin_inff();
    uint32_t alive = 0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
        const bool in = takes_part(s[e]);
        alive += (uint32_t)__popcll(__ballot(in));
        most = fmaxf(most, s[e]);
        least_score = fminf(least_score, in ? s[e] : __builtin_inff());
    }
    if (alive == 0) {
        for (uint32_t j = lane; j < (uint32_t)set.n_draws; j += 64) {
            idx[j] = -1;
            if (prob) prob[j] = 0.0f;
        }
        if (lane == 0 && kept_out) kept_out[p] = 0;
        return;
    }
    most = score_of(wave_max(order_key(most + 0.0f)));
    least_score = -score_of(wave_max(order_key(0.0f - least_score)));
    Limits lim;
    read_settings(set, p, most, q, lim);
    if (lim.k == 1) {
        uint32_t first = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < EACH / 4; ++i)
            first = first_best(q, (f32x4u_t){s[4 * i], s[4 * i + 1], s[4 * i + 2], s[4 * i + 3]}, i * 256 + lane * 4, first);
        write_one<64>((int32_t)~wave_max(~first), lane, set.n_draws, idx, prob);
        if (lane == 0 && kept_out) kept_out[p] = 1;
        return;
    }
    uint32_t w[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) w[e] = weight32(exponent_of(q, s[e]));

    const bool by_count = lim.k < alive, by_mass = lim.top_p < 1.0f;
    Cut cut{0, 0x7fffffff};
    if (by_count || by_mass) {
        const float t_least = -exponent_of(q, least_score), span = t_least < 34.0f ? t_least : 34.0f;
        const float bin_scale = span > 0.0f ? fminf((float)(kSmallBins - 1) / span, 1e30f) : 1.0f;
        uint32_t in_bins = 0;
        uint64_t mass = 0;
        wave_sync();
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            if (w[e] != 0) {
                const uint32_t bin = (uint32_t)(-exponent_of(q, s[e]) * bin_scale);
                atomicAdd((unsigned long long *)&lds.mass[bin], (unsigned long long)whole(w[e]));
                atomicAdd(&lds.count[bin], 1u);
                mass += whole(w[e]);
            }
            in_bins += (uint32_t)__popcll(__ballot(w[e] != 0));
        }
        wave_sync();
        mass = lane_u64(wave_scan52(mass), 63);
        // first the k best, then the share of their mass
#pragma unroll 1
        for (int turn = by_count && lim.k < in_bins ? 0 : 1; turn < (by_mass ? 2 : 1); ++turn)
            cut = small_cut(q, s, w, bin_scale, turn, turn ? share_of(lim, mass) : lim.k, mass, lds);
        wave_sync();                                        // (the histogram is read)
    }

    const uint32_t floor32 = lim.least < 0xffffffffull ? (uint32_t)lim.least : 0xffffffffu;
    uint32_t kept = 0;
    uint64_t four[EACH / 4], run[EACH / 4], total = 0;
#pragma unroll
    for (int i = 0; i < EACH / 4; ++i) {
        four[i] = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const int e = 4 * i + c;
            const bool in = w[e] >= floor32 && within(cut, key_of(s[e]), small_index(lane, e));
            kept += (uint32_t)__popcll(__ballot(in));
            w[e] = in ? w[e] : 0;
            four[i] += whole(w[e]);
        }
        run[i] = total + wave_scan52(four[i]);
        total = lane_u64(run[i], 63);
    }
    if (lane == 0 && kept_out) kept_out[p] = (int32_t)kept;
    if (set.n_draws <= 8) {                                 // the wave finds one after another
        for (int32_t j = 0; j < set.n_draws; ++j) {
            const uint64_t r = point_of(__uint_as_float((uint32_t)__builtin_amdgcn_readlane(__float_as_int(u_first), j)), total);
            bool found = false;
#pragma unroll
            for (int i = 0; i < EACH / 4; ++i) {
                const uint64_t over = found ? 0 : __ballot(run[i] > r);
                if (over == 0) continue;
                found = true;
                if (lane != __builtin_ctzll(over)) continue;
                uint64_t left = r - (run[i] - four[i]);
                int c = 0;
                uint32_t at = w[4 * i];
#pragma unroll
                for (int e = 0; e < 3; ++e)
                    if (c == e && whole(w[4 * i + e]) <= left) {
                        left -= whole(w[4 * i + e]);
                        at = w[4 * i + e + 1];
                        ++c;
                    }
                idx[j] = small_index(lane, 4 * i + c);
                if (prob) prob[j] = (float)((double)whole(at) / (double)total);
            }
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < EACH / 4; ++i) {
        lds.run[i * 64 + lane] = run[i];
        *reinterpret_cast<u32x4_t *>(lds.w + (i * 64 + lane) * 4) = (u32x4_t){w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
    }
    wave_sync();
    for (uint32_t j = lane; j < (uint32_t)set.n_draws; j += 64) {      // a lane a draw
        uint64_t r = point_of(j < 64 ? u_first : u[j], total);
        int at = 0;
#pragma unroll
        for (int step = EACH * 8; step > 0; step >>= 1)
            if (lds.run[at + step - 1] <= r) at += step;
        r -= at ? lds.run[at - 1] : 0;
        const u32x4_t v = *reinterpret_cast<const u32x4_t *>(lds.w + at * 4);
        int c = 0;
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (c == e && whole(v[e]) <= r) {
                r -= whole(v[e]);
                ++c;
            }
        idx[j] = at * 4 + c;
        if (prob) prob[j] = (float)((double)whole(v[c]) / (double)total);
    }
}

// `each` problems a workgroup: those of up to kSmall candidates a wave each,
// then the others by the whole workgroup, one after another.
template <int NT, int BINS, int CACHED>
__global__ __launch_bounds__(NT, 3) void k_sample_waves(const float *__restrict__ scores, int64_t R, const int64_t *__restrict__ seg,
                                                        int32_t P, int32_t each, Settings set, const float *__restrict__ u,
                                                        int32_t *__restrict__ idx, float *__restrict__ prob,
                                                        int32_t *__restrict__ kept_out)
{
    __shared__ union {
        Lds<NT, BINS, CACHED> lds;
        SmallLds small[NT / 64];
    } sh;
    const int32_t wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), p0 = (int32_t)blockIdx.x * each;
    if (wave < each && p0 + wave < P) {
        const Problem q = problem_of(scores, R, seg, p0 + wave);
        if (q.n <= 256) sample_small<4>(q, p0 + wave, set, u, idx, prob, kept_out, sh.small[wave]);
        else if (q.n <= 512) sample_small<8>(q, p0 + wave, set, u, idx, prob, kept_out, sh.small[wave]);
        else if (q.n <= kSmall) sample_small<16>(q, p0 + wave, set, u, idx, prob, kept_out, sh.small[wave]);
    }
#pragma unroll 1
    for (int32_t p = p0; p < p0 + each && p < P; ++p) {
        if (problem_of(scores, R, seg, p).n <= kSmall) continue;           // (the same for all threads)
        __syncthreads();                                    // (LDS is free again)
        sample_problem<NT, BINS, CACHED>(sh.lds, p, scores, R, seg, set, u, idx, prob, kept_out);
    }
}

// Few problems of many candidates: each is shared by many workgroups, in
// passes that hand their results on in the workspace: best score; histogram;
// candidates around the cut, ranked by one workgroup (once for top-k, once for
// top-p); sums of parts; draws.  A compute unit takes in some 100 GB/s, so 3
// problems of 534,600 take 881 us in a workgroup each, 53 so.  (Ending a pass
// by its last workgroup instead of a launch: 64 problems of 131,072 82 -> 358
// us, its fences write back L2.)
constexpr int kWide = 1024, kWideBins = 4096, kWideNear = 1536, kWideParts = 1024, kWideBlocks = 512;

struct WideBest {                                           // keys of a workgroup's best score and of its least's negative
    uint32_t best, least, alive, pad;
};

struct WideState {
    WideBest best_of[kWideBlocks];
    uint32_t best, least, alive, bin, before_count, n_near, tied_key, first;    // first: the lowest index of the best score
    uint64_t before_mass, want, mass;
    Cut cut;
    uint64_t mass_of[kWideBins], part[kWideParts];
    uint64_t near[kWideNear];                               // as they are ranked
    uint32_t count_of[kWideBins], kept_of[kWideParts];
    uint32_t tied_of[kWideBlocks * (kWide / 64)];           // of each wave
};

struct WideArgs {
    const float *scores;
    int64_t R;
    const int64_t *seg;
    WideState *state;
    Settings set;
};

// This wave's steps of problem blockIdx.y among those of all its workgroups.
__device__ __forceinline__ Walk shared_walk(int32_t n)
{
    const int32_t waves = (int32_t)gridDim.x * (kWide / 64);
    const int32_t wave = __builtin_amdgcn_readfirstlane((int)blockIdx.x * (kWide / 64) + (threadIdx.x >> 6));
    Walk w;
    w.n = n;
    w.steps = (int32_t)(((int64_t)n + 256 * (int64_t)waves - 1) / (256 * (int64_t)waves));
    w.base = (int32_t)((int64_t)wave * w.steps * 256 < n ? (int64_t)wave * w.steps * 256 : n);
    w.each = w.steps;
    w.per_wave = 1;
    return w;
}

// Steps of one of at most kWideParts parts of n candidates.
__device__ __forceinline__ int32_t wide_each(int32_t n)
{
    return (int32_t)(((int64_t)n + 256 * kWideParts - 1) / (256 * kWideParts));
}

// Best and least score of each workgroup's candidates; clears what the later
// passes count in.
__global__ __launch_bounds__(kWide) void k_wide_best(WideArgs a)
{
    const int32_t p = blockIdx.y;
    WideState &st = a.state[p];
    const Problem q = problem_of(a.scores, a.R, a.seg, p);
    const Walk walk = shared_walk(q.n);
    for (int i = (int)blockIdx.x * kWide + (int)threadIdx.x; i < kWideBins; i += (int)gridDim.x * kWide) {
        st.mass_of[i] = 0;
        st.count_of[i] = 0;
    }
    float most = -__builtin_inff(), least = __builtin_inff();
    uint32_t alive = 0;
    each_step(q.s, walk, 0, walk.steps, [&](int32_t, const f32x4u_t &t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const bool in = takes_part(t[c]);
            alive += in;
            most = fmaxf(most, t[c]);
            least = fminf(least, in ? t[c] : __builtin_inff());
        }
    });
    alive = wave_sum(alive);
    const uint32_t hi = wave_max(order_key(most + 0.0f)), lo = wave_max(order_key(0.0f - least));
    __shared__ uint32_t sh[3];
    if (threadIdx.x < 3) sh[threadIdx.x] = 0;
    __syncthreads();
    if ((threadIdx.x & 63) == 0 && alive != 0) {
        atomicMax(&sh[0], hi);
        atomicMax(&sh[1], lo);
        atomicAdd(&sh[2], alive);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        st.best_of[blockIdx.x] = {sh[0], sh[1], sh[2], 0};
        if (blockIdx.x == 0) {
            st.first = 0xffffffffu;
            st.n_near = 0;
            st.mass = 0;
            st.cut = {0, 0x7fffffff};
        }
    }
}

// A problem with its settings read, and its bins' scale.
__device__ __forceinline__ float wide_settings(const WideArgs &a, int32_t p, uint32_t best, uint32_t least, Problem &q, Limits &lim)
{
    read_settings(a.set, p, score_of(best), q, lim);
    const float t_least = -exponent_of(q, -score_of(least)), span = t_least < 34.0f ? t_least : 34.0f;
    return span > 0.0f ? fminf((float)(kWideBins - 1) / span, 1e30f) : 1.0f;
}

__global__ __launch_bounds__(kWide) void k_wide_bins(WideArgs a)
{
    __shared__ uint64_t mass[kWideBins];
    __shared__ uint32_t count[kWideBins];
    const int32_t p = blockIdx.y;
    WideState &st = a.state[p];
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    uint32_t best = 0, least = 0, alive = 0;                // of all workgroups', by each wave
    for (int i = threadIdx.x & 63; i < (int)gridDim.x; i += 64) {
        const WideBest b = st.best_of[i];
        best = b.best > best ? b.best : best;
        least = b.least > least ? b.least : least;
        alive += b.alive;
    }
    best = wave_max(best);
    least = wave_max(least);
    alive = wave_sum(alive);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        st.best = best;
        st.least = least;
        st.alive = alive;
    }
    if (alive == 0) return;
    Limits lim;
    const float bin_scale = wide_settings(a, p, best, least, q, lim);
    const bool by_count = lim.k < alive;
    const Walk walk = shared_walk(q.n);
    if (lim.k == 1) {
        uint32_t first = 0xffffffffu;
        each_step(q.s, walk, 0, walk.steps, [&](int32_t i, const f32x4u_t &t) { first = first_best(q, t, walk.base + i * 256 + (int)(threadIdx.x & 63) * 4, first); });
        first = ~wave_max(~first);
        if ((threadIdx.x & 63) == 0 && first != 0xffffffffu) atomicMin(&st.first, first);
        return;
    }
    if (!by_count && !(lim.top_p < 1.0f)) return;
    for (int i = threadIdx.x; i < kWideBins; i += kWide) {
        mass[i] = 0;
        count[i] = 0;
    }
    __syncthreads();
    each_step(q.s, walk, 0, walk.steps, [&](int32_t, const f32x4u_t &t) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            const float e = exponent_of(q, t[c]);
            const uint32_t w = weight32(e);
            if (w != 0) {
                const uint32_t bin = (uint32_t)(-e * bin_scale);
                atomicAdd((unsigned long long *)&mass[bin], (unsigned long long)whole(w));
                if (by_count) atomicAdd(&count[bin], 1u);
            }
        }
    });
    __syncthreads();
    for (int i = threadIdx.x; i < kWideBins; i += kWide)
        if (mass[i] != 0) {
            atomicAdd((unsigned long long *)&st.mass_of[i], (unsigned long long)mass[i]);
            if (by_count) atomicAdd(&st.count_of[i], count[i]);
        }
}

// Before each cut, a workgroup a problem: its bin, or that there is none to
// find (want = 0).  turn 0: top-k, 1: top-p.
__global__ __launch_bounds__(kWide) void k_wide_find(WideArgs a, int turn)
{
    __shared__ Lds<kWide, kWideBins, 4> lds;
    const int32_t p = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    WideState &st = a.state[p];
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    if (threadIdx.x == 0) {
        st.want = 0;
        st.n_near = 0;
    }
    if (st.alive == 0) return;
    Limits lim;
    const float bin_scale = wide_settings(a, p, st.best, st.least, q, lim);
    if (lim.k == 1 || (turn ? !(lim.top_p < 1.0f) : !(lim.k < st.alive))) return;
    // 4,096 scores from here and there, among which one that many share will be found (16,384 singly: 14 us more)
    constexpr int kLook = 4;
    float look[kLook];
#pragma unroll
    for (int j = 0; j < kLook; ++j) {
        const int64_t at = (int64_t)wave * q.n / (kWide / 64) + lane * kLook + j;
        look[j] = q.s[at < q.n ? at : q.n - 1];
    }
    if (threadIdx.x == 0) lds.n_near = 0;
    uint64_t mass = 0;
    uint32_t n = 0;
    for (int i = threadIdx.x; i < kWideBins; i += kWide) {
        lds.mass[i] = st.mass_of[i];
        lds.count[i] = st.count_of[i];
        mass += lds.mass[i];
        n += lds.count[i];
    }
    n = wave_sum(n);
    mass = wave_sum(mass);
    if (lane == 0) {
        lds.wave_count[wave] = n;
        lds.wave_mass[wave] = mass;
    }
    __syncthreads();
    n = 0;
    mass = 0;
    for (int w = 0; w < kWide / 64; ++w) {
        n += lds.wave_count[w];
        mass += lds.wave_mass[w];
    }
    __syncthreads();
    if (turn == 0 && !(lim.k < n)) return;                  // (scores that weigh nothing are in no bin)
    const uint64_t want = turn ? share_of(lim, st.mass != 0 ? st.mass : mass) : lim.k;
    uint32_t bin, before_count;
    uint64_t before_mass;
    find_bin<kWide, kWideBins>(lds, turn, want, bin, before_count, before_mass);
#pragma unroll
    for (int j = 0; j < kLook; ++j)
        if (takes_part(look[j]) && (uint32_t)(-exponent_of(q, look[j]) * bin_scale) == bin) {
            const uint32_t at = atomicAdd(&lds.n_near, 1u);
            if (at < 64) lds.near[at] = key_of(look[j]);
        }
    __syncthreads();
    if (wave != 0) return;
    const uint32_t tied_key = commonest((uint32_t)lane < lds.n_near ? lds.near[lane] : 0);
    if (threadIdx.x == 0) {
        st.want = want;
        st.tied_key = tied_key;
        st.bin = bin;
        st.before_count = before_count;
        st.before_mass = before_mass;
    }
}

__global__ __launch_bounds__(kWide) void k_wide_list(WideArgs a)
{
    const int32_t p = blockIdx.y, lane = threadIdx.x & 63;
    WideState &st = a.state[p];
    if (st.alive == 0 || st.want == 0) return;
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    Limits lim;
    const float bin_scale = wide_settings(a, p, st.best, st.least, q, lim);
    const uint32_t bin = st.bin, tied_key = st.tied_key;
    const Walk walk = shared_walk(q.n);
    uint32_t tied = 0;
    each_step(q.s, walk, 0, walk.steps, [&](int32_t i, const f32x4u_t &t) {
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (takes_part(t[c]) && (uint32_t)(-exponent_of(q, t[c]) * bin_scale) == bin) {
                if (key_of(t[c]) == tied_key) {
                    ++tied;
                    continue;
                }
                const uint32_t at = atomicAdd(&st.n_near, 1u);
                if (at < kWideNear) st.near[at] = rank_of(t[c], (uint32_t)(walk.base + i * 256 + lane * 4 + c));
            }
    });
    tied = wave_sum(tied);
    if (lane == 0) st.tied_of[(int)blockIdx.x * (kWide / 64) + (int)(threadIdx.x >> 6)] = tied;
}

__global__ __launch_bounds__(kWide) void k_wide_cut(WideArgs a, int turn, int32_t blocks)
{
    __shared__ Lds<kWide, kWideBins, 4> lds;
    static_assert(Lds<kWide, kWideBins, 4>::kList == kWideNear, "the list fits");
    const int32_t p = blockIdx.x;
    WideState &st = a.state[p];
    constexpr int kNear = (kWideNear + kWide - 1) / kWide;  // (on their way before it is known how many there are)
    uint64_t near[kNear];
#pragma unroll
    for (int i = 0; i < kNear; ++i) near[i] = threadIdx.x + i * kWide < kWideNear ? st.near[threadIdx.x + i * kWide] : 0;
    if (st.alive == 0 || st.want == 0) return;
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    Limits lim;
    wide_settings(a, p, st.best, st.least, q, lim);
    const uint32_t m = st.n_near;
    uint64_t upto;
    Cut cut;
    // the tied ones: a thread takes consecutive waves of k_wide_list
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blocks * (kWide / 64), own = (waves + kWide - 1) / kWide;
    Tied tied{st.tied_key, 0};
    uint32_t here = 0;
    for (int i = 0; i < own; ++i) {
        const int w = (int)threadIdx.x * own + i;
        here += w < waves ? st.tied_of[w] : 0;
    }
    const uint32_t scan = wave_scan(here);
    if (lane == 63) lds.wave_count[wave] = scan;
    __syncthreads();
    uint32_t before = scan - here;
    for (int w = 0; w < kWide / 64; ++w) {
        before += w < wave ? lds.wave_count[w] : 0;
        tied.count += lds.wave_count[w];
    }
    if (tied.count == 0) tied.key = 0;
    __syncthreads();
    if (m + (tied.key != 0) <= kWideNear) {
#pragma unroll
        for (int i = 0; i < kNear; ++i)
            if (threadIdx.x + i * kWide < m) lds.list[threadIdx.x + i * kWide] = near[i];
        if (threadIdx.x < kWide / 64) lds.wave_count[threadIdx.x] = threadIdx.x == 0 ? m : 0;
        uint32_t ties;
        cut = rank_bin<kWide>(q, m, tied, turn, st.before_count, st.before_mass, st.want, upto, ties, lds);
        if (ties != 0) {                                    // which wave's it is, and what is before that wave
            if (ties > before && ties <= before + here) {
                int w = (int)threadIdx.x * own;
                while (ties > before + st.tied_of[w]) before += st.tied_of[w++];
                lds.found_bin = (uint32_t)w;
                lds.found_count = ties - before;
            }
            __syncthreads();
            const uint32_t w = lds.found_bin, left = lds.found_count;
            __syncthreads();
            if (wave == 0) {
                const int32_t steps = (int32_t)(((int64_t)q.n + 256 * (int64_t)waves - 1) / (256 * (int64_t)waves));
                const Walk walk{q.n, steps, (int32_t)w * steps * 256, steps, 1};
                const int32_t at = tied_at<4>(q, walk, 0, steps, cut.key, left);
                if (lane == 0) lds.found_bin = (uint32_t)at;
            }
            __syncthreads();
            cut.last = (int32_t)lds.found_bin;
        }
    } else {
        cut = cut_by_digits<kWide, kWideBins>(q, walk_of<kWide>(q.n, (int)(threadIdx.x >> 6)), turn, st.want, upto, lds);
    }
    if (threadIdx.x == 0) {
        st.cut = cut;
        st.mass = upto;
    }
}

__global__ __launch_bounds__(kWide) void k_wide_sums(WideArgs a)
{
    const int32_t p = blockIdx.y, lane = threadIdx.x & 63;
    WideState &st = a.state[p];
    if (st.alive == 0) return;
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    Limits lim;
    wide_settings(a, p, st.best, st.least, q, lim);
    if (lim.k == 1) return;
    const Cut cut = st.cut;
    const int32_t each = wide_each(q.n), parts = (int32_t)(((int64_t)q.n + 256 * (int64_t)each - 1) / (256 * (int64_t)each));
    for (int32_t e = __builtin_amdgcn_readfirstlane((int)blockIdx.x * (kWide / 64) + (threadIdx.x >> 6)); e < parts;
         e += (int32_t)gridDim.x * (kWide / 64)) {
        const Walk walk{q.n, each, e * each * 256, each, 1};
        uint64_t sum = 0;
        uint32_t kept = 0;
        each_step(q.s, walk, 0, each, [&](int32_t i, const f32x4u_t &t) {
            uint64_t w[4];
            kept_weights(q, cut, lim.least, t, walk.base + i * 256 + lane * 4, w);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                sum += w[c];
                kept += w[c] != 0;
            }
        });
        sum = wave_sum(sum);
        kept = wave_sum(kept);
        if (lane == 0) {
            st.part[e] = sum;
            st.kept_of[e] = kept;
        }
    }
}

__global__ __launch_bounds__(kWide) void k_wide_draw(WideArgs a, const float *__restrict__ u, int32_t *__restrict__ idx,
                                                     float *__restrict__ prob, int32_t *__restrict__ kept_out)
{
    __shared__ uint64_t part[kWideParts + 1], wave_mass[kWide / 64];
    __shared__ uint32_t wave_kept[kWide / 64];
    const int32_t p = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int32_t n_draws = a.set.n_draws;
    const WideState &st = a.state[p];
    u += (int64_t)p * n_draws;
    idx += (int64_t)p * n_draws;
    if (prob) prob += (int64_t)p * n_draws;
    if (st.alive == 0) {
        if (threadIdx.x == 0 && kept_out) kept_out[p] = 0;
        for (uint32_t j = threadIdx.x; j < (uint32_t)n_draws; j += kWide) {
            idx[j] = -1;
            if (prob) prob[j] = 0.0f;
        }
        return;
    }
    Problem q = problem_of(a.scores, a.R, a.seg, p);
    Limits lim;
    wide_settings(a, p, st.best, st.least, q, lim);
    if (lim.k == 1) {
        write_one<kWide>((int32_t)st.first, threadIdx.x, n_draws, idx, prob);
        if (threadIdx.x == 0 && kept_out) kept_out[p] = 1;
        return;
    }
    const Cut cut = st.cut;
    const int32_t each = wide_each(q.n), parts = (int32_t)(((int64_t)q.n + 256 * (int64_t)each - 1) / (256 * (int64_t)each));
    const uint64_t own = (int)threadIdx.x < parts ? st.part[threadIdx.x] : 0, scan = wave_scan(own);
    uint32_t kept = wave_sum((int)threadIdx.x < parts ? st.kept_of[threadIdx.x] : 0);
    if (lane == 63) {
        wave_mass[wave] = scan;
        wave_kept[wave] = kept;
    }
    __syncthreads();
    uint64_t before = scan - own, total = 0;
    kept = 0;
    for (int w = 0; w < kWide / 64; ++w) {
        if (w < wave) before += wave_mass[w];
        total += wave_mass[w];
        kept += wave_kept[w];
    }
    if (threadIdx.x == 0 && kept_out) kept_out[p] = (int32_t)kept;
    part[threadIdx.x] = before;
    if (threadIdx.x == 0) part[kWideParts] = total;
    __syncthreads();
    for (uint32_t j = wave; j < (uint32_t)n_draws; j += kWide / 64) {
        uint64_t r = point_of(u[j], total);
        int32_t e = 0;
        for (int step = kWideParts / 2; step > 0; step >>= 1)
            if (e + step < parts && part[e + step] <= r) e += step;
        draw_in(q, cut, lim.least, Walk{q.n, each, e * each * 256, each, 1}, 0, each, r - part[e], total, idx + j,
                prob ? prob + j : nullptr);
    }
}

}  // namespace

// Segment lengths are not known here; their mean is.  Few problems of many
// candidates are shared by workgroups, which costs seven launches for top-k or
// top-p and ten for both: 8 problems of 49,152 38 us (a workgroup each: 40), 8 of 32,768 35 (30); 64 of 131,072 74
// (83), 64 of 65,536 65 (50); 128 of 262,144 157 (163), 128 of 131,072 101 (92).
static bool shared_problems(int64_t R, int32_t P) { return P <= 128 && R / P > 36864 + 1280 * (int64_t)P; }

// A wave a problem, for problems of up to kSmall candidates on average: 16 problems of 64 6.3 us (512 threads each:
// 12.7), of 512 7.7 (12.8), of 1,000 11.3 (12.9); 4,096 of 64 13 (90), of 512 17.6 (90), of 1,000 50 (93).  Longer
// ones among them go by 256 threads: 600 of up to 1,400 17.4 (23.5), 1,000 of up to 2,000 27.0 (34.4), but 100 of up
// to 1,400 14.0 (13.6).
constexpr int64_t kSmallMean = kSmall;

size_t sample_workspace_bytes(int64_t R, int32_t P, int32_t)
{
    return shared_problems(R, P) ? (size_t)P * sizeof(WideState) : 0;
}

static void launch_shared(const WideArgs &a, int32_t P, const float *u, int32_t *idx, float *prob, int32_t *kept, hipStream_t s)
{
    // sixteen steps or so a wave, the machine filled about twice
    int64_t blocks = (a.R + 16383) / 16384;
    for (const int64_t most : {(2 * (int64_t)compute_units() + P - 1) / P, (int64_t)kWideBlocks}) blocks = blocks < most ? blocks : most;
    const dim3 shared((unsigned)blocks, (unsigned)P), one((unsigned)P), block(kWide);
    hipLaunchKernelGGL(k_wide_best, shared, block, 0, s, a);
    const bool by_count = a.set.how.top_k_of || a.set.how.top_k > 0 || a.set.how.temperature_of || !(a.set.how.temperature > 0.0f),
               by_mass = a.set.how.top_p_of || a.set.how.top_p < 1.0f;
    hipLaunchKernelGGL(k_wide_bins, shared, block, 0, s, a);  // (also where no prefix is wanted: it says which score is the best)
    const bool one_each = (!a.set.how.temperature_of && !(a.set.how.temperature > 0.0f)) ||
                          (!a.set.how.top_k_of && a.set.how.top_k == 1);   // only the best of every problem
    for (int turn = one_each ? 2 : 0; turn < 2; ++turn) {
        if (!(turn ? by_mass : by_count)) continue;
        hipLaunchKernelGGL(k_wide_find, one, block, 0, s, a, turn);
        hipLaunchKernelGGL(k_wide_list, shared, block, 0, s, a);
        hipLaunchKernelGGL(k_wide_cut, one, block, 0, s, a, turn, (int32_t)blocks);
    }
    if (!one_each) hipLaunchKernelGGL(k_wide_sums, shared, block, 0, s, a);
    hipLaunchKernelGGL(k_wide_draw, one, block, 0, s, a, u, idx, prob, kept);
}

// launch(problems, seg, settings, u, idx, prob, kept) for spans of problems.
template <class F>
static void each_problems(const int64_t *seg, int32_t P, const hwsel_sampling_t &how, const float *u, int32_t n_draws, int32_t *idx,
                          float *prob, int32_t *kept, F &&launch)
{
    each_span(P, [&](int32_t p0, int32_t n) {
        hwsel_sampling_t h = how;
        if (h.temperature_of) h.temperature_of += p0;
        if (h.top_k_of) h.top_k_of += p0;
        if (h.top_p_of) h.top_p_of += p0;
        if (h.min_p_of) h.min_p_of += p0;
        const int64_t o = (int64_t)p0 * n_draws;
        launch(n, seg + p0, Settings{h, n_draws}, u + o, idx + o, prob ? prob + o : nullptr, kept ? kept + p0 : nullptr);
    });
}

template <int NT, int BINS, int CACHED, int WAVES>
static void launch_problems(const float *scores, int64_t R, const int64_t *seg, int32_t P, const hwsel_sampling_t &how,
                            const float *u, int32_t n_draws, int32_t *idx, float *prob, int32_t *kept, hipStream_t s)
{
    each_problems(seg, P, how, u, n_draws, idx, prob, kept, [&](int32_t n, auto... rest) {
        hipLaunchKernelGGL((k_sample<NT, BINS, CACHED, WAVES>), dim3(n), dim3(NT), 0, s, scores, R, rest...);
    });
}

// Enough workgroups for every compute unit first, then as many problems as a workgroup has waves, but one where half
// of the problems may be longer and follow each other (1,000 of up to 2,000: 27 us, four by four 49).
static void launch_waves(const float *scores, int64_t R, const int64_t *seg, int32_t P, const hwsel_sampling_t &how, const float *u,
                         int32_t n_draws, int32_t *idx, float *prob, int32_t *kept, hipStream_t s)
{
    constexpr int NT = 256;
    each_problems(seg, P, how, u, n_draws, idx, prob, kept, [&](int32_t n, const int64_t *seg_n, auto... rest) {
        const int32_t cus = compute_units(), each = n <= cus || R / P > kSmall / 2 ? 1 : n >= cus * (NT / 64) ? NT / 64 : (n + cus - 1) / cus;
        hipLaunchKernelGGL((k_sample_waves<NT, 1024, 4096>), dim3((n + each - 1) / each), dim3(NT), 0, s, scores, R, seg_n, n, each, rest...);
    });
}

hipError_t launch_sample(const float *scores, int64_t R, const int64_t *seg, int32_t P, const hwsel_sampling_t &how,
                         const float *u, int32_t n_draws, int32_t *idx, float *prob, int32_t *kept, void *ws, hipStream_t s)
{
    if (shared_problems(R, P))
        launch_shared(WideArgs{scores, R, seg, static_cast<WideState *>(ws), Settings{how, n_draws}}, P, u, idx, prob, kept, s);
    else if (R / P <= kSmallMean) launch_waves(scores, R, seg, P, how, u, n_draws, idx, prob, kept, s);
    // Where problems outnumber compute units, three workgroups share one, of 256 threads for up to 12,288 candidates and
    // of 512 (in 80 registers) for more: 600 problems of up to 8,192 with 64 draws 26.8 us (512: 29.6), 600 of 4,000
    // 21.1 (26.8), 600 of 12,000 37.8 (42.7), 600 of 16,384 44.0 (44.2), but 300 of 16,000 40 (36), 300 of 65,536 134
    // (103; 1,024 threads: 125), 2,000 of 32,768 218 (193; 305).  Otherwise 512 up to 8,192 candidates, which wait for
    // each other less than 1,024, which keep more than three times as many candidates in LDS: 16 of 4,000 15.0 (256
    // threads: 16.9), 128 of 8,192 16.8 (1,024 threads: 17.6), but 8 of 12,288 21.2 (19.4) and 256 of 24,576 33 (26).
    else if (P > compute_units()) {
        if (R / P <= 12288) launch_problems<256, 1024, 8192, 3>(scores, R, seg, P, how, u, n_draws, idx, prob, kept, s);
        else launch_problems<512, 1024, 8192, 6>(scores, R, seg, P, how, u, n_draws, idx, prob, kept, s);
    }
    else if (R / P <= 8192) launch_problems<512, 1024, 8192, 4>(scores, R, seg, P, how, u, n_draws, idx, prob, kept, s);
    else launch_problems<1024, 2048, 28672, 4>(scores, R, seg, P, how, u, n_draws, idx, prob, kept, s);
    return hipGetLastError();
}

}  // namespace hwsel
