// Drawing candidates from a problem's scores: softmax at a temperature, limited
// by top-k, top-p and min-p, by given random numbers.
//
// Weights are whole numbers, so sums do not depend on their order and every
// comparison is exact.  The kept set is a prefix of the order (score
// descending, index ascending) without sorting: the key of its last score is
// found digit by digit from histograms of count and mass (11 + 11 + 10 bits),
// the ones tied with it are kept from the lowest index on.
#include "internal.hpp"

namespace hwsel {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64, kBins = 2048;

struct Settings {
    hwsel_sampling_t how;
    int32_t n_draws;
};

// floor(2^32 2^t) in stated steps, t = (s - best) * rate (compiled without
// multiply-add contraction: every product and sum rounds).
__device__ __forceinline__ uint64_t weight_of(float s, float best, float rate)
{
    float t = (s - best) * rate;
    t = s == best ? 0.0f : t;
    t = t > -60.0f ? t : -60.0f;
    const float n = rintf(t), f = t - n;
    float p = 1.5403530e-04f;                               // ln(2)^i / i!, i = 6 .. 0
    p = p * f + 1.3333558e-03f;
    p = p * f + 9.6181291e-03f;
    p = p * f + 5.5504109e-02f;
    p = p * f + 2.4022651e-01f;
    p = p * f + 6.9314718e-01f;
    p = p * f + 1.0f;
    return ((uint64_t)(uint32_t)(p * 16777216.0f) << 8) >> (int)-n;
}

// Key of a score that takes part (larger is better), 0 for NaN and -inf.
__device__ __forceinline__ uint32_t key_of(float s) { return s > -__builtin_inff() ? order_key(s + 0.0f) : 0u; }

__device__ __forceinline__ float score_of(uint32_t key)
{
    return __uint_as_float((key & 0x80000000u) ? key ^ 0x80000000u : ~key);
}

template <class T>
__device__ __forceinline__ T wave_sum(T v)
{
#pragma unroll
    for (int l = 1; l < 64; l <<= 1) v += __shfl_xor(v, l);
    return v;
}

template <class T>
__device__ __forceinline__ T wave_scan(T v, int lane)      // inclusive
{
#pragma unroll
    for (int l = 1; l < 64; l <<= 1) {
        const T o = __shfl_up(v, l);
        v += lane >= l ? o : T(0);
    }
    return v;
}

struct Lds {
    uint64_t mass[kBins];
    uint32_t count[kBins];
    uint64_t wave_mass[kWaves];
    uint32_t wave_count[kWaves];
    uint64_t found_mass;                                    // above the found digit
    uint32_t found_count, found_bin;
};

// The largest key K at which the count (BY_MASS: the mass) of scores with keys
// >= K reaches `want`, which the whole does; count and mass strictly above K.
template <bool BY_MASS>
__device__ __forceinline__ uint32_t descend(const float *__restrict__ s, int32_t n, float best, float rate, uint64_t want,
                                            uint32_t &above_count, uint64_t &above_mass, Lds &lds)
{
    uint32_t prefix = 0;
    above_count = 0;
    above_mass = 0;
    constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};
    for (int level = 0; level < 3; ++level) {
        const int shift = kShift[level], bits = kBits[level];
        for (int b = threadIdx.x; b < kBins; b += kThreads) {
            lds.mass[b] = 0;
            lds.count[b] = 0;
        }
        __syncthreads();
        for (int32_t i = threadIdx.x; i < n; i += kThreads) {
            const float v = s[i];
            const uint32_t key = key_of(v);
            const uint32_t high = level == 0 ? 0u : key >> (shift + bits);
            if (key == 0 || high != prefix) continue;
            const uint32_t bin = (key >> shift) & ((1u << bits) - 1);
            atomicAdd(&lds.count[bin], 1u);
            atomicAdd((unsigned long long *)&lds.mass[bin], (unsigned long long)weight_of(v, best, rate));
        }
        __syncthreads();
        // from the top bin down: thread t has bins kBins - 1 - 2 t and the one below
        const int hi = kBins - 1 - 2 * (int)threadIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        const uint64_t m2 = lds.mass[hi] + lds.mass[hi - 1];
        const uint32_t c2 = lds.count[hi] + lds.count[hi - 1];
        const uint64_t m_scan = wave_scan(m2, lane);
        const uint32_t c_scan = wave_scan(c2, lane);
        if (lane == 63) {
            lds.wave_mass[wave] = m_scan;
            lds.wave_count[wave] = c_scan;
        }
        __syncthreads();
        uint64_t m_at = above_mass + m_scan - m2;           // above this thread's bins
        uint32_t c_at = above_count + c_scan - c2;
        for (int w = 0; w < wave; ++w) {
            m_at += lds.wave_mass[w];
            c_at += lds.wave_count[w];
        }
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const uint64_t m = lds.mass[hi - j];
            const uint32_t c = lds.count[hi - j];
            const bool here = BY_MASS ? m_at < want && m_at + m >= want : c_at < want && (uint64_t)c_at + c >= want;
            if (here) {
                lds.found_bin = (uint32_t)(hi - j);
                lds.found_mass = m_at;
                lds.found_count = c_at;
            }
            m_at += m;
            c_at += c;
        }
        __syncthreads();
        prefix = (prefix << bits) | lds.found_bin;
        above_mass = lds.found_mass;
        above_count = lds.found_count;
    }
    __syncthreads();
    return prefix;
}

__global__ __launch_bounds__(kThreads) void k_sample(const float *__restrict__ scores, int64_t R,
                                                     const int64_t *__restrict__ seg, Settings set,
                                                     const float *__restrict__ u, int32_t *__restrict__ idx,
                                                     float *__restrict__ prob, int32_t *__restrict__ kept_out)
{
    __shared__ Lds lds;
    const int32_t p = blockIdx.x, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    int64_t lo = seg[p], hi = seg[p + 1];
    lo = lo < 0 ? 0 : lo > R ? R : lo;
    hi = hi < lo ? lo : hi > R ? R : hi;
    const float *s = scores + lo;
    const int32_t n = (int32_t)(hi - lo);
    u += (int64_t)p * set.n_draws;
    idx += (int64_t)p * set.n_draws;
    if (prob) prob += (int64_t)p * set.n_draws;

    // the best score, and how many take part
    uint32_t best_key = 0, alive = 0;
    for (int32_t i = threadIdx.x; i < n; i += kThreads) {
        const uint32_t k = key_of(s[i]);
        best_key = k > best_key ? k : best_key;
        alive += k != 0;
    }
#pragma unroll
    for (int l = 1; l < 64; l <<= 1) {
        const uint32_t o = (uint32_t)__shfl_xor((int)best_key, l);
        best_key = o > best_key ? o : best_key;
    }
    alive = wave_sum(alive);
    if (lane == 0) {
        lds.count[wave] = best_key;
        lds.wave_count[wave] = alive;
    }
    __syncthreads();
    alive = 0;
    for (int w = 0; w < kWaves; ++w) {
        best_key = lds.count[w] > best_key ? lds.count[w] : best_key;
        alive += lds.wave_count[w];
    }
    __syncthreads();
    if (alive == 0) {
        for (int32_t j = threadIdx.x; j < set.n_draws; j += kThreads) {
            idx[j] = -1;
            if (prob) prob[j] = 0.0f;
        }
        if (threadIdx.x == 0 && kept_out) kept_out[p] = 0;
        return;
    }
    const float best = score_of(best_key);
    const float T = set.how.temperature_of ? set.how.temperature_of[p] : set.how.temperature;
    const int32_t k_set = set.how.top_k_of ? set.how.top_k_of[p] : set.how.top_k;
    const float top_p = set.how.top_p_of ? set.how.top_p_of[p] : set.how.top_p;
    const float min_p = set.how.min_p_of ? set.how.min_p_of[p] : set.how.min_p;
    const bool cold = !(T > 0.0f);
    const float rate = cold ? 1.0f : (float)(1.4426950408889634 / (double)T);
    const uint32_t k = cold ? 1u : k_set > 0 ? (uint32_t)k_set : 0xffffffffu;

    // the prefix: keys above `cut`, and the first `ties` of those equal to it
    uint32_t cut = 0, ties = 0xffffffffu, above_count;
    uint64_t above_mass, mass;
    if (k < alive) {
        cut = descend<false>(s, n, best, rate, k, above_count, above_mass, lds);
        ties = k - above_count;
        mass = above_mass + ties * weight_of(score_of(cut), best, rate);
    } else if (top_p < 1.0f) {
        mass = 0;
        for (int32_t i = threadIdx.x; i < n; i += kThreads) mass += key_of(s[i]) ? weight_of(s[i], best, rate) : 0;
        mass = wave_sum(mass);
        if (lane == 0) lds.wave_mass[wave] = mass;
        __syncthreads();
        mass = 0;
        for (int w = 0; w < kWaves; ++w) mass += lds.wave_mass[w];
        __syncthreads();
    }
    if (top_p < 1.0f) {
        const double share = (double)mass * (double)(top_p > 0.0f ? top_p : 0.0f);
        uint64_t need = (uint64_t)ceil(share);
        need = need < 1 ? 1 : need;
        cut = descend<true>(s, n, best, rate, need, above_count, above_mass, lds);
        const uint64_t w = weight_of(score_of(cut), best, rate), t = (need - above_mass + w - 1) / w;
        ties = t < 0xffffffffull ? (uint32_t)t : 0xffffffffu;
    }
    const double floor_p = min_p > 0.0f ? (min_p < 1.0f ? (double)min_p : 1.0) * 4294967296.0 : 0.0;
    uint64_t least = (uint64_t)ceil(floor_p);
    least = least < 1 ? 1 : least;

    // A wave has a range of consecutive candidates; last: the index of the last
    // tied one that is kept.
    const int32_t range = (n + kThreads - 1) / kThreads * 64, w_lo = wave * range < n ? wave * range : n,
                  w_hi = w_lo + range < n ? w_lo + range : n;
    int32_t last = n;
    if (ties != 0xffffffffu) {
        uint32_t c = 0;
        for (int32_t i = w_lo + lane; i < w_hi; i += 64) c += key_of(s[i]) == cut;
        c = wave_sum(c);
        if (lane == 0) lds.wave_count[wave] = c;
        if (threadIdx.x == 0) lds.found_bin = (uint32_t)n;
        __syncthreads();
        uint32_t before = 0;
        for (int w = 0; w < wave; ++w) before += lds.wave_count[w];
        if (before < ties && before + c >= ties) {
            for (int32_t i0 = w_lo; i0 < w_hi; i0 += 64) {
                const int32_t i = i0 + lane;
                const uint64_t tied = __ballot(i < w_hi && key_of(s[i < w_hi ? i : i0]) == cut);
                const uint32_t here = (uint32_t)__popcll(tied);
                if (before + here >= ties) {
                    uint64_t left = tied;
                    for (uint32_t j = 1; j < ties - before; ++j) left &= left - 1;
                    if (lane == 0) lds.found_bin = (uint32_t)(i0 + __builtin_ctzll(left));
                    break;
                }
                before += here;
            }
        }
        __syncthreads();
        last = (int32_t)lds.found_bin;
        __syncthreads();
    }
    auto kept_weight = [&](int32_t i) -> uint64_t {
        const uint32_t key = key_of(s[i]);
        if (key == 0 || key < cut || (key == cut && i > last)) return 0;
        const uint64_t w = weight_of(s[i], best, rate);
        return w >= least ? w : 0;
    };
    uint64_t sum = 0;
    uint32_t kept = 0;
    for (int32_t i = w_lo + lane; i < w_hi; i += 64) {
        const uint64_t w = kept_weight(i);
        sum += w;
        kept += w != 0;
    }
    sum = wave_sum(sum);
    kept = wave_sum(kept);
    if (lane == 0) {
        lds.wave_mass[wave] = sum;
        lds.wave_count[wave] = kept;
    }
    __syncthreads();
    uint64_t total = 0;
    kept = 0;
    for (int w = 0; w < kWaves; ++w) {
        total += lds.wave_mass[w];
        kept += lds.wave_count[w];
    }
    if (threadIdx.x == 0 && kept_out) kept_out[p] = (int32_t)kept;
    for (int32_t j = wave; j < set.n_draws; j += kWaves) {
        const float v = floorf(u[j] * 16777216.0f);
        const uint32_t u24 = v > 0.0f ? (v < 16777215.0f ? (uint32_t)v : 16777215u) : 0u;
        uint64_t r = (total >> 24) * u24 + (((total & 0xffffffull) * u24) >> 24);
        int w = 0;
        while (w < kWaves - 1 && r >= lds.wave_mass[w]) r -= lds.wave_mass[w++];
        const int32_t b = w * range, e = b + range < n ? b + range : n;
        for (int32_t i0 = b; i0 < e; i0 += 64) {
            const uint64_t mine = i0 + lane < e ? kept_weight(i0 + lane) : 0, scan = wave_scan(mine, lane);
            const uint64_t over = __ballot(scan > r);
            if (over) {
                const int l = __builtin_ctzll(over);
                if (lane == l) {
                    idx[j] = i0 + l;
                    if (prob) prob[j] = (float)((double)mine / (double)total);
                }
                break;
            }
            r -= __shfl(scan, 63);
        }
    }
}

}  // namespace

size_t sample_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }

hipError_t launch_sample(const float *scores, int64_t R, const int64_t *seg, int32_t P, const hwsel_sampling_t &how,
                         const float *u, int32_t n_draws, int32_t *idx, float *prob, int32_t *kept, void *, hipStream_t s)
{
    each_span(P, [&](int32_t p0, int32_t n) {
        hwsel_sampling_t h = how;
        if (h.temperature_of) h.temperature_of += p0;
        if (h.top_k_of) h.top_k_of += p0;
        if (h.top_p_of) h.top_p_of += p0;
        if (h.min_p_of) h.min_p_of += p0;
        const int64_t o = (int64_t)p0 * n_draws;
        hipLaunchKernelGGL(k_sample, dim3(n), dim3(kThreads), 0, s, scores, R, seg + p0, Settings{h, n_draws}, u + o, idx + o,
                           prob ? prob + o : nullptr, kept ? kept + p0 : nullptr);
    });
    return hipGetLastError();
}

}  // namespace hwsel
