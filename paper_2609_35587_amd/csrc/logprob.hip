// Log probabilities of given candidates with entropy and best alternatives, and
// their gradient with respect to the scores.
//   t = (s - best) / T;  Z = sum exp t;  log p = t - log Z;  H = log Z - sum(exp(t) t) / Z
// Scores are read once, with the running best score and the sums that go by it.
#include "internal.hpp"

namespace hwsel {
namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNone = -__builtin_inff();

// A problem's rows, within [0, R], and its temperature.
struct Problem {
    const float *s;
    int64_t at;
    int32_t n;
    float T;
    bool cold;                                              // the first best candidate alone
};

__device__ __forceinline__ int64_t within(int64_t v, int64_t R) { return v < 0 ? 0 : v > R ? R : v; }

__device__ __forceinline__ Problem problem_of(const float *scores, int64_t R, const int64_t *seg, int32_t p, float temperature,
                                              const float *temperature_of)
{
    const int64_t a = within(seg[p], R), b = within(seg[p + 1], R);
    const float T = temperature_of ? temperature_of[p] : temperature;
    return {scores + a, a, (int32_t)(b > a ? b - a : 0), T, !(T > 0.0f)};
}

// NaN takes no part, as -inf does.
__device__ __forceinline__ float taking_part(float s) { return s > kNone ? s : kNone; }

// log2 of a candidate's weight against the best one's; -200 (weight 0) for what
// has none: -inf against anything, and NaN, as of 0 times infinity.
__device__ __forceinline__ float weight_exponent(float s, float best, float rate) { return fmaxf((s - best) * rate, -200.0f); }

// Some candidates: the best score, how many equal it, the sum of the others'
// weights 2^t and of 2^t t.  Weights of the best are counted and not added, so
// that log Z = log1p of the others keeps its digits where one has nearly all.
struct Mass {
    float best, equal, less, weighted;
};

// The sums as they are once another score is the best.
__device__ __forceinline__ Mass lowered(const Mass &m, float best, float rate)
{
    const float t = weight_exponent(m.best, best, rate), e = __builtin_amdgcn_exp2f(t), all = m.equal + m.less;
    return {best, 0.0f, e * all, e > 0.0f ? e * (m.weighted + t * all) : 0.0f};
}

__device__ __forceinline__ Mass joined(const Mass &a, const Mass &b, float rate)
{
    const Mass x = a.best < b.best ? lowered(a, b.best, rate) : a, y = b.best < a.best ? lowered(b, a.best, rate) : b;
    return {x.best, x.equal + y.equal, x.less + y.less, x.weighted + y.weighted};
}

template <int N>
__device__ __forceinline__ void take(Mass &m, const float (&v)[N], float rate)
{
    float top = v[0];
#pragma unroll
    for (int i = 1; i < N; ++i) top = fmaxf(top, v[i]);
    if (top > m.best) m = lowered(m, top, rate);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = weight_exponent(v[i], m.best, rate), e = __builtin_amdgcn_exp2f(t);
        const bool is_best = v[i] == m.best;
        m.equal += is_best ? 1.0f : 0.0f;
        m.less += is_best ? 0.0f : e;
        m.weighted += is_best ? 0.0f : e * t;
    }
}

__device__ __forceinline__ Mass lane_of(const Mass &m, int l)
{
    return {__shfl(m.best, l), __shfl(m.equal, l), __shfl(m.less, l), __shfl(m.weighted, l)};
}

__device__ __forceinline__ Mass wave_mass(Mass m, float rate)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const Mass o = {__shfl_xor(m.best, d), __shfl_xor(m.equal, d), __shfl_xor(m.less, d), __shfl_xor(m.weighted, d)};
        m = joined(m, o, rate);
    }
    return lane_of(m, 0);
}

// What log probabilities are made from.
struct Norm {
    float best, log_mass, entropy;
    int32_t first;                                          // of a cold problem: the candidate (else -1)
};

__device__ __forceinline__ Norm norm_of(const Mass &m, const Problem &q, int32_t first)
{
    if (!(m.best > kNone)) return {kNone, kNone, 0.0f, -1};
    if (q.cold) return {m.best, 0.0f, 0.0f, first};
    const float log_mass = log1pf((m.equal - 1.0f) + m.less);
    return {m.best, log_mass, log_mass - m.weighted * kLn2 / (m.equal + m.less), -1};
}

__device__ __forceinline__ float log_probability(const Problem &q, const Norm &z, int32_t j, float s)
{
    if (!(s > kNone)) return kNone;
    if (q.cold) return j == z.first ? 0.0f : kNone;
    return (s == z.best ? 0.0f : (s - z.best) / q.T) - z.log_mass;
}

__device__ __forceinline__ uint64_t key_of(float s, int32_t j)   // 0: takes no part
{
    return s > kNone ? ((uint64_t)order_key(s + 0.0f) << 32) | (0xffffffffu - (uint32_t)j) : 0ull;
}

constexpr int kThreads = 256;

template <int NT>
__device__ __forceinline__ uint64_t block_max(uint64_t v, uint64_t *sh)
{
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) {
        const uint64_t o = __shfl_xor((unsigned long long)v, d);
        v = o > v ? o : v;
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
    __syncthreads();
    for (int w = 0; w < NT / 64; ++w) v = sh[w] > v ? sh[w] : v;
    return v;
}

struct LogprobArgs {
    const float *scores;
    int64_t R;
    const int64_t *seg;
    float temperature;
    const float *temperature_of;
    const int32_t *picks;
    int32_t n_picks, top;
    float *logp, *entropy, *norm;
    int32_t *top_idx;
    float *top_logp;
    int32_t p0;
};

// A workgroup has a problem.
__global__ __launch_bounds__(kThreads) void k_logprob(LogprobArgs a)
{
    __shared__ Mass part[kThreads / 64];
    __shared__ uint64_t sh[kThreads / 64];
    const int32_t p = a.p0 + (int32_t)blockIdx.x;
    const Problem q = problem_of(a.scores, a.R, a.seg, p, a.temperature, a.temperature_of);
    const float rate = kLog2e / q.T;
    Mass m = {kNone, 0.0f, 0.0f, 0.0f};
    for (int64_t i = threadIdx.x; i < q.n; i += kThreads) {
        const float v[1] = {taking_part(q.s[i])};
        take(m, v, rate);
    }
    m = wave_mass(m, rate);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    m = part[0];
    for (int w = 1; w < kThreads / 64; ++w) m = joined(m, part[w], rate);
    int32_t first = -1;
    auto best_below = [&](uint64_t limit) {
        uint64_t k = 0;
        for (int64_t i = threadIdx.x; i < q.n; i += kThreads) {
            const uint64_t v = key_of(q.s[i], (int32_t)i);
            k = v < limit && v > k ? v : k;
        }
        return block_max<kThreads>(k, sh);
    };
    if (q.cold) first = (int32_t)(0xffffffffu - (uint32_t)best_below(~0ull));
    const Norm z = norm_of(m, q, first);
    if (threadIdx.x == 0) {
        if (a.entropy) a.entropy[p] = z.entropy;
        if (a.norm) {
            a.norm[2 * (int64_t)p] = z.best;
            a.norm[2 * (int64_t)p + 1] = z.log_mass;
        }
    }
    for (int64_t i = threadIdx.x; i < a.n_picks; i += kThreads) {
        const int32_t j = a.picks[(int64_t)p * a.n_picks + i];
        a.logp[(int64_t)p * a.n_picks + i] = j < 0 || j >= q.n ? 0.0f : log_probability(q, z, j, q.s[j]);
    }
    uint64_t limit = ~0ull;
    for (int32_t r = 0; r < a.top; ++r) {
        const uint64_t k = limit ? best_below(limit) : 0ull;
        limit = k;
        if (threadIdx.x == 0) {
            const int32_t j = (int32_t)(0xffffffffu - (uint32_t)k);
            const float lp = k ? log_probability(q, z, j, q.s[j]) : kNone;
            a.top_idx[(int64_t)p * a.top + r] = lp > kNone ? j : -1;
            a.top_logp[(int64_t)p * a.top + r] = lp;
        }
    }
}

struct GradientArgs {
    const float *scores;
    int64_t R;
    const int64_t *seg;
    int32_t P, p0;
    float temperature;
    const float *temperature_of, *norm;
    const int32_t *picks;
    int32_t n_picks;
    const float *d_logp, *entropy, *d_entropy;
    float *d_scores;
};

// A pick that counts: inside the problem, with a probability.
__device__ __forceinline__ bool counts(const Problem &q, const Norm &z, int32_t j)
{
    return j >= 0 && j < q.n && log_probability(q, z, j, q.s[j]) > kNone;
}

constexpr int kPart = 4096;                                 // candidates whose picks are summed at once

// A workgroup has a problem, a part of its candidates at a time: the picks'
// gradients are added in fixed point in LDS, by a unit of 2^-62 n of the largest,
// so their order does not matter.
__global__ __launch_bounds__(kThreads) void k_logprob_gradient(GradientArgs a)
{
    __shared__ unsigned long long acc[kPart];
    __shared__ unsigned long long total;
    __shared__ uint32_t largest;
    const int32_t p = a.p0 + (int32_t)blockIdx.x;
    // rows of no problem: this workgroup's share
    const int64_t before = within(a.seg[0], a.R), behind = within(a.seg[a.P], a.R);
    for (int64_t i = (int64_t)p * kThreads + threadIdx.x; i < before; i += (int64_t)a.P * kThreads) a.d_scores[i] = 0.0f;
    for (int64_t i = behind + (int64_t)p * kThreads + threadIdx.x; i < a.R; i += (int64_t)a.P * kThreads) a.d_scores[i] = 0.0f;

    const Problem q = problem_of(a.scores, a.R, a.seg, p, a.temperature, a.temperature_of);
    const Norm z = {a.norm[2 * (int64_t)p], a.norm[2 * (int64_t)p + 1], a.entropy ? a.entropy[p] : 0.0f, -1};
    float *d = a.d_scores + q.at;
    if (q.cold) {
        for (int64_t i = threadIdx.x; i < q.n; i += kThreads) d[i] = 0.0f;
        return;
    }
    const int32_t *picks = a.picks + (int64_t)p * a.n_picks;
    const float *dl = a.d_logp + (int64_t)p * a.n_picks;
    if (threadIdx.x == 0) {
        largest = 0;
        total = 0;
    }
    __syncthreads();
    for (int64_t i = threadIdx.x; i < a.n_picks; i += kThreads)
        if (counts(q, z, picks[i])) atomicMax(&largest, __float_as_uint(dl[i]) & 0x7fffffffu);
    __syncthreads();
    // unit 2^e: the largest is below 2^x, n of them below 2^(62 + e)
    const uint32_t most = largest;
    const bool fine = most < 0x7f800000u;
    const int bits = 32 - __builtin_clz((uint32_t)a.n_picks | 1u);
    const int e = (int)(most >> 23) - 126 + bits - 62;
    auto fixed = [&](float v) { return (unsigned long long)(long long)__builtin_rint(__builtin_ldexp((double)v, -e)); };
    auto value = [&](unsigned long long v) { return (float)__builtin_ldexp((double)(long long)v, e); };
    if (fine)
        for (int64_t i = threadIdx.x; i < a.n_picks; i += kThreads)
            if (counts(q, z, picks[i])) atomicAdd(&total, fixed(dl[i]));
    __syncthreads();
    const float S = fine ? value(total) : __uint_as_float(most);
    const float de = a.d_entropy ? a.d_entropy[p] : 0.0f;
    for (int64_t part = 0; part < q.n; part += kPart) {
        const int32_t n = (int32_t)(q.n - part < kPart ? q.n - part : kPart);
        __syncthreads();
        for (int32_t i = threadIdx.x; i < n; i += kThreads) acc[i] = 0;
        __syncthreads();
        if (fine)
            for (int64_t i = threadIdx.x; i < a.n_picks; i += kThreads) {
                const int64_t j = picks[i] - part;
                if (j >= 0 && j < n && counts(q, z, picks[i])) atomicAdd(&acc[j], fixed(dl[i]));
            }
        __syncthreads();
        for (int32_t i = threadIdx.x; i < n; i += kThreads) {
            const float s = q.s[part + i], lp = log_probability(q, z, (int32_t)(part + i), s);
            const float pr = __builtin_amdgcn_exp2f(lp * kLog2e), g = value(acc[i]);
            // g (1 - p) without the difference where p is nearly 1
            const float own = g != 0.0f ? -g * expm1f(lp) : 0.0f;
            const float v = own - pr * (S - g) - de * (pr > 0.0f ? pr * (lp + z.entropy) : 0.0f);
            d[part + i] = lp > kNone ? v / q.T : 0.0f;
        }
    }
}

}  // namespace

size_t logprob_workspace_bytes(int64_t, int32_t, int32_t) { return 0; }

hipError_t launch_logprob(const float *scores, int64_t R, const int64_t *seg, int32_t P, float temperature, const float *temperature_of,
                          const int32_t *picks, int32_t n_picks, int32_t top, float *logp, float *entropy, float *norm, int32_t *top_idx,
                          float *top_logp, void *, hipStream_t s)
{
    LogprobArgs a{scores, R, seg, temperature, temperature_of, picks, n_picks, top, logp, entropy, norm, top_idx, top_logp, 0};
    each_span(P, [&](int32_t p0, int32_t n) {
        a.p0 = p0;
        hipLaunchKernelGGL(k_logprob, dim3(n), dim3(kThreads), 0, s, a);
    });
    return hipGetLastError();
}

hipError_t launch_logprob_gradient(const float *scores, int64_t R, const int64_t *seg, int32_t P, float temperature,
                                   const float *temperature_of, const float *norm, const int32_t *picks, int32_t n_picks,
                                   const float *d_logp, const float *entropy, const float *d_entropy, float *d_scores, hipStream_t s)
{
    GradientArgs a{scores, R, seg, P, 0, temperature, temperature_of, norm, picks, n_picks, d_logp, entropy, d_entropy, d_scores};
    each_span(P, [&](int32_t p0, int32_t n) {
        a.p0 = p0;
        hipLaunchKernelGGL(k_logprob_gradient, dim3(n), dim3(kThreads), 0, s, a);
    });
    return hipGetLastError();
}

}  // namespace hwsel
