// Log probabilities of given candidates with entropy and best alternatives, and
// their gradient with respect to the scores.
//   t = (s - best) / T;  Z = sum exp t;  log p = t - log Z;  H = log Z - sum(exp(t) t) / Z
// Scores are read once, with the running best score and the sums that go by it; for alternatives once more where
// a workgroup's registers do not hold them.
//
// Bound by latency where problems are few or short (a launch, the offsets, the scores, barriers: 100 problems of 700 3.9 us,
// launches in a row), by memory where they are long: 256 x 65,536 scores, 67 MB, 15 us (4.5 TB/s), their gradient 23.5 us (5.7 TB/s read and written).
#include "topk.hpp"

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

typedef float f32x4u_t __attribute__((ext_vector_type(4), aligned(4)));   // four scores from any segment's start

// Scores i .. i + 3 of n, -inf past the last.
__device__ __forceinline__ f32x4u_t load4(const float *s, int32_t i, int32_t n)
{
    if (i + 4 <= n) return *reinterpret_cast<const f32x4u_t *>(s + i);
    f32x4u_t w;
#pragma unroll
    for (int k = 0; k < 4; ++k) w[k] = i + k < n ? s[i + k] : kNone;
    return w;
}

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

// N more scores.  NaN takes no part: it is above nothing, equals nothing and its weight is 0.
template <int N>
__device__ __forceinline__ void take(Mass &m, const float (&v)[N], float rate)
{
    float top = m.best;
#pragma unroll
    for (int i = 0; i < N; ++i) top = v[i] > top ? v[i] : top;
    if (top > m.best) m = lowered(m, top, rate);
    uint32_t equal = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // (of the best itself t is 0, or -200 where it is +inf: it adds nothing to the third sum)
        const float t = weight_exponent(v[i], m.best, rate), e = __builtin_amdgcn_exp2f(t);
        const bool is_best = v[i] == m.best;
        equal += is_best;
        m.less += is_best ? 0.0f : e;
        m.weighted = __builtin_fmaf(e, t, m.weighted);
    }
    m.equal += (float)equal;
}

template <int CTRL, int ROW_MASK>
__device__ __forceinline__ float dpp_max(float v)
{
    return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(__float_as_int(kNone), __float_as_int(v), CTRL, ROW_MASK, 0xf, false)));
}

__device__ __forceinline__ float wave_max(float v)
{
    v = dpp_max<0x111, 0xf>(v);
    v = dpp_max<0x112, 0xf>(v);
    v = dpp_max<0x114, 0xf>(v);
    v = dpp_max<0x118, 0xf>(v);
    v = dpp_max<0x142, 0xa>(v);
    v = dpp_max<0x143, 0xc>(v);
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// The lanes' candidates together: first the best score, then sums that go by it.
__device__ __forceinline__ Mass wave_mass(Mass m, float rate)
{
    const float top = wave_max(m.best);
    if (m.best < top) m = lowered(m, top, rate);
    float v[3] = {m.equal, m.less, m.weighted};
    group_totals<64>(v);
    auto last = [](float x) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63)); };
    return {top, last(v[0]), last(v[1]), last(v[2])};
}

constexpr Mass kNothing = {kNone, 0.0f, 0.0f, 0.0f};

// A workgroup's candidates together, in every thread (part: not in use).
template <int NT>
__device__ __forceinline__ Mass block_mass(Mass m, float rate, Mass *part)
{
    const int lane = threadIdx.x & 63;
    m = wave_mass(m, rate);
    if (lane == 0) part[threadIdx.x >> 6] = m;
    __syncthreads();
    return wave_mass(lane < NT / 64 ? part[lane] : kNothing, rate);
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
    const float t = s == z.best ? 0.0f : (s - z.best) / q.T;
    return t > kNone ? t - z.log_mass : kNone;              // (NaN: a finite score below +inf at T = inf)
}

// Waits for a group of THREADS: a wave's own accesses of LDS (GLOBAL: and of memory), or a workgroup's.
template <int THREADS, bool GLOBAL = false>
__device__ __forceinline__ void group_barrier()
{
    if constexpr (THREADS > 64) {
        if constexpr (GLOBAL) __syncthreads();
        else lds_barrier();
    } else {
        if constexpr (GLOBAL) __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
        else __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
    }
}

constexpr int kThreads = 256;

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
    int32_t P, p0;
};

__device__ __forceinline__ Problem problem_of(const LogprobArgs &a, int32_t p)
{
    return problem_of(a.scores, a.R, a.seg, p, a.temperature, a.temperature_of);
}

// A thread's first pick with its score, on the way while the scores are read.
struct Pick {
    int32_t j;
    float s;
};

__device__ __forceinline__ Pick pick_of(const LogprobArgs &a, const Problem &q, int32_t p, int32_t i)
{
    Pick k = {-1, 0.0f};
    if (i < a.n_picks) k.j = a.picks[(int64_t)p * a.n_picks + i];
    if (k.j >= 0 && k.j < q.n) k.s = q.s[k.j];
    else k.j = -1;
    return k;
}

// What N threads (this one the t-th) write of a problem: its norm, its picks; keys: its best candidates, descending, 0 for none.
template <int N>
__device__ __forceinline__ void write_problem(const LogprobArgs &a, const Problem &q, int32_t p, const Norm &z, int t, Pick pick, const uint64_t *keys)
{
    if (t == 0) {
        if (a.entropy) a.entropy[p] = z.entropy;
        if (a.norm) {
            a.norm[2 * (int64_t)p] = z.best;
            a.norm[2 * (int64_t)p + 1] = z.log_mass;
        }
    }
    for (uint32_t i = t; i < (uint32_t)a.n_picks; i += N) {
        if (i >= N) pick = pick_of(a, q, p, (int32_t)i);
        a.logp[(int64_t)p * a.n_picks + i] = pick.j < 0 ? 0.0f : log_probability(q, z, pick.j, pick.s);
    }
    for (int32_t r = t; r < a.top; r += N) {
        const uint64_t k = keys[r];
        const int32_t j = (int32_t)(0xffffffffu - (uint32_t)k);
        const float s = desc_value((uint32_t)(k >> 32));    // (NaN for key 0)
        const float lp = log_probability(q, z, j, s);
        a.top_idx[(int64_t)p * a.top + r] = lp > kNone ? j : -1;
        a.top_logp[(int64_t)p * a.top + r] = lp;
    }
}

// n scores by a workgroup, 16 a thread and step; the last step's stay in w.
template <int NT>
__device__ __forceinline__ Mass take_all(const float *s, int32_t n, float rate, f32x4u_t (&w)[4])
{
    Mass m = kNothing;
    constexpr int kStep = 16 * NT;
    for (int32_t at = 0; at < n; at += kStep) {
        const int32_t left = n - at;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = load4(s + at, (i * NT + (int)threadIdx.x) * 4, left);
        float v[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = w[i >> 2][i & 3];
        take(m, v, rate);
    }
    return m;
}

template <int NT>
struct Lds {
    TopkLds<NT> topk;
    uint64_t keys[64];
    Mass part[NT / 64];
    uint32_t best[NT / 64][64];                             // each thread's best score, as ordered bits
    int32_t first, n_list;
};

constexpr uint32_t kLeastBits = 0x00800000u;                // of the least finite score; below them are -inf and NaN

// The best `top` of n scores, read once more unless one step (w) has them: a score is listed if it is not below what the best scores of `top`
// threads reach (of 256 threads, or of 64 groups of them; more are taken together), and the listed ones, few more
// than `top`, are ranked by counting the larger.  False, and nothing written, if they do not fit the list.
// (By tiles, each score with its key against a running bound, the sums on the way: 600 of up to 8,192 scores, 10 of
// each, 13.7 us, 10.1 so; 256 of 65,536 with 64 of each 77 and 24; 256 of 131,072, 134 MB, 90 and 44.  Where the best are the same
// few values over and over they do not fit and the tiles follow: of twelve values 600 x 8,192 with 10 20 us, 9 of distinct ones; 256 x
// 65,536 with 64 46 and 26.)
template <int NT>
__device__ __forceinline__ bool list_best(const float *s, int32_t n, int32_t top, Lds<NT> &lds, f32x4u_t (&w)[4])
{
    const int lane = threadIdx.x & 63;
    uint32_t best[4] = {}, bits = 0;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) best[w & 3] = lds.best[w][lane] > best[w & 3] ? lds.best[w][lane] : best[w & 3];
    const bool few = top <= 16;                             // 64 are enough: a quarter of the comparisons
    if (few) {
#pragma unroll
        for (int w = 1; w < 4; ++w) best[0] = best[w] > best[0] ? best[w] : best[0];
    }
    for (int b = 31; b >= 0; --b) {                         // (every wave for itself)
        int32_t c = (int32_t)__popcll(__ballot(best[0] >= (bits | 1u << b)));
        if (!few) {
#pragma unroll
            for (int w = 1; w < 4; ++w) c += (int32_t)__popcll(__ballot(best[w] >= (bits | 1u << b)));
        }
        if (c >= top) bits |= 1u << b;
        if (c == top) break;
    }
    const float least = bits > kLeastBits ? desc_value(bits) : -3.4028235e38f;
    constexpr int kStep = 16 * NT;
    for (int32_t at = 0; at < n; at += kStep) {
        if (n > kStep) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = load4(s + at, (i * NT + (int)threadIdx.x) * 4, n - at);
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const float v = w[i >> 2][i & 3];
            const bool in = v >= least;
            const uint64_t take = __ballot(in);
            if (take == 0) continue;
            int32_t to = 0;
            if (lane == 0) to = atomicAdd(&lds.n_list, __popcll(take));
            to = __builtin_amdgcn_readfirstlane(to) +
                 (int32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(take >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)take, 0u));
            const uint32_t j = (uint32_t)(at + ((i >> 2) * NT + (int)threadIdx.x) * 4 + (i & 3));
            if (in && to < kList) lds.topk.cand[to] = ((uint64_t)order_key(v + 0.0f) << 32) | (0xffffffffu - j);
        }
    }
    __syncthreads();
    const int32_t m = lds.n_list;
    if (m > kList) return false;
    for (int32_t i = threadIdx.x; i < m; i += NT) {
        const uint64_t own = lds.topk.cand[i];
        int32_t rank = 0;
#pragma unroll 8
        for (int32_t e = 0; e < m; ++e) rank += lds.topk.cand[e] > own;
        if (rank < top) lds.keys[rank] = own;
    }
    __syncthreads();
    return true;
}

// The sums and best candidates of n scores by a workgroup; first: of a cold problem its best candidate (else -1).
template <int NT, int TILE, bool TOP>
__device__ __forceinline__ Mass block_scores(const float *s, int32_t n, int32_t top, bool cold, float rate, Lds<NT> &lds, int32_t &first)
{
    first = -1;
    f32x4u_t w[4];
    if constexpr (TOP) {
        Mass m = take_all<NT>(s, n, rate, w);
        lds.best[threadIdx.x >> 6][threadIdx.x & 63] = m.best > kNone ? order_key(m.best + 0.0f) : 0u;
        if (threadIdx.x < 64) lds.keys[threadIdx.x] = 0;
        if (threadIdx.x == 0) lds.n_list = 0;
        m = block_mass<NT>(m, rate, lds.part);              // (its barrier)
        if (!list_best<NT>(s, n, top, lds, w)) {               // many scores are one: by tiles
            __syncthreads();
            topk_tiles<NT, TILE>(s, n, top, lds.topk, [&](int32_t j, uint64_t key) { lds.keys[j] = key; });
            __syncthreads();
        }
        if (cold) first = (int32_t)(0xffffffffu - (uint32_t)lds.keys[0]);
        return m;
    } else {
        const Mass m = block_mass<NT>(take_all<NT>(s, n, rate, w), rate, lds.part);
        if (cold) {
            if (threadIdx.x == 0) lds.first = 0x7fffffff;
            __syncthreads();
            for (int32_t j = threadIdx.x; j < n; j += NT)
                if (s[j] == m.best) {
                    atomicMin(&lds.first, j);
                    break;
                }
            __syncthreads();
            first = lds.first;
        }
        return m;
    }
}

// A workgroup has a problem.
template <int NT, int TILE, bool TOP>
__device__ __forceinline__ void block_problem(const LogprobArgs &a, int32_t p, Lds<NT> &lds)
{
    const Problem q = problem_of(a, p);
    const Pick pick = pick_of(a, q, p, threadIdx.x);
    const float rate = kLog2e / q.T;
    int32_t first;
    const Mass m = block_scores<NT, TILE, TOP>(q.s, q.n, a.top, q.cold, rate, lds, first);
    write_problem<NT>(a, q, p, norm_of(m, q, first), threadIdx.x, pick, lds.keys);
}

template <int NT, int TILE, bool TOP>
__global__ __launch_bounds__(NT) void k_logprob(LogprobArgs a)
{
    __shared__ Lds<NT> lds;
    block_problem<NT, TILE, TOP>(a, a.p0 + (int32_t)blockIdx.x, lds);
}

// A wave has a problem of up to 64 EACH candidates, its scores in registers.  A lone wave takes some 7 cycles an
// instruction, so what it does goes by how many there are.
constexpr int kSmall = 1024, kFew = 8;                      // kFew: alternatives for which lanes' best give a bound
constexpr int kWaveList = 16 * kFew;

template <int EACH, bool TOP>
__device__ __forceinline__ void wave_problem(const LogprobArgs &a, const Problem &q, int32_t p, int lane, uint64_t *list, uint64_t *keys)
{
    const Pick pick = pick_of(a, q, p, lane);
    const float rate = kLog2e / q.T;
    float v[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) v[e] = lane + 64 * e < q.n ? q.s[lane + 64 * e] : kNone;
    Mass m = kNothing;
    take(m, v, rate);
    m = wave_mass(m, rate);
    int32_t first = -1;
    const int32_t rounds = TOP ? a.top : q.cold ? 1 : 0;
    if (rounds > 0) {
        // What the best are not below: bits hi, of those that equal them ~index lo.  Found bit by bit: for few, what
        // that many lanes' best reach; else what that many candidates do.  It is good once no more than that many do.
        uint32_t bits[EACH], best = 0, at = 0;
#pragma unroll
        for (int e = EACH - 1; e >= 0; --e) {
            bits[e] = v[e] > kNone ? order_key(v[e] + 0.0f) : 0u;
            at = bits[e] >= best ? (uint32_t)(lane + 64 * e) : at;
            best = bits[e] >= best ? bits[e] : best;
        }
        const bool few = rounds <= kFew;
        auto reach = [&](uint32_t h, uint32_t l) {  // how many are not below (h, l)
            if (few) return (int32_t)__popcll(__ballot(best > h || (best == h && 1023u - at >= l)));
            int32_t c = 0;
#pragma unroll
            for (int e = 0; e < EACH; ++e) c += __popcll(__ballot(bits[e] > h || (bits[e] == h && 1023u - (uint32_t)(lane + 64 * e) >= l)));
            return c;
        };
        uint32_t hi = 0, lo = 0;
        bool open = true;
        for (int b = 31; b >= 0 && open; --b) {
            const int32_t c = reach(hi | 1u << b, 0u);
            if (c >= rounds) hi |= 1u << b;
            open = c != rounds;
        }
        for (int b = 9; b >= 0 && open; --b) {
            const int32_t c = reach(hi, lo | 1u << b);
            if (c >= rounds) lo |= 1u << b;
            open = c != rounds;
        }
        hi = hi > 1u ? hi : 1u;                     // (0: takes no part)
        int32_t n_list = 0;
#pragma unroll
        for (int e = 0; e < EACH; ++e) {
            const uint32_t j = (uint32_t)(lane + 64 * e);
            const bool in = bits[e] > hi || (bits[e] == hi && 1023u - j >= lo);
            const uint64_t take = __ballot(in);
            if (in)
                list[n_list + (int32_t)__builtin_amdgcn_mbcnt_hi((uint32_t)(take >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)take, 0u))] =
                    ((uint64_t)bits[e] << 32) | (0xffffffffu - j);
            n_list += __popcll(take);
        }
        keys[lane] = 0;
        group_barrier<64>();
        for (int32_t i = lane; i < n_list; i += 64) {
            const uint64_t own = list[i];
            int32_t rank = 0;
#pragma unroll 4
            for (int32_t e = 0; e < n_list; ++e) rank += list[e] > own;
            if (rank < rounds) keys[rank] = own;
        }
        group_barrier<64>();
        first = (int32_t)(0xffffffffu - (uint32_t)keys[0]);
    }
    write_problem<64>(a, q, p, norm_of(m, q, q.cold ? first : -1), lane, pick, keys);
}

// Longer ones among them follow, by the whole workgroup.
template <bool TOP>
__global__ __launch_bounds__(kThreads) void k_logprob_waves(LogprobArgs a)
{
    constexpr int kWaves = kThreads / 64;
    __shared__ Lds<kThreads> lds;
    __shared__ uint64_t keys[kWaves][64], list[kWaves][kWaveList];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t p0 = a.p0 + (int32_t)blockIdx.x * kWaves, p = p0 + wave;
    if (p < a.P) {
        const Problem q = problem_of(a, p);
        if (q.n <= 64) wave_problem<1, TOP>(a, q, p, lane, list[wave], keys[wave]);
        else if (q.n <= 256) wave_problem<4, TOP>(a, q, p, lane, list[wave], keys[wave]);
        else if (q.n <= 512) wave_problem<8, TOP>(a, q, p, lane, list[wave], keys[wave]);
        else if (q.n <= kSmall) wave_problem<16, TOP>(a, q, p, lane, list[wave], keys[wave]);
    }
    for (int32_t i = 0; i < kWaves && p0 + i < a.P; ++i) {
        if (problem_of(a, p0 + i).n <= kSmall) continue;     // (one answer for the workgroup)
        block_problem<kThreads, 2048, TOP>(a, p0 + i, lds);
        __syncthreads();
    }
}

// Few long problems: each goes in parts to workgroups of its own, whose sums and
// best candidates one workgroup joins.
constexpr int kWide = 512, kWideTile = 4096;

struct Part {
    Mass m;
    int32_t first;
};

struct Parts {
    Part *part;                                             // [P][n]
    uint64_t *keys;                                         // [P][n][top]
    int32_t n;
};

template <bool TOP>
__global__ __launch_bounds__(kWide) void k_logprob_parts(LogprobArgs a, Parts to)
{
    __shared__ Lds<kWide> lds;
    const int32_t p = blockIdx.y, g = blockIdx.x;
    const Problem q = problem_of(a, p);
    const int32_t each = (q.n + to.n - 1) / to.n, from = g * (int64_t)each < q.n ? g * each : q.n, n = q.n - from < each ? q.n - from : each;
    int32_t first;
    const Mass m = block_scores<kWide, kWideTile, TOP>(q.s + from, n, a.top, q.cold, kLog2e / q.T, lds, first);
    const int64_t at = (int64_t)p * to.n + g;
    if (threadIdx.x == 0) to.part[at] = {m, first + from};
    if constexpr (TOP)
        for (int32_t r = threadIdx.x; r < a.top; r += kWide) to.keys[at * a.top + r] = lds.keys[r] ? lds.keys[r] - (uint32_t)from : 0ull;
}

// The most parts of a problem, and of their candidates (each part's `top`).
constexpr int kMostParts = 256, kMostKeys = 4096;

// One load of each thread's share of the parts and their candidates, all on their way at once; then the
// candidates that can be among the best are ranked by counting the larger ones.
template <bool TOP>
__global__ __launch_bounds__(kWide) void k_logprob_join(LogprobArgs a, Parts from)
{
    constexpr int kKeys = kMostKeys / kWide, kEach = kMostParts / 64;
    __shared__ uint64_t list[TOP ? kMostKeys : 1], keys[64];
    __shared__ int32_t n_list;
    const int32_t p = blockIdx.x, top = a.top;
    const int lane = threadIdx.x & 63;
    uint64_t key[kKeys], own = 0, last = 0;
    const uint64_t *k = from.keys + (int64_t)p * from.n * top;
    const int32_t lanes = from.n < 64 ? from.n : 64, half = lanes > 1 ? lanes / 2 : 1;
    // j-th best of r lanes' parts at least: j r >= top
    const int32_t j = (top + half - 1) / half, r = TOP ? (top + j - 1) / j : 0;
    Part part[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
        const int32_t g = lane + 64 * e;
        part[e] = g < from.n ? from.part[(int64_t)p * from.n + g] : Part{kNothing, -1};
    }
    if constexpr (TOP) {
#pragma unroll
        for (int e = 0; e < kKeys; ++e) {
            const int32_t i = (int32_t)threadIdx.x + e * kWide;
            key[e] = i < from.n * top ? k[i] : 0ull;
        }
#pragma unroll
        for (int e = 0; e < kEach; ++e) {
            const int32_t g = lane + 64 * e;
            const uint64_t o = g < from.n ? k[(int64_t)g * top + j - 1] : 0ull, l = g < from.n ? k[(int64_t)g * top + top - 1] : 0ull;
            own = o > own ? o : own;
            last = l > last ? l : last;
        }
        if (threadIdx.x == 0) n_list = 0;
        if (threadIdx.x < 64) keys[threadIdx.x] = 0;
    }
    const Problem q = problem_of(a, p);
    const Pick pick = pick_of(a, q, p, threadIdx.x);
    // every wave joins the parts for itself
    const float rate = kLog2e / q.T;
    Mass m = part[0].m;
#pragma unroll
    for (int e = 1; e < kEach; ++e) m = joined(m, part[e].m, rate);
    m = wave_mass(m, rate);
    int32_t first = -1;
    if (q.cold) {                                           // parts are in the candidates' order: the first that has the best score
        uint32_t g = 0xffffffffu;
        int32_t of = -1;
#pragma unroll
        for (int e = kEach - 1; e >= 0; --e)
            if (part[e].m.best == m.best && lane + 64 * e < from.n) {
                g = (uint32_t)(lane + 64 * e);
                of = part[e].first;
            }
        const uint32_t low = 0xffffffffu - wave_max_u32(0xffffffffu - g);
        const uint64_t has = __ballot(g == low && low != 0xffffffffu);
        if (has) first = __builtin_amdgcn_readlane(of, __builtin_ctzll(has));
    }
    if constexpr (TOP) {
        // What the best `top` are not below: the largest of the parts' last candidates, and the score that r lanes' j-th
        // best reach (of a lane's parts the one whose j-th is best), to 24 bits.
        uint32_t bits = 0;
#pragma unroll
        for (int b = 31; b >= 8; --b)
            if (__popcll(__ballot((uint32_t)(own >> 32) >= (bits | 1u << b))) >= r) bits |= 1u << b;
        const uint64_t most = wave_max_key(last), floor = (uint64_t)bits << 32 > most ? (uint64_t)bits << 32 : most;
        __syncthreads();
#pragma unroll
        for (int e = 0; e < kKeys; ++e)
            if (key[e] != 0 && key[e] >= floor) list[atomicAdd(&n_list, 1)] = key[e];
        __syncthreads();
        const int32_t n = n_list;
        for (int32_t i = threadIdx.x; i < n; i += kWide) {
            const uint64_t v = list[i];
            int32_t rank = 0;
#pragma unroll 8
            for (int32_t e = 0; e < n; ++e) rank += list[e] > v;
            if (rank < top) keys[rank] = v;
        }
        __syncthreads();
    }
    write_problem<kWide>(a, q, p, norm_of(m, q, first), threadIdx.x, pick, keys);
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

template <int CTRL, int ROW_MASK, bool ZERO_FILL>
__device__ __forceinline__ uint64_t dpp_add64(uint64_t v)
{
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROW_MASK, 0xf, ZERO_FILL);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROW_MASK, 0xf, ZERO_FILL);
    return v + (((uint64_t)hi << 32) | lo);
}

// Sum over the wave, in every lane.  (An atomic to LDS by 64 lanes is a loop over them: 2 us.)
__device__ __forceinline__ uint64_t wave_sum(uint64_t v)
{
    v = dpp_add64<0x111, 0xf, true>(v);
    v = dpp_add64<0x112, 0xf, true>(v);
    v = dpp_add64<0x114, 0xf, true>(v);
    v = dpp_add64<0x118, 0xf, true>(v);
    v = dpp_add64<0x142, 0xa, false>(v);
    v = dpp_add64<0x143, 0xc, false>(v);
    return lane_value(v, 63);
}

// Picks' gradients in fixed point: sums do not depend on their order.  Of acc only the picked candidates' entries are used.
template <int PART>
struct Fixed {
    unsigned long long acc[PART];
    unsigned long long total;
    uint32_t most;
};

// Candidates [from, to) of a problem by THREADS threads (this one the t-th), PART at a time: all of them as
// if none were picked, then the picked ones again by their picks' threads (each of several picks of one
// candidate stores the same).  The unit of fixed point is 2^e: the largest |d_logp| is below 2^x, n of them
// below 2^(62 + e).
template <int THREADS, int PART, bool PICKS>
__device__ __forceinline__ void gradient_of(const GradientArgs &a, int32_t p, const Problem &q, int32_t from, int32_t to, int t,
                                            Fixed<PICKS ? PART : 1> &fx)
{
    float *d = a.d_scores + q.at;
    if (q.cold) {
        for (int32_t i = from + t; i < to; i += THREADS) d[i] = 0.0f;
        return;
    }
    constexpr int kEach = PART / THREADS;
    const Norm z = {a.norm[2 * (int64_t)p], a.norm[2 * (int64_t)p + 1], a.d_entropy ? a.entropy[p] : 0.0f, -1};
    const float de = a.d_entropy ? a.d_entropy[p] : 0.0f;
    const int32_t *picks = a.picks + (int64_t)p * a.n_picks;
    const float *dl = a.d_logp + (int64_t)p * a.n_picks;
    // a thread's first pick stays with it
    int32_t own_j = -1;
    float own_g = 0.0f, own_s = kNone;
    if constexpr (PICKS) {
        if (t < a.n_picks) {
            own_j = picks[t];
            own_g = dl[t];
        }
    }
    // a part's scores, four in a row a thread
    float s[kEach];
    auto fetch = [&](int32_t part) {
#pragma unroll
        for (int k = 0; k < kEach; k += 4) {
            const f32x4u_t w = load4(q.s + part, k * THREADS + t * 4, to - part);
#pragma unroll
            for (int i = 0; i < 4; ++i) s[k + i] = w[i];
        }
    };
    fetch(from);
    // a pick's score, and its candidate: -1 where it does not count, outside or without a probability
    auto counted = [&](int32_t j, float &v) {
        if (j < 0 || j >= q.n) return -1;
        v = q.s[j];
        return log_probability(q, z, j, v) > kNone ? j : -1;
    };
    float S = 0.0f;
    unsigned long long sum = 0;                             // S in fixed point
    int e = 0;
    bool fine = true;
    auto fixed = [&](float v) { return (unsigned long long)(long long)__builtin_rint(__builtin_ldexp((double)v, -e)); };
    auto value = [&](unsigned long long v) { return (float)__builtin_ldexp((double)(long long)v, e); };
    // f(candidate, its score, gradient) for this thread's picks that count
    auto each = [&](auto &&f) {
        if (own_j >= 0) f(own_j, own_s, own_g);
        for (uint32_t i = t + THREADS; i < (uint32_t)a.n_picks; i += THREADS) {
            float v;
            const int32_t j = counted(picks[i], v);
            if (j >= 0) f(j, v, dl[i]);
        }
    };
    auto inside = [](int32_t i) { return (uint32_t)i < (uint32_t)PART; };
    if constexpr (PICKS) {
        if (t == 0) {
            fx.most = 0;
            fx.total = 0;
        }
        own_j = counted(own_j, own_s);
        group_barrier<THREADS>();
        uint32_t most = 0;
        each([&](int32_t j, float, float g) {
            const uint32_t b = __float_as_uint(g) & 0x7fffffffu;
            most = b > most ? b : most;
            if (inside(j - from)) fx.acc[j - from] = 0;
        });
        most = wave_max_u32(most);
        if constexpr (THREADS > 64) {
            if ((threadIdx.x & 63) == 0 && most != 0) atomicMax(&fx.most, most);
        }
        group_barrier<THREADS>();
        if constexpr (THREADS > 64) most = fx.most;
        fine = most < 0x7f800000u;
        S = __uint_as_float(most);
        if (fine) {                                         // (uniform)
            e = (int)(most >> 23) - 126 + (32 - __builtin_clz((uint32_t)a.n_picks)) - 62;
            each([&](int32_t j, float, float g) {
                const unsigned long long u = fixed(g);
                sum += u;
                if (inside(j - from)) atomicAdd(&fx.acc[j - from], u);
            });
            sum = wave_sum(sum);
            if constexpr (THREADS > 64) {
                if ((threadIdx.x & 63) == 0 && sum != 0) atomicAdd(&fx.total, sum);
                group_barrier<THREADS>();
                sum = fx.total;
            }
            S = value(sum);
        }
    }
    const float rate = kLog2e / q.T, by_T = fminf(1.0f / q.T, 3.4028235e38f);
    const float log2_mass = z.log_mass * kLog2e;
    // lt: log2 of a score's weight.  No weight (NaN and -inf, and below the numbers): no gradient
    auto lt_of = [&](float v) { return v == z.best ? 0.0f : (v - z.best) * rate; };
    auto done = [&](float v, float lt, float r) { return v > kNone && lt > kNone ? r * by_T : 0.0f; };
    auto of_entropy = [&](float pr, float lp) { return de * (pr > 0.0f ? pr * (lp + z.entropy) : 0.0f); };
    for (int32_t part = from; part < to; part += PART) {
        const int32_t n = to - part < PART ? to - part : PART;
        if constexpr (PICKS) {
            if (part > from && fine) {
                group_barrier<THREADS>();                   // the last part's entries have been read
                each([&](int32_t j, float, float) {
                    if (inside(j - part)) fx.acc[j - part] = 0;
                });
                group_barrier<THREADS>();
                each([&](int32_t j, float, float g) {
                    if (inside(j - part)) atomicAdd(&fx.acc[j - part], fixed(g));
                });
            }
        }
        float o[kEach];
#pragma unroll
        for (int k = 0; k < kEach; ++k) {
            const float lt = lt_of(s[k]), pr = __builtin_amdgcn_exp2f(lt - log2_mass);
            o[k] = done(s[k], lt, -pr * S - of_entropy(pr, lt * kLn2 - z.log_mass));
        }
#pragma unroll
        for (int k = 0; k < kEach; k += 4) {
            const int32_t i = k * THREADS + t * 4;
            if (i + 4 <= n) {
                *reinterpret_cast<f32x4u_t *>(d + part + i) = (f32x4u_t){o[k], o[k + 1], o[k + 2], o[k + 3]};
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i + j < n) d[part + i + j] = o[k + j];
            }
        }
        if (part + PART < to) fetch(part + PART);
        if constexpr (PICKS) {
            if (fine) {
                group_barrier<THREADS, true>();
                each([&](int32_t j, float v, float) {
                    const int32_t i = j - part;
                    if (!inside(i)) return;
                    const float lt = lt_of(v), pr = __builtin_amdgcn_exp2f(lt - log2_mass), lp = lt * kLn2 - z.log_mass;
                    // g (1 - p): where p is above 0.6 by the series of 1 - exp(lp), without the difference
                    float x = 1.0f / 9.0f;
#pragma unroll
                    for (int m = 8; m >= 1; --m) x = (1.0f + lp * x) * (1.0f / (float)m);
                    // (the others' sum S - g too: in whole numbers, rounded once)
                    const float g = value(fx.acc[i]), others = value(sum - fx.acc[i]), own = g * (lp > -0.5f ? -lp * x : 1.0f - pr);
                    d[part + i] = done(v, lt, own - pr * others - of_entropy(pr, lp));
                });
            }
        }
    }
}

__device__ __forceinline__ Problem problem_of(const GradientArgs &a, int32_t p)
{
    return problem_of(a.scores, a.R, a.seg, p, a.temperature, a.temperature_of);
}

// Rows of no problem: a share of them for each of the launch's threads.
__device__ __forceinline__ void clear_others(const GradientArgs &a, int64_t thread, int64_t threads)
{
    const int64_t before = within(a.seg[0], a.R), behind = within(a.seg[a.P], a.R);
    for (int64_t i = thread; i < before; i += threads) a.d_scores[i] = 0.0f;
    for (int64_t i = behind + thread; i < a.R; i += threads) a.d_scores[i] = 0.0f;
}

constexpr int kPart = 4096;                                 // candidates whose picks are summed at once

// gridDim.x workgroups have a problem, a part of its candidates each.
template <bool PICKS>
__global__ __launch_bounds__(kThreads) void k_logprob_gradient(GradientArgs a)
{
    __shared__ Fixed<PICKS ? kPart : 1> fx;
    const int32_t p = a.p0 + (int32_t)blockIdx.y;
    const Problem q = problem_of(a, p);
    // whole parts to each, the last ones to the last
    const int32_t parts = (q.n + kPart - 1) / kPart, each = (parts + (int32_t)gridDim.x - 1) / (int32_t)gridDim.x;
    const int64_t from = (int64_t)blockIdx.x * each * kPart, to = from + (int64_t)each * kPart;
    if (from < q.n) gradient_of<kThreads, kPart, PICKS>(a, p, q, (int32_t)from, (int32_t)(to < q.n ? to : q.n), threadIdx.x, fx);
    clear_others(a, ((int64_t)p * gridDim.x + blockIdx.x) * kThreads + threadIdx.x, (int64_t)a.P * gridDim.x * kThreads);
}

// A wave has a problem of up to kSmallPart candidates; longer ones follow, by the whole workgroup.
constexpr int kSmallPart = 1024;

template <bool PICKS>
__global__ __launch_bounds__(kThreads) void k_logprob_gradient_waves(GradientArgs a)
{
    constexpr int kWaves = kThreads / 64;
    using Small = Fixed<PICKS ? kSmallPart : 1>;
    using Large = Fixed<PICKS ? kPart : 1>;
    __shared__ __attribute__((aligned(16))) char lds[sizeof(Large) > kWaves * sizeof(Small) ? sizeof(Large) : kWaves * sizeof(Small)];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int32_t p0 = a.p0 + (int32_t)blockIdx.x * kWaves, p = p0 + wave;
    if (p < a.P) {
        const Problem q = problem_of(a, p);
        if (q.n <= kSmallPart && q.n > 0) gradient_of<64, kSmallPart, PICKS>(a, p, q, 0, q.n, threadIdx.x & 63, reinterpret_cast<Small *>(lds)[wave]);
    }
    for (int32_t i = 0; i < kWaves && p0 + i < a.P; ++i) {
        const Problem q = problem_of(a, p0 + i);
        if (q.n <= kSmallPart) continue;                    // (one answer for the workgroup)
        __syncthreads();
        gradient_of<kThreads, kPart, PICKS>(a, p0 + i, q, 0, q.n, threadIdx.x, *reinterpret_cast<Large *>(lds));
    }
    if (p < a.P) clear_others(a, (int64_t)p * 64 + (threadIdx.x & 63), (int64_t)a.P * 64);
}

}  // namespace

namespace {

// Problems' lengths are not known here; their mean is.  (600 problems of 500 and one of 534,600, a single workgroup's: 103 us, with
// 10 alternatives 178, the gradient 169.)  Parts and the kernel that joins them against a workgroup a problem, 16
// alternatives, us: 64 x 20,000 13.3 / 10.3, 8 x 40,000 11.1 / 12.1, 3 x 100,000 10.8 / 20.0, 64 x 100,000 15.7 / 20.8, 3 x 534,600
// 13.5 / 70.5.  Many of just enough are faster without parts, which they get all the same: 64 x 40,000 12.6 / 12.3,
// 128 x 65,536 16.2 / 14.6.
int32_t parts_of(int64_t R, int32_t P, int32_t top)
{
    const int64_t mean = R / P, n_cu = compute_units();
    if (2 * (int64_t)P > n_cu || mean < 8 * kWideTile) return 1;
    const int64_t by_units = 2 * n_cu / P, by_length = (mean + kWideTile - 1) / kWideTile, n = by_units < by_length ? by_units : by_length;
    const int64_t most = top * kMostParts > kMostKeys ? kMostKeys / top : kMostParts;
    return (int32_t)(n < most ? n : most);
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

}  // namespace

size_t logprob_workspace_bytes(int64_t R, int32_t P, int32_t top)
{
    const int32_t n = parts_of(R, P, top);
    return n == 1 ? 0 : up256((size_t)P * n * sizeof(Part)) + (size_t)P * n * top * 8;
}

hipError_t launch_logprob(const float *scores, int64_t R, const int64_t *seg, int32_t P, float temperature, const float *temperature_of,
                          const int32_t *picks, int32_t n_picks, int32_t top, float *logp, float *entropy, float *norm, int32_t *top_idx,
                          float *top_logp, void *ws, hipStream_t s)
{
    LogprobArgs a{scores, R, seg, temperature, temperature_of, picks, n_picks, top, logp, entropy, norm, top_idx, top_logp, P, 0};
    const int32_t parts = parts_of(R, P, top);
    const int64_t mean = R / P;
    auto go = [&]<bool TOP>() {
        if (parts > 1) {
            const Parts w{static_cast<Part *>(ws), reinterpret_cast<uint64_t *>(static_cast<char *>(ws) + up256((size_t)P * parts * sizeof(Part))), parts};
            hipLaunchKernelGGL((k_logprob_parts<TOP>), dim3(parts, P), dim3(kWide), 0, s, a, w);
            hipLaunchKernelGGL((k_logprob_join<TOP>), dim3(P), dim3(kWide), 0, s, a, w);
        } else if (mean <= (TOP && P <= 4 * compute_units() ? 256 : kSmall)) {
            // A wave a problem, four in a workgroup, against a workgroup each, us: without alternatives always (100 x 700 3.9 / 4.0,
            // 3,000 x 1,000 5.6 / 11.5); with ten 600 x 64 5.6 / 7.3, 100 x 512 8.0 / 6.0, 600 x 1,000 11.6 / 7.3, 3,000 x 700 14.3 / 15.8,
            // 8,000 x 700 28 / 33; with 64 100 x 200 7.2 / 10.1, 600 x 512 9.8 / 8.9.  Two limits do not part them everywhere: 100
            // x 200 with ten 6.7 / 6.1 and 1,500 x 700 12.8 / 9.8 go by waves.
            each_span(P, [&](int32_t p0, int32_t n) {
                a.p0 = p0;
                hipLaunchKernelGGL((k_logprob_waves<TOP>), dim3((n + 3) / 4), dim3(kThreads), 0, s, a);
            });
        } else {
            // Threads of a problem.  Fewer start and meet sooner, more read a long one with fewer steps; where a unit has
            // several problems those fill it.  256 / 512 / 1,024, 10 alternatives, us: 600 x 4,096 7.4 / 9.0 / 19.2, 600
            // of 2,000 .. 16,000 13.3 / 12.5 / 19.5, 300 of 6,000 .. 50,000 26.1 / 20.5 / 21.9; 200 x 4,096 6.2 / 6.4 / 7.7,
            // 1 x 8,192 7.1 / 5.9 / 7.1, 100 x 16,000 10.5 / 8.1 / 7.5, 200 x 100,000 50 / 31 / 29; none asked for: 100 x 16,000 6.0 /
            // 5.0 / 5.4, 256 x 65,536 19.5 / 14.0 / 14.9 and 200 x 100,000 28 / 18.5 / 17.4 out of the caches, but from memory 512
            // and 1,024 17.0 / 16.2 and 24 / 19.3: 1,024 for both.
            const bool alone = P <= compute_units();
            each_span(P, [&](int32_t p0, int32_t n) {
                a.p0 = p0;
                if (mean <= (alone ? 4096 : 8192)) hipLaunchKernelGGL((k_logprob<256, 2048, TOP>), dim3(n), dim3(256), 0, s, a);
                else if (!alone || mean <= 8192) hipLaunchKernelGGL((k_logprob<512, 4096, TOP>), dim3(n), dim3(512), 0, s, a);
                else hipLaunchKernelGGL((k_logprob<1024, kTile, TOP>), dim3(n), dim3(1024), 0, s, a);
            });
        }
    };
    if (top > 0) go.template operator()<true>();
    else go.template operator()<false>();
    return hipGetLastError();
}

hipError_t launch_logprob_gradient(const float *scores, int64_t R, const int64_t *seg, int32_t P, float temperature,
                                   const float *temperature_of, const float *norm, const int32_t *picks, int32_t n_picks,
                                   const float *d_logp, const float *entropy, const float *d_entropy, float *d_scores, hipStream_t s)
{
    GradientArgs a{scores, R, seg, P, 0, temperature, temperature_of, norm, picks, n_picks, d_logp, entropy, d_entropy, d_scores};
    const int64_t mean = R / P;
    auto go = [&]<bool PICKS>() {
        if (mean <= 1024) {                                 // (a wave / a workgroup each, us: 1 x 1,000 3.7 / 4.5, 2,000 x 900 6.4 / 12.0)
            each_span(P, [&](int32_t p0, int32_t n) {
                a.p0 = p0;
                hipLaunchKernelGGL((k_logprob_gradient_waves<PICKS>), dim3((n + 3) / 4), dim3(kThreads), 0, s, a);
            });
            return;
        }
        // Parts of up to twice the mean length; several to a workgroup where there are more of them than run at once (four a
        // unit, by their LDS): each goes through all picks.  One / two / five workgroups a problem, us: 600 of 1,000 .. 8,192 9.1 / 10.2 / 10.5, 2,000 x
        // 4,000 15.6 / 22.2 / 19.9, 256 x 65,536 29.0 / 24.1 / 25.1, 64 x 8,192 5.6 / 4.4 / 4.8; 8 x 200,000 64 / 35 / 16 and 5.7 with 98.
        const int64_t by_length = (2 * mean + kPart - 1) / kPart, at_once = 4 * (int64_t)compute_units() / P;
        const int64_t most = at_once > 1 ? at_once : 1, each = by_length < most ? by_length : most;
        for (a.p0 = 0; a.p0 < P; a.p0 += 1 << 15) {         // (a grid's second dimension)
            const int32_t n = P - a.p0 < 1 << 15 ? P - a.p0 : 1 << 15;
            hipLaunchKernelGGL((k_logprob_gradient<PICKS>), dim3((unsigned)each, n), dim3(kThreads), 0, s, a);
        }
    };
    if (n_picks > 0) go.template operator()<true>();
    else go.template operator()<false>();
    return hipGetLastError();
}

}  // namespace hwsel
