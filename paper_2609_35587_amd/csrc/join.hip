// Joining a block's result to the residual stream, with the norms after the
// block and before the next one, gate, dropout and scales; and its gradients.
//   u = w_branch norm(y);  v = dropout(branch g u);  x1 = stream x + v;  z = w_pre norm(x1)
// With d = d_x1 + r1 (dn - xn mean(dn xn)), dn = d_z w_pre, xn = x1 r1:
//   dx = stream d;  dv = dropout(branch d);  dg = dv u;  du = dv g;  dw_branch = sum du yn;
//   dy = r (dn' - yn mean(dn' yn)), dn' = du w_branch;  dw_pre = sum d_z xn
//
// Bound by memory: each operand is read once and each result written once where a row fits the registers of the threads
// that have it.  Measured (HBM bytes over time): 1,048,576 x 512, fp32 stream and bf16 block with an element gate, 1,456 us, 5.2
// TB/s, what a copy reaches; 65,536 x 1,024 in bf16 with gate and dropout forward 128 us, 5.2 TB/s, backward 209 us, 5.2 TB/s.
#include "rows.hpp"

namespace hwsel {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

struct In {
    const void *p;
    int64_t ld;
};

struct Out {
    void *p;
    int64_t ld;
};

enum { kNoGate = 0, kRowGate = 1, kElementGate = 2 };

struct Common {
    int32_t rows, cols;
    Ends ends;
    const float *wb, *wp;
    float eps, inv_cols, stream, branch;
    int32_t post_norm, gate_kind, sigmoid;
    Dropout drop;
    int64_t row0;                                           // the launch's first row
};

struct Forward {
    Common c;
    In x, y, gate;
    Out x1, z;
};

struct Backward {
    Common c;
    In x1, y, gate, dx1, dz;
    Out dx, dy, dgate;
    float *stats;                                           // [rows][4] of the long rows: r1, m1, r, m
    float *parts;                                           // [parts][2][cols]
    int32_t n_parts, rows_each, want_wb, want_wp;
};

__device__ __forceinline__ float norm_factor(float sum, const Common &c) { return 1.0f / __builtin_sqrtf(sum * c.inv_cols + c.eps); }

__device__ __forceinline__ float gate_value(float a, int sigmoid)
{
    return sigmoid ? __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2e * a)) : a;
}

// The gate's slope: s (1 - s) of a sigmoid, without the difference.
__device__ __forceinline__ float gate_slope(float a, int sigmoid)
{
    const float e = __builtin_amdgcn_exp2f(-kLog2e * __builtin_fabsf(a)), q = __builtin_amdgcn_rcpf(1.0f + e);
    return sigmoid ? e * q * q : 1.0f;
}

// Sums of N values over a workgroup, in every thread.
template <int NT, int N>
__device__ __forceinline__ void block_sums(float (&v)[N], float (&sh)[N][NT / 64])
{
    group_totals<64>(v);
    __syncthreads();                                        // the last sums have been read
    if ((threadIdx.x & 63) == 63) {
#pragma unroll
        for (int i = 0; i < N; ++i) sh[i][threadIdx.x >> 6] = v[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v[i] = 0.0f;
#pragma unroll
        for (int w = 0; w < NT / 64; ++w) v[i] += sh[i][w];
    }
}

template <int CTRL, int ROW_MASK, bool ZERO_FILL>
__device__ __forceinline__ double dpp_add64(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)b, CTRL, ROW_MASK, 0xf, ZERO_FILL);
    const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(b >> 32), CTRL, ROW_MASK, 0xf, ZERO_FILL);
    return v + __builtin_bit_cast(double, ((uint64_t)hi << 32) | lo);
}

// The wave's sum, in its last lane.
__device__ __forceinline__ double wave_total(double v)
{
    v = dpp_add64<0x111, 0xf, true>(v);
    v = dpp_add64<0x112, 0xf, true>(v);
    v = dpp_add64<0x114, 0xf, true>(v);
    v = dpp_add64<0x118, 0xf, true>(v);
    v = dpp_add64<0x142, 0xa, false>(v);
    return dpp_add64<0x143, 0xc, false>(v);
}

template <class E>
__device__ __forceinline__ void weights8(const float *w, int32_t col, const Common &c, const E &ends, float (&v)[8])
{
    if (w) {
        Eight<false> e = load8<false>(w, col, c.cols - col, ends);
        settle8(e, c.cols - col, ends);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = e.at(i);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = 1.0f;
    }
}

// d of eight columns: d_x1 and the norm before the next block; dn and xn of that.
template <bool SBF, bool BBF>
struct Stream8 {
    Eight<SBF> x1, dx1;
    Eight<BBF> dz;

    template <class E>
    __device__ __forceinline__ void load(const Backward &a, int64_t row, int32_t col, int32_t n, const E &ends)
    {
        x1 = load8<SBF>(a.dz.p ? a.x1.p : nullptr, row * a.x1.ld + col, n, ends);   // (of no use without d_z)
        dx1 = load8<SBF>(a.dx1.p, row * a.dx1.ld + col, n, ends);
        dz = load8<BBF>(a.dz.p, row * a.dz.ld + col, n, ends);
    }
    template <class E>
    __device__ __forceinline__ void settle(int32_t n, const E &ends)
    {
        settle8(x1, n, ends);
        settle8(dx1, n, ends);
        settle8(dz, n, ends);
    }
    __device__ __forceinline__ float d(int i, float wp, float r1, float m1) const
    {
        return dx1.at(i) + r1 * (dz.at(i) * wp - x1.at(i) * r1 * m1);
    }
};

// dv of eight columns from their d.
__device__ __forceinline__ void branch8(const Common &c, const Mask &m, int64_t row, int32_t col, const float (&d)[8], float (&dv)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) dv[i] = c.branch * d[i];
    if (m.least != 0) drop8(m, (uint32_t)row, (uint32_t)(col >> 3), dv);
}

template <int CTRL>
__device__ __forceinline__ float dpp_moved_add(float v)
{
    return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sums of N values over LANES neighbouring threads (0: the workgroup's), in
// each of them: lane moves within 8 or 16 lanes, the four rows of a wave by
// scalar reads, waves through LDS (two buffers in turn, so that a sum costs one
// barrier).
struct Shared {
    float v[2][3][16];
};

template <int LANES, int N>
__device__ __forceinline__ void lane_sums(float (&v)[N], Shared &sh, int &turn)
{
    static_assert(N <= 3, "room in Shared");
#pragma unroll
    for (int i = 0; i < N; ++i) {
        // lanes i ^ 1, i ^ 2, then the other four of eight; rotations by 8 of 16
        v[i] = dpp_moved_add<0x141>(dpp_moved_add<0x4e>(dpp_moved_add<0xb1>(v[i])));
        if constexpr (LANES != 8) v[i] = dpp_moved_add<0x128>(v[i]);
    }
    if constexpr (LANES == 0 || LANES >= 32) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int b = __float_as_int(v[i]);
            const float low = __int_as_float(__builtin_amdgcn_readlane(b, 0)) + __int_as_float(__builtin_amdgcn_readlane(b, 16));
            const float high = __int_as_float(__builtin_amdgcn_readlane(b, 32)) + __int_as_float(__builtin_amdgcn_readlane(b, 48));
            v[i] = LANES != 32 ? low + high : threadIdx.x & 32 ? high : low;
        }
    }
    if constexpr (LANES == 0) {
        auto &to = sh.v[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int i = 0; i < N; ++i) to[i][threadIdx.x >> 6] = v[i];
        }
        lds_barrier();
        const int waves = (int)blockDim.x >> 6;
#pragma unroll
        for (int i = 0; i < N; ++i) {
            v[i] = to[i][0];
            for (int w = 1; w < waves; ++w) v[i] += to[i][w];
        }
    }
}

// ---------------------------------------------------------------------------
// Rows that fit the registers of LANES threads, 8 K columns each: a row is read
// once and written once.  Threads keep their columns from row to row, so weights
// are read once a launch and their gradients are summed in registers.
// ---------------------------------------------------------------------------
// How a thread's k-th eight of K is read: but for the last all are there.
template <bool EDGE, int K, int k>
__device__ __forceinline__ auto ends_of_eight(const Common &c)
{
    if constexpr (k < K - 1) return AllThere{};
    else if constexpr (EDGE) return c.ends;
    else return NoEnds{};
}

// f(k, ends) for a thread's K eights.
template <bool EDGE, int K, class F>
__device__ __forceinline__ void each_eight(const Common &c, F &&f)
{
    if constexpr (K == 2) f(0, ends_of_eight<EDGE, K, 0>(c));
    f(K - 1, ends_of_eight<EDGE, K, K - 1>(c));
}

// Rows that a workgroup has at once: of 256 threads, or one.
template <int LANES>
constexpr int kRows = LANES ? 256 / LANES : 1;

template <int LANES>
__device__ __forceinline__ int64_t first_row()
{
    if constexpr (LANES == 0) return blockIdx.x;
    const int group = (int)threadIdx.x / (LANES ? LANES : 1);
    return (int64_t)blockIdx.x * kRows<LANES> + (LANES == 64 ? __builtin_amdgcn_readfirstlane(group) : group);
}

// The first of a thread's columns in its k-th eight.
template <int LANES>
__device__ __forceinline__ int32_t column(int k)
{
    const int lanes = LANES ? LANES : (int)blockDim.x;
    return (LANES ? threadIdx.x % (LANES ? LANES : 1) : threadIdx.x) * 8 + k * lanes * 8;
}

// Whether a thread of this wave has the last columns of rows that are no whole number of eights.
template <int LANES, int K>
__device__ __forceinline__ bool has_last(const Common &c)
{
    const int32_t n = c.cols - column<LANES>(K - 1);
    return c.ends.shift != 0 && __ballot(n > 0 && n < 8) != 0;
}

template <bool SBF, bool BBF, int LANES, int K, bool EDGE>
__global__ __launch_bounds__(LANES ? 256 : 1024) void k_join(Forward a)
{
    __shared__ Shared sh;
    const Common &c = a.c;
    const Mask m = mask_of(c.drop);
    auto col_of = [&](int k) { return column<LANES>(k); };
    float wb[K][8], wp[K][8];
    each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
        weights8(c.wb, col_of(k), c, ends, wb[k]);
        weights8(c.wp, col_of(k), c, ends, wp[k]);
    });
    const bool ragged = EDGE && has_last<LANES, K>(c);
    int turn = 0;
    for (int64_t row = first_row<LANES>(); row < c.rows; row += (int64_t)gridDim.x * kRows<LANES>) {
        Eight<SBF> x[K];
        Eight<BBF> y[K], g[K];
        each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
            const int32_t col = col_of(k), n = c.cols - col;
            x[k] = load8<SBF>(a.x.p, row * a.x.ld + col, n, ends);
            y[k] = load8<BBF>(a.y.p, row * a.y.ld + col, n, ends);
            g[k] = load8<BBF>(c.gate_kind == kElementGate ? a.gate.p : nullptr, row * a.gate.ld + col, n, ends);
        });
        if (ragged) {
            settle8(x[K - 1], c.cols - col_of(K - 1), c.ends);
            settle8(y[K - 1], c.cols - col_of(K - 1), c.ends);
            if (c.gate_kind == kElementGate) settle8(g[K - 1], c.cols - col_of(K - 1), c.ends);
        }
        float x1[K][8];
        if (a.y.p) {
            const float row_gate = c.gate_kind == kRowGate ? gate_value(load1<BBF>(a.gate.p, row * a.gate.ld), c.sigmoid) : 1.0f;
            float r = 1.0f;
            if (c.post_norm) {
                float t[1] = {0.0f};
#pragma unroll
                for (int k = 0; k < K; ++k)
#pragma unroll
                    for (int i = 0; i < 8; ++i) t[0] += y[k].at(i) * y[k].at(i);
                lane_sums<LANES>(t, sh, turn);
                r = norm_factor(t[0], c);
            }
            const float scale = c.branch * row_gate * r;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                float v[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = scale * (y[k].at(i) * wb[k][i]);
                if (c.gate_kind == kElementGate) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[i] *= gate_value(g[k].at(i), c.sigmoid);
                }
                if (m.least != 0) drop8(m, (uint32_t)row, (uint32_t)(col_of(k) >> 3), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) x1[k][i] = c.stream * x[k].at(i) + v[i];
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) x1[k][i] = c.stream * x[k].at(i);
        }
        if (a.x1.p)
            each_eight<EDGE, K>(c, [&](int k, const auto &ends) { store8<SBF>(a.x1.p, row * a.x1.ld + col_of(k), c.cols - col_of(k), ends, x1[k]); });
        if (a.z.p) {
            float t[1] = {0.0f};
#pragma unroll
            for (int k = 0; k < K; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) t[0] += col_of(k) + i < c.cols ? x1[k][i] * x1[k][i] : 0.0f;
            lane_sums<LANES>(t, sh, turn);
            const float r1 = norm_factor(t[0], c);
            each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
                float z[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) z[i] = x1[k][i] * r1 * wp[k][i];
                store8<BBF>(a.z.p, row * a.z.ld + col_of(k), c.cols - col_of(k), ends, z);
            });
        }
    }
}

// Two rounds of sums a row: x1^2, dn x1 and y^2 together, then what goes by d.
// A workgroup's sums over its rows go to a part of their own, joined in a fixed
// order by k_join_sums: atomics would add in any order.  The second launch takes 5 us.
// Five operands and two sums of 16 columns are 190 to 225 registers, two waves a SIMD; vector units are busy 59 % of the time.  One
// eight a thread takes 103 to 125 where a wave or a workgroup has a row, up to 151 for several rows of a wave: the waves that
// the launch bounds promise are what the compiler reaches without them too, and what groups_of counts on.
template <bool SBF, bool BBF, int LANES, int K, bool EDGE>
__global__ __launch_bounds__(LANES ? 256 : 512, K == 2 ? 2 : LANES == 64 || LANES == 0 ? 4 : 3) void k_join_gradient(Backward a)
{
    constexpr int kGroups = kRows<LANES>;
    __shared__ Shared sh;
    __shared__ __attribute__((aligned(16))) float sums[kGroups][LANES ? LANES * 8 * K : 1];
    const Common &c = a.c;
    const Mask m = mask_of(c.drop);
    auto col_of = [&](int k) { return column<LANES>(k); };
    float wb[K][8], wp[K][8], swb[K][8] = {}, swp[K][8] = {};
    each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
        weights8(c.wb, col_of(k), c, ends, wb[k]);
        weights8(c.wp, col_of(k), c, ends, wp[k]);
    });
    const bool ragged = EDGE && has_last<LANES, K>(c);
    int turn = 0;
    for (int64_t row = first_row<LANES>(); row < c.rows; row += (int64_t)gridDim.x * kRows<LANES>) {
        Stream8<SBF, BBF> q[K];
        Eight<BBF> y[K], g[K];
        each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
            const int32_t col = col_of(k), n = c.cols - col;
            q[k].load(a, row, col, n, ends);
            y[k] = load8<BBF>(a.y.p, row * a.y.ld + col, n, ends);
            g[k] = load8<BBF>(c.gate_kind == kElementGate ? a.gate.p : nullptr, row * a.gate.ld + col, n, ends);
        });
        if (ragged) {
            q[K - 1].settle(c.cols - col_of(K - 1), c.ends);
            settle8(y[K - 1], c.cols - col_of(K - 1), c.ends);
            if (c.gate_kind == kElementGate) settle8(g[K - 1], c.cols - col_of(K - 1), c.ends);
        }
        float s[3] = {};
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                s[0] += q[k].x1.at(i) * q[k].x1.at(i);
                s[1] += q[k].dz.at(i) * wp[k][i] * q[k].x1.at(i);
                s[2] += y[k].at(i) * y[k].at(i);
            }
        lane_sums<LANES>(s, sh, turn);
        const float r1 = a.dz.p ? norm_factor(s[0], c) : 0.0f, m1 = r1 * s[1] * c.inv_cols;
        float d[K][8];
        each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
            float o[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                d[k][i] = q[k].d(i, wp[k][i], r1, m1);
                swp[k][i] += q[k].dz.at(i) * (q[k].x1.at(i) * r1);
                o[i] = c.stream * d[k][i];
            }
            if (a.dx.p) store8<SBF>(a.dx.p, row * a.dx.ld + col_of(k), c.cols - col_of(k), ends, o);
        });
        if (!a.y.p) continue;
        const float r = c.post_norm ? norm_factor(s[2], c) : 1.0f;
        const float gate = c.gate_kind == kRowGate ? load1<BBF>(a.gate.p, row * a.gate.ld) : 1.0f;
        const float row_gate = c.gate_kind == kRowGate ? gate_value(gate, c.sigmoid) : 1.0f;
        float t[2] = {};                                    // of dn' yn; of dv u, the gradient of a row's gate
        each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
            float dv[8], dg[8];
            branch8(c, m, row, col_of(k), d[k], dv);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float yn = y[k].at(i) * r, gi = c.gate_kind == kElementGate ? gate_value(g[k].at(i), c.sigmoid) : row_gate;
                const float u = yn * wb[k][i], du = dv[i] * gi;
                t[1] += dv[i] * u;
                dg[i] = dv[i] * u;
                swb[k][i] += du * yn;
                d[k][i] = du * wb[k][i];                    // dn' from here on
                t[0] += d[k][i] * yn;
            }
            if (a.dgate.p && c.gate_kind == kElementGate) {
#pragma unroll
                for (int i = 0; i < 8; ++i) dg[i] *= gate_slope(g[k].at(i), c.sigmoid);
                store8<BBF>(a.dgate.p, row * a.dgate.ld + col_of(k), c.cols - col_of(k), ends, dg);
            }
        });
        if (c.post_norm || c.gate_kind == kRowGate) lane_sums<LANES>(t, sh, turn);
        const float mean = c.post_norm ? t[0] * c.inv_cols : 0.0f;
        if (a.dy.p) {
            each_eight<EDGE, K>(c, [&](int k, const auto &ends) {
                float o[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) o[i] = r * (d[k][i] - y[k].at(i) * r * mean);
                store8<BBF>(a.dy.p, row * a.dy.ld + col_of(k), c.cols - col_of(k), ends, o);
            });
        }
        if (col_of(0) == 0 && a.dgate.p && c.gate_kind == kRowGate) {
            const float dg = t[1] * gate_slope(gate, c.sigmoid);
            if constexpr (BBF) static_cast<uint16_t *>(a.dgate.p)[row * a.dgate.ld] = (uint16_t)bf16_pair(dg, 0.0f);
            else static_cast<float *>(a.dgate.p)[row * a.dgate.ld] = dg;
        }
    }
    float *part = a.parts + (int64_t)blockIdx.x * 2 * c.cols;
    auto hand_on = [&](float (&v)[K][8], float *to) {
        if constexpr (kGroups > 1) {
            __syncthreads();
            each_eight<EDGE, K>(c, [&](int k, const auto &ends) { store8<false>(&sums[threadIdx.x / LANES][0], col_of(k), 8, ends, v[k]); });
            __syncthreads();
            for (int col = threadIdx.x; col < LANES * 8 * K && col < c.cols; col += 256) {
                float t = sums[0][col];
#pragma unroll
                for (int i = 1; i < kGroups; ++i) t += sums[i][col];
                to[col] = t;
            }
        } else {
            each_eight<EDGE, K>(c, [&](int k, const auto &ends) { store8<false>(to, col_of(k), c.cols - col_of(k), ends, v[k]); });
        }
    };
    if (a.want_wb) hand_on(swb, part);
    if (a.want_wp) hand_on(swp, part + c.cols);
}

// ---------------------------------------------------------------------------
// Rows of any length: a workgroup goes through a row several times, from the
// second on out of the caches where it fits them.  Forward: 2,000 x 30,000 in bf16 188 us (3.2 TB/s of each operand once).
// Backward: two kernels, the rows' sums, then columns, whose sums over a part of the rows stay in registers, at 4.1 and 5.0 TB/s
// of their operands: 4,000 x 16,384 385 us (2.7 TB/s of each operand once), 2,000 x 30,000 355 us (2.7 TB/s); 401 and 385 with
// what goes by d in a second pass of the first kernel.  Rows are in 256 parts: up to 256 rows are a part each, whose sums are
// its own terms, written and read again (8 bytes a column and part).
// ---------------------------------------------------------------------------
constexpr int kLong = 512;

template <bool SBF, bool BBF>
__global__ __launch_bounds__(kLong) void k_join_long(Forward a)
{
    __shared__ float sh[1][kLong / 64];
    const Common &c = a.c;
    const Ends ends = c.ends;
    const int64_t row = c.row0 + blockIdx.x;
    const Mask m = mask_of(c.drop);
    float r = 1.0f;
    if (a.y.p && c.post_norm) {
        float s[1] = {0.0f};
        for (int32_t col = threadIdx.x * 8; col < c.cols; col += kLong * 8) {
            Eight<BBF> y = load8<BBF>(a.y.p, row * a.y.ld + col, c.cols - col, ends);
            settle8(y, c.cols - col, ends);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += y.at(i) * y.at(i);
        }
        block_sums<kLong>(s, sh);
        r = norm_factor(s[0], c);
    }
    const float row_gate = c.gate_kind == kRowGate ? gate_value(load1<BBF>(a.gate.p, row * a.gate.ld), c.sigmoid) : 1.0f;
    auto joined = [&](int32_t col, float (&x1)[8]) {
        const int32_t n = c.cols - col;
        Eight<SBF> x = load8<SBF>(a.x.p, row * a.x.ld + col, n, ends);
        settle8(x, n, ends);
        float v[8] = {};
        if (a.y.p) {
            Eight<BBF> y = load8<BBF>(a.y.p, row * a.y.ld + col, n, ends);
            settle8(y, n, ends);
            float w[8];
            weights8(c.wb, col, c, ends, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = c.branch * row_gate * (y.at(i) * r * w[i]);
            if (c.gate_kind == kElementGate) {
                Eight<BBF> g = load8<BBF>(a.gate.p, row * a.gate.ld + col, n, ends);
                settle8(g, n, ends);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] *= gate_value(g.at(i), c.sigmoid);
            }
            if (m.least != 0) drop8(m, (uint32_t)row, (uint32_t)(col >> 3), v);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) x1[i] = i < n ? c.stream * x.at(i) + v[i] : 0.0f;
    };
    float r1 = 1.0f;
    if (a.z.p) {
        float s[1] = {0.0f};
        for (int32_t col = threadIdx.x * 8; col < c.cols; col += kLong * 8) {
            float x1[8];
            joined(col, x1);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[0] += x1[i] * x1[i];
        }
        block_sums<kLong>(s, sh);
        r1 = norm_factor(s[0], c);
    }
    for (int32_t col = threadIdx.x * 8; col < c.cols; col += kLong * 8) {
        const int32_t n = c.cols - col;
        float x1[8];
        joined(col, x1);
        if (a.x1.p) store8<SBF>(a.x1.p, row * a.x1.ld + col, n, ends, x1);
        if (a.z.p) {
            float w[8], z[8];
            weights8(c.wp, col, c, ends, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) z[i] = x1[i] * r1 * w[i];
            store8<BBF>(a.z.p, row * a.z.ld + col, n, ends, z);
        }
    }
}

// What the columns' pass needs of each row, and the gradient of its gate, in one pass over the row.  d is linear in
// d_x1, dn and x1 with factors that are known once the row has been read, so what goes by d is made of three
// sums with h = dropout(branch) w_branch y (and an element's gate): sum h d = sum h d_x1 + r1 (sum h dn - r1 m1 sum h x1).
// Where the parts of d cancel so do the three sums, but not their errors: they are made in 64 bits, of products that these
// hold whole.  (In 32 bits 4,000 x 16,384 took 376 us, and dy kept the error of what had cancelled.)
template <bool SBF, bool BBF>
__global__ __launch_bounds__(kLong) void k_join_long_stats(Backward a)
{
    __shared__ float sh[3][kLong / 64];
    __shared__ double sh64[3][kLong / 64];
    const Common &c = a.c;
    const Ends ends = c.ends;
    const int64_t row = c.row0 + blockIdx.x;
    const Mask m = mask_of(c.drop);
    const bool by_d = a.y.p && (c.post_norm || c.gate_kind == kRowGate);
    float s[3] = {};
    double t[3] = {};
    for (int32_t col = threadIdx.x * 8; col < c.cols; col += kLong * 8) {
        const int32_t n = c.cols - col;
        Stream8<SBF, BBF> q;
        q.load(a, row, col, n, ends);
        Eight<BBF> y = load8<BBF>(by_d ? a.y.p : nullptr, row * a.y.ld + col, n, ends);
        Eight<BBF> g = load8<BBF>(by_d && c.gate_kind == kElementGate ? a.gate.p : nullptr, row * a.gate.ld + col, n, ends);
        float wp[8], wb[8];
        weights8(c.wp, col, c, ends, wp);
        weights8(c.wb, col, c, ends, wb);
        q.settle(n, ends);
        settle8(y, n, ends);
        settle8(g, n, ends);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s[0] += q.x1.at(i) * q.x1.at(i);
            s[1] += q.dz.at(i) * wp[i] * q.x1.at(i);
            s[2] += y.at(i) * y.at(i);
        }
        if (!by_d) continue;
        float share[8];                                     // of the branch: 0 where it is dropped
#pragma unroll
        for (int i = 0; i < 8; ++i) share[i] = 1.0f;
        if (m.least != 0) drop8(m, (uint32_t)row, (uint32_t)(col >> 3), share);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float h = share[i] * c.branch * wb[i] * y.at(i) * (c.gate_kind == kElementGate ? gate_value(g.at(i), c.sigmoid) : 1.0f);
            t[0] += share[i] != 0.0f ? (double)h * q.dx1.at(i) : 0.0;
            t[1] += (double)h * ((double)q.dz.at(i) * wp[i]);
            t[2] += (double)h * q.x1.at(i);
        }
    }
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        t[i] = wave_total(t[i]);
        if ((threadIdx.x & 63) == 63) sh64[i][threadIdx.x >> 6] = t[i];
    }
    block_sums<kLong>(s, sh);                               // (its barriers)
    if (threadIdx.x != 0) return;
    const float r1 = a.dz.p ? norm_factor(s[0], c) : 0.0f, m1 = r1 * s[1] * c.inv_cols;
    const float r = c.post_norm ? norm_factor(s[2], c) : 1.0f;
#pragma unroll
    for (int i = 0; i < 3; ++i) {
        t[i] = sh64[i][0];
#pragma unroll
        for (int w = 1; w < kLong / 64; ++w) t[i] += sh64[i][w];
    }
    // of dv u, the gradient of a row's gate; its gate times that: of dn' yn
    const float by_u = (float)(r * (t[0] + (double)r1 * (t[1] - (double)r1 * m1 * t[2])));
    float row_gate = 1.0f;
    if (c.gate_kind == kRowGate) {
        const float gate = load1<BBF>(a.gate.p, row * a.gate.ld);
        row_gate = gate_value(gate, c.sigmoid);
        if (a.dgate.p) {
            const float dg = by_u * gate_slope(gate, c.sigmoid);
            if constexpr (BBF) static_cast<uint16_t *>(a.dgate.p)[row * a.dgate.ld] = (uint16_t)bf16_pair(dg, 0.0f);
            else static_cast<float *>(a.dgate.p)[row * a.dgate.ld] = dg;
        }
    }
    float *st = a.stats + row * 4;
    st[0] = r1;
    st[1] = m1;
    st[2] = r;
    st[3] = c.post_norm ? row_gate * by_u * c.inv_cols : 0.0f;
}

// The gradients of 2,048 columns of some rows, and their sums over those rows.
constexpr int kTile = 256;

template <bool SBF, bool BBF>
__global__ __launch_bounds__(kTile) void k_join_long_columns(Backward a)
{
    const Common &c = a.c;
    const Ends ends = c.ends;
    const int32_t col = (int32_t)(blockIdx.x * kTile + threadIdx.x) * 8, n = c.cols - col;
    if (n <= 0) return;
    const Mask m = mask_of(c.drop);
    float wp[8], wb[8], swb[8] = {}, swp[8] = {};
    weights8(c.wp, col, c, ends, wp);
    weights8(c.wb, col, c, ends, wb);
    const int64_t first = (int64_t)blockIdx.y * a.rows_each, last = first + a.rows_each < c.rows ? first + a.rows_each : c.rows;
    for (int64_t row = first; row < last; ++row) {
        const float *st = a.stats + row * 4;
        const float r1 = st[0], m1 = st[1], r = st[2], mean = st[3];
        Stream8<SBF, BBF> q;
        q.load(a, row, col, n, ends);
        Eight<BBF> y = load8<BBF>(a.y.p, row * a.y.ld + col, n, ends);
        Eight<BBF> g = load8<BBF>(c.gate_kind == kElementGate ? a.gate.p : nullptr, row * a.gate.ld + col, n, ends);
        q.settle(n, ends);
        settle8(y, n, ends);
        settle8(g, n, ends);
        float d[8], o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            d[i] = q.d(i, wp[i], r1, m1);
            swp[i] += q.dz.at(i) * (q.x1.at(i) * r1);
            o[i] = c.stream * d[i];
        }
        if (a.dx.p) store8<SBF>(a.dx.p, row * a.dx.ld + col, n, ends, o);
        if (!a.y.p) continue;
        const float row_gate = c.gate_kind == kRowGate ? gate_value(load1<BBF>(a.gate.p, row * a.gate.ld), c.sigmoid) : 1.0f;
        float dv[8];
        branch8(c, m, row, col, d, dv);
        float dg[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float yn = y.at(i) * r, gi = c.gate_kind == kElementGate ? gate_value(g.at(i), c.sigmoid) : row_gate;
            dg[i] = dv[i] * (yn * wb[i]) * (c.gate_kind == kElementGate ? gate_slope(g.at(i), c.sigmoid) : 0.0f);
            const float du = dv[i] * gi;
            swb[i] += du * yn;
            o[i] = r * (du * wb[i] - yn * mean);
        }
        if (a.dy.p) store8<BBF>(a.dy.p, row * a.dy.ld + col, n, ends, o);
        if (a.dgate.p && c.gate_kind == kElementGate) store8<BBF>(a.dgate.p, row * a.dgate.ld + col, n, ends, dg);
    }
    float *part = a.parts + (int64_t)blockIdx.y * 2 * c.cols;
    if (a.want_wb) store8<false>(part, col, n, ends, swb);
    if (a.want_wp) store8<false>(part, c.cols + col, n, ends, swp);
}

// Sums of the parts: dw_branch and dw_pre.  A workgroup has 32 columns, 32
// threads each, every one a 32nd of the parts: 512 parts of 1,024 columns in two
// rounds of eight loads.
constexpr int kSumCols = 32, kSumThreads = 1024;

__global__ __launch_bounds__(kSumThreads) void k_join_sums(const float *__restrict__ parts, int32_t n_parts, int64_t cols, int64_t col0, float *dwb,
                                                           float *dwp)
{
    constexpr int kSlices = kSumThreads / kSumCols;
    __shared__ float sh[kSlices][kSumCols + 1];
    float *out = blockIdx.y ? dwp : dwb;
    if (!out) return;
    const int slice = threadIdx.x / kSumCols, at = threadIdx.x % kSumCols;
    const int64_t col = col0 + (int64_t)blockIdx.x * kSumCols + at;
    float s = 0.0f;
    if (col < cols) {
        const float *from = parts + (int64_t)blockIdx.y * cols + col;
        for (int32_t i = slice; i < n_parts; i += 8 * kSlices) {
            float v[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                const int32_t g = i + k * kSlices;
                v[k] = g < n_parts ? from[(int64_t)g * 2 * cols] : 0.0f;
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) s += v[k];
        }
    }
    sh[slice][at] = s;
    __syncthreads();
    if (slice != 0 || col >= cols) return;
#pragma unroll
    for (int i = 1; i < kSlices; ++i) s += sh[i][at];
    out[col] = s;
}

Common common_of(const hwsel_join_t &j, bool has_y)
{
    Common c{};
    c.cols = (int32_t)j.cols;
    c.ends = ends_of(j.cols);
    c.rows = (int32_t)j.rows;
    c.wb = j.w_branch;
    c.wp = j.w_pre;
    c.eps = j.eps;
    c.inv_cols = 1.0f / (float)j.cols;
    c.stream = j.stream_scale;
    c.branch = j.branch_scale;
    c.post_norm = has_y && j.post_norm;
    c.gate_kind = j.gate_cols == 0 ? kNoGate : j.gate_cols == 1 && j.cols != 1 ? kRowGate : kElementGate;
    c.sigmoid = j.gate_sigmoid;
    c.drop = dropout_of(j.dropout);
    return c;
}

In in_of(const hwsel_matrix_t &m) { return {m.data, m.ld}; }
Out out_of(const hwsel_matrix_t &m) { return {m.data, m.ld}; }

// go<stream in bf16, block in bf16>()
template <class F>
void by_types(bool sbf, bool bbf, F &&go)
{
    if (sbf) bbf ? go.template operator()<true, true>() : go.template operator()<true, false>();
    else bbf ? go.template operator()<false, true>() : go.template operator()<false, false>();
}

// f(rows) with c.row0 set for spans of rows that are a launch each of kLong threads a row: fewer than 2^32.
template <class F>
void each_row_span(Common &c, F &&f)
{
    constexpr int64_t kSpan = (int64_t)1 << 21;
    for (c.row0 = 0; c.row0 < c.rows; c.row0 += kSpan) f((unsigned)(c.rows - c.row0 < kSpan ? c.rows - c.row0 : kSpan));
    c.row0 = 0;
}

size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

// The longest rows that registers hold: 1,024 threads of two eights forward; backward 512, since 1,024 threads leave each
// 128 registers and the gradient takes up to 225.
constexpr int64_t kLongestForward = 16384, kLongestBackward = 8192;

// How rows of some length lie in registers: `lanes` threads of K eights each (0: all of the workgroup's `threads`).
// Fewer threads a row leave fewer without columns and add up in fewer steps; two eights a thread have more loads on the way.
// Forward in bf16, us: 1,000,000 x 64 by 8 lanes 113, by 16 227; 200,000 x 250 by 32 lanes 115, by 64 205; 65,536 x 1,024 by one
// wave of two eights 131, by two waves of one 147; 16,384 x 4,096 with two eights 127, with one 147; 8,192 x 8,192 130 and 152.
struct Shape {
    int lanes, K, threads;
    int rows() const { return lanes ? 256 / lanes : 1; }
};

Shape shape_of(int64_t cols)
{
    if (cols <= 64) return {8, 1, 256};
    if (cols <= 128) return {16, 1, 256};
    if (cols <= 256) return {32, 1, 256};
    if (cols <= 512) return {64, 1, 256};
    if (cols <= 1024) return {64, 2, 256};
    if (cols <= 1536) return {0, 1, 192};                   // (128 threads of two eights leave more of them without columns)
    return {0, 2, (int)((cols + 1023) / 1024) * 64};
}

// Workgroups that run at once where a SIMD holds `waves` of their waves, at most one for each row (or rows).
// 65,536 x 1,024 in bf16, us: forward 4 waves 131, 6 142, 8 136; backward 2 waves 213, 3 231, 4 215 (and twice the parts).
// One eight a thread, bf16, forward 4 / 6 / 8 waves: several rows of a wave 1,000,000 x 64 121 / 123 / 139, 250,000 x 256 119 / 124 / 139;
// else 262,144 x 512 246 / 261 / 272, but rows that are no whole number of eights 200,000 x 300 226 / 183 / 215, 60,000 x 1,500 248 / 194 / 245: 6.
// Backward 2 / 3 / 4: 1,000,000 x 64 196 / 204 / 211, 262,144 x 512 439 / 438 / 464 (though 200,000 x 300 366 / 303 / 283): 2; a workgroup's row
// 60,000 x 1,500 500 / 339 / 333: 4.
int32_t groups_of(const Shape &f, int64_t rows, int waves)
{
    const int64_t each = 4 * waves * 64 / f.threads, most = (int64_t)compute_units() * (each > 1 ? each : 1), need = (rows + f.rows() - 1) / f.rows();
    return (int32_t)(need < most ? need : most);
}

int32_t forward_groups(const hwsel_join_t &j)
{
    const Shape f = shape_of(j.cols);
    return groups_of(f, j.rows, f.K == 1 && (f.lanes == 64 || f.lanes == 0) ? 6 : 4);
}

// A workgroup of the gradient has a part of the sums over rows.
int32_t gradient_parts(const hwsel_join_t &j)
{
    const Shape f = shape_of(j.cols);
    return groups_of(f, j.rows, f.K == 1 && !f.lanes ? 4 : 2);
}

// go<LANES, K>() of a shape.
template <class F>
void by_shape(const Shape &f, F &&go)
{
    if (f.lanes == 8) go.template operator()<8, 1>();
    else if (f.lanes == 16) go.template operator()<16, 1>();
    else if (f.lanes == 32) go.template operator()<32, 1>();
    else if (f.lanes == 64) f.K == 1 ? go.template operator()<64, 1>() : go.template operator()<64, 2>();
    else f.K == 1 ? go.template operator()<0, 1>() : go.template operator()<0, 2>();
}

// Of rows that are too long, the columns' pass has its rows in this many parts.
constexpr int32_t kLongParts = 256;

int32_t long_rows_each(int64_t rows) { return (int32_t)((rows + kLongParts - 1) / kLongParts); }

}  // namespace

size_t join_gradient_workspace_bytes(const hwsel_join_t &j)
{
    if (j.cols <= kLongestBackward) return (size_t)gradient_parts(j) * 2 * (size_t)j.cols * 4;
    const int64_t each = long_rows_each(j.rows), parts = (j.rows + each - 1) / each;
    return up256((size_t)j.rows * 16) + (size_t)parts * 2 * (size_t)j.cols * 4;
}

hipError_t launch_block_join(const hwsel_join_t &j, const hwsel_matrix_t &x, const hwsel_matrix_t &y, const hwsel_matrix_t &gate,
                             const hwsel_matrix_t &x1, const hwsel_matrix_t &z, bool sbf, bool bbf, hipStream_t s)
{
    Forward a{common_of(j, y.data != nullptr), in_of(x), in_of(y), in_of(gate), out_of(x1), out_of(z)};
    by_types(sbf, bbf, [&]<bool SBF, bool BBF>() {
        if (j.cols > kLongestForward) {
            each_row_span(a.c, [&](unsigned n) { hipLaunchKernelGGL((k_join_long<SBF, BBF>), dim3(n), dim3(kLong), 0, s, a); });
            return;
        }
        const Shape f = shape_of(j.cols);
        by_shape(f, [&]<int LANES, int K>() {
            const auto kernel = j.cols % 8 ? k_join<SBF, BBF, LANES, K, true> : k_join<SBF, BBF, LANES, K, false>;
            hipLaunchKernelGGL(kernel, dim3((unsigned)forward_groups(j)), dim3(f.threads), 0, s, a);
        });
    });
    return hipGetLastError();
}

hipError_t launch_block_join_gradient(const hwsel_join_t &j, const hwsel_matrix_t &x1, const hwsel_matrix_t &y,
                                      const hwsel_matrix_t &gate, const hwsel_matrix_t &dx1, const hwsel_matrix_t &dz,
                                      const hwsel_matrix_t &dx, const hwsel_matrix_t &dy, const hwsel_matrix_t &dgate, float *dwb,
                                      float *dwp, void *ws, bool sbf, bool bbf, hipStream_t s)
{
    Backward a{common_of(j, y.data != nullptr), in_of(x1), in_of(y), in_of(gate), in_of(dx1), in_of(dz), out_of(dx), out_of(dy), out_of(dgate),
               nullptr, static_cast<float *>(ws), 0, 0, dwb != nullptr, dwp != nullptr};
    if (j.cols <= kLongestBackward) {
        a.n_parts = gradient_parts(j);
        by_types(sbf, bbf, [&]<bool SBF, bool BBF>() {
            const Shape f = shape_of(j.cols);
            by_shape(f, [&]<int LANES, int K>() {
                const auto kernel = j.cols % 8 ? k_join_gradient<SBF, BBF, LANES, K, true> : k_join_gradient<SBF, BBF, LANES, K, false>;
                hipLaunchKernelGGL(kernel, dim3((unsigned)a.n_parts), dim3(f.threads), 0, s, a);
            });
        });
    } else {
        a.stats = static_cast<float *>(ws);
        a.parts = reinterpret_cast<float *>(static_cast<char *>(ws) + up256((size_t)j.rows * 16));
        a.rows_each = long_rows_each(j.rows);
        a.n_parts = (int32_t)((j.rows + a.rows_each - 1) / a.rows_each);
        const unsigned strips = (unsigned)((j.cols + kTile * 8 - 1) / (kTile * 8));
        by_types(sbf, bbf, [&]<bool SBF, bool BBF>() {
            each_row_span(a.c, [&](unsigned n) { hipLaunchKernelGGL((k_join_long_stats<SBF, BBF>), dim3(n), dim3(kLong), 0, s, a); });
            hipLaunchKernelGGL((k_join_long_columns<SBF, BBF>), dim3(strips, (unsigned)a.n_parts), dim3(kTile), 0, s, a);
        });
    }
    constexpr int64_t kSpan = (int64_t)1 << 26;             // columns of a launch: fewer than 2^32 threads
    for (int64_t c0 = 0; (dwb || dwp) && c0 < j.cols; c0 += kSpan) {
        const int64_t n = j.cols - c0 < kSpan ? j.cols - c0 : kSpan;
        hipLaunchKernelGGL(k_join_sums, dim3((unsigned)((n + kSumCols - 1) / kSumCols), 2), dim3(kSumThreads), 0, s, a.parts, a.n_parts, j.cols, c0, dwb, dwp);
    }
    return hipGetLastError();
}

}  // namespace hwsel
