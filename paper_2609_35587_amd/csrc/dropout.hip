// Dropout by a mask that is made from a counter: Y = residual + mask(X) / share.
//
// One pass, bound by memory: 16 bytes of bf16 (32 of fp32) of a row a thread and group, whose eight numbers are one
// counter's, so the mask costs ten rounds for eight elements and no memory.  Measured on 65,536 x 1,024 in bf16 (134 MB read,
// 134 written): 45 us, 5.9 TB/s with the vector units busy 58 % of the time, most of it the rounds' 32 x 32-bit products; onto a residual 72 us,
// 5.6 TB/s.  (Calls over the same memory again and again: one group a thread 55 and 72 us, two 40 and 71.)  1 x 1,024 takes
// 1.8 us, a launch.
#include "rows.hpp"

namespace hwsel {
namespace {

constexpr int kThreads = 256;

// i / d for i < 2^31 by a product: (i + high word of i m) >> s, 2^s the power of two from d on and m = 2^32 (2^s - d) / d + 1
// (Granlund and Montgomery, 1994).
struct Divisor {
    uint32_t d, m, s;
    explicit Divisor(uint32_t d_) : d(d_), m(0), s(0)
    {
        while (((uint64_t)1 << s) < d) ++s;
        m = (uint32_t)((((uint64_t)1 << 32) * (((uint64_t)1 << s) - d)) / d + 1);
    }
    __device__ __forceinline__ uint32_t of(uint32_t i) const { return (__umulhi(i, m) + i) >> s; }
};

struct DropoutArgs {
    const void *X, *residual;
    void *Y;
    int64_t ldx, ldr, ldy;
    int32_t cols;
    Ends ends;
    Divisor groups;                                         // of eight columns, in a row
    uint32_t items, row0;                                   // all groups; the first row
    Dropout how;
};

constexpr int kEach = 2;                                    // groups of a thread, their loads on the way together

template <bool XBF, bool YBF, bool RES>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutArgs a)
{
    const Mask m = mask_of(a.how);
    uint32_t row[kEach], g[kEach];
    int32_t n[kEach];
    Eight<XBF> x[kEach];
    Eight<YBF> r[kEach];
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        const uint32_t i = (blockIdx.x * kEach + k) * kThreads + threadIdx.x;
        row[k] = a.groups.of(i);
        g[k] = i - row[k] * a.groups.d;
        const int32_t c = (int32_t)g[k] * 8;
        n[k] = i < a.items ? a.cols - c : 0;
        x[k] = load8<XBF>(a.X, (int64_t)row[k] * a.ldx + c, n[k], a.ends);
        if constexpr (RES) r[k] = load8<YBF>(a.residual, (int64_t)row[k] * a.ldr + c, n[k], a.ends);
    }
#pragma unroll
    for (int k = 0; k < kEach; ++k) {
        settle8(x[k], n[k], a.ends);
        if constexpr (RES) settle8(r[k], n[k], a.ends);
        float v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = x[k].at(e);
        if (m.least != 0) drop8(m, a.row0 + row[k], g[k], v);
        if constexpr (RES) {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] += r[k].at(e);
        }
        store8<YBF>(a.Y, (int64_t)row[k] * a.ldy + (int64_t)g[k] * 8, n[k], a.ends, v);
    }
}

}  // namespace

hipError_t launch_dropout(const hwsel_dropout_t &how, int64_t rows, int64_t cols, const hwsel_matrix_t &X,
                          const hwsel_matrix_t &residual, const hwsel_matrix_t &Y, hipStream_t s)
{
    const bool xbf = X.dtype == HWSEL_DTYPE_BF16, ybf = Y.dtype == HWSEL_DTYPE_BF16;
    const int64_t groups = (cols + 7) / 8;
    const int64_t span = (((int64_t)1 << 31) - kEach * kThreads) / groups;   // rows of a launch: fewer than 2^31 groups
    auto at = [](const hwsel_matrix_t &m, int64_t row) {
        return static_cast<char *>(m.data) + (m.dtype == HWSEL_DTYPE_BF16 ? 2 : 4) * row * m.ld;
    };
    for (int64_t r0 = 0; r0 < rows; r0 += span) {
        const int64_t n = rows - r0 < span ? rows - r0 : span;
        DropoutArgs a{at(X, r0), residual.data ? at(residual, r0) : nullptr, at(Y, r0), X.ld, residual.ld, Y.ld, (int32_t)cols, ends_of(cols),
                      Divisor((uint32_t)groups), (uint32_t)(n * groups), (uint32_t)r0, dropout_of(how)};
        const dim3 grid((unsigned)((a.items + (kEach * kThreads - 1ull)) / (kEach * kThreads)));
        auto go = [&](auto *kernel) { hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, s, a); };
        if (residual.data) {
            if (xbf) ybf ? go(k_dropout<true, true, true>) : go(k_dropout<true, false, true>);
            else ybf ? go(k_dropout<false, true, true>) : go(k_dropout<false, false, true>);
        } else {
            if (xbf) ybf ? go(k_dropout<true, true, false>) : go(k_dropout<true, false, false>);
            else ybf ? go(k_dropout<false, true, false>) : go(k_dropout<false, false, false>);
        }
    }
    return hipGetLastError();
}

}  // namespace hwsel
