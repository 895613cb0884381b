// Dropout by a mask that is made from a counter: Y = residual + mask(X) / share.
#include "rows.hpp"

namespace hwsel {
namespace {

constexpr int kThreads = 256;

struct DropoutArgs {
    const void *X, *residual;
    void *Y;
    int64_t ldx, ldr, ldy, cols;
    uint32_t groups, items, row0;                           // of eight columns: a row's, all; the first row
    Dropout how;
};

// A thread has eight columns of a row.
template <bool XBF, bool YBF, bool RES>
__global__ __launch_bounds__(kThreads) void k_dropout(DropoutArgs a)
{
    const uint32_t i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= a.items) return;
    const Mask m = mask_of(a.how);
    const uint32_t row = i / a.groups, g = i - row * a.groups;
    const int64_t c = (int64_t)g * 8, n = a.cols - c;
    const Eight<XBF> x = load8<XBF>(a.X, (int64_t)row * a.ldx + c, n);
    Eight<YBF> r;
    if constexpr (RES) r = load8<YBF>(a.residual, (int64_t)row * a.ldr + c, n);
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = x.at(e);
    if (m.least != 0) drop8(m, a.row0 + row, g, v);
    if constexpr (RES) {
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] += r.at(e);
    }
    store8<YBF>(a.Y, (int64_t)row * a.ldy + c, n, v);
}

}  // namespace

hipError_t launch_dropout(const hwsel_dropout_t &how, int64_t rows, int64_t cols, const hwsel_matrix_t &X,
                          const hwsel_matrix_t &residual, const hwsel_matrix_t &Y, hipStream_t s)
{
    const bool xbf = X.dtype == HWSEL_DTYPE_BF16, ybf = Y.dtype == HWSEL_DTYPE_BF16;
    const int64_t groups = (cols + 7) / 8;
    const int64_t span = ((int64_t)1 << 31) / groups;       // rows of a launch: fewer than 2^32 threads
    auto at = [](const hwsel_matrix_t &m, int64_t row) {
        return static_cast<char *>(m.data) + (m.dtype == HWSEL_DTYPE_BF16 ? 2 : 4) * row * m.ld;
    };
    for (int64_t r0 = 0; r0 < rows; r0 += span) {
        const int64_t n = rows - r0 < span ? rows - r0 : span;
        DropoutArgs a{at(X, r0), residual.data ? at(residual, r0) : nullptr, at(Y, r0), X.ld, residual.ld, Y.ld, cols,
                      (uint32_t)groups, (uint32_t)(n * groups), (uint32_t)r0, dropout_of(how)};
        const dim3 grid((unsigned)((a.items + (kThreads - 1ull)) / kThreads));
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
