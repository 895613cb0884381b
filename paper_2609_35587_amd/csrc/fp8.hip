// 8-bit matrices with block scales: quantising (rows, 128 x 128 blocks,
// transposed), restoring, and transposing what is already in 8 bits.
//
// For a block of 128 elements (or 128 x 128) with largest finite magnitude
// amax: e = the least exponent with amax <= max_code 2^e, q = rne(x 2^-e).
// All are bound by HBM: every element is read once and its code written once.
#include "fp8.hpp"

namespace hwsel {
namespace {

constexpr int kThreads = 256;

// Eight consecutive elements of a row, zeros from column C on.
template <bool BF16>
__device__ __forceinline__ void load8(const void *X, int64_t row_at, int64_t c0, int64_t C, float (&v)[8])
{
    if (c0 + 8 <= C) {
        if constexpr (BF16) {
            const u32x4_any_t w = *reinterpret_cast<const u32x4_any_t *>(static_cast<const uint16_t *>(X) + row_at + c0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                v[2 * i] = __uint_as_float(w[i] << 16);
                v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
            }
        } else {
            const f32x4_any_t *at = reinterpret_cast<const f32x4_any_t *>(static_cast<const float *>(X) + row_at + c0);
            const f32x4_any_t a = at[0], b = at[1];
            v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
            v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        v[i] = 0.0f;
        if (c0 + i < C) {
            if constexpr (BF16) v[i] = bf16_value(static_cast<const uint16_t *>(X)[row_at + c0 + i]);
            else v[i] = static_cast<const float *>(X)[row_at + c0 + i];
        }
    }
}

// A scale for each row's 128 columns.  Sixteen lanes share a block, eight
// elements each, and find its maximum by rotations; a wave takes 4 / KBW rows
// of KBW blocks at once, kRowsInFlight times.  Bound by HBM: 4.9 M x 128 fp32
// standardised 534 us, 5.9 TB/s (means read singly and a byte stored of each
// row's word: 814; workgroups that go through many steps: 600).
constexpr int kRowsInFlight = 2;

template <bool BF16, bool STD, int KBW>
__global__ __launch_bounds__(kThreads) void k_quantise_rows(const void *__restrict__ X, int64_t ld, const float *__restrict__ mean,
                                                             const float *__restrict__ inv_std, hwsel_fp8_t out)
{
    constexpr int kRows = 4 / KBW;                          // rows of one wave step
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t kb = (int64_t)blockIdx.y * KBW + (lane >> 4) % KBW;
    const bool in_block = kb < (out.cols + kFp8Block - 1) / kFp8Block;
    const int64_t c0 = kb * kFp8Block + (lane & 15) * 8;
    float mu[8], is[8];
    if constexpr (STD) {
        typedef float f32x8u_t __attribute__((ext_vector_type(8), aligned(4)));
        if (c0 + 8 <= out.cols) {
            const f32x8u_t a = *reinterpret_cast<const f32x8u_t *>(mean + c0), b = *reinterpret_cast<const f32x8u_t *>(inv_std + c0);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                mu[i] = a[i];
                is[i] = b[i];
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                mu[i] = c0 + i < out.cols ? mean[c0 + i] : 0.0f;
                is[i] = c0 + i < out.cols ? inv_std[c0 + i] : 0.0f;
            }
        }
    }
    constexpr int64_t kStep = 4 * kRows * kRowsInFlight;    // rows of a workgroup step
    for (int64_t r0 = (int64_t)blockIdx.x * kStep; r0 < out.rows; r0 += (int64_t)gridDim.x * kStep) {
        float v[kRowsInFlight][8];
        const int64_t first = r0 + (int64_t)wave * kRows * kRowsInFlight + (lane >> 4) / KBW;
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int64_t r = first + j * kRows;            // (past the end the last row again: its codes are not stored)
            load8<BF16>(X, (r < out.rows ? r : out.rows - 1) * ld, c0, out.cols, v[j]);
        }
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int64_t r = first + j * kRows;
            uint32_t m = 0, all = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                if constexpr (STD) {
                    const float x = __builtin_isfinite(v[j][i]) ? v[j][i] : 0.0f;
                    v[j][i] = c0 + i < out.cols ? __fmul_rn(__fsub_rn(x, mu[i]), is[i]) : 0.0f;
                }
                const uint32_t a = __float_as_uint(v[j][i]) & 0x7fffffffu, f = a < 0x7f800000u ? a : 0u;
                all = a > all ? a : all;
                m = f > m ? f : m;
            }
            const bool odd = all >= 0x7f800000u;
            const uint32_t byte = scale_byte(row16_max(m), out.format);
            if (r < out.rows && in_block) {
                const float s = inverse_scale(byte);
                const uint2 w = make_uint2(codes4_checked(&v[j][0], s, out.format, odd),
                                           codes4_checked(&v[j][4], s, out.format, odd));
                *reinterpret_cast<uint2 *>(out.q + r * out.ld + c0) = w;
                if ((lane & 15) == 0) {
                    uint8_t *at = out.scale + r * out.ld_scale + kb;
                    if constexpr (KBW == 1) *reinterpret_cast<uint32_t *>(at) = byte;  // (the row's only block: its word whole)
                    else *at = (uint8_t)byte;
                }
            }
        }
    }
}

// What a tile of 128 rows by 128 columns is read from.
enum class Source { fp32, bf16, fp8 };

struct TileIn {
    const void *X;
    int64_t rows, cols, ld;
    const uint8_t *scale;                                   // of an 8-bit source
    int64_t ld_scale;
    int32_t format, block_rows;
};

// Four columns of sixteen rows in fp32 or bf16, zeros outside.
template <Source S>
__device__ __forceinline__ void load16x4(const TileIn &in, int64_t r0, int64_t c, float (&v)[16][4])
{
    if (c + 4 <= in.cols) {                                 // all on their way at once; the last row again past the end
#pragma unroll
        for (int j = 0; j < 16; ++j) {
            const int64_t at = (r0 + j < in.rows ? r0 + j : in.rows - 1) * in.ld + c;
            if constexpr (S == Source::fp32) {
                const f32x4_any_t w = *reinterpret_cast<const f32x4_any_t *>(static_cast<const float *>(in.X) + at);
                v[j][0] = w.x; v[j][1] = w.y; v[j][2] = w.z; v[j][3] = w.w;
            } else {
                const u32x2_any_t w = *reinterpret_cast<const u32x2_any_t *>(static_cast<const uint16_t *>(in.X) + at);
                v[j][0] = __uint_as_float(w.x << 16);
                v[j][1] = __uint_as_float(w.x & 0xffff0000u);
                v[j][2] = __uint_as_float(w.y << 16);
                v[j][3] = __uint_as_float(w.y & 0xffff0000u);
            }
        }
        if (r0 + 16 > in.rows) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[j][i] = r0 + j < in.rows ? v[j][i] : 0.0f;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 16; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v[j][i] = 0.0f;
            if (r0 + j < in.rows && c + i < in.cols) {
                if constexpr (S == Source::fp32) v[j][i] = static_cast<const float *>(in.X)[(r0 + j) * in.ld + c + i];
                else v[j][i] = bf16_value(static_cast<const uint16_t *>(in.X)[(r0 + j) * in.ld + c + i]);
            }
        }
}

// A workgroup takes tiles of 128 x 128; a thread has 16 rows of four columns,
// so that a column's codes are 16 bytes of an output row when TRANSPOSED.  The
// codes then go through LDS (rows 144 bytes apart) to be stored as whole lines.
// BLOCK: one scale for the tile, else one for each of its columns (TRANSPOSED).
template <Source S, bool TRANSPOSED, bool BLOCK>
__global__ __launch_bounds__(kThreads) void k_quantise_tiles(TileIn in, hwsel_fp8_t out)
{
    static_assert(TRANSPOSED || BLOCK, "rows have their own kernel");
    constexpr int kRow = 144;
    __shared__ uint32_t part[8][128];
    __shared__ __attribute__((aligned(16))) uint8_t lds[TRANSPOSED ? 128 * kRow : 16];
    __shared__ __attribute__((aligned(16))) float row_scale[S == Source::fp8 ? 128 : 4];
    const int64_t n_ct = (in.cols + 127) / 128, n_tiles = (in.rows + 127) / 128 * n_ct;
    const int c4 = (threadIdx.x & 31) * 4, group = threadIdx.x >> 5;
    for (int64_t tile = blockIdx.x; tile < n_tiles; tile += gridDim.x) {
        const int64_t rt = tile / n_ct, ct = tile % n_ct, c = ct * 128 + c4;
        float v[16][4];
        if constexpr (S == Source::fp8) {
            // sixteen loads on their way at once, from the last row where the tile goes past it; rows are
            // padded with zeros to whole blocks, so four codes can always be read
            const uint8_t *q = static_cast<const uint8_t *>(in.X) + c;
            const int64_t r0 = rt * 128 + 16 * group;
            int w[16];
#pragma unroll
            for (int j = 0; j < 16; ++j)
                w[j] = *reinterpret_cast<const int *>(q + (r0 + j < in.rows ? r0 + j : in.rows - 1) * in.ld);
            if (threadIdx.x < 128) {
                int64_t r = rt * 128 + threadIdx.x;
                r = r < in.rows ? r : in.rows - 1;
                row_scale[threadIdx.x] = scale_value(in.scale[(in.block_rows == 1 ? r : rt) * in.ld_scale + ct]);
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const float s = row_scale[16 * group + j];
                const int u = r0 + j < in.rows ? w[j] : 0;
                f32x2_t a, b;
                if (in.format == HWSEL_FP8_E4M3) {
                    a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false);
                    b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                } else {
                    a = __builtin_amdgcn_cvt_pk_f32_bf8(u, false);
                    b = __builtin_amdgcn_cvt_pk_f32_bf8(u, true);
                }
                v[j][0] = a.x * s; v[j][1] = a.y * s; v[j][2] = b.x * s; v[j][3] = b.y * s;
            }
        } else {
            load16x4<S>(in, rt * 128 + 16 * group, c, v);
        }
        uint32_t m[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t a = __float_as_uint(v[j][i]) & 0x7fffffffu;
                m[i] = a > m[i] ? a : m[i];
            }
        const bool odd = (m[0] > m[1] ? m[0] : m[1]) >= 0x7f800000u || (m[2] > m[3] ? m[2] : m[3]) >= 0x7f800000u;
        if (odd) {                                          // scales go by the finite elements
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                m[i] = 0;
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    const uint32_t f = finite_bits(v[j][i]);
                    m[i] = f > m[i] ? f : m[i];
                }
            }
        }
        *reinterpret_cast<uint4 *>(&part[group][c4]) = make_uint4(m[0], m[1], m[2], m[3]);
        __syncthreads();
        uint32_t byte[4];
        if constexpr (BLOCK) {
            uint32_t most = 0;
            for (int g = 0; g < 8; ++g) {
                const uint32_t a = part[g][threadIdx.x & 63], b = part[g][64 + (threadIdx.x & 63)];
                most = a > most ? a : most;
                most = b > most ? b : most;
            }
            most = row16_max(most);
#pragma unroll
            for (int l = 16; l < 64; l <<= 1) {
                const uint32_t o = (uint32_t)__shfl_xor((int)most, l);
                most = o > most ? o : most;
            }
            byte[0] = byte[1] = byte[2] = byte[3] = scale_byte(most, out.format);
        } else {
#pragma unroll
            for (int g = 0; g < 8; ++g) {
                const uint4 w = *reinterpret_cast<const uint4 *>(&part[g][c4]);
                m[0] = w.x > m[0] ? w.x : m[0];
                m[1] = w.y > m[1] ? w.y : m[1];
                m[2] = w.z > m[2] ? w.z : m[2];
                m[3] = w.w > m[3] ? w.w : m[3];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) byte[i] = scale_byte(m[i], out.format);
        }
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float s = inverse_scale(byte[i]);
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const float x[4] = {v[4 * q][i], v[4 * q + 1][i], v[4 * q + 2][i], v[4 * q + 3][i]};
                    w[q] = codes4_checked(x, s, out.format, odd);
                }
                *reinterpret_cast<uint4 *>(lds + (c4 + i) * kRow + 16 * group) = make_uint4(w[0], w[1], w[2], w[3]);
                if (!BLOCK && group == 0 && c + i < in.cols) out.scale[(c + i) * out.ld_scale + rt] = (uint8_t)byte[i];
            }
            if (BLOCK && threadIdx.x == 0) out.scale[ct * out.ld_scale + rt] = (uint8_t)byte[0];
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int row = (threadIdx.x >> 3) + 32 * j;
                if (ct * 128 + row < out.rows)
                    *reinterpret_cast<uint4 *>(out.q + (ct * 128 + row) * out.ld + rt * 128 + (threadIdx.x & 7) * 16) =
                        *reinterpret_cast<const uint4 *>(lds + row * kRow + (threadIdx.x & 7) * 16);
            }
            __syncthreads();
        } else {
            const float s = inverse_scale(byte[0]);
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                const int64_t r = rt * 128 + 16 * group + j;
                if (r < out.rows)
                    *reinterpret_cast<uint32_t *>(out.q + r * out.ld + c) = codes4_checked(v[j], s, out.format, odd);
            }
            if (threadIdx.x == 0) out.scale[rt * out.ld_scale + ct] = (uint8_t)byte[0];
            __syncthreads();
        }
    }
}

// Sixteen lanes a block, eight elements each.
template <bool BF16, int KBW>
__global__ __launch_bounds__(kThreads) void k_dequantise(hwsel_fp8_t in, void *__restrict__ X, int64_t ld)
{
    constexpr int kRows = 4 / KBW;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int64_t kb = (int64_t)blockIdx.y * KBW + (lane >> 4) % KBW;
    const int64_t c0 = kb * kFp8Block + (lane & 15) * 8;
    if (c0 >= in.cols) return;
    constexpr int64_t kStep = 4 * kRows * kRowsInFlight;
    for (int64_t r0 = (int64_t)blockIdx.x * kStep; r0 < in.rows; r0 += (int64_t)gridDim.x * kStep) {
        const int64_t first = r0 + (int64_t)wave * kRows * kRowsInFlight + (lane >> 4) / KBW;
        uint2 w[kRowsInFlight];
        uint32_t byte[kRowsInFlight];
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int64_t r = first + j * kRows < in.rows ? first + j * kRows : in.rows - 1;
            w[j] = *reinterpret_cast<const uint2 *>(in.q + r * in.ld + c0);
            byte[j] = in.scale[(in.block_rows == 1 ? r : r / kFp8Block) * in.ld_scale + kb];
        }
#pragma unroll
        for (int j = 0; j < kRowsInFlight; ++j) {
            const int64_t r = first + j * kRows;
            if (r >= in.rows) continue;
            const float s = scale_value(byte[j]);
            float v[8];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int u = (int)(h ? w[j].y : w[j].x);
                f32x2_t a, b;
                if (in.format == HWSEL_FP8_E4M3) {
                    a = __builtin_amdgcn_cvt_pk_f32_fp8(u, false);
                    b = __builtin_amdgcn_cvt_pk_f32_fp8(u, true);
                } else {
                    a = __builtin_amdgcn_cvt_pk_f32_bf8(u, false);
                    b = __builtin_amdgcn_cvt_pk_f32_bf8(u, true);
                }
                v[4 * h] = a.x * s;
                v[4 * h + 1] = a.y * s;
                v[4 * h + 2] = b.x * s;
                v[4 * h + 3] = b.y * s;
            }
            if (c0 + 8 <= in.cols) {
                if constexpr (BF16) {
                    *reinterpret_cast<u32x4_any_t *>(static_cast<uint16_t *>(X) + r * ld + c0) =
                        (u32x4_any_t){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
                } else {
                    f32x4_any_t *at = reinterpret_cast<f32x4_any_t *>(static_cast<float *>(X) + r * ld + c0);
                    at[0] = (f32x4_any_t){v[0], v[1], v[2], v[3]};
                    at[1] = (f32x4_any_t){v[4], v[5], v[6], v[7]};
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (c0 + i < in.cols) {
                        if constexpr (BF16) static_cast<uint16_t *>(X)[r * ld + c0 + i] = (uint16_t)bf16_pair(v[i], 0.0f);
                        else static_cast<float *>(X)[r * ld + c0 + i] = v[i];
                    }
            }
        }
    }
}

// Workgroups of a launch: enough for every row step, at most 2^20 in all (the
// kernels step on by the grid's size).
unsigned row_groups(int64_t rows, int64_t step, int64_t chunks)
{
    const int64_t most = (int64_t)(1 << 20) / chunks > 1 ? (1 << 20) / chunks : 1, n = (rows + step - 1) / step;
    return (unsigned)(n < most ? n : most);
}

template <class F>
void by_blocks(int64_t nkb, F &&f)
{
    if (nkb == 1) f(std::integral_constant<int, 1>{});
    else if (nkb == 2) f(std::integral_constant<int, 2>{});
    else f(std::integral_constant<int, 4>{});
}

template <Source S>
void launch_tiles(const TileIn &in, bool transposed, const hwsel_fp8_t &out, hipStream_t s)
{
    const int64_t n = (in.rows + 127) / 128 * ((in.cols + 127) / 128);
    const dim3 grid((unsigned)(n < (1 << 20) ? n : 1 << 20)), block(kThreads);
    if (!transposed) hipLaunchKernelGGL((k_quantise_tiles<S, false, true>), grid, block, 0, s, in, out);
    else if (out.block_rows == 1) hipLaunchKernelGGL((k_quantise_tiles<S, true, false>), grid, block, 0, s, in, out);
    else hipLaunchKernelGGL((k_quantise_tiles<S, true, true>), grid, block, 0, s, in, out);
}

}  // namespace

hipError_t launch_fp8_quantise(const void *X, bool bf16, int64_t ld, bool transposed, const float *mean,
                               const float *inv_std, const hwsel_fp8_t &out, hipStream_t s)
{
    if (transposed || out.block_rows != 1) {
        const TileIn in{X, transposed ? out.cols : out.rows, transposed ? out.rows : out.cols, ld, nullptr, 0, 0, 1};
        if (bf16) launch_tiles<Source::bf16>(in, transposed, out, s);
        else launch_tiles<Source::fp32>(in, transposed, out, s);
        return hipGetLastError();
    }
    by_blocks(fp8_blocks(out.cols), [&](auto kbw) {
        constexpr int KBW = decltype(kbw)::value;
        const int64_t chunks = (fp8_blocks(out.cols) + KBW - 1) / KBW;
        const dim3 grid(row_groups(out.rows, 4 * (4 / KBW) * kRowsInFlight, chunks), (unsigned)chunks), block(kThreads);
        if (mean && bf16) hipLaunchKernelGGL((k_quantise_rows<true, true, KBW>), grid, block, 0, s, X, ld, mean, inv_std, out);
        else if (mean) hipLaunchKernelGGL((k_quantise_rows<false, true, KBW>), grid, block, 0, s, X, ld, mean, inv_std, out);
        else if (bf16) hipLaunchKernelGGL((k_quantise_rows<true, false, KBW>), grid, block, 0, s, X, ld, mean, inv_std, out);
        else hipLaunchKernelGGL((k_quantise_rows<false, false, KBW>), grid, block, 0, s, X, ld, mean, inv_std, out);
    });
    return hipGetLastError();
}

hipError_t launch_fp8_transpose(const hwsel_fp8_t &in, const hwsel_fp8_t &out, hipStream_t s)
{
    const TileIn t{in.q, in.rows, in.cols, in.ld, in.scale, in.ld_scale, in.format, in.block_rows};
    launch_tiles<Source::fp8>(t, true, out, s);
    return hipGetLastError();
}

hipError_t launch_fp8_dequantise(const hwsel_fp8_t &in, void *X, bool bf16, int64_t ld, hipStream_t s)
{
    by_blocks(fp8_blocks(in.cols), [&](auto kbw) {
        constexpr int KBW = decltype(kbw)::value;
        const int64_t chunks = (fp8_blocks(in.cols) + KBW - 1) / KBW;
        const dim3 grid(row_groups(in.rows, 4 * (4 / KBW) * kRowsInFlight, chunks), (unsigned)chunks), block(kThreads);
        if (bf16) hipLaunchKernelGGL((k_dequantise<true, KBW>), grid, block, 0, s, in, X, ld);
        else hipLaunchKernelGGL((k_dequantise<false, KBW>), grid, block, 0, s, in, X, ld);
    });
    return hipGetLastError();
}

}  // namespace hwsel
