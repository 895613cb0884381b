// Products of 8-bit matrices with block scales, C = act(A B^T + bias).
//
// v_mfma_scale_f32_16x16x128_f8f6f4 multiplies 16 x 128 by 128 x 16 codes and
// scales each row of either by a power of two as it does so; one instruction
// covers exactly one block of 128, so the scales cost no arithmetic and the
// sums run on in fp32 accumulators over all of K.  The weights (B) are the
// instruction's first operand: a lane then holds four consecutive columns n
// of one row m of C.
//
// Within the instruction the products of eight neighbouring k are aligned to
// the largest of them and kept to 2^-13 of it (measured: one product 2^-14 of
// its neighbour's is lost, one eight places on is not; the groups are added as
// fp32 sums are).  On random data that is 1.5e-5 of the result's norm, a
// hundredth of a bf16 rounding, and of no account for one result in bf16 or 8
// bits (through a layer re-quantised to 8 bits, where it moves values across the
// boundaries of codes, the next result is off by 0.00195 of its norm, with fp32
// sums by 0.00166).  For results in fp32 it would be a hundred times their rounding: they
// take the bf16 instruction instead (EXACT), whose sums are fp32's, on codes
// decoded and scaled in registers, at half the rate.
#include "fp8.hpp"

namespace hwsel {
namespace {

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef int i32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));

enum OutKind { kOutF32, kOutBf16, kOutFp8, kOutPart };

// What becomes of a sum.
struct Out {
    void *C;                                                // fp32, bf16 or codes; partial sums
    int64_t ld;
    uint8_t *scale;
    int64_t ld_scale;
    const float *bias;
    int32_t gelu;
};

struct Operand {
    const uint8_t *q;
    int64_t ld;
    const uint8_t *scale;
    int64_t ld_scale;
    int32_t rows, shift;                                    // shift: rows >> shift is a row's scale row
};

// GELU(a) = max(a, 0) - |a| Phi(-|a|), Phi(-x) = 2^P(x) for x >= 0 with the
// polynomial P of degree 5 fitted on [0, 5] by gelu_fit.py: |error| <= 7e-7 for
// every finite a, near the rounding of an fp32 sum of a few hundred terms.
// Past the fitted range P keeps falling and the result is max(a, 0); the
// maximum is the one that keeps a NaN, and |a| stops at 64, where 2^P is 0, so
// that an infinity meets no 0 times infinity.  Nine instructions.
__device__ __forceinline__ float gelu_fine(float a)
{
    constexpr float c5 = -0.00047442156937904656f, c4 = 0.007105245254933834f, c3 = -0.0519152507185936f,
                    c2 = -0.45985135436058044f, c1 = -1.1508772373199463f, c0 = -1.000020146369934f;
    const float x = __builtin_amdgcn_fmed3f(fabsf(a), 0.0f, 64.0f);
    float p = fmaf(c5, x, c4);
    p = fmaf(p, x, c3);
    p = fmaf(p, x, c2);
    p = fmaf(p, x, c1);
    p = fmaf(p, x, c0);
    return fmaf(-x, __builtin_amdgcn_exp2f(p), __builtin_elementwise_maximum(a, 0.0f));
}

// The same with degree 4 and |a| up to 5.5, where 2^P is 2e-8: |error| <= 8.4e-6,
// for results in bf16 and 8 bits, where it is no more than the products' own
// (see above) and an instruction in eleven is worth having: with the longer one
// two layers of 4.9 M rows take 3.41 ms instead of 3.36, and their result is off
// by 0.001942 of its norm instead of 0.001945.
__device__ __forceinline__ float gelu_short(float a)
{
    constexpr float c4 = 0.00369689567014575f, c3 = -0.04334138706326485f, c2 = -0.4690028131008148f,
                    c1 = -1.146939754486084f, c0 = -1.000515103340149f;
    const float x = __builtin_amdgcn_fmed3f(fabsf(a), 0.0f, 5.5f);
    float p = fmaf(c4, x, c3);
    p = fmaf(p, x, c2);
    p = fmaf(p, x, c1);
    p = fmaf(p, x, c0);
    return fmaf(-x, __builtin_amdgcn_exp2f(p), __builtin_elementwise_maximum(a, 0.0f));
}

template <OutKind KIND>
__device__ __forceinline__ float gelu(float a) { return KIND == kOutF32 ? gelu_fine(a) : gelu_short(a); }

// v[i] = act(v[i] + bias[n + i]); columns from N on are set to 0.
template <OutKind KIND>
__device__ __forceinline__ void finish4(const Out &o, int32_t n, int32_t N, float (&v)[4])
{
    if (o.bias) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (n + i < N) v[i] += o.bias[n + i];
    }
    if (o.gelu) {
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = gelu<KIND>(v[i]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = n + i < N ? v[i] : 0.0f;
}

template <OutKind KIND>
__device__ __forceinline__ void store4(const Out &o, int64_t m, int32_t n, int32_t N, const float (&v)[4])
{
    static_assert(KIND == kOutF32 || KIND == kOutBf16 || KIND == kOutPart, "codes have their own way");
    if (n >= N) return;
    if constexpr (KIND == kOutBf16) {
        uint16_t *at = static_cast<uint16_t *>(o.C) + m * o.ld + n;
        const uint32_t a = bf16_pair(v[0], v[1]), b = bf16_pair(v[2], v[3]);
        if (n + 4 <= N) {
            *reinterpret_cast<u32x2_any_t *>(at) = (u32x2_any_t){a, b};
        } else {
            at[0] = (uint16_t)a;
            if (n + 1 < N) at[1] = (uint16_t)(a >> 16);
            if (n + 2 < N) at[2] = (uint16_t)b;
            if (n + 3 < N) at[3] = (uint16_t)(b >> 16);
        }
    } else {
        float *at = static_cast<float *>(o.C) + m * o.ld + n;
        if (KIND == kOutPart || n + 4 <= N) {
            *reinterpret_cast<f32x4_any_t *>(at) = (f32x4_any_t){v[0], v[1], v[2], v[3]};
        } else {
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if (n + i < N) at[i] = v[i];
        }
    }
}

// 1,024 bytes (8 rows of 128) from rows r0.. of a tile to LDS at `to`: lane i
// brings 16-byte chunk (i % 8) ^ swizzle of row r0 + i / 8 to place i.  With
// chunks swizzled by (row / 2) % 8, the 16 rows that a fragment read touches
// at one logical chunk lie on 16 different 16-byte bank groups.  Rows past the
// end read the last one: what they give is not stored.
__device__ __forceinline__ uint32_t lds_source(int r0, int lane, int32_t rows_left, int64_t ld)
{
    const int row = r0 + (lane >> 3), chunk = (lane & 7) ^ ((row >> 1) & 7);
    return __umul24((uint32_t)(row < rows_left ? row : rows_left - 1), (uint32_t)ld) + chunk * 16;
}

// The codes from a tile's first row on as a buffer: its base and the step along
// K stay in scalar registers.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t tile_buffer(const uint8_t *base)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t *>(base), 0, 0xffffffff, 0x00027000);
}

__device__ __forceinline__ void to_lds(__amdgpu_buffer_rsrc_t tile, uint32_t offset, uint32_t k, uint8_t *to)
{
    __builtin_amdgcn_raw_ptr_buffer_load_lds(tile, (__attribute__((address_space(3))) void *)to, 16, offset, k, 0, 0);
}

// One word a lane to LDS.
__device__ __forceinline__ void word_to_lds(const uint8_t *from, uint8_t *to)
{
    __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void *)from,
                                     (__attribute__((address_space(3))) void *)to, 4, 0, 0);
}

// A fragment: 32 bytes of row lane % 16, chunks lane / 16 and lane / 16 + 4 (any
// pairing of k serves, if it is the same for both operands).
__device__ __forceinline__ i32x8_t fragment(const uint8_t *tile, int lane)
{
    const int row = lane & 15, sw = (row >> 1) & 7, g = lane >> 4;
    const i32x4_t a = *reinterpret_cast<const i32x4_t *>(tile + row * 128 + ((g ^ sw) << 4));
    const i32x4_t b = *reinterpret_cast<const i32x4_t *>(tile + row * 128 + (((g ^ sw) ^ 4) << 4));
    return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// A fragment's 32 codes as bf16 values, scaled by 2^(lowest byte of scale - 127).
// The instruction goes by the exponent bits of its scale alone: 0 is 2^-127 and
// 255 gives NaN (measured), as the format has it.  (Decoding the next fragment
// between this one's products, an instruction to each: 3% slower.)
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

template <int FMT>
__device__ __forceinline__ void decode(const i32x8_t &x, uint32_t scale, bf16x8_t (&out)[4])
{
    const float s = __uint_as_float((scale & 0xffu) << 23);
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        bf16x2_t v[4];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t w = (uint32_t)x[2 * q + h];
            if constexpr (FMT == 0) {
                v[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, false);
                v[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, s, true);
            } else {
                v[2 * h] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, false);
                v[2 * h + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, s, true);
            }
        }
        const auto lo = __builtin_shufflevector(v[0], v[1], 0, 1, 2, 3), hi = __builtin_shufflevector(v[2], v[3], 0, 1, 2, 3);
        out[q] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    }
}

// The scale bytes of blocks 4 j .. 4 j + 3 of a row, the first lowest.
__device__ __forceinline__ uint32_t scale_word(const Operand &x, int32_t row, int32_t kb)
{
    const int32_t r = row < x.rows ? row : x.rows - 1;
    return *reinterpret_cast<const uint32_t *>(x.scale + (int64_t)(r >> x.shift) * x.ld_scale + (kb & ~3));
}

// Four registers seen by the four groups of 16 lanes as a 4 x 4 matrix, transposed:
// x[j] of group g becomes x[g] of group j.
__device__ __forceinline__ void transpose_groups(uint32_t &a, uint32_t &b, uint32_t &c, uint32_t &d)
{
    const auto ac = __builtin_amdgcn_permlane32_swap(a, c, false, false), bd = __builtin_amdgcn_permlane32_swap(b, d, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(ac[0], bd[0], false, false),
               hi = __builtin_amdgcn_permlane16_swap(ac[1], bd[1], false, false);
    a = lo[0];
    b = lo[1];
    c = hi[0];
    d = hi[1];
}

// Maximum over the four groups of 16 lanes, in every lane, of bits of floats >= 0.
__device__ __forceinline__ uint32_t groups_max(uint32_t v)
{
    const auto h = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    const uint32_t m = h[0] > h[1] ? h[0] : h[1];
    const auto q = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    return q[0] > q[1] ? q[0] : q[1];
}

// The sums' first values: the bias, for a product that ends in this launch.
template <int MT, OutKind KIND>
__device__ __forceinline__ void start_tiles(f32x4_t (&acc)[MT][8], int32_t n0, int32_t N, const Out &o, int lane)
{
    const int32_t n_lane = n0 + 4 * (lane >> 4);
#pragma unroll
    for (int nt = 0; nt < 8; ++nt) {
        f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (KIND != kOutPart && o.bias) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int32_t n = n_lane + 16 * nt + i;
                v[i] = o.bias[n < N ? n : N - 1];
            }
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) acc[mt][nt] = v;
    }
}

// What becomes of a wave's MT x 8 tiles, rows from m0, columns from n0 (a whole
// block).  Lane l, element i of a tile: row m = l % 16, column n = 4 (l / 16) + i.
// The lanes of a row exchange what they hold so that each stores 16 bytes.
template <int MT, OutKind KIND>
__device__ __forceinline__ void finish_tiles(const f32x4_t (&acc)[MT][8], int32_t m0, int32_t n0, int32_t M, int32_t N,
                                             int32_t split, const Out &o, int lane)
{
    constexpr int NT = 8;
    if (n0 >= N || m0 >= M) return;                         // (the whole wave)
    const int32_t g = lane >> 4, n_lane = n0 + 4 * g;
    const bool whole = n0 + 128 <= N;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int32_t m = m0 + 16 * mt + (lane & 15);
        float v[NT][4];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int i = 0; i < 4; ++i) v[nt][i] = acc[mt][nt][i];
        if (KIND != kOutPart && o.gelu) {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int i = 0; i < 4; ++i) v[nt][i] = gelu<KIND>(v[nt][i]);
        }
        if constexpr (KIND == kOutFp8) {
            if (!whole) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[nt][i] = n_lane + 16 * nt + i < N ? v[nt][i] : 0.0f;
            }
            float most = 0.0f;                              // (NaN do not count)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                most = fmaxf(fmaxf(fabsf(v[nt][0]), fabsf(v[nt][1])), most);
                most = fmaxf(fmaxf(fabsf(v[nt][2]), fabsf(v[nt][3])), most);
            }
            const uint32_t top = groups_max(__float_as_uint(most));
            uint32_t w[NT], byte;
            if (__any(top == 0x7f800000u)) {                // infinities do not count either
                uint32_t bits = 0;
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t f = finite_bits(v[nt][i]);
                        bits = f > bits ? f : bits;
                    }
                byte = scale_byte(groups_max(bits), HWSEL_FP8_E4M3);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) w[nt] = codes4_checked(v[nt], inverse_scale(byte), HWSEL_FP8_E4M3, true);
            } else {
                byte = scale_byte(top, HWSEL_FP8_E4M3);
                const float s = __uint_as_float(byte << 23);
#pragma unroll
                for (int nt = 0; nt < NT; ++nt) w[nt] = scaled_codes4(v[nt], s);
            }
            transpose_groups(w[0], w[1], w[2], w[3]);
            transpose_groups(w[4], w[5], w[6], w[7]);
            if (m < M) {
                uint8_t *at = static_cast<uint8_t *>(o.C) + (int64_t)m * o.ld + n0 + 16 * g;
                *reinterpret_cast<uint4 *>(at) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4 *>(at + 64) = make_uint4(w[4], w[5], w[6], w[7]);
                if (g == 0) o.scale[(int64_t)m * o.ld_scale + (n0 >> 7)] = (uint8_t)byte;
            }
        } else if (KIND == kOutBf16 && whole) {
            uint32_t lo[NT], hi[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                lo[nt] = bf16_pair(v[nt][0], v[nt][1]);
                hi[nt] = bf16_pair(v[nt][2], v[nt][3]);
            }
#pragma unroll
            for (int h = 0; h < NT; h += 4) {
                transpose_groups(lo[h], lo[h + 1], lo[h + 2], lo[h + 3]);
                transpose_groups(hi[h], hi[h + 1], hi[h + 2], hi[h + 3]);
            }
            if (m < M) {
#pragma unroll
                for (int h = 0; h < NT; h += 4) {
                    auto *at = reinterpret_cast<u32x4_any_t *>(static_cast<uint16_t *>(o.C) + (int64_t)m * o.ld + n0 + 16 * (h + g));
                    at[0] = (u32x4_any_t){lo[h], hi[h], lo[h + 1], hi[h + 1]};
                    at[1] = (u32x4_any_t){lo[h + 2], hi[h + 2], lo[h + 3], hi[h + 3]};
                }
            }
        } else if (m < M) {
            Out to = o;
            if constexpr (KIND == kOutPart) to.C = static_cast<float *>(o.C) + (int64_t)split * M * o.ld;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) store4<KIND>(to, m, n_lane + 16 * nt, N, v[nt]);
        }
        __builtin_amdgcn_sched_barrier(0);                  // (one row of tiles at a time: registers)
    }
}

// The tile that workgroup b of n works on: the eight XCDs take consecutive
// ranges of the tiles, so that neighbours share an L2, and within those
// 8 tiles along m go with every n before the next 8.
__device__ __forceinline__ void tile_of(int32_t b, int32_t m_tiles, int32_t n_tiles, int32_t &mt, int32_t &nt)
{
    const int32_t n = m_tiles * n_tiles, q = n / 8, r = n % 8, x = b % 8;
    const int32_t t = x * q + (x < r ? x : r) + b / 8, band = t / (8 * n_tiles), first = band * 8;
    const int32_t rows = m_tiles - first < 8 ? m_tiles - first : 8, in = t - band * 8 * n_tiles;
    mt = first + in % rows;
    nt = in / rows;
}

// Four waves, each MT x 8 tiles of 16 x 16: 128 columns, a whole block of the
// next layer's operand.  Two LDS stages: the next block of K is on its way while
// one is multiplied.  (Three and four stages, eight waves or two: no faster
// anywhere from 300 x 300 x 2,000 to 8,192 x 1,024 x 1,024.)
template <int MT, int FA, OutKind KIND>
__global__ __launch_bounds__(256, 2) void k_product(Operand A, Operand B, int32_t nkb, int32_t per_split, Out o)
{
    constexpr int NT = 8, BM = 64 * MT, kStage = (BM + 128) * 128, kLoadsA = BM / 8 / 4, kLoadsB = 4;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int32_t m_tile, n_tile;
    tile_of(blockIdx.x, (A.rows + BM - 1) / BM, (B.rows + 127) / 128, m_tile, n_tile);
    const int32_t m0 = m_tile * BM, n0 = n_tile * 128;
    const int32_t k_begin = (int32_t)blockIdx.y * per_split, k_end = k_begin + per_split < nkb ? k_begin + per_split : nkb;
    const auto a_tile = tile_buffer(A.q + (int64_t)m0 * A.ld), b_tile = tile_buffer(B.q + (int64_t)n0 * B.ld);
    uint32_t a_at[kLoadsA], b_at[kLoadsB];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) a_at[i] = lds_source((wave * kLoadsA + i) * 8, lane, A.rows - m0, A.ld);
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i) b_at[i] = lds_source((wave * kLoadsB + i) * 8, lane, B.rows - n0, B.ld);
    auto fetch = [&](int32_t kb) {
        const uint32_t k = (uint32_t)kb * 128;
        uint8_t *stage = lds + (kb & 1) * kStage;
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i) to_lds(a_tile, a_at[i], k, stage + (wave * kLoadsA + i) * 1024);
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i) to_lds(b_tile, b_at[i], k, stage + BM * 128 + (wave * kLoadsB + i) * 1024);
    };
    const int32_t row_a = m0 + wave * MT * 16 + (lane & 15), row_b = n0 + (lane & 15);
    uint32_t sa[MT], sb[NT], sa_next[MT], sb_next[NT];
    auto scales = [&](int32_t kb) {                         // (of the last blocks again past the end)
        kb = kb < nkb ? kb : nkb - 1;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sa_next[mt] = scale_word(A, row_a + 16 * mt, kb);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sb_next[nt] = scale_word(B, row_b + 16 * nt, kb);
    };
    fetch(k_begin);
    scales(k_begin);
    f32x4_t acc[MT][NT];
    start_tiles<MT, KIND>(acc, n0, B.rows, o, lane);
    for (int32_t kb = k_begin; kb < k_end; ++kb) {
        if (((kb - k_begin) & 3) == 0) {                    // (splits start at multiples of four blocks)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sa[mt] = sa_next[mt];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sb[nt] = sb_next[nt];
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);                 // vmcnt(0): the barrier alone does not wait for loads to LDS
        __syncthreads();                                    // this stage has come; the other one is read
        if (kb + 1 < k_end) fetch(kb + 1);
        if (((kb - k_begin) & 3) == 0) scales(kb + 4);
        const uint8_t *stage = lds + (kb & 1) * kStage;
        i32x8_t a[MT];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) a[mt] = fragment(stage + (wave * MT + mt) * 2048, lane);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const i32x8_t b = fragment(stage + BM * 128 + nt * 2048, lane);
#pragma unroll
            for (int mt = 0; mt < MT; ++mt)
                acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b, a[mt], acc[mt][nt], 0, FA, 0, (int)sb[nt], 0,
                                                                              (int)sa[mt]);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sa[mt] >>= 8;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sb[nt] >>= 8;
    }
    finish_tiles<MT, KIND>(acc, m0 + wave * MT * 16, n0, A.rows, B.rows, (int32_t)blockIdx.y, o, lane);
}

// 256 x 256 tiles by eight waves in two groups, a wave of each on every SIMD.
// A step of K has two phases with a barrier after each: while one group reads
// its fragments from LDS the other one multiplies, so the matrix cores and LDS
// are both busy all the time.  The second group runs a phase behind.
template <int FA, OutKind KIND>
__global__ __launch_bounds__(512) void k_product_deep(Operand A, Operand B, int32_t nkb, Out o)
{
    constexpr int MT = 4, NT = 8, BM = 256, BN = 256, kStage = (BM + BN) * 128;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStage];
    // Exponent bytes of four blocks of K: [block][A: wave rows, row % 16, tile][B: alike],
    // so that one read brings a lane the bytes of its row of every tile.
    __shared__ __attribute__((aligned(16))) uint8_t scale_lds[2][4][512];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool second = wave >= 4;                          // the second group: rows 128 .. 255
    const int wm = wave >> 1, wn = wave & 1;                // the wave's 64 rows and 128 columns
    int32_t m_tile, n_tile;
    tile_of(blockIdx.x, (A.rows + BM - 1) / BM, (B.rows + BN - 1) / BN, m_tile, n_tile);
    const int32_t m0 = m_tile * BM, n0 = n_tile * BN;
    const auto a_tile = tile_buffer(A.q + (int64_t)m0 * A.ld), b_tile = tile_buffer(B.q + (int64_t)n0 * B.ld);
    // a wave brings 32 rows of A, those of its own group; a wave of the first group 64 of B
    uint32_t a_at[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) a_at[i] = lds_source(wave * 32 + i * 8, lane, A.rows - m0, A.ld);
    // (past the end the last block is brought again, to a stage that is not read)
    auto k_of = [&](int32_t kb) { return (uint32_t)(kb < nkb ? kb : nkb - 1) * 128; };
    // thread t brings the bytes of row t of A's 256, then of B's
    const int32_t own = (int32_t)threadIdx.x & 255;
    const bool of_b = threadIdx.x >= 256;
    const int scale_at = of_b ? 256 + (own & 128) + (own & 15) * 8 + ((own >> 4) & 7) : (own & 192) + (own & 15) * 4 + ((own >> 4) & 3);
    auto load_scales = [&](int32_t kb) -> uint32_t {        // (of the last blocks again past the end)
        kb = kb < nkb ? kb : nkb - 1;
        return of_b ? scale_word(B, n0 + own, kb) : scale_word(A, m0 + own, kb);
    };
    auto put_scales = [&](int32_t kb, uint32_t w) {
        uint8_t *to = &scale_lds[(kb >> 2) & 1][0][scale_at];
#pragma unroll
        for (int i = 0; i < 4; ++i) to[512 * i] = (uint8_t)(w >> (8 * i));
    };
    f32x4_t acc[MT][NT];
    start_tiles<MT, KIND>(acc, n0 + wn * 128, B.rows, o, lane);
    auto barrier = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    auto fetch_a = [&](int32_t kb, int i) { to_lds(a_tile, a_at[i], k_of(kb), lds + (kb & 1) * kStage + (wave * 4 + i) * 1024); };
    auto fetch_b = [&](int32_t kb) {
        int l = lane;                                       // (offsets made anew each time: no registers to keep them)
        asm volatile("" : "+v"(l));
#pragma unroll
        for (int i = 0; i < 8; ++i)
            to_lds(b_tile, lds_source((wave & 3) * 64 + i * 8, l, B.rows - n0, B.ld), k_of(kb), lds + (kb & 1) * kStage + BM * 128 + ((wave & 3) * 8 + i) * 1024);
    };
    auto lds_done = [] { __builtin_amdgcn_s_waitcnt(0xc07f); };           // lgkmcnt(0)
    if (!second) fetch_b(0);
#pragma unroll
    for (int i = 0; i < 4; ++i) fetch_a(0, i);
    put_scales(0, load_scales(0));
    if (!second) fetch_b(0 + 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) fetch_a(0 + 1, i);
    __builtin_amdgcn_s_waitcnt(0x0f70);                     // vmcnt(0)
    lds_done();
    barrier();
    if (second) barrier();
    uint32_t next_scales = 0;
    for (int32_t kb = 0; kb < nkb; ++kb) {
        const uint8_t *stage = lds + (kb & 1) * kStage;
        const uint8_t *sc = scale_lds[(kb >> 2) & 1][kb & 3];
        i32x8_t a[MT], b[NT];
        const uint32_t sa = *reinterpret_cast<const uint32_t *>(sc + wm * 64 + (lane & 15) * 4);
        const u32x2_t sb = *reinterpret_cast<const u32x2_t *>(sc + 256 + wn * 128 + (lane & 15) * 8);
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) a[mt] = fragment(stage + (wm * MT + mt) * 2048, lane);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) b[nt] = fragment(stage + BM * 128 + (wn * NT + nt) * 2048, lane);
        __builtin_amdgcn_sched_barrier(0);
        // the other stage: the second group has read it in the phase before
        if (!second && kb > 0) fetch_b(kb + 1);
        if ((kb & 3) == 2) put_scales(kb + 2, next_scales);
        lds_done();                                         // the fragments are here
        barrier();
        __builtin_amdgcn_sched_barrier(0);
        if ((kb & 3) == 1) next_scales = load_scales(kb + 3);
        __builtin_amdgcn_s_setprio(1);
#define TILE(nt, mt)                                                                                                          \
    acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[nt], a[mt], acc[mt][nt], 0, FA, (nt) & 3,                 \
                                                                   (int)((nt) < 4 ? sb.x : sb.y), mt, (int)sa)
#define TILES(nt) TILE(nt, 0); TILE(nt, 1); TILE(nt, 2); TILE(nt, 3)
#define STEP(i)                                                                                                               \
    TILES(2 * i);                                                                                                             \
    __builtin_amdgcn_sched_barrier(0);                                                                                        \
    fetch_a(kb + 2, i);                                                                                                       \
    __builtin_amdgcn_sched_barrier(0);                                                                                        \
    TILES(2 * i + 1)
        // this stage's rows of A: the group itself has read them
        STEP(0); STEP(1); STEP(2); STEP(3);
#undef STEP
#undef TILES
#undef TILE
        __builtin_amdgcn_s_setprio(0);
        // all but the four loads just made have landed
        __builtin_amdgcn_s_waitcnt(0x0f74);
        __builtin_amdgcn_sched_barrier(0);
        barrier();
    }
    if (!second) barrier();
    __builtin_amdgcn_s_waitcnt(0x0f70);                     // (no load to LDS outlives the workgroup)
    finish_tiles<MT, KIND>(acc, m0 + wm * 64, n0 + wn * 128, A.rows, B.rows, 0, o, lane);
}

// Short sums (K up to 128 NKB), many rows.  A wave keeps its MT x 16 rows of A in
// registers, all of K, and goes through the columns 128 at a time; B comes by
// in LDS, a ring of four stages of 128 columns by one block of K that runs on
// from one 128 columns to the next, three stages ahead; their exponent bytes and bias come by the same way.
// Blocks of K past the
// end are zeros of A against the last block of B, both with scale 1.
// 4.9 M x 512 -> 512 with GELU to 8 bits 2.02 ms, by counters: vector units (GELU,
// scales, codes) busy 62 % of the time, matrix cores 28 %, both at once 8 %, LDS
// 17 %.  Fragments are read just before the products that take them, and GELU
// comes after all of a tile's products.
template <int NKB, int MT, int FA, OutKind KIND>
__global__ __launch_bounds__(256, 2) void k_product_rows(Operand A, Operand B, int32_t nkb, int32_t tiles_each, Out o)
{
    constexpr int NT = 8, BM = 64 * MT, kStage = 128 * 128, kAhead = 3;
    static_assert(MT * NKB <= 8, "registers");
    constexpr int kWords = (NKB + 3) / 4, kSide = 512 * (kWords + 1);      // exponent words and bias of 128 columns
    __shared__ __attribute__((aligned(1024))) uint8_t lds[4 * kStage + 4 * kSide];
    uint8_t *side = lds + 4 * kStage;                       // of tile t at t % 4
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int32_t N = B.rows, n_tiles = (N + 127) / 128;
    const int32_t m0 = (int32_t)blockIdx.x * BM + wave * MT * 16;
    const int32_t t_begin = (int32_t)blockIdx.y * tiles_each, t_end = t_begin + tiles_each < n_tiles ? t_begin + tiles_each : n_tiles;
    const int32_t stages = (t_end - t_begin) * NKB;
    uint32_t b_at[4];                                       // (made anew for a last tile of fewer columns)
#pragma unroll
    for (int i = 0; i < 4; ++i) b_at[i] = lds_source(wave * 32 + i * 8, lane, N - t_begin * 128, B.ld);
    auto fetch = [&](int32_t at) {                          // (past the end the last stage again: it is not read)
        const int32_t s = at < stages ? at : stages - 1, n0 = (t_begin + s / NKB) * 128, kb = s % NKB;
        const auto tile = tile_buffer(B.q + (int64_t)n0 * B.ld);
        if (kb == 0) {                                      // 64 words a load: words 64 i .. of the tile's
            const int32_t t = at / NKB;
            if (n0 + 128 > N) {
#pragma unroll
                for (int i = 0; i < 4; ++i) b_at[i] = lds_source(wave * 32 + i * 8, lane, N - n0, B.ld);
            }
#pragma unroll
            for (int i = wave; i < 2 * (kWords + 1); i += 4) {
                const int j = i >> 1;
                int32_t n = n0 + (i & 1) * 64 + lane;
                n = n < N ? n : N - 1;
                uint8_t *to = side + (t & 3) * kSide + i * 256;
                if (j < kWords)
                    word_to_lds(B.scale + (int64_t)(n >> B.shift) * B.ld_scale + (4 * j < nkb ? 4 * j : 0), to);
                else if (o.bias)
                    word_to_lds(reinterpret_cast<const uint8_t *>(o.bias + n), to);
            }
        }
        uint8_t *to = lds + (at & 3) * kStage + wave * 4096;
        const uint32_t k = (uint32_t)(kb < nkb ? kb : nkb - 1) * 128;
#pragma unroll
        for (int i = 0; i < 4; ++i) to_lds(tile, b_at[i], k, to + i * 1024);
    };
    // vmcnt(8): of this wave's loads all but the next two stages' have come.  lgkmcnt(0):
    // its fragments of the stage before have been read, which is loaded anew behind the
    // barrier (the products that take them may follow it; without the wait up to a
    // whole stage's reads were on their way here).
    auto stage_barrier = [] {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0078);
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
#pragma unroll
    for (int s = 0; s < kAhead; ++s) fetch(s);
    auto clean = [&](uint32_t w, int j) {                   // bytes past the blocks may be anything
        if (nkb == NKB) return w;
        const int32_t have = nkb - 4 * j;
        const uint32_t mask = have >= 4 ? 0xffffffffu : have > 0 ? (1u << (8 * have)) - 1u : 0u;
        return (w & mask) | (0x7f7f7f7fu & ~mask);
    };
    i32x8_t a[MT][NKB];
    uint32_t sa[MT][(NKB + 3) / 4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int32_t row = m0 + 16 * mt + (lane & 15), r = row < A.rows ? row : A.rows - 1;
        const uint8_t *at = A.q + (int64_t)r * A.ld + g * 16;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb) {
            const int32_t k = (kb < nkb ? kb : nkb - 1) * 128;
            const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(at + k), hi = *reinterpret_cast<const i32x4_t *>(at + k + 64);
            a[mt][kb] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
            if (kb >= nkb) a[mt][kb] = (i32x8_t){0, 0, 0, 0, 0, 0, 0, 0};
        }
#pragma unroll
        for (int j = 0; j < (NKB + 3) / 4; ++j) sa[mt][j] = clean(scale_word(A, row, 4 * j < nkb ? 4 * j : 0), j);
    }
    for (int32_t t = t_begin; t < t_end; ++t) {
        const int32_t n0 = t * 128;
        f32x4_t acc[MT][NT];
        uint32_t sb[NT][kWords];
#define BLOCK(kb)                                                                                                             \
    if constexpr ((kb) < NKB) {                                                                                               \
        const int32_t s = (t - t_begin) * NKB + (kb);                                                                         \
        stage_barrier();                                                                                                      \
        fetch(s + kAhead);                                                                                                    \
        __builtin_amdgcn_sched_barrier(0);                                                                                    \
        if constexpr ((kb) == 0) {                                                                                            \
            const uint8_t *own = side + ((t - t_begin) & 3) * kSide;                                                          \
            _Pragma("unroll") for (int nt = 0; nt < NT; ++nt)                                                                 \
            {                                                                                                                 \
                f32x4_t first = {0.0f, 0.0f, 0.0f, 0.0f};                                                                     \
                if (o.bias) first = *reinterpret_cast<const f32x4_t *>(own + 512 * kWords + nt * 64 + g * 16);                \
                _Pragma("unroll") for (int mt = 0; mt < MT; ++mt) acc[mt][nt] = first;                                        \
                _Pragma("unroll") for (int j = 0; j < kWords; ++j)                                                            \
                    sb[nt][j] = clean(*reinterpret_cast<const uint32_t *>(own + 512 * j + nt * 64 + (lane & 15) * 4), j);     \
            }                                                                                                                 \
        }                                                                                                                     \
        const uint8_t *stage = lds + (s & 3) * kStage;                                                                        \
        _Pragma("unroll") for (int nt = 0; nt < NT; ++nt)                                                                     \
        {                                                                                                                     \
            const i32x8_t b = fragment(stage + nt * 2048, lane);                                                              \
            _Pragma("unroll") for (int mt = 0; mt < MT; ++mt) acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4( \
                b, a[mt][kb], acc[mt][nt], 0, FA, (kb) & 3, (int)sb[nt][(kb) / 4], (kb) & 3, (int)sa[mt][(kb) / 4]);          \
        }                                                                                                                     \
    }
        BLOCK(0) BLOCK(1) BLOCK(2) BLOCK(3) BLOCK(4) BLOCK(5) BLOCK(6) BLOCK(7)
#undef BLOCK
        // the sums are taken here: left to itself the compiler moves every product
        // behind the last barrier, with all fragments kept in registers till then
#pragma unroll
        for (int mt = 0; mt < MT; ++mt)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) asm volatile("" : "+v"(acc[mt][nt]));
        __builtin_amdgcn_sched_barrier(0);
        finish_tiles<MT, KIND>(acc, m0, n0, A.rows, N, 0, o, lane);
    }
    __builtin_amdgcn_s_waitcnt(0x0f70);                     // (no load to LDS outlives the workgroup)
}

// Results in fp32: products of decoded codes by the bf16 instruction (see above).
// Four waves, WM along the rows, each 16 MT x 16 NT: a fragment decoded serves MT
// or NT products.  Two stages in LDS, the next block of K on its way meanwhile.
template <int WM, int MT, int FA, OutKind KIND>
__global__ __launch_bounds__(256, 2) void k_product_exact(Operand A, Operand B, int32_t nkb, int32_t per_split, Out o)
{
    constexpr int NT = 2 * WM, BM = 16 * WM * MT, BN = 128, kStage = (BM + BN) * 128;
    constexpr int kLoadsA = (BM / 8 + 3) / 4, kLoadsB = BN / 8 / 4;
    __shared__ __attribute__((aligned(1024))) uint8_t lds[2 * kStage];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wm = wave % WM, wn = wave / WM;
    int32_t m_tile, n_tile;
    tile_of(blockIdx.x, (A.rows + BM - 1) / BM, (B.rows + BN - 1) / BN, m_tile, n_tile);
    const int32_t m0 = m_tile * BM, n0 = n_tile * BN, N = B.rows;
    const int32_t k_begin = (int32_t)blockIdx.y * per_split, k_end = k_begin + per_split < nkb ? k_begin + per_split : nkb;
    const auto a_tile = tile_buffer(A.q + (int64_t)m0 * A.ld), b_tile = tile_buffer(B.q + (int64_t)n0 * B.ld);
    uint32_t a_at[kLoadsA], b_at[kLoadsB];
#pragma unroll
    for (int i = 0; i < kLoadsA; ++i) a_at[i] = lds_source((wave * kLoadsA + i) * 8, lane, A.rows - m0, A.ld);
#pragma unroll
    for (int i = 0; i < kLoadsB; ++i) b_at[i] = lds_source((wave * kLoadsB + i) * 8, lane, N - n0, B.ld);
    auto fetch = [&](int32_t kb) {
        const uint32_t k = (uint32_t)kb * 128;
        uint8_t *stage = lds + (kb & 1) * kStage;
#pragma unroll
        for (int i = 0; i < kLoadsA; ++i)
            if (BM % 32 == 0 || wave * kLoadsA + i < BM / 8) to_lds(a_tile, a_at[i], k, stage + (wave * kLoadsA + i) * 1024);
#pragma unroll
        for (int i = 0; i < kLoadsB; ++i) to_lds(b_tile, b_at[i], k, stage + BM * 128 + (wave * kLoadsB + i) * 1024);
    };
    f32x4_t acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
    const int32_t row_a = m0 + wm * 16 * MT + (lane & 15), row_b = n0 + wn * 16 * NT + (lane & 15);
    uint32_t sa[MT], sb[NT], sa_next[MT], sb_next[NT];
    auto scales = [&](int32_t kb) {                         // (of the last blocks again past the end)
        kb = kb < nkb ? kb : nkb - 1;
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sa_next[mt] = scale_word(A, row_a + 16 * mt, kb);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sb_next[nt] = scale_word(B, row_b + 16 * nt, kb);
    };
    fetch(k_begin);
    scales(k_begin);
    for (int32_t kb = k_begin; kb < k_end; ++kb) {
        if (((kb - k_begin) & 3) == 0) {                    // (splits start at multiples of four blocks)
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sa[mt] = sa_next[mt];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sb[nt] = sb_next[nt];
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);                 // vmcnt(0): the barrier alone does not wait for loads to LDS
        __syncthreads();                                    // this stage has come; the other one is read
        if (kb + 1 < k_end) fetch(kb + 1);
        if (((kb - k_begin) & 3) == 0) scales(kb + 4);
        const uint8_t *stage = lds + (kb & 1) * kStage;
        bf16x8_t wide[MT][4];
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            decode<FA>(fragment(stage + (wm * MT + mt) * 2048, lane), sa[mt], wide[mt]);
            sa[mt] >>= 8;
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            bf16x8_t w[4];
            decode<0>(fragment(stage + BM * 128 + (wn * NT + nt) * 2048, lane), sb[nt], w);
            sb[nt] >>= 8;
#pragma unroll
            for (int q = 0; q < 4; ++q)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[q], wide[mt][q], acc[mt][nt], 0, 0, 0);
        }
    }
    Out to = o;
    if constexpr (KIND == kOutPart) to.C = static_cast<float *>(o.C) + (int64_t)blockIdx.y * A.rows * o.ld;
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int32_t m = row_a + 16 * mt;
        if (m >= A.rows) continue;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int32_t n = n0 + (wn * NT + nt) * 16 + 4 * (lane >> 4);
            float v[4] = {acc[mt][nt][0], acc[mt][nt][1], acc[mt][nt][2], acc[mt][nt][3]};
            if constexpr (KIND != kOutPart) finish4<KIND>(o, n, N, v);
            store4<KIND>(to, m, n, N, v);
        }
    }
}

// Few rows (up to 16 MT): bound by reading B.  A workgroup has 16 NT columns, its
// eight waves a run of K each; fragments go from memory to registers, the next
// block's while one is multiplied, and the waves' sums are added in LDS in the
// order of K.
template <int MT, int NT, int FA, bool EXACT, OutKind KIND>
__global__ __launch_bounds__(512) void k_product_few(Operand A, Operand B, int32_t nkb, int32_t per_split, Out o)
{
    constexpr int kWaves = 8, kTiles = MT * NT;
    __shared__ f32x4_t sums[kWaves][kTiles][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = lane >> 4;
    const int32_t N = B.rows, n0 = (int32_t)blockIdx.x * 16 * NT;
    const int32_t s_begin = (int32_t)blockIdx.y * per_split, s_end = s_begin + per_split < nkb ? s_begin + per_split : nkb;
    const int32_t each = (s_end - s_begin + kWaves - 1) / kWaves;
    const int32_t k_begin = s_begin + wave * each < s_end ? s_begin + wave * each : s_end,
                  k_end = k_begin + each < s_end ? k_begin + each : s_end;
    const uint8_t *a_at[MT], *b_at[NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
        const int32_t r = 16 * mt + (lane & 15);
        a_at[mt] = A.q + (int64_t)(r < A.rows ? r : A.rows - 1) * A.ld + g * 16;
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
        const int32_t r = n0 + 16 * nt + (lane & 15);
        b_at[nt] = B.q + (int64_t)(r < N ? r : N - 1) * B.ld + g * 16;
    }
    struct Block {
        i32x8_t a[MT], b[NT];
    };
    auto load = [&](int32_t kb, Block &x) {
        const int64_t k = (int64_t)kb * 128;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(b_at[nt] + k), hi = *reinterpret_cast<const i32x4_t *>(b_at[nt] + k + 64);
            x.b[nt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) {
            const i32x4_t lo = *reinterpret_cast<const i32x4_t *>(a_at[mt] + k), hi = *reinterpret_cast<const i32x4_t *>(a_at[mt] + k + 64);
            x.a[mt] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        }
    };
    uint32_t sa[MT], sb[NT];
    auto scales = [&](int32_t kb) {
#pragma unroll
        for (int mt = 0; mt < MT; ++mt) sa[mt] = scale_word(A, 16 * mt + (lane & 15), kb) >> (8 * (kb & 3));
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sb[nt] = scale_word(B, n0 + 16 * nt + (lane & 15), kb) >> (8 * (kb & 3));
    };
    f32x4_t acc[MT][NT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) acc[mt][nt] = (f32x4_t){0.0f, 0.0f, 0.0f, 0.0f};
    auto multiply = [&](const Block &x) {
        if constexpr (EXACT) {
            bf16x8_t wide[MT][4];
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) decode<FA>(x.a[mt], sa[mt], wide[mt]);
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                bf16x8_t w[4];
                decode<0>(x.b[nt], sb[nt], w);
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int mt = 0; mt < MT; ++mt)
                        acc[mt][nt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[q], wide[mt][q], acc[mt][nt], 0, 0, 0);
            }
        } else {
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int mt = 0; mt < MT; ++mt)
                    acc[mt][nt] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x.b[nt], x.a[mt], acc[mt][nt], 0, FA, 0,
                                                                                  (int)sb[nt], 0, (int)sa[mt]);
        }
    };
    auto next_scales = [&](int32_t kb) {                    // of block kb, after kb - 1
        if ((kb & 3) == 0) {
            if (kb < k_end) scales(kb);
        } else {
#pragma unroll
            for (int mt = 0; mt < MT; ++mt) sa[mt] >>= 8;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) sb[nt] >>= 8;
        }
    };
    if (k_begin < k_end) {
        Block x, y;
        load(k_begin, x);
        scales(k_begin);
        int32_t kb = k_begin;
        for (; kb + 1 < k_end; kb += 2) {
            load(kb + 1, y);
            multiply(x);
            next_scales(kb + 1);
            if (kb + 2 < k_end) load(kb + 2, x);
            multiply(y);
            next_scales(kb + 2);
        }
        if (kb < k_end) multiply(x);
    }
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sums[wave][mt * NT + nt][lane] = acc[mt][nt];
    __syncthreads();
    for (int e = threadIdx.x; e < kTiles * 64; e += 512) {
        const int tile = e >> 6, l = e & 63;
        f32x4_t v = sums[0][tile][l];
#pragma unroll
        for (int w = 1; w < kWaves; ++w) v += sums[w][tile][l];
        const int32_t m = 16 * (tile / NT) + (l & 15), n = n0 + 16 * (tile % NT) + 4 * (l >> 4);
        if (m >= A.rows) continue;
        float out[4] = {v[0], v[1], v[2], v[3]};
        Out to = o;
        if constexpr (KIND == kOutPart) to.C = static_cast<float *>(o.C) + (int64_t)blockIdx.y * A.rows * o.ld;
        else finish4<KIND>(o, n, N, out);
        store4<KIND>(to, m, n, N, out);
    }
}

// Sum of the splits' partial sums, in the order of K, and what becomes of it:
// 32 lanes take 128 columns of a row.
template <OutKind KIND>
__global__ __launch_bounds__(256) void k_product_join(const float *__restrict__ part, int32_t splits, int32_t M, int32_t N,
                                                      int64_t ldp, Out o)
{
    const int32_t blocks = (N + 127) / 128;
    const int64_t items = (int64_t)M * blocks;
    for (int64_t it = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); it < items; it += (int64_t)gridDim.x * 8) {
        const int64_t m = it / blocks;
        const int32_t kb = (int32_t)(it % blocks), n = kb * 128 + (threadIdx.x & 31) * 4;
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (n < N) {
            for (int32_t z = 0; z < splits; ++z) {
                const float4 p = *reinterpret_cast<const float4 *>(part + ((int64_t)z * M + m) * ldp + n);
                v[0] += p.x; v[1] += p.y; v[2] += p.z; v[3] += p.w;
            }
        }
        finish4<KIND>(o, n, N, v);
        if constexpr (KIND == kOutFp8) {
            uint32_t most = 0, all = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t f = finite_bits(v[i]), x = __float_as_uint(v[i]) & 0x7fffffffu;
                most = f > most ? f : most;
                all = x > all ? x : all;
            }
#pragma unroll
            for (int l = 1; l < 32; l <<= 1) {
                const uint32_t x = (uint32_t)__shfl_xor((int)most, l, 32);
                most = x > most ? x : most;
            }
            const uint32_t byte = scale_byte(most, HWSEL_FP8_E4M3);
            *reinterpret_cast<uint32_t *>(static_cast<uint8_t *>(o.C) + m * o.ld + n) =
                codes4_checked(v, inverse_scale(byte), HWSEL_FP8_E4M3, all >= 0x7f800000u);
            if ((threadIdx.x & 31) == 0) o.scale[m * o.ld_scale + kb] = (uint8_t)byte;
        } else {
            store4<KIND>(o, m, n, N, v);
        }
    }
}

constexpr int kBM = 128, kBN = 128;

enum class Way { few, rows, deep, tiles };                  // the kernels above

struct Plan {
    Way way;
    int32_t splits, per_split, nt, bm;                      // nt: column tiles of a workgroup, few rows; bm: rows of a tile
};

// The kernel, and how many parts K is split into, by sizes alone (codes: results in 8 bits).  us are of
// calls in a graph, results in bf16 where nothing else is said.
Plan plan_product(int64_t M, int64_t N, int64_t nkb, bool exact, bool codes = false)
{
    const int64_t cus = compute_units();
    auto plan = [&](Way way, int64_t s, int64_t unit, int32_t nt, int32_t bm) {
        s = s < 1 ? 1 : s;
        const int64_t per = (nkb + unit * s - 1) / (unit * s) * unit;
        return Plan{way, (int32_t)((nkb + per - 1) / per), (int32_t)per, nt, bm};
    };
    // Few rows.  K = N = 8,192: 13.6 us (1 row), 14.9 (16), 19.4 (32), where tiles take 20.2, 20.5 and 20.7.  With
    // 64 rows, a weight for four products, only small B: 64 x 1,024 x 1,024 4.9 (tiles 8.4), 64 x 4,096 x 4,096 13.0
    // (14.3), but 64 x 8,192 x 8,192 39 (22).  Wider workgroups read A less often, where there are columns enough:
    // 16 x 16,384 x 4,096 18.1, 15.4 and 13.3 with 1, 2 and 4 tiles of columns, 16 x 8,192 x 8,192 18.1, 14.8 and
    // 16.2, 32 x 16,384 x 16,384 97, 67 and 92 (registers), 32 x 4,096 x 4,096 8.5, 10.6 and 21.
    // Codes need the sums of whole blocks joined, a second launch: up to K = 1,024 a tile does both, 4 x 581 x 126 3.8
    // us (4.7; called from Python 6.4 and 9.1), 16 x 1,024 x 512 5.1 (5.1), 32 x 1,024 x 1,024 6.9 (6.2; 6.9 and 9.2).
    if (!(codes && nkb <= 8) && (M <= 32 || (M <= 64 && N * nkb < (1 << 17)))) {
        const int nt = M <= 16 && N >= 64 * cus ? 4 : M <= 32 && N >= 32 * cus ? 2 : 1;
        const int64_t s = cus / ((N + 16 * nt - 1) / (16 * nt));
        return plan(Way::few, s < nkb / 32 ? s : nkb / 32, 1, nt, 0);
    }
    auto tiles_of = [&](int64_t m, int64_t n) { return (M + m - 1) / m * ((N + n - 1) / n); };
    // Tiles of 256 x 256, if they fill five compute units in eight: 2,816 x 4,096 x 4,096 47 us (128 x 128: 62),
    // 8,192 x 8,192 x 2,048 128 (155), 4,096 x 4,096 x 1,024 23.1 (24.0), but 2,048 x 4,096 x 4,096 44 (37) and
    // 4,096 x 4,096 x 768 20.9 (21.3), where their start weighs as much as they win.
    if (!exact && M >= 256 && N >= 256 && nkb >= 8 && tiles_of(256, 256) * 8 >= cus * 5) return plan(Way::deep, 1, 4, 0, 256);
    // Short sums over many tiles: 65,536 x 1,024 x 512 53.9 us (tiles one by one: 57.2), with K = 128 30.8 (35.9),
    // 262,144 x 1,024 x 512 to 8 bits 210 (277), but 32,768 x 1,024 x 512 33.6 (31.0) and 8,192 13.5 (11.4).
    if (!exact && nkb <= 4 && tiles_of(kBM, kBN) >= 12 * cus) return plan(Way::rows, 1, 4, 0, kBM);
    // Lower tiles where there are no more than compute units: 1,024 x 1,024 x 1,024 6.7 us (128 rows: 8.3), 2,048 x
    // 2,048 x 4,096 26 (32), 512 x 8,192 x 8,192 46 (49), but 8,192 x 1,024 x 1,024 18.7 (15.4).
    int32_t bm = !exact && tiles_of(kBM, kBN) <= cus ? 64 : kBM;
    // Heights in fp32, where K is too short to split instead: the rows that the busiest compute unit gets, a tenth
    // and a fifth more work to a row in the lower ones (8,192 x 8,192 x 2,048: 128 rows 272 us, 64 304, 48 333), and
    // a workgroup alone has no other to hide its waits.  4,099 x 1,000 x 2,500: 43.9, 39.5 and 34.6 us (31.5 by now); 4,096 x
    // 1,024 x 4,096: 47.0, 43.2 (41.2), 47.5; 8,192 x 1,000 x 2,500: 45.7, 49.8, 58.5; 1,024 x 1,024 x 1,024: 15.1, 10.1,
    // 8.7; 512 x 1,024 x 65,536, split: 75.5, 80.8, 99.0.
    if (exact && nkb < 64) {
        auto cost = [&](int64_t m) {
            const int64_t each = (tiles_of(m, kBN) + cus - 1) / cus;
            return (each > 1 ? 4 * each : 5) * m * (m == 128 ? 10 : m == 64 ? 11 : 12);
        };
        for (const int32_t m : {64, 48})
            if (cost(m) < cost(bm)) bm = m;
    }
    // K in parts, two workgroups a compute unit, eight blocks at least: 1,024 x 1,024 x 8,192 26 us (whole: 77),
    // 100 x 4,096 x 4,096 15.5 (25; parts of four blocks 17.4), 64 x 16,384 x 16,384 54 (one workgroup: 78);
    // 1,024 x 1,024 x 1,024 in fp32 10.6 whole and 12.9 in two.
    const int64_t s = 2 * cus / tiles_of(bm, kBN);
    return plan(Way::tiles, s < nkb / 8 ? s : nkb / 8, 4, 0, bm);
}

Operand operand(const hwsel_fp8_t &x)
{
    return {x.q, x.ld, x.scale, x.ld_scale, (int32_t)x.rows, x.block_rows == 1 ? 0 : 7};
}

// Rows first .. first + n of an operand (whole blocks before them).
Operand part_of(Operand x, int64_t first, int64_t n)
{
    x.q += first * x.ld;
    x.scale += (first >> x.shift) * x.ld_scale;
    x.rows = (int32_t)n;
    return x;
}

// A result from column n on.
template <OutKind KIND>
Out columns_from(Out o, int64_t n)
{
    static_assert(KIND != kOutFp8, "codes have scales beside them");
    o.C = static_cast<uint8_t *>(o.C) + n * (KIND == kOutBf16 ? 2 : 4);
    if (o.bias) o.bias += n;
    return o;
}

template <int MT, bool EXACT, OutKind KIND>
void launch_few(const hwsel_fp8_t &A, const hwsel_fp8_t &B, const Plan &p, const Out &o, hipStream_t s)
{
    const int32_t nkb = (int32_t)fp8_blocks(A.cols);
    // (a launch has fewer than 2^32 threads: many columns, which leave K whole, go in spans of 2^22 workgroups)
    auto go = [&](auto kernel) {
        const int64_t span = ((int64_t)1 << 22) * 16 * p.nt;
        for (int64_t n0 = 0; n0 < B.rows; n0 += span) {
            const int64_t n = B.rows - n0 < span ? B.rows - n0 : span;
            const dim3 grid((unsigned)((n + 16 * p.nt - 1) / (16 * p.nt)), (unsigned)p.splits);
            hipLaunchKernelGGL(kernel, grid, dim3(512), 0, s, operand(A), part_of(operand(B), n0, n), nkb, p.per_split,
                               columns_from<KIND>(o, n0));
        }
    };
    auto by_columns = [&](auto fa) {
        constexpr int FA = decltype(fa)::value;
        if constexpr (MT == 1)
            if (p.nt == 4) return go(k_product_few<MT, 4, FA, EXACT, KIND>);
        if constexpr (MT <= 2)
            if (p.nt == 2) return go(k_product_few<MT, 2, FA, EXACT, KIND>);
        go(k_product_few<MT, 1, FA, EXACT, KIND>);
    };
    if (A.format == HWSEL_FP8_E4M3) by_columns(std::integral_constant<int, 0>{});
    else by_columns(std::integral_constant<int, 1>{});
}

template <bool EXACT, OutKind KIND>
void launch_tiles(const hwsel_fp8_t &A, const hwsel_fp8_t &B, const Plan &p, const Out &o, hipStream_t s)
{
    const int32_t nkb = (int32_t)fp8_blocks(A.cols);
    if constexpr (KIND != kOutFp8) {                        // (to 8 bits through the workspace)
        if (p.way == Way::few)
            return A.rows <= 16 ? launch_few<1, EXACT, KIND>(A, B, p, o, s)
                 : A.rows <= 32 ? launch_few<2, EXACT, KIND>(A, B, p, o, s) : launch_few<4, EXACT, KIND>(A, B, p, o, s);
    }
    if constexpr (!EXACT && KIND != kOutPart) {
        if (p.way == Way::rows) {
            const int32_t n_tiles = (int32_t)((B.rows + 127) / 128), m_tiles = (int32_t)((A.rows + 127) / 128);
            int32_t each = (int32_t)((int64_t)m_tiles * n_tiles / (4 * compute_units()));
            each = each < 1 ? 1 : each > n_tiles ? n_tiles : each;
            const dim3 grid((unsigned)m_tiles, (unsigned)((n_tiles + each - 1) / each));
            auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, operand(A), operand(B), nkb, each, o); };
            if (A.format == HWSEL_FP8_E4M3) {
                if (nkb == 1) go(k_product_rows<1, 2, 0, KIND>);
                else if (nkb == 2) go(k_product_rows<2, 2, 0, KIND>);
                else go(k_product_rows<4, 2, 0, KIND>);
            } else {
                if (nkb == 1) go(k_product_rows<1, 2, 1, KIND>);
                else if (nkb == 2) go(k_product_rows<2, 2, 1, KIND>);
                else go(k_product_rows<4, 2, 1, KIND>);
            }
            return;
        }
        if (p.way == Way::deep) {
            const dim3 grid((unsigned)((B.rows + 255) / 256 * ((A.rows + 255) / 256)));
            if (A.format == HWSEL_FP8_E4M3)
                hipLaunchKernelGGL((k_product_deep<0, KIND>), grid, dim3(512), 0, s, operand(A), operand(B), nkb, o);
            else
                hipLaunchKernelGGL((k_product_deep<1, KIND>), grid, dim3(512), 0, s, operand(A), operand(B), nkb, o);
            return;
        }
    }
    const dim3 grid((unsigned)((B.rows + kBN - 1) / kBN * ((A.rows + p.bm - 1) / p.bm)), (unsigned)p.splits);
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, grid, dim3(256), 0, s, operand(A), operand(B), nkb, p.per_split, o); };
    if constexpr (EXACT) {
        auto by_rows = [&](auto fa) {
            constexpr int FA = decltype(fa)::value;
            if (p.bm == 48) go(k_product_exact<1, 3, FA, KIND>);
            else if (p.bm == 64) go(k_product_exact<1, 4, FA, KIND>);
            else go(k_product_exact<2, 4, FA, KIND>);
        };
        if (A.format == HWSEL_FP8_E4M3) by_rows(std::integral_constant<int, 0>{});
        else by_rows(std::integral_constant<int, 1>{});
    } else if (A.format == HWSEL_FP8_E4M3) {
        if (p.bm == 64) go(k_product<1, 0, KIND>);
        else go(k_product<2, 0, KIND>);
    } else {
        if (p.bm == 64) go(k_product<1, 1, KIND>);
        else go(k_product<2, 1, KIND>);
    }
}

int64_t part_ld(int64_t N) { return (N + 3) / 4 * 4; }

template <OutKind KIND>
hipError_t run_product(const hwsel_fp8_t &A, const hwsel_fp8_t &B, const Out &o, void *ws, hipStream_t s)
{
    const Plan p = plan_product(A.rows, B.rows, fp8_blocks(A.cols), KIND == kOutF32, KIND == kOutFp8);
    if (p.splits == 1 && !(KIND == kOutFp8 && p.way == Way::few)) {
        launch_tiles<KIND == kOutF32, KIND>(A, B, p, o, s);
    } else {
        Out part = o;
        part.C = ws;
        part.ld = part_ld(B.rows);
        launch_tiles<KIND == kOutF32, kOutPart>(A, B, p, part, s);
        const int64_t items = A.rows * ((B.rows + 127) / 128), groups = (items + 7) / 8;
        hipLaunchKernelGGL(k_product_join<KIND>, dim3((unsigned)(groups < 65536 ? groups : 65536)), dim3(256), 0, s,
                           static_cast<const float *>(ws), p.splits, (int32_t)A.rows, (int32_t)B.rows, part.ld, o);
    }
    return hipGetLastError();
}

}  // namespace

// Enough for whatever the result is held in.
size_t fp8_matmul_workspace_bytes(int64_t M, int64_t N, int64_t K)
{
    size_t most = 0;
    for (int exact = 0; exact < 2; ++exact) {
        const Plan p = plan_product(M, N, fp8_blocks(K), exact);
        const bool used = p.splits > 1 || (!exact && p.way == Way::few);
        const size_t bytes = used ? (size_t)p.splits * (size_t)M * (size_t)part_ld(N) * 4 : 0;
        most = bytes > most ? bytes : most;
    }
    return most;
}

bool fp8_product_fits(int64_t M, int64_t N, int64_t K, bool fp32, bool codes)
{
    const Plan p = plan_product(M, N, fp8_blocks(K), fp32, codes);
    return p.way != Way::tiles || (M + p.bm - 1) / p.bm * ((N + kBN - 1) / kBN) * p.splits < (int64_t)1 << 24;
}

hipError_t launch_fp8_matmul(const hwsel_fp8_t &A, const hwsel_fp8_t &B, const float *bias, bool gelu, void *C, bool bf16,
                             int64_t ldc, void *ws, hipStream_t s)
{
    const Out o{C, ldc, nullptr, 0, bias, gelu};
    return bf16 ? run_product<kOutBf16>(A, B, o, ws, s) : run_product<kOutF32>(A, B, o, ws, s);
}

hipError_t launch_fp8_layer(const hwsel_fp8_t &A, const hwsel_fp8_t &B, const float *bias, bool gelu, const hwsel_fp8_t &C,
                            void *ws, hipStream_t s)
{
    return run_product<kOutFp8>(A, B, Out{C.q, C.ld, C.scale, C.ld_scale, bias, gelu}, ws, s);
}

}  // namespace hwsel
