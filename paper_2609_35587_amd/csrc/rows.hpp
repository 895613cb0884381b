// Rows of plain fp32 and bf16 matrices eight elements at a time, dropout's mask,
// and sums over lanes: shared by dropout.hip and join.hip.
#pragma once

#include "fp8.hpp"

namespace hwsel {

// Eight consecutive elements as they lie in memory.
template <bool BF16>
struct Eight;

template <>
struct Eight<true> {
    u32x4_any_t w;
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(i & 1 ? w[i >> 1] & 0xffff0000u : w[i >> 1] << 16); }
};

template <>
struct Eight<false> {
    f32x4_any_t a, b;
    __device__ __forceinline__ float at(int i) const { return i < 4 ? a[i & 3] : b[i & 3]; }
};

// Elements at .. at + 7 of X, zeros from the n-th on (n >= 8: all; n <= 0: none is read).
template <bool BF16>
__device__ __forceinline__ Eight<BF16> load8(const void *X, int64_t at, int64_t n)
{
    Eight<BF16> v;
    if (n >= 8) {
        if constexpr (BF16) {
            v.w = *reinterpret_cast<const u32x4_any_t *>(static_cast<const uint16_t *>(X) + at);
        } else {
            const f32x4_any_t *p = reinterpret_cast<const f32x4_any_t *>(static_cast<const float *>(X) + at);
            v.a = p[0];
            v.b = p[1];
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if constexpr (BF16) {
            const uint32_t e = i < n ? static_cast<const uint16_t *>(X)[at + i] : 0u;
            v.w[i >> 1] = i & 1 ? v.w[i >> 1] | (e << 16) : e;
        } else {
            const float e = i < n ? static_cast<const float *>(X)[at + i] : 0.0f;
            if (i < 4) v.a[i & 3] = e;
            else v.b[i & 3] = e;
        }
    }
    return v;
}

// The first n of eight values to elements at .. of X, rounded to nearest even.
template <bool BF16>
__device__ __forceinline__ void store8(void *X, int64_t at, int64_t n, const float (&v)[8])
{
    if (n >= 8) {
        if constexpr (BF16) {
            *reinterpret_cast<u32x4_any_t *>(static_cast<uint16_t *>(X) + at) =
                (u32x4_any_t){bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        } else {
            f32x4_any_t *p = reinterpret_cast<f32x4_any_t *>(static_cast<float *>(X) + at);
            p[0] = (f32x4_any_t){v[0], v[1], v[2], v[3]};
            p[1] = (f32x4_any_t){v[4], v[5], v[6], v[7]};
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i)
        if (i < n) {
            if constexpr (BF16) static_cast<uint16_t *>(X)[at + i] = (uint16_t)bf16_pair(v[i], 0.0f);
            else static_cast<float *>(X)[at + i] = v[i];
        }
}

template <bool BF16>
__device__ __forceinline__ float load1(const void *X, int64_t at)
{
    if constexpr (BF16) return bf16_value(static_cast<const uint16_t *>(X)[at]);
    else return static_cast<const float *>(X)[at];
}

// A call's dropout as the kernels take it.
struct Dropout {
    uint64_t seed, offset;
    const uint64_t *state;                                  // (seed, offset) on the device, or null
    uint32_t least;                                         // numbers below it are dropped, of 2^16
    float factor;                                           // 1 / share kept; 0 where nothing is
};

inline Dropout dropout_of(const hwsel_dropout_t &d)
{
    const uint32_t least = (uint32_t)__builtin_rintf(d.p * 65536.0f);
    return {d.seed, d.offset, d.state, least, least < 65536u ? 65536.0f / (float)(65536u - least) : 0.0f};
}

// The mask's key and offset, in scalar registers.
struct Mask {
    uint32_t k0, k1, o0, o1, least;
    float factor;
};

__device__ __forceinline__ Mask mask_of(const Dropout &d)
{
    const uint64_t seed = d.state ? d.state[0] : d.seed, offset = d.state ? d.state[1] : d.offset;
    return {(uint32_t)seed, (uint32_t)(seed >> 32), (uint32_t)offset, (uint32_t)(offset >> 32), d.least, d.factor};
}

// The eight values of columns 8 g .. 8 g + 7 of a row: kept ones times the
// factor, dropped ones 0.  Ten rounds of Philox4x32: two 32 x 32-bit products,
// two exclusive ors of three each, the key moved on by a constant.
__device__ __forceinline__ void drop8(const Mask &m, uint32_t row, uint32_t g, float (&v)[8])
{
    uint32_t c0 = g, c1 = row, c2 = m.o0, c3 = m.o1, k0 = m.k0, k1 = m.k1;
#pragma unroll
    for (int i = 0; i < 10; ++i) {
        const uint64_t p0 = (uint64_t)c0 * 0xd2511f53u, p1 = (uint64_t)c2 * 0xcd9e8d57u;
        c0 = (uint32_t)(p1 >> 32) ^ c1 ^ k0;
        c1 = (uint32_t)p1;
        c2 = (uint32_t)(p0 >> 32) ^ c3 ^ k1;
        c3 = (uint32_t)p0;
        k0 += 0x9e3779b9u;
        k1 += 0xbb67ae85u;
    }
    const uint32_t w[4] = {c0, c1, c2, c3};
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t number = i & 1 ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
        v[i] = number >= m.least ? v[i] * m.factor : 0.0f;
    }
}

}  // namespace hwsel
