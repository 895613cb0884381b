// Rows of plain fp32 and bf16 matrices eight elements at a time, dropout's mask,
// and sums over lanes: shared by dropout.hip and join.hip.
#pragma once

#include <type_traits>

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

typedef float f32x2_any_t __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_any_t __attribute__((aligned(2)));

// How rows of some length are read eight elements at a time.  The last ones of
// a row that is no whole number of eights are read with those before them, as
// one load like all others, and moved down once they are there: loads wait for
// nothing and go the same way in every thread.  (The last ones as four, two and
// one, with waits in between, 30,000 rows of 1,100 took 229 us.)
struct Ends {
    int32_t tail, shift;                                    // elements past the last whole eight; places they are moved
    bool narrow;                                            // rows of less than eight
};

// Rows of whole eights, and eights that every thread has, known when a kernel is compiled.
struct NoEnds {
    static constexpr int32_t tail = 0, shift = 0;
    static constexpr bool narrow = false;
};

struct AllThere : NoEnds {};

inline Ends ends_of(int64_t cols)
{
    const int32_t tail = (int32_t)(cols & 7);
    return {tail, cols > 8 && tail ? 8 - tail : 0, cols < 8};
}

// Elements at .. of X, n of them left in the row (zeros where n <= 0 or there is no X: none is read); settle8 comes
// before their use.
template <bool BF16, class E>
__device__ __forceinline__ Eight<BF16> load8(const void *X, int64_t at, int32_t n, const E &ends)
{
    Eight<BF16> v{};
    if (!ends.narrow) {
        if (X && (std::is_same_v<E, AllThere> || n > 0)) {
            if (ends.shift != 0) at += n < 8 ? n - 8 : 0;
            if constexpr (BF16) {
                v.w = *reinterpret_cast<const u32x4_any_t *>(static_cast<const uint16_t *>(X) + at);
            } else {
                v.a = *reinterpret_cast<const f32x4_any_t *>(static_cast<const float *>(X) + at);
                v.b = *reinterpret_cast<const f32x4_any_t *>(static_cast<const float *>(X) + at + 4);
            }
        }
        return v;
    }
#pragma unroll
    for (int i = 0; i < 7; ++i) {
        if constexpr (BF16) {
            const uint32_t e = X && i < n ? static_cast<const uint16_t *>(X)[at + i] : 0u;
            v.w[i >> 1] = i & 1 ? v.w[i >> 1] | (e << 16) : e;
        } else {
            const float e = X && i < n ? static_cast<const float *>(X)[at + i] : 0.0f;
            if (i < 4) v.a[i & 3] = e;
            else v.b[i & 3] = e;
        }
    }
    return v;
}

// A row's last elements to their places, zeros behind them (ends.shift is the same for all threads).
template <bool BF16, class E>
__device__ __forceinline__ void settle8(Eight<BF16> &v, int32_t n, const E &ends)
{
    if (ends.shift == 0) return;
    const bool mine = n > 0 && n < 8;
    if constexpr (BF16) {
        uint32_t w[5] = {v.w[0], v.w[1], v.w[2], v.w[3], 0u};
        if (ends.shift & 4) w[0] = w[2], w[1] = w[3], w[2] = 0u, w[3] = 0u;
        if (ends.shift & 2) w[0] = w[1], w[1] = w[2], w[2] = w[3], w[3] = 0u;
        if (ends.shift & 1) {
#pragma unroll
            for (int i = 0; i < 4; ++i) w[i] = __builtin_amdgcn_alignbit(w[i + 1], w[i], 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) v.w[i] = mine ? w[i] : v.w[i];
    } else {
        float w[9] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w, 0.0f};
        if (ends.shift & 4) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < 4 ? w[i + 4] : 0.0f;
        }
        if (ends.shift & 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = i < 6 ? w[i + 2] : 0.0f;
        }
        if (ends.shift & 1) {
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = w[i + 1];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            v.a[i] = mine ? w[i] : v.a[i];
            v.b[i] = mine ? w[i + 4] : v.b[i];
        }
    }
}

// The first n of eight values to elements at .. of X, rounded to nearest even; a
// row's last ones as four, two and one.
template <bool BF16, class E>
__device__ __forceinline__ void store8(void *X, int64_t at, int32_t n, const E &ends, const float (&v)[8])
{
    const int32_t tail = ends.tail;
    const bool two = tail & 2, four = tail & 4;
    if constexpr (BF16) {
        uint16_t *p = static_cast<uint16_t *>(X) + at;
        const uint32_t w[4] = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]), bf16_pair(v[6], v[7])};
        if (std::is_same_v<E, AllThere> || n >= 8) {
            *reinterpret_cast<u32x4_any_t *>(p) = (u32x4_any_t){w[0], w[1], w[2], w[3]};
        } else if (n > 0) {
            const uint32_t first = four ? w[2] : w[0], second = four ? w[3] : w[1];
            if (four) *reinterpret_cast<u32x2_any_t *>(p) = (u32x2_any_t){w[0], w[1]};
            if (two) *reinterpret_cast<u32_any_t *>(p + (tail & 4)) = first;
            if (tail & 1) p[tail & 6] = (uint16_t)(two ? second : first);
        }
    } else {
        float *p = static_cast<float *>(X) + at;
        const f32x4_any_t a = {v[0], v[1], v[2], v[3]}, b = {v[4], v[5], v[6], v[7]};
        if (std::is_same_v<E, AllThere> || n >= 8) {
            *reinterpret_cast<f32x4_any_t *>(p) = a;
            *reinterpret_cast<f32x4_any_t *>(p + 4) = b;
        } else if (n > 0) {
            const f32x4_any_t rest = four ? b : a;
            if (four) *reinterpret_cast<f32x4_any_t *>(p) = a;
            if (two) *reinterpret_cast<f32x2_any_t *>(p + (tail & 4)) = (f32x2_any_t){rest.x, rest.y};
            if (tail & 1) p[tail & 6] = two ? rest.z : rest.x;
        }
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
