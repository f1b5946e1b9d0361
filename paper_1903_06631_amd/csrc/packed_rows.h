// Rows of a cache in few bits: how a row of bytes is laid out and what it stands for.
//
// Elements come in groups of 32 (the last one of a row perhaps shorter).  Of L = 2^bits - 1 levels, lo the least element and
// step the least number of the elements' type from (largest - least) / L on, element x is held as u, the whole number
// nearest to (x - lo) / step, and stands for lo + u step, rounded once (binary16) or to 32 bits and then to the type (bfloat16).  Bytes of a row: the words of all groups, `bits` of 32
// bits for each; then lo and step of each group, 16 bits each; then zeros up to a multiple of 16.
//
// A word's low half holds its even elements from the lowest bits up, its high half the odd ones at the same places.  So one
// mask leaves a pair of levels in two halves, as the packed instructions of binary16 take them; and the low halves of the words
// of two rows, put side by side, are pairs of one element of both rows: a matrix operand along the rows needs no
// transposition through LDS, which rows of plain numbers do.
#pragma once
#include "attn_core.h"

namespace lap {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// words of two rows: their low halves side by side, and their high halves
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }

// Levels as numbers, two by two.  Words of 4 bits are split into two whose bytes are levels below 16: as numbers of eight bits with
// three of fraction, such a byte is that many 2^-9, exactly, and one instruction converts two.  Masks, shifts to the right,
// sums and products of 32 bits take half of the time of other vector instructions (and of packed ones of 16 bits), so a pair of binary16
// costs 2.4 of the latter (with masked levels as the fraction of 1024 or 64, less that: 3.1), one of bfloat16 3.4 (each level
// masked and converted alone: 4.4).  In 8 bits 3 and 4.
template <int BITS> struct Levels;
template <> struct Levels<4> {
    uint32_t w[2];
    __device__ __forceinline__ explicit Levels(uint32_t x) : w{x & 0x0F0F0F0Fu, (x >> 4) & 0x0F0F0F0Fu} {}
};
template <> struct Levels<8> {
    uint32_t w;
    __device__ __forceinline__ explicit Levels(uint32_t x) : w(x) {}
};

// Words of two slots, their levels two by two of the same element: place p of the low (or high) halves holds element 2 p (+ 1).
template <int BITS> __device__ __forceinline__ Levels<BITS> side_by_side(uint32_t a, uint32_t b, bool high)
{
    const uint32_t sel = BITS == 4 ? (high ? 0x07030602u : 0x05010400u) : high ? 0x07060302u : 0x05040100u;
    return Levels<BITS>(__builtin_amdgcn_perm(b, a, sel));
}
// A word of one row: place p holds, in 4 bits, elements e and e + 4, e = 0 2 1 3; in 8 bits 2 p and 2 p + 1.
constexpr int HELD_4[8] = {0, 4, 2, 6, 1, 5, 3, 7};
template <int BITS> __device__ __forceinline__ constexpr int held(int i) { return BITS == 4 ? HELD_4[i] : i; }      // of eight elements

// lo and step of the two numbers of a pair, and what a pair of levels stands for
template <class T, int BITS> struct Pair;

// binary16: one instruction for both, lo + u step is rounded once
template <int BITS> struct Pair<_Float16, BITS> {
    f16x2 lo, step;
    __device__ __forceinline__ explicit Pair(uint32_t ends) : Pair(ends, ends) {}      // of one group
    __device__ __forceinline__ Pair(uint32_t a, uint32_t b)                            // of two rows' groups
    {
        lo = __builtin_bit_cast(f16x2, low_halves(a, b)), step = __builtin_bit_cast(f16x2, high_halves(a, b));
    }
    template <int PLACE> __device__ __forceinline__ uint32_t get(const Levels<BITS> &x) const
    {
        f16x2 u;
        if constexpr (BITS == 4) {
            u = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x.w[PLACE & 1], 512.f, PLACE >> 1));
        } else {      // as the fraction of 1024
            u = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, x.w, PLACE ? 0x04030401u : 0x04020400u)) - (_Float16)1024;
        }
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(u, step, lo));
    }
};

// bfloat16 has no such instruction: u step exact, the sum rounded to 24 bits and then to eight
template <int BITS> struct Pair<__bf16, BITS> {
    float lo[2], step[2];
    __device__ __forceinline__ explicit Pair(uint32_t ends) : Pair(ends, ends) {}
    __device__ __forceinline__ Pair(uint32_t a, uint32_t b)
    {
        lo[0] = __uint_as_float(a << 16), step[0] = __uint_as_float(a & 0xFFFF0000u);
        lo[1] = __uint_as_float(b << 16), step[1] = __uint_as_float(b & 0xFFFF0000u);
    }
    template <int PLACE> __device__ __forceinline__ uint32_t get(const Levels<BITS> &x) const
    {
        float u[2];
        if constexpr (BITS == 4) {
            const auto y = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(x.w[PLACE & 1], 512.f, PLACE >> 1);
            u[0] = y[0], u[1] = y[1];
        } else {
            u[0] = (float)((x.w >> (8 * PLACE)) & 0xFF), u[1] = (float)((x.w >> (16 + 8 * PLACE)) & 0xFF);
        }
        const bf16x2 y = {(__bf16)__builtin_fmaf(u[0], step[0], lo[0]), (__bf16)__builtin_fmaf(u[1], step[1], lo[1])};
        return __builtin_bit_cast(uint32_t, y);
    }
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// eight elements of a row from BITS / 4 words, as they are held
template <class T, int BITS> __device__ __forceinline__ u32x4 eight_as_held(const uint32_t *words, const Pair<T, BITS> &ends)
{
    if constexpr (BITS == 4) {
        const Levels<4> x(words[0]);
        return u32x4{ends.template get<0>(x), ends.template get<1>(x), ends.template get<2>(x), ends.template get<3>(x)};
    } else {
        const Levels<8> x(words[0]), y(words[1]);
        return u32x4{ends.template get<0>(x), ends.template get<1>(x), ends.template get<0>(y), ends.template get<1>(y)};
    }
}
// and in order
template <class T, int BITS> __device__ __forceinline__ typename Elem<T>::x8 eight_of(const uint32_t *words, const Pair<T, BITS> &ends)
{
    u32x4 x = eight_as_held<T, BITS>(words, ends);
    if (BITS == 4) x = u32x4{low_halves(x[0], x[2]), low_halves(x[1], x[3]), high_halves(x[0], x[2]), high_halves(x[1], x[3])};
    return __builtin_bit_cast(typename Elem<T>::x8, x);
}

// What a slot receives from a row of queries: from its product, the row's largest one and the logarithm to base 2 of the row's sum on
// that, with c, products to exponents of two.  A slot that the row does not see (minus infinity) receives nothing, also where the row's sum
// is not a number.
__device__ __forceinline__ float received(float x, float2 whole, float c)
{
    const float p = exp2_fast(__builtin_fmaf(x - whole.x, c, -whole.y));
    return x == -ATTN_INF ? 0.f : p;
}

}  // namespace lap
