// Rows of a cache in few bits: how a row of bytes is laid out and what it stands for.
//
// Elements come in groups of 32 (the last one of a row perhaps shorter).  Of L = 2^bits - 1 levels, lo the least element and
// step the least number of the elements' type from (largest - least) / L on, element x is held as u, the whole number
// nearest to (x - lo) / step, and stands for lo + u step, rounded once.  Bytes of a row: the words of all groups, `bits` of 32
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

// lo and step of the two numbers of a pair, and a pair of levels as the numbers that they stand for: `place` counts the
// pairs of a word from its lowest bits
template <class T, int BITS> struct Pair;

// binary16: levels as the fraction of 1024 or 64 plus themselves, less that; one instruction for both of a pair, and lo + u
// step is rounded once
template <int BITS> struct Pair<_Float16, BITS> {
    f16x2 lo, step;
    __device__ __forceinline__ explicit Pair(uint32_t ends)      // of one group
    {
        lo = __builtin_bit_cast(f16x2, low_halves(ends, ends)), step = __builtin_bit_cast(f16x2, high_halves(ends, ends));
    }
    __device__ __forceinline__ Pair(uint32_t a, uint32_t b)      // of two rows' groups
    {
        lo = __builtin_bit_cast(f16x2, low_halves(a, b)), step = __builtin_bit_cast(f16x2, high_halves(a, b));
    }
    __device__ __forceinline__ uint32_t get(uint32_t w, int place) const
    {
        f16x2 u;
        if (BITS == 8) {
            u = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, w, place ? 0x04030401u : 0x04020400u)) - (_Float16)1024;
        } else {
            if (place >= 2) w >>= 8;
            if (place & 1) u = __builtin_bit_cast(f16x2, (w & 0x00F000F0u) | 0x54005400u) - (_Float16)64;
            else u = __builtin_bit_cast(f16x2, (w & 0x000F000Fu) | 0x64006400u) - (_Float16)1024;
        }
        return __builtin_bit_cast(uint32_t, __builtin_elementwise_fma(u, step, lo));
    }
};

// bfloat16 has no such instructions: levels as 32-bit numbers, one at a time, u step exact, the sum rounded to 24 bits and then
// to eight
template <int BITS> struct Pair<__bf16, BITS> {
    float lo[2], step[2];
    __device__ __forceinline__ explicit Pair(uint32_t ends) : Pair(ends, ends) {}
    __device__ __forceinline__ Pair(uint32_t a, uint32_t b)
    {
        lo[0] = __uint_as_float(a << 16), step[0] = __uint_as_float(a & 0xFFFF0000u);
        lo[1] = __uint_as_float(b << 16), step[1] = __uint_as_float(b & 0xFFFF0000u);
    }
    __device__ __forceinline__ uint32_t get(uint32_t w, int place) const
    {
        if (BITS == 4) w = (place & 1 ? w >> 4 : w) & 0x0F0F0F0Fu;
        const int byte = BITS == 4 ? place / 2 : place;
        const float u0 = (float)((w >> (8 * byte)) & 0xFF), u1 = (float)((w >> (16 + 8 * byte)) & 0xFF);
        const bf16x2 x = {(__bf16)__builtin_fmaf(u0, step[0], lo[0]), (__bf16)__builtin_fmaf(u1, step[1], lo[1])};
        return __builtin_bit_cast(uint32_t, x);
    }
};

// eight elements of a row in order, from BITS / 4 words
template <class T, int BITS> __device__ __forceinline__ typename Elem<T>::x8 eight_of(const uint32_t *words, const Pair<T, BITS> &ends)
{
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    u32x4 x;
#pragma unroll
    for (int p = 0; p < 4; ++p) x[p] = BITS == 4 ? ends.get(words[0], p) : ends.get(words[p / 2], p % 2);
    return __builtin_bit_cast(typename Elem<T>::x8, x);
}

}  // namespace lap
