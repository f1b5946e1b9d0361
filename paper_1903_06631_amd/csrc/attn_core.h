// What the attention kernels share: element types, tiles of rows in LDS, matrix operands out of them, visible ranges.
//
// All products go through the 32x32x16 matrix instruction (C = A B, lane l with h = l / 32):
//   A: row l % 32, contraction indices 8 h .. 8 h + 7          B: column l % 32, the same contraction indices
//   C: column l % 32, element i of 16 is row 8 (i / 4) + 4 h + i % 4
// Scores are computed with the side that a wave keeps in registers as B, so a lane holds scores of one kept row only, 16
// of every 32 of the streamed rows.  Those 16, rounded and in order, are the B operand of the next product over the
// streamed rows (elements 8 s .. 8 s + 7 for its step s), if its A operand takes the streamed rows in the order
// 4 h .. 4 h + 3, 8 + 4 h .. 8 + 4 h + 3: the transposing LDS read fetches four rows at a time, from anywhere, so the
// order costs nothing and no lane has to pass anything on.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_kernels.h"

namespace lap {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

#define ATTN_LDS __attribute__((address_space(3)))
#define ATTN_GLB __attribute__((address_space(1)))

template <class T> struct Elem;
template <> struct Elem<__bf16> {
    typedef __bf16 x8 __attribute__((ext_vector_type(8)));
    typedef __bf16 x4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Elem<_Float16> {
    typedef _Float16 x8 __attribute__((ext_vector_type(8)));
    typedef _Float16 x4 __attribute__((ext_vector_type(4)));
    static __device__ __forceinline__ f32x16 mfma(x8 a, x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

constexpr float LOG2E = 1.4426950408889634f;
constexpr float LN2 = 0.6931471805599453f;
constexpr float LOWEST = -1e30f;      // running maximum of a row's products before its first key; times 1.5e6 still a number
#define ATTN_INF __builtin_inff()

// a number that all lanes hold alike, told to the compiler (divisions leave theirs in vector registers)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// the larger of a lane's value and its partner's in the other half of the wave (and the same for a sum)
__device__ __forceinline__ float half_max(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Rows in LDS.  An asynchronous load puts 64 times 16 bytes side by side, G rows of DP elements; such groups of rows stand
// 16 bytes apart, and within one, chunk c (16 bytes) of row r stands at place c ^ swz(r).  LDS serves 256 bytes at a time
// from 64 banks: 16 rows that follow each other, read at one chunk, or four rows at four neighbouring chunks, then come
// from 16 different places, so neither kind of read below has conflicts (a layout whose places repeat after eight rows took
// twice the LDS cycles).  The places of other groups are a constant away, and go into the instruction.
template <int DP> struct Tile {
    static constexpr int CH = DP / 8;            // chunks of a row
    static constexpr int G = 64 / CH;            // rows of a group
    static constexpr int GROUP = 64 * 8 + 8;     // elements from group to group
    static constexpr int size(int rows) { return rows / G * GROUP; }
    static __device__ __forceinline__ int swz(int row) { return DP == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2 | ((row >> 2) & 1) << 1; }
    static __device__ __forceinline__ int place(int row, int chunk) { return row / G * GROUP + row % G * DP + (chunk ^ swz(row)) * 8; }
};

// ROWS rows from global memory into LDS, asynchronously, by NW waves.  Rows past `last` are copies of it: padding is never
// read.  Chunks past the last one of a row are left alone by lanes that sit out; zero_tiles() has put zeros there, or what comes of them
// is thrown away.  (Copies of the last chunk, times the zeros on the other side of a product, are not a number where that
// chunk holds an infinity.)
// The compiler does not see these loads: it would wait for the ones just sent off before any read of LDS, as it cannot
// tell the tiles apart.  tiles_arrive() waits for them.
template <int DP, int ROWS, int NW> struct TileLoad {
    typedef Tile<DP> L;
    static constexpr int PER = ROWS / L::G / NW;      // instructions of a wave
    static_assert(PER * NW * L::G == ROWS, "whole instructions");
    uint32_t off;           // this lane's bytes of the first instruction; the others are a number of rows further on
    uint32_t stride;        // bytes of a row (at most 2^25 - 16: the start of a tile's 128th row, and that row, are within 32 bits)
    int row0;
    bool takes_part;
    static_assert(ROWS <= 128, "offsets within 32 bits");
    __device__ __forceinline__ TileLoad(int64_t row_stride, int last_chunk, int wave, int lane)
    {
        stride = (uint32_t)row_stride * 2u;
        row0 = wave * PER * L::G + lane / L::CH;
        const int chunk = (lane % L::CH) ^ L::swz(lane / L::CH);
        off = (uint32_t)row0 * stride + (uint32_t)chunk * 16u;
        takes_part = chunk <= last_chunk;
    }
    // rows first .. first + ROWS - 1 of g; first <= last
    template <class T> __device__ __forceinline__ void issue(T *lds, const T *g, int first, int last, int wave) const
    {
        const char *base = (const char *)g + (int64_t)first * stride;
        const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(ATTN_LDS void *)lds + (uint32_t)(wave * PER * L::GROUP * 2));
        const int left = last - first;
        if (!takes_part) return;
        if (left >= ROWS - 1) {
#pragma unroll
            for (int j = 0; j < PER; ++j) send(to + j * (L::GROUP * 2u), off, base + (uint64_t)(j * L::G) * stride);
        } else {
#pragma unroll
            for (int j = 0; j < PER; ++j)
                send(to + j * (L::GROUP * 2u), off + (uint32_t)(min(row0 + j * L::G, left) - row0) * stride, base);
        }
    }
    // 16 bytes for every lane, from base + its offset, to LDS address `to` + 16 times the lane (the register that holds
    // that address is not the compiler's to use)
    static __device__ __forceinline__ void send(uint32_t to, uint32_t offset, const char *base)
    {
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base) : "memory");
    }
};

// Floats from g + first on into LDS, 64 of them by one wave, the part-th 64 of a tile; those past index `last` are copies of
// that one (first <= last)
__device__ __forceinline__ void load_floats(float *lds, const float *g, int first, int last, int part, int lane)
{
    const char *base = (const char *)(g + first);
    const uint32_t to = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(ATTN_LDS void *)(lds + 64 * part));
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(4u * (uint32_t)min(64 * part + lane, last - first)), "s"(base) : "memory");
}

// Zeros into tiles of rows with fewer than DP elements, before the first of them is asked for.
template <int DP, int NT, class T> __device__ __forceinline__ void zero_tiles(T *tiles, int n, uint32_t head_dim)
{
    if (head_dim == DP) return;
    for (int i = threadIdx.x * 8; i < n; i += NT * 8) *(s16x8 *)(tiles + i) = s16x8{};
    __syncthreads();
}

// what has been asked for has arrived in LDS, for every wave, and every wave is done with what it has read there
__device__ __forceinline__ void tiles_arrive()
{
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0070);      // no memory or LDS access under way
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// Operands out of a tile.  RowRead: A of a product over the elements of a row (lane l: row l % 32 of a block of 32).
template <int DP, class T> struct RowRead {
    int at[4];
    __device__ __forceinline__ explicit RowRead(int lane)
    {
#pragma unroll
        for (int i = 0; i < 4; ++i) at[i] = Tile<DP>::place(lane & 31, (DP == 128 ? 4 * i : 2 * i) | (lane >> 5));
    }
    // elements 16 k + 8 h .. of rows 32 block ..
    __device__ __forceinline__ typename Elem<T>::x8 get(const T *tile, int block, int k) const
    {
        return *(const typename Elem<T>::x8 *)(tile + (DP == 128 ? at[k >> 1] + (k & 1) * 16 : at[k]) + Tile<DP>::size(32) * block);
    }
};

// ColRead: A of a product over the rows of the tile (lane l: element 32 d + l % 32 of rows 16 s .., in the order above)
template <int DP, class T> struct ColRead {
    int at[DP / 32];
    __device__ __forceinline__ explicit ColRead(int lane)
    {
        const int g = lane >> 4, i = lane & 15;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) at[d] = Tile<DP>::place(4 * (g >> 1) + (i >> 2), 4 * d + 2 * (g & 1) + ((i & 3) >> 1)) + (i & 1) * 4;
    }
    __device__ __forceinline__ typename Elem<T>::x8 get(const T *tile, int s, int d) const
    {
        T *p = const_cast<T *>(tile) + at[d] + Tile<DP>::size(16) * s;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS s16x4 *)p);
        const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((ATTN_LDS s16x4 *)(p + Tile<DP>::size(8)));
        const s16x8 both = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename Elem<T>::x8, both);
    }
};

// The order of a run of N products with PER LDS reads each: reads stay AHEAD products in front of their use, where the
// compiler, saving registers, would wait for each as it comes.
template <int N, int PER, int AHEAD> __device__ __forceinline__ void reads_ahead()
{
    __builtin_amdgcn_sched_group_barrier(0x100, AHEAD * PER, 0);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        if (i < N - AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, PER, 0);
    }
}

// B of a product over the elements of a row, straight from memory: lane l holds elements 16 k + 8 h .. of its row
template <int DP, class T>
__device__ __forceinline__ void load_kept(typename Elem<T>::x8 (&f)[DP / 16], const T *row, int head_dim, int lane)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k) {
        const int e = 16 * k + 8 * (lane >> 5);
        typename Elem<T>::x8 z = {};
        f[k] = e < head_dim ? *(const typename Elem<T>::x8 *)(row + e) : z;
    }
}

// the same rows into a tile, as rows 32 block ..: zeros included where a row has fewer than DP elements
template <int DP, class T>
__device__ __forceinline__ void keep_in_lds(T *tile, int block, const typename Elem<T>::x8 *f, int lane)
{
#pragma unroll
    for (int k = 0; k < DP / 16; ++k)
        *(typename Elem<T>::x8 *)(tile + Tile<DP>::size(32) * block + Tile<DP>::place(lane & 31, 2 * k + (lane >> 5))) = f[k];
}

// Hidden pairs have weight zero, but zero times infinity is not a number, and so then is the sum.  A workgroup whose sums are
// all numbers is done.  One with a sum that is not (which pairs that are seen may have made so too) runs again with care:
// where some pairs of a block of 32 rows are hidden, the block is looked over, one with a value that is not finite is left
// out, and after the loop its rows are added one by one, from memory, to the sums of the kept rows that see them.  The look
// at the sums takes 1 to 3 % of a call; a look at every such block in the first place took 1 to 13 %.
template <int N> __device__ __forceinline__ bool sums_are_numbers(const f32x16 (&c)[N])
{
    float x[4] = {};      // infinities count as well
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) x[i % 4] = __builtin_fmaf(c[d][i], 0.f, x[i % 4]);
    return __ballot(!((x[0] + x[1]) + (x[2] + x[3]) == 0.f)) == 0;
}
template <int DP, class T> __device__ __forceinline__ bool block_is_finite(const T *tile, int block, int lane)
{
    typedef unsigned short u16x8 __attribute__((ext_vector_type(8)));
    constexpr unsigned short MAGNITUDE = 0x7FFF, TOP = __is_same(T, __bf16) ? 0x7F80 : 0x7C00;
    u16x8 most = {};
#pragma unroll
    for (int j = 0; j < 32 * DP / 8 / 64; ++j) {
        const u16x8 x = *(const u16x8 *)(tile + Tile<DP>::size(32) * block + j * Tile<DP>::GROUP + lane * 8) & MAGNITUDE;
        most = __builtin_elementwise_max(most, x);
    }
    bool fine = true;
#pragma unroll
    for (int j = 0; j < 8; ++j) fine &= most[j] < TOP;
    return __ballot(!fine) == 0;
}
// The same of rows first .. first + 31 in memory, those past `last` as copies of it.
template <class T> __device__ __forceinline__ bool rows_are_finite(const T *g, int64_t stride, int first, int last, uint32_t head_dim, int lane)
{
    const T *row = g + (int64_t)min(first + (lane & 31), last) * stride;
    bool fine = true;
#pragma unroll 1
    for (uint32_t e = 0; e < head_dim; ++e) fine &= __builtin_fabsf((float)row[e]) < ATTN_INF;
    return __ballot(!fine) == 0;
}
template <class T> __device__ __forceinline__ float dot(const T *a, const T *b, uint32_t head_dim)
{
    float x = 0.f;
#pragma unroll 1
    for (uint32_t e = 0; e < head_dim; ++e) x = __builtin_fmaf((float)a[e], (float)b[e], x);
    return x;
}
// a row in memory times its weight added to the sums of a kept row
template <int DP, class T>
__device__ __forceinline__ void add_row(f32x16 (&c)[DP / 32], const T *row, float weight, uint32_t head_dim, int lane)
{
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const uint32_t e = 32 * d + 2 * i + 4 * (lane >> 5);
            if (e < head_dim) {
                const auto x = *(const typename Elem<T>::x4 *)(row + e);
#pragma unroll
                for (int j = 0; j < 4; ++j) c[d][i + j] = __builtin_fmaf((float)x[j], weight, c[d][i + j]);
            }
        }
}

// A wave's sums through LDS to the wave that adds them up: N times 16 numbers of each lane, lanes side by side
template <int N> __device__ __forceinline__ void put_sums(float *box, const f32x16 (&c)[N], int lane)
{
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) box[(16 * d + i) * 64 + lane] = c[d][i];
}
template <int N> __device__ __forceinline__ void add_sums(const float *box, f32x16 (&c)[N], float times, int lane)
{
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) c[d][i] = __builtin_fmaf(box[(16 * d + i) * 64 + lane], times, c[d][i]);
}

// binary16 ends at 65504 and has full precision above 2^-14 only, and a gradient may be of any size.  So what enters a product
// is a multiple of a power of two: probabilities, which are at most 1, of 2^-P16 (those above 2^-26 keep their precision), and
// the ds = p z, z = g.v - delta, of a kept row of 1 / f, f a power of two of the row's own.  f starts high enough for anything
// that the type can show, and comes down, and the row's sums with it, whenever a z times f passes 2^MOST, so that this one is
// then between 2^(MOST - 4) and 2^(MOST - 3).  MOST is 15 less what p is multiplied by: a ds below 2^-25 of the row's largest
// z loses precision, and none passes 2^15.  f moves a few times in a row's first
// blocks and then hardly ever.  The look at 16 values stands in front of the exponentials, which the next reads of LDS then
// hide behind: it takes 3 to 6 % of a backward pass (8 x 16 heads x 2048 tokens x 128, causal: 573 -> 590 us), after them 7 to 12 %.
constexpr int P16 = 12;
constexpr float FIRST_F = 0x1p64f;
template <class T> constexpr bool IS_F16 = __is_same(T, _Float16);
// z times 1, or of a row with one that is too large times what makes f smaller; f and the row's sums likewise
template <int MOST, int N> __device__ __forceinline__ void hold_in_range(float (&z)[16], float &f, f32x16 (&c)[N])
{
    constexpr float LIMIT = (float)(1 << MOST);
    float top = __builtin_fabsf(z[0]);
#pragma unroll
    for (int i = 1; i < 16; ++i) top = fmaxf(top, __builtin_fabsf(z[i]));
    if (!__ballot(top > LIMIT)) return;
    top = half_max(top);
    const float by = top > LIMIT && top < ATTN_INF ? __builtin_ldexpf(1.f, MOST - 3 - __builtin_amdgcn_frexp_expf(top)) : 1.f;
    f *= by;
#pragma unroll
    for (int i = 0; i < 16; ++i) z[i] *= by;
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) c[d][i] *= by;
}
template <int N> __device__ __forceinline__ void times(f32x16 (&c)[N], float by)
{
#pragma unroll
    for (int d = 0; d < N; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) c[d][i] *= by;
}

// eight values of C, from element `first` on, rounded to the nearest: B of the next product
template <class T, int N>
__device__ __forceinline__ typename Elem<T>::x8 round8(const float (&x)[N], int first)
{
    typename Elem<T>::x8 r;
#pragma unroll
    for (int j = 0; j < 8; ++j) r[j] = (T)x[first + j];
    return r;
}

// C with the kept row as its column: elements 32 d + 8 (i / 4) + 4 h .. of that row, times `by`, rounded once
template <int DP, class T>
__device__ __forceinline__ void store_kept(T *row, const f32x16 (&c)[DP / 32], float by, int head_dim, int lane)
{
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
        for (int i = 0; i < 16; i += 4) {
            const int e = 32 * d + 2 * i + 4 * (lane >> 5);
            typename Elem<T>::x4 x;
#pragma unroll
            for (int j = 0; j < 4; ++j) x[j] = (T)(c[d][i + j] * by);
            if (e < head_dim) *(typename Elem<T>::x4 *)(row + e) = x;
        }
}

// How the waves of a workgroup share its work out, by the number of its blocks of 128 kept rows: few leave units empty, so
// more waves take part in each.  Times in us, forward and backward, one sequence of 2048 tokens x 128 with so many heads (16
// blocks each).  Under a causal mask, long tiles first:
//                                                 2         12        20        32        48        64
//   4 blocks of 32 rows, a wave each          41  137    42  139   44  145   50  161   64  196   82  260
//   4 blocks of 32 rows, two waves each       35  106    35  108   38  114   48  149   76  231   99  301
//   2 blocks of 32 rows, four waves each      25   70    29   84   48  138   67  196  102  296  138  400
// Without, equal tiles, which units take in whole rounds:
//                                                 6          9        15        20        32
//   4 blocks of 32 rows, a wave each          42  139    43  141   44  145   62  188   75  232
//   4 blocks of 32 rows, two waves each       35  107    36  109   41  125   72  227   81  252
//   2 blocks of 32 rows, four waves each      25   72    51  145   55  161   78  227  105  310
enum class Share { FOUR, FOUR_BY_TWO, TWO_BY_FOUR };
inline Share share_of(const AttnShape &s, uint32_t heads, uint32_t len)
{
    const uint64_t blocks = (uint64_t)s.batch * heads * ((len + 127) / 128), round = s.causal ? 256 : 128;
    return blocks > 2 * round ? Share::FOUR : blocks > round ? Share::FOUR_BY_TWO : Share::TWO_BY_FOUR;
}

// ---- who sees whom ------------------------------------------------------------------------------------------------

struct Span {
    int ql, kl;      // rows in use
    int off;         // a query's place among the keys is its row + off
};

__device__ __forceinline__ int clamp_len(const int32_t *lens, uint32_t b, uint32_t most)
{
    return lens ? max(0, min(lens[b], (int)most)) : (int)most;
}
__device__ __forceinline__ Span span_of(const AttnShape &s, uint32_t b)
{
    Span p;
    p.ql = clamp_len(s.q_lens, b, s.q_len);
    p.kl = clamp_len(s.k_lens, b, s.k_len);
    p.off = p.kl - p.ql;
    return p;
}
// keys lo .. hi - 1 are visible to query row i (hi <= lo: none)
__device__ __forceinline__ int key_hi(const AttnShape &s, const Span &p, int i) { return s.causal ? min(p.kl, i + p.off + 1) : p.kl; }
__device__ __forceinline__ int key_lo(const AttnShape &s, const Span &p, int i) { return s.window ? max(0, i + p.off + 1 - s.window) : 0; }
// query rows lo .. hi - 1 see key j
__device__ __forceinline__ int row_lo(const AttnShape &s, const Span &p, int j) { return s.causal ? max(0, j - p.off) : 0; }
__device__ __forceinline__ int row_hi(const AttnShape &s, const Span &p, int j)
{
    return s.window ? (int)min((int64_t)p.ql, (int64_t)j - p.off + s.window) : p.ql;
}

// Work of all tiles of the rows of `caches` key heads (times `group` query heads): tile by tile, key heads next to each
// other.  Workgroups are dealt to the eight dies in turn, each with an L2 cache of its own, so with a multiple of eight key
// heads (padded to one where there are many) all that reads one head's rows shares a die, at the same time; and where
// tiles differ in length, all long ones come before all short ones, so that no unit is left with a long one at the end.
struct Work {
    uint32_t tile, b, g, kvh;
};
inline uint32_t padded_caches(uint32_t caches) { return caches < 32 ? caches : (caches + 7) / 8 * 8; }
__device__ __forceinline__ bool work_item(const AttnShape &s, uint32_t group, Work &w)
{
    const uint32_t caches = s.batch * s.kv_heads, padded = caches < 32 ? caches : (caches + 7) / 8 * 8;
    const uint32_t n = blockIdx.x / padded, c = blockIdx.x % padded;
    w.tile = n / group, w.g = n % group;
    w.b = c / s.kv_heads, w.kvh = c % s.kv_heads;
    return c < caches;
}

}  // namespace lap
