// Rows of keys and values into a cache in 4 or 8 bits an element, and what such rows stand for (packed_rows.h has the layout).
//
// Bound by memory: a row of 128 elements is 256 bytes and 80 (144 in 8 bits) packed.  Lanes have eight elements each, next to each
// other, so four of them share a group.  What is computed once for a group, two divisions' worth, would be most of the work of
// packing; so four lanes go through four rows at a time, and each computes it for one of them.
//
// Measured, kernels alone: a token of 64 sequences x 8 heads in 4 bits 3.5 us packed and 3.0 us unpacked, a launch; 8 x 8 x up
// to 16 384 rows 68 us (5.8 TB/s; 300 MB of plain rows and 94 of packed; of the cycles of all SIMDs 77 % go to vector instructions) and,
// with the rows past the lengths written as zeros, 82 us (630 MB, 7.7 TB/s); 2 x 8 x 131 072 rows
// unpacked 223 us, 1.41 GB at 6.3 TB/s, beyond what a copy reaches (4.9), as less is read than written.
#include "lap_dev.h"
#include "packed_rows.h"

namespace lap {
namespace {

constexpr int NT = 256;
constexpr float WIDEST = 0x1p100f;      // of a group's range: u step and the quotients below stay numbers

// not a number if either is
__device__ __forceinline__ float least(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float most(float a, float b) { return __builtin_elementwise_maximum(a, b); }

template <class T> __device__ __forceinline__ uint32_t bits_of(T x) { return __builtin_bit_cast(uint16_t, x); }

// a / b rounded to the nearest, from y near 1 / b: the remainder is exact
__device__ __forceinline__ float quotient(float a, float b, float y)
{
    const float q = a * y;
    return __builtin_fmaf(__builtin_fmaf(-q, b, a), y, q);
}

// quad_perm moves: a lane's neighbour by one and by two in the four of a group, and the value of one of the four for all
__device__ __forceinline__ float next_one(float x) { return __uint_as_float(dpp_mov<0xB1>(0u, __float_as_uint(x))); }
__device__ __forceinline__ float next_two(float x) { return __uint_as_float(dpp_mov<0x4E>(0u, __float_as_uint(x))); }
template <int LANE> __device__ __forceinline__ float of_lane(float x) { return __uint_as_float(dpp_mov<LANE * 0x55>(0u, __float_as_uint(x))); }

// one value of each of four rows in each of four lanes: f over the lanes, of row q in lane q
template <class F> __device__ __forceinline__ float each_its_row(const float (&x)[1], int, F &&f)      // (of one row: in all four)
{
    const float a = f(x[0], next_one(x[0]));
    return f(a, next_two(a));
}
template <class F> __device__ __forceinline__ float each_its_row(const float (&x)[4], int lane, F &&f)
{
    const bool odd = lane & 1, high = lane & 2;
    // rows 0 and 2, or 1 and 3, of two lanes; then of four
    const float a = f(odd ? x[1] : x[0], next_one(odd ? x[0] : x[1])), b = f(odd ? x[3] : x[2], next_one(odd ? x[2] : x[3]));
    return f(high ? b : a, next_two(high ? a : b));
}

template <int N> struct Int {
    static constexpr int value = N;
};

// What a group's elements are held by.  Small ranges are taken times a power of two, so that nothing loses bits.
struct Group {
    float up, base, step, inverse;      // base: lo, and step, times up; 1 / step, nearly
    uint32_t ends;                      // lo | step << 16
    bool over, any;                     // step was cut; levels are not all 0
};
template <class T, int BITS> __device__ __forceinline__ Group group_of(float lo, float hi)
{
    constexpr float L = (float)((1 << BITS) - 1);
    Group r;
    lo += 0.f, hi += 0.f;      // no minus zero
    const float span = hi - lo;
    const bool good = span <= WIDEST;
    const float down = span < 0x1p-60f ? 0x1p-100f : 1.f;
    r.up = span < 0x1p-60f ? 0x1p100f : 1.f;
    const float want = quotient(span * r.up, L, 1.f / L) * down;      // step is this, rounded up
    uint32_t step_bits;
    if constexpr (IS_F16<T>) {
        step_bits = bits_of((T)want);
        step_bits += (float)(T)want < want;
    } else {
        step_bits = (__float_as_uint(want) + 0xFFFFu) >> 16;
    }
    const auto number = [](uint32_t bits) { return (float)__builtin_bit_cast(T, (uint16_t)bits); };
    r.over = good && __builtin_fabsf((float)(T)__builtin_fmaf(L, number(step_bits), lo)) == ATTN_INF;
    step_bits = good ? step_bits - r.over : 0;
    r.any = step_bits != 0;
    r.step = number(step_bits) * r.up;
    const float y = __builtin_amdgcn_rcpf(r.step);
    r.inverse = __builtin_fmaf(__builtin_fmaf(-y, r.step, 1.f), y, y);
    r.base = lo * r.up;
    r.ends = (good ? bits_of((T)lo) : bits_of((T)__builtin_nanf(""))) | step_bits << 16;
    return r;
}

// levels of eight elements: the nearest whole numbers of their quotients, ties to even
template <int BITS, bool CUT> __device__ __forceinline__ void levels_of(const float (&x)[8], float up, float base, float step, float inverse, uint32_t (&words)[BITS / 4])
{
    const auto level = [&](float y, int byte, uint32_t old) {
        float q = quotient(__builtin_fmaf(y, up, -base), step, inverse);
        if (BITS == 4 && CUT) q = fminf(q, 15.f);
        return __builtin_amdgcn_cvt_pk_u8_f32(q, byte, old);      // 255 at most, and 0 for what is not a number
    };
    if constexpr (BITS == 8) {
#pragma unroll
        for (int w = 0; w < 2; ++w) words[w] = level(x[4 * w + 3], 3, level(x[4 * w + 1], 2, level(x[4 * w + 2], 1, level(x[4 * w], 0, 0))));
    } else {
        words[0] = level(x[5], 3, level(x[1], 2, level(x[4], 1, level(x[0], 0, 0)))) | level(x[7], 3, level(x[3], 2, level(x[6], 1, level(x[2], 0, 0)))) << 4;
    }
}

struct Place {      // of a workgroup: `each` rows of one head's keys or values
    uint32_t b, h;
    int begin, len, to;      // first row, rows in use, slot of row 0
    int from, until;         // the rows that have a slot
    Rows plain, cache;
};
__device__ __forceinline__ Place place_of(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, uint32_t pieces, uint32_t each)
{
    Place p;
    const uint32_t head = blockIdx.x / pieces;
    p.b = head / s.kv_heads, p.h = head % s.kv_heads;
    p.begin = (int)((blockIdx.x - head * pieces) * each);
    p.len = clamp_len(s.lens, p.b, s.n), p.to = s.first ? s.first[p.b] : 0;
    p.from = (int)min(max(-(int64_t)p.to, (int64_t)0), (int64_t)s.n);
    p.until = (int)min(max((int64_t)s.slots - p.to, (int64_t)0), (int64_t)p.len);
    p.plain = blockIdx.y ? v : k, p.cache = blockIdx.y ? v_cache : k_cache;
    return p;
}

// Few rows: one for a thread, which is a shorter chain (64 x 8 rows packed 5.7 us in a row of launches and 6.4 with four; 1430
// workgroups' worth 8.2 and 7.9).  More: several (unpacked 1, 2, 4 and 8 rows to a thread: 6 x 4 x up to 4099 rows of 80 in 12.3, 9.2, 8.8 and
// 9.1 us, 2 x 8 x 131 072 in 303, 231, 245 and 252).  Many: plain rows that do not stay in the caches anyway pass them by, so
// that packed ones, and what is written, do not make way for them (8 x 8 x up to 16 384 rows packed and unpacked 154 us, otherwise 202).
// From 32 MiB of plain rows on, which is where unpacking alone gains: 52 MiB 10.2 us in place of 12.5, 128 MiB 26 and 27, 256 MiB 50 and 63.  Where attention
// reads the unpacked rows next it would be from some 256 MiB on: both calls, 8 key heads and 16 (512) new tokens of 32 query heads, 52 MiB 48 (181) us
// and with rows that stay 42 (158), 128 MiB 91 (422) and 79 (373), 256 MiB 170 (849) and 186 (819).
enum class How { FEW, SOME, PASSING };
__host__ __device__ constexpr int rows_of_thread(How how, bool write) { return how == How::FEW ? 1 : write || how == How::SOME ? 4 : 2; }

// all of a workgroup's threads side by side, 4 G for a row
template <class T, int BITS, int G, How HOW>
__global__ __launch_bounds__(NT) void k_pack(PackShape s, Rows k, Rows v, Rows k_cache, Rows v_cache, uint32_t pieces, uint32_t each)
{
    constexpr int ROWS = rows_of_thread(HOW, true), LANES = 4 * G, SIDE = NT / LANES, ENDS = G * BITS * 4, PAD = ((ENDS + G * 4 + 15) / 16 * 16 - ENDS - G * 4) / 4;
    const Place p = place_of(s, k, v, k_cache, v_cache, pieces, each);
    const int begin = max(p.begin, p.from), end = min(p.begin + (int)each, p.until), lane = threadIdx.x % LANES;
    if (threadIdx.x >= SIDE * LANES || begin >= end) return;
    const int first = begin + (int)threadIdx.x / LANES;
    // lanes without elements: those of the group's last eight again
    const T *const from = (const T *)p.plain.data + (int64_t)p.b * p.plain.batch + (int64_t)p.h * p.plain.head + (int64_t)first * p.plain.row + min(lane * 8, (int)s.head_dim - 8);
    char *const to = (char *)p.cache.data + (int64_t)p.b * p.cache.batch + (int64_t)p.h * p.cache.head + ((int64_t)p.to + first) * p.cache.row;
    const int64_t side = SIDE * p.cache.row;
    const bool has = lane * 8 < (int)s.head_dim;
    const int left = end - 1 - first;      // rows from this lane's first on, less one; rows past the end: the last one again
    float x[ROWS][8], lows[ROWS], highs[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const auto *const row = (const typename Elem<T>::x8 *)(from + (int64_t)min(r * SIDE, left) * (int)p.plain.row);
        const auto y = HOW == How::PASSING ? __builtin_nontemporal_load(row) : *row;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[r][j] = (float)y[j];
        lows[r] = highs[r] = x[r][0];
#pragma unroll
        for (int j = 1; j < 8; ++j) lows[r] = least(lows[r], x[r][j]), highs[r] = most(highs[r], x[r][j]);
    }
    const Group mine = group_of<T, BITS>(each_its_row(lows, lane, least), each_its_row(highs, lane, most));      // of row lane % ROWS
    const float any = mine.any ? 1.f : 0.f;
    const auto one_row = [&](auto which, auto cut) {
        constexpr int R = decltype(which)::value;
        uint32_t words[BITS / 4];
        levels_of<BITS, decltype(cut)::value != 0>(x[R], of_lane<R>(mine.up), of_lane<R>(mine.base), of_lane<R>(mine.step), of_lane<R>(mine.inverse), words);
        const bool any_r = of_lane<R>(any) != 0.f, some = has && any_r;      // (the lane with that row may have no elements itself)
        if (R * SIDE > left) return;
        char *const row = to + R * side;
        if constexpr (BITS == 4) *(uint32_t *)(row + lane * 4) = some ? words[0] : 0;
        else *(u32x2 *)(row + lane * 8) = some ? u32x2{words[0], words[1]} : u32x2{};
        if (lane < PAD) *(uint32_t *)(row + ENDS + G * 4 + lane * 4) = 0;
    };
    const auto all_rows = [&](auto cut) {
        one_row(Int<0>(), cut);
        if constexpr (ROWS == 4) one_row(Int<1>(), cut), one_row(Int<2>(), cut), one_row(Int<3>(), cut);
    };
    if (ballot(mine.over)) all_rows(Int<1>());
    else all_rows(Int<0>());
    if (ROWS == 4 ? lane % 4 * SIDE <= left : lane % 4 == 0 && left >= 0) *(uint32_t *)(to + lane % ROWS * side + ENDS + lane / 4 * 4) = mine.ends;
}

// and the other way
template <class T, int BITS, int G, How HOW>
__global__ __launch_bounds__(NT) void k_unpack(PackShape s, Rows k, Rows v, Rows k_cache, Rows v_cache, uint32_t pieces, uint32_t each)
{
    constexpr int ROWS = rows_of_thread(HOW, false), LANES = 4 * G, SIDE = NT / LANES, ENDS = G * BITS * 4;
    const Place p = place_of(s, k, v, k_cache, v_cache, pieces, each);
    const int lane = threadIdx.x % LANES, first = p.begin + (int)threadIdx.x / LANES;
    if (threadIdx.x >= SIDE * LANES || lane * 8 >= (int)s.head_dim) return;
    T *const to = (T *)p.plain.data + (int64_t)p.b * p.plain.batch + (int64_t)p.h * p.plain.head + (int64_t)first * p.plain.row + lane * 8;
    const char *const from = (const char *)p.cache.data + (int64_t)p.b * p.cache.batch + (int64_t)p.h * p.cache.head + ((int64_t)p.to + first) * p.cache.row;
    uint32_t words[ROWS][BITS / 4], ends[ROWS];
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        const int i = first + r * SIDE;
        const char *const row = from + (int64_t)(r * SIDE) * p.cache.row;
        const bool some = i >= p.from && i < p.until;      // else zeros, as lo and step
#pragma unroll
        for (int j = 0; j < BITS / 4; ++j) words[r][j] = some ? ((const uint32_t *)(row + lane * BITS))[j] : 0;
        ends[r] = some ? *(const uint32_t *)(row + ENDS + lane / 4 * 4) : 0;
    }
#pragma unroll
    for (int r = 0; r < ROWS; ++r) {
        if (first + r * SIDE >= (int)s.n) return;
        const auto y = eight_of<T, BITS>(words[r], Pair<T, BITS>(ends[r]));
        auto *const row = (typename Elem<T>::x8 *)(to + (int64_t)(r * SIDE) * p.plain.row);
        if (HOW == How::PASSING) __builtin_nontemporal_store(y, row);
        else *row = y;
    }
}

constexpr uint64_t MANY_BYTES = 32 << 20, FEW_GROUPS = 1024;
template <class T, int BITS, bool WRITE, How HOW>
hipError_t launch(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st)
{
    const uint32_t g = pack_groups(s.head_dim), heads = s.batch * s.kv_heads;
    const auto kernel = WRITE ? (g == 1 ? k_pack<T, BITS, 1, HOW> : g == 2 ? k_pack<T, BITS, 2, HOW> : g == 3 ? k_pack<T, BITS, 3, HOW> : k_pack<T, BITS, 4, HOW>)
                              : (g == 1 ? k_unpack<T, BITS, 1, HOW> : g == 2 ? k_unpack<T, BITS, 2, HOW> : g == 3 ? k_unpack<T, BITS, 3, HOW> : k_unpack<T, BITS, 4, HOW>);
    const uint32_t each = NT / (4 * g) * rows_of_thread(HOW, WRITE), pieces = (s.n + each - 1) / each;
    kernel<<<dim3(heads * pieces, 2), NT, 0, st>>>(s, k, v, k_cache, v_cache, pieces, each);
    return hipGetLastError();
}
template <class T, int BITS, bool WRITE>
hipError_t launch(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st)
{
    const uint64_t heads = (uint64_t)s.batch * s.kv_heads, side = NT / (4 * pack_groups(s.head_dim));
    if (heads * s.n * s.head_dim * 4 > MANY_BYTES) return launch<T, BITS, WRITE, How::PASSING>(s, k, v, k_cache, v_cache, st);
    if (2 * heads * ((s.n + side - 1) / side) <= FEW_GROUPS) return launch<T, BITS, WRITE, How::FEW>(s, k, v, k_cache, v_cache, st);
    return launch<T, BITS, WRITE, How::SOME>(s, k, v, k_cache, v_cache, st);
}
template <bool WRITE>
hipError_t launch(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st)
{
    if (s.half) return s.bits == 4 ? launch<_Float16, 4, WRITE>(s, k, v, k_cache, v_cache, st) : launch<_Float16, 8, WRITE>(s, k, v, k_cache, v_cache, st);
    return s.bits == 4 ? launch<__bf16, 4, WRITE>(s, k, v, k_cache, v_cache, st) : launch<__bf16, 8, WRITE>(s, k, v, k_cache, v_cache, st);
}

}  // namespace

hipError_t launch_cache_pack(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st)
{
    return launch<true>(s, k, v, k_cache, v_cache, st);
}
hipError_t launch_cache_unpack(const PackShape &s, const Rows &k_cache, const Rows &v_cache, const Rows &k, const Rows &v, hipStream_t st)
{
    return launch<false>(s, k, v, k_cache, v_cache, st);
}

}  // namespace lap
