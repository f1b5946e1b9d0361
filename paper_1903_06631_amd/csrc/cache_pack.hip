// Rows of keys and values into a cache in 4 or 8 bits an element, and what such rows stand for (packed_rows.h has the layout).
//
// Bound by memory: a row of 128 elements is 256 bytes and 80 (144 in 8 bits) packed.  Four lanes share a group of 32, eight
// elements each; its least and largest element go round them by lane moves.
#include "lap_dev.h"
#include "packed_rows.h"

namespace lap {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

constexpr int NT = 256;
constexpr float WIDEST = 0x1p100f;      // of a group's range: u step and the quotients below stay numbers

// over the four lanes of a group
__device__ __forceinline__ float quad(float x, float (*f)(float, float))
{
    x = f(x, __uint_as_float(dpp_mov<0xB1>(0u, __float_as_uint(x))));      // quad_perm 1 0 3 2
    return f(x, __uint_as_float(dpp_mov<0x4E>(0u, __float_as_uint(x))));      // quad_perm 2 3 0 1
}
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

// eight elements of a group (has: this lane has any), the others by its three neighbours: words and lo | step << 16
template <class T, int BITS> __device__ __forceinline__ void pack(const float (&x)[8], bool has, uint32_t (&words)[BITS / 4], uint32_t &ends)
{
    constexpr float L = (float)((1 << BITS) - 1);
    float lo = x[0], hi = x[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) lo = least(lo, x[i]), hi = most(hi, x[i]);
    lo = quad(has ? lo : ATTN_INF, least) + 0.f, hi = quad(has ? hi : -ATTN_INF, most) + 0.f;      // no minus zero
    const float span = hi - lo;
    const bool good = span <= WIDEST;
    // step: span / L rounded up.  Small ranges are taken times a power of two, so that nothing below loses bits.
    const float up = span < 0x1p-60f ? 0x1p100f : 1.f, down = span < 0x1p-60f ? 0x1p-100f : 1.f;
    const float want = quotient(span * up, L, 1.f / L) * down;
    uint32_t step_bits;
    if constexpr (IS_F16<T>) {
        step_bits = bits_of((T)want);
        step_bits += (float)(T)want < want;
    } else {
        step_bits = (__float_as_uint(want) + 0xFFFFu) >> 16;
    }
    const auto number = [](uint32_t bits) { return (float)__builtin_bit_cast(T, (uint16_t)bits); };
    const bool over = __builtin_fabsf((float)(T)__builtin_fmaf(L, number(step_bits), lo)) == ATTN_INF;
    if (over && good) step_bits -= 1;
    step_bits = good ? step_bits : 0;
    const float step = number(step_bits) * up;
    float inverse = __builtin_amdgcn_rcpf(step);
    inverse = __builtin_fmaf(__builtin_fmaf(-inverse, step, 1.f), inverse, inverse);
    const float base = lo * up;
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = __builtin_rintf(quotient(__builtin_fmaf(x[i], up, -base), step, inverse));
    if (ballot(over)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) u[i] = fminf(u[i], L);
    }
    const bool any = has && step_bits != 0;
#pragma unroll
    for (int w = 0; w < BITS / 4; ++w) {      // places of a half are digits of a whole number, exact in 24 bits
        float half[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float *e = u + w * 4 + h;
            half[h] = BITS == 4 ? __builtin_fmaf(__builtin_fmaf(__builtin_fmaf(e[6], 16.f, e[4]), 16.f, e[2]), 16.f, e[0]) : __builtin_fmaf(e[2], 256.f, e[0]);
        }
        words[w] = any ? (uint32_t)half[0] | (uint32_t)half[1] << 16 : 0;
    }
    ends = (good ? bits_of((T)lo) : bits_of((T)__builtin_nanf(""))) | step_bits << 16;
}

// A workgroup goes through `each` rows of one head's keys or values, all of its threads side by side on rows of 4 G lanes.
template <class T, int BITS, int G, bool WRITE>
__global__ __launch_bounds__(NT) void k_pack(PackShape s, Rows k, Rows v, Rows k_cache, Rows v_cache, uint32_t pieces, uint32_t each)
{
    constexpr int LANES = 4 * G, ROW = (G * (BITS * 4 + 4) + 15) / 16 * 16, PAD = (ROW - G * (BITS * 4 + 4)) / 4;
    const uint32_t piece = blockIdx.x % pieces, head = blockIdx.x / pieces;
    const uint32_t b = head / s.kv_heads, h = head % s.kv_heads;
    const Rows &plain = blockIdx.y ? v : k, &cache = blockIdx.y ? v_cache : k_cache;
    const int lane = threadIdx.x % LANES;
    const int len = clamp_len(s.lens, b, s.n), to = s.first ? s.first[b] : 0;
    const int begin = piece * each, end = min(begin + (int)each, WRITE ? len : (int)s.n);
    T *const rows = (T *)plain.data + (int64_t)b * plain.batch + (int64_t)h * plain.head + lane * 8;
    char *const packed = (char *)cache.data + (int64_t)b * cache.batch + (int64_t)h * cache.head;
    const bool has = lane * 8 < (int)s.head_dim;
    const uint32_t at = lane / 4 * (BITS * 4) + lane % 4 * BITS, ends_at = G * BITS * 4 + lane / 4 * 4;
    for (int i = begin + (int)threadIdx.x / LANES; i < end; i += NT / LANES) {
        if (threadIdx.x >= NT / LANES * LANES) break;
        const int64_t slot = (int64_t)to + i;
        const bool inside = slot >= 0 && slot < (int64_t)s.slots;
        char *const row = packed + slot * cache.row;
        T *const mine = rows + (int64_t)i * plain.row;
        uint32_t words[BITS / 4] = {}, ends = 0;
        if constexpr (WRITE) {
            if (!inside) continue;
            float x[8] = {};
            if (has) {
                const auto y = *(const typename Elem<T>::x8 *)mine;
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = (float)y[j];
            }
            pack<T, BITS>(x, has, words, ends);
            if constexpr (BITS == 4) *(uint32_t *)(row + at) = words[0];
            else *(u32x2 *)(row + at) = u32x2{words[0], words[1]};
            if (lane % 4 == 0) *(uint32_t *)(row + ends_at) = ends;
            if (lane < PAD) *(uint32_t *)(row + ROW - PAD * 4 + lane * 4) = 0;
        } else if (has) {
            typename Elem<T>::x8 y = {};
            if (inside && i < len) {
#pragma unroll
                for (int j = 0; j < BITS / 4; ++j) words[j] = ((const uint32_t *)(row + at))[j];
                y = eight_of<T, BITS>(words, Pair<T, BITS>(*(const uint32_t *)(row + ends_at)));
            }
            *(typename Elem<T>::x8 *)mine = y;
        }
    }
}

template <class T, int BITS, bool WRITE>
hipError_t launch(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st)
{
    const uint32_t groups = pack_groups(s.head_dim), heads = s.batch * s.kv_heads;
    const auto kernel = groups == 1 ? k_pack<T, BITS, 1, WRITE> : groups == 2 ? k_pack<T, BITS, 2, WRITE> : groups == 3 ? k_pack<T, BITS, 3, WRITE> : k_pack<T, BITS, 4, WRITE>;
    const uint32_t each = 256, pieces = (s.n + each - 1) / each;
    kernel<<<dim3(heads * pieces, 2), NT, 0, st>>>(s, k, v, k_cache, v_cache, pieces, each);
    return hipGetLastError();
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
