// Attention of one or a few new tokens of every sequence over a cache in 4 or 8 bits an element, and the weight that every slot
// receives from them:
//   o_i = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j - lse_i), over the slots in use that row i sees; w_j += sum_i p_ij
// with k and v the numbers that the packed rows stand for, rounded to the element type as in cache_unpack.
//
// p is rounded to the values' type for its product with them (a matrix operand), in binary16 as a multiple of 2^-12, so that
// those below 2^-26 of the largest of their wave lose precision and none of them vanishes above 2^-36.  Sums, scores and weights
// are 32 bits.
//
// Every packed row is read once.  The rows of queries that share a key head, heads times tokens, are the columns of 16 of the
// 16x16x32 matrix instruction (C = A B, lane l with g = l / 16):
//   A: row l % 16, contraction indices 8 g .. 8 g + 7      B: column l % 16, the same      C: column l % 16, rows 4 g .. 4 g + 3
// Keys are A of the scores: a lane holds a fourth of a slot's row, which is one group of 32 elements where rows have 128, so it
// needs one lo and one step.  Values are A of the outputs, elements along the rows: a lane holds one word of eight slots,
// whose low and high halves, side by side for two slots, are the operand's pairs (packed_rows.h).  So both go from memory
// straight into registers and from there into the products, without LDS; the contraction over slots runs in the order in which
// the scores stand in C.  Waves go through 32 slots at a time of their own, without waiting for each other, and ask for the
// next keys when these ones are decoded, for the next values likewise.
//
// Chunks of long caches, one workgroup for short ones, the scores kept for the weights: as in attention_step.hip.
#include "packed_rows.h"

namespace lap {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int TS = 32;                      // slots of a wave's tile
constexpr uint32_t CHUNK_WAVES = 4;         // waves of a chunk's workgroup
constexpr uint32_t WHOLE_WAVES = 8;         // and of one that goes through a whole cache
constexpr uint32_t WHOLE_SCORES = 6144;     // scores that the latter keeps in LDS

__host__ __device__ __forceinline__ uint32_t score_pitch(uint32_t slots) { return (slots + TS - 1) / TS * TS + 4; }

// CHUNK: one of several workgroups of a cache, to be joined.  Or the only one, of up to 32 rows, with its scores in the
// workspace (WHOLE) or in LDS.
enum class Form { CHUNK, WHOLE, WHOLE_IN_LDS };

template <class T> struct Small;
template <> struct Small<__bf16> {
    static __device__ __forceinline__ f32x4 mfma(Elem<__bf16>::x8 a, Elem<__bf16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Small<_Float16> {
    static __device__ __forceinline__ f32x4 mfma(Elem<_Float16>::x8 a, Elem<_Float16>::x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
};

// over the four lanes that hold the same column of C
__device__ __forceinline__ float column_max(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_max(fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1])));
}
__device__ __forceinline__ float column_sum(float x)
{
    const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return half_sum(__uint_as_float(r[0]) + __uint_as_float(r[1]));
}

// The packed words of 32 slots that a lane holds, and where they stand in a row.  Lanes whose share of a row is past its last
// group hold the last group's: queries are zero there, and outputs thrown away.
template <int BITS, int DP> struct Words {
    static constexpr int KW = DP * BITS / 128;                       // words of a key's fourth
    static constexpr int VW = DP * BITS >= 512 ? DP * BITS / 512 : 1;      // of a value's sixteenth (of 32 bytes: half a word)
    uint32_t k[2][KW], k_ends[2], v[8][VW], v_ends[8];
};

template <int BITS, int DP> struct Loader {
    typedef Words<BITS, DP> W;
    const char *k, *v;                     // of the cache
    int64_t k_row, v_row;
    uint32_t k_at, k_ends, v_at, v_ends;   // bytes from the start of a tile
    uint32_t k_lane, v_lane;               // the same without the lane's slot
    uint32_t k_gap, v_gap;                 // from the words to lo and step
    int n, g;
    __device__ __forceinline__ Loader(const Rows &rk, const Rows &rv, uint32_t b, uint32_t kvh, uint32_t head_dim, int lane)
    {
        n = lane & 15, g = lane >> 4;
        k = (const char *)rk.data + (int64_t)b * rk.batch + (int64_t)kvh * rk.head;
        v = (const char *)rv.data + (int64_t)b * rv.batch + (int64_t)kvh * rv.head;
        k_row = rk.row, v_row = rv.row;
        const uint32_t groups = pack_groups(head_dim), ends = pack_ends(head_dim, BITS);
        const uint32_t kg = min((uint32_t)(DP == 128 ? g : g >> 1), groups - 1), vg = min((uint32_t)(DP == 128 ? n >> 2 : n >> 3), groups - 1);
        k_lane = kg * (BITS * 4) + (DP == 128 ? 0 : (g & 1) * (BITS * 2));
        v_lane = vg * (BITS * 4) + (DP == 128 ? (n & 3) * BITS : BITS == 8 ? (n & 7) * 4 : (n >> 1 & 3) * 4);
        k_gap = ends + kg * 4 - k_lane, v_gap = ends + vg * 4 - v_lane;
        k_at = n * (uint32_t)k_row + k_lane, v_at = 4 * g * (uint32_t)v_row + v_lane;
    }
    static __device__ __forceinline__ int slot(int i) { return i < 4 ? i : 12 + i; }      // of a lane's i-th value, less 4 g
    static __device__ __forceinline__ uint32_t word(const char *p, uint32_t off) { return *(const uint32_t *)(p + off); }
    template <int N> static __device__ __forceinline__ void words(uint32_t (&w)[N], const char *p, uint32_t off)
    {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const u32x4 x = *(const u32x4 *)(p + off + 4 * i);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i + j] = x[j];
            }
        } else if constexpr (N == 2) {
            const uint2 x = *(const uint2 *)(p + off);
            w[0] = x.x, w[1] = x.y;
        } else {
            w[0] = word(p, off);
        }
    }
    // keys of slots at .. at + 31; those past `last` are copies of it (at <= last)
    __device__ __forceinline__ void keys(W &w, int at, int last) const
    {
        const char *base = k + (int64_t)at * k_row;
        if (at + TS - 1 <= last) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const char *p = base + 16 * h * k_row;
                words(w.k[h], p, k_at), w.k_ends[h] = word(p, k_at + k_gap);
            }
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t off = (uint32_t)min(16 * h + n, last - at) * (uint32_t)k_row + k_lane;
                words(w.k[h], base, off), w.k_ends[h] = word(base, off + k_gap);
            }
        }
    }
    __device__ __forceinline__ void values(W &w, int at, int last) const
    {
        const char *base = v + (int64_t)at * v_row;
        if (at + TS - 1 <= last) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const char *p = base + slot(i) * v_row;
                words(w.v[i], p, v_at), w.v_ends[i] = word(p, v_at + v_gap);
            }
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t off = (uint32_t)min(4 * g + slot(i), last - at) * (uint32_t)v_row + v_lane;
                words(w.v[i], base, off), w.v_ends[i] = word(base, off + v_gap);
            }
        }
    }
};

// Columns of values: operand j of DP / 16 is one element of eight slots, element at(i, j) of the DP / 4 of the lanes 4 g + i.
template <class T, int BITS, int DP> struct Columns {
    static constexpr int N = DP / 16;
    static __device__ __forceinline__ constexpr int at(int i, int j)
    {
        if (DP == 128) return BITS == 4 ? 8 * i + 2 * (j & 3) + (j >> 2) : 8 * i + 4 * (j >> 2) + 2 * (j & 1) + (j >> 1 & 1);
        return BITS == 4 ? 8 * (i >> 1) + 2 * j + (i & 1) : 4 * i + 2 * (j & 1) + (j >> 1);
    }
    template <class F> static __device__ __forceinline__ void for_all(const Words<BITS, DP> &w, int lane, F &&f)
    {
        constexpr int PER = BITS == 4 ? 4 : 2;                  // places of a half
        constexpr int HALVES = N / PER;                         // low and high ones of a lane's words
        u32x4 x[N];
#pragma unroll
        for (int s = 0; s < 4; ++s) {                           // two slots at a time
            const Pair<T, BITS> ends(w.v_ends[2 * s], w.v_ends[2 * s + 1]);
#pragma unroll
            for (int h = 0; h < HALVES; ++h) {
                const uint32_t a = w.v[2 * s][h / 2], b = w.v[2 * s + 1][h / 2];
                const uint32_t side = HALVES == 1 ? __builtin_amdgcn_perm(b, a, lane & 1 ? 0x07060302u : 0x05040100u) : h % 2 ? high_halves(a, b) : low_halves(a, b);
#pragma unroll
                for (int p = 0; p < PER; ++p) x[h * PER + p][s] = ends.get(side, p);
            }
        }
#pragma unroll
        for (int j = 0; j < N; ++j) f(j, __builtin_bit_cast(typename Elem<T>::x8, x[j]));
    }
};

template <class T, int BITS, int DP, int NR, int NW, Form FORM>
__global__ __launch_bounds__(NW * 64, 2) void k_step_packed(StepShape s, StepWork w)
{
    constexpr bool WHOLE = FORM != Form::CHUNK, IN_LDS = FORM == Form::WHOLE_IN_LDS;
    constexpr int R = 16 * NR, BOXES = NW / 2, PITCH = BOXES * DP + 4;
    __shared__ __align__(16) float kept[IN_LDS ? WHOLE_SCORES : 4];
    __shared__ __align__(16) float outs[R * PITCH];      // [row][half of the waves][DP]
    __shared__ float2 sums[NW][R];
    __shared__ float l2[R], totals[R];      // of a row: logarithm to base 2 of the whole sum, the sum on the maximum
    const uint32_t group = s.q_heads / s.kv_heads * s.tokens, parts = (group + R - 1) / R;      // rows of queries of a key head
    const uint32_t rows = s.batch * s.kv_heads * parts;
    const uint32_t row = rows >= 256 ? blockIdx.x % rows : blockIdx.x / s.splits;
    const uint32_t split = rows >= 256 ? blockIdx.x / rows : (blockIdx.x + row) % s.splits, part = row % parts;
    const uint32_t kvh = row / parts % s.kv_heads, b = row / parts / s.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int n_rows = min(R, (int)(group - part * R)), first = (int)(kvh * group + part * R);      // of this workgroup, first of all of the sequence
    const int64_t row0 = (int64_t)b * s.q_heads * s.tokens + first;
    const int len = clamp_len(s.lens, b, s.slots), tokens = clamp_len(s.q_lens, b, s.tokens);
    const int c0 = split * s.chunk, c1 = min(c0 + (int)s.chunk, len);

    typename Elem<T>::x8 qf[NR][DP / 32];
    int sees[NR];      // slots below this one
#pragma unroll
    for (int a = 0; a < NR; ++a) {
        const uint32_t of = (uint32_t)(first + min(16 * a + n, n_rows - 1)), head = of / s.tokens, token = of % s.tokens;
        sees[a] = (int)token < tokens ? len - (tokens - 1 - (int)token) : 0;
        const T *q = (const T *)w.q.data + (int64_t)b * w.q.batch + (int64_t)head * w.q.head + (int64_t)token * w.q.row;
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
            const uint32_t e = (DP / 4) * g + 8 * j;
            const typename Elem<T>::x8 z = {};
            qf[a][j] = e < s.head_dim ? *(const typename Elem<T>::x8 *)(q + e) : z;
        }
    }
    const int all_see = tokens == (int)s.tokens ? len - (int)(s.tokens - 1) : 0;      // slots below this one: every row
    const Loader<BITS, DP> from(w.k, w.v, b, kvh, s.head_dim, lane);
    const int32_t *pos = w.positions ? w.positions + ((int64_t)b * s.kv_heads + kvh) * s.slots : nullptr;
    const uint32_t pitch = IN_LDS ? score_pitch(s.slots) : 0;
    const float c = s.scale * LOG2E;
    constexpr float TIMES = IS_F16<T> ? 12.f : 0.f;      // p as a multiple of 2^-TIMES

    f32x4 acc[NR][DP / 16] = {};
    float m[NR], l[NR];
#pragma unroll
    for (int a = 0; a < NR; ++a) m[a] = LOWEST * c, l[a] = 0.f;
    Words<BITS, DP> words;
    int at = c0 + wave * TS;
    int held = 0;
    const auto places = [&](int at) { return pos ? pos[min(at + (lane & 31), len - 1)] : 0; };
    if (at < c1) held = places(at), from.keys(words, at, len - 1), from.values(words, at, len - 1);
    for (; at < c1; at += NW * TS) {
        const bool more = at + NW * TS < c1;
        f32x4 x[NR][2] = {};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const Pair<T, BITS> ends(words.k_ends[h]);
#pragma unroll
            for (int j = 0; j < DP / 32; ++j) {
                const auto k = eight_of<T, BITS>(words.k[h] + j * (BITS / 4), ends);
#pragma unroll
                for (int a = 0; a < NR; ++a) x[a][h] = Small<T>::mfma(k, qf[a][j], x[a][h]);
            }
        }
        const uint32_t live = (uint32_t)__ballot(held >= 0);      // one bit for each slot of the tile
        if (more) held = places(at + NW * TS), from.keys(words, at + NW * TS, len - 1);
        float p[NR][8];
#pragma unroll
        for (int a = 0; a < NR; ++a)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[a][i] = x[a][i / 4][i % 4] * c;
        if (live != ~0u || at + TS > all_see) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int slot = 4 * g + from.slot(i);
                const bool used = (live >> slot) & 1;
#pragma unroll
                for (int a = 0; a < NR; ++a) p[a][i] = used && at + slot < sees[a] ? p[a][i] : -ATTN_INF;
                // what an empty slot holds may be anything, and past the length stand copies of the last slot: zero times
                // what is not a number is not zero
                words.v_ends[i] = used && at + slot < len ? words.v_ends[i] : 0;
            }
            // a slot that only some of the rows see, with a value that is not a number: left out of the product, and added to those rows
            for (int slot = max(len - (tokens - 1) - at, 0); slot < min(TS, len - at); ++slot) {
                if (!((live >> slot) & 1)) continue;
                const uint32_t groups = pack_groups(s.head_dim);
                const char *ends = from.v + (int64_t)(at + slot) * w.v.row + pack_ends(s.head_dim, BITS);
                const uint32_t mine = *(const uint32_t *)(ends + 4 * min((uint32_t)(DP == 128 ? g : g >> 1), groups - 1));      // of this lane's outputs
                const float lo = IS_F16<T> ? (float)__builtin_bit_cast(f16x2, mine)[0] : __uint_as_float(mine << 16);
#pragma unroll
                for (int a = 0; a < NR; ++a)
                    if (lo != lo && at + slot < sees[a])
#pragma unroll
                        for (int j = 0; j < DP / 16; ++j) acc[a][j] = f32x4{lo, lo, lo, lo};
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint32_t e = words.v_ends[i];
                    const float y = IS_F16<T> ? (float)__builtin_bit_cast(f16x2, e)[0] : __uint_as_float(e << 16);
                    if (4 * g + from.slot(i) == slot && y != y) words.v_ends[i] = 0;
                }
            }
        }
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            if (w.weights && 16 * a + n < n_rows) {
                float *const to = IN_LDS ? kept + (16 * a + n) * pitch : w.scores + (row0 + 16 * a + n) * (int64_t)s.score_row;
                *(f32x4 *)(to + at + 4 * g) = f32x4{p[a][0], p[a][1], p[a][2], p[a][3]};
                *(f32x4 *)(to + at + 16 + 4 * g) = f32x4{p[a][4], p[a][5], p[a][6], p[a][7]};
            }
            float top = p[a][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, p[a][i]);
            top = column_max(top);
            if (__ballot(top > m[a])) {
                const float up = fmaxf(m[a], top), by = exp2_fast(m[a] - up);
                m[a] = up;
                l[a] *= by;
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) acc[a][j] *= by;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[a][i] = exp2_fast(p[a][i] - (m[a] - TIMES));
                l[a] += p[a][i];
            }
        }
        typename Elem<T>::x8 pf[NR];
#pragma unroll
        for (int a = 0; a < NR; ++a) pf[a] = round8<T>(p[a], 0);
        Columns<T, BITS, DP>::for_all(words, lane, [&](int j, typename Elem<T>::x8 v) {
#pragma unroll
            for (int a = 0; a < NR; ++a) acc[a][j] = Small<T>::mfma(v, pf[a], acc[a][j]);
        });
        if (more) from.values(words, at + NW * TS, len - 1);
    }

    // join the waves: their sums, then their outputs, each on the workgroup's maximum
    constexpr float ONE = IS_F16<T> ? 0x1p-12f : 1.f;
#pragma unroll
    for (int a = 0; a < NR; ++a) {
        l[a] = column_sum(l[a]) * ONE;
        if (g == 0) sums[wave][16 * a + n] = make_float2(m[a], l[a]);
    }
    __syncthreads();
    float y[NR][DP / 4];      // this wave's outputs in order, elements (DP / 4) g ..
#pragma unroll
    for (int a = 0; a < NR; ++a) {
        const int r = 16 * a + n;
        float top = sums[0][r].x;
        for (int i = 1; i < NW; ++i) top = fmaxf(top, sums[i][r].x);
        const float by = exp2_fast(m[a] - top) * ONE;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[a][Columns<T, BITS, DP>::at(i, j)] = sees[a] > 0 ? acc[a][j][i] * by : 0.f;
        if (wave == 0 && g == 0 && r < n_rows) {
            float total = 0.f;
            for (int i = 0; i < NW; ++i) total += sums[i][r].y * exp2_fast(sums[i][r].x - top);
            const bool some = total != 0.f;
            if constexpr (WHOLE) {
                w.lse[row0 + r] = some ? top * LN2 + __logf(total) : -ATTN_INF;
                l2[r] = some ? top + __log2f(total) : ATTN_INF;
                totals[r] = total;
            } else {
                w.sums[(row0 + r) * s.splits + split] = make_float2(top, total);
            }
        }
    }
    // half of the waves hand theirs to the other half
    for (int turn = 0; turn < 2; ++turn) {
        if ((wave < BOXES) == (turn == 1))
#pragma unroll
            for (int a = 0; a < NR; ++a)
                if (16 * a + n < n_rows)
#pragma unroll
                    for (int e = 0; e < DP / 4; e += 4) {
                        f32x4 *box = (f32x4 *)(outs + (16 * a + n) * PITCH + wave % BOXES * DP + (DP / 4) * g + e);
                        const f32x4 z = {y[a][e], y[a][e + 1], y[a][e + 2], y[a][e + 3]};
                        *box = turn ? *box + z : z;
                    }
        __syncthreads();
    }
    for (int i = threadIdx.x; i < n_rows * (DP / 4); i += NW * 64) {
        const int r = i / (DP / 4), e = i % (DP / 4) * 4;
        f32x4 z = *(f32x4 *)(outs + r * PITCH + e);
        for (int box = 1; box < BOXES; ++box) z += *(f32x4 *)(outs + r * PITCH + box * DP + e);
        if constexpr (WHOLE) {
            typename Elem<T>::x4 o;
            for (int j = 0; j < 4; ++j) o[j] = (T)(totals[r] != 0.f ? z[j] / totals[r] : 0.f);
            const uint32_t of = (uint32_t)(first + r);
            if (e < (int)s.head_dim)
                *(typename Elem<T>::x4 *)((T *)w.out.data + (int64_t)b * w.out.batch + (int64_t)(of / s.tokens) * w.out.head + (int64_t)(of % s.tokens) * w.out.row + e) = o;
        } else {
            *(f32x4 *)(w.outs + ((row0 + r) * s.splits + split) * DP + e) = z;
        }
    }
    if constexpr (WHOLE) {
        if (!w.weights) return;
        const float *const all = w.scores + row0 * (int64_t)s.score_row;
        const int64_t to = ((int64_t)b * s.kv_heads + kvh) * s.slots;
        const bool aligned = s.slots % 4 == 0 && ((uintptr_t)w.weights | (uintptr_t)w.before) % 16 == 0;
        for (uint32_t slot = threadIdx.x * 4; slot < s.slots; slot += NW * 64 * 4) {
            f32x4 sum = {};
            if ((int)slot < len) {
#pragma unroll 4
                for (int r = 0; r < n_rows; ++r) {
                    const f32x4 x = *(const f32x4 *)(IN_LDS ? kept + r * pitch + slot : all + (int64_t)r * s.score_row + slot);
                    for (int j = 0; j < 4; ++j) sum[j] += exp2_fast(x[j] - l2[r]);
                }
                for (int j = 1; j < 4; ++j) sum[j] = (int)slot + j < len ? sum[j] : 0.f;
            }
            if (aligned) {
                *(f32x4 *)(w.weights + to + slot) = *(const f32x4 *)(w.before + to + slot) + sum;
            } else {
                for (int j = 0; j < 4; ++j)
                    if (slot + j < s.slots) w.weights[to + slot + j] = w.before[to + slot + j] + sum[j];
            }
        }
    }
}

template <class T, int BITS, int DP, int NR> hipError_t launch(const StepShape &s, const StepWork &w, hipStream_t st)
{
    const uint32_t rows = s.batch * s.kv_heads;
    if (s.whole) {
        if (s.score_row) k_step_packed<T, BITS, DP, NR, WHOLE_WAVES, Form::WHOLE><<<rows, WHOLE_WAVES * 64, 0, st>>>(s, w);
        else k_step_packed<T, BITS, DP, NR, WHOLE_WAVES, Form::WHOLE_IN_LDS><<<rows, WHOLE_WAVES * 64, 0, st>>>(s, w);
        return hipGetLastError();
    }
    const uint32_t group = s.q_heads / s.kv_heads * s.tokens, parts = (group + 16 * NR - 1) / (16 * NR);
    k_step_packed<T, BITS, DP, NR, CHUNK_WAVES, Form::CHUNK><<<s.splits * parts * rows, CHUNK_WAVES * 64, 0, st>>>(s, w);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_step_join(s, w, st) : e;
}
template <class T, int BITS, int DP> hipError_t launch(const StepShape &s, const StepWork &w, hipStream_t st)
{
    return s.q_heads / s.kv_heads * s.tokens <= 16 ? launch<T, BITS, DP, 1>(s, w, st) : launch<T, BITS, DP, 2>(s, w, st);
}
template <class T> hipError_t launch(const StepShape &s, const StepWork &w, uint32_t bits, hipStream_t st)
{
    if (bits == 4) return s.head_dim <= 64 ? launch<T, 4, 64>(s, w, st) : launch<T, 4, 128>(s, w, st);
    return s.head_dim <= 64 ? launch<T, 8, 64>(s, w, st) : launch<T, 8, 128>(s, w, st);
}

}  // namespace

static bool whole_caches(uint64_t rows, uint32_t slots)
{
    const uint64_t rounds = (rows + 255) / 256;
    return slots <= 1024 || (slots <= 2048 && rows >= 128) || (slots <= 4096 && rows >= 192 * rounds);
}

void packed_step_split(StepShape &s)
{
    const uint32_t group = s.q_heads / s.kv_heads * s.tokens, of_part = group <= 16 ? 16 : 32;
    const uint64_t rows = (uint64_t)s.batch * s.kv_heads * ((group + of_part - 1) / of_part);
    const uint64_t least = CHUNK_WAVES * TS, most = 2048;
    const uint64_t want = (uint64_t)s.slots * rows / 2048;
    const uint64_t chunk = (want < least ? least : want > most ? most : want) / least * least;
    s.chunk = (uint32_t)chunk;
    s.splits = (uint32_t)((s.slots + chunk - 1) / chunk);
    if (!s.splits) s.splits = 1;
    s.score_row = ((uint64_t)s.slots + TS - 1) / TS * TS;
    s.whole = group <= 32 && whole_caches(rows, s.slots);
    if (!s.whole) return;
    s.chunk = s.slots, s.splits = 1;
    if ((uint64_t)group * score_pitch(s.slots) <= WHOLE_SCORES) s.score_row = 0;
}

hipError_t launch_attention_step_packed(const StepShape &s, const StepWork &w, uint32_t bits, hipStream_t st)
{
    return s.half ? launch<_Float16>(s, w, bits, st) : launch<__bf16>(s, w, bits, st);
}

}  // namespace lap
