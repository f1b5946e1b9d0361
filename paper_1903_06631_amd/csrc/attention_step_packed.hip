// Attention of one or a few new tokens of every sequence over a cache in 4 or 8 bits an element, and the weight that every slot
// receives from them:
//   o_i = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j - lse_i), over the slots in use that row i sees; w_j += sum_i p_ij
// with k and v the numbers that the packed rows stand for, rounded to the element type as in cache_unpack.
//
// p is rounded to the values' type for its product with them (a matrix operand), in binary16 as a multiple of 2^-10, so that
// those below 2^-24 of the largest of their wave lose precision and none vanishes above 2^-35.  Sums, scores and weights are
// 32 bits.
//
// Every packed row is read once for each 16 rows of queries that share a key head, heads times tokens, or for each 32 where there are
// more than 16.  These rows are the columns, 16 each, of the 16x16x32 matrix instruction (C = A B, lane l with g = l / 16):
//   A: row l % 16, contraction indices 8 g .. 8 g + 7      B: column l % 16, the same      C: column l % 16, rows 4 g .. 4 g + 3
// Keys are A of the scores: a lane holds a fourth of a slot's row, which is one group of 32 elements where rows have 128, so it
// needs one lo and one step.  Values are A of the outputs, elements along the rows: a lane holds one word of eight slots,
// whose low and high halves, side by side for two slots, are the operand's pairs (packed_rows.h).  So both go from memory
// straight into registers and from there into the products, without LDS; the contraction over slots runs in the order in which
// the scores stand in C.  Waves go through 32 slots at a time of their own, without waiting for each other, and ask for the
// next keys when these ones are decoded, for the next values likewise (with two tiles on their way, and a fourth of the waves less,
// 64 caches of 8 heads x up to 4096 slots took 55 us in place of 50, 24 of 4 x up to 6001 of 8 bits 37 in place of 27).
//
// Bound by memory where caches are long, and not by much: a tile of 32 slots of 128 elements is 10 KB and some 400 vector
// instructions in bfloat16 (280 in binary16), four cycles each, of which a third would do for rows of 16 bits.  So every
// instruction of a tile counts: levels are converted two by two, loads need no addresses of their own, the running maximum is
// left behind by up to 2^5 before sums are taken down to a new one, and lanes compare with it on their own.  Short caches are bound by a
// launch or two and the chain of a tile, some 1.3 us.
//
// Long caches are cut into chunks, a workgroup of four waves each; what these leave is joined by a second kernel, which adds the
// weights as well (packed_join.hip).  Short ones have a workgroup of eight waves each, which does all of it.
//
// Measured, kernels alone, 4 bits and 128 elements where nothing else is said: 16 x 1000 slots of one sequence 12.4 us (a launch
// and a chain of four tiles); 64 ragged sequences of 8 heads x up to 4096 slots, 4 query heads each and weights, 45 us (188 MB of rows
// and results at 4.2 TB/s, vector instructions in 51 % of all cycles, the matrix units busy 7 %); 2 x 8 x 131 072 slots likewise 76 us and 12 to
// join (4.9 TB/s, 39 %, 9 %); 24 ragged x 4 x up to 6001 slots of 96 in 8 bits, 8 query heads each, 19 us and 4.4; 16 ragged x 8 x up
// to 8192 slots, five tokens of 4 query heads, 30 us and 5.3; 32 x 2047 slots of 64, 32 query heads, 10 us and 6.0.
//
// More than 32 rows to a key head are parts of 32, workgroups of their own, of which each reads the cache from memory: the 64
// sequences, without weights, 50 us with 16 rows and 173 MB read, 66 and 175 with 32, 111 and 351 with 40, 120 and 358 with 64, 454 and 1429 with 256.
// The floor, the rows read once, is 35 us.
#include "lap_dev.h"
#include "packed_rows.h"

namespace lap {
namespace {

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

__device__ __forceinline__ __amdgpu_buffer_rsrc_t bytes_at(const void *from, int size)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(from), 0, size, 0x00020000);
}

// The packed words of 32 slots that a lane holds, and where they stand in a row.  Lanes whose share of a row is past its last
// group hold the last group's: queries are zero there, and outputs thrown away.
template <int BITS, int DP> struct Words {
    static constexpr int KW = DP * BITS / 128;                       // words of a key's fourth
    static constexpr int VW = DP * BITS >= 512 ? DP * BITS / 512 : 1;      // of a value's sixteenth (of 32 bytes: half a word)
    uint32_t k[2][KW], k_ends[2], v[8][VW], v_ends[8];
};

// Buffer loads: a lane's place within a tile does not change, the tile's start is in the scalar descriptor and so is its end, past
// which such a load reads nothing and gives zeros.  (Ordinary loads took two 64-bit additions each, and with rows past the length
// to be told from others their addresses took 32 registers.)
template <int BITS, int DP> struct Loader {
    typedef Words<BITS, DP> W;
    const char *k, *v;                     // of the cache
    int64_t k_row, v_row;
    uint32_t row_bytes;
    int k_at, k_ends, v_at, v_ends;        // bytes from the start of a tile
    __device__ __forceinline__ Loader(const Rows &rk, const Rows &rv, uint32_t b, uint32_t kvh, uint32_t head_dim, int lane)
    {
        const int n = lane & 15, g = lane >> 4;
        k = (const char *)rk.data + (int64_t)b * rk.batch + (int64_t)kvh * rk.head;
        v = (const char *)rv.data + (int64_t)b * rv.batch + (int64_t)kvh * rv.head;
        k_row = rk.row, v_row = rv.row;
        row_bytes = pack_row_bytes(head_dim, BITS);
        const uint32_t groups = pack_groups(head_dim), ends = pack_ends(head_dim, BITS);
        const uint32_t kg = min((uint32_t)(DP == 128 ? g : g >> 1), groups - 1), vg = min((uint32_t)(DP == 128 ? n >> 2 : n >> 3), groups - 1);
        const uint32_t k_slot = n * (uint32_t)k_row, v_slot = 4 * g * (uint32_t)v_row;
        k_at = k_slot + kg * (BITS * 4) + (DP == 128 ? 0 : (g & 1) * (BITS * 2));
        v_at = v_slot + vg * (BITS * 4) + (DP == 128 ? (n & 3) * BITS : BITS == 8 ? (n & 7) * 4 : (n >> 1 & 3) * 4);
        k_ends = k_slot + ends + kg * 4, v_ends = v_slot + ends + vg * 4;
    }
    static __device__ __forceinline__ constexpr int slot(int i) { return i < 4 ? i : 12 + i; }      // of a lane's i-th value, less 4 g
    // Rows at .. last, 32 at most, which are less than 2^30 bytes; none if there are none, however far `at` is behind.  (A load's
    // scalar offset is taken off the range before it is checked, so there is none: rows further on have a descriptor of their own.)
    struct Tile32 {
        const char *base;
        int row, size;
        __device__ __forceinline__ Tile32(const char *from, int64_t row_, int at, int last, uint32_t row_bytes) : base(from + (int64_t)at * row_), row((int)row_)
        {
            const int n = last - at;
            size = (int)(((uint32_t)min(TS - 1, n) * (uint32_t)row + row_bytes) & ~(uint32_t)(n >> 31));
        }
        __device__ __forceinline__ __amdgpu_buffer_rsrc_t from(int i) const { return bytes_at(base + i * row, max(size - i * row, 0)); }
    };
    template <int N> static __device__ __forceinline__ void words(uint32_t (&w)[N], __amdgpu_buffer_rsrc_t from, int off)
    {
        if constexpr (N % 4 == 0) {
#pragma unroll
            for (int i = 0; i < N; i += 4) {
                const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(from, off + 4 * i, 0, 0);
#pragma unroll
                for (int j = 0; j < 4; ++j) w[i + j] = x[j];
            }
        } else if constexpr (N == 2) {
            const u32x2 x = __builtin_amdgcn_raw_buffer_load_b64(from, off, 0, 0);
            w[0] = x[0], w[1] = x[1];
        } else {
            w[0] = __builtin_amdgcn_raw_buffer_load_b32(from, off, 0, 0);
        }
    }
    // keys of slots at .. at + 31, as far as `last`
    __device__ __forceinline__ void keys(W &w, int at, int last) const
    {
        const Tile32 tile(k, k_row, at, last, row_bytes);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const auto from = tile.from(16 * h);
            words(w.k[h], from, k_at);
            w.k_ends[h] = __builtin_amdgcn_raw_buffer_load_b32(from, k_ends, 0, 0);
        }
    }
    __device__ __forceinline__ void values(W &w, int at, int last) const
    {
        const Tile32 tile(v, v_row, at, last, row_bytes);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const auto from = tile.from(slot(i));
            words(w.v[i], from, v_at);
            w.v_ends[i] = __builtin_amdgcn_raw_buffer_load_b32(from, v_ends, 0, 0);
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
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
            u32x4 x[PER];
#pragma unroll
            for (int s = 0; s < 4; ++s) {                       // two slots at a time
                const Pair<T, BITS> ends(w.v_ends[2 * s], w.v_ends[2 * s + 1]);
                const Levels<BITS> side = side_by_side<BITS>(w.v[2 * s][h / 2], w.v[2 * s + 1][h / 2], HALVES == 1 ? lane & 1 : h % 2);
                x[0][s] = ends.template get<0>(side), x[1][s] = ends.template get<1>(side);
                if constexpr (PER == 4) x[2][s] = ends.template get<2>(side), x[3][s] = ends.template get<3>(side);
            }
#pragma unroll
            for (int j = 0; j < PER; ++j) f(h * PER + j, __builtin_bit_cast(typename Elem<T>::x8, x[j]));
            __builtin_amdgcn_sched_barrier(0);
        }
    }
};

// inclusive prefix sum over the wave
__device__ __forceinline__ uint32_t wave_sums(uint32_t v)
{
    v += dpp_mov<0x111>(0u, v);
    v += dpp_mov<0x112>(0u, v);
    v += dpp_mov<0x114>(0u, v);
    v += dpp_mov<0x118>(0u, v);
    v += dpp_mov<0x142, 0xA>(0u, v);
    v += dpp_mov<0x143, 0xC>(0u, v);
    return v;
}

// Which slots of which sequence are a workgroup's.  Without lengths, chunks of s.chunk slots, s.splits for each sequence.  Lengths
// are known on the GPU only, so it is there that all sequences are cut into chunks of one size, a number of tiles for each wave:
// the least that makes no more than s.splits of them (for each key head), so that workgroups fill the card's places evenly,
// whatever the lengths are; or, of more sequences than a wave has lanes and where no size below it does, the least that surely makes no
// more than s.shares, as chunks of all tiles plus one for each sequence are.  (16 ragged sequences of 8 heads x up to 8192 slots,
// five tokens: 35.0 us, with the sure size alone 36.9.)
struct Share {
    uint32_t b;
    int len, first, slots;
    bool any;
};
__device__ __forceinline__ Share share_of(const StepShape &s, uint32_t turn, uint2 *table, int lane)
{
    Share r = {};
    if (!s.lens) {
        const uint32_t n = s.splits;
        r.any = true;
        r.b = turn / n, r.len = (int)s.slots;
        r.first = (int)((turn - r.b * n) * s.chunk), r.slots = (int)s.chunk;
        return r;
    }
    const auto length = [&](uint32_t b) { return b < s.batch ? (uint32_t)clamp_len(s.lens, b, s.slots) : 0; };
    uint32_t own = length(lane), all = read_lane(wave_sums((own + TS - 1) / TS), 63);
    for (uint32_t b = 64; b < s.batch; b += 64) all += read_lane(wave_sums((length(b + lane) + TS - 1) / TS), 63);
    const auto at_least = [&](uint32_t chunks) { return uniform(max(1u, (all + chunks * CHUNK_WAVES - 1) / (chunks * CHUNK_WAVES))); };
    const uint32_t surely = at_least(s.shares - s.batch);
    uint32_t for_wave = surely;      // tiles
    if (s.batch <= 64)
        for (for_wave = at_least(s.splits); for_wave < surely; ++for_wave)
            if (read_lane(wave_sums(((own + TS - 1) / TS + for_wave * CHUNK_WAVES - 1) / (for_wave * CHUNK_WAVES)), 63) <= s.splits) break;
    const uint32_t each = for_wave * CHUNK_WAVES;
    uint32_t before = 0;
    for (uint32_t b0 = 0; b0 < s.batch; b0 += 64) {
        if (b0) own = length(b0 + lane);
        const uint32_t n = ((own + TS - 1) / TS + each - 1) / each, up = before + wave_sums(n);
        if (table && b0 + lane < s.batch) table[b0 + lane] = make_uint2(up - n, n);
        const int at = __popcll(ballot(up <= turn));      // sequences whose chunks all come before
        if (!r.any && at < 64) {
            r.any = true;
            r.b = b0 + at;
            r.len = (int)read_lane(own, at);
            r.first = uniform((int)((turn - (read_lane(up, at) - read_lane(n, at))) * each * TS));
            r.slots = (int)(each * TS);
            if (!table) break;
        }
        before = read_lane(up, 63);
    }
    return r;
}

template <class T, int BITS, int DP, int NR, int NW, Form FORM>
__global__ __launch_bounds__(NW * 64, NR == 2 ? 3 : 4) void k_step_packed(StepShape s, StepWork w)
{
    constexpr bool WHOLE = FORM != Form::CHUNK, IN_LDS = FORM == Form::WHOLE_IN_LDS;
    constexpr int R = 16 * NR, BOXES = NW / 2, PITCH = BOXES * DP + 4;
    __shared__ __align__(16) float kept[IN_LDS ? WHOLE_SCORES : 4];
    __shared__ __align__(16) float outs[R * PITCH];      // [row][half of the waves][DP]
    __shared__ typename Elem<T>::x8 queries[NR][DP / 32][64];
    __shared__ float2 sums[NW][R];
    __shared__ float2 whole[R];      // of a row: its largest product and the logarithm to base 2 of its sum on that
    __shared__ float totals[R];      // that sum
    const uint32_t group = s.group, parts = (group + R - 1) / R;      // rows of queries of a key head
    const uint32_t turn = WHOLE ? blockIdx.y : blockIdx.x, kvh = WHOLE ? blockIdx.x : blockIdx.y, part = blockIdx.z;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 15, g = lane >> 4;
    const int n_rows = min(R, (int)(group - part * R)), first = (int)(kvh * group + part * R);      // of this workgroup, first of all of the sequence
    uint32_t b = turn;
    int len, c0 = 0, c1;
    if constexpr (WHOLE) {
        c1 = len = clamp_len(s.lens, b, s.slots);
    } else {
        const Share mine = share_of(s, turn, turn + kvh + part + wave == 0 ? w.table : nullptr, lane);
        if (!mine.any) return;
        b = mine.b, len = mine.len, c0 = mine.first, c1 = min(c0 + mine.slots, len);
    }
    const int tokens = clamp_len(s.q_lens, b, s.tokens);
    const int64_t row0 = (int64_t)b * s.q_heads * s.tokens + first;      // of lse
    const int64_t partial = ((int64_t)(kvh * parts + part) * s.shares + turn) * R;      // of outs and sums: [key head][part][share][row]

    const int all_see = tokens == (int)s.tokens ? len - (int)(s.tokens - 1) : 0;      // slots below this one: every row
    // Queries as operands, a wave's share of them for all waves: in registers they would cost a fifth of the waves that fit.
    static_assert(NW >= DP / 32, "an operand for each wave at most");
    typename Elem<T>::x8 mine[NR];
    int sees[NR];      // slots below this one
#pragma unroll
    for (int a = 0; a < NR; ++a) {
        const uint32_t of = (uint32_t)(first + min(16 * a + n, n_rows - 1)), head = s.tokens == 1 ? of : of / s.tokens, token = of - head * s.tokens;
        sees[a] = (int)token < tokens ? len - (tokens - 1 - (int)token) : 0;
        const uint32_t e = (DP / 4) * g + 8 * wave;
        mine[a] = typename Elem<T>::x8{};
        if (wave < DP / 32 && e < s.head_dim)
            mine[a] = *(const typename Elem<T>::x8 *)((const T *)w.q.data + (int64_t)b * w.q.batch + (int64_t)head * w.q.head + (int64_t)token * w.q.row + e);
    }
    const Loader<BITS, DP> from(w.k, w.v, b, kvh, s.head_dim, lane);
    const int32_t *pos = w.positions ? w.positions + ((int64_t)b * s.kv_heads + kvh) * s.slots : nullptr;
    // Every pass asks for the same loads and stores, of nothing where there is nothing: what is in flight is then known when
    // the code is compiled, and a wait for the keys is none for the values that were asked for after them.
    const auto places = [&](int at) {
        return (int)__builtin_amdgcn_raw_buffer_load_b32(bytes_at(pos + at, uniform(pos ? max(0, min(TS, c1 - at)) * 4 : 0)), (lane & 31) * 4, 0, 0);
    };
    Words<BITS, DP> words;
    int place;
    int at = c0 + wave * TS;
    place = places(at), from.keys(words, at, c1 - 1);
    __builtin_amdgcn_sched_barrier(0);      // in the order in which the loop asks for them
    from.values(words, at, c1 - 1);
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int a = 0; a < NR; ++a)
        if (wave < DP / 32) {
            typename Elem<T>::x8 y;
#pragma unroll
            for (int i = 0; i < 8; ++i) y[i] = mine[a][held<BITS>(i)];
            queries[a][wave][lane] = y;
        }
    __syncthreads();
    // of the chunk's tiles: [tile][row of the key head][slot]
    float *const scores = w.scores + (int64_t)(b * s.kv_heads + kvh) * s.score_row * group + (int64_t)part * R * TS;
    const uint32_t pitch = IN_LDS ? score_pitch(s.slots) : 0;
    const float c = s.scale * LOG2E;
    constexpr float TIMES = IS_F16<T> ? 10.f : 0.f;      // p as a multiple of 2^-TIMES
    const float slack = 5.f / c;                         // by how much the running maximum may be left behind: 2^5
    // Maxima are those of the products, and differences are taken before the scale comes in: a scaled score may be so large that
    // 32 bits hold it to whole powers of two only, and its own maximum's exponent has to be 0 all the same.  (With scaled
    // maxima inside the multiplication, a subtraction less for each score, the 16 sequences with five tokens took 32.9 us in
    // place of 33.3, the two long ones the same.)

    f32x4 acc[NR][DP / 16] = {};
    float m[NR], l[NR];
#pragma unroll
    for (int a = 0; a < NR; ++a) m[a] = LOWEST, l[a] = 0.f;
    for (; at < c1; at += NW * TS) {
        const int next = at + NW * TS;
        asm volatile("" ::: "memory");      // the queries are not to be kept in registers
        f32x4 x[NR][2] = {};
        const Pair<T, BITS> ends[2] = {Pair<T, BITS>(words.k_ends[0]), Pair<T, BITS>(words.k_ends[1])};
#pragma unroll
        for (int j = 0; j < DP / 32; ++j) {
            typename Elem<T>::x8 q[NR];
#pragma unroll
            for (int a = 0; a < NR; ++a) q[a] = queries[a][j][lane];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const auto k = __builtin_bit_cast(typename Elem<T>::x8, eight_as_held<T, BITS>(words.k[h] + j * (BITS / 4), ends[h]));
#pragma unroll
                for (int a = 0; a < NR; ++a) x[a][h] = Small<T>::mfma(k, q[a], x[a][h]);
            }
        }
        const uint32_t live = (uint32_t)__ballot(place >= 0);      // one bit for each slot of the tile
        place = places(next), from.keys(words, next, c1 - 1);
        float p[NR][8];
#pragma unroll
        for (int a = 0; a < NR; ++a)
#pragma unroll
            for (int i = 0; i < 8; ++i) p[a][i] = x[a][i / 4][i % 4];
        if (live != ~0u || at + TS > all_see) {
            int g4 = 4 * g;
            asm volatile("" : "+v"(g4));      // or what comes of it is kept in registers throughout the loop
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int slot = g4 + from.slot(i);
                const bool used = (live >> slot) & 1;
#pragma unroll
                for (int a = 0; a < NR; ++a) p[a][i] = used && at + slot < sees[a] ? p[a][i] : -ATTN_INF;
                // what an empty slot holds may be anything, and past the length may stand the last slot again (rows of stride
                // zero): zero times what is not a number is not zero
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
                    if (g4 + from.slot(i) == slot && y != y) words.v_ends[i] = 0;
                }
            }
        }
#pragma unroll
        for (int a = 0; a < NR; ++a) {
            const int r = 16 * a + n;
            if constexpr (IN_LDS) {
                if (w.weights && r < n_rows) {
                    *(f32x4 *)(kept + r * pitch + at + 4 * g) = f32x4{p[a][0], p[a][1], p[a][2], p[a][3]};
                    *(f32x4 *)(kept + r * pitch + at + 16 + 4 * g) = f32x4{p[a][4], p[a][5], p[a][6], p[a][7]};
                }
            } else {
                const auto to = bytes_at(scores + (int64_t)at * group, w.weights ? n_rows * TS * 4 : 0);
#pragma unroll
                for (int h = 0; h < 2; ++h)
                    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4, f32x4{p[a][4 * h], p[a][4 * h + 1], p[a][4 * h + 2], p[a][4 * h + 3]}), to,
                                                           r * (TS * 4) + 64 * h + 16 * g, 0, 0);
            }
            float top = p[a][0];
#pragma unroll
            for (int i = 1; i < 8; ++i) top = fmaxf(top, p[a][i]);
            if (__ballot(top - m[a] > slack)) {
                const float up = fmaxf(m[a], column_max(top)), by = exp2_fast((m[a] - up) * c);
                m[a] = up;
                l[a] *= by;
#pragma unroll
                for (int j = 0; j < DP / 16; ++j) acc[a][j] *= by;
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                p[a][i] = exp2_fast(__builtin_fmaf(p[a][i] - m[a], c, TIMES));
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
        from.values(words, next, c1 - 1);
    }

    // join the waves: their sums, then their outputs, each on the workgroup's maximum
    constexpr float ONE = IS_F16<T> ? 0x1p-10f : 1.f;
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
        const float by = exp2_fast((m[a] - top) * c) * ONE;
#pragma unroll
        for (int j = 0; j < DP / 16; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) y[a][Columns<T, BITS, DP>::at(i, j)] = sees[a] > 0 ? acc[a][j][i] * by : 0.f;
        if (wave == 0 && g == 0 && r < n_rows) {
            float total = 0.f;
            for (int i = 0; i < NW; ++i) total += sums[i][r].y * exp2_fast((sums[i][r].x - top) * c);
            const bool some = total != 0.f;
            if constexpr (WHOLE) {
                w.lse[row0 + r] = some ? top * s.scale + __logf(total) : -ATTN_INF;
                whole[r] = some ? make_float2(top, __log2f(total)) : make_float2(ATTN_INF, 0.f);
                totals[r] = total;
            } else {
                w.sums[partial + r] = make_float2(top, total);
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
            *(f32x4 *)(w.outs + (partial + r) * DP + e) = z;
        }
    }
    if constexpr (WHOLE) {
        if (!w.weights) return;
        const int64_t to = ((int64_t)b * s.kv_heads + kvh) * s.slots;
        const bool aligned = s.slots % 4 == 0 && ((uintptr_t)w.weights | (uintptr_t)w.before) % 16 == 0;
        for (uint32_t slot = threadIdx.x * 4; slot < s.slots; slot += NW * 64 * 4) {
            f32x4 sum = {};
            if ((int)slot < len) {
#pragma unroll 4
                for (int r = 0; r < n_rows; ++r) {
                    const f32x4 x = *(const f32x4 *)(IN_LDS ? kept + r * pitch + slot : scores + (int64_t)(slot / TS) * (TS * n_rows) + r * TS + slot % TS);
                    for (int j = 0; j < 4; ++j) sum[j] += received(x[j], whole[r], c);
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
    if (s.whole) {
        const dim3 grid(s.kv_heads, s.batch);      // the heads of a sequence to all dies (the other way 64 us in place of 50)
        if (s.score_row) k_step_packed<T, BITS, DP, NR, WHOLE_WAVES, Form::WHOLE><<<grid, WHOLE_WAVES * 64, 0, st>>>(s, w);
        else k_step_packed<T, BITS, DP, NR, WHOLE_WAVES, Form::WHOLE_IN_LDS><<<grid, WHOLE_WAVES * 64, 0, st>>>(s, w);
        return hipGetLastError();
    }
    k_step_packed<T, BITS, DP, NR, CHUNK_WAVES, Form::CHUNK><<<dim3(s.shares, s.kv_heads, step_parts(s.group)), CHUNK_WAVES * 64, 0, st>>>(s, w);
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? launch_packed_join(s, w, st) : e;
}
template <class T, int BITS, int DP> hipError_t launch(const StepShape &s, const StepWork &w, hipStream_t st)
{
    return s.group <= 16 ? launch<T, BITS, DP, 1>(s, w, st) : launch<T, BITS, DP, 2>(s, w, st);
}
template <class T> hipError_t launch(const StepShape &s, const StepWork &w, uint32_t bits, hipStream_t st)
{
    if (bits == 4) return s.head_dim <= 64 ? launch<T, 4, 64>(s, w, st) : launch<T, 4, 128>(s, w, st);
    return s.head_dim <= 64 ? launch<T, 8, 64>(s, w, st) : launch<T, 8, 128>(s, w, st);
}

}  // namespace

// Whether one workgroup goes through all of a cache.  It needs no second launch, 3 us of the card's and 5 of the call, but has a
// compute unit's waves for itself only where there are as many caches.  So: for short ones; for those of 1024 to 1536 slots, where
// units are not left idle for long; and for up to 8192 slots where the last round of workgroups leaves at most an eighth of
// them idle (up to 2800 with lengths and one round: the longest cache's unit then works alone).  Measured (8 key heads of 128 elements in 4 bits, 4 query heads each; whole, and in the best chunks):
//   caches x slots     whole   chunks          caches x slots     whole   chunks
//        8 x 500         9.1      9.5 us          128 x 4000        36.9     28.4 us
//        8 x 1000       12.7      9.7 *           192 x 4000        37.5     33.2
//        8 x 2000       20        9.8             256 x 4000        42.7     47.6
//       32 x 1000       13.2     11.2 *           320 x 4000        70.4     59.7
//       32 x 2000       20.5     12.5             384 x 4000        63.1     56.5
//      128 x 1000       13.8     15.8             512 x 4000        82       90
//      128 x 2000       21.6     18.9             512 x 8000       169      174
//      192 x 2000       21.9     23.6             768 x 4000       124.5    133
// (* on the card alone: called one after the other 12.1 and 17.)
// Ragged, lengths evenly spread up to these, 256 x 2000 19.5 and 21.0, x 4096 33.6 and 28.7, 240 x 6000 46.6 and 35.5, 512 x 4096 45.8 and 49.0,
// x 8192 84.4 and 82.7.
static bool whole_caches(uint64_t rows, uint32_t slots, bool lens)
{
    const uint64_t rounds = (rows + 255) / 256;
    return slots <= 1024 || (slots <= 1536 && slots <= 8 * rows) || (slots <= (lens && rounds == 1 ? 2800 : 8192) && 8 * rows >= 7 * 256 * rounds);
}

// Into how many chunks caches are cut: as many as the card has places for workgroups of CHUNK_WAVES waves, four or (with 32 rows
// of queries in the registers) three a unit.  Half of the places are better for shorter ones: fewer start and fewer are joined, and up
// to 32 tiles a chunk that is the more; with lengths up to 24, as these make the tiles fewer than there may be and the chunks of all
// less even.  Chunks of over 64 tiles are cut smaller, so that units that are done early go on.  Measured (4 bits, 8 key heads of 128
// elements, 4 query heads each; tiles a chunk with half of the places, that, all of them):
//   without lengths   16 x 3500 slots   27    21.9  22.8 us      ragged    4 x 5000 slots   10    14.7  16.2 us
//                     16 x 4500         35    25.1  26.0                  2 x 20000         20    18.2  20.4
//                     16 x 6500         51    31.8  31.5                  8 x 5000          20    20.6  20.0
//                      1 x 30000        15    17.4  20.5                 16 x 3500          27    22.2  18.6
//                      1 x 131072       64    40.0  42.2                  8 x 8000          31    27.2  25.2
constexpr uint64_t FEW = 512, PLACES = 1024, PLACES_32 = 768;
void packed_step_split(StepShape &s)
{
    s.group = s.q_heads / s.kv_heads * s.tokens;
    const uint64_t heads = (uint64_t)s.kv_heads * step_parts(s.group), rows = s.batch * heads;
    s.score_row = ((uint64_t)s.slots + TS - 1) / TS * TS;
    s.whole = s.group <= 32 && whole_caches(rows, s.slots, s.lens);
    s.chunk = s.splits = s.shares = 0;
    if (!s.whole) {
        const uint64_t tiles = s.score_row / TS, places = s.group <= 16 ? PLACES : PLACES_32;
        // for each key head, of one sequence or of all of them
        const uint64_t sequences = s.lens ? s.batch : 1, all = tiles * sequences, few = FEW / heads / (s.batch / sequences);
        uint64_t n = places / heads / (s.batch / sequences);
        if (all <= few * (s.lens ? 24 : 32)) n = few;
        if (all > n * 64) n = (all + 63) / 64;
        if (!n) n = 1;      // (no slots, and more heads than places)
        if (s.lens) {
            s.splits = (uint32_t)n;
            s.shares = (uint32_t)((n > s.batch ? n - s.batch / 2 : n - n / 2) + s.batch);
        } else {
            const uint64_t each = (tiles + n - 1) / n;
            s.chunk = (uint32_t)((each < CHUNK_WAVES ? CHUNK_WAVES : each) * TS);
            s.splits = s.slots ? (uint32_t)((s.slots + s.chunk - 1) / s.chunk) : 1;      // without slots one that finds none
            s.shares = s.splits * s.batch;
        }
        return;
    }
    if ((uint64_t)s.group * score_pitch(s.slots) <= WHOLE_SCORES) s.score_row = 0;
}

hipError_t launch_attention_step_packed(const StepShape &s, const StepWork &w, uint32_t bits, hipStream_t st)
{
    return s.half ? launch<_Float16>(s, w, bits, st) : launch<__bf16>(s, w, bits, st);
}

}  // namespace lap
