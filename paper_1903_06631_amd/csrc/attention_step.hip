// Attention of one new token of every sequence over its cache, and the weight that every slot receives from it:
//   o = sum_j p_j v_j, p_j = exp(scale q.k_j - lse), over the slots in use; w_j += sum of p_j over the heads that share slot j
//
// p is rounded to the values' type for its product with them (a matrix operand); in binary16, those below 2^-25 of the largest
// of their wave, which has up to 512 slots, vanish: less than 2^-16 of the row.  Sums, scores and weights are 32 bits.
//
// Every key and value is read once and takes part in a few products only: the pass is bound by memory.  Waves go through 32
// slots at a time of their own, without waiting for each other: keys from memory straight into registers as a matrix operand,
// values through LDS, which is where they are transposed.  The heads of a group are the kept rows (up to 32; with fewer,
// part of the matrix instructions runs empty, at a rate that is far from binding).  Few long caches are cut into chunks of up to
// 512 slots, a workgroup of four waves each, and a second kernel joins their sums and outputs; the weights need the joined
// sums, so the first one leaves the scores (4 bytes for each slot and head beside the slot's 4 head_dim).  Short ones, and many, have
// a workgroup of eight waves each, which adds the weights too: one launch, and nothing to join.
//
// Measured: 2 caches of 8 heads x 131072 slots x 128, 4 query heads each, 216 + 16 us, the first kernel at 5.1 TB/s (a copy of
// 2 GiB: 4.9); 64 ragged caches of 8 heads x up to 4096 slots 124 us in a workgroup each (in chunks 123 + 12); one of 16
// heads x 1000 slots 14.5 us, a launch and a chain of four tiles a wave.  With positions, which a tile waits for before the next
// is asked for, 2 to 3 % more in long caches and 4 to 15 % in that one.
#include "attn_core.h"

namespace lap {
namespace {

constexpr int TS = 32;                      // slots of a wave's tile
constexpr uint32_t CHUNK_WAVES = 4;         // waves of a chunk's workgroup
constexpr uint32_t WHOLE_WAVES = 8;         // and of one that goes through a whole cache
constexpr uint32_t WHOLE_SCORES = 6144;     // scores that the latter keeps in LDS

// floats from one head's scores to the next's there
__host__ __device__ __forceinline__ uint32_t score_pitch(uint32_t slots) { return (slots + TS - 1) / TS * TS + 4; }

// CHUNK: one of several workgroups of a cache, to be joined.  Or the only one, of up to 32 heads, with its scores in the
// workspace (WHOLE) or in LDS.
enum class Form { CHUNK, WHOLE, WHOLE_IN_LDS };

template <class T, int DP, int NW, Form FORM>
__global__ __launch_bounds__(NW * 64, 2) void k_step(StepShape s, StepWork w)
{
    constexpr bool WHOLE = FORM != Form::CHUNK, IN_LDS = FORM == Form::WHOLE_IN_LDS;
    constexpr int TILE = Tile<DP>::size(TS);
    __shared__ __align__(16) float kept[IN_LDS ? WHOLE_SCORES : 4];
    __shared__ float l2[32], totals[32];      // of a row: logarithm to base 2 of the whole sum, the sum on the maximum
    __shared__ __align__(16) char raw[NW * 2 * TILE * sizeof(T)];      // the waves' values; their outputs at the end
    __shared__ float2 sums[NW][32];
    T *const lv = (T *)raw;
    const uint32_t group = s.q_heads / s.kv_heads, parts = (group + 31) / 32;
    // Many caches: next to each other, so that the last chunks of ragged ones, which are empty, come last and to all dies
    // (64 caches of 8 heads, up to 4096 slots: 135 us, the other way 143).  Few: the chunks of one next to each other, which
    // memory prefers (2 x 8 x 131072 slots: 231 us, the other way 245).
    const uint32_t rows = s.batch * s.kv_heads * parts;
    const uint32_t row = rows >= 256 ? blockIdx.x % rows : blockIdx.x / s.splits;
    const uint32_t split = rows >= 256 ? blockIdx.x / rows : (blockIdx.x + row) % s.splits, part = row % parts;
    const uint32_t kvh = row / parts % s.kv_heads, b = row / parts / s.kv_heads;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
    const int n_rows = min(32, (int)(group - part * 32));
    const uint32_t head0 = kvh * group + part * 32;
    const int len = clamp_len(s.lens, b, s.slots);
    const int c0 = split * s.chunk, c1 = min(c0 + (int)s.chunk, len);

    const int r = lane & 31;
    typename Elem<T>::x8 qf[DP / 16], kf[DP / 16];
    load_kept<DP>(qf, (const T *)w.q.data + (int64_t)b * w.q.batch + (int64_t)(head0 + min(r, n_rows - 1)) * w.q.head, s.head_dim, lane);
    const T *gk = (const T *)w.k.data + (int64_t)b * w.k.batch + (int64_t)kvh * w.k.head;
    const T *gv = (const T *)w.v.data + (int64_t)b * w.v.batch + (int64_t)kvh * w.v.head;
    const int32_t *pos = w.positions ? w.positions + ((int64_t)b * s.kv_heads + kvh) * s.slots : nullptr;
    float *const scores = w.scores + ((int64_t)b * s.q_heads + head0 + r) * s.score_row;      // of the lane's head
    const uint32_t pitch = score_pitch(s.slots);
    const float c = s.scale * LOG2E;
    const ColRead<DP, T> cols(lane);
    const TileLoad<DP, TS, 1> tv(w.v.row, (int)s.head_dim / 8 - 1, 0, lane);
    T *const mine = lv + wave * 2 * TILE;

    f32x16 acc[DP / 32] = {};
    float m = LOWEST * c, l = 0.f;
    const auto fetch = [&](int at, int to) {      // slots at .. at + 31
        tv.issue(mine + to * TILE, gv, at, len - 1, 0);
        load_kept<DP>(kf, gk + (int64_t)min(at + r, len - 1) * w.k.row, s.head_dim, lane);
    };
    int at = c0 + wave * TS, buf = 0;
    if (at < c1) fetch(at, 0);
    for (; at < c1; at += NW * TS, buf ^= 1) {
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);      // this wave's keys and values are here
        asm volatile("" ::: "memory");
        f32x16 x = {};
#pragma unroll
        for (int d = 0; d < DP / 16; ++d) x = Elem<T>::mfma(kf[d], qf[d], x);
        const int32_t held = pos ? pos[min(at + r, len - 1)] : 0;
        if (at + NW * TS < c1) fetch(at + NW * TS, buf ^ 1);
        float p[16];
#pragma unroll
        for (int i = 0; i < 16; ++i) p[i] = x[i] * c;
        const uint32_t live = (uint32_t)__ballot(at + r < len && held >= 0);      // one bit for each slot of the tile
        if (live != ~0u) {
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = (live >> (8 * (i / 4) + 4 * h + i % 4)) & 1 ? p[i] : -ATTN_INF;
            // what an empty slot holds may be anything, and past the length stand copies of the last slot, which may be
            // infinite: zero times it is not always zero
            for (int n = lane; n < TS * DP / 8; n += 64)
                if (!((live >> (n / (DP / 8))) & 1)) *(s16x8 *)(mine + buf * TILE + Tile<DP>::place(n / (DP / 8), n % (DP / 8))) = s16x8{};
        }
        if (w.weights && r < n_rows) {
            float *const to = IN_LDS ? kept + r * pitch : scores;
#pragma unroll
            for (int i = 0; i < 16; i += 4) *(f32x4 *)(to + at + 2 * i + 4 * h) = f32x4{p[i], p[i + 1], p[i + 2], p[i + 3]};
        }
        float top = p[0];
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(top, p[i]);
        top = half_max(top);
        if (__ballot(top > m)) {
            const float up = fmaxf(m, top), by = exp2_fast(m - up);
            m = up;
            l *= by;
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= by;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            p[i] = exp2_fast(p[i] - m);
            l += p[i];
        }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
            const auto pf = round8<T>(p, 8 * t);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) acc[d] = Elem<T>::mfma(cols.get(mine + buf * TILE, t, d), pf, acc[d]);
        }
    }
    // join the waves: their sums, then their outputs, each on the workgroup's maximum
    l = half_sum(l);
    if (lane < 32) sums[wave][r] = make_float2(m, l);
    __syncthreads();
    float top = sums[0][r].x;
    for (int i = 1; i < NW; ++i) top = fmaxf(top, sums[i][r].x);
    const float by = exp2_fast(m - top);
    float *out = (float *)raw;      // [row][wave][DP]
    static_assert(2 * TS * sizeof(T) >= 32 * sizeof(float), "the outputs fit where the values were");
    if (r < n_rows)
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                f32x4 y;
#pragma unroll
                for (int j = 0; j < 4; ++j) y[j] = acc[d][i + j] * by;
                *(f32x4 *)(out + (r * NW + wave) * DP + 32 * d + 2 * i + 4 * h) = y;
            }
    float total = 0.f;      // of row r
    for (int i = 0; i < NW; ++i) total += sums[i][r].y * exp2_fast(sums[i][r].x - top);
    const bool some = total != 0.f;
    if (wave == 0 && lane < n_rows) {
        if constexpr (WHOLE) {
            w.lse[(int64_t)b * s.q_heads + head0 + r] = some ? top * LN2 + __logf(total) : -ATTN_INF;
            l2[r] = some ? top + __log2f(total) : ATTN_INF;
            totals[r] = total;
        } else {
            w.sums[((int64_t)b * s.q_heads + head0 + r) * s.splits + split] = make_float2(top, total);
        }
    }
    __syncthreads();
    for (int n = threadIdx.x; n < n_rows * (DP / 4); n += NW * 64) {
        const int row = n / (DP / 4), e = n % (DP / 4) * 4;
        f32x4 y = *(f32x4 *)(out + row * NW * DP + e);
        for (int i = 1; i < NW; ++i) y += *(f32x4 *)(out + (row * NW + i) * DP + e);
        if constexpr (WHOLE) {
            typename Elem<T>::x4 z;
            for (int j = 0; j < 4; ++j) z[j] = (T)(totals[row] != 0.f ? y[j] / totals[row] : 0.f);
            if (e < (int)s.head_dim) *(typename Elem<T>::x4 *)((T *)w.out.data + (int64_t)b * w.out.batch + (int64_t)(head0 + row) * w.out.head + e) = z;
        } else {
            *(f32x4 *)(w.outs + (((int64_t)b * s.q_heads + head0 + row) * s.splits + split) * DP + e) = y;
        }
    }
    if constexpr (WHOLE) {
        if (!w.weights) return;
        const float *const all = w.scores + ((int64_t)b * s.q_heads + head0) * s.score_row;
        const int64_t to = ((int64_t)b * s.kv_heads + kvh) * s.slots;
        const bool aligned = s.slots % 4 == 0 && ((uintptr_t)w.weights | (uintptr_t)w.before) % 16 == 0;
        for (uint32_t slot = threadIdx.x * 4; slot < s.slots; slot += NW * 64 * 4) {
            f32x4 sum = {};
            if ((int)slot < len) {
#pragma unroll 4
                for (int g = 0; g < n_rows; ++g) {
                    const f32x4 x = *(const f32x4 *)(IN_LDS ? kept + g * pitch + slot : all + (int64_t)g * s.score_row + slot);
                    for (int j = 0; j < 4; ++j) sum[j] += exp2_fast(x[j] - l2[g]);
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

constexpr int JOIN = 256, JOIN_SLOTS = 1024;

// maximum and sum of a head over its chunks, by a wave
__device__ __forceinline__ float2 join_sums(const float2 *sums, uint32_t n, int lane)
{
    float m = sums[0].x;
    for (uint32_t i = lane; i < n; i += 64) m = fmaxf(m, sums[i].x);
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d, 64));
    float l = 0.f;
    for (uint32_t i = lane; i < n; i += 64) l += sums[i].y * exp2_fast(sums[i].x - m);
    for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d, 64);
    return make_float2(m, l);
}

// The first batch * q_heads workgroups join the outputs of a head each, the others add the weights of JOIN_SLOTS slots.
template <class T, int DP> __global__ __launch_bounds__(JOIN) void k_step_join(StepShape s, StepWork w, uint32_t pieces)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t heads = s.batch * s.q_heads;
    if (blockIdx.x < heads) {
        constexpr int ACROSS = DP / 4, LANES = JOIN / ACROSS;      // threads of a row, rows at a time
        __shared__ f32x4 part[LANES][ACROSS];
        const uint32_t b = blockIdx.x / s.q_heads, head = blockIdx.x % s.q_heads;
        const float2 *sums = w.sums + (int64_t)blockIdx.x * s.splits;
        const float2 all = join_sums(sums, s.splits, lane);
        const int e = threadIdx.x % ACROSS, first = threadIdx.x / ACROSS;
        f32x4 y = {};
        const f32x4 *outs = (const f32x4 *)(w.outs + (int64_t)blockIdx.x * s.splits * DP);
#pragma unroll 4
        for (uint32_t i = first; i < s.splits; i += LANES) {
            // a chunk without slots has written zeros
            y += outs[(int64_t)i * ACROSS + e] * exp2_fast(sums[i].x - all.x);
        }
        part[first][e] = y;
        __syncthreads();
        if (first == 0) {
            for (int i = 1; i < LANES; ++i) y += part[i][e];
            const bool some = all.y != 0.f;
            typename Elem<T>::x4 z;
            for (int j = 0; j < 4; ++j) z[j] = (T)(some ? y[j] / all.y : 0.f);
            if (e * 4 < (int)s.head_dim) *(typename Elem<T>::x4 *)((T *)w.out.data + (int64_t)b * w.out.batch + (int64_t)head * w.out.head + e * 4) = z;
            if (threadIdx.x == 0) w.lse[blockIdx.x] = some ? all.x * LN2 + __logf(all.y) : -ATTN_INF;
        }
        return;
    }
    __shared__ float l2[MAX_GROUP];
    const uint32_t group = s.q_heads / s.kv_heads;
    const uint32_t item = (blockIdx.x - heads) / pieces, piece = (blockIdx.x - heads) % pieces;
    const uint32_t b = item / s.kv_heads, head0 = b * s.q_heads + item % s.kv_heads * group;
    for (uint32_t g = wave; g < group; g += JOIN / 64) {
        const float2 all = join_sums(w.sums + (int64_t)(head0 + g) * s.splits, s.splits, lane);
        if (lane == 0) l2[g] = all.y != 0.f ? all.x + __log2f(all.y) : ATTN_INF;
    }
    __syncthreads();
    const int len = clamp_len(s.lens, b, s.slots);
    const int64_t row = (int64_t)item * s.slots;
    const float *scores = w.scores + (int64_t)head0 * s.score_row;
    if (s.slots % 4 == 0 && ((uintptr_t)w.weights | (uintptr_t)w.before) % 16 == 0) {      // four slots for each thread
        const uint32_t slot = piece * JOIN_SLOTS + threadIdx.x * 4;
        if (slot >= s.slots) return;
        f32x4 sum = {};
        if ((int)slot < len) {
#pragma unroll 4
            for (uint32_t g = 0; g < group; ++g) {
                const f32x4 x = *(const f32x4 *)(scores + (int64_t)g * s.score_row + slot);
                for (int j = 0; j < 4; ++j) sum[j] += exp2_fast(x[j] - l2[g]);
            }
            for (int j = 1; j < 4; ++j) sum[j] = (int)slot + j < len ? sum[j] : 0.f;
        }
        *(f32x4 *)(w.weights + row + slot) = *(const f32x4 *)(w.before + row + slot) + sum;
        return;
    }
    for (uint32_t i = 0; i < JOIN_SLOTS; i += JOIN) {
        const uint32_t slot = piece * JOIN_SLOTS + i + threadIdx.x;
        if (slot >= s.slots) return;
        float sum = 0.f;
        if ((int)slot < len)
            for (uint32_t g = 0; g < group; ++g) sum += exp2_fast(scores[(int64_t)g * s.score_row + slot] - l2[g]);
        w.weights[row + slot] = w.before[row + slot] + sum;
    }
}

template <class T, int DP> hipError_t launch(const StepShape &s, const StepWork &w, hipStream_t st)
{
    const uint32_t parts = (s.q_heads / s.kv_heads + 31) / 32;
    if (s.whole) {
        const uint32_t grid = s.batch * s.kv_heads;
        if (s.score_row) k_step<T, DP, WHOLE_WAVES, Form::WHOLE><<<grid, WHOLE_WAVES * 64, 0, st>>>(s, w);
        else k_step<T, DP, WHOLE_WAVES, Form::WHOLE_IN_LDS><<<grid, WHOLE_WAVES * 64, 0, st>>>(s, w);
        return hipGetLastError();
    }
    k_step<T, DP, CHUNK_WAVES, Form::CHUNK><<<s.splits * parts * s.batch * s.kv_heads, CHUNK_WAVES * 64, 0, st>>>(s, w);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    const uint32_t pieces = w.weights ? (s.slots + JOIN_SLOTS - 1) / JOIN_SLOTS : 0;
    k_step_join<T, DP><<<s.batch * (s.q_heads + s.kv_heads * pieces), JOIN, 0, st>>>(s, w, pieces);
    return hipGetLastError();
}

}  // namespace

// One workgroup for a cache, in us, chunks beside it (keys of 128 elements, b caches of 8 heads, lengths all equal or ragged):
//   1 x 16 heads   500 slots 12.9 17.2, 1000 14.1 17.3, 1500 18.6 17.5      b = 16   1500 22 26, 2900 36 41, 4000 60 53
//   b = 24         2000 33 42, 4000 81 94, 16000 363 293                    b = 36   2000 74 71 (ragged 31 43), 4000 153 123 (70 70)
//   b = 48         2000 87 100, 4000 162 160 (87 101)                       b = 64   1000 46 56, 4000 188 210, 16000 961 931
//   b = 96         2000 145 161, 4000 278 305, 8000 622 603                 (b = 64, ragged, 4 query heads each: 4096 123 135)
// So up to 1024 slots always, up to 2048 where there are workgroups for half the units, up to 4096 where the last round of
// workgroups fills three quarters of them (eight waves take up a unit's LDS).
static bool whole_caches(uint64_t rows, uint32_t slots)
{
    const uint64_t rounds = (rows + 255) / 256;
    return slots <= 1024 || (slots <= 2048 && rows >= 128) || (slots <= 4096 && rows >= 192 * rounds);
}

// Chunks: workgroups enough to keep the chip evenly loaded to the end, of a tile for each wave at least and 512 slots at
// most (64 caches of 8 heads, up to 4096 slots: 135 us, with 1024 slots 157, with 256 142; with eight waves and 1024 slots 144).
void step_split(StepShape &s)
{
    const uint64_t rows = (uint64_t)s.batch * s.kv_heads * ((s.q_heads / s.kv_heads + 31) / 32);
    const uint64_t least = CHUNK_WAVES * TS, most = 512;
    const uint64_t want = (uint64_t)s.slots * rows / 4096;
    const uint64_t chunk = (want < least ? least : want > most ? most : want) / least * least;
    s.chunk = (uint32_t)chunk;
    s.splits = (uint32_t)((s.slots + chunk - 1) / chunk);
    if (!s.splits) s.splits = 1;
    s.score_row = ((uint64_t)s.slots + TS - 1) / TS * TS;
    const uint32_t group = s.q_heads / s.kv_heads;
    s.whole = group <= 32 && whole_caches(rows, s.slots);
    if (!s.whole) return;
    s.chunk = s.slots, s.splits = 1;
    if ((uint64_t)group * score_pitch(s.slots) <= WHOLE_SCORES) s.score_row = 0;
}

hipError_t launch_attention_step(const StepShape &s, const StepWork &w, hipStream_t st)
{
    if (s.half) return s.head_dim <= 64 ? launch<_Float16, 64>(s, w, st) : launch<_Float16, 128>(s, w, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, w, st) : launch<__bf16, 128>(s, w, st);
}

}  // namespace lap
