// What attention of new tokens over packed caches in chunks ends with: outputs and sums of the chunks joined, and the weights,
// which need the joined sums.  A launch and a chain of a few accesses; with weights bound by memory where caches are long (the
// scores, 4 bytes for each slot and row of queries, are mostly still in the last cache).  Measured: 2 caches of 8 heads x 131 072
// slots with weights of 4 query heads each 12.2 us (34 MB of scores, 17 of weights read and written), 32 of 2047 slots and 32 query heads 6.1,
// without weights 4.3 to 5.6.
#include "packed_rows.h"

namespace lap {
namespace {

constexpr int JOIN = 256, JOIN_WAVES = JOIN / 64, AHEAD = 8;

// maximum of the products and sum, over this many lanes next to each other; c: products to exponents of two
__device__ __forceinline__ float2 join_lanes(float2 a, uint32_t lanes, float c)
{
    for (uint32_t d = lanes / 2; d; d >>= 1) {
        const float m = __shfl_xor(a.x, d, 64), l = __shfl_xor(a.y, d, 64), top = fmaxf(a.x, m);
        a = make_float2(top, a.y * exp2_fast((a.x - top) * c) + l * exp2_fast((m - top) * c));
    }
    return a;
}
// and over a row's chunks, the lane-th of `lanes`
__device__ __forceinline__ float2 join_chunks(const float2 *sums, uint32_t n, uint32_t stride, uint32_t lane, uint32_t lanes, float c)
{
    float2 a = make_float2(-__FLT_MAX__, 0.f);
#pragma unroll 4
    for (uint32_t i = lane; i < n; i += lanes) {
        const float2 x = sums[(int64_t)i * stride];
        const float top = fmaxf(a.x, x.x);
        a = make_float2(top, a.y * exp2_fast((a.x - top) * c) + x.y * exp2_fast((x.x - top) * c));
    }
    return a;
}

// a sequence's first chunk, how many it has
__device__ __forceinline__ uint2 chunks_of(const StepShape &s, const StepWork &w, uint32_t b) { return s.lens ? w.table[b] : make_uint2(b * s.splits, s.splits); }

// Workgroups below row_groups join the outputs of JOIN_WAVES / waves rows each, `waves` waves for one; the others add the
// weights of `each` slots, four to a thread, the rows of the key head shared out where that leaves threads over.
template <class T, int DP>
__global__ __launch_bounds__(JOIN) void k_packed_join(StepShape s, StepWork w, uint32_t row_groups, uint32_t waves, uint32_t pieces, uint32_t each)
{
    constexpr int E = DP / 64;      // elements of a lane
    typedef float f32xE __attribute__((ext_vector_type(E)));
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const uint32_t of_one = s.q_heads * s.tokens, rows = s.batch * of_one;      // rows of queries
    const float c = s.scale * LOG2E;
    if (blockIdx.x < row_groups) {
        __shared__ f32xE part[JOIN_WAVES][64];
        const uint32_t row = blockIdx.x * (JOIN_WAVES / waves) + wave / waves, first = wave % waves;
        f32xE y = {};
        float2 all = {};
        const uint32_t b = row / of_one, of = row - b * of_one;
        if (row < rows) {
            const uint32_t kvh = of / s.group, r = of - kvh * s.group, parts = step_parts(s.group), of_part = step_part(s.group);
            const uint2 chunks = chunks_of(s, w, b);
            const int64_t at = ((int64_t)(kvh * parts + r / of_part) * s.shares + chunks.x) * of_part + r % of_part;
            const float2 *sums = w.sums + at;
            const f32xE *outs = (const f32xE *)(w.outs + at * DP) + lane;
            all = join_lanes(join_chunks(sums, chunks.y, of_part, lane, 64, c), 64, c);
            for (uint32_t i = first; i < chunks.y; i += waves * AHEAD) {
                f32xE x[AHEAD];
                float m[AHEAD];
#pragma unroll
                for (int j = 0; j < AHEAD; ++j) {
                    const int64_t k = (int64_t)min(i + j * waves, chunks.y - 1) * of_part;
                    x[j] = outs[k * 64], m[j] = sums[k].x;
                }
#pragma unroll
                for (int j = 0; j < AHEAD; ++j)
                    if (i + j * waves < chunks.y) y += x[j] * exp2_fast((m[j] - all.x) * c);
            }
        }
        if (waves > 1) {
            part[wave][lane] = y;
            __syncthreads();
            if (first == 0)
                for (uint32_t i = 1; i < waves; ++i) y += part[wave + i][lane];
        }
        if (row >= rows || first) return;
        const bool some = all.y != 0.f;
        const uint32_t head = s.tokens == 1 ? of : of / s.tokens, token = of - head * s.tokens, e = lane * E;
        typedef T TE __attribute__((ext_vector_type(E)));
        TE z;
        for (int j = 0; j < E; ++j) z[j] = (T)(some ? y[j] / all.y : 0.f);
        if (e < s.head_dim) *(TE *)((T *)w.out.data + (int64_t)b * w.out.batch + (int64_t)head * w.out.head + (int64_t)token * w.out.row + e) = z;
        if (lane == 0) w.lse[row] = some ? all.x * s.scale + __logf(all.y) : -ATTN_INF;
        return;
    }
    __shared__ float2 whole[MAX_GROUP];      // of a row: its largest product and the logarithm to base 2 of its sum on that
    __shared__ f32x4 shares[JOIN];
    const uint32_t group = s.group;
    const uint32_t item = (blockIdx.x - row_groups) / pieces, piece = (blockIdx.x - row_groups) % pieces;
    const uint32_t b = item / s.kv_heads, row0 = item * group, of_part = step_part(group);
    const int len = clamp_len(s.lens, b, s.slots);
    const uint32_t quads = each / 4, share = threadIdx.x / quads, of = JOIN / quads;
    const uint32_t slot = piece * each + threadIdx.x % quads * 4;
    // the first scores are on their way while the sums are joined
    const float *from = w.scores + (int64_t)row0 * s.score_row + (int64_t)(slot / SCORE_TILE) * group * SCORE_TILE + slot % SCORE_TILE;
    f32x4 x[AHEAD] = {};
    if ((int)slot < len)
#pragma unroll
        for (int j = 0; j < AHEAD; ++j)
            if (share + j * of < group) x[j] = *(const f32x4 *)(from + (share + j * of) * SCORE_TILE);
    const uint32_t lanes = group <= 4 ? 64 : group <= 8 ? 32 : group <= 16 ? 16 : 8, at_once = JOIN / lanes;      // lanes of a row
    const uint2 chunks = chunks_of(s, w, b);
    const int64_t of_head = (int64_t)(item - b * s.kv_heads) * step_parts(group);
    for (uint32_t r = threadIdx.x / lanes; r < (group + at_once - 1) / at_once * at_once; r += at_once) {
        const uint32_t l = lane % lanes, row = min(r, group - 1);
        const float2 *sums = w.sums + ((of_head + row / of_part) * s.shares + chunks.x) * of_part + row % of_part;
        const float2 all = join_lanes(join_chunks(sums, chunks.y, of_part, l, lanes, c), lanes, c);
        if (l == 0 && r < group) whole[r] = all.y != 0.f ? make_float2(all.x, __log2f(all.y)) : make_float2(ATTN_INF, 0.f);
    }
    __syncthreads();
    f32x4 sum = {};
    if ((int)slot < len)
        for (uint32_t r0 = share; r0 < group; r0 += AHEAD * of) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const uint32_t r = r0 + i * of;
                if (r < group)
                    for (int j = 0; j < 4; ++j) sum[j] += received(x[i][j], whole[r], c);
            }
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                const uint32_t r = r0 + (AHEAD + i) * of;
                if (r < group) x[i] = *(const f32x4 *)(from + r * SCORE_TILE);
            }
        }
    if (of > 1) {
        shares[threadIdx.x] = sum;
        __syncthreads();
        if (share) return;
        for (uint32_t i = 1; i < of; ++i) sum += shares[i * quads + threadIdx.x];
    }
    for (int j = 0; j < 4; ++j) sum[j] = (int)slot + j < len ? sum[j] : 0.f;
    const int64_t to = (int64_t)item * s.slots + slot;
    if (s.slots % 4 == 0 && ((uintptr_t)w.weights | (uintptr_t)w.before) % 16 == 0) {
        if (slot < s.slots) *(f32x4 *)(w.weights + to) = *(const f32x4 *)(w.before + to) + sum;
    } else {
        for (int j = 0; j < 4; ++j)
            if (slot + j < s.slots) w.weights[to + j] = w.before[to + j] + sum[j];
    }
}

template <class T, int DP> hipError_t launch(const StepShape &s, const StepWork &w, hipStream_t st)
{
    const uint32_t rows = s.batch * s.q_heads * s.tokens, waves = rows >= 1024 || s.shares <= AHEAD * s.batch ? 1 : JOIN_WAVES;
    const uint32_t row_groups = (rows * waves + JOIN_WAVES - 1) / JOIN_WAVES;
    const uint64_t quads = (uint64_t)s.batch * s.kv_heads * ((s.slots + 3) / 4);
    const uint32_t each = quads >= 512 * JOIN ? 1024 : quads >= 128 * JOIN ? 256 : 128;
    const uint32_t pieces = w.weights ? (s.slots + each - 1) / each : 0;
    k_packed_join<T, DP><<<row_groups + s.batch * s.kv_heads * pieces, JOIN, 0, st>>>(s, w, row_groups, waves, pieces, each);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_packed_join(const StepShape &s, const StepWork &w, hipStream_t st)
{
    if (s.half) return s.head_dim <= 64 ? launch<_Float16, 64>(s, w, st) : launch<_Float16, 128>(s, w, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, w, st) : launch<__bf16, 128>(s, w, st);
}

}  // namespace lap
