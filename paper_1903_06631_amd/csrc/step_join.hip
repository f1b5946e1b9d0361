// What attention of new tokens over caches in chunks ends with: outputs and sums of the chunks joined, and the weights, which
// need the joined sums.  Bound by memory where weights are asked for (the scores, 4 bytes for each slot and row of queries, are
// mostly still in the caches), else a launch and a chain of a few accesses.
#include "attn_core.h"

namespace lap {
namespace {

constexpr int JOIN = 256, JOIN_SLOTS = 1024;

// maximum and sum of a row over its chunks, by a wave
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

// The first batch * q_heads * tokens workgroups join the outputs of a row each, the others add the weights of JOIN_SLOTS slots.
template <class T, int DP> __global__ __launch_bounds__(JOIN) void k_step_join(StepShape s, StepWork w, uint32_t pieces)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t of_one = s.q_heads * s.tokens, rows = s.batch * of_one;      // rows of queries
    if (blockIdx.x < rows) {
        constexpr int ACROSS = DP / 4, LANES = JOIN / ACROSS;      // threads of a row, rows at a time
        __shared__ f32x4 part[LANES][ACROSS];
        const uint32_t b = blockIdx.x / of_one, head = blockIdx.x % of_one / s.tokens, token = blockIdx.x % s.tokens;
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
            if (e * 4 < (int)s.head_dim) *(typename Elem<T>::x4 *)((T *)w.out.data + (int64_t)b * w.out.batch + (int64_t)head * w.out.head + (int64_t)token * w.out.row + e * 4) = z;
            if (threadIdx.x == 0) w.lse[blockIdx.x] = some ? all.x * LN2 + __logf(all.y) : -ATTN_INF;
        }
        return;
    }
    __shared__ float l2[MAX_GROUP];
    const uint32_t group = s.q_heads / s.kv_heads * s.tokens;
    const uint32_t item = (blockIdx.x - rows) / pieces, piece = (blockIdx.x - rows) % pieces;
    const uint32_t b = item / s.kv_heads, head0 = b * of_one + item % s.kv_heads * group;
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
    const uint32_t pieces = w.weights ? (s.slots + JOIN_SLOTS - 1) / JOIN_SLOTS : 0;
    k_step_join<T, DP><<<s.batch * (s.q_heads * s.tokens + s.kv_heads * pieces), JOIN, 0, st>>>(s, w, pieces);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_step_join(const StepShape &s, const StepWork &w, hipStream_t st)
{
    if (s.half) return s.head_dim <= 64 ? launch<_Float16, 64>(s, w, st) : launch<_Float16, 128>(s, w, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, w, st) : launch<__bf16, 128>(s, w, st);
}

}  // namespace lap
