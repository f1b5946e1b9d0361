// Host-side launch wrappers of the attention and cache kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lap {

// rows of [batch, heads, length, head_dim], elements of a row one after the other; strides in elements
struct Rows {
    void *data;
    int64_t batch, head, row;
};

struct AttnShape {
    uint32_t batch, q_heads, kv_heads, q_len, k_len, head_dim;
    int32_t causal, window;
    float scale;
    const int32_t *q_lens, *k_lens;
    bool half;      // IEEE binary16, else bfloat16
};

uint32_t forward_parts(const AttnShape &s);
size_t forward_workspace(const AttnShape &s);
hipError_t launch_attention(const AttnShape &s, const Rows &q, const Rows &k, const Rows &v, const Rows &out, float *lse, void *ws, hipStream_t st);

struct AttnGrad {
    Rows g, q, k, v, out, dq, dk, dv;
    const float *lse;
    float *stats;       // sums in base 2 (plus infinity: no key) [batch, q_heads, q_len], then delta likewise
    float *sums;        // grad_sums(s) bytes
};
uint32_t grad_parts(const AttnShape &s);
size_t grad_sums(const AttnShape &s);
hipError_t launch_attention_grad(const AttnShape &s, const AttnGrad &a, hipStream_t st);
// sums: [batch, kv_heads, weights_parts(s), k_len], unless that is one part
uint32_t weights_blocks(const AttnShape &s);
uint32_t weights_parts(const AttnShape &s);
hipError_t launch_attention_weights(const AttnShape &s, const Rows &q, const Rows &k, const float *lse, const float *before, float *weights,
                                    float *sums, hipStream_t st);

constexpr uint32_t SCORE_TILE = 32;
constexpr uint32_t MAX_GROUP = 256;      // rows of queries (heads times tokens) that share one key head in a step

struct StepShape {
    uint32_t batch, q_heads, kv_heads, slots, head_dim;
    float scale;
    const int32_t *lens;
    bool half;
    uint32_t tokens;             // of every sequence (of rows in 16 bits: 1)
    const int32_t *q_lens;       // how many of them are in use, NULL: all
    uint32_t group;              // rows of queries of a key head; this and the next by packed_step_split
    uint32_t shares;             // workgroups for each part of a key head's rows, among which all sequences are shared out
    uint32_t chunk, splits;      // (packed, with lengths: what to cut all of a key head's into) slots of a workgroup, workgroups of a cache (step_split)
    uint64_t score_row;          // floats between two heads' scores (0: they stay in LDS)
    bool whole;                  // one workgroup for all of a cache, and nothing to join
};
struct StepWork {
    Rows q, k, v, out;      // q, out: row unused where there is one token; packed k, v: strides in bytes
    const int32_t *positions;
    const float *before;
    float *lse, *weights;
    float *outs;            // [batch, q_heads, splits, 64 or 128]; packed: [kv_heads, parts, shares, rows of a part, 64 or 128]
    float2 *sums;           // the same without the last: maximum in base 2 (packed: of q.k), sum
    float *scores;          // [batch, q_heads, tokens, score_row] in base 2, where weights are asked for; packed: q.k [batch,
                            // kv_heads, score_row / SCORE_TILE, rows of a key head, SCORE_TILE]
    uint2 *table;           // packed: [batch] a sequence's first share, how many it has
};
void step_split(StepShape &s);
hipError_t launch_attention_step(const StepShape &s, const StepWork &w, hipStream_t st);

// caches in 4 or 8 bits an element: packed_rows.h
constexpr int PACK_GROUP = 32;
__host__ __device__ __forceinline__ uint32_t pack_groups(uint32_t head_dim) { return (head_dim + PACK_GROUP - 1) / PACK_GROUP; }
// byte of a row where lo and step of its groups begin
__host__ __device__ __forceinline__ uint32_t pack_ends(uint32_t head_dim, uint32_t bits) { return pack_groups(head_dim) * bits * 4; }
__host__ __device__ __forceinline__ uint32_t pack_row_bytes(uint32_t head_dim, uint32_t bits)
{
    return (pack_ends(head_dim, bits) + pack_groups(head_dim) * 4 + 15) / 16 * 16;
}

__host__ __device__ __forceinline__ uint32_t step_part(uint32_t group) { return group <= 16 ? 16 : 32; }      // rows of a workgroup
__host__ __device__ __forceinline__ uint32_t step_parts(uint32_t group) { return (group + step_part(group) - 1) / step_part(group); }
void packed_step_split(StepShape &s);
hipError_t launch_packed_join(const StepShape &s, const StepWork &w, hipStream_t st);
hipError_t launch_attention_step_packed(const StepShape &s, const StepWork &w, uint32_t bits, hipStream_t st);

struct PackShape {
    uint32_t batch, kv_heads, slots, n, head_dim, bits;      // n: rows of the plain tensors
    const int32_t *lens, *first;      // rows in use, slot of the first one; NULL: n, 0
    bool half;
};
// k, v: plain rows; k_cache, v_cache: strides in bytes
hipError_t launch_cache_pack(const PackShape &s, const Rows &k, const Rows &v, const Rows &k_cache, const Rows &v_cache, hipStream_t st);
hipError_t launch_cache_unpack(const PackShape &s, const Rows &k_cache, const Rows &v_cache, const Rows &k, const Rows &v, hipStream_t st);

struct EvictShape {
    uint32_t batch, kv_heads, slots, slots_out, head_dim, keep, recent;
    const int32_t *lens;
};
struct InsertShape {
    uint32_t batch, kv_heads, slots, head_dim, recent;
};
// kept [batch, kv_heads, slots_out] scratch
hipError_t launch_cache_evict(const EvictShape &s, const Rows &k, const Rows &v, const float *weights, const int32_t *positions,
                              const Rows &k_out, const Rows &v_out, float *weights_out, int32_t *positions_out, int32_t *lens_out,
                              int32_t *kept, hipStream_t st);
hipError_t launch_cache_insert(const InsertShape &s, const Rows &k_new, const Rows &v_new, const Rows &k, const Rows &v, float *weights,
                               int32_t *positions, const int32_t *position, int32_t *slots_out, hipStream_t st);

}  // namespace lap
