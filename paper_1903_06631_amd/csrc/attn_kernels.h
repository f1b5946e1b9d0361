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

constexpr uint32_t MAX_GROUP = 256;      // query heads that share one key head, in attention_step.hip

struct StepShape {
    uint32_t batch, q_heads, kv_heads, slots, head_dim;
    float scale;
    const int32_t *lens;
    bool half;
    uint32_t chunk, splits;      // slots of a workgroup, workgroups of a cache (step_split)
    uint64_t score_row;          // floats between two heads' scores (0: they stay in LDS)
    bool whole;                  // one workgroup for all of a cache, and nothing to join
};
struct StepWork {
    Rows q, k, v, out;      // q, out: row unused
    const int32_t *positions;
    const float *before;
    float *lse, *weights;
    float *outs;            // [batch, q_heads, splits, 64 or 128]
    float2 *sums;           // [batch, q_heads, splits]: maximum in base 2, sum
    float *scores;          // [batch, q_heads, score_row] in base 2, where weights are asked for
};
void step_split(StepShape &s);
hipError_t launch_attention_step(const StepShape &s, const StepWork &w, hipStream_t st);

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
