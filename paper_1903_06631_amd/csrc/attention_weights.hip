// The attention weight that every key has received: w_j += sum over rows i and the query heads that share the key of
// p_ij = exp(scale q_i.k_j - lse_i), with the sums of the forward pass.
//
// A workgroup keeps keys and streams the rows of their heads; a lane adds up the probabilities of one key for each block of
// 32 that its wave keeps.  Where that makes too few workgroups, or under a causal mask too few to share out long and short
// ones, the rows are cut into parts, whose sums a second kernel adds in order.  For a block of 32 x 32 pairs of 128 elements 8
// products of 32 cycles stand against some 90 vector instructions (16 exponentials among them).  Measured: 2 x 32 heads on 8 x
// 8192 tokens, causal, 560 us = 980 TFLOP/s, at 2.0 GHz and 47 % of the matrix cycles: bound by power.
#include <algorithm>

#include "attn_core.h"

namespace lap {
namespace {

constexpr int QT = 64, NW = 4;      // rows of a tile, waves

template <class T, int DP, int KB>
__global__ __launch_bounds__(NW * 64, 2) void k_attention_weights(AttnShape s, Rows q, Rows k, const float *lse, const float *before,
                                                               float *weights, uint32_t parts)
{
    constexpr int BK = 32 * KB * NW;
    __shared__ __align__(16) T lq[2][Tile<DP>::size(QT)];
    __shared__ __align__(16) float lst[2][64];
    static_assert(QT == 64, "a wave fetches the numbers of 64 rows at once");
    Work wk;
    if (!work_item(s, parts, wk)) return;
    const uint32_t b = wk.b, kvh = wk.kvh;
    const int first = (int)wk.tile * BK;      // the first keys of a causal head are seen by the most rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span sp = span_of(s, b);
    const uint32_t group = s.q_heads / s.kv_heads;

    const int w0 = first + 32 * KB * wave;
    float sum[KB] = {};
    const int end = min(first + BK, sp.kl);
    const int r0 = first < sp.kl ? row_lo(s, sp, first) / QT * QT : 0;
    const int r1 = first < sp.kl ? row_hi(s, sp, end - 1) : 0;
    const int per = r0 < r1 ? (r1 - r0 + QT - 1) / QT : 0;
    const int n0 = uniform((int)((int64_t)per * group * wk.g / parts)), n1 = uniform((int)((int64_t)per * group * (wk.g + 1) / parts));
    if (n0 < n1) {
        typename Elem<T>::x8 kf[KB][DP / 16];
        int hi[KB], lo[KB];
#pragma unroll
        for (int n = 0; n < KB; ++n) {
            const int used = min(w0 + 32 * n + (lane & 31), sp.kl - 1);
            load_kept<DP>(kf[n], (const T *)k.data + (int64_t)b * k.batch + (int64_t)kvh * k.head + (int64_t)used * k.row, s.head_dim, lane);
            hi[n] = row_hi(s, sp, used), lo[n] = row_lo(s, sp, used);
        }
        const int w_last = min(w0 + 32 * KB - 1, sp.kl - 1), w_first = min(w0, sp.kl - 1);
        const int all_hi = row_hi(s, sp, w_first), all_lo = row_lo(s, sp, w_last);
        const int any_hi = row_hi(s, sp, w_last), any_lo = row_lo(s, sp, w_first);
        const float c = s.scale * LOG2E;
        const RowRead<DP, T> rows(lane);
        const TileLoad<DP, QT, NW> tq(q.row, (int)s.head_dim / 8 - 1, wave, lane);
        const int64_t head0 = uniform((int)(kvh * group) + n0 / per);
        const T *gq = (const T *)q.data + (int64_t)b * q.batch + head0 * q.head;
        const float *gs = lse + ((int64_t)b * s.q_heads + head0) * s.q_len;
        int next = uniform(r0 + n0 % per * QT);      // rows of the next tile to ask for
        const auto issue = [&](int to) {
            tq.issue(lq[to], gq, next, sp.ql - 1, wave);
            if (wave == 0) load_floats(lst[to], gs, next, sp.ql - 1, 0, lane);
            next += QT;
            if (next >= r1) next = r0, gq += q.head, gs += s.q_len;
        };
        int buf = 0, qt = next;
        zero_tiles<DP, NW * 64>(lq[0], sizeof(lq) / sizeof(T), s.head_dim);
        issue(0);
        for (int n = n0; n < n1; ++n, buf ^= 1) {
            tiles_arrive();
            if (n + 1 < n1) issue(buf ^ 1);
            const int tile = qt;
            qt = qt + QT >= r1 ? r0 : qt + QT;
#pragma unroll
            for (int qb = 0; qb < QT / 32; ++qb) {
                const int at = tile + 32 * qb;
                if (at >= any_hi || at + 32 <= any_lo) continue;
                f32x16 x[KB];
#pragma unroll
                for (int m = 0; m < KB; ++m) x[m] = f32x16{};
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) {
                    const auto a = rows.get(lq[buf], qb, d);
#pragma unroll
                    for (int m = 0; m < KB; ++m) x[m] = Elem<T>::mfma(a, kf[m][d], x[m]);
                }
                float l2[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    // minus infinity: a row without keys, or whose scores are all below what counts; others as they are, so
                    // that what is not a number stays so
                    const float sum = lst[buf][32 * qb + 8 * (i / 4) + 4 * (lane >> 5) + i % 4];
                    l2[i] = sum == -ATTN_INF ? sum : -LOG2E * sum;
                }
                const bool whole = at + 32 <= all_hi && at >= all_lo;
#pragma unroll
                for (int m = 0; m < KB; ++m) {
                    float p[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) p[i] = exp2_fast(__builtin_fmaf(x[m][i], c, l2[i]));
                    if (!whole) {
                        const int row0 = at + 4 * (lane >> 5);
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int row = row0 + 8 * (i / 4) + i % 4;
                            p[i] = row < hi[m] && row >= lo[m] ? p[i] : 0.f;
                        }
                    }
                    // the block's own sum first: 16 small terms at a time lose less in a long one
                    float part = 0.f;
#pragma unroll
                    for (int i = 0; i < 16; ++i) part += p[i];
                    sum[m] += part;
                }
            }
        }
    }
#pragma unroll
    for (int n = 0; n < KB; ++n) {
        const int key = w0 + 32 * n + (lane & 31);
        const float all = half_sum(sum[n]);
        if (key < (int)s.k_len && lane < 32) {
            const int64_t at = (((int64_t)b * s.kv_heads + kvh) * parts + wk.g) * s.k_len + key;
            weights[at] = (before ? before[at] : 0.f) + (key < sp.kl ? all : 0.f);
        }
    }
}

__global__ __launch_bounds__(256) void k_add_parts(const float *sums, uint32_t parts, const float *before, float *weights, uint32_t len)
{
    const uint32_t j = blockIdx.x * 256 + threadIdx.x;
    if (j >= len) return;
    const float *from = sums + (int64_t)blockIdx.y * parts * len + j;
    float sum = 0.f;
    for (uint32_t i = 0; i < parts; ++i) sum += from[(int64_t)i * len];
    const int64_t at = (int64_t)blockIdx.y * len + j;
    weights[at] = (before ? before[at] : 0.f) + sum;
}

template <class T, int DP>
hipError_t launch(const AttnShape &s, const Rows &q, const Rows &k, const float *lse, const float *before, float *weights, float *sums, hipStream_t st)
{
    const uint32_t caches = padded_caches(s.batch * s.kv_heads), parts = weights_parts(s);
    const uint32_t keys = 32 * NW * weights_blocks(s), total = caches * ((s.k_len + keys - 1) / keys) * parts;
    const float *first = parts > 1 ? nullptr : before;
    float *to = parts > 1 ? sums : weights;
    if (weights_blocks(s) == 2) k_attention_weights<T, DP, 2><<<total, NW * 64, 0, st>>>(s, q, k, lse, first, to, parts);
    else k_attention_weights<T, DP, 1><<<total, NW * 64, 0, st>>>(s, q, k, lse, first, to, parts);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    k_add_parts<<<dim3((s.k_len + 255) / 256, s.batch * s.kv_heads), 256, 0, st>>>(sums, parts, before, weights, s.k_len);
    return hipGetLastError();
}

}  // namespace

// Blocks of 32 keys that a wave keeps: two, so that what it reads from LDS serves two products (2 x 32 heads x 8192 tokens:
// 558 us, with one 628 us), unless that leaves units without work.
uint32_t weights_blocks(const AttnShape &s)
{
    return (uint64_t)s.batch * s.kv_heads * ((s.k_len + 127) / 128) * (s.q_heads / s.kv_heads) * ((s.q_len + 255) / 256) >= 512 ? 2 : 1;
}
// Parts of the rows: enough for 2048 workgroups (2 x 32 heads x 8192 tokens: 558 us, with 1024 of them 582, with 4096 561), of
// 512 rows each at least (16 x 16 heads on 4 x 600 tokens: 28 us, with 256 rows 33); where that leaves fewer than 512
// workgroups, as many as that, of 256 rows at least (8 heads of 1500 tokens: 16 us, with 512 rows 26, with 1024 40).
uint32_t weights_parts(const AttnShape &s)
{
    const uint32_t keys = 32 * NW * weights_blocks(s);
    const uint64_t groups = (uint64_t)s.batch * s.kv_heads * ((s.k_len + keys - 1) / keys), rows = (uint64_t)(s.q_heads / s.kv_heads) * s.q_len;
    if (!groups) return 1;
    uint64_t parts = std::min((2048 + groups - 1) / groups, rows / 512);
    if (groups * parts < 512) parts = std::min((512 + groups - 1) / groups, rows / 256);
    return (uint32_t)std::max<uint64_t>(parts, 1);
}

hipError_t launch_attention_weights(const AttnShape &s, const Rows &q, const Rows &k, const float *lse, const float *before, float *weights,
                                    float *sums, hipStream_t st)
{
    if (s.half)
        return s.head_dim <= 64 ? launch<_Float16, 64>(s, q, k, lse, before, weights, sums, st) : launch<_Float16, 128>(s, q, k, lse, before, weights, sums, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, q, k, lse, before, weights, sums, st) : launch<__bf16, 128>(s, q, k, lse, before, weights, sums, st);
}

}  // namespace lap
