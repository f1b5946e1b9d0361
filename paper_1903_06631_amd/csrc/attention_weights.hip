// The attention weight that every key has received: w_j += sum over rows i and the query heads that share the key of
// p_ij = exp(scale q_i.k_j - lse_i), with the sums of the forward pass.
//
// A workgroup keeps keys and streams the rows of their heads; a lane adds up the probabilities of one key.
#include "attn_core.h"

namespace lap {
namespace {

constexpr int QT = 32;      // rows of a tile

template <class T, int DP, int NW>
__global__ __launch_bounds__(NW * 64, 2) void k_attention_weights(AttnShape s, Rows q, Rows k, const float *lse, const float *before,
                                                               float *weights, uint32_t tiles)
{
    constexpr int BK = 32 * NW;
    __shared__ __align__(16) T lq[2][QT * DP];
    __shared__ __align__(16) float lst[2][QT];
    uint32_t item;
    if (!work_item(s.batch * s.kv_heads * tiles, item)) return;
    const uint32_t head = item / tiles, b = head / s.kv_heads, kvh = head % s.kv_heads;
    const int first = (int)(item % tiles) * BK;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span sp = span_of(s, b);
    const uint32_t group = s.q_heads / s.kv_heads;

    const int w0 = first + 32 * wave;
    const int key = w0 + (lane & 31);
    float sum = 0.f;
    const int end = min(first + BK, sp.kl);
    const int r0 = first < sp.kl ? row_lo(s, sp, first) / QT * QT : 0;
    const int r1 = first < sp.kl ? row_hi(s, sp, end - 1) : 0;
    if (r0 < r1) {
        const int used = min(key, sp.kl - 1);
        typename Elem<T>::x8 kf[DP / 16];
        load_kept<DP>(kf, (const T *)k.data + (int64_t)b * k.batch + (int64_t)kvh * k.head + (int64_t)used * k.row, s.head_dim, lane);
        const int hi = row_hi(s, sp, used), lo = row_lo(s, sp, used);
        const int w_last = min(w0 + 31, sp.kl - 1), w_first = min(w0, sp.kl - 1);
        const int all_hi = row_hi(s, sp, w_first), all_lo = row_lo(s, sp, w_last);
        const int any_hi = row_hi(s, sp, w_last), any_lo = row_lo(s, sp, w_first);
        const float c = s.scale * LOG2E;
        const RowRead<DP, T> rows(lane);
        const TileLoad<DP, QT, NW> tq(q.row, (int)s.head_dim / 8 - 1, wave, lane);
        const int per = (r1 - r0 + QT - 1) / QT, count = per * (int)group;
        const T *gq = (const T *)q.data + (int64_t)b * q.batch + (int64_t)kvh * group * q.head;
        const float *gs = lse + ((int64_t)b * s.q_heads + (int64_t)kvh * group) * s.q_len;
        int next = r0;
        auto issue = [&](int to) {
            tq.issue(lq[to], gq, next, sp.ql - 1, wave);
            if (wave == 0 && lane < QT) {
                const float x = gs[min(next + lane, sp.ql - 1)];
                lst[to][lane] = x == -ATTN_INF ? ATTN_INF : x * LOG2E;
            }
            next += QT;
            if (next >= r1) next = r0, gq += q.head, gs += s.q_len;
        };
        issue(0);
        int buf = 0, qt = r0;
        for (int n = 0; n < count; ++n, buf ^= 1) {
            tiles_arrive();
            if (n + 1 < count) issue(buf ^ 1);
            const int at = qt;
            qt = qt + QT >= r1 ? r0 : qt + QT;
            if (at >= any_hi || at + QT <= any_lo) continue;
            f32x16 x = {};
#pragma unroll
            for (int d = 0; d < DP / 16; ++d) x = Elem<T>::mfma(rows.get(lq[buf], 0, d), kf[d], x);
            float p[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) p[i] = exp2_fast(__builtin_fmaf(x[i], c, -lst[buf][8 * (i / 4) + 4 * (lane >> 5) + i % 4]));
            if (at + QT > all_hi || at < all_lo) {
                const int row0 = at + 4 * (lane >> 5);
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const int row = row0 + 8 * (i / 4) + i % 4;
                    p[i] = row < hi && row >= lo ? p[i] : 0.f;
                }
            }
            // the tile's own sum first: 16 small terms at a time lose less in a long one
            float part = 0.f;
#pragma unroll
            for (int i = 0; i < 16; ++i) part += p[i];
            sum += part;
        }
    }
    sum = half_sum(sum);
    if (key < (int)s.k_len && lane < 32) {
        const int64_t at = ((int64_t)b * s.kv_heads + kvh) * s.k_len + key;
        weights[at] = (before ? before[at] : 0.f) + (key < sp.kl ? sum : 0.f);
    }
}

template <class T, int DP>
hipError_t launch(const AttnShape &s, const Rows &q, const Rows &k, const float *lse, const float *before, float *weights, hipStream_t st)
{
    constexpr int NW = 4;
    const uint32_t tiles = (s.k_len + 32 * NW - 1) / (32 * NW), total = s.batch * s.kv_heads * tiles;
    k_attention_weights<T, DP, NW><<<(total + 7) / 8 * 8, NW * 64, 0, st>>>(s, q, k, lse, before, weights, tiles);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_weights(const AttnShape &s, const Rows &q, const Rows &k, const float *lse, const float *before, float *weights,
                                    hipStream_t st)
{
    if (s.half)
        return s.head_dim <= 64 ? launch<_Float16, 64>(s, q, k, lse, before, weights, st) : launch<_Float16, 128>(s, q, k, lse, before, weights, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, q, k, lse, before, weights, st) : launch<__bf16, 128>(s, q, k, lse, before, weights, st);
}

}  // namespace lap
