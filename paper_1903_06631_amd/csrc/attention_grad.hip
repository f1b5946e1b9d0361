// Attention's backward pass.  With p_ij = exp(scale q_i.k_j - lse_i) computed again from the rows and the forward pass's
// sums, g_i the gradient of o_i and delta_i = g_i.o_i:
//   dv_j = sum_i p_ij g_i      ds_ij = p_ij (g_i.v_j - delta_i)      dq_i = scale sum_j ds_ij k_j      dk_j = scale sum_i ds_ij q_i
// p and ds are rounded to the rows' type where they enter a product, which is what the matrix instruction takes (in binary16 as
// multiples of a power of two: hold_in_range); scores, g.v, p and ds themselves and all sums are 32 bits.
//
// Two kernels, each with its sums in registers from the first product to the last, added in a fixed order: one keeps
// query rows and streams keys (dq; it also leaves delta and the sums in base 2 in the workspace), the other keeps keys and
// streams the rows of every query head that shares them (dk and dv).  Scores and g.v are computed in both, seven products
// in place of five: the price for results that do not depend on the order in which workgroups finish.  Where there are few
// keys and many rows, the second kernel's rows are cut into parts, whose sums a third adds in order.
//
// Measured, 8 x 16 heads x 2048 tokens x 128, causal, bfloat16: 228 + 313 us = 635 TFLOP/s of the five products that a backward
// pass cannot do without (890 of the seven), the matrix units busy in 44 % of the cycles at 2.0 GHz.  6 ragged sequences of up to
// 1001 tokens x 80, 12 heads on 4, binary16: 36 + 59 us, with the compute units busy in 48 % of the cycles: bound by the longest
// workgroup's chain of tiles, a third of whose products are of the padding to 128 elements.
#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attn_core.h"

namespace lap {
namespace {

// QW blocks of 32 rows, the keys of each dealt to KG waves, a block of 32 at a time of KT
template <class T, int DP, int QW, int KG, int KT>
__global__ __launch_bounds__(QW * KG * 64, 2) void k_attention_dq(AttnShape s, Rows g, Rows q, Rows k, Rows v, Rows o, const float *lse,
                                                          Rows dq, float *stats, uint32_t tiles)
{
    constexpr int NW = QW * KG, BQ = 32 * QW;
    __shared__ __align__(16) T tiles_kv[4][Tile<DP>::size(KT)];
    T(*const lk)[Tile<DP>::size(KT)] = tiles_kv, (*const lv)[Tile<DP>::size(KT)] = tiles_kv + 2;
    const uint32_t group = s.q_heads / s.kv_heads;
    Work wk;
    if (!work_item(s, group, wk)) return;
    const uint32_t b = wk.b, kvh = wk.kvh, h = kvh * group + wk.g;
    const int first = (int)(tiles - 1 - wk.tile) * BQ;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span sp = span_of(s, b);

    const int qw = wave % QW, kg = wave / QW;
    const int w0 = first + 32 * qw;
    const int row = w0 + (lane & 31);
    T *drow = (T *)dq.data + (int64_t)b * dq.batch + (int64_t)h * dq.head + (int64_t)row * dq.row;
    const int64_t at = ((int64_t)b * s.q_heads + h) * s.q_len;

    __shared__ int again;
    if (threadIdx.x == 0) again = 0;
    f32x16 acc[DP / 32] = {};
    const int end = min(first + BQ, sp.ql);
    const int k0 = first < sp.ql ? key_lo(s, sp, first) / KT * KT : 0;
    const int k1 = first < sp.ql ? key_hi(s, sp, end - 1) : 0;
    if (first < sp.ql) {
        const int used = min(row, sp.ql - 1);
        typename Elem<T>::x8 qf[DP / 16], gf[DP / 16];
        load_kept<DP>(qf, (const T *)q.data + (int64_t)b * q.batch + (int64_t)h * q.head + (int64_t)used * q.row, s.head_dim, lane);
        load_kept<DP>(gf, (const T *)g.data + (int64_t)b * g.batch + (int64_t)h * g.head + (int64_t)used * g.row, s.head_dim, lane);
        float delta = 0.f;
        {
            typename Elem<T>::x8 of[DP / 16];
            load_kept<DP>(of, (const T *)o.data + (int64_t)b * o.batch + (int64_t)h * o.head + (int64_t)used * o.row, s.head_dim, lane);
#pragma unroll
            for (int d = 0; d < DP / 16; ++d)
#pragma unroll
                for (int j = 0; j < 8; ++j) delta = __builtin_fmaf((float)gf[d][j], (float)of[d][j], delta);
            delta = half_sum(delta);
        }
        // a row without keys gets probabilities of zero
        const float sum = lse[at + used], l2 = sum == -ATTN_INF ? ATTN_INF : sum * LOG2E;
        if (row < sp.ql && lane < 32 && kg == 0) {
            stats[at + row] = IS_F16<T> ? l2 - P16 : l2;      // probabilities times 2^P16 in the second kernel
            stats[(int64_t)s.batch * s.q_heads * s.q_len + at + row] = IS_F16<T> ? -delta : delta;      // there the second kernel's sums start with it
        }

        if (k0 < k1) {
            const int hi = key_hi(s, sp, used), lo = key_lo(s, sp, used);
            const int w_last = min(w0 + 31, sp.ql - 1), w_first = min(w0, sp.ql - 1);
            const int all_hi = key_hi(s, sp, w_first), all_lo = key_lo(s, sp, w_last);
            const int any_hi = key_hi(s, sp, w_last), any_lo = key_lo(s, sp, w_first);
            const float c = s.scale * LOG2E;
            const T *gk = (const T *)k.data + (int64_t)b * k.batch + (int64_t)kvh * k.head;
            const T *gv = (const T *)v.data + (int64_t)b * v.batch + (int64_t)kvh * v.head;
            const int last_chunk = (int)s.head_dim / 8 - 1;
            const RowRead<DP, T> rows(lane);
            const ColRead<DP, T> cols(lane);
            const TileLoad<DP, KT, NW> tk(k.row, last_chunk, wave, lane), tv(v.row, last_chunk, wave, lane);
            float f;      // what z and ds are multiplied by, in binary16
            zero_tiles<DP, NW * 64>(tiles_kv[0], sizeof(tiles_kv) / sizeof(T), s.head_dim);
            const auto pass = [&](auto careful) {
                constexpr bool care = decltype(careful)::value;
                bool odd = false;      // blocks have been left out
                f = IS_F16<T> ? FIRST_F : 1.f;
                tk.issue(lk[0], gk, k0, sp.kl - 1, wave);
                tv.issue(lv[0], gv, k0, sp.kl - 1, wave);
                int buf = 0;
                for (int kt = k0; kt < k1; kt += KT, buf ^= 1) {
                    tiles_arrive();
                    if (kt + KT < k1) {
                        tk.issue(lk[buf ^ 1], gk, kt + KT, sp.kl - 1, wave);
                        tv.issue(lv[buf ^ 1], gv, kt + KT, sp.kl - 1, wave);
                    }
#pragma unroll
                    for (int n = 0; n < KT / 32 / KG; ++n) {
                        const int kb = KT / 32 / KG * kg + n, at = kt + 32 * kb;
                        if (at >= any_hi || at + 32 <= any_lo) continue;
                        f32x16 x = {}, y = {};
#pragma unroll
                        for (int d = 0; d < DP / 16; ++d) x = Elem<T>::mfma(rows.get(lk[buf], kb, d), qf[d], x);
#pragma unroll
                        for (int d = 0; d < DP / 16; ++d) y = Elem<T>::mfma(rows.get(lv[buf], kb, d), gf[d], y);
                        const bool part = at + 32 > all_hi || at < all_lo;
                        const int key0 = at + 4 * (lane >> 5);
                        float z[16], ds[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) z[i] = IS_F16<T> ? __builtin_fmaf(y[i], f, -delta * f) : y[i] - delta;
                        if constexpr (IS_F16<T>) {
                            if (part)
#pragma unroll
                                for (int i = 0; i < 16; ++i) {
                                    const int key = key0 + 8 * (i / 4) + i % 4;
                                    z[i] = key < hi && key >= lo ? z[i] : 0.f;
                                }
                            hold_in_range<15>(z, f, acc);
                        }
#pragma unroll
                        for (int i = 0; i < 16; ++i) ds[i] = exp2_fast(__builtin_fmaf(x[i], c, -l2)) * z[i];
                        if (part) {
#pragma unroll
                            for (int i = 0; i < 16; ++i) {
                                const int key = key0 + 8 * (i / 4) + i % 4;
                                ds[i] = key < hi && key >= lo ? ds[i] : 0.f;
                            }
                            if (care && !block_is_finite<DP>(lk[buf], kb, lane)) {
                                odd = true;
                                continue;
                            }
                        }
#pragma unroll
                        for (int t = 0; t < 2; ++t) {
                            const auto df = round8<T>(ds, 8 * t);
#pragma unroll
                            for (int d = 0; d < DP / 32; ++d) acc[d] = Elem<T>::mfma(cols.get(lk[buf], 2 * kb + t, d), df, acc[d]);
                        }
                    }
                }
                if constexpr (care) {
                    if (!odd) return;
                    const T *const qrow = (const T *)q.data + (int64_t)b * q.batch + (int64_t)h * q.head + (int64_t)used * q.row;
                    const T *const grow = (const T *)g.data + (int64_t)b * g.batch + (int64_t)h * g.head + (int64_t)used * g.row;
#pragma unroll 1
                    for (int kt = k0; kt < k1; kt += KT)
#pragma unroll 1
                        for (int n = 0; n < KT / 32 / KG; ++n) {
                            const int at = kt + 32 * (KT / 32 / KG * kg + n);
                            if (at >= any_hi || at + 32 <= any_lo || (at + 32 <= all_hi && at >= all_lo)) continue;
                            if (rows_are_finite(gk, k.row, at, sp.kl - 1, s.head_dim, lane)) continue;
#pragma unroll 1
                            for (int key = max(at, lo); key < min(at + 32, hi); ++key) {
                                const T *const krow = gk + (int64_t)key * k.row;
                                const float p = exp2_fast(__builtin_fmaf(dot(qrow, krow, s.head_dim), c, -l2));
                                add_row<DP>(acc, krow, p * ((dot(grow, gv + (int64_t)key * v.row, s.head_dim) - delta) * f), s.head_dim, lane);
                            }
                        }
                }
            };
            pass(std::false_type());
            if (!sums_are_numbers(acc) && lane == 0) again = 1;
            __syncthreads();
            if (again) {
#pragma unroll
                for (int d = 0; d < DP / 32; ++d) acc[d] = f32x16{};
                pass(std::true_type());
            }
            if constexpr (IS_F16<T>) times(acc, 1.f / f);
        }
    }
    if constexpr (KG > 1) {
        static_assert((KG - 1) * QW * DP / 2 * 64 * sizeof(float) <= sizeof(tiles_kv), "the sums fit where the tiles were");
        float *const box = (float *)tiles_kv + qw * (DP / 2 * 64);
        __syncthreads();
        if (kg > 0) put_sums(box + (kg - 1) * QW * (DP / 2 * 64), acc, lane);
        __syncthreads();
        if (kg > 0) return;
#pragma unroll
        for (int n = 1; n < KG; ++n) add_sums(box + (n - 1) * QW * (DP / 2 * 64), acc, 1.f, lane);
    }
    if (row < (int)s.q_len) {
        if (row >= sp.ql)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) acc[d] = f32x16{};
        store_kept<DP>(drow, acc, s.scale, s.head_dim, lane);
    }
}

// KW blocks of 32 keys, the rows of each dealt to RG waves, a block of 32 at a time
template <class T, int DP, int KW, int RG>
__global__ __launch_bounds__(KW * RG * 64, 2) void k_attention_dkv(AttnShape s, Rows g, Rows q, Rows k, Rows v, const float *stats, Rows dk,
                                                                Rows dv, uint32_t parts, float *sums)
{
    constexpr int NW = KW * RG, BK = 32 * KW, QT = 32 * RG;
    __shared__ __align__(16) T tiles_qg[4][Tile<DP>::size(QT)];
    T(*const lq)[Tile<DP>::size(QT)] = tiles_qg, (*const lg)[Tile<DP>::size(QT)] = tiles_qg + 2;
    // The values of the kept rows are read from here: in registers they and the sums of two waves on a SIMD do not fit, and
    // what the compiler then keeps in memory has to be waited for together with the next tile (8 x 16 heads x 2048 tokens x
    // 128: both passes 566 us; with 26 registers in memory 753, with one wave on a SIMD 668).
    __shared__ __align__(16) T lkept[Tile<DP>::size(BK)];
    constexpr int PARTS = (QT + 63) / 64;      // a wave fetches the numbers of 64 rows at once
    __shared__ __align__(16) float lst[2][2][64 * PARTS];
    Work wk;
    if (!work_item(s, RG > 2 ? parts : 1, wk)) return;
    const uint32_t b = wk.b, kvh = wk.kvh;
    const int first = (int)wk.tile * BK;      // the first keys of a causal head are seen by the most rows
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span sp = span_of(s, b);
    const uint32_t group = s.q_heads / s.kv_heads;

    const int kw = wave % KW, rg = wave / KW;
    const int w0 = first + 32 * kw;
    const int key = w0 + (lane & 31);
    __shared__ int again;
    if (threadIdx.x == 0) again = 0;
    f32x16 ak[DP / 32] = {}, av[DP / 32] = {};
    const int end = min(first + BK, sp.kl);
    const int r0 = first < sp.kl ? row_lo(s, sp, first) / QT * QT : 0;
    const int r1 = first < sp.kl ? row_hi(s, sp, end - 1) : 0;
    const int per = r0 < r1 ? (r1 - r0 + QT - 1) / QT : 0;      // tiles of a head, of which this part takes n0 .. n1 - 1
    int n0 = 0, n1 = per * (int)group, head0 = (int)(kvh * group), begin = r0;
    if constexpr (RG > 2) {      // (the few workgroups of the others are enough)
        n0 = uniform((int)((int64_t)n1 * wk.g / parts)), n1 = uniform((int)((int64_t)n1 * (wk.g + 1) / parts));
        if (per) head0 = uniform(head0 + n0 / per), begin = uniform(r0 + n0 % per * QT);
    }
    if (n0 < n1) {
        const int used = min(key, sp.kl - 1);
        typename Elem<T>::x8 kf[DP / 16];
        load_kept<DP>(kf, (const T *)v.data + (int64_t)b * v.batch + (int64_t)kvh * v.head + (int64_t)used * v.row, s.head_dim, lane);
        if (rg == 0) keep_in_lds<DP>(lkept, kw, kf, lane);
        load_kept<DP>(kf, (const T *)k.data + (int64_t)b * k.batch + (int64_t)kvh * k.head + (int64_t)used * k.row, s.head_dim, lane);
        const int hi = row_hi(s, sp, used), lo = row_lo(s, sp, used);
        const int w_last = min(w0 + 31, sp.kl - 1), w_first = min(w0, sp.kl - 1);
        const int all_hi = row_hi(s, sp, w_first), all_lo = row_lo(s, sp, w_last);
        const int any_hi = row_hi(s, sp, w_last), any_lo = row_lo(s, sp, w_first);
        const float c = s.scale * LOG2E;
        const int last_chunk = (int)s.head_dim / 8 - 1;
        const RowRead<DP, T> rows(lane);
        const ColRead<DP, T> cols(lane);
        const TileLoad<DP, QT, NW> tq(q.row, last_chunk, wave, lane), tg(g.row, last_chunk, wave, lane);
        const int64_t to_delta = (int64_t)s.batch * s.q_heads * s.q_len;
        zero_tiles<DP, NW * 64>(tiles_qg[0], sizeof(tiles_qg) / sizeof(T), s.head_dim);
        float f;      // what z and ds are multiplied by, in binary16 (ds beside the 2^P16 of its probability)
        const auto pass = [&](auto careful) {
            constexpr bool care = decltype(careful)::value;
            bool odd = false;      // blocks have been left out
            f = IS_F16<T> ? FIRST_F : 1.f;
            const T *gq = (const T *)q.data + (int64_t)b * q.batch + head0 * q.head;
            const T *gg = (const T *)g.data + (int64_t)b * g.batch + head0 * g.head;
            const float *gs = stats + ((int64_t)b * s.q_heads + head0) * s.q_len;
            int next = begin;      // rows and head of the next tile to ask for
            const auto issue = [&](int to) {
                tq.issue(lq[to], gq, next, sp.ql - 1, wave);
                tg.issue(lg[to], gg, next, sp.ql - 1, wave);
                if (wave < 2 * PARTS) load_floats(lst[to][wave / PARTS], gs + wave / PARTS * to_delta, next, sp.ql - 1, wave % PARTS, lane);
                next += QT;
                if (next >= r1) next = r0, gq += q.head, gg += g.head, gs += s.q_len;
            };
            int buf = 0, qt = next;
            issue(0);
            for (int n = n0; n < n1; ++n, buf ^= 1) {
                tiles_arrive();
                if (n + 1 < n1) issue(buf ^ 1);
                const int tile = qt;
                qt = qt + QT >= r1 ? r0 : qt + QT;
                const int at = tile + 32 * rg;
                if (at >= any_hi || at + 32 <= any_lo) continue;
                const float *const l2 = lst[buf][0] + 32 * rg + 4 * (lane >> 5), *const delta = lst[buf][1] + 32 * rg + 4 * (lane >> 5);
                f32x16 x = {}, y = {};
                if constexpr (IS_F16<T>)      // (minus delta there: the difference comes out of the product)
#pragma unroll
                    for (int i = 0; i < 16; ++i) y[i] = delta[8 * (i / 4) + i % 4];
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) x = Elem<T>::mfma(rows.get(lq[buf], rg, d), kf[d], x);
#pragma unroll
                for (int d = 0; d < DP / 16; ++d) y = Elem<T>::mfma(rows.get(lg[buf], rg, d), rows.get(lkept, kw, d), y);
                const bool part = at + 32 > all_hi || at < all_lo;
                const int row0 = at + 4 * (lane >> 5);
                float z[16], p[16], ds[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) z[i] = IS_F16<T> ? y[i] * f : y[i] - delta[8 * (i / 4) + i % 4];
                if constexpr (IS_F16<T>) {
                    if (part)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int row = row0 + 8 * (i / 4) + i % 4;
                            z[i] = row < hi && row >= lo ? z[i] : 0.f;
                        }
                    hold_in_range<15 - P16>(z, f, ak);
                }
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    p[i] = exp2_fast(__builtin_fmaf(x[i], c, -l2[8 * (i / 4) + i % 4]));
                    ds[i] = p[i] * z[i];
                }
                if (part) {
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const int row = row0 + 8 * (i / 4) + i % 4;
                        const bool in = row < hi && row >= lo;
                        p[i] = in ? p[i] : 0.f;
                        ds[i] = in ? ds[i] : 0.f;
                    }
                    if (care && (!block_is_finite<DP>(lq[buf], rg, lane) || !block_is_finite<DP>(lg[buf], rg, lane))) {
                        odd = true;
                        continue;
                    }
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const auto pf = round8<T>(p, 8 * t), df = round8<T>(ds, 8 * t);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) {
                        av[d] = Elem<T>::mfma(cols.get(lg[buf], 2 * rg + t, d), pf, av[d]);
                        ak[d] = Elem<T>::mfma(cols.get(lq[buf], 2 * rg + t, d), df, ak[d]);
                    }
                }
            }
            if constexpr (care) {
                if (!odd) return;
                const T *const krow = (const T *)k.data + (int64_t)b * k.batch + (int64_t)kvh * k.head + (int64_t)used * k.row;
                const T *const vrow = (const T *)v.data + (int64_t)b * v.batch + (int64_t)kvh * v.head + (int64_t)used * v.row;
#pragma unroll 1
                for (int n = n0; n < n1; ++n) {
                    const int at = r0 + n % per * QT + 32 * rg;
                    if (at >= any_hi || at + 32 <= any_lo || (at + 32 <= all_hi && at >= all_lo)) continue;
                    const int64_t head = (int64_t)kvh * group + n / per;
                    const T *const q0 = (const T *)q.data + (int64_t)b * q.batch + head * q.head;
                    const T *const g0 = (const T *)g.data + (int64_t)b * g.batch + head * g.head;
                    const float *const st = stats + ((int64_t)b * s.q_heads + head) * s.q_len;
                    if (rows_are_finite(q0, q.row, at, sp.ql - 1, s.head_dim, lane) && rows_are_finite(g0, g.row, at, sp.ql - 1, s.head_dim, lane)) continue;
#pragma unroll 1
                    for (int row = max(at, lo); row < min(at + 32, hi); ++row) {
                        const T *const qrow = q0 + (int64_t)row * q.row, *const grow = g0 + (int64_t)row * g.row;
                        const float p = exp2_fast(__builtin_fmaf(dot(qrow, krow, s.head_dim), c, -st[row]));
                        add_row<DP>(av, grow, p, s.head_dim, lane);
                        add_row<DP>(ak, qrow, p * ((dot(grow, vrow, s.head_dim) - (IS_F16<T> ? -st[to_delta + row] : st[to_delta + row])) * f), s.head_dim, lane);
                    }
                }
            }
        };
        pass(std::false_type());
        if (!(sums_are_numbers(ak) && sums_are_numbers(av)) && lane == 0) again = 1;
        __syncthreads();
        if (again) {
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) ak[d] = av[d] = f32x16{};
            pass(std::true_type());
        }
        if constexpr (IS_F16<T>) times(av, 1.f / (1 << P16)), times(ak, 1.f / (1 << P16) / f);
    }
    if constexpr (RG > 1) {
        static_assert((RG - 1) * KW * DP / 2 * 64 * sizeof(float) <= sizeof(tiles_qg), "the sums fit where the tiles were");
        float *const box = (float *)tiles_qg + kw * (DP / 2 * 64);
        __syncthreads();
        if (rg > 0) put_sums(box + (rg - 1) * KW * (DP / 2 * 64), ak, lane);
        __syncthreads();
        if (rg == 0)
#pragma unroll
            for (int n = 1; n < RG; ++n) add_sums(box + (n - 1) * KW * (DP / 2 * 64), ak, 1.f, lane);
        __syncthreads();
        if (rg > 0) put_sums(box + (rg - 1) * KW * (DP / 2 * 64), av, lane);
        __syncthreads();
        if (rg > 0) return;
#pragma unroll
        for (int n = 1; n < RG; ++n) add_sums(box + (n - 1) * KW * (DP / 2 * 64), av, 1.f, lane);
    }
    if (RG > 2 && parts > 1) {      // [part][batch, kv_heads, k_len][dk, dv][DP]
        if (key >= sp.kl) return;
        float *to = sums + (((int64_t)wk.g * s.batch * s.kv_heads + (int64_t)b * s.kv_heads + kvh) * s.k_len + key) * 2 * DP + 4 * (lane >> 5);
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4) {
                *(f32x4 *)(to + 32 * d + 2 * i) = f32x4{ak[d][i], ak[d][i + 1], ak[d][i + 2], ak[d][i + 3]};
                *(f32x4 *)(to + DP + 32 * d + 2 * i) = f32x4{av[d][i], av[d][i + 1], av[d][i + 2], av[d][i + 3]};
            }
        return;
    }
    if (key < (int)s.k_len) {
        if (key >= sp.kl)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) ak[d] = av[d] = f32x16{};
        store_kept<DP>((T *)dk.data + (int64_t)b * dk.batch + (int64_t)kvh * dk.head + (int64_t)key * dk.row, ak, s.scale, s.head_dim, lane);
        store_kept<DP>((T *)dv.data + (int64_t)b * dv.batch + (int64_t)kvh * dv.head + (int64_t)key * dv.row, av, 1.f, s.head_dim, lane);
    }
}

// Eight elements of a key's dk or dv for each thread: the parts in order, rounded once.
template <class T, int DP> __global__ __launch_bounds__(256) void k_dkv_join(AttnShape s, Rows dk, Rows dv, uint32_t parts, const float *sums)
{
    constexpr int ACROSS = 2 * DP / 8;
    const int64_t at = (int64_t)blockIdx.x * (256 / ACROSS) + threadIdx.x / ACROSS, all = (int64_t)s.batch * s.kv_heads * s.k_len;
    if (at >= all) return;
    const uint32_t e = threadIdx.x % ACROSS * 8 % DP, key = (uint32_t)(at % s.k_len);
    const bool second = threadIdx.x % ACROSS >= DP / 8;
    const uint32_t h = (uint32_t)(at / s.k_len % s.kv_heads), b = (uint32_t)(at / s.k_len / s.kv_heads);
    if (e >= s.head_dim) return;
    f32x4 y[2] = {};
    if ((int)key < span_of(s, b).kl) {
        const f32x4 *from = (const f32x4 *)(sums + (at * 2 + second) * DP + e);
        for (uint32_t i = 0; i < parts; ++i, from += all * 2 * DP / 4) y[0] += from[0], y[1] += from[1];
    }
    const float by = second ? 1.f : s.scale;
    typename Elem<T>::x8 z;
#pragma unroll
    for (int j = 0; j < 8; ++j) z[j] = (T)(y[j / 4][j % 4] * by);
    const Rows &to = second ? dv : dk;
    *(typename Elem<T>::x8 *)((T *)to.data + (int64_t)b * to.batch + (int64_t)h * to.head + (int64_t)key * to.row + e) = z;
}

template <class T, int DP, int QW, int KG, int KT> hipError_t launch_dq(const AttnShape &s, const AttnGrad &a, hipStream_t st)
{
    const uint32_t tiles = (s.q_len + 32 * QW - 1) / (32 * QW);
    const uint32_t total = padded_caches(s.batch * s.kv_heads) * (s.q_heads / s.kv_heads) * tiles;
    k_attention_dq<T, DP, QW, KG, KT><<<total, QW * KG * 64, 0, st>>>(s, a.g, a.q, a.k, a.v, a.out, a.lse, a.dq, a.stats, tiles);
    return hipGetLastError();
}
template <class T, int DP, int KW, int RG> hipError_t launch_dkv(const AttnShape &s, const AttnGrad &a, hipStream_t st)
{
    const uint32_t tiles = (s.k_len + 32 * KW - 1) / (32 * KW), parts = grad_parts(s), total = padded_caches(s.batch * s.kv_heads) * tiles * parts;
    k_attention_dkv<T, DP, KW, RG><<<total, KW * RG * 64, 0, st>>>(s, a.g, a.q, a.k, a.v, a.stats, a.dk, a.dv, parts, a.sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    const uint64_t rows = (uint64_t)s.batch * s.kv_heads * s.k_len, per = 256 / (2 * DP / 8);
    k_dkv_join<T, DP><<<(uint32_t)((rows + per - 1) / per), 256, 0, st>>>(s, a.dk, a.dv, parts, a.sums);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t launch(const AttnShape &s, const AttnGrad &a, hipStream_t st)
{
    if (s.q_len) {
        const Share share = share_of(s, s.q_heads, s.q_len);
        const hipError_t e = share == Share::FOUR ? launch_dq<T, DP, 4, 1, 64>(s, a, st) : share == Share::FOUR_BY_TWO ? launch_dq<T, DP, 4, 2, 64>(s, a, st)
                                                                                                                         : launch_dq<T, DP, 2, 4, 128>(s, a, st);
        if (e != hipSuccess) return e;
    }
    if (!s.k_len) return hipSuccess;
    const Share share = share_of(s, s.kv_heads, s.k_len);
    return share == Share::FOUR ? launch_dkv<T, DP, 4, 1>(s, a, st) : share == Share::FOUR_BY_TWO ? launch_dkv<T, DP, 4, 2>(s, a, st) : launch_dkv<T, DP, 2, 4>(s, a, st);
}

}  // namespace

// Parts of the rows that the second kernel streams: where there are few keys and many rows (query heads that share a key
// head are rows too), the number that ends first by this estimate, in us: a workgroup's 64 keys take 2.2 for each 128
// rows, 256 workgroups at a time; under a causal mask half of that on the average, the longest first; every part's sums are
// written and read once at 5 TB/s, by a kernel more.  Backward passes, causal, 8 heads on one x 2048 tokens 80 us (in one part
// 255), 16 on 2 x 4096 tokens 274 (542); all keys visible, 2 sequences of 5013 tokens, 4 heads on one 444 (469).
uint32_t grad_parts(const AttnShape &s)
{
    if (!s.k_len || !s.q_len || share_of(s, s.kv_heads, s.k_len) != Share::TWO_BY_FOUR) return 1;
    const double groups = (double)s.batch * s.kv_heads * ((s.k_len + 63) / 64), rows = (double)(s.q_heads / s.kv_heads) * s.q_len;
    const double whole = rows / 128 * 2.2, sums = groups * 64 * 2 * (s.head_dim <= 64 ? 64 : 128) * 8 / 5e6;
    uint32_t best = 1;
    double least = 0;
    for (uint32_t p = 1; p <= 16 && (p == 1 || rows / p >= 512); ++p) {
        const double time = (s.causal ? std::max(groups * whole / 512, whole / p) : std::ceil(groups * p / 256) * whole / p) + (p > 1 ? 6 + p * sums : 0);
        if (p == 1 || time < least) best = p, least = time;
    }
    return best;
}
size_t grad_sums(const AttnShape &s)
{
    const uint32_t parts = grad_parts(s);
    return parts == 1 ? 0 : (size_t)parts * s.batch * s.kv_heads * s.k_len * 2 * (s.head_dim <= 64 ? 64 : 128) * sizeof(float);
}

hipError_t launch_attention_grad(const AttnShape &s, const AttnGrad &a, hipStream_t st)
{
    if (s.half) return s.head_dim <= 64 ? launch<_Float16, 64>(s, a, st) : launch<_Float16, 128>(s, a, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, a, st) : launch<__bf16, 128>(s, a, st);
}

}  // namespace lap
