// Attention of a training step or a prompt: o_i = sum_j p_ij v_j, p_ij = exp(scale q_i.k_j - lse_i), lse_i = the logarithm
// of the sum of exp(scale q_i.k_j) over the keys that row i sees.
//
// One pass over the keys with a running maximum m and sum l for every row: a tile of keys gives s = K Q^T, p = 2^(c s - c m)
// with c = scale log2(e), l += sum p, O^T += V^T P^T.  The matrix instruction takes p in the values' type: each is off by half a
// unit of that at most, as each value is already, and a product of 32-bit operands runs at a sixteenth of the rate; l is the sum
// of the unrounded ones, so that lse has 32 bits.  Nothing of the size queries x keys is ever stored.  Where there are few
// rows and many keys, the keys are cut into parts, a workgroup each, which leave m, l and O in the workspace for a second
// kernel to join.
//
// A wave keeps 32 rows and their outputs in registers; four waves share tiles of keys and values in LDS, fetched while the
// tile before is worked on.  For 32 rows and 64 keys of 128 elements a wave has 32 products of 32 cycles and 230 vector
// instructions of 4 (exponentials 8); two or three waves on a SIMD overlap the two in part.  Measured: 32 heads x 12345 rows on
// 13370 keys, causal, 1.36 ms = 1070 TFLOP/s, 88 % of what a large matrix product reaches on the same card, with the matrix
// unit busy in 60 % of the cycles and the clock down to 1.7 GHz: bound by power, and other orders of the instructions (scores
// of the next tile worked out beside the exponentials, products and vector instructions dealt out by hand) came out within
// 3 % or worse.  Shorter rows are slower, causal ones most (16 heads of 128 elements, TFLOP/s of the visible pairs):
//   tokens       8 x 1024   8 x 2048   8 x 4096   4 x 8192   1 x 16384
//   causal            608        866        941       1042        1064
//   all keys          826        989       1007       1076        1069
// Starts and ends of workgroups are what shorter rows without a mask lose.  Causal ones lose 12 % more at 2048 tokens: 6 % are the
// diagonal's hidden pairs and the waves that wait for the last of four there, the rest is not accounted for.
#include <type_traits>

#include "attn_core.h"

namespace lap {
namespace {

// What probabilities are multiplied by, in base 2: they are taken from a maximum that may be passed by 2^8 (below), and in
// binary16 all that are below 2^-25 of it would be nothing (400 000 keys at 2^-25.5 beside one at 1: 0.8 % of the row).
template <class T> constexpr float SHIFT = __is_same(T, _Float16) ? 7.f : 0.f;

// QW blocks of 32 rows; their keys are dealt to KG waves each, NB blocks of 32 keys at a time.  Where rows are few, waves that
// share them fill the units that would have none; they join their sums at the end.
template <class T, int DP, int QW, int KG, int NB>
__global__ __launch_bounds__(QW * KG * 64, NB == 1 && KG == 1 ? 3 : 2) void k_attention(AttnShape s, Rows q, Rows k, Rows v, Rows o, float *lse, uint32_t tiles,
                                                                     uint32_t parts, float *outs, float2 *out_sums)
{
    constexpr int NW = QW * KG, BQ = 32 * QW, KT = 32 * KG * NB;
    __shared__ __align__(16) T tiles_kv[4][Tile<DP>::size(KT)];
    T(*const lk)[Tile<DP>::size(KT)] = tiles_kv, (*const lv)[Tile<DP>::size(KT)] = tiles_kv + 2;
    const uint32_t group = s.q_heads / s.kv_heads;
    Work wk;
    if (!work_item(s, group * parts, wk)) return;
    const uint32_t b = wk.b, h = wk.kvh * group + wk.g % group, part = wk.g / group;
    const int first = (int)(tiles - 1 - wk.tile) * BQ;      // the longest rows of a causal head first
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const Span sp = span_of(s, b);

    const int qw = wave % QW, kg = wave / QW;
    const int w0 = first + 32 * qw;                 // this wave's rows
    const int row = w0 + (lane & 31);
    T *orow = (T *)o.data + (int64_t)b * o.batch + (int64_t)h * o.head + (int64_t)row * o.row;
    float *lrow = lse + ((int64_t)b * s.q_heads + h) * s.q_len + row;

    f32x16 acc[DP / 32];
    float m, l;
    __shared__ int again;
    if (threadIdx.x == 0) again = 0;
    const auto clear = [&] {
        m = LOWEST, l = 0.f;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d) acc[d] = f32x16{};
    };
    clear();
    const int end = min(first + BQ, sp.ql);         // rows in use
    int k0 = first < sp.ql ? key_lo(s, sp, first) / KT * KT : 0;
    int k1 = first < sp.ql ? key_hi(s, sp, end - 1) : 0;
    if (parts > 1 && k0 < k1) {      // this part's share of the tiles
        const int64_t n = (k1 - k0 + KT - 1) / KT;
        k1 = uniform(min(k1, k0 + (int)(n * (part + 1) / parts) * KT));
        k0 = uniform(k0 + (int)(n * part / parts) * KT);
    }
    if (k0 < k1) {
        zero_tiles<DP, NW * 64>(tiles_kv[0], sizeof(tiles_kv) / sizeof(T), s.head_dim);
        const int used = min(row, sp.ql - 1);       // padding takes the last row's part and is thrown away
        const int last_chunk = (int)s.head_dim / 8 - 1, last = sp.kl - 1;
        const T *gk = (const T *)k.data + (int64_t)b * k.batch + (int64_t)wk.kvh * k.head;
        const T *gv = (const T *)v.data + (int64_t)b * v.batch + (int64_t)wk.kvh * v.head;
        const TileLoad<DP, KT, NW> tk(k.row, last_chunk, wave, lane), tv(v.row, last_chunk, wave, lane);
        typename Elem<T>::x8 qf[DP / 16];
        load_kept<DP>(qf, (const T *)q.data + (int64_t)b * q.batch + (int64_t)h * q.head + (int64_t)used * q.row, s.head_dim, lane);
        const int hi = key_hi(s, sp, used), lo = key_lo(s, sp, used);
        const int w_last = min(w0 + 31, sp.ql - 1), w_first = min(w0, sp.ql - 1);
        const int all_hi = key_hi(s, sp, w_first), all_lo = key_lo(s, sp, w_last);      // every row of the wave sees these
        const int any_hi = key_hi(s, sp, w_last), any_lo = key_lo(s, sp, w_first);      // and some row these
        const float c = s.scale * LOG2E;
        const RowRead<DP, T> rows(lane);
        const ColRead<DP, T> cols(lane);

        const auto pass = [&](auto careful) {
            constexpr bool care = decltype(careful)::value;
            bool odd = false;      // blocks have been left out
            tk.issue(lk[0], gk, k0, last, wave);
            tv.issue(lv[0], gv, k0, last, wave);
            int buf = 0;
            for (int kt = k0; kt < k1; kt += KT, buf ^= 1) {
                tiles_arrive();
                if (kt + KT < k1) {
                    tk.issue(lk[buf ^ 1], gk, kt + KT, last, wave);
                    tv.issue(lv[buf ^ 1], gv, kt + KT, last, wave);
                }
                const int mine = kt + 32 * NB * kg;
                if (mine >= any_hi || mine + 32 * NB <= any_lo) continue;
                f32x16 x[NB] = {};
#pragma unroll
                for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                    for (int d = 0; d < DP / 16; ++d) x[kb] = Elem<T>::mfma(rows.get(lk[buf], NB * kg + kb, d), qf[d], x[kb]);
                reads_ahead<NB * DP / 16, 1, NB * DP / 32>();
                bool finite = true;
                if (mine + 32 * NB > all_hi || mine < all_lo) {
#pragma unroll
                    for (int kb = 0; kb < NB; ++kb)
                        if (care) finite &= block_is_finite<DP>(lv[buf], NB * kg + kb, lane);
                    const int at = mine + 4 * (lane >> 5);
#pragma unroll
                    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const int key = at + 32 * kb + 8 * (i / 4) + i % 4;
                            x[kb][i] = key < hi && key >= lo ? x[kb][i] : -ATTN_INF;
                        }
                }
                float top = x[0][0];
#pragma unroll
                for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                    for (int i = 0; i < 16; ++i) top = fmaxf(top, x[kb][i]);
                top = half_max(top);
                // The sums stay on an old maximum until a score passes it by a factor of 2^8: what is rounded to 16 bits keeps
                // its relative error, and rows seldom come to that more than once or twice.
                if (__ballot((top - m) * c > 8.f)) {
                    const float up = fmaxf(m, top), by = exp2_fast((m - up) * c);
                    m = up;
                    l *= by;
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[d][i] *= by;
                }
                const float mc = m * c - SHIFT<T>;
                float part = 0.f;
                if (!finite) {
                    odd = true;
#pragma unroll
                    for (int kb = 0; kb < NB; ++kb)
#pragma unroll
                        for (int i = 0; i < 16; ++i) l += exp2_fast(__builtin_fmaf(x[kb][i], c, -mc));
                    continue;
                }
#pragma unroll
                for (int t = 0; t < 2 * NB; ++t) {
                    float p[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        p[i] = exp2_fast(__builtin_fmaf(x[t / 2][8 * (t % 2) + i], c, -mc));
                        part += p[i];
                    }
                    const auto pf = round8<T>(p, 0);
#pragma unroll
                    for (int d = 0; d < DP / 32; ++d) acc[d] = Elem<T>::mfma(cols.get(lv[buf], 2 * NB * kg + t, d), pf, acc[d]);
                }
                l += part;
            }
            if constexpr (care) {
                if (!odd) return;
                const T *const qrow = (const T *)q.data + (int64_t)b * q.batch + (int64_t)h * q.head + (int64_t)used * q.row;
#pragma unroll 1
                for (int kt = k0; kt < k1; kt += KT) {
                    const int mine = kt + 32 * NB * kg;
                    if (mine >= any_hi || mine + 32 * NB <= any_lo || (mine + 32 * NB <= all_hi && mine >= all_lo)) continue;
                    bool finite = true;
                    for (int kb = 0; kb < NB; ++kb) finite &= rows_are_finite(gv, v.row, mine + 32 * kb, last, s.head_dim, lane);
                    if (finite) continue;
#pragma unroll 1
                    for (int key = max(mine, lo); key < min(mine + 32 * NB, hi); ++key) {
                        const float x = dot(qrow, gk + (int64_t)key * k.row, s.head_dim);
                        add_row<DP>(acc, gv + (int64_t)key * v.row, exp2_fast((x - m) * c + SHIFT<T>), s.head_dim, lane);
                    }
                }
            }
        };
        pass(std::false_type());
        if (!sums_are_numbers(acc) && lane == 0) again = 1;
        __syncthreads();
        if (again) {
            clear();
            pass(std::true_type());
        }
    }
    l = half_sum(l);
    if constexpr (KG > 1) {
        __shared__ float2 sums[KG][QW][32];
        static_assert((KG - 1) * QW * DP / 2 * 64 * sizeof(float) <= sizeof(tiles_kv), "the sums fit where the tiles were");
        float *const box = (float *)tiles_kv + qw * (DP / 2 * 64);
        __syncthreads();
        if (kg > 0) {
            put_sums(box + (kg - 1) * QW * (DP / 2 * 64), acc, lane);
            if (lane < 32) sums[kg][qw][lane] = make_float2(m, l);
        }
        __syncthreads();
        if (kg > 0) return;
        const float c = s.scale * LOG2E;
#pragma unroll 1
        for (int g = 1; g < KG; ++g) {
            const float2 other = sums[g][qw][lane & 31];
            const float up = fmaxf(m, other.x), by = exp2_fast((m - up) * c), times = exp2_fast((other.x - up) * c);
#pragma unroll
            for (int d = 0; d < DP / 32; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) acc[d][i] *= by;
            add_sums(box + (g - 1) * QW * (DP / 2 * 64), acc, times, lane);
            l = l * by + other.y * times;
            m = up;
        }
    }
    if (parts > 1) {
        if (row >= sp.ql) return;
        const int64_t at = (((int64_t)b * s.q_heads + h) * s.q_len + row) * parts + part;
#pragma unroll
        for (int d = 0; d < DP / 32; ++d)
#pragma unroll
            for (int i = 0; i < 16; i += 4)
                *(f32x4 *)(outs + at * DP + 32 * d + 2 * i + 4 * (lane >> 5)) = f32x4{acc[d][i], acc[d][i + 1], acc[d][i + 2], acc[d][i + 3]};
        if (lane < 32) out_sums[at] = make_float2(m, l);
        return;
    }
    if (row < (int)s.q_len) {
        const bool some = row < sp.ql && l != 0.f;      // (a sum that is not a number is some)
        if (!some)
#pragma unroll
            for (int d = 0; d < DP / 32; ++d) acc[d] = f32x16{};
        store_kept<DP>(orow, acc, some ? 1.f / l : 0.f, s.head_dim, lane);
        if (lane < 32) *lrow = some ? m * s.scale + __logf(l) - SHIFT<T> * LN2 : -ATTN_INF;
    }
}

// A wave joins the parts of a row.
template <class T, int DP>
__global__ __launch_bounds__(256) void k_attention_join(AttnShape s, Rows o, float *lse, uint32_t parts, const float *outs, const float2 *sums)
{
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    if (at >= (int64_t)s.batch * s.q_heads * s.q_len) return;
    const uint32_t row = (uint32_t)(at % s.q_len), h = (uint32_t)(at / s.q_len % s.q_heads), b = (uint32_t)(at / s.q_len / s.q_heads);
    constexpr int N = DP / 64;      // elements of a lane
    const float c = s.scale * LOG2E;
    float m = LOWEST, l = 0.f, y[N] = {};
    if ((int)row < span_of(s, b).ql) {
        for (uint32_t i = 0; i < parts; ++i) m = fmaxf(m, sums[at * parts + i].x);
#pragma unroll 4
        for (uint32_t i = 0; i < parts; ++i) {
            const float2 x = sums[at * parts + i];
            const float by = exp2_fast((x.x - m) * c);
            l += x.y * by;
#pragma unroll
            for (int j = 0; j < N; ++j) y[j] += outs[(at * parts + i) * DP + lane * N + j] * by;
        }
    }
    const bool some = l != 0.f;
    T *to = (T *)o.data + (int64_t)b * o.batch + (int64_t)h * o.head + (int64_t)row * o.row + lane * N;
    typedef T TN __attribute__((ext_vector_type(N)));
    TN z;
#pragma unroll
    for (int j = 0; j < N; ++j) z[j] = (T)(some ? y[j] / l : 0.f);
    if (lane * N < (int)s.head_dim) *(TN *)to = z;
    if (lane == 0) lse[at] = some ? m * s.scale + __logf(l) - SHIFT<T> * LN2 : -ATTN_INF;
}

template <class T, int DP, int QW, int KG, int NB>
hipError_t launch_as(const AttnShape &s, const Rows &q, const Rows &k, const Rows &v, const Rows &out, float *lse, void *ws, hipStream_t st)
{
    const uint32_t tiles = (s.q_len + 32 * QW - 1) / (32 * QW), parts = forward_parts(s);
    const uint32_t total = padded_caches(s.batch * s.kv_heads) * (s.q_heads / s.kv_heads) * tiles * parts;
    const uint64_t rows = (uint64_t)s.batch * s.q_heads * s.q_len;
    float *outs = (float *)ws;
    float2 *sums = (float2 *)(outs + rows * parts * DP);
    k_attention<T, DP, QW, KG, NB><<<total, QW * KG * 64, 0, st>>>(s, q, k, v, out, lse, tiles, parts, outs, sums);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || parts == 1) return e;
    k_attention_join<T, DP><<<(uint32_t)((rows + 3) / 4), 256, 0, st>>>(s, out, lse, parts, outs, sums);
    return hipGetLastError();
}

template <class T, int DP>
hipError_t launch(const AttnShape &s, const Rows &q, const Rows &k, const Rows &v, const Rows &out, float *lse, void *ws, hipStream_t st)
{
    switch (share_of(s, s.q_heads, s.q_len)) {
    case Share::FOUR:
        // 32 keys a tile leave registers for a third wave on a SIMD, where there are that many (3104 blocks of 128
        // rows: 1325 us for 32 heads of 12345 rows, with 64 keys 1360; 640 blocks: 61 us and 54)
        if ((uint64_t)s.batch * s.q_heads * ((s.q_len + 127) / 128) > 1024) return launch_as<T, DP, 4, 1, 1>(s, q, k, v, out, lse, ws, st);
        return launch_as<T, DP, 4, 1, 2>(s, q, k, v, out, lse, ws, st);
    case Share::FOUR_BY_TWO: return launch_as<T, DP, 4, 2, 2>(s, q, k, v, out, lse, ws, st);
    default: return launch_as<T, DP, 2, 4, 1>(s, q, k, v, out, lse, ws, st);
    }
}

}  // namespace

// Parts of the keys: as many as workgroups of 64 rows (the last of the sharings above) leave units for, of four tiles of 128
// keys at least.  Of 17 rows on 12000 keys, two sequences of 16 heads, 25 us (in one part 111); 500 rows on 8000 keys 52 us
// (77); twice as many parts, which units then take in turn, 30 and 60 us; two tiles to a part in place of four 26 us where
// that is 19 (2 heads of 2048 rows, causal; one part 25).
uint32_t forward_parts(const AttnShape &s)
{
    const uint64_t groups = (uint64_t)s.batch * s.q_heads * ((s.q_len + 63) / 64);
    const uint64_t want = groups ? 256 / groups : 0, most = s.k_len / 512;
    return (uint32_t)(want < 2 || most < 2 ? 1 : want > most ? most : want);
}
size_t forward_workspace(const AttnShape &s)
{
    const uint32_t parts = forward_parts(s);
    return parts == 1 ? 0 : (size_t)s.batch * s.q_heads * s.q_len * parts * ((s.head_dim <= 64 ? 64 : 128) * sizeof(float) + sizeof(float2));
}

hipError_t launch_attention(const AttnShape &s, const Rows &q, const Rows &k, const Rows &v, const Rows &out, float *lse, void *ws, hipStream_t st)
{
    if (s.half)
        return s.head_dim <= 64 ? launch<_Float16, 64>(s, q, k, v, out, lse, ws, st) : launch<_Float16, 128>(s, q, k, v, out, lse, ws, st);
    return s.head_dim <= 64 ? launch<__bf16, 64>(s, q, k, v, out, lse, ws, st) : launch<__bf16, 128>(s, q, k, v, out, lse, ws, st);
}

}  // namespace lap
