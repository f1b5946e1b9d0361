// Which slots of a key/value cache stay, by the attention weight they have received.
//
// Order of a row's slots (one cache of one head): empty ones, then those in use by weight (not a number counts as the
// least), equal ones with the higher index first, then the newest `recent` positions.  An eviction keeps the last `keep`
// of that order and copies them, in the order of their slots, into another cache; an insertion overwrites the first.
//
// Measured: 8 ragged prompts of up to 16384 tokens, 8 heads, into 2048 slots of 128 elements, 32 us: the choice is a chain of some
// 18 in the longest rows (by leaving its steps out one by one: 2.6 to read 16384 weights, 6 for the first digit of the search, 4
// for the others, 5 to place), while shorter ones are copied (134 MB read and written in all, 20 us alone); waves wait in 62 % of
// their cycles.  Rows that do not fit into registers: 8 heads of 60000 slots into 8000 76 us, where every workgroup of a row
// reads its weights up to five times.  An insertion into 64 x 8 caches of 2048 slots 4.7 us,
// most of it a launch and three dependent accesses.
#include "attn_core.h"
#include "lap_dev.h"

namespace lap {
namespace {

constexpr uint32_t NEWEST = 0xFFFFFFFFu, LEAST = 1u, EMPTY = 0u;

// weights as whole numbers in the same order (minus zero is zero)
__device__ __forceinline__ uint32_t weight_key(float w)
{
    const uint32_t u = __float_as_uint(w + 0.f);
    return w != w ? LEAST : u & 0x80000000u ? ~u : u | 0x80000000u;
}

constexpr int EV = 1024, EW = EV / 64, BIN_BITS = 13, BINS = 1 << BIN_BITS;

struct EvictRow {
    const float *weights;
    const int32_t *positions;
    int len, newest, recent;      // slots in use; the largest position; how many up to it are among the newest
    __device__ __forceinline__ uint32_t key(float w, int p) const { return p < 0 ? EMPTY : newest - p < recent ? NEWEST : weight_key(w); }
};

// how many of the lanes before this one are among `set`
__device__ __forceinline__ uint32_t before_lane(uint64_t set)
{
    return __builtin_amdgcn_mbcnt_hi((uint32_t)(set >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)set, 0));
}

// one more in the counter of every lane's bin; lanes with the bin of the first one that counts add up in one go (many
// weights are equal, and additions to one counter take turns)
__device__ __forceinline__ void count(uint32_t *bins, bool counts, uint32_t bin, int lane)
{
    const uint64_t who = ballot(counts);
    if (!who) return;
    const int first = __ffsll((unsigned long long)who) - 1;
    const uint32_t of = read_lane(bin, first);
    const uint64_t same = ballot(counts && bin == of);
    if (counts && (bin != of || lane == first)) atomicAdd(&bins[bin], bin == of ? (uint32_t)__popcll(same) : 1u);
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
constexpr int COPY_ROWS = 4;      // rows of keys and of values that a thread has on their way

// The slots that stay, ascending, and their rows of keys and values.  `pieces` workgroups for each row find the same order each,
// write a share of the new cache's slots, and copy these: a copy that starts with a row's choice and spreads over the chip, in
// one launch (a choice by one workgroup a row, then a copy of all rows: 38 us in place of 32 above).  A stretch of the row
// for each wave, with the weights of EACH x 64 slots in registers (EACH 0: read again from the L2 cache each time).  The key of
// the last one that stays is found digit by digit (13, 13 and 6 bits: the first one has four bits of a weight's fraction, so
// that weights of one size do not all meet in one counter) from counts in LDS.
template <int EACH>
__global__ __launch_bounds__(EV) void k_evict(EvictShape s, Rows k, Rows v, const float *weights, const int32_t *positions, Rows k_out, Rows v_out,
                                            int32_t *kept, float *weights_out, int32_t *positions_out, int32_t *lens_out, uint32_t pieces)
{
    __shared__ uint32_t bins[BINS];
    __shared__ uint32_t part[EW][2];
    __shared__ uint32_t found[3];
    const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const uint32_t rows = s.batch * s.kv_heads, at_row = blockIdx.x % rows, piece = blockIdx.x / rows;      // (the pieces of a row on one die, mostly)
    const uint32_t b = at_row / s.kv_heads, h = at_row % s.kv_heads;
    const uint32_t first = (uint32_t)((uint64_t)s.slots_out * piece / pieces), last = (uint32_t)((uint64_t)s.slots_out * (piece + 1) / pieces);
    EvictRow row;
    row.weights = weights + (int64_t)at_row * s.slots;
    row.positions = positions ? positions + (int64_t)at_row * s.slots : nullptr;
    row.len = clamp_len(s.lens, b, s.slots);

    int newest = row.len - 1, used = row.len;
    if (positions) {
        newest = -1, used = 0;
        for (int i = t; i < row.len; i += EV) {
            const int p = row.positions[i];
            newest = max(newest, p);
            used += p >= 0;
        }
        for (int d = 32; d; d >>= 1) newest = max(newest, __shfl_xor(newest, d, 64)), used += __shfl_xor(used, d, 64);
        if (lane == 0) part[wave][0] = (uint32_t)newest, part[wave][1] = (uint32_t)used;
        __syncthreads();
        used = 0;
        for (int i = 0; i < EW; ++i) newest = max(newest, (int)part[i][0]), used += (int)part[i][1];
        __syncthreads();
    }
    row.newest = newest, row.recent = (int)s.recent;
    const int keep = min((int)s.keep, used);

    // this wave's slots, in whole 64s
    const int each = ((row.len + EW - 1) / EW + 63) / 64 * 64, i0 = wave * each, i1 = min(i0 + each, row.len);
    constexpr int AHEAD = EACH ? EACH : 16;      // times 64 weights, asked for before the first is looked at
    float mine[AHEAD];
    uint32_t keys[AHEAD];
    const auto read = [&](int from) {
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) mine[j] = row.weights[min(from + 64 * j + lane, i1 - 1)];
#pragma unroll
        for (int j = 0; j < AHEAD; ++j) {
            const int i = from + 64 * j + lane, p = positions ? row.positions[min(i, i1 - 1)] : i;
            keys[j] = i < i1 ? row.key(mine[j], p) : EMPTY;
        }
    };
    if (EACH > 0 && i0 < i1) read(i0);
    const auto for_all = [&](auto &&f) {      // f(first slot, this lane's key and weight), for 64 slots at a time
        if constexpr (EACH > 0) {
#pragma unroll
            for (int j = 0; j < EACH; ++j)
                if (i0 + 64 * j < i1) f(i0 + 64 * j, keys[j], mine[j]);
        } else
            for (int from = i0; from < i1; from += 64 * AHEAD) {
                read(from);
#pragma unroll
                for (int j = 0; j < AHEAD; ++j)
                    if (from + 64 * j < i1) f(from + 64 * j, keys[j], mine[j]);
            }
    };

    // everything above `bound` stays, and the first `equal` slots whose key is `bound`
    uint32_t bound = LEAST, equal = 0xFFFFFFFFu;      // all slots in use
    if (keep < used) {
        uint32_t prefix = 0, mask = 0, want = (uint32_t)keep;      // of the slots whose key begins with prefix, the want-th
        for (int digit = 0; digit < 3; ++digit) {
            const int shift = digit == 0 ? 19 : digit == 1 ? 6 : 0;
            const uint32_t ones = digit == 2 ? 63 : BINS - 1;
            for (int i = t; i < BINS; i += EV) bins[i] = 0;
            __syncthreads();
            for_all([&](int, uint32_t k, float) { count(bins, k != EMPTY && (k & mask) == prefix, (k >> shift) & ones, lane); });
            __syncthreads();
            // counts from the top: a thread holds eight bins, the highest first
            constexpr int OWN = BINS / EV;
            const int lo = BINS - OWN * (t + 1);
            uint32_t c[OWN], own = 0;
#pragma unroll
            for (int i = 0; i < OWN; ++i) own += c[i] = bins[lo + i];
            uint32_t up = own;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t x = __shfl_up(up, d, 64);
                if (lane >= d) up += x;
            }
            if (lane == 63) part[wave][0] = up;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < EW; ++i) up += i < wave ? part[i][0] : 0;
            uint32_t before = up - own;
            if (before < want && want <= up) {
#pragma unroll
                for (int i = OWN - 1; i >= 0; --i) {
                    if (before < want && want <= before + c[i]) found[0] = (uint32_t)(lo + i), found[1] = want - before, found[2] = c[i];
                    before += c[i];
                }
            }
            __syncthreads();
            prefix |= found[0] << shift;
            mask |= ones << shift;
            want = found[1];
            const bool all = want == found[2];      // all that begin like this: nothing left to tell apart (prefix is not 0: if the least stay, all do)
            __syncthreads();
            if (all) {
                prefix -= 1, want = 0;
                break;
            }
        }
        bound = prefix, equal = want;
    }

    // how many of every wave's are above the bound and at it, then the places
    uint32_t above = 0, at = 0;
    for_all([&](int, uint32_t k, float) {
        above += k > bound;
        at += k == bound && k != EMPTY;
    });
    above = wave_reduce_add32(above), at = wave_reduce_add32(at);
    if (lane == 0) part[wave][0] = above, part[wave][1] = at;
    __syncthreads();
    uint32_t place = 0, seen = 0;
#pragma unroll
    for (int i = 0; i < EW; ++i)
        if (i < wave) place += part[i][0] + min(equal - min(equal, seen), part[i][1]), seen += part[i][1];
    const int64_t out = (int64_t)at_row * s.slots_out;
    kept += out, weights_out += out, positions_out += out;
    for_all([&](int base, uint32_t k, float w) {
        const uint64_t eq = ballot(k == bound && k != EMPTY);
        bool stays = k > bound;
        if (eq) {
            stays |= k == bound && k != EMPTY && seen + before_lane(eq) < equal;
            seen += __popcll(eq);
        }
        const uint64_t all = ballot(stays);
        if (stays) {
            const uint32_t to = place + before_lane(all);
            if (to >= first && to < last) {
                kept[to] = base + lane;
                weights_out[to] = w;
                positions_out[to] = positions ? row.positions[base + lane] : base + lane;
            }
        }
        place += __popcll(all);
    });
    for (uint32_t i = max((uint32_t)keep, first) + t; i < last; i += EV) {
        kept[i] = -1;
        weights_out[i] = 0.f;
        positions_out[i] = -1;
    }
    if (h == 0 && piece == 0 && t == 0) lens_out[b] = min((int)s.keep, row.len);
    __syncthreads();

    // keys and values: 16 bytes for each thread, rows side by side
    const uint32_t across = s.head_dim / 8, side = EV / across, r = t / across, e = t % across * 8;
    if (r >= side) return;
    const uint16_t *gk = (const uint16_t *)k.data + (int64_t)b * k.batch + (int64_t)h * k.head + e;
    const uint16_t *gv = (const uint16_t *)v.data + (int64_t)b * v.batch + (int64_t)h * v.head + e;
    uint16_t *ok = (uint16_t *)k_out.data + (int64_t)b * k_out.batch + (int64_t)h * k_out.head + e;
    uint16_t *ov = (uint16_t *)v_out.data + (int64_t)b * v_out.batch + (int64_t)h * v_out.head + e;
    for (uint32_t to = first + r; to < last; to += side * COPY_ROWS) {
        u32x4 x[COPY_ROWS] = {}, y[COPY_ROWS] = {};
        int from[COPY_ROWS];
#pragma unroll
        for (int i = 0; i < COPY_ROWS; ++i) from[i] = to + i * side < last ? kept[to + i * side] : -1;
#pragma unroll
        for (int i = 0; i < COPY_ROWS; ++i)
            if (from[i] >= 0) x[i] = *(const u32x4 *)(gk + (int64_t)from[i] * k.row), y[i] = *(const u32x4 *)(gv + (int64_t)from[i] * v.row);
#pragma unroll
        for (int i = 0; i < COPY_ROWS; ++i)
            if (to + i * side < last) {
                *(u32x4 *)(ok + (int64_t)(to + i * side) * k_out.row) = x[i];
                *(u32x4 *)(ov + (int64_t)(to + i * side) * v_out.row) = y[i];
            }
    }
}

// One workgroup for each row: the first slot in the order above, and the new token into it.
constexpr int IN = 256;
__global__ __launch_bounds__(IN) void k_insert(InsertShape s, Rows k_new, Rows v_new, Rows k, Rows v, float *weights, int32_t *positions,
                                             const int32_t *position, int32_t *slots_out)
{
    __shared__ uint64_t part[IN / 64];
    const int t = threadIdx.x, lane = t & 63;
    const uint32_t b = blockIdx.x / s.kv_heads, h = blockIdx.x % s.kv_heads;
    const int at = position[b];
    if (at < 0) {
        if (t == 0) slots_out[blockIdx.x] = -1;
        return;
    }
    float *w = weights + (int64_t)blockIdx.x * s.slots;
    int32_t *pos = positions + (int64_t)blockIdx.x * s.slots;
    uint64_t least = ~0ull;
    for (uint32_t first = t; first < s.slots; first += 8 * IN) {      // eight at a time; past the end the last one again
        int p[8];
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) p[j] = pos[min(first + j * IN, s.slots - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = w[min(first + j * IN, s.slots - 1)];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const uint32_t i = min(first + j * IN, s.slots - 1);
            const uint32_t key = p[j] < 0 ? EMPTY : (int64_t)p[j] > (int64_t)at - (int64_t)s.recent ? NEWEST : weight_key(x[j]);
            const uint64_t y = (uint64_t)key << 32 | (p[j] < 0 ? i : ~i);
            least = y < least ? y : least;
        }
    }
    for (int d = 32; d; d >>= 1) {
        const uint64_t x = __shfl_xor((unsigned long long)least, d, 64);
        least = x < least ? x : least;
    }
    if (lane == 0) part[t >> 6] = least;
    __syncthreads();
    for (int i = 0; i < IN / 64; ++i) least = part[i] < least ? part[i] : least;
    const uint32_t slot = (least >> 32) == EMPTY ? (uint32_t)least : ~(uint32_t)least;
    const uint32_t across = s.head_dim / 8;
    if (t < (int)(2 * across)) {
        const bool second = t >= (int)across;
        const uint32_t e = (second ? t - across : t) * 8;
        const Rows &from = second ? v_new : k_new, &to = second ? v : k;
        *(uint4 *)((uint16_t *)to.data + (int64_t)b * to.batch + (int64_t)h * to.head + (int64_t)slot * to.row + e) =
            *(const uint4 *)((const uint16_t *)from.data + (int64_t)b * from.batch + (int64_t)h * from.head + e);
    }
    if (t == 0) {
        w[slot] = 0.f;
        pos[slot] = at;
        slots_out[blockIdx.x] = (int32_t)slot;
    }
}

}  // namespace

// Workgroups for a row: as many as rows leave units for (with twice as many, which take turns, 44 us in place of 32 above), of
// 256 slots of the new cache at least.
constexpr uint32_t EVICT_UNITS = 256, EVICT_LEAST = 256;

hipError_t launch_cache_evict(const EvictShape &s, const Rows &k, const Rows &v, const float *weights, const int32_t *positions,
                              const Rows &k_out, const Rows &v_out, float *weights_out, int32_t *positions_out, int32_t *lens_out,
                              int32_t *kept, hipStream_t st)
{
    const uint32_t rows = s.batch * s.kv_heads;
    const uint32_t spread = rows < EVICT_UNITS ? EVICT_UNITS / rows : 1, most = (s.slots_out + EVICT_LEAST - 1) / EVICT_LEAST;
    const uint32_t pieces = spread < most ? spread : most, grid = rows * pieces;
    const auto kernel = s.slots <= 4 * EV ? k_evict<4> : s.slots <= 16 * EV ? k_evict<16> : k_evict<0>;
    kernel<<<grid, EV, 0, st>>>(s, k, v, weights, positions, k_out, v_out, kept, weights_out, positions_out, lens_out, pieces);
    return hipGetLastError();
}

hipError_t launch_cache_insert(const InsertShape &s, const Rows &k_new, const Rows &v_new, const Rows &k, const Rows &v, float *weights,
                               int32_t *positions, const int32_t *position, int32_t *slots_out, hipStream_t st)
{
    k_insert<<<s.batch * s.kv_heads, IN, 0, st>>>(s, k_new, v_new, k, v, weights, positions, position, slots_out);
    return hipGetLastError();
}

}  // namespace lap
