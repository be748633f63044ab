// libcsr5: attention over packed sequences and over a paged cache of keys and values.  Its gradients are in attention_back.hip.
// The C ABI is declared in include/csr5.h.
//
// Rows are folded: the query heads that share a head of keys are rows side by side, r = token * shared + head, so that they
// read its keys once.  A score is s = q.k in units of 1 / (scale * log2 e); softmax by a running base b, with p = 2^(c (s - b)), c = scale log2 e.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "csr5.h"
#include "heads.h"
#include "numbers.h"
#include "sequences.h"
#include "to_lds.h"

namespace {

template <typename T, typename KV> struct Attend {
    int32_t sequences, rows, heads, kv_heads, shared, d;
    const int32_t* q_offset;
    float scale;
    bool causal;
    Heads<const T> q;
    KV kv;
    Heads<T> out;
    float* lse;
    int32_t tiles;
    int32_t chunk;          // keys of a workgroup, where the work is split over them (0: it is not)
    float *part, *stats;    // ... and what it leaves: [chunk][row][head][d] sums, [chunk][row][head] their base and total
};

// The base rises where a score passes it by more than this many powers of two: sums are rescaled seldom, and p is at most 256.
constexpr float RISE = 8.f;
// The same in scores; finite (the smallest scales would make it infinite), so that the first score, from a base of -inf, passes it.
__device__ __forceinline__ float rise_of(float c) { return fminf(RISE / c, 0x1.fffffep127f); }

__device__ __forceinline__ float half_most(float v) {       // over lanes l and l ^ 32
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(both[0]) + __uint_as_float(both[1]);
}
__device__ __forceinline__ float quarter_most(float v) {    // over lanes l, l ^ 16, l ^ 32, l ^ 48
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_most(fmaxf(__uint_as_float(both[0]), __uint_as_float(both[1])));
}
__device__ __forceinline__ float quarter_sum(float v) {
    const auto both = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return half_sum(__uint_as_float(both[0]) + __uint_as_float(both[1]));
}
// What a workgroup leaves of one row: the result, or its part of it.
template <typename T, typename KV> struct Leave {
    T* out;
    float *part, *lse, *stats;
    __device__ __forceinline__ Leave(const Attend<T, KV>& a, int32_t row, int32_t h) {
        const int64_t at = (int64_t(blockIdx.y) * a.rows + row) * a.heads + h;
        out = a.out.p + row * a.out.row + h * a.out.head;
        part = a.chunk ? a.part + at * a.d : nullptr, stats = a.chunk ? a.stats + at * 2 : nullptr;
        lse = !a.chunk && a.lse ? a.lse + int64_t(h) * a.rows + row : nullptr;
    }
    // four neighbouring values of the sum from c on; inverse: of the total
    template <bool WIDE> __device__ __forceinline__ void four(int c, int d, const float (&v)[4], float inverse) const {
        if (part) {
#pragma unroll
            for (int e = 0; e < 4; e++)
                if (c + e < d) part[c + e] = v[e];
        } else {
            const float w[4] = {v[0] * inverse, v[1] * inverse, v[2] * inverse, v[3] * inverse};
            store_values<4, WIDE>(out + c, d - c, w);
        }
    }
    __device__ __forceinline__ void more(int c, float v) const {
        if (part) part[c] += v;
        else out[c] = T(float(out[c]) + v);
    }
    __device__ __forceinline__ void total(float base, float sum, float scale) const {
        if (stats) stats[0] = base, stats[1] = sum;
        else if (lse) *lse = sum == 0.f ? -INFINITY : base * scale + logf(sum);
    }
};

// ---------------------------------------------------------------------------------------------------------------
// Many rows.  128 folded rows, 32 to each of four wavefronts, which go through the keys in tiles of 32.
// Scores are computed as keys x rows, k q^T: a lane has 16 of the 32 scores of one row, so the maximum and the sum need one exchange
// with the lane's other half, and what it has is, rounded, the second operand of out^T = v^T p^T as it is: the order of the depth (keys) is free as
// long as v's, which a transposing read of LDS brings, is the same.  Two tiles of keys and of values are in LDS, the next on its way, at fixed places, so
// that the reads' addresses need no arithmetic.  170 registers at most: three workgroups to a CU, whose products and powers go on side by side.
// Bound by power and by what products and powers take of each other: 3 sequences up to 8001, 32 heads of 128 with 8 of keys, 794 us, 916 TFLOP/s
// (a library product of 8192^3: 1598), the matrix units busy 48 % of the time at 1.85 GHz.  Without powers it takes 700 us, without loads 645, with products alone 545.
// Tiles of 64 and two workgroups: 775 against 740; the next scores beside this tile's powers in one stream of instructions: 908; eight wavefronts to 256
// rows: 874 against 775; rings of three and four tiles: no change.
// ---------------------------------------------------------------------------------------------------------------
constexpr int MANY_ROWS = 128, MANY_SHIFT = 7, MANY_KEYS = 32;

// What a lane left of a row (values c = dt * 32 + i * 8 + half * 4 on) sees of keys [from, to), whose values that are not finite were left out.
template <int ND, typename T, typename KV, typename One> __device__ __forceinline__ void repair(const Leave<T, KV>& leave, const One& kv, int32_t from, int32_t to, int d) {
    for (int32_t j = from; j < to; j++) {
        const T* const v = kv.any_value(j);
        if (!v) continue;
        for (int i = 0; i < 4 * ND; i++)
            for (int e = 0; e < 4; e++) {
                const int c = i * 8 + ((threadIdx.x >> 5) & 1) * 4 + e;
                if (c < d && !finite(float(v[c]))) leave.more(c, float(v[c]));
            }
    }
}

template <typename T, typename KV, int ND, bool WIDE, int KG> __global__ __launch_bounds__(256, KG == 1 ? 3 : 2) void k_attend_many(Attend<T, KV> a) {
    constexpr int D = ND <= 2 ? 64 : 128, KEYS = MANY_KEYS * KG, TILE = KEYS * D * 2, ROWS = MANY_ROWS / KG;
    constexpr int SHIFT = KG == 1 ? MANY_SHIFT : KG == 2 ? MANY_SHIFT - 1 : MANY_SHIFT - 2;
    typedef Bring<T, D, WIDE, false, KEYS, 4> B;
    extern __shared__ __align__(16) uint8_t lds[];          // begins at 0: nothing else is in LDS, so bits of addresses can be turned over
    int32_t& cleansed = *reinterpret_cast<int32_t*>(lds + 4 * TILE);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, kg = KG == 1 ? 0 : wave / (4 / KG);
    const int32_t hk = blockIdx.x % a.kv_heads;
    TileOf at;
    if (!tile_of(a.q_offset, a.sequences, a.rows, a.shared, SHIFT, a.tiles - 1 - int32_t(blockIdx.x / a.kv_heads), at)) return;
    const auto kv = a.kv.one(at.s, hk);
    const int32_t m = at.rows.count, n = kv.count;
    const int64_t first = at.first + wave % (4 / KG) * 32;
    const Row row = row_of(first + (lane & 31), m, n, a.shared, a.causal);
    // the keys that this wavefront's first and last row see, and the workgroup's
    const int32_t least = __builtin_amdgcn_readfirstlane(row.limit), most = __builtin_amdgcn_readlane(row.limit, 31);
    const int32_t all = __builtin_amdgcn_readfirstlane(row_of(at.first + ROWS - 1, m, n, a.shared, a.causal).limit);
    const int32_t fewest = __builtin_amdgcn_readfirstlane(row_of(at.first, m, n, a.shared, a.causal).limit);
    const int32_t begin = a.chunk * int32_t(blockIdx.y), end = a.chunk ? min(all, begin + a.chunk) : all;
    if (a.chunk && begin >= end) return;
    if (threadIdx.x == 0) cleansed = 0;

    vec<T, 8> q[2 * ND];
    {
        const T* const from = a.q.p + (at.rows.first + row.token) * a.q.row + (hk * a.shared + row.head) * a.q.head;
#pragma unroll
        for (int kk = 0; kk < 2 * ND; kk++) q[kk] = eight_values<WIDE>(from + (2 * kk + half) * 8, row.there ? a.d - (2 * kk + half) * 8 : 0);
    }
    // LDS: two tiles of keys, then two of values
    const uint32_t lds0 = lds_address(lds);
    const B bring(kv, wave, a.d);
    typename decltype(kv)::Ahead ahead[B::LOADS];
    const ReadFixed<ND> read(lds0 + kg * MANY_KEYS * D * 2);      // its 32 keys of a tile

    const float c = a.scale * LOG2_E, rise = rise_of(c);
    float base = -INFINITY, sum = 0.f;
    f32x16 o[ND] = {};
    auto tile = [&](auto at_place, int32_t j0) {
        constexpr int NOW = decltype(at_place)::value;
        landed<0>();
        if (j0 + KEYS > fewest && fewest < n) {        // some row does not see some key
            if (cleanse<T>(lds + (2 + NOW) * TILE, TILE, threadIdx.x, 256)) cleansed = 1;
            __syncthreads();
        }
        if (j0 + KEYS < end) {
            bring(kv, j0 + KEYS, ahead, a.d, lds0 + (1 - NOW) * TILE, lds0 + (3 - NOW) * TILE);
            bring.look(kv, j0 + 2 * KEYS, ahead);
        }
        const int32_t mine = j0 + kg * MANY_KEYS;           // this wavefront's keys
        if (mine >= most) return;
        f32x16 s = {};
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int kk = 0; kk < 2 * ND; kk++) s = product32(read.template row<T>(NOW * TILE, kk), q[kk], s);
        if (mine + MANY_KEYS > least) {
#pragma unroll
            for (int i = 0; i < 16; i++) s[i] = or_none(s[i], row.limit - 1 - (mine + 8 * (i / 4) + 4 * half + i % 4));
        }
        __builtin_amdgcn_s_setprio(0);
        float top = s[0];
#pragma unroll
        for (int i = 1; i < 16; i++) top = fmaxf(s[i], top);
        top = half_most(top);
        if (__any(top > base + rise)) {
            const float higher = fmaxf(base, top), less = higher == base ? 1.f : power((base - higher) * c);
            base = higher, sum *= less;
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[dt][i] *= less;
        }
        const float zero = base == -INFINITY ? 0.f : base * c;
        vec<T, 8> p[2];
#pragma unroll
        for (int i = 0; i < 16; i++) {
            const float e = power(fmaf(s[i], c, -zero));
            sum += e;
            p[i / 8][i % 8] = T(e);
        }
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int dt = 0; dt < ND; dt++) o[dt] = product32(read.template turned<T>((2 + NOW) * TILE + k * 16 * D * 2, dt), p[k], o[dt]);
        __builtin_amdgcn_s_setprio(0);
    };
    if (bring.ragged) {
        zeros_to(lds0, 4 * TILE, threadIdx.x, 256);
        landed<0>();
    }
    if (begin < end) {
        bring.look(kv, begin, ahead);
        bring(kv, begin, ahead, a.d, lds0, lds0 + 2 * TILE);
        bring.look(kv, begin + KEYS, ahead);
    }
    for (int32_t j0 = begin; j0 < end; j0 += 2 * KEYS) {
        tile(std::integral_constant<int, 0>(), j0);
        if (j0 + KEYS < end) tile(std::integral_constant<int, 1>(), j0 + KEYS);
    }
    own_landed<0>();
    __syncthreads();
    sum = half_sum(sum);
    // the sums of the wavefronts that have the same rows by way of LDS: the upper half's to the lower's, until one has them all
#pragma unroll
    for (int more = KG / 2; more > 0; more /= 2) {
        float* const place = reinterpret_cast<float*>(lds) + (wave % (4 / KG) + kg % more * (4 / KG)) * (ND * 1024 + 128) + lane;
        if (kg >= more && kg < 2 * more) {
            place[0] = base, place[64] = sum;
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) place[(2 + dt * 16 + i) * 64] = o[dt][i];
        }
        __syncthreads();
        if (kg < more) {
            const float other = place[0], higher = fmaxf(base, other);
            const float less = base == higher ? 1.f : power((base - higher) * c), weight = other == higher ? 1.f : power((other - higher) * c);
            base = higher, sum = sum * less + place[64] * weight;
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) o[dt][i] = o[dt][i] * less + place[(2 + dt * 16 + i) * 64] * weight;
        }
        __syncthreads();
    }
    if (kg > 0 || !row.there) return;
    const Leave<T, KV> leave(a, at.rows.first + row.token, hk * a.shared + row.head);
    const float inverse = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int dt = 0; dt < ND; dt++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float v[4] = {o[dt][4 * i], o[dt][4 * i + 1], o[dt][4 * i + 2], o[dt][4 * i + 3]};
            leave.template four<WIDE>(dt * 32 + i * 8 + half * 4, a.d, v, inverse);
        }
    if (half == 0) leave.total(base, sum, a.scale);
    // the tiles that were cleansed begin with the first that some row does not see whole
    if (cleansed) repair<ND>(leave, kv, max(begin, fewest / KEYS * KEYS), min(row.limit, end), a.d);
}

// ---------------------------------------------------------------------------------------------------------------
// Few rows: 16 RB folded rows, and the keys dealt to four wavefronts in tiles of 32, each with LDS of its own and no barrier; what they
// have of the rows is joined at the end.  Bound by the keys' and values' way from memory: 16 KB (8 where d <= 64) of each wavefront, eight of them on a
// CU, are on their way but for the moment in which it reads what has come into registers.  48 single tokens of 64 heads with 8 of keys over 3000 to
// 24000 tokens 519 us, 5.1 TB/s (two tiles to a wavefront and one workgroup to a CU: 551); 8 over 200 to 2200 15 us and 4.5 to join the parts.  Products are keys x rows as above, of 16 x 16 x 32.
// ---------------------------------------------------------------------------------------------------------------
constexpr int FEW_KEYS = 32;

template <typename T, typename KV, int ND, bool WIDE, int RB> __global__ __launch_bounds__(256, RB <= 2 ? 2 : 1) void k_attend_few(Attend<T, KV> a) {
    constexpr int D = ND <= 2 ? 64 : 128, TILE = FEW_KEYS * D * 2, ROWS = 16 * RB;
    typedef Bring<T, D, WIDE, true, FEW_KEYS, 1> B;
    constexpr int SHIFT = RB == 1 ? 4 : RB == 2 ? 5 : 6;
    extern __shared__ __align__(16) uint8_t lds[];
    __shared__ int32_t cleansed[4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), quarter = lane >> 4, li = lane & 15;
    const int32_t hk = blockIdx.x % a.kv_heads;
    TileOf at;
    if (!tile_of(a.q_offset, a.sequences, a.rows, a.shared, SHIFT, a.tiles - 1 - int32_t(blockIdx.x / a.kv_heads), at)) return;
    const auto kv = a.kv.one(at.s, hk);
    const int32_t m = at.rows.count, n = kv.count;
    const int32_t least = __builtin_amdgcn_readfirstlane(row_of(at.first, m, n, a.shared, a.causal).limit);
    const int32_t all = __builtin_amdgcn_readfirstlane(row_of(at.first + ROWS - 1, m, n, a.shared, a.causal).limit);
    const int32_t begin = a.chunk * int32_t(blockIdx.y), end = a.chunk ? min(all, begin + a.chunk) : all;
    if (a.chunk && begin >= end) return;

    Row row[RB];
    vec<T, 8> q[RB][ND];
#pragma unroll
    for (int b = 0; b < RB; b++) {
        row[b] = row_of(at.first + b * 16 + li, m, n, a.shared, a.causal);
        const T* const from = a.q.p + (at.rows.first + row[b].token) * a.q.row + (hk * a.shared + row[b].head) * a.q.head;
#pragma unroll
        for (int kk = 0; kk < ND; kk++) q[b][kk] = eight_values<WIDE>(from + (4 * kk + quarter) * 8, row[b].there ? a.d - (4 * kk + quarter) * 8 : 0);
    }
    uint8_t* const mine = lds + wave * 2 * TILE;
    const B bring(kv, 0, a.d);
    typename decltype(kv)::Ahead ahead[B::LOADS];
    const uint32_t lds0 = lds_address(mine);
    const int vr = quarter * 4 + (li >> 2);
    uint32_t k_at[ND], v_at[2 * ND];
#pragma unroll
    for (int kk = 0; kk < ND; kk++) k_at[kk] = li * D * 2 + chunk_at<D, true>(li, 4 * kk + quarter) * 16;
#pragma unroll
    for (int dt = 0; dt < 2 * ND; dt++) v_at[dt] = TILE + vr * D * 2 + chunk_at<D, true>(vr, dt * 2 + ((li & 3) >> 1)) * 16 + (li & 1) * 8;

    const float c = a.scale * LOG2_E, rise = rise_of(c);
    float base[RB], sum[RB];
    f32x4 o[RB][2 * ND] = {};
#pragma unroll
    for (int b = 0; b < RB; b++) base[b] = -INFINITY, sum[b] = 0.f;
    const int32_t start = begin + wave * FEW_KEYS;
    if (bring.ragged) {
        zeros_to(lds0, 2 * TILE, lane, 64);
        own_read();
    }
    if (start < end) {
        bring.look(kv, start, ahead);
        bring(kv, start, ahead, a.d, lds0, lds0 + TILE);
        bring.look(kv, start + 4 * FEW_KEYS, ahead);
    }
    bool found = false;
    for (int32_t j0 = start; j0 < end; j0 += 4 * FEW_KEYS) {
        own_landed<0>();
        const bool some = j0 + FEW_KEYS > least;
        if (some && least < n) {
            found = __any(cleanse<T>(mine + TILE, TILE, lane, 64)) || found;
            wave_order();
        }
        // everything of the tile into registers, and the next one on its way before this one's products
        vec<T, 8> k[2][ND], v[2 * ND];
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
            for (int kk = 0; kk < ND; kk++) k[kb][kk] = chunk_from<T>(lds0 + k_at[kk] + kb * 16 * D * 2);
#pragma unroll
        for (int dt = 0; dt < 2 * ND; dt++) v[dt] = turned_from<T>(lds0 + v_at[dt], lds0 + v_at[dt] + 16 * D * 2);
        if (j0 + 4 * FEW_KEYS < end) {
            own_read();
            bring(kv, j0 + 4 * FEW_KEYS, ahead, a.d, lds0, lds0 + TILE);
            bring.look(kv, j0 + 8 * FEW_KEYS, ahead);
        }
        f32x4 s[RB][2] = {};
#pragma unroll
        for (int kb = 0; kb < 2; kb++)
#pragma unroll
            for (int kk = 0; kk < ND; kk++)
#pragma unroll
                for (int b = 0; b < RB; b++) s[b][kb] = product16(k[kb][kk], q[b][kk], s[b][kb]);
        vec<T, 8> p[RB];
#pragma unroll
        for (int b = 0; b < RB; b++) {
            if (some)
#pragma unroll
                for (int i = 0; i < 8; i++)
                    s[b][i / 4][i % 4] = or_none(s[b][i / 4][i % 4], row[b].limit - 1 - (j0 + i / 4 * 16 + quarter * 4 + i % 4));
            float top = s[b][0][0];
#pragma unroll
            for (int i = 1; i < 8; i++) top = fmaxf(top, s[b][i / 4][i % 4]);
            top = quarter_most(top);
            if (__any(top > base[b] + rise)) {
                const float higher = fmaxf(base[b], top), less = higher == base[b] ? 1.f : power((base[b] - higher) * c);
                base[b] = higher, sum[b] *= less;
#pragma unroll
                for (int dt = 0; dt < 2 * ND; dt++)
#pragma unroll
                    for (int i = 0; i < 4; i++) o[b][dt][i] *= less;
            }
            const float zero = base[b] == -INFINITY ? 0.f : base[b] * c;
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float e = power(fmaf(s[b][i / 4][i % 4], c, -zero));
                sum[b] += e;
                p[b][i] = T(e);
            }
        }
#pragma unroll
        for (int dt = 0; dt < 2 * ND; dt++)
#pragma unroll
            for (int b = 0; b < RB; b++) o[b][dt] = product16(v[dt], p[b], o[b][dt]);
    }
    // Joined by way of LDS: [wave][row][d], and their bases and totals.
    own_landed<0>();
    __syncthreads();
    constexpr int PITCH = ND * 32 + 4;      // floats of a row: 16 rows' four values from one column on begin in other banks
    float* const sums = reinterpret_cast<float*>(lds);
    __shared__ float bases[4][ROWS], totals[4][ROWS];
    if (lane == 0) cleansed[wave] = found;
#pragma unroll
    for (int b = 0; b < RB; b++) {
        const float total = quarter_sum(sum[b]);
        if (quarter == 0) bases[wave][b * 16 + li] = base[b], totals[wave][b * 16 + li] = total;
#pragma unroll
        for (int dt = 0; dt < 2 * ND; dt++) *reinterpret_cast<f32x4*>(sums + (wave * ROWS + b * 16 + li) * PITCH + dt * 16 + quarter * 4) = o[b][dt];
    }
    __syncthreads();
    for (int i = threadIdx.x; i < ROWS * ND * 8; i += 256) {
        const int r = i / (ND * 8), x = i % (ND * 8) * 4;
        const Row it = row_of(at.first + r, m, n, a.shared, a.causal);
        if (!it.there) continue;
        float top = bases[0][r], total = 0.f, v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 1; w < 4; w++) top = fmaxf(top, bases[w][r]);
#pragma unroll
        for (int w = 0; w < 4; w++) {
            // a wavefront without keys has base -inf: nothing
            const float less = bases[w][r] == -INFINITY ? 0.f : power((bases[w][r] - top) * c);
            if (bases[w][r] == -INFINITY && totals[w][r] == 0.f) continue;
            total += totals[w][r] * less;
            const f32x4 part = *reinterpret_cast<const f32x4*>(sums + (w * ROWS + r) * PITCH + x);
#pragma unroll
            for (int e = 0; e < 4; e++) v[e] += part[e] * less;
        }
        const Leave<T, KV> leave(a, at.rows.first + it.token, hk * a.shared + it.head);
        leave.template four<WIDE>(x, a.d, v, total == 0.f ? 0.f : 1.f / total);
        if (x == 0) leave.total(top, total, a.scale);
        if (cleansed[0] | cleansed[1] | cleansed[2] | cleansed[3])
            for (int32_t j = max(begin, least / FEW_KEYS * FEW_KEYS); j < min(it.limit, end); j++) {
                const T* const from = kv.any_value(j);
                for (int e = 0; from && e < 4; e++)
                    if (x + e < a.d && !finite(float(from[x + e]))) leave.more(x + e, float(from[x + e]));
            }
    }
}

// The parts of a row that workgroups left, one for each `chunk` keys that it sees: one wavefront per row and head.
template <typename T, typename KV> __global__ __launch_bounds__(256) void k_join(Attend<T, KV> a) {
    const int64_t at = workgroup() * 4 + (threadIdx.x >> 6);
    if (at >= int64_t(a.rows) * a.heads) return;
    const int32_t row = __builtin_amdgcn_readfirstlane(int32_t(at / a.heads)), h = __builtin_amdgcn_readfirstlane(int32_t(at % a.heads)), lane = threadIdx.x & 63;
    Span rows;
    const int32_t s = last_of(a.q_offset, a.sequences, a.rows, rows, [&](int32_t begin, int32_t) { return begin <= row; });
    if (s < 0 || row >= rows.first + rows.count) return;
    const auto kv = a.kv.one(s, 0);
    const int32_t limit = seen(a.causal, row - rows.first, rows.count, kv.count), parts = (limit + a.chunk - 1) / a.chunk;
    const int64_t step = int64_t(a.rows) * a.heads;
    const float* const stats = a.stats + at * 2;
    const float* const part = a.part + at * a.d;
    const float c = a.scale * LOG2_E;
    float top = -INFINITY, total = 0.f, v[2] = {0.f, 0.f};
    // 64 parts at a time: their bases and totals by the lanes, what they count by then one after the other
    for (int32_t i0 = 0; i0 < parts; i0 += 64) {
        const int32_t have = min(parts - i0, 64);
        const float base = lane < have ? stats[(i0 + lane) * step * 2] : -INFINITY, sum = lane < have ? stats[(i0 + lane) * step * 2 + 1] : 0.f;
        float higher = fmaxf(top, base);
#pragma unroll
        for (int e = 1; e < 64; e *= 2) higher = fmaxf(higher, __shfl_xor(higher, e));
        const float less = top == higher ? 1.f : power((top - higher) * c), weight = lane >= have ? 0.f : base == higher ? 1.f : power((base - higher) * c);
        top = higher, total = total * less + wave_sum(sum * weight), v[0] *= less, v[1] *= less;
        for (int32_t i = 0; i < have; i += 8) {
            float from[8][2];
#pragma unroll
            for (int u = 0; u < 8; u++)
#pragma unroll
                for (int e = 0; e < 2; e++) from[u][e] = lane + e * 64 < a.d ? part[(i0 + min(i + u, have - 1)) * step * a.d + lane + e * 64] : 0.f;
#pragma unroll
            for (int u = 0; u < 8; u++) {
                const float w = i + u < have ? __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(weight), i + u)) : 0.f;
#pragma unroll
                for (int e = 0; e < 2; e++) v[e] = fmaf(from[u][e], w, v[e]);
            }
        }
    }
    const float inverse = total == 0.f ? 0.f : 1.f / total;
    T* const out = a.out.p + row * a.out.row + h * a.out.head;
#pragma unroll
    for (int e = 0; e < 2; e++)
        if (lane + e * 64 < a.d) out[lane + e * 64] = T(v[e] * inverse);
    if (a.lse && lane == 0) a.lse[int64_t(h) * a.rows + row] = total == 0.f ? -INFINITY : top * a.scale + logf(total);
}

// ---------------------------------------------------------------------------------------------------------------
// Which kernel
// ---------------------------------------------------------------------------------------------------------------
struct Plan {
    int blocks;             // of 16 rows: few rows; 0: many
    int sides;              // many rows: wavefronts that share a row's keys, 128 / sides rows to a workgroup
    int64_t tiles, chunk, chunks;
};
// By the rows that a sequence has on average (the host does not know each): 64 are where few rows' kernel ends (sequences of 131 to 420 rows
// by it 38 -> 138 us, by 32 rows to a workgroup 86).  The keys are split where there are not enough workgroups, into parts of 256 or 512 and more, for about 2048
// of them (chunks up to 700 over 2000 to 12000 tokens: 457 us unsplit, 453 for 1024, 407 for 2048; 48 single tokens over long histories: 519 for 2048
// and 4096, 527 for 8192; parts of 128 for 8 short ones: 23.7 against 18.6).
Plan plan_of(int64_t rows, int64_t heads, int64_t kv_heads, int64_t sequences, int64_t most_keys, bool split) {
    const int64_t shared = kv_heads ? heads / kv_heads : 1, each = (rows + sequences - 1) / sequences * shared;
    Plan p{each <= 16 ? 1 : each <= 32 ? 2 : each <= 64 ? 4 : 0, 1, 0, 0, 1};
    p.tiles = tiles_at_most(sequences, rows, shared, p.blocks == 1 ? 4 : p.blocks == 2 ? 5 : p.blocks == 4 ? 6 : MANY_SHIFT);
    if (p.blocks == 0) {
        const int64_t groups = p.tiles * kv_heads;
        p.sides = sides_of(groups);
        if (p.sides > 1) p.tiles = tiles_at_most(sequences, rows, shared, p.sides == 2 ? MANY_SHIFT - 1 : MANY_SHIFT - 2);
    }
    if (split) {
        const int64_t groups = p.tiles * kv_heads, least = p.blocks ? 256 : 512, unit = 128;
        int64_t chunk = (most_keys * groups / 2048 + unit - 1) / unit * unit;
        chunk = chunk < least ? least : chunk;
        if (chunk < most_keys) p.chunk = chunk, p.chunks = (most_keys + chunk - 1) / chunk;
    }
    return p;
}

template <typename T, typename KV> int attend(Attend<T, KV> a, const Plan& p, bool wide, hipStream_t s) {
    const int64_t groups = p.tiles * a.kv_heads;
    if (groups > MOST_SIZE || groups * 256 > UINT32_MAX) return CSR5_ERANGE;
    a.tiles = int32_t(p.tiles), a.chunk = int32_t(p.chunk);
    const dim3 grid(uint32_t(groups), uint32_t(p.chunks));
    auto go = [&](auto nd, auto w) {
        constexpr int ND = decltype(nd)::value, TILE = (ND <= 2 ? 64 : 128) * 2;
        constexpr bool WIDE = decltype(w)::value;
        auto few = [&](auto rb) {
            constexpr int RB = decltype(rb)::value, ring = 8 * FEW_KEYS * TILE, join = 4 * 16 * RB * (ND * 32 + 4) * 4;
            k_attend_few<T, KV, ND, WIDE, RB><<<grid, 256, ring > join ? ring : join, s>>>(a);
        };
        if (p.blocks == 1) few(std::integral_constant<int, 1>());
        else if (p.blocks == 2) few(std::integral_constant<int, 2>());
        else if (p.blocks == 4) few(std::integral_constant<int, 4>());
        else {
            auto many = [&](auto kg) {
                constexpr int KG = decltype(kg)::value;
                k_attend_many<T, KV, ND, WIDE, KG><<<grid, 256, 4 * KG * MANY_KEYS * TILE + 16, s>>>(a);
            };
            if (p.sides == 4) many(std::integral_constant<int, 4>());
            else if (p.sides == 2) many(std::integral_constant<int, 2>());
            else many(std::integral_constant<int, 1>());
        }
    };
    auto by = [&](auto nd) {
        if (wide) go(nd, std::true_type());
        else go(nd, std::false_type());
    };
    if (a.d <= 64) by(std::integral_constant<int, 2>());
    else if (a.d <= 96) by(std::integral_constant<int, 3>());
    else by(std::integral_constant<int, 4>());
    if constexpr (!KV::One::PACKED)         // packed keys are not split
        if (p.chunk) k_join<T, KV><<<workgroups((int64_t(a.rows) * a.heads + 3) / 4), 256, 0, s>>>(a);
    return launched();
}

}  // namespace

extern "C" {

int csr5_attention(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset,
                   const int32_t* k_offset, float scale, int causal, csr5_heads_t q, csr5_heads_t k, csr5_heads_t v, csr5_heads_t out, float* lse, void* hip_stream) {
    if (const int bad = attention_sizes(sequences, rows, k_rows, heads, kv_heads, d, dtype, scale)) return bad;
    if (!heads_ok(q, rows, heads, d, 2) || !heads_ok(k, k_rows, kv_heads, d, 2) || !heads_ok(v, k_rows, kv_heads, d, 2) || !output_ok(out, rows, heads, d, 2)) return CSR5_EINVAL;
    if (!words({q_offset, k_offset, lse})) return CSR5_EINVAL;
    if (sequences == 0 || rows == 0 || heads == 0) return CSR5_OK;
    if (!q_offset || !k_offset) return CSR5_EINVAL;
    const Plan p = plan_of(rows, heads, kv_heads, sequences, k_rows, false);
    const bool w = d % 8 == 0 && wide(q, 2) && wide(k, 2) && wide(v, 2) && wide(out, 2);
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        const Attend<T, Packed<T>> a{sequences, rows, heads, kv_heads, heads / kv_heads, d, q_offset, scale, causal != 0, typed<const T>(q), {k_offset, k_rows, typed<const T>(k), typed<const T>(v)},
                                     typed<T>(out), lse, 0, 0, nullptr, nullptr};
        return attend(a, p, w, static_cast<hipStream_t>(hip_stream));
    });
}

size_t csr5_attention_paged_workspace_bytes(int32_t rows, int32_t heads, int32_t kv_heads, int32_t d, int32_t sequences, int64_t max_length) {
    if (rows <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads || d < 0 || sequences <= 0 || max_length < 0 || max_length > CSR5_ATTENTION_MAX_ROWS) return 0;
    const Plan p = plan_of(rows, heads, kv_heads, sequences, max_length, true);
    return p.chunk ? size_t(p.chunks) * size_t(rows) * size_t(heads) * size_t(d + 2) * 4 : 0;
}

int csr5_attention_paged(int32_t sequences, int32_t rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset, const int32_t* length,
                         const int32_t* table, int32_t width, int64_t ldt, int32_t pages, int32_t page, float scale, csr5_heads_t q, csr5_cache_t k_cache, csr5_cache_t v_cache,
                         csr5_heads_t out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = attention_sizes(sequences, rows, 0, heads, kv_heads, d, dtype, scale)) return bad;
    if (width < 0 || pages < 0 || !power_of_two(page)) return CSR5_EINVAL;
    if (int64_t(width) * page > CSR5_ATTENTION_MAX_ROWS) return CSR5_ERANGE;
    if (!heads_ok(q, rows, heads, d, 2) || !output_ok(out, rows, heads, d, 2) || !cache_ok(k_cache, pages, page, kv_heads, d, 2) || !cache_ok(v_cache, pages, page, kv_heads, d, 2) ||
        !rows_ok(table, sequences, ldt, width, 4))
        return CSR5_EINVAL;
    if (!words({q_offset, length, lse, workspace})) return CSR5_EINVAL;
    if (sequences == 0 || rows == 0 || heads == 0) return CSR5_OK;
    if (!q_offset || !length) return CSR5_EINVAL;
    const int64_t most = int64_t(width) * page;
    const size_t need = csr5_attention_paged_workspace_bytes(rows, heads, kv_heads, d, sequences, most);
    if (need && (!workspace || workspace_bytes < need)) return CSR5_ENOMEM;
    const Plan p = plan_of(rows, heads, kv_heads, sequences, most, true);
    const bool w = d % 8 == 0 && wide(q, 2) && wide(k_cache, 2) && wide(v_cache, 2) && wide(out, 2);
    float* const part = static_cast<float*>(workspace);
    float* const stats = p.chunk ? part + size_t(p.chunks) * size_t(rows) * size_t(heads) * size_t(d) : nullptr;
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        const Attend<T, Paged<T>> a{sequences, rows, heads, kv_heads, heads / kv_heads, d, q_offset, scale, true, typed<const T>(q),
                                    {length, table, width, pages, __builtin_ctz(page), ldt, typed<const T>(k_cache), typed<const T>(v_cache)}, typed<T>(out), lse, 0, 0, part, stats};
        return attend(a, p, w, static_cast<hipStream_t>(hip_stream));
    });
}

}  // extern "C"
