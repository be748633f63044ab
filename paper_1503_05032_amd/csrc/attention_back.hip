// libcsr5: the gradients of attention over packed sequences.  The C ABI is declared in include/csr5.h.
//
// With p = 2^(c q.k - lse log2 e), c = scale log2 e, and ds = p (dout.v - delta), delta = dout.out:
//   dv = p^T dout,  dk = scale ds^T q  by workgroups that have keys and go through the queries,
//   dq = scale ds k                    by workgroups that have queries and go through the keys,
// so that every sum has one owner and one order; p is computed in both: seven products for the five that there are with one pass, whose dq would
// be added up between workgroups.  p and ds are, rounded, the second operands of the next products as the lanes have them, as in attention.hip.
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

template <typename T> struct Back {
    int32_t sequences, rows, k_rows, heads, kv_heads, shared, d;
    const int32_t *q_offset, *k_offset;
    float scale;
    bool causal;
    Heads<const T> dout, q, out, k, v;
    const float* lse;
    float *delta, *base;        // [heads][rows]: dout . out, and lse log2 e (infinity where lse is -inf)
    Heads<T> dq, dk, dv;
    int32_t tiles;
    float* part;                // sums of dk, then of dv, by workgroups that have some of the heads only: [part][2][k_rows][kv_heads][d]; NULL: there are none
};

// ---------------------------------------------------------------------------------------------------------------
// delta and base: D / 8 lanes to a row and head.  Bound by memory: 7751 x 20 heads of 128 17.5 us (4.6 TB/s).
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int LANES, bool WIDE> __global__ __launch_bounds__(256) void k_delta(Back<T> a) {
    const int64_t at = workgroup() * (256 / LANES) + threadIdx.x / LANES;
    const int c = threadIdx.x % LANES * 8;
    const bool there = at < int64_t(a.rows) * a.heads;
    const int64_t row = there ? at / a.heads : 0, h = there ? at % a.heads : 0;
    float x[8], y[8], sum = 0.f;
    load_values<8, WIDE>(a.dout.p + row * a.dout.row + h * a.dout.head + c, there ? a.d - c : 0, x);
    load_values<8, WIDE>(a.out.p + row * a.out.row + h * a.out.head + c, there ? a.d - c : 0, y);
#pragma unroll
    for (int e = 0; e < 8; e++) sum = fmaf(x[e], y[e], sum);
    sum = lanes_sum<LANES>(sum);
    if (there && c == 0) {
        const float lse = a.lse[h * a.rows + row];
        // a row whose scores are all -inf: with this base its weights are 0, as in its result
        a.delta[h * a.rows + row] = sum, a.base[h * a.rows + row] = lse == -INFINITY ? INFINITY : lse * LOG2_E;
    }
}

// Where a wavefront reads rows of LDS for products of 32 x 32 x 16: rows as first operands (chunks 2 kk on), and turned (columns 32 dt on).  Tiles begin at
// multiples of 256 bytes, so other chunks are other patterns in bits 5 to 7: one register for all of them.
template <int ND> struct Read {
    static constexpr int D = ND <= 2 ? 64 : 128;
    uint32_t row_, turned_;
    __device__ __forceinline__ Read() {
        const int lane = threadIdx.x & 63, half = lane >> 5, li = lane & 15, r = half * 4 + (li >> 2);
        row_ = (lane & 31) * D * 2 + chunk_at<D, false>(lane & 31, half) * 16;
        turned_ = r * D * 2 + chunk_at<D, false>(r, ((lane >> 4) & 1) * 2 + ((li & 3) >> 1)) * 16 + (li & 1) * 8;
    }
    __device__ __forceinline__ uint32_t row(uint32_t tile, int kk) const { return (tile + row_) ^ (kk * 32); }
    __device__ __forceinline__ uint32_t turned(uint32_t tile, int dt) const { return (tile + turned_) ^ (dt * 64); }
};

// A head's values of this lane's column, for second operands.
template <int ND, bool WIDE, typename T> __device__ __forceinline__ void column(vec<T, 8> (&to)[2 * ND], const T* from, bool there, int d) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int kk = 0; kk < 2 * ND; kk++) to[kk] = eight_values<WIDE>(from + (2 * kk + half) * 8, there ? d - (2 * kk + half) * 8 : 0);
}
// A column of a result that lies as [values][columns].
template <int ND, bool WIDE, typename T> __device__ __forceinline__ void leave(T* to, const f32x16 (&acc)[ND], float scale, int d) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int dt = 0; dt < ND; dt++)
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const int c = dt * 32 + i * 8 + half * 4;
            const float v[4] = {acc[dt][4 * i] * scale, acc[dt][4 * i + 1] * scale, acc[dt][4 * i + 2] * scale, acc[dt][4 * i + 3] * scale};
            store_values<4, WIDE>(to + c, d - c, v);
        }
}

constexpr int DQ_ROWS = 128, DQ_SHIFT = 7, DQ_STEP = 32;
constexpr int DKV_KEYS = 64, DKV_SHIFT = 6;

// ---------------------------------------------------------------------------------------------------------------
// dq: 128 folded rows (as in attention.hip), 32 to each wavefront, which go through keys and values in tiles of 32.
// 5 sequences up to 2801, 20 heads of 128 with 5 of keys: 171 us, 711 TFLOP/s of its three products.  Keys are cleansed between the scores and dq's product: 1 us.
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int ND, bool WIDE, int KG> __global__ __launch_bounds__(256, 2) void k_attend_dq(Back<T> a) {
    constexpr int D = ND <= 2 ? 64 : 128, KEYS = DQ_STEP * KG, TILE = KEYS * D * 2, ROWS = DQ_ROWS / KG;
    typedef Bring<T, D, WIDE, false, KEYS, 4> B;
    extern __shared__ __align__(16) uint8_t lds[];          // begins at 0: nothing else is in LDS, so bits of addresses can be turned over
    int32_t& cleansed = *reinterpret_cast<int32_t*>(lds + 4 * TILE);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, kg = KG == 1 ? 0 : wave / (4 / KG);
    const int32_t hk = blockIdx.x % a.kv_heads;
    TileOf at;
    if (!tile_of(a.q_offset, a.sequences, a.rows, a.shared, KG == 1 ? DQ_SHIFT : KG == 2 ? DQ_SHIFT - 1 : DQ_SHIFT - 2, a.tiles - 1 - int32_t(blockIdx.x / a.kv_heads), at)) return;
    const Span keys = span_of(a.k_offset, at.s, a.k_rows);
    const int32_t m = at.rows.count, n = keys.count;
    const Row row = row_of(at.first + wave % (4 / KG) * 32 + (lane & 31), m, n, a.shared, a.causal);
    const int32_t least = __builtin_amdgcn_readfirstlane(row.limit), most = __builtin_amdgcn_readlane(row.limit, 31);
    const int32_t end = __builtin_amdgcn_readfirstlane(row_of(at.first + ROWS - 1, m, n, a.shared, a.causal).limit);
    const int32_t fewest = __builtin_amdgcn_readfirstlane(row_of(at.first, m, n, a.shared, a.causal).limit);
    if (threadIdx.x == 0) cleansed = 0;
    const int64_t token = at.rows.first + row.token;
    const int h = hk * a.shared + row.head;
    vec<T, 8> q[2 * ND], dout[2 * ND];
    column<ND, WIDE>(q, a.q.p + token * a.q.row + h * a.q.head, row.there, a.d);
    column<ND, WIDE>(dout, a.dout.p + token * a.dout.row + h * a.dout.head, row.there, a.d);
    const float delta = a.delta[int64_t(h) * a.rows + token], base = a.base[int64_t(h) * a.rows + token], c = a.scale * LOG2_E;

    const typename Packed<T>::One kv{same(a.k.p + keys.first * a.k.row + hk * a.k.head), same(a.v.p + keys.first * a.v.row + hk * a.v.head), a.k.row, a.v.row, __builtin_amdgcn_readfirstlane(n)};
    const B bring(kv, wave, a.d);
    const int none[B::LOADS] = {};
    // LDS: two tiles of keys, then two of values
    const uint32_t lds0 = lds_address(lds);
    const ReadFixed<ND> read(lds0 + kg * DQ_STEP * D * 2);        // its 32 keys of a tile
    f32x16 dq[ND] = {};
    auto tile = [&](auto at_place, int32_t j0) {
        constexpr int NOW = decltype(at_place)::value;
        landed<0>();
        if (j0 + KEYS < end) bring(kv, j0 + KEYS, none, a.d, lds0 + (1 - NOW) * TILE, lds0 + (3 - NOW) * TILE);
        const int32_t mine = j0 + kg * DQ_STEP;             // this wavefront's keys
        const bool some = mine < most;
        vec<T, 8> ds[2];
        if (some) {
            f32x16 s = {}, dp = {};
#pragma unroll
            for (int kk = 0; kk < 2 * ND; kk++) s = product32(read.template row<T>(NOW * TILE, kk), q[kk], s);
#pragma unroll
            for (int kk = 0; kk < 2 * ND; kk++) dp = product32(read.template row<T>((2 + NOW) * TILE, kk), dout[kk], dp);
#pragma unroll
            for (int i = 0; i < 16; i++) s[i] = power(fmaf(s[i], c, -base)) * (dp[i] - delta);
            if (mine + DQ_STEP > least) {
#pragma unroll
                for (int i = 0; i < 16; i++) s[i] = or_zero(s[i], row.limit - 1 - (mine + 8 * (i / 4) + 4 * half + i % 4));
            }
#pragma unroll
            for (int i = 0; i < 16; i++) ds[i / 8][i % 8] = T(s[i]);
        }
        // Some row does not see some key: cleansed after the scores, which a key's values decide as they are (one of -inf may make its p 0).
        if (j0 + KEYS > fewest && fewest < n) {
            __syncthreads();
            if (cleanse<T>(lds + NOW * TILE, TILE, threadIdx.x, 256)) cleansed = 1;
            __syncthreads();
        }
        if (!some) return;
#pragma unroll
        for (int k = 0; k < 2; k++)
#pragma unroll
            for (int dt = 0; dt < ND; dt++) dq[dt] = product32(read.template turned<T>(NOW * TILE + k * 16 * D * 2, dt), ds[k], dq[dt]);
    };
    if (bring.ragged) {
        zeros_to(lds0, 4 * TILE, threadIdx.x, 256);
        landed<0>();
    }
    if (end > 0) bring(kv, 0, none, a.d, lds0, lds0 + 2 * TILE);
    for (int32_t j0 = 0; j0 < end; j0 += 2 * KEYS) {
        tile(std::integral_constant<int, 0>(), j0);
        if (j0 + KEYS < end) tile(std::integral_constant<int, 1>(), j0 + KEYS);
    }
    own_landed<0>();
    __syncthreads();
    // the sums of the wavefronts that have the same rows by way of LDS, as in attention.hip
#pragma unroll
    for (int more = KG / 2; more > 0; more /= 2) {
        float* const place = reinterpret_cast<float*>(lds) + (wave % (4 / KG) + kg % more * (4 / KG)) * (ND * 1024) + lane;
        if (kg >= more && kg < 2 * more) {
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) place[(dt * 16 + i) * 64] = dq[dt][i];
        }
        __syncthreads();
        if (kg < more) {
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) dq[dt][i] += place[(dt * 16 + i) * 64];
        }
        __syncthreads();
    }
    if (kg > 0 || !row.there) return;
    T* const to = a.dq.p + token * a.dq.row + h * a.dq.head;
    leave<ND, WIDE>(to, dq, a.scale, a.d);
    // a key that is not finite makes the values of dq not finite that it has so; the others have had it by way of the scores
    if (cleansed)
        for (int32_t j = fewest / KEYS * KEYS; j < row.limit; j++)
            for (int i = 0; i < 16 * ND; i++) {
                const int x = i / 4 * 8 + half * 4 + i % 4;
                if (x < a.d && !finite(float(kv.any_key(j)[x]))) to[x] = T(NAN);
            }
}

// ---------------------------------------------------------------------------------------------------------------
// dk and dv: 64 keys to a workgroup, which go through the queries that see them in tiles of 32 RG, head by head of those that share the keys: each
// wavefront has 32 of the keys and takes 32 of the queries, and what RG of them have of the same keys is added up in the end.  (With 128 keys, 32 to a
// wavefront and all queries, there are half as many workgroups and the first keys' are twice as long.)  5 sequences up to 2801, 20 heads of 128 with 5 of keys: 330 us,
// 489 TFLOP/s of its four products; 557 with 128 keys and one wavefront to a SIMD, whose accumulators went to and fro between the two halves of the registers.
// Scores are computed as queries x keys, so that a lane has a key's column of p and ds.
// ---------------------------------------------------------------------------------------------------------------
template <typename T, int ND, bool WIDE, int RG> __global__ __launch_bounds__(128 * RG, 2) void k_attend_dkv(Back<T> a) {
    constexpr int DKV_STEP = 32 * RG, WAVES = 2 * RG;
    constexpr int D = ND <= 2 ? 64 : 128, TILE = DKV_STEP * D * 2, STAGE = 2 * TILE + DKV_STEP * 8;
    typedef Bring<T, D, WIDE, false, DKV_STEP, WAVES> B;
    extern __shared__ __align__(16) uint8_t lds[];          // begins at 0
    int32_t& cleansed = *reinterpret_cast<int32_t*>(lds + 2 * STAGE);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), half = lane >> 5, rb = wave >> 1;
    const int32_t hk = blockIdx.x % a.kv_heads;
    TileOf at;
    if (!tile_of(a.k_offset, a.sequences, a.k_rows, 1, DKV_SHIFT, blockIdx.x / a.kv_heads, at)) return;
    const Span mine = span_of(a.q_offset, at.s, a.rows);
    const int32_t m = mine.count, n = at.rows.count, first = int32_t(at.first) + (wave & 1) * 32, key = first + (lane & 31);
    const bool there = key < n;
    const int64_t token = at.rows.first + min(key, n - 1);
    vec<T, 8> k[2 * ND], v[2 * ND];
    column<ND, WIDE>(k, a.k.p + token * a.k.row + hk * a.k.head, there, a.d);
    column<ND, WIDE>(v, a.v.p + token * a.v.row + hk * a.v.head, there, a.d);
    const float c = a.scale * LOG2_E;
    // query i sees key j where j <= i + ahead
    const int32_t ahead = a.causal ? n - m : n;         // sums of two are below 2^31
    const int32_t whole = max(0, int32_t(at.first) + DKV_KEYS - 1 - ahead);      // the first query that sees all of the workgroup's keys
    if (threadIdx.x == 0) cleansed = 0;
    const int32_t start = max(0, int32_t(at.first) - ahead) / DKV_STEP * DKV_STEP, steps = m > start ? (m - start + DKV_STEP - 1) / DKV_STEP : 0;

    // the heads of this workgroup, of those that share the keys
    const int first_head = int(int64_t(blockIdx.y) * a.shared / gridDim.y), last_head = int(int64_t(blockIdx.y + 1) * a.shared / gridDim.y);
    // the queries of a head, and their dout, as rows side by side
    auto of = [&](int h) {
        return typename Packed<T>::One{same(a.q.p + mine.first * a.q.row + h * a.q.head), same(a.dout.p + mine.first * a.dout.row + h * a.dout.head), a.q.row, a.dout.row, __builtin_amdgcn_readfirstlane(m)};
    };
    const B bring(of(hk * a.shared), wave, a.d);
    const int none[B::LOADS] = {};
    const uint32_t lds0 = lds_address(lds);
    auto load = [&](int h, int32_t i0, uint32_t to) {
        bring(of(h), i0, none, a.d, to, to + TILE);
        // base, and delta: a wavefront for each 64
        const int32_t i = i0 + wave % (RG / 2) * 64 + lane;
        if (wave < RG) word_to_lds(i < m ? static_cast<const void*>((wave < RG / 2 ? a.base : a.delta) + int64_t(h) * a.rows + mine.first + i) : &ZEROS, lds + (to - lds0) + 2 * TILE + wave * 256);
    };
    const Read<ND> read;
    f32x16 dk[ND] = {}, dv[ND] = {};
    // the step that is loaded next
    int h = hk * a.shared + first_head;
    int32_t i1 = start;
    const int32_t total = steps * (last_head - first_head);
    auto load_next = [&](uint32_t to) {
        load(h, i1, to);
        if ((i1 += DKV_STEP) >= m) i1 = start, h++;
    };
    if (bring.ragged) {
        zeros_to(lds0, 2 * STAGE, threadIdx.x, 128 * RG);
        landed<0>();
    }
    if (total > 0) load_next(lds0);
    int now = 0;
    int32_t i0 = start;
    for (int32_t step = 0; step < total; step++, now ^= 1, i0 = i0 + DKV_STEP < m ? i0 + DKV_STEP : start) {
        landed<0>();
        if (i0 < whole && i0 + ahead < n - 1) {             // some query does not see some key
            if (cleanse<T>(lds + now * STAGE, 2 * TILE, threadIdx.x, 128 * RG)) cleansed = 1;
            __syncthreads();
        }
        if (step + 1 < total) load_next(lds0 + (now ^ 1) * STAGE);
        const int32_t i = i0 + rb * 32;
        if (i >= m || i + 31 + ahead < first) continue;     // no query, or none that sees one of these keys
        const uint32_t tile = lds0 + now * STAGE + rb * 32 * D * 2, words = lds0 + now * STAGE + 2 * TILE + rb * 128 + half * 16;
        f32x16 s = {}, dp = {};
#pragma unroll
        for (int kk = 0; kk < 2 * ND; kk++) s = product32(chunk_from<T>(read.row(tile, kk)), k[kk], s);
#pragma unroll
        for (int kk = 0; kk < 2 * ND; kk++) dp = product32(chunk_from<T>(read.row(tile + TILE, kk)), v[kk], dp);
        // all 256 registers are in use: without these borders, loads that are moved up put 45 of them into memory
        __builtin_amdgcn_sched_barrier(0);
        vec<T, 8> p[2], ds[2];
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const f32x4 base = *(const __attribute__((address_space(3))) f32x4*)uintptr_t(words + e * 32), delta = *(const __attribute__((address_space(3))) f32x4*)uintptr_t(words + DKV_STEP * 4 + e * 32);
#pragma unroll
            for (int u = 0; u < 4; u++) {
                const int w = e * 4 + u;
                s[w] = power(fmaf(s[w], c, -base[u])), dp[w] = s[w] * (dp[w] - delta[u]);
            }
        }
        if (i + ahead < first + 31 || i + 32 > m) {         // some query does not see some key; or there is none
#pragma unroll
            for (int w = 0; w < 16; w++) {
                const int32_t r = i + 8 * (w / 4) + 4 * half + w % 4, unseen = (m - 1 - r) | (r + ahead - key);
                s[w] = or_zero(s[w], unseen), dp[w] = or_zero(dp[w], unseen);
            }
        }
#pragma unroll
        for (int w = 0; w < 16; w++) p[w / 8][w % 8] = T(s[w]), ds[w / 8][w % 8] = T(dp[w]);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int x = 0; x < 2; x++)
#pragma unroll
            for (int dt = 0; dt < ND; dt++) {
                dv[dt] = product32(turned32<D, T>(read.turned(tile + TILE + x * 16 * D * 2, dt)), p[x], dv[dt]);
                dk[dt] = product32(turned32<D, T>(read.turned(tile + x * 16 * D * 2, dt)), ds[x], dk[dt]);
            }
    }
    own_landed<0>();
    __syncthreads();
    // the sums of the wavefronts that have the same keys by way of LDS: the upper half's to the lower's, until one has them all
#pragma unroll
    for (int more = RG / 2; more > 0; more /= 2) {
        float* const sums = reinterpret_cast<float*>(lds) + ((wave & 1) + rb % more * 2) * (ND * 2048) + lane;
        if (rb >= more && rb < 2 * more) {
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) sums[(dt * 16 + i) * 64] = dk[dt][i], sums[(dt * 16 + i) * 64 + ND * 1024] = dv[dt][i];
        }
        __syncthreads();
        if (rb < more) {
#pragma unroll
            for (int dt = 0; dt < ND; dt++)
#pragma unroll
                for (int i = 0; i < 16; i++) dk[dt][i] += sums[(dt * 16 + i) * 64], dv[dt][i] += sums[(dt * 16 + i) * 64 + ND * 1024];
        }
        __syncthreads();
    }
    if (rb > 0 || !there) return;
    T *const to_k = a.dk.p + token * a.dk.row + hk * a.dk.head, *const to_v = a.dv.p + token * a.dv.row + hk * a.dv.head;
    const int64_t step = int64_t(a.k_rows) * a.kv_heads * a.d;
    float* const part = a.part ? a.part + blockIdx.y * 2 * step + (token * a.kv_heads + hk) * a.d : nullptr;
    if (part) {
#pragma unroll
        for (int dt = 0; dt < ND; dt++)
#pragma unroll
            for (int i = 0; i < 16; i++) {
                const int x = dt * 32 + i / 4 * 8 + half * 4 + i % 4;
                if (x < a.d) part[x] = dk[dt][i], part[step + x] = dv[dt][i];
            }
    } else {
        leave<ND, WIDE>(to_k, dk, a.scale, a.d);
        leave<ND, WIDE>(to_v, dv, 1.f, a.d);
    }
    if (!cleansed) return;
    // a query that is not finite makes all of dk and dv so of the keys that it sees (where its scores are all -inf: the values of dk that it has so), a dout that is not all
    // of dk, and the values of dv that it has so
    for (int g = first_head; g < last_head; g++)
        for (int32_t i = max(start, key - ahead); i < min(m, start + (whole - start + DKV_STEP - 1) / DKV_STEP * DKV_STEP); i++) {
            const T *const q = a.q.p + (mine.first + i) * a.q.row + (hk * a.shared + g) * a.q.head, *const o = a.dout.p + (mine.first + i) * a.dout.row + (hk * a.shared + g) * a.dout.head;
            bool bad_q = false, bad_o = false;
            for (int x = 0; x < a.d; x++) bad_q = bad_q || !finite(float(q[x])), bad_o = bad_o || !finite(float(o[x]));
            if (!bad_q && !bad_o) continue;
            const bool none = a.base[int64_t(hk * a.shared + g) * a.rows + mine.first + i] == INFINITY;      // all its weights are 0
            for (int e = 0; e < 16 * ND; e++) {
                const int x = e / 4 * 8 + half * 4 + e % 4;
                if (x >= a.d) continue;
                const float of_v = bad_q && !none ? NAN : finite(float(o[x])) ? 0.f : none ? NAN : float(o[x]);
                const float of_k = bad_o || !none || !finite(float(q[x])) ? NAN : 0.f;
                if (part) part[x] += of_k, part[step + x] += of_v;
                else to_k[x] = T(float(to_k[x]) + of_k), to_v[x] = T(float(to_v[x]) + of_v);
            }
        }
}

// The parts of dk and dv, added up in their order: a wavefront for each key and head.
template <typename T> __global__ __launch_bounds__(256) void k_add(Back<T> a, int parts) {
    const int64_t at = workgroup() * 4 + (threadIdx.x >> 6);
    if (at >= int64_t(a.k_rows) * a.kv_heads) return;
    const int32_t row = __builtin_amdgcn_readfirstlane(int32_t(at / a.kv_heads)), hk = __builtin_amdgcn_readfirstlane(int32_t(at % a.kv_heads)), lane = threadIdx.x & 63;
    Span keys;
    const int32_t s = last_of(a.k_offset, a.sequences, a.k_rows, keys, [&](int32_t begin, int32_t) { return begin <= row; });
    if (s < 0 || row >= keys.first + keys.count) return;
    const int64_t step = int64_t(a.k_rows) * a.kv_heads * a.d;
    for (int x = lane; x < a.d; x += 64) {
        float dk = 0.f, dv = 0.f;
        for (int p = 0; p < parts; p++) dk += a.part[p * 2 * step + at * a.d + x], dv += a.part[(p * 2 + 1) * step + at * a.d + x];
        a.dk.p[row * a.dk.row + hk * a.dk.head + x] = T(dk * a.scale), a.dv.p[row * a.dv.row + hk * a.dv.head + x] = T(dv);
    }
}

// Workgroups that have the same keys and some of the heads each, where there are few workgroups and many heads share keys: dk and dv are then added up
// from their parts, in 32 bits in the workspace.  (One sequence of 3549, 16 heads of 80 with one of keys, 56 workgroups: all
// gradients and the attention 1275 us, 464 in ten parts.)
constexpr size_t MOST_PARTS = size_t(32) << 20;
int parts_of(int64_t groups, int64_t shared, int64_t k_values, size_t room) {
    if (groups > 256 || groups == 0 || shared < 2 || k_values == 0) return 1;
    int64_t parts = (512 + groups - 1) / groups;
    const int64_t fit = int64_t(room) / (k_values * 8);
    parts = parts < shared ? parts : shared, parts = parts < fit ? parts : fit;
    return parts < 2 ? 1 : int(parts);
}

}  // namespace

extern "C" {

size_t csr5_attention_backward_workspace_bytes(int32_t rows, int32_t heads) {
    if (rows <= 0 || heads <= 0) return 0;
    const size_t all = size_t(rows) * size_t(heads), parts = all * 1024;        // of all heads, with as many keys as queries and 128 values to a head
    return all * 8 + (parts < MOST_PARTS ? parts : MOST_PARTS);
}

int csr5_attention_backward(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset,
                            const int32_t* k_offset, float scale, int causal, csr5_heads_t dout, csr5_heads_t q, csr5_heads_t k, csr5_heads_t v, csr5_heads_t out,
                            const float* lse, csr5_heads_t dq, csr5_heads_t dk, csr5_heads_t dv, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = attention_sizes(sequences, rows, k_rows, heads, kv_heads, d, dtype, scale)) return bad;
    if (!heads_ok(q, rows, heads, d, 2) || !heads_ok(k, k_rows, kv_heads, d, 2) || !heads_ok(v, k_rows, kv_heads, d, 2) || !heads_ok(out, rows, heads, d, 2) ||
        !heads_ok(dout, rows, heads, d, 2) || !output_ok(dq, rows, heads, d, 2) || !output_ok(dk, k_rows, kv_heads, d, 2) || !output_ok(dv, k_rows, kv_heads, d, 2))
        return CSR5_EINVAL;
    if (!words({q_offset, k_offset, lse, workspace})) return CSR5_EINVAL;
    if (sequences == 0 || kv_heads == 0 || d == 0 || (rows == 0 && k_rows == 0)) return CSR5_OK;
    const bool queries_there = rows > 0 && heads > 0;        // without them dk and dv are 0
    if (!q_offset || !k_offset || (queries_there && !lse)) return CSR5_EINVAL;
    if (queries_there && (!workspace || workspace_bytes < csr5_attention_backward_workspace_bytes(rows, heads))) return CSR5_ENOMEM;
    const int64_t wide_tiles = tiles_at_most(sequences, rows, heads / kv_heads, DQ_SHIFT);
    const int sides = sides_of(wide_tiles * kv_heads);
    const int64_t q_tiles = tiles_at_most(sequences, rows, heads / kv_heads, sides == 1 ? DQ_SHIFT : sides == 2 ? DQ_SHIFT - 1 : DQ_SHIFT - 2), k_tiles = tiles_at_most(sequences, k_rows, 1, DKV_SHIFT);
    if (q_tiles * kv_heads * 256 > UINT32_MAX || k_tiles * kv_heads * 256 > UINT32_MAX) return CSR5_ERANGE;
    const size_t room = csr5_attention_backward_workspace_bytes(rows, heads) - size_t(rows) * size_t(heads) * 8;
    const int parts = !queries_there ? 1 : parts_of(k_tiles * kv_heads, heads / kv_heads, int64_t(k_rows) * kv_heads * d, room);
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    const bool w = d % 8 == 0 && wide(q, 2) && wide(k, 2) && wide(v, 2) && wide(out, 2) && wide(dout, 2) && wide(dq, 2) && wide(dk, 2) && wide(dv, 2);
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        float* const delta = static_cast<float*>(workspace);
        const Back<T> a{sequences, rows, k_rows, heads, kv_heads, heads / kv_heads, d, q_offset, k_offset, scale, causal != 0, typed<const T>(dout), typed<const T>(q), typed<const T>(out),
                        typed<const T>(k), typed<const T>(v), lse, delta, delta + size_t(rows) * size_t(heads), typed<T>(dq), typed<T>(dk), typed<T>(dv), int32_t(q_tiles),
                        parts > 1 ? delta + 2 * size_t(rows) * size_t(heads) : nullptr};
        auto go = [&](auto nd, auto is_wide) {
            constexpr int ND = decltype(nd)::value, D = ND <= 2 ? 64 : 128;
            constexpr bool WIDE = decltype(is_wide)::value;
            if (queries_there) {
                k_delta<T, D / 8, WIDE><<<workgroups((int64_t(rows) * heads + 2048 / D - 1) / (2048 / D)), 256, 0, s>>>(a);
                auto queries = [&](auto kg) {
                    constexpr int KG = decltype(kg)::value;
                    k_attend_dq<T, ND, WIDE, KG><<<uint32_t(q_tiles * kv_heads), 256, 4 * KG * DQ_STEP * D * 2 + 16, s>>>(a);
                };
                if (sides == 4) queries(std::integral_constant<int, 4>());
                else if (sides == 2) queries(std::integral_constant<int, 2>());
                else queries(std::integral_constant<int, 1>());
            }
            auto keys = [&](auto rg) {
                constexpr int RG = decltype(rg)::value, STEP = 32 * RG;
                k_attend_dkv<T, ND, WIDE, RG><<<dim3(uint32_t(k_tiles * kv_heads), parts), 128 * RG, 4 * STEP * D * 2 + 16 * STEP + 16, s>>>(a);
            };
            if (k_rows > 0) {
                // long sequences of few workgroups: what the longest takes counts (5 sequences up to 2801, 5 heads of keys: 618 us for 657, all gradients; 9 up
                // to 1025, 12 heads: 128 for 121)
                if (rows > 96 * int64_t(sequences) && k_tiles * kv_heads * parts <= 768) keys(std::integral_constant<int, 4>());
                else keys(std::integral_constant<int, 2>());
                if (parts > 1) k_add<T><<<workgroups((int64_t(k_rows) * kv_heads + 3) / 4), 256, 0, s>>>(a, parts);
            }
        };
        auto by = [&](auto nd) {
            if (w) go(nd, std::true_type());
            else go(nd, std::false_type());
        };
        if (d <= 64) by(std::integral_constant<int, 2>());
        else if (d <= 96) by(std::integral_constant<int, 3>());
        else by(std::integral_constant<int, 4>());
        return launched();
    });
}

}  // extern "C"
