// Packed sequences, paged caches and the tiles of keys and values that the attention's kernels take through LDS.
#ifndef CSR5_SEQUENCES_H
#define CSR5_SEQUENCES_H

#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <initializer_list>
#include <type_traits>

#include "csr5.h"
#include "heads.h"
#include "numbers.h"
#include "to_lds.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

constexpr float LOG2_E = 1.44269504088896340736f, LN_2 = 0.69314718055994530942f;

struct Span {
    int32_t first, count;
};
// Rows of sequence s.  Whatever the offsets hold, these are rows that there are.
__device__ __forceinline__ int32_t begin_of(const int32_t* offset, int32_t s, int32_t rows) { return min(max(offset[s], 0), rows); }
__device__ __forceinline__ Span span_of(const int32_t* offset, int32_t s, int32_t rows) {
    const int32_t a = begin_of(offset, s, rows), b = begin_of(offset, s + 1, rows);
    return {a, max(b - a, 0)};
}

// Sequences in tiles of 2^SHIFT of their rows times `times` (heads that share): sequence s has the tiles from
// (begin * times >> SHIFT) + s on, as many as it needs or one more, so that no sum over the sequences before it is needed and
// the host knows how many there are at most.
inline int64_t tiles_at_most(int64_t sequences, int64_t rows, int64_t times, int shift) { return (rows * times >> shift) + sequences; }

// The sequence that has tile t and where in it the tile begins, by all lanes of a wavefront: 64 sequences at a time are looked at.
// Whatever the offsets hold, the tile begins before the end of the sequence's rows, or false is returned.
struct TileOf {
    int32_t s;
    Span rows;
    int64_t first;          // of rows.count * times
};
__device__ __forceinline__ bool tile_of(const int32_t* offset, int32_t sequences, int32_t rows, int64_t times, int shift, int64_t t, TileOf& out) {
    const int lane = threadIdx.x & 63;
    int32_t low = 0, count = sequences;
    for (;;) {
        const int32_t step = (count + 63) / 64;
        const int64_t i = int64_t(low) + int64_t(lane) * step;
        const bool before = int64_t(lane) * step < count && (int64_t(begin_of(offset, int32_t(i), rows)) * times >> shift) + i <= t;
        const uint64_t votes = __ballot(before);
        if (!votes) return false;
        const int last = 63 - __builtin_clzll(votes);
        low += last * step, count = min(step, count - last * step);
        if (step == 1) break;
    }
    out.s = __builtin_amdgcn_readfirstlane(low);
    out.rows = span_of(offset, out.s, rows);
    out.first = (t - ((int64_t(out.rows.first) * times >> shift) + out.s)) << shift;
    return out.first >= 0 && out.first < int64_t(out.rows.count) * times;
}

// Keys and values of one sequence and head, packed or in a cache: where row j of either is.
template <typename T> struct Packed {
    const int32_t* offset;
    int32_t rows;
    Heads<const T> k, v;
    struct One {
        const T *k, *v;
        int64_t k_row, v_row;
        int32_t count;
        // What is looked up ahead of a row's loads (a packed row needs nothing).
        struct Ahead {};
        __device__ __forceinline__ Ahead ahead(int32_t) const { return {}; }
        __device__ __forceinline__ const T* key(int32_t j, Ahead) const { return k + j * k_row; }
        __device__ __forceinline__ const T* value(int32_t j, Ahead) const { return v + j * v_row; }
    };
    __device__ __forceinline__ One one(int32_t s, int32_t h) const {
        const Span at = span_of(offset, s, rows);
        return {same(k.p + at.first * k.row + h * k.head), same(v.p + at.first * v.row + h * v.head), k.row, v.row, at.count};
    }
};
template <typename T> struct Paged {
    const int32_t *length, *table;
    int32_t width, pages, shift;
    int64_t ldt;
    Cache<const T> k, v;
    struct One {
        const int32_t* table;
        int32_t pages, shift;
        const T *k, *v;
        int64_t k_page, k_row, v_page, v_row;
        int32_t count;
        typedef int32_t Ahead;      // the page; -1: a row of zeros
        __device__ __forceinline__ int32_t ahead(int32_t j) const {
            const int32_t page = j < count ? table[j >> shift] : -1;
            return uint32_t(page) < uint32_t(pages) ? page : -1;
        }
        __device__ __forceinline__ const T* key(int32_t j, int32_t page) const { return page < 0 ? nullptr : k + page * k_page + (j & ((1 << shift) - 1)) * k_row; }
        __device__ __forceinline__ const T* value(int32_t j, int32_t page) const { return page < 0 ? nullptr : v + page * v_page + (j & ((1 << shift) - 1)) * v_row; }
    };
    __device__ __forceinline__ One one(int32_t s, int32_t h) const {
        return {same(table + s * ldt), pages, shift, same(k.p + h * k.head), same(v.p + h * v.head), k.page, k.row, v.page, v.row, int32_t(min(int64_t(max(length[s], 0)), int64_t(width) << shift))};
    }
};

// Keys that query i of m sees, of n.
__device__ __forceinline__ int32_t seen(bool causal, int32_t i, int32_t m, int32_t n) { return causal ? min(max(n - m + i + 1, 0), n) : n; }

__device__ __forceinline__ float power(float v) { return __builtin_amdgcn_exp2f(v); }

// A row of the folded ones, its query and the keys that it sees.
struct Row {
    int32_t token, head, limit;
    bool there;
};
__device__ __forceinline__ Row row_of(int64_t r, int32_t m, int32_t n, int32_t shared, bool causal) {
    const int64_t count = int64_t(m) * shared, at = r < count ? r : count - 1;
    Row x;
    if (at >> 32) {
        x.token = int32_t(at / shared), x.head = int32_t(at % shared);
    } else {
        x.token = int32_t(uint32_t(at) / uint32_t(shared)), x.head = int32_t(uint32_t(at) % uint32_t(shared));
    }
    x.limit = seen(causal, x.token, m, n), x.there = r < count;
    return x;
}

// ---------------------------------------------------------------------------------------------------------------
// Matrix instructions, 16 bits in and 32 out.  Of 32 x 32 x 16 (16 x 16 x 32) a lane has row (column) lane % 32 (16) of the first
// (second) operand, values 8 * (lane / 32 (16)) to + 7 of the depth; of the result column lane % 32 (16), and rows 8 * (i / 4) + 4 * (lane / 32) + i % 4
// (4 * (lane / 16) + i).
// ---------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ f32x16 product32(vec<bf16, 8> a, vec<bf16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 product32(vec<f16, 8> a, vec<f16, 8> b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 product16(vec<bf16, 8> a, vec<bf16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 product16(vec<f16, 8> a, vec<f16, 8> b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// ---------------------------------------------------------------------------------------------------------------
// Tiles in LDS: rows of D values (64 or 128), 16-byte chunks c of row r swizzled so that the 64 banks are read evenly.
//   rows are read (the first operand of a product over d): 16 rows' chunk c has to be in 16 places
//   columns are read (over the rows: transposing reads of 4 rows x 16 values by 16 lanes): for 32 x 32 x 16 half a wavefront reads 64 bytes
//   of 4 rows, chunks 4g to 4g + 3; for 16 x 16 x 32 32 bytes of 8 rows, chunks 2g and 2g + 1
// SMALL false: c ^ (r % 4, r / 4 % 4) (as four bits) is both, for 32 x 32 x 16; true: c ^ (r % 8, r / 8 % 2), for 16 x 16 x 32.  Rows of 128 bytes have
// r / 2 for r, and the two of a pair are next to each other.
// ---------------------------------------------------------------------------------------------------------------
template <int D, bool SMALL> __device__ __forceinline__ uint32_t chunk_at(int r, int c) {      // where chunk c is in row r, in chunks; its own inverse
    if (D == 128) return SMALL ? c ^ ((r & 7) << 1 | (r >> 3 & 1)) : c ^ ((r & 3) << 2 | (r >> 2 & 3));
    return SMALL ? c ^ ((r >> 1 & 3) << 1 | (r >> 3 & 1)) : c ^ ((r >> 1 & 1) << 2 | (r >> 2 & 3));
}

template <typename T> __device__ __forceinline__ vec<T, 8> chunk_from(uint32_t at) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    return __builtin_bit_cast(vec<T, 8>, *(const __attribute__((address_space(3))) u32x4*)uintptr_t(at));
}
// The rows at `at` and those at `other`, four rows each of 16 columns, as a lane's eight values of one column.
template <typename T> __device__ __forceinline__ vec<T, 8> turned_from(uint32_t at, uint32_t other) {
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4* lds_ptr;
    const s16x4 low = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)uintptr_t(at)), high = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)uintptr_t(other));
    const uint2 a = __builtin_bit_cast(uint2, low), b = __builtin_bit_cast(uint2, high);
    return __builtin_bit_cast(vec<T, 8>, make_uint4(a.x, a.y, b.x, b.y));
}

// For 32 x 32 x 16: columns of four rows and of those 8 rows on, where bit 1 of a chunk's place is the other one.
template <int D, typename T> __device__ __forceinline__ vec<T, 8> turned32(uint32_t at) { return turned_from<T>(at, (at ^ 32) + 8 * D * 2); }

// One wavefront's load into LDS: 1024 bytes, lane by lane 16 of them; `from` NULL, or values from `have` on: zeros.
template <bool WIDE, typename T> __device__ __forceinline__ void chunk_to_lds(const T* from, int have, uint8_t* to) {
    if (WIDE) to_lds(from && have > 0 ? static_cast<const void*>(from) : &ZEROS, to);
    else *reinterpret_cast<vec<T, 8>*>(to + (threadIdx.x & 63) * 16) = eight_values<false>(from, from ? have : 0);
}

// The largest magnitude of 16-bit values, in pairs of them: whether one is not finite.
template <typename T> constexpr uint32_t NOT_FINITE = std::is_same<T, f16>::value ? 0x7c00u : 0x7f80u;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void most_of(u16x2& most, uint32_t w) {
    const u16x2 v = __builtin_bit_cast(u16x2, w & 0x7fff7fffu);
    most = __builtin_elementwise_max(most, v);
}
template <typename T> __device__ __forceinline__ bool not_finite(u16x2 most) { return most[0] >= NOT_FINITE<T> || most[1] >= NOT_FINITE<T>; }

template <typename T> constexpr uint32_t ONE = std::is_same<T, f16>::value ? 0x3c00u : 0x3f80u;
typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
// v without what is not finite; up: 1 where it is +inf or NaN, down: where it is -inf or NaN.  (By packed arithmetic: comparisons would need
// a register of the scalar file each.)
template <typename T> __device__ __forceinline__ void parted(vec<T, 8>& v, vec<T, 8>& up, vec<T, 8>& down) {
    const u16x8 w = __builtin_bit_cast(u16x8, v), size = w & uint16_t(0x7fff), finite = uint16_t(NOT_FINITE<T> - 1), inf = uint16_t(NOT_FINITE<T>), one = 1;
    const u16x8 bad = __builtin_elementwise_min(__builtin_elementwise_max(size, finite) - finite, one), nan = __builtin_elementwise_min(__builtin_elementwise_max(size, inf) - inf, one);
    const u16x8 minus = w >> 15;
    up = __builtin_bit_cast(vec<T, 8>, u16x8((bad & (nan | (minus ^ one))) * uint16_t(ONE<T>)));
    down = __builtin_bit_cast(vec<T, 8>, u16x8((bad & (nan | minus)) * uint16_t(ONE<T>)));
    v = __builtin_bit_cast(vec<T, 8>, u16x8(w & (bad - one)));
}
// 1 where `margin` is positive
template <typename T> __device__ __forceinline__ uint32_t one_if(int32_t margin) { return uint32_t(min(max(margin, 0), 1)) * ONE<T>; }
// x, and 0 (-inf) where `hidden` is negative
__device__ __forceinline__ float or_zero(float x, int32_t hidden) { return __uint_as_float(__float_as_uint(x) & ~uint32_t(hidden >> 31)); }
__device__ __forceinline__ float or_none(float x, int32_t hidden) {
    const uint32_t mask = uint32_t(hidden >> 31);
    return __uint_as_float((__float_as_uint(x) & ~mask) | (mask & 0xff800000u));
}

// What counts of values that are not finite do to a sum: a count becomes 0 or infinity (no contraction: a fused product would stay below it).
template <bool SIGNED> __device__ __forceinline__ float counted(float up, float down) {
#pragma clang fp contract(off)
    const float x = up * 0x1p127f * 0x1p127f, y = down * 0x1p127f * 0x1p127f;
    return SIGNED ? x - y : (x - x) + (y - y);
}

// acc += v p over a depth of 32 K for products of 32 x 32 x 16, v turned on the way (at[i]: where this lane reads the first four rows of columns 32 i on),
// p the second operand, where some p are 0 because the mask hides that depth from that column and v has values that are not finite: a product
// 0 * inf must not show.  Such values are left out, and what they do to the columns that see them is found by counting; see(k): positive where
// this lane's column sees depth k.  SIGNED: p is positive, so their sign is the sum's; else they make it NaN.
template <int K, bool SIGNED, int D, typename T, int ND, typename See> __device__ __forceinline__ void careful(const vec<T, 8>* p, const uint32_t (&at)[ND], f32x16 (&acc)[ND], See see) {
    const int half = (threadIdx.x >> 5) & 1;
#pragma unroll
    for (int dt = 0; dt < ND; dt++) {
        f32x16 up = {}, down = {};
#pragma unroll
        for (int k = 0; k < 2 * K; k++) {
            __builtin_amdgcn_sched_barrier(0);      // one after the other: registers count here, not time
            vec<T, 8> v = turned32<D, T>(at[dt] + k * 16 * D * 2), u, w;
            parted<T>(v, u, w);
            uint32_t sees[4];
#pragma unroll
            for (int e = 0; e < 4; e++) {
                const int at_k = k * 16 + (e / 2) * 8 + half * 4 + e % 2 * 2;
                sees[e] = one_if<T>(see(at_k)) | one_if<T>(see(at_k + 1)) << 16;
            }
            const vec<T, 8> s = __builtin_bit_cast(vec<T, 8>, make_uint4(sees[0], sees[1], sees[2], sees[3]));
            acc[dt] = product32(v, p[k], acc[dt]), up = product32(u, s, up), down = product32(w, s, down);
        }
#pragma unroll
        for (int i = 0; i < 16; i++) acc[dt][i] += counted<SIGNED>(up[i], down[i]);
    }
}
// Whether `bytes` of LDS have a value that is not finite, by all lanes of a wavefront.
template <typename T> __device__ __forceinline__ bool any_not_finite(uint32_t at, int bytes) {
    u16x2 size = {0, 0};
    for (int i = (threadIdx.x & 63) * 16; i < bytes; i += 1024) {
        const uint4 w = __builtin_bit_cast(uint4, chunk_from<T>(at + i));
        most_of(size, w.x), most_of(size, w.y), most_of(size, w.z), most_of(size, w.w);
    }
    return __any(not_finite<T>(size));
}

// ---------------------------------------------------------------------------------------------------------------
// What calls ask of their sizes
// ---------------------------------------------------------------------------------------------------------------
template <typename F> int with_half(int dtype, F f) { return dtype == CSR5_DTYPE_F16 ? f(f16()) : f(bf16()); }

inline int attention_sizes(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, float scale) {
    if ((dtype != CSR5_DTYPE_BF16 && dtype != CSR5_DTYPE_F16) || sequences < 0 || rows < 0 || k_rows < 0 || heads < 0 || kv_heads < 0 || d < 0) return CSR5_EINVAL;
    if (kv_heads == 0 ? heads != 0 : heads % kv_heads != 0) return CSR5_EINVAL;
    if (!(scale > 0.f) || !std::isfinite(scale)) return CSR5_EINVAL;
    if (sequences > MOST_SIZE || rows > CSR5_ATTENTION_MAX_ROWS || k_rows > CSR5_ATTENTION_MAX_ROWS || heads > CSR5_ATTENTION_MAX_HEADS || d > CSR5_ATTENTION_MAX_D) return CSR5_ERANGE;
    return CSR5_OK;
}
inline bool words(std::initializer_list<const void*> all) {
    for (const void* p : all)
        if (reinterpret_cast<uintptr_t>(p) & 3) return false;
    return true;
}

}  // namespace

#endif
