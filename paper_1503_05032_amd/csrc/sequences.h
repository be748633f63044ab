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

// Where there are few workgroups of 128 rows, two or four wavefronts share a row's keys instead, and workgroups have 64 rows or 32 (one sequence
// of 861, 7 heads with one of keys: 48 workgroups, attention 32 us for 19; above some 500 of them it is the other way round, as keys are brought more often).
inline int sides_of(int64_t groups) { return groups <= 128 ? 4 : groups <= 320 ? 2 : 1; }

// The sequence that has tile t and where in it the tile begins, by all lanes of a wavefront: 64 sequences at a time are looked at.
// Whatever the offsets hold, the tile begins before the end of the sequence's rows, or false is returned.
struct TileOf {
    int32_t s;
    Span rows;
    int64_t first;          // of rows.count * times
};
// The last of the sequences for which f(its first row, its number) holds, where it holds for those before too, and its rows; -1: none.
template <typename F> __device__ __forceinline__ int32_t last_of(const int32_t* offset, int32_t sequences, int32_t rows, Span& span, F f) {
    const int lane = threadIdx.x & 63;
    int32_t low = 0, count = sequences;
    for (;;) {
        const int32_t step = (count + 63) / 64;
        const int64_t i = int64_t(low) + int64_t(lane) * step;
        const int32_t begin = i <= sequences ? begin_of(offset, int32_t(i), rows) : rows;
        const uint64_t votes = __ballot(int64_t(lane) * step < count && f(begin, int32_t(i)));
        if (!votes) return -1;
        const int last = 63 - __builtin_clzll(votes);
        if (step == 1) {
            const int32_t s = low + last, first = __builtin_amdgcn_readlane(begin, last);
            const int32_t end = last < 63 ? __builtin_amdgcn_readlane(begin, last + 1) : begin_of(offset, s + 1, rows);
            span = {first, max(end - first, 0)};
            return __builtin_amdgcn_readfirstlane(s);
        }
        low += last * step, count = min(step, count - last * step);
    }
}
__device__ __forceinline__ bool tile_of(const int32_t* offset, int32_t sequences, int32_t rows, int64_t times, int shift, int64_t t, TileOf& out) {
    out.s = last_of(offset, sequences, rows, out.rows, [&](int32_t begin, int32_t i) { return (int64_t(begin) * times >> shift) + i <= t; });
    if (out.s < 0) return false;
    out.first = (t - ((int64_t(out.rows.first) * times >> shift) + out.s)) << shift;
    return out.first >= 0 && out.first < int64_t(out.rows.count) * times;
}

// Keys and values of one sequence and head, packed or in a cache: where row j of either is, and whether rows from j on (a multiple of
// their number) lie side by side, so that one address serves a wavefront's load.
template <typename T> struct Packed {
    const int32_t* offset;
    int32_t rows;
    Heads<const T> k, v;
    struct One {
        const T *k, *v;
        int64_t k_row, v_row;
        int32_t count;
        static constexpr bool PACKED = true;
        typedef int Ahead;          // what is looked up ahead of a load (for packed rows nothing)
        __device__ __forceinline__ Ahead ahead(int32_t) const { return 0; }
        template <int ROWS> __device__ __forceinline__ bool together(Ahead) const { return true; }
        __device__ __forceinline__ const T* key(int32_t j, Ahead) const { return k + j * k_row; }
        __device__ __forceinline__ const T* value(int32_t j, Ahead) const { return v + j * v_row; }
        __device__ __forceinline__ const T* any_key(int32_t j) const { return k + j * k_row; }
        __device__ __forceinline__ const T* any_value(int32_t j) const { return v + j * v_row; }
    };
    __device__ __forceinline__ One one(int32_t s, int32_t h) const {
        const Span at = span_of(offset, s, rows);
        return {same(k.p + at.first * k.row + h * k.head), same(v.p + at.first * v.row + h * v.head), k.row, v.row, __builtin_amdgcn_readfirstlane(at.count)};
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
        static constexpr bool PACKED = false;
        typedef int32_t Ahead;      // the page of a row that is the same in every lane; -1: none
        __device__ __forceinline__ int32_t ahead(int32_t j) const {
            typedef const __attribute__((address_space(4))) int32_t* constant;      // a scalar load
            const int32_t page = j < count ? ((constant)(uintptr_t)table)[j >> shift] : -1;
            return uint32_t(page) < uint32_t(pages) ? page : -1;
        }
        template <int ROWS> __device__ __forceinline__ bool together(int32_t page) const { return page >= 0 && (1 << shift) >= ROWS; }
        __device__ __forceinline__ const T* key(int32_t j, int32_t page) const { return k + page * k_page + (j & ((1 << shift) - 1)) * k_row; }
        __device__ __forceinline__ const T* value(int32_t j, int32_t page) const { return v + page * v_page + (j & ((1 << shift) - 1)) * v_row; }
        // of any row, j < count, which may be another one in every lane; NULL: a row of zeros
        __device__ __forceinline__ const T* any_key(int32_t j) const {
            const int32_t page = table[j >> shift];
            return uint32_t(page) < uint32_t(pages) ? key(j, page) : nullptr;
        }
        __device__ __forceinline__ const T* any_value(int32_t j) const {
            const int32_t page = table[j >> shift];
            return uint32_t(page) < uint32_t(pages) ? value(j, page) : nullptr;
        }
    };
    __device__ __forceinline__ One one(int32_t s, int32_t h) const {
        const int32_t count = int32_t(min(int64_t(max(length[s], 0)), int64_t(width) << shift));
        return {same(table + s * ldt), pages, shift, same(k.p + h * k.head), same(v.p + h * v.head), k.page, k.row, v.page, v.row, __builtin_amdgcn_readfirstlane(count)};
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

// Where a wavefront reads tiles for products of 32 x 32 x 16: rows as first operands (chunks 2 kk on), and turned (columns 32 dt on).  Tiles begin at
// multiples of 256 bytes.  Other chunks are other patterns in bits 5 to 7: with a register for each, a tile at a fixed place needs no arithmetic; with one
// register for all, one instruction a read.
template <int ND> struct ReadFixed {
    static constexpr int D = ND <= 2 ? 64 : 128;
    uint32_t rows[2 * ND], first[ND], second[ND];
    __device__ __forceinline__ ReadFixed(uint32_t lds) {
        const int lane = threadIdx.x & 63, half = lane >> 5, li = lane & 15, r = half * 4 + (li >> 2);
#pragma unroll
        for (int kk = 0; kk < 2 * ND; kk++) rows[kk] = lds + (lane & 31) * D * 2 + chunk_at<D, false>(lane & 31, 2 * kk + half) * 16;
#pragma unroll
        for (int dt = 0; dt < ND; dt++) {
            first[dt] = lds + r * D * 2 + chunk_at<D, false>(r, dt * 4 + ((lane >> 4) & 1) * 2 + ((li & 3) >> 1)) * 16 + (li & 1) * 8;
            second[dt] = (first[dt] ^ 32) + 8 * D * 2;
        }
    }
    template <typename T> __device__ __forceinline__ vec<T, 8> row(int tile, int kk) const { return chunk_from<T>(rows[kk] + tile); }
    template <typename T> __device__ __forceinline__ vec<T, 8> turned(int tile, int dt) const { return turned_from<T>(first[dt] + tile, second[dt] + tile); }
};

// One wavefront's load into LDS, from an address of each lane: 1024 bytes, lane by lane 16 of them; `from` NULL, or values from `have` on: zeros.
template <bool WIDE, typename T> __device__ __forceinline__ void chunk_to_lds(const T* from, int have, uint32_t to) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    if (WIDE) to_lds_at(from && have > 0 ? static_cast<const void*>(from) : &ZEROS, to);
    else *(__attribute__((address_space(3))) u32x4*)uintptr_t(to + (threadIdx.x & 63) * 16) = __builtin_bit_cast(u32x4, eight_values<false>(from, from ? have : 0));
}

// Zeros to `bytes` of LDS, by `lanes` lanes of which this is one.
__device__ __forceinline__ void zeros_to(uint32_t at, int bytes, int lane, int lanes) {
    typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
    for (int i = lane * 16; i < bytes; i += lanes * 16) *(__attribute__((address_space(3))) u32x4*)uintptr_t(at + i) = u32x4{0, 0, 0, 0};
}

// A tile of keys and one of values (or of any two arrays with the same rows) into LDS by WAVES wavefronts, each LOADS times a load of EACH rows of both: where
// they lie side by side from one address on, that and one offset of each lane serve a load; else each lane looks for its row (heads of 80 over pages of 16,
// 32 single tokens over 4000 to 8000: 262 us so, 135 by offsets).
template <typename T, int D, bool WIDE, bool SMALL, int ROWS, int WAVES> struct Bring {
    static constexpr int LANES = D / 8, EACH = 64 / LANES;      // lanes of a row, rows of a load
    static constexpr int LOADS = ROWS / EACH / WAVES;
    // Rows that all loads of a lane have the swizzle of; where WAVES is 1, loads differ in it.
    static constexpr int KINDS = WAVES * EACH >= 16 ? 1 : 16 / (WAVES * EACH);
    int wave, row;                                  // this lane's row of a load
    int chunk[KINDS];
    uint32_t k_off[LOADS], v_off[LOADS];            // in bytes: packed, from the tile's first row; else from the load's
    bool near;                                      // 16-byte rows, and no offset passes 32 bits
    bool ragged;                                    // lanes whose chunk is beside the row, but is read, ask for nothing: their place has zeros from the beginning
    template <typename One> __device__ __forceinline__ Bring(const One& kv, int wave, int d) : wave(wave) {
        const int lane = threadIdx.x & 63;
        row = lane / LANES;
        // a chunk that is not read may be another one
        ragged = d != D && !(D == 128 && d == 96);
        near = WIDE && (ROWS * kv.k_row | ROWS * kv.v_row) < (1 << 28);
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int r = (i * WAVES + wave) * EACH + row, from = One::PACKED ? r : row;
            const int c = int(chunk_at<D, SMALL>(r, lane % LANES)) * 8, in = c < d ? c : 0;
            chunk[i % KINDS] = c;
            k_off[i] = uint32_t(from * kv.k_row + in) * 2, v_off[i] = uint32_t(from * kv.v_row + in) * 2;
        }
    }
    // The loads' pages, of the tile from j0 on.
    template <typename One> __device__ __forceinline__ void look(const One& kv, int32_t j0, typename One::Ahead (&ahead)[LOADS]) const {
#pragma unroll
        for (int i = 0; i < LOADS; i++) ahead[i] = kv.ahead(j0 + (i * WAVES + wave) * EACH);
    }
    // k, v: where the tiles are in LDS
    template <typename One> __device__ __forceinline__ void operator()(const One& kv, int32_t j0, const typename One::Ahead (&ahead)[LOADS], int d, uint32_t k, uint32_t v) const {
        const bool whole = near && j0 + ROWS <= kv.count;
        if (One::PACKED && whole) {
            const T *const from = kv.key(j0, ahead[0]), *const of = kv.value(j0, ahead[0]);
#pragma unroll
            for (int i = 0; i < LOADS; i++) {
                if (ragged && chunk[i % KINDS] >= d) continue;
                to_lds_at(from, k_off[i], k + (i * WAVES + wave) * 1024);
                to_lds_at(of, v_off[i], v + (i * WAVES + wave) * 1024);
            }
            return;
        }
#pragma unroll
        for (int i = 0; i < LOADS; i++) {
            const int32_t j = j0 + (i * WAVES + wave) * EACH;
            const uint32_t to = (i * WAVES + wave) * 1024;
            if (!One::PACKED && whole && kv.template together<EACH>(ahead[i])) {
                if (ragged && chunk[i % KINDS] >= d) continue;
                to_lds_at(kv.key(j, ahead[i]), k_off[i], k + to), to_lds_at(kv.value(j, ahead[i]), v_off[i], v + to);
            } else {
                const bool there = j + row < kv.count;
                const T *const from = there ? kv.any_key(j + row) : nullptr, *const of = there ? kv.any_value(j + row) : nullptr;
                const int c = chunk[i % KINDS];
                chunk_to_lds<WIDE>(from ? from + c : from, d - c, k + to), chunk_to_lds<WIDE>(of ? of + c : of, d - c, v + to);
            }
        }
    }
};

// x, and 0 (-inf) where `hidden` is negative
__device__ __forceinline__ float or_zero(float x, int32_t hidden) { return __uint_as_float(__float_as_uint(x) & ~uint32_t(hidden >> 31)); }
__device__ __forceinline__ float or_none(float x, int32_t hidden) {
    const uint32_t mask = uint32_t(hidden >> 31);
    return __uint_as_float((__float_as_uint(x) & ~mask) | (mask & 0xff800000u));
}

// Where a mask hides some depth of a product from some columns, their p are 0, and a value there that is not finite must not show, as 0 * inf would.
// So a tile with such values, seldom as they are, is cleansed of them in LDS before it is read so (keys after the scores, which their values decide as they are), and what they do to the columns that do see them is
// added to the results in the end, from memory.  (A second way through the products for such tiles would take the first one's registers: the attention of
// 3 sequences up to 8001 took 985 us with it.)  Bytes [from, to) of this tile by lanes that have `lane` of `lanes`; whether there were some.
template <typename T> __device__ __forceinline__ bool cleanse(uint8_t* tile, int bytes, int lane, int lanes) {
    typedef uint16_t u16x8 __attribute__((ext_vector_type(8)));
    constexpr uint16_t LARGEST = std::is_same<T, f16>::value ? 0x7bff : 0x7f7f;
    bool found = false;
    for (int i = lane * 16; i < bytes; i += lanes * 16) {
        u16x8* const at = reinterpret_cast<u16x8*>(tile + i);
        const u16x8 w = *at, over = __builtin_elementwise_max(w & uint16_t(0x7fff), u16x8(LARGEST)) - LARGEST;     // 0: finite
        const uint4 some = __builtin_bit_cast(uint4, over);
        if (!(some.x | some.y | some.z | some.w)) continue;
        *at = w & (__builtin_elementwise_min(over, u16x8(1)) - uint16_t(1));
        found = true;
    }
    return found;
}
__device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }

// ---------------------------------------------------------------------------------------------------------------
// What calls ask of their sizes
// ---------------------------------------------------------------------------------------------------------------
template <typename F> int with_half(int dtype, F f) { return dtype == CSR5_DTYPE_F16 ? f(f16()) : f(bf16()); }

inline int attention_sizes(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, float scale) {
    if ((dtype != CSR5_DTYPE_BF16 && dtype != CSR5_DTYPE_F16) || sequences < 0 || rows < 0 || k_rows < 0 || heads < 0 || kv_heads < 0 || d < 0) return CSR5_EINVAL;
    if (kv_heads == 0 ? heads != 0 : heads % kv_heads != 0) return CSR5_EINVAL;
    if (!(scale > 0.f) || !std::isfinite(scale * LOG2_E)) return CSR5_EINVAL;       // infinite, it would make a score of 0 NaN
    if (sequences > MOST_SIZE || rows > CSR5_ATTENTION_MAX_ROWS || k_rows > CSR5_ATTENTION_MAX_ROWS || heads > CSR5_ATTENTION_MAX_HEADS || kv_heads > CSR5_ATTENTION_MAX_HEADS || d > CSR5_ATTENTION_MAX_D) return CSR5_ERANGE;
    return CSR5_OK;
}
inline bool words(std::initializer_list<const void*> all) {
    for (const void* p : all)
        if (reinterpret_cast<uintptr_t>(p) & 3) return false;
    return true;
}

}  // namespace

#endif
