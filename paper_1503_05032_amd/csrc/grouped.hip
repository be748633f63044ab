// libcsr5: products of a layer of experts -- grouped by expert over ragged groups, in 16 bits with their gradients and in
// 8 bits with a scale for each block of 128.  The C ABI is declared in include/csr5.h.
//
// Every product here is out[i][j] = sum_c X[i][c] W[j][c]:
//
//   FWD   y = x w^T      i: rows of a group    j: n      c: k       X, W as they lie in memory
//   DX    dx = dy w      i: rows of a group    j: k      c: n       W lies with j contiguous: transposed on the way
//   DW    dw = dy^T x    i: n                  j: k      c: rows    both transposed on the way
//
// The matrix instructions take W for their first operand and X for their second, so that a lane of the result holds
// four neighbouring columns j of one row i (one row's scale, one 8-byte store).
#include <hip/hip_runtime.h>

#include <cstdint>
#include <type_traits>

#include "csr5.h"
#include "numbers.h"

namespace {

enum { FWD, DX, DW };

typedef uint8_t f8;
template <typename T> constexpr bool is_f8 = std::is_same<T, f8>::value;

struct Product {
    const void* x;              // FWD: x; DX, DW: dy
    int64_t ldx;
    const void* w;              // FWD, DX: w; DW: x
    int64_t ldw, w_group;
    void* y;
    int64_t ldy, y_group;       // y_group: DW
    const int32_t* offset;      // NULL: one group of all rows
    const int32_t* source;      // of the rows of x, wherever x is; NULL: themselves
    int32_t source_rows;        // rows that a source may name
    int32_t groups, rows;
    int32_t out_rows;           // DW: n
    int32_t cols, depth;        // j and c (DW: depth is the group's)
    const float *xs, *ws;       // 8 bits: the scales
    int64_t xs_row, xs_block, ws_row, ws_block, ws_group;
    int32_t w_rows;
    bool far;                   // bytes from the beginning of x to a row that a source names may pass 32 bits
};

// ---------------------------------------------------------------------------------------------------------------
// Which rows
// ---------------------------------------------------------------------------------------------------------------
struct Span {
    int group;
    int32_t first, last;        // rows [first, last) of the group that are this workgroup's
};

__device__ __forceinline__ int32_t offset_at(const Product& a, int g) { return min(max(a.offset[g], 0), a.rows); }
__device__ __forceinline__ Span group_span(const Product& a, int g) {
    if (!a.offset) return {0, 0, a.rows};
    const int32_t first = offset_at(a, g);
    return {g, first, max(offset_at(a, g + 1), first)};
}

// The same in every lane, for the compiler to know.
__device__ __forceinline__ Span uniform(Span s) {
    return {__builtin_amdgcn_readfirstlane(s.group), __builtin_amdgcn_readfirstlane(s.first), __builtin_amdgcn_readfirstlane(s.last)};
}

// The t-th tile of BM rows, counted through the groups in order; group -1: there are fewer.  The whole wavefront takes part:
// a lane per group.  At most rows / BM + groups tiles where no groups overlap; there are no workgroups for more.
template <int BM> __device__ __forceinline__ Span find_tile(const Product& a, int32_t t) {
    if (!a.offset) {
        const int64_t first = int64_t(t) * BM;
        return {first < a.rows ? 0 : -1, int32_t(min(first, int64_t(a.rows))), int32_t(min(first + BM, int64_t(a.rows)))};
    }
    const int lane = threadIdx.x & 63;
    int32_t before = 0;
    for (int g0 = 0; g0 < a.groups; g0 += 64) {
        const int g = g0 + lane;
        Span s{-1, 0, 0};
        if (g < a.groups) s = group_span(a, g);
        const int32_t tiles = (s.last - s.first + BM - 1) / BM;
        const int32_t upto = wave_prefix(tiles);
        const uint64_t past = __ballot(before + upto > t);
        if (past) {
            const int l = __ffsll((unsigned long long)past) - 1;
            const int32_t first = __builtin_amdgcn_readlane(s.first, l) + (t - before - __builtin_amdgcn_readlane(upto - tiles, l)) * BM;
            return uniform({g0 + l, first, min(first + BM, __builtin_amdgcn_readlane(s.last, l))});
        }
        before += __builtin_amdgcn_readlane(upto, 63);
    }
    return {-1, 0, 0};
}
// How many there are; `most`: of dense rows.
template <int BM> __device__ __forceinline__ int32_t count_tiles(const Product& a, int32_t most) {
    if (!a.offset) return most;
    int32_t all = 0;
    for (int g0 = 0; g0 < a.groups; g0 += 64) {
        const int g = g0 + int(threadIdx.x & 63);
        int32_t tiles = 0;
        if (g < a.groups) {
            const Span s = group_span(a, g);
            tiles = (s.last - s.first + BM - 1) / BM;
        }
        all += __builtin_amdgcn_readlane(wave_prefix(tiles), 63);
    }
    return all;
}
// The group with the rank-th most rows (the rank-th, where there are more than 64 or none has more than 256: to sort takes
// longer than such a tile; 60 groups of 2 rows, 1408 x 3200: 152 us instead of 191).
__device__ __forceinline__ int largest_group(const Product& a, int rank) {
    if (a.groups > 64) return rank;
    const int lane = threadIdx.x & 63;
    uint32_t rows = 0;
    if (lane < a.groups) {
        const Span s = group_span(a, lane);
        rows = uint32_t(s.last - s.first);
    }
    if (wave_max(rows) <= 256) return rank;
    const uint32_t key = min(rows, (1u << 26) - 1) << 6 | uint32_t(63 - lane);      // no two alike
    int above = 0;
    for (int g = 0; g < a.groups; g++) above += uint32_t(__builtin_amdgcn_readlane(int(key), g)) > key;
    return __ffsll((unsigned long long)__ballot(lane < a.groups && above == rank)) - 1;
}

__device__ __forceinline__ int64_t source_of(const Product& a, int64_t row) {       // -1: a row of zeros
    const int64_t r = a.source ? a.source[row] : row;
    return r >= 0 && r < a.source_rows ? r : -1;
}

// ---------------------------------------------------------------------------------------------------------------
// The matrix instructions: 16 x 16 results from 16 bytes (8 bits: 32) of each lane
// ---------------------------------------------------------------------------------------------------------------
typedef vec<float, 4> f32x4;
typedef vec<bf16, 8> bf16x8;
typedef vec<f16, 8> f16x8;

__device__ __forceinline__ f32x4 multiply(const uint4& w, const uint4& x, f32x4 acc, bf16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, w), __builtin_bit_cast(bf16x8, x), acc, 0, 0, 0);
}
__device__ __forceinline__ f32x4 multiply(const uint4& w, const uint4& x, f32x4 acc, f16) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, w), __builtin_bit_cast(f16x8, x), acc, 0, 0, 0);
}
// 8 e4m3 values in 16 bits, exactly
__device__ __forceinline__ bf16x8 widen(uint32_t a, uint32_t b) {
    const vec<float, 2> v[4] = {__builtin_amdgcn_cvt_pk_f32_fp8(int(a), false), __builtin_amdgcn_cvt_pk_f32_fp8(int(a), true),
                                __builtin_amdgcn_cvt_pk_f32_fp8(int(b), false), __builtin_amdgcn_cvt_pk_f32_fp8(int(b), true)};
    bf16x8 r;
#pragma unroll
    for (int i = 0; i < 8; i++) r[i] = bf16(v[i / 2][i % 2]);
    return r;
}
// In 8 bits, added up in 32: by the instruction for 16.
__device__ __forceinline__ f32x4 multiply(const uint4& w, const uint4& x, f32x4 acc, f8) {
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.x, w.y), widen(x.x, x.y), acc, 0, 0, 0);
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(w.z, w.w), widen(x.z, x.w), acc, 0, 0, 0);
}

typedef int i32x8 __attribute__((ext_vector_type(8)));

// A block's 128 products in 8 bits, of 32 bytes of each lane (as two pieces of 16 neighbouring values).  The instruction for 8
// bits adds up every eight neighbouring products in units of 2^(E-13), E the largest sum of the exponents of two factors whose
// product is not 0 (-6 for subnormal ones), and cuts what a product has below that; it adds the eights in 32 bits.  (Measured: of
// 120000 random rows of 128 values every one within 2^-22 of that, and those of one eight equal to it.)  So an eight is off by
// less than 7 * 2^-13 of its largest product, and normal values by 2e-6 of the sum of the magnitudes, where a sum in 32 bits is
// off by 1e-9.  That is a choice for results that are rounded to 16 bits, 2^-9 or 2^-12 of them; results in 32 bits get sums in
// 32 bits, by four instructions for 16.
template <typename Y> __device__ __forceinline__ f32x4 multiply_block(const i32x8& w, const i32x8& x) {
    if constexpr (std::is_same<Y, float>::value) {
        f32x4 part = {0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < 8; h += 4)
            part = multiply(make_uint4(w[h], w[h + 1], w[h + 2], w[h + 3]), make_uint4(x[h], x[h + 1], x[h + 2], x[h + 3]), part, f8());
        return part;
    } else {
        // scales 0: the form of the instruction without scales
        return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, x, f32x4{0, 0, 0, 0}, 0, 0, 0, 0, 0, 0);
    }
}

// Four neighbouring values of a row of y.
template <typename Y, bool VEC> __device__ __forceinline__ void store_four(Y* p, int have, f32x4 v) {
    const float f[4] = {v[0], v[1], v[2], v[3]};
    store_values<4, VEC>(p, have, f);
}

// ---------------------------------------------------------------------------------------------------------------
// The plain kernel: right for any strides, alignment and sizes.  128 x 128 results per workgroup of four wavefronts; the
// depth goes by in steps of 128 bytes (in 8 bits a block of scales) through registers into LDS, where rows of both
// operands are contiguous along it.
// ---------------------------------------------------------------------------------------------------------------
constexpr int PLAIN_TILE = 128;
constexpr int PLAIN_PITCH = 128 + 16;       // bytes of a row in LDS

template <typename T, typename Y, int OP> __global__ __launch_bounds__(256) void k_product_plain(Product a) {
    constexpr int SIZE = sizeof(T), STEP = 128 / SIZE;
    __shared__ __align__(16) uint8_t lds[2][PLAIN_TILE * PLAIN_PITCH];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int col_tiles = (a.cols + PLAIN_TILE - 1) / PLAIN_TILE;
    const int j0 = int(blockIdx.x % col_tiles) * PLAIN_TILE;
    Span s;
    int32_t i0;                             // first row of the results
    int32_t i_end, depth;
    if (OP == DW) {
        const int row_tiles = (a.out_rows + PLAIN_TILE - 1) / PLAIN_TILE;
        s = group_span(a, int(blockIdx.x / col_tiles / row_tiles));
        i0 = int32_t(blockIdx.x / col_tiles % row_tiles) * PLAIN_TILE;
        i_end = a.out_rows, depth = s.last - s.first;
    } else {
        s = find_tile<PLAIN_TILE>(a, int32_t(blockIdx.x / col_tiles));
        if (s.group < 0) return;
        i0 = s.first, i_end = s.last, depth = a.depth;
    }
    const T* const w = static_cast<const T*>(a.w) + (OP == DW ? 0 : s.group * a.w_group);

    // One value of each operand, 0 outside.
    auto x_at = [&](int32_t i, int32_t c) -> T {
        if (i >= i_end || c >= depth) return T(0);
        if (OP == DW) return static_cast<const T*>(a.x)[int64_t(s.first + c) * a.ldx + i];
        const int64_t r = OP == FWD ? source_of(a, i) : i;
        return r < 0 ? T(0) : static_cast<const T*>(a.x)[r * a.ldx + c];
    };
    auto w_at = [&](int32_t j, int32_t c) -> T {
        if (j >= a.cols || c >= depth) return T(0);
        if (OP == FWD) return w[int64_t(j) * a.ldw + c];
        if (OP == DX) return w[int64_t(c) * a.ldw + j];
        const int64_t r = source_of(a, s.first + c);
        return r < 0 ? T(0) : w[r * a.ldw + j];
    };
    f32x4 acc[4][4] = {};                   // [j][i] of this wavefront's 64 x 64
    const int wi = (wave & 1) * 64, wj = (wave >> 1) * 64;
    for (int32_t c0 = 0; c0 < depth; c0 += STEP) {
        // neighbouring threads along what is contiguous in memory
        for (int e = tid; e < PLAIN_TILE * STEP; e += 256) {
            const int i = OP == DW ? e % PLAIN_TILE : e / STEP, c = OP == DW ? e / PLAIN_TILE : e % STEP;
            *reinterpret_cast<T*>(&lds[0][i * PLAIN_PITCH + c * SIZE]) = x_at(i0 + i, c0 + c);
        }
        for (int e = tid; e < PLAIN_TILE * STEP; e += 256) {
            const int j = OP != FWD ? e % PLAIN_TILE : e / STEP, c = OP != FWD ? e / PLAIN_TILE : e % STEP;
            *reinterpret_cast<T*>(&lds[1][j * PLAIN_PITCH + c * SIZE]) = w_at(j0 + j, c0 + c);
        }
        __syncthreads();
        f32x4 part[4][4] = {};
#pragma unroll
        for (int k = 0; k < 128; k += 64) {
            uint4 xv[4], wv[4];
#pragma unroll
            for (int i = 0; i < 4; i++) {
                xv[i] = *reinterpret_cast<const uint4*>(&lds[0][(wi + i * 16 + (lane & 15)) * PLAIN_PITCH + k + (lane >> 4) * 16]);
                wv[i] = *reinterpret_cast<const uint4*>(&lds[1][(wj + i * 16 + (lane & 15)) * PLAIN_PITCH + k + (lane >> 4) * 16]);
            }
#pragma unroll
            for (int j = 0; j < 4; j++)
#pragma unroll
                for (int i = 0; i < 4; i++) {
                    f32x4& to = is_f8<T> ? part[j][i] : acc[j][i];
                    to = multiply(wv[j], xv[i], to, T());
                }
        }
        if (is_f8<T>) {
            const int b = c0 / CSR5_F8_BLOCK;
#pragma unroll
            for (int i = 0; i < 4; i++) {
                const int32_t row = i0 + wi + i * 16 + (lane & 15);
                const int64_t r = row < i_end ? source_of(a, row) : -1;
                const float xs = r < 0 ? 0.f : a.xs[r * a.xs_row + b * a.xs_block];
#pragma unroll
                for (int j = 0; j < 4; j++)
#pragma unroll
                    for (int q = 0; q < 4; q++) {
                        const int32_t col = j0 + wj + j * 16 + (lane >> 4) * 4 + q;
                        const float ws = col < a.cols ? a.ws[s.group * a.ws_group + col / a.w_rows * a.ws_row + b * a.ws_block] : 0.f;
                        acc[j][i][q] += part[j][i][q] * (xs * ws);
                    }
            }
        }
        __syncthreads();
    }
    Y* const y = static_cast<Y*>(a.y) + (OP == DW ? s.group * a.y_group : 0);
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const int32_t row = i0 + wi + i * 16 + (lane & 15);
        if (row >= i_end) continue;
        const bool zero = OP == FWD && source_of(a, row) < 0;       // whatever w holds
#pragma unroll
        for (int j = 0; j < 4; j++) {
            const int32_t col = j0 + wj + j * 16 + (lane >> 4) * 4;
            store_four<Y, false>(y + int64_t(row) * a.ldy + col, a.cols - col, zero ? f32x4{0, 0, 0, 0} : acc[j][i]);
        }
    }
}

// ---------------------------------------------------------------------------------------------------------------
// The tiled kernels, for rows of whole 16-byte chunks.  BI x BJ results per workgroup of WI x WJ wavefronts; the depth goes by
// in steps of 128 bytes, from memory straight into LDS, ahead of the matrix instructions.
//
// A tile whose rows are contiguous along the depth (Straight) lies in LDS as rows of one step, 128 bytes: whole lines (64
// bytes a step took twice the requests to the L2); one whose rows are contiguous along i or j (Turned: W of DX, both of DW)
// as 64 rows of the tile's width, and is turned by the LDS read.  A wavefront's load fills 1024 contiguous bytes of LDS;
// which 16 bytes of memory each lane asks for is what spreads the reads over the 64 banks (no conflicts counted):
//   Straight   chunk c of row r is at place c ^ (r >> 1 & 7): the 16 rows that a read takes a chunk of fill all banks
//   Turned     32-byte segment g of row c is at segment g ^ (c & 3 | c >> 1 & 4): so do the 8 rows of half a read
// Chunks past the depth (or the row, where that is contiguous) come from 16 bytes of zeros; rows past the end are some
// other row, and their results are not stored.
// ---------------------------------------------------------------------------------------------------------------
__device__ const uint4 ZEROS = {0, 0, 0, 0};

// 16 (4) bytes of each lane's address to lds + 16 (4) * lane; lds is the same for the whole wavefront.  In assembly because
// the compiler, which knows these loads as writes to all of LDS, would wait for later steps' before it reads this one's;
// they write no vector register, and the compiler keeps nothing in m0 (hence no warning that it would not be kept).  What
// waits for them is landed().  The compiler does not look into the assembly, so the waits that the instructions need are in it:
// one state after m0; and a base, which may come from a vector instruction (same()) less than the five states before that a load
// needs then, is moved by a scalar one, which the hardware waits for on both sides.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ uint32_t lds_address(const void* lds) {
    return __builtin_amdgcn_readfirstlane(uint32_t(uintptr_t((const __attribute__((address_space(3))) void*)lds)));
}
// An address that is the same in every lane, for the compiler to know.
template <typename P> __device__ __forceinline__ P* same(P* p) {
    const uint64_t v = reinterpret_cast<uintptr_t>(p);
    // the builtin's result is signed
    const uint32_t low = uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v))), high = uint32_t(__builtin_amdgcn_readfirstlane(uint32_t(v >> 32)));
    return reinterpret_cast<P*>(uint64_t(low) | uint64_t(high) << 32);
}
__device__ __forceinline__ void to_lds(const void* from, const void* lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds_address(lds)), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void to_lds(const void* base, uint32_t offset, const void* lds) {      // base: the same in every lane
    const void* at;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(at) : "s"(lds_address(lds)), "v"(offset), "s"(same(base)) : "memory", "m0");
}
__device__ __forceinline__ void word_to_lds(const void* from, const void* lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds_address(lds)), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void word_to_lds(const void* base, uint32_t offset, const void* lds) {
    const void* at;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dword %2, %0" : "=&s"(at) : "s"(lds_address(lds)), "v"(offset), "s"(same(base)) : "memory", "m0");
}
#pragma clang diagnostic pop
// This wavefront's loads into LDS have landed but for the last LATER, and its reads of LDS have returned; then the others' too.
template <int LATER> __device__ __forceinline__ void landed() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

template <int HEIGHT, int WAVES> struct Straight {                  // HEIGHT rows of 128 bytes
    static constexpr int LOADS = HEIGHT / 8 / WAVES;
    static_assert(WAVES % 2 == 0, "bit 3 of a row is that of the wavefront, so a lane's chunk is the same in every load");
    const uint8_t* base;        // moves on with the steps, the same in every lane
    uint32_t offset[LOADS];     // from it, in 16 bytes
    int chunk;                  // of a step, that this lane asks for
    // row(r): bytes from `at` to the tile's row r
    template <typename Row> __device__ __forceinline__ void start(int lane, int wave, const void* at, Row row) {
        base = same(static_cast<const uint8_t*>(at));
        chunk = (lane & 7) ^ (((wave * 8 + lane / 8) >> 1) & 7);
#pragma unroll
        for (int q = 0; q < LOADS; q++) offset[q] = uint32_t(uint64_t(row((q * WAVES + wave) * 8 + lane / 8)) >> 4) + chunk;
    }
    // left: bytes of a row from this step on.  FAST: a whole step, and no offset passes 32 bits.
    template <bool FAST> __device__ __forceinline__ void load(int q, uint8_t* lds, int wave, int64_t left) {
        uint8_t* const to = lds + (q * WAVES + wave) * 1024;
        if (FAST) to_lds(base, offset[q] << 4, to);
        else to_lds(chunk * 16 < left ? base + (uint64_t(offset[q]) << 4) : reinterpret_cast<const uint8_t*>(&ZEROS), to);
        if (q == LOADS - 1) base += 128;
    }
    // Where in a tile this lane reads the first of the 16 x 64 bytes of rows from `first` on (a multiple of a wavefront's
    // share), and the e-th from there on of its 64 bytes k, given the address of that in a tile.
    __device__ static __forceinline__ uint32_t where(int first, int lane) { return (first + (lane & 15)) * 128 + (((lane >> 4) ^ ((lane >> 1) & 7)) * 16); }
    __device__ static __forceinline__ uint4 read(uint32_t at, int e, int k) {
        typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
        const u32x4 v = *(const __attribute__((address_space(3))) u32x4*)uintptr_t((at ^ (k * 64)) + e * 2048);
        return make_uint4(v[0], v[1], v[2], v[3]);
    }
};

template <int COLS, int WAVES> struct Turned {                      // 64 rows of COLS 16-bit values
    static constexpr int PITCH = COLS * 2, LANES = PITCH / 16, EACH = 64 / LANES, LOADS = 64 / EACH / WAVES;     // lanes of a row, rows of a load
    static_assert(COLS >= 128 && LANES <= 64, "a swizzle is over 256 bytes; a load is whole rows");
    static_assert(WAVES * EACH % 16 == 0, "bits 0, 1 and 3 of a row are the same in every load of a lane");
    const uint8_t* base;        // row 0 of the next step (with source: of all), the same in every lane
    int64_t pitch;              // bytes of a row in memory
    int32_t next[LOADS][EACH];  // with source: what it says for the next step, the same in every lane
    int32_t from[LOADS];        // ... and for this one, for this lane's row
    bool all_named;             // ... of which every one is a row
    int c;                      // row of load 0 within a step
    uint32_t col;               // where this lane's chunk begins in a row, in bytes; past its end: at its last chunk
    // values: row 0; first: the tile's first value in it; width: values of a row
    template <typename T> __device__ __forceinline__ void start(int lane, int wave, const T* values, int64_t ld, int first, int width) {
        c = wave * EACH + lane / LANES;
        const int place = lane % LANES, at = first + (((place >> 1) ^ ((c & 3) | (c >> 1 & 4))) << 4) + (place & 1) * 8;
        base = same(reinterpret_cast<const uint8_t*>(values)), pitch = ld * sizeof(T), col = min(at, width - 8) * sizeof(T);
    }
    // left: rows from this step on.  FAST: a whole step.
    template <bool FAST> __device__ __forceinline__ void load(int q, uint8_t* lds, int wave, int left) {
        const int at = c + q * WAVES * EACH;
        uint8_t* const to = lds + (q * WAVES + wave) * 1024;
        if (FAST) to_lds(base, uint32_t(at) * uint32_t(pitch) + col, to);
        else to_lds(at < left ? base + at * pitch + col : reinterpret_cast<const uint8_t*>(&ZEROS), to);
        if (q == LOADS - 1) base += 64 * pitch;
    }
    // source: from the step's first row on; left: its rows.  Scalar loads: they do not wait with the loads into LDS.
    __device__ __forceinline__ void by_source(const int32_t* source, int left, int wave) {
        typedef const __attribute__((address_space(4))) int32_t* constant;
#pragma unroll
        for (int q = 0; q < LOADS; q++)
#pragma unroll
            for (int r = 0; r < EACH; r++) next[q][r] = left > 0 ? ((constant)(uintptr_t)source)[min((q * WAVES + wave) * EACH + r, left - 1)] : -1;
    }
    // Before the first of a step's loads, after the wait of landed(): the compiler's own wait for them goes here, where it
    // is for nothing.
    // rows: that a source may name
    __device__ __forceinline__ void here(int lane, int32_t rows) {
        bool named = true;
#pragma unroll
        for (int q = 0; q < LOADS; q++) {
            from[q] = next[q][0];
#pragma unroll
            for (int e = 1; e < EACH; e++) from[q] = lane / LANES == e ? next[q][e] : from[q];
            asm volatile("" : "+v"(from[q]));
            named = named && uint32_t(from[q]) < uint32_t(rows);
        }
        all_named = __all(named);
    }
    // what by_source() asked for a step ago
    template <bool FAST> __device__ __forceinline__ void load_by_source(int q, uint8_t* lds, int wave, int left, int32_t rows) {
        uint8_t* const to = lds + (q * WAVES + wave) * 1024;
        if (FAST && all_named) {
            to_lds(base, uint32_t(from[q]) * uint32_t(pitch) + col, to);
        } else {
            const bool there = c + q * WAVES * EACH < left && uint32_t(from[q]) < uint32_t(rows);
            to_lds(there ? base + from[q] * pitch + col : reinterpret_cast<const uint8_t*>(&ZEROS), to);
        }
    }
    // As Straight's, for 16 columns from `first` on; slots and rows are multiples of 256 bytes, so the e-th segment's place is
    // another pattern in bits 5 to 7.
    __device__ static __forceinline__ uint32_t where(int first, int lane) {
        const int li = lane & 15, q = lane >> 4;
        return (q * 8 + (li >> 2)) * PITCH + (((first >> 4) ^ ((li >> 2) | (q & 1) << 2)) * 32) + (li & 3) * 8;
    }
    __device__ static __forceinline__ uint4 read(uint32_t at, int e, int k) {
        typedef short s16x4 __attribute__((ext_vector_type(4)));
        typedef __attribute__((address_space(3))) s16x4* lds_ptr;
        at = (at ^ (e * 32)) + k * 32 * PITCH;
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)uintptr_t(at)),
                    hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_ptr)uintptr_t(at + 4 * PITCH));
        const uint2 a = __builtin_bit_cast(uint2, lo), b = __builtin_bit_cast(uint2, hi);
        return make_uint4(a.x, a.y, b.x, b.y);
    }
};

// The order of the tiles, which suits the caches: 8 tiles of rows go with one tile of columns after the other.
__device__ __forceinline__ void tile_at(int32_t at, int row_tiles, int col_tiles, int32_t& i, int32_t& j) {
    const int32_t strip = at / (8 * col_tiles), in = at - strip * 8 * col_tiles, high = min(8, row_tiles - strip * 8);
    i = __builtin_amdgcn_readfirstlane(strip * 8 + in % high), j = __builtin_amdgcn_readfirstlane(in / high);
}

// The rows, columns and depth of a workgroup's tile.  Workgroups go to the 8 XCDs by turns, so each XCD gets a contiguous part
// of the order: of the tiles that there are, which is for the device to say (with a part of the most that there can be, one
// XCD had mostly tiles that there were not).  DW: of each group's, the groups with most rows first, as a tile takes as long
// as its group has rows.
struct Tile {
    Span s;
    int32_t i0, i_end, j0, depth;
};
template <int OP, int BI, int BJ> __device__ __forceinline__ bool find(const Product& a, int row_tiles, int col_tiles, Tile& t) {
    const int32_t xcd = blockIdx.x & 7, m = blockIdx.x >> 3;
    int32_t it, jt;
    if (OP == DW) {
        const int32_t total = row_tiles * col_tiles, per = (total + 7) / 8, at = xcd * per + m % per;
        if (at >= total) return false;
        t.s.group = largest_group(a, m / per);
        if (t.s.group < 0 || t.s.group >= a.groups) return false;
        tile_at(at, row_tiles, col_tiles, it, jt);
        t.s = uniform(group_span(a, t.s.group));
        t.i0 = it * BI, t.i_end = a.out_rows, t.depth = t.s.last - t.s.first;
    } else {
        row_tiles = __builtin_amdgcn_readfirstlane(min(count_tiles<BI>(a, row_tiles), row_tiles));
        const int32_t total = row_tiles * col_tiles, per = (total + 7) / 8, at = xcd * per + m;
        if (m >= per || at >= total) return false;
        tile_at(at, row_tiles, col_tiles, it, jt);
        t.s = find_tile<BI>(a, it);
        t.i0 = t.s.first, t.i_end = t.s.last, t.depth = a.depth;
    }
    t.j0 = jt * BJ;
    return t.s.group >= 0;
}

// A wavefront's 16 TI x 16 TJ results from row i0 and column j0 on.  A lane has four columns of a row; in 16 bits, lanes of
// neighbouring columns exchange halves, so that a store is 16 bytes of a lane and 64 contiguous ones of a row (8192 x 4096 x
// 64, two rounds of tiles: 38.7 us with 8-byte stores, 21.8 so).
template <int OP, typename Y, int TI, int TJ> __device__ __forceinline__ void store_tile(const Product& a, const Tile& t, int32_t i0, int32_t j0, int lane, const f32x4 (&acc)[TJ][TI]) {
    constexpr int SIZE = sizeof(Y), VALUES = 16 / SIZE, TILES = 4 / SIZE;       // of a store: values, tiles of columns
    static_assert(TJ % TILES == 0, "tiles of columns in pairs");
    Y* const y = static_cast<Y*>(a.y) + (OP == DW ? t.s.group * a.y_group : 0);
    const int q = lane >> 4;
    j0 += SIZE == 2 ? (q & 1) * 16 + (q >> 1) * 8 : q * 4;
#pragma unroll
    for (int i = 0; i < TI; i++) {
        const int32_t row = i0 + i * 16 + (lane & 15);
        const bool zero = OP == FWD && a.source && source_of(a, min(row, t.i_end - 1)) < 0;
#pragma unroll
        for (int j = 0; j < TJ; j += TILES) {
            typedef uint32_t u32x4 __attribute__((ext_vector_type(4), aligned(8)));        // y may be aligned to 8 bytes only
            u32x4 v;
            if constexpr (SIZE == 2) {
                auto pack = [](f32x4 f) { return __builtin_bit_cast(uint2, vec<Y, 4>{Y(f[0]), Y(f[1]), Y(f[2]), Y(f[3])}); };
                const uint2 l = pack(acc[j][i]), r = pack(acc[j + 1][i]);
                // l's odd rows of 16 lanes change places with r's even ones
                const auto x = __builtin_amdgcn_permlane16_swap(l.x, r.x, false, false), y = __builtin_amdgcn_permlane16_swap(l.y, r.y, false, false);
                v = u32x4{x[0], y[0], x[1], y[1]};
            } else {
                v = __builtin_bit_cast(u32x4, acc[j][i]);
            }
            if (zero) v = u32x4{0, 0, 0, 0};
            const int32_t col = j0 + j * 16;
            if (row >= t.i_end || col >= a.cols) continue;
            Y* const p = y + int64_t(row) * a.ldy + col;
            if (col + VALUES <= a.cols) {
                *reinterpret_cast<u32x4*>(p) = v;
            } else {
                const vec<Y, VALUES> values = __builtin_bit_cast(vec<Y, VALUES>, v);
#pragma unroll
                for (int e = 0; e < VALUES; e++)
                    if (col + e < a.cols) p[e] = values[e];
            }
        }
    }
}

// Where a straight tile's rows are.  With a source, from the beginning of x on; then an offset may pass 32 bits (a.far).
template <typename T, int OP, typename X> __device__ __forceinline__ void start_x(const Product& a, const Tile& t, int lane, int wave, X& tx) {
    const T* const x = static_cast<const T*>(a.x);
    const int64_t pitch = a.ldx * int64_t(sizeof(T));
    const bool by_source = OP == FWD && a.source;
    tx.start(lane, wave, by_source ? x : x + int64_t(t.i0) * a.ldx, [&](int r) {
        const int32_t i = min(t.i0 + r, t.i_end - 1);
        return (by_source ? max(source_of(a, i), int64_t(0)) : i - t.i0) * pitch;
    });
}
template <typename T, typename W> __device__ __forceinline__ void start_w(const Product& a, const Tile& t, int lane, int wave, W& tw) {
    const T* const w = static_cast<const T*>(a.w) + t.s.group * a.w_group + int64_t(t.j0) * a.ldw;
    tw.start(lane, wave, w, [&](int r) { return min(r, a.cols - 1 - t.j0) * (a.ldw * int64_t(sizeof(T))); });
}

// 16 bits.  A step is 64 values of the depth, in two halves of TI rows of TJ matrix instructions.  The operands of a half are
// read while the one before it is multiplied.  After the first half of step s both tiles of s have been read: at the
// barrier there, those of step s + 1 have to have landed.  LDS is a ring of five tiles, w 0, x 0, w 1, x 1 and so on; in the
// second half of step s the tiles x s + 2 and w s + 3 are asked for, in the places of w s and x s.  So half of the loads
// have a step to land, the others two.  Reads and loads are dealt out between the rows of products: together they held them up.
// Bound by the matrix instructions at the clock that the card's power leaves them: 8192^3 in bf16 746 us, 1470 TFLOP/s (dx
// 747, dw 789; matrix instructions alone 711; with zeros for data a fifth less), the matrix pipe busy 76% of the cycles.  A
// tile costs about 8 us beside its steps: 756 GFLOP over 32 groups of 2048 rows or so, 2816 x 2048, 670 us, 1130 TFLOP/s.
template <typename T, int OP, int BI, int BJ, int WI, int WJ>
__global__ __launch_bounds__(WI * WJ * 64, BI * BJ / (WI * WJ) < 64 * 64 ? 4 : 2) void k_product(Product a, int row_tiles, int col_tiles) {
    constexpr int WAVES = WI * WJ, TI = BI / WI / 16, TJ = BJ / WJ / 16, TILE = BI * 128, RING = 5;
    static_assert(BI == BJ && TI >= 4 && TJ % 2 == 0, "places of a ring");
    constexpr bool X_TURNED = OP == DW, W_TURNED = OP != FWD;
    using X = std::conditional_t<X_TURNED, Turned<BI, WAVES>, Straight<BI, WAVES>>;
    using W = std::conditional_t<W_TURNED, Turned<BJ, WAVES>, Straight<BJ, WAVES>>;
    constexpr int LOADS = X::LOADS, EACH = 2 * LOADS / TI;      // loads of a tile, loads beside a row
    static_assert(X::LOADS == W::LOADS && 2 * LOADS % TI == 0, "loads are dealt out evenly");
    __shared__ __align__(1024) uint8_t lds[RING * TILE];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Tile t;
    if (!find<OP, BI, BJ>(a, row_tiles, col_tiles, t)) return;
    const T* const w = static_cast<const T*>(a.w) + (OP == DW ? 0 : t.s.group * a.w_group);
    const T* const x = static_cast<const T*>(a.x);
    const bool by_source = OP == DW && a.source;
    X tx;
    W tw;
    if constexpr (X_TURNED) {
        tx.start(lane, wave, x + int64_t(t.s.first) * a.ldx, a.ldx, t.i0, t.i_end);
    } else {
        start_x<T, OP>(a, t, lane, wave, tx);
    }
    if constexpr (W_TURNED) {
        tw.start(lane, wave, OP == DW && !by_source ? w + int64_t(t.s.first) * a.ldw : w, a.ldw, t.j0, a.cols);
        if (by_source) tw.by_source(a.source + t.s.first, t.depth, wave);
    } else {
        start_w<T>(a, t, lane, wave, tw);
    }
    // load q of the tile of the step from c0 on (past the depth: zeros)
    auto load_x = [&](auto fast, int q, uint8_t* tile, int32_t c0) __attribute__((always_inline)) {
        constexpr bool FAST = decltype(fast)::value;
        if constexpr (X_TURNED) tx.template load<FAST>(q, tile, wave, t.depth - c0);
        else tx.template load<FAST>(q, tile, wave, int64_t(t.depth - c0) * 2);
    };
    auto load_w = [&](auto fast, int q, uint8_t* tile, int32_t c0) __attribute__((always_inline)) {
        constexpr bool FAST = decltype(fast)::value;
        if constexpr (OP == DW) {
            if (by_source) {
                tw.template load_by_source<FAST>(q, tile, wave, t.depth - c0, a.source_rows);
                if (q == LOADS - 1) tw.by_source(a.source + t.s.first + c0 + 64, t.depth - c0 - 64, wave);
                return;
            }
        }
        if constexpr (W_TURNED) tw.template load<FAST>(q, tile, wave, t.depth - c0);
        else tw.template load<FAST>(q, tile, wave, int64_t(t.depth - c0) * 2);
    };
    auto load_row = [&](auto fast, int i, uint8_t* xt, uint8_t* wt, int32_t c0) __attribute__((always_inline)) {     // those beside row i: x of the step from c0 on, w of the next
        constexpr bool FAST = decltype(fast)::value;
#pragma unroll
        for (int p = i * EACH; p < (i + 1) * EACH; p++) {
            if (p < LOADS) {
                if (FAST || c0 < t.depth) load_x(fast, p, xt, c0);
            } else {
                if (FAST || c0 + 64 < t.depth) load_w(fast, p - LOADS, wt, c0 + 64);
            }
        }
    };

    f32x4 acc[TJ][TI] = {};
    const int wi = wave / WJ * (TI * 16), wj = wave % WJ * (TJ * 16);      // this wavefront's part of the tile
    const bool some = __builtin_amdgcn_readfirstlane(t.i0 + wi < t.i_end); // ... has a row
    const uint32_t x_at = X::where(wi, lane), w_at = W::where(wj, lane);
    // X's rows but the last two are read into the registers of the rows just multiplied; W's and those have two sets.
    struct Operands {
        uint4 w[TJ], last[2];
    };
    uint4 rows[TI - 2];
    // A half: its products, the reads of the half k from these tiles, and, LOAD, the loads into x_free, w_free.
    auto half = [&](auto load, auto fast, const Operands& now, Operands& next, const uint8_t* xt, const uint8_t* wt, int k, uint8_t* x_free, uint8_t* w_free, int32_t c0) __attribute__((always_inline)) {
        constexpr bool LOAD = decltype(load)::value;
        if (!some) {
            if (LOAD)
#pragma unroll
                for (int i = 0; i < TI; i++) load_row(fast, i, x_free, w_free, c0);
            return;
        }
        const uint32_t xr = lds_address(xt) + x_at, wr = lds_address(wt) + w_at;
#pragma unroll
        for (int i = 0; i < TI; i++) {
            if (i < 2)
#pragma unroll
                for (int j = i * TJ / 2; j < (i + 1) * TJ / 2; j++) next.w[j] = W::read(wr, j, k);
            else if (i < 4) next.last[i - 2] = X::read(xr, TI - 4 + i, k);
            if (i > 0 && i < TI - 1) rows[i - 1] = X::read(xr, i - 1, k);
            if (LOAD) load_row(fast, i, x_free, w_free, c0);
#pragma unroll
            for (int j = 0; j < TJ; j++) acc[j][i] = multiply(now.w[j], i < TI - 2 ? rows[i] : now.last[i - TI + 2], acc[j][i], T());
            __builtin_amdgcn_sched_barrier(0);
        }
    };
    if (t.depth > 0) {
        Operands even, odd;
        // tiles in the ring: w 0, x 0, w 1, x 1, w 2
        uint8_t* place[RING] = {lds, lds + TILE, lds + 2 * TILE, lds + 3 * TILE, lds + 4 * TILE};
#pragma unroll
        for (int s = 0; s < RING; s++) {
            if (s / 2 * 64 >= t.depth) continue;
#pragma unroll
            for (int q = 0; q < LOADS; q++) {
                if (s & 1) {
                    load_x(std::false_type(), q, place[s], s / 2 * 64);
                } else {
                    if constexpr (OP == DW) {
                        if (by_source && q == 0) tw.here(lane, a.source_rows);
                    }
                    load_w(std::false_type(), q, place[s], s / 2 * 64);
                }
            }
        }
        if (t.depth > 128) landed<3 * LOADS>();
        else landed<0>();
        const uint32_t xr = lds_address(place[1]) + x_at, wr = lds_address(place[0]) + w_at;
#pragma unroll
        for (int j = 0; j < TJ; j++) even.w[j] = W::read(wr, j, 0);
#pragma unroll
        for (int i = 0; i < TI - 2; i++) rows[i] = X::read(xr, i, 0);
        even.last[0] = X::read(xr, TI - 2, 0), even.last[1] = X::read(xr, TI - 1, 0);
        uint8_t *w_now = place[0], *x_now = place[1], *w_next = place[2], *x_next = place[3], *w_after = place[4];
        auto step = [&](auto fast, int32_t c0) __attribute__((always_inline)) {
            half(std::false_type(), fast, even, odd, x_now, w_now, 1, nullptr, nullptr, 0);
            // all but the loads of w_after, where there are some
            if (decltype(fast)::value || c0 + 128 < t.depth) landed<LOADS>();
            else landed<0>();
            if constexpr (OP == DW) {
                if (by_source) tw.here(lane, a.source_rows);
            }
            // x of the step after the next goes to w_now, w of the one after that to x_now
            half(std::true_type(), fast, odd, even, x_next, w_next, 0, w_now, x_now, c0 + 128);
            uint8_t *const xa = w_now, *const wa = x_now;
            w_now = w_next, x_now = x_next, w_next = w_after, x_next = xa, w_after = wa;
        };
        int32_t c0 = 0;
        if (!a.far)
            for (; c0 + 256 <= t.depth; c0 += 64) step(std::true_type(), c0);
        for (; c0 < t.depth; c0 += 64) step(std::false_type(), c0);
        landed<0>();            // nothing is on its way to this LDS when it becomes another workgroup's
    }
    store_tile<OP, T>(a, t, t.i0 + wi, t.j0 + wj, lane, acc);
}

// 8 bits.  A step is a block of 128 values: one matrix instruction per 16 x 16 results (four where they stay in 32 bits), which
// starts from 0 and whose result is scaled and added in 32 bits, beside the instructions of the next row of tiles.  LDS holds two tiles of w, XRING of x and three sets of scales.  Two rows of tiles before a step's
// end everything of the step has been read; at the barrier there the next step has to have landed, and its first operands
// are read beside the last two rows.  From there on the loads of w s + 2 are asked for, then, XRING = 3, of x s + 3: that
// half of the loads has two steps to land.  W1: a scale per row of w.
// Bound by power as above and by what a wavefront issues beside the products (four adds for each): 8192^3 483 us, 2275
// TFLOP/s, the matrix pipe busy 55% of the cycles (on another card 528; 1111 with results in 32 bits); without loads 2530
// TFLOP/s, without LDS reads 2880.  A scale per row of w costs a seventh more (603 for the 528), for the registers and LDS reads of
// four scales instead of one.  Short depths pay for their tiles: 275 GFLOP in 64 groups of 512 rows, 2048 x 2048, 191 to 203 us.
template <typename Y, int BI, int BJ, int WI, int WJ, int XRING, bool W1>
__global__ __launch_bounds__(WI * WJ * 64, 2) void k_product_f8(Product a, int row_tiles, int col_tiles) {
    constexpr int WAVES = WI * WJ, TI = BI / WI / 16, TJ = BJ / WJ / 16;
    static_assert(BI + BJ <= WAVES * 64 && 128 % (TJ * 16) == 0 && TI >= 4, "a thread per scale; a wavefront's columns share one");
    using X = Straight<BI, WAVES>;
    using W = Straight<BJ, WAVES>;
    constexpr int LOADS = W::LOADS + 1 + X::LOADS, EACH = (LOADS + TI - 2) / (TI - 1), SETS = TI % 3 ? 4 : 3;
    constexpr int X_TILE = BI * 128, W_TILE = BJ * 128, S_TILE = WAVES * 256;
    __shared__ __align__(1024) uint8_t lds[XRING * X_TILE + 2 * W_TILE + 3 * S_TILE];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    Tile t;
    if (!find<FWD, BI, BJ>(a, row_tiles, col_tiles, t)) return;
    X tx;
    W tw;
    start_x<f8, FWD>(a, t, lane, wave, tx);
    start_w<f8>(a, t, lane, wave, tw);
    // A thread's scale: the first wavefronts' of x, the next ones' of w (whatever the last ones get is not used).
    const bool of_x = wave * 64 < BI;
    const float* scale = same(of_x ? a.xs : a.ws + t.s.group * a.ws_group);
    const int64_t scale_step = of_x ? a.xs_block : a.ws_block;
    const int64_t scale_at = of_x ? max(source_of(a, min(t.i0 + tid, t.i_end - 1)), int64_t(0)) * a.xs_row : min(t.j0 + tid - BI, a.cols - 1) / a.w_rows * a.ws_row;
    auto load_scales = [&](auto fast, uint8_t* tile, int32_t c0) __attribute__((always_inline)) {
        if (decltype(fast)::value) word_to_lds(scale, uint32_t(scale_at) * 4, tile + wave * 256);
        else word_to_lds(c0 < t.depth ? static_cast<const void*>(scale + scale_at) : &ZEROS, tile + wave * 256);
        scale += scale_step;
    };

    f32x4 acc[TJ][TI] = {};
    const int wi = wave / WJ * (TI * 16), wj = wave % WJ * (TJ * 16);
    const uint32_t x_at = X::where(wi, lane), w_at = W::where(wj, lane);
    auto both = [](uint4 lo, uint4 hi) { return i32x8{int(lo.x), int(lo.y), int(lo.z), int(lo.w), int(hi.x), int(hi.y), int(hi.z), int(hi.w)}; };
    if (t.depth > 0) {
        uint8_t *x_now = lds, *x_next = lds + X_TILE, *x_free = lds + (XRING - 1) * X_TILE;
        uint8_t *w_now = lds + XRING * X_TILE, *w_next = w_now + W_TILE;
        uint8_t *s_now = w_next + W_TILE, *s_next = s_now + S_TILE, *s_after = s_next + S_TILE;
        // Turn `turn` of the loads that a step's barrier lets go: w and the scales of the step from c0 on, then x of that
        // or, XRING = 3, the next one.
        auto load = [&](auto fast, int turn, uint8_t* wt, uint8_t* st, uint8_t* xt, int32_t c0) __attribute__((always_inline)) {
            constexpr bool FAST = decltype(fast)::value;
#pragma unroll
            for (int p = turn * EACH; p < min((turn + 1) * EACH, LOADS); p++) {
                if (p < W::LOADS) tw.template load<FAST>(p, wt, wave, t.depth - c0);
                else if (p == W::LOADS) load_scales(fast, st, c0);
                else tx.template load<FAST>(p - W::LOADS - 1, xt, wave, t.depth - c0 - (XRING - 2) * 128);
            }
        };
        // As a step finds it: step 0 (of x, XRING = 3, step 1 too), and the first two turns of what comes next.
#pragma unroll
        for (int q = 0; q < W::LOADS; q++) tw.template load<false>(q, w_now, wave, t.depth);
        load_scales(std::false_type(), s_now, 0);
#pragma unroll
        for (int r = 0; r < XRING - 1; r++)
#pragma unroll
            for (int q = 0; q < X::LOADS; q++) tx.template load<false>(q, lds + r * X_TILE, wave, t.depth - r * 128);
        landed<0>();
        load(std::false_type(), 0, w_next, s_next, x_free, 128);
        load(std::false_type(), 1, w_next, s_next, x_free, 128);
        i32x8 wv[TJ], xv[SETS];         // w's operands, x's two rows ahead of the products
        f32x4 part[2][TJ] = {}, ws[W1 ? TJ : 1] = {}, ws_before[W1 ? TJ : 1];
        float before = 0.f, one_before = 0.f;       // x's scale of the row of tiles before, w's
#pragma unroll
        for (int j = 0; j < TJ; j++) wv[j] = both(W::read(lds_address(w_now) + w_at, j, 0), W::read(lds_address(w_now) + w_at, j, 1));
#pragma unroll
        for (int i = 0; i < 2; i++) xv[i] = both(X::read(lds_address(x_now) + x_at, i, 0), X::read(lds_address(x_now) + x_at, i, 1));
        auto step = [&](auto fast, int32_t c0) __attribute__((always_inline)) {
            const float* const xs_at = reinterpret_cast<const float*>(s_now) + wi + (lane & 15);
            const float* const ws_at = reinterpret_cast<const float*>(s_now) + BI + wj;
            float one = 1.f;
            if (W1) {
#pragma unroll
                for (int j = 0; j < TJ; j++) ws_before[W1 ? j : 0] = ws[W1 ? j : 0], ws[W1 ? j : 0] = *reinterpret_cast<const f32x4*>(ws_at + j * 16 + (lane >> 4) * 4);
            } else {
                one = *ws_at;
            }
#pragma unroll
            for (int i = 0; i < TI; i++) {
                if (i == TI - 2) landed<(XRING - 2) * X::LOADS>();
                // From the barrier on the loads into what has been read: w_now, the scales of the step before, x_now.
                if (i >= TI - 2) load(fast, i - (TI - 2), w_now, s_after, x_now, c0 + 256);
                else load(fast, i + 2, w_next, s_next, x_free, c0 + 128);
                const uint32_t xr = lds_address(i < TI - 2 ? x_now : x_next) + x_at, wr = lds_address(w_next) + w_at;
                const int e = i < TI - 2 ? i + 2 : i - (TI - 2);
                xv[(i + 2) % SETS] = both(X::read(xr, e, 0), X::read(xr, e, 1));
                const float by_x = before * one_before, xs = xs_at[i * 16];
#pragma unroll
                for (int j = 0; j < TJ; j++) {
                    part[i & 1][j] = multiply_block<Y>(wv[j], xv[i % SETS]);
                    if (i == TI - 1) wv[j] = both(W::read(wr, j, 0), W::read(wr, j, 1));
                    f32x4& to = acc[j][(i + TI - 1) % TI];
                    const f32x4 by = i > 0 ? ws[W1 ? j : 0] : ws_before[W1 ? j : 0];
#pragma unroll
                    for (int q = 0; q < 4; q++) to[q] = fmaf(part[~i & 1][j][q], W1 ? before * by[q] : by_x, to[q]);
                    __builtin_amdgcn_sched_barrier(0);
                }
                before = xs, one_before = one;
            }
            uint8_t *const w_old = w_now, *const x_old = x_now, *const s_old = s_now;
            w_now = w_next, w_next = w_old;
            s_now = s_next, s_next = s_after, s_after = s_old;
            x_now = x_next, x_next = XRING == 3 ? x_free : x_old, x_free = x_old;
        };
        int32_t c0 = 0;
        if (!a.far)
            for (; c0 + 128 * (XRING + 1) <= t.depth; c0 += 128) step(std::true_type(), c0);
        for (; c0 < t.depth; c0 += 128) step(std::false_type(), c0);
#pragma unroll
        for (int j = 0; j < TJ; j++)        // the last row of tiles
#pragma unroll
            for (int q = 0; q < 4; q++) acc[j][TI - 1][q] = fmaf(part[(TI - 1) & 1][j][q], W1 ? before * ws[W1 ? j : 0][q] : before * one_before, acc[j][TI - 1][q]);
        landed<0>();            // nothing is on its way to this LDS when it becomes another workgroup's
    }
    store_tile<FWD, Y>(a, t, t.i0 + wi, t.j0 + wj, lane, acc);
}

// ---------------------------------------------------------------------------------------------------------------
// Few rows (a step of serving): bound by reading the weights once.  A workgroup of 8 wavefronts has 16 columns and 16 TI rows;
// its wavefronts take the steps of the depth by turns, several at a time, from memory straight into the registers of the
// matrix instructions (a load takes 64 contiguous bytes of 16 rows), and add up their sums in LDS in a fixed order.  64 rows
// over 64 experts of 1536 x 2048 in bf16 41 us, 6.2 TB/s of the weights they name; 8 rows by 8192 x 4096 in 8 bits 9.2 us, 3.6 TB/s.
// ---------------------------------------------------------------------------------------------------------------
constexpr int FEW_WAVES = 8;
// 8 bits: 32 columns to a workgroup where that still makes 256 of them (8 x 8192 x 4096 10.2 us against 11.2 with 16; 8 x 4096 x
// 14336 25 against 16).  16 bits: always (64 rows over 64 groups of 1536 x 2048 46 against 49).
constexpr int FEW_WIDE = 32 * 256;

template <typename T, typename Y, int TI, int TJ, bool W1> __global__ __launch_bounds__(FEW_WAVES * 64) void k_product_few(Product a, int col_tiles) {
    constexpr bool F8 = is_f8<T>, WIDE = F8 && TJ == 2;
    constexpr int SIZE = sizeof(T), STEP = 128 / SIZE, AHEAD = WIDE ? 4 : 2, WS = W1 ? 4 : 1;
    __shared__ __align__(16) f32x4 sums[FEW_WAVES][TJ][TI][64];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), li = lane & 15, q = lane >> 4;
    const Span s = find_tile<16 * TI>(a, int32_t(blockIdx.x / col_tiles));
    if (s.group < 0) return;
    const int32_t j0 = int32_t(blockIdx.x % col_tiles) * (16 * TJ);
    const uint8_t *w[TJ], *x[TI];
    const float *xs[TI], *ws[TJ][WS];
#pragma unroll
    for (int j = 0; j < TJ; j++) {
        w[j] = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.w) + s.group * a.w_group + int64_t(min(j0 + j * 16 + li, a.cols - 1)) * a.ldw);
        if (F8)
#pragma unroll
            for (int c = 0; c < WS; c++) ws[j][c] = a.ws + s.group * a.ws_group + min(j0 + j * 16 + (W1 ? q * 4 + c : 0), a.cols - 1) / a.w_rows * a.ws_row;
    }
#pragma unroll
    for (int i = 0; i < TI; i++) {
        const int64_t r = max(source_of(a, min(s.first + i * 16 + li, s.last - 1)), int64_t(0));
        x[i] = reinterpret_cast<const uint8_t*>(static_cast<const T*>(a.x) + r * a.ldx);
        if (F8) xs[i] = a.xs + r * a.xs_row;
    }
    const int64_t bytes = int64_t(a.depth) * SIZE;
    const int steps = (a.depth + STEP - 1) / STEP;
    f32x4 acc[TJ][TI] = {};
    for (int at = wave; at < steps; at += FEW_WAVES * AHEAD) {
        uint4 wv[AHEAD][TJ][2], xv[AHEAD][TI][2];
        float xf[AHEAD][TI], wf[AHEAD][TJ][WS];
#pragma unroll
        for (int u = 0; u < AHEAD; u++) {
            const int b = at + u * FEW_WAVES;
#pragma unroll
            for (int k = 0; k < 2; k++) {
                const int64_t o = int64_t(b) * 128 + k * 64 + q * 16;
                const bool in = o < bytes;
#pragma unroll
                for (int j = 0; j < TJ; j++) wv[u][j][k] = *reinterpret_cast<const uint4*>(in ? w[j] + o : reinterpret_cast<const uint8_t*>(&ZEROS));
#pragma unroll
                for (int i = 0; i < TI; i++) xv[u][i][k] = *reinterpret_cast<const uint4*>(in ? x[i] + o : reinterpret_cast<const uint8_t*>(&ZEROS));
            }
            if (F8) {
                const int64_t block = min(b, steps - 1);
#pragma unroll
                for (int i = 0; i < TI; i++) xf[u][i] = b < steps ? xs[i][block * a.xs_block] : 0.f;
#pragma unroll
                for (int j = 0; j < TJ; j++)
#pragma unroll
                    for (int c = 0; c < WS; c++) wf[u][j][c] = b < steps ? ws[j][c][block * a.ws_block] : 0.f;
            }
        }
        if (!WIDE) __builtin_amdgcn_sched_barrier(0);       // all loads before the first product: the compiler would keep fewer in flight
#pragma unroll
        for (int u = 0; u < AHEAD; u++)
#pragma unroll
            for (int j = 0; j < TJ; j++)
#pragma unroll
                for (int i = 0; i < TI; i++) {
                    if constexpr (F8) {
                        const uint4 wl = wv[u][j][0], wh = wv[u][j][1], xl = xv[u][i][0], xh = xv[u][i][1];
                        const i32x8 w8 = {int(wl.x), int(wl.y), int(wl.z), int(wl.w), int(wh.x), int(wh.y), int(wh.z), int(wh.w)};
                        const i32x8 x8 = {int(xl.x), int(xl.y), int(xl.z), int(xl.w), int(xh.x), int(xh.y), int(xh.z), int(xh.w)};
                        const f32x4 part = multiply_block<Y>(w8, x8);
                        // Past the depth products and scales are 0.  No branch around the sum: where one skipped what reads a
                        // matrix instruction's result, the compiler wrote its registers again too early for the instruction,
                        // whose write came after (one in some thousand results was wrong).
#pragma unroll
                        for (int c = 0; c < 4; c++) acc[j][i][c] = fmaf(part[c], xf[u][i] * wf[u][j][W1 ? c : 0], acc[j][i][c]);
                    } else {
#pragma unroll
                        for (int k = 0; k < 2; k++) acc[j][i] = multiply(wv[u][j][k], xv[u][i][k], acc[j][i], T());
                    }
                }
    }
#pragma unroll
    for (int j = 0; j < TJ; j++)
#pragma unroll
        for (int i = 0; i < TI; i++) sums[wave][j][i][lane] = acc[j][i];
    __syncthreads();
    // a thread per four columns of a row
    for (int e = tid; e < TJ * TI * 64; e += FEW_WAVES * 64) {
        const int l = e % 64, i = e / 64 % TI, j = e / 64 / TI;
        f32x4 sum = sums[0][j][i][l];
#pragma unroll
        for (int v = 1; v < FEW_WAVES; v++) sum += sums[v][j][i][l];
        const int32_t row = s.first + i * 16 + (l & 15), col = j0 + j * 16 + (l >> 4) * 4;
        if (row >= s.last || col >= a.cols) continue;
        if (a.source && source_of(a, row) < 0) sum = f32x4{0, 0, 0, 0};
        store_four<Y, true>(static_cast<Y*>(a.y) + int64_t(row) * a.ldy + col, a.cols - col, sum);
    }
}

// ---------------------------------------------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------------------------------------------
// A launch has fewer than 2^32 threads.
bool threads_fit(int64_t groups, int threads) { return groups * threads <= int64_t(UINT32_MAX); }

template <typename T, typename Y, int OP> int launch_plain(const Product& a, hipStream_t s) {
    const int64_t cols = divide_up(a.cols, PLAIN_TILE);
    const int64_t tiles = OP == DW ? int64_t(a.groups) * divide_up(a.out_rows, PLAIN_TILE) : int64_t(divide_up(a.rows, PLAIN_TILE)) + (a.offset ? a.groups : 0);
    if (!threads_fit(tiles * cols, 256)) return CSR5_ERANGE;
    k_product_plain<T, Y, OP><<<uint32_t(tiles * cols), 256, 0, s>>>(a);
    return launched();
}

template <typename T, typename Y, int OP, int BI, int BJ, int WI, int WJ> int launch_tiled(const Product& a, hipStream_t s) {
    const int64_t cols = divide_up(a.cols, BJ);
    const int64_t rows = OP == DW ? int64_t(divide_up(a.out_rows, BI)) : int64_t(divide_up(a.rows, BI)) + (a.offset ? a.groups : 0);
    const int64_t grid = (rows * cols + 7) / 8 * 8 * (OP == DW ? a.groups : 1);
    if (!threads_fit(grid, WI * WJ * 64)) return CSR5_ERANGE;
    if constexpr (is_f8<T>) {
        constexpr int XRING = BI > 128 ? 3 : 2;         // 128 x 128: two workgroups on a CU
        if (a.w_rows == 1) k_product_f8<Y, BI, BJ, WI, WJ, XRING, true><<<uint32_t(grid), WI * WJ * 64, 0, s>>>(a, int(rows), int(cols));
        else k_product_f8<Y, BI, BJ, WI, WJ, XRING, false><<<uint32_t(grid), WI * WJ * 64, 0, s>>>(a, int(rows), int(cols));
    } else {
        k_product<T, OP, BI, BJ, WI, WJ><<<uint32_t(grid), WI * WJ * 64, 0, s>>>(a, int(rows), int(cols));
    }
    return launched();
}

template <typename T, typename Y, int TI, int TJ> int launch_few(const Product& a, hipStream_t s) {
    const int64_t cols = divide_up(a.cols, 16 * TJ), rows = int64_t(divide_up(a.rows, 16 * TI)) + (a.offset ? a.groups : 0);
    if (!threads_fit(rows * cols, FEW_WAVES * 64)) return CSR5_ERANGE;
    if (is_f8<T> && a.w_rows == 1) k_product_few<T, Y, TI, TJ, is_f8<T>><<<uint32_t(rows * cols), FEW_WAVES * 64, 0, s>>>(a, int(cols));
    else k_product_few<T, Y, TI, TJ, false><<<uint32_t(rows * cols), FEW_WAVES * 64, 0, s>>>(a, int(cols));
    return launched();
}
template <typename T, typename Y, int TI> int launch_few(const Product& a, hipStream_t s) {
    if constexpr (is_f8<T>)
        if (int64_t(a.cols) * divide_up(a.rows, 16 * TI) < FEW_WIDE) return launch_few<T, Y, TI, 1>(a, s);
    return launch_few<T, Y, TI, 2>(a, s);
}

// Offsets that do not fit 32 bits.
constexpr int64_t MOST_BYTES = int64_t(1) << 32;
bool far(const Product& a, int64_t named_pitch) {
    auto past = [](int64_t rows, int64_t pitch) { return pitch < 0 || rows * pitch >= MOST_BYTES; };
    return (a.source && past(a.source_rows, named_pitch)) || past(a.source_rows, a.xs_row * 4) || past(a.cols, a.ws_row * 4);
}

// Rows of whole 16-byte chunks, at 16-byte addresses, a tile of which offsets of 32 bits reach; results at addresses of four
// values; and a row of x to read in place of those that a source does not name.
template <typename T, typename Y, int OP> bool chunks_fit(const Product& a) {
    constexpr int SIZE = sizeof(T);
    auto whole = [](int64_t n) { return n * SIZE % 16 == 0; };
    return aligned(a.x, a.ldx, SIZE, 16) && aligned(a.w, a.ldw, SIZE, 16) && whole(a.w_group) && aligned(a.y, a.ldy, sizeof(Y), 4 * sizeof(Y)) &&
           a.y_group % 4 == 0 && a.ldx * SIZE < MOST_BYTES / 256 && a.ldw * SIZE < MOST_BYTES / 256 && (OP != FWD || !a.source || int64_t(a.source_rows) * a.ldx * SIZE < 16 * MOST_BYTES) &&
           (OP != FWD || a.source_rows > 0) && (OP == FWD ? whole(a.depth) : OP == DX ? whole(a.depth) && whole(a.cols) : whole(a.out_rows) && whole(a.cols));
}

// Which kernel.  Measured at k = 1408 to 4096, n = 1024 to 8192 (us in 16 bits, in 8):
//   few rows    groups of up to 12 rows on average (8 bits: 4): 64 groups of 1536 x 2048 with 10 rows each 86 against 97 in
//               128 x 128 tiles, with 16 rows 112 against 103; 8 bits with 6 rows 57 against 53; and where there are so few
//               tiles that a step of their depth takes as long whatever they are: 32 rows of n = 8192, k = 4096 21 against 34
//               (12 against 20), 64 of them 36 against 35 (23 against 22)
//   64 x 128    8 bits, up to 128 tiles of 128 x 128: 512 rows of 2048 x 2048 12.6 in 128 x 128, 9.8 so; 200 of 8192 x 8192 48, 41;
//               1024 of 2048 x 4096 28, 22; with 256 tiles of 128 x 128 (1024 of 4096 x 8192) 52, 53, with 512 40, 53
//   128 x 128   by four wavefronts, DW by eight (2048 x 2048 of 2048 rows 22 against 26; the others gain nothing by it)
//   large tiles 256 rows and more where there are enough to go round the CUs: 4096 x 4096 x 2048 55 against 67, 2048 x 4096 x
//               4096 78 against 61
constexpr int FEW_ROWS16 = 12, FEW_ROWS8 = 4, FEW_AREA = 12288;
constexpr int LARGE_TILES = 192;
constexpr int HALF_TILES = 128;

template <typename T, typename Y, int OP> int launch(Product a, hipStream_t s) {
    constexpr bool F8 = is_f8<T>;
    if (!chunks_fit<T, Y, OP>(a)) return launch_plain<T, Y, OP>(a, s);
    a.far = far(a, (OP == DW ? a.ldw : a.ldx) * int64_t(sizeof(T)));
    const int64_t height = OP == DW ? a.out_rows : a.rows / a.groups;
    if constexpr (OP == FWD) {
        const int64_t tiles = divide_up(a.rows, 32) + (a.offset ? a.groups - 1 : 0);
        if (height <= (F8 ? FEW_ROWS8 : FEW_ROWS16) || tiles * a.cols <= FEW_AREA)
            return height <= 16 ? launch_few<T, Y, 1>(a, s) : launch_few<T, Y, 2>(a, s);
    }
    constexpr int BI = F8 ? 192 : 256;
    const int64_t large = (OP == DW ? int64_t(a.groups) * divide_up(a.out_rows, BI) : a.rows / BI + (a.offset ? a.groups / 2 : 0)) * divide_up(a.cols, 256);
    if constexpr (!F8 || sizeof(Y) == 2)        // sums of 8 bits in 32 have no registers for them
        if (height >= 192 && large >= LARGE_TILES) return launch_tiled<T, Y, OP, BI, 256, 2, 4>(a, s);
    if constexpr (F8)
        if ((a.rows / 128 + (a.offset ? a.groups / 2 : 0)) * int64_t(divide_up(a.cols, 128)) <= HALF_TILES) return launch_tiled<T, Y, OP, 64, 128, 1, 4>(a, s);
    return launch_tiled<T, Y, OP, 128, 128, 2, OP == DW ? 4 : 2>(a, s);
}

bool half_type(int dtype) { return dtype == CSR5_DTYPE_BF16 || dtype == CSR5_DTYPE_F16; }
template <int OP> int launch_half(int dtype, const Product& a, void* hip_stream) {
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return dtype == CSR5_DTYPE_BF16 ? launch<bf16, bf16, OP>(a, s) : launch<f16, f16, OP>(a, s);
}

int launch_f8(int dtype, const Product& a, void* hip_stream) {
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    switch (dtype) {
        case CSR5_DTYPE_BF16: return launch<f8, bf16, FWD>(a, s);
        case CSR5_DTYPE_F16: return launch<f8, f16, FWD>(a, s);
        default: return launch<f8, float, FWD>(a, s);
    }
}

bool groups_ok(int32_t groups, int32_t rows, int32_t n, int32_t k, const int32_t* offset) {
    return groups >= 0 && rows >= 0 && n >= 0 && k >= 0 && (groups == 0 || offset) && !(reinterpret_cast<uintptr_t>(offset) & 3);
}
bool sizes_fit(int32_t groups, int32_t rows, int32_t n, int32_t k) { return max(max(groups, rows), max(n, k)) <= MOST_SIZE; }
// what `source` may name is there
bool source_ok(int32_t rows, int32_t x_rows, const int32_t* source) {
    return x_rows >= 0 && (source || x_rows >= rows) && !(reinterpret_cast<uintptr_t>(source) & 3);
}

}  // namespace

extern "C" {

int csr5_grouped_gemm(int32_t groups, int32_t rows, int32_t n, int32_t k, int dtype, const int32_t* offset, const void* x, int32_t x_rows,
                      int64_t ldx, const int32_t* source, const void* w, int64_t ldw, int64_t w_group, void* y, int64_t ldy, void* hip_stream) {
    if (!half_type(dtype) || !groups_ok(groups, rows, n, k, offset) || !source_ok(rows, x_rows, source)) return CSR5_EINVAL;
    if (!sizes_fit(groups, rows, n, k)) return CSR5_ERANGE;
    if (!rows_ok(x, x_rows, ldx, k, 2) || !rows_ok(w, int64_t(groups) * n, ldw, k, 2) || !rows_ok(y, rows, ldy, n, 2)) return CSR5_EINVAL;
    if (groups == 0 || rows == 0 || n == 0) return CSR5_OK;
    Product a{};
    a.x = x, a.ldx = ldx, a.w = w, a.ldw = ldw, a.w_group = w_group, a.y = y, a.ldy = ldy;
    a.offset = offset, a.source = source, a.source_rows = x_rows, a.groups = groups, a.rows = rows, a.cols = n, a.depth = k;
    return launch_half<FWD>(dtype, a, hip_stream);
}

int csr5_grouped_gemm_dx(int32_t groups, int32_t rows, int32_t n, int32_t k, int dtype, const int32_t* offset, const void* dy, int64_t lddy,
                         const void* w, int64_t ldw, int64_t w_group, void* dx, int64_t lddx, void* hip_stream) {
    if (!half_type(dtype) || !groups_ok(groups, rows, n, k, offset)) return CSR5_EINVAL;
    if (!sizes_fit(groups, rows, n, k)) return CSR5_ERANGE;
    if (!rows_ok(dy, rows, lddy, n, 2) || !rows_ok(w, int64_t(groups) * n, ldw, k, 2) || !rows_ok(dx, rows, lddx, k, 2)) return CSR5_EINVAL;
    if (groups == 0 || rows == 0 || k == 0) return CSR5_OK;
    Product a{};
    a.x = dy, a.ldx = lddy, a.w = w, a.ldw = ldw, a.w_group = w_group, a.y = dx, a.ldy = lddx;
    a.offset = offset, a.groups = groups, a.rows = rows, a.cols = k, a.depth = n;
    return launch_half<DX>(dtype, a, hip_stream);
}

int csr5_grouped_gemm_dw(int32_t groups, int32_t rows, int32_t n, int32_t k, int dtype, const int32_t* offset, const void* dy, int64_t lddy,
                         const void* x, int32_t x_rows, int64_t ldx, const int32_t* source, void* dw, int64_t lddw, int64_t dw_group, void* hip_stream) {
    if (!half_type(dtype) || !groups_ok(groups, rows, n, k, offset) || !source_ok(rows, x_rows, source)) return CSR5_EINVAL;
    if (!sizes_fit(groups, rows, n, k)) return CSR5_ERANGE;
    if (!rows_ok(dy, rows, lddy, n, 2) || !rows_ok(x, x_rows, ldx, k, 2) || !rows_ok(dw, int64_t(groups) * n, lddw, k, 2)) return CSR5_EINVAL;
    if (groups == 0 || n == 0 || k == 0) return CSR5_OK;
    Product a{};
    a.x = dy, a.ldx = lddy, a.w = x, a.ldw = ldx, a.y = dw, a.ldy = lddw, a.y_group = dw_group;
    a.offset = offset, a.source = source, a.source_rows = x_rows, a.groups = groups, a.rows = rows, a.out_rows = n, a.cols = k;
    return launch_half<DW>(dtype, a, hip_stream);
}

int csr5_grouped_gemm_f8(int32_t groups, int32_t rows, int32_t n, int32_t k, int dtype, const int32_t* offset, const uint8_t* x, int32_t x_rows,
                         int64_t ldx, const float* x_scale, int64_t xs_row, int64_t xs_block, const int32_t* source, const uint8_t* w, int64_t ldw,
                         int64_t w_group, const float* w_scale, int32_t w_rows, int64_t ws_row, int64_t ws_block, int64_t ws_group, void* y,
                         int64_t ldy, void* hip_stream) {
    const size_t size = half_type(dtype) ? 2 : 4;
    if (!(half_type(dtype) || dtype == CSR5_DTYPE_F32) || !groups_ok(groups, rows, n, k, offset) || !source_ok(rows, x_rows, source)) return CSR5_EINVAL;
    if (!sizes_fit(groups, rows, n, k)) return CSR5_ERANGE;
    if (w_rows != 1 && w_rows != CSR5_F8_BLOCK) return CSR5_EINVAL;
    if (!rows_ok(x, x_rows, ldx, k, 1) || !rows_ok(w, int64_t(groups) * n, ldw, k, 1) || !rows_ok(y, rows, ldy, n, size)) return CSR5_EINVAL;
    if (groups == 0 || rows == 0 || n == 0) return CSR5_OK;
    if (k > 0 && ((x_rows > 0 && !x_scale) || !w_scale || ((reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(w_scale)) & 3))) return CSR5_EINVAL;
    Product a{};
    a.x = x, a.ldx = ldx, a.w = w, a.ldw = ldw, a.w_group = w_group, a.y = y, a.ldy = ldy;
    a.offset = offset, a.source = source, a.source_rows = x_rows, a.groups = groups, a.rows = rows, a.cols = n, a.depth = k;
    a.xs = x_scale, a.xs_row = xs_row, a.xs_block = xs_block;
    a.ws = w_scale, a.ws_row = ws_row, a.ws_block = ws_block, a.ws_group = ws_group, a.w_rows = w_rows;
    return launch_f8(dtype, a, hip_stream);
}

int csr5_gemm_f8(int32_t m, int32_t n, int32_t k, int dtype, const uint8_t* x, int64_t ldx, const float* x_scale, int64_t xs_row, int64_t xs_block,
                 const uint8_t* w, int64_t ldw, const float* w_scale, int32_t w_rows, int64_t ws_row, int64_t ws_block, void* y, int64_t ldy,
                 void* hip_stream) {
    const size_t size = half_type(dtype) ? 2 : 4;
    if (!(half_type(dtype) || dtype == CSR5_DTYPE_F32) || m < 0 || n < 0 || k < 0 || (w_rows != 1 && w_rows != CSR5_F8_BLOCK)) return CSR5_EINVAL;
    if (!sizes_fit(1, m, n, k)) return CSR5_ERANGE;
    if (!rows_ok(x, m, ldx, k, 1) || !rows_ok(w, n, ldw, k, 1) || !rows_ok(y, m, ldy, n, size)) return CSR5_EINVAL;
    if (m == 0 || n == 0) return CSR5_OK;
    if (k > 0 && (!x_scale || !w_scale || ((reinterpret_cast<uintptr_t>(x_scale) | reinterpret_cast<uintptr_t>(w_scale)) & 3))) return CSR5_EINVAL;
    Product a{};
    a.x = x, a.ldx = ldx, a.w = w, a.ldw = ldw, a.y = y, a.ldy = ldy;
    a.source_rows = m, a.groups = 1, a.rows = m, a.cols = n, a.depth = k;
    a.xs = x_scale, a.xs_row = xs_row, a.xs_block = xs_block;
    a.ws = w_scale, a.ws_row = ws_row, a.ws_block = ws_block, a.w_rows = w_rows;
    return launch_f8(dtype, a, hip_stream);
}

}  // extern "C"
