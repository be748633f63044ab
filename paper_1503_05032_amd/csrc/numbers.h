// Types, rounding, rows and sums over a wavefront, for the kernels of a layer of experts.
#ifndef CSR5_NUMBERS_H
#define CSR5_NUMBERS_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

typedef __bf16 bf16;
typedef _Float16 f16;
template <typename T, int N> using vec = T __attribute__((ext_vector_type(N)));

constexpr float F8_MAX = 448.f;             // largest finite e4m3 value
constexpr float F8_SCALE_MIN = 0x1p-126f;   // the smallest normal float: its reciprocal is finite

// Values of a load or a store: as many of N as 16 bytes hold.
template <typename T, int N> constexpr int PIECE = N * sizeof(T) <= 16 ? N : 16 / int(sizeof(T));

// N values at p, of which the first `have` exist; the others are 0.  VEC: p is aligned to N values, or to 16 bytes where they are more.
// (Value by value each load is waited for: 8192 x 4096 in bf16, norm 148 us against 40, its gradients 154, 52, quantisation 48, 21,
// combination of 4 rows 197, 78, its gradients 402, 127.)
template <int N, bool VEC, typename T> __device__ __forceinline__ void load_values(const T* p, int have, float (&out)[N]) {
    if (VEC && have >= N) {
#pragma unroll
        for (int i = 0; i < N; i += PIECE<T, N>) {
            const vec<T, PIECE<T, N>> v = *reinterpret_cast<const vec<T, PIECE<T, N>>*>(p + i);
#pragma unroll
            for (int j = 0; j < PIECE<T, N>; j++) out[i + j] = float(v[j]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i++) out[i] = i < have ? float(p[i]) : 0.f;
    }
}

// Eight of them as they are.
template <bool VEC, typename T> __device__ __forceinline__ vec<T, 8> eight_values(const T* p, int have) {
    vec<T, 8> v;
    if (VEC && have >= 8) {
#pragma unroll
        for (int i = 0; i < 8; i += PIECE<T, 8>) {
            const vec<T, PIECE<T, 8>> part = *reinterpret_cast<const vec<T, PIECE<T, 8>>*>(p + i);
#pragma unroll
            for (int j = 0; j < PIECE<T, 8>; j++) v[i + j] = part[j];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) v[i] = i < have ? p[i] : T(0.f);
    }
    return v;
}

// Rounds to the nearest T, ties to even.
template <int N, bool VEC, typename T> __device__ __forceinline__ void store_values(T* p, int have, const float (&in)[N]) {
    if (VEC && have >= N) {
#pragma unroll
        for (int i = 0; i < N; i += PIECE<T, N>) {
            vec<T, PIECE<T, N>> v;
#pragma unroll
            for (int j = 0; j < PIECE<T, N>; j++) v[j] = T(in[i + j]);
            *reinterpret_cast<vec<T, PIECE<T, N>>*>(p + i) = v;
        }
    } else {
#pragma unroll
        for (int i = 0; i < N; i++)
            if (i < have) p[i] = T(in[i]);
    }
}

// Four e4m3 values, rounded to the nearest, ties to even.  A value that its scale's rounding left a little
// above the largest becomes the largest.
__device__ __forceinline__ uint32_t f8_pack(float a, float b, float c, float d) {
    a = fminf(fmaxf(a, -F8_MAX), F8_MAX), b = fminf(fmaxf(b, -F8_MAX), F8_MAX);
    c = fminf(fmaxf(c, -F8_MAX), F8_MAX), d = fminf(fmaxf(d, -F8_MAX), F8_MAX);
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true));
}

// The scale of a block, from the bits of its largest magnitude.  Magnitudes are compared as whole numbers: that order is
// the floats' own, with infinity and then NaN above them, so that neither gets lost.
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
struct Scale {
    float scale;            // largest / 448
    float divisor, inverse; // x / scale = 0.875 x / divisor
};
__device__ __forceinline__ Scale f8_scale(uint32_t largest) {
    const float least = F8_SCALE_MIN * F8_MAX, most = __uint_as_float(largest), l = most < least ? least : most;
    const float d = l * 0x1p-9f;
    return {l / F8_MAX, d, 1.f / d};
}
// x / scale, correctly rounded as a quotient of x and the magnitude: 16-bit inputs often lie halfway between two e4m3
// values, and come out as that and are then rounded to even.  (0.875 x is exact in 16 bits and cannot overflow.)
__device__ __forceinline__ float f8_quotient(float x, const Scale& s) {
    const float v = x * 0.875f, q = v * s.inverse;
    return fmaf(fmaf(-q, s.divisor, v), s.inverse, q);
}

// 8 values in units of their scale, rounded to e4m3
template <bool VEC> __device__ __forceinline__ void f8_store(uint8_t* q, int have, const float (&v)[8], const Scale& s) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; i++) w[i] = f8_pack(f8_quotient(v[4 * i], s), f8_quotient(v[4 * i + 1], s), f8_quotient(v[4 * i + 2], s), f8_quotient(v[4 * i + 3], s));
    if (VEC && have >= 8) {
        *reinterpret_cast<uint2*>(q) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++)
            if (i < have) q[i] = uint8_t(w[i / 4] >> (8 * (i % 4)));
    }
}

// over aligned groups of LANES lanes, everybody gets the result
template <int LANES> __device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v += __shfl_xor(v, d);
    return v;
}
template <int LANES> __device__ __forceinline__ uint32_t lanes_max(uint32_t v) {
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) v = max(v, uint32_t(__shfl_xor(int(v), d)));
    return v;
}

// Over the whole wavefront, by data-parallel moves: row shifts by 1, 2, 4 and 8, then the last lane of a row of 16 to the
// next row and of the first half to the second; lane 63 has it all.  (A shuffle through LDS takes some 100 cycles a step.)
template <int CTRL, int ROWS> __device__ __forceinline__ uint32_t moved(uint32_t v, uint32_t identity) {
    return uint32_t(__builtin_amdgcn_update_dpp(int(identity), int(v), CTRL, ROWS, 0xf, false));
}
// With sums, a lane has those up to itself.
template <typename F> __device__ __forceinline__ uint32_t wave_upto(uint32_t v, uint32_t identity, F f) {
    v = f(v, moved<0x111, 0xf>(v, identity));
    v = f(v, moved<0x112, 0xf>(v, identity));
    v = f(v, moved<0x114, 0xf>(v, identity));
    v = f(v, moved<0x118, 0xf>(v, identity));
    v = f(v, moved<0x142, 0xa>(v, identity));
    return f(v, moved<0x143, 0xc>(v, identity));
}
template <typename F> __device__ __forceinline__ uint32_t wave_all(uint32_t v, uint32_t identity, F f) {
    return uint32_t(__builtin_amdgcn_readlane(int(wave_upto(v, identity, f)), 63));
}
__device__ __forceinline__ int32_t wave_prefix(int32_t v) {
    return int32_t(wave_upto(uint32_t(v), 0u, [](uint32_t a, uint32_t b) { return a + b; }));
}
// Over each row of 16 lanes, by rotations: every lane has the result.
template <typename F> __device__ __forceinline__ uint32_t row_all(uint32_t v, F f) {
    v = f(v, moved<0x128, 0xf>(v, v));
    v = f(v, moved<0x124, 0xf>(v, v));
    v = f(v, moved<0x122, 0xf>(v, v));
    return f(v, moved<0x121, 0xf>(v, v));
}
__device__ __forceinline__ uint32_t row_max(uint32_t v) {
    return row_all(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float row_sum(float v) {
    return __uint_as_float(row_all(__float_as_uint(v), [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
    return wave_all(v, 0u, [](uint32_t a, uint32_t b) { return max(a, b); });
}
__device__ __forceinline__ float wave_sum(float v) {
    return __uint_as_float(wave_all(__float_as_uint(v), 0u, [](uint32_t a, uint32_t b) { return __float_as_uint(__uint_as_float(a) + __uint_as_float(b)); }));
}

// What the lanes of this wavefront wrote to LDS before is what they read after it (their LDS accesses are in order).
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

inline bool aligned(const void* p, int64_t ld, size_t element, size_t bytes) {
    return (reinterpret_cast<uintptr_t>(p) % bytes) == 0 && (size_t(ld) * element) % bytes == 0;
}
// an array of `rows` rows may be given: its address, and a stride that its columns fit
inline bool rows_ok(const void* p, int64_t rows, int64_t ld, int64_t columns, size_t element) {
    if (rows == 0 || columns == 0) return true;
    return p && ld >= columns && (reinterpret_cast<uintptr_t>(p) % element) == 0;
}
inline int divide_up(int64_t a, int64_t b) { return int((a + b - 1) / b); }

// The largest size that every loop may count past.
constexpr int32_t MOST_SIZE = INT32_MAX - 65536;

// n workgroups in two dimensions, as one holds 2^32 threads at most; the last ones may have nothing to do.
inline dim3 workgroups(int64_t n) {
    constexpr int64_t ROW = 1 << 20;
    return dim3(uint32_t(n < ROW ? n : ROW), uint32_t((n + ROW - 1) / ROW));
}
__device__ __forceinline__ int64_t workgroup() { return int64_t(blockIdx.y) * gridDim.x + blockIdx.x; }

inline int launched() { return hipGetLastError() == hipSuccess ? CSR5_OK : CSR5_EHIP; }

}  // namespace

#endif
