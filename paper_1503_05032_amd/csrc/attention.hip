// libcsr5: attention over packed sequences and over a paged cache of keys and values, and its gradients.  The C ABI is declared in
// include/csr5.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>
#include <type_traits>

#include "csr5.h"
#include "heads.h"
#include "numbers.h"

namespace {

// ---------------------------------------------------------------------------------------------------------------
// Sequences
// ---------------------------------------------------------------------------------------------------------------
struct Span {
    int32_t first, count;
};
// Rows of sequence s.  Whatever the offsets hold, these are rows that there are.
__device__ __forceinline__ Span span_of(const int32_t* offset, int32_t s, int32_t rows) {
    const int32_t a = min(max(offset[s], 0), rows), b = min(max(offset[s + 1], 0), rows);
    return {a, max(b - a, 0)};
}
// The sequence that row i lies in, by bisection; -1: none.
__device__ __forceinline__ int32_t sequence_of(const int32_t* offset, int32_t sequences, int32_t rows, int32_t i) {
    int32_t low = 0, high = sequences;
    while (high - low > 1) {
        const int32_t mid = low + (high - low) / 2;
        if (offset[mid] <= i) low = mid;
        else high = mid;
    }
    const Span s = span_of(offset, low, rows);
    return i >= s.first && i < s.first + s.count ? low : -1;
}

// Keys and values, packed or in a cache.
template <typename T> struct Packed {
    const int32_t* offset;
    int32_t rows;
    Heads<const T> k, v;
    __device__ __forceinline__ Span span(int32_t s) const { return span_of(offset, s, rows); }
    __device__ __forceinline__ const T* key(int32_t s, const Span& at, int32_t j, int h) const { return k.p + int64_t(at.first + j) * k.row + h * k.head; }
    __device__ __forceinline__ const T* value(int32_t s, const Span& at, int32_t j, int h) const { return v.p + int64_t(at.first + j) * v.row + h * v.head; }
};
template <typename T> struct Paged {
    const int32_t *length, *table;
    int32_t width, pages, shift;
    int64_t ldt;
    Cache<const T> k, v;
    __device__ __forceinline__ Span span(int32_t s) const { return {0, int32_t(min(int64_t(max(length[s], 0)), int64_t(width) << shift))}; }
    __device__ __forceinline__ const T* row(const Cache<const T>& c, int32_t s, int32_t j, int h) const {
        const int32_t page = table[s * ldt + (j >> shift)];
        return uint32_t(page) < uint32_t(pages) ? c.p + page * c.page + (j & ((1 << shift) - 1)) * c.row + h * c.head : nullptr;
    }
    __device__ __forceinline__ const T* key(int32_t s, const Span&, int32_t j, int h) const { return row(k, s, j, h); }
    __device__ __forceinline__ const T* value(int32_t s, const Span&, int32_t j, int h) const { return row(v, s, j, h); }
};

template <typename T, typename KV> struct Attend {
    int32_t sequences, rows, heads, shared, d;
    const int32_t* q_offset;
    float scale;
    bool causal;
    Heads<const T> q;
    KV kv;
    Heads<T> out;
    float* lse;
};

// Keys that query i of m sees, of n.
__device__ __forceinline__ int32_t seen(bool causal, int32_t i, int32_t m, int32_t n) { return causal ? min(max(n - m + i + 1, 0), n) : n; }

template <typename T> __device__ __forceinline__ float dot(const T* a, const T* b, int d) {
    float sum = 0.f;
    if (b)
        for (int c = 0; c < d; c++) sum = fmaf(float(a[c]), float(b[c]), sum);
    return sum;
}
__device__ __forceinline__ float wave_most(float v) {
#pragma unroll
    for (int e = 1; e < 64; e *= 2) v = fmaxf(v, __shfl_xor(v, e));
    return v;
}

// One wavefront per row and head: 64 scores at a time, a running maximum and sum.
template <typename T, typename KV> __global__ __launch_bounds__(64) void k_attend(Attend<T, KV> a) {
    const int64_t at = workgroup();
    if (at >= int64_t(a.rows) * a.heads) return;
    const int32_t row = int32_t(at / a.heads), h = int32_t(at % a.heads), hk = h / a.shared, lane = threadIdx.x;
    const int32_t s = sequence_of(a.q_offset, a.sequences, a.rows, row);
    if (s < 0) return;
    const Span mine = span_of(a.q_offset, s, a.rows), keys = a.kv.span(s);
    const int32_t n = seen(a.causal, row - mine.first, mine.count, keys.count);
    const T* const q = a.q.p + row * a.q.row + h * a.q.head;
    float top = -INFINITY, sum = 0.f, acc[2] = {0.f, 0.f};
    for (int32_t j0 = 0; j0 < n; j0 += 64) {
        const int32_t j = j0 + lane;
        const float x = j < n ? a.scale * dot(q, a.kv.key(s, keys, j, hk), a.d) : -INFINITY;
        const float higher = fmaxf(top, wave_most(x)), base = higher == -INFINITY ? 0.f : higher;
        const float p = expf(x - base), less = expf(top - base);
        top = higher, sum = sum * less + wave_sum(p);
        acc[0] *= less, acc[1] *= less;
        for (int e = 0; e < min(64, n - j0); e++) {
            const float w = __shfl(p, e);
            const T* const v = a.kv.value(s, keys, j0 + e, hk);
            for (int i = 0; i < 2; i++)
                if (v && i * 64 + lane < a.d) acc[i] = fmaf(w, float(v[i * 64 + lane]), acc[i]);
        }
    }
    for (int i = 0; i < 2; i++)
        if (i * 64 + lane < a.d) a.out.p[row * a.out.row + h * a.out.head + i * 64 + lane] = T(n > 0 ? acc[i] / sum : 0.f);
    if (a.lse && lane == 0) a.lse[int64_t(h) * a.rows + row] = n > 0 ? top + logf(sum) : -INFINITY;
}

template <typename T> struct Back {
    int32_t sequences, rows, heads, shared, d;
    const int32_t* q_offset;
    float scale;
    bool causal;
    Heads<const T> dout, q, out;
    Packed<T> kv;
    const float* lse;
    float* delta;               // [heads][rows]
    Heads<T> dq, dk, dv;
};

template <typename T> __global__ __launch_bounds__(64) void k_delta(Back<T> a) {
    const int64_t at = workgroup() * 64 + threadIdx.x;
    if (at >= int64_t(a.rows) * a.heads) return;
    const int32_t row = int32_t(at % a.rows), h = int32_t(at / a.rows);
    a.delta[at] = dot(a.dout.p + row * a.dout.row + h * a.dout.head, a.out.p + row * a.out.row + h * a.out.head, a.d);
}

// One wavefront per row and head.
template <typename T> __global__ __launch_bounds__(64) void k_attend_dq(Back<T> a) {
    const int64_t at = workgroup();
    if (at >= int64_t(a.rows) * a.heads) return;
    const int32_t row = int32_t(at / a.heads), h = int32_t(at % a.heads), hk = h / a.shared, lane = threadIdx.x;
    const int32_t s = sequence_of(a.q_offset, a.sequences, a.rows, row);
    if (s < 0) return;
    const Span mine = span_of(a.q_offset, s, a.rows), keys = a.kv.span(s);
    const int32_t n = seen(a.causal, row - mine.first, mine.count, keys.count);
    const float lse = a.lse[int64_t(h) * a.rows + row], delta = a.delta[int64_t(h) * a.rows + row];
    float acc[2] = {0.f, 0.f};
    for (int32_t j0 = 0; j0 < n; j0 += 64) {
        const int32_t j = j0 + lane;
        float ds = 0.f;
        if (j < n) {
            const float p = expf(a.scale * dot(a.q.p + row * a.q.row + h * a.q.head, a.kv.key(s, keys, j, hk), a.d) - lse);
            ds = p * (dot(a.dout.p + row * a.dout.row + h * a.dout.head, a.kv.value(s, keys, j, hk), a.d) - delta);
        }
        for (int e = 0; e < min(64, n - j0); e++) {
            const float w = __shfl(ds, e);
            const T* const k = a.kv.key(s, keys, j0 + e, hk);
            for (int i = 0; i < 2; i++)
                if (i * 64 + lane < a.d) acc[i] = fmaf(w, float(k[i * 64 + lane]), acc[i]);
        }
    }
    for (int i = 0; i < 2; i++)
        if (i * 64 + lane < a.d) a.dq.p[row * a.dq.row + h * a.dq.head + i * 64 + lane] = T(a.scale * acc[i]);
}

// One wavefront per key and head of keys; the query heads that share it one after the other.
template <typename T> __global__ __launch_bounds__(64) void k_attend_dkv(Back<T> a) {
    const int64_t at = workgroup();
    const int32_t kv_heads = a.heads / a.shared;
    if (at >= int64_t(a.kv.rows) * kv_heads) return;
    const int32_t row = int32_t(at / kv_heads), hk = int32_t(at % kv_heads), lane = threadIdx.x;
    const int32_t s = sequence_of(a.kv.offset, a.sequences, a.kv.rows, row);
    if (s < 0) return;
    const Span mine = span_of(a.q_offset, s, a.rows), keys = a.kv.span(s);
    const int32_t j = row - keys.first, from = a.causal ? max(0, j - (keys.count - mine.count)) : 0;     // the first query that sees it
    float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    for (int g = 0; g < a.shared; g++) {
        const int h = hk * a.shared + g;
        for (int32_t i0 = from; i0 < mine.count; i0 += 64) {
            const int32_t i = i0 + lane, r = mine.first + i;
            float p = 0.f, ds = 0.f;
            if (i < mine.count) {
                p = expf(a.scale * dot(a.q.p + r * a.q.row + h * a.q.head, a.kv.key(s, keys, j, hk), a.d) - a.lse[int64_t(h) * a.rows + r]);
                ds = p * (dot(a.dout.p + r * a.dout.row + h * a.dout.head, a.kv.value(s, keys, j, hk), a.d) - a.delta[int64_t(h) * a.rows + r]);
            }
            for (int e = 0; e < min(64, mine.count - i0); e++) {
                const float w = __shfl(p, e), u = __shfl(ds, e);
                const int64_t q = mine.first + i0 + e;
                for (int c = lane; c < a.d; c += 64) {
                    dv[c / 64] = fmaf(w, float(a.dout.p[q * a.dout.row + h * a.dout.head + c]), dv[c / 64]);
                    dk[c / 64] = fmaf(u, float(a.q.p[q * a.q.row + h * a.q.head + c]), dk[c / 64]);
                }
            }
        }
    }
    for (int c = lane; c < a.d; c += 64) {
        a.dk.p[row * a.dk.row + hk * a.dk.head + c] = T(a.scale * dk[c / 64]);
        a.dv.p[row * a.dv.row + hk * a.dv.head + c] = T(dv[c / 64]);
    }
}

template <typename F> int with_half(int dtype, F f) { return dtype == CSR5_DTYPE_F16 ? f(f16()) : f(bf16()); }

// What all calls ask of their sizes
int sizes(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, float scale) {
    if ((dtype != CSR5_DTYPE_BF16 && dtype != CSR5_DTYPE_F16) || sequences < 0 || rows < 0 || k_rows < 0 || heads < 0 || kv_heads < 0 || d < 0) return CSR5_EINVAL;
    if (kv_heads == 0 ? heads != 0 : heads % kv_heads != 0) return CSR5_EINVAL;
    if (!(scale > 0.f) || !std::isfinite(scale)) return CSR5_EINVAL;
    if (sequences > MOST_SIZE || rows > MOST_SIZE || k_rows > MOST_SIZE || heads > CSR5_ATTENTION_MAX_HEADS || d > CSR5_ATTENTION_MAX_D) return CSR5_ERANGE;
    return CSR5_OK;
}
bool words(std::initializer_list<const void*> all) {
    for (const void* p : all)
        if (reinterpret_cast<uintptr_t>(p) & 3) return false;
    return true;
}

}  // namespace

extern "C" {

int csr5_attention(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset,
                   const int32_t* k_offset, float scale, int causal, csr5_heads_t q, csr5_heads_t k, csr5_heads_t v, csr5_heads_t out, float* lse, void* hip_stream) {
    if (const int bad = sizes(sequences, rows, k_rows, heads, kv_heads, d, dtype, scale)) return bad;
    if (!heads_ok(q, rows, heads, d, 2) || !heads_ok(k, k_rows, kv_heads, d, 2) || !heads_ok(v, k_rows, kv_heads, d, 2) || !output_ok(out, rows, heads, d, 2)) return CSR5_EINVAL;
    if (!words({q_offset, k_offset, lse})) return CSR5_EINVAL;
    if (sequences == 0 || rows == 0 || heads == 0) return CSR5_OK;
    if (!q_offset || !k_offset) return CSR5_EINVAL;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        const Attend<T, Packed<T>> a{sequences, rows, heads, heads / kv_heads, d, q_offset, scale, causal != 0, typed<const T>(q), {k_offset, k_rows, typed<const T>(k), typed<const T>(v)}, typed<T>(out), lse};
        k_attend<T><<<workgroups(int64_t(rows) * heads), 64, 0, s>>>(a);
        return launched();
    });
}

size_t csr5_attention_backward_workspace_bytes(int32_t rows, int32_t heads) { return rows <= 0 || heads <= 0 ? 0 : size_t(rows) * size_t(heads) * 4; }

int csr5_attention_backward(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset,
                            const int32_t* k_offset, float scale, int causal, csr5_heads_t dout, csr5_heads_t q, csr5_heads_t k, csr5_heads_t v, csr5_heads_t out,
                            const float* lse, csr5_heads_t dq, csr5_heads_t dk, csr5_heads_t dv, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = sizes(sequences, rows, k_rows, heads, kv_heads, d, dtype, scale)) return bad;
    if (!heads_ok(q, rows, heads, d, 2) || !heads_ok(k, k_rows, kv_heads, d, 2) || !heads_ok(v, k_rows, kv_heads, d, 2) || !heads_ok(out, rows, heads, d, 2) ||
        !heads_ok(dout, rows, heads, d, 2) || !output_ok(dq, rows, heads, d, 2) || !output_ok(dk, k_rows, kv_heads, d, 2) || !output_ok(dv, k_rows, kv_heads, d, 2))
        return CSR5_EINVAL;
    if (!words({q_offset, k_offset, lse, workspace})) return CSR5_EINVAL;
    if (sequences == 0 || heads == 0 || d == 0) return CSR5_OK;
    if (!q_offset || !k_offset || (rows > 0 && !lse)) return CSR5_EINVAL;
    if (rows > 0 && (!workspace || workspace_bytes < csr5_attention_backward_workspace_bytes(rows, heads))) return CSR5_ENOMEM;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        const Back<T> a{sequences, rows, heads, heads / kv_heads, d, q_offset, scale, causal != 0, typed<const T>(dout), typed<const T>(q), typed<const T>(out),
                        {k_offset, k_rows, typed<const T>(k), typed<const T>(v)}, lse, static_cast<float*>(workspace), typed<T>(dq), typed<T>(dk), typed<T>(dv)};
        if (rows > 0) {
            k_delta<T><<<workgroups((int64_t(rows) * heads + 63) / 64), 64, 0, s>>>(a);
            k_attend_dq<T><<<workgroups(int64_t(rows) * heads), 64, 0, s>>>(a);
        }
        if (k_rows > 0) k_attend_dkv<T><<<workgroups(int64_t(k_rows) * kv_heads), 64, 0, s>>>(a);
        return launched();
    });
}

size_t csr5_attention_paged_workspace_bytes(int32_t rows, int32_t heads, int32_t kv_heads, int32_t d, int32_t sequences, int64_t max_length) { return 0; }

int csr5_attention_paged(int32_t sequences, int32_t rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset, const int32_t* length,
                         const int32_t* table, int32_t width, int64_t ldt, int32_t pages, int32_t page, float scale, csr5_heads_t q, csr5_cache_t k_cache, csr5_cache_t v_cache,
                         csr5_heads_t out, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = sizes(sequences, rows, 0, heads, kv_heads, d, dtype, scale)) return bad;
    if (width < 0 || pages < 0 || !power_of_two(page)) return CSR5_EINVAL;
    if (int64_t(width) * page > MOST_SIZE) return CSR5_ERANGE;
    if (!heads_ok(q, rows, heads, d, 2) || !output_ok(out, rows, heads, d, 2) || !cache_ok(k_cache, pages, page, kv_heads, d, 2) || !cache_ok(v_cache, pages, page, kv_heads, d, 2) ||
        !rows_ok(table, sequences, ldt, width, 4))
        return CSR5_EINVAL;
    if (!words({q_offset, length, lse, workspace})) return CSR5_EINVAL;
    if (sequences == 0 || rows == 0 || heads == 0) return CSR5_OK;
    if (!q_offset || !length) return CSR5_EINVAL;
    const size_t need = csr5_attention_paged_workspace_bytes(rows, heads, kv_heads, d, sequences, int64_t(width) * page);
    if (need && (!workspace || workspace_bytes < need)) return CSR5_ENOMEM;
    hipStream_t s = static_cast<hipStream_t>(hip_stream);
    return with_half(dtype, [&](auto zero) {
        using T = decltype(zero);
        const Attend<T, Paged<T>> a{sequences, rows, heads, heads / kv_heads, d, q_offset, scale, true, typed<const T>(q), {length, table, width, pages, __builtin_ctz(page), ldt, typed<const T>(k_cache), typed<const T>(v_cache)}, typed<T>(out), lse};
        k_attend<T><<<workgroups(int64_t(rows) * heads), 64, 0, s>>>(a);
        return launched();
    });
}

}  // extern "C"
