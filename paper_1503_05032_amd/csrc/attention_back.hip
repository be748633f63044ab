// libcsr5: the gradients of attention over packed sequences.  The C ABI is declared in include/csr5.h.
#include <hip/hip_runtime.h>

#include <cmath>
#include <cstdint>

#include "csr5.h"
#include "heads.h"
#include "numbers.h"
#include "sequences.h"

namespace {

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

template <typename T> __device__ __forceinline__ float dot(const T* a, const T* b, int d) {
    float sum = 0.f;
    if (b)
        for (int c = 0; c < d; c++) sum = fmaf(float(a[c]), float(b[c]), sum);
    return sum;
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
    const Span mine = span_of(a.q_offset, s, a.rows), keys = span_of(a.kv.offset, s, a.kv.rows);
    const int32_t n = seen(a.causal, row - mine.first, mine.count, keys.count);
    const float lse = a.lse[int64_t(h) * a.rows + row], delta = a.delta[int64_t(h) * a.rows + row];
    float acc[2] = {0.f, 0.f};
    for (int32_t j0 = 0; j0 < n; j0 += 64) {
        const int32_t j = j0 + lane;
        float ds = 0.f;
        if (j < n) {
            const float p = expf(a.scale * dot(a.q.p + row * a.q.row + h * a.q.head, (a.kv.k.p + (keys.first + j) * a.kv.k.row + hk * a.kv.k.head), a.d) - lse);
            ds = p * (dot(a.dout.p + row * a.dout.row + h * a.dout.head, (a.kv.v.p + (keys.first + j) * a.kv.v.row + hk * a.kv.v.head), a.d) - delta);
        }
        for (int e = 0; e < min(64, n - j0); e++) {
            const float w = __shfl(ds, e);
            const T* const k = a.kv.k.p + (keys.first + j0 + e) * a.kv.k.row + hk * a.kv.k.head;
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
    const Span mine = span_of(a.q_offset, s, a.rows), keys = span_of(a.kv.offset, s, a.kv.rows);
    const int32_t j = row - keys.first, from = a.causal ? max(0, j - (keys.count - mine.count)) : 0;     // the first query that sees it
    float dk[2] = {0.f, 0.f}, dv[2] = {0.f, 0.f};
    for (int g = 0; g < a.shared; g++) {
        const int h = hk * a.shared + g;
        for (int32_t i0 = from; i0 < mine.count; i0 += 64) {
            const int32_t i = i0 + lane, r = mine.first + i;
            float p = 0.f, ds = 0.f;
            if (i < mine.count) {
                p = expf(a.scale * dot(a.q.p + r * a.q.row + h * a.q.head, (a.kv.k.p + (keys.first + j) * a.kv.k.row + hk * a.kv.k.head), a.d) - a.lse[int64_t(h) * a.rows + r]);
                ds = p * (dot(a.dout.p + r * a.dout.row + h * a.dout.head, (a.kv.v.p + (keys.first + j) * a.kv.v.row + hk * a.kv.v.head), a.d) - a.delta[int64_t(h) * a.rows + r]);
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

}  // namespace

extern "C" {

size_t csr5_attention_backward_workspace_bytes(int32_t rows, int32_t heads) { return rows <= 0 || heads <= 0 ? 0 : size_t(rows) * size_t(heads) * 4; }

int csr5_attention_backward(int32_t sequences, int32_t rows, int32_t k_rows, int32_t heads, int32_t kv_heads, int32_t d, int dtype, const int32_t* q_offset,
                            const int32_t* k_offset, float scale, int causal, csr5_heads_t dout, csr5_heads_t q, csr5_heads_t k, csr5_heads_t v, csr5_heads_t out,
                            const float* lse, csr5_heads_t dq, csr5_heads_t dk, csr5_heads_t dv, void* workspace, size_t workspace_bytes, void* hip_stream) {
    if (const int bad = attention_sizes(sequences, rows, k_rows, heads, kv_heads, d, dtype, scale)) return bad;
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

}  // extern "C"
