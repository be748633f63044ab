// Rows of heads, caches of pages and packed sequences, for the attention and what stands around it.
#ifndef CSR5_HEADS_H
#define CSR5_HEADS_H

#include <hip/hip_runtime.h>

#include <cstdint>

#include "csr5.h"
#include "numbers.h"

namespace {

template <typename T> struct Heads {
    T* p;
    int64_t row, head;
};
template <typename T> struct Cache {
    T* p;
    int64_t page, row, head;
};
template <typename T> Heads<T> typed(const csr5_heads_t& h) { return {static_cast<T*>(h.p), h.row, h.head}; }
template <typename T> Cache<T> typed(const csr5_cache_t& c) { return {static_cast<T*>(c.p), c.page, c.row, c.head}; }

inline bool power_of_two(int32_t n) { return n > 0 && (n & (n - 1)) == 0; }

// given, at an address of its type, with strides that are not negative
inline bool heads_ok(const csr5_heads_t& h, int64_t rows, int64_t heads, int64_t d, size_t element) {
    if (rows == 0 || heads == 0 || d == 0) return true;
    return h.p && (reinterpret_cast<uintptr_t>(h.p) % element) == 0 && h.row >= 0 && h.head >= 0;
}
// Values of `levels` dimensions with these counts and strides around d neighbouring ones: no two at one address.  By strides in
// ascending order, each is at least the extent of those below.
inline bool apart(int64_t d, int levels, int64_t* count, int64_t* stride) {
    for (int i = 0; i < levels; i++)
        for (int j = i + 1; j < levels; j++)
            if (stride[j] < stride[i]) {
                const int64_t c = count[i], s = stride[i];
                count[i] = count[j], stride[i] = stride[j], count[j] = c, stride[j] = s;
            }
    int64_t extent = d;
    for (int i = 0; i < levels; i++) {
        if (count[i] <= 1) continue;
        if (stride[i] < extent) return false;
        extent += (count[i] - 1) * stride[i];
    }
    return true;
}
inline bool output_ok(const csr5_heads_t& h, int64_t rows, int64_t heads, int64_t d, size_t element) {
    if (rows == 0 || heads == 0 || d == 0) return true;
    int64_t count[2] = {rows, heads}, stride[2] = {h.row, h.head};
    return heads_ok(h, rows, heads, d, element) && apart(d, 2, count, stride);
}
inline bool cache_ok(const csr5_cache_t& c, int64_t pages, int64_t page, int64_t heads, int64_t d, size_t element) {
    if (pages == 0 || heads == 0 || d == 0) return true;
    return c.p && (reinterpret_cast<uintptr_t>(c.p) % element) == 0 && c.page >= 0 && c.row >= 0 && c.head >= 0;
}
inline bool cache_output_ok(const csr5_cache_t& c, int64_t pages, int64_t page, int64_t heads, int64_t d, size_t element) {
    if (pages == 0 || heads == 0 || d == 0) return true;
    int64_t count[3] = {pages, page, heads}, stride[3] = {c.page, c.row, c.head};
    return cache_ok(c, pages, page, heads, d, element) && apart(d, 3, count, stride);
}
// rows of whole 16 bytes at 16-byte addresses
inline bool wide(const csr5_heads_t& h, size_t element) {
    return (reinterpret_cast<uintptr_t>(h.p) % 16) == 0 && (size_t(h.row) * element) % 16 == 0 && (size_t(h.head) * element) % 16 == 0;
}
inline bool wide(const csr5_cache_t& c, size_t element) {
    return (reinterpret_cast<uintptr_t>(c.p) % 16) == 0 && (size_t(c.page) * element) % 16 == 0 && (size_t(c.row) * element) % 16 == 0 && (size_t(c.head) * element) % 16 == 0;
}

}  // namespace

#endif
