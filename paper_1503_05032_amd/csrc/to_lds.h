// Loads from memory straight into LDS, and the wait for them.
#ifndef CSR5_TO_LDS_H
#define CSR5_TO_LDS_H

#include <hip/hip_runtime.h>

#include <cstdint>

namespace {

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
// To an LDS address that is the same in every lane.
__device__ __forceinline__ void to_lds_at(const void* from, uint32_t lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(uint32_t(__builtin_amdgcn_readfirstlane(lds))), "v"(from) : "memory", "m0");
}
__device__ __forceinline__ void to_lds_at(const void* base, uint32_t offset, uint32_t lds) {
    const void* at;
    asm volatile("s_mov_b32 m0, %1\n\ts_mov_b64 %0, %3\n\tglobal_load_lds_dwordx4 %2, %0" : "=&s"(at) : "s"(uint32_t(__builtin_amdgcn_readfirstlane(lds))), "v"(offset), "s"(same(base)) : "memory", "m0");
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
// The same without the others: for LDS that one wavefront has to itself.
template <int LATER> __device__ __forceinline__ void own_landed() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(LATER) : "memory");
}

// This wavefront's reads of LDS have returned: it may be loaded anew.
__device__ __forceinline__ void own_read() {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
}

}  // namespace

#endif
