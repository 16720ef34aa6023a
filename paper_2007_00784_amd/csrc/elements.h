// Elements in memory as vectors, and rows of lanes: what the kernels that stream over tensors share.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace kfac {

// N consecutive elements from anywhere: tensors may start at any element, and the loads are as wide as N allows all the same (global memory
// takes unaligned vectors).
template <typename T, int N> struct Vec { T x[N]; };
template <typename T, int N> __device__ inline Vec<T, N> load(const void *p, int64_t i) {
    Vec<T, N> r;
    __builtin_memcpy(&r, (const char *)p + i * (int64_t)sizeof(T), sizeof(r));
    return r;
}
template <typename T, int N> __device__ inline void store(void *p, int64_t i, const Vec<T, N> &r) {
    __builtin_memcpy((char *)p + i * (int64_t)sizeof(T), &r, sizeof(r));
}
// The same past the caches, for what is too long to stay there or is not read again by this launch.
typedef unsigned AnyVector __attribute__((ext_vector_type(4), aligned(1)));
template <typename T, int N> __device__ inline Vec<T, N> load_past(const void *p, int64_t i) {
    static_assert(sizeof(Vec<T, N>) == 16, "one vector");
    return __builtin_bit_cast(Vec<T, N>, (AnyVector)__builtin_nontemporal_load((const AnyVector *)((const char *)p + i * (int64_t)sizeof(T))));
}
template <typename T, int N> __device__ inline void store_past(void *p, int64_t i, const Vec<T, N> &r) {
    static_assert(sizeof(Vec<T, N>) == 16, "one vector");
    __builtin_nontemporal_store(__builtin_bit_cast(AnyVector, r), (AnyVector *)((char *)p + i * (int64_t)sizeof(T)));
}
__device__ inline float widen(unsigned short b) { return __uint_as_float((unsigned)b << 16); }
__device__ inline unsigned short round_bf16(float x) {   // half to even; NaN stays NaN
    const unsigned u = __float_as_uint(x);
    if ((u & 0x7fffffffu) > 0x7f800000u) return (unsigned short)((u >> 16) | 0x40u);
    return (unsigned short)((u + 0x7fffu + ((u >> 16) & 1u)) >> 16);
}

// An element as fp32, and fp32 as an element (bf16: half to even, by the conversion instruction).
__device__ inline float value_of(float x) { return x; }
__device__ inline float value_of(unsigned short x) { return widen(x); }
template <typename T> __device__ inline T element_of(float x);
template <> __device__ inline float element_of<float>(float x) { return x; }
template <> __device__ inline unsigned short element_of<unsigned short>(float x) {
    const __bf16 b = (__bf16)x;
    return __builtin_bit_cast(unsigned short, b);
}

// The largest of the sixteen lanes of a row, in all of them.
__device__ inline float row_max(float x) {
#define KFAC_ROW_STEP(ctrl) x = fmaxf(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), ctrl, 0xf, 0xf, true)))
    KFAC_ROW_STEP(0xB1);     // lanes 1 0 3 2
    KFAC_ROW_STEP(0x4E);     // lanes 2 3 0 1
    KFAC_ROW_STEP(0x141);    // the other four of each eight
    KFAC_ROW_STEP(0x140);    // the other eight of the sixteen
#undef KFAC_ROW_STEP
    return x;
}

}  // namespace kfac
