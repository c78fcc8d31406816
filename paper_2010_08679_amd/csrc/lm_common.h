// Shared by the operators for language models (lm_*.hip, compiled so that infinities and NaN are ordinary values).
#pragma once

#include "cnr_common.h"
#include "cnr_lm.h"

static inline bool cnr_valid_float_type(int t) { return t == CNR_FLOAT_F32 || t == CNR_FLOAT_BF16 || t == CNR_FLOAT_F16; }
static inline size_t cnr_float_bytes(cnr_float_type t) { return t == CNR_FLOAT_F32 ? 4 : 2; }
static inline bool cnr_aligned(const void *p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }
static inline uint64_t cnr_ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

#ifdef __HIPCC__
// Elements of the three types: to fp32 exactly, from fp32 with one rounding to nearest even.
template <int TYPE>
struct Element;
template <>
struct Element<CNR_FLOAT_F32> {
    typedef float type;
    static __device__ __forceinline__ float wide(float v) { return v; }
    static __device__ __forceinline__ float narrow(float v) { return v; }
};
template <>
struct Element<CNR_FLOAT_BF16> {
    typedef __bf16 type;
    static __device__ __forceinline__ float wide(__bf16 v) { return (float)v; }
    static __device__ __forceinline__ __bf16 narrow(float v) { return (__bf16)v; }
};
template <>
struct Element<CNR_FLOAT_F16> {
    typedef _Float16 type;
    static __device__ __forceinline__ float wide(_Float16 v) { return (float)v; }
    static __device__ __forceinline__ _Float16 narrow(float v) { return (_Float16)v; }
};

// N elements side by side that need no more alignment than one of them: rows of an odd length start anywhere, and
// the memory system takes a wide access at any element's address.
template <typename T, int N>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[N];
};

// 16 bytes of elements that need no more alignment than one of them, in one access, as words.
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));
template <typename T>
__device__ __forceinline__ u32x4 load16(const T *p) {
    return *reinterpret_cast<const u32x4_anywhere *>(p);
}
template <typename T>
__device__ __forceinline__ void store16(T *p, const u32x4 &w) {
    *reinterpret_cast<u32x4_anywhere *>(p) = w;
}
#endif
