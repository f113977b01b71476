// What the operators of an autoregressive model (linear, attention over a paged cache, selection over a vocabulary) share: element
// types, 16-byte pieces and the matrix instruction over them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tbs.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 op_bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 op_f16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;

// A fragment is 16 bytes a lane: a piece of one row, row (lane & 15) of sixteen, piece (lane >> 4) of four.
template <class T>
struct OpPiece {
    static constexpr int E = 16 / sizeof(T);   // elements of a piece
};

__device__ __forceinline__ float op_float(float x) { return x; }
__device__ __forceinline__ float op_float(__bf16 x) { return (float)x; }
__device__ __forceinline__ float op_float(_Float16 x) { return (float)x; }

// 16 bytes from any address that is a multiple of the element's size (the hardware takes unaligned vector loads)
template <class T>
__device__ __forceinline__ uint4 op_load16(const T *p) {
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}

// ... of which only the first n elements are there (n <= 0: none); the others are zero
template <class T>
__device__ __forceinline__ uint4 op_load16_part(const T *p, int n) {
    T e[OpPiece<T>::E];
#pragma unroll
    for (int i = 0; i < OpPiece<T>::E; ++i) e[i] = i < n ? p[i] : (T)0.f;
    uint4 v;
    __builtin_memcpy(&v, e, 16);
    return v;
}

// c += a b over the four pieces: c's rows are a's, its columns b's; a lane holds rows 4 (lane >> 4) .. + 3 of column lane & 15.
// (float32: four steps, the i-th over the i-th elements of the pieces; the order of the sum is the same for both operands)
template <class T>
__device__ __forceinline__ floatx4 op_mma(const uint4 &a, const uint4 &b, floatx4 c) {
    if constexpr (sizeof(T) == 4) {
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    } else if constexpr (__is_same(T, __bf16)) {
        op_bf16x8 x, y;
        __builtin_memcpy(&x, &a, 16);
        __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, c, 0, 0, 0);
    } else {
        op_f16x8 x, y;
        __builtin_memcpy(&x, &a, 16);
        __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, y, c, 0, 0, 0);
    }
}

static inline size_t op_dtype_size(int32_t dtype) { return dtype == TBS_F32 ? 4 : 2; }
static inline bool op_dtype_known(int32_t dtype) { return dtype >= TBS_F32 && dtype <= TBS_F16; }
