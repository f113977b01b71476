// What the operators of an autoregressive model (linear, attention over a paged cache and of prompts, selection over a vocabulary) share: element
// types, 16-byte pieces and the matrix instructions over them.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <initializer_list>

#include "tbs.h"

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 op_bf16x8;
typedef __attribute__((__vector_size__(8 * sizeof(_Float16)))) _Float16 op_f16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float floatx4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float floatx16;

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

// The same over two pieces a row and 32 rows of each side: a fragment is row (lane & 31), piece (lane >> 5) of two; a lane holds of column lane & 31, with
// h = lane >> 5, the rows 8 (i / 4) + 4 h + i % 4 as its i-th number.
template <class T>
__device__ __forceinline__ floatx16 op_mma32(const uint4 &a, const uint4 &b, floatx16 c) {
    if constexpr (sizeof(T) == 4) {
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.x), __uint_as_float(b.x), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.y), __uint_as_float(b.y), c, 0, 0, 0);
        c = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.z), __uint_as_float(b.z), c, 0, 0, 0);
        return __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(a.w), __uint_as_float(b.w), c, 0, 0, 0);
    } else if constexpr (__is_same(T, __bf16)) {
        op_bf16x8 x, y;
        __builtin_memcpy(&x, &a, 16);
        __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, c, 0, 0, 0);
    } else {
        op_f16x8 x, y;
        __builtin_memcpy(&x, &a, 16);
        __builtin_memcpy(&y, &b, 16);
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(x, y, c, 0, 0, 0);
    }
}

// A direct load to LDS, 16 bytes a lane, lane l's at lds + 16 l.  The compiler, which does not see these loads for what they are, adds no
// waits of its own: it would wait for all of them in front of every fragment read (it counts a direct load against any read
// of the array), and the loads of what comes next would be on their way for a part of the time only.  Every wait stands in the kernel.
__device__ __forceinline__ void op_load_lds(const char *from, unsigned lds) {
    unsigned m0_was;   // (whatever the compiler may keep there)
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %2, off\n\ts_mov_b32 m0, %0" : "=&s"(m0_was) : "s"(lds), "v"(from) : "memory");
}

// Rows of bytes: whether two sets of them have one in common.  (Rows of one stride, as of two slices of a tensor, by what their distance leaves; others
// row by row, where the memory between their ends overlaps at all.)
struct OpRows {
    const void *at;
    int64_t rows, ld, width;
};
static inline bool op_overlap(OpRows a, OpRows b) {
    if (a.rows > b.rows) {
        const OpRows t = a;
        a = b, b = t;
    }
    const int64_t d = (int64_t)((uintptr_t)b.at - (uintptr_t)a.at);
    if (d >= (a.rows - 1) * a.ld + a.width || -d >= (b.rows - 1) * b.ld + b.width) return false;
    auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    if (a.ld == b.ld) {
        const int64_t q = floor_div(d, a.ld), r = d - q * a.ld;   // row j of b begins r bytes behind row q + j of a
        return (r < a.width && q < a.rows && q + b.rows > 0) || (r + b.width > a.ld && q + 1 < a.rows && q + 1 + b.rows > 0);
    }
    for (int64_t i = 0; i < a.rows; ++i) {
        const int64_t s = i * a.ld - d;   // row i of a, from b's first byte
        const int64_t first = floor_div(s - b.width, b.ld) + 1, last = floor_div(s + a.width - 1, b.ld);
        if ((first > 0 ? first : 0) <= (last < b.rows ? last : b.rows - 1)) return true;
    }
    return false;
}

// rows of 32-bit or longer numbers that a call reads or writes as they are (none: at nothing)
static inline OpRows op_rows(const void *at, int64_t rows, int64_t ld, int64_t cols, int64_t size) {
    return {at, at && cols > 0 ? rows : 0, (rows > 1 ? ld : cols) * size, cols * size};
}
// whether what is written lies over itself or over what is read
static inline bool op_written_over(std::initializer_list<OpRows> written, std::initializer_list<OpRows> read) {
    for (const OpRows *w = written.begin(); w != written.end(); ++w) {
        if (w->rows < 1) continue;
        for (const OpRows *x = written.begin(); x != w; ++x)
            if (x->rows > 0 && op_overlap(*w, *x)) return true;
        for (const OpRows &x : read)
            if (x.rows > 0 && op_overlap(*w, x)) return true;
    }
    return false;
}

// [tokens, heads, dim] by elements, a head's side by side
struct OpHeads {
    const void *at;
    int64_t tokens, heads, dim, row, head;
};
// rows of `bytes` bytes, `ld` apart, among heads of numbers of `size` (none: at nothing)
static inline OpHeads op_plain(const void *at, int64_t rows, int64_t ld, int64_t bytes, int64_t size) { return {at, at && bytes > 0 ? rows : 0, 1, bytes / size, ld / size, 0}; }
static inline bool op_same(const OpHeads &a, const OpHeads &b) {
    return a.at == b.at && (a.row == b.row || a.tokens <= 1) && (a.head == b.head || a.heads <= 1);
}
// whether its heads may lie over each other: tokens in rows, or (a head's tokens together) heads in rows
static inline bool op_folded(const OpHeads &a) {
    const int64_t token = (a.heads > 1 ? (a.heads - 1) * a.head : 0) + a.dim, head = (a.tokens > 1 ? (a.tokens - 1) * a.row : 0) + a.dim;
    const bool by_token = (a.heads <= 1 || a.head >= a.dim) && (a.tokens <= 1 || a.row >= token);
    const bool by_head = (a.tokens <= 1 || a.row >= a.dim) && (a.heads <= 1 || a.head >= head);
    return !by_token && !by_head;
}
// whether heads of the one lie over heads of the other: rows of a token's heads, or of a head's tokens, where both are that; all memory between first and last otherwise
static inline bool op_overlap(const OpHeads &a, const OpHeads &b, int64_t size) {
    if (a.tokens < 1 || b.tokens < 1) return false;
    auto by = [&](const OpHeads &x, bool heads) {
        const int64_t n = heads ? x.heads : x.tokens, m = heads ? x.tokens : x.heads, ld = heads ? x.head : x.row, in = heads ? x.row : x.head;
        OpRows r = {x.at, n, ld * size, ((m - 1) * in + x.dim) * size};
        if (r.rows > 1 && r.ld < r.width) r.width += (r.rows - 1) * r.ld, r.rows = 1;
        if (r.rows == 1) r.ld = r.width;
        return r;
    };
    return op_overlap(by(a, false), by(b, false)) && op_overlap(by(a, true), by(b, true));
}

static inline size_t op_dtype_size(int32_t dtype) { return dtype == TBS_F32 ? 4 : 2; }
static inline bool op_dtype_known(int32_t dtype) { return dtype >= TBS_F32 && dtype <= TBS_F16; }

// [pages, page, heads, dim] by elements
struct OpCache {
    const void *at;
    int64_t pages, page, heads, dim, page_stride, token, head;
};
// Its dimensions of more than one place, from the longest stride on, and its numbers
struct OpStrides {
    int64_t count[3], stride[3], dim;
    int n;
    int64_t extent(int i) const {   // from the first number to behind the last, of the dimensions from the i-th on
        int64_t e = dim;
        for (; i < n; ++i) e += (count[i] - 1) * stride[i];
        return e;
    }
};
static inline OpStrides op_strides(const OpCache &a, int64_t size) {
    OpStrides x = {};
    x.dim = a.dim * size;
    const int64_t count[] = {a.pages, a.page, a.heads}, stride[] = {a.page_stride, a.token, a.head};
    for (int i = 0; i < 3; ++i) {
        if (count[i] <= 1) continue;
        int at = x.n++;
        for (; at > 0 && x.stride[at - 1] < stride[i] * size; --at) x.count[at] = x.count[at - 1], x.stride[at] = x.stride[at - 1];
        x.count[at] = count[i], x.stride[at] = stride[i] * size;
    }
    return x;
}
// whether its numbers may lie over each other
static inline bool op_folded(const OpCache &a, int64_t size) {
    const OpStrides x = op_strides(a, size);
    for (int i = 0; i < x.n; ++i)
        if (x.stride[i] < x.extent(i + 1)) return true;
    return false;
}
// Whether numbers of b, which begins d bytes behind a, lie over numbers of a, neither of them folded: while both have a dimension alike, by the places whose distance can make
// up for d (two at most); otherwise all memory between first and last
static inline bool op_meet(const OpStrides &a, const OpStrides &b, int i, int64_t d) {
    const int64_t na = a.extent(i), nb = b.extent(i);
    if (d >= na || -d >= nb) return false;
    if (i == a.n || i == b.n || a.count[i] != b.count[i] || a.stride[i] != b.stride[i]) return true;
    const int64_t s = a.stride[i], q = d / s;
    for (int64_t k = q - 1; k <= q + 1; ++k)
        if (k > -a.count[i] && k < a.count[i] && op_meet(a, b, i + 1, d - k * s)) return true;
    return false;
}
static inline bool op_overlap(const OpCache &a, const OpCache &b, int64_t size) {
    return op_meet(op_strides(a, size), op_strides(b, size), 0, (int64_t)((uintptr_t)b.at - (uintptr_t)a.at));
}
// whether all memory between a cache's first and last number meets that of heads (a call that writes the one and reads the other is refused)
static inline bool op_overlap(const OpCache &a, const OpHeads &b, int64_t size) {
    if (!a.at || !b.at || b.tokens < 1) return false;
    const int64_t na = ((a.pages - 1) * a.page_stride + (a.page - 1) * a.token + (a.heads - 1) * a.head + a.dim) * size, nb = ((b.tokens - 1) * b.row + (b.heads - 1) * b.head + b.dim) * size;
    return (uintptr_t)a.at < (uintptr_t)b.at + nb && (uintptr_t)b.at < (uintptr_t)a.at + na;
}
