// Queries and keys turned by their positions, keys and values into their places in the cache.
//
// A pair (a, b) becomes (a cos - b sin, b cos + a sin) with the angle position x frequency.  The angle is a product of float64 (at 10^6 positions
// float32 leaves it four digits), brought to quarters of a turn there, and the rest's sine and cosine are float32's.
#include "op_device.h"

#define ROTARY_THREADS 256
#define ROTARY_ANGLES 1024   // of a workgroup at most

struct RotaryP {
    const char *q, *k, *v;
    char *q_out, *k_out, *k_cache, *v_cache;
    const int *positions;
    const double *freqs;
    const int64_t *slots;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, qo_row, qo_head, ko_row, ko_head;   // bytes
    int64_t kp, kt, kh, vp, vt, vh, places;
    int tokens, heads, kv_heads, dim, pairs, page;
    int per, lanes;   // tokens of a workgroup, lanes of a head (a power of two)
};

__device__ __forceinline__ float2 rotary_angle(double position, double freq) {
    const double turns = position * freq * 0.15915494309189535;   // 1 / (2 pi)
    const double rest = turns - rint(turns), quarter = rint(4 * rest);
    float s, c;
    sincospif((float)(2 * rest - 0.5 * quarter), &s, &c);   // (at most a quarter of pi on both sides of 0)
    const int n = (int)quarter & 3;
    return n == 0 ? make_float2(c, s) : n == 1 ? make_float2(-s, c) : n == 2 ? make_float2(-c, -s) : make_float2(s, -c);
}

// the first n elements of 16 bytes (n of all of them: one store)
template <class T>
__device__ __forceinline__ void rotary_store(T *to, const T *x, int n) {
    constexpr int E = OpPiece<T>::E;
    if (n >= E) {
        __builtin_memcpy(to, x, 16);
        return;
    }
#pragma unroll
    for (int i = 0; i < E; ++i)
        if (i < n) to[i] = x[i];
}

template <class T>
__device__ __forceinline__ void rotary_load(T *x, const T *from, int n) {
    const uint4 u = n >= OpPiece<T>::E ? op_load16(from) : op_load16_part(from, n);
    __builtin_memcpy(x, &u, 16);
}

// A workgroup takes `per` tokens: their angles once into LDS, then all their heads by pieces of 16 bytes, `lanes` threads to a head; of the values a
// copy.  HALF: a pair is i and i + pairs, a thread takes both pieces; otherwise 2 i and 2 i + 1.
template <class T, bool HALF>
__global__ void __launch_bounds__(ROTARY_THREADS)
k_rotary(RotaryP p) {
    constexpr int E = OpPiece<T>::E;
    __shared__ float2 s_angle[ROTARY_ANGLES];
    const int t0 = (int)blockIdx.x * p.per, mine = min(p.per, p.tokens - t0);
    for (int i = threadIdx.x; i < mine * p.pairs; i += ROTARY_THREADS) {
        const int t = i / p.pairs;
        s_angle[i] = rotary_angle((double)p.positions[t0 + t], p.freqs[i - t * p.pairs]);
    }
    __syncthreads();
    const int turned = HALF ? (p.pairs + E - 1) / E : (2 * p.pairs + E - 1) / E, rest = p.dim - 2 * p.pairs;
    const int rows = p.heads + p.kv_heads + (p.slots ? p.kv_heads : 0), step = ROTARY_THREADS / p.lanes, lane = threadIdx.x & (p.lanes - 1);
    for (int r = threadIdx.x / p.lanes; r < mine * rows; r += step) {
        const int u = r / rows, h = r - u * rows, t = t0 + u;
        const bool is_q = h < p.heads, is_v = h >= p.heads + p.kv_heads;
        const int kvh = is_v ? h - p.heads - p.kv_heads : h - p.heads;
        char *cache = nullptr;   // where a key or value goes as well
        if (p.slots && !is_q) {
            const int64_t slot = p.slots[t];
            if (slot >= 0 && slot < p.places) {
                const int64_t page = slot <= UINT32_MAX ? (unsigned)slot / (unsigned)p.page : slot / p.page, off = slot - page * p.page;
                cache = is_v ? p.v_cache + page * p.vp + off * p.vt + kvh * p.vh : p.k_cache + page * p.kp + off * p.kt + kvh * p.kh;
            }
        }
        T x[E], y[E];
        if (is_v) {
            if (!cache) continue;
            const T *from = (const T *)(p.v + t * p.v_row + kvh * p.v_head);
            for (int c = lane * E; c < p.dim; c += p.lanes * E) {
                rotary_load(x, from + c, p.dim - c);
                rotary_store((T *)cache + c, x, p.dim - c);
            }
            continue;
        }
        const T *from = (const T *)(is_q ? p.q + t * p.q_row + h * p.q_head : p.k + t * p.k_row + kvh * p.k_head);
        T *to = (T *)(is_q ? p.q_out + t * p.qo_row + h * p.qo_head : p.k_out + t * p.ko_row + kvh * p.ko_head);
        if (lane < turned) {
            const int c = lane * E;
            const float2 *angle = s_angle + u * p.pairs;
            if constexpr (HALF) {
                const int n = p.pairs - c;
                rotary_load(x, from + c, n);
                rotary_load(y, from + p.pairs + c, n);
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float2 w = angle[min(c + i, p.pairs - 1)];
                    const float a = op_float(x[i]), b = op_float(y[i]);
                    x[i] = (T)(a * w.x - b * w.y);
                    y[i] = (T)(b * w.x + a * w.y);
                }
                rotary_store(to + c, x, n);
                rotary_store(to + p.pairs + c, y, n);
                if (cache) {
                    rotary_store((T *)cache + c, x, n);
                    rotary_store((T *)cache + p.pairs + c, y, n);
                }
            } else {
                const int n = 2 * p.pairs - c;
                rotary_load(x, from + c, n);
#pragma unroll
                for (int i = 0; i < E; i += 2) {
                    const float2 w = angle[min((c + i) / 2, p.pairs - 1)];
                    const float a = op_float(x[i]), b = op_float(x[i + 1]);
                    x[i] = (T)(a * w.x - b * w.y);
                    x[i + 1] = (T)(b * w.x + a * w.y);
                }
                rotary_store(to + c, x, n);
                if (cache) rotary_store((T *)cache + c, x, n);
            }
        } else if ((lane - turned) * E < rest) {   // what is behind the pairs stays as it is
            const int c = 2 * p.pairs + (lane - turned) * E;
            rotary_load(x, from + c, p.dim - c);
            rotary_store(to + c, x, p.dim - c);
            if (cache) rotary_store((T *)cache + c, x, p.dim - c);
        }
    }
}

template <class T>
static void rotary_run(const RotaryP &p, bool half, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)p.tokens + p.per - 1) / p.per)), block(ROTARY_THREADS);
    if (half) hipLaunchKernelGGL((k_rotary<T, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_rotary<T, false>), grid, block, 0, st, p);
}

extern "C" int tbs_rotary(const tbs_rotary_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_rotary_args &a = *args;
    if (!op_dtype_known(a.dtype) || a.tokens < 0 || a.heads < 1 || a.heads > 65535 || a.kv_heads < 1 || a.kv_heads > 65535 || a.dim < 1 || a.dim > 512 || a.pairs < 0 ||
        2 * a.pairs > a.dim || (a.interleaved != 0 && a.interleaved != 1))
        return TBS_EINVAL;
    const bool cached = a.slots != nullptr;
    if (cached && (a.pages < 1 || a.page < 1 || a.page > 65536)) return TBS_EINVAL;
    if (a.tokens == 0) return TBS_OK;
    if (!a.q || !a.k || !a.q_out || !a.k_out || !a.positions || (!a.freqs && a.pairs > 0)) return TBS_EINVAL;
    if (cached ? !a.v || !a.k_cache || !a.v_cache : a.v || a.k_cache || a.v_cache) return TBS_EINVAL;
    const int64_t strides[] = {a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.q_out_row, a.q_out_head, a.k_out_row, a.k_out_head,
                               a.k_cache_page, a.k_cache_token, a.k_cache_head, a.v_cache_page, a.v_cache_token, a.v_cache_head};
    for (int64_t s : strides)
        if (s < 0 || s > INT64_MAX / 64 / INT32_MAX) return TBS_EINVAL;
    const int64_t es = (int64_t)op_dtype_size(a.dtype);
    const void *ptrs[] = {a.q, a.k, a.v, a.q_out, a.k_out, a.k_cache, a.v_cache};
    for (const void *x : ptrs)
        if ((uintptr_t)x % es) return TBS_EINVAL;
    // what is written lies neither over itself nor over what others read
    const OpHeads q = {a.q, a.tokens, a.heads, a.dim, a.q_row, a.q_head}, k = {a.k, a.tokens, a.kv_heads, a.dim, a.k_row, a.k_head},
                  qo = {a.q_out, a.tokens, a.heads, a.dim, a.q_out_row, a.q_out_head}, ko = {a.k_out, a.tokens, a.kv_heads, a.dim, a.k_out_row, a.k_out_head};
    if (op_folded(qo) || op_folded(ko) || op_overlap(qo, ko, es) || op_overlap(qo, k, es) || op_overlap(ko, q, es) || (!op_same(q, qo) && op_overlap(qo, q, es)) ||
        (!op_same(k, ko) && op_overlap(ko, k, es)))
        return TBS_EINVAL;
    if (cached) {
        if ((a.kv_heads > 1 && (a.k_cache_head < a.dim || a.v_cache_head < a.dim)) || (a.page > 1 && (a.k_cache_token < a.dim || a.v_cache_token < a.dim)) ||
            (a.pages > 1 && (a.k_cache_page < a.dim || a.v_cache_page < a.dim)))
            return TBS_EINVAL;
        const OpHeads v = {a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head};
        if (op_overlap(qo, v, es) || op_overlap(ko, v, es)) return TBS_EINVAL;
    }
    RotaryP p = {};
    p.q = (const char *)a.q, p.k = (const char *)a.k, p.v = (const char *)a.v, p.q_out = (char *)a.q_out, p.k_out = (char *)a.k_out;
    p.k_cache = (char *)a.k_cache, p.v_cache = (char *)a.v_cache, p.positions = a.positions, p.freqs = a.freqs, p.slots = a.slots;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.k_row = a.k_row * es, p.k_head = a.k_head * es, p.v_row = a.v_row * es, p.v_head = a.v_head * es;
    p.qo_row = a.q_out_row * es, p.qo_head = a.q_out_head * es, p.ko_row = a.k_out_row * es, p.ko_head = a.k_out_head * es;
    p.kp = a.k_cache_page * es, p.kt = a.k_cache_token * es, p.kh = a.k_cache_head * es, p.vp = a.v_cache_page * es, p.vt = a.v_cache_token * es, p.vh = a.v_cache_head * es;
    p.places = cached ? (int64_t)a.pages * a.page : 0;
    p.tokens = a.tokens, p.heads = a.heads, p.kv_heads = a.kv_heads, p.dim = a.dim, p.pairs = a.pairs, p.page = cached ? a.page : 1;
    const int e = (int)(16 / es), pieces = (a.interleaved ? (2 * a.pairs + e - 1) / e : (a.pairs + e - 1) / e) + (a.dim - 2 * a.pairs + e - 1) / e;
    p.lanes = 1;
    while (p.lanes < pieces) p.lanes *= 2;   // (at most 129 pieces)
    const int rows = a.heads + a.kv_heads * (cached ? 2 : 1);
    int64_t per = ((int64_t)ROTARY_THREADS / p.lanes * 4 + rows - 1) / rows;   // four heads a thread
    if (a.pairs > 0 && per > ROTARY_ANGLES / a.pairs) per = ROTARY_ANGLES / a.pairs;
    if (per > a.tokens / 1024) per = a.tokens / 1024;   // (few tokens: one a workgroup)
    p.per = per < 1 ? 1 : (int)per;
    const hipStream_t st = (hipStream_t)stream;
    a.dtype == TBS_F32 ? rotary_run<float>(p, !a.interleaved, st) : a.dtype == TBS_BF16 ? rotary_run<__bf16>(p, !a.interleaved, st) : rotary_run<_Float16>(p, !a.interleaved, st);
    return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
}
