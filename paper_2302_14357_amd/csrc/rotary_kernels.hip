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

// A head's row is pieces of 16 bytes: those of its pairs, then those of what is behind them.  A lane has two of every row that it takes.
struct RotaryPieces {
    int c[2], n[2], turned;   // first element, elements (none: 0 or fewer); bits of those that turn
};

template <int E, bool HALF>
__device__ __forceinline__ RotaryPieces rotary_pieces(const RotaryP &p, int lane) {
    const int front = 2 * p.pairs, turned = ((HALF ? p.pairs : front) + E - 1) / E, rest = (p.dim - front + E - 1) / E;
    RotaryPieces x;
    if (HALF && lane < turned) {   // both members of its pairs
        x.c[0] = lane * E, x.c[1] = p.pairs + lane * E;
        x.n[0] = x.n[1] = p.pairs - lane * E;
        x.turned = 3;
        return x;
    }
    const int count = HALF ? rest : turned + rest, half = (count + 1) / 2, mine = HALF ? lane - turned : lane;
    x.turned = 0;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int i = mine + j * half;
        const bool turns = !HALF && i < turned;
        x.c[j] = turns || HALF ? i * E + (HALF ? front : 0) : front + (i - turned) * E;
        x.n[j] = mine < half && i < count ? (turns ? front : p.dim) - x.c[j] : 0;
        x.turned |= (int)turns << j;
    }
    return x;
}

// A workgroup takes `per` tokens: their angles once into LDS, then all their heads, `lanes` threads to a head, the next head's pieces on their way while
// one is turned; of the values a copy.  HALF: a pair is i and i + pairs; otherwise 2 i and 2 i + 1.  WHOLE: all of a head turns, and every
// lane has two whole pieces.
// Bound by memory: 8000 tokens, heads of 32 + 8 + 8 x 128, bfloat16, with the cache 42 to 45 us, 4.7 to 5.1 TB/s (on inputs that the caches hold in part 34; 36 without the next
// head's loads ahead, 37 without WHOLE); 500 tokens of them 5.4 us.  A half of 256 turned, 16 + 4 + 4 heads, 4000 tokens, float16: 23 us (one piece a lane 31).
template <class T, bool HALF, bool WHOLE>
__global__ void __launch_bounds__(ROTARY_THREADS)
k_rotary(RotaryP p) {
    constexpr int E = OpPiece<T>::E;
    __shared__ float2 s_angle[ROTARY_ANGLES];
    const int t0 = (int)blockIdx.x * p.per, mine = min(p.per, p.tokens - t0);
    const int rows = p.heads + p.kv_heads + (p.slots ? p.kv_heads : 0), all = mine * rows, step = ROTARY_THREADS / p.lanes;
    const int lane = threadIdx.x & (p.lanes - 1);
    RotaryPieces at = rotary_pieces<E, HALF>(p, lane);
    if (WHOLE) at.c[0] = lane * E, at.c[1] = p.pairs + at.c[0];
    struct Row {
        T x[2][E];
        int64_t slot;
    };
    auto load = [&](Row &row, int r) {
        const int u = r / rows, h = r - u * rows, t = t0 + u;
        const bool is_q = h < p.heads, is_v = h >= p.heads + p.kv_heads;
        row.slot = p.slots && !is_q ? p.slots[t] : -1;
        const T *from = (const T *)(is_q ? p.q + t * p.q_row + h * p.q_head : is_v ? p.v + t * p.v_row + (h - p.heads - p.kv_heads) * p.v_head : p.k + t * p.k_row + (h - p.heads) * p.k_head);
#pragma unroll
        for (int j = 0; j < 2; ++j)
            if (WHOLE || at.n[j] > 0) rotary_load(row.x[j], from + at.c[j], WHOLE ? E : at.n[j]);
    };
    int r = threadIdx.x / p.lanes;
    Row row, next;
    if (r < all) load(row, r);
    for (int i = threadIdx.x; i < mine * p.pairs; i += ROTARY_THREADS) {
        const int t = i / p.pairs;
        s_angle[i] = rotary_angle((double)p.positions[t0 + t], p.freqs[i - t * p.pairs]);
    }
    __syncthreads();
    for (; r < all; r += step) {
        if (r + step < all) load(next, r + step);
        const int u = r / rows, h = r - u * rows, t = t0 + u;
        const bool is_q = h < p.heads, is_v = h >= p.heads + p.kv_heads;
        const int kvh = is_v ? h - p.heads - p.kv_heads : h - p.heads;
        const float2 *angle = s_angle + u * p.pairs;
        if ((WHOLE || at.turned) && !is_v) {
            if constexpr (HALF) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    const float2 w = angle[WHOLE ? at.c[0] + i : min(at.c[0] + i, p.pairs - 1)];
                    const float a = op_float(row.x[0][i]), b = op_float(row.x[1][i]);
                    row.x[0][i] = (T)(a * w.x - b * w.y);
                    row.x[1][i] = (T)(b * w.x + a * w.y);
                }
            } else {
#pragma unroll
                for (int j = 0; j < 2; ++j)
                    if (WHOLE || at.turned >> j & 1)
#pragma unroll
                        for (int i = 0; i < E; i += 2) {
                            const float2 w = angle[WHOLE ? (at.c[j] + i) / 2 : min((at.c[j] + i) / 2, p.pairs - 1)];
                            const float a = op_float(row.x[j][i]), b = op_float(row.x[j][i + 1]);
                            row.x[j][i] = (T)(a * w.x - b * w.y);
                            row.x[j][i + 1] = (T)(b * w.x + a * w.y);
                        }
            }
        }
        if (!is_v) {
            T *to = (T *)(is_q ? p.q_out + t * p.qo_row + h * p.qo_head : p.k_out + t * p.ko_row + kvh * p.ko_head);
#pragma unroll
            for (int j = 0; j < 2; ++j) rotary_store(to + at.c[j], row.x[j], WHOLE ? E : at.n[j]);
        }
        if (row.slot >= 0 && row.slot < p.places) {   // where a key or value goes as well
            const int64_t page = row.slot <= UINT32_MAX ? (unsigned)row.slot / (unsigned)p.page : row.slot / p.page, off = row.slot - page * p.page;
            T *to = (T *)(is_v ? p.v_cache + page * p.vp + off * p.vt + kvh * p.vh : p.k_cache + page * p.kp + off * p.kt + kvh * p.kh);
#pragma unroll
            for (int j = 0; j < 2; ++j) rotary_store(to + at.c[j], row.x[j], WHOLE ? E : at.n[j]);
        }
        row = next;
    }
}

template <class T>
static void rotary_run(const RotaryP &p, bool half, hipStream_t st) {
    const dim3 grid((unsigned)(((int64_t)p.tokens + p.per - 1) / p.per)), block(ROTARY_THREADS);
    const bool whole = p.dim == 2 * p.pairs && p.lanes * OpPiece<T>::E == p.pairs;
    if (whole) {
        if (half) hipLaunchKernelGGL((k_rotary<T, true, true>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((k_rotary<T, false, true>), grid, block, 0, st, p);
    } else {
        if (half) hipLaunchKernelGGL((k_rotary<T, true, false>), grid, block, 0, st, p);
        else hipLaunchKernelGGL((k_rotary<T, false, false>), grid, block, 0, st, p);
    }
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
    const OpHeads plain[] = {op_plain(a.positions, 1, 0, 4ll * a.tokens, es), op_plain(a.freqs, 1, 0, 8ll * a.pairs, es), op_plain(a.slots, 1, 0, 8ll * a.tokens, es)};
    for (const OpHeads &x : plain)
        if (op_overlap(qo, x, es) || op_overlap(ko, x, es)) return TBS_EINVAL;
    if (cached) {
        if ((a.kv_heads > 1 && (a.k_cache_head < a.dim || a.v_cache_head < a.dim)) || (a.page > 1 && (a.k_cache_token < a.dim || a.v_cache_token < a.dim)) ||
            (a.pages > 1 && (a.k_cache_page < a.dim || a.v_cache_page < a.dim)))
            return TBS_EINVAL;
        const OpHeads v = {a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head};
        const OpCache kc = {a.k_cache, a.pages, a.page, a.kv_heads, a.dim, a.k_cache_page, a.k_cache_token, a.k_cache_head},
                      vc = {a.v_cache, a.pages, a.page, a.kv_heads, a.dim, a.v_cache_page, a.v_cache_token, a.v_cache_head};
        if (op_overlap(qo, v, es) || op_overlap(ko, v, es) || op_folded(kc, es) || op_folded(vc, es) || op_overlap(kc, vc, es)) return TBS_EINVAL;
        for (const OpCache &cache : {kc, vc}) {
            if (op_overlap(cache, q, es) || op_overlap(cache, k, es) || op_overlap(cache, v, es) || op_overlap(cache, qo, es) || op_overlap(cache, ko, es)) return TBS_EINVAL;
            for (const OpHeads &x : plain)
                if (op_overlap(cache, x, es)) return TBS_EINVAL;
        }
    }
    RotaryP p = {};
    p.q = (const char *)a.q, p.k = (const char *)a.k, p.v = (const char *)a.v, p.q_out = (char *)a.q_out, p.k_out = (char *)a.k_out;
    p.k_cache = (char *)a.k_cache, p.v_cache = (char *)a.v_cache, p.positions = a.positions, p.freqs = a.freqs, p.slots = a.slots;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.k_row = a.k_row * es, p.k_head = a.k_head * es, p.v_row = a.v_row * es, p.v_head = a.v_head * es;
    p.qo_row = a.q_out_row * es, p.qo_head = a.q_out_head * es, p.ko_row = a.k_out_row * es, p.ko_head = a.k_out_head * es;
    p.kp = a.k_cache_page * es, p.kt = a.k_cache_token * es, p.kh = a.k_cache_head * es, p.vp = a.v_cache_page * es, p.vt = a.v_cache_token * es, p.vh = a.v_cache_head * es;
    p.places = cached ? (int64_t)a.pages * a.page : 0;
    p.tokens = a.tokens, p.heads = a.heads, p.kv_heads = a.kv_heads, p.dim = a.dim, p.pairs = a.pairs, p.page = cached ? a.page : 1;
    const int e = (int)(16 / es), turned = ((a.interleaved ? 2 * a.pairs : a.pairs) + e - 1) / e, behind = (a.dim - 2 * a.pairs + e - 1) / e;
    const int pieces = a.interleaved ? (turned + behind + 1) / 2 : turned + (behind + 1) / 2;   // lanes that a head needs
    p.lanes = 1;
    while (p.lanes < pieces) p.lanes *= 2;   // (at most 65)
    const int rows = a.heads + a.kv_heads * (cached ? 2 : 1);
    int64_t per = ((int64_t)ROTARY_THREADS / p.lanes * 4 + rows - 1) / rows;   // four heads a thread
    if (a.pairs > 0 && per > ROTARY_ANGLES / a.pairs) per = ROTARY_ANGLES / a.pairs;
    if (per > a.tokens / 1024) per = a.tokens / 1024;   // (few tokens: one a workgroup)
    p.per = per < 1 ? 1 : (int)per;
    const hipStream_t st = (hipStream_t)stream;
    a.dtype == TBS_F32 ? rotary_run<float>(p, !a.interleaved, st) : a.dtype == TBS_BF16 ? rotary_run<__bf16>(p, !a.interleaved, st) : rotary_run<_Float16>(p, !a.interleaved, st);
    return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
}
