// Attention of one new token per row over a paged cache of keys and values.
//
// With t = log2(e) scale q.k of a token and a running maximum m over the tokens seen, o = sum 2^(t - m) v and l = sum 2^(t - m) are kept in
// float32 registers; a larger m multiplies both by 2^(m_old - m_new).  One pass over the cache, no score is stored.
//
// Sixteen queries are the columns of the matrix instructions (the query heads of one key head; fewer leave columns idle, which costs
// nothing: the cache's bytes bound the kernel).  A wave takes tiles of 32 tokens (float32: 16) without LDS or barriers:
//  - scores: keys are the rows, S^T = K Q^T.  A lane then has, of one query, the tokens 16 b + 4 (lane / 16) + r of the tile;
//  - output: O^T = V^T P^T.  The order of the tokens in the sum is free, so it is made the order in which a lane has its weights: what the
//    scores' instruction returns goes into the next one as it is.  V comes in rows of whole heads, W = dim / 16 elements a
//    lane; the i-th row of the n-th instruction is made dimension W i + n, so that a lane has its eight tokens' values of that dimension in
//    its own registers, and only halves of registers change places (four byte permutes an instruction).
// A lane keeps maximum, sum and output of one query: nothing but the maximum crosses lanes.
#include "op_device.h"

#define ATT_WAVES 4
#define ATT_TABLE 1024   // page table entries in LDS at a time

struct AttendP {
    const char *q, *k_new, *v_new;
    char *k_cache, *v_cache;
    const int *tables, *lens;
    char *out;
    float *part_o, *part_ml;   // [rows, heads, splits, dim], [rows, heads, splits, 2]; only with more than one split
    int64_t q_row, q_head, kn_row, kn_head, vn_row, vn_head, o_row, o_head, kp, kt, kh, vp, vt, vh, ld_tables;   // bytes (ld_tables: elements)
    int rows, heads, kv_heads, group, dim, page, pages, width, splits, split_len, qblocks;
    unsigned page_mul, page_shift;
    float scale2;   // scale * log2(e)
};

// t / page for 0 <= t < 2^31 (by multiplication: page_mul = floor(2^(32 + s) / page) + 1 with s = floor(log2 page) errs by less than 2^-31 a unit)
__device__ __forceinline__ int att_page(const AttendP &p, int t) {
    return p.page_mul ? (int)(__umulhi((unsigned)t, p.page_mul) >> p.page_shift) : (int)((unsigned)t >> p.page_shift);
}

// tokens that row r attends to; *pos: place of its new token (-1: none)
__device__ __forceinline__ int att_tokens(const AttendP &p, int r, int *pos) {
    const int len = p.lens[r];
    const int64_t cap = (int64_t)p.width * p.page;
    *pos = -1;
    if (len < 0) return 0;
    if (p.k_new && len < cap) {
        *pos = len;
        return len + 1;
    }
    return (int)(len < cap ? len : cap);
}

template <int N>
struct AttWords {
    unsigned w[N];
};

template <class T, int DP>
struct AttTile {
    static constexpr int NB = sizeof(T) == 4 ? 1 : 2;          // blocks of 16 tokens
    static constexpr int TK = 16 * NB, NV = 4 * NB;            // tokens of a tile; of V a lane
    static constexpr int KS = DP * (int)sizeof(T) / 64;        // 16-byte pieces of a key a lane
    static constexpr int W = DP / 16, WW = W * (int)sizeof(T) / 4;   // dimensions of V a lane, in 4-byte words
    uint4 k[NB][KS];
    unsigned v[NV][WW];
    unsigned ok;   // bit j: V's token j exists
};

// DP: dim rounded up to 32, 64, 128 or 256 (PAD: it was not that already)
template <class T, int DP, bool PAD>
__global__ void __launch_bounds__(64 * ATT_WAVES, 2)
k_attend(AttendP p) {
    typedef AttTile<T, DP> Tile;
    constexpr int E = OpPiece<T>::E, NB = Tile::NB, TK = Tile::TK, NV = Tile::NV, KS = Tile::KS, W = Tile::W, WW = Tile::WW;
    __shared__ int s_table[ATT_TABLE + 1];
    __shared__ float s_o[ATT_WAVES / 2][W * 4][64];
    __shared__ float s_ml[ATT_WAVES][2][16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int kvh = (int)blockIdx.x % p.kv_heads, qblk = (int)blockIdx.x / p.kv_heads, split = blockIdx.y, row = blockIdx.z;
    int pos;
    const int n = att_tokens(p, row, &pos);
    const int k0 = split * p.split_len;
    if (k0 >= n && split > 0) return;   // (of a row without tokens the first workgroup writes the zeros)
    const int k1 = split == p.splits - 1 ? n : min(n, k0 + p.split_len);   // (the last goes on to the row's end, whatever max_len said)
    const int qh = qblk * 16 + c;       // query head within the group
    const bool has_q = qh < p.group;
    const int head = kvh * p.group + min(qh, p.group - 1);
    const char *kb = p.k_cache + kvh * p.kh, *vb = p.v_cache + kvh * p.vh;
    const char *kn = p.k_new ? p.k_new + row * p.kn_row + kvh * p.kn_head : nullptr, *vn = kn ? p.v_new + row * p.vn_row + kvh * p.vn_head : nullptr;
    const bool quad = (p.page & 3) == 0;   // four tokens from a multiple of four on lie in one page

    uint4 q[KS];
    {
        const T *src = (const T *)(p.q + row * p.q_row + head * p.q_head);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = has_q && (!PAD || (s * 4 + kg) * E < p.dim) ? op_load16(src + (s * 4 + kg) * E) : make_uint4(0, 0, 0, 0);
    }
    floatx4 o[W];
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] = floatx4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY, l = 0.f;

    for (int c0 = k0; c0 < k1; c0 += ATT_TABLE * p.page) {
        const int first = att_page(p, c0), c1 = min((int64_t)k1, (int64_t)c0 + (int64_t)ATT_TABLE * p.page);
        if (c0 > k0) __syncthreads();
        for (int i = threadIdx.x; i <= att_page(p, c1 - 1) - first; i += 64 * ATT_WAVES) s_table[i] = p.tables[row * p.ld_tables + first + i];
        __syncthreads();
        // a token's page in the pool (negative: it does not exist) and its place there
        auto page_of = [&](int t, int &off) {
            const int i = att_page(p, t), id = s_table[i - first];
            off = t - i * p.page;
            return (unsigned)id < (unsigned)p.pages ? id : -1;
        };
        auto load = [&](Tile &x, int t0) {
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                const int t = min(t0 + b * 16 + c, c1 - 1);
                int off;
                const int id = page_of(t, off);
                const char *at = t == pos ? kn : id < 0 ? kb : kb + id * p.kp + off * p.kt;
#pragma unroll
                for (int s = 0; s < KS; ++s)
                    x.k[b][s] = !PAD || (s * 4 + kg) * E < p.dim ? op_load16((const T *)at + (s * 4 + kg) * E) : make_uint4(0, 0, 0, 0);
            }
            x.ok = 0;
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                int off = 0, id = 0;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int want = t0 + b * 16 + kg * 4 + r, t = min(want, c1 - 1);
                    if (r == 0 || !quad) id = page_of(t, off);
                    const char *at = t == pos ? vn : id < 0 ? vb : vb + id * p.vp + (quad ? off + (t - min(want - r, c1 - 1)) : off) * p.vt;
                    if (want < c1 && (id >= 0 || t == pos)) x.ok |= 1u << (b * 4 + r);
                    unsigned *v = x.v[b * 4 + r];
                    constexpr int G = W < 8 ? W : 8;   // elements that are there together or not at all: dim is a multiple of 8
#pragma unroll
                    for (int g = 0; g < W / G; ++g) {
                        constexpr int GW = G * (int)sizeof(T) / 4;
                        AttWords<GW> u = {};
                        if (!PAD || c * W + g * G < p.dim) __builtin_memcpy(&u, (const T *)at + c * W + g * G, sizeof u);
#pragma unroll
                        for (int i = 0; i < GW; ++i) v[g * GW + i] = u.w[i];
                    }
                }
            }
        };
        auto compute = [&](Tile &x) {
            const bool whole = __all(x.ok == (1u << NV) - 1);
            if (!whole) {   // what stands in places without a token may be anything
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < WW; ++i) x.v[j][i] = x.ok >> j & 1 ? x.v[j][i] : 0;
            }
            float t[NV];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
                floatx4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int i = 0; i < KS; ++i) s = op_mma<T>(x.k[b][i], q[i], s);
#pragma unroll
                for (int r = 0; r < 4; ++r) t[b * 4 + r] = whole || (x.ok >> (b * 4 + r) & 1) ? s[r] * p.scale2 : -INFINITY;
            }
            float top = t[0];
#pragma unroll
            for (int j = 1; j < NV; ++j) top = fmaxf(top, t[j]);
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            if (__any(top > m)) {
                const float m1 = fmaxf(m, top), a = m1 == m ? 1.f : __builtin_amdgcn_exp2f(m - m1);
                m = m1;
                l *= a;
#pragma unroll
                for (int i = 0; i < W; ++i) o[i] *= a;
            }
            // (fp16: weights up to 2^12 instead of 1, so that small ones keep their digits)
            const float base = m == -INFINITY ? 0.f : m - (__is_same(T, _Float16) ? 12.f : 0.f);
#pragma unroll
            for (int j = 0; j < NV; ++j) {
                t[j] = __builtin_amdgcn_exp2f(t[j] - base);
                l += t[j];
            }
            if constexpr (sizeof(T) == 4) {
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int i = 0; i < W; ++i) o[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[r][i]), t[r], o[i], 0, 0, 0);
            } else {
                // A weight goes into the matrix instruction as two numbers of 16 bits, its rounding and what that left out: a weight's error
                // is then 2^-17 (fp16: 2^-22) instead of 2^-9, and the output's own rounding is all that shows.  (The second half of the
                // products costs no time: memory bounds the kernel.)
                T hi[8], lo[8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    hi[j] = (T)t[j];
                    lo[j] = (T)(t[j] - (float)hi[j]);
                }
                uint4 ph, pl;
                __builtin_memcpy(&ph, hi, 16);
                __builtin_memcpy(&pl, lo, 16);
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    const unsigned sel = i & 1 ? 0x07060302u : 0x05040100u;
                    const uint4 a = make_uint4(__builtin_amdgcn_perm(x.v[1][i / 2], x.v[0][i / 2], sel), __builtin_amdgcn_perm(x.v[3][i / 2], x.v[2][i / 2], sel),
                                               __builtin_amdgcn_perm(x.v[5][i / 2], x.v[4][i / 2], sel), __builtin_amdgcn_perm(x.v[7][i / 2], x.v[6][i / 2], sel));
                    o[i] = op_mma<T>(a, ph, o[i]);
                    o[i] = op_mma<T>(a, pl, o[i]);
                }
            }
        };
        for (int t0 = c0 + wave * TK; t0 < c1; t0 += ATT_WAVES * TK) {
            Tile x;
            load(x, t0);
            compute(x);
        }
    }
    // the waves' shares: 3 and 2 to 1 and 0, 1 to 0; every lane has the same place in all of them
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (lane < 16) {
        s_ml[wave][0][c] = m;
        s_ml[wave][1][c] = l;
    }
    __syncthreads();
    float top = m;
#pragma unroll
    for (int i = 0; i < ATT_WAVES; ++i) top = fmaxf(top, s_ml[i][0][c]);
    auto share = [&](float x) { return x == top ? 1.f : __builtin_amdgcn_exp2f(x - top); };   // (-inf of -inf: nothing there, 1 x 0)
    const float a = share(m);
    l = 0.f;
#pragma unroll
    for (int i = 0; i < ATT_WAVES; ++i) l += s_ml[i][1][c] * share(s_ml[i][0][c]);
#pragma unroll
    for (int i = 0; i < W; ++i) o[i] *= a;
#pragma unroll
    for (int h = ATT_WAVES / 2; h > 0; h >>= 1) {
        if (wave >= h && wave < 2 * h)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) s_o[wave - h][i * 4 + r][lane] = o[i][r];
        __syncthreads();
        if (wave < h)
#pragma unroll
            for (int i = 0; i < W; ++i)
#pragma unroll
                for (int r = 0; r < 4; ++r) o[i][r] += s_o[wave][i * 4 + r][lane];
        __syncthreads();
    }
    if (wave == 0) {
        const float inv = l == 0.f ? 0.f : 1.f / l;   // (no weight at all: 0)
        if (has_q) {
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                const int d = (kg * 4 + r) * W;
                constexpr int G = W < 8 ? W : 8;
#pragma unroll
                for (int g = 0; g < W / G; ++g) {
                    if (PAD && d + g * G >= p.dim) continue;
                    if (p.splits > 1) {
                        float *dst = p.part_o + (((int64_t)row * p.heads + head) * p.splits + split) * p.dim + d + g * G;
#pragma unroll
                        for (int i = 0; i < G; ++i) dst[i] = o[g * G + i][r];
                    } else {
                        T y[G];
#pragma unroll
                        for (int i = 0; i < G; ++i) y[i] = (T)(l == 0.f ? 0.f : o[g * G + i][r] * inv);
                        __builtin_memcpy((T *)(p.out + row * p.o_row + head * p.o_head) + d + g * G, y, sizeof y);
                    }
                }
            }
            if (p.splits > 1 && kg == 0) {
                float *ml = p.part_ml + (((int64_t)row * p.heads + head) * p.splits + split) * 2;
                ml[0] = top;
                ml[1] = l;
            }
        }
    } else if (wave == 1 && qblk == 0 && pos >= k0 && pos < k1) {
        // the new token's place in the cache (this launch reads the token from k_new and v_new, whoever attends to it)
        const int i = att_page(p, pos), id = p.tables[row * p.ld_tables + i], off = pos - i * p.page;
        if ((unsigned)id < (unsigned)p.pages)
            for (int d = lane; d < p.dim; d += 64) {
                ((T *)(p.k_cache + id * p.kp + off * p.kt + kvh * p.kh))[d] = ((const T *)kn)[d];
                ((T *)(p.v_cache + id * p.vp + off * p.vt + kvh * p.vh))[d] = ((const T *)vn)[d];
            }
    }
}

// The splits' shares of one row and head: a workgroup of four waves, a share of the splits each.
template <class T>
__global__ void __launch_bounds__(256)
k_attend_join(AttendP p) {
    __shared__ float s_o[4][256], s_l[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, row = blockIdx.y, head = blockIdx.x;
    int pos;
    const int n = att_tokens(p, row, &pos), used = n == 0 ? 1 : min(p.splits, (int)(((int64_t)n + p.split_len - 1) / p.split_len));
    const float *ml = p.part_ml + ((int64_t)row * p.heads + head) * p.splits * 2;
    const float *po = p.part_o + ((int64_t)row * p.heads + head) * p.splits * p.dim;
    float top = -INFINITY;
    for (int s = lane; s < used; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    float o[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
    for (int s = wave; s < used; s += 4) {
        const float m = ml[2 * s], a = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top);
        l += a * ml[2 * s + 1];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (i * 64 + lane < p.dim) o[i] += a * po[(int64_t)s * p.dim + i * 64 + lane];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) s_o[wave][i * 64 + lane] = o[i];
    if (lane == 0) s_l[wave] = l;
    __syncthreads();
    const int d = threadIdx.x;
    l = s_l[0] + s_l[1] + s_l[2] + s_l[3];
    if (d < p.dim)
        ((T *)(p.out + row * p.o_row + head * p.o_head))[d] = (T)(l == 0.f ? 0.f : (s_o[0][d] + s_o[1][d] + s_o[2][d] + s_o[3][d]) / l);
}

// How the work is split: workgroups of a row and key head (and sixteen query heads), and over the tokens where those are fewer than the
// chip holds at once.
struct AttendPlan {
    int qblocks, splits, split_len;
};

static AttendPlan attend_plan(const tbs_attend_args &a) {
    const int group = a.heads / a.kv_heads, tile = a.dtype == TBS_F32 ? 16 : 32;
    AttendPlan pl;
    pl.qblocks = (group + 15) / 16;
    const int64_t cap = (int64_t)a.table_width * a.page;
    const int64_t longest = a.max_len > 0 && a.max_len < cap ? a.max_len : cap;
    const int64_t units = (int64_t)a.rows * a.kv_heads * pl.qblocks;
    const int64_t step = ATT_WAVES * tile;   // a tile for every wave
    int64_t splits = 1024 / units, most = (longest + 2 * step - 1) / (2 * step);
    if (splits > most) splits = most;
    if (splits < 1) splits = 1;
    int64_t len = (longest + splits - 1) / splits;
    len = (len + step - 1) / step * step;
    if (len < step) len = step;
    pl.split_len = (int)len;
    pl.splits = (int)((longest + len - 1) / len);
    if (pl.splits < 1) pl.splits = 1;
    return pl;
}

static int attend_check(const tbs_attend_args &a) {
    if (!op_dtype_known(a.dtype) || a.rows < 0 || a.kv_heads < 1 || a.heads < a.kv_heads || a.heads % a.kv_heads || a.dim < 8 || a.dim > 256 || a.dim % 8)
        return TBS_EINVAL;
    if (a.page < 1 || a.page > 65536 || a.pages < 1 || a.table_width < 1 || a.max_len < 0 || a.beams < 1 || a.rows % a.beams) return TBS_EINVAL;
    if (a.rows > 65535 || a.heads > 65535 || (int64_t)a.table_width * a.page > (1 << 30)) return TBS_EINVAL;
    return TBS_OK;
}

extern "C" int64_t tbs_attend_workspace(const tbs_attend_args *args) {
    if (!args || attend_check(*args) != TBS_OK) return TBS_EINVAL;
    const AttendPlan pl = attend_plan(*args);
    return pl.splits > 1 ? (int64_t)args->rows * args->heads * pl.splits * (args->dim + 2) * 4 : 0;
}

template <class T, int DP>
static void attend_launch(const AttendP &p, hipStream_t st) {
    const dim3 grid(p.kv_heads * p.qblocks, p.splits, p.rows), block(64 * ATT_WAVES);
    if (p.dim == DP) hipLaunchKernelGGL((k_attend<T, DP, false>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_attend<T, DP, true>), grid, block, 0, st, p);
}

template <class T>
static hipError_t attend_run(const AttendP &p, hipStream_t st) {
    if (p.dim <= 32) attend_launch<T, 32>(p, st);
    else if (p.dim <= 64) attend_launch<T, 64>(p, st);
    else if (p.dim <= 128) attend_launch<T, 128>(p, st);
    else attend_launch<T, 256>(p, st);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        hipLaunchKernelGGL((k_attend_join<T>), dim3(p.heads, p.rows), dim3(256), 0, st, p);
        e = hipGetLastError();
    }
    return e;
}

extern "C" int tbs_attend_paged(const tbs_attend_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_attend_args &a = *args;
    if (attend_check(a) != TBS_OK) return TBS_EINVAL;
    if (a.rows == 0) return TBS_OK;
    if (!a.q || !a.k_cache || !a.v_cache || !a.tables || !a.lens || !a.out || !a.k_new != !a.v_new || a.ld_tables < a.table_width) return TBS_EINVAL;
    const int64_t es = (int64_t)op_dtype_size(a.dtype);
    const int64_t strides[] = {a.q_row, a.q_head, a.k_new_row, a.k_new_head, a.v_new_row, a.v_new_head, a.out_row, a.out_head,
                               a.k_page, a.k_token, a.k_head, a.v_page, a.v_token, a.v_head};
    for (int64_t s : strides)
        if (s < 0 || s > INT64_MAX / 64 / INT32_MAX) return TBS_EINVAL;
    // what is written may not lie over itself: a head after the other in the outputs and the cache
    if ((a.heads > 1 && a.out_head < a.dim) || (a.rows > 1 && a.out_row < a.dim)) return TBS_EINVAL;
    if (a.k_new && ((a.kv_heads > 1 && (a.k_head < a.dim || a.v_head < a.dim)) || (a.page > 1 && (a.k_token < a.dim || a.v_token < a.dim)) ||
                    (a.pages > 1 && (a.k_page < a.dim || a.v_page < a.dim))))
        return TBS_EINVAL;
    const void *ptrs[] = {a.q, a.k_new, a.v_new, a.k_cache, a.v_cache, a.out};
    for (const void *x : ptrs)
        if ((uintptr_t)x % es) return TBS_EINVAL;
    const AttendPlan pl = attend_plan(a);
    const int64_t need = tbs_attend_workspace(&a);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return TBS_EINVAL;
    AttendP p = {};
    p.q = (const char *)a.q, p.k_new = (const char *)a.k_new, p.v_new = (const char *)a.v_new;
    p.k_cache = (char *)a.k_cache, p.v_cache = (char *)a.v_cache, p.out = (char *)a.out;
    p.tables = a.tables, p.lens = a.lens;
    p.part_o = (float *)a.workspace;
    p.part_ml = p.part_o + (int64_t)a.rows * a.heads * pl.splits * a.dim;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.kn_row = a.k_new_row * es, p.kn_head = a.k_new_head * es;
    p.vn_row = a.v_new_row * es, p.vn_head = a.v_new_head * es, p.o_row = a.out_row * es, p.o_head = a.out_head * es;
    p.kp = a.k_page * es, p.kt = a.k_token * es, p.kh = a.k_head * es, p.vp = a.v_page * es, p.vt = a.v_token * es, p.vh = a.v_head * es;
    p.ld_tables = a.ld_tables;
    p.rows = a.rows, p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = a.heads / a.kv_heads, p.dim = a.dim;
    p.page = a.page, p.pages = a.pages, p.width = a.table_width, p.splits = pl.splits, p.split_len = pl.split_len, p.qblocks = pl.qblocks;
    const unsigned lg = 31 - __builtin_clz((unsigned)a.page);
    p.page_shift = lg;
    p.page_mul = (a.page & (a.page - 1)) ? (unsigned)((((uint64_t)1 << (32 + lg)) / (unsigned)a.page) + 1) : 0;
    p.scale2 = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.dim)) * 1.44269504f;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = a.dtype == TBS_F32 ? attend_run<float>(p, st) : a.dtype == TBS_BF16 ? attend_run<__bf16>(p, st) : attend_run<_Float16>(p, st);
    return e == hipSuccess ? TBS_OK : TBS_EHIP;
}
