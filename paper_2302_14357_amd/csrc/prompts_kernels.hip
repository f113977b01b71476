// Causal attention of packed prompts: new tokens side by side, what came before them in a paged cache.
//
// With t = log2(e) scale q.k and a reference m near the largest t seen, o = sum 2^(t - m) v and l = sum 2^(t - m) are kept in float32 registers while the keys
// pass once, 32 or 64 at a time; where a tile's largest t is above m by more than PROMPTS_SLACK, m becomes it and o and l are multiplied by
// 2^(m_old - m).  (Below that a weight is at most 2^8: float32 and bfloat16 hold it as well as 1, and most tiles then multiply nothing.)
//
// The rows of a prompt and key head are its tokens' queries of that head's group, token after token: one product for all of a group's heads, and
// few rows per key on the diagonal.  A wave has 32 of them as the columns of the matrix instructions:
//  - scores: S^T = K Q^T, keys the rows, so that a lane has 16 of 32 keys' scores of one query, the other half's lane the others;
//  - output: O^T = V^T P^T.  The order of the keys in the sum is free, so the weights go into the instruction as the scores' came out; V's fragments
//    come from LDS by the reads that transpose 4 x 16 blocks, from the rows that this order names.
// Keys and values of a tile go to LDS by direct loads, the next tile's while this one is worked on.  Pieces of 16 bytes of a row are permuted by bits
// of the row, so that a fragment's reads are all LDS banks once.
//
// Weights are rounded to the 16 bits of the values' type: a weight's relative error is half a step of it, as large as the output's own rounding; two
// numbers a weight would cost half as many matrix instructions again.  Sums, statistics and the weights' sum are float32.
#include "op_device.h"

#define PROMPTS_SLACK 8.f
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short prompts_b64;

struct PromptsP {
    const char *q, *k, *v, *k_cache, *v_cache;
    const int *starts, *past, *tables;
    char *out;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, kp, kt, kh, vp, vt, vh, ld_tables;   // bytes (ld_tables: elements)
    int tokens, prompts, heads, kv_heads, group, dim, page, pages, width;
    bool direct;    // everything on 16-byte boundaries
    float scale2;   // |scale| log2(e)
    unsigned flip;  // sign bits of a word of queries where the scale is negative
};

struct PromptsAt {
    int start, n, past;   // of a prompt: its first token's row, its tokens, those in the cache
};

__device__ __forceinline__ int prompts_start(const PromptsP &p, int i) { return min(max(p.starts[i], 0), p.tokens); }
// its tokens: starts may be any numbers, and each is brought into the batch before they are subtracted
__device__ __forceinline__ int prompts_length(const PromptsP &p, int i) { return max(prompts_start(p, i + 1) - prompts_start(p, i), 0); }

__device__ __forceinline__ PromptsAt prompts_at(const PromptsP &p, int i) {
    PromptsAt x;
    x.start = prompts_start(p, i);
    x.n = prompts_length(p, i);
    x.past = p.past ? (int)min((int64_t)max(p.past[i], 0), (int64_t)p.width * p.page) : 0;
    return x;
}

// The tile `unit` of `rows` rows among all prompts' tiles, by every wave for itself: its prompt and its number in the prompt, a prompt's last first
// (they have the most keys); prompt -1 for one behind all of them, and then the number of tiles.
__device__ __forceinline__ int2 prompts_find(const PromptsP &p, int unit, int rows) {
    const int lane = threadIdx.x & 63;
    auto tiles = [&](int i) { return (prompts_length(p, i) * p.group + rows - 1) / rows; };   // (below 2^31: tokens x heads is)
    int from = 0, count = p.prompts;
    int64_t before = 0;   // (starts in no order may give any sum)
    for (;;) {
        const int each = (count + 63) / 64;   // prompts a lane
        int64_t mine = 0;
        for (int i = lane * each; i < min((lane + 1) * each, count); ++i) mine += tiles(from + i);
        int64_t end = mine;
#pragma unroll
        for (int i = 1; i < 64; i <<= 1) {
            const int64_t y = __shfl_up(end, i);
            if (lane >= i) end += y;
        }
        end += before;
        const unsigned long long has = __ballot(end > unit);
        if (!has) return make_int2(-1, (int)__shfl(end, 63));   // (at most `unit`)
        const int l = __ffsll((long long)has) - 1;
        const int64_t all = __shfl(mine, l);
        before = __shfl(end, l) - all;
        if (each == 1) return make_int2(from + l, (int)(all - 1 - (unit - before)));
        from += l * each;
        count = min(each, count - l * each);
    }
}

template <class T, int DP>
struct PromptsTile {
    static constexpr int E = OpPiece<T>::E, KEYS = sizeof(T) == 4 || DP > 128 ? 32 : 64;
    static constexpr int USED = DP / E;                                       // pieces of a row
    static constexpr int PITCH = USED <= 4 ? 4 : USED <= 8 ? 8 : USED <= 16 ? 16 : USED <= 32 ? 32 : 64;   // ... in LDS
    static constexpr int BYTES = KEYS * PITCH * 16;                           // of keys, or values
    // Keys: 32 rows' pieces of one place.  Values: four rows' two or four pieces side by side (float32: a row's eight, and those of the row four behind).
    static __device__ __forceinline__ int k_swizzle(int row) { return PITCH >= 16 ? row & 15 : PITCH == 8 ? row >> 1 & 7 : row >> 2 & 3; }
    static __device__ __forceinline__ int v_swizzle(int row) {
        if (sizeof(T) == 4) return PITCH >= 16 ? (row >> 2 & 1) << 3 : 0;
        return PITCH >= 16 ? (row & 2) << 2 | (row & 1) << 2 | (row & 2) : PITCH == 8 ? (row & 2) << 1 | (row & 1) << 1 : row & 2;
    }
};

// DP: dim rounded up to 32, 64, 96, 128 or 256; NW: waves of 32 rows each
template <class T, int DP, int NW>
__global__ void __launch_bounds__(64 * NW, DP > 128 || sizeof(T) == 4 ? 1 : 2)
k_prompts(PromptsP p) {
    typedef PromptsTile<T, DP> Tile;
    constexpr int E = Tile::E, TK = Tile::KEYS, PITCH = Tile::PITCH, KB = TK / 32, DB = DP / 32, KS = DP * (int)sizeof(T) / 32, ROWS = 32 * NW;
    constexpr int CHUNKS = TK * PITCH / 64, MINE = (CHUNKS + NW - 1) / NW;   // loads of 64 pieces, and those of a wave
    constexpr int VS = sizeof(T) == 4 ? 1 : DB;   // addresses of V
    __shared__ __align__(16) char s_kv[2][2][Tile::BYTES];
    __shared__ unsigned long long s_there[2];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
    const int kvh = (int)blockIdx.x % p.kv_heads, unit = (int)blockIdx.x / p.kv_heads;
    const int2 found = prompts_find(p, unit, ROWS);
    if (found.x < 0) {   // rows of no prompt are 0: those before the first and behind the last, shared among the workgroups without a tile
        const int first = p.prompts > 0 ? prompts_start(p, 0) : p.tokens, last = p.prompts > 0 ? max(prompts_start(p, p.prompts), first) : p.tokens;
        const int spare = (int)gridDim.x / p.kv_heads - found.y, rows = first + p.tokens - last;
        for (int i = unit - found.y; i < rows; i += spare) {
            T *to = (T *)(p.out + (i < first ? i : last + i - first) * p.o_row + kvh * p.group * p.o_head);
            for (int j = threadIdx.x; j < p.group * p.dim; j += 64 * NW) {
                const int head = j / p.dim;
                *(T *)((char *)to + head * p.o_head + (j - head * p.dim) * sizeof(T)) = (T)0.f;
            }
        }
        return;
    }
    const PromptsAt at = prompts_at(p, found.x);
    const int *table = p.past ? p.tables + found.x * p.ld_tables : nullptr;
    const int rows = at.n * p.group, row0 = found.y * ROWS;   // (below 2^31: tokens x heads is)
    const int keys = at.past + (min(row0 + ROWS, rows) - 1) / p.group + 1, steps = (keys + TK - 1) / TK;
    // this lane's query, and the last key that it sees; the first and last of the wave's
    const int row = row0 + wave * 32 + c, token = row / p.group, head = kvh * p.group + row - token * p.group;
    const bool live = row < rows;
    const int sees = live ? at.past + token : -1;
    const int w0 = row0 + wave * 32, wave_first = w0 + 32 <= rows ? at.past + w0 / p.group : -1, wave_last = w0 < rows ? at.past + (min(w0 + 32, rows) - 1) / p.group : -1;
    uint4 q[KS];
    {
        const T *src = (const T *)(p.q + (int64_t)(at.start + (live ? token : 0)) * p.q_row + (live ? head : 0) * p.q_head);
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            q[s] = live && (s * 2 + h) * E < p.dim ? op_load16(src + (s * 2 + h) * E) : make_uint4(0, 0, 0, 0);
            q[s].x ^= p.flip, q[s].y ^= p.flip, q[s].z ^= p.flip, q[s].w ^= p.flip;
        }
    }

    // ---- tiles into LDS
    const char *k_new = p.k + (int64_t)at.start * p.k_row + kvh * p.k_head, *v_new = p.v + (int64_t)at.start * p.v_row + kvh * p.v_head;
    const char *k_old = p.k_cache + kvh * p.kh, *v_old = p.v_cache + kvh * p.vh;
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)&s_kv[0][0][0];
    int id[MINE], id_mask = 0;   // the pages of this lane's keys in the tile to be asked for next, and of key `lane` of it
    auto page_of = [&](int t) { return t < at.past ? table[(unsigned)t / (unsigned)p.page] : 0; };
    auto row_of = [&](int i) { return ((wave + i * NW) * 64 + lane) / PITCH; };
    auto look = [&](int step) {
        if (step * TK >= at.past) return;
#pragma unroll
        for (int i = 0; i < MINE; ++i) id[i] = page_of(step * TK + row_of(i));
        if (wave == 0) id_mask = page_of(step * TK + (lane & (TK - 1)));
    };
    auto ask = [&](int step) {
        const int t0 = step * TK, buffer = step & 1;
        const bool old = t0 < at.past;
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int chunk = wave + i * NW;
            if (CHUNKS % NW && chunk >= CHUNKS) continue;
            const int r = row_of(i), slot = (chunk * 64 + lane) % PITCH;
            const int t = min(t0 + r, keys - 1);   // (behind the last: anything that is there)
            const char *k = k_new + (int64_t)(t - at.past) * p.k_row, *v = v_new + (int64_t)(t - at.past) * p.v_row;
            if (old && t < at.past) {
                const unsigned page = (unsigned)t / (unsigned)p.page, off = (unsigned)t - page * (unsigned)p.page;
                const int n = (unsigned)id[i] < (unsigned)p.pages ? id[i] : 0;   // (a page that does not exist: the first's, masked)
                k = k_old + n * p.kp + off * p.kt;
                v = v_old + n * p.vp + off * p.vt;
            }
            const int ks = slot ^ Tile::k_swizzle(r), vs = slot ^ Tile::v_swizzle(r);
            const unsigned to = lds + buffer * 2 * Tile::BYTES + chunk * 1024;
            if (p.direct) {
                if (ks * E < p.dim) op_load_lds(k + ks * 16, to);
                if (vs * E < p.dim) op_load_lds(v + vs * 16, to + Tile::BYTES);
            } else {
                if (ks * E < p.dim) *(uint4 *)(&s_kv[buffer][0][0] + chunk * 1024 + lane * 16) = op_load16((const T *)k + ks * E);
                if (vs * E < p.dim) *(uint4 *)(&s_kv[buffer][1][0] + chunk * 1024 + lane * 16) = op_load16((const T *)v + vs * E);
            }
        }
        if (old && wave == 0) {
            const int t = t0 + lane;
            const unsigned long long there = __ballot(lane < TK && (t >= at.past || (unsigned)id_mask < (unsigned)p.pages));
            if (lane == 0) s_there[buffer] = there;
        }
    };
    // pieces behind the head's end are 0 in both buffers, and stay so
    if (p.dim < PITCH * E) {
        for (int i = threadIdx.x; i < 4 * TK * PITCH; i += 64 * NW) {
            const int in = i % (TK * PITCH), r = in / PITCH, slot = in % PITCH;
            if ((slot ^ ((i / (TK * PITCH)) & 1 ? Tile::v_swizzle(r) : Tile::k_swizzle(r))) * E >= p.dim) ((uint4 *)&s_kv[0][0][0])[i] = make_uint4(0, 0, 0, 0);
        }
    }
    look(0);
    ask(0);
    look(1);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");

    // ---- fragments: where this lane's begin
    int k_at[KS], v_at[VS];
#pragma unroll
    for (int s = 0; s < KS; ++s) k_at[s] = (c * PITCH + ((s * 2 + h) ^ Tile::k_swizzle(c))) * 16;
    const int v_row = sizeof(T) == 4 ? 4 * h : 4 * h + (lane >> 2 & 3);
#pragma unroll
    for (int d = 0; d < VS; ++d)
        v_at[d] = sizeof(T) == 4 ? v_row * PITCH * 16 : (v_row * PITCH + ((d * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ Tile::v_swizzle(v_row))) * 16 + (lane & 1) * 8;
    // V^T of 16 keys from `key` on (in the order of the weights) and the d-th 32 dimensions
    auto v_frag = [&](int buffer, int key, int d) {
        uint4 u;
        typedef __attribute__((address_space(3))) prompts_b64 *Lds;
        const unsigned from = lds + (buffer * 2 + 1) * Tile::BYTES + v_at[d] + key * PITCH * 16;
        const prompts_b64 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)from), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(uintptr_t)(from + 8 * PITCH * 16));
        __builtin_memcpy(&u, &x, 8);
        __builtin_memcpy((char *)&u + 8, &y, 8);
        return u;
    };
    auto v_one = [&](int buffer, int key, int d) {   // float32: dimension 32 d + c of key `key` + 4 h
        return *(const float *)(&s_kv[buffer][1][0] + v_at[0] + key * PITCH * 16 + (((d * 8 + c / 4) ^ (PITCH >= 16 ? h << 3 : 0)) * 16 + c % 4 * 4));
    };

    floatx16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float m = -INFINITY, l = 0.f;
    // (float16: weights up to 2^7 more, so that small ones keep their digits: with the slack's 2^8 at most half its largest number)
    constexpr float MORE = __is_same(T, _Float16) ? 7.f : 0.f;

    for (int step = 0; step < steps; ++step) {
        const int t0 = step * TK, buffer = step & 1;
        if (step + 1 < steps) {
            ask(step + 1);
            look(step + 2);
        }
        if (t0 <= wave_last) {
            unsigned long long there = keys - t0 >= TK ? (TK == 64 ? ~0ull : (1ull << (TK & 63)) - 1) : (1ull << (keys - t0)) - 1;
            const unsigned long long whole = TK == 64 ? ~0ull : (1ull << (TK & 63)) - 1;
            if (t0 < at.past) there &= s_there[buffer];
            there = (unsigned long long)__builtin_amdgcn_readfirstlane((int)(there >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)there);
            const bool mixed = there != whole || t0 + TK - 1 > wave_first;   // some key is not some query's
            floatx16 s[KB];
#pragma unroll
            for (int b = 0; b < KB; ++b) {
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = 0.f;
#pragma unroll
                for (int j = 0; j < KS; ++j) s[b] = op_mma32<T>(*(const uint4 *)(&s_kv[buffer][0][0] + k_at[j] + b * 32 * PITCH * 16), q[j], s[b]);
            }
            unsigned long long mine = ~0ull;   // this lane's query's keys of the tile
            if (mixed) {
                const int last = sees - t0;   // (its last key's place)
                mine = last < 0 ? 0 : last >= 63 ? there : there & ((2ull << last) - 1);
                const unsigned long long bits = mine >> (4 * h);
#pragma unroll
                for (int b = 0; b < KB; ++b)
#pragma unroll
                    for (int i = 0; i < 16; ++i) s[b][i] = bits >> (32 * b + 8 * (i / 4) + i % 4) & 1 ? s[b][i] : -INFINITY;
            }
            float top = s[0][0];
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
            {
                typedef unsigned uint2_ __attribute__((ext_vector_type(2)));
                const uint2_ u = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);
                top = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1])) * p.scale2;
            }
            if (__any(top > m + PROMPTS_SLACK)) {
                const float m1 = fmaxf(m, top), a = m1 == m ? 1.f : __builtin_amdgcn_exp2f(m - m1);
                m = m1;
                l *= a;
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] *= a;
            }
            const float base = m == -INFINITY ? 0.f : m - MORE;
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    s[b][i] = __builtin_amdgcn_exp2f(fmaf(s[b][i], p.scale2, -base));
                    l += s[b][i];
                }
            // A value that is NaN or infinite would reach, times the weight 0, the queries that do not see it.  Where some do not, such a tile's keys are
            // added one by one to those that do.
            bool odd = false;
            if constexpr (sizeof(T) == 4) {
                if (mixed) {
                    floatx16 z = {};
#pragma unroll
                    for (int key = 0; key < TK; key += 8)
#pragma unroll
                        for (int r = 0; r < 4; ++r)
#pragma unroll
                            for (int d = 0; d < DB; ++d) z = __builtin_amdgcn_mfma_f32_32x32x2f32(v_one(buffer, key + r, d), 0.f, z, 0, 0, 0);
                    bool none = false;
#pragma unroll
                    for (int i = 0; i < 16; ++i) none |= z[i] != 0.f;
                    odd = __any(none);
                }
                if (!odd) {
#pragma unroll
                    for (int i = 0; i < 16; ++i)
#pragma unroll
                        for (int d = 0; d < DB; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_one(buffer, 8 * (i / 4) + i % 4, d), s[0][i], o[d], 0, 0, 0);
                } else {
                    for (int key = 0; key < TK; ++key) {
                        const bool seen = mine >> key & 1;
                        if (!__any(seen)) continue;
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (8 * (i / 4) + i % 4 != (key & ~4)) continue;
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                const float x = v_one(buffer, key & ~4, d);
                                floatx16 z = {};
                                z = __builtin_amdgcn_mfma_f32_32x32x2f32(h == (key >> 2 & 1) ? x : 0.f, h == (key >> 2 & 1) && seen ? s[0][i] : 0.f, z, 0, 0, 0);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[d][j] = seen ? o[d][j] + z[j] : o[d][j];
                            }
                        }
                    }
                }
            } else {
                uint4 w[TK / 16];
#pragma unroll
                for (int i = 0; i < TK / 16; ++i) {
                    T x[8];
#pragma unroll
                    for (int j = 0; j < 8; ++j) x[j] = (T)s[i / 2][i % 2 * 8 + j];
                    __builtin_memcpy(&w[i], x, 16);
                }
                if (mixed) {
                    floatx16 z = {};
#pragma unroll
                    for (int i = 0; i < TK / 16; ++i)
#pragma unroll
                        for (int d = 0; d < DB; ++d) z = op_mma32<T>(v_frag(buffer, i * 16, d), make_uint4(0, 0, 0, 0), z);
                    bool none = false;
#pragma unroll
                    for (int i = 0; i < 16; ++i) none |= z[i] != 0.f;
                    odd = __any(none);
                }
                if (!odd) {
#pragma unroll
                    for (int i = 0; i < TK / 16; ++i)
#pragma unroll
                        for (int d = 0; d < DB; ++d) o[d] = op_mma32<T>(v_frag(buffer, i * 16, d), w[i], o[d]);
                } else {
                    for (int key = 0; key < TK; ++key) {
                        const bool seen = mine >> key & 1;
                        if (!__any(seen)) continue;
                        // its place in the fragments: half and element
                        const int half = key >> 2 & 1, e = (key >> 3 & 1) * 4 + (key & 3);
                        const unsigned keep = h == half ? (e & 1 ? 0xffff0000u : 0xffffu) : 0;
#pragma unroll
                        for (int i = 0; i < TK / 16; ++i) {
                            if (i != key >> 4) continue;
#pragma unroll
                            for (int d = 0; d < DB; ++d) {
                                uint4 x = v_frag(buffer, i * 16, d);
                                x.x &= e / 2 == 0 ? keep : 0, x.y &= e / 2 == 1 ? keep : 0, x.z &= e / 2 == 2 ? keep : 0, x.w &= e / 2 == 3 ? keep : 0;
                                floatx16 z = {};
                                z = op_mma32<T>(x, w[i], z);
#pragma unroll
                                for (int j = 0; j < 16; ++j) o[d][j] = seen ? o[d][j] + z[j] : o[d][j];
                            }
                        }
                    }
                }
            }
        }
        if (step + 1 < steps) {   // the next tile is there, and everybody has read this one
            asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        }
    }

    l += __shfl_xor(l, 32);
    const float f = l == 0.f ? 0.f : 1.f / l;   // (no weight at all: 0)
    if (!live) return;
    char *to = p.out + (int64_t)(at.start + token) * p.o_row + head * p.o_head;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int e = d * 32 + b * 8 + h * 4;   // (dim is a multiple of 8)
            if (e >= p.dim) continue;
            T y[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) y[i] = (T)(l == 0.f ? 0.f : o[d][b * 4 + i] * f);
            __builtin_memcpy((T *)to + e, y, sizeof y);
        }
}

static int64_t prompts_units(const tbs_attend_prompts_args &a, int rows) { return (int64_t)a.tokens * (a.heads / a.kv_heads) / rows + a.prompts + 1; }

template <class T, int DP>
static hipError_t prompts_waves(const PromptsP &p, const tbs_attend_prompts_args &a, hipStream_t st) {
    constexpr int MOST = DP > 128 || sizeof(T) == 4 ? 4 : 8;
    int waves = MOST;
    while (waves > 2 && prompts_units(a, 32 * waves) * a.kv_heads < 512) waves /= 2;
    const int64_t blocks = prompts_units(a, 32 * waves) * a.kv_heads;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(64 * waves);
    if (waves == 2) hipLaunchKernelGGL((k_prompts<T, DP, 2>), grid, block, 0, st, p);
    else if (waves == 4) hipLaunchKernelGGL((k_prompts<T, DP, 4>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_prompts<T, DP, MOST>), grid, block, 0, st, p);
    return hipGetLastError();
}

template <class T>
static hipError_t prompts_dims(const PromptsP &p, const tbs_attend_prompts_args &a, hipStream_t st) {
    if (p.dim <= 32) return prompts_waves<T, 32>(p, a, st);
    if (p.dim <= 64) return prompts_waves<T, 64>(p, a, st);
    if (p.dim <= 96) return prompts_waves<T, 96>(p, a, st);
    if (p.dim <= 128) return prompts_waves<T, 128>(p, a, st);
    return prompts_waves<T, 256>(p, a, st);
}

static int prompts_check(const tbs_attend_prompts_args &a) {
    if (!op_dtype_known(a.dtype) || a.tokens < 0 || a.prompts < 0 || a.kv_heads < 1 || a.heads < a.kv_heads || a.heads % a.kv_heads || a.heads > 65535 || a.dim < 8 ||
        a.dim > 256 || a.dim % 8 || a.tokens > (1 << 30) || (int64_t)a.tokens * a.heads > INT32_MAX - 65536)
        return TBS_EINVAL;
    if (a.past && (a.page < 1 || a.page > 65536 || a.pages < 1 || a.table_width < 1 || (int64_t)a.table_width * a.page + a.tokens > (1 << 30))) return TBS_EINVAL;
    return TBS_OK;
}

extern "C" int64_t tbs_attend_prompts_workspace(const tbs_attend_prompts_args *args) {
    if (!args || prompts_check(*args) != TBS_OK) return TBS_EINVAL;
    return 0;
}

extern "C" int tbs_attend_prompts(const tbs_attend_prompts_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_attend_prompts_args &a = *args;
    if (prompts_check(a) != TBS_OK) return TBS_EINVAL;
    if (a.past ? !a.k_cache || !a.v_cache || !a.tables || a.ld_tables < a.table_width : a.k_cache || a.v_cache || a.tables) return TBS_EINVAL;
    if (a.tokens == 0) return TBS_OK;
    if (!a.q || !a.k || !a.v || !a.starts || !a.out) return TBS_EINVAL;
    const int64_t es = (int64_t)op_dtype_size(a.dtype);
    const int64_t strides[] = {a.q_row, a.q_head, a.k_row, a.k_head, a.v_row, a.v_head, a.out_row, a.out_head,
                               a.k_cache_page, a.k_cache_token, a.k_cache_head, a.v_cache_page, a.v_cache_token, a.v_cache_head};
    bool direct = true;
    for (int64_t s : strides) {
        if (s < 0 || s > INT64_MAX / 64 / INT32_MAX) return TBS_EINVAL;
        direct &= s * es % 16 == 0;
    }
    const void *ptrs[] = {a.q, a.k, a.v, a.k_cache, a.v_cache, a.out};
    for (const void *x : ptrs) {
        if ((uintptr_t)x % es) return TBS_EINVAL;
        direct &= (uintptr_t)x % 16 == 0;
    }
    // what is written lies neither over itself nor over what others read; queries are read by those who write in their place
    const OpHeads q = {a.q, a.tokens, a.heads, a.dim, a.q_row, a.q_head}, out = {a.out, a.tokens, a.heads, a.dim, a.out_row, a.out_head};
    if (op_folded(out) || (!op_same(q, out) && op_overlap(out, q, es)) || op_overlap(out, {a.k, a.tokens, a.kv_heads, a.dim, a.k_row, a.k_head}, es) ||
        op_overlap(out, {a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head}, es))
        return TBS_EINVAL;
    PromptsP p = {};
    p.q = (const char *)a.q, p.k = (const char *)a.k, p.v = (const char *)a.v, p.k_cache = (const char *)a.k_cache, p.v_cache = (const char *)a.v_cache, p.out = (char *)a.out;
    p.starts = a.starts, p.past = a.past, p.tables = a.tables;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.k_row = a.k_row * es, p.k_head = a.k_head * es, p.v_row = a.v_row * es, p.v_head = a.v_head * es;
    p.o_row = a.out_row * es, p.o_head = a.out_head * es;
    p.kp = a.k_cache_page * es, p.kt = a.k_cache_token * es, p.kh = a.k_cache_head * es, p.vp = a.v_cache_page * es, p.vt = a.v_cache_token * es, p.vh = a.v_cache_head * es;
    p.ld_tables = a.ld_tables;
    p.tokens = a.tokens, p.prompts = a.prompts, p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = a.heads / a.kv_heads, p.dim = a.dim;
    p.page = a.past ? a.page : 1, p.pages = a.pages, p.width = a.table_width;
    p.direct = direct;
    const float scale = a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.dim);
    p.scale2 = fabsf(scale) * 1.44269504f;
    p.flip = scale < 0.f ? (a.dtype == TBS_F32 ? 0x80000000u : 0x80008000u) : 0;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = a.dtype == TBS_F32 ? prompts_dims<float>(p, a, st) : a.dtype == TBS_BF16 ? prompts_dims<__bf16>(p, a, st) : prompts_dims<_Float16>(p, a, st);
    return e == hipSuccess ? TBS_OK : e == hipErrorInvalidValue ? TBS_EINVAL : TBS_EHIP;
}
