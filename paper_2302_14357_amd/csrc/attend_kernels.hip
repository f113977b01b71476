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

//
// Hypotheses of one utterance (beams) name the same pages for most of their length.  A workgroup then takes a key head and a piece of the
// length for all of them: the pages at the piece's head that their tables have in common are read once, with all hypotheses' queries as
// columns, and behind those each hypothesis' own tokens, which count for its columns alone.
#define ATT_TABLE 1024   // page table entries in LDS at a time, of all hypotheses of a workgroup

struct AttendP {
    const char *q, *k_new, *v_new;
    char *k_cache, *v_cache;
    const int *tables, *lens;
    char *out;
    float *part_o, *part_ml;   // [rows, heads, splits, dim], [rows, heads, splits, 2]; only with more than one split
    int64_t q_row, q_head, kn_row, kn_head, vn_row, vn_head, o_row, o_head, kh, vh, ld_tables;   // bytes (ld_tables: elements)
    unsigned kp, kt, vp, vt;
    int rows, heads, kv_heads, group, dim, page, pages, width, splits, split_len, qblocks, beams;
    unsigned page_mul, page_shift;
    float scale2;   // scale * log2(e)
};

// t / page = 2 t / (2 page) for 0 <= t <= 2^30, by multiplication: page_mul = floor(2^(32 + s) / (2 page)) + 1 with s = floor(log2 (2 page)) is at most
// 2^(s + 1) / 2^(32 + s) of a unit too large for numerators below 2^31 (powers of two: 2^32 / (2 page), which is exact)
__device__ __forceinline__ int att_page(const AttendP &p, int t) { return (int)(__umulhi((unsigned)t << 1, p.page_mul) >> p.page_shift); }

// the larger of a lane's number and those 16 and 32 lanes away (rows of 16 lanes, and halves, change places)
__device__ __forceinline__ float att_max4(float x) {
    typedef unsigned uint2_ __attribute__((ext_vector_type(2)));
    uint2_ u = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
    u = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    return fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1]));
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

// two numbers cut to the first bits that their 16-bit type holds (none of them is above its largest)
__device__ __forceinline__ void att_first_bits(float a, float b, __bf16 *to) {
    const unsigned u = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
    __builtin_memcpy(to, &u, 4);
}
__device__ __forceinline__ void att_first_bits(float a, float b, _Float16 *to) {
    const auto u = __builtin_amdgcn_cvt_pkrtz(a, b);
    __builtin_memcpy(to, &u, 4);
}
// what weights are made larger by: enough for 16 bits to hold the excess (fp16: of weights from 2^-26 of the row's largest on)
template <class T>
struct AttMore {
    static constexpr float F = sizeof(T) == 4 ? 1.f : __is_same(T, __bf16) ? 1.f + 0x1p-16f : 1.f + 0x1p-11f;
};

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

// DP: dim rounded up to 32, 64, 128 or 256 (PAD: it was not that already); QB: blocks of sixteen queries a wave takes together;
// NW: waves, of which four write the outputs; GROUP: hypotheses together, otherwise row by row
template <class T, int DP, int QB, bool PAD, int NW, bool GROUP>
__global__ void __launch_bounds__(64 * NW, 2)
k_attend(AttendP p) {
    typedef AttTile<T, DP> Tile;
    constexpr int E = OpPiece<T>::E, NB = Tile::NB, TK = Tile::TK, NV = Tile::NV, KS = Tile::KS, W = Tile::W, WW = Tile::WW;
    constexpr bool LATE = DP > 128;   // (registers for keys and values at the same time are missing: values are asked for when the scores are made)
    __shared__ int s_table[ATT_TABLE + TBS_MAX_BEAM];
    __shared__ float s_o[NW][4][W][64];
    __shared__ float s_ml[NW][2][QB * 16];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int c = lane & 15, kg = lane >> 4;
    const int kvh = (int)blockIdx.x % p.kv_heads, qblk = (int)blockIdx.x / p.kv_heads, split = p.splits - 1 - (int)blockIdx.z, N = GROUP ? p.beams : 1, r0 = (int)blockIdx.y * N;   // (a row's end takes longest: first)
    // hypothesis `lane` of the group: its tokens, and those of them that are in the cache
    int n_l = 0, pos_l = -1;
    if (lane < N) n_l = att_tokens(p, r0 + lane, &pos_l);
    int n = n_l, cached = lane < N && n_l > 0 ? (pos_l >= 0 ? pos_l : n_l) : INT32_MAX;
    if (N > 1)
#pragma unroll
        for (int i = 1; i < 32; i <<= 1) {
            n = max(n, __shfl_xor(n, i));
            cached = min(cached, __shfl_xor(cached, i));
        }
    n = __builtin_amdgcn_readfirstlane(n);   // of the longest
    cached = __builtin_amdgcn_readfirstlane(cached);   // of the shortest that takes part
    const unsigned live = (unsigned)__ballot(n_l > 0);
    const int k0 = split * p.split_len;
    if (k0 >= n && split > 0) return;   // (of a group without tokens the first workgroup writes the zeros)
    const int k1 = split == p.splits - 1 ? n : min(n, k0 + p.split_len);   // (the last goes on to the end, whatever max_len said)
    const char *kb = p.k_cache + kvh * p.kh, *vb = p.v_cache + kvh * p.vh;
    const bool quad = (p.page & 3) == 0;   // four tokens from a multiple of four on lie in one page

    int col_row[QB], col_head[QB];   // whose query a lane's column is
    bool col_live[QB];
    uint4 q[QB][KS];
    floatx4 o[QB][W];
    float m[QB], l[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int col = (qblk * QB + b) * 16 + c;
        col_row[b] = col / p.group;
        col_head[b] = kvh * p.group + col - col_row[b] * p.group;
        const bool there = col_row[b] < N;
        col_live[b] = there && (live >> col_row[b] & 1);
        const T *src = (const T *)(p.q + (r0 + min(col_row[b], N - 1)) * p.q_row + col_head[b] * p.q_head);
#pragma unroll
        for (int s = 0; s < KS; ++s) q[b][s] = there && (!PAD || (s * 4 + kg) * E < p.dim) ? op_load16(src + (s * 4 + kg) * E) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < W; ++i) o[b][i] = floatx4{0.f, 0.f, 0.f, 0.f};
        m[b] = -INFINITY;
        l[b] = 0.f;
    }

    const int per_row = ATT_TABLE / N, chunk = per_row * p.page;   // table entries of a hypothesis at a time, their tokens
    for (int c0 = k0; c0 < k1; c0 += chunk) {
        const int first = att_page(p, c0), c1 = min(k1, c0 + chunk), pages = att_page(p, c1 - 1) - first + 1;
        if (c0 > k0) __syncthreads();
        for (int b = wave; b < N; b += NW) {
            const int mine = __shfl(n_l, b), have = mine > 0 ? att_page(p, mine - 1) - first + 1 : 0;
            for (int i = lane; i < pages; i += 64) {
                const int id = p.tables[(r0 + b) * p.ld_tables + first + i];   // (in the table: i < width)
                s_table[b * (per_row + 1) + i] = i < have && (unsigned)id < (unsigned)p.pages ? id : -1;   // (negative: its tokens do not exist)
            }
        }
        __syncthreads();
        // tokens up to `common` are everybody's: pages of the same numbers, whole, in the cache of all
        int common = c0;
        const int lead = __ffs(live) - 1;
        if (N > 1) {
            int same = 0;
            for (int i0 = 0; i0 < pages; i0 += 64) {
                const int i = i0 + lane;
                bool differ = i >= pages;
                for (unsigned rest = live & (live - 1); rest; rest &= rest - 1)
                    differ |= i < pages && s_table[lead * (per_row + 1) + i] != s_table[(__ffs(rest) - 1) * (per_row + 1) + i];
                const unsigned long long d = __ballot(differ);
                same += d ? __ffsll((long long)d) - 1 : 64;
                if (d) break;
            }
            common = max(c0, min((int)min((int64_t)c1, (int64_t)(first + same) * p.page), att_page(p, min(cached, c1)) * p.page));
        }
        // tiles: those of the common tokens, then each hypothesis' own
        const int shared = (common - c0 + TK - 1) / TK, end_l = min(n_l, c1), own = end_l > common ? (end_l - common + TK - 1) / TK : 0;
        int start = own;
        if (N > 1)
#pragma unroll
            for (int i = 1; i < 32; i <<= 1) {
                const int x = __shfl_up(start, i);
                if (lane >= i) start += x;
            }
        const int tiles = shared + __builtin_amdgcn_readlane(start, N - 1);
        start += shared - own;
        struct Where {
            int t0, end, row, b;   // row: whose it is (-1: everybody's, by the table of hypothesis b)
        };
        auto place = [&](int tile) {
            Where w = {c0 + tile * TK, common, -1, lead};
            if (tile >= shared) {
                w.row = w.b = 31 - __clz((unsigned)__ballot(lane < N && own > 0 && start <= tile));
                w.t0 = common + (tile - __builtin_amdgcn_readlane(start, w.b)) * TK;
                w.end = __builtin_amdgcn_readlane(end_l, w.b);
            }
            return w;
        };
        // A token's address in the cache; one whose page does not exist has the first page's.  No branch in here: the loads of a tile have to
        // leave together.
        auto address = [&](const char *base, unsigned page_bytes, unsigned token_bytes, const Where &w, int t, bool &there) {
            const int i = att_page(p, t), id = s_table[w.b * (per_row + 1) + i - first];
            there = id >= 0;
            return base + (uint64_t)(unsigned)max(id, 0) * page_bytes + (unsigned)(t - i * p.page) * token_bytes;
        };
        auto take_k = [&](Tile &x, int b, const char *at) {
#pragma unroll
            for (int s = 0; s < KS; ++s) x.k[b][s] = !PAD || (s * 4 + kg) * E < p.dim ? op_load16((const T *)at + (s * 4 + kg) * E) : make_uint4(0, 0, 0, 0);
        };
        auto take_v = [&](Tile &x, int j, const char *at) {
            constexpr int G = W < 8 ? W : 8, GW = G * (int)sizeof(T) / 4;   // elements that are there together or not at all: dim is a multiple of 8
#pragma unroll
            for (int g = 0; g < W / G; ++g) {
                AttWords<GW> u = {};
                if (!PAD || c * W + g * G < p.dim) __builtin_memcpy(&u, (const T *)at + c * W + g * G, sizeof u);
#pragma unroll
                for (int i = 0; i < GW; ++i) x.v[j][g * GW + i] = u.w[i];
            }
        };
        // whole tiles of tokens in the cache, pages of a multiple of four tokens: a lane's four tokens of V lie in one page
        auto plain = [&](const Where &w) { return quad && w.t0 + TK + (w.row >= 0 ? 1 : 0) <= w.end; };   // (the new token is its row's last)
        auto load_k = [&](Tile &x, const Where &w) {
            bool there;
            if (plain(w)) {
#pragma unroll
                for (int b = 0; b < NB; ++b) take_k(x, b, address(kb, p.kp, p.kt, w, w.t0 + b * 16 + c, there));
            } else {
                const int pos = w.row >= 0 ? __builtin_amdgcn_readlane(pos_l, w.b) : -1;
                const char *kn = p.k_new + (r0 + w.b) * p.kn_row + kvh * p.kn_head;
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const int t = min(w.t0 + b * 16 + c, w.end - 1);
                    const char *at = address(kb, p.kp, p.kt, w, t, there);
                    take_k(x, b, t == pos ? kn : at);
                }
            }
        };
        auto load_v = [&](Tile &x, const Where &w) {
            bool there;
            x.ok = 0;
            if (plain(w)) {
#pragma unroll
                for (int b = 0; b < NB; ++b) {
                    const char *at = address(vb, p.vp, p.vt, w, w.t0 + b * 16 + kg * 4, there);
                    x.ok |= there ? 15u << (b * 4) : 0;
#pragma unroll
                    for (int r = 0; r < 4; ++r) take_v(x, b * 4 + r, at + (uint64_t)r * p.vt);
                }
            } else {
                const int pos = w.row >= 0 ? __builtin_amdgcn_readlane(pos_l, w.b) : -1;
                const char *vn = p.v_new + (r0 + w.b) * p.vn_row + kvh * p.vn_head;
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    const int want = w.t0 + (j / 4) * 16 + kg * 4 + j % 4, t = min(want, w.end - 1);
                    const char *at = address(vb, p.vp, p.vt, w, t, there);
                    x.ok |= want < w.end && (there || t == pos) ? 1u << j : 0;
                    take_v(x, j, t == pos ? vn : at);
                }
            }
        };
        auto compute = [&](Tile &x, const Where &w) {
            floatx4 s[QB][NB];
#pragma unroll
            for (int b = 0; b < QB; ++b)
#pragma unroll
                for (int i = 0; i < NB; ++i) {
                    s[b][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int j = 0; j < KS; ++j) s[b][i] = op_mma<T>(x.k[i][j], q[b][j], s[b][i]);
                }
            if (LATE) load_v(x, w);
            const bool whole = __all(x.ok == (1u << NV) - 1);
            if (!whole) {   // what stands in places without a token may be anything
#pragma unroll
                for (int j = 0; j < NV; ++j)
#pragma unroll
                    for (int i = 0; i < WW; ++i) x.v[j][i] = x.ok >> j & 1 ? x.v[j][i] : 0;
            }
#pragma unroll
            for (int b = 0; b < QB; ++b) {
                // (a hypothesis' own tokens: blocks without a query of its own have nothing to do)
                if (QB > 1 && w.row >= 0 && ((w.row + 1) * p.group <= (qblk * QB + b) * 16 || w.row * p.group >= (qblk * QB + b + 1) * 16)) continue;
                const bool mine = w.row < 0 ? col_live[b] : col_row[b] == w.row;
                float t[NV];
#pragma unroll
                for (int j = 0; j < NV; ++j) t[j] = mine && (whole || (x.ok >> j & 1)) ? s[b][j / 4][j % 4] * p.scale2 : -INFINITY;
                float top = t[0];
#pragma unroll
                for (int j = 1; j < NV; ++j) top = fmaxf(top, t[j]);
                top = att_max4(top);
                if (__any(top > m[b])) {
                    const float m1 = fmaxf(m[b], top), a = m1 == m[b] ? 1.f : __builtin_amdgcn_exp2f(m[b] - m1);
                    m[b] = m1;
                    l[b] *= a;
#pragma unroll
                    for (int i = 0; i < W; ++i) o[b][i] *= a;
                }
                // (fp16: weights up to 2^12 instead of 1, so that small ones keep their digits)
                const float base = m[b] == -INFINITY ? 0.f : m[b] - (__is_same(T, _Float16) ? 12.f : 0.f);
#pragma unroll
                for (int j = 0; j < NV; ++j) {
                    t[j] = __builtin_amdgcn_exp2f(t[j] - base);
                    l[b] += t[j];
                }
                // One hypothesis' own tokens add to its own columns only: the others' weights are 0 here, but 0 times a NaN or an infinity of this
                // one's is not.  (1 % of the time of hypotheses together; row by row there are no others.)
                auto add = [&](int i, const floatx4 &y) {
#pragma unroll
                    for (int r = 0; r < 4; ++r) o[b][i][r] = !GROUP || mine ? y[r] : o[b][i][r];
                };
                if constexpr (sizeof(T) == 4) {
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        floatx4 y = o[b][i];
#pragma unroll
                        for (int r = 0; r < 4; ++r) y = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[r][i]), t[r], y, 0, 0, 0);
                        add(i, y);
                    }
                } else {
                    // A weight goes into the matrix instruction as two numbers of 16 bits, what its first bits are and what they leave out: a weight's
                    // error is then 2^-16 (fp16: 2^-21) instead of 2^-9, and the output's own rounding is all that shows.  (The second half
                    // of the products costs no time: memory bounds the kernel.)  Both are made a little larger together, and the sum of the weights with
                    // them, so that the second is never 0 or below where the weight is not: times an infinity it would be NaN, not that infinity.
                    T hi[8], lo[8];
#pragma unroll
                    for (int j = 0; j < 8; j += 2) att_first_bits(t[j], t[j + 1], hi + j);
#pragma unroll
                    for (int j = 0; j < 8; ++j) lo[j] = (T)fmaf(t[j], AttMore<T>::F, -(float)hi[j]);
                    uint4 ph, pl;
                    __builtin_memcpy(&ph, hi, 16);
                    __builtin_memcpy(&pl, lo, 16);
#pragma unroll
                    for (int i = 0; i < W; ++i) {
                        const unsigned sel = i & 1 ? 0x07060302u : 0x05040100u;
                        const uint4 a = make_uint4(__builtin_amdgcn_perm(x.v[1][i / 2], x.v[0][i / 2], sel), __builtin_amdgcn_perm(x.v[3][i / 2], x.v[2][i / 2], sel),
                                                   __builtin_amdgcn_perm(x.v[5][i / 2], x.v[4][i / 2], sel), __builtin_amdgcn_perm(x.v[7][i / 2], x.v[6][i / 2], sel));
                        add(i, op_mma<T>(a, pl, op_mma<T>(a, ph, o[b][i])));
                    }
                }
            }
        };
        // (No tile ahead: with the next one's loads in front of this one's products the kernel takes 20 to 90 registers more, so fewer waves a SIMD, and
        // was 0 to 20 % slower: 320 rows of up to 400 tokens 29.0 us against 24.0 at two splits, 17.1 against 16.6 at one.)
        for (int tile = wave; tile < tiles; tile += NW) {
            const Where w = place(tile);
            Tile x;
            load_k(x, w);
            if (!LATE) load_v(x, w);
            compute(x, w);
        }
    }
    // The waves' shares meet in LDS; a lane has the same place in all of them.  Wave r then adds up and writes the r-th of the four rows of every
    // block that a lane has: W dimensions side by side.
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (lane < 16) {
            s_ml[wave][0][b * 16 + c] = m[b];
            s_ml[wave][1][b * 16 + c] = l[b] * AttMore<T>::F;
        }
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        if (b > 0) __syncthreads();
#pragma unroll
        for (int i = 0; i < W; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) s_o[wave][r][i][lane] = o[b][i][r];
        __syncthreads();
        float top = s_ml[0][0][b * 16 + c];
#pragma unroll
        for (int i = 1; i < NW; ++i) top = fmaxf(top, s_ml[i][0][b * 16 + c]);
        float y[W], sum = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) y[i] = 0.f;
#pragma unroll
        for (int j = 0; j < NW; ++j) {
            const float x = s_ml[j][0][b * 16 + c], a = x == top ? 1.f : __builtin_amdgcn_exp2f(x - top);   // (-inf of -inf: nothing there, 1 x 0)
            sum += a * s_ml[j][1][b * 16 + c];
#pragma unroll
            for (int i = 0; i < W; ++i) y[i] += a * s_o[j][wave & 3][i][lane];
        }
        if (wave < 4 && col_row[b] < N) {
            const int64_t row = r0 + col_row[b];
            const int head = col_head[b], d = (kg * 4 + wave) * W;
            constexpr int G = W < 8 ? W : 8;
#pragma unroll
            for (int g = 0; g < W / G; ++g) {
                if (PAD && d + g * G >= p.dim) continue;
                if (p.splits > 1) {
                    __builtin_memcpy(p.part_o + ((row * p.heads + head) * p.splits + split) * p.dim + d + g * G, y + g * G, G * 4);
                } else {
                    T z[G];
#pragma unroll
                    for (int i = 0; i < G; ++i) z[i] = (T)(sum == 0.f ? 0.f : y[g * G + i] / sum);   // (no weight at all: 0)
                    __builtin_memcpy((T *)(p.out + row * p.o_row + head * p.o_head) + d + g * G, z, sizeof z);
                }
            }
            if (p.splits > 1 && kg == 0 && wave == 0) {
                float *ml = p.part_ml + ((row * p.heads + head) * p.splits + split) * 2;
                ml[0] = top;
                ml[1] = sum;
            }
        }
    }
    if (qblk == 0)   // the new tokens' places in the cache (this launch reads them from k_new and v_new, whoever attends to them)
        for (int b = wave; b < N; b += NW) {
            const int pos = __shfl(pos_l, b);
            if (pos < k0 || pos >= k1) continue;
            const int i = att_page(p, pos), id = p.tables[(r0 + b) * p.ld_tables + i], off = pos - i * p.page;
            if ((unsigned)id >= (unsigned)p.pages) continue;
            const T *kn = (const T *)(p.k_new + (r0 + b) * p.kn_row + kvh * p.kn_head), *vn = (const T *)(p.v_new + (r0 + b) * p.vn_row + kvh * p.vn_head);
            for (int d = lane; d < p.dim; d += 64) {
                ((T *)(p.k_cache + (uint64_t)(unsigned)id * p.kp + (unsigned)off * p.kt + kvh * p.kh))[d] = kn[d];
                ((T *)(p.v_cache + (uint64_t)(unsigned)id * p.vp + (unsigned)off * p.vt + kvh * p.vh))[d] = vn[d];
            }
        }
}

// The splits' shares of one row and head.  Four dimensions a thread: dim / 4 threads (rounded up to 2^x) to a split, the workgroup's
// threads over as many splits as fit, four of each asked for at a time.
template <class T>
__global__ void __launch_bounds__(256)
k_attend_join(AttendP p, int threads) {
    __shared__ float s_o[256][4], s_l[256];
    const int lane = threadIdx.x & 63, row = blockIdx.y, head = blockIdx.x, d = (int)threadIdx.x % threads * 4, from = (int)threadIdx.x / threads, step = 256 / threads;
    int pos;
    const int n = att_tokens(p, row, &pos), used = n == 0 ? 1 : min(p.splits, (int)(((int64_t)n + p.split_len - 1) / p.split_len));
    const float *ml = p.part_ml + ((int64_t)row * p.heads + head) * p.splits * 2;
    const float *po = p.part_o + ((int64_t)row * p.heads + head) * p.splits * p.dim + min(d, p.dim - 4);
    float top = -INFINITY;
    for (int s = lane; s < used; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    float o[4] = {0.f, 0.f, 0.f, 0.f}, l = 0.f;
    for (int s0 = from; s0 < used; s0 += 4 * step) {
        float x[4][4], w[4], y[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int s = min(s0 + i * step, used - 1);
            w[i] = ml[2 * s];
            y[i] = ml[2 * s + 1];
            __builtin_memcpy(x[i], po + (int64_t)s * p.dim, 16);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (s0 + i * step >= used) continue;
            const float a = w[i] == top ? 1.f : __builtin_amdgcn_exp2f(w[i] - top);
            l += a * y[i];
#pragma unroll
            for (int j = 0; j < 4; ++j) o[j] += a * x[i][j];
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) s_o[threadIdx.x][j] = o[j];
    s_l[threadIdx.x] = l;
    __syncthreads();
    if (from > 0 || d >= p.dim) return;
    for (int i = 1; i < step; ++i) {
        l += s_l[i * threads];
#pragma unroll
        for (int j = 0; j < 4; ++j) o[j] += s_o[i * threads + threadIdx.x][j];
    }
    T y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = (T)(l == 0.f ? 0.f : o[j] / l);
    __builtin_memcpy((T *)(p.out + row * p.o_row + head * p.o_head) + d, y, sizeof y);
}

// How the work is split: workgroups of a key head, a row or a group of hypotheses and 16 or 32 queries, and over the tokens where those are
// fewer than the chip holds at once.
struct AttendPlan {
    int beams, qb, qblocks, waves, splits, split_len;
    double us;   // estimated
};

// beams: how many hypotheses a workgroup takes together; piece: 0 = by the rule, else tokens of a piece, in whole steps
static AttendPlan attend_form(const tbs_attend_args &a, int beams, int piece) {
    const int group = a.heads / a.kv_heads, tile = a.dtype == TBS_F32 ? 16 : 32;
    const int64_t cap = (int64_t)a.table_width * a.page;
    const int64_t longest = a.max_len > 0 && a.max_len < cap ? a.max_len : cap;
    AttendPlan pl;
    pl.beams = beams;
    const int columns = beams * group;
    pl.qb = columns > 16 && a.dim <= 128 ? 2 : 1;
    pl.qblocks = (columns + 16 * pl.qb - 1) / (16 * pl.qb);
    const int64_t units = (int64_t)a.rows / beams * a.kv_heads * pl.qblocks;
    const int64_t step = 4 * tile;   // a tile for each of four waves
    // As many pieces as take the least time, in tokens that a workgroup handles meanwhile (100 a us): turns of the 256 CUs, of a piece and 500 for a
    // workgroup's start and end, and 400 for the join.  (us by pieces: 16 units of 131071 tokens 16 177, 24 215, 32 184, 64 190; 128 units of 3000 2 30, 3 28,
    // 6 27, 12 33; 256 of up to 4000 1 101, 2 118, 4 127; 512 of 400 1 16.6, 2 24; 16 of 300 1 8.4, 2 10.3.)
    const int64_t most = (longest + 2 * step - 1) / (2 * step);
    int64_t splits = 1, least = (units + 255) / 256 * (longest + 500);
    for (int turns = 1; turns <= 4; ++turns) {   // (the pieces that fill so many turns)
        const int64_t fill = 256 * turns / units, k = fill < most ? fill : most;
        if (k < 2) continue;
        const int64_t t = (units * k + 255) / 256 * ((longest + k - 1) / k + 500) + 400;
        if (t < least) least = t, splits = k;
    }
    int64_t len = (longest + splits - 1) / splits;
    len = (len + step - 1) / step * step;
    if (len < step) len = step;
    if (piece > 0) len = (piece + step - 1) / step * step;
    pl.split_len = (int)len;
    pl.splits = (int)((longest + len - 1) / len);
    if (pl.splits < 1) pl.splits = 1;
    // Hypotheses together, up to two workgroups a CU: eight waves, to have more loads on their way (us with eight / four: 32 x 8 rows of up to 4000 tokens
    // 101 / 120, 4 x 8 of 2000 25.2 / 28.4, 64 x 8 of 40 15.3 / 16.0; nothing shared, 64 x 4 of 500 to 1500 121 / 117).  More workgroups four (128 x 8 of 200
    // 39.4 / 36.1), row by row four (4 rows of 131071 183 / 170, 128 of 4000 379 / 374; one of 300 8.1 / 8.7), and where dim leaves room for the sums of no more.
    pl.waves = beams > 1 && a.dim <= 128 && units * pl.splits <= 512 ? 8 : 4;
    const double mb = (double)units * longest * a.dim * 2 * (double)op_dtype_size(a.dtype) * 1e-6, join = pl.splits > 1 ? 5 : 0;
    pl.us = beams == 1 ? 4.5 + 0.0045 * units + (a.dtype == TBS_F32 ? 0.12 : 0.08) * mb + join
                       : 7.5 + beams * (columns > 16 ? 0.75 : 0.25) + 0.0015 * beams * units + 0.2 * mb + join;
    return pl;
}

// (together: 0 = by the rule below, 1 = row by row, 2 = hypotheses together)
static AttendPlan attend_plan(const tbs_attend_args &a, int together = 0, int piece = 0) {
    const AttendPlan rows = attend_form(a, 1, piece);
    if (a.beams == 1 || a.beams > TBS_MAX_BEAM || together == 1) return rows;
    // Hypotheses together where that is estimated to take less time.  Row by row what they share comes from the caches at 12 TB/s (float32's matrix
    // instructions: 8), but is computed again; together every hypothesis' own end costs, and memory gives 5 TB/s.  us together / row by row, estimated and
    // measured: 64 x 8 rows of 40 tokens 17, 26; 15.3, 24.8.  16 x 5 of 400 12.3, 12.6; 11.5, 13.5.  8 x 8 of 500 (four queries to a key head) 22.5, 17.3; 21.5, 16.6,
    // of 1000 25.8, 27.8; 25.2, 25.5.  2 x 16 of 1000 27, 16; 27.4, 18, of 4000 38, 47; 29, 48.  8 x 32 of 200 35, 22; 32, 19.7, of 800 40, 47; 36.6, 45.8.
    const AttendPlan groups = attend_form(a, a.beams, piece);
    return together == 2 || groups.us < rows.us ? groups : rows;
}

static int attend_check(const tbs_attend_args &a) {
    if (!op_dtype_known(a.dtype) || a.rows < 0 || a.kv_heads < 1 || a.heads < a.kv_heads || a.heads % a.kv_heads || a.dim < 8 || a.dim > 256 || a.dim % 8)
        return TBS_EINVAL;
    if (a.page < 1 || a.page > 65536 || a.pages < 1 || a.table_width < 1 || a.max_len < 0 || a.beams < 1 || a.rows % a.beams) return TBS_EINVAL;
    if (a.rows > 65535 || a.heads > 65535 || (int64_t)a.table_width * a.page > (1 << 30)) return TBS_EINVAL;
    return TBS_OK;
}

static int64_t attend_bytes(const tbs_attend_args &a, const AttendPlan &pl) { return pl.splits > 1 ? (int64_t)a.rows * a.heads * pl.splits * (a.dim + 2) * 4 : 0; }

extern "C" int64_t tbs_attend_workspace(const tbs_attend_args *args) {
    if (!args || attend_check(*args) != TBS_OK) return TBS_EINVAL;
    return args->rows == 0 ? 0 : attend_bytes(*args, attend_plan(*args));
}

template <class T, int DP, int QB, int NW, bool GROUP>
static void attend_launch(const AttendP &p, hipStream_t st) {
    const dim3 grid(p.kv_heads * p.qblocks, p.rows / p.beams, p.splits), block(64 * NW);
    if (p.dim == DP) hipLaunchKernelGGL((k_attend<T, DP, QB, false, NW, GROUP>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_attend<T, DP, QB, true, NW, GROUP>), grid, block, 0, st, p);
}

template <class T, int QB, int NW, bool GROUP>
static void attend_dims(const AttendP &p, hipStream_t st) {
    if (p.dim > 128) {   // (one block of queries, four waves: attend_form)
        if constexpr (QB == 1 && NW == 4) attend_launch<T, 256, 1, 4, GROUP>(p, st);
    } else if (p.dim <= 32) attend_launch<T, 32, QB, NW, GROUP>(p, st);
    else if (p.dim <= 64) attend_launch<T, 64, QB, NW, GROUP>(p, st);
    else attend_launch<T, 128, QB, NW, GROUP>(p, st);
}

template <class T>
static hipError_t attend_run(const AttendP &p, int qb, int waves, hipStream_t st) {
    if (p.beams == 1) qb == 1 ? attend_dims<T, 1, 4, false>(p, st) : attend_dims<T, 2, 4, false>(p, st);
    else if (waves == 8) qb == 1 ? attend_dims<T, 1, 8, true>(p, st) : attend_dims<T, 2, 8, true>(p, st);
    else qb == 1 ? attend_dims<T, 1, 4, true>(p, st) : attend_dims<T, 2, 4, true>(p, st);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && p.splits > 1) {
        int threads = 2;
        while (threads * 4 < p.dim) threads *= 2;
        hipLaunchKernelGGL((k_attend_join<T>), dim3(p.heads, p.rows), dim3(256), 0, st, p, threads);
        e = hipGetLastError();
    }
    return e;
}

static int attend_call(const tbs_attend_args *args, int together, int piece, void *stream) {
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
    // (addresses in the cache: a page's number times 32 bits, a place in the page of 32 bits)
    const int64_t wide[] = {a.k_page * es, a.v_page * es, a.k_token * es * a.page, a.v_token * es * a.page};
    for (int i = 0; i < 4; ++i)
        if ((i >= 2 || a.pages > 1) && wide[i] > UINT32_MAX) return TBS_EINVAL;
    // what is written may not lie over itself: a head after the other in the outputs and the cache
    if ((a.heads > 1 && a.out_head < a.dim) || (a.rows > 1 && a.out_row < a.dim)) return TBS_EINVAL;
    if (a.k_new && ((a.kv_heads > 1 && (a.k_head < a.dim || a.v_head < a.dim)) || (a.page > 1 && (a.k_token < a.dim || a.v_token < a.dim)) ||
                    (a.pages > 1 && (a.k_page < a.dim || a.v_page < a.dim))))
        return TBS_EINVAL;
    const void *ptrs[] = {a.q, a.k_new, a.v_new, a.k_cache, a.v_cache, a.out};
    for (const void *x : ptrs)
        if ((uintptr_t)x % es) return TBS_EINVAL;
    const AttendPlan pl = attend_plan(a, together, piece);
    const int64_t need = attend_bytes(a, pl);
    if (need > 0 && (!a.workspace || a.workspace_bytes < need || (uintptr_t)a.workspace % 16)) return TBS_EINVAL;
    AttendP p = {};
    p.q = (const char *)a.q, p.k_new = (const char *)a.k_new, p.v_new = (const char *)a.v_new;
    p.k_cache = (char *)a.k_cache, p.v_cache = (char *)a.v_cache, p.out = (char *)a.out;
    p.tables = a.tables, p.lens = a.lens;
    p.part_o = (float *)a.workspace;
    p.part_ml = p.part_o + (int64_t)a.rows * a.heads * pl.splits * a.dim;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.kn_row = a.k_new_row * es, p.kn_head = a.k_new_head * es;
    p.vn_row = a.v_new_row * es, p.vn_head = a.v_new_head * es, p.o_row = a.out_row * es, p.o_head = a.out_head * es;
    p.kp = (unsigned)(a.k_page * es), p.kt = (unsigned)(a.k_token * es), p.kh = a.k_head * es, p.vp = (unsigned)(a.v_page * es), p.vt = (unsigned)(a.v_token * es), p.vh = a.v_head * es;
    p.ld_tables = a.ld_tables;
    p.rows = a.rows, p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = a.heads / a.kv_heads, p.dim = a.dim;
    p.page = a.page, p.pages = a.pages, p.width = a.table_width, p.splits = pl.splits, p.split_len = pl.split_len, p.qblocks = pl.qblocks, p.beams = pl.beams;
    const unsigned twice = 2 * (unsigned)a.page, lg = 31 - __builtin_clz(twice);
    p.page_shift = (twice & (twice - 1)) ? lg : 0;
    p.page_mul = (unsigned)((((uint64_t)1 << (32 + p.page_shift)) / twice) + (p.page_shift ? 1 : 0));
    p.scale2 = (a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.dim)) * 1.44269504f;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = a.dtype == TBS_F32 ? attend_run<float>(p, pl.qb, pl.waves, st) : a.dtype == TBS_BF16 ? attend_run<__bf16>(p, pl.qb, pl.waves, st) : attend_run<_Float16>(p, pl.qb, pl.waves, st);
    return e == hipSuccess ? TBS_OK : TBS_EHIP;
}

extern "C" int tbs_attend_paged(const tbs_attend_args *args, void *stream) { return attend_call(args, 0, 0, stream); }

// one way of splitting the work, for the tests (not in the header)
extern "C" int attend_by(const tbs_attend_args *args, int together, int piece, void *stream) { return attend_call(args, together, piece, stream); }
