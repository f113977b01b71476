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
// Keys and values of a tile go to LDS by direct loads, those of new tokens while the tile before is worked on.  Behind a cache that holds in part only: the number of a later tile's page is
// looked up behind these loads and copied at once (look()), and what waits for it waits for them too.  Pieces of 16 bytes of a row are permuted by bits
// of the row, so that a fragment's reads are all LDS banks once.
//
// Weights are rounded to the 16 bits of the values' type: a weight's relative error is half a step of it, as large as the output's own rounding.  Where values are independent the two add up
// to sqrt(2) times the one (measured against 64 bits: 1.17 to 1.41 times the error that float32 weights leave); a mean of like values hardly has the weights' part.  Two
// numbers a weight would cost half as many matrix instructions again.  Sums, statistics and the weights' sum are float32.
//
// Bound by the matrix and the vector units together.  Prompts of 16000 and 7001 tokens, 32 heads on 8 of 128, bfloat16: 2.4 ms, 1.03 PFLOP/s (a large product of the library 1.45),
// the matrix pipes 50 % busy, the vector units (32 exponentials, roundings and sums a lane of 64 keys) 44 %; two waves a SIMD overlap the two only in part.  16000 tokens, 32 heads
// on 8 of 64: 1.2 ms, 0.87 PFLOP/s, half as many products for the same exponentials.  4000 in float32, 16 heads on 4 of 128: 600 us, 110 TFLOP/s of 153 (where
// the rest goes is not known).
// Four waves and 32 queries each: eight in two groups half a tile apart gained 2 %, eight behind one barrier 3 % of long prompts and lost 10 % of a batch's short ones; 64 queries
// a wave spill; 32 keys a tile 7 % slower at 128; three tiles on their way 12 %; halves of a tile worked on in turn inside a wave 15 %.
#include "op_device.h"

#define PROMPTS_SLACK 8.f
#define PROMPTS_WAVES 4   // of 32 rows each: a workgroup (two, for more workgroups where tiles are few, took as long or twice as long: fewer loads are on their way)
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short prompts_b64;

struct PromptsP {
    const char *q, *k, *v, *k_cache, *v_cache;
    const int *starts, *past, *tables;
    char *out;
    int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head, kh, vh, ld_tables;   // bytes (ld_tables: elements)
    unsigned kp, kt, vp, vt;
    int tokens, prompts, heads, kv_heads, group, dim, page, pages, width;
    bool direct;    // everything on 16-byte boundaries
    unsigned page_mul, page_shift;
    float scale2;   // |scale| log2(e)
    unsigned flip;  // sign bits of a word of queries where the scale is negative
    // where the keys of a tile are shared among workgroups (otherwise null): the list of pieces, and what they leave
    struct PromptsPiece *pieces;
    int *count;               // pieces, and tiles
    struct PromptsSplit *splits;
    float *part_o, *part_ml;  // [pieces, kv_heads, rows, dim], [pieces, kv_heads, rows, 2]
};

// Steps k0 .. k1 - 1 of a tile's keys; apart: not all of them, and the piece's sums go to its place in part_o
struct PromptsPiece {
    int prompt, tile, k0, k1, apart;
};
// A tile's pieces
struct PromptsSplit {
    int prompt, tile, first, count;
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
// (they have the most keys); prompt -1 for one behind all of them, and then the number of tiles.  Every workgroup adds all prompts up, so that the time grows as prompts times tiles: of prompts of
// one token, 8 heads of 64, 512 take 42 us, 4096 970 and 16384 14600.
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
    static constexpr int E = OpPiece<T>::E, KEYS = sizeof(T) == 4 || DP > 128 ? 32 : 64;   // (prompts_form() counts with them)
    static constexpr int USED = DP / E;                                       // pieces of a row
    static constexpr int PITCH = USED <= 4 ? 4 : USED <= 8 ? 8 : sizeof(T) == 2 && USED <= 12 ? 12 : USED <= 16 ? 16 : USED <= 32 ? 32 : 64;   // ... in LDS
    static constexpr int BYTES = KEYS * PITCH * 16;                           // of keys, or values
    static constexpr int SPAN = PITCH >= 16 ? 16 : PITCH == 8 ? 8 : 4;        // pieces that a swizzle changes among each other
    // (12: 64 bytes a row fewer to load and to keep than with 16; rows of 192 bytes, four of which begin at different quarters of all banks)
    // Keys: 32 rows' pieces of one place.  Values: four rows' two or four pieces side by side (float32: a row's eight, and those of the row four behind).
    static __device__ __forceinline__ int k_swizzle(int row) { return PITCH >= 16 ? row & 15 : PITCH == 8 ? row >> 1 & 7 : row >> 2 & 3; }
    static __device__ __forceinline__ int v_swizzle(int row) {
        if (sizeof(T) == 4) return PITCH >= 16 ? (row >> 2 & 1) << 3 : 0;
        return PITCH >= 16 ? (row & 2) << 2 | (row & 1) << 2 | (row & 2) : PITCH == 8 ? (row & 2) << 1 | (row & 1) << 1 : row & 2;
    }
};

// t / page = 2 t / (2 page) for 0 <= t <= 2^30 by multiplication, as for one token over the cache: page_mul = floor(2^(32 + s) / (2 page)) + 1 with
// s = floor(log2 (2 page)) is at most 2^(s + 1) / 2^(32 + s) of a unit too large for numerators below 2^31 (powers of two: exact)
__device__ __forceinline__ unsigned prompts_page(const PromptsP &p, int t) { return __umulhi((unsigned)t << 1, p.page_mul) >> p.page_shift; }

// what all lanes have alike, in scalar registers
__device__ __forceinline__ const char *prompts_uniform(const char *x) {
    const uint64_t u = (uint64_t)(uintptr_t)x;
    return (const char *)(uintptr_t)((uint64_t)(unsigned)__builtin_amdgcn_readfirstlane((int)(u >> 32)) << 32 | (unsigned)__builtin_amdgcn_readfirstlane((int)u));
}

// Direct loads to LDS, N up to four times 16 bytes a lane, from base + off[i] + 1024 i to lds + 1024 i + 16 lane: the instruction adds its own offset on both sides, so that
// neither has an address to be made
template <int N>
__device__ __forceinline__ void prompts_load_lds(const char *base, unsigned off0, unsigned off1, unsigned off2, unsigned off3, unsigned lds) {
    unsigned m0_was;
    const unsigned to = __builtin_amdgcn_readfirstlane(lds);
    if constexpr (N == 1)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\ts_mov_b32 m0, %0" : "=&s"(m0_was) : "s"(to), "s"(base), "v"(off0) : "memory");
    else if constexpr (N == 2)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\tglobal_load_lds_dwordx4 %4, %2 offset:1024\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_was) : "s"(to), "s"(base), "v"(off0), "v"(off1) : "memory");
    else if constexpr (N == 3)
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\tglobal_load_lds_dwordx4 %4, %2 offset:1024\n\t"
                     "global_load_lds_dwordx4 %5, %2 offset:2048\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_was) : "s"(to), "s"(base), "v"(off0), "v"(off1), "v"(off2) : "memory");
    else
        asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %3, %2\n\tglobal_load_lds_dwordx4 %4, %2 offset:1024\n\t"
                     "global_load_lds_dwordx4 %5, %2 offset:2048\n\tglobal_load_lds_dwordx4 %6, %2 offset:3*1024\n\ts_mov_b32 m0, %0"
                     : "=&s"(m0_was) : "s"(to), "s"(base), "v"(off0), "v"(off1), "v"(off2), "v"(off3) : "memory");
}

// The order of N matrix instructions and the R LDS reads that each wants: those of the first A instructions, then an instruction and the reads of the one A
// behind it.  (All reads first would take 64 registers.)
template <int N, int R, int A>
__device__ __forceinline__ void prompts_interleave() {
    __builtin_amdgcn_sched_group_barrier(0x100, R * (A < N ? A : N), 0);
#pragma unroll
    for (int i = 0; i < N - A; ++i) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, R, 0);
    }
    __builtin_amdgcn_sched_group_barrier(0x008, A < N ? A : N, 0);
}

// What a workgroup does.  DP: dim rounded up to 32, 64, 96, 128 or 256, or 80 itself; SHARED: by the list of pieces (its few scalars more cost 7 % in
// the loop).  A class whose functions are all inlined: everything in it is in registers.
#define PROMPTS_INLINE __device__ __forceinline__
template <class T, int DP, bool SHARED>
struct PromptsWork {
    typedef PromptsTile<T, DP> Tile;
    static constexpr int E = Tile::E, TK = Tile::KEYS, PITCH = Tile::PITCH, DB = (DP + 31) / 32, KS = DP * (int)sizeof(T) / 32, NW = PROMPTS_WAVES, ROWS = 32 * NW;
    static constexpr int CHUNKS = TK * PITCH / 64, MINE = (CHUNKS + NW - 1) / NW;   // loads of 64 pieces, and those of a wave
    static constexpr int RUN = MINE * 64 / PITCH;                                   // rows of a wave's
    // addresses of fragments: the swizzles change 4, 8 or 16 pieces among each other, and what is so many further has the same address and a constant
    static constexpr int KA = Tile::SPAN / 2 < KS ? Tile::SPAN / 2 : KS, VA = sizeof(T) == 4 ? 1 : Tile::SPAN / 4 < DB ? Tile::SPAN / 4 : DB;
    static constexpr int KB = TK / 32;
    // (float16: weights up to 2^7 more, so that small ones keep their digits: with the slack's 2^8 at most half its largest number)
    static constexpr float MORE = __is_same(T, _Float16) ? 7.f : 0.f;
    static constexpr bool KEY = false, VALUE = true;

    const PromptsP &p;
    char *kv;   // LDS: keys and values of two tiles
    int lane, wave, c, h;
    PromptsAt at;
    const int *table;
    int keys, first_step, steps;             // up to the last that a row of the workgroup sees; steps to do
    int sees, wave_first, wave_last;         // the last key that this lane's query sees; the first and last of the wave's
    bool holes;                              // whether some of its pages do not exist
    bool runs;                               // whether a wave's keys of a tile lie in one page, on 16-byte boundaries
    uint4 q[KS];
    const char *k_new, *v_new, *k_old, *v_old;
    unsigned lds;
    unsigned k_off[MINE], v_off[MINE];   // bytes of a lane's pieces from 3 KiB before the wave's first key, less 1024 times their number among four: in a page, and then among new tokens
    bool k_in[MINE], v_in[MINE];         // (pieces behind the head's end are not there)
    int id[MINE], v_id[MINE];            // the pages of the keys and of the values that are asked for next, looked up a tile ahead: of this lane's (a wave's may be one)
    const char *k_at[KA], *v_at[VA];   // where this lane's fragments begin
    floatx16 o[DB];
    float m, l;
    uint4 w[sizeof(T) == 4 ? 1 : TK / 16];   // a tile's weights (float32: in place of the scores)

    PROMPTS_INLINE PromptsWork(const PromptsP &p_, char *kv_) : p(p_), kv(kv_) {}

    // ---- tiles into LDS: a lane's pieces are places of its rows
    // (what is seldom wanted is worked out where it is, not kept in registers)
    static PROMPTS_INLINE int again() {
        int x = threadIdx.x & 63;
        asm volatile("" : "+v"(x));
        return x;
    }
    PROMPTS_INLINE int row_of(int i, int lane) const { return ((wave * MINE + i) * 64 + lane) / PITCH; }
    PROMPTS_INLINE int piece_of(int i, int lane, bool value) const {
        return (((wave * MINE + i) * 64 + lane) % PITCH) ^ (value ? Tile::v_swizzle(row_of(i, lane)) : Tile::k_swizzle(row_of(i, lane)));
    }
    PROMPTS_INLINE bool takes_part(int i) const { return CHUNKS % NW == 0 || wave * MINE + i < CHUNKS; }
    // where the pieces of a lane are: keys, or values, `bytes` apart
    template <bool V>
    PROMPTS_INLINE void places(unsigned bytes) {
        const int lane = again();
#pragma unroll
        for (int i = 0; i < MINE; ++i) {
            const int piece = piece_of(i, lane, V);   // (dim = DP: places behind the head's end are never looked at, and have its first piece)
            (V ? v_off : k_off)[i] = (row_of(i, lane) - wave * RUN) * bytes + (piece < Tile::USED ? piece : 0) * 16 + (3 - i % 4) * 1024;
        }
    }
    PROMPTS_INLINE int page_of(int t) const { return t < at.past ? table[prompts_page(p, t)] : 0; }
    PROMPTS_INLINE void look(int step) {   // (the values follow the keys a tile later, with the pages of the last look)
        const int t0 = step * TK;
        if (t0 >= at.past + TK) return;
        const int lane = again();
        int x[MINE];
        if (runs) {
            x[0] = page_of(t0 + wave * RUN);
#pragma unroll
            for (int i = 1; i < MINE; ++i) x[i] = x[0];
        } else {
#pragma unroll
            for (int i = 0; i < MINE; ++i) x[i] = page_of(t0 + row_of(i, lane));
        }
#pragma unroll
        for (int i = 0; i < MINE; ++i) v_id[i] = id[i], id[i] = x[i];
    }
    template <bool V>
    PROMPTS_INLINE void load(const char *from, unsigned to) {
        from -= 3 * 1024;   // (offsets are unsigned)
        constexpr int N = MINE < 4 ? MINE : 4;
        auto off = [&](int i) __attribute__((always_inline)) { return V ? v_off[i] : k_off[i]; };
#pragma unroll
        for (int i = 0; i < MINE; i += N) {
            if (p.dim == DP) {
                if (takes_part(i)) prompts_load_lds<N>(from, off(i), off(N > 1 ? i + 1 : i), off(N > 2 ? i + 2 : i), off(N > 3 ? i + 3 : i), to + i * 1024);
            } else {
#pragma unroll
                for (int j = 0; j < N; ++j)
                    if (takes_part(i + j) && (V ? v_in[i + j] : k_in[i + j])) prompts_load_lds<1>(from + j * 1024, off(i + j), 0, 0, 0, to + (i + j) * 1024);
            }
        }
    }
    template <bool V>
    PROMPTS_INLINE void ask(int step) {
        const int t0 = step * TK, buffer = step & 1, t = t0 + wave * RUN;
        const unsigned to = lds + (buffer * 2 + V) * Tile::BYTES + wave * MINE * 1024;
        const bool fresh = t0 >= at.past;
        const char *newer = V ? v_new : k_new, *older = V ? v_old : k_old;
        const int64_t row_bytes = V ? p.v_row : p.k_row;
        const unsigned page_bytes = V ? p.vp : p.kp, token_bytes = V ? p.vt : p.kt;
        if (fresh ? p.direct && t0 + TK <= keys : runs && t0 + TK <= at.past) {   // new tokens or ones of the cache, all there: scalar addresses
            const char *from;
            if (fresh) {
                if (t0 < at.past + TK) places<V>((unsigned)row_bytes);   // (the first of the new ones)
                from = newer + (int64_t)(t - at.past) * row_bytes;
            } else {
                const unsigned n = (unsigned)__builtin_amdgcn_readfirstlane(V ? v_id[0] : id[0]), use = n < (unsigned)p.pages ? n : 0;   // (a page that does not exist: the first's, masked)
                from = older + (uint64_t)use * page_bytes + ((unsigned)t - prompts_page(p, t) * (unsigned)p.page) * token_bytes;
            }
            load<V>(prompts_uniform(from), to);
        } else {
            const int lane = again();
            int n[MINE];
            if (!fresh) {
#pragma unroll
                for (int i = 0; i < MINE; ++i) {
                    n[i] = V ? v_id[i] : id[i];
                    asm volatile("" : "+v"(n[i]));   // (here, before the first load: it would be waited for)
                }
            }
#pragma unroll
            for (int i = 0; i < MINE; ++i) {
                if (!takes_part(i)) continue;
                const int key = min(t0 + row_of(i, lane), keys - 1), piece = piece_of(i, lane, V);   // (behind the last: anything that is there)
                const char *from = newer + (int64_t)(key - at.past) * row_bytes;
                if (key < at.past) {
                    const unsigned use = (unsigned)n[i] < (unsigned)p.pages ? n[i] : 0;
                    from = older + (uint64_t)use * page_bytes + ((unsigned)key - prompts_page(p, key) * (unsigned)p.page) * token_bytes;
                }
                if (piece * E >= p.dim) continue;
                if (p.direct) op_load_lds(from + piece * 16, __builtin_amdgcn_readfirstlane(to + i * 1024));
                else *(uint4 *)(kv + (buffer * 2 + V) * Tile::BYTES + (wave * MINE + i) * 1024 + lane * 16) = op_load16((const T *)from + piece * E);
            }
        }
    }
    static PROMPTS_INLINE void landed() {
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    // ---- fragments
    PROMPTS_INLINE uint4 k_frag(int step, int b, int j) const {   // 32 keys, two pieces
        return *(const uint4 *)(k_at[j % KA] + j / KA * Tile::SPAN * 16 + (step & 1) * 2 * Tile::BYTES + b * 32 * PITCH * 16);
    }
    PROMPTS_INLINE int v_row() const { return sizeof(T) == 4 ? 4 * h : 4 * h + (lane >> 2 & 3); }
    PROMPTS_INLINE const char *v_place(int d) const {
        return kv + Tile::BYTES + (sizeof(T) == 4 ? v_row() * PITCH * 16 : (v_row() * PITCH + ((d * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1)) ^ Tile::v_swizzle(v_row()))) * 16 + (lane & 1) * 8);
    }
    // V^T of 16 keys from `key` on (in the order of the weights) and 32 dimensions from `from` on
    static PROMPTS_INLINE uint4 v_frag(const char *from, int step, int key) {
        uint4 u;
        typedef __attribute__((address_space(3))) prompts_b64 *Lds;
        from += (step & 1) * 2 * Tile::BYTES;
        const prompts_b64 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from + key * PITCH * 16)), y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(from + (key + 8) * PITCH * 16));
        __builtin_memcpy(&u, &x, 8);
        __builtin_memcpy((char *)&u + 8, &y, 8);
        return u;
    }
    PROMPTS_INLINE float v_one(int step, int key, int d) const {   // float32: dimension 32 d + c of key `key` + 4 h
        return *(const float *)(v_at[0] + (step & 1) * 2 * Tile::BYTES + key * PITCH * 16 + (((d * 8 + c / 4) ^ (PITCH >= 16 ? h << 3 : 0)) * 16 + c % 4 * 4));
    }
    // which of a tile's keys there are (bit i: key i), for all of the wave
    static constexpr unsigned long long WHOLE = TK == 64 ? ~0ull : (1ull << (TK & 63)) - 1;
    PROMPTS_INLINE unsigned long long there_of(int step) const {
        const int t0 = step * TK;
        unsigned long long there = keys - t0 >= TK ? WHOLE : (1ull << (keys - t0)) - 1;
        if (holes && t0 < at.past) {
            const int t = t0 + (int)(threadIdx.x & (TK - 1));
            there &= __ballot(t >= at.past || (unsigned)page_of(t) < (unsigned)p.pages);
        }
        return there;
    }
    // ... and which of them this lane's query sees
    PROMPTS_INLINE unsigned long long mine_of(int step, unsigned long long there) const {
        const int last = sees - step * TK;   // (its last key's place)
        return last < 0 ? 0 : last >= 63 ? there : there & ((2ull << last) - 1);
    }
    PROMPTS_INLINE bool mixed(int step, unsigned long long there) const { return there != WHOLE || step * TK + TK - 1 > wave_first; }   // some key is not some query's

    PROMPTS_INLINE void scores(floatx16 (&s)[KB], int step) {
        __builtin_amdgcn_s_setprio(1);
#pragma unroll
        for (int j = 0; j < KS; ++j)
#pragma unroll
            for (int b = 0; b < KB; ++b) s[b] = op_mma32<T>(k_frag(step, b, j), q[j], j == 0 ? floatx16{} : s[b]);
        if constexpr (sizeof(T) == 2) prompts_interleave<KS * KB, 1, 4>();
        __builtin_amdgcn_s_setprio(0);
        __builtin_amdgcn_sched_barrier(0);
    }
    // the scores of keys that this lane's query does not see
    PROMPTS_INLINE void hide(floatx16 (&s)[KB], int step, unsigned long long there) const {
        if (mixed(step, there)) {
            const unsigned long long bits = mine_of(step, there) >> (4 * h);
#pragma unroll
            for (int b = 0; b < KB; ++b)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[b][i] = bits >> (32 * b + 8 * (i / 4) + i % 4) & 1 ? s[b][i] : -INFINITY;
        }
    }
    // Scores into weights, 2^(t - m), and these to their sum
    PROMPTS_INLINE void weigh(floatx16 (&s)[KB]) {
        const float base = m == -INFINITY ? 0.f : m - MORE;
        float sum[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < TK / 16; ++i) {
            T x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float y = __builtin_amdgcn_exp2f(fmaf(s[i / 2][i % 2 * 8 + j], p.scale2, -base));
                if constexpr (sizeof(T) == 4) s[i / 2][i % 2 * 8 + j] = y;
                sum[j & 1] += y;
                x[j] = (T)y;
            }
            if constexpr (sizeof(T) == 2) __builtin_memcpy(&w[i], x, 16);
        }
        l += sum[0] + sum[1];
        __builtin_amdgcn_sched_barrier(0);
    }
    PROMPTS_INLINE void softmax(floatx16 (&s)[KB], int step, unsigned long long there) {
        hide(s, step, there);
        float top = s[0][0];
#pragma unroll
        for (int b = 0; b < KB; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = fmaxf(top, s[b][i]);
        typedef unsigned uint2_ __attribute__((ext_vector_type(2)));
        const uint2_ u = __builtin_amdgcn_permlane32_swap(__float_as_uint(top), __float_as_uint(top), false, false);   // (this lane's and its other half's)
        top = fmaxf(__uint_as_float(u[0]), __uint_as_float(u[1])) * p.scale2;
        if (__any(top > m + PROMPTS_SLACK)) {
            const float m1 = fmaxf(m, top), a = m1 == m ? 1.f : __builtin_amdgcn_exp2f(m - m1);
            m = m1;
            l *= a;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= a;
        }
        weigh(s);
    }
    PROMPTS_INLINE void values(const floatx16 (&s)[KB], int step) {   // the weights with their values
        __builtin_amdgcn_s_setprio(1);
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < 16 * KB; ++i)
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x2f32(v_one(step, i / 16 * 32 + 8 * (i % 16 / 4) + i % 4, d), s[i / 16][i % 16], o[d], 0, 0, 0);
        } else {
#pragma unroll
            for (int i = 0; i < TK / 16; ++i)
#pragma unroll
                for (int d = 0; d < DB; ++d) o[d] = op_mma32<T>(v_frag(v_at[d % VA] + d / VA * Tile::SPAN * 16, step, i * 16), w[i], o[d]);
            prompts_interleave<TK / 16 * DB, 2, 4>();
        }
        __builtin_amdgcn_s_setprio(0);
    }

    PROMPTS_INLINE void start() {
#pragma unroll
        for (int d = 0; d < DB; ++d) o[d] = floatx16{};
        l = 0.f;
        if (first_step * TK < at.past) places<false>(p.kt), places<true>(p.vt);
        else if (first_step * TK >= at.past + TK) places<false>((unsigned)p.k_row), places<true>((unsigned)p.v_row);   // (ask() has them with the first new tile)
    }
    // a tile's values, and the keys of the next one
    PROMPTS_INLINE void ask_for(int step) {
        if (step < steps) ask<true>(step);
        if (step + 1 < steps) {
            ask<false>(step + 1);
            look(step + 2);
        }
    }
    // All tiles.  A value that is NaN or infinite reaches, times the weight 0, the queries that do not see it, and a sum of weights up to 2^8 and large values may be beyond
    // float32 where their mean is not: of the outputs of this pass nothing is kept then.
    PROMPTS_INLINE void pass() {
        start();
        m = -INFINITY;
        floatx16 s[KB];
        const int mine = min(steps, wave_last < 0 ? 0 : wave_last / TK + 1);   // steps in which the wave has something to do
        int step = first_step;
        look(step);
        ask<false>(step);
        look(step + 1);
        landed();
        ask_for(step);
        if (step < mine) {
            scores(s, step);
            for (;;) {
                softmax(s, step, there_of(step));
                landed();
                ask_for(step + 1);
                values(s, step);
                if (++step >= mine) break;
                __builtin_amdgcn_sched_barrier(0);
                scores(s, step);
            }
        }
        for (; step < steps; ++step) {   // (the others have)
            landed();
            ask_for(step + 1);
        }
    }
    // The d-th 32 dimensions, in o[0], with the reference that m is; keys are added one by one to the queries that see them.
    PROMPTS_INLINE void pass_apart(int d) {
        start();
        const char *place = v_place(sizeof(T) == 4 ? 0 : d);
        for (int step = first_step; step < steps; ++step) {
            look(step);
            ask<false>(step);
            look(step + 1);
            ask<true>(step);
            landed();
            if (step * TK <= wave_last) {
                const unsigned long long there = there_of(step);
                floatx16 s[KB];
                scores(s, step);
                hide(s, step, there);
                weigh(s);
                const unsigned long long mine = mixed(step, there) ? mine_of(step, there) : ~0ull;
#pragma unroll 1
                for (int key = 0; key < TK; ++key) {
                    const bool seen = mine >> key & 1;
                    if (!__any(seen)) continue;
                    const int half = key >> 2 & 1;   // its place in the fragments: half, and element
                    floatx16 z = {};
                    if constexpr (sizeof(T) == 4) {
                        float one = 0.f;
#pragma unroll
                        for (int i = 0; i < 16 * KB; ++i) one = i / 16 * 32 + 8 * (i % 16 / 4) + i % 4 == (key & ~4) ? s[i / 16][i % 16] : one;
                        const float v = v_one(step, key & ~4, d);
                        z = __builtin_amdgcn_mfma_f32_32x32x2f32(h == half ? v : 0.f, h == half && seen ? one : 0.f, z, 0, 0, 0);
                    } else {
                        const int e = (key >> 3 & 1) * 4 + (key & 3);
                        const unsigned keep = h == half ? (e & 1 ? 0xffff0000u : 0xffffu) : 0;
                        uint4 x = v_frag(place, step, key & ~15), y = w[0];
#pragma unroll
                        for (int i = 1; i < TK / 16; ++i)
                            if (i == key >> 4) y = w[i];
                        x.x &= e / 2 == 0 ? keep : 0, x.y &= e / 2 == 1 ? keep : 0, x.z &= e / 2 == 2 ? keep : 0, x.w &= e / 2 == 3 ? keep : 0;
                        z = op_mma32<T>(x, y, z);
                    }
#pragma unroll
                    for (int j = 0; j < 16; ++j) o[0][j] = seen ? o[0][j] + z[j] : o[0][j];
                }
            }
            landed();
        }
    }

    PROMPTS_INLINE void run() {
        lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), c = lane & 31, h = lane >> 5;
        const int kvh = (int)blockIdx.x % p.kv_heads, unit = (int)blockIdx.x / p.kv_heads;
        PromptsPiece piece = {0, 0, 0, INT32_MAX, 0};
        int2 found;
        if (SHARED) {
            const int n = *p.count;
            if (unit < n) piece = p.pieces[unit];
            found = unit < n ? make_int2(piece.prompt, piece.tile) : make_int2(-1, n);
        } else {
            found = prompts_find(p, unit, ROWS);
        }
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
        const int prompt = __builtin_amdgcn_readfirstlane(found.x), tile = __builtin_amdgcn_readfirstlane(found.y);
        at = prompts_at(p, prompt);
        at.start = __builtin_amdgcn_readfirstlane(at.start), at.n = __builtin_amdgcn_readfirstlane(at.n), at.past = __builtin_amdgcn_readfirstlane(at.past);   // (in scalar registers)
        table = p.past ? p.tables + prompt * p.ld_tables : nullptr;
        const int rows = at.n * p.group, row0 = tile * ROWS;   // (below 2^31: tokens x heads is)
        keys = at.past + (min(row0 + ROWS, rows) - 1) / p.group + 1;
        first_step = __builtin_amdgcn_readfirstlane(piece.k0), steps = min((keys + TK - 1) / TK, __builtin_amdgcn_readfirstlane(piece.k1));
        const int row = row0 + wave * 32 + c, token = row / p.group, w0 = row0 + wave * 32;
        const bool live = row < rows;
        sees = live ? at.past + token : -1;
        wave_first = w0 + 32 <= rows ? at.past + w0 / p.group : -1, wave_last = w0 < rows ? at.past + (min(w0 + 32, rows) - 1) / p.group : -1;
        holes = false, runs = p.direct && p.page % RUN == 0;
        if (at.past > 0) {
            const int from = first_step * TK, to = min(at.past, steps * TK);
            for (int i = (int)prompts_page(p, from) + threadIdx.x; from < to && i <= (int)prompts_page(p, to - 1); i += 64 * NW) holes |= (unsigned)table[i] >= (unsigned)p.pages;
            holes = __syncthreads_or(holes);
        }
        {
            const int head = kvh * p.group + row - token * p.group;
            const T *src = (const T *)(p.q + (int64_t)(at.start + (live ? token : 0)) * p.q_row + (live ? head : 0) * p.q_head);
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                q[s] = live && (s * 2 + h) * E < p.dim ? op_load16(src + (s * 2 + h) * E) : make_uint4(0, 0, 0, 0);
                q[s].x ^= p.flip, q[s].y ^= p.flip, q[s].z ^= p.flip, q[s].w ^= p.flip;
            }
        }
        k_new = p.k + (int64_t)at.start * p.k_row + kvh * p.k_head, v_new = p.v + (int64_t)at.start * p.v_row + kvh * p.v_head;
        k_old = p.k_cache + kvh * p.kh, v_old = p.v_cache + kvh * p.vh;
        lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)kv;
#pragma unroll
        for (int i = 0; i < MINE; ++i) k_in[i] = piece_of(i, lane, false) * E < p.dim, v_in[i] = piece_of(i, lane, true) * E < p.dim;
        // pieces behind the head's end are 0 in both buffers, and stay so
        if (p.dim < DP) {
            for (int i = threadIdx.x; i < 4 * TK * PITCH; i += 64 * NW) {
                const int in = i % (TK * PITCH), r = in / PITCH, slot = in % PITCH;
                if ((slot ^ ((i / (TK * PITCH)) & 1 ? Tile::v_swizzle(r) : Tile::k_swizzle(r))) * E >= p.dim) ((uint4 *)kv)[i] = make_uint4(0, 0, 0, 0);
            }
        }
#pragma unroll
        for (int s = 0; s < KA; ++s) k_at[s] = kv + (c * PITCH + ((s * 2 + h) ^ Tile::k_swizzle(c))) * 16;
#pragma unroll
        for (int d = 0; d < VA; ++d) v_at[d] = v_place(d);

        auto store = [&](const floatx16 &x, int d) __attribute__((always_inline)) {
            const float sum = l + __shfl_xor(l, 32), f = sum == 0.f ? 0.f : 1.f / sum;   // (no weight at all: 0)
            if (!live) return;
            if (SHARED && piece.apart) {
                const int64_t place = ((int64_t)unit * p.kv_heads + kvh) * ROWS + wave * 32 + c;
#pragma unroll
                for (int b = 0; b < 4; ++b)
                    if (d * 32 + b * 8 + h * 4 < p.dim) *(float4 *)(p.part_o + place * p.dim + d * 32 + b * 8 + h * 4) = make_float4(x[b * 4], x[b * 4 + 1], x[b * 4 + 2], x[b * 4 + 3]);
                if (h == 0 && d == 0) *(float2 *)(p.part_ml + place * 2) = make_float2(m, sum);
                return;
            }
            char *to = p.out + (int64_t)(at.start + token) * p.o_row + (kvh * p.group + row - token * p.group) * p.o_head;
#pragma unroll
            for (int b = 0; b < 4; ++b) {
                const int e = d * 32 + b * 8 + h * 4;   // (dim is a multiple of 8)
                if (e >= p.dim) continue;
                T y[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) y[i] = (T)(sum == 0.f ? 0.f : x[b * 4 + i] * f);
                __builtin_memcpy((T *)to + e, y, sizeof y);
            }
        };
        pass();
        float none = 0.f;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i)
                if (d * 32 + i / 4 * 8 < DP) none = fmaf(o[d][i], 0.f, none);   // (behind the head's end there may be anything)
        if (!__syncthreads_or(live && none != 0.f)) {
#pragma unroll
            for (int d = 0; d < DB; ++d) store(o[d], d);
        } else {
            // With the weights' sum in the reference they are parts of 1, and no sum of them is larger than the largest value.  (float16, whose small weights would
            // lose digits: parts of 2^15, its values are 2^16 at most.)
            m += __builtin_amdgcn_logf(l + __shfl_xor(l, 32)) - (__is_same(T, _Float16) ? 15.f : 0.f);   // (the logarithm to 2; -inf where there is no weight)
            asm volatile("" : "+v"(h), "+v"(lane));   // (nothing of what follows is worked out ahead of the first pass, whose registers are few)
#pragma unroll 1
            for (int d = 0; d < DB; ++d) {
                pass_apart(d);
                store(o[0], d);
                __syncthreads();
            }
        }
    }
};

template <class T, int DP, bool SHARED>
__global__ void __launch_bounds__(64 * PROMPTS_WAVES, DP > 128 || sizeof(T) == 4 ? 1 : DP <= 80 ? 3 : 2)   // (three at 80: 4 to 9 registers spill, and 16000 tokens take 771 us in place of 863; float32's shared form at 256 spills 36)
k_prompts(PromptsP p) {
    __shared__ __align__(16) char s_kv[4 * PromptsTile<T, DP>::BYTES];
    PromptsWork<T, DP, SHARED> work(p, s_kv);
    work.run();
}

#define PROMPTS_PLAN 1024     // threads of the plan; tiles, and prompts, at most
#define PROMPTS_LENGTHS 16    // lengths of pieces that are looked at
#define PROMPTS_PIECES 4      // pieces of an equal share at most
#define PROMPTS_LEAST 4       // steps of a piece at least, where a tile has more than one
__device__ const int prompts_parts[PROMPTS_LENGTHS] = {16, 18, 20, 22, 25, 28, 32, 36, 40, 44, 50, 56, 64, 96, 128, 0};   // 64ths of a share; 0: whole tiles

// workgroups of four waves that the chip runs at a time, one to three a CU, as the plan and the choice of the form count them.  (Registers allow four at 32 in 16 bits, three at 32 in float32 and
// two of the shared form at 80 in float32, of which the measured rules know nothing.)
static int prompts_slots(const tbs_attend_prompts_args &a) { return 256 * (a.dtype == TBS_F32 ? (a.dim <= 64 ? 2 : 1) : a.dim <= 64 || a.dim == 80 ? 3 : a.dim <= 128 ? 2 : 1); }

// Whose keys are shared, one workgroup: a thread a tile, or prompt.  A piece is at most `len` steps long: of sixteen lengths, from a quarter of an equal share of all work up, the one that
// is estimated to take the fewest steps one after the other.  That is the turns that the slots take, whole ones, of a mean piece and eight steps for its start, its end and the way
// of its sums through memory; where one turn is enough, the longest piece; and six steps for the join.  (Measured by the lengths, in shares.  Four chunks of 100 to 512
// tokens behind 20001 to 60000, 32 heads of 128: 1/4 1153 us, 1/3 1128, 1/2 1304, 2/3 1067, 1 1326, all 2254.  256 tokens behind 100000, 8 heads: 1/4 291, 2/3 270, 1 204, 3/2 242, all 3945.
// 2100 tokens, 8 heads: 1/4 51, 1/3 42, 1/2 45, 1 52, all 84.  4000 in float32: 1/4 778, 1 803, all 689.)
__global__ void __launch_bounds__(PROMPTS_PLAN)
k_prompts_plan(PromptsP p, int rows, int step, int most, int slots) {
    __shared__ int s_first[PROMPTS_PLAN], s_wave[PROMPTS_PLAN / 64], s_sum[PROMPTS_LENGTHS], s_longest;
    __shared__ unsigned long long s_all;
    __shared__ int4 s_tile[PROMPTS_PLAN];
    const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
    auto before = [&](int x, int *all) {   // the sum over smaller threads, and over all
        int sum = x;
#pragma unroll
        for (int j = 1; j < 64; j <<= 1) {
            const int y = __shfl_up(sum, j);
            if (lane >= j) sum += y;
        }
        __syncthreads();
        if (lane == 63) s_wave[wave] = sum;
        __syncthreads();
        int less = sum - x, total = 0;
        for (int j = 0; j < (int)blockDim.x / 64; ++j) {
            less += j < wave ? s_wave[j] : 0;
            total += s_wave[j];
        }
        *all = total;
        return less;
    };
    if (i < PROMPTS_LENGTHS) s_sum[i] = 0;   // (there is a wave at least)
    if (i == 0) s_longest = 0, s_all = 0;
    int tiles;
    const int mine = i < p.prompts ? (prompts_length(p, i) * p.group + rows - 1) / rows : 0;
    const int first = before(min(mine, PROMPTS_PLAN + 1), &tiles);
    tiles = min(tiles, most);   // (starts in no order may give more: there is no room for them)
    s_first[i] = first;
    __syncthreads();
    int prompt = 0, tile = 0, steps = 0;
    if (i < tiles) {
#pragma unroll
        for (int w = PROMPTS_PLAN / 2; w > 0; w /= 2)
            if (prompt + w < p.prompts && s_first[prompt + w] <= i) prompt += w;
        const PromptsAt at = prompts_at(p, prompt);
        const int count = (at.n * p.group + rows - 1) / rows;
        tile = count - 1 - (i - s_first[prompt]);   // (a prompt's last tiles, which have the most keys, first)
        steps = (at.past + (min(tile * rows + rows, at.n * p.group) - 1) / p.group + 1 + step - 1) / step;
    }
    int64_t all_steps = steps;
    int most_steps = steps;
#pragma unroll
    for (int k = 1; k < 64; k <<= 1) all_steps += __shfl_xor(all_steps, k), most_steps = max(most_steps, __shfl_xor(most_steps, k));
    if (lane == 0 && most_steps > 0) {
        atomicAdd(&s_all, (unsigned long long)all_steps);
        atomicMax(&s_longest, most_steps);
    }
    __syncthreads();
    const int longest = max(s_longest, 1);
    const int64_t all = (int64_t)s_all, share = max((all * p.kv_heads + slots - 1) / slots, (int64_t)PROMPTS_LEAST * PROMPTS_PIECES);
    // a lane a length, and a quarter of the wave's tiles
    const int part = prompts_parts[lane & (PROMPTS_LENGTHS - 1)], length = part ? (int)min((int64_t)longest, (share * part + 63) / 64) : longest;
    if (wave * 64 < tiles) {
        int n = 0;
        for (int k = 0; k < PROMPTS_LENGTHS; ++k) n += (int)((unsigned)(__shfl(steps, (lane & ~(PROMPTS_LENGTHS - 1)) + k) + length - 1) / (unsigned)length);   // (of no tile: none)
        n += __shfl_xor(n, 16);
        n += __shfl_xor(n, 32);
        if (lane < PROMPTS_LENGTHS) atomicAdd(&s_sum[lane], n);
    }
    __syncthreads();
    const float n = (float)max(s_sum[lane & (PROMPTS_LENGTHS - 1)], 1), turns = n * p.kv_heads / slots;
    float least = (turns <= 1.f ? length + 8.f : ceilf(turns) * ((float)all / n + 8.f)) + (length < longest ? 6.f : 0.f);
    int len = length;
#pragma unroll
    for (int k = 1; k < PROMPTS_LENGTHS; k <<= 1) {
        const float t = __shfl_xor(least, k);
        const int other = __shfl_xor(len, k);
        if (t < least || (t == least && other > len)) least = t, len = other;   // (the same for all)
    }
    const int count = i < tiles ? (steps + len - 1) / len : 0;
    int total;
    const int at = before(count, &total);
    if (i == 0) p.count[0] = total, p.count[1] = tiles;
    if (i < tiles) p.splits[i] = {prompt, tile, at, count};
    __syncthreads();
    s_first[i] = i < tiles ? at : total;   // (a tile's first piece now, and of the others what follows)
    s_tile[i] = {prompt, tile, steps, count};
    __syncthreads();
    for (int q = i; q < total; q += blockDim.x) {
        int u = 0;
#pragma unroll
        for (int w = PROMPTS_PLAN / 2; w > 0; w /= 2)
            if (u + w < tiles && s_first[u + w] <= q) u += w;
        const int4 x = s_tile[u];
        const int j = q - s_first[u];
        const int even = (int)((unsigned)x.z / (unsigned)x.w), rest = x.z - even * x.w;   // (the first ones have a step more)
        p.pieces[q] = {x.x, x.y, even * j + min(j, rest), even * (j + 1) + min(j + 1, rest), x.w > 1};
    }
}

// The pieces of a tile and key head: four rows of a wave at a time where heads are of 64, a row's numbers by lanes side by side
template <class T>
__global__ void __launch_bounds__(256)
k_prompts_join(PromptsP p, int rows) {
    const int kvh = (int)blockIdx.x % p.kv_heads, u = (int)blockIdx.x / p.kv_heads;
    if (u >= p.count[1]) return;
    const PromptsSplit s = p.splits[u];
    if (s.count <= 1) return;
    const PromptsAt at = prompts_at(p, s.prompt);
    int lanes = 2;   // of a row, four numbers each
    while (lanes * 4 < p.dim) lanes *= 2;
    const int d = (threadIdx.x & (lanes - 1)) * 4, step = 256 / lanes * gridDim.y;
    for (int r = blockIdx.y * (256 / lanes) + threadIdx.x / lanes; r < rows; r += step) {
        const int row = s.tile * rows + r, token = row / p.group;
        if (row >= at.n * p.group || d >= p.dim) continue;
        float top = -INFINITY, l = 0.f;
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int j0 = 0; j0 < s.count; j0 += 8) {   // eight pieces' sums on their way
            float2 ml[8];
            float4 x[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int64_t from = ((int64_t)(s.first + min(j0 + j, s.count - 1)) * p.kv_heads + kvh) * rows + r;
                ml[j] = *(const float2 *)(p.part_ml + from * 2);
                x[j] = *(const float4 *)(p.part_o + from * p.dim + d);
            }
            float m = top;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = fmaxf(m, ml[j].x);
            const float a = top == m ? 1.f : __builtin_amdgcn_exp2f(top - m);
            top = m;
            l *= a;
            o = make_float4(o.x * a, o.y * a, o.z * a, o.w * a);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (j0 + j >= s.count) continue;
                const float b = ml[j].x == m ? 1.f : __builtin_amdgcn_exp2f(ml[j].x - m);
                l += ml[j].y * b;
                o = make_float4(o.x + x[j].x * b, o.y + x[j].y * b, o.z + x[j].z * b, o.w + x[j].w * b);
            }
        }
        float f = l == 0.f ? 0.f : 1.f / l;
        if (!(fabsf(o.x) < INFINITY && fabsf(o.y) < INFINITY && fabsf(o.z) < INFINITY && fabsf(o.w) < INFINITY)) {   // a sum beyond float32, where the mean may not be: each piece by its share
            o = make_float4(0.f, 0.f, 0.f, 0.f);
            for (int j = 0; j < s.count; ++j) {
                const int64_t from = ((int64_t)(s.first + j) * p.kv_heads + kvh) * rows + r;
                const float mj = p.part_ml[from * 2], b = (mj == top ? 1.f : __builtin_amdgcn_exp2f(mj - top)) * f;
                const float4 x = *(const float4 *)(p.part_o + from * p.dim + d);
                o = make_float4(o.x + x.x * b, o.y + x.y * b, o.z + x.z * b, o.w + x.w * b);
            }
            f = 1.f;
        }
        const T y[4] = {(T)(l == 0.f ? 0.f : o.x * f), (T)(l == 0.f ? 0.f : o.y * f), (T)(l == 0.f ? 0.f : o.z * f), (T)(l == 0.f ? 0.f : o.w * f)};
        __builtin_memcpy((T *)(p.out + (int64_t)(at.start + token) * p.o_row + (kvh * p.group + row - token * p.group) * p.o_head) + d, y, sizeof y);
    }
}

// How a call is done: whether the keys of a tile are shared out, and how many there are at most: tiles; tiles, or pieces, and one more
struct PromptsForm {
    bool shared;
    int64_t tiles, units;
};

// Shared out where there are few workgroups for their keys: the plan and the join take about 14 us, a piece's sums go through memory, and a turn that is not full is waited for.  The
// longest prompt is the largest that the tables can hold, or the mean one.  (A tile a workgroup and shared, bfloat16, at blocks by slots.  32 heads on 8 of 128, four
// prompts behind 8000 each: 0.3 235 and 113 us, 0.6 239 and 199, 0.8 275 and 291, 1.1 305 and 341; behind 500 to 8000: 0.6 244 and 140, 0.8 243 and 189, 1.1 265 and 232, 1.3 257 and 278.  One of
// 4000, nothing before it: 0.5 101 and 89, 0.7 103 and 105, 1.0 106 and 126.  One of 1000, 8 heads of 64: 28 and 21; two of 1000, 16 heads on 4, 31 and 40; 8 of one token behind
// 1500: 52 and 25.)
static PromptsForm prompts_form(const tbs_attend_prompts_args &a, int force) {
    const int group = a.heads / a.kv_heads;
    PromptsForm f = {};
    f.tiles = (int64_t)a.tokens * group / (32 * PROMPTS_WAVES) + a.prompts;
    const int64_t longest = a.past ? (int64_t)a.table_width * a.page : a.prompts > 0 ? a.tokens / a.prompts : 0, blocks = f.tiles * a.kv_heads, slots = prompts_slots(a);
    const bool few = longest >= 768 && blocks * 4096 < slots * std::min<int64_t>(longest, a.past ? 4096 : 2867);
    f.shared = f.tiles <= PROMPTS_PLAN && a.prompts > 0 && (force ? force == 2 : few);
    f.units = f.tiles + 1;
    if (f.shared) {   // a piece is a quarter of an equal share of all steps, or more, and four steps or a whole tile
        const int64_t keys = (a.past ? (int64_t)a.table_width * a.page : 0) + a.tokens, step = PROMPTS_LEAST * (a.dtype == TBS_F32 || a.dim > 128 ? 32 : 64);
        f.units += std::min<int64_t>(slots * PROMPTS_PIECES / a.kv_heads + 1, f.tiles * ((keys + step - 1) / step - 1));
    }
    return f;
}

struct PromptsSpace {
    int64_t pieces, splits, o, ml, bytes;
};

static PromptsSpace prompts_space(const tbs_attend_prompts_args &a, const PromptsForm &f) {
    PromptsSpace s = {};
    if (!f.shared) return s;
    const int64_t rows = f.units * a.kv_heads * 32 * PROMPTS_WAVES;
    auto after = [](int64_t at, int64_t n) { return (at + n + 15) / 16 * 16; };
    s.pieces = 16;
    s.splits = after(s.pieces, f.units * (int64_t)sizeof(PromptsPiece));
    s.ml = after(s.splits, PROMPTS_PLAN * (int64_t)sizeof(PromptsSplit));
    s.o = after(s.ml, rows * 8);
    s.bytes = after(s.o, rows * a.dim * 4);
    return s;
}

template <class T, int DP>
static hipError_t prompts_launch(const PromptsP &p, const tbs_attend_prompts_args &a, const PromptsForm &f, hipStream_t st) {
    const int64_t blocks = f.units * a.kv_heads;
    if (blocks > INT32_MAX) return hipErrorInvalidValue;
    const dim3 grid((unsigned)blocks), block(64 * PROMPTS_WAVES);
    if (f.shared) {
        hipLaunchKernelGGL(k_prompts_plan, dim3(1), dim3((unsigned)(f.tiles + 63) / 64 * 64), 0, st,   // (tiles: no fewer than prompts)
                           p, 32 * PROMPTS_WAVES, PromptsTile<T, DP>::KEYS, (int)f.tiles, prompts_slots(a));
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (f.shared) hipLaunchKernelGGL((k_prompts<T, DP, true>), grid, block, 0, st, p);
    else hipLaunchKernelGGL((k_prompts<T, DP, false>), grid, block, 0, st, p);
    if (f.shared) {
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((k_prompts_join<T>), dim3((unsigned)(f.tiles * a.kv_heads), 16), dim3(256), 0, st, p, 32 * PROMPTS_WAVES);
    }
    return hipGetLastError();
}

template <class T>
static hipError_t prompts_dims(const PromptsP &p, const tbs_attend_prompts_args &a, const PromptsForm &f, hipStream_t st) {
    if (p.dim <= 32) return prompts_launch<T, 32>(p, a, f, st);
    if (p.dim <= 64) return prompts_launch<T, 64>(p, a, f, st);
    if (p.dim == 80) return prompts_launch<T, 80>(p, a, f, st);
    if (p.dim <= 96) return prompts_launch<T, 96>(p, a, f, st);
    if (p.dim <= 128) return prompts_launch<T, 128>(p, a, f, st);
    return prompts_launch<T, 256>(p, a, f, st);
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
    return args->tokens == 0 ? 0 : prompts_space(*args, prompts_form(*args, 0)).bytes;
}

// force: 0 = by the rule, 1 = a workgroup a tile, 2 = the keys shared out
static int prompts_call(const tbs_attend_prompts_args *args, int force, void *stream) {
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
    // Addresses in the cache: a page's number times 32 bits, a place in the page of 32 bits.
    const int64_t wide[] = {a.k_cache_token * es * a.page, a.v_cache_token * es * a.page, a.k_cache_page * es, a.v_cache_page * es};
    for (int i = 0; i < (a.past ? a.pages > 1 ? 4 : 2 : 0); ++i)
        if (wide[i] > UINT32_MAX - 8192ll) return TBS_EINVAL;
    // ... and of direct loads from new tokens 32 bits from a tile's first; rows that are further apart than that go through registers
    if (a.tokens > 1 && (a.k_row * es * 64 > INT32_MAX || a.v_row * es * 64 > INT32_MAX)) direct = false;
    // what is written lies neither over itself nor over what others read; queries are read by those who write in their place
    const OpHeads q = {a.q, a.tokens, a.heads, a.dim, a.q_row, a.q_head}, out = {a.out, a.tokens, a.heads, a.dim, a.out_row, a.out_head};
    if (op_folded(out) || (!op_same(q, out) && op_overlap(out, q, es)) || op_overlap(out, {a.k, a.tokens, a.kv_heads, a.dim, a.k_row, a.k_head}, es) ||
        op_overlap(out, {a.v, a.tokens, a.kv_heads, a.dim, a.v_row, a.v_head}, es) || op_overlap(out, op_plain(a.starts, 1, 0, 4ll * a.prompts + 4, es), es) ||
        op_overlap(out, op_plain(a.past, 1, 0, 4ll * a.prompts, es), es) || op_overlap(out, op_plain(a.tables, a.prompts, a.ld_tables * 4, 4ll * a.table_width, es), es))
        return TBS_EINVAL;
    if (a.past && (op_overlap(OpCache{a.k_cache, a.pages, a.page, a.kv_heads, a.dim, a.k_cache_page, a.k_cache_token, a.k_cache_head}, out, es) ||
                   op_overlap(OpCache{a.v_cache, a.pages, a.page, a.kv_heads, a.dim, a.v_cache_page, a.v_cache_token, a.v_cache_head}, out, es)))
        return TBS_EINVAL;
    const PromptsForm f = prompts_form(a, force);
    const PromptsSpace space = prompts_space(a, f);
    if (space.bytes > 0 && (!a.workspace || a.workspace_bytes < space.bytes || (uintptr_t)a.workspace % 16)) return TBS_EINVAL;
    PromptsP p = {};
    if (f.shared) {
        char *w = (char *)a.workspace;
        p.count = (int *)w, p.pieces = (PromptsPiece *)(w + space.pieces), p.splits = (PromptsSplit *)(w + space.splits), p.part_ml = (float *)(w + space.ml), p.part_o = (float *)(w + space.o);
    }
    p.q = (const char *)a.q, p.k = (const char *)a.k, p.v = (const char *)a.v, p.k_cache = (const char *)a.k_cache, p.v_cache = (const char *)a.v_cache, p.out = (char *)a.out;
    p.starts = a.starts, p.past = a.past, p.tables = a.tables;
    p.q_row = a.q_row * es, p.q_head = a.q_head * es, p.k_row = a.k_row * es, p.k_head = a.k_head * es, p.v_row = a.v_row * es, p.v_head = a.v_head * es;
    p.o_row = a.out_row * es, p.o_head = a.out_head * es;
    p.kp = (unsigned)(a.k_cache_page * es), p.kt = (unsigned)(a.k_cache_token * es), p.kh = a.k_cache_head * es;
    p.vp = (unsigned)(a.v_cache_page * es), p.vt = (unsigned)(a.v_cache_token * es), p.vh = a.v_cache_head * es;
    p.ld_tables = a.ld_tables;
    p.tokens = a.tokens, p.prompts = a.prompts, p.heads = a.heads, p.kv_heads = a.kv_heads, p.group = a.heads / a.kv_heads, p.dim = a.dim;
    p.page = a.past ? a.page : 1, p.pages = a.pages, p.width = a.table_width;
    const unsigned twice = 2 * (unsigned)p.page, lg = 31 - __builtin_clz(twice);
    p.page_shift = (twice & (twice - 1)) ? lg : 0;
    p.page_mul = (unsigned)((((uint64_t)1 << (32 + p.page_shift)) / twice) + (p.page_shift ? 1 : 0));
    p.direct = direct;
    const float scale = a.scale != 0.f ? a.scale : 1.f / sqrtf((float)a.dim);
    p.scale2 = fabsf(scale) * 1.44269504f;
    p.flip = scale < 0.f ? (a.dtype == TBS_F32 ? 0x80000000u : 0x80008000u) : 0;
    const hipStream_t st = (hipStream_t)stream;
    const hipError_t e = a.dtype == TBS_F32 ? prompts_dims<float>(p, a, f, st) : a.dtype == TBS_BF16 ? prompts_dims<__bf16>(p, a, f, st) : prompts_dims<_Float16>(p, a, f, st);
    return e == hipSuccess ? TBS_OK : e == hipErrorInvalidValue ? TBS_EINVAL : TBS_EHIP;
}

extern "C" int tbs_attend_prompts(const tbs_attend_prompts_args *args, void *stream) { return prompts_call(args, 0, stream); }

// one way of splitting the work, for the tests (not in the header)
extern "C" int prompts_by(const tbs_attend_prompts_args *args, int force, void *stream) { return prompts_call(args, force, stream); }
extern "C" int64_t prompts_by_workspace(const tbs_attend_prompts_args *args, int force) { return prompts_space(*args, prompts_form(*args, force)).bytes; }
