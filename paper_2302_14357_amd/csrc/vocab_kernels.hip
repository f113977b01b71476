// The best continuations of groups of hypotheses over a vocabulary (no transducer blank): scores + log softmax(logits), the best
// `beams` of beams x vocabulary.
//
// One launch for small vocabularies (k_vocab_small), else two.  k_vocab_part reads the logits once, a workgroup a slice of at most 8192 of a row, in registers: its maximum, sum of
// exponentials and best candidates.  k_vocab_join has a workgroup a group: the slices' sums give each row's normaliser, their lists its best
// logits, and the rows' lists the group's best scores.
#include "op_device.h"

typedef unsigned long long vk_u64;

#define VOC_SLICE 8192
#define VOC_ELEMS (VOC_SLICE / 256)
#define VOC_SMALL (64 * VOC_ELEMS)
#define VOC_SPLITS (TBS_MAX_VOCAB / VOC_SLICE)   // at most a wave's lanes

struct VocabP {
    const void *logits;
    const double *scores;
    const uint8_t *finished;
    double *out_scores;
    int *out_tokens, *out_parents;
    uint8_t *out_finished;
    double *sum;      // [rows, splits] sum of e^(l - max)
    float *top;       // [rows, splits] max; NaN: the slice has a logit that is NaN or +inf
    float *val;       // [rows, splits, beams] best logits, then their tokens
    int *tok;
    int64_t ld;
    int rows, beams, vocab, eos, splits, slice;
};

// e^x for -690 <= x <= 0, in float64: 2^(k + f), |f| <= 1/2, 2^f by the polynomial of degree 8 that agrees with it in nine Chebyshev
// points (relative error 1.1e-12).  k and its place in the exponent come out of the addition of 1.5 2^52.  Scores of different hypotheses
// are compared, so what a float32 exponential loses (1e-8 of a normaliser) could put near ones in the wrong order; float64 instructions
// run at float32's rate here.
__device__ __forceinline__ double voc_exp(double x) {
    const double magic = 6755399441055744.0;
    const double z = fma(x, 1.4426950408889634, magic), f = fma(x, 1.4426950408889634, magic - z);
    double y = 1.3255179556479267e-06;
    y = fma(y, f, 1.5310080611926545e-05);
    y = fma(y, f, 0.00015403456082633648);
    y = fma(y, f, 0.0013333450563173552);
    y = fma(y, f, 0.009618129159053034);
    y = fma(y, f, 0.055504109412108156);
    y = fma(y, f, 0.24022650695814518);
    y = fma(y, f, 0.6931471805459332);
    y = fma(y, f, 1.0000000000000004);
    return __hiloint2double(__double2hiint(y) + (__double2loint(z) << 20), __double2loint(y));
}

// numbers in the order of whole numbers (no NaN; -0 is made 0 before)
__device__ __forceinline__ unsigned voc_key(float v) {
    const unsigned u = __float_as_uint(v);
    return u ^ (unsigned)(((int)u >> 31) | 0x80000000);
}
__device__ __forceinline__ float voc_unkey(unsigned k) { return __uint_as_float(k & 0x80000000 ? k ^ 0x80000000 : ~k); }

__device__ __forceinline__ vk_u64 voc_shfl_xor(vk_u64 v, int i) {
    return (vk_u64)__shfl_xor((unsigned)(v >> 32), i) << 32 | (unsigned)__shfl_xor((unsigned)v, i);
}

// The other operand of a reduction over the wave that any order of lanes serves, step 0 to 5: lanes 1 and 2 away, mirrored in 8 and in 16, and
// rows of 16 and halves exchanged; all without LDS.
typedef unsigned voc_uint2 __attribute__((ext_vector_type(2)));
template <int STEP>
__device__ __forceinline__ unsigned voc_other(unsigned x) {
    if constexpr (STEP < 4) {
        constexpr int CTRL[4] = {0xB1, 0x4E, 0x141, 0x140};   // quad_perm 1 0 3 2, quad_perm 2 3 0 1, row_half_mirror, row_mirror
        return __builtin_amdgcn_update_dpp(0u, x, CTRL[STEP], 0xF, 0xF, true);
    } else {
        const voc_uint2 u = STEP == 4 ? __builtin_amdgcn_permlane16_swap(x, x, false, false) : __builtin_amdgcn_permlane32_swap(x, x, false, false);
        const bool upper = (threadIdx.x & (STEP == 4 ? 16 : 32)) != 0;   // (u[0]: the lower row or half in both, u[1]: the upper)
        return upper ? u[0] : u[1];
    }
}
template <int STEP = 0>
__device__ __forceinline__ float voc_max(float x) {
    if constexpr (STEP == 6) return x;
    else return voc_max<STEP + 1>(fmaxf(x, __uint_as_float(voc_other<STEP>(__float_as_uint(x)))));
}
template <int STEP = 0>
__device__ __forceinline__ double voc_add(double x) {
    if constexpr (STEP == 6) return x;
    else return voc_add<STEP + 1>(x + __hiloint2double((int)voc_other<STEP>((unsigned)__double2hiint(x)), (int)voc_other<STEP>((unsigned)__double2loint(x))));
}

// what lanes of a wave wrote to LDS is there for its others
__device__ __forceinline__ void voc_wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// A wave's N best of `used` numbers a lane, those from `from` on, one after the other: for many equal ones.
template <int ELEMS, class Token>
__device__ __forceinline__ void voc_wave_slow(float (&v)[ELEMS], float from, int used, int N, vk_u64 *best, Token token) {
    for (int i = 0; i < N; ++i) {
        vk_u64 k = 0;
        const vk_u64 before = i > 0 ? best[i - 1] : ~0ull;
        int zero = 0;
        asm volatile("" : "+v"(zero));   // (made anew each time: 32 keys kept over the loop would cost every call its registers)
#pragma unroll
        for (int j = 0; j < ELEMS; ++j) {
            asm volatile("" : "+v"(v[j]));
            const vk_u64 kj = (vk_u64)voc_key(v[j]) << 32 | (unsigned)~token(j, zero);
            if (j < used && v[j] >= from && kj > k && kj < before) k = kj;
        }
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) k = max(k, voc_shfl_xor(k, x));
        if ((threadIdx.x & 63) == 0) best[i] = k;
        voc_wave_sync();
    }
}

// The numbers of a wave from `from` on, as keys, into cand (64 at most are written); how many they are.
template <int ELEMS, class Token>
__device__ __forceinline__ int voc_collect(const float (&v)[ELEMS], float from, int used, vk_u64 *cand, Token token) {
    int found = 0;
#pragma unroll
    for (int j = 0; j < ELEMS; ++j) {
        if (j >= used) continue;
        const vk_u64 m = __ballot(v[j] >= from);
        if (m) {
            const int at = found + (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)m, 0));
            if (v[j] >= from && at < 64) cand[at] = (vk_u64)voc_key(v[j]) << 32 | (unsigned)~token(j, 0);
            found += __popcll(m);
        }
    }
    return found;
}

// how many of a list's `count` keys are better than k (eight reads of LDS on their way; a list has room for 64)
__device__ __forceinline__ int voc_rank(const vk_u64 *list, int count, vk_u64 k) {
    int rank = 0;
    for (int i = 0; i < count; i += 8)
#pragma unroll
        for (int j = 0; j < 8; ++j) rank += i + j < count && list[i + j] > k;
    return rank;
}

// the N-th largest of a wave's numbers, `used` a lane, if it is `from` or more
template <int ELEMS>
__device__ __forceinline__ float voc_nth(const float (&v)[ELEMS], float from, int used, int N) {
    unsigned least = 0;
#pragma unroll 1
    for (int b = 31; b >= 0; --b) {
        const unsigned t = least | 1u << b;
        const float x = voc_unkey(t);   // (no number at all: nothing is as large)
        int count = 0;
#pragma unroll
        for (int j = 0; j < ELEMS; ++j)
            if (j < used) count += __popcll(__ballot(v[j] >= x));
        if (count >= N) least = t;
    }
    return fmaxf(from, voc_unkey(least));
}

// A wave's N best of `used` numbers a lane, best first, into best[0 .. N) in LDS: keys of (number, the lower token first), 0 where there are fewer
// above -inf.  At least N lanes have a maximum of `least` or more, so the N best are among the numbers from there on: the N-th
// largest lane maximum, cut to its first 16 bits (what a bf16 has), found bit by bit.  They are collected, at most 64 of them, and a lane
// each finds its rank by counting.  More than 64 are collected from the N-th largest number on, and taken one after the other if they are more than that still (many equal
// logits).
template <int ELEMS, class Token>
__device__ __forceinline__ void voc_wave_best(float (&v)[ELEMS], float mine, int used, int N, vk_u64 *cand, vk_u64 *best, Token token) {
    const int lane = threadIdx.x & 63;
    unsigned least = 0;
    const unsigned key = voc_key(mine);
#pragma unroll
    for (int b = 31; b >= 16; --b) {
        const unsigned t = least | 1u << b;
        if (__popcll(__ballot(key >= t)) >= N) least = t;
    }
    float from = voc_unkey(max(least, voc_key(-INFINITY) + 1));   // (-inf is no candidate)
    int found = voc_collect(v, from, used, cand, token);
    if (found > 64) {
        from = voc_nth(v, from, used, N);
        found = voc_collect(v, from, used, cand, token);
    }
    if (lane < N) best[lane] = 0;
    voc_wave_sync();
    if (found <= 64) {
        const vk_u64 k = lane < found ? cand[lane] : 0;
        const int rank = voc_rank(cand, found, k);
        if (lane < found && rank < N) best[rank] = k;
        voc_wave_sync();
    } else {
        voc_wave_slow(v, from, used, N, best, token);
    }
}

// `count` logits, pieces of 16 bytes dealt out to `threads` threads one after the other; -inf behind the last
template <class T>
__device__ __forceinline__ void voc_load(const T *l, int count, int threads, float (&v)[VOC_ELEMS]) {
    constexpr int E = OpPiece<T>::E, P = VOC_ELEMS / E;
    const int mine = (int)threadIdx.x % threads * E;
    if (count == threads * VOC_ELEMS) {   // the loads leave together
        uint4 u[P];
#pragma unroll
        for (int i = 0; i < P; ++i) u[i] = op_load16(l + mine + i * threads * E);
#pragma unroll
        for (int i = 0; i < P; ++i) {
            T e[E];
            __builtin_memcpy(e, &u[i], 16);
#pragma unroll
            for (int j = 0; j < E; ++j) v[i * E + j] = op_float(e[j]) + 0.f;   // (+ 0: -0 and 0 are equal logits)
        }
        return;
    }
#pragma unroll
    for (int i = 0; i < P; ++i) {
        const int at = i * threads * E + mine;
        uint4 u = make_uint4(0, 0, 0, 0);
        if (at + E <= count) u = op_load16(l + at);
        T e[E];
        __builtin_memcpy(e, &u, 16);
        if (at < count && at + E > count)
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (at + j < count) e[j] = l[at + j];
#pragma unroll
        for (int j = 0; j < E; ++j) v[i * E + j] = at + j < count ? op_float(e[j]) + 0.f : -INFINITY;
    }
}

// a lane's maximum, and the wave's: NaN where one of its logits is NaN or +inf
__device__ __forceinline__ float voc_top(const float (&v)[VOC_ELEMS], float &mine) {
    mine = -INFINITY;
    int largest = INT32_MIN;   // as whole numbers +inf and positive NaN come behind all others, without a sign negative NaN do
    unsigned last = 0;
#pragma unroll
    for (int j = 0; j < VOC_ELEMS; ++j) {
        mine = fmaxf(mine, v[j]);
        largest = max(largest, __float_as_int(v[j]));
        last = max(last, __float_as_uint(v[j]));
    }
    const float top = voc_max(mine);
    return __any(largest >= 0x7F800000 || last > 0xFF800000u) ? NAN : top;
}

// the wave's sum of e^(v - top), `used` numbers a lane (top: not -inf)
template <int E>
__device__ __forceinline__ double voc_sum(const float (&v)[VOC_ELEMS], float top, int used) {
    double sum = 0.;
#pragma unroll
    for (int i = 0; i < VOC_ELEMS / E; ++i)
        if (i * E < used)
#pragma unroll
            for (int j = 0; j < E; ++j) sum += voc_exp(fmax((double)v[i * E + j] - (double)top, -690.));   // (e^-690 for nothing at all: 1e-300)
    return voc_add(sum);
}

// A slice's best: as voc_wave_best, with the line drawn by all 256 lane maxima, so that the four waves together collect little more than N.
// Eight waves a SIMD: a slice's loads wait behind other slices' arithmetic.  (512 rows of 131000 in float32, groups of 16: 75 to 79 us, 3.5 TB/s; the float64
// exponentials, sixteen instructions a logit, are most of what keeps the vector units busy for 69 % of that.  Slices of 4096 100 us; waves that go on through 32768 each with a list
// of its own 106.)
template <class T>
__global__ void __launch_bounds__(256, 8)
k_vocab_part(VocabP p) {
    constexpr int E = OpPiece<T>::E, PASS = 256 * E;
    __shared__ vk_u64 s_cand[4][64], s_best[4][TBS_MAX_BEAM];
    __shared__ double s_sum[4];
    __shared__ float s_top[4];
    __shared__ int s_found[4];
    __shared__ __attribute__((aligned(8))) uint16_t s_key[256];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.y, split = blockIdx.x;
    if (p.finished && p.finished[row]) return;   // (nobody reads its lists)
    const int v0 = split * p.slice, count = min(p.slice, p.vocab - v0), N = p.beams, used = (count + PASS - 1) / PASS * E;
    auto token = [&](int j, int zero) { return v0 + tid * E + zero + (j / E) * PASS + j % E; };
    float v[VOC_ELEMS], mine;
    voc_load((const T *)p.logits + row * p.ld + v0, count, 256, v);
    float top = voc_top(v, mine);
    if (lane == 0) s_top[wave] = top;
    s_key[tid] = (uint16_t)(voc_key(mine) >> 16);
    if (lane < N) s_best[wave][lane] = 0;
    __syncthreads();
    unsigned k4[4], least = 0;
    {
        const uint2 u = *reinterpret_cast<const uint2 *>(s_key + 4 * lane);
        k4[0] = u.x & 0xFFFF, k4[1] = u.x >> 16, k4[2] = u.y & 0xFFFF, k4[3] = u.y >> 16;
    }
#pragma unroll
    for (int b = 15; b >= 0; --b) {
        const unsigned t = least | 1u << b;
        if (__popcll(__ballot(k4[0] >= t)) + __popcll(__ballot(k4[1] >= t)) + __popcll(__ballot(k4[2] >= t)) + __popcll(__ballot(k4[3] >= t)) >= N) least = t;
    }
    const float from = voc_unkey(max(least << 16, voc_key(-INFINITY) + 1));   // (-inf is no candidate)
    const int found = voc_collect(v, from, used, s_cand[wave], token);
    if (lane == 0) s_found[wave] = found;
    top = s_top[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) top = top != top || s_top[i] != s_top[i] ? NAN : fmaxf(top, s_top[i]);
    const double sum = top > -INFINITY ? voc_sum<E>(v, top, used) : 0.;
    if (lane == 0) s_sum[wave] = sum;
    __syncthreads();
    const int n[4] = {s_found[0], s_found[1], s_found[2], s_found[3]}, all = n[0] + n[1] + n[2] + n[3];
    const int64_t list = ((int64_t)row * p.splits + split) * N;
    auto put = [&](int rank, vk_u64 k) {
        p.val[list + rank] = k ? voc_unkey((unsigned)(k >> 32)) : -INFINITY;
        p.tok[list + rank] = (int)~(unsigned)k;
    };
    if (all <= 64) {   // (the same for every wave) one of them has a lane each
        if (wave == 0) {
            const int w = lane < n[0] ? 0 : lane < n[0] + n[1] ? 1 : lane < n[0] + n[1] + n[2] ? 2 : 3;
            const vk_u64 k = lane < all ? s_cand[w][lane - (w > 0 ? n[0] : 0) - (w > 1 ? n[1] : 0) - (w > 2 ? n[2] : 0)] : 0;
            int rank = 0;
#pragma unroll
            for (int i = 0; i < 4; ++i)
                for (int j = 0; j < n[i]; ++j) rank += s_cand[i][j] > k;
            if (lane < all && rank < N) put(rank, k);
            if (lane < N && lane >= all) put(lane, 0);
        }
    } else {
        voc_wave_slow(v, from, used, N, s_best[wave], token);
        __syncthreads();
        // the four waves' lists: a key's rank is its place in its own and the larger ones in the others
        if (lane < N) {
            const vk_u64 k = s_best[wave][lane];
            int rank = lane;
#pragma unroll
            for (int w = 1; w < 4; ++w) {
                const vk_u64 *b = s_best[(wave + w) & 3];
                int lo = 0, hi = N;   // keys before lo are larger, from hi on they are not
                while (lo < hi) {
                    const int mid = (lo + hi) >> 1;
                    if (b[mid] > k || (b[mid] == k && ((wave + w) & 3) < wave)) lo = mid + 1;   // (equal: 0, no candidate)
                    else hi = mid;
                }
                rank += lo;
            }
            if (rank < N) put(rank, k);
        }
    }
    if (tid == 0) {
        p.sum[row * p.splits + split] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
        p.top[row * p.splits + split] = top;
    }
}

// A row's list from its N best keys: scores, tokens (a lane each).  The row has none where its maximum is NaN or -inf.
__device__ __forceinline__ void voc_row(int lane, int N, const vk_u64 *best, double score, float top, double sum, double *scores, int *tokens) {
    if (lane >= N) return;
    const vk_u64 k = best[lane];
    const double lse = (double)top + log(sum), x = score + ((double)voc_unkey((unsigned)(k >> 32)) - lse);
    const bool there = k != 0 && top > -INFINITY && x > -INFINITY;
    scores[lane] = there ? x : -INFINITY;
    tokens[lane] = there ? (int)~(unsigned)k : -1;
}

__device__ __forceinline__ void voc_row_finished(int lane, int N, double score, int eos, double *scores, int *tokens) {
    if (lane >= N) return;
    scores[lane] = lane == 0 && score > -INFINITY ? score : -INFINITY;
    tokens[lane] = eos;
}

// The group's N best of its rows' lists.  The entry at place e of a list (sorted, from 0) to which the entries at place e of h others are better (the lower
// row first at a tie) has h (e + 1) + e better ones at least: only N + N / 2 + N / 3 + ... entries are looked at further, 119 of 1024 for 32.  An entry's rank is its place
// in its own list and the better ones in the others, a binary search in each of them, a thread an entry and another row: the searches' steps wait
// for LDS, so as many as can run beside each other.
struct VocGroup {
    int count, entry[128], rank[128];
};
template <int STRIDE>
__device__ __forceinline__ void voc_group(const VocabP &p, int64_t r0, const double (*scores)[STRIDE], const int (*tokens)[STRIDE], VocGroup &g) {
    const int N = p.beams, tid = threadIdx.x, entries = N * N;
    const bool all = entries <= 128;   // (looking at all of them took 1 us less of five rows of 32001, 0.7 of ten of 50000; at some, 50 us less of 32 of 131000)
    if (tid == 0) g.count = all ? entries : 0;
    if (!all) __syncthreads();   // (the lists are complete, too)
    for (int i = tid; i < entries; i += blockDim.x) {
        const int row = i / N, e = i - row * N;
        if (all) {
            g.entry[i] = row << 8 | e;
            g.rank[i] = e;
            continue;
        }
        const double x = scores[row][e];
        int h = 0;
#pragma unroll 8
        for (int r = 0; r < N; ++r) {
            const double y = scores[r][e];
            h += y > x || (y == x && r < row);
        }
        if (h * (e + 1) + e < N) {
            const int at = atomicAdd(&g.count, 1);   // (in any order)
            g.entry[at] = row << 8 | e;
            g.rank[at] = e;
        }
    }
    __syncthreads();
    const int count = g.count;
    for (int i = tid; i < count * N; i += blockDim.x) {
        const int at = i / N, r = i - at * N, row = g.entry[at] >> 8;
        if (r == row) continue;
        const double x = scores[row][g.entry[at] & 255];
        int lo = 0, hi = N;
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            const double y = scores[r][mid];
            if (y > x || (y == x && r < row)) lo = mid + 1;
            else hi = mid;
        }
        if (lo > 0) atomicAdd(&g.rank[at], lo);
    }
    __syncthreads();
    for (int i = tid; i < count; i += blockDim.x) {
        const int rank = g.rank[i], row = g.entry[i] >> 8, e = g.entry[i] & 255;
        if (rank >= N) continue;
        const double x = scores[row][e];
        const bool none = !(x > -INFINITY);
        const int token = none ? -1 : tokens[row][e];
        p.out_scores[r0 + rank] = x;
        p.out_tokens[r0 + rank] = token;
        p.out_parents[r0 + rank] = none ? -1 : row;
        p.out_finished[r0 + rank] = none || token == p.eos || (p.finished && p.finished[r0 + row]);
    }
}

// Rows' lists from their slices' (a wave a row), and the group's.  (Steps that wait for each other: 5 us for 64 groups of five rows of 32001, 10 for 32 of sixteen rows
// of 131000.)
__global__ void __launch_bounds__(1024)
k_vocab_join(VocabP p) {
    __shared__ double s_score[TBS_MAX_BEAM][TBS_MAX_BEAM + 1];   // (places of one number in neighbouring lists: neighbouring LDS banks)
    __shared__ int s_token[TBS_MAX_BEAM][TBS_MAX_BEAM + 1];
    __shared__ vk_u64 s_cand[16][64], s_best[16][TBS_MAX_BEAM];
    __shared__ VocGroup s_group;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, N = p.beams;
    const int64_t r0 = (int64_t)blockIdx.x * N;
    for (int i = wave; i < N; i += waves) {
        const int64_t row = r0 + i;
        const double score = p.scores[row];
        if (p.finished && p.finished[row]) {
            voc_row_finished(lane, N, score, p.eos, s_score[i], s_token[i]);
            continue;
        }
        const bool in = lane < p.splits;
        const float top = in ? p.top[row * p.splits + lane] : -INFINITY;
        const double part = in ? p.sum[row * p.splits + lane] : 0.;
        float best = voc_max(top);
        const double sum = voc_add(top > -INFINITY ? part * exp((double)top - (double)best) : 0.);
        if (__any(top != top)) best = NAN;
        // 512 entries of the lists at a time, and the best of those before
        const int all = p.splits * N;
        const float one_n = 1.f / N;
        for (int from = 0; from < all; from += 512) {
            float v[9], mine = -INFINITY;
            int tok[9];
            const vk_u64 k = from > 0 && lane % 2 == 0 && lane / 2 < N ? s_best[wave][lane / 2] : 0;   // (theirs, too)
            v[8] = k ? voc_unkey((unsigned)(k >> 32)) : -INFINITY;
            tok[8] = (int)~(unsigned)k;
            const float *val = p.val + row * all;
            const int *token = p.tok + row * all;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                // (lists side by side, each turned by another number of places, so that their best ones are different lanes': every lane's maximum then
                // says something about where the line is)
                v[j] = -INFINITY;
                tok[j] = 0;
                if (from + j * 64 >= all) continue;
                const int at = from + j * 64 + lane, list = (int)((at + 0.5f) * one_n), turn = (list * N * N) >> 9;
                int place = at - list * N + turn - (int)((turn + 0.5f) * one_n) * N;
                place = list * N + (place >= N ? place - N : place);
                v[j] = at < all ? val[place] : -INFINITY;
                tok[j] = at < all ? token[place] : 0;
            }
#pragma unroll
            for (int j = 0; j < 9; ++j) mine = fmaxf(mine, v[j]);
            voc_wave_best(v, mine, 9, N, s_cand[wave], s_best[wave], [&](int j, int) { return tok[j]; });
        }
        voc_row(lane, N, s_best[wave], score, best, sum, s_score[i], s_token[i]);
        voc_wave_sync();
    }
    voc_group(p, r0, s_score, s_token, s_group);
}

// Vocabularies of up to 2048 and groups of up to 16: one launch, a workgroup a group, a wave a row.
template <class T>
__global__ void __launch_bounds__(1024)
k_vocab_small(VocabP p) {
    constexpr int E = OpPiece<T>::E, PASS = 64 * E;
    __shared__ double s_score[16][17];
    __shared__ int s_token[16][17];
    __shared__ vk_u64 s_cand[16][64], s_best[16][16];
    __shared__ VocGroup s_group;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), N = p.beams;
    const int64_t r0 = (int64_t)blockIdx.x * N, row = r0 + wave;
    const double score = p.scores[row];
    if (p.finished && p.finished[row]) {
        voc_row_finished(lane, N, score, p.eos, s_score[wave], s_token[wave]);
    } else {
        const int used = (p.vocab + PASS - 1) / PASS * E;
        float v[VOC_ELEMS], mine;
        voc_load((const T *)p.logits + row * p.ld, p.vocab, 64, v);
        const float top = voc_top(v, mine);
        voc_wave_best(v, mine, used, N, s_cand[wave], s_best[wave], [&](int j, int zero) { return lane * E + zero + (j / E) * PASS + j % E; });
        const double sum = top > -INFINITY ? voc_sum<E>(v, top, used) : 0.;
        voc_row(lane, N, s_best[wave], score, top, sum, s_score[wave], s_token[wave]);
    }
    voc_group(p, r0, s_score, s_token, s_group);
}

struct VocabPlan {
    int splits, slice;
    bool small;
};

static VocabPlan vocab_plan(const tbs_beam_select_args &a) {
    // One launch where a wave has a row's logits in registers (five rows of 1024: 7 us a call, by two launches 14.6).  Else slices of 8192, smaller ones (2048 at
    // least) while these are fewer than two workgroups a CU
    int64_t splits = (a.vocab + VOC_SLICE - 1) / VOC_SLICE, more = 512 / a.rows;
    if (more > (a.vocab + 2047) / 2048) more = (a.vocab + 2047) / 2048;
    if (more > VOC_SPLITS) more = VOC_SPLITS;
    if (splits < more) splits = more;
    const int pass = 256 * (int)(16 / op_dtype_size(a.dtype));
    VocabPlan pl;
    pl.small = a.vocab <= VOC_SMALL && a.beams <= 16;
    pl.slice = (int)((a.vocab + splits - 1) / splits + pass - 1) / pass * pass;
    pl.splits = (a.vocab + pl.slice - 1) / pl.slice;
    return pl;
}

static int vocab_check(const tbs_beam_select_args &a) {
    if (!op_dtype_known(a.dtype) || a.beams < 1 || a.beams > TBS_MAX_BEAM || a.rows < 0 || a.rows % a.beams || a.rows > 65535 || a.vocab < 1 ||
        a.vocab > TBS_MAX_VOCAB)
        return TBS_EINVAL;
    return TBS_OK;
}

// doubles, then floats, then whole numbers
static int64_t vocab_bytes(const tbs_beam_select_args &a, const VocabPlan &pl) {
    const int64_t lists = (int64_t)a.rows * pl.splits;
    return lists * (8 + 4 + (int64_t)a.beams * 8);
}

extern "C" int64_t tbs_beam_select_workspace(const tbs_beam_select_args *args) {
    if (!args || vocab_check(*args) != TBS_OK) return TBS_EINVAL;
    if (args->rows == 0) return 0;
    const VocabPlan pl = vocab_plan(*args);
    return pl.small ? 0 : vocab_bytes(*args, pl);
}

extern "C" int tbs_beam_select(const tbs_beam_select_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_beam_select_args &a = *args;
    if (vocab_check(a) != TBS_OK) return TBS_EINVAL;
    if (a.rows == 0) return TBS_OK;
    if (!a.logits || !a.scores || !a.out_scores || !a.out_tokens || !a.out_parents || !a.out_finished || a.ld_logits < a.vocab ||
        (uintptr_t)a.logits % op_dtype_size(a.dtype))
        return TBS_EINVAL;
    const VocabPlan pl = vocab_plan(a);
    if (!pl.small && (!a.workspace || a.workspace_bytes < vocab_bytes(a, pl) || (uintptr_t)a.workspace % 16)) return TBS_EINVAL;
    VocabP p = {};
    p.logits = a.logits, p.scores = a.scores, p.finished = a.finished;
    p.out_scores = a.out_scores, p.out_tokens = a.out_tokens, p.out_parents = a.out_parents, p.out_finished = a.out_finished;
    const int64_t lists = (int64_t)a.rows * pl.splits;
    p.sum = (double *)a.workspace;
    p.top = (float *)(p.sum + lists);
    p.val = p.top + lists;
    p.tok = (int *)(p.val + lists * a.beams);
    p.ld = a.ld_logits;
    p.rows = a.rows, p.beams = a.beams, p.vocab = a.vocab, p.eos = a.eos, p.splits = pl.splits, p.slice = pl.slice;
    const hipStream_t st = (hipStream_t)stream;
    if (pl.small) {
        const dim3 groups(a.rows / a.beams), block(64 * a.beams);
        if (a.dtype == TBS_F32) hipLaunchKernelGGL((k_vocab_small<float>), groups, block, 0, st, p);
        else if (a.dtype == TBS_BF16) hipLaunchKernelGGL((k_vocab_small<__bf16>), groups, block, 0, st, p);
        else hipLaunchKernelGGL((k_vocab_small<_Float16>), groups, block, 0, st, p);
        return hipGetLastError() == hipSuccess ? TBS_OK : TBS_EHIP;
    }
    const dim3 grid(pl.splits, a.rows);
    if (a.dtype == TBS_F32) hipLaunchKernelGGL((k_vocab_part<float>), grid, dim3(256), 0, st, p);
    else if (a.dtype == TBS_BF16) hipLaunchKernelGGL((k_vocab_part<__bf16>), grid, dim3(256), 0, st, p);
    else hipLaunchKernelGGL((k_vocab_part<_Float16>), grid, dim3(256), 0, st, p);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess) {
        hipLaunchKernelGGL(k_vocab_join, dim3(a.rows / a.beams), dim3(64 * (a.beams < 16 ? a.beams : 16)), 0, st, p);
        e = hipGetLastError();
    }
    return e == hipSuccess ? TBS_OK : TBS_EHIP;
}
