// The best continuations of groups of hypotheses over a vocabulary (no transducer blank): scores + log softmax(logits), the best
// `beams` of beams x vocabulary.
//
// Two launches.  k_vocab_part reads the logits once, a workgroup a slice of at most 8192 of a row, in registers: its maximum, sum of
// exponentials and best candidates.  k_vocab_join has a workgroup a group: the slices' sums give each row's normaliser, their lists its best
// logits, and the rows' lists the group's best scores.
#include "op_device.h"

typedef unsigned long long vk_u64;

#define VOC_SLICE 8192
#define VOC_ELEMS (VOC_SLICE / 256)
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

// what lanes of a wave wrote to LDS is there for its others
__device__ __forceinline__ void voc_wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <class T>
__global__ void __launch_bounds__(256)
k_vocab_part(VocabP p) {
    constexpr int E = OpPiece<T>::E, PASS = 256 * E, PASSES = VOC_SLICE / PASS;
    __shared__ vk_u64 s_cand[4][64], s_best[4][TBS_MAX_BEAM];
    __shared__ double s_sum[4];
    __shared__ float s_top[4];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), row = blockIdx.y, split = blockIdx.x;
    if (p.finished && p.finished[row]) return;   // (nobody reads its lists)
    const int v0 = split * p.slice, count = min(p.slice, p.vocab - v0), N = p.beams;
    const T *l = (const T *)p.logits + row * p.ld + v0;
    float v[VOC_ELEMS];
#pragma unroll
    for (int i = 0; i < PASSES; ++i) {
        const int at = i * PASS + tid * E;
        if (i * PASS < count && at + E <= count) {
            const uint4 u = op_load16(l + at);
            T e[E];
            __builtin_memcpy(e, &u, 16);
#pragma unroll
            for (int j = 0; j < E; ++j) v[i * E + j] = op_float(e[j]) + 0.f;   // (+ 0: -0 and 0 are equal logits)
        } else {
#pragma unroll
            for (int j = 0; j < E; ++j) v[i * E + j] = i * PASS < count && at + j < count ? op_float(l[at + j]) + 0.f : -INFINITY;
        }
    }
    float mine = -INFINITY;
    bool bad = false;   // NaN or +inf
#pragma unroll
    for (int j = 0; j < VOC_ELEMS; ++j) {
        mine = fmaxf(mine, v[j]);
        bad |= !(v[j] < INFINITY);
    }
    float top = mine;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) top = fmaxf(top, __shfl_xor(top, i));
    if (__any(bad)) top = NAN;
    if (lane == 0) s_top[wave] = top;
    // The wave's N best.  At least N lanes have a maximum of `least` or more, so the N best are among the elements from there on: the
    // N-th largest lane maximum, cut to its first 16 bits (what a bf16 has), found bit by bit.
    unsigned least = 0;
    const unsigned key = voc_key(mine);
#pragma unroll
    for (int b = 31; b >= 16; --b) {
        const unsigned t = least | 1u << b;
        if (__popcll(__ballot(key >= t)) >= N) least = t;
    }
    const float from = voc_unkey(max(least, voc_key(-INFINITY) + 1));   // (-inf is no candidate)
    int found = 0;
#pragma unroll
    for (int j = 0; j < VOC_ELEMS; ++j) {
        const vk_u64 m = __ballot(v[j] >= from);
        if (m) {
            const int at = found + __popcll(m & ((1ull << lane) - 1));
            if (v[j] >= from && at < 64) s_cand[wave][at] = (vk_u64)voc_key(v[j]) << 32 | (unsigned)~(v0 + (j / E) * PASS + tid * E + j % E);
            found += __popcll(m);
        }
    }
    if (lane < N) s_best[wave][lane] = 0;
    voc_wave_sync();
    if (found <= 64) {   // each lane one of them: its rank is the number of larger ones
        const vk_u64 k = lane < found ? s_cand[wave][lane] : 0;
        int rank = 0;
        for (int i = 0; i < found; ++i) rank += s_cand[wave][i] > k;
        if (lane < found && rank < N) s_best[wave][rank] = k;
    } else {   // many equal logits: one after the other
        for (int i = 0; i < N; ++i) {
            vk_u64 k = 0;
#pragma unroll
            for (int j = 0; j < VOC_ELEMS; ++j) {
                const vk_u64 kj = (vk_u64)voc_key(v[j]) << 32 | (unsigned)~(v0 + (j / E) * PASS + tid * E + j % E);
                if (v[j] >= from && kj > k && (i == 0 || kj < s_best[wave][i - 1])) k = kj;
            }
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) k = max(k, voc_shfl_xor(k, x));
            if (lane == 0) s_best[wave][i] = k;
            voc_wave_sync();
        }
    }
    __syncthreads();
    top = s_top[0];
#pragma unroll
    for (int i = 1; i < 4; ++i) top = top != top || s_top[i] != s_top[i] ? NAN : fmaxf(top, s_top[i]);
    double sum = 0.;
    if (top > -INFINITY) {
#pragma unroll
        for (int i = 0; i < PASSES; ++i)
            if (i * PASS < count)
#pragma unroll
                for (int j = 0; j < E; ++j) sum += voc_exp(fmax((double)v[i * E + j] - (double)top, -690.));   // (e^-690 for nothing at all: 1e-300)
    }
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
    if (lane == 0) s_sum[wave] = sum;
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
        if (rank < N) {
            const int64_t at = ((int64_t)row * p.splits + split) * N + rank;
            p.val[at] = k ? voc_unkey((unsigned)(k >> 32)) : -INFINITY;
            p.tok[at] = (int)~(unsigned)k;
        }
    }
    __syncthreads();
    if (tid == 0) {
        p.sum[row * p.splits + split] = s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
        p.top[row * p.splits + split] = top;
    }
}

// the larger of two candidates: by score, the lower row at a tie
struct VocBest {
    double score;
    int row;
};
__device__ __forceinline__ VocBest voc_best(VocBest a, VocBest b) { return b.score > a.score || (b.score == a.score && b.row < a.row) ? b : a; }

__global__ void __launch_bounds__(1024)
k_vocab_join(VocabP p) {
    __shared__ double s_score[TBS_MAX_BEAM][TBS_MAX_BEAM];
    __shared__ int s_token[TBS_MAX_BEAM][TBS_MAX_BEAM];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6, N = p.beams;
    const int64_t r0 = (int64_t)blockIdx.x * N;
    for (int i = wave; i < N; i += waves) {
        const int64_t row = r0 + i;
        const double score = p.scores[row];
        if (p.finished && p.finished[row]) {
            if (lane < N) {
                s_score[i][lane] = lane == 0 && score > -INFINITY ? score : -INFINITY;
                s_token[i][lane] = p.eos;
            }
            continue;
        }
        const bool in = lane < p.splits;
        const float top = in ? p.top[row * p.splits + lane] : -INFINITY;
        float best = top;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) best = fmaxf(best, __shfl_xor(best, x));
        double sum = in && top > -INFINITY ? p.sum[row * p.splits + lane] * exp((double)top - (double)best) : 0.;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) sum += __shfl_xor(sum, x);
        const bool none = __any(top != top) || best == -INFINITY;
        const double lse = (double)best + log(sum);
        // the slices' lists, a lane each: whoever has the largest logit (the lower slice at a tie: its tokens come first) goes on to its next
        int at = 0;
        const int64_t base = (row * p.splits + lane) * N;
        float v = in ? p.val[base] : -INFINITY;
        for (int k = 0; k < N; ++k) {
            float m = v;
#pragma unroll
            for (int x = 1; x < 64; x <<= 1) m = fmaxf(m, __shfl_xor(m, x));
            const int from = __ffsll((long long)__ballot(v == m)) - 1;
            if (lane == from) {
                const double s = score + ((double)v - lse);
                s_score[i][k] = none || !(s > -INFINITY) ? -INFINITY : s;
                if (v > -INFINITY) {   // (so it is one of its list)
                    s_token[i][k] = p.tok[base + at];
                    ++at;
                    v = at < N ? p.val[base + at] : -INFINITY;
                }
            }
        }
    }
    __syncthreads();
    if (wave > 0) return;
    int at = 0;
    VocBest b = {lane < N ? s_score[lane][0] : -INFINITY, lane};
    for (int k = 0; k < N; ++k) {
        VocBest m = b;
#pragma unroll
        for (int x = 1; x < 64; x <<= 1) m = voc_best(m, VocBest{__shfl_xor(m.score, x), __shfl_xor(m.row, x)});
        if (lane == m.row) {
            const bool none = !(m.score > -INFINITY);
            const int token = none ? -1 : s_token[lane][at];
            p.out_scores[r0 + k] = m.score;
            p.out_tokens[r0 + k] = token;
            p.out_parents[r0 + k] = none ? -1 : lane;
            p.out_finished[r0 + k] = none || token == p.eos || (p.finished && p.finished[r0 + lane]);
            if (!none) {
                ++at;
                b.score = at < N ? s_score[lane][at] : -INFINITY;
            }
        }
    }
}

struct VocabPlan {
    int splits, slice;
};

static VocabPlan vocab_plan(const tbs_beam_select_args &a) {
    // slices of 8192, smaller ones (2048 at least) while these are fewer than two workgroups a CU
    int64_t splits = (a.vocab + VOC_SLICE - 1) / VOC_SLICE, more = 512 / a.rows;
    if (more > (a.vocab + 2047) / 2048) more = (a.vocab + 2047) / 2048;
    if (more > VOC_SPLITS) more = VOC_SPLITS;
    if (splits < more) splits = more;
    const int pass = 256 * (int)(16 / op_dtype_size(a.dtype));
    VocabPlan pl;
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
    return args->rows == 0 ? 0 : vocab_bytes(*args, vocab_plan(*args));
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
    if (!a.workspace || a.workspace_bytes < vocab_bytes(a, pl) || (uintptr_t)a.workspace % 16) return TBS_EINVAL;
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
