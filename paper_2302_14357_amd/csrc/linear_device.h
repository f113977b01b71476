// Products with their epilogue: out = act(x w^T + bias) + residual, float32 sums, one rounding.  The kernels of all element types, each
// instantiated in a file of its own (linear_kernels.hip, linear_f16_kernels.hip, linear_f32_kernels.hip).
#pragma once
#include <math.h>

#include "op_device.h"

struct LinearEp {
    const float *bias;
    const void *residual;
    void *out;
    int64_t ld_r, ld_o;
    int act;
};

// y P(y) = max(y, 0) - |y| P(-|y|) with the normal distribution function P, for outputs of 16 bits: log2 P(-a) by a polynomial of degree 8, found by linear
// programming over 0 <= a <= 13.2, where a P(-a) leaves the normal numbers.  |y| P(-|y|) is then off by 2.2e-7 at most and, as a part of itself, by 8.1e-5 down to
// 6e-5 (a sixth of fp16's half step; below it numbers of fp16 are 6e-8 apart, and it is off by 4.9e-9) and 1e-3 below (a quarter of bf16's).  The polynomial falls
// without end, so that nothing is left from 20 on.  Half of it is the exponent and the exponential goes in twice: it is 0 where its result is below the normal
// numbers, which P is before a P is.
__device__ __forceinline__ float linear_gelu16(float y) {
    const float a = fminf(fabsf(y), 20.f);
    float p = fmaf(a, 2.4074848781197034e-08f, -1.3808490848532529e-06f);
    p = fmaf(a, fmaf(a, fmaf(a, p, 3.389550693100318e-05f), -0.0004732646921183914f), 0.004258902743458748f);
    p = fmaf(a, fmaf(a, fmaf(a, fmaf(a, p, -0.02697637677192688f), -0.22922585904598236f), -0.5756383538246155f), -0.499994695186615f);
    const float e = __builtin_amdgcn_exp2f(p);
    return fmaf(-a * e, e, y <= 0.f ? 0.f : y);   // (NaN stays)
}

// ... hyperbolic tangent and logistic function for such outputs: hardware exponential and reciprocal (a few units of float32), near 0, where
// 1 - 2 / (e^2x + 1) would lose digits, the series
__device__ __forceinline__ float linear_tanh16(float x) {
    const float s = x * x, near = x * fmaf(s, fmaf(s, fmaf(s, -17.f / 315.f, 2.f / 15.f), -1.f / 3.f), 1.f);
    return fabsf(x) < 0.25f ? near : 1.f - 2.f * __builtin_amdgcn_rcpf(__expf(2.f * x) + 1.f);
}

template <int ACT, bool F32>
__device__ __forceinline__ float linear_act(float y) {
    if constexpr (ACT == TBS_ACT_RELU) return y > 0.f || y != y ? y : 0.f;   // (NaN stays)
    else if constexpr (ACT == TBS_ACT_TANH) return F32 ? tanhf(y) : linear_tanh16(y);
    else if constexpr (ACT == TBS_ACT_GELU) return F32 ? 0.5f * y * erfcf(y * -0.70710678f) : linear_gelu16(y);   // (1 + erf would cancel where y is far below 0)
    else if constexpr (ACT == TBS_ACT_SILU) return F32 ? y / (1.f + expf(-y)) : y * __builtin_amdgcn_rcpf(1.f + __expf(-y));
    else return y;
}

// The residual of N columns c .. of row `row`, where they are all there (asked for ahead of the arithmetic).
template <class TO, int N>
__device__ __forceinline__ void linear_residual(const LinearEp &ep, int64_t row, int c, int n, TO (&r)[N]) {
    if (ep.residual && c + N <= n) __builtin_memcpy(r, (const TO *)ep.residual + row * ep.ld_r + c, sizeof r);
}

// N columns c .. of row `row`, some of them perhaps behind the last: activation of sum + bias, residual, one rounding.
template <class TO, int N>
__device__ __forceinline__ void linear_finish(const LinearEp &ep, int64_t row, int c, int n, float (&y)[N], const float (&bias)[N], const TO (&r)[N]) {
    constexpr bool F32 = sizeof(TO) == 4;
    switch (ep.act) {
#define LINEAR_EACH(A)                                                                   \
    case A:                                                                              \
        _Pragma("unroll") for (int q = 0; q < N; ++q) y[q] = linear_act<A, F32>(y[q] + bias[q]); \
        break;
        LINEAR_EACH(TBS_ACT_RELU)
        LINEAR_EACH(TBS_ACT_TANH)
        LINEAR_EACH(TBS_ACT_GELU)
        LINEAR_EACH(TBS_ACT_SILU)
#undef LINEAR_EACH
        default:
#pragma unroll
            for (int q = 0; q < N; ++q) y[q] += bias[q];
    }
    TO *o = (TO *)ep.out + row * ep.ld_o + c;
    if (c + N <= n) {
        TO v[N];
#pragma unroll
        for (int q = 0; q < N; ++q) v[q] = (TO)(ep.residual ? y[q] + op_float(r[q]) : y[q]);
        __builtin_memcpy(o, v, sizeof v);
    } else {
        const TO *pr = (const TO *)ep.residual + row * ep.ld_r + c;
#pragma unroll
        for (int q = 0; q < N - 1; ++q)
            if (c + q < n) o[q] = (TO)(ep.residual ? y[q] + op_float(pr[q]) : y[q]);
    }
}

template <int N>
__device__ __forceinline__ void linear_bias(const LinearEp &ep, int c, int n, float (&bias)[N]) {
#pragma unroll
    for (int q = 0; q < N; ++q) bias[q] = ep.bias ? ep.bias[min(c + q, n - 1)] : 0.f;
}

// Any sizes, strides and alignments: 64 x 64 outputs a workgroup of four waves, K through two LDS buffers by way of registers, rows
// of four 16-byte pieces.  Piece c of row r lies at c ^ (r / 4 % 4): sixteen rows' pieces at one place are then all LDS banks once.
template <class T, class TO>
__global__ void __launch_bounds__(256)
k_linear_any(const T *__restrict__ x, const T *__restrict__ w, int64_t ld_x, int64_t ld_w, int m, int n, int k, int tiles_n, LinearEp ep) {
    constexpr int E = OpPiece<T>::E;
    __shared__ uint4 lds[2][2][64 * 4];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int m0 = (int)(blockIdx.x / tiles_n) * 64, n0 = (int)(blockIdx.x % tiles_n) * 64;
    const int row = tid >> 2, piece = tid & 3, put = row * 4 + (piece ^ ((row >> 2) & 3));
    const T *px = x + min(m0 + row, m - 1) * ld_x, *pw = w + min(n0 + row, n - 1) * ld_w;
    uint4 rx, rw;
    auto fetch = [&](int k0) {
        const int at = k0 + piece * E;
        if (at + E <= k) {
            rx = op_load16(px + at);
            rw = op_load16(pw + at);
        } else {
            rx = op_load16_part(px + at, k - at);
            rw = op_load16_part(pw + at, k - at);
        }
    };
    const int fr = lane & 15, fp = (lane >> 4) ^ (fr >> 2);
    const int wm = wave >> 1, wn = wave & 1;
    floatx4 acc[2][2] = {};
    fetch(0);
    int buf = 0;
    for (int k0 = 0; k0 < k; k0 += 4 * E, buf ^= 1) {
        lds[buf][0][put] = rx;
        lds[buf][1][put] = rw;
        __syncthreads();   // (the other buffer was read before the last barrier)
        if (k0 + 4 * E < k) fetch(k0 + 4 * E);
        uint4 a[2], b[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) a[i] = lds[buf][0][(wm * 32 + i * 16 + fr) * 4 + fp];
#pragma unroll
        for (int j = 0; j < 2; ++j) b[j] = lds[buf][1][(wn * 32 + j * 16 + fr) * 4 + fp];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = op_mma<T>(b[j], a[i], acc[i][j]);   // (a lane: four columns of one row)
    }
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int c = n0 + wn * 32 + j * 16 + (lane >> 4) * 4;
        float bias[4];
        linear_bias(ep, c, n, bias);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = m0 + wm * 32 + i * 16 + fr;
            float y[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (r < m && c < n) {
                TO before[4];
                linear_residual(ep, r, c, n, before);
                linear_finish<TO>(ep, r, c, n, y, bias, before);
            }
        }
    }
}

// The 8 XCDs (workgroup id modulo 8) form a grid of gm x 8 / gm rectangles of tiles, each tm x tn of them, so that an XCD's L2 fetches a part of each operand
// instead of all of both.
struct LinearXcd {
    int gm, tm, tn;
};
__device__ __forceinline__ bool linear_tile_of(const LinearXcd &g, int tiles_m, int tiles_n, int &m, int &n) {
    const int xcd = blockIdx.x & 7, j = blockIdx.x >> 3, jn = j / g.tm, gn = 8 / g.gm;
    m = xcd / gn * g.tm + j - jn * g.tm;
    n = xcd % gn * g.tn + jn;
    return jn < g.tn && m < tiles_m && n < tiles_n;
}
// (host) the grid for which an XCD reads the fewest rows of both operands
static LinearXcd linear_xcds(int64_t tiles_m, int64_t tiles_n, int rows_m, int rows_n) {
    LinearXcd best = {1, 1, 1};
    int64_t least = INT64_MAX;
    for (int gm = 1; gm <= 8; gm *= 2) {
        const int64_t tm = (tiles_m + gm - 1) / gm, tn = (tiles_n + 8 / gm - 1) / (8 / gm);
        const int64_t rows = (tm * rows_m + tn * rows_n) * ((tm * tn * 8 + 255) / 256);   // (and no more turns of the chip than it takes)
        if (rows < least) least = rows, best = {gm, (int)tm, (int)tn};
    }
    return best;
}

#define LINEAR_WAVES 8
#define LINEAR_U 4
// The waves' shares of 16 TM x 16 TN outputs meet in LDS, are added up in the waves' order and finished, four columns a thread.
template <class TO, int TM, int TN>
__device__ __forceinline__ void linear_shares(const LinearEp &ep, const floatx4 (&acc)[TM][TN], floatx4 *s_acc, int m0, int n0, int m, int n) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fq = lane >> 4;
#pragma unroll
    for (int i = 0; i < TM * TN; ++i) s_acc[(wave * TM * TN + i) * 64 + lane] = acc[i / TN][i % TN];
    __syncthreads();
    if (wave >= TM * TN) return;
    floatx4 t = s_acc[wave * 64 + lane];
#pragma unroll
    for (int i = 1; i < LINEAR_WAVES; ++i) t += s_acc[(i * TM * TN + wave) * 64 + lane];
    const int r = m0 + wave / TN * 16 + fr, c = n0 + wave % TN * 16 + fq * 4;
    float y[4] = {t[0], t[1], t[2], t[3]}, bias[4];
    linear_bias(ep, c, n, bias);
    if (r < m && c < n) {
        TO before[4];
        linear_residual(ep, r, c, n, before);
        linear_finish<TO>(ep, r, c, n, y, bias, before);
    }
}

// Few rows: a workgroup of eight waves makes 16 TM x 16 TN outputs, each wave over its share of K, from registers alone: a wave asks for
// LINEAR_U steps of four pieces of every row at once (256 bytes of a row side by side; eight waves 2 KB), and its matrix instructions take
// them as they come.  The shares meet in LDS at the end.  What bounds it is how many bytes of the weights are on their way; any strides,
// alignments and K.
template <class T, class TO, int TM, int TN>
__global__ void __launch_bounds__(64 * LINEAR_WAVES)
k_linear_few(const T *__restrict__ x, const T *__restrict__ w, int64_t ld_x, int64_t ld_w, int m, int n, int k, LinearXcd grid, LinearEp ep) {
    constexpr int E = OpPiece<T>::E, STEP = 4 * E, CHUNK = LINEAR_U * STEP;
    __shared__ floatx4 s_acc[LINEAR_WAVES * TM * TN * 64];
    static_assert(TM * TN <= LINEAR_WAVES, "a wave finishes a block of 16 x 16");
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fq = lane >> 4;
    int tile_m, tile_n;
    if (!linear_tile_of(grid, (m + 16 * TM - 1) / (16 * TM), (n + 16 * TN - 1) / (16 * TN), tile_m, tile_n)) return;   // before any barrier
    const int m0 = tile_m * 16 * TM, n0 = tile_n * 16 * TN;
    const T *px[TM], *pw[TN];
#pragma unroll
    for (int i = 0; i < TM; ++i) px[i] = x + min(m0 + i * 16 + fr, m - 1) * ld_x + fq * E;
#pragma unroll
    for (int j = 0; j < TN; ++j) pw[j] = w + min(n0 + j * 16 + fr, n - 1) * ld_w + fq * E;
    floatx4 acc[TM][TN] = {};
    constexpr int EVERY = LINEAR_WAVES * CHUNK;
    struct Chunk {
        uint4 a[LINEAR_U][TM], b[LINEAR_U][TN];
    } one, two;
    auto load = [&](Chunk &q, int from) {
#pragma unroll
        for (int u = 0; u < LINEAR_U; ++u) {
#pragma unroll
            for (int j = 0; j < TN; ++j) q.b[u][j] = op_load16(pw[j] + from + u * STEP);
#pragma unroll
            for (int i = 0; i < TM; ++i) q.a[u][i] = op_load16(px[i] + from + u * STEP);
        }
        asm volatile("" ::: "memory");   // (asked for here, not where it is used)
    };
    auto multiply = [&](const Chunk &q) {
#pragma unroll
        for (int u = 0; u < LINEAR_U; ++u)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = op_mma<T>(q.b[u][j], q.a[u][i], acc[i][j]);
    };
    int at = wave * CHUNK;
    // 16 bits: the next chunk is on its way while the matrix instructions take the last (64 x 4096 x 4096 20.6 -> 17.8 us, 320 x 640 x 2560
    // 14.3 -> 11.7); float32, whose matrix instructions take sixteen times as long, has other waves for that (320 x 512 x 2048 17.8, like this 20.2)
    if constexpr (sizeof(T) == 2) {
        if (at + CHUNK <= k) {
            load(one, at);
            for (;;) {
                at += EVERY;
                const bool more = at + CHUNK <= k;
                if (more) load(two, at);
                multiply(one);
                if (!more) break;
                at += EVERY;
                const bool still = at + CHUNK <= k;
                if (still) load(one, at);
                multiply(two);
                if (!still) break;
            }
        }
    } else {
        for (; at + CHUNK <= k; at += EVERY) {
            load(one, at);
            multiply(one);
        }
    }
    for (const int end = min(at + CHUNK, k); at < end; at += STEP) {   // the last, partial chunk is one wave's
        uint4 a[TM], b[TN];
        const int left = k - at - fq * E;
        auto get = [&](const T *p) { return left >= E ? op_load16(p + at) : op_load16_part(p + at, left); };
#pragma unroll
        for (int j = 0; j < TN; ++j) b[j] = get(pw[j]);
#pragma unroll
        for (int i = 0; i < TM; ++i) a[i] = get(px[i]);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = op_mma<T>(b[j], a[i], acc[i][j]);
    }
    linear_shares<TO, TM, TN>(ep, acc, s_acc, m0, n0, m, n);
}

// Many rows: one tile of 32 TM x 64 TN outputs a workgroup of eight waves (2 x 4), a wave 16 TM x 16 TN.  Rows of 128 bytes of K (8 pieces,
// piece c of row r at c ^ (r / 2 % 8): sixteen rows' pieces of one place are then all LDS banks once) pass through NS stages of LDS by direct
// loads; a stage is asked for again as soon as every wave has its last fragments, and the fragments of the next 64 bytes are read
// while the matrix instructions take the last ones.  Rows on 16-byte boundaries, K in whole pieces; pieces behind K come from zeros.
#define LT_ROW 128                                             // bytes of a row and stage
#define LT_LDS_READ (15 | (7 << 4) | (0 << 8) | (3 << 14))     // s_waitcnt: LDS reads only
#define LT_VMCNT(n) (((n) & 15) | (7 << 4) | (15 << 8) | (((n) >> 4) << 14))   // ... all but n loads from memory
__device__ const uint4 linear_zeros = {0, 0, 0, 0};

// what lanes of a wave wrote to LDS is there for its others
__device__ __forceinline__ void lt_wave_sync() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Few rows on 16-byte boundaries: as k_linear_few, but through LDS, D steps of PB pieces of every row on their way.  A load's neighbouring lanes take neighbouring
// pieces of a row (PB x 16 bytes together), as the first-level cache wants them; the matrix instructions' lanes, of which neighbours are
// different rows, get theirs from LDS, each wave from a ring of its own, without barriers.  Piece c of row r lies at c ^ swz(r): sixteen rows' pieces of one
// place are then all LDS banks once.
template <class T, class TO, int TM, int TN, int PB, int D>
__global__ void __launch_bounds__(64 * LINEAR_WAVES)
k_linear_stream(const char *__restrict__ x, const char *__restrict__ w, int64_t ld_x, int64_t ld_w, int m, int n, int k_bytes, LinearXcd grid, LinearEp ep) {
    constexpr int STEP = PB * 16, PER = LINEAR_U * 64 / STEP, CHUNK = PER * STEP, R = TM + TN, L = PB / 4;   // bytes; L loads to 16 rows
    constexpr int BLOCK = 16 * STEP, RING = D * R * BLOCK;
    static_assert(TM * TN <= LINEAR_WAVES && TM * TN * 1024 <= RING, "a wave finishes a block of 16 x 16; the shares lie in the rings");
    extern __shared__ __attribute__((aligned(16))) char lt_smem[];   // a ring of D steps for every wave
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), fr = lane & 15, fq = lane >> 4;
    int tile_m, tile_n;
    if (!linear_tile_of(grid, (m + 16 * TM - 1) / (16 * TM), (n + 16 * TN - 1) / (16 * TN), tile_m, tile_n)) return;   // before any barrier
    const int m0 = tile_m * 16 * TM, n0 = tile_n * 16 * TN;
    auto swz = [](int r) { return PB == 8 ? (r >> 1) & 7 : (r >> 2) & 3; };
    const char *p[R][L];   // weights first
    int piece[L];
#pragma unroll
    for (int q = 0; q < L; ++q) {
        const int row = q * (64 / PB) + lane / PB;
        piece[q] = ((lane % PB) ^ swz(row)) * 16;
#pragma unroll
        for (int j = 0; j < TN; ++j) p[j][q] = w + min(n0 + j * 16 + row, n - 1) * ld_w + piece[q];
#pragma unroll
        for (int i = 0; i < TM; ++i) p[TN + i][q] = x + min(m0 + i * 16 + row, m - 1) * ld_x + piece[q];
    }
    // this wave's steps: those of chunks wave, wave + 8, ...; the last chunk may have fewer
    const int chunks = (k_bytes + CHUNK - 1) / CHUNK, mine = chunks > wave ? (chunks - wave + LINEAR_WAVES - 1) / LINEAR_WAVES : 0;
    const int missing = mine > 0 && (chunks - 1) % LINEAR_WAVES == wave ? (int)(((int64_t)chunks * CHUNK - k_bytes) / STEP) : 0, steps = mine * PER - missing;
    char *ring = lt_smem + wave * RING;
    const unsigned lds = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)ring;
    int asked = 0, slot_in = 0;
    auto ask = [&]() {
        const int at = ((asked / PER) * LINEAR_WAVES + wave) * CHUNK + asked % PER * STEP;
#pragma unroll
        for (int q = 0; q < L; ++q) {
            const bool behind = at + STEP > k_bytes && at + piece[q] >= k_bytes;   // (pieces behind K, in the last step only)
#pragma unroll
            for (int r = 0; r < R; ++r) op_load_lds(behind ? (const char *)&linear_zeros : p[r][q] + at, lds + (slot_in * R + r) * BLOCK + q * 1024);
        }
        slot_in = slot_in + 1 == D ? 0 : slot_in + 1;
        ++asked;
    };
#pragma unroll
    for (int s = 0; s < D; ++s)
        if (s < steps) ask();
    floatx4 acc[TM][TN] = {};
    int slot = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + D <= steps) asm volatile("s_waitcnt vmcnt(%0)" ::"n"((D - 1) * R * L) : "memory");   // this step's have landed; the younger ones may be on their way
        else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        uint4 f[L][R];
#pragma unroll
        for (int h = 0; h < L; ++h)
#pragma unroll
            for (int r = 0; r < R; ++r) f[h][r] = *reinterpret_cast<const uint4 *>(ring + (slot * R + r) * BLOCK + fr * STEP + ((h * 4 + fq) ^ swz(fr)) * 16);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");   // and have been read before their place is asked for again
        __builtin_amdgcn_sched_barrier(0);
        if (asked < steps) ask();
        slot = slot + 1 == D ? 0 : slot + 1;
#pragma unroll
        for (int h = 0; h < L; ++h)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = op_mma<T>(f[h][j], f[h][TN + i], acc[i][j]);
    }
    __syncthreads();   // (the shares lie where the other waves' rings were)
    linear_shares<TO, TM, TN>(ep, acc, reinterpret_cast<floatx4 *>(lt_smem), m0, n0, m, n);
}

template <class T, class TO, int TM, int TN, int NS>
__global__ void __launch_bounds__(512, 2)
k_linear_tile(const char *__restrict__ x, const char *__restrict__ w, int64_t ld_x, int64_t ld_w, int m, int n, int k_bytes, LinearXcd grid, LinearEp ep) {
    constexpr int BM = 32 * TM, BN = 64 * TN, RA = BM / 64, RB = BN / 64, STAGE = (BM + BN) * LT_ROW;
    extern __shared__ __attribute__((aligned(16))) char lt_smem[];   // NS stages
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), wm = wave >> 2, wn = wave & 3;
    const int tiles_m = (m + BM - 1) / BM, tiles_n = (n + BN - 1) / BN;
    int tile_m, tile_n;
    if (!linear_tile_of(grid, tiles_m, tiles_n, tile_m, tile_n)) return;   // before any barrier
    const int kt_n = (k_bytes + LT_ROW - 1) / LT_ROW;
    // a pass: 64 rows, eight a wave; position lane % 8 of its row receives piece position ^ (row / 2 % 8)
    const int lrow = wave * 8 + (lane >> 3), lch = ((lane & 7) ^ ((lrow >> 1) & 7)) * 16;
    const char *pa[RA], *pb[RB];
#pragma unroll
    for (int i = 0; i < RA; ++i) pa[i] = x + min(tile_m * BM + i * 64 + lrow, m - 1) * ld_x + lch;
#pragma unroll
    for (int i = 0; i < RB; ++i) pb[i] = w + min(tile_n * BN + i * 64 + lrow, n - 1) * ld_w + lch;
    int asked = 0;
    const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char *)lt_smem + wave * 8 * LT_ROW;
    auto fetch = [&](int stage) {
        const unsigned dst = lds0 + stage * STAGE;
        if ((asked + 1) * LT_ROW > k_bytes && asked * LT_ROW + lch >= k_bytes) {   // (pieces behind K, in the last K tile only)
#pragma unroll
            for (int i = 0; i < RA; ++i) pa[i] = (const char *)&linear_zeros;
#pragma unroll
            for (int i = 0; i < RB; ++i) pb[i] = (const char *)&linear_zeros;
        }
#pragma unroll
        for (int i = 0; i < RA; ++i) {
            op_load_lds(pa[i], dst + i * 64 * LT_ROW);
            pa[i] += LT_ROW;
        }
#pragma unroll
        for (int i = 0; i < RB; ++i) {
            op_load_lds(pb[i], dst + (BM + i * 64) * LT_ROW);
            pb[i] += LT_ROW;
        }
        ++asked;
    };
#pragma unroll
    for (int q = 0; q < NS; ++q)
        if (q < kt_n) fetch(q);
    const int frow = lane & 15, fq = lane >> 4, fsw = (frow >> 1) & 7;
    const int fa = (wm * 16 * TM + frow) * LT_ROW, fb = (BM + wn * 16 * TN + frow) * LT_ROW;
    const int ch[2] = {(fq ^ fsw) * 16, ((4 + fq) ^ fsw) * 16};
    uint4 xa[2][TM], xb[2][TN];
    auto read = [&](int h, int stage) {
        const char *s = lt_smem + stage * STAGE + ch[h];
#pragma unroll
        for (int b = 0; b < TN; ++b) xb[h][b] = *reinterpret_cast<const uint4 *>(s + fb + b * 16 * LT_ROW);
#pragma unroll
        for (int i = 0; i < TM; ++i) xa[h][i] = *reinterpret_cast<const uint4 *>(s + fa + i * 16 * LT_ROW);
    };
    floatx4 acc[TM][TN] = {};
    auto mma = [&](int h) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int b = 0; b < TN; ++b) acc[i][b] = op_mma<T>(xb[h][b], xa[h][i], acc[i][b]);
        __builtin_amdgcn_sched_barrier(0);
    };
    // this wave's share of the K tile after kt has landed (the NS - 2 behind it may be on their way), and so has everybody's
    auto landed = [&](int kt) {
        if (kt + NS <= kt_n) __builtin_amdgcn_s_waitcnt(LT_VMCNT((NS - 2) * (RA + RB)));
        else __builtin_amdgcn_s_waitcnt(LT_VMCNT(0));
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    if (kt_n >= NS) __builtin_amdgcn_s_waitcnt(LT_VMCNT((NS - 1) * (RA + RB)));
    else __builtin_amdgcn_s_waitcnt(LT_VMCNT(0));
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    read(0, 0);
    int stage = 0;
    for (int kt = 0; kt < kt_n; ++kt) {
        __builtin_amdgcn_s_waitcnt(LT_LDS_READ);
        __builtin_amdgcn_sched_barrier(0);
        read(1, stage);
        mma(0);
        __builtin_amdgcn_s_waitcnt(LT_LDS_READ);
        if (kt + 1 < kt_n) {
            landed(kt);   // (and every wave has read this stage)
            const int next = stage + 1 == NS ? 0 : stage + 1;
            read(0, next);
            if (kt + NS < kt_n) fetch(stage);
            stage = next;
        }
        mma(1);
    }
    // The result goes through LDS, a wave's part in a region of its own, in one piece or two halves: a lane then has eight columns of a row
    // (whole lines of memory are read and written together), and the activations' code is there once, in a loop.  Piece c of row r
    // at c ^ swz(r), as above, for rows of 4 TN pieces.
    constexpr int HALVES = 8 * 16 * TM * 16 * TN * 4 > NS * STAGE ? 2 : 1, TH = TM / HALVES, RL = 64 * TN;   // (bytes of a row)
    static_assert(8 * 16 * TH * RL <= NS * STAGE && TM % HALVES == 0, "");
    auto swz = [](int r) { return TN == 4 ? r & 15 : TN == 2 ? (r >> 1) & 7 : (r >> 2) & 3; };
    char *mine = lt_smem + wave * 16 * TH * RL;
    const int col = lane % (2 * TN) * 8, c = tile_n * BN + wn * 16 * TN + col;
    // Passes of 32 / TN rows, G of them in one turn of the loop; the residual of the next turn's rows is asked for before this turn's arithmetic (8000 x 4096 x 1024 with gelu
    // and residual 98 us; asked for with its own row 109, eight passes a turn 103).
    constexpr int PASSES = 16 * TH * TN / 32, G = PASSES % 4 == 0 && sizeof(TO) == 2 ? 4 : PASSES % 2 == 0 ? 2 : 1;
    const int row0 = tile_m * BM + wm * 16 * TM + lane / (2 * TN);
    float bias[8];
    linear_bias(ep, c, n, bias);
    TO next[G][8];   // the residual of the next turn's rows
    auto ask = [&](int row) {
#pragma unroll
        for (int i = 0; i < G; ++i) linear_residual(ep, min(row + i * (32 / TN), m - 1), c, n, next[i]);
    };
    ask(row0);
    __builtin_amdgcn_s_waitcnt(LT_LDS_READ);
    __builtin_amdgcn_s_barrier();   // every wave has read its last fragments
    asm volatile("" ::: "memory");
    for (int h = 0; h < HALVES; ++h) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
            if (HALVES == 1 || (h == 0) == (i < TH))
#pragma unroll
                for (int b = 0; b < TN; ++b) {
                    const int r = (i % TH) * 16 + frow;
                    *reinterpret_cast<floatx4 *>(mine + r * RL + ((b * 4 + fq) ^ swz(r)) * 16) = acc[i][b];
                }
        lt_wave_sync();
        for (int g = 0; g < PASSES; g += G) {
            TO before[G][8];
            __builtin_memcpy(before, next, sizeof next);
            ask(row0 + h * 16 * TH + (g + G) * (32 / TN));   // (the turn after a half's last is the next half's first)
#pragma unroll
            for (int i = 0; i < G; ++i) {
                const int r = lane / (2 * TN) + (g + i) * (32 / TN), row = row0 + h * 16 * TH + (g + i) * (32 / TN);
                const floatx4 u = *reinterpret_cast<const floatx4 *>(mine + r * RL + ((col / 4) ^ swz(r)) * 16);
                const floatx4 v = *reinterpret_cast<const floatx4 *>(mine + r * RL + ((col / 4 + 1) ^ swz(r)) * 16);
                float y[8] = {u[0], u[1], u[2], u[3], v[0], v[1], v[2], v[3]};
                if (row < m && c < n) linear_finish<TO>(ep, row, c, n, y, bias, before[i]);
            }
        }
        lt_wave_sync();
    }
}

template <class T, class TO, int TM, int TN, int NS>
static hipError_t linear_tile_launch(const tbs_linear_args &a, const LinearEp &ep, hipStream_t st) {
    constexpr int BM = 32 * TM, BN = 64 * TN, SHM = NS * (BM + BN) * LT_ROW;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_linear_tile<T, TO, TM, TN, NS>), hipFuncAttributeMaxDynamicSharedMemorySize, SHM);
    if (e != hipSuccess) return e;
    const LinearXcd g = linear_xcds(((int64_t)a.m + BM - 1) / BM, ((int64_t)a.n + BN - 1) / BN, BM, BN);
    hipLaunchKernelGGL((k_linear_tile<T, TO, TM, TN, NS>), dim3((unsigned)(8 * (int64_t)g.tm * g.tn)), dim3(512), SHM, st, (const char *)a.x, (const char *)a.w, a.ld_x * (int64_t)sizeof(T),
                       a.ld_w * (int64_t)sizeof(T), a.m, a.n, (int)(a.k * sizeof(T)), g, ep);
    return hipGetLastError();
}

template <class T, class TO, int TM, int TN, int PB, int D>
static hipError_t linear_stream_launch(const tbs_linear_args &a, const LinearEp &ep, hipStream_t st) {
    constexpr int SHM = LINEAR_WAVES * D * (TM + TN) * PB * 256;
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(&k_linear_stream<T, TO, TM, TN, PB, D>), hipFuncAttributeMaxDynamicSharedMemorySize, SHM);
    if (e != hipSuccess) return e;
    const LinearXcd g = linear_xcds(((int64_t)a.m + 16 * TM - 1) / (16 * TM), ((int64_t)a.n + 16 * TN - 1) / (16 * TN), 16 * TM, 16 * TN);
    hipLaunchKernelGGL((k_linear_stream<T, TO, TM, TN, PB, D>), dim3((unsigned)(8 * (int64_t)g.tm * g.tn)), dim3(64 * LINEAR_WAVES), SHM, st, (const char *)a.x, (const char *)a.w,
                       a.ld_x * (int64_t)sizeof(T), a.ld_w * (int64_t)sizeof(T), a.m, a.n, (int)(a.k * sizeof(T)), g, ep);
    return hipGetLastError();
}

template <class T, class TO, int TM, int TN>
static hipError_t linear_few_launch(const tbs_linear_args &a, const LinearEp &ep, hipStream_t st) {
    const LinearXcd g = linear_xcds(((int64_t)a.m + 16 * TM - 1) / (16 * TM), ((int64_t)a.n + 16 * TN - 1) / (16 * TN), 16 * TM, 16 * TN);
    hipLaunchKernelGGL((k_linear_few<T, TO, TM, TN>), dim3((unsigned)(8 * (int64_t)g.tm * g.tn)), dim3(64 * LINEAR_WAVES), 0, st, (const T *)a.x, (const T *)a.w, a.ld_x, a.ld_w, a.m,
                       a.n, a.k, g, ep);
    return hipGetLastError();
}

// Which kernel?  The one whose estimated time is least, in us; K in units of 2048 bytes (1024 numbers of 16 bits), "turns" of the chip's 256
// CUs.  Fitted to 30 sizes of 1 to 8192 rows, operands in the caches or from memory (us, estimated / measured):
//   k_linear_stream: 1.3, and for every turn 2 (2.8 where they are more than two) and what a workgroup reads at so many bytes a ns: 100 (16 x 16 outputs), 90 (16 x 32, 32 x 16, 32 x 32),
//     60 (64 x 32), all of it at 6.5 TB/s at most: 5 x 2560 x 640 3.7 / 4.5, 16 x 4096 x 4096 8.4 / 7.7, 64 x 4096 x 4096 9.1 / 9.3, 320 x 640 x 2560 6.9 / 6.9,
//     320 x 1024 x 1024 6.6 / 6.4; float32, whose matrix instructions take their time, 60, 45, 40, 30: 320 x 512 x 2048 16.4 / 16.5
//   k_linear_few: 3.3, and what a CU's workgroups read at 47 (16 x 16) or 37 bytes a ns (32 x 32; float32 37, 34), all of it at 5.5 TB/s at most: its neighbouring
//     lanes are different rows, which the first-level cache serves 16 bytes at a time; several workgroups a CU, though, and no alignment: 5 x 32000 x 1024 15 / 14
//   k_linear_tile (operands at 3.4 TB/s at most) 64 x 64, two workgroups a CU: 3 + 5.5 K for up to one a CU, else 8 K a turn of 512: 256 x 4096 x 1024 8.5 / 9.4,
//     1000 x 4096 x 1024 19 / 22, 64 x 32000 x 1024 22 / 18
//   128 x 128, two a CU: 12.5 K for one a CU, 18 K + 4 for two: 1000 x 4096 x 1024 15.5 / 16.5, 8000 x 1024 x 4096 79 / 75
//   192 x 256: 22 K + 6 a turn: 2560 x 4096 x 1024 30 / 30;  256 x 256: 28 K + 9 a turn: 8000 x 4096 x 1024 76 / 81, 8192 x 4096 x 4096 244 / 237
//   float32's matrix instructions take their own time: 64 x 64 11 K and 20 K: 256 x 4096 x 1024 25 / 28, 1000 x 4096 x 1024 83 / 94, 8000 x 1024 x 4096 643 / 612;
//     128 x 128 32 K and 70 K: 256 x 4096 x 1024 67 / 71, 1000 x 4096 x 1024 67 / 83, 8000 x 1024 x 4096 563 / 563;  192 x 256 112 K: 2560 x 4096 x 1024 232 / 204, 8192 x
//     4096 x 4096 2708 / 2209;  256 x 256 137 K: 8000 x 1024 x 4096 1107 / 970, 8192 x 4096 x 4096 2212 / 1955
//   k_linear_any, where the tiles' alignment is missing: 10 K, or 18.5 K for every 1024 tiles: 300 x 1001 x 2001 23 / 18, 1000 x 1000 x 999 13 / 11, 2000 x 2001 x 2001
//     39 / 52, 4000 x 4999 x 4999 442 / 792 (nothing else comes near there); float32 15 and 48: 62 / 54, 32 / 33, 191 / 196, 2281 / 1964
struct LinearChoice {
    int kernel;
    double us;
};

static LinearChoice linear_choice(const tbs_linear_args &a, int es, bool tiles) {
    const double K = (double)a.k * es / 2048, m = a.m, n = a.n, bytes = (m + n) * a.k * es;
    const bool f32 = es == 4;
    LinearChoice best = {0, 1e30};
    auto consider = [&](int kernel, double us) {
        if (us < best.us) best = {kernel, us};
    };
    auto up = [](double x, double d) { return ceil(x / d); };
    auto few = [&](int kernel, int tm, int tn, double rate) {
        const double groups = up(m, 16 * tm) * up(n, 16 * tn), turns = groups < 1024 ? up(groups, 256) : groups / 256;
        consider(kernel, 3.3 + fmax(turns * 16 * (tm + tn) * a.k * es / (rate * 1000), bytes / 5.5e6));
    };
    few(11, 1, 1, f32 ? 37 : 47), few(22, 2, 2, f32 ? 34 : 37);
    if (tiles) {
        auto stream = [&](int kernel, int tm, int tn, double rate) {
            const double turns = up(up(m, 16 * tm) * up(n, 16 * tn), 256);
            consider(kernel, 1.3 + fmax(turns * (16 * (tm + tn) * a.k * es / (rate * 1000) + (turns > 2 ? 2.8 : 2)), bytes / 6.5e6 + 2));
        };
        stream(311, 1, 1, f32 ? 60 : 100), stream(312, 1, 2, f32 ? 45 : 90), stream(321, 2, 1, f32 ? 45 : 90), stream(322, 2, 2, f32 ? 40 : 90), stream(342, 4, 2, f32 ? 30 : 60);
        auto two = [&](int kernel, double bm, double bn, double one_a_cu, double two_a_cu, double end) {   // two workgroups a CU
            const double t = up(m, bm) * up(n, bn), whole = floor(t / 512), rest = t - 512 * whole;
            consider(kernel, 3 + fmax(whole * (two_a_cu * K + end) + (rest == 0 ? 0 : (rest <= 256 ? one_a_cu : two_a_cu) * K + (whole ? end : 0)), bytes / 3.4e6));
        };
        two(121, 64, 64, f32 ? 11 : 5.5, f32 ? 20 : 8, 0);
        two(142, 128, 128, f32 ? 32 : 12.5, f32 ? 70 : 18, 4);
        consider(164, 2 + up(up(m, 192) * up(n, 256), 256) * ((f32 ? 112 : 22) * K + 6));
        consider(184, 2 + up(up(m, 256) * up(n, 256), 256) * ((f32 ? 137 : 28) * K + 9));
    } else {
        const double t = up(m, 64) * up(n, 64) / 1024;
        consider(1, 3 + fmax(K * fmax(f32 ? 15 : 10, t * (f32 ? 48 : 18.5)), bytes / 3.6e6));
    }
    return best;
}

// kernel: 0 = the choice for the sizes; otherwise that one (10 TM + TN of k_linear_few, 300 + that of k_linear_stream, 100 + that of k_linear_tile,
// 1 = k_linear_any)
template <class T, class TO>
static hipError_t linear_run(const tbs_linear_args &a, int kernel, hipStream_t st) {
    const LinearEp ep = {a.bias, a.residual, a.out, a.ld_residual, a.ld_out, a.act};
    const bool tiles = (uintptr_t)a.x % 16 == 0 && (uintptr_t)a.w % 16 == 0 && a.ld_x * sizeof(T) % 16 == 0 && a.ld_w * sizeof(T) % 16 == 0 && a.k * sizeof(T) % 16 == 0 &&
                       a.k <= INT32_MAX / 8;
    if (kernel == 0) kernel = linear_choice(a, sizeof(T), tiles).kernel;
    if (kernel >= 100 && !tiles) return hipErrorInvalidValue;
    switch (kernel) {
        case 11: return linear_few_launch<T, TO, 1, 1>(a, ep, st);
        case 22: return linear_few_launch<T, TO, 2, 2>(a, ep, st);
        case 311: return linear_stream_launch<T, TO, 1, 1, 8, 4>(a, ep, st);
        case 312: return linear_stream_launch<T, TO, 1, 2, 8, 2>(a, ep, st);
        case 321: return linear_stream_launch<T, TO, 2, 1, 8, 2>(a, ep, st);
        case 322:   // (us by steps of 64 / 128 bytes: float32 320 x 512 x 2048 16.5 / 17.3, 64 x 2048 x 2048 15.8 / 16.7; bf16 64 x 4096 x 4096 12.6 / 9.3)
            if constexpr (sizeof(T) == 4) return linear_stream_launch<T, TO, 2, 2, 4, 4>(a, ep, st);
            else return linear_stream_launch<T, TO, 2, 2, 8, 2>(a, ep, st);
        case 342: return linear_stream_launch<T, TO, 4, 2, 4, 3>(a, ep, st);
        case 121: return linear_tile_launch<T, TO, 2, 1, 4>(a, ep, st);
        case 142: return linear_tile_launch<T, TO, 4, 2, 2>(a, ep, st);
        case 164: return linear_tile_launch<T, TO, 6, 4, 2>(a, ep, st);
        case 184: return linear_tile_launch<T, TO, 8, 4, 2>(a, ep, st);
        case 1: break;
        default: return hipErrorInvalidValue;
    }
    const int64_t tiles_m = ((int64_t)a.m + 63) / 64, tiles_n = ((int64_t)a.n + 63) / 64;
    if (tiles_m * tiles_n > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_linear_any<T, TO>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, st, (const T *)a.x, (const T *)a.w, a.ld_x,
                       a.ld_w, a.m, a.n, a.k, (int)tiles_n, ep);
    return hipGetLastError();
}

