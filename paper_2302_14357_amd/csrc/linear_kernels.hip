// Products with their epilogue: out = act(x w^T + bias) + residual, float32 sums, one rounding.
#include "op_device.h"

struct LinearEp {
    const float *bias;
    const void *residual;
    void *out;
    int64_t ld_r, ld_o;
    int act;
};

// Error function by the rational approximation 7.1.26 of Abramowitz and Stegun, Handbook of Mathematical Functions (absolute
// error 1.5e-7): for outputs of 16 bits, whose rounding is far larger.
__device__ __forceinline__ float linear_erf16(float x) {
    const float a = fabsf(x), t = __builtin_amdgcn_rcpf(fmaf(0.3275911f, a, 1.f));
    const float p = t * fmaf(t, fmaf(t, fmaf(t, fmaf(t, 1.061405429f, -1.453152027f), 1.421413741f), -0.284496736f), 0.254829592f);
    return copysignf(1.f - p * __expf(-a * a), x);
}

template <bool F32>
__device__ __forceinline__ float linear_act(float y, int act) {
    switch (act) {
        case TBS_ACT_RELU: return y > 0.f || y != y ? y : 0.f;   // (NaN stays)
        case TBS_ACT_TANH: return tanhf(y);
        case TBS_ACT_GELU: return 0.5f * y * (1.f + (F32 ? erff(y * 0.70710678f) : linear_erf16(y * 0.70710678f)));
        case TBS_ACT_SILU: return y / (1.f + expf(-y));
        default: return y;
    }
}

// Four columns j .. j + 3 of row i of the result.
template <class TO>
__device__ __forceinline__ void linear_store(const LinearEp &ep, int i, int j, int n, floatx4 acc) {
    float y[4];
    const int c = min(4, n - j);
#pragma unroll
    for (int q = 0; q < 4; ++q) y[q] = linear_act<sizeof(TO) == 4>(acc[q] + (ep.bias && q < c ? ep.bias[j + q] : 0.f), ep.act);
    TO *o = (TO *)ep.out + i * ep.ld_o + j;
    const TO *r = ep.residual ? (const TO *)ep.residual + i * ep.ld_r + j : nullptr;
    TO v[4];
    if (c == 4) {
        if (r) {
            __builtin_memcpy(v, r, sizeof v);
#pragma unroll
            for (int q = 0; q < 4; ++q) y[q] += op_float(v[q]);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = (TO)y[q];
        __builtin_memcpy(o, v, sizeof v);
    } else {
#pragma unroll
        for (int q = 0; q < 3; ++q)
            if (q < c) o[q] = (TO)(y[q] + (r ? op_float(r[q]) : 0.f));
    }
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
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const int r = m0 + wm * 32 + i * 16 + fr, c = n0 + wn * 32 + j * 16 + (lane >> 4) * 4;
            if (r < m && c < n) linear_store<TO>(ep, r, c, n, acc[i][j]);
        }
}

template <class T, class TO>
static hipError_t linear_run(const tbs_linear_args &a, hipStream_t st) {
    const LinearEp ep = {a.bias, a.residual, a.out, a.ld_residual, a.ld_out, a.act};
    const int64_t tiles_m = ((int64_t)a.m + 63) / 64, tiles_n = ((int64_t)a.n + 63) / 64;
    if (tiles_m * tiles_n > INT32_MAX) return hipErrorInvalidValue;
    hipLaunchKernelGGL((k_linear_any<T, TO>), dim3((unsigned)(tiles_m * tiles_n)), dim3(256), 0, st, (const T *)a.x, (const T *)a.w, a.ld_x,
                       a.ld_w, a.m, a.n, a.k, (int)tiles_n, ep);
    return hipGetLastError();
}

extern "C" int tbs_linear(const tbs_linear_args *args, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_linear_args &a = *args;
    if (!op_dtype_known(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != TBS_F32) || a.act < TBS_ACT_NONE || a.act > TBS_ACT_SILU)
        return TBS_EINVAL;
    if (a.m < 0 || a.n < 1 || a.k < 1 || a.k > INT32_MAX - 64 || a.n > INT32_MAX - 64 || a.m > INT32_MAX - 64) return TBS_EINVAL;
    if (a.m == 0) return TBS_OK;
    if (!a.x || !a.w || !a.out || a.ld_x < a.k || a.ld_w < a.k || a.ld_out < a.n || (a.residual && a.ld_residual < a.n)) return TBS_EINVAL;
    const size_t es = op_dtype_size(a.dtype), os = op_dtype_size(a.out_dtype);
    if ((uintptr_t)a.x % es || (uintptr_t)a.w % es || (uintptr_t)a.out % os || (uintptr_t)a.residual % os || (uintptr_t)a.bias % 4) return TBS_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    hipError_t e;
    if (a.dtype == TBS_F32) e = linear_run<float, float>(a, st);
    else if (a.dtype == TBS_BF16) e = a.out_dtype == TBS_F32 ? linear_run<__bf16, float>(a, st) : linear_run<__bf16, __bf16>(a, st);
    else e = a.out_dtype == TBS_F32 ? linear_run<_Float16, float>(a, st) : linear_run<_Float16, _Float16>(a, st);
    return e == hipSuccess ? TBS_OK : e == hipErrorInvalidValue ? TBS_EINVAL : TBS_EHIP;
}
