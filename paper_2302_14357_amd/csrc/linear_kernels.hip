// The products' entry point, and their kernels for bf16.
#include "linear_device.h"

hipError_t linear_f16(const tbs_linear_args &a, int kernel, hipStream_t st);
hipError_t linear_f32(const tbs_linear_args &a, int kernel, hipStream_t st);

static int linear_call(const tbs_linear_args *args, int kernel, void *stream) {
    if (!args) return TBS_EINVAL;
    const tbs_linear_args &a = *args;
    if (!op_dtype_known(a.dtype) || (a.out_dtype != a.dtype && a.out_dtype != TBS_F32) || a.act < TBS_ACT_NONE || a.act > TBS_ACT_SILU)
        return TBS_EINVAL;
    if (a.m < 0 || a.n < 1 || a.k < 1 || a.k > (1 << 30) || a.n > INT32_MAX - 64 || a.m > INT32_MAX - 64) return TBS_EINVAL;
    if (a.m == 0) return TBS_OK;
    if (!a.x || !a.w || !a.out || a.ld_x < a.k || a.ld_w < a.k || a.ld_out < a.n || (a.residual && a.ld_residual < a.n)) return TBS_EINVAL;
    const size_t es = op_dtype_size(a.dtype), os = op_dtype_size(a.out_dtype);
    if ((uintptr_t)a.x % es || (uintptr_t)a.w % es || (uintptr_t)a.out % os || (uintptr_t)a.residual % os || (uintptr_t)a.bias % 4) return TBS_EINVAL;
    // what is written is nothing that other workgroups read: only a residual's own places are its writer's alone
    const int64_t e = (int64_t)es, oe = (int64_t)os;
    const OpRows out = {a.out, a.m, a.ld_out * oe, a.n * oe};
    if (op_overlap(out, {a.x, a.m, a.ld_x * e, a.k * e}) || op_overlap(out, {a.w, a.n, a.ld_w * e, a.k * e}) || (a.bias && op_overlap(out, {a.bias, 1, 4ll * a.n, 4ll * a.n})))
        return TBS_EINVAL;
    if (a.residual && !(a.residual == a.out && (a.ld_residual == a.ld_out || a.m == 1)) && op_overlap(out, {a.residual, a.m, a.ld_residual * oe, a.n * oe})) return TBS_EINVAL;
    const hipStream_t st = (hipStream_t)stream;
    hipError_t err;
    if (a.dtype == TBS_F32) err = linear_f32(a, kernel, st);
    else if (a.dtype == TBS_BF16) err = a.out_dtype == TBS_F32 ? linear_run<__bf16, float>(a, kernel, st) : linear_run<__bf16, __bf16>(a, kernel, st);
    else err = linear_f16(a, kernel, st);
    return err == hipSuccess ? TBS_OK : err == hipErrorInvalidValue ? TBS_EINVAL : TBS_EHIP;
}

extern "C" int tbs_linear(const tbs_linear_args *args, void *stream) { return linear_call(args, 0, stream); }

// one kernel of them all, for the tests and for timing (not in the header)
extern "C" int linear_by(const tbs_linear_args *args, int kernel, void *stream) { return linear_call(args, kernel, stream); }
