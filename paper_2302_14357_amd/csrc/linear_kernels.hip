// The products' entry point, and their kernels for bf16.
#include "linear_device.h"

hipError_t linear_f16(const tbs_linear_args &a, int kernel, hipStream_t st);
hipError_t linear_f32(const tbs_linear_args &a, int kernel, hipStream_t st);

// Rows of bytes: whether two sets of them have one in common.  (Rows of one stride, as of two slices of a tensor, by what their distance leaves; others
// row by row, where the memory between their ends overlaps at all.)
struct LinearRows {
    const void *at;
    int64_t rows, ld, width;
};
static bool linear_overlap(LinearRows a, LinearRows b) {
    if (a.rows > b.rows) {
        const LinearRows t = a;
        a = b, b = t;
    }
    const int64_t d = (int64_t)((uintptr_t)b.at - (uintptr_t)a.at);
    if (d >= (a.rows - 1) * a.ld + a.width || -d >= (b.rows - 1) * b.ld + b.width) return false;
    auto floor_div = [](int64_t x, int64_t y) { return x / y - (x % y < 0); };
    if (a.ld == b.ld) {
        const int64_t q = floor_div(d, a.ld), r = d - q * a.ld;   // row j of b begins r bytes behind row q + j of a
        return (r < a.width && q < a.rows && q + b.rows > 0) || (r + b.width > a.ld && q + 1 < a.rows && q + 1 + b.rows > 0);
    }
    for (int64_t i = 0; i < a.rows; ++i) {
        const int64_t s = i * a.ld - d;   // row i of a, from b's first byte
        const int64_t first = floor_div(s - b.width, b.ld) + 1, last = floor_div(s + a.width - 1, b.ld);
        if ((first > 0 ? first : 0) <= (last < b.rows ? last : b.rows - 1)) return true;
    }
    return false;
}

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
    const LinearRows out = {a.out, a.m, a.ld_out * oe, a.n * oe};
    if (linear_overlap(out, {a.x, a.m, a.ld_x * e, a.k * e}) || linear_overlap(out, {a.w, a.n, a.ld_w * e, a.k * e}) || (a.bias && linear_overlap(out, {a.bias, 1, 4ll * a.n, 4ll * a.n})))
        return TBS_EINVAL;
    if (a.residual && !(a.residual == a.out && (a.ld_residual == a.ld_out || a.m == 1)) && linear_overlap(out, {a.residual, a.m, a.ld_residual * oe, a.n * oe})) return TBS_EINVAL;
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
