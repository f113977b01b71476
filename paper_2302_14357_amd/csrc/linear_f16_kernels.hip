#include "linear_device.h"

hipError_t linear_f16(const tbs_linear_args &a, int kernel, hipStream_t st) {
    return a.out_dtype == TBS_F32 ? linear_run<_Float16, float>(a, kernel, st) : linear_run<_Float16, _Float16>(a, kernel, st);
}
