#include "linear_device.h"

hipError_t linear_f32(const tbs_linear_args &a, int kernel, hipStream_t st) { return linear_run<float, float>(a, kernel, st); }
