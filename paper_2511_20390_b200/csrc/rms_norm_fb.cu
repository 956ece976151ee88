// Root-mean-square norm: kernels for rows of fp32 and a residual of bf16.
#include "rms_norm.cuh"

int rms_norm_fb(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s) { return rms::launch_y<float, __nv_bfloat16>(a, vw, y_dtype, s); }
