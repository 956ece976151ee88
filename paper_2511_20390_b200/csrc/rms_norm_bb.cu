// Root-mean-square norm: kernels for rows of bf16 and a residual of bf16.
#include "rms_norm.cuh"

int rms_norm_bb(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s) { return rms::launch_y<__nv_bfloat16, __nv_bfloat16>(a, vw, y_dtype, s); }
