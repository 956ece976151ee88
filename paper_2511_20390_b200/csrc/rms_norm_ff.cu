// Root-mean-square norm: kernels for rows of fp32 and a residual of fp32.
#include "rms_norm.cuh"

int rms_norm_ff(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s) { return rms::launch_y<float, float>(a, vw, y_dtype, s); }
