// Internal interfaces of the root-mean-square norm (rms_norm_*.cu).
#pragma once
#include "internal.h"

constexpr int kRmsMaxD = 8192;

struct RmsArgs {
    long long M;                              // rows: tokens x heads
    int D, heads, rows_per_group, warps;
    const void* x; long long x_tok, x_head;
    const void* res; long long res_stride;    // or nullptr
    void* h; long long h_stride;              // the sum, or nullptr
    const float* weight; long long mod_stride; float unit;    // unit: 1 where the weight is stored as an offset from one
    float eps;
    void* y; long long y_tok, y_head;
    float* scales; long long scale_stride; int scale_block;   // 8-bit results; scale_block 0: one scale a row
    float* rstd;                              // [M] or nullptr
    long long rows_per_team;
};

// vw: consecutive columns of one access, 8 (bf16 only), 4 or 1.  One function per pair of types (x, residual).
int rms_norm_ff(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s);
int rms_norm_fb(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s);
int rms_norm_bf(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s);
int rms_norm_bb(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s);

// Backward pass: the kernels of layer_norm.cu without a mean.
struct RmsBwdArgs {
    int x_dtype, dy_dtype, D, heads, groups, rows_per_group;
    const void* x; long long x_tok, x_head;
    const void* dy; long long dy_tok, dy_head;
    const float *rstd, *weight; long long mod_stride; float unit;
    const void* dres; long long dres_tok, dres_head;
    void* dx; long long dx_tok, dx_head;
    float* dw; long long dmod_stride;
    float* ws; size_t ws_bytes;
};
size_t rms_norm_bwd_bytes(int groups, int rows_per_group, int D);
bool rms_norm_bwd_takes_heads(int D);        // whether rows of D columns may be heads with strides of their own
int rms_norm_bwd(const RmsBwdArgs& a, cudaStream_t s);
