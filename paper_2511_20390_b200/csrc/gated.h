// Internal interfaces of the gated linear layer: gated_tc.cu (bf16, tensor cores), gated_simt.cu (fp32, CUDA cores),
// gated_rows.cu (few rows) and gated_api.cu (elementwise gradients, sums of parts, entry points).
#pragma once
#include "internal.h"

// ---- activations of the gate -------------------------------------------------------------------
// act and d act / dg.  GELU is the tanh form, written with the logistic function: (1 + tanh v) / 2 = 1 / (1 + e^(-2 v)).
#define FREE_GELU_2K 1.5957691216057308f                     /* 2 sqrt(2 / pi) */
#define FREE_GELU_C  0.044715f

__device__ __forceinline__ float free_logistic(float v) { return 1.f / (1.f + expf(-v)); }
// The same from the fast exponential and reciprocal, for the bf16 mode: off by at most (8 + 1.2 |v|) 2^-23 of the value (the
// exponential's argument is rounded after its scaling by log2 e, so its error grows with |v|).  Everything that is rounded to bf16 (half a step:
// 2^-8) uses it, and so does the bias gradient of that mode, whose terms come from the same pass: it is fp32 but holds this
// error.  e^-v overflows to infinity for v < -88 and the reciprocal is 0, the limit.
__device__ __forceinline__ float free_logistic_fast(float v) {
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + __expf(-v)));
    return r;
}
__device__ __forceinline__ float free_gate_arg(int act, float g) { return act == FREE_ACT_SILU ? g : FREE_GELU_2K * (g + FREE_GELU_C * g * g * g); }
__device__ __forceinline__ float free_gate_act_fast(int act, float g) { return g * free_logistic_fast(free_gate_arg(act, g)); }
__device__ __forceinline__ float free_gate_act(int act, float g) { return g * free_logistic(free_gate_arg(act, g)); }
// derivative from the logistic value s: s + g s (1 - s) d(arg)/dg.  Beyond |g| = 20 s is 0 or 1 and the second term 0; its last factor
// is kept finite (the square of 2e19 is not, and 0 times infinity is NaN).
__device__ __forceinline__ float free_gate_slope(int act, float g, float s) {
    const float d = act == FREE_ACT_SILU ? 1.f : FREE_GELU_2K * fminf(1.f + 3.f * FREE_GELU_C * g * g, 1e7f);
    return s + g * s * (1.f - s) * d;
}

// ---- products split along the contraction -------------------------------------------------------
struct GatedSplit {
    int parts;                   // 1: written straight to the output
    long long plane_rows;        // rows of a part in the workspace
    int half;                    // tensor cores: columns of a tile per CTA of a pair (128 or 64)
};

// ---- bf16 (tcgen05): F % 8 == 0, K % 8 == 0 ------------------------------------------------------
bool gated_tc_supported(int F, int K);
int gated_tc_forward(int act, int M, int F, int K, const void* x, const void* w, const float* bias, void* h, void* preact, uint32_t* err, cudaStream_t s);
GatedSplit gated_tc_split(bool dw, int M, int F, int K);
// dw false: out [M, K] = dz W; true: out [2F, K] = dz^T x.  g: of gated_tc_split(); with several parts they go to `parts`,
// plane_rows * K elements apart, and `out` is not written
int gated_tc_backward(bool dw, const GatedSplit& g, int M, int F, int K, const void* x, const void* w, const void* dz, void* out, float* parts, uint32_t* err, cudaStream_t s);

// ---- few rows (CUDA cores, both types); bf16: K % 8 == 0 -----------------------------------------
bool gated_rows_wanted(int dtype, int M, int F, int K);
int gated_rows_forward(int dtype, int act, int M, int F, int K, const void* x, const void* w, const float* bias, void* h, void* preact, cudaStream_t s);

// ---- fp32 (CUDA cores), any sizes ----------------------------------------------------------------
int gated_simt_forward(int act, int M, int F, int K, const float* x, const float* w, const float* bias, float* h, float* preact, cudaStream_t s);
GatedSplit gated_simt_split(bool dw, int M, int F, int K);
int gated_simt_backward(bool dw, const GatedSplit& g, int M, int F, int K, const float* x, const float* w, const float* dz, float* out, float* parts, cudaStream_t s);
