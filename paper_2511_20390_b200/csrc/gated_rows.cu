// Gated linear layer for few rows (single tokens) or few columns: h = act(x Wg^T + bg) (x Wu^T + bu) on CUDA cores.
//
// Bound by the weights' bytes, which are read once: a warp takes one gate row and the matching up row of W, 16 bytes per lane
// and load with several loads in flight, and multiplies them with all MR rows of x (which come from the L1).  Sums are fp32,
// joined by exchanges at the end; the warp that holds z_gate holds z_up, so the activation and the product follow at once.
// With one warp per column the weights of a 4608 x 1152 layer are in flight on all SMs at the same time.
#include "gated.h"

namespace {

constexpr int kWarps = 8;

template <typename T, int V> struct Chunk;                         // V values of a row
template <> struct Chunk<__nv_bfloat16, 8> {
    uint4 d;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { d = __ldg(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void load_once(const __nv_bfloat16* p) { d = __ldcs(reinterpret_cast<const uint4*>(p)); }
    __device__ __forceinline__ void zero() { d = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {d.x, d.y, d.z, d.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) { f[2 * i] = __uint_as_float(w[i] << 16); f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
    }
};
template <> struct Chunk<float, 4> {
    float4 d;
    __device__ __forceinline__ void load(const float* p) { d = __ldg(reinterpret_cast<const float4*>(p)); }
    __device__ __forceinline__ void load_once(const float* p) { d = __ldcs(reinterpret_cast<const float4*>(p)); }
    __device__ __forceinline__ void zero() { d = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = d.x; f[1] = d.y; f[2] = d.z; f[3] = d.w; }
};
template <> struct Chunk<float, 1> {
    float d;
    __device__ __forceinline__ void load(const float* p) { d = __ldg(p); }
    __device__ __forceinline__ void load_once(const float* p) { d = __ldcs(p); }
    __device__ __forceinline__ void zero() { d = 0.f; }
    __device__ __forceinline__ void get(float (&f)[1]) const { f[0] = d; }
};

__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

template <typename T, int V, int MR, int ACT>
__global__ void __launch_bounds__(kWarps * 32) gated_rows_kernel(int M, int F, int K, const T* __restrict__ x, const T* __restrict__ w,
                                                                 const float* __restrict__ bias, T* __restrict__ h, T* __restrict__ pre) {
    constexpr int U = MR <= 2 ? 4 : 2;                             // loads of each row in flight
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, f = blockIdx.x * kWarps + (threadIdx.x >> 5);
    if (f >= F) return;
    const int m0 = blockIdx.y * MR;                                // more than MR rows: the weights come again, from the L2
    x += (long long)m0 * K;
    M -= m0;
    const T *wg = w + (long long)f * K, *wu = w + (long long)(F + f) * K;
    float g[MR] = {}, u[MR] = {};
    for (int k0 = lane * V; k0 < K; k0 += 32 * V * U) {
        Chunk<T, V> cg[U], cu[U];
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = k0 + i * 32 * V;
            if (k < K) { cg[i].load_once(wg + k); cu[i].load_once(wu + k); }
            else { cg[i].zero(); cu[i].zero(); }
        }
#pragma unroll
        for (int i = 0; i < U; ++i) {
            const int k = k0 + i * 32 * V;
            if (k >= K) break;
            float a[V], b[V];
            cg[i].get(a); cu[i].get(b);
#pragma unroll
            for (int m = 0; m < MR; ++m) {
                Chunk<T, V> cx;
                if (m < M) cx.load(x + (long long)m * K + k); else cx.zero();
                float v[V];
                cx.get(v);
#pragma unroll
                for (int e = 0; e < V; ++e) { g[m] = fmaf(a[e], v[e], g[m]); u[m] = fmaf(b[e], v[e], u[m]); }
            }
        }
    }
    const float bg = bias ? __ldg(bias + f) : 0.f, bu = bias ? __ldg(bias + F + f) : 0.f;
#pragma unroll
    for (int m = 0; m < MR; ++m) {
        const float zg = free_warp_sum(g[m]) + bg, zu = free_warp_sum(u[m]) + bu;
        if (lane == m && m < M) {
            const long long row = m0 + m;
            put(h + row * F + f, free_gate_act(ACT, zg) * zu);
            if (pre) { put(pre + row * 2 * F + f, zg); put(pre + row * 2 * F + F + f, zu); }
        }
    }
}

template <typename T, int V, int MR>
int launch(int act, int M, int F, int K, const T* x, const T* w, const float* bias, T* h, T* pre, cudaStream_t s) {
    auto kernel = act == FREE_ACT_SILU ? gated_rows_kernel<T, V, MR, FREE_ACT_SILU> : gated_rows_kernel<T, V, MR, FREE_ACT_GELU>;
    return free_launch(free_overlap_for_rows(M), kernel, dim3((unsigned)((F + kWarps - 1) / kWarps), (unsigned)((M + MR - 1) / MR)),
                       dim3(kWarps * 32), 0, s, M, F, K, x, w, bias, h, pre);
}

template <typename T, int V>
int rows(int act, int M, int F, int K, const void* x, const void* w, const float* bias, void* h, void* pre, cudaStream_t s) {
    const T *xt = (const T*)x, *wt = (const T*)w;
    T *ht = (T*)h, *pt = (T*)pre;
    if (M == 1) return launch<T, V, 1>(act, M, F, K, xt, wt, bias, ht, pt, s);
    if (M == 2) return launch<T, V, 2>(act, M, F, K, xt, wt, bias, ht, pt, s);
    if (M <= 4) return launch<T, V, 4>(act, M, F, K, xt, wt, bias, ht, pt, s);
    return launch<T, V, 8>(act, M, F, K, xt, wt, bias, ht, pt, s);
}

}  // namespace

// The time here goes with M F K, that of the tiled kernels, while their tiles are few, with K alone.  Measured (us, rows here /
// tiled): bf16, F = 4608, K = 1152, 1 / 4 / 8 rows 5.6 / 8.9 / 13.5, tiled 10.6 to 12.6; F = 1536, K = 384, 8 / 16 rows 4.7 / 7.3,
// tiled 5.8; F = 216, K = 1144, 16 rows 5.8, tiled 8.2.  fp32, F = 4608, K = 1152, 1 / 8 / 24 / 32 rows 5.3 / 18 / 38 / 49, tiled 49;
// F = 12288, K = 2048, 16 / 24 rows 115 / 174, tiled 164; F = 256, K = 4608, 96 / 128 rows 31 / 55, tiled 41; F = 216, K = 1146, 64 /
// 96 rows 15 / 21, tiled 17.  Short contractions, which the tiled fp32 kernel does not split: F = K = 64, 1024 rows 9.9, tiled 10.7.
bool gated_rows_wanted(int dtype, int M, int F, int K) {
    const long long work = (long long)M * F;
    return dtype == FREE_BF16 ? M <= 4 || work <= 14000 : M <= 24 || work <= (K < 128 ? 70000 : 20000);
}

int gated_rows_forward(int dtype, int act, int M, int F, int K, const void* x, const void* w, const float* bias, void* h, void* preact, cudaStream_t s) {
    if (dtype == FREE_BF16) return rows<__nv_bfloat16, 8>(act, M, F, K, x, w, bias, h, preact, s);
    return K % 4 == 0 ? rows<float, 4>(act, M, F, K, x, w, bias, h, preact, s) : rows<float, 1>(act, M, F, K, x, w, bias, h, preact, s);
}
