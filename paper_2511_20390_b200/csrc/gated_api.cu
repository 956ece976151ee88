// Gated linear layer: the elementwise part of its backward pass, sums of split products, and the entry points.
//
//   forward    z = x W^T + b;  h = act(z_gate) z_up                                      (one kernel)
//   backward   dz_gate = dh z_up act'(z_gate),  dz_up = dh act(z_gate),  db = sum_rows dz  (one pass over z and dh)
//              dx = dz W,  dW = dz^T x                                                    (two products)
// In bf16 dz is rounded to bf16 once, because both products take their operands in bf16: relative to a product's terms that
// is 2^-9, as large as the rounding of the outputs themselves.  db is summed from the unrounded values.
#include "gated.h"

namespace {

constexpr int kSms = 148;
constexpr int kThreads = 128;
constexpr int kRows = 4;                    // rows whose loads are in flight

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16(v); }

// dz of a block of V * kThreads columns over a run of rows; a thread keeps its columns, so db stays in its registers.
template <typename T, int V, bool FAST>
__global__ void __launch_bounds__(kThreads) gated_grad_kernel(int act, int M, int F, int chunks, const T* pre, const T* dh, T* dz, float* db) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int col = (blockIdx.x * kThreads + threadIdx.x) * V;
    if (col >= F) return;
    const int r0 = (int)((long long)M * blockIdx.y / chunks), r1 = (int)((long long)M * (blockIdx.y + 1) / chunks);
    float sg[V] = {}, su[V] = {};
    using P = Pack<T, V>;
    for (int r = r0; r < r1; r += kRows) {
        P g[kRows], u[kRows], d[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k)
            if (r + k < r1) {
                const long long row = r + k;
                g[k] = *reinterpret_cast<const P*>(pre + row * 2 * F + col);
                u[k] = *reinterpret_cast<const P*>(pre + row * 2 * F + F + col);
                d[k] = *reinterpret_cast<const P*>(dh + row * F + col);
            }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            if (r + k >= r1) break;
            const long long row = r + k;
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float zg = to_f(g[k].v[e]), zu = to_f(u[k].v[e]), dd = to_f(d[k].v[e]);
                const float arg = free_gate_arg(act, zg);
                const float s = FAST ? free_logistic_fast(arg) : free_logistic(arg);
                const float dg = dd * zu * free_gate_slope(act, zg, s), du = dd * zg * s;
                sg[e] += dg; su[e] += du;
                from_f(g[k].v[e], dg); from_f(u[k].v[e], du);
            }
            *reinterpret_cast<P*>(dz + row * 2 * F + col) = g[k];
            *reinterpret_cast<P*>(dz + row * 2 * F + F + col) = u[k];
        }
    }
    if (db) {
        float* o = db + (long long)blockIdx.y * 2 * F + col;
#pragma unroll
        for (int e = 0; e < V; ++e) { o[e] = sg[e]; o[F + e] = su[e]; }
    }
}

// out[c] = sum of rows [n][cols]: 32 columns x 16 slices per CTA, slices joined in order
__global__ void __launch_bounds__(512) gated_bias_kernel(int n, int cols, const float* p, float* out) {
    __shared__ float sh[16][33];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int c = blockIdx.x * 32 + tx;
    float s = 0.f;
    if (c < cols)
        for (int k = ty; k < n; k += 16) s += p[(long long)k * cols + c];
    sh[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && c < cols) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += sh[k][tx];
        out[c] = t;
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(256) gated_add_kernel(int parts, long long plane, long long n, const float* src, T* out) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * V; i < n; i += (long long)gridDim.x * 256 * V) {
        Pack<float, V> s = *reinterpret_cast<const Pack<float, V>*>(src + i);
        for (int p = 1; p < parts; ++p) {
            const Pack<float, V> t = *reinterpret_cast<const Pack<float, V>*>(src + p * plane + i);
#pragma unroll
            for (int e = 0; e < V; ++e) s.v[e] += t.v[e];
        }
        Pack<T, V> o;
#pragma unroll
        for (int e = 0; e < V; ++e) from_f(o.v[e], s.v[e]);
        *reinterpret_cast<Pack<T, V>*>(out + i) = o;
    }
}

int vec_of(int dtype, int F) { return dtype == FREE_BF16 ? 8 : (F % 4 == 0 ? 4 : 1); }

// Runs of rows of the elementwise pass: enough CTAs for the GPU, at least 16 rows each.
int chunks_of(int dtype, int M, int F) {
    const int v = vec_of(dtype, F), blocks = (F / v + kThreads - 1) / kThreads;
    int c = (kSms * 8 + blocks - 1) / blocks;
    if (c > M / 16) c = M / 16;
    return c < 1 ? 1 : (c > 65535 ? 65535 : c);
}

struct Layout { size_t dz, db, parts, total; };
Layout layout_of(int dtype, int M, int F, int K) {
    Layout l{};
    const size_t e = dtype == FREE_BF16 ? 2 : 4;
    l.dz = 0;
    l.db = free_round_up((size_t)M * 2 * F * e, 256);
    const int c = chunks_of(dtype, M, F);
    l.parts = l.db + (c > 1 ? free_round_up((size_t)c * 2 * F * 4, 256) : 0);
    size_t most = 0;                        // both products use the same part: they run one after the other
    for (int dw = 0; dw < 2; ++dw) {
        const GatedSplit g = dtype == FREE_BF16 ? gated_tc_split(dw != 0, M, F, K) : gated_simt_split(dw != 0, M, F, K);
        const size_t b = g.parts > 1 ? (size_t)g.parts * g.plane_rows * K * 4 : 0;
        if (b > most) most = b;
    }
    l.total = l.parts + most;
    return l;
}

bool known(int dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }
bool known_act(int act) { return act == FREE_ACT_SILU || act == FREE_ACT_GELU; }

template <typename T, int V, bool FAST>
int grad(int act, int M, int F, int chunks, const void* pre, const void* dh, void* dz, float* db, cudaStream_t s) {
    const dim3 grid((unsigned)((F / V + kThreads - 1) / kThreads), (unsigned)chunks);
    return free_launch(free_overlap_for_rows(M), gated_grad_kernel<T, V, FAST>, grid, dim3(kThreads), 0, s, act, M, F, chunks, (const T*)pre,
                       (const T*)dh, (T*)dz, db);
}

}  // namespace

int gated_add_parts(int dtype, int parts, long long plane, long long n, const float* src, void* out, cudaStream_t s) {
    const bool vec = n % 4 == 0 && plane % 4 == 0;
    const long long want = (n / (vec ? 4 : 1) + 255) / 256;
    const dim3 grid((unsigned)(want > kSms * 16 ? kSms * 16 : want));
    const bool ov = free_launch_overlap_enabled();
    if (dtype == FREE_BF16)                 // n and plane are multiples of K, a multiple of 8
        return free_launch(ov, gated_add_kernel<__nv_bfloat16, 4>, grid, dim3(256), 0, s, parts, plane, n, src, (__nv_bfloat16*)out);
    if (vec) return free_launch(ov, gated_add_kernel<float, 4>, grid, dim3(256), 0, s, parts, plane, n, src, (float*)out);
    return free_launch(ov, gated_add_kernel<float, 1>, grid, dim3(256), 0, s, parts, plane, n, src, (float*)out);
}

extern "C" int free_op_gated_linear(int dtype, int act, int M, int F, int K, const void* x, const void* w, const float* bias,
                                    void* h, void* preact, uint32_t* device_error, void* stream) {
    if (!known(dtype) || !known_act(act)) return FREE_ERR_ARG;
    if (M < 0 || F < 1 || K < 1) return FREE_ERR_SHAPE;
    if (F > 0x3fffffff) return FREE_ERR_UNSUPPORTED;
    if (dtype == FREE_BF16 && !gated_tc_supported(F, K)) return FREE_ERR_UNSUPPORTED;
    if (M == 0) return FREE_OK;
    if (!x || !w || !h || (dtype == FREE_BF16 && !device_error)) return FREE_ERR_ARG;
    if (!free_aligned16(x) || !free_aligned16(w) || !free_aligned16(h) || !free_aligned16(preact) || (reinterpret_cast<uintptr_t>(bias) & 3u) ||
        (reinterpret_cast<uintptr_t>(device_error) & 3u)) return FREE_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (dtype == FREE_FP32) return gated_simt_forward(act, M, F, K, (const float*)x, (const float*)w, bias, (float*)h, (float*)preact, s);
    return gated_tc_forward(act, M, F, K, x, w, bias, h, preact, device_error, s);
}

extern "C" size_t free_op_gated_linear_bwd_workspace_bytes(int dtype, int M, int F, int K) {
    if (!known(dtype) || M < 1 || F < 1 || F > 0x3fffffff || K < 1 || (dtype == FREE_BF16 && !gated_tc_supported(F, K))) return 0;
    return layout_of(dtype, M, F, K).total;
}

extern "C" int free_op_gated_linear_bwd(int dtype, int act, int M, int F, int K, const void* x, const void* w, const void* preact,
                                        const void* dh, void* dx, void* dw, float* dbias, void* ws, size_t ws_bytes,
                                        uint32_t* device_error, void* stream) {
    if (!known(dtype) || !known_act(act)) return FREE_ERR_ARG;
    if (M < 0 || F < 1 || K < 1) return FREE_ERR_SHAPE;
    if (F > 0x3fffffff) return FREE_ERR_UNSUPPORTED;
    if (dtype == FREE_BF16 && !gated_tc_supported(F, K)) return FREE_ERR_UNSUPPORTED;
    if (!dx && !dw && !dbias) return FREE_OK;
    if (M > 0 && (!preact || !dh || (dx && !w) || (dw && !x))) return FREE_ERR_ARG;
    if (M > 0 && dtype == FREE_BF16 && !device_error) return FREE_ERR_ARG;
    if (!free_aligned16(x) || !free_aligned16(w) || !free_aligned16(preact) || !free_aligned16(dh) || !free_aligned16(dx) || !free_aligned16(dw) ||
        !free_aligned16(ws) || (reinterpret_cast<uintptr_t>(dbias) & 3u) || (reinterpret_cast<uintptr_t>(device_error) & 3u)) return FREE_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const size_t e = dtype == FREE_BF16 ? 2 : 4;
    if (M == 0) {                           // sums over no rows
        if (dw) FREE_CUDA_TRY(cudaMemsetAsync(dw, 0, (size_t)2 * F * K * e, s));
        if (dbias) FREE_CUDA_TRY(cudaMemsetAsync(dbias, 0, (size_t)2 * F * 4, s));
        return FREE_OK;
    }
    const Layout l = layout_of(dtype, M, F, K);
    if (!ws || ws_bytes < l.total) return FREE_ERR_WORKSPACE;
    char* base = (char*)ws;
    void* dz = base + l.dz;
    float* parts = (float*)(base + l.parts);
    const int chunks = chunks_of(dtype, M, F);
    float* db = !dbias ? nullptr : (chunks > 1 ? (float*)(base + l.db) : dbias);
    if (dtype == FREE_BF16) FREE_TRY((grad<__nv_bfloat16, 8, true>(act, M, F, chunks, preact, dh, dz, db, s)));
    else if (vec_of(dtype, F) == 4) FREE_TRY((grad<float, 4, false>(act, M, F, chunks, preact, dh, dz, db, s)));
    else FREE_TRY((grad<float, 1, false>(act, M, F, chunks, preact, dh, dz, db, s)));
    if (dbias && chunks > 1)
        FREE_TRY(free_launch(free_launch_overlap_enabled(), gated_bias_kernel, dim3((2u * F + 31) / 32), dim3(512), 0, s, chunks, 2 * F, (const float*)db, dbias));
    if (dtype == FREE_BF16) {
        if (dw) FREE_TRY(gated_tc_backward(true, M, F, K, x, w, dz, dw, parts, device_error, s));
        if (dx) FREE_TRY(gated_tc_backward(false, M, F, K, x, w, dz, dx, parts, device_error, s));
    } else {
        if (dw) FREE_TRY(gated_simt_backward(true, M, F, K, (const float*)x, (const float*)w, (const float*)dz, (float*)dw, parts, s));
        if (dx) FREE_TRY(gated_simt_backward(false, M, F, K, (const float*)x, (const float*)w, (const float*)dz, (float*)dx, parts, s));
    }
    return FREE_OK;
}
