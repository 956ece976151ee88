// Gated linear layer: the elementwise part of its backward pass, the sums that end it, and the entry points.
//
//   forward    z = x W^T + b;  h = act(z_gate) z_up                                      (one kernel)
//   backward   dz_gate = dh z_up act'(z_gate),  dz_up = dh act(z_gate),  db = sum_rows dz  (one pass over z and dh)
//              dx = dz W,  dW = dz^T x                                                    (two products)
// The elementwise pass is bound by HBM (z and dh in, dz out): 193 us for 24576 rows, F = 4608 (1.13 GB, 5.9 TB/s).
// In bf16 dz is rounded to bf16 once, because both products take their operands in bf16: each term of a product is off by half
// a step at most (2^-8 of it; 1.7e-3 root mean square), as much as the outputs' own rounding, so gradients are off by 2.3e-3 in
// the 2-norm instead of 1.7e-3.  db is summed from the unrounded values.
#include "gated.h"

namespace {

constexpr int kSms = 148;
constexpr int kMaxThreads = 256;
constexpr int kPerSm = 4;                    // such CTAs per SM (register budget)
constexpr int kRows = 2;                     // rows whose loads are in flight

template <typename T, int V> struct alignas(sizeof(T) * V) Pack { T v[V]; };
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16(v); }

// V values as one access; bf16 pairs stay packed in 32-bit words
template <typename T, int V> struct Vals {
    Pack<uint32_t, V * (int)sizeof(T) / 4> d;
    __device__ __forceinline__ float operator[](int i) const {
        if (sizeof(T) == 4) return __uint_as_float(d.v[i]);
        return __uint_as_float(i % 2 ? d.v[i / 2] & 0xffff0000u : d.v[i / 2] << 16);
    }
    __device__ __forceinline__ void set(const float (&f)[V]) {
        if (sizeof(T) == 4) {
#pragma unroll
            for (int i = 0; i < V; ++i) d.v[i % (V * (int)sizeof(T) / 4)] = __float_as_uint(f[i]);
        } else {
#pragma unroll
            for (int i = 0; i < V / 2; ++i) {
                const __nv_bfloat162 b = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
                d.v[i] = *reinterpret_cast<const uint32_t*>(&b);
            }
        }
    }
    __device__ __forceinline__ void load(const T* p) { d = *reinterpret_cast<const decltype(d)*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<decltype(d)*>(p) = d; }
};

// dz of a block of columns over a run of rows; a thread keeps its V columns, so db stays in its registers.
template <typename T, int V, int ACT>
__global__ void __launch_bounds__(kMaxThreads, kPerSm) gated_grad_kernel(int M, int F, int chunks, const T* __restrict__ pre,
                                                                         const T* __restrict__ dh, T* __restrict__ dz, float* __restrict__ db) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int col = (blockIdx.x * blockDim.x + threadIdx.x) * V;
    if (col >= F) return;
    float sg[V] = {}, su[V] = {};
    using P = Vals<T, V>;
    // rows blockIdx.y, blockIdx.y + chunks, ...: the CTAs in flight work on neighbouring rows
    for (long long r = blockIdx.y; r < M; r += (long long)kRows * chunks) {
        P g[kRows], u[kRows], d[kRows];
#pragma unroll
        for (int k = 0; k < kRows; ++k) {                          // past the last row: this one again, not counted or stored
            const long long row = r + (long long)k * chunks < M ? r + (long long)k * chunks : r;
            g[k].load(pre + row * 2 * F + col);
            u[k].load(pre + row * 2 * F + F + col);
            d[k].load(dh + row * F + col);
        }
#pragma unroll
        for (int k = 0; k < kRows; ++k) {
            const long long row = r + (long long)k * chunks;
            if (row >= M) break;
            float dg[V], du[V];
#pragma unroll
            for (int e = 0; e < V; ++e) {
                const float zg = g[k][e], dd = d[k][e], arg = free_gate_arg(ACT, zg);
                const float s = sizeof(T) == 2 ? free_logistic_fast(arg) : free_logistic(arg);
                // rounded products: the sums take the same values whether dz is stored or not
                dg[e] = __fmul_rn(dd * u[k][e], free_gate_slope(ACT, zg, s)); du[e] = __fmul_rn(dd, zg * s);
                sg[e] += dg[e]; su[e] += du[e];
            }
            if (dz) {                                              // not where the bias gradient alone is wanted
                P o;
                o.set(dg);
                o.store(dz + row * 2 * F + col);
                o.set(du);
                o.store(dz + row * 2 * F + F + col);
            }
        }
    }
    if (db) {
        float* o = db + (long long)blockIdx.y * 2 * F + col;
#pragma unroll
        for (int e = 0; e < V; ++e) { o[e] = sg[e]; o[F + e] = su[e]; }
    }
}

// What is left once the products are done, in one launch: the parts of dx and of dw added in their order and rounded, and the
// partial rows of db added (32 columns x 8 slices of the rows per CTA, slices joined in order).
// Launched plainly: brought up early, as the kernels before it are, its blocks wait beside the product and the whole pass takes
// longer (300 rows, F = 4608: 40 us against 35; 8192 rows, F = 1024: 64 against 58).  Two sums of a thread are in flight: one is 3 us slower where there are many,
// four 13 us slower where there are few and many parts (20000 rows, F = 256).
constexpr int kSums = 2;
template <typename T> struct Sum { const float* src; T* out; long long n, plane; int parts, blocks; };
template <typename T> struct FinishArgs {
    Sum<T> dx, dw;
    const float* db; float* dbias; int chunks, cols, db_blocks;
};
template <typename T, int V>
__global__ void __launch_bounds__(256) gated_finish_kernel(const FinishArgs<T> a) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    int block = blockIdx.x;
    if (block < a.db_blocks) {                  // first: these are the longest
        __shared__ float sh[8][33];
        const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
        const int c = block * 32 + tx;
        float s = 0.f;
        if (c < a.cols) {
#pragma unroll 8
            for (int k = ty; k < a.chunks; k += 8) s += a.db[(long long)k * a.cols + c];
        }
        sh[ty][tx] = s;
        __syncthreads();
        if (ty == 0 && c < a.cols) {
            float t = 0.f;
#pragma unroll
            for (int k = 0; k < 8; ++k) t += sh[k][tx];
            a.dbias[c] = t;
        }
        return;
    }
    block -= a.db_blocks;
    const Sum<T> j = block < a.dx.blocks ? a.dx : a.dw;
    if (block >= a.dx.blocks) block -= a.dx.blocks;
    for (long long i = ((long long)block * kSums * 256 + threadIdx.x) * V; i < j.n; i += (long long)j.blocks * kSums * 256 * V) {
        Pack<float, V> s[kSums];
#pragma unroll
        for (int u = 0; u < kSums; ++u)
            if (i + u * 256 * V < j.n) s[u] = *reinterpret_cast<const Pack<float, V>*>(j.src + i + u * 256 * V);
#pragma unroll 2
        for (int p = 1; p < j.parts; ++p) {
#pragma unroll
            for (int u = 0; u < kSums; ++u) {
                if (i + u * 256 * V >= j.n) break;
                const Pack<float, V> t = *reinterpret_cast<const Pack<float, V>*>(j.src + p * j.plane + i + u * 256 * V);
#pragma unroll
                for (int e = 0; e < V; ++e) s[u].v[e] += t.v[e];
            }
        }
#pragma unroll
        for (int u = 0; u < kSums; ++u) {
            if (i + u * 256 * V >= j.n) break;
            Pack<T, V> o;
#pragma unroll
            for (int e = 0; e < V; ++e) from_f(o.v[e], s[u].v[e]);
            *reinterpret_cast<Pack<T, V>*>(j.out + i + u * 256 * V) = o;
        }
    }
}

int vec_of(int dtype, int F) { return dtype == FREE_BF16 ? 8 : (F % 4 == 0 ? 4 : 1); }

// CTAs of the elementwise pass: column blocks of equal width, and runs of rows, enough for the GPU and at least 16 rows each
// (fewer, down to 4, where that would leave SMs idle).
struct GradGrid { int blocks, threads, chunks; };
GradGrid grad_grid(int dtype, int M, int F) {
    const int v = vec_of(dtype, F), vecs = F / v;
    GradGrid g;
    g.blocks = (vecs + kMaxThreads - 1) / kMaxThreads;
    g.threads = ((vecs + g.blocks - 1) / g.blocks + 31) / 32 * 32;
    g.chunks = (int)(((long long)kSms * 16 * 128 / g.threads + g.blocks - 1) / g.blocks);
    // (every run leaves a partial row of db: 4173 rows, F = 1536, whole backward pass: 48.7 us with 16 rows, 52 with 8; 300 rows,
    // F = 4608: 41 us with 16 rows, 37 with 8)
    int least = 16;
    while (least > 4 && (long long)g.blocks * (M / least) < kSms) least /= 2;
    if (g.chunks > M / least) g.chunks = M / least;
    if (g.chunks < 1) g.chunks = 1;
    return g;
}

// Workspace: dz, the partial rows of db, the parts of dx, the parts of dw.
struct Layout { size_t dz, db, dx, dw, total; int chunks; GatedSplit gx, gw; };
Layout layout_of(int dtype, int M, int F, int K) {
    Layout l{};
    const size_t e = dtype == FREE_BF16 ? 2 : 4;
    l.chunks = grad_grid(dtype, M, F).chunks;
    l.gx = dtype == FREE_BF16 ? gated_tc_split(false, M, F, K) : gated_simt_split(false, M, F, K);
    l.gw = dtype == FREE_BF16 ? gated_tc_split(true, M, F, K) : gated_simt_split(true, M, F, K);
    auto parts = [&](const GatedSplit& g) { return g.parts > 1 ? free_round_up((size_t)g.parts * g.plane_rows * K * 4, 256) : 0; };
    l.dz = 0;
    l.db = free_round_up((size_t)M * 2 * F * e, 256);
    l.dx = l.db + (l.chunks > 1 ? free_round_up((size_t)l.chunks * 2 * F * 4, 256) : 0);
    l.dw = l.dx + parts(l.gx);
    l.total = l.dw + parts(l.gw);
    return l;
}

template <typename T, int V>
Sum<T> sum_of(const GatedSplit& g, long long rows, int K, const float* src, void* out) {
    Sum<T> j{src, (T*)out, rows * K, g.plane_rows * K, g.parts, 0};
    if (!out || g.parts == 1) return j;
    const long long want = (j.n / V + kSums * 256 - 1) / (kSums * 256);
    j.blocks = (int)(want > kSms * 16 ? kSms * 16 : want);
    return j;
}

template <typename T, int V>
int finish(const Layout& l, int M, int F, int K, char* base, void* dx, void* dw, float* dbias, cudaStream_t s) {
    FinishArgs<T> a{};
    a.dx = sum_of<T, V>(l.gx, M, K, (const float*)(base + l.dx), dx);
    a.dw = sum_of<T, V>(l.gw, 2LL * F, K, (const float*)(base + l.dw), dw);
    a.db = (const float*)(base + l.db); a.dbias = dbias; a.chunks = l.chunks; a.cols = 2 * F;
    a.db_blocks = dbias && l.chunks > 1 ? (a.cols + 31) / 32 : 0;
    const long long grid = (long long)a.dx.blocks + a.dw.blocks + a.db_blocks;
    if (grid == 0) return FREE_OK;
    return free_launch(false, gated_finish_kernel<T, V>, dim3((unsigned)grid), dim3(256), 0, s, a);
}

// Sizes whose tile counts and coordinates fit 32 bits.
constexpr int kMaxRows = 1 << 30, kMaxCols = 1 << 28;
bool too_large(int M, int F, int K) { return M > kMaxRows || F > kMaxCols || K > kMaxCols; }
bool known(int dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }
bool known_act(int act) { return act == FREE_ACT_SILU || act == FREE_ACT_GELU; }

template <typename T, int V>
int grad(int dtype, int act, int M, int F, const void* pre, const void* dh, void* dz, float* db, cudaStream_t s) {
    const GradGrid g = grad_grid(dtype, M, F);
    auto kernel = act == FREE_ACT_SILU ? gated_grad_kernel<T, V, FREE_ACT_SILU> : gated_grad_kernel<T, V, FREE_ACT_GELU>;
    return free_launch(free_overlap_for_rows(M), kernel, dim3((unsigned)g.blocks, (unsigned)g.chunks), dim3(g.threads), 0, s, M, F, g.chunks,
                       (const T*)pre, (const T*)dh, (T*)dz, db);
}

}  // namespace

extern "C" int free_op_gated_linear(int dtype, int act, int M, int F, int K, const void* x, const void* w, const float* bias,
                                    void* h, void* preact, uint32_t* device_error, void* stream) {
    if (!known(dtype) || !known_act(act)) return FREE_ERR_ARG;
    if (M < 0 || F < 1 || K < 1) return FREE_ERR_SHAPE;
    if (too_large(M, F, K)) return FREE_ERR_UNSUPPORTED;
    if (dtype == FREE_BF16 && !gated_tc_supported(F, K)) return FREE_ERR_UNSUPPORTED;
    if (M == 0) return FREE_OK;
    if (!x || !w || !h || (dtype == FREE_BF16 && !device_error)) return FREE_ERR_ARG;
    if (!free_aligned16(x) || !free_aligned16(w) || !free_aligned16(bias) || !free_aligned16(h) || !free_aligned16(preact) ||
        (reinterpret_cast<uintptr_t>(device_error) & 3u)) return FREE_ERR_ALIGN;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    if (gated_rows_wanted(dtype, M, F, K)) return gated_rows_forward(dtype, act, M, F, K, x, w, bias, h, preact, s);
    if (dtype == FREE_FP32) return gated_simt_forward(act, M, F, K, (const float*)x, (const float*)w, bias, (float*)h, (float*)preact, s);
    return gated_tc_forward(act, M, F, K, x, w, bias, h, preact, device_error, s);
}

extern "C" size_t free_op_gated_linear_bwd_workspace_bytes(int dtype, int M, int F, int K) {
    if (!known(dtype) || M < 1 || F < 1 || K < 1 || too_large(M, F, K) || (dtype == FREE_BF16 && !gated_tc_supported(F, K))) return 0;
    return layout_of(dtype, M, F, K).total;
}

extern "C" int free_op_gated_linear_bwd(int dtype, int act, int M, int F, int K, const void* x, const void* w, const void* preact,
                                        const void* dh, void* dx, void* dw, float* dbias, void* ws, size_t ws_bytes,
                                        uint32_t* device_error, void* stream) {
    if (!known(dtype) || !known_act(act)) return FREE_ERR_ARG;
    if (M < 0 || F < 1 || K < 1) return FREE_ERR_SHAPE;
    if (too_large(M, F, K)) return FREE_ERR_UNSUPPORTED;
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
    void* dz = dx || dw ? base + l.dz : nullptr;
    float* db = !dbias ? nullptr : (l.chunks > 1 ? (float*)(base + l.db) : dbias);
    float *px = (float*)(base + l.dx), *pw = (float*)(base + l.dw);
    if (dtype == FREE_BF16) {
        FREE_TRY((grad<__nv_bfloat16, 8>(dtype, act, M, F, preact, dh, dz, db, s)));
        // dx walks over dz from its end, dw then from its start: each begins with what the L2 still holds
        if (dx) FREE_TRY(gated_tc_backward(false, l.gx, M, F, K, x, w, dz, dx, px, device_error, s));
        if (dw) FREE_TRY(gated_tc_backward(true, l.gw, M, F, K, x, w, dz, dw, pw, device_error, s));
        return finish<__nv_bfloat16, 4>(l, M, F, K, base, dx, dw, dbias, s);        // K % 8 == 0
    }
    const float *xf = (const float*)x, *wf = (const float*)w, *zf = (const float*)dz;
    if (vec_of(dtype, F) == 4) FREE_TRY((grad<float, 4>(dtype, act, M, F, preact, dh, dz, db, s)));
    else FREE_TRY((grad<float, 1>(dtype, act, M, F, preact, dh, dz, db, s)));
    if (dw) FREE_TRY(gated_simt_backward(true, l.gw, M, F, K, xf, wf, zf, (float*)dw, pw, s));
    if (dx) FREE_TRY(gated_simt_backward(false, l.gx, M, F, K, xf, wf, zf, (float*)dx, px, s));
    return K % 4 == 0 ? finish<float, 4>(l, M, F, K, base, dx, dw, dbias, s) : finish<float, 1>(l, M, F, K, base, dx, dw, dbias, s);
}
