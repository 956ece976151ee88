// fp32 products of the gated linear layer on CUDA cores (the exact-arithmetic mode), forward and backward: any sizes.
//
//   GATED   z = x W^T + b, h = act(z_gate) z_up;   DX  dx = dz W;   DW  dW = dz^T x
//
// A CTA computes a tile of TM x 128 outputs with 8 x 8 per thread, the contraction staged 16 deep through two shared-memory
// buffers (the next stage's global loads are in flight while this one is multiplied).  A thread's eight columns are four of
// each half of the tile: in GATED the halves are 64 gate columns and the matching 64 up columns, so the thread that holds
// z_gate holds z_up.  Bound by the fp32 pipe: 64 multiply-adds against four 16-byte shared-memory reads per thread and step.
// 4096 rows, F = 1536, K = 384: 226 us forward, 43 TFLOP/s (the pipe 0.65 active), 460 us for the whole backward pass.
// TM is 64 where 128-row tiles would leave SMs idle in the last wave.  Few tiles and a long contraction are split and the parts
// added in order: forward by the CTAs of a cluster, through their shared memory (z has to be whole before the activation), backward
// through the workspace.  F = 256, K = 4608, 1024 rows: 129 us, unsplit 291; F = 1536, K = 384, 100 rows: 16, unsplit 30.
#include "gated.h"

namespace {

enum { GATED = 0, DX = 1, DW = 2 };

constexpr int TN = 128, TK = 16;
constexpr int kSms = 148;
constexpr int kMaxGridY = 65535;           // column tiles of a launch

struct Args {
    int M, N, depth;                       // output rows and columns (GATED: N = F), contraction
    const float *A, *B;
    long long lda, ldb;
    const float* bias;
    int act, F;
    float *out, *pre;                      // GATED: pre [M, 2F] or nullptr
    int parts; long long plane;            // elements between the parts
    int tile_n0;                           // first column tile of the launch
};

// Two multiply-adds as one instruction (each rounded as fmaf): the FMA pipe is fed with half the issue slots.
__device__ __forceinline__ void fma2(uint64_t& acc, uint64_t a, uint64_t b) {
    asm("fma.rn.f32x2 %0, %1, %2, %0;" : "+l"(acc) : "l"(a), "l"(b));
}
__device__ __forceinline__ uint64_t both(float v) {
    uint64_t r;
    asm("mov.b64 %0, {%1, %1};" : "=l"(r) : "f"(v));
    return r;
}
__device__ __forceinline__ void split2(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }

// A stage of one operand: ROWS x 16 values, contraction-major in shared memory ([16][ROWS + 4]).
// KMAJOR: memory holds rows of the contraction (element (r, k) at r * ld + k); otherwise k * ld + r.
template <int ROWS, int THREADS, bool KMAJOR, bool VEC> struct Loader {
    static constexpr int N = ROWS * TK / 4 / THREADS;       // 16-byte groups per thread
    float v[N][4];
    // split: the upper half of the rows is read from `shift` rows further on (gate rows, then up rows)
    __device__ __forceinline__ void fetch(const float* p, long long ld, int row0, int rows, int half_rows, int shift, int k0, int k1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int idx = threadIdx.x + i * THREADS;
            if (KMAJOR) {
                const int lr = idx / 4, k = k0 + (idx % 4) * 4;
                const int local = lr < half_rows ? lr : lr - half_rows;
                const bool in = row0 + local < rows;
                const float* q = p + (long long)(row0 + local + (lr < half_rows ? 0 : shift)) * ld + k;
                if (VEC && in && k + 3 < k1) {
                    const float4 f = __ldg(reinterpret_cast<const float4*>(q));
                    v[i][0] = f.x; v[i][1] = f.y; v[i][2] = f.z; v[i][3] = f.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = in && k + e < k1 ? __ldg(q + e) : 0.f;
                }
            } else {
                const int k = k0 + idx / (ROWS / 4), r = row0 + idx % (ROWS / 4) * 4;
                const float* q = p + (long long)k * ld + r;
                if (VEC && k < k1 && r + 3 < rows) {
                    const float4 f = __ldg(reinterpret_cast<const float4*>(q));
                    v[i][0] = f.x; v[i][1] = f.y; v[i][2] = f.z; v[i][3] = f.w;
                } else {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[i][e] = k < k1 && r + e < rows ? __ldg(q + e) : 0.f;
                }
            }
        }
    }
    __device__ __forceinline__ void store(float (*sm)[ROWS + 4]) const {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const int idx = threadIdx.x + i * THREADS;
            if (KMAJOR) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sm[(idx % 4) * 4 + e][idx / 4] = v[i][e];
            } else {
                *reinterpret_cast<float4*>(&sm[idx / (ROWS / 4)][idx % (ROWS / 4) * 4]) = make_float4(v[i][0], v[i][1], v[i][2], v[i][3]);
            }
        }
    }
};

// bias, activation and product of four columns of row m
__device__ __forceinline__ void finish(const Args& a, int m, int n0, const float* gate, const float* up) {
    if (m >= a.M) return;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int n = n0 + j;
        if (n >= a.F) continue;
        float g = gate[j], u = up[j];
        if (a.bias) { g += __ldg(a.bias + n); u += __ldg(a.bias + a.F + n); }
        a.out[(long long)m * a.F + n] = free_gate_act(a.act, g) * u;
        if (a.pre) { a.pre[(long long)m * 2 * a.F + n] = g; a.pre[(long long)m * 2 * a.F + a.F + n] = u; }
    }
}
__device__ __forceinline__ float4 cluster_read(const void* mine, int rank) {       // what another CTA has at the same place
    uint32_t at;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(at) : "r"((uint32_t)__cvta_generic_to_shared(mine)), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(at) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_barrier() {
    asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");     // release, acquire
}

// S > 1 (GATED): the S CTAs of a cluster take parts of the contraction; each then joins and finishes 8 / S rows of every thread.
template <int MODE, int TM, bool VEC, int S>
__device__ __forceinline__ void gated_simt_tile(const Args& a) {
    constexpr int THREADS = TM * 2;
    constexpr int HALF = MODE == GATED ? TN / 2 : TN;       // output columns of a tile
    constexpr int STAGES = 2 * TK * (TM + 4 + TN + 4), JOIN = S > 1 ? TM * TN : 0;
    __shared__ __align__(16) float smem[STAGES > JOIN ? STAGES : JOIN];
    float (*As)[TK][TM + 4] = reinterpret_cast<float (*)[TK][TM + 4]>(smem);
    float (*Bs)[TK][TN + 4] = reinterpret_cast<float (*)[TK][TN + 4]>(smem + 2 * TK * (TM + 4));
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    const int m0 = blockIdx.x * TM, n0 = (a.tile_n0 + blockIdx.y) * HALF;
    const int kbeg = (int)((long long)a.depth * blockIdx.z / a.parts), kend = (int)((long long)a.depth * (blockIdx.z + 1) / a.parts);
    // parts begin at multiples of four so that 16-byte reads along the contraction stay aligned
    const int k0 = kbeg / 4 * 4, k1 = blockIdx.z + 1 == a.parts ? kend : kend / 4 * 4;
    Loader<TM, THREADS, MODE != DW, VEC> la;
    Loader<TN, THREADS, MODE == GATED, VEC> lb;
    uint64_t acc2[8][4] = {};                              // columns (0, 1), (2, 3) of the lower half, then of the upper
    auto fetch = [&](int k) {
        la.fetch(a.A, a.lda, m0, a.M, TM, 0, k, k1);
        lb.fetch(a.B, a.ldb, n0, a.N, HALF, MODE == GATED ? a.F : 0, k, k1);
    };
    if (k0 < k1) {
        fetch(k0);
        la.store(As[0]); lb.store(Bs[0]);
    }
    __syncthreads();
    int buf = 0;
    for (int k = k0; k < k1; k += TK, buf ^= 1) {
        const bool more = k + TK < k1;
        if (more) fetch(k + TK);
        // the fragments of the next step are read while this one is multiplied
        float4 a0 = *reinterpret_cast<const float4*>(&As[buf][0][ty * 4]), a1 = *reinterpret_cast<const float4*>(&As[buf][0][TM / 2 + ty * 4]);
        ulonglong2 b0 = *reinterpret_cast<const ulonglong2*>(&Bs[buf][0][tx * 4]), b1 = *reinterpret_cast<const ulonglong2*>(&Bs[buf][0][TN / 2 + tx * 4]);
#pragma unroll
        for (int kk = 0; kk < TK; ++kk) {
            const float av[8] = {a0.x, a0.y, a0.z, a0.w, a1.x, a1.y, a1.z, a1.w};
            const ulonglong2 c0 = b0, c1 = b1;
            if (kk + 1 < TK) {
                a0 = *reinterpret_cast<const float4*>(&As[buf][kk + 1][ty * 4]);
                a1 = *reinterpret_cast<const float4*>(&As[buf][kk + 1][TM / 2 + ty * 4]);
                b0 = *reinterpret_cast<const ulonglong2*>(&Bs[buf][kk + 1][tx * 4]);
                b1 = *reinterpret_cast<const ulonglong2*>(&Bs[buf][kk + 1][TN / 2 + tx * 4]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint64_t a2 = both(av[i]);
                fma2(acc2[i][0], a2, c0.x); fma2(acc2[i][1], a2, c0.y);
                fma2(acc2[i][2], a2, c1.x); fma2(acc2[i][3], a2, c1.y);
            }
        }
        if (more) { la.store(As[buf ^ 1]); lb.store(Bs[buf ^ 1]); }   // last read before the previous barrier
        __syncthreads();
    }
    if constexpr (S > 1) {
        float4* mine = reinterpret_cast<float4*>(smem) + threadIdx.x;          // [row][gate or up][thread]
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            ulonglong2 lo, hi;
            lo.x = acc2[i][0]; lo.y = acc2[i][1]; hi.x = acc2[i][2]; hi.y = acc2[i][3];
            *reinterpret_cast<ulonglong2*>(mine + (2 * i) * THREADS) = lo;
            *reinterpret_cast<ulonglong2*>(mine + (2 * i + 1) * THREADS) = hi;
        }
        cluster_barrier();
#pragma unroll
        for (int r = 0; r < 8 / S; ++r) {
            const int i = blockIdx.z * (8 / S) + r;
            float4 g = make_float4(0.f, 0.f, 0.f, 0.f), u = g;
#pragma unroll
            for (int q = 0; q < S; ++q) {
                const float4 p = cluster_read(mine + (2 * i) * THREADS, q), t = cluster_read(mine + (2 * i + 1) * THREADS, q);
                g.x += p.x; g.y += p.y; g.z += p.z; g.w += p.w;
                u.x += t.x; u.y += t.y; u.z += t.z; u.w += t.w;
            }
            finish(a, m0 + (i < 4 ? ty * 4 + i : TM / 2 + ty * 4 + i - 4), n0 + tx * 4, &g.x, &u.x);
        }
        cluster_barrier();                                  // nobody leaves while its sums are read
        return;
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int m = m0 + (i < 4 ? ty * 4 + i : TM / 2 + ty * 4 + i - 4);
        if (m >= a.M) continue;
        float acc[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) split2(acc2[i][j], acc[2 * j], acc[2 * j + 1]);
        if (MODE == GATED) {
            finish(a, m, n0 + tx * 4, acc, acc + 4);
        } else {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = n0 + h * (TN / 2) + tx * 4;
                float* q = a.out + blockIdx.z * a.plane + (long long)m * a.N + n;
                if (VEC && n + 3 < a.N) *reinterpret_cast<float4*>(q) = make_float4(acc[4 * h], acc[4 * h + 1], acc[4 * h + 2], acc[4 * h + 3]);
                else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n + j < a.N) q[j] = acc[4 * h + j];
                }
            }
        }
    }
}

template <int MODE, int TM, bool VEC> __global__ void __launch_bounds__(TM * 2) gated_simt_kernel(const Args a) { gated_simt_tile<MODE, TM, VEC, 1>(a); }
template <bool VEC, int S> __global__ void __launch_bounds__(128) __cluster_dims__(1, 1, S) gated_simt_split_kernel(const Args a) {
    gated_simt_tile<GATED, 64, VEC, S>(a);
}

template <int MODE>
int launch(Args a, bool vec, cudaStream_t s) {
    constexpr int cols = MODE == GATED ? TN / 2 : TN;
    const long long nn = (a.N + cols - 1) / cols, m128 = ((long long)a.M + 127) / 128, m64 = ((long long)a.M + 63) / 64;
    // time of a wave in 64-row units; equal: the larger tile (fewer shared-memory reads per product)
    const long long w128 = 2 * ((m128 * nn * a.parts + kSms - 1) / kSms), w64 = (m64 * nn * a.parts + kSms - 1) / kSms;
    for (a.tile_n0 = 0; a.tile_n0 < nn; a.tile_n0 += kMaxGridY) {
        const dim3 grid((unsigned)(w64 < w128 ? m64 : m128), (unsigned)(nn - a.tile_n0 < kMaxGridY ? nn - a.tile_n0 : kMaxGridY), (unsigned)a.parts);
        if (w64 < w128) {
            if (vec) gated_simt_kernel<MODE, 64, true><<<grid, 128, 0, s>>>(a);
            else gated_simt_kernel<MODE, 64, false><<<grid, 128, 0, s>>>(a);
        } else {
            if (vec) gated_simt_kernel<MODE, 128, true><<<grid, 256, 0, s>>>(a);
            else gated_simt_kernel<MODE, 128, false><<<grid, 256, 0, s>>>(a);
        }
        FREE_TRY(free_check_launch());
    }
    return FREE_OK;
}

}  // namespace

int gated_simt_forward(int act, int M, int F, int K, const float* x, const float* w, const float* bias, float* h, float* preact, cudaStream_t s) {
    Args a{};
    a.M = M; a.N = F; a.depth = K; a.A = x; a.B = w; a.lda = K; a.ldb = K; a.bias = bias; a.act = act; a.F = F; a.out = h; a.pre = preact; a.parts = 1;
    // few tiles: as many CTAs to each as leave an SM three at most, with at least 64 of the contraction (at most two: 0 to 30% slower,
    // 12288 columns, 40 rows 223 against 164 us; at most four: 0 to 18% slower)
    const long long tiles = ((long long)M + 63) / 64 * (((long long)F + TN / 2 - 1) / (TN / 2));
    const bool vec = K % 4 == 0;
    if (tiles * 2 <= 3 * kSms && K >= 128) {
        a.parts = tiles * 8 <= 3 * kSms && K >= 512 ? 8 : tiles * 4 <= 3 * kSms && K >= 256 ? 4 : 2;
        const dim3 grid((unsigned)((M + 63) / 64), (unsigned)((F + TN / 2 - 1) / (TN / 2)), (unsigned)a.parts);
        if (vec) (a.parts == 8 ? gated_simt_split_kernel<true, 8> : a.parts == 4 ? gated_simt_split_kernel<true, 4> : gated_simt_split_kernel<true, 2>)<<<grid, 128, 0, s>>>(a);
        else (a.parts == 8 ? gated_simt_split_kernel<false, 8> : a.parts == 4 ? gated_simt_split_kernel<false, 4> : gated_simt_split_kernel<false, 2>)<<<grid, 128, 0, s>>>(a);
        return free_check_launch();
    }
    return launch<GATED>(a, vec, s);
}

// Enough parts to give every SM two tiles, each at least 256 deep.
GatedSplit gated_simt_split(bool dw, int M, int F, int K) {
    const long long rows = dw ? 2LL * F : M, depth = dw ? M : 2LL * F;
    const long long tiles = (rows + 63) / 64 * (((long long)K + TN - 1) / TN);
    long long s = (2 * kSms + tiles - 1) / tiles;
    if (s > depth / 256) s = depth / 256;
    if (s > 64) s = 64;
    return {s < 1 ? 1 : (int)s, rows, 0};
}

int gated_simt_backward(bool dw, const GatedSplit& g, int M, int F, int K, const float* x, const float* w, const float* dz, float* out, float* parts, cudaStream_t s) {
    Args a{};
    a.M = dw ? 2 * F : M; a.N = K; a.depth = dw ? M : 2 * F; a.F = F;
    a.A = dz; a.lda = 2LL * F; a.B = dw ? x : w; a.ldb = K;
    a.parts = g.parts; a.plane = g.plane_rows * K; a.out = g.parts > 1 ? parts : out;
    const bool vec = K % 4 == 0 && F % 2 == 0;
    return dw ? launch<DW>(a, vec, s) : launch<DX>(a, vec, s);
}
