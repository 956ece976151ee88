// Layer norm with an optional weight and bias per group of rows, and its backward pass.
//
//   forward    mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r,  y = xh w + b
//   backward   v = dy w;  dx = r (v - mean(v) - xh mean(v xh)) + dres;  dw = sum_rows dy xh;  db = sum_rows dy
//
// w and b belong to a group of consecutive rows (a sequence, for adaptive norms, where w = 1 + scale) or to all of them.
// Both directions are one pass over the data and bound by HBM: every row is read once into registers.  A row is held by
// a team of warps, eight columns per lane: one warp for rows of at most 512 columns (eight teams per CTA), ceil(D / 256)
// warps beyond.  Statistics are fp32: each warp takes the mean of its own columns and their squared deviations from it,
// and the parts are combined with the exact formula M2 = sum M2_k + n_k (mean_k - mean)^2, so that a large mean cancels
// nothing and a row costs one CTA barrier.
// The gradients of w and b are column sums over a group's rows.  A CTA keeps them in fp32 registers over a run of rows of
// one group and writes one partial row; a second, small launch adds the partial rows of a group in a fixed order, so that
// repeats are bit-identical (no atomics).
#include "internal.h"

namespace {

constexpr int kMaxWarps = 32;
constexpr int kMaxD = kMaxWarps * 256;
constexpr int kSms = 148;

template <typename T> __device__ __forceinline__ void ld8(const T* p, float (&v)[8]);
template <> __device__ __forceinline__ void ld8<float>(const float* p, float (&v)[8]) {
    const float4 a = __ldcs(reinterpret_cast<const float4*>(p)), b = __ldcs(reinterpret_cast<const float4*>(p) + 1);
    v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}
template <> __device__ __forceinline__ void ld8<__nv_bfloat16>(const __nv_bfloat16* p, float (&v)[8]) {
    const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) { v[2 * i] = __uint_as_float(w[i] << 16); v[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u); }
}
__device__ __forceinline__ void st8(float* p, const float (&v)[8]) {
    reinterpret_cast<float4*>(p)[0] = make_float4(v[0], v[1], v[2], v[3]);
    reinterpret_cast<float4*>(p)[1] = make_float4(v[4], v[5], v[6], v[7]);
}
__device__ __forceinline__ void st8(__nv_bfloat16* p, const float (&v)[8]) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    *reinterpret_cast<uint4*>(p) = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// The columns of a lane.  Warp k of a team of W owns the 256-column blocks k, W + k, ...  (step i: block i W + k).
// VEC: lane l holds columns 8 l .. 8 l + 7 of a block as 16-byte accesses (D % 8 == 0, row starts 16-byte aligned);
// otherwise columns l, l + 32, ..., l + 224: any D, any row stride, whole-warp runs of consecutive elements.
template <bool VEC> struct Cols {
    int D, W, k, lane;
    __device__ __forceinline__ int at(int i, int e) const { return (i * W + k) * 256 + (VEC ? lane * 8 + e : e * 32 + lane); }
    __device__ __forceinline__ bool in(int i, int e) const { return at(i, VEC ? 0 : e) < D; }
    template <typename E> __device__ __forceinline__ void load(const E* row, int i, float (&v)[8]) const {
        if (VEC) {
            if (in(i, 0)) ld8<E>(row + at(i, 0), v);
            else {
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = 0.f;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = in(i, e) ? to_f(row[at(i, e)]) : 0.f;
        }
    }
    template <typename E> __device__ __forceinline__ void store(E* row, int i, const float (&v)[8]) const {
        if (VEC) {
            if (in(i, 0)) st8(row + at(i, 0), v);
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (in(i, e)) st1(row + at(i, e), v[e]);
        }
    }
};

struct NormArgs {
    long long M;
    int D, groups, rows_per_group, warps;     // warps: warps of a team
    const void* x; long long x_stride;
    const float *weight, *bias; long long mod_stride; float unit;   // unit: 1 where the weight is stored as an offset from one
    float eps;
    void* y; long long y_stride;
    float* stats;                             // [M][2]: mu, r
    long long rows_per_team;                  // forward: consecutive rows of a team
    // backward
    const void* dy; long long dy_stride;
    const float* stats_in;
    const void* dres; long long dres_stride;
    void* dx; long long dx_stride;
    float *dw, *db; long long dmod_stride;    // final gradients
    float* partial;                           // [groups][chunks][2][D]; with one chunk per group the kernel writes dw, db itself
    int chunks;
};

// NV: 256-column blocks per warp; R: rows in flight per team
template <typename TX, typename TY, int NV, bool VEC, int MAXT, int R>
__global__ void __launch_bounds__(MAXT) layer_norm_kernel(const NormArgs a) {
    __shared__ float2 part[2][R][kMaxWarps];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int W = NV > 1 ? 1 : a.warps;                            // several blocks per warp: teams of one warp
    const int teams = W == 1 ? blockDim.x >> 5 : 1;
    const Cols<VEC> c{a.D, W, W == 1 ? 0 : warp, lane};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long first = ((long long)blockIdx.x * teams + (W == 1 ? warp : 0)) * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    const float inv_d = 1.f / (float)a.D;
    const float n_last = (float)(a.D - (W - 1) * 256);             // columns of the team's last warp; the others hold 256
    const float inv_n = W == 1 ? inv_d : (c.k < W - 1 ? 1.f / 256.f : 1.f / n_last);
    float w[NV][8], b[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) { w[i][e] = 1.f; b[i][e] = 0.f; }
    long long group_end = a.weight || a.bias ? first : a.M;        // first row that the registers' w and b do not belong to
    int buf = 0;
    for (long long row = first; row < last; row += R, buf ^= 1) {
        float v[R][NV][8], mu[R], m2[R];
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                if (row + r < last) c.load(x + (row + r) * a.x_stride, i, v[r][i]);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) v[r][i][e] = 0.f;
                }
            }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float s = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) s += v[r][i][e];
            mu[r] = free_warp_sum(s) * inv_n;
            float q = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) { const float d = v[r][i][e] - mu[r]; q += c.in(i, e) ? d * d : 0.f; }
            m2[r] = free_warp_sum(q);                              // squared deviations from this warp's mean
        }
        if (W > 1) {
            if (lane == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) part[buf][r][warp] = make_float2(mu[r], m2[r]);
            }
            __syncthreads();                                       // a buffer is rewritten two barriers after its last read
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float s = 0.f;
                for (int k = 0; k < W - 1; ++k) s += part[buf][r][k].x;
                const float2 pl = part[buf][r][W - 1];
                const float m = (256.f * s + n_last * pl.x) * inv_d;
                float q = 0.f, t = 0.f;
                for (int k = 0; k < W - 1; ++k) { const float2 p = part[buf][r][k]; q += p.y; t += (p.x - m) * (p.x - m); }
                mu[r] = m;
                m2[r] = q + pl.y + 256.f * t + n_last * (pl.x - m) * (pl.x - m);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long rr = row + r;
            if (rr >= last) break;
            const float rstd = rsqrtf(m2[r] * inv_d + a.eps);
            if (rr >= group_end) {                                 // uniform over the team
                const long long g = rr / a.rows_per_group, mo = g * a.mod_stride;
                group_end = (g + 1) * a.rows_per_group;
#pragma unroll
                for (int i = 0; i < NV; ++i)
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (c.in(i, e)) {
                            if (a.weight) w[i][e] = __ldg(a.weight + mo + c.at(i, e)) + a.unit;
                            if (a.bias) b[i][e] = __ldg(a.bias + mo + c.at(i, e));
                        }
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (v[r][i][e] - mu[r]) * rstd * w[i][e] + b[i][e];
                c.store(y + rr * a.y_stride, i, o);
            }
            if (a.stats && c.k == 0 && lane == 0) { a.stats[2 * rr] = mu[r]; a.stats[2 * rr + 1] = rstd; }
        }
    }
}

// One CTA per (group, chunk): a run of the group's rows, walked by the CTA's teams in turn.
template <typename TX, typename TY, int NV, bool VEC, int MAXT, int R>
__global__ void __launch_bounds__(MAXT) layer_norm_bwd_kernel(const NormArgs a) {
    __shared__ float2 part[2][R][kMaxWarps];
    __shared__ float cols[NV > 1 ? MAXT / 32 : 1][NV > 1 ? NV * 512 : 1];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int W = NV > 1 ? 1 : a.warps;
    const int teams = NV > 1 ? blockDim.x >> 5 : 1;                // NV == 1: the CTA is one team
    const Cols<VEC> c{a.D, W, NV > 1 ? 0 : warp, lane};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const TY* dy = reinterpret_cast<const TY*>(a.dy);
    const TX* dres = reinterpret_cast<const TX*>(a.dres);
    TX* dx = reinterpret_cast<TX*>(a.dx);
    const int g = blockIdx.x / a.chunks, ch = blockIdx.x % a.chunks;
    const long long base = (long long)g * a.rows_per_group;
    const long long lo = base + (long long)a.rows_per_group * ch / a.chunks, hi = base + (long long)a.rows_per_group * (ch + 1) / a.chunks;
    const float inv_d = 1.f / (float)a.D;
    float w[NV][8], dw[NV][8], db[NV][8];
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            w[i][e] = 1.f; dw[i][e] = 0.f; db[i][e] = 0.f;
            if (a.weight && c.in(i, e)) w[i][e] = __ldg(a.weight + (long long)g * a.mod_stride + c.at(i, e)) + a.unit;
        }
    int buf = 0;
    for (long long row = lo + (NV > 1 ? warp * R : 0); row < hi; row += (long long)teams * R, buf ^= 1) {
        float xh[R][NV][8], gy[R][NV][8], res[R][NV][8];
        float2 st[R], sums[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long rr = row + r < hi ? row + r : hi - 1;  // past the run: the last row again, not counted or stored
            st[r] = make_float2(__ldg(a.stats_in + 2 * rr), __ldg(a.stats_in + 2 * rr + 1));
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                c.load(x + rr * a.x_stride, i, xh[r][i]);
                c.load(dy + rr * a.dy_stride, i, gy[r][i]);
                if (dres) c.load(dres + rr * a.dres_stride, i, res[r][i]);
                else {
#pragma unroll
                    for (int e = 0; e < 8; ++e) res[r][i][e] = 0.f;
                }
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live = row + r < hi;
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int i = 0; i < NV; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float h = (xh[r][i][e] - st[r].x) * st[r].y, d = gy[r][i][e], v = d * w[i][e];
                    const bool in = c.in(i, e);                    // outside the row d = 0, but h is not
                    xh[r][i][e] = h; gy[r][i][e] = v;
                    if (in) {
                        s1 += v; s2 = fmaf(v, h, s2);
                        if (live) { dw[i][e] = fmaf(d, h, dw[i][e]); db[i][e] += d; }
                    }
                }
            sums[r] = make_float2(free_warp_sum(s1), free_warp_sum(s2));
        }
        if (W > 1) {
            if (lane == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) part[buf][r][warp] = sums[r];
            }
            __syncthreads();                                       // a buffer is rewritten two barriers after its last read
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float s1 = 0.f, s2 = 0.f;
                for (int k = 0; k < W; ++k) { const float2 p = part[buf][r][k]; s1 += p.x; s2 += p.y; }
                sums[r] = make_float2(s1, s2);
            }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row + r >= hi) break;
            const float m1 = sums[r].x * inv_d, m2 = sums[r].y * inv_d;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                float o[8];
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = fmaf(st[r].y, gy[r][i][e] - m1 - xh[r][i][e] * m2, res[r][i][e]);
                c.store(dx + (row + r) * a.dx_stride, i, o);
            }
        }
    }
    if (!a.dw && !a.db) return;
    float *ow = a.dw ? a.dw + (long long)g * a.dmod_stride : nullptr, *ob = a.db ? a.db + (long long)g * a.dmod_stride : nullptr;
    if (a.chunks > 1) {
        ow = a.partial + (long long)blockIdx.x * 2 * a.D;
        ob = ow + a.D;
    }
    if (NV > 1) {                                                  // the teams' sums, added in the order of the warps
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (c.in(i, e)) { cols[warp][c.at(i, e)] = dw[i][e]; cols[warp][NV * 256 + c.at(i, e)] = db[i][e]; }
        __syncthreads();
        for (int j = threadIdx.x; j < a.D; j += blockDim.x) {
            float s = 0.f, t = 0.f;
            for (int k = 0; k < teams; ++k) { s += cols[k][j]; t += cols[k][NV * 256 + j]; }
            if (ow) ow[j] = s;
            if (ob) ob[j] = t;
        }
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c.in(0, e)) {
                if (ow) ow[c.at(0, e)] = dw[0][e];
                if (ob) ob[c.at(0, e)] = db[0][e];
            }
    }
}

// dw, db of a group = the sum of its chunks' partial rows: 32 columns x 16 slices of the chunks per CTA, slices joined in order.
__global__ void __launch_bounds__(512) layer_norm_reduce_kernel(const NormArgs a) {
    __shared__ float sh[16][33];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int blocks = (2 * a.D + 31) / 32, g = blockIdx.x / blocks, j = (blockIdx.x % blocks) * 32 + tx;   // j: column of [2][D]
    const float* p = a.partial + (long long)g * a.chunks * 2 * a.D;
    float s = 0.f;
    if (j < 2 * a.D)
        for (int k = ty; k < a.chunks; k += 16) s += p[(long long)k * 2 * a.D + j];
    sh[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && j < 2 * a.D) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += sh[k][tx];
        float* out = j < a.D ? a.dw : a.db;
        if (out) out[(long long)g * a.dmod_stride + (j < a.D ? j : j - a.D)] = t;
    }
}

// Shape of a launch for width D: blocks per warp, warps of a team, threads of a CTA.
// Rows of at most 512 columns fit one warp (two blocks): no barrier, eight rows side by side.
struct Shape { int nv, warps, threads; };
Shape shape_of(int D) {
    if (D <= 512) return {2, 1, 256};
    const int w = (D + 255) / 256;
    return {1, w, w * 32};
}

// Chunks of a group in the backward pass: enough CTAs to fill the GPU, at least eight rows per team.
int chunks_of(int groups, int rows_per_group, int D) {
    const Shape s = shape_of(D);
    const int per_cta = 8 * (s.warps == 1 ? s.threads / 32 : 1);
    const long long want = ((long long)kSms * (s.threads <= 256 ? 1024 / s.threads : 1) + groups - 1) / groups;
    const long long most = rows_per_group / per_cta;
    const long long c = want < most ? want : most;
    return c < 1 ? 1 : (int)c;
}

template <typename TX, typename TY, bool VEC>
int launch_fwd(NormArgs a, cudaStream_t s) {
    const Shape sh = shape_of(a.D);
    const int teams = sh.warps == 1 ? sh.threads / 32 : 1;
    a.warps = sh.warps;
    // a whole number of waves of the CTAs that the GPU holds at once; few rows: as many teams as there are rows
    const long long resident = (long long)kSms * (2048 / sh.threads < 1 ? 1 : 2048 / sh.threads) * teams;
    a.rows_per_team = (a.M + resident - 1) / resident;
    const unsigned grid = (unsigned)((a.M + a.rows_per_team * teams - 1) / (a.rows_per_team * teams));
    const bool ov = free_overlap_for_rows(a.M);
    if (sh.nv == 2) return free_launch(ov, layer_norm_kernel<TX, TY, 2, VEC, 256, 1>, dim3(grid), dim3(sh.threads), 0, s, a);
    if (sh.threads <= 256) return free_launch(ov, layer_norm_kernel<TX, TY, 1, VEC, 256, 2>, dim3(grid), dim3(sh.threads), 0, s, a);
    return free_launch(ov, layer_norm_kernel<TX, TY, 1, VEC, 1024, 1>, dim3(grid), dim3(sh.threads), 0, s, a);
}

template <typename TX, typename TY, bool VEC>
int launch_bwd(NormArgs a, cudaStream_t s) {
    const Shape sh = shape_of(a.D);
    a.warps = sh.warps;
    const dim3 grid((unsigned)a.groups * (unsigned)a.chunks), block(sh.threads);
    const bool ov = free_overlap_for_rows(a.M);
    int r;
    if (sh.nv == 2) r = free_launch(ov, layer_norm_bwd_kernel<TX, TY, 2, VEC, 256, 1>, grid, block, 0, s, a);
    else if (sh.threads <= 256) r = free_launch(ov, layer_norm_bwd_kernel<TX, TY, 1, VEC, 256, 2>, grid, block, 0, s, a);
    else r = free_launch(ov, layer_norm_bwd_kernel<TX, TY, 1, VEC, 1024, 1>, grid, block, 0, s, a);
    if (r != FREE_OK || a.chunks == 1 || (!a.dw && !a.db)) return r;
    return free_launch(free_launch_overlap_enabled(), layer_norm_reduce_kernel, dim3((unsigned)a.groups * ((2u * a.D + 31) / 32)), dim3(512), 0, s, a);
}

bool row_vec(int dtype, const void* p, long long stride) {
    return !p || (stride % (dtype == FREE_BF16 ? 8 : 4) == 0);     // base pointers are 16-byte aligned (checked)
}

bool known(int dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }

}  // namespace

extern "C" int free_op_layer_norm(int x_dtype, int y_dtype, int n_groups, int rows_per_group, int D,
                                  const void* x, int64_t x_stride, const float* weight, const float* bias, int64_t mod_stride,
                                  int unit_offset, float eps, void* y, int64_t y_stride, float* stats, void* stream) {
    if (!known(x_dtype) || !known(y_dtype) || !(eps >= 0.f)) return FREE_ERR_ARG;
    if (n_groups < 0 || rows_per_group < 0 || D < 1) return FREE_ERR_SHAPE;
    const long long M = (long long)n_groups * rows_per_group;
    if (M == 0) return FREE_OK;
    if (!x || !y) return FREE_ERR_ARG;
    if (x_stride < D || y_stride < D || ((weight || bias) && n_groups > 1 && mod_stride < 0)) return FREE_ERR_SHAPE;
    if (!free_aligned16(x) || !free_aligned16(y) || (reinterpret_cast<uintptr_t>(weight) & 3u) || (reinterpret_cast<uintptr_t>(bias) & 3u) ||
        (reinterpret_cast<uintptr_t>(stats) & 3u)) return FREE_ERR_ALIGN;
    if (D > kMaxD) return FREE_ERR_UNSUPPORTED;
    NormArgs a{};
    a.M = M; a.D = D; a.groups = n_groups; a.rows_per_group = rows_per_group;
    a.x = x; a.x_stride = x_stride; a.weight = weight; a.bias = bias; a.mod_stride = mod_stride; a.unit = unit_offset ? 1.f : 0.f;
    a.eps = eps; a.y = y; a.y_stride = y_stride; a.stats = stats;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool vec = D % 8 == 0 && row_vec(x_dtype, x, x_stride) && row_vec(y_dtype, y, y_stride);
    const int which = (x_dtype == FREE_BF16 ? 4 : 0) + (y_dtype == FREE_BF16 ? 2 : 0) + (vec ? 1 : 0);
    using bf = __nv_bfloat16;
    switch (which) {
        case 0: return launch_fwd<float, float, false>(a, s);
        case 1: return launch_fwd<float, float, true>(a, s);
        case 2: return launch_fwd<float, bf, false>(a, s);
        case 3: return launch_fwd<float, bf, true>(a, s);
        case 4: return launch_fwd<bf, float, false>(a, s);
        case 5: return launch_fwd<bf, float, true>(a, s);
        case 6: return launch_fwd<bf, bf, false>(a, s);
        default: return launch_fwd<bf, bf, true>(a, s);
    }
}

extern "C" size_t free_op_layer_norm_bwd_workspace_bytes(int n_groups, int rows_per_group, int D) {
    if (n_groups < 1 || rows_per_group < 1 || D < 1 || D > kMaxD) return 0;
    const int c = chunks_of(n_groups, rows_per_group, D);
    return c > 1 ? (size_t)n_groups * c * 2 * D * sizeof(float) : 0;
}

extern "C" int free_op_layer_norm_bwd(int x_dtype, int y_dtype, int n_groups, int rows_per_group, int D,
                                      const void* x, int64_t x_stride, const void* dy, int64_t dy_stride, const float* stats,
                                      const float* weight, int64_t mod_stride, int unit_offset,
                                      const void* dres, int64_t dres_stride, void* dx, int64_t dx_stride,
                                      float* dweight, float* dbias, int64_t dmod_stride, void* ws, size_t ws_bytes, void* stream) {
    if (!known(x_dtype) || !known(y_dtype)) return FREE_ERR_ARG;
    if (n_groups < 0 || rows_per_group < 0 || D < 1) return FREE_ERR_SHAPE;
    if (n_groups == 0) return FREE_OK;
    const long long M = (long long)n_groups * rows_per_group;
    const bool grads = dweight || dbias;
    if (M > 0 && (!x || !dy || !stats || !dx)) return FREE_ERR_ARG;
    if (M > 0 && (x_stride < D || dy_stride < D || dx_stride < D || (dres && dres_stride < D))) return FREE_ERR_SHAPE;
    if ((weight && n_groups > 1 && mod_stride < 0) || (grads && n_groups > 1 && dmod_stride < D)) return FREE_ERR_SHAPE;
    if (!free_aligned16(x) || !free_aligned16(dy) || !free_aligned16(dres) || !free_aligned16(dx) || !free_aligned16(ws) ||
        (reinterpret_cast<uintptr_t>(stats) & 3u) || (reinterpret_cast<uintptr_t>(weight) & 3u) ||
        (reinterpret_cast<uintptr_t>(dweight) & 3u) || (reinterpret_cast<uintptr_t>(dbias) & 3u)) return FREE_ERR_ALIGN;
    if (D > kMaxD) return FREE_ERR_UNSUPPORTED;
    if (M == 0 && !grads) return FREE_OK;
    const int chunks = rows_per_group ? chunks_of(n_groups, rows_per_group, D) : 1;
    if ((long long)n_groups * chunks > 0x7fffffffLL || (long long)n_groups * ((2LL * D + 31) / 32) > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    if (grads && chunks > 1 && (!ws || ws_bytes < free_op_layer_norm_bwd_workspace_bytes(n_groups, rows_per_group, D))) return FREE_ERR_WORKSPACE;
    NormArgs a{};
    a.M = M; a.D = D; a.groups = n_groups; a.rows_per_group = rows_per_group;
    a.x = x; a.x_stride = x_stride; a.weight = weight; a.mod_stride = mod_stride; a.unit = unit_offset ? 1.f : 0.f;
    a.dy = dy; a.dy_stride = dy_stride; a.stats_in = stats; a.dres = dres; a.dres_stride = dres_stride; a.dx = dx; a.dx_stride = dx_stride;
    a.dw = dweight; a.db = dbias; a.dmod_stride = dmod_stride; a.partial = (float*)ws; a.chunks = chunks;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool vec = D % 8 == 0 && row_vec(x_dtype, x, x_stride) && row_vec(y_dtype, dy, dy_stride) && row_vec(x_dtype, dres, dres_stride) &&
                     row_vec(x_dtype, dx, dx_stride);
    const int which = (x_dtype == FREE_BF16 ? 4 : 0) + (y_dtype == FREE_BF16 ? 2 : 0) + (vec ? 1 : 0);
    using bf = __nv_bfloat16;
    switch (which) {
        case 0: return launch_bwd<float, float, false>(a, s);
        case 1: return launch_bwd<float, float, true>(a, s);
        case 2: return launch_bwd<float, bf, false>(a, s);
        case 3: return launch_bwd<float, bf, true>(a, s);
        case 4: return launch_bwd<bf, float, false>(a, s);
        case 5: return launch_bwd<bf, float, true>(a, s);
        case 6: return launch_bwd<bf, bf, false>(a, s);
        default: return launch_bwd<bf, bf, true>(a, s);
    }
}
