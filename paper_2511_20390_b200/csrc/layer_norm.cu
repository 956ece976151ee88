// Layer norm with an optional weight and bias per group of rows, and its backward pass.
//
//   forward    mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r,  y = xh w + b
//   backward   v = dy w;  dx = r (v - mean(v) - xh mean(v xh)) + dres;  dw = sum_rows dy xh;  db = sum_rows dy
//
// w and b belong to a group of consecutive rows (a sequence, for adaptive norms, where w = 1 + scale) or to all of them.
// Both directions are one pass over the data and bound by HBM: every row is read once.  Statistics are fp32: each warp takes
// the mean of its own columns and their squared deviations from it, and the parts are combined with the exact formula
// M2 = sum M2_k + n_k (mean_k - mean)^2, so that a large mean cancels nothing.
// Forward: a warp holds a row in registers (up to 2048 columns; several warps beyond), so a row costs ten exchanges and no
// barrier; the weight and bias of a group come from the L1.  24 x 1024 rows of 1152, fp32 to bf16, weight and bias per sequence:
// 29.5 us, 5.8 TB/s (a CTA per row with a barrier each: 41 us); 6144 rows of 4608: 33 us.
// Backward: the column sums need registers too, so a row is spread over ceil(D / 256) warps, eight columns per lane, with one
// barrier; rows are copied to shared memory one ahead of their use, every thread its own columns, so that the bytes in flight do
// not cost registers.  The same rows with the residual path's gradient added: 65 us, 6.1 TB/s, and 5 us for the sums.
// The gradients of w and b are column sums over a group's rows.  A CTA keeps them in fp32 registers over a run of rows of
// one group and writes one partial row; a second, small launch adds the partial rows of a group in a fixed order, so that
// repeats are bit-identical (no atomics).
#include "internal.h"

namespace {

constexpr int kMaxWarps = 32;
constexpr int kMaxD = kMaxWarps * 256;
constexpr int kSms = 148;

// Eight columns as they come from memory (bf16 stays packed until it is used).
template <typename T, bool VEC> struct Raw {
    uint32_t r[VEC ? 2 * sizeof(T) : 8];
    __device__ __forceinline__ float operator[](int i) const {
        if (!VEC || sizeof(T) == 4) return __uint_as_float(r[i]);
        return __uint_as_float(i % 2 ? r[i / 2] & 0xffff0000u : r[i / 2] << 16);
    }
};
// four columns, global to shared memory
template <typename T> __device__ __forceinline__ void copy4_async(uint32_t smem, const T* g) {
    if (sizeof(T) == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(g) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem), "l"(g) : "memory");
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void st4(float* p, const float* v) { *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]); }
__device__ __forceinline__ void st4(__nv_bfloat16* p, const float* v) {
    const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
    *reinterpret_cast<uint2*>(p) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void st1(float* p, float v) { *p = v; }
__device__ __forceinline__ void st1(__nv_bfloat16* p, float v) { *p = __float2bfloat16(v); }

// The columns of a lane: warp k of a team owns the 256-column blocks k NV .. k NV + NV - 1.
// VEC: lane l holds columns 4 l .. 4 l + 3 of each half of a block, so that the accesses of a warp are whole runs of 512
// (fp32) or 256 (bf16) bytes; D % 4 == 0, rows aligned to four elements.  (Eight consecutive columns per lane, two 16-byte
// accesses 32 bytes apart in fp32, make two half-used sectors of every sector: measured 20 to 40% slower.)
// Otherwise columns l, l + 32, ..., l + 224: any D, any row stride.
template <bool VEC> struct Cols {
    int D, k, lane;
    __device__ __forceinline__ int at(int i, int e) const {
        return (k + i) * 256 + (VEC ? (e / 4) * 128 + lane * 4 + e % 4 : e * 32 + lane);
    }
    __device__ __forceinline__ bool in(int i, int e) const { return at(i, VEC ? e / 4 * 4 : e) < D; }
    // straight into registers
    template <typename E> __device__ __forceinline__ void load(const E* row, int i, Raw<E, VEC>& v) const {
        if (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                constexpr int N = (int)sizeof(E);                  // 32-bit words of four columns
                const E* p = row + at(i, 4 * h);
                const bool ok = in(i, 4 * h);
                if (N == 4) {
                    const uint4 u = ok ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
                    v.r[h * N] = u.x; v.r[h * N + 1] = u.y; v.r[h * N + N - 2] = u.z; v.r[h * N + N - 1] = u.w;
                } else {
                    const uint2 u = ok ? __ldcs(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
                    v.r[h * N] = u.x; v.r[h * N + 1] = u.y;
                }
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v.r[e] = in(i, e) ? __float_as_uint(to_f(row[at(i, e)])) : 0u;
        }
    }
    // a table's row
    __device__ __forceinline__ void table(const float* row, int i, float add, float (&v)[8]) const {
        if (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const float4 f = in(i, 4 * h) ? __ldg(reinterpret_cast<const float4*>(row + at(i, 4 * h))) : make_float4(0.f, 0.f, 0.f, 0.f);
                v[4 * h] = f.x + add; v[4 * h + 1] = f.y + add; v[4 * h + 2] = f.z + add; v[4 * h + 3] = f.w + add;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = in(i, e) ? __ldg(row + at(i, e)) + add : 0.f;
        }
    }
    // vector form, ahead of time: into shared memory, [half][thread] of a region of 8 elements per thread, and back from there
    template <typename E> __device__ __forceinline__ uint32_t place(uint32_t region, int half) const {
        return region + (half * blockDim.x + threadIdx.x) * 4 * (uint32_t)sizeof(E);
    }
    template <typename E> __device__ __forceinline__ void send(const E* row, int i, uint32_t region) const {
#pragma unroll
        for (int h = 0; h < 2; ++h)
            if (in(i, 4 * h)) copy4_async<E>(place<E>(region, h), row + at(i, 4 * h));
    }
    template <typename E> __device__ __forceinline__ void take(uint32_t region, int i, Raw<E, VEC>& v) const {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            constexpr int N = (int)sizeof(E);                      // 32-bit words of four columns
            uint32_t u[4];
            if (N == 4) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(place<E>(region, h)) : "memory");
            else asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(u[0]), "=r"(u[1]) : "r"(place<E>(region, h)) : "memory");
#pragma unroll
            for (int q = 0; q < N; ++q) v.r[h * N + q] = in(i, 4 * h) ? u[q] : 0u;      // outside: nothing was copied there
        }
    }
    template <typename E> __device__ __forceinline__ void store(E* row, int i, const float (&v)[8]) const {
        if (VEC) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                if (in(i, 4 * h)) st4(row + at(i, 4 * h), v + 4 * h);
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

// Sums over a team's warps (at most MAXW), every thread for itself.
template <int MAXW> __device__ __forceinline__ float2 team_sum(const float2* part, int W) {
    float2 s = make_float2(0.f, 0.f);
    if (MAXW <= 8) {
#pragma unroll
        for (int k = 0; k < MAXW; ++k)
            if (k < W) { const float2 p = part[k]; s.x += p.x; s.y += p.y; }
    } else {
#pragma unroll 8
        for (int k = 0; k < W; ++k) { const float2 p = part[k]; s.x += p.x; s.y += p.y; }
    }
    return s;
}

// Forward: a warp of a team owns NH blocks of 128 columns, four per lane and block (Cols, with half the width).
// FULL: the row is exactly the team's blocks, nothing is checked.
template <bool VEC, int NH, bool FULL> struct Cols4 {
    int D, k, lane;
    __device__ __forceinline__ int at(int h, int e) const { return (k * NH + h) * 128 + (VEC ? lane * 4 + e : e * 32 + lane); }
    __device__ __forceinline__ bool in(int h, int e) const { return FULL || at(h, VEC ? 0 : e) < D; }
    template <typename E> __device__ __forceinline__ void load(const E* row, int h, uint32_t (&v)[VEC ? sizeof(E) : 4]) const {
        if (VEC) {
            const E* p = row + at(h, 0);
            if (sizeof(E) == 4) {
                const uint4 u = in(h, 0) ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
                v[0] = u.x; v[1] = u.y; v[sizeof(E) - 2] = u.z; v[sizeof(E) - 1] = u.w;
            } else {
                const uint2 u = in(h, 0) ? __ldcs(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
                v[0] = u.x; v[1] = u.y;
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = in(h, e) ? __float_as_uint(to_f(row[at(h, e)])) : 0u;
        }
    }
    template <typename E> static __device__ __forceinline__ float value(const uint32_t (&v)[VEC ? sizeof(E) : 4], int e) {
        if (!VEC || sizeof(E) == 4) return __uint_as_float(v[e]);
        return __uint_as_float(e % 2 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
    }
    // a table's row
    __device__ __forceinline__ void table(const float* row, int h, float add, float (&v)[4]) const {
        if (VEC) {
            const float4 f = in(h, 0) ? __ldg(reinterpret_cast<const float4*>(row + at(h, 0))) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[0] = f.x + add; v[1] = f.y + add; v[2] = f.z + add; v[3] = f.w + add;
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = in(h, e) ? __ldg(row + at(h, e)) + add : 0.f;
        }
    }
    template <typename E> __device__ __forceinline__ void store(E* row, int h, const float (&v)[4]) const {
        if (VEC) {
            if (in(h, 0)) st4(row + at(h, 0), v);
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (in(h, e)) st1(row + at(h, e), v[e]);
        }
    }
};

// A team is one warp where NH blocks hold the row (MAXW == 1), else the CTA.  The next row's loads are in flight while this one is
// reduced; the weight and bias come from the L1 (in registers they cost more rows in flight than they save: 31.2 against 30.7 us
// for 24 x 1024 rows of 1152, 4.8 against 3.5 for 2048 rows).
template <typename TX, typename TY, int NH, bool VEC, bool FULL, int MAXT, int MINB, int MAXW>
__global__ void __launch_bounds__(MAXT, MINB) layer_norm_kernel(const NormArgs a) {
    __shared__ float2 part[2][MAXW];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int W = MAXW > 1 ? a.warps : 1;
    using C = Cols4<VEC, NH, FULL>;
    const C c{a.D, W > 1 ? warp : 0, lane};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long team = MAXW > 1 ? blockIdx.x : (long long)blockIdx.x * (blockDim.x >> 5) + warp;
    const long long first = team * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    constexpr float full = NH * 128.f;                             // columns of all of a team's warps but the last
    const float inv_d = 1.f / (float)a.D, n_last = (float)a.D - (float)(W - 1) * full;
    const float inv_n = c.k < W - 1 ? 1.f / full : 1.f / n_last;
    uint32_t nx[NH][VEC ? sizeof(TX) : 4];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int h = 0; h < NH; ++h) c.template load<TX>(x + row * a.x_stride, h, nx[h]);
    };
    const bool tables = a.weight || a.bias;
    // the first row that the weight and bias at hand do not belong to, where they lie, and how far away the next group's are
    // (one division per warp: the code stays short, which counts more than anything else for small calls)
    const long long g0 = !tables ? 0 : first <= 0xffffffffLL ? (long long)((uint32_t)first / (uint32_t)a.rows_per_group) : first / a.rows_per_group;
    long long group_end = tables ? g0 * a.rows_per_group : a.M, mo = g0 * a.mod_stride, step = 0;
    if (first < last) fetch(first);
    int it = 0;
    for (long long row = first; row < last; ++row, ++it) {
        if (row >= group_end) {                                    // uniform over the team
            mo += step;
            step = a.mod_stride;
            group_end += a.rows_per_group;
        }
        float v[NH][4];
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) v[h][e] = C::template value<TX>(nx[h], e);
        if (row + 1 < last) fetch(row + 1);
        float s = 0.f;
#pragma unroll
        for (int h = 0; h < NH; ++h) s += (v[h][0] + v[h][1]) + (v[h][2] + v[h][3]);
        float mu = free_warp_sum(s) * inv_n, q = 0.f;
#pragma unroll
        for (int h = 0; h < NH; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) { const float d = v[h][e] - mu; q += c.in(h, e) ? d * d : 0.f; }
        float m2 = free_warp_sum(q);                               // squared deviations from this warp's mean
        if (MAXW > 1) {
            float2* now = part[it & 1];                            // a buffer is rewritten two barriers after its last read
            if (lane == 0) now[warp] = make_float2(mu, m2);
            __syncthreads();
            const float2 pl = now[W - 1], t = team_sum<MAXW>(now, W - 1);
            mu = (full * t.x + n_last * pl.x) * inv_d;
            float d2 = 0.f;
#pragma unroll
            for (int k = 0; k < MAXW; ++k)
                if (k < W - 1) { const float d = now[k].x - mu; d2 = fmaf(d, d, d2); }
            m2 = t.y + pl.y + full * d2 + n_last * (pl.x - mu) * (pl.x - mu);
        }
        const float rstd = rsqrtf(m2 * inv_d + a.eps);
#pragma unroll
        for (int h = 0; h < NH; ++h) {
            float o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] = (v[h][e] - mu) * rstd;
            float t[4];
            if (a.weight) {
                c.table(a.weight + mo, h, a.unit, t);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] *= t[e];
            }
            if (a.bias) {
                c.table(a.bias + mo, h, 0.f, t);
#pragma unroll
                for (int e = 0; e < 4; ++e) o[e] += t[e];
            }
            c.store(y + row * a.y_stride, h, o);
        }
        if (a.stats && c.k == 0 && lane == 0) { a.stats[2 * row] = mu; a.stats[2 * row + 1] = rstd; }
    }
}

// One CTA, a team of ceil(D / 256) warps, per (group, chunk): a run of the group's rows, R of them per barrier.
// DEPTH: groups of R rows in flight (vector form).  T: threads per SM that the register budget is set for.
template <typename TX, typename TY, bool VEC, int MAXT, int T, int R, int DEPTH>
__global__ void __launch_bounds__(MAXT, T / MAXT) layer_norm_bwd_kernel(const NormArgs a) {
    __shared__ float2 part[2][R][MAXT / 32];
    extern __shared__ uint4 ring[];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, W = a.warps;
    const Cols<VEC> c{a.D, warp, lane};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const TY* dy = reinterpret_cast<const TY*>(a.dy);
    const TX* dres = reinterpret_cast<const TX*>(a.dres);
    TX* dx = reinterpret_cast<TX*>(a.dx);
    const int g = blockIdx.x / a.chunks, ch = blockIdx.x % a.chunks;
    const long long base = (long long)g * a.rows_per_group;
    const long long lo = base + (long long)a.rows_per_group * ch / a.chunks, hi = base + (long long)a.rows_per_group * (ch + 1) / a.chunks;
    const float inv_d = 1.f / (float)a.D;
    const uint32_t ring0 = (uint32_t)__cvta_generic_to_shared(ring);
    const uint32_t bx = blockDim.x * 8 * (uint32_t)sizeof(TX), by = blockDim.x * 8 * (uint32_t)sizeof(TY);   // regions of x and dres, of dy
    auto unit = [&](int it, int r) { return ring0 + (uint32_t)(it % DEPTH * R + r) * (2 * bx + by); };
    auto fetch = [&](int it) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const long long row = lo + (long long)it * R + r;
            if (row < hi) {
                const uint32_t u = unit(it, r);
                c.send(x + row * a.x_stride, 0, u);
                if (dres) c.send(dres + row * a.dres_stride, 0, u + bx);
                c.send(dy + row * a.dy_stride, 0, u + 2 * bx);
            }
        }
        copy_commit();
    };
    auto stats_of = [&](long long row) {
        return row < hi ? make_float2(__ldg(a.stats_in + 2 * row), __ldg(a.stats_in + 2 * row + 1)) : make_float2(0.f, 0.f);
    };
    if (VEC) {
#pragma unroll
        for (int k = 0; k < DEPTH - 1; ++k) fetch(k);
    }
    float w[8], dw[8], db[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) { w[e] = 1.f; dw[e] = 0.f; db[e] = 0.f; }
    if (a.weight) c.table(a.weight + (long long)g * a.mod_stride, 0, a.unit, w);
    float2 next[R];                                                // statistics of the rows to come
#pragma unroll
    for (int r = 0; r < R; ++r) next[r] = stats_of(lo + r);
    int it = 0;
    for (long long row = lo; row < hi; row += R, ++it) {
        Raw<TX, VEC> res[R];
        float2 st[R], sum[R];
        float xh[R][8], v[R][8];
        if (VEC) {
            fetch(it + DEPTH - 1);                                 // into the slot that the previous rows left
            copy_wait<DEPTH - 1>();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            Raw<TX, VEC> rx;
            Raw<TY, VEC> ry;
            const bool live = row + r < hi;                        // past the run: nothing is counted or stored
            if (VEC) {
                c.take(unit(it, r), 0, rx);
                c.take(unit(it, r) + 2 * bx, 0, ry);
            } else if (live) {
                c.load(x + (row + r) * a.x_stride, 0, rx);
                c.load(dy + (row + r) * a.dy_stride, 0, ry);
                if (dres) c.load(dres + (row + r) * a.dres_stride, 0, res[r]);
            }
            st[r] = next[r];
            next[r] = stats_of(row + R + r);
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const bool in = live && c.in(0, e);
                const float d = in ? ry[e] : 0.f;
                xh[r][e] = in ? (rx[e] - st[r].x) * st[r].y : 0.f;
                v[r][e] = d * w[e];
                s1 += v[r][e]; s2 = fmaf(v[r][e], xh[r][e], s2);
                dw[e] = fmaf(d, xh[r][e], dw[e]); db[e] += d;
            }
            sum[r] = make_float2(free_warp_sum(s1), free_warp_sum(s2));
        }
        if (W > 1) {
            float2 (*now)[MAXT / 32] = part[it & 1];               // a buffer is rewritten two barriers after its last read
            if (lane == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) now[r][warp] = sum[r];
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] = team_sum<MAXT / 32>(now[r], W);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row + r >= hi) break;
            const float m1 = sum[r].x * inv_d, m2 = sum[r].y * inv_d;
            float o[8];
            if (VEC && dres) c.take(unit(it, r) + bx, 0, res[r]);
#pragma unroll
            for (int e = 0; e < 8; ++e) o[e] = fmaf(st[r].y, v[r][e] - m1 - xh[r][e] * m2, dres ? res[r][e] : 0.f);
            c.store(dx + (row + r) * a.dx_stride, 0, o);
        }
    }
    if (VEC) copy_wait<0>();                                       // nothing is in flight when the CTA ends
    if (!a.dw && !a.db) return;
    float *ow = a.dw ? a.dw + (long long)g * a.dmod_stride : nullptr, *ob = a.db ? a.db + (long long)g * a.dmod_stride : nullptr;
    if (a.chunks > 1) {
        ow = a.partial + (long long)blockIdx.x * 2 * a.D;
        ob = ow + a.D;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (c.in(0, e)) {
            if (ow) ow[c.at(0, e)] = dw[e];
            if (ob) ob[c.at(0, e)] = db[e];
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
    if (j < 2 * a.D) {
#pragma unroll 8
        for (int k = ty; k < a.chunks; k += 16) s += p[(long long)k * 2 * a.D + j];
    }
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

// Threads per SM of the backward kernel.  The scalar form has no copies ahead of their use: two rows per barrier, in twice the registers.
constexpr int kBwdT = 1024, kBwdScalarT = 512;

int bwd_threads(int D) { return (D + 255) / 256 * 32; }

// Chunks of a group in the backward pass: one wave of CTAs, at least eight rows each.  (A function of the sizes alone: the
// workspace depends on it.)
int chunks_of(int groups, int rows_per_group, int D) {
    const int t = bwd_threads(D);
    const int per_sm = t > 256 ? 1 : (D % 4 ? kBwdScalarT : kBwdT) / t;
    const long long want = ((long long)kSms * per_sm + groups - 1) / groups;
    const long long most = rows_per_group / 8;
    const long long c = want < most ? want : most;
    return c < 1 ? 1 : (int)c;
}

template <typename TX, typename TY, int NH, bool VEC, bool FULL, int MAXT, int MINB, int MAXW>
int start_fwd(NormArgs a, int warps, cudaStream_t s) {
    const int threads = MAXW > 1 ? warps * 32 : MAXT, teams = MAXW > 1 ? 1 : MAXT / 32;
    a.warps = warps;
    // one wave of the CTAs that the GPU holds at once; few rows: as many teams as there are rows
    const long long resident = (long long)kSms * (MINB * MAXT / threads) * teams;
    a.rows_per_team = (a.M + resident - 1) / resident;
    const long long grid = (a.M + a.rows_per_team * teams - 1) / (a.rows_per_team * teams);
    return free_launch(free_overlap_for_rows(a.M), layer_norm_kernel<TX, TY, NH, VEC, FULL, MAXT, MINB, MAXW>, dim3((unsigned)grid), dim3(threads),
                       0, s, a);
}

// As many blocks of 128 columns per warp as the row needs (registers decide how many rows an SM holds); several warps beyond 2048
// columns.  Widths that the blocks fill exactly have kernels without checks (24 x 1024 rows of 1152: 29.5 us, with checks 34).
template <typename TX, typename TY, bool VEC>
int launch_fwd(const NormArgs& a, cudaStream_t s) {
    if constexpr (VEC) {
        const int n = a.D % 128 == 0 ? a.D / 128 : 0;
        switch (n) {
            case 2: return start_fwd<TX, TY, 2, true, true, 128, 8, 1>(a, 1, s);
            case 3: return start_fwd<TX, TY, 3, true, true, 128, 7, 1>(a, 1, s);
            case 4: return start_fwd<TX, TY, 4, true, true, 128, 6, 1>(a, 1, s);
            case 5: return start_fwd<TX, TY, 5, true, true, 128, 5, 1>(a, 1, s);
            case 6: return start_fwd<TX, TY, 6, true, true, 128, 4, 1>(a, 1, s);
            case 8: return start_fwd<TX, TY, 8, true, true, 128, 4, 1>(a, 1, s);
            case 9: return start_fwd<TX, TY, 9, true, true, 128, 3, 1>(a, 1, s);
            case 10: return start_fwd<TX, TY, 10, true, true, 128, 3, 1>(a, 1, s);
            case 12: return start_fwd<TX, TY, 12, true, true, 128, 3, 1>(a, 1, s);
            case 16: return start_fwd<TX, TY, 16, true, true, 128, 2, 1>(a, 1, s);
            default: break;
        }
        if (n > 16 && n % 9 == 0) return start_fwd<TX, TY, 9, true, true, 256, 2, 8>(a, n / 9, s);
        if (n > 16 && n % 8 == 0) return start_fwd<TX, TY, 8, true, true, 256, 2, 8>(a, n / 8, s);
    }
    if (a.D <= 512) return start_fwd<TX, TY, 4, VEC, false, 128, 6, 1>(a, 1, s);
    if (a.D <= 768) return start_fwd<TX, TY, 6, VEC, false, 128, 5, 1>(a, 1, s);
    if (a.D <= 1280) return start_fwd<TX, TY, 10, VEC, false, 128, 4, 1>(a, 1, s);
    if (a.D <= 2048) return start_fwd<TX, TY, 16, VEC, false, 128, 2, 1>(a, 1, s);
    constexpr int per = 1280;
    return start_fwd<TX, TY, 10, VEC, false, 256, 2, (kMaxD + per - 1) / per>(a, (a.D + per - 1) / per, s);
}

template <typename TX, typename TY, bool VEC, int MAXT, int T, int R>
int start_bwd(const NormArgs& a, int threads, cudaStream_t s) {
    constexpr int DEPTH = 2;
    auto kernel = layer_norm_bwd_kernel<TX, TY, VEC, MAXT, T, R, DEPTH>;
    const size_t smem = VEC ? (size_t)threads * DEPTH * R * 8 * (2 * sizeof(TX) + sizeof(TY)) : 0;
    if (smem > 47 * 1024) FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem));
    return free_launch(free_overlap_for_rows(a.M), kernel, dim3((unsigned)a.groups * (unsigned)a.chunks), dim3(threads), smem, s, a);
}

template <typename TX, typename TY, bool VEC>
int launch_bwd(NormArgs a, cudaStream_t s) {
    const int threads = bwd_threads(a.D);
    a.warps = threads / 32;
    // wide rows leave an SM one CTA: two rows per barrier where shared memory holds them
    const int r = threads <= 256 ? start_bwd<TX, TY, VEC, 256, VEC ? kBwdT : kBwdScalarT, VEC ? 1 : 2>(a, threads, s)
                : threads <= 576 ? start_bwd<TX, TY, VEC, 576, 576, 2>(a, threads, s) : start_bwd<TX, TY, VEC, 1024, 1024, 1>(a, threads, s);
    if (r != FREE_OK || a.chunks == 1 || (!a.dw && !a.db)) return r;
    return free_launch(free_launch_overlap_enabled(), layer_norm_reduce_kernel, dim3((unsigned)a.groups * ((2u * a.D + 31) / 32)), dim3(512), 0, s, a);
}

bool tables_vec(const float* w, const float* b, int groups, long long stride) {
    return ((reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(b)) & 15u) == 0 && (groups == 1 || stride % 4 == 0);
}
bool row_vec(const void* p, long long stride) { return !p || stride % 4 == 0; }    // base pointers are 16-byte aligned (checked)

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
    const bool vec = D % 4 == 0 && row_vec(x, x_stride) && row_vec(y, y_stride) && tables_vec(weight, bias, n_groups, mod_stride);
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
    const bool vec = D % 4 == 0 && row_vec(x, x_stride) && row_vec(dy, dy_stride) && row_vec(dres, dres_stride) &&
                     row_vec(dx, dx_stride) && tables_vec(weight, nullptr, n_groups, mod_stride);
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
