// Layer norm with an optional weight and bias per group of rows, and its backward pass.
//
//   forward    mu = mean(x), r = 1 / sqrt(mean((x - mu)^2) + eps), xh = (x - mu) r,  y = xh w + b
//   backward   v = dy w;  dx = r (v - mean(v) - xh mean(v xh)) + dres;  dw = sum_rows dy xh;  db = sum_rows dy
//
// w and b belong to a group of consecutive rows (a sequence, for adaptive norms, where w = 1 + scale) or to all of them.
// Both directions are one pass over the data and bound by HBM: every row is read once.  Statistics are fp32: each warp takes
// the mean of its own columns and their squared deviations from it, and the parts are combined with the exact formula
// M2 = sum M2_k + n_k (mean_k - mean)^2, so that a large mean cancels nothing.
// Forward: where a warp can hold a row in registers it does, so that a row costs ten exchanges and no barrier: up to 2048 columns in
// whole blocks of 128, 1280 of other widths, 768 in accesses of two columns, 256 of one; wider rows take the warps of a CTA
// (launch_fwd).  With four columns per access the weight and bias of a group come from the L1, with fewer they stay in
// registers.  24 x 1024 rows of 1152, fp32 to bf16, weight and bias per sequence: 31 us as calls on new inputs (5.5 TB/s), 27 without
// the statistics, 25 where a replayed graph finds part of its one input in the L2; a CTA per row with a barrier each took 41.
// 6144 rows of 4608: 33 us.
// Backward: the column sums need registers too, so a row is spread over warps with 12 or 16 columns per lane and one
// barrier; rows are copied to shared memory one ahead of their use, every thread its own columns, so that the bytes in flight do
// not cost registers.  The same rows with the residual path's gradient added: 72 us as calls (5.5 TB/s), of which the kernel takes
// 62 to 65 and the sums 5.
// The gradients of w and b are column sums over a group's rows.  A CTA keeps them in fp32 registers over a run of rows of
// one group and writes one partial row; a second, small launch adds the partial rows of a group in a fixed order, so that
// repeats are bit-identical (no atomics).
#include "rms_norm.h"

namespace {

constexpr int kMaxWarps = 32;
constexpr int kMaxD = kMaxWarps * 256;
constexpr int kSms = 148;
constexpr int kNarrowPerSm = 4, kNarrowBwdPerSm = 2;   // CTAs of the kernels for narrow rows on an SM

// ---- VW consecutive columns: 4 (rows aligned to four elements, D % 4 == 0), 2, or 1 (any D, any row stride) ------------------
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
// 32-bit words that they are held in: as they come from memory, bf16 packed two by two (single ones as floats)
template <typename E, int VW> constexpr int kWords = sizeof(E) == 4 || VW == 1 ? VW : VW / 2;
template <typename E, int VW> __device__ __forceinline__ float value(const uint32_t* w, int e) {
    if (sizeof(E) == 4 || VW == 1) return __uint_as_float(w[e]);
    return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}
// ONCE: read past the caches' older lines.  Not for single fp32 columns in the backward and narrow kernels, where two accesses share a
// line and the second comes late (20000 x 1001, fp32 and bf16, backward: 63 us, with it 152; forward the other way, 39 and 32).
template <typename E, int VW, bool ONCE = true> __device__ __forceinline__ void load(const E* p, bool ok, uint32_t* w) {
    constexpr int B = VW * (int)sizeof(E);
    if (B == 16) {
        const uint4 u = ok ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
        w[0] = u.x; w[1] = u.y; w[2 % kWords<E, VW>] = u.z; w[3 % kWords<E, VW>] = u.w;
    } else if (B == 8) {
        const uint2 u = ok ? __ldcs(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
        w[0] = u.x; w[1 % kWords<E, VW>] = u.y;
    } else if (B == 4) {
        const uint32_t* q = reinterpret_cast<const uint32_t*>(p);
        w[0] = !ok ? 0u : ONCE || VW > 1 ? __ldcs(q) : *q;
    } else {
        w[0] = ok ? __float_as_uint(to_f(*p)) : 0u;
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int VW> __device__ __forceinline__ void store(float* p, const float* v) {
    if (VW == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1 % VW], v[2 % VW], v[3 % VW]);
    else if (VW == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1 % VW]);
    else *p = v[0];
}
template <int VW> __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
    if (VW == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1 % VW]), pack2(v[2 % VW], v[3 % VW]));
    else if (VW == 2) *reinterpret_cast<uint32_t*>(p) = pack2(v[0], v[1 % VW]);
    else *p = __float2bfloat16(v[0]);
}
// a table's row: fp32, aligned as the rows are
template <int VW> __device__ __forceinline__ void table(const float* p, bool ok, float add, float* v) {
    uint32_t w[VW];
    if (VW == 4) {
        const float4 f = ok ? __ldg(reinterpret_cast<const float4*>(p)) : make_float4(0.f, 0.f, 0.f, 0.f);
        w[0] = __float_as_uint(f.x); w[1 % VW] = __float_as_uint(f.y); w[2 % VW] = __float_as_uint(f.z); w[3 % VW] = __float_as_uint(f.w);
    } else if (VW == 2) {
        const float2 f = ok ? __ldg(reinterpret_cast<const float2*>(p)) : make_float2(0.f, 0.f);
        w[0] = __float_as_uint(f.x); w[1 % VW] = __float_as_uint(f.y);
    } else {
        w[0] = ok ? __float_as_uint(__ldg(p)) : 0u;
    }
#pragma unroll
    for (int e = 0; e < VW; ++e) v[e] = __uint_as_float(w[e]) + add;
}
// asynchronously to shared memory (not for single bf16 columns), and back from there
template <typename E, int VW> __device__ __forceinline__ void send(uint32_t smem, const E* g) {
    constexpr int B = VW * (int)sizeof(E);
    if (B == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem), "l"(g) : "memory");
    else if (B == 8) asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem), "l"(g) : "memory");
    else if (B == 4) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem), "l"(g) : "memory");
}
template <typename E, int VW> __device__ __forceinline__ void take(uint32_t smem, bool ok, uint32_t* w) {
    constexpr int B = VW * (int)sizeof(E), N = kWords<E, VW>;
    uint32_t u[4] = {0u, 0u, 0u, 0u};
    if (B == 16) asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(u[0]), "=r"(u[1]), "=r"(u[2]), "=r"(u[3]) : "r"(smem) : "memory");
    else if (B == 8) asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(u[0]), "=r"(u[1]) : "r"(smem) : "memory");
    else if (B == 4) asm volatile("ld.shared.b32 %0, [%1];" : "=r"(u[0]) : "r"(smem) : "memory");
#pragma unroll
    for (int q = 0; q < N; ++q) w[q] = ok ? u[q] : 0u;             // outside the row nothing was copied there
}
__device__ __forceinline__ void copy_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copy_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

// The columns of a lane: N columns of a block of 32 N that starts at `base`, in pieces of VW consecutive ones, so that the
// accesses of a warp are whole runs of 32 VW elements.  (Eight consecutive fp32 columns per lane, two 16-byte accesses 32 bytes
// apart, make two half-used sectors of every sector: measured 20 to 40% slower.)  FULL: the row fills the block, nothing is checked.
template <int N, int VW, bool FULL> struct Cols {
    int D, base, lane;
    __device__ __forceinline__ int at(int piece) const { return base + piece * 32 * VW + lane * VW; }
    __device__ __forceinline__ bool in(int piece) const { return FULL || at(piece) < D; }
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
    const float* rstd_in;                     // without a mean: [M], in place of stats_in
    int heads;                                // without a mean: row i is head i % heads of token i / heads; the strides above are the
    long long x_head, dy_head, dres_head, dx_head;    // tokens', these the heads' (narrow rows only)
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

// A team is one warp where NH blocks hold the row (MAXW == 1), else the CTA.  The next row's loads are in flight while this one is
// reduced; the weight and bias come from the L1 (in registers they cost more rows in flight than they save: 31.2 against 30.7 us
// for 24 x 1024 rows of 1152, 4.8 against 3.5 for 2048 rows).
template <typename TX, typename TY, int NH, int VW, bool FULL, int MAXT, int MINB, int MAXW>
__global__ void __launch_bounds__(MAXT, MINB) layer_norm_kernel(const NormArgs a) {
    __shared__ float2 part[2][MAXW];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int W = MAXW > 1 ? a.warps : 1;
    constexpr int P = 4 * NH / VW, XW = kWords<TX, VW>;         // pieces of a lane, words of a piece
    const Cols<4 * NH, VW, FULL> c{a.D, (W > 1 ? warp : 0) * NH * 128, lane};
    const int k = W > 1 ? warp : 0;
    const TX* x = reinterpret_cast<const TX*>(a.x);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long team = MAXW > 1 ? blockIdx.x : (long long)blockIdx.x * (blockDim.x >> 5) + warp;
    const long long first = team * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    constexpr float full = NH * 128.f;                             // columns of all of a team's warps but the last
    const float inv_d = 1.f / (float)a.D, n_last = (float)a.D - (float)(W - 1) * full;
    const float inv_n = k < W - 1 ? 1.f / full : 1.f / n_last;
    uint32_t nx[P][XW];
    auto fetch = [&](long long row) {
#pragma unroll
        for (int p = 0; p < P; ++p) load<TX, VW>(x + row * a.x_stride + c.at(p), c.in(p), nx[p]);
    };
    const bool tables = a.weight || a.bias;
    // the first row that the weight and bias at hand do not belong to, where they lie, and how far away the next group's are
    // (one division per warp: the code stays short, which counts more than anything else for small calls)
    const long long g0 = !tables ? 0 : first <= 0xffffffffLL ? (long long)((uint32_t)first / (uint32_t)a.rows_per_group) : first / a.rows_per_group;
    long long group_end = tables ? g0 * a.rows_per_group : a.M, mo = g0 * a.mod_stride, step = 0;
    if (first < last) fetch(first);
    // narrow accesses: the tables would cost as many as the rows, so the current group's stay in registers
    constexpr bool KEEP = VW < 4;
    float w[KEEP ? P : 1][VW], b[KEEP ? P : 1][VW];
    if (KEEP) {
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) { w[p][e] = 1.f; b[p][e] = 0.f; }
    }
    int it = 0;
    for (long long row = first; row < last; ++row, ++it) {
        if (row >= group_end) {                                    // uniform over the team
            mo += step;
            step = a.mod_stride;
            group_end += a.rows_per_group;
            if (KEEP) {
#pragma unroll
                for (int p = 0; p < P; ++p) {
                    if (a.weight) table<VW>(a.weight + mo + c.at(p), c.in(p), a.unit, w[p]);
                    if (a.bias) table<VW>(a.bias + mo + c.at(p), c.in(p), 0.f, b[p]);
                }
            }
        }
        float v[P][VW];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) v[p][e] = value<TX, VW>(nx[p], e);
        if (row + 1 < last) fetch(row + 1);
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) s += VW == 4 ? (v[p][0] + v[p][1 % VW]) + (v[p][2 % VW] + v[p][3 % VW]) : VW == 2 ? v[p][0] + v[p][1 % VW] : v[p][0];
        float mu = free_warp_sum(s) * inv_n, q = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) { const float d = v[p][e] - mu; q += c.in(p) ? d * d : 0.f; }
        float m2 = free_warp_sum(q);                               // squared deviations from this warp's mean
        if (MAXW > 1) {
            float2* now = part[it & 1];                            // a buffer is rewritten two barriers after its last read
            if (lane == 0) now[warp] = make_float2(mu, m2);
            __syncthreads();
            const float2 pl = now[W - 1], t = team_sum<MAXW>(now, W - 1);
            mu = (full * t.x + n_last * pl.x) * inv_d;
            float d2 = 0.f;
#pragma unroll
            for (int j = 0; j < MAXW; ++j)
                if (j < W - 1) { const float d = now[j].x - mu; d2 = fmaf(d, d, d2); }
            m2 = t.y + pl.y + full * d2 + n_last * (pl.x - mu) * (pl.x - mu);
        }
        const float rstd = rsqrtf(m2 * inv_d + a.eps);
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float o[VW], t[VW];
#pragma unroll
            for (int e = 0; e < VW; ++e) o[e] = (v[p][e] - mu) * rstd;
            if (KEEP) {
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] = o[e] * w[p][e] + b[p][e];
            } else {
                if (a.weight) {
                    table<VW>(a.weight + mo + c.at(p), c.in(p), a.unit, t);
#pragma unroll
                    for (int e = 0; e < VW; ++e) o[e] *= t[e];
                }
                if (a.bias) {
                    table<VW>(a.bias + mo + c.at(p), c.in(p), 0.f, t);
#pragma unroll
                    for (int e = 0; e < VW; ++e) o[e] += t[e];
                }
            }
            if (c.in(p)) store<VW>(y + row * a.y_stride + c.at(p), o);
        }
        if (a.stats && k == 0 && lane == 0) { a.stats[2 * row] = mu; a.stats[2 * row + 1] = rstd; }
    }
}

// Whether rows are copied to shared memory ahead of their use: copies are of 4, 8 or 16 bytes.
template <typename TX, typename TY, int VW> constexpr bool kAhead = VW * sizeof(TX) >= 4 && VW * sizeof(TY) >= 4;

// One CTA, a team of warps with C columns per lane, per (group, chunk): a run of the group's rows, R of them per barrier and R more in
// flight.  T: threads per SM that the register budget is set for.
// RMS: the norm without a mean and bias, dx = r (v - xh mean(v xh)) + dres with xh = x r (24 x 1024 rows of 1152, fp32 with the residual's
// gradient, bf16 dy: 60 us, 69 with the sums of the table's columns).
template <typename TX, typename TY, int C, int VW, int MAXT, int T, int R, bool RMS>
__global__ void __launch_bounds__(MAXT, T / MAXT) layer_norm_bwd_kernel(const NormArgs a) {
    constexpr int P = C / VW, XW = kWords<TX, VW>, YW = kWords<TY, VW>;      // pieces of a lane, words of a piece
    constexpr bool AHEAD = kAhead<TX, TY, VW>;
    __shared__ float2 part[2][R][MAXT / 32];
    extern __shared__ uint4 ring[];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, W = a.warps;
    const Cols<C, VW, false> c{a.D, warp * 32 * C, lane};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const TY* dy = reinterpret_cast<const TY*>(a.dy);
    const TX* dres = reinterpret_cast<const TX*>(a.dres);
    TX* dx = reinterpret_cast<TX*>(a.dx);
    const int g = blockIdx.x / a.chunks, ch = blockIdx.x % a.chunks;
    const long long base = (long long)g * a.rows_per_group;
    const long long lo = base + (long long)a.rows_per_group * ch / a.chunks, hi = base + (long long)a.rows_per_group * (ch + 1) / a.chunks;
    const float inv_d = 1.f / (float)a.D;
    // shared memory: two groups of R rows, of each x, dres and dy, [warp][piece][lane]; running addresses, for the pass counts every
    // instruction (24 x 1024 rows of 1152 bf16, this kernel alone: 46.3 us, with products of row and stride 48.4)
    const uint32_t T0 = blockDim.x, bx = T0 * C * (uint32_t)sizeof(TX), one = 2 * bx + T0 * C * (uint32_t)sizeof(TY);
    const uint32_t place = warp * 32 * C + lane * VW;
    uint32_t now = (uint32_t)__cvta_generic_to_shared(ring), then = now + R * one;
    auto px = [&](uint32_t u, int p) { return u + place * (uint32_t)sizeof(TX) + p * 32 * VW * (uint32_t)sizeof(TX); };
    auto py = [&](uint32_t u, int p) { return u + 2 * bx + place * (uint32_t)sizeof(TY) + p * 32 * VW * (uint32_t)sizeof(TY); };
    const TX *fx = x + lo * a.x_stride + c.at(0), *fr = dres + lo * a.dres_stride + c.at(0);
    const TY* fy = dy + lo * a.dy_stride + c.at(0);
    long long ahead = lo;                                          // the row to copy next
    auto fetch = [&](uint32_t to) {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (ahead < hi) {
                const uint32_t u = to + r * one;
#pragma unroll
                for (int p = 0; p < P; ++p)
                    if (c.in(p)) {
                        send<TX, VW>(px(u, p), fx + p * 32 * VW);
                        if (dres) send<TX, VW>(px(u + bx, p), fr + p * 32 * VW);
                        send<TY, VW>(py(u, p), fy + p * 32 * VW);
                    }
            }
            ++ahead; fx += a.x_stride; fr += a.dres_stride; fy += a.dy_stride;
        }
        copy_commit();
    };
    auto stats_of = [&](long long row) {
        if (RMS) return make_float2(0.f, row < hi ? __ldg(a.rstd_in + row) : 0.f);
        return row < hi ? make_float2(__ldg(a.stats_in + 2 * row), __ldg(a.stats_in + 2 * row + 1)) : make_float2(0.f, 0.f);
    };
    if (AHEAD) fetch(now);
    float w[P][VW], dw[P][VW], db[P][VW];
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int e = 0; e < VW; ++e) { w[p][e] = 1.f; dw[p][e] = 0.f; db[p][e] = 0.f; }
        if (a.weight) table<VW>(a.weight + (long long)g * a.mod_stride + c.at(p), c.in(p), a.unit, w[p]);
    }
    float2 next[R];                                                // statistics of the rows to come
#pragma unroll
    for (int r = 0; r < R; ++r) next[r] = stats_of(lo + r);
    int it = 0;
    for (long long row = lo; row < hi; row += R, ++it) {
        uint32_t res[R][P][XW];
        float2 st[R], sum[R];
        float xh[R][P][VW], v[R][P][VW];
        if (AHEAD) {
            fetch(then);                                           // into the slot that the previous rows left
            copy_wait<1>();
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool live = R == 1 || row + r < hi;              // past the run: nothing is counted or stored
            const long long rr = live ? row + r : row;
            st[r] = next[r];
            next[r] = stats_of(row + R + r);
            uint32_t rx[P][XW], ry[P][YW];
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (AHEAD) {
                    take<TX, VW>(px(now + r * one, p), c.in(p), rx[p]);
                    take<TY, VW>(py(now + r * one, p), c.in(p), ry[p]);
                } else {
                    load<TX, VW, false>(x + rr * a.x_stride + c.at(p), c.in(p), rx[p]);
                    load<TY, VW, false>(dy + rr * a.dy_stride + c.at(p), c.in(p), ry[p]);
                    if (dres) load<TX, VW, false>(dres + rr * a.dres_stride + c.at(p), c.in(p), res[r][p]);
                }
            }
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                const bool in = live && c.in(p);
#pragma unroll
                for (int e = 0; e < VW; ++e) {
                    const float d = in ? value<TY, VW>(ry[p], e) : 0.f;
                    xh[r][p][e] = in ? (RMS ? value<TX, VW>(rx[p], e) : value<TX, VW>(rx[p], e) - st[r].x) * st[r].y : 0.f;
                    v[r][p][e] = d * w[p][e];
                    if (!RMS) s1 += v[r][p][e];
                    s2 = fmaf(v[r][p][e], xh[r][p][e], s2);
                    dw[p][e] = fmaf(d, xh[r][p][e], dw[p][e]);
                    if (!RMS) db[p][e] += d;
                }
            }
            sum[r] = make_float2(RMS ? 0.f : free_warp_sum(s1), free_warp_sum(s2));
        }
        if (W > 1) {
            float2 (*sums)[MAXT / 32] = part[it & 1];               // a buffer is rewritten two barriers after its last read
            if (lane == 0) {
#pragma unroll
                for (int r = 0; r < R; ++r) sums[r][warp] = sum[r];
            }
            __syncthreads();
#pragma unroll
            for (int r = 0; r < R; ++r) sum[r] = team_sum<MAXT / 32>(sums[r], W);
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            if (row + r >= hi) break;
            const float m1 = sum[r].x * inv_d, m2 = sum[r].y * inv_d;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float o[VW];
                if (AHEAD && dres) take<TX, VW>(px(now + r * one + bx, p), c.in(p), res[r][p]);
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] = fmaf(st[r].y, (RMS ? v[r][p][e] : v[r][p][e] - m1) - xh[r][p][e] * m2, dres ? value<TX, VW>(res[r][p], e) : 0.f);
                if (c.in(p)) store<VW>(dx + (row + r) * a.dx_stride + c.at(p), o);
            }
        }
        const uint32_t t = now;
        now = then;
        then = t;
    }
    if (AHEAD) copy_wait<0>();                                     // nothing is in flight when the CTA ends
    if (!a.dw && !a.db) return;
    float *ow = a.dw ? a.dw + (long long)g * a.dmod_stride : nullptr, *ob = a.db ? a.db + (long long)g * a.dmod_stride : nullptr;
    if (a.chunks > 1) {
        ow = a.partial + (long long)blockIdx.x * (RMS ? 1 : 2) * a.D;
        ob = RMS ? nullptr : ow + a.D;
    }
#pragma unroll
    for (int p = 0; p < P; ++p)
        if (c.in(p)) {
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                if (ow) ow[c.at(p) + e] = dw[p][e];
                if (ob && !RMS) ob[c.at(p) + e] = db[p][e];
            }
        }
}

// ---- narrow rows (norms over a head; up to 256 columns) ---------------------------------------------------------------------
// L lanes hold a row, C columns each, and a warp 32 / L rows at a time: fewer exchanges per row and no idle lanes.  393216 rows of
// 64, bf16: forward 22.5 us (a warp per row 160), backward 37 (139); 65536 rows of 192: 15 (19) and 26 (43).  Fewer columns per
// lane are slower (forward 29, four instead of eight), but for single columns (65536 rows of 127: 15 against 17, backward 27
// against 51).
template <int VW> constexpr int kNarrowCols = VW == 1 ? 4 : 8;     // C, for rows of 33 to 128 columns
template <int L> __device__ __forceinline__ float part_sum(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}
template <int L, int C, int VW> struct NarrowCols {
    int D, lane;
    __device__ __forceinline__ int at(int piece) const { return (piece * L + lane) * VW; }
    __device__ __forceinline__ bool in(int piece) const { return at(piece) < D; }
};

// A warp takes rows_per_team consecutive rows, its parts neighbouring ones.  The tables stay in registers until the group changes.
template <typename TX, typename TY, int L, int C, int VW>
__global__ void __launch_bounds__(256, kNarrowPerSm) layer_norm_narrow_kernel(const NormArgs a) {
    constexpr int P = C / VW, XW = kWords<TX, VW>, R = 32 / L;
    free_grid_dep_wait();
    free_grid_dep_launch();
    const NarrowCols<L, C, VW> c{a.D, (int)(threadIdx.x % L)};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    const float inv_d = 1.f / (float)a.D;
    long long row = first + (threadIdx.x & 31) / L;
    uint32_t nx[P][XW];
    auto fetch = [&](long long r) {
#pragma unroll
        for (int p = 0; p < P; ++p) load<TX, VW, false>(x + r * a.x_stride + c.at(p), r < last && c.in(p), nx[p]);
    };
    const bool tables = a.weight || a.bias;
    const long long g0 = !tables ? 0 : first <= 0xffffffffLL ? (long long)((uint32_t)first / (uint32_t)a.rows_per_group) : first / a.rows_per_group;
    long long group_end = tables ? g0 * a.rows_per_group : a.M, mo = g0 * a.mod_stride, step = 0;
    fetch(row);
    float w[P][VW], b[P][VW];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < VW; ++e) { w[p][e] = 1.f; b[p][e] = 0.f; }
    for (long long base = first; base < last; base += R, row += R) {
        const bool live = row < last;                              // all lanes take part in the exchanges
        if (live && row >= group_end) {
            do {
                mo += step;
                step = a.mod_stride;
                group_end += a.rows_per_group;
            } while (row >= group_end);
#pragma unroll
            for (int p = 0; p < P; ++p) {
                if (a.weight) table<VW>(a.weight + mo + c.at(p), c.in(p), a.unit, w[p]);
                if (a.bias) table<VW>(a.bias + mo + c.at(p), c.in(p), 0.f, b[p]);
            }
        }
        float v[P][VW], s = 0.f, q = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) { v[p][e] = value<TX, VW>(nx[p], e); s += v[p][e]; }
        fetch(row + R);
        const float mu = part_sum<L>(s) * inv_d;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) { v[p][e] -= mu; q += c.in(p) ? v[p][e] * v[p][e] : 0.f; }
        const float rstd = rsqrtf(part_sum<L>(q) * inv_d + a.eps);
        if (live) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float o[VW];
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] = v[p][e] * rstd * w[p][e] + b[p][e];
                if (c.in(p)) store<VW>(y + row * a.y_stride + c.at(p), o);
            }
            if (a.stats && c.lane == 0) { a.stats[2 * row] = mu; a.stats[2 * row + 1] = rstd; }
        }
    }
}

// One CTA per (group, chunk) as for wide rows; its warps take the run's rows in turn and their column sums are added at the end.
template <typename TX, typename TY, int L, int C, int VW, bool RMS>
__global__ void __launch_bounds__(256, kNarrowBwdPerSm) layer_norm_narrow_bwd_kernel(const NormArgs a) {
    constexpr int P = C / VW, XW = kWords<TX, VW>, YW = kWords<TY, VW>, R = 32 / L, N = L * C;
    __shared__ float sums[8][2][N];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int warp = threadIdx.x >> 5, W = blockDim.x >> 5;
    const NarrowCols<L, C, VW> c{a.D, (int)(threadIdx.x % L)};
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const TY* dy = reinterpret_cast<const TY*>(a.dy);
    const TX* dres = reinterpret_cast<const TX*>(a.dres);
    TX* dx = reinterpret_cast<TX*>(a.dx);
    const int g = blockIdx.x / a.chunks, ch = blockIdx.x % a.chunks;
    const long long base = (long long)g * a.rows_per_group;
    const long long lo = base + (long long)a.rows_per_group * ch / a.chunks, hi = base + (long long)a.rows_per_group * (ch + 1) / a.chunks;
    const float inv_d = 1.f / (float)a.D;
    uint32_t nx[P][XW], ny[P][YW], nr[P][XW];
    float2 ns;
    // without a mean: heads of tokens; the row's token and head are counted on
    const int H = RMS ? a.heads : 1;
    long long tok = lo + warp * R + (threadIdx.x & 31) / L;
    int head = 0;
    if (RMS && H > 1) { head = (int)(tok % H); tok /= H; }
    const int step_tok = W * R / H, step_head = W * R % H;
    auto fetch = [&](long long r) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool ok = r < hi && c.in(p);
            if (RMS) {
                load<TX, VW, false>(x + tok * a.x_stride + head * a.x_head + c.at(p), ok, nx[p]);
                load<TY, VW, false>(dy + tok * a.dy_stride + head * a.dy_head + c.at(p), ok, ny[p]);
                load<TX, VW, false>(dres + tok * a.dres_stride + head * a.dres_head + c.at(p), ok && dres, nr[p]);
                continue;
            }
            load<TX, VW, false>(x + r * a.x_stride + c.at(p), ok, nx[p]);
            load<TY, VW, false>(dy + r * a.dy_stride + c.at(p), ok, ny[p]);
            load<TX, VW, false>(dres + r * a.dres_stride + c.at(p), ok && dres, nr[p]);
        }
        if (RMS) ns = make_float2(0.f, r < hi ? __ldg(a.rstd_in + r) : 0.f);
        else ns = r < hi ? make_float2(__ldg(a.stats_in + 2 * r), __ldg(a.stats_in + 2 * r + 1)) : make_float2(0.f, 0.f);
    };
    long long row = lo + warp * R + (threadIdx.x & 31) / L;
    fetch(row);
    float w[P][VW], dw[P][VW], db[P][VW];
#pragma unroll
    for (int p = 0; p < P; ++p) {
#pragma unroll
        for (int e = 0; e < VW; ++e) { w[p][e] = 1.f; dw[p][e] = 0.f; db[p][e] = 0.f; }
        if (a.weight) table<VW>(a.weight + (long long)g * a.mod_stride + c.at(p), c.in(p), a.unit, w[p]);
    }
    for (long long first = lo + warp * R; first < hi; first += W * R, row += W * R) {
        const bool live = row < hi;
        const float2 st = ns;
        float xh[P][VW], v[P][VW], s1 = 0.f, s2 = 0.f;
        uint32_t res[P][XW];
#pragma unroll
        for (int p = 0; p < P; ++p) {
            const bool in = live && c.in(p);
#pragma unroll
            for (int e = 0; e < VW; ++e) {
                const float d = value<TY, VW>(ny[p], e);           // zero outside the row
                xh[p][e] = in ? (RMS ? value<TX, VW>(nx[p], e) : value<TX, VW>(nx[p], e) - st.x) * st.y : 0.f;
                v[p][e] = d * w[p][e];
                if (!RMS) s1 += v[p][e];
                s2 = fmaf(v[p][e], xh[p][e], s2);
                dw[p][e] = fmaf(d, xh[p][e], dw[p][e]);
                if (!RMS) db[p][e] += d;
            }
#pragma unroll
            for (int q = 0; q < XW; ++q) res[p][q] = nr[p][q];
        }
        TX* out = dx + (RMS ? tok * a.dx_stride + head * a.dx_head : row * a.dx_stride);
        if (RMS) {
            tok += step_tok; head += step_head;
            if (head >= H) { head -= H; ++tok; }
        }
        fetch(row + W * R);
        const float m1 = RMS ? 0.f : part_sum<L>(s1) * inv_d, m2 = part_sum<L>(s2) * inv_d;
        if (live) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float o[VW];
#pragma unroll
                for (int e = 0; e < VW; ++e) o[e] = fmaf(st.y, (RMS ? v[p][e] : v[p][e] - m1) - xh[p][e] * m2, value<TX, VW>(res[p], e));
                if (c.in(p)) store<VW>(out + c.at(p), o);
            }
        }
    }
    if (!a.dw && !a.db) return;
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < VW; ++e) {
#pragma unroll
            for (int o = L; o < 32; o <<= 1) {
                dw[p][e] += __shfl_xor_sync(~0u, dw[p][e], o);
                if (!RMS) db[p][e] += __shfl_xor_sync(~0u, db[p][e], o);
            }
            if ((threadIdx.x & 31) < L) { sums[warp][0][c.at(p) + e] = dw[p][e]; if (!RMS) sums[warp][1][c.at(p) + e] = db[p][e]; }
        }
    __syncthreads();
    float *ow = a.dw ? a.dw + (long long)g * a.dmod_stride : nullptr, *ob = a.db ? a.db + (long long)g * a.dmod_stride : nullptr;
    if (a.chunks > 1) {
        ow = a.partial + (long long)blockIdx.x * (RMS ? 1 : 2) * a.D;
        ob = RMS ? nullptr : ow + a.D;
    }
    for (int i = threadIdx.x; i < (RMS ? 1 : 2) * N; i += blockDim.x) {
        const int col = i % N;
        float* out = i < N ? ow : ob;
        if (col >= a.D || !out) continue;
        float t = 0.f;
        for (int k = 0; k < W; ++k) t += sums[k][i / N][col];
        out[col] = t;
    }
}

// dw, db of a group = the sum of its chunks' partial rows: 32 columns x 16 slices of the chunks per CTA, slices joined in order.
__global__ void __launch_bounds__(512) layer_norm_reduce_kernel(const NormArgs a, int width) {
    __shared__ float sh[16][33];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int tx = threadIdx.x & 31, ty = threadIdx.x >> 5;
    const int blocks = (width + 31) / 32, g = blockIdx.x / blocks, j = (blockIdx.x % blocks) * 32 + tx;   // j: column of a partial row, [2][D] or, without a mean, [D]
    const float* p = a.partial + (long long)g * a.chunks * width;
    float s = 0.f;
    if (j < width) {
#pragma unroll 8
        for (int k = ty; k < a.chunks; k += 16) s += p[(long long)k * width + j];
    }
    sh[ty][tx] = s;
    __syncthreads();
    if (ty == 0 && j < width) {
        float t = 0.f;
#pragma unroll
        for (int k = 0; k < 16; ++k) t += sh[k][tx];
        float* out = j < a.D ? a.dw : a.db;
        if (out) out[(long long)g * a.dmod_stride + (j < a.D ? j : j - a.D)] = t;
    }
}

// Columns per lane of the backward kernel for wide rows.  It is bound by issue slots where the rows are bf16, and a row takes each of
// its warps what 16 columns take besides (exchanges, addresses, the barrier): so the number whose warps cost least, 12 or 16.
// 24 x 1024 rows of 1152 bf16: 48.6 us with 12, 61.6 with 8; 8192 rows of 4096: 53 with 16, 66 with 8.  Eight columns and two rows
// per barrier: odd widths, which are not copied ahead, and 4097 to 4608 columns, of which 16 would leave an SM with one CTA of nine
// warps.  8192 rows of 4608 bf16: 77 us, with 16 columns 83 (fp32 rows, bf16 gradients: 102 and 99).  Beyond 4608 eight columns
// would take more than 576 threads, whose registers hold one row instead of two: 8192 rows of 5000 bf16 114 us, with 16 columns 86
// (fp32 115 and 106), of 8192 153 and 110 (162 and 150).
int bwd_cols(int D) {
    if (D % 2 || (D > 4096 && D <= 4608)) return 8;
    const int w12 = (D + 383) / 384, w16 = (D + 511) / 512;
    return D <= 1536 && w12 * (12 + 16) < w16 * (16 + 16) ? 12 : 16;
}
// Threads of an SM that the registers are shared among, so that sums and rows stay in them (twelve columns: 640 and 768 threads are
// 3 and 7% slower).  Sixteen columns of fp32 rows still spill 32 to 80 bytes per thread, and so do a few forward kernels at their
// numbers of CTAs per SM (4 to 72 bytes).
constexpr int kBwdT = 512;
int bwd_threads(int D) { return (D + 32 * bwd_cols(D) - 1) / (32 * bwd_cols(D)) * 32; }
bool narrow(int D) { return D <= 128 || (D <= 256 && D % 2 == 0); }      // (single columns beyond 128: 32 us the wide way, 56 this)

// Chunks of a group in the backward pass: full waves of CTAs, at least eight rows each (64 where rows are narrow).  (A function of the sizes alone: the
// workspace depends on it.)
int chunks_of(int groups, int rows_per_group, int D) {
    const int t = bwd_threads(D);
    const int per_sm = narrow(D) ? kNarrowBwdPerSm : t >= kBwdT ? 1 : kBwdT / t;
    // the first number of waves that whole chunks fill to nine tenths, or else the best of four (one wave and a few CTAs more
    // take two: 4200 rows of 4608 in 14 groups 83 us, so 50)
    const long long resident = (long long)kSms * per_sm;
    long long want = 1;
    double best = 1e30;
    for (int k = 1; k <= 4 && best > 1.1; ++k) {
        const long long n = k * resident / groups;
        const double cost = n > 0 ? (double)k * resident / ((double)n * groups) : 1e30;
        if (cost < best) { best = cost; want = n; }
    }
    const long long most = rows_per_group / (narrow(D) ? 64 : 8);
    const long long c = want < most ? want : most;
    return c < 1 ? 1 : (int)c;
}

template <typename TX, typename TY, int NH, int VW, bool FULL, int MAXT, int MINB, int MAXW>
int start_fwd(NormArgs a, int warps, cudaStream_t s) {
    const int threads = MAXW > 1 ? warps * 32 : MAXT, teams = MAXW > 1 ? 1 : MAXT / 32;
    a.warps = warps;
    // one wave of the CTAs that the GPU holds at once; few rows: as many teams as there are rows
    const long long resident = (long long)kSms * (MINB * MAXT / threads) * teams;
    a.rows_per_team = (a.M + resident - 1) / resident;
    const long long grid = (a.M + a.rows_per_team * teams - 1) / (a.rows_per_team * teams);
    return free_launch(free_overlap_for_rows(a.M), layer_norm_kernel<TX, TY, NH, VW, FULL, MAXT, MINB, MAXW>, dim3((unsigned)grid), dim3(threads),
                       0, s, a);
}

template <typename TX, typename TY, int L, int C, int VW>
int start_narrow(NormArgs a, cudaStream_t s) {
    constexpr int R = 32 / L;
    const long long resident = (long long)kSms * kNarrowPerSm * 8;
    const long long steps = (a.M + resident * R - 1) / (resident * R);
    a.rows_per_team = steps * R;
    const long long grid = (a.M + a.rows_per_team * 8 - 1) / (a.rows_per_team * 8);
    return free_launch(free_overlap_for_rows(a.M), layer_norm_narrow_kernel<TX, TY, L, C, VW>, dim3((unsigned)grid), dim3(256), 0, s, a);
}
template <typename TX, typename TY, int L, int C, int VW, bool RMS>
int start_narrow_bwd(const NormArgs& a, cudaStream_t s) {
    const int steps = a.rows_per_group / a.chunks / (64 / L);      // a warp takes two steps of 32 / L rows at least
    const int warps = steps < 1 ? 1 : steps > 8 ? 8 : steps;
    return free_launch(free_overlap_for_rows(a.M), layer_norm_narrow_bwd_kernel<TX, TY, L, C, VW, RMS>, dim3((unsigned)a.groups * (unsigned)a.chunks),
                       dim3(warps * 32), 0, s, a);
}

// As many blocks of 128 columns per warp as the row needs (registers decide how many rows an SM holds), several warps beyond 2048
// columns.  Widths that the blocks fill exactly have kernels without checks (24 x 1024 rows of 1152: 29.5 us, with checks 34).  7, 11 and
// 13 to 15 blocks have none as yet and take the kernels with checks, which costs them 24 x 1024 rows, fp32 / bf16 to bf16: 896 columns
// 29 / 27 us, without checks 20 / 16; 1408 49 / 46, 33 / 25; 1664 66 / 61, 43 / 35; 1920 65 / 59, 49 / 39.
// With checks a warp holds up to 1280 columns (20000 rows of 1300, fp32 to bf16: 35 us by three warps, 56 by one; of 700: 25 by
// two, 18 by one); with one or two columns per access, where the tables need registers too, 256 (20000 rows of 1001, bf16: 35 us,
// with all in one warp 60; 690 in pairs: 19 and 15).
template <typename TX, typename TY, int VW>
int launch_fwd(const NormArgs& a, cudaStream_t s) {
    constexpr int C = kNarrowCols<VW>;
    if (a.D <= 32) return start_narrow<TX, TY, 8, 4, VW>(a, s);
    if (a.D <= 64) return start_narrow<TX, TY, 64 / C, C, VW>(a, s);
    if (a.D <= 128) return start_narrow<TX, TY, 128 / C, C, VW>(a, s);
    if constexpr (VW == 4) {
        const int n = a.D % 128 == 0 ? a.D / 128 : 0;
        switch (n) {
            case 2: return start_fwd<TX, TY, 2, 4, true, 128, 8, 1>(a, 1, s);
            case 3: return start_fwd<TX, TY, 3, 4, true, 128, 7, 1>(a, 1, s);
            case 4: return start_fwd<TX, TY, 4, 4, true, 128, 6, 1>(a, 1, s);
            case 5: return start_fwd<TX, TY, 5, 4, true, 128, 5, 1>(a, 1, s);
            case 6: return start_fwd<TX, TY, 6, 4, true, 128, 4, 1>(a, 1, s);
            case 8: return start_fwd<TX, TY, 8, 4, true, 128, 4, 1>(a, 1, s);
            case 9: return start_fwd<TX, TY, 9, 4, true, 128, 3, 1>(a, 1, s);
            case 10: return start_fwd<TX, TY, 10, 4, true, 128, 3, 1>(a, 1, s);
            case 12: return start_fwd<TX, TY, 12, 4, true, 128, 3, 1>(a, 1, s);
            case 16: return start_fwd<TX, TY, 16, 4, true, 128, 2, 1>(a, 1, s);
            default: break;
        }
        if (n > 16 && n % 9 == 0) return start_fwd<TX, TY, 9, 4, true, 256, 2, 8>(a, n / 9, s);
        if (n > 16 && n % 8 == 0) return start_fwd<TX, TY, 8, 4, true, 256, 2, 8>(a, n / 8, s);
    }
    if (a.D <= 256) return start_narrow<TX, TY, 32, 8, VW>(a, s);
    if constexpr (VW > 1) {
        if (a.D <= 512) return start_fwd<TX, TY, 4, VW, false, 128, VW == 4 ? 6 : 5, 1>(a, 1, s);
        if (a.D <= 768) return start_fwd<TX, TY, 6, VW, false, 128, VW == 4 ? 5 : 4, 1>(a, 1, s);
    }
    if constexpr (VW == 4) {
        if (a.D <= 1024) return start_fwd<TX, TY, 8, VW, false, 128, 4, 1>(a, 1, s);
        if (a.D <= 1280) return start_fwd<TX, TY, 10, VW, false, 128, 4, 1>(a, 1, s);
        if (a.D <= 4096) return start_fwd<TX, TY, 4, VW, false, 256, 3, 8>(a, (a.D + 511) / 512, s);
        constexpr int per = 1280;
        return start_fwd<TX, TY, 10, VW, false, 256, 2, (kMaxD + per - 1) / per>(a, (a.D + per - 1) / per, s);
    } else {
        if (a.D <= 2048) return start_fwd<TX, TY, 2, VW, false, 256, 3, 8>(a, (a.D + 255) / 256, s);
        return start_fwd<TX, TY, 4, VW, false, 512, 1, 16>(a, (a.D + 511) / 512, s);
    }
}

template <typename TX, typename TY, int C, int VW, int MAXT, int T, int R, bool RMS>
int start_bwd(const NormArgs& a, int threads, cudaStream_t s) {
    auto kernel = layer_norm_bwd_kernel<TX, TY, C, VW, MAXT, T, R, RMS>;
    constexpr size_t per = kAhead<TX, TY, VW> ? 2 * R * C * (2 * sizeof(TX) + sizeof(TY)) : 0;
    const size_t smem = threads * per;
    // the most that the kernel takes: another thread's call with narrower rows must not set it below this one's
    if (smem > 47 * 1024) FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)(MAXT * per)));
    return free_launch(free_overlap_for_rows(a.M), kernel, dim3((unsigned)a.groups * (unsigned)a.chunks), dim3(threads), smem, s, a);
}
template <typename TX, typename TY, int VW, bool RMS>
int start_wide_bwd(const NormArgs& a, int threads, cudaStream_t s) {
    const int cols = bwd_cols(a.D);
    if (cols == 12) return start_bwd<TX, TY, 12, VW, 128, kBwdT, 1, RMS>(a, threads, s);
    if (cols == 16) return start_bwd<TX, TY, 16, VW, 512, kBwdT, 1, RMS>(a, threads, s);
    if constexpr (VW == 1) {
        if (threads <= 256) return start_bwd<TX, TY, 8, VW, 256, kBwdT, 2, RMS>(a, threads, s);
        if (threads > 576) return start_bwd<TX, TY, 8, VW, 1024, 1024, 1, RMS>(a, threads, s);
    }
    return start_bwd<TX, TY, 8, VW, 576, 576, 2, RMS>(a, threads, s);
}

template <typename TX, typename TY, int VW, bool RMS>
int launch_bwd(NormArgs a, cudaStream_t s) {
    const int threads = bwd_threads(a.D);
    a.warps = threads / 32;
    constexpr int C = kNarrowCols<VW>;
    const int r = a.D <= 32 ? start_narrow_bwd<TX, TY, 8, 4, VW, RMS>(a, s) : a.D <= 64 ? start_narrow_bwd<TX, TY, 64 / C, C, VW, RMS>(a, s)
                : a.D <= 128 ? start_narrow_bwd<TX, TY, 128 / C, C, VW, RMS>(a, s)
                : narrow(a.D) ? start_narrow_bwd<TX, TY, 32, 8, VW, RMS>(a, s) : start_wide_bwd<TX, TY, VW, RMS>(a, threads, s);
    if (r != FREE_OK || a.chunks == 1 || (!a.dw && !a.db)) return r;
    return free_launch(free_launch_overlap_enabled(), layer_norm_reduce_kernel,
                       dim3((unsigned)a.groups * (((RMS ? 1u : 2u) * a.D + 31) / 32)), dim3(512), 0, s, a, (RMS ? 1 : 2) * a.D);
}

template <typename TX, typename TY>
int launch_fwd_vw(const NormArgs& a, int vw, cudaStream_t s) {
    return vw == 4 ? launch_fwd<TX, TY, 4>(a, s) : vw == 2 ? launch_fwd<TX, TY, 2>(a, s) : launch_fwd<TX, TY, 1>(a, s);
}
template <typename TX, typename TY, bool RMS = false>
int launch_bwd_vw(const NormArgs& a, int vw, cudaStream_t s) {
    return vw == 4 ? launch_bwd<TX, TY, 4, RMS>(a, s) : vw == 2 ? launch_bwd<TX, TY, 2, RMS>(a, s) : launch_bwd<TX, TY, 1, RMS>(a, s);
}

// Consecutive columns of one access: what D, the row strides and the tables' rows are aligned to (base pointers of rows are
// 16-byte aligned, which is checked; strides that are not used are passed as 0).
int width_of(int D, long long strides, const float* w, const float* b, int groups, long long mod_stride) {
    if (groups > 1 && (w || b)) strides |= mod_stride;
    const uintptr_t tables = reinterpret_cast<uintptr_t>(w) | reinterpret_cast<uintptr_t>(b);
    for (int v = 4; v > 1; v /= 2)
        if (D % v == 0 && strides % v == 0 && tables % (4 * v) == 0) return v;
    return 1;
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
    const int vw = width_of(D, x_stride | y_stride, weight, bias, n_groups, mod_stride);
    using bf = __nv_bfloat16;
    if (x_dtype == FREE_FP32) return y_dtype == FREE_FP32 ? launch_fwd_vw<float, float>(a, vw, s) : launch_fwd_vw<float, bf>(a, vw, s);
    return y_dtype == FREE_FP32 ? launch_fwd_vw<bf, float>(a, vw, s) : launch_fwd_vw<bf, bf>(a, vw, s);
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
    const int vw = width_of(D, x_stride | dy_stride | (dres ? dres_stride : 0) | dx_stride, weight, nullptr, n_groups, mod_stride);
    using bf = __nv_bfloat16;
    if (x_dtype == FREE_FP32) return y_dtype == FREE_FP32 ? launch_bwd_vw<float, float>(a, vw, s) : launch_bwd_vw<float, bf>(a, vw, s);
    return y_dtype == FREE_FP32 ? launch_bwd_vw<bf, float>(a, vw, s) : launch_bwd_vw<bf, bf>(a, vw, s);
}

size_t rms_norm_bwd_bytes(int groups, int rows_per_group, int D) { return free_op_layer_norm_bwd_workspace_bytes(groups, rows_per_group, D) / 2; }

bool rms_norm_bwd_takes_heads(int D) { return narrow(D); }

int rms_norm_bwd(const RmsBwdArgs& b, cudaStream_t s) {
    NormArgs a{};
    a.M = (long long)b.groups * b.rows_per_group; a.D = b.D; a.groups = b.groups; a.rows_per_group = b.rows_per_group;
    a.heads = b.heads;
    a.x = b.x; a.x_stride = b.x_tok; a.x_head = b.x_head; a.dy = b.dy; a.dy_stride = b.dy_tok; a.dy_head = b.dy_head;
    a.rstd_in = b.rstd; a.weight = b.weight; a.mod_stride = b.mod_stride; a.unit = b.unit;
    a.dres = b.dres; a.dres_stride = b.dres_tok; a.dres_head = b.dres_head; a.dx = b.dx; a.dx_stride = b.dx_tok; a.dx_head = b.dx_head;
    a.dw = b.dw; a.dmod_stride = b.dmod_stride; a.partial = b.ws;
    a.chunks = b.rows_per_group ? chunks_of(b.groups, b.rows_per_group, b.D) : 1;
    if ((long long)b.groups * a.chunks > 0x7fffffffLL || (long long)b.groups * ((b.D + 31LL) / 32) > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    if (b.dw && a.chunks > 1 && (!b.ws || b.ws_bytes < rms_norm_bwd_bytes(b.groups, b.rows_per_group, b.D))) return FREE_ERR_WORKSPACE;
    const long long strides = b.x_tok | b.dy_tok | b.dx_tok | (b.dres ? b.dres_tok : 0) | (b.heads > 1 ? b.x_head | b.dy_head | b.dx_head | (b.dres ? b.dres_head : 0) : 0);
    // addresses counted in elements: accesses are as wide as their low bits allow
    auto place = [](const void* p, int dtype) { return (long long)(reinterpret_cast<uintptr_t>(p) / (dtype == FREE_FP32 ? 4 : 2)) & 7; };
    const long long places = place(b.x, b.x_dtype) | place(b.dy, b.dy_dtype) | place(b.dx, b.x_dtype) | place(b.dres, b.x_dtype);
    const int vw = width_of(b.D, strides | places, b.weight, nullptr, b.groups, b.mod_stride);
    using bf = __nv_bfloat16;
    if (b.x_dtype == FREE_FP32) return b.dy_dtype == FREE_FP32 ? launch_bwd_vw<float, float, true>(a, vw, s) : launch_bwd_vw<float, bf, true>(a, vw, s);
    return b.dy_dtype == FREE_FP32 ? launch_bwd_vw<bf, float, true>(a, vw, s) : launch_bwd_vw<bf, bf, true>(a, vw, s);
}
