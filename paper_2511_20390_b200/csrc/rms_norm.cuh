// Root-mean-square norm of rows, with the residual's addition in front of it and a 32-, 16- or 8-bit result.
//
//   h = x + residual,   r = 1 / sqrt(mean(h^2) + eps),   y = h r w        (w: a weight per group of rows, or 1)
//   8 bits: for every run of 128 columns (or the row) s = max |y| / 448, q = e4m3(y / s)
//
// One pass over the data, bound by HBM: every row is read once and kept in registers as h in fp32 (the norm is of the unrounded
// sum; what is stored of h is rounded to the residual's type).  Rows of up to 1024 columns (512 of single accesses, and 1152) take one warp, P
// pieces of 128 columns (four consecutive ones per lane: whole 16- or 8-byte accesses, and one piece is one run of an 8-bit result's
// scale) or of 256 (eight); wider rows take several warps of a CTA, joined through shared memory.  The next row's loads are in flight while this one is reduced.
// Heads of up to 128 columns: four rows share a warp, or eight (rms_norm_heads_kernel).
// Measured, 24 x 1024 rows of 1152, bf16 onto an fp32 residual, per sequence: 53 us on its own, 59 to 62 one call after another (what they
// wrote leaves the L2 meanwhile; 340 MB, 52 us at a copy's rate).  16 heads of 72 in as many tokens: 23 us (18).  4100 rows of 4096 onto
// a bf16 residual, 8-bit values and a scale per 128 columns: 23 us (18).  256 rows of 384: 2 us in a graph of them, the launch.
#pragma once
#include "rms_norm.h"
#include <cuda_fp8.h>

namespace rms {

constexpr int kSms = 148;
using e4m3 = __nv_fp8_e4m3;

// VW columns as they come from memory, bf16 packed two by two (single ones as floats)
template <typename E, int VW> constexpr int kWords = sizeof(E) == 4 || VW == 1 ? VW : VW / 2;
template <typename E, int VW> __device__ __forceinline__ float value(const uint32_t* w, int e) {
    if (sizeof(E) == 4 || VW == 1) return __uint_as_float(w[e]);
    return __uint_as_float(e % 2 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
}
template <typename E, int VW> __device__ __forceinline__ void load(const E* p, bool ok, uint32_t* w) {
    if constexpr (VW * sizeof(E) == 16) {
        const uint4 u = ok ? __ldcs(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
        w[0] = u.x; w[1] = u.y; w[2] = u.z; w[3] = u.w;
    } else if constexpr (VW == 4) {
        const uint2 u = ok ? __ldcs(reinterpret_cast<const uint2*>(p)) : make_uint2(0u, 0u);
        w[0] = u.x; w[1] = u.y;
    } else if constexpr (sizeof(E) == 4) {
        w[0] = ok ? __float_as_uint(*p) : 0u;
    } else {
        w[0] = ok ? (uint32_t)*reinterpret_cast<const unsigned short*>(p) << 16 : 0u;
    }
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
template <int VW> __device__ __forceinline__ void store(float* p, const float* v) {
    static_assert(VW <= 4, "16-byte accesses");
    if constexpr (VW == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
    else *p = v[0];
}
template <int VW> __device__ __forceinline__ void store(__nv_bfloat16* p, const float* v) {
    if constexpr (VW == 8) *reinterpret_cast<uint4*>(p) = make_uint4(pack2(v[0], v[1]), pack2(v[2], v[3]), pack2(v[4], v[5]), pack2(v[6], v[7]));
    else if constexpr (VW == 4) *reinterpret_cast<uint2*>(p) = make_uint2(pack2(v[0], v[1]), pack2(v[2], v[3]));
    else *p = __float2bfloat16(v[0]);
}
__device__ __forceinline__ uint32_t pack4(const float* v) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(v[2], v[3]), __NV_SATFINITE, __NV_E4M3);
    return lo | hi << 16;
}
template <int VW> __device__ __forceinline__ void store(e4m3* p, const float* v) {
    if constexpr (VW == 8) *reinterpret_cast<uint2*>(p) = make_uint2(pack4(v), pack4(v + 4));
    else if constexpr (VW == 4) *reinterpret_cast<uint32_t*>(p) = pack4(v);
    else *reinterpret_cast<__nv_fp8_storage_t*>(p) = __nv_cvt_float_to_fp8(v[0], __NV_SATFINITE, __NV_E4M3);
}
template <int VW> __device__ __forceinline__ void table(const float* p, bool ok, float add, float* v) {
    if constexpr (VW == 1) {
        v[0] = (ok ? __ldg(p) : 0.f) + add;
    } else {
#pragma unroll
        for (int k = 0; k < VW; k += 4) {
            const float4 f = ok ? __ldg(reinterpret_cast<const float4*>(p + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
            v[k] = f.x + add; v[k + 1] = f.y + add; v[k + 2] = f.z + add; v[k + 3] = f.w + add;
        }
    }
}
// NaN is kept: a run with a NaN gets a NaN scale
__device__ __forceinline__ float max_nan(float a, float b) {
    float r;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
    return r;
}
template <int L = 32> __device__ __forceinline__ float warp_max(float v) {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) v = max_nan(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
// scale of a run whose largest magnitude is `top`, and its inverse; a run without anything above 2^-100 is zeros at scale 1
__device__ __forceinline__ float2 scale_of(float top) {
    const bool none = top < 7.888609e-31f;
    return none ? make_float2(1.f, 1.f) : make_float2(top * (1.f / 448.f), 448.f / top);
}

// W = a.warps warps hold a row (one of them: every warp of the CTA for itself).  FULL: P pieces fill it exactly.
template <typename TX, typename TR, typename TY, int P, int VW, bool FULL, int MAXT, int MINB>
__global__ void __launch_bounds__(MAXT, MINB) rms_norm_kernel(const RmsArgs a) {
    __shared__ float part[2][MAXT / 32], tops[2][MAXT / 32];
    constexpr bool Y8 = sizeof(TY) == 1;
    constexpr int XW = kWords<TX, VW>, RW = kWords<TR, VW>;
    constexpr int RUN = VW == 8 ? 1 : 4 / VW, SHARE = VW == 8 ? 16 : 32;      // pieces and lanes of a run of 128 columns
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, W = a.warps;
    const int col0 = (W > 1 ? warp : 0) * P * 32 * VW + lane * VW;
    auto at = [&](int p) { return col0 + p * 32 * VW; };
    auto in = [&](int p) { return FULL || at(p) < a.D; };
    const TX* x = reinterpret_cast<const TX*>(a.x);
    const TR* res = reinterpret_cast<const TR*>(a.res);
    TR* hout = reinterpret_cast<TR*>(a.h);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long team = W > 1 ? blockIdx.x : (long long)blockIdx.x * (blockDim.x >> 5) + warp;
    const long long first = team * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    const float inv_d = 1.f / (float)a.D;
    uint32_t nx[P][XW], nr[P][RW];
    auto fetch = [&](long long row) {
        const TX* px = x + (a.heads > 1 ? row / a.heads * a.x_tok + row % a.heads * a.x_head : row * a.x_tok);
#pragma unroll
        for (int p = 0; p < P; ++p) load<TX, VW>(px + at(p), in(p), nx[p]);
        if (res) {
#pragma unroll
            for (int p = 0; p < P; ++p) load<TR, VW>(res + row * a.res_stride + at(p), in(p), nr[p]);
        }
    };
    const long long g0 = a.weight ? first / a.rows_per_group : 0;
    long long group_end = a.weight ? (g0 + 1) * a.rows_per_group : a.M, mo = g0 * a.mod_stride;
    if (first < last) fetch(first);
    int it = 0;
    for (long long row = first; row < last; ++row, ++it) {
        if (row >= group_end) {                                    // uniform over the team
            mo += a.mod_stride;
            group_end += a.rows_per_group;
        }
        float v[P][VW];
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) v[p][e] = value<TX, VW>(nx[p], e);
        if (res) {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < VW; ++e) v[p][e] += value<TR, VW>(nr[p], e);
        }
        if (row + 1 < last) fetch(row + 1);
        if (res && hout) {
#pragma unroll
            for (int p = 0; p < P; ++p)
                if (in(p)) store<VW>(hout + row * a.h_stride + at(p), v[p]);
        }
        float s = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p) {
            float t = 0.f;
#pragma unroll
            for (int e = 0; e < VW; ++e) t = fmaf(v[p][e], v[p][e], t);
            s += t;
        }
        s = free_warp_sum(s);
        if (W > 1) {
            float* now = part[it & 1];                             // a buffer is rewritten two barriers after its last read
            if (lane == 0) now[warp] = s;
            __syncthreads();
            s = 0.f;
            for (int k = 0; k < W; ++k) s += now[k];
        }
        const float r = rsqrtf(s * inv_d + a.eps);
        if (a.rstd && threadIdx.x % (32 * W) == 0) a.rstd[row] = r;
        if (a.weight) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
                float w[VW];
                table<VW>(a.weight + mo + at(p), in(p), a.unit, w);
#pragma unroll
                for (int e = 0; e < VW; ++e) v[p][e] = v[p][e] * r * w[e];
            }
        } else {
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < VW; ++e) v[p][e] *= r;
        }
        TY* py = y + (a.heads > 1 ? row / a.heads * a.y_tok + row % a.heads * a.y_head : row * a.y_tok);
        if constexpr (Y8) {
            if (a.scale_block) {
#pragma unroll
                for (int b = 0; b < (P + RUN - 1) / RUN; ++b) {
                    float top = 0.f;
#pragma unroll
                    for (int p = b * RUN; p < (b + 1) * RUN && p < P; ++p)
#pragma unroll
                        for (int e = 0; e < VW; ++e) top = max_nan(top, fabsf(v[p][e]));
                    const float2 f = scale_of(warp_max<SHARE>(top));
#pragma unroll
                    for (int p = b * RUN; p < (b + 1) * RUN && p < P; ++p)
#pragma unroll
                        for (int e = 0; e < VW; ++e) v[p][e] *= f.y;
                    const int run = at(b * RUN) >> 7;
                    if (lane % SHARE == 0 && run * 128 < a.D) a.scales[row * a.scale_stride + run] = f.x;
                }
            } else {
                float top = 0.f;
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int e = 0; e < VW; ++e) top = max_nan(top, fabsf(v[p][e]));
                top = warp_max(top);
                if (W > 1) {
                    float* now = tops[it & 1];
                    if (lane == 0) now[warp] = top;
                    __syncthreads();
                    for (int k = 0; k < W; ++k) top = max_nan(top, now[k]);
                }
                const float2 f = scale_of(top);
#pragma unroll
                for (int p = 0; p < P; ++p)
#pragma unroll
                    for (int e = 0; e < VW; ++e) v[p][e] *= f.y;
                if (threadIdx.x % (32 * W) == 0) a.scales[row * a.scale_stride] = f.x;
            }
        }
#pragma unroll
        for (int p = 0; p < P; ++p)
            if (in(p)) store<VW>(py + at(p), v[p]);
    }
}

// Heads: L lanes hold a row of up to L * C columns, 32 / L neighbouring rows a warp.  No residual, no 8-bit result.
template <typename TX, typename TY, int L, int C, int VW>
__global__ void __launch_bounds__(256, 4) rms_norm_heads_kernel(const RmsArgs a) {
    constexpr int P = C / VW, XW = kWords<TX, VW>, R = 32 / L;
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int sub = (threadIdx.x & 31) / L, col0 = (threadIdx.x % L) * VW;
    auto at = [&](int p) { return col0 + p * L * VW; };
    auto in = [&](int p) { return at(p) < a.D; };
    const TX* x = reinterpret_cast<const TX*>(a.x);
    TY* y = reinterpret_cast<TY*>(a.y);
    const long long first = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * a.rows_per_team;
    const long long last = first + a.rows_per_team < a.M ? first + a.rows_per_team : a.M;
    const float inv_d = 1.f / (float)a.D;
    long long row = first + sub, tok = row / a.heads;
    int head = (int)(row % a.heads);
    const int step_tok = R / a.heads, step_head = R % a.heads;
    uint32_t nx[P][XW];
    auto fetch = [&](long long r, long long t, int h) {
#pragma unroll
        for (int p = 0; p < P; ++p) load<TX, VW>(x + t * a.x_tok + h * a.x_head + at(p), r < last && in(p), nx[p]);
    };
    fetch(row, tok, head);
    float w[P][VW];
#pragma unroll
    for (int p = 0; p < P; ++p)
#pragma unroll
        for (int e = 0; e < VW; ++e) w[p][e] = 1.f;
    long long group_end = a.weight ? 0 : a.M;
    for (long long base = first; base < last; base += R) {
        const bool live = row < last;                              // all lanes take part in the exchanges
        if (live && row >= group_end) {
            const long long g = row / a.rows_per_group;
            group_end = (g + 1) * a.rows_per_group;
#pragma unroll
            for (int p = 0; p < P; ++p) table<VW>(a.weight + g * a.mod_stride + at(p), in(p), a.unit, w[p]);
        }
        float v[P][VW], s = 0.f;
#pragma unroll
        for (int p = 0; p < P; ++p)
#pragma unroll
            for (int e = 0; e < VW; ++e) { v[p][e] = value<TX, VW>(nx[p], e); s = fmaf(v[p][e], v[p][e], s); }
        TY* py = y + tok * a.y_tok + head * a.y_head;
        const long long now = row;
        row += R; tok += step_tok; head += step_head;
        if (head >= a.heads) { head -= a.heads; ++tok; }
        fetch(row, tok, head);
#pragma unroll
        for (int o = L / 2; o > 0; o >>= 1) s += __shfl_xor_sync(~0u, s, o);
        const float r = rsqrtf(s * inv_d + a.eps);
        if (live) {
#pragma unroll
            for (int p = 0; p < P; ++p) {
#pragma unroll
                for (int e = 0; e < VW; ++e) v[p][e] = v[p][e] * r * w[p][e];
                if (in(p)) store<VW>(py + at(p), v[p]);
            }
            if (a.rstd && threadIdx.x % L == 0) a.rstd[now] = r;
        }
    }
}

template <typename TX, typename TR, typename TY, int P, int VW, bool FULL, int MAXT, int MINB>
int start(RmsArgs a, int warps, cudaStream_t s) {
    const int threads = warps > 1 ? warps * 32 : MAXT, teams = warps > 1 ? 1 : MAXT / 32;
    a.warps = warps;
    // one wave of the CTAs that the GPU holds at once; few rows: as many teams as there are rows
    const long long resident = (long long)kSms * (MINB * MAXT / threads) * teams;
    a.rows_per_team = (a.M + resident - 1) / resident;
    const long long grid = (a.M + a.rows_per_team * teams - 1) / (a.rows_per_team * teams);
    return free_launch(free_overlap_for_rows(a.M), rms_norm_kernel<TX, TR, TY, P, VW, FULL, MAXT, MINB>, dim3((unsigned)grid), dim3(threads), 0, s, a);
}
template <typename TX, typename TY, int L, int C, int VW> int start_heads(RmsArgs a, cudaStream_t s) {
    constexpr int R = 32 / L;
    const long long resident = (long long)kSms * 4 * 8;
    const long long steps = (a.M + resident * R - 1) / (resident * R);
    a.rows_per_team = steps * R;
    const long long grid = (a.M + a.rows_per_team * 8 - 1) / (a.rows_per_team * 8);
    return free_launch(free_overlap_for_rows(a.M), rms_norm_heads_kernel<TX, TY, L, C, VW>, dim3((unsigned)grid), dim3(256), 0, s, a);
}

// As many pieces per warp as the row needs (registers decide how many rows an SM holds), several warps beyond 1024 columns.  Whole pieces of 128
// columns, up to nine, have kernels of their own, without guards and the lanes behind the row's end (200 MB of bf16 rows of 640 columns
// onto fp32 ones: 208 us, in the kernel for up to 1024 columns 224; 8-bit results with a scale per run: 112 and 174).
template <typename TX, typename TR, typename TY, int P> int start_exact(const RmsArgs& a, cudaStream_t s) {
    return start<TX, TR, TY, P, 4, true, 128, P <= 2 ? 8 : P <= 4 ? 6 : P == 5 ? 5 : P <= 8 ? 4 : 3>(a, 1, s);
}
template <typename TX, typename TR, typename TY, int VW> int launch(const RmsArgs& a, cudaStream_t s) {
    if constexpr (sizeof(TY) > 1) {
        if (!a.res && a.D <= 128) {
            if (a.D <= 32) return start_heads<TX, TY, 4, 8, VW>(a, s);
            if (a.D <= 64) return start_heads<TX, TY, 8, 8, VW>(a, s);
            if constexpr (VW < 8)
                if (a.D <= 96) return start_heads<TX, TY, 8, 12, VW>(a, s);
            return start_heads<TX, TY, 8, 16, VW>(a, s);
        }
    }
    const int D = a.D;
    if constexpr (VW == 8) {
        if (D > 1024 && D % 1024 == 0) return start<TX, TR, TY, 4, 8, true, 256, 2>(a, D / 1024, s);
        if (D <= 256) return start<TX, TR, TY, 1, 8, false, 128, 8>(a, 1, s);
        if (D <= 512) return start<TX, TR, TY, 2, 8, false, 128, 6>(a, 1, s);
        if (D <= 1024) return start<TX, TR, TY, 4, 8, false, 128, 4>(a, 1, s);
        return start<TX, TR, TY, 4, 8, false, 256, 2>(a, (D + 1023) / 1024, s);
    } else if constexpr (VW == 4) {
        switch (D % 128 == 0 ? D / 128 : 0) {
            case 1: return start_exact<TX, TR, TY, 1>(a, s);
            case 2: return start_exact<TX, TR, TY, 2>(a, s);
            case 3: return start_exact<TX, TR, TY, 3>(a, s);
            case 4: return start_exact<TX, TR, TY, 4>(a, s);
            case 5: return start_exact<TX, TR, TY, 5>(a, s);
            case 6: return start_exact<TX, TR, TY, 6>(a, s);
            case 7: return start_exact<TX, TR, TY, 7>(a, s);
            case 8: return start_exact<TX, TR, TY, 8>(a, s);
            case 9: return start_exact<TX, TR, TY, 9>(a, s);
            default: break;
        }
        if (D > 1024 && D % 1024 == 0) return start<TX, TR, TY, 8, 4, true, 256, 2>(a, D / 1024, s);
        if (D <= 256) return start<TX, TR, TY, 2, 4, false, 128, 8>(a, 1, s);
        if (D <= 512) return start<TX, TR, TY, 4, 4, false, 128, 6>(a, 1, s);
        if (D <= 1024) return start<TX, TR, TY, 8, 4, false, 128, 4>(a, 1, s);
        return start<TX, TR, TY, 4, 4, false, 512, 1>(a, (D + 511) / 512, s);
    } else {
        if (D <= 256) return start<TX, TR, TY, 8, 1, false, 128, 8>(a, 1, s);
        return start<TX, TR, TY, 16, 1, false, 512, 1>(a, (D + 511) / 512, s);
    }
}
template <typename TX, typename TR> int launch_y(const RmsArgs& a, int vw, int y_dtype, cudaStream_t s) {
    using bf = __nv_bfloat16;
    if constexpr (sizeof(TX) == 2 && sizeof(TR) == 2)
        if (vw == 8) return y_dtype == FREE_BF16 ? launch<TX, TR, bf, 8>(a, s) : launch<TX, TR, e4m3, 8>(a, s);
    if (y_dtype == FREE_FP32) return vw == 4 ? launch<TX, TR, float, 4>(a, s) : launch<TX, TR, float, 1>(a, s);
    if (y_dtype == FREE_BF16) return vw == 4 ? launch<TX, TR, bf, 4>(a, s) : launch<TX, TR, bf, 1>(a, s);
    return vw == 4 ? launch<TX, TR, e4m3, 4>(a, s) : launch<TX, TR, e4m3, 1>(a, s);
}

}  // namespace rms
