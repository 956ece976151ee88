// Attention to an encoder's states on CUDA cores (fp32 arithmetic throughout): the exact mode, and bf16 inputs that the tensor
// cores' tile copies cannot take (rows that are not 16-byte aligned, odd head sizes).
//
//   forward   S = scale q k^T, p = e^(S - max), out = p v / sum p, lse = max + log sum p     one pass, running maximum and sum
//   dq        p = e^(S - lse), dS = p (g v^T - delta) scale, dq = dS k                        g: the gradient of out
//   dk, dv    dk = dS^T q, dv = p^T g, summed over the queries, heads and sequences that share the states (in parts, joined in order)
//
// Tiles of 64 x 64 scores, 256 threads.  Thread (ty, tx) forms the scores of rows 4 ty .. and columns tx, tx + 16, ..: both
// operands are read as four consecutive channels (16 bytes), eight reads for 64 multiply-adds; a row of a tile is d + 4 floats
// (rounded up), so that eight threads' reads lie in different banks.  Scores go through shared memory to be the left operand
// of the second product.  Bound by the fp32 pipe and shared memory's bandwidth; small calls by latency (3 x 333 tokens, 6 heads of 40,
// up to 77 states: 17 us).
// States that do not count are read as zeros and their scores are masked, so nothing in them reaches a result.
#include "cross.h"

namespace {

constexpr int T = 64, kThreads = 256, PS = T + 4;

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16(v); }

__host__ __device__ constexpr int pitch(int d) { return (d + 7) / 8 * 8 + 4; }

// rows [r0, r0 + T) of a matrix of heads -> shared memory; rows that are not `live` and channels behind d are zeros.  A warp's eight rows
// are under way together (one after the other, 3 x 333 tokens, 6 heads of 40 took 29 us).
template <typename E, typename Live>
__device__ __forceinline__ void load_tile(float* dst, const E* base, long long stride, int r0, int d, int P, Live live) {
    constexpr int WARPS = kThreads / 32, R = T / WARPS;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    bool ok[R];
#pragma unroll
    for (int i = 0; i < R; ++i) ok[i] = live(r0 + warp + i * WARPS);
    const E* src = base + (long long)(r0 + warp) * stride;
    for (int c = lane; c < P; c += 32) {
        E v[R];
#pragma unroll
        for (int i = 0; i < R; ++i) v[i] = ok[i] && c < d ? src[i * WARPS * stride + c] : E(0.f);
#pragma unroll
        for (int i = 0; i < R; ++i) dst[(warp + i * WARPS) * P + c] = to_f(v[i]);
    }
}

// s[r][k] = <A row 4 ty + r, B row tx + 16 k>
__device__ __forceinline__ void scores(const float* A, const float* B, int P, int ty, int tx, float (&s)[4][4]) {
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int k = 0; k < 4; ++k) s[r][k] = 0.f;
    for (int c = 0; c < P - 4; c += 4) {
        float4 a[4], b[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) a[r] = *reinterpret_cast<const float4*>(A + (4 * ty + r) * P + c);
#pragma unroll
        for (int k = 0; k < 4; ++k) b[k] = *reinterpret_cast<const float4*>(B + (tx + 16 * k) * P + c);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int k = 0; k < 4; ++k)
                s[r][k] = fmaf(a[r].x, b[k].x, fmaf(a[r].y, b[k].y, fmaf(a[r].z, b[k].z, fmaf(a[r].w, b[k].w, s[r][k]))));
    }
}
// acc[r][i] += sum over j of W[4 ty + r][j] * B[j][channel], channels 4 tx + 64 (i / 4) + i % 4
template <int ND> __device__ __forceinline__ void product(const float* W, const float* B, int P, int ty, int tx, float (&acc)[4][4 * ND]) {
    for (int j = 0; j < T; j += 4) {
        float4 w[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) w[r] = *reinterpret_cast<const float4*>(W + (4 * ty + r) * PS + j);
#pragma unroll
        for (int q = 0; q < ND; ++q) {
            if (ND > 1 && 4 * tx + 64 * q >= P - 4) break;
            const int c = ND == 1 ? min(4 * tx, P - 4) : 4 * tx + 64 * q;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const float4 b = *reinterpret_cast<const float4*>(B + (j + u) * P + c);
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const float x = u == 0 ? w[r].x : u == 1 ? w[r].y : u == 2 ? w[r].z : w[r].w;
                    acc[r][4 * q] = fmaf(x, b.x, acc[r][4 * q]);
                    acc[r][4 * q + 1] = fmaf(x, b.y, acc[r][4 * q + 1]);
                    acc[r][4 * q + 2] = fmaf(x, b.z, acc[r][4 * q + 2]);
                    acc[r][4 * q + 3] = fmaf(x, b.w, acc[r][4 * q + 3]);
                }
            }
        }
    }
}
template <typename E, int ND> __device__ __forceinline__ void store_rows(E* base, long long stride, int r0, int rows, int d, int ty, int tx, const float (&acc)[4][4 * ND]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = r0 + 4 * ty + r;
        if (row >= rows) continue;
#pragma unroll
        for (int q = 0; q < ND; ++q)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const int c = 4 * tx + 64 * q + u;
                if (c < d) from_f(base[(long long)row * stride + c], acc[r][4 * q + u]);
            }
    }
}
template <typename E> __device__ __forceinline__ void zero_rows(E* base, long long stride, int r0, int rows, int d) {
    for (int r = r0 + (int)(threadIdx.x >> 5); r < rows; r += kThreads / 32)
        for (int c = threadIdx.x & 31; c < d; c += 32) base[(long long)r * stride + c] = E(0.f);
}
template <typename E> __device__ __forceinline__ const E* at(const CrossMat& m, int s, long long row, int h) {
    return reinterpret_cast<const E*>(m.p) + s * m.seq + row * m.tok + h * m.head;
}
template <typename E> __device__ __forceinline__ E* at_out(const CrossMat& m, int s, long long row, int h) { return const_cast<E*>(at<E>(m, s, row, h)); }

__device__ __forceinline__ float row_max(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
    return v;
}
__device__ __forceinline__ float row_sum(float v) {
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
    return v;
}

template <typename E, int ND> __global__ void __launch_bounds__(kThreads) cross_simt_kernel(const CrossArgs a) {
    extern __shared__ float smem[];
    const int d = a.d, P = pitch(d);
    float *Q = smem, *K = Q + T * P, *V = K + T * P, *W = V + T * P;
    const int tiles = (a.n_q + T - 1) / T;
    const int tile = (int)(blockIdx.x % tiles), sh = (int)(blockIdx.x / tiles), h = sh % a.heads, s = sh / a.heads, kh = h / a.group;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, q0 = tile * T;
    const CrossSpan sp = cross_span(a.where, s);
    const uint8_t* mask = cross_mask(a.where, sp);
    auto counts = [&](int j) { return j < sp.len && (!mask || mask[j]); };
    load_tile<E>(Q, at<E>(a.q, s, 0, h), a.q.tok, q0, d, P, [&](int r) { return r < a.n_q; });
    const E *kb = at<E>(a.k, sp.enc, sp.row0, kh), *vb = at<E>(a.v, sp.enc, sp.row0, kh);
    float acc[4][4 * ND], top[4], sum[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        top[r] = -INFINITY; sum[r] = 0.f;
#pragma unroll
        for (int i = 0; i < 4 * ND; ++i) acc[r][i] = 0.f;
    }
    for (int j0 = 0; j0 < sp.len; j0 += T) {
        __syncthreads();
        load_tile<E>(K, kb, a.k.tok, j0, d, P, counts);
        load_tile<E>(V, vb, a.v.tok, j0, d, P, counts);
        __syncthreads();
        float sc[4][4];
        scores(Q, K, P, ty, tx, sc);
        bool ok[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) ok[k] = counts(j0 + tx + 16 * k);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            float m = -INFINITY;
#pragma unroll
            for (int k = 0; k < 4; ++k) { sc[r][k] = ok[k] ? sc[r][k] * a.scale : -INFINITY; m = fmaxf(m, sc[r][k]); }
            m = fmaxf(top[r], row_max(m));
            const float base = m == -INFINITY ? 0.f : m;           // no state so far
            const float alpha = expf(top[r] - base);
            float part = 0.f;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float p = expf(sc[r][k] - base);
                part += p;
                W[(4 * ty + r) * PS + tx + 16 * k] = p;
            }
            sum[r] = sum[r] * alpha + row_sum(part);
            top[r] = m;
#pragma unroll
            for (int i = 0; i < 4 * ND; ++i) acc[r][i] *= alpha;
        }
        __syncwarp();                                              // a row of W is written and read by one half of a warp
        product<ND>(W, V, P, ty, tx, acc);
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const float inv = sum[r] == 0.f ? 0.f : 1.f / sum[r];
#pragma unroll
        for (int i = 0; i < 4 * ND; ++i) acc[r][i] *= inv;
        const int row = q0 + 4 * ty + r;
        if (a.lse && tx == 0 && row < a.n_q) a.lse[((long long)s * a.heads + h) * a.n_q + row] = top[r] + logf(sum[r]);      // no state: both -inf
    }
    store_rows<E, ND>(at_out<E>(a.o, s, 0, h), a.o.tok, q0, a.n_q, d, ty, tx, acc);
}

// delta = <dout, out> of every token and head.  L lanes hold a row, V consecutive channels each (16 bytes, or 1 element where the rows
// allow no more), R rows of a group of lanes are in flight.  Rows are counted on, not divided out.  (24 x 1024 tokens, 16 heads of 72: 42 us,
// nine of sixteen lanes busy; the kernel for matrices without gaps 23, 4.9 TB/s.)
template <typename E, int V> struct Chunk {
    E v[V];
    __device__ __forceinline__ void load(const E* p, bool ok) {
        if constexpr (V == 1) {
            v[0] = ok ? *p : E(0.f);
        } else {
            const uint4 u = ok ? __ldg(reinterpret_cast<const uint4*>(p)) : make_uint4(0u, 0u, 0u, 0u);
            *reinterpret_cast<uint4*>(v) = u;
        }
    }
};
template <typename E, int V, int L> __global__ void __launch_bounds__(256) cross_delta_kernel(const CrossArgs a) {
    constexpr int R = V == 1 ? 1 : 4, P = V == 1 ? kCrossMaxD / L : 1;        // pieces of a lane
    free_grid_dep_wait();
    free_grid_dep_launch();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.next = 0;
    const long long rows = (long long)a.n_seq * a.n_q * a.heads;
    const int lane = threadIdx.x % L, groups = (int)(gridDim.x * (256 / L)), step_h = groups % a.heads;
    const int step_t = groups / a.heads % a.n_q, step_s = groups / a.heads / a.n_q;
    long long i = (long long)blockIdx.x * (256 / L) + threadIdx.x / L;
    int h = (int)(i % a.heads), t, s;
    { const long long st = i / a.heads; t = (int)(st % a.n_q); s = (int)(st / a.n_q); }
    // whole groups of lanes leave together, so the exchanges name the group's lanes only
    const unsigned mates = L == 32 ? 0xffffffffu : ((1u << L) - 1u) << ((threadIdx.x & 31) / L * L);
    while (i < rows) {
        Chunk<E, V> g[R][P], o[R][P];
        long long out[R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bool ok = i < rows;
            const E *pg = at<E>(a.g, s, t, h) + lane * V, *po = at<E>(a.o, s, t, h) + lane * V;
#pragma unroll
            for (int p = 0; p < P; ++p) {
                g[r][p].load(pg + p * L * V, ok && lane * V + p * L * V < a.d);
                o[r][p].load(po + p * L * V, ok && lane * V + p * L * V < a.d);
            }
            out[r] = ok ? ((long long)s * a.heads + h) * a.n_q + t : -1;
            i += groups; h += step_h; t += step_t; s += step_s;
            if (h >= a.heads) { h -= a.heads; ++t; }
            if (t >= a.n_q) { t -= a.n_q; ++s; }
        }
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float v = 0.f;
#pragma unroll
            for (int p = 0; p < P; ++p)
#pragma unroll
                for (int e = 0; e < V; ++e) v = fmaf(to_f(g[r][p].v[e]), to_f(o[r][p].v[e]), v);
#pragma unroll
            for (int k = L / 2; k > 0; k >>= 1) v += __shfl_xor_sync(mates, v, k);
            if (lane == 0 && out[r] >= 0) a.delta[out[r]] = v;
        }
    }
}

// The same of matrices without gaps: a warp takes 32 rows and reads their pieces of 16 bytes in the order of memory; the pieces' sums meet
// in shared memory, where each lane adds those of a row.
template <typename E, int L> __global__ void __launch_bounds__(256) cross_delta_dense_kernel(const CrossArgs a) {
    constexpr int V = 16 / (int)sizeof(E);
    __shared__ float part[8][32 * (L + 1)];
    free_grid_dep_wait();
    free_grid_dep_launch();
    if (blockIdx.x == 0 && threadIdx.x == 0) *a.next = 0;
    const int lane = threadIdx.x & 31, units = a.d / V, pitch = units | 1, magic = (65535 + units) / units;
    const long long rows = (long long)a.n_seq * a.n_q * a.heads;
    float* mine = part[threadIdx.x >> 5];
    for (long long i0 = ((long long)blockIdx.x * 8 + (threadIdx.x >> 5)) * 32; i0 < rows; i0 += (long long)gridDim.x * 256) {
        const E *g = static_cast<const E*>(a.g.p) + i0 * a.d, *o = static_cast<const E*>(a.o.p) + i0 * a.d;
        const int n = (int)(rows - i0 < 32 ? rows - i0 : 32) * units;
#pragma unroll 4
        for (int x = lane; x < 32 * units; x += 32) {
            Chunk<E, V> cg, co;
            cg.load(g + (long long)x * V, x < n);
            co.load(o + (long long)x * V, x < n);
            float v = 0.f;
#pragma unroll
            for (int e = 0; e < V; ++e) v = fmaf(to_f(cg.v[e]), to_f(co.v[e]), v);
            const int row = x * magic >> 16;
            mine[row * pitch + x - row * units] = v;
        }
        __syncwarp();
        float t[L];                                                // added in the order of the kernel above: the same sums
#pragma unroll
        for (int u = 0; u < L; ++u) t[u] = u < units ? mine[lane * pitch + u] : 0.f;
#pragma unroll
        for (int k = L / 2; k > 0; k >>= 1)
#pragma unroll
            for (int u = 0; u < k; ++u) t[u] += t[u + k];
        __syncwarp();
        const long long i = i0 + lane;
        if (i < rows) {
            const int h = (int)(i % a.heads);
            const long long st = i / a.heads;
            a.delta[(st / a.n_q * a.heads + h) * a.n_q + st % a.n_q] = t[0];
        }
    }
}

template <typename E, int ND> __global__ void __launch_bounds__(kThreads) cross_simt_dq_kernel(const CrossArgs a) {
    extern __shared__ float smem[];
    const int d = a.d, P = pitch(d);
    float *Q = smem, *G = Q + T * P, *K = G + T * P, *V = K + T * P, *W = V + T * P;
    const int tiles = (a.n_q + T - 1) / T;
    const int tile = (int)(blockIdx.x % tiles), sh = (int)(blockIdx.x / tiles), h = sh % a.heads, s = sh / a.heads, kh = h / a.group;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, q0 = tile * T;
    const CrossSpan sp = cross_span(a.where, s);
    const uint8_t* mask = cross_mask(a.where, sp);
    auto counts = [&](int j) { return j < sp.len && (!mask || mask[j]); };
    auto live = [&](int r) { return r < a.n_q; };
    load_tile<E>(Q, at<E>(a.q, s, 0, h), a.q.tok, q0, d, P, live);
    load_tile<E>(G, at<E>(a.g, s, 0, h), a.g.tok, q0, d, P, live);
    const E *kb = at<E>(a.k, sp.enc, sp.row0, kh), *vb = at<E>(a.v, sp.enc, sp.row0, kh);
    float acc[4][4 * ND], lse[4], delta[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const int row = q0 + 4 * ty + r;
        const long long i = ((long long)s * a.heads + h) * a.n_q + row;
        lse[r] = row < a.n_q ? a.lse[i] : 0.f;
        delta[r] = row < a.n_q ? a.delta[i] : 0.f;
#pragma unroll
        for (int k = 0; k < 4 * ND; ++k) acc[r][k] = 0.f;
    }
    for (int j0 = 0; j0 < sp.len; j0 += T) {
        __syncthreads();
        load_tile<E>(K, kb, a.k.tok, j0, d, P, counts);
        load_tile<E>(V, vb, a.v.tok, j0, d, P, counts);
        __syncthreads();
        float sc[4][4], dp[4][4];
        scores(Q, K, P, ty, tx, sc);
        scores(G, V, P, ty, tx, dp);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const bool ok = counts(j0 + tx + 16 * k);
#pragma unroll
            for (int r = 0; r < 4; ++r)
                W[(4 * ty + r) * PS + tx + 16 * k] = ok ? expf(sc[r][k] * a.scale - lse[r]) * (dp[r][k] - delta[r]) * a.scale : 0.f;
        }
        __syncwarp();
        product<ND>(W, K, P, ty, tx, acc);
    }
    store_rows<E, ND>(at_out<E>(a.dq, s, 0, h), a.dq.tok, q0, a.n_q, d, ty, tx, acc);
}

// A CTA per (64 states, key head, encoder sequence, part); it walks over its part of the tiles of tokens: of every sequence that reads the
// states, in order, the query heads of the key head and 64 tokens.
// PACKED: blocks may be counted by the rows, and a sequence's last may have rows behind it to write (2.4% of 2.9 ms where there are none).
template <typename E, int ND, bool PACKED> __global__ void __launch_bounds__(kThreads) cross_simt_dkv_kernel(const CrossArgs a, int blocks, int parts, float* part_out) {
    extern __shared__ float smem[];
    const int d = a.d, P = pitch(d);
    float *K = smem, *V = K + T * P, *Q = V + T * P, *G = Q + T * P, *W = G + T * P, *L = W + T * PS, *D = L + T;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, part = (int)(blockIdx.x % parts);
    const CrossBlock block = PACKED && !blocks ? cross_block<T, true>(a.where, a.kv_heads, 0, blockIdx.x / parts) : cross_block<T, false>(a.where, a.kv_heads, blocks, blockIdx.x / parts);
    if (PACKED && block.row0 < 0) return;
    const int kh = block.head, e = block.e, j0 = block.row0;
    const CrossSpan sp = cross_span_of_enc(a.where, e);
    const int rows = !PACKED || block.last || sp.rows - j0 < T ? sp.rows : j0 + T;      // that are written up to
    if (j0 >= rows) return;
    const uint8_t* mask = cross_mask(a.where, sp);
    auto counts = [&](int j) { return j < sp.len && (!mask || mask[j]); };
    load_tile<E>(K, at<E>(a.k, sp.enc, sp.row0, kh), a.k.tok, j0, d, P, counts);
    load_tile<E>(V, at<E>(a.v, sp.enc, sp.row0, kh), a.v.tok, j0, d, P, counts);
    float dk[4][4 * ND], dv[4][4 * ND];
#pragma unroll
    for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int i = 0; i < 4 * ND; ++i) dk[r][i] = dv[r][i] = 0.f;
    bool ok[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) ok[r] = counts(j0 + 4 * ty + r);
    const int first = a.where.seq_of ? 0 : e * a.where.share, last = a.where.seq_of || first + a.where.share > a.n_seq ? a.n_seq : first + a.where.share;
    const long long per = (long long)a.group * ((a.n_q + T - 1) / T);           // tiles of a sequence
    long long lo = 0, hi = per * (last - first), at_tile = 0;
    if (parts > 1) {
        if (a.where.seq_of) {
            int n = 0;
            for (int s = 0; s < a.n_seq; s += kThreads) n += __syncthreads_count(s + (int)threadIdx.x < a.n_seq && cross_enc_of(a.where, s + threadIdx.x) == e);
            hi = per * n;
        }
        lo = hi * part / parts;
        hi = hi * (part + 1) / parts;
    }
    for (int s = first; s < last && j0 < sp.len && at_tile < hi; ++s) {
        if (cross_enc_of(a.where, s) != e) continue;
        if (at_tile + per <= lo) { at_tile += per; continue; }
        for (int h = kh * a.group; h < (kh + 1) * a.group; ++h)
            for (int q0 = 0; q0 < a.n_q; q0 += T, ++at_tile) {
                if (at_tile < lo || at_tile >= hi) continue;
                __syncthreads();
                auto live = [&](int r) { return r < a.n_q; };
                load_tile<E>(Q, at<E>(a.q, s, 0, h), a.q.tok, q0, d, P, live);
                load_tile<E>(G, at<E>(a.g, s, 0, h), a.g.tok, q0, d, P, live);
                if (threadIdx.x < T) {
                    const int row = q0 + threadIdx.x;
                    const long long i = ((long long)s * a.heads + h) * a.n_q + row;
                    L[threadIdx.x] = row < a.n_q ? a.lse[i] : INFINITY;      // rows behind the last: p = 0
                    D[threadIdx.x] = row < a.n_q ? a.delta[i] : 0.f;
                }
                __syncthreads();
                float sc[4][4], dp[4][4];
                scores(K, Q, P, ty, tx, sc);
                scores(V, G, P, ty, tx, dp);
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const int t = tx + 16 * k;
                        sc[r][k] = ok[r] ? expf(sc[r][k] * a.scale - L[t]) : 0.f;
                        dp[r][k] = ok[r] ? sc[r][k] * (dp[r][k] - D[t]) * a.scale : 0.f;
                        W[(4 * ty + r) * PS + t] = sc[r][k];
                    }
                __syncwarp();
                product<ND>(W, G, P, ty, tx, dv);
                __syncwarp();
#pragma unroll
                for (int r = 0; r < 4; ++r)
#pragma unroll
                    for (int k = 0; k < 4; ++k) W[(4 * ty + r) * PS + tx + 16 * k] = dp[r][k];
                __syncwarp();
                product<ND>(W, Q, P, ty, tx, dk);
            }
    }
#pragma unroll
    for (int r = 0; r < 4; ++r)
        if (!ok[r]) {                                              // whatever dout and q hold
#pragma unroll
            for (int i = 0; i < 4 * ND; ++i) dk[r][i] = dv[r][i] = 0.f;
        }
    if (parts > 1) {
        const long long all = (long long)(a.where.offsets ? 1 : a.where.n_enc) * a.where.kv_rows * a.kv_heads * d, step = (long long)a.kv_heads * d;
        float* out = part_out + 2 * part * all + (((long long)sp.enc * a.where.kv_rows + sp.row0) * a.kv_heads + kh) * d;
        store_rows<float, ND>(out, step, j0, rows, d, ty, tx, dk);
        store_rows<float, ND>(out + all, step, j0, rows, d, ty, tx, dv);
        if (PACKED) {
            zero_rows(out, step, j0 + T, rows, d);
            zero_rows(out + all, step, j0 + T, rows, d);
        }
        return;
    }
    store_rows<E, ND>(at_out<E>(a.dk, sp.enc, sp.row0, kh), a.dk.tok, j0, rows, d, ty, tx, dk);
    store_rows<E, ND>(at_out<E>(a.dv, sp.enc, sp.row0, kh), a.dv.tok, j0, rows, d, ty, tx, dv);
    if (PACKED) {
        zero_rows(at_out<E>(a.dk, sp.enc, sp.row0, kh), a.dk.tok, j0 + T, rows, d);
        zero_rows(at_out<E>(a.dv, sp.enc, sp.row0, kh), a.dv.tok, j0 + T, rows, d);
    }
}

template <typename K, typename... A> int launch(K kernel, long long ctas, int tiles_held, int extra, cudaStream_t s, const CrossArgs& a, A... rest) {
    if (ctas > 0x7fffffffLL) return FREE_ERR_SHAPE;
    auto bytes = [&](int d) { return (tiles_held * T * pitch(d) + T * PS + extra) * (int)sizeof(float); };
    const int smem = bytes(a.d);
    // the most that the kernel takes: another thread's smaller call must not set it below this one's
    FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes(a.d <= 64 ? 64 : kCrossMaxD)));
    kernel<<<(unsigned)ctas, kThreads, smem, s>>>(a, rest...);
    return free_check_launch();
}
long long q_tiles(const CrossArgs& a) { return (long long)((a.n_q + T - 1) / T) * a.n_seq * a.heads; }

}  // namespace

int cross_simt_forward(int dtype, const CrossArgs& a, cudaStream_t s) {
    if (dtype == FREE_FP32) return a.d <= 64 ? launch(cross_simt_kernel<float, 1>, q_tiles(a), 3, 0, s, a) : launch(cross_simt_kernel<float, 2>, q_tiles(a), 3, 0, s, a);
    return a.d <= 64 ? launch(cross_simt_kernel<__nv_bfloat16, 1>, q_tiles(a), 3, 0, s, a) : launch(cross_simt_kernel<__nv_bfloat16, 2>, q_tiles(a), 3, 0, s, a);
}
namespace {

template <typename E, int V, int L> int start_delta(const CrossArgs& a, cudaStream_t s) {
    const long long rows = (long long)a.n_seq * a.n_q * a.heads, ctas = (rows + 256 / L - 1) / (256 / L);
    return free_launch(free_overlap_for_rows((long long)a.n_seq * a.n_q), cross_delta_kernel<E, V, L>, dim3((unsigned)(ctas < 148 * 8 ? ctas : 148 * 8)), dim3(256), 0, s, a);
}
template <typename E> int delta_of(const CrossArgs& a, cudaStream_t s) {
    constexpr int V = 16 / (int)sizeof(E);
    bool wide = a.d % V == 0;
    for (const CrossMat* m : {&a.g, &a.o}) wide = wide && free_aligned16(m->p) && m->seq % V == 0 && m->tok % V == 0 && m->head % V == 0;
    if (!wide) return start_delta<E, 1, 32>(a, s);
    const int units = a.d / V;
    bool dense = true;
    for (const CrossMat* m : {&a.g, &a.o})
        dense = dense && (a.heads == 1 || m->head == a.d) && (a.n_q == 1 || m->tok == (long long)a.heads * a.d) && (a.n_seq == 1 || m->seq == (long long)a.n_q * a.heads * a.d);
    if (dense) {
        const long long ctas = ((long long)a.n_seq * a.n_q * a.heads + 255) / 256;
        auto kernel = units <= 8 ? cross_delta_dense_kernel<E, 8> : units <= 16 ? cross_delta_dense_kernel<E, 16> : cross_delta_dense_kernel<E, 32>;
        return free_launch(free_overlap_for_rows((long long)a.n_seq * a.n_q), kernel, dim3((unsigned)(ctas < 148 * 6 ? ctas : 148 * 6)), dim3(256), 0, s, a);
    }
    return units <= 8 ? start_delta<E, V, 8>(a, s) : units <= 16 ? start_delta<E, V, 16>(a, s) : start_delta<E, V, 32>(a, s);
}

}  // namespace

int cross_delta(int dtype, const CrossArgs& a, cudaStream_t s) { return dtype == FREE_FP32 ? delta_of<float>(a, s) : delta_of<__nv_bfloat16>(a, s); }
int cross_simt_dq(int dtype, const CrossArgs& a, cudaStream_t s) {
    if (dtype == FREE_FP32) return a.d <= 64 ? launch(cross_simt_dq_kernel<float, 1>, q_tiles(a), 4, 0, s, a) : launch(cross_simt_dq_kernel<float, 2>, q_tiles(a), 4, 0, s, a);
    return a.d <= 64 ? launch(cross_simt_dq_kernel<__nv_bfloat16, 1>, q_tiles(a), 4, 0, s, a) : launch(cross_simt_dq_kernel<__nv_bfloat16, 2>, q_tiles(a), 4, 0, s, a);
}

// Parts of the tokens where the blocks of states leave SMs without one (all gradients of 2 x 512 tokens, 8 heads of 64, 300 states: 158 ->
// 139 us; of 3 x 333 tokens, 77 states, 6 heads of 40: 84 -> 52)
int cross_simt_dkv_parts(const CrossArgs& a) {
    const long long items = cross_blocks(a.where, T) * a.kv_heads, tiles = (long long)a.n_seq * a.group * ((a.n_q + T - 1) / T) / (a.where.n_enc > 0 ? a.where.n_enc : 1);
    if (items < 1 || items >= 2 * 148) return 1;
    long long p = (3 * 148 + items - 1) / items;
    if (p > tiles) p = tiles;
    if (p > cross_parts_held(a)) p = cross_parts_held(a);
    return p < 1 ? 1 : (int)p;
}
namespace {
template <bool PACKED> auto dkv_kernel(int dtype, int d) {
    const bool slim = d <= 64;
    return dtype == FREE_FP32 ? slim ? cross_simt_dkv_kernel<float, 1, PACKED> : cross_simt_dkv_kernel<float, 2, PACKED>
                              : slim ? cross_simt_dkv_kernel<__nv_bfloat16, 1, PACKED> : cross_simt_dkv_kernel<__nv_bfloat16, 2, PACKED>;
}
}  // namespace
int cross_simt_dkv(int dtype, const CrossArgs& a, int parts, float* part_out, cudaStream_t s) {
    const long long n = cross_blocks(a.where, T) * a.kv_heads * parts;
    FREE_TRY(launch(a.where.offsets ? dkv_kernel<true>(dtype, a.d) : dkv_kernel<false>(dtype, a.d), n, 4, 2 * T, s, a, cross_blocks_per(a.where, T), parts, part_out));
    return parts > 1 ? cross_bwd_join(dtype, a, parts, part_out, s) : FREE_OK;
}
