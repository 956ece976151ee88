// Rotary positions with several axes: every pair (a, b) of a head is turned by an angle that grows with the token's
// position on the pair's axis,
//   t = pos[axis(pair)] * freq(pair),   (a, b) -> (a cos t - b sin t, a sin t + b cos t);   inverse: -t (also the backward pass).
//
// Bound by HBM (each element is read and written once; 3 FLOPs).  The angle of a far position needs more than fp32: it is
// formed in turns, t / 2 pi, as one fp64 product, reduced to [-1/2, 1/2] there, and only the remainder goes to fp32
// sincospif.  All heads of a token share its angles, and so do the sequences that share positions: a CTA takes a few tokens of
// a run of sequences, fills a table [tokens][pairs] of (cos, sin) in shared memory once while its first loads are in flight, and
// streams the heads through it.  A thread keeps one slot (one vector of a head, or the two that it couples), so that the index
// arithmetic is done once, and has kUnroll tokens' loads in flight.  The frequencies are formed on the host in fp64 and travel
// as a kernel argument.
// Measured on B200: 41 us in a replayed graph, 43 as calls on new inputs, for the 113 MB of queries and keys of 24 x 1024 tokens,
// 16 heads of 72, bf16 (5.5 and 5.3 TB/s read and written; in place 44), 73 us for the same in fp32 (6.2 TB/s).
#include "internal.h"
#include <math.h>

namespace {

constexpr int kMaxPairs = 128;                     // rotated pairs of a head
constexpr int kMaxAxes = 4;
constexpr int kThreads = 512;                     // most threads of a CTA
constexpr int kTableBytes = 16384;                 // (cos, sin) entries of a CTA
// Tokens that a thread has in flight.
// (A bf16 slot of two halves is up to eight pairs: more of those cost registers, 23 instead of 20 us for four on 8 x 4096 tokens of
// 12 heads of 64.  Narrower slots take four: 16 heads of 72 on 24 x 1024 tokens 22.7 us, one 30.8.)
template <typename T, int V, bool HALVES> constexpr int kUnroll = HALVES && sizeof(T) == 2 && V > 4 ? 1 : 4;
constexpr int kSms = 148;

struct RopeArgs {
    int n_seq, n_tok, n_axes, pairs;               // pairs: rotated pairs of a head
    int heads, d_head;
    int slots_per_head, slots;                     // slots: slots_per_head * heads
    int width, lanes_tok;                          // a CTA's threads: width slots side by side, for lanes_tok tokens at a time
    int passes;                                    // runs of `width` slots that cover a token
    int tok_per_cta, seq_per_cta;
    const float* pos; long long pos_seq_stride;
    const void* x; long long xs, xt, xh;           // strides of sequence, token, head in elements
    void* y; long long ys, yt, yh;
    float sign;
    double turns[kMaxPairs];                       // angle per unit of position, in turns
    unsigned char axis[kMaxPairs];
};

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };

// V elements of a head.  bf16 pairs stay packed in 32-bit words: one shift or mask to unpack, one conversion to pack two.
template <typename T, int V> struct Vec;
template <int V> struct Vec<float, V> {
    Pack<float, V> d;
    __device__ __forceinline__ void get2(int i, float& a, float& b) const { a = d.v[2 * i]; b = d.v[2 * i + 1]; }
    __device__ __forceinline__ void set2(int i, float a, float b) { d.v[2 * i] = a; d.v[2 * i + 1] = b; }
};
template <int V> struct Vec<__nv_bfloat16, V> {
    Pack<uint32_t, V / 2> d;
    __device__ __forceinline__ void get2(int i, float& a, float& b) const {
        a = __uint_as_float(d.v[i] << 16); b = __uint_as_float(d.v[i] & 0xffff0000u);
    }
    __device__ __forceinline__ void set2(int i, float a, float b) {
        const __nv_bfloat162 r = __floats2bfloat162_rn(a, b);
        d.v[i] = *reinterpret_cast<const uint32_t*>(&r);
    }
};
// one element (halves of an odd number of pairs)
template <> struct Vec<float, 1> {
    Pack<float, 1> d;
    __device__ __forceinline__ void get2(int, float& a, float& b) const { a = d.v[0]; b = 0.f; }
    __device__ __forceinline__ void set2(int, float a, float) { d.v[0] = a; }
};
template <> struct Vec<__nv_bfloat16, 1> {
    Pack<__nv_bfloat16, 1> d;
    __device__ __forceinline__ void get2(int, float& a, float& b) const { a = __bfloat162float(d.v[0]); b = 0.f; }
    __device__ __forceinline__ void set2(int, float a, float) { d.v[0] = __float2bfloat16(a); }
};
// as one access, or (ALIGNED false) element by element
template <typename T, int V, bool ALIGNED> __device__ __forceinline__ Vec<T, V> get(const T* p) {
    Vec<T, V> r;
    using D = decltype(r.d);
    if (ALIGNED) r.d = *reinterpret_cast<const D*>(p);
    else {
        Pack<T, V> e;
#pragma unroll
        for (int i = 0; i < V; ++i) e.v[i] = p[i];
        r.d = *reinterpret_cast<const D*>(&e);
    }
    return r;
}
template <typename T, int V, bool ALIGNED> __device__ __forceinline__ void put(T* p, const Vec<T, V>& r) {
    if (ALIGNED) *reinterpret_cast<decltype(r.d)*>(p) = r.d;
    else {
        const Pack<T, V> e = *reinterpret_cast<const Pack<T, V>*>(&r.d);
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = e.v[i];
    }
}

// One pair turned by (cos, sin).
__device__ __forceinline__ void turn(float& a, float& b, float cs, float sn) {
    const float p = a, q = b;
    a = p * cs - q * sn;
    b = p * sn + q * cs;
}
// The pairs of a slot, their (cos, sin) two by two in f[0], f[plane], ...  PART: only the first `pairs`, the elements behind
// stay as they are (bit for bit).
template <typename T, int V, bool HALVES, bool PART>
__device__ __forceinline__ void rotate(Vec<T, V>& u, Vec<T, V>& w, const float4* f, int plane, int pairs) {
    constexpr int PV = HALVES ? V : V / 2;
#pragma unroll
    for (int q = 0; q < (PV + 1) / 2; ++q) {
        const float4 c = f[q * plane];
        float a0, a1, b0, b1;
        if (HALVES) {                                              // pairs (u0, w0), (u1, w1)
            u.get2(q, a0, a1); w.get2(q, b0, b1);
            turn(a0, b0, c.x, c.y); turn(a1, b1, c.z, c.w);
            u.set2(q, a0, a1); w.set2(q, b0, b1);
        } else {                                                   // pairs (u0, u1), (u2, u3)
            if (!PART || 2 * q < pairs) { u.get2(2 * q, a0, b0); turn(a0, b0, c.x, c.y); u.set2(2 * q, a0, b0); }
            if (2 * q + 1 < PV && (!PART || 2 * q + 1 < pairs)) { u.get2((2 * q + 1) % (V / 2), a1, b1); turn(a1, b1, c.z, c.w); u.set2((2 * q + 1) % (V / 2), a1, b1); }
        }
    }
}

// HALVES false: a slot is V consecutive elements (V / 2 pairs (2i, 2i + 1)); elements past the rotated ones are copied.
// HALVES true: pair i couples elements i and i + pairs; a slot is V elements of the first half with their partners, or V
// elements behind both halves, which are copied.
template <typename T, int V, bool HALVES, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) rope_axes_kernel(const __grid_constant__ RopeArgs a) {
    constexpr int U = kUnroll<T, V, HALVES>;
    // Pairs of a slot: PV.  They lie in planes of two, [plane][token][slot group], so that a warp's 16-byte reads are one run
    // (with a slot's pairs side by side they would be 32 bytes apart and meet in the same banks: 61 against 44 us for the
    // queries and keys of 24 x 1024 tokens, 16 heads of 72, both in an older form that unpacked its words; this one takes 41).
    constexpr int PV = HALVES ? V : V / 2;
    __shared__ float4 table[kTableBytes / 16];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int P = a.pairs, G = (P + PV - 1) / PV, plane = a.tok_per_cta * G;
    const int t0 = blockIdx.x * a.tok_per_cta, n = a.n_tok - t0 < a.tok_per_cta ? a.n_tok - t0 : a.tok_per_cta;
    const int s0 = blockIdx.y * a.seq_per_cta, s1 = a.n_seq - s0 < a.seq_per_cta ? a.n_seq : s0 + a.seq_per_cta;
    const int lt = threadIdx.x / a.width, lane = threadIdx.x - lt * a.width;
    const long long xstep = a.lanes_tok * a.xt, ystep = a.lanes_tok * a.yt;
    for (int s = s0; s < s1; ++s) {
        const bool fill = s == s0 || a.pos_seq_stride != 0;        // sequences that share positions share the table
        for (int pass = 0; pass < a.passes; ++pass) {
            const int slot = pass * a.width + lane;
            const bool live = lt < a.lanes_tok && lt < n && slot < a.slots;
            const int h = slot / a.slots_per_head, j = slot - h * a.slots_per_head;
            const int pair0 = j * PV;                              // first pair of the slot
            const bool turned = pair0 < P;
            const int col = HALVES && !turned ? pair0 + P : HALVES ? pair0 : j * V;
            Vec<T, V> u[U], w[U];
            if (live) {
                const T* q = reinterpret_cast<const T*>(a.x) + s * a.xs + (t0 + lt) * a.xt + h * a.xh + col;
#pragma unroll
                for (int k = 0; k < U; ++k) {
                    u[k] = get<T, V, ALIGNED>(q);
                    if (HALVES && turned) w[k] = get<T, V, ALIGNED>(q + P);
                    if (lt + (k + 1) * a.lanes_tok < n) q += xstep;   // past the last token: the last one again, not stored
                }
            }
            if (fill && pass == 0) {                               // while the first loads are in flight
                if (s > s0) __syncthreads();
                const float* pos = a.pos + s * a.pos_seq_stride + (long long)t0 * a.n_axes;
                // a thread keeps its pair: lanes that each read another kernel argument wait for one another (32768 tokens of eight
                // heads of 128, bf16: 30 us, 44 with a pair looked up for every angle; 131072 of one head 33, 132)
                const int wide = P < (int)blockDim.x ? P : (int)blockDim.x, side = blockDim.x / wide, first = threadIdx.x / wide;
                for (int p = threadIdx.x - first * wide; first < side && p < P; p += wide) {
                    const double freq = a.turns[p];
                    const float* at = pos + a.axis[p];
                    const int r = p % PV;
                    float2* to = reinterpret_cast<float2*>(table + r / 2 * plane + p / PV) + (r & 1);
                    for (int k = first; k < n; k += side) {
                        double turns = (double)at[k * a.n_axes] * freq;
                        turns -= rint(turns);
                        float cs, sn;
                        sincospif((float)(turns + turns), &sn, &cs);
                        to[2 * k * G] = make_float2(cs, a.sign * sn);
                    }
                }
                __syncthreads();
            }
            if (!live) continue;
            T* q = reinterpret_cast<T*>(a.y) + s * a.ys + (t0 + lt) * a.yt + h * a.yh + col;
            const float4* f = table + lt * G + j;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                if (lt + k * a.lanes_tok >= n) break;
                if (pair0 + PV <= P) rotate<T, V, HALVES, false>(u[k], w[k], f, plane, PV);
                else if (turned) rotate<T, V, HALVES, true>(u[k], w[k], f, plane, P - pair0);
                if (HALVES && turned) put<T, V, ALIGNED>(q + P, w[k]);
                put<T, V, ALIGNED>(q, u[k]);
                q += ystep;
                f += a.lanes_tok * G;
            }
        }
    }
}

template <typename T, int V, bool HALVES, bool ALIGNED>
int launch(RopeArgs& a, cudaStream_t s) {
    a.slots_per_head = HALVES ? (a.d_head - a.pairs) / V : a.d_head / V;
    const long long slots = (long long)a.slots_per_head * a.heads;
    if (slots > (1 << 24)) return FREE_ERR_UNSUPPORTED;
    a.slots = (int)slots;
    // a token with few slots shares the CTA with others; one with many takes equal passes of at most kThreads slots
    a.passes = (a.slots + kThreads - 1) / kThreads;
    a.width = (a.slots + a.passes - 1) / a.passes;
    a.lanes_tok = a.width >= 256 ? 1 : 256 / a.width;
    if (a.lanes_tok > a.n_tok) a.lanes_tok = a.n_tok;
    constexpr int PV = HALVES ? V : V / 2, U = kUnroll<T, V, HALVES>;
    // tokens of a CTA: as many as a thread unrolls, less when the table is full or the GPU would stand idle
    long long tok = (long long)a.lanes_tok * U;
    const long long spread = ((long long)a.n_tok * a.n_seq + 2 * kSms - 1) / (2 * kSms);
    if (tok > spread) tok = spread;
    const int entry = (a.pairs + PV - 1) / PV * ((PV + 1) / 2) * 16;   // table bytes of a token
    if (tok > kTableBytes / entry) tok = kTableBytes / entry;
    if (tok > a.n_tok) tok = a.n_tok;
    a.tok_per_cta = (int)tok;
    if (a.lanes_tok > tok) a.lanes_tok = (int)tok;
    const int threads = (a.width * a.lanes_tok + 31) / 32 * 32;
    // the sequences of a CTA follow one another (and share the table where they share positions): about two waves of CTAs
    const long long tok_blocks = (a.n_tok + tok - 1) / tok, want = (long long)kSms * (2048 / threads);
    long long seq_blocks = (want + tok_blocks - 1) / tok_blocks;
    if (seq_blocks > a.n_seq || a.pos_seq_stride) seq_blocks = a.n_seq;
    if (seq_blocks > 65535) seq_blocks = 65535;
    a.seq_per_cta = (int)((a.n_seq + seq_blocks - 1) / seq_blocks);
    seq_blocks = (a.n_seq + a.seq_per_cta - 1) / a.seq_per_cta;
    return free_launch(free_overlap_for_rows((long long)a.n_tok * a.n_seq), rope_axes_kernel<T, V, HALVES, ALIGNED>,
                       dim3((unsigned)tok_blocks, (unsigned)seq_blocks), dim3(threads), 0, s, a);
}

// The widest vector whose size divides every offset that a slot can have.
template <typename T>
int dispatch(RopeArgs& a, bool halves, cudaStream_t s) {
    constexpr int W = 16 / (int)sizeof(T);
    auto fits = [&](int v) {
        const long long all = a.xs | a.xt | a.xh | a.ys | a.yt | a.yh | a.d_head | (halves ? a.pairs : 0);
        const uintptr_t at = reinterpret_cast<uintptr_t>(a.x) | reinterpret_cast<uintptr_t>(a.y);
        return all % v == 0 && at % (v * sizeof(T)) == 0;
    };
    if (halves) {
        if (fits(W)) return launch<T, W, true, true>(a, s);
        if (W > 4 && fits(4)) return launch<T, 4, true, true>(a, s);
        if (fits(2)) return launch<T, 2, true, true>(a, s);
        return launch<T, 1, true, true>(a, s);
    }
    if (fits(W)) return launch<T, W, false, true>(a, s);
    if (W > 4 && fits(4)) return launch<T, 4, false, true>(a, s);
    if (fits(2)) return launch<T, 2, false, true>(a, s);
    return launch<T, 2, false, false>(a, s);
}

}  // namespace

extern "C" int free_op_rope_axes(int dtype, int pairing, int freq_mode, int inverse, int n_seq, int n_tok, int heads, int d_head,
                                 int n_axes, const int32_t* axis_dims, double base, const float* pos, int64_t pos_seq_stride,
                                 const void* x, int64_t x_seq_stride, int64_t x_tok_stride, int64_t x_head_stride,
                                 void* y, int64_t y_seq_stride, int64_t y_tok_stride, int64_t y_head_stride, void* stream) {
    if (dtype != FREE_FP32 && dtype != FREE_BF16) return FREE_ERR_ARG;
    if (pairing != FREE_ROPE_INTERLEAVED && pairing != FREE_ROPE_HALVES) return FREE_ERR_ARG;
    if (freq_mode != FREE_ROPE_FREQ_PER_AXIS && freq_mode != FREE_ROPE_FREQ_JOINT) return FREE_ERR_ARG;
    if (!axis_dims || !(base > 0.0) || !isfinite(base)) return FREE_ERR_ARG;
    if (n_seq < 0 || n_tok < 0 || heads < 1 || d_head < 1 || n_axes < 1 || n_axes > kMaxAxes) return FREE_ERR_SHAPE;
    long long total = 0;
    for (int i = 0; i < n_axes; ++i) {
        if (axis_dims[i] < 0 || axis_dims[i] % 2) return FREE_ERR_SHAPE;
        total += axis_dims[i];
    }
    if (total < 2 || total > d_head) return FREE_ERR_SHAPE;
    if (d_head % 2 || total > 2 * kMaxPairs) return FREE_ERR_UNSUPPORTED;
    if (n_seq == 0 || n_tok == 0) return FREE_OK;
    if (!pos || !x || !y) return FREE_ERR_ARG;
    if (x_seq_stride < 0 || x_tok_stride < 0 || x_head_stride < 0 || y_seq_stride < 0 || y_tok_stride < 0 || y_head_stride < 0 ||
        pos_seq_stride < 0) return FREE_ERR_SHAPE;
    // strides of axes with one entry say nothing and must not decide the vector width
    if (n_seq == 1) x_seq_stride = y_seq_stride = 0;
    if (n_tok == 1) x_tok_stride = y_tok_stride = 0;
    if (heads == 1) x_head_stride = y_head_stride = 0;
    // outputs that would fall on one another
    if ((heads > 1 && y_head_stride < d_head) || (n_tok > 1 && y_tok_stride < d_head) || (n_seq > 1 && y_seq_stride < d_head)) return FREE_ERR_SHAPE;
    const uintptr_t elem = dtype == FREE_FP32 ? 4 : 2;
    if (reinterpret_cast<uintptr_t>(x) % elem || reinterpret_cast<uintptr_t>(y) % elem || (reinterpret_cast<uintptr_t>(pos) & 3u)) return FREE_ERR_ALIGN;
    RopeArgs a{};
    a.n_seq = n_seq; a.n_tok = n_tok; a.n_axes = n_axes; a.pairs = (int)(total / 2);
    a.heads = heads; a.d_head = d_head; a.pos = pos; a.pos_seq_stride = pos_seq_stride;
    a.x = x; a.xs = x_seq_stride; a.xt = x_tok_stride; a.xh = x_head_stride;
    a.y = y; a.ys = y_seq_stride; a.yt = y_tok_stride; a.yh = y_head_stride;
    a.sign = inverse ? -1.f : 1.f;
    const double two_pi = 6.283185307179586476925286766559;
    // consecutive pairs differ by one factor.  Each product adds its own rounding (2^-53) and the factor's error (pow: 2^-52) once
    // more, so the last of 128 is off by 3 x 128 units of 2^-53 at most: 4e-14, 4e-9 of a turn after 100000 turns.  128 powers cost more.
    int p = 0;
    double ratio = pow(base, -1.0 / a.pairs), t = 1.0 / two_pi;
    for (int ax = 0; ax < n_axes; ++ax) {
        const int n = axis_dims[ax] / 2;
        if (freq_mode == FREE_ROPE_FREQ_PER_AXIS && n > 0) { ratio = pow(base, -1.0 / n); t = 1.0 / two_pi; }
        for (int i = 0; i < n; ++i, ++p, t *= ratio) { a.turns[p] = t; a.axis[p] = (unsigned char)ax; }
    }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool halves = pairing == FREE_ROPE_HALVES;
    return dtype == FREE_FP32 ? dispatch<float>(a, halves, s) : dispatch<__nv_bfloat16>(a, halves, s);
}
