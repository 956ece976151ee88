// Rotary positions with several axes: every pair (a, b) of a head is turned by an angle that grows with the token's
// position on the pair's axis,
//   t = pos[axis(pair)] * freq(pair),   (a, b) -> (a cos t - b sin t, a sin t + b cos t);   inverse: -t (also the backward pass).
//
// Bound by HBM (each element is read and written once; 3 FLOPs).  The angle of a far position needs more than fp32: it is
// formed in turns, t / 2 pi, as one fp64 product, reduced to [-1/2, 1/2] there, and only the remainder goes to fp32
// sincospif.  All heads of a token share its angles, so a CTA first fills a table [tokens][pairs] of (cos, sin) in shared
// memory and then streams its tokens' heads through it.  A thread keeps one slot (one vector of a head, or the two that it
// couples) and walks over the tokens, so that the index arithmetic is done once per thread, and has kUnroll tokens' loads
// in flight.  The table of frequencies is formed on the host in fp64 and travels as a kernel argument.
#include "internal.h"
#include <math.h>

namespace {

constexpr int kMaxPairs = 128;                     // rotated pairs of a head
constexpr int kMaxAxes = 4;
constexpr int kThreads = 512;                      // most threads of a CTA
constexpr int kTable = 2048;                       // (cos, sin) entries of a CTA: 16 KB
constexpr int kMaxTok = 256;                       // tokens of a CTA
constexpr int kUnroll = 4;
constexpr int kSms = 148;

struct RopeArgs {
    long long tokens;                              // n_seq * n_tok
    int n_tok, n_axes, pairs;                      // pairs: rotated pairs of a head
    int heads, d_head;
    int slots_per_head, slots;                     // slots: slots_per_head * heads
    int tok_per_cta;
    int width, lanes_tok;                          // a CTA's threads: width slots side by side, for lanes_tok tokens at a time
    const float* pos; long long pos_seq_stride;
    const void* x; long long xs, xt, xh;           // strides of sequence, token, head in elements
    void* y; long long ys, yt, yh;
    float sign;
    double turns[kMaxPairs];                       // angle per unit of position, in turns
    unsigned char axis[kMaxPairs];
};

template <typename T, int N> struct alignas(sizeof(T) * N) Pack { T v[N]; };
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16(v); }

// V elements as one access, or (ALIGNED false) one by one
template <typename T, int V, bool ALIGNED> __device__ __forceinline__ Pack<T, V> get(const T* p) {
    Pack<T, V> r;
    if (ALIGNED) r = *reinterpret_cast<const Pack<T, V>*>(p);
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) r.v[i] = p[i];
    }
    return r;
}
template <typename T, int V, bool ALIGNED> __device__ __forceinline__ void put(T* p, const Pack<T, V>& r) {
    if (ALIGNED) *reinterpret_cast<Pack<T, V>*>(p) = r;
    else {
#pragma unroll
        for (int i = 0; i < V; ++i) p[i] = r.v[i];
    }
}

// HALVES false: a slot is V consecutive elements (V / 2 pairs (2i, 2i + 1)); elements past the rotated ones are copied.
// HALVES true: pair i couples elements i and i + pairs; a slot is V elements of the first half with their partners, or V
// elements behind both halves, which are copied.
template <typename T, int V, bool HALVES, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) rope_axes_kernel(const __grid_constant__ RopeArgs a) {
    __shared__ float2 table[kTable];
    __shared__ long long off_x[kMaxTok], off_y[kMaxTok];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const long long tok0 = (long long)blockIdx.x * a.tok_per_cta;
    const int n = (int)(a.tokens - tok0 < a.tok_per_cta ? a.tokens - tok0 : a.tok_per_cta);
    const int P = a.pairs;
    for (int i = threadIdx.x; i < n; i += blockDim.x) {
        const long long q = (tok0 + i) / a.n_tok, t = (tok0 + i) % a.n_tok;
        off_x[i] = q * a.xs + t * a.xt;
        off_y[i] = q * a.ys + t * a.yt;
    }
    for (int i = threadIdx.x; i < n * P; i += blockDim.x) {
        const int k = i / P, p = i - k * P;
        const long long q = (tok0 + k) / a.n_tok, t = (tok0 + k) % a.n_tok;
        double turn = (double)a.pos[q * a.pos_seq_stride + t * a.n_axes + a.axis[p]] * a.turns[p];
        turn -= rint(turn);
        float s, c;
        sincospif((float)(turn + turn), &s, &c);
        table[i] = make_float2(c, a.sign * s);
    }
    __syncthreads();
    const T* x = reinterpret_cast<const T*>(a.x);
    T* y = reinterpret_cast<T*>(a.y);
    const int width = a.width, lt = threadIdx.x / width;
    if (lt >= a.lanes_tok) return;
    for (int slot = threadIdx.x - lt * width; slot < a.slots; slot += width) {
        const int h = slot / a.slots_per_head, j = slot - h * a.slots_per_head;
        const int pair0 = HALVES ? j * V : j * (V / 2);            // first pair of the slot
        const int col = HALVES ? (pair0 < P ? pair0 : pair0 + P) : j * V;
        const T* xp = x + h * a.xh + col;
        T* yp = y + h * a.yh + col;
        for (int t0 = lt; t0 < n; t0 += a.lanes_tok * kUnroll) {
            Pack<T, V> u[kUnroll], w[kUnroll];
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int t = t0 + k * a.lanes_tok;
                if (t < n) {
                    u[k] = get<T, V, ALIGNED>(xp + off_x[t]);
                    if (HALVES && pair0 < P) w[k] = get<T, V, ALIGNED>(xp + off_x[t] + P);
                }
            }
#pragma unroll
            for (int k = 0; k < kUnroll; ++k) {
                const int t = t0 + k * a.lanes_tok;
                if (t >= n) break;
                const float2* cs = table + t * P + pair0;
                if (HALVES) {
                    if (pair0 < P) {
#pragma unroll
                        for (int e = 0; e < V; ++e) {
                            const float2 f = cs[e];
                            const float p = to_f(u[k].v[e]), q = to_f(w[k].v[e]);
                            from_f(u[k].v[e], p * f.x - q * f.y);
                            from_f(w[k].v[e], p * f.y + q * f.x);
                        }
                        put<T, V, ALIGNED>(yp + off_y[t] + P, w[k]);
                    }
                } else {
#pragma unroll
                    for (int e = 0; e < V / 2; ++e)
                        if (pair0 + e < P) {                       // elements past the rotated ones stay as they are
                            const float2 f = cs[e];
                            const float p = to_f(u[k].v[2 * e]), q = to_f(u[k].v[2 * e + 1]);
                            from_f(u[k].v[2 * e], p * f.x - q * f.y);
                            from_f(u[k].v[2 * e + 1], p * f.y + q * f.x);
                        }
                }
                put<T, V, ALIGNED>(yp + off_y[t], u[k]);
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
    const int passes = (a.slots + kThreads - 1) / kThreads;
    a.width = (a.slots + passes - 1) / passes;
    a.lanes_tok = a.width >= 256 ? 1 : 256 / a.width;
    const int threads = (a.width * a.lanes_tok + 31) / 32 * 32;
    // tokens of a CTA: four slots of a thread's loads in flight, less when the table is full or the GPU would stand idle
    long long tok = (long long)a.lanes_tok * kUnroll;
    const long long spread = (a.tokens + 2 * kSms - 1) / (2 * kSms);
    if (tok > spread) tok = spread;
    if (tok > kTable / a.pairs) tok = kTable / a.pairs;
    if (tok > kMaxTok) tok = kMaxTok;
    if (tok < 1) tok = 1;
    a.tok_per_cta = (int)tok;
    const long long grid = (a.tokens + tok - 1) / tok;
    if (grid > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    return free_launch(free_overlap_for_rows(a.tokens), rope_axes_kernel<T, V, HALVES, ALIGNED>, dim3((unsigned)grid), dim3(threads), 0, s, a);
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
    a.tokens = (long long)n_seq * n_tok; a.n_tok = n_tok; a.n_axes = n_axes; a.pairs = (int)(total / 2);
    a.heads = heads; a.d_head = d_head; a.pos = pos; a.pos_seq_stride = pos_seq_stride;
    a.x = x; a.xs = x_seq_stride; a.xt = x_tok_stride; a.xh = x_head_stride;
    a.y = y; a.ys = y_seq_stride; a.yt = y_tok_stride; a.yh = y_head_stride;
    a.sign = inverse ? -1.f : 1.f;
    const double two_pi = 6.283185307179586476925286766559;
    int p = 0;
    for (int ax = 0; ax < n_axes; ++ax)
        for (int i = 0; i < axis_dims[ax] / 2; ++i, ++p) {
            const double e = freq_mode == FREE_ROPE_FREQ_JOINT ? (double)p / a.pairs : (double)i / (axis_dims[ax] / 2);
            a.turns[p] = pow(base, -e) / two_pi;
            a.axis[p] = (unsigned char)ax;
        }
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool halves = pairing == FREE_ROPE_HALVES;
    return dtype == FREE_FP32 ? dispatch<float>(a, halves, s) : dispatch<__nv_bfloat16>(a, halves, s);
}
