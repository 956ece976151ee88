// Attention to an encoder's states for few tokens (single ones above all): tokens x query heads of a key head are up to eight rows.
//
//   S = scale q k^T, p = 2^(c S - m), out = sum p v / sum p
//
// Bound by HBM (K and V are read once, 2 rows of multiply-adds per element) or, for short state sequences, by latency: no tensor
// memory, no tile copies, one launch.  L lanes hold a state's row, one 16-byte unit each, and a warp 32 / L states; every group of
// lanes takes KEYS states at a time.  Units are copied to shared memory several steps ahead, every lane its own, so that the bytes in
// flight do not cost registers.  Scores are summed over the lanes by exchanges that halve the values as they go, so that every lane ends
// with its own (row, state) and takes its exponential; the probabilities are then passed to all lanes of the group.  The parts of a
// CTA's groups are joined through shared memory; long state sequences are split over CTAs as well and joined by cross_join_kernel.
// Measured: 4 sequences of 77 states, 6 heads of 64: 4.4 us (8.7 by the tensor cores' kernel).  8 of up to 16384 states, 32 heads of 128
// on 8: 80 us with the join, 4.5 TB/s of K and V (120 us with every score summed over all lanes).  Neither issue slots (0.67) nor HBM (0.55)
// are full; what is left are the ends: parts of unequal length, which only the device knows, make two rounds of CTAs and a bit.
#include "cross_tc.cuh"

namespace {

using namespace cross_tc;

constexpr int kThreads = 128, kWarps = kThreads / 32, kSms = 148;
// Steps of copies in the ring.  Four rows: three, with 128 registers a thread, so that an SM holds four CTAs (8 of up to 16384 states 90 -> 84 us;
// eight rows have no registers to spare, 33 -> 41 us for 2 x 8192 states, and one row with three steps 91 -> 98 us).
template <int ROWS> constexpr int kStepsOf = ROWS == 4 ? 3 : 4;

template <typename E> struct Unit;            // 16 bytes of a row, as pairs of fp32 numbers
template <> struct Unit<float> {
    static constexpr int V = 4;
    static __device__ __forceinline__ void values(const uint4& u, uint64_t (&f)[2]) {
        f[0] = pair(__uint_as_float(u.x), __uint_as_float(u.y)); f[1] = pair(__uint_as_float(u.z), __uint_as_float(u.w));
    }
};
template <> struct Unit<__nv_bfloat16> {
    static constexpr int V = 8;
    static __device__ __forceinline__ void values(const uint4& u, uint64_t (&f)[4]) {
        const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = pair(__uint_as_float(w[i] << 16), __uint_as_float(w[i] & 0xffff0000u));
    }
};
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ void from_f(float& d, float v) { d = v; }
__device__ __forceinline__ void from_f(__nv_bfloat16& d, float v) { d = __float2bfloat16(v); }
// fp32 results are compared with 64 bits: the exact exponential there, the fast one (2 units) for bf16
template <typename E> __device__ __forceinline__ float power(float x) {
    if constexpr (sizeof(E) == 4) return exp2f(x);
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// R: rows held; L: lanes of a state's row
template <typename E, int R, int L> __global__ void __launch_bounds__(kThreads, R == 4 ? 4 : 1) cross_rows_kernel(const CrossArgs a, const CrossParts parts) {
    constexpr int kSteps = kStepsOf<R>;
    constexpr int V = Unit<E>::V, G = 32 / L, GROUPS = kWarps * G, KEYS = R <= 4 ? 4 : 2;
    extern __shared__ uint4 ring[];           // [step][warp][2 KEYS][lane]; at the end the groups' parts
    __shared__ float2 stats[GROUPS][R];       // maximum, sum
    float* acc_of = reinterpret_cast<float*>(ring);      // [group][row][channel]
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x % L, group = threadIdx.x / L;
    const int part = blockIdx.x % parts.n, sh = blockIdx.x / parts.n, kh = sh % a.kv_heads, s = sh / a.kv_heads;
    const int rows = a.n_q * a.group;
    const CrossSpan sp = cross_span(a.where, s);
    const uint8_t* mask = cross_mask(a.where, sp);
    const int lo = (int)((long long)sp.len * part / parts.n), hi = (int)((long long)sp.len * (part + 1) / parts.n);
    const bool in = lane * V < a.d;
    const E* kb = reinterpret_cast<const E*>(a.k.p) + sp.enc * a.k.seq + (long long)sp.row0 * a.k.tok + kh * a.k.head + lane * V;
    const E* vb = reinterpret_cast<const E*>(a.v.p) + sp.enc * a.v.seq + (long long)sp.row0 * a.v.tok + kh * a.v.head + lane * V;
    constexpr int N = R * KEYS, NF = N >= L ? N / L : 1, D = N >= L ? 1 : L / N;     // scores of a group and step, of a lane; lanes of a score
    constexpr int SAME = NF < KEYS ? NF : KEYS, ROWL = KEYS * D / NF > 1 ? KEYS * D / NF : 1;      // of a lane's scores, those of one row; lanes of a row
    uint64_t q[R][V / 2], acc[R][V / 2];
    float top[NF], sum[NF];
    const float c = a.scale * 1.4426950408889634f;
#pragma unroll
    for (int v = 0; v < NF; ++v) { top[v] = -INFINITY; sum[v] = 0.f; }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const E* qp = reinterpret_cast<const E*>(a.q.p) + s * a.q.seq + (r / a.group) * a.q.tok + (kh * a.group + r % a.group) * a.q.head + lane * V;
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            q[r][e] = r < rows && in ? pair(to_f(qp[2 * e]), to_f(qp[2 * e + 1])) : 0ull;
            acc[r][e] = 0ull;
        }
    }
    // score i of a group is in slot i % NF of lane i / NF * D
    auto from_lane = [&](const float (&v)[NF], int i) { return __shfl_sync(0xffffffffu, v[i % NF], i / NF * D, L); };
    const uint32_t mine = (uint32_t)__cvta_generic_to_shared(ring) + ((threadIdx.x >> 5) * 2 * KEYS * 32 + (threadIdx.x & 31)) * 16u;
    constexpr uint32_t STEP = kThreads * 2 * KEYS * 16;
    auto counts = [&](int j) { return j < hi && (!mask || mask[j] != 0); };
    int ahead = lo + group * KEYS;                                 // first state of the step to copy next
    uint32_t to = 0;
    const E *kp = kb + (long long)ahead * a.k.tok, *vp = vb + (long long)ahead * a.v.tok;     // running addresses, which may lie behind the last state
    const long long k_step = (long long)(GROUPS * KEYS) * a.k.tok, v_step = (long long)(GROUPS * KEYS) * a.v.tok;
    auto copy = [&]() {
        const int left = in ? hi - ahead : 0;
        const E *k1 = kp, *v1 = vp;
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            const bool ok = k < left && (!mask || mask[ahead + k] != 0);      // else zeros, and nothing is read
            const uint32_t dst = mine + to + k * 512u, size = ok ? 16u : 0u;
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(ok ? k1 : kb), "r"(size) : "memory");
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst + KEYS * 512u), "l"(ok ? v1 : vb), "r"(size) : "memory");
            k1 += a.k.tok; v1 += a.v.tok;
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
        ahead += GROUPS * KEYS;
        kp += k_step; vp += v_step;
        to = to + STEP == kSteps * STEP ? 0 : to + STEP;
    };
#pragma unroll
    for (int i = 0; i < kSteps - 1; ++i) copy();
    uint32_t from = 0;
    for (int j0 = lo + group * KEYS; j0 - group * KEYS < hi; j0 += GROUPS * KEYS) {       // all lanes take part in the exchanges
        asm volatile("cp.async.wait_group %0;" ::"n"(kSteps - 2) : "memory");
        uint4 ku[KEYS], vu[KEYS];
        bool ok[KEYS];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            ok[k] = counts(j0 + k);
            const uint32_t src = mine + from + k * 512u;
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(ku[k].x), "=r"(ku[k].y), "=r"(ku[k].z), "=r"(ku[k].w) : "r"(src) : "memory");
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(vu[k].x), "=r"(vu[k].y), "=r"(vu[k].z), "=r"(vu[k].w) : "r"(src + KEYS * 512u) : "memory");
        }
        from = from + STEP == kSteps * STEP ? 0 : from + STEP;
        copy();                                                    // into the step that was read before this one
        float sc[N];
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            uint64_t f[V / 2];
            Unit<E>::values(ku[k], f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                uint64_t t = 0ull;
#pragma unroll
                for (int e = 0; e < V / 2; ++e) t = fma2(q[r][e], f[e], t);
                sc[r * KEYS + k] = low(t) + high(t);
            }
        }
        {
            int n = N;
#pragma unroll
            for (int o = L / 2; o > 0; o >>= 1) {
                if (n > 1) {
                    n >>= 1;
                    const bool up = lane & o;
#pragma unroll
                    for (int i = 0; i < N / 2; ++i)
                        if (i < n) {
                            const float keep = up ? sc[n + i] : sc[i], give = up ? sc[i] : sc[n + i];
                            sc[i] = keep + __shfl_xor_sync(0xffffffffu, give, o);
                        }
                } else {
                    sc[0] += __shfl_xor_sync(0xffffffffu, sc[0], o);
                }
            }
        }
        float p[NF], alpha[NF];
        bool moved = false;
#pragma unroll
        for (int v = 0; v < NF; ++v) {
            const int k = (lane / D * NF + v) % KEYS;              // this score's state
            bool good = ok[0];
#pragma unroll
            for (int u = 1; u < KEYS; ++u) good = k == u ? ok[u] : good;
            p[v] = good ? sc[v] : -INFINITY;
        }
#pragma unroll
        for (int v = 0; v < NF; v += SAME) {
            float m = p[v];
#pragma unroll
            for (int u = 1; u < SAME; ++u) m = fmaxf(m, p[v + u]);
#pragma unroll
            for (int o = D; o < ROWL; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
            const float now = fmaxf(top[v], m), base = now == -INFINITY ? 0.f : now;
            const float al = now == top[v] ? 1.f : power<E>((top[v] - base) * c);
            moved = moved || now != top[v];
#pragma unroll
            for (int u = 0; u < SAME; ++u) {
                p[v + u] = power<E>((p[v + u] - base) * c);
                sum[v + u] = fmaf(sum[v + u], al, p[v + u]);
                top[v + u] = now;
                alpha[v + u] = al;
            }
        }
        if (__any_sync(0xffffffffu, moved)) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float al = from_lane(alpha, r * KEYS);
                const uint64_t a2 = pair(al, al);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) acc[r][e] = mul2(acc[r][e], a2);
            }
        }
#pragma unroll
        for (int k = 0; k < KEYS; ++k) {
            uint64_t f[V / 2];
            Unit<E>::values(vu[k], f);
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const float pr = from_lane(p, r * KEYS + k);
                const uint64_t p2 = pair(pr, pr);
#pragma unroll
                for (int e = 0; e < V / 2; ++e) acc[r][e] = fma2(p2, f[e], acc[r][e]);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    __syncthreads();                                               // the ring is free for the parts
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const float m = from_lane(top, r * KEYS);
        float l = 0.f;
#pragma unroll
        for (int k = 0; k < KEYS; ++k) l += from_lane(sum, r * KEYS + k);
        if (lane == 0) stats[group][r] = make_float2(m, l);
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
            acc_of[(group * R + r) * L * V + lane * V + 2 * e] = low(acc[r][e]);
            acc_of[(group * R + r) * L * V + lane * V + 2 * e + 1] = high(acc[r][e]);
        }
    }
    __syncthreads();
    const long long all = (long long)a.n_seq * a.heads * a.n_q;
    for (int i = threadIdx.x; i < R * L * V; i += kThreads) {
        const int r = i / (L * V), ch = i % (L * V);
        if (r >= rows || ch >= a.d) continue;
        float m = -INFINITY;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) m = fmaxf(m, stats[g][r].x);
        const float base = m == -INFINITY ? 0.f : m;
        float l = 0.f, o = 0.f;
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) {
            const float f = power<E>((stats[g][r].x - base) * c);
            l = fmaf(f, stats[g][r].y, l);
            o = fmaf(f, acc_of[(g * R + r) * L * V + ch], o);
        }
        // no state: the sum tells, which a NaN among the scores reaches (the maximum leaves it out), and both terms of lse are -inf
        const float out = l == 0.f ? 0.f : o / l, lse = m * a.scale + logf(l);
        const int t = r / a.group, h = kh * a.group + r % a.group;
        const long long row = ((long long)s * a.heads + h) * a.n_q + t;
        if (parts.n > 1) {
            parts.out[(part * all + row) * a.d + ch] = out;
            if (ch == 0) parts.lse[part * all + row] = lse;
        } else {
            from_f(reinterpret_cast<E*>(const_cast<void*>(a.o.p))[s * a.o.seq + t * a.o.tok + h * a.o.head + ch], out);
            if (ch == 0 && a.lse) a.lse[row] = lse;
        }
    }
}

template <typename E, int R> int start(const CrossArgs& a, const CrossParts& parts, cudaStream_t s) {
    const int units = (a.d + Unit<E>::V - 1) / Unit<E>::V;
    const long long ctas = (long long)a.n_seq * a.kv_heads * parts.n;
    if (ctas > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    auto kernel = units <= 4 ? cross_rows_kernel<E, R, 4> : units <= 8 ? cross_rows_kernel<E, R, 8> : units <= 16 ? cross_rows_kernel<E, R, 16> : cross_rows_kernel<E, R, 32>;
    constexpr int copies = kStepsOf<R> * kThreads * 2 * (R <= 4 ? 4 : 2) * 16, joined = kThreads * R * Unit<E>::V * 4, smem = copies > joined ? copies : joined;
    if (smem > 47 * 1024) FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem));
    return free_launch(free_overlap_for_rows(a.n_seq), kernel, dim3((unsigned)ctas), dim3(kThreads), smem, s, a, parts);
}
template <typename E> int rows_of(const CrossArgs& a, const CrossParts& parts, cudaStream_t s) {
    const int rows = a.n_q * a.group;
    return rows == 1 ? start<E, 1>(a, parts, s) : rows == 2 ? start<E, 2>(a, parts, s) : rows <= 4 ? start<E, 4>(a, parts, s) : start<E, 8>(a, parts, s);
}

}  // namespace

// Whole 16-byte units of K and V, and few rows
bool cross_rows_supported(int dtype, const CrossArgs& a) {
    if ((long long)a.n_q * a.group > 8 || a.where.n_kv < 1) return false;
    const int v = dtype == FREE_FP32 ? 4 : 8;
    bool ok = a.d % v == 0;
    for (const CrossMat* m : {&a.k, &a.v}) ok = ok && free_aligned16(m->p) && m->seq % v == 0 && m->tok % v == 0 && m->head % v == 0;
    return ok;
}

// Parts: enough CTAs for eight on every SM, 128 states each at least (twelve took 2% longer, 24 a fifth).
int cross_rows_parts(const CrossArgs& a) {
    const long long ctas = (long long)a.n_seq * a.kv_heads, most = (a.where.n_kv + 127) / 128;
    long long n = (8 * kSms + ctas - 1) / ctas;
    if (n > most) n = most;
    return n < 1 ? 1 : (int)n;
}

int cross_rows_forward(int dtype, const CrossArgs& a, const CrossParts& parts, cudaStream_t s) {
    FREE_TRY(dtype == FREE_FP32 ? rows_of<float>(a, parts, s) : rows_of<__nv_bfloat16>(a, parts, s));
    return parts.n > 1 ? cross_join(dtype, a, parts, s) : FREE_OK;
}
