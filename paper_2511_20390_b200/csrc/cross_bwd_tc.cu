// Gradients of the attention to an encoder's states on the tensor cores (bf16 operands, fp32 accumulation).
//
//   p = 2^(c S - lse log2 e), S = q k^T;   dP = g v^T (g: the gradient of out);   dS = p (dP - delta) scale, delta = <g, out>
//   dq = dS k                 rows are 128 tokens of one head, columns the states
//   dk = dS^T q, dv = p^T g   rows are 128 states of one key head, columns the tokens of every head and sequence that reads them
//
// Both are one kernel: two 128 x 64 products S and dP from the rows' two operands (resident) and a column tile's two (a ring), the
// elementwise part in registers, and p and dS, rounded to bf16, back to tensor memory as left operands of the products that
// accumulate.  Transposing the problem for dk and dv (rows are states) leaves every operand as it lies in memory: a column tile serves
// as K-major operand of S or dP and, read along its rows, as operand of the accumulation.
// Persistent CTAs, one per SM: two warpgroups for the elementwise part, a column tile each in turn; one that writes results; a warp that
// finds items (dk, dv: takes the next as its CTA comes free; 24 x 1024 tokens of 16 heads of 72 leave some SMs seven blocks of states and
// others four where they are dealt out), one that loads tiles, one that brings the tokens' lse and delta (dk, dv); one each that issues S,
// dP and either accumulating product, in order, so that sums have a fixed order whichever CTA forms them.  Nothing is added atomically; S
// and dP are formed twice instead (once here, once for the other direction).
// What bounds it: the way of a tile through the warps.  Those 24 x 1024 tokens take 89 us for dq and 107 for dk, dv; the tensor cores
// work for 20% of that, the exponentials' unit for 22%; a tile's elementwise part takes 1300 to 2000 clocks, its copies 2300 when they
// compete with a block of rows, a wait 115 when it is over already.  Before S, dP, dk and dv had a warp each, and dP its own tensor memory,
// free once it is read: 95 and 160.
// States that do not count: p and dS are replaced by zeros, and (dq) their rows of K zeroed in shared memory, for 0 x NaN is NaN.
#include "cross_tc.cuh"

namespace {

using namespace cross_tc;

constexpr int BR = 128, BC = 64;
constexpr int kThreads = 640, kSms = 148;     // warps 0 - 7 elementwise, 8 - 11 results, 12 loads, 13 statistics, 14 S, 15 dP, 16 zeros, 17 dq or dk, 18 dv, 19 items
constexpr int kMathRegs = 136, kOtherRegs = 64;
static_assert(256 * kMathRegs + 384 * kOtherRegs <= kThreads * 96, "registers of the launch");
constexpr uint32_t kChunk = BR * 128, kColChunk = BC * 128;
constexpr uint32_t kStage = 32 * 128;     // staging: 128 bytes of 32 rows, pieces of 16 swizzled

// NCH: chunks of 64 channels; W: columns of tensor memory per sum; AB: sets of the rows' operands; N1, N2: ring slots of the columns'
// operands; NS, ND: buffers of S (p and dS go over it) and of dP (free once read); NA: sets of sums
template <bool DKV, int NCH, int W, int AB, int N1, int N2, int NS, int ND, int NA> struct Mem {
    static constexpr uint32_t queue = DKV ? 2 : 4;        // items
    static constexpr uint32_t a = NCH * kChunk, b = NCH * kColChunk;
    static constexpr uint32_t ctrl = 1024 + (DKV ? N1 * BC * 8 : 0);
    static constexpr uint32_t ctrl_bytes = (ctrl + 1023) / 1024 * 1024;
    static constexpr uint32_t bytes = 1024 + ctrl_bytes + AB * 2 * a + (N1 + N2) * b + 4 * kStage;
    static constexpr uint32_t dp_col = NS * 64, acc_col = (NS + ND) * 64, acc_set = (DKV ? 2 : 1) * W;
    static_assert(acc_col + NA * acc_set <= 512, "tensor memory of an SM");
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
    static_assert((2 * AB + 2 * N1 + 2 * N2 + 3 * NS + ND + 2 * NA + 2 * queue + 1) * 8 <= 512, "barriers");
};

struct Args {
    CrossWhere where;
    int n_seq, n_q, heads, kv_heads, d, group;
    int q_seq_mul, q_head_mul, g_seq_mul, g_head_mul, k_seq_mul, k_head_mul, v_seq_mul, v_head_mul;     // 0 where one matrix serves all
    int blocks, parts;                        // row blocks of a (sequence, head), or cross_block's of an encoder sequence; parts of the columns
    long long items;
    float c, scale;
    const float *lse, *delta;
    CrossMat o1, o2;                          // results: dq, or dk and dv
    float* part_out;                          // [part][2][encoder row][key head][d]
    long long part_rows;
    unsigned long long* next;                 // dk, dv: the next item that no CTA has
    uint32_t* err;
};

struct alignas(16) Item {
    int live, idx, head, row0;                // idx: sequence (dq) or encoder sequence (dk, dv); head: of the rows; row0: first row's token or state
    int tiles, part, enc, row;                // column tiles; enc, row: where the first state lies
    int left, first, limit, kv_head;          // states from `row` on; first column tile of the part; rows that are written (the last block of states: behind it, too)
};

__device__ __forceinline__ int sequences_of(const Args& a, int e) {      // that read encoder sequence e; whole warp
    if (!a.where.seq_of) return a.n_seq ? a.where.share : 0;
    int n = 0;
    for (int s0 = 0; s0 < a.n_seq; s0 += 32) {
        const int s = s0 + (threadIdx.x & 31);
        n += __popc(__ballot_sync(0xffffffffu, s < a.n_seq && __ldg(a.where.seq_of + s) == e));
    }
    return n;
}

template <bool DKV, bool ROWS> __device__ __forceinline__ Item item_of(const Args& a, long long i) {     // whole warp
    Item it;
    it.live = i < a.items;
    it.tiles = it.part = it.first = 0;
    if (!it.live) return it;
    if (DKV) {
        it.part = (int)(i % a.parts);
        const CrossBlock b = cross_block<BR, ROWS>(a.where, a.kv_heads, a.blocks, i / a.parts);
        it.live = b.more; it.idx = b.e; it.head = it.kv_head = b.head; it.row0 = b.row0; it.limit = 0;
        if (ROWS && b.row0 < 0) return it;
        const CrossSpan sp = cross_span_of_enc(a.where, it.idx);
        it.enc = sp.enc; it.row = sp.row0 + it.row0; it.left = sp.len - it.row0;
        it.limit = b.last ? sp.rows - it.row0 : min(sp.rows - it.row0, BR);
        if (it.left > 0) {
            const long long all = (long long)sequences_of(a, it.idx) * a.group * ((a.n_q + BC - 1) / BC);
            it.first = (int)(all * it.part / a.parts);
            it.tiles = (int)(all * (it.part + 1) / a.parts) - it.first;
        }
    } else {
        const int blk = (int)(i % a.blocks); i /= a.blocks;
        it.head = (int)(i % a.heads); it.idx = (int)(i / a.heads);
        it.kv_head = it.head / a.group;
        const CrossSpan sp = cross_span(a.where, it.idx);
        it.row0 = blk * BR;
        it.enc = sp.enc; it.row = sp.row0; it.left = sp.len;
        it.limit = a.n_q - it.row0;
        it.tiles = (sp.len + BC - 1) / BC;
    }
    return it;
}

// dk, dv: the column tiles of an item, in order: (sequence, head of the group, 64 tokens)
struct Columns {
    int s, g, t, tiles_q;
    __device__ __forceinline__ void seek(const Args& a, const Item& it) {
        tiles_q = (a.n_q + BC - 1) / BC;
        const int per = a.group * tiles_q, skip = it.first / per, rest = it.first % per;
        g = rest / tiles_q; t = rest % tiles_q;
        if (!a.where.seq_of) { s = it.idx * a.where.share + skip; return; }
        s = -1;
        for (int k = 0; k <= skip; ++k) next_sequence(a, it.idx);
    }
    __device__ __forceinline__ void next_sequence(const Args& a, int e) {
        ++s;
        if (a.where.seq_of)
            while (s < a.n_seq && __ldg(a.where.seq_of + s) != e) ++s;
    }
    __device__ __forceinline__ void next(const Args& a, int e) {
        if (++t < tiles_q) return;
        t = 0;
        if (++g < a.group) return;
        g = 0;
        next_sequence(a, e);
    }
};

template <bool DKV, bool ROWS, int NCH, int W, int AB, int N1, int N2, int NS, int ND, int NA>
__global__ void __launch_bounds__(kThreads, 1)
cross_bwd_kernel(const __grid_constant__ CUtensorMap mapA1, const __grid_constant__ CUtensorMap mapA2, const __grid_constant__ CUtensorMap mapB1,
                 const __grid_constant__ CUtensorMap mapB2, const Args a) {
    using M = Mem<DKV, NCH, W, AB, N1, N2, NS, ND, NA>;
    constexpr uint32_t kQueue = M::queue;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* a_full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* a_empty = a_full + AB;
    uint64_t* b1_full = a_empty + AB;
    uint64_t* b1_empty = b1_full + N1;
    uint64_t* b2_full = b1_empty + N1;
    uint64_t* b2_empty = b2_full + N2;
    uint64_t* s_full = b2_empty + N2;         // S and dP of a buffer
    uint64_t* p_full = s_full + NS;           // p and dS
    uint64_t* s_free = p_full + NS;           // the accumulating products have read them
    uint64_t* d_free = s_free + NS;           // dP has been read
    uint64_t* acc_full = d_free + ND;
    uint64_t* acc_free = acc_full + NA;
    uint64_t* item_full = acc_free + NA;
    uint64_t* item_free = item_full + kQueue;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(item_free + kQueue);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    Item* queue = reinterpret_cast<Item*>(smem + 512);
    static_assert(512 + kQueue * sizeof(Item) <= 1024, "control block");
    float* stats = reinterpret_cast<float*>(smem + 1024);     // dk, dv: [slot of B1][-lse log2 e, -scale delta][column]
    uint8_t* sA = smem + M::ctrl_bytes;
    uint8_t* ring1 = sA + AB * 2 * M::a;
    uint8_t* ring2 = ring1 + N1 * M::b;

    uint8_t* staging = ring2 + N2 * M::b;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < AB; ++i) { tc::mbar_init(&a_full[i], 1); tc::mbar_init(&a_empty[i], 2); }
        for (int i = 0; i < N1; ++i) { tc::mbar_init(&b1_full[i], DKV ? 2 : 1); tc::mbar_init(&b1_empty[i], 1); }
        for (int i = 0; i < N2; ++i) { tc::mbar_init(&b2_full[i], 1); tc::mbar_init(&b2_empty[i], 1); }
        for (int i = 0; i < NS; ++i) { tc::mbar_init(&s_full[i], 2); tc::mbar_init(&p_full[i], 4); tc::mbar_init(&s_free[i], DKV ? 2 : 1); }
        for (int i = 0; i < ND; ++i) tc::mbar_init(&d_free[i], 4);
        for (int i = 0; i < NA; ++i) { tc::mbar_init(&acc_full[i], DKV ? 2 : 1); tc::mbar_init(&acc_free[i], 4); }
        for (uint32_t i = 0; i < kQueue; ++i) { tc::mbar_init(&item_full[i], 1); tc::mbar_init(&item_free[i], DKV ? 18 : 16); }    // 8 + 4 + 4 (+ 2)
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::fence_proxy_async();
    }
    if (warp == 12) { tc::tmem_alloc(tmem_slot, 512); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() { *abort_flag = 1; atomicOr(a.err, FREE_DEV_ERR_ATTN); };
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int ks = (a.d + 15) / 16;
    auto see = [&](uint32_t n) { return cross_tc::wait(&item_full[n % kQueue], n / kQueue & 1u, abort_flag); };
    auto leave = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&item_free[n % kQueue]);
    };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kMathRegs));
        // ------------------------------------------------------------------ elementwise: a warpgroup per column tile, a thread per row
        const int w = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16);
        const uint64_t c2 = pair(a.c, a.c), sc2 = pair(a.scale, a.scale);
        uint32_t tile = 0, buf = 0, buf_ph = 0, dbuf = 0, slot = 0, slot_ph = 0;   // column tiles of the CTA so far; buffers and ring slot of the next
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            ok = see(n);
            if (!ok) break;
            const Item& item = queue[n % kQueue];
            const int live = item.live, tiles = item.tiles, left = item.left, idx = item.idx, head = item.head, row0 = item.row0;
            const uint8_t* mask = a.where.mask ? a.where.mask + (a.where.offsets ? 0 : (long long)item.enc * a.where.n_kv) + item.row : nullptr;
            leave(n);
            if (!live) break;
            uint64_t row_l = 0ull, row_d = 0ull;         // -lse log2 e and -scale delta of the row, twice
            if (!DKV && row0 + r < a.n_q) {
                const long long i = ((long long)idx * a.heads + head) * a.n_q + row0 + r;
                const float l = -1.4426950408889634f * __ldg(a.lse + i), dl = -a.scale * __ldg(a.delta + i);
                row_l = pair(l, l);
                row_d = pair(dl, dl);
            }
            for (int j = 0; ok && j < tiles; ++j, ++tile) {
                if ((tile & 1u) == (uint32_t)w) {
                    uint32_t bits[2] = {0xffffffffu, 0xffffffffu};
                    const bool whole = DKV || (left - j * BC >= BC && !mask);
                    if (!whole) count_bits(bits, mask, j * BC, left, lane);
                    ok = DKV ? cross_tc::wait2(&s_full[buf], buf_ph, &b1_full[slot], slot_ph, abort_flag) :      // (and the statistics, first hand)
                               cross_tc::wait(&s_full[buf], buf_ph, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint32_t ts = lanes + buf * 64u, td = lanes + M::dp_col + dbuf * 64u;
                    const ulonglong2 *cl = reinterpret_cast<const ulonglong2*>(stats + slot * 2 * BC), *cd = cl + BC / 4;
#pragma unroll 1                                                         // (half the code: instructions come in time)
                    for (int h = 0; h < 2; ++h) {
                        uint32_t s[32], d[32], ps[16], ds[16];
                        tc::tmem_ld32(ts + 32 * h, s);
                        tc::tmem_ld32(td + 32 * h, d);
                        tc::tmem_wait_ld();
                        if (h) {
                            tc::tc_fence_before();
                            __syncwarp();
                            if (lane == 0) tc::mbar_arrive(&d_free[dbuf]);
                        }
                        const uint32_t bit = h ? bits[1] : bits[0];
#pragma unroll
                        for (int e = 0; e < 32; e += 4) {
                            // pairs: p = 2^(c S - lse'), dS = p (scale dP - scale delta)
                            uint64_t l2[2] = {row_l, row_l}, d2[2] = {row_d, row_d};
                            if (DKV) {
                                const ulonglong2 lv = cl[8 * h + e / 4], dv = cd[8 * h + e / 4];
                                l2[0] = lv.x; l2[1] = lv.y; d2[0] = dv.x; d2[1] = dv.y;
                            }
#pragma unroll
                            for (int u = 0; u < 2; ++u) {
                                const int k = e + 2 * u;
                                const uint64_t y = fma2(pair(__uint_as_float(s[k]), __uint_as_float(s[k + 1])), c2, l2[u]);
                                const uint64_t z = fma2(pair(__uint_as_float(d[k]), __uint_as_float(d[k + 1])), sc2, d2[u]);
                                float p0 = ex2(low(y)), p1 = ex2(high(y));
                                const uint64_t x = mul2(pair(p0, p1), z);
                                float x0 = low(x), x1 = high(x);
                                if (!whole) {                      // (dk, dv: rows that do not count are dropped at the end)
                                    x0 = bit >> k & 1u ? x0 : 0.f;
                                    x1 = bit >> (k + 1) & 1u ? x1 : 0.f;
                                }
                                if (DKV) ps[k / 2] = pack2(p0, p1);
                                ds[k / 2] = pack2(x0, x1);
                            }
                        }
                        // over scores that have been read: p in the first half of their columns, dS in the other
                        if (DKV) tc::tmem_st16(ts + 32 * h, ps);
                        tc::tmem_st16(ts + 32 * h + 16, ds);
                    }
                    if (!whole) {
                        const int cols = left - j * BC >= BC ? BC : (left - j * BC + 15) & ~15;
                        const uint32_t out0 = ~bits[0] & low_bits(cols), out1 = ~bits[1] & low_bits(cols - 32);
                        if (out0 | out1) {                         // K has landed: S is complete
                            uint8_t* kt = ring1 + slot * M::b;
                            constexpr int PER = 8 * NCH;           // 16-byte pieces of a row
#pragma unroll
                            for (int u = 0; u < BC * PER / 128; ++u) {
                                const uint32_t i = u * 128u + r, k = i / PER, piece = i % PER;
                                if ((k < 32 ? out0 >> k : out1 >> (k - 32)) & 1u)
                                    *reinterpret_cast<uint4*>(kt + (piece >> 3) * kColChunk + k * 128 + (piece & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            tc::fence_proxy_async();
                        }
                    }
                    tc::tmem_wait_st();
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&p_full[buf]);
                }
                if (++buf == NS) { buf = 0; buf_ph ^= 1u; }
                if (++dbuf == ND) dbuf = 0;
                if (++slot == N1) { slot = 0; slot_ph ^= 1u; }
            }
        }
        if (!ok && lane == 0) fail();
        __syncwarp();
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        // ------------------------------------------------------------------ results
        const int q = warp & 3, r = q * 32 + lane;
        uint8_t* mine = staging + (uint32_t)q * kStage;
        uint32_t set = 0, ph = 0;
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            ok = see(n);
            if (!ok) break;
            const Item it = queue[n % kQueue];
            leave(n);
            if (!it.live) break;
            const uint8_t* mask = a.where.mask ? a.where.mask + (a.where.offsets ? 0 : (long long)it.enc * a.where.n_kv) + it.row : nullptr;
            const bool keep = !DKV || (r < it.left && (!mask || mask[r] != 0));    // states that do not count: zeros, whatever the sums are
            const int seq = DKV ? it.enc : it.idx, tok0 = DKV ? it.row : it.row0;
            const bool split = a.parts > 1, whole = a.d % (split ? 4 : 8) == 0;
            const int rows = it.limit - 32 * q;
            // the warp's first row of either result, and how far rows lie apart
            uint8_t* dst[DKV ? 2 : 1];
            long long apart[DKV ? 2 : 1];
#pragma unroll
            for (int o = 0; o < (DKV ? 2 : 1); ++o) {
                const CrossMat& mat = o ? a.o2 : a.o1;
                dst[o] = split ? reinterpret_cast<uint8_t*>(a.part_out + (((long long)it.part * 2 + o) * a.part_rows +
                                                                          ((long long)seq * a.where.kv_rows + tok0 + 32 * q) * a.kv_heads + it.head) * a.d) :
                                 reinterpret_cast<uint8_t*>(const_cast<void*>(mat.p)) + 2 * (seq * mat.seq + (long long)(tok0 + 32 * q) * mat.tok + it.head * mat.head);
                apart[o] = split ? 4ll * a.kv_heads * a.d : 2 * mat.tok;
            }
            ok = cross_tc::wait(&acc_full[set], ph, abort_flag);
            if (!ok) break;
            tc::tc_fence_after();
#pragma unroll
            for (int o = 0; o < (DKV ? 2 : 1); ++o) {
                const uint32_t acc = tmem + M::acc_col + set * M::acc_set + o * W + ((uint32_t)(q * 32) << 16);
                auto flush = [&](int col, int n) {       // n pieces of 16 bytes of every row, from byte `col`; neighbours by neighbouring lanes
                    __syncwarp();
                    if (n == 8) {
                        uint8_t* to = dst[o] + (lane >> 3) * apart[o] + col + 16 * (lane & 7);
                        const uint8_t* from = mine + (lane >> 3) * 128;
                        uint4 v[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = *reinterpret_cast<const uint4*>(from + i * 512 + 16 * ((lane & 7) ^ (lane >> 3) ^ (4 * (i & 1))));
#pragma unroll
                        for (int i = 0; i < 8; ++i)
                            if (4 * i + (lane >> 3) < rows) *reinterpret_cast<uint4*>(to + 4 * i * apart[o]) = v[i];
                    } else {
                        const int magic = (65535 + n) / n;
#pragma unroll 1
                        for (int i = lane; i < 32 * n; i += 32) {
                            const int row = i * magic >> 16, piece = i - row * n;
                            if (row < rows) *reinterpret_cast<uint4*>(dst[o] + row * apart[o] + col + 16 * piece) = *reinterpret_cast<const uint4*>(mine + row * 128 + 16 * (piece ^ (row & 7)));
                        }
                    }
                    __syncwarp();
                };
#pragma unroll 1
                for (int c0 = 0; c0 < a.d; c0 += 32) {
                    uint32_t v[32];
                    tc::tmem_ld32(acc + c0, v);
                    tc::tmem_wait_ld();
                    if (o == (DKV ? 1 : 0) && c0 + 32 >= a.d) {
                        tc::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) tc::mbar_arrive(&acc_free[set]);
                    }
                    if (rows <= 0) continue;
                    if (!keep) {
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0u;
                    }
                    if (!whole) {
#pragma unroll
                        for (int e = 0; e < 32; ++e)
                            if (c0 + e < a.d && lane < rows) {
                                if (split) reinterpret_cast<float*>(dst[o] + lane * apart[o])[c0 + e] = __uint_as_float(v[e]);
                                else reinterpret_cast<__nv_bfloat16*>(dst[o] + lane * apart[o])[c0 + e] = __float2bfloat16(__uint_as_float(v[e]));
                            }
                        __syncwarp();
                    } else if (split) {
#pragma unroll
                        for (int u = 0; u < 8; ++u) *reinterpret_cast<uint4*>(mine + lane * 128 + 16 * (u ^ (lane & 7))) = make_uint4(v[4 * u], v[4 * u + 1], v[4 * u + 2], v[4 * u + 3]);
                        flush(4 * c0, a.d - c0 < 32 ? (a.d - c0) / 4 : 8);
                    } else {
                        const int first = (c0 & 32) / 8;
#pragma unroll
                        for (int u = 0; u < 4; ++u) {
                            uint32_t pk[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) pk[e] = pack2(__uint_as_float(v[8 * u + 2 * e]), __uint_as_float(v[8 * u + 2 * e + 1]));
                            *reinterpret_cast<uint4*>(mine + lane * 128 + 16 * ((first + u) ^ (lane & 7))) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                        }
                        const int from = c0 & ~63;
                        if ((c0 & 32) || c0 + 32 >= a.d) flush(2 * from, a.d - from < 64 ? (a.d - from) / 8 : 8);
                    }
                }
            }
            if (++set == NA) { set = 0; ph ^= 1u; }
        }
        if (!ok && lane == 0) fail();
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 12) {
            // ------------------------------------------------------------------ TMA loads
            if (lane == 0) { tc::tma_prefetch_desc(&mapA1); tc::tma_prefetch_desc(&mapA2); tc::tma_prefetch_desc(&mapB1); tc::tma_prefetch_desc(&mapB2); }
            uint32_t set = 0, a_ph = 1, s1 = 0, ph1 = 1, s2 = 0, ph2 = 1;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = see(n);
                if (!ok) break;
                const Item it = queue[n % kQueue];
                leave(n);
                if (!it.live) break;
                Columns col;
                if (DKV) col.seek(a, it);
                auto rows_load = [&]() {
                    ok = cross_tc::wait(&a_empty[set], a_ph, abort_flag);
                    if (!ok) return;
                    if (tc::elect_one()) {
                        tc::mbar_expect_tx(&a_full[set], 2 * M::a);
                        const int seq = DKV ? it.enc : it.idx, tok = DKV ? it.row : it.row0;
                        for (int ch = 0; ch < NCH; ++ch) {
                            load_4d(tc::smem_u32(sA + (2 * set) * M::a + ch * kChunk), &mapA1, &a_full[set], 64 * ch, it.head * (DKV ? a.k_head_mul : a.q_head_mul), tok,
                                    seq * (DKV ? a.k_seq_mul : a.q_seq_mul));
                            load_4d(tc::smem_u32(sA + (2 * set + 1) * M::a + ch * kChunk), &mapA2, &a_full[set], 64 * ch, it.head * (DKV ? a.v_head_mul : a.g_head_mul), tok,
                                    seq * (DKV ? a.v_seq_mul : a.g_seq_mul));
                        }
                    }
                    __syncwarp();
                    if (++set == AB) { set = 0; a_ph ^= 1u; }
                };
                if (AB > 1) rows_load();
                for (int j = 0; ok && j < it.tiles; ++j) {
                    const int seq = DKV ? col.s : it.enc, head = DKV ? it.kv_head * a.group + col.g : it.kv_head, tok = DKV ? col.t * BC : it.row + j * BC;
                    ok = cross_tc::wait(&b1_empty[s1], ph1, abort_flag);
                    if (ok && tc::elect_one()) {
                        tc::mbar_expect_tx(&b1_full[s1], M::b);
                        for (int ch = 0; ch < NCH; ++ch)
                            load_4d(tc::smem_u32(ring1 + s1 * M::b + ch * kColChunk), &mapB1, &b1_full[s1], 64 * ch, head * (DKV ? a.q_head_mul : a.k_head_mul), tok,
                                    seq * (DKV ? a.q_seq_mul : a.k_seq_mul));
                    }
                    __syncwarp();
                    if (ok) ok = cross_tc::wait(&b2_empty[s2], ph2, abort_flag);
                    if (ok && tc::elect_one()) {
                        tc::mbar_expect_tx(&b2_full[s2], M::b);
                        for (int ch = 0; ch < NCH; ++ch)
                            load_4d(tc::smem_u32(ring2 + s2 * M::b + ch * kColChunk), &mapB2, &b2_full[s2], 64 * ch, head * (DKV ? a.g_head_mul : a.v_head_mul), tok,
                                    seq * (DKV ? a.g_seq_mul : a.v_seq_mul));
                    }
                    __syncwarp();
                    if (++s1 == N1) { s1 = 0; ph1 ^= 1u; }
                    if (++s2 == N2) { s2 = 0; ph2 ^= 1u; }
                    if (AB == 1 && j == 0 && ok) rows_load();        // one set: while the last item's products still read it, a tile may come
                    if (DKV) col.next(a, it.idx);
                }
            }
            if (!ok) {
                if (lane == 0) fail();
                const long long t0 = clock64();          // loads in flight must land before the shared memory is given back
                while (clock64() - t0 < 400000ll) { }
            }
            __syncwarp();
        } else if (warp == 13 && DKV) {
            // ------------------------------------------------------------------ the tokens' lse (in log2) and delta, beside their tiles
            uint32_t slot = 0, ph = 1;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = see(n);
                if (!ok) break;
                const Item it = queue[n % kQueue];
                leave(n);
                if (!it.live) break;
                Columns col;
                col.seek(a, it);
                for (int j = 0; ok && j < it.tiles; ++j) {
                    float l[2], dl[2];
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int t = col.t * BC + lane + 32 * u;
                        const long long i = ((long long)col.s * a.heads + it.kv_head * a.group + col.g) * a.n_q + t;
                        const float v = t < a.n_q ? __ldg(a.lse + i) : -INFINITY;
                        l[u] = v == -INFINITY ? -INFINITY : -1.4426950408889634f * v;    // tokens without a state, or behind the last: p = 0
                        dl[u] = t < a.n_q ? -a.scale * __ldg(a.delta + i) : 0.f;
                    }
                    ok = cross_tc::wait(&b1_empty[slot], ph, abort_flag);
                    if (!ok) break;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        stats[slot * 2 * BC + lane + 32 * u] = l[u];
                        stats[slot * 2 * BC + BC + lane + 32 * u] = dl[u];
                    }
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&b1_full[slot]);
                    if (++slot == N1) { slot = 0; ph ^= 1u; }
                    col.next(a, it.idx);
                }
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp == 14 || warp == 15) {
            // ------------------------------------------------------------------ S; dP
            const bool first = warp == 14;
            const uint32_t leader = tc::elect_one() ? 1u : 0u, idesc = tc::idesc_bf16(BR, BC);
            const uint32_t slots = first ? N1 : N2, bufs = first ? NS : ND;
            const uint64_t a_desc = tc::smem_desc(tc::smem_u32(sA) + (first ? 0 : M::a), 1024, 2), b_desc = tc::smem_desc(tc::smem_u32(first ? ring1 : ring2), 1024, 2);
            const uint32_t out = tmem + (first ? 0 : M::dp_col);
            uint64_t *full = first ? b1_full : b2_full, *free = first ? s_free : d_free;
            uint32_t set = 0, a_ph = 0, slot = 0, slot_ph = 0, buf = 0, buf_ph = 1, sbuf = 0;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = see(n);
                if (!ok) break;
                const int live = queue[n % kQueue].live, tiles = queue[n % kQueue].tiles;
                leave(n);
                if (!live) break;
                ok = cross_tc::wait(&a_full[set], a_ph, abort_flag);
                const uint64_t x = a_desc + (2 * set) * (M::a >> 4);
                for (int j = 0; ok && j < tiles; ++j) {
                    ok = cross_tc::wait2(&full[slot], slot_ph, &free[buf], buf_ph, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const uint64_t y = b_desc + slot * (M::b >> 4);
#pragma unroll
                    for (int k = 0; k < 4 * NCH; ++k)
                        if (k < ks) tc::mma_bf16_if(leader, out + buf * 64u, x + ((k >> 2) * (kChunk >> 4) + (k & 3) * 2), y + ((k >> 2) * (kColChunk >> 4) + (k & 3) * 2), idesc, k != 0);
                    tc::mma_commit_if(leader, &s_full[sbuf]);
                    if (!DKV && !first) tc::mma_commit_if(leader, &b2_empty[slot]);
                    if (++slot == slots) { slot = 0; slot_ph ^= 1u; }
                    if (++buf == bufs) { buf = 0; buf_ph ^= 1u; }
                    if (++sbuf == NS) sbuf = 0;
                }
                if (ok) tc::mma_commit_if(leader, &a_empty[set]);
                if (++set == AB) { set = 0; a_ph ^= 1u; }
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp == 17 || (DKV && warp == 18)) {
            // ------------------------------------------------------------------ the accumulating products: dq or dk; dv
            const bool first = warp == 17;
            const uint32_t leader = tc::elect_one() ? 1u : 0u, idesc = tc::idesc_bf16(BR, ks * 16) | kBMajorMN;
            const uint64_t b_desc = desc_mn(tc::smem_u32(first ? ring1 : ring2), kColChunk);
            const uint32_t slots = first ? N1 : N2;
            uint64_t* empty = first ? b1_empty : b2_empty;
            uint32_t slot = 0, buf = 0, buf_ph = 0, set = 0, acc_ph = 1;
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = see(n);
                if (!ok) break;
                const int live = queue[n % kQueue].live, tiles = queue[n % kQueue].tiles, left = queue[n % kQueue].left;
                leave(n);
                if (!live) break;
                ok = cross_tc::wait(&acc_free[set], acc_ph, abort_flag);
                const uint32_t acc = tmem + M::acc_col + set * M::acc_set + (first ? 0 : W);
                for (int j = 0; ok && j < tiles; ++j) {
                    ok = cross_tc::wait(&p_full[buf], buf_ph, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const int cols = DKV || left - j * BC >= BC ? BC : (left - j * BC + 15) & ~15;
                    const uint32_t x = tmem + buf * 64u + (first ? 16u : 0u);        // dS; p
                    const uint64_t y = b_desc + slot * (M::b >> 4);
#pragma unroll
                    for (int k = 0; k < BC / 16; ++k)
                        if (DKV || 16 * k < cols) mma_ts_if(leader, acc, x + 8u * k + 16u * (k / 2), y + k * (2048u >> 4), idesc, j > 0 || k > 0);
                    tc::mma_commit_if(leader, &s_free[buf]);
                    tc::mma_commit_if(leader, &empty[slot]);
                    if (++slot == slots) slot = 0;
                    if (++buf == NS) { buf = 0; buf_ph ^= 1u; }
                }
                if (ok) tc::mma_commit_if(leader, &acc_full[set]);
                if (++set == NA) { set = 0; acc_ph ^= 1u; }
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp == 19) {
            // ------------------------------------------------------------------ the items that have a column tile
            bool ok = true;
            long long i = blockIdx.x;
            auto next_item = [&]() {
                if (DKV) {
                    unsigned long long v = 0;
                    if (lane == 0) v = atomicAdd(a.next, 1ull);
                    i = (long long)__shfl_sync(0xffffffffu, v, 0);
                }
                const Item it = item_of<DKV, ROWS>(a, i);
                if (!DKV) i += gridDim.x;
                return it;
            };
            for (uint32_t n = 0; ok; ++n) {
                // dk, dv: no sooner than the item before is begun, so that the CTAs end together
                if (DKV) ok = cross_tc::wait(&item_free[n % kQueue], (n / kQueue & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                Item it = next_item();
                while (it.live && it.tiles == 0) it = next_item();
                if (!DKV) ok = cross_tc::wait(&item_free[n % kQueue], (n / kQueue & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                if (lane == 0) {
                    queue[n % kQueue] = it;
                    tc::mbar_arrive(&item_full[n % kQueue]);
                }
                __syncwarp();
                if (!it.live) break;
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp == 16) {
            // ------------------------------------------------------------------ rows that nothing reaches
            for (long long i = blockIdx.x; i < a.items; i += gridDim.x) {
                const Item it = item_of<DKV, ROWS>(a, i);
                if (ROWS && !it.live) break;
                const int skip = it.tiles > 0 ? BR : 0, rows = (DKV || it.limit < BR ? it.limit : BR) - skip, seq = DKV ? it.enc : it.idx, tok0 = (DKV ? it.row : it.row0) + skip;
                if (rows <= 0) continue;
                for (int o = 0; o < (DKV ? 2 : 1); ++o) {
                    const CrossMat& mat = o ? a.o2 : a.o1;
                    if (a.parts > 1)
                        zero_rows(a.part_out + (((long long)it.part * 2 + o) * a.part_rows + ((long long)seq * a.where.kv_rows + tok0) * a.kv_heads + it.head) * a.d, 4ll * a.kv_heads * a.d,
                                  rows, 4 * a.d, lane);
                    else
                        zero_rows(reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(mat.p)) + seq * mat.seq + (long long)tok0 * mat.tok + it.head * mat.head, 2 * mat.tok, rows,
                                  2 * a.d, lane);
                }
            }
        }
    }
    // ---------------------------------------------------------------------- teardown
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 12) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, 512); }
}

// dk and dv from their parts: a warp per state and key head, parts in order
template <typename E> __global__ void __launch_bounds__(256) cross_bwd_join_kernel(const CrossArgs a, int parts, const float* part_out, long long part_rows) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31;
    // packed: the rows from the first sequence's first to the last's last
    long long first = 0, last = (long long)a.where.n_enc * a.where.n_kv;
    if (a.where.offsets) {
        first = min(max(__ldg(a.where.offsets), 0), a.where.kv_rows);
        last = min(max(__ldg(a.where.offsets + a.where.n_enc), 0), a.where.kv_rows);
    }
    for (long long i = first * a.kv_heads + (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < last * a.kv_heads; i += (long long)gridDim.x * 8) {
        const int h = (int)(i % a.kv_heads);
        const long long row = i / a.kv_heads;
        const int e = a.where.offsets ? 0 : (int)(row / a.where.n_kv), j = (int)(row - (long long)e * a.where.n_kv);
        for (int o = 0; o < 2; ++o) {
            const CrossMat& mat = o ? a.dv : a.dk;
            E* dst = reinterpret_cast<E*>(const_cast<void*>(mat.p)) + e * mat.seq + j * mat.tok + h * mat.head;
            for (int c = lane; c < a.d; c += 32) {
                float v = 0.f;
                for (int p = 0; p < parts; ++p) v += part_out[(((long long)p * 2 + o) * part_rows + i) * a.d + c];
                if constexpr (sizeof(E) == 4) dst[c] = v;
                else dst[c] = __float2bfloat16(v);
            }
        }
    }
}

template <bool DKV, bool ROWS, int NCH, int W, int AB, int N1, int N2, int NS, int ND, int NA>
int launch(const CUtensorMap (&m)[4], const Args& a, cudaStream_t s) {
    auto kernel = cross_bwd_kernel<DKV, ROWS, NCH, W, AB, N1, N2, NS, ND, NA>;
    constexpr uint32_t bytes = Mem<DKV, NCH, W, AB, N1, N2, NS, ND, NA>::bytes;
    FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    const int grid = (int)(a.items < kSms ? a.items : kSms);
    return free_launch(free_overlap_for_rows((long long)a.n_seq * a.n_q), kernel, dim3(grid), dim3(kThreads), bytes, s, m[0], m[1], m[2], m[3], a);
}

// (heads of 72 with two buffers of S instead of three: 116 us for 107; with five and three slots of the ring for four each 114)
template <bool ROWS> int launch_dkv(int d, const CUtensorMap (&m)[4], const Args& a, cudaStream_t s) {
    return d <= 64 ? launch<true, ROWS, 1, 64, 2, 6, 6, 3, 3, 1>(m, a, s) : d <= 96 ? launch<true, ROWS, 2, 96, 1, 4, 4, 3, 2, 1>(m, a, s) :
                     launch<true, ROWS, 2, 128, 1, 4, 4, 2, 2, 1>(m, a, s);
}

Args args_of(const CrossArgs& c) {
    Args a{};
    a.where = c.where;
    a.n_seq = c.n_seq; a.n_q = c.n_q; a.heads = c.heads; a.kv_heads = c.kv_heads; a.d = c.d; a.group = c.group;
    a.q_seq_mul = c.q.seq > 0; a.q_head_mul = c.q.head > 0; a.g_seq_mul = c.g.seq > 0; a.g_head_mul = c.g.head > 0;
    a.k_seq_mul = c.k.seq > 0; a.k_head_mul = c.k.head > 0; a.v_seq_mul = c.v.seq > 0; a.v_head_mul = c.v.head > 0;
    a.scale = c.scale; a.c = c.scale * 1.4426950408889634f;
    a.lse = c.lse; a.delta = c.delta; a.err = c.err;
    a.parts = 1;
    return a;
}

}  // namespace

bool cross_bwd_tc_supported(const CrossArgs& c) {
    if (c.where.n_kv < 1 || c.n_seq < 1 || c.n_q < 1) return false;
    const int enc = c.where.offsets ? 1 : c.where.n_enc, rows = c.where.kv_rows;
    using cross_tc::mappable;
    return mappable(c.q, c.n_seq, c.n_q, c.heads) && mappable(c.g, c.n_seq, c.n_q, c.heads) && mappable(c.k, enc, rows, c.kv_heads) && mappable(c.v, enc, rows, c.kv_heads);
}

// Parts of the tokens' tiles where the blocks of states leave SMs without one: two tiles at least, an fp32 row of dk and dv each.  Items of
// more than a million tiles, a second's work, are split too: waits for them give up after two.
int cross_bwd_tc_parts(const CrossArgs& c) {
    const long long items = cross_blocks(c.where, BR) * c.kv_heads;
    const long long all = (long long)c.n_seq * c.group * ((c.n_q + BC - 1) / BC), tiles = all / (c.where.n_enc > 0 ? c.where.n_enc : 1);
    long long p = items >= kSms || items < 1 ? 1 : (2 * kSms + items - 1) / items;
    if (p > tiles / 2) p = tiles / 2;
    if (p > cross_parts_held(c)) p = cross_parts_held(c);
    const long long least = ((c.where.seq_of ? all : tiles) + (1 << 20) - 1) >> 20;
    if (p < least) p = least;
    return p < 1 ? 1 : (int)p;
}

int cross_bwd_tc_dq(const CrossArgs& c, cudaStream_t s) {
    Args a = args_of(c);
    const int enc = c.where.offsets ? 1 : c.where.n_enc, rows = c.where.kv_rows;
    a.blocks = (c.n_q + BR - 1) / BR;
    a.items = (long long)c.n_seq * c.heads * a.blocks;
    a.o1 = a.o2 = c.dq;
    CUtensorMap m[4];
    using cross_tc::map_heads;
    FREE_TRY(map_heads(&m[0], c.q, c.n_seq, c.n_q, c.heads, c.d, 1, BR));
    FREE_TRY(map_heads(&m[1], c.g, c.n_seq, c.n_q, c.heads, c.d, 1, BR));
    FREE_TRY(map_heads(&m[2], c.k, enc, rows, c.kv_heads, c.d, 1, BC));
    FREE_TRY(map_heads(&m[3], c.v, enc, rows, c.kv_heads, c.d, 1, BC));
    // two sets of sums, so that results leave while the next item's are formed (24 x 1024 tokens of 16 heads of 72: 92 us; one set and a
    // third buffer of dP 95)
    if (c.d <= 64) return launch<false, false, 1, 64, 2, 6, 4, 3, 3, 2>(m, a, s);
    return c.d <= 96 ? launch<false, false, 2, 96, 2, 3, 2, 3, 2, 2>(m, a, s) : launch<false, false, 2, 128, 2, 3, 2, 2, 2, 2>(m, a, s);
}

int cross_bwd_tc_dkv(const CrossArgs& c, int parts, float* part_out, cudaStream_t s) {
    Args a = args_of(c);
    const int enc = c.where.offsets ? 1 : c.where.n_enc, rows = c.where.kv_rows;
    a.blocks = cross_blocks_per(c.where, BR);
    a.parts = parts; a.part_out = part_out; a.part_rows = (long long)enc * rows * c.kv_heads;
    a.items = cross_blocks(c.where, BR) * c.kv_heads * parts;
    a.next = c.next;
    a.o1 = c.dk; a.o2 = c.dv;
    CUtensorMap m[4];
    using cross_tc::map_heads;
    FREE_TRY(map_heads(&m[0], c.k, enc, rows, c.kv_heads, c.d, 1, BR));
    FREE_TRY(map_heads(&m[1], c.v, enc, rows, c.kv_heads, c.d, 1, BR));
    FREE_TRY(map_heads(&m[2], c.q, c.n_seq, c.n_q, c.heads, c.d, 1, BC));
    FREE_TRY(map_heads(&m[3], c.g, c.n_seq, c.n_q, c.heads, c.d, 1, BC));
    FREE_TRY(a.blocks ? launch_dkv<false>(c.d, m, a, s) : launch_dkv<true>(c.d, m, a, s));
    if (parts == 1) return FREE_OK;
    return cross_bwd_join(FREE_BF16, c, parts, part_out, s);
}

int cross_bwd_join(int dtype, const CrossArgs& c, int parts, const float* part_out, cudaStream_t s) {
    const long long n = (c.where.offsets ? c.where.kv_rows : (long long)c.where.n_enc * c.where.n_kv) * c.kv_heads, ctas = (n + 7) / 8;
    const long long rows = (long long)(c.where.offsets ? 1 : c.where.n_enc) * c.where.kv_rows * c.kv_heads;
    auto kernel = dtype == FREE_FP32 ? cross_bwd_join_kernel<float> : cross_bwd_join_kernel<__nv_bfloat16>;
    return free_launch(false, kernel, dim3((unsigned)(ctas < kSms * 8 ? ctas : kSms * 8)), dim3(256), 0, s, c, parts, part_out, rows);
}
