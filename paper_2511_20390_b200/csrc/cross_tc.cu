// Attention to an encoder's states on the tensor cores (bf16 operands, fp32 softmax and accumulation), forward.
//
//   S = Q K^T (tcgen05, fp32 in tensor memory);  p = 2^(c S - m), c = scale log2 e;  O += p V;  out = O / sum p
//
// Persistent CTAs, one per SM.  An item is two tiles of 128 rows of one (sequence, key head), rows being (token, query head of the key
// head's group), so that shared key heads are read once.  A warpgroup per tile does the softmax, a thread per row; one warp
// loads tiles by TMA, one issues the MMAs.  While one tile's exponentials run, the tensor pipe does the other tile's products.
//   - p goes back to tensor memory, over its own scores, as the left operand of O += p V: it never passes shared memory.
//   - Blocks of 64 states, the scores of two of them per tile in tensor memory: while the softmax works on one, the next (of the next
//     item, too) is there already.  Scores are issued right behind the O += p V that reads the p in their columns; the pipe runs in order.
//   - V is the right operand as it lies in memory (contraction along its rows), so nothing is transposed.
//   - The maximum that p is taken against moves only when it has grown by 2^8; then O is rescaled in tensor memory.
//   - The last block of a sequence costs the 16-column steps that it has.  States that do not count: scores are replaced by -inf, and the
//     rows of V are zeroed in shared memory (0 x NaN would be NaN).
// Long states and few rows: the states are split into parts, each with its own softmax, joined by cross_join_kernel.
#include "cross_tc.cuh"

namespace cross_tc {

bool mappable(const CrossMat& m, int n_seq, int n_tok, int heads) {
    auto fits = [](long long stride, int n) { return n <= 1 || (stride % 8 == 0 && stride < (1LL << 38)); };
    return free_aligned16(m.p) && fits(m.seq, n_seq) && fits(m.tok, n_tok) && m.tok * (n_tok > 1) >= (n_tok > 1) && fits(m.head, heads);
}
int map_heads(CUtensorMap* map, const CrossMat& m, int n_seq, int n_tok, int heads, int d, int heads_box, int tok_box) {
    const bool hs = heads > 1 && m.head > 0, ss = n_seq > 1 && m.seq > 0;
    const uint64_t dims[4] = {(uint64_t)d, hs ? (uint64_t)heads : 1, (uint64_t)n_tok, ss ? (uint64_t)n_seq : 1};
    const uint64_t strides[3] = {hs ? (uint64_t)m.head * 2 : 256, n_tok > 1 ? (uint64_t)m.tok * 2 : 256, ss ? (uint64_t)m.seq * 2 : 256};
    const uint32_t box[4] = {64, (uint32_t)heads_box, (uint32_t)tok_box, 1};
    return free_tensor_map_4d(map, m.p, dims, strides, box);
}

}  // namespace cross_tc

namespace {

using namespace cross_tc;

constexpr int BQ = 128, BK = 64;
constexpr int kThreads = 512, kSms = 148;     // warps 0 - 7 softmax, 8 - 11 results, 12 loads, 13, 14 MMAs
// Registers: 512 x 128 at launch, of which the softmax takes 152 each (64 scores of a row at a time) and the others keep 104.
constexpr int kSoftmaxRegs = 152, kOtherRegs = 104;
static_assert(256 * (kSoftmaxRegs + kOtherRegs) <= kThreads * 128, "registers of the launch");
constexpr uint32_t kChunk = BQ * 128, kKvChunk = BK * 128;      // rows x 64 channels, 128-byte rows
constexpr uint32_t kTmemCols = 512;           // scores: tile w, buffer b at column 128 w + 64 b; O of tile w at 256 + 128 w
constexpr uint32_t kCtrl = 2048;              // barriers, and 1 / sum p of the rows of both tiles
template <int NCH> struct Mem {               // NCH: chunks of 64 channels
    static constexpr int slots = NCH == 1 ? 12 : 6;
    static constexpr uint32_t q = NCH * kChunk, kv = NCH * kKvChunk;
    static constexpr uint32_t bytes = 1024 + kCtrl + 2 * q + slots * kv + 2 * q;
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
};

// n / d for n below 2^31: a product with m = ceil(2^(31 + s) / d), s = ceil(log2 d), whose excess m d - 2^(31 + s) < 2^s is too small
// to reach the next quotient.
struct Div {
    uint32_t m, s;
    __device__ __forceinline__ uint32_t operator()(uint32_t n) const { return (uint32_t)((uint64_t)n * m >> (31 + s)); }
};
Div div_by(uint32_t d) {
    uint32_t s = 0;
    while ((1ull << s) < d) ++s;
    return Div{(uint32_t)(((1ull << (31 + s)) + d - 1) / d), s};
}

struct Args {
    CrossWhere where;
    Div by_parts, by_pairs, by_kv_heads, by_share;
    int n_q, heads, d, group, tt;             // tt: tokens of a tile
    int tiles;                                // of an item
    uint32_t pairs, parts, items;             // pairs: of tiles, per (sequence, key head); parts of the states
    uint32_t kv_heads;
    int kv_head_mul, kv_seq_mul, v_head_mul, v_seq_mul, q_seq_mul, q_head_mul;      // 0 where one matrix serves all
    long long rows;                           // n_seq * heads * n_q
    float c, ln2_over_c, scale;               // c: scale * log2 e
    float *lse, *part_out, *part_lse;
    uint32_t* err;
};

// One item: its place and the blocks of states that it covers.
struct Item {
    int s, kh, t0, part, tiles, b0, nb, limit;      // limit: tokens; blocks b0 .. b0 + nb - 1
    CrossSpan sp;
};
__device__ __forceinline__ Item item_of(const Args& a, uint32_t i) {
    Item it;
    const uint32_t k = a.by_parts(i), sh = a.by_pairs(k);
    it.part = (int)(i - k * a.parts);
    const int pair = (int)(k - sh * a.pairs);
    it.s = (int)a.by_kv_heads(sh); it.kh = (int)(sh - it.s * a.kv_heads);
    it.t0 = pair * a.tiles * a.tt;
    it.tiles = a.tiles == 2 && it.t0 + a.tt < a.n_q ? 2 : 1;
    it.sp = cross_span_of_enc(a.where, a.where.seq_of ? __ldg(a.where.seq_of + it.s) : (int)a.by_share(it.s));
    const int blocks = (it.sp.len + BK - 1) / BK;
    it.b0 = 0; it.nb = blocks;
    if (a.parts > 1) {
        it.b0 = (int)((long long)blocks * it.part / a.parts);
        it.nb = (int)((long long)blocks * (it.part + 1) / a.parts) - it.b0;
    }
    return it;
}
__device__ __forceinline__ int columns_of(const Item& it, int j) {       // of scores, in steps of 16
    const int left = it.sp.len - (it.b0 + j) * BK;
    return left >= BK ? BK : (left + 15) & ~15;
}

// Walks over the blocks of all of a CTA's items that have any.
struct Steps {
    const Args& a;
    uint32_t i, step;
    Item it;
    int j;
    bool live;
    __device__ __forceinline__ Steps(const Args& args, uint32_t first, uint32_t stride) : a(args), i(first - stride), step(stride), j(0), live(true) { next_item(); }
    __device__ __forceinline__ void next_item() {
        for (;;) {
            i += step;
            if (i >= a.items) { live = false; return; }
            it = item_of(a, i);
            j = 0;
            if (it.nb > 0) return;
        }
    }
    __device__ __forceinline__ void next() { if (++j == it.nb) next_item(); }
    __device__ __forceinline__ bool last() const { return j == it.nb - 1; }
};

// One step of 16 of a product, issued by the leader of a converged warp; descriptors differ in their low words only.
__device__ __forceinline__ void mma_ts_if(uint32_t issue, uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate), "r"(issue) : "memory");
}

template <int NCH>
__global__ void __launch_bounds__(kThreads, 1)
cross_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                const __grid_constant__ CUtensorMap mapO, const Args a) {
    using M = Mem<NCH>;
    constexpr uint32_t NS = M::slots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* kv_empty = kv_full + NS;
    uint64_t* q_full = kv_empty + NS;         // [tile]
    uint64_t* q_empty = q_full + 2;
    uint64_t* o_free = q_empty + 2;           // results have been read from tensor memory
    uint64_t* pv_done = o_free + 2;           // every O += p V
    uint64_t* o_full = pv_done + 2;           // an item's last
    uint64_t* inv_full = o_full + 2;
    uint64_t* inv_free = inv_full + 2;
    uint64_t* s_full = inv_free + 2;          // [tile][buffer]
    uint64_t* p_full = s_full + 4;
    uint64_t* group = p_full + 4;             // the warps that write results meet
    uint64_t* turn = group + 1;               // tile 0 has done an item's first exponentials
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(turn + 1);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    float* invs = reinterpret_cast<float*>(smem + 1024);      // [tile][row]
    uint8_t* sQ = smem + kCtrl;
    uint8_t* ring = sQ + 2 * M::q;
    uint8_t* staging = ring + NS * M::kv;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < NS; ++i) { tc::mbar_init(&kv_full[i], 1); tc::mbar_init(&kv_empty[i], 2); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&q_full[i], 1); tc::mbar_init(&q_empty[i], 1); tc::mbar_init(&o_free[i], 4); tc::mbar_init(&pv_done[i], 1); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&o_full[i], 1); tc::mbar_init(&inv_full[i], 4); tc::mbar_init(&inv_free[i], 4); }
        tc::mbar_init(group, 4);
        tc::mbar_init(turn, 4);
        for (int i = 0; i < 4; ++i) { tc::mbar_init(&s_full[i], 1); tc::mbar_init(&p_full[i], 4); }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::fence_proxy_async();
    }
    if (warp == 12) { tc::tmem_alloc(tmem_slot, kTmemCols); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() { *abort_flag = 1; atomicOr(a.err, FREE_DEV_ERR_ATTN); };
    free_grid_dep_wait();                                // only this CTA's shared and tensor memory was touched so far
    free_grid_dep_launch();
    const int ks = (a.d + 15) / 16;                      // 16-channel steps

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ------------------------------------------------------------------ softmax: a warpgroup per tile, a thread per row
        const int w = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t ts = tmem + w * 128u + ((uint32_t)(q * 32) << 16), to = ts + 256u;
        const int row_t = r / a.group, row_h = r - row_t * a.group;
        uint32_t n = 0, ns = 0, inv_ph = 1, turn_ph = 0;    // blocks of the CTA (a pair of slots each), and of this tile, so far
        bool ok = true;
        Item ahead = item_of(a, blockIdx.x);             // its loads are under way while the item before is worked on
        for (uint32_t i = blockIdx.x; ok && i < a.items; i += gridDim.x) {
            const Item it = ahead;
            if (i + gridDim.x < a.items) ahead = item_of(a, i + gridDim.x);
            const uint32_t first = n;
            n += (uint32_t)it.nb;
            if (w >= it.tiles) continue;
            const uint8_t* mask = cross_mask(a.where, it.sp);
            float top = -INFINITY, sum = 0.f;            // maximum in use
            for (int j = 0; j < it.nb; ++j, ++ns) {
                const uint32_t tsb = ts + (ns & 1u) * 64u, bar = 2 * w + (ns & 1u);
                const int left = it.sp.len - (it.b0 + j) * BK;
                const bool whole = left >= BK && !mask;
                ok = tc::wait_uniform(&s_full[bar], ns >> 1 & 1u, abort_flag);
                if (!ok) break;
                tc::tc_fence_after();
                uint32_t x[64];
                tc::tmem_ld64(tsb, x);
                tc::tmem_wait_ld();
                uint32_t bits[2];
                if (!whole) {
                    count_bits(bits, mask, (it.b0 + j) * BK, it.sp.len, lane);
#pragma unroll
                    for (int e = 0; e < 64; ++e) x[e] = bits[e >> 5] >> (e & 31) & 1u ? x[e] : 0xff800000u;
                }
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 64; e += 2) m4[e / 2 & 3] = fmaxf(fmaxf(m4[e / 2 & 3], __uint_as_float(x[e])), __uint_as_float(x[e + 1]));
                const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                const bool grown = !((mx - top) * a.c <= 8.f) && mx > top;      // also the first block with a state that counts
                if (__any_sync(0xffffffffu, grown)) {
                    const float nt = fmaxf(top, mx);
                    const float alpha = nt == -INFINITY ? 1.f : ex2((top - nt) * a.c);
                    top = nt;
                    sum *= alpha;
                    if (j > 0) {
                        ok = tc::wait_uniform(&pv_done[w], (ns - 1u) & 1u, abort_flag);
                        if (!ok) break;
                        tc::tc_fence_after();
                        for (int c = 0; c < ks; ++c) {
                            uint32_t o[16];
                            tc::tmem_ld16(to + 16 * c, o);
                            tc::tmem_wait_ld();
#pragma unroll
                            for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * alpha);
                            tc::tmem_st16(to + 16 * c, o);
                        }
                    }
                }
                const float base = top == -INFINITY ? 0.f : top * a.c;
                // the tiles start an item one behind the other, so that one's exponentials run beside the other's remaining work
                if (j == 0 && it.tiles == 2 && w == 1) {
                    ok = tc::wait_uniform(turn, turn_ph, abort_flag);
                    turn_ph ^= 1u;
                    if (!ok) break;
                }
                float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t pk[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        const float p0 = ex2(fmaf(__uint_as_float(x[32 * c + 2 * e]), a.c, -base)), p1 = ex2(fmaf(__uint_as_float(x[32 * c + 2 * e + 1]), a.c, -base));
                        s4[e & 3] += p0;
                        s4[(e + 2) & 3] += p1;
                        pk[e] = pack2(p0, p1);
                    }
                    tc::tmem_st16(tsb + 16 * c, pk);
                }
                sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                if (j == 0 && it.tiles == 2 && w == 0) {
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(turn);
                }
                if (!whole) {
                    // rows of V that do not count and that the product would read (both tiles' groups write the same zeros)
                    const int cols = left >= BK ? BK : (left + 15) & ~15;
                    const uint32_t out0 = ~bits[0] & low_bits(cols), out1 = ~bits[1] & low_bits(cols - 32);
                    if (out0 | out1) {
                        const uint32_t v = 2u * (first + j) + 1u, slot = v % NS;
                        ok = tc::wait_uniform(&kv_full[slot], v / NS & 1u, abort_flag);
                        if (!ok) break;
                        uint8_t* vt = ring + slot * M::kv;
#pragma unroll 1
                        for (uint32_t o = out0, k0 = 0;; o = out1, k0 = 32) {
                            for (; o; o &= o - 1u) {
                                const uint32_t k = k0 + (uint32_t)__ffs((int)o) - 1u;
                                if ((k & 3u) == (uint32_t)q && lane < 8 * NCH)
                                    *reinterpret_cast<uint4*>(vt + (lane >> 3) * kKvChunk + k * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                            }
                            if (k0) break;
                        }
                        tc::fence_proxy_async();
                    }
                }
                tc::tmem_wait_st();
                tc::tc_fence_before();
                // at most one product of the tile is under way, so that the parity tells which one was the last
                if (j > 0) ok = tc::wait_uniform(&pv_done[w], (ns - 1u) & 1u, abort_flag);
                if (!ok) break;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&p_full[bar]);
            }
            if (!ok) break;
            const int t = it.t0 + w * a.tt + row_t;
            if (row_t < a.tt && t < a.n_q) {
                const long long row = ((long long)it.s * a.heads + it.kh * a.group + row_h) * a.n_q + t;
                const float lse = top == -INFINITY ? -INFINITY : top * a.scale + logf(sum);
                if (a.parts > 1) a.part_lse[it.part * a.rows + row] = lse;
                else if (a.lse) a.lse[row] = lse;
            }
            if (it.nb > 0) {
                ok = tc::wait_uniform(&inv_free[w], inv_ph, abort_flag);
                inv_ph ^= 1u;
                if (!ok) break;
                invs[w * BQ + r] = sum == 0.f ? 0.f : 1.f / sum;
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&inv_full[w]);
            }
        }
        if (!ok && lane == 0) fail();
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 12) {
            // ------------------------------------------------------------------ TMA producer
            if (lane == 0) { tc::tma_prefetch_desc(&mapQ); tc::tma_prefetch_desc(&mapK); tc::tma_prefetch_desc(&mapV); }
            const uint32_t q_bytes = (uint32_t)(a.tt * a.group) * 128u * NCH;
            uint32_t slot = 0, ph = 0, q_ph = 0;             // bit w of q_ph: parity of tile w's loads
            bool ok = true;
            for (Steps st(a, blockIdx.x, gridDim.x); ok && st.live; st.next()) {
                const Item& it = st.it;
                if (st.j == 0)
                    for (int w = 0; ok && w < it.tiles; ++w, __syncwarp()) {
                        ok = tc::wait_uniform(&q_empty[w], (q_ph >> w & 1u) ^ 1u, abort_flag);
                        q_ph ^= 1u << w;
                        if (ok && tc::elect_one()) {
                            tc::mbar_expect_tx(&q_full[w], q_bytes);
                            for (int ch = 0; ch < NCH; ++ch)
                                load_4d(tc::smem_u32(sQ + w * M::q + ch * kChunk), &mapQ, &q_full[w], 64 * ch, it.kh * a.group * a.q_head_mul, it.t0 + w * a.tt, it.s * a.q_seq_mul);
                        }
                    }
                for (int kv = 0; ok && kv < 2; ++kv, __syncwarp()) {
                    ok = tc::wait_uniform(&kv_empty[slot], ph ^ 1u, abort_flag);
                    if (ok && tc::elect_one()) {
                        tc::mbar_expect_tx(&kv_full[slot], M::kv);
                        for (int ch = 0; ch < NCH; ++ch)
                            load_4d(tc::smem_u32(ring + slot * M::kv + ch * kKvChunk), kv ? &mapV : &mapK, &kv_full[slot], 64 * ch,
                                    it.kh * (kv ? a.v_head_mul : a.kv_head_mul), it.sp.row0 + (it.b0 + st.j) * BK, it.sp.enc * (kv ? a.v_seq_mul : a.kv_seq_mul));
                    }
                    if (++slot == NS) { slot = 0; ph ^= 1u; }
                }
            }
            if (!ok) {
                if (lane == 0) fail();
                const long long t0 = clock64();              // loads in flight must land before the shared memory is given back
                while (clock64() - t0 < 400000ll) { }
            }
            __syncwarp();
        } else if (warp == 13 || warp == 14) {
            // ------------------------------------------------------------------ MMA issuers, one per tile: O += p V of a block, then the scores of the block after next
            const int w = warp - 13;
            const uint32_t leader = tc::elect_one() ? 1u : 0u;
            const uint32_t idesc_o = tc::idesc_bf16(BQ, ks * 16) | kBMajorMN;
            const uint64_t q_desc = tc::smem_desc(tc::smem_u32(sQ + w * M::q), 1024, 2), k_desc = tc::smem_desc(tc::smem_u32(ring), 1024, 2);
            const uint64_t v_desc = desc_mn(tc::smem_u32(ring), kKvChunk);
            const uint32_t d_s = tmem + w * 128u, d_o = tmem + 256u + w * 128u;
            uint32_t q_ph = 0, o_ph = 1, s_buf = 0, p_buf = 0, p_ph = 0;
            uint32_t k_slot = 0, k_ph = 0, v_slot = 1, v_ph = 0;
            bool ok = true;
            Steps sc(a, blockIdx.x, gridDim.x), pv = sc;
            // a slot is free when both issuers are done with it: one that has no tile in this item is so as soon as it is full (not
            // earlier, or it would count twice for one use of the slot)
            auto scores = [&]() {
                if (w < sc.it.tiles) {
                    if (sc.j == 0) {
                        ok = tc::wait_uniform(&q_full[w], q_ph, abort_flag);
                        q_ph ^= 1u;
                    }
                    if (ok) ok = tc::wait_uniform(&kv_full[k_slot], k_ph, abort_flag);
                    if (!ok) return;
                    tc::tc_fence_after();
                    const uint32_t idesc = tc::idesc_bf16(BQ, columns_of(sc.it, sc.j)), d = d_s + s_buf * 64u;
                    const uint64_t kd = k_desc + k_slot * (M::kv >> 4);
    #pragma unroll
                    for (int k = 0; k < 4 * NCH; ++k)
                        if (k < ks) tc::mma_bf16_if(leader, d, q_desc + ((k >> 2) * (kChunk >> 4) + (k & 3) * 2), kd + ((k >> 2) * (kKvChunk >> 4) + (k & 3) * 2), idesc, k != 0);
                    tc::mma_commit_if(leader, &s_full[2 * w + s_buf]);
                    s_buf ^= 1u;
                    if (sc.last()) tc::mma_commit_if(leader, &q_empty[w]);
                    tc::mma_commit_if(leader, &kv_empty[k_slot]);
                } else {
                    ok = tc::wait_uniform(&kv_full[k_slot], k_ph, abort_flag);
                    if (!ok) return;
                    if (leader) tc::mbar_arrive(&kv_empty[k_slot]);
                }
                sc.next();
                k_slot += 2;
                if (k_slot >= NS) { k_slot -= NS; k_ph ^= 1u; }
            };
            for (int i = 0; i < 2 && ok && sc.live; ++i) scores();
            while (ok && pv.live) {
                if (w < pv.it.tiles) {
                    if (pv.j == 0) {
                        ok = tc::wait_uniform(&o_free[w], o_ph, abort_flag);
                        o_ph ^= 1u;
                    }
                    if (ok) ok = tc::wait_uniform(&kv_full[v_slot], v_ph, abort_flag);
                    if (ok) ok = tc::wait_uniform(&p_full[2 * w + p_buf], p_ph >> p_buf & 1u, abort_flag);
                    if (!ok) break;
                    tc::tc_fence_after();
                    const int steps = columns_of(pv.it, pv.j) / 16;
                    const uint32_t p = d_s + p_buf * 64u;
                    const uint64_t vd = v_desc + v_slot * (M::kv >> 4);
                    p_ph ^= 1u << p_buf;
                    p_buf ^= 1u;
    #pragma unroll
                    for (int k = 0; k < BK / 16; ++k)
                        if (k < steps) mma_ts_if(leader, d_o, p + 8u * k, vd + k * (2048u >> 4), idesc_o, pv.j > 0 || k > 0);
                    tc::mma_commit_if(leader, &pv_done[w]);
                    if (pv.last()) tc::mma_commit_if(leader, &o_full[w]);
                    tc::mma_commit_if(leader, &kv_empty[v_slot]);
                } else {
                    ok = tc::wait_uniform(&kv_full[v_slot], v_ph, abort_flag);
                    if (!ok) break;
                    if (leader) tc::mbar_arrive(&kv_empty[v_slot]);
                }
                if (sc.live) scores();
                pv.next();
                v_slot += 2;
                if (v_slot >= NS) { v_slot -= NS; v_ph ^= 1u; }
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp < 12) {
            // ------------------------------------------------------------------ results, tile after tile, while the softmax is at the next item
            const int q = warp & 3, r = q * 32 + lane;
            const int row_t = r / a.group, row_h = r - row_t * a.group;
            const bool writer = q == 0 && lane == 0;         // the thread that issues the copies
            uint32_t met = 0, staged = 0, ph = 0;            // ph: bit w, parity of tile w's barriers
            bool ok = true;
            auto meet = [&]() {                              // a bounded wait, as everywhere: a warp that gave up does not come
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(group);
                ok = tc::wait_uniform(group, met++ & 1u, abort_flag);
            };
            for (uint32_t i = blockIdx.x; ok && i < a.items; i += gridDim.x) {
                const Item it = item_of(a, i);
                for (int w = 0; ok && w < it.tiles; ++w) {
                    const uint32_t to = tmem + 256u + w * 128u + ((uint32_t)(q * 32) << 16);
                    uint8_t* mine = staging + (staged & 1u) * M::q;
                    if (a.parts == 1) {
                        if (writer) tc::bulk_wait_read<1>(); // the copies that last used this staging tile have read it
                        meet();
                    }
                    float inv = 0.f;
                    if (ok && it.nb > 0) {
                        ok = tc::wait_uniform(&inv_full[w], ph >> w & 1u, abort_flag);
                        if (ok) ok = tc::wait_uniform(&o_full[w], ph >> w & 1u, abort_flag);
                        ph ^= 1u << w;
                        tc::tc_fence_after();
                        inv = invs[w * BQ + r];
                    }
                    if (!ok) break;
                    const int t = it.t0 + w * a.tt + row_t;
                    const bool row_ok = row_t < a.tt && t < a.n_q;
                    float* dst = a.part_out + (it.part * a.rows + ((long long)it.s * a.heads + it.kh * a.group + row_h) * a.n_q + t) * a.d;
    #pragma unroll 1
                    for (int h = 0; 2 * h < ks; ++h) {       // 32 channels
                        uint32_t o[32];
                        tc::tmem_ld32(to + 32 * h, o);
                        tc::tmem_wait_ld();
                        if (a.parts > 1) {
                            if (row_ok && it.nb > 0) {
    #pragma unroll
                                for (int e = 0; e < 32; ++e)
                                    if (32 * h + e < a.d) dst[32 * h + e] = __uint_as_float(o[e]) * inv;
                            }
                        } else {
    #pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t pk[4];
    #pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    pk[e] = it.nb > 0 ? pack2(__uint_as_float(o[8 * c + 2 * e]) * inv, __uint_as_float(o[8 * c + 2 * e + 1]) * inv) : 0u;
                                *reinterpret_cast<uint4*>(mine + (h >> 1) * kChunk + r * 128 + (((4 * (h & 1) + c) ^ (r & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                            }
                        }
                    }
                    if (it.nb > 0) {
                        tc::tc_fence_before();
                        __syncwarp();
                        if (lane == 0) { tc::mbar_arrive(&o_free[w]); tc::mbar_arrive(&inv_free[w]); }
                    }
                    if (a.parts == 1) {
                        tc::fence_proxy_async();
                        meet();
                        if (ok && writer) {
                            for (int ch = 0; ch < NCH; ++ch) store_4d(&mapO, tc::smem_u32(mine + ch * kChunk), 64 * ch, it.kh * a.group, it.t0 + w * a.tt, it.s);
                            tc::bulk_commit();
                        }
                        ++staged;
                    }
                }
            }
            if (!ok && lane == 0) fail();
            if (writer) tc::bulk_wait<0>();                  // every store complete before the CTA ends
            __syncwarp();
        }
    }
    // ---------------------------------------------------------------------- teardown
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 12) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, kTmemCols); }
}

// out, lse of a row from its parts' own: a warp per row.
template <typename E> __global__ void __launch_bounds__(256) cross_join_kernel(const CrossArgs a, const CrossParts p, long long rows) {
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31;
    for (long long i = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); i < rows; i += (long long)gridDim.x * 8) {
        float top = -INFINITY;
        for (int k = lane; k < p.n; k += 32) top = fmaxf(top, p.lse[k * rows + i]);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
        float sum = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
        if (top != -INFINITY)
            for (int k = 0; k < p.n; ++k) {
                const float l = p.lse[k * rows + i];
                if (l == -INFINITY) continue;                      // a part without a state wrote nothing else
                const float f = expf(l - top);
                sum += f;
                const float* o = p.out + (k * rows + i) * a.d;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (lane + 32 * c < a.d) acc[c] = fmaf(f, o[lane + 32 * c], acc[c]);
            }
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        const int t = (int)(i % a.n_q), h = (int)(i / a.n_q % a.heads), s = (int)(i / a.n_q / a.heads);
        E* out = reinterpret_cast<E*>(const_cast<void*>(a.o.p)) + s * a.o.seq + t * a.o.tok + h * a.o.head;
#pragma unroll
        for (int c = 0; c < 4; ++c)
            if (lane + 32 * c < a.d) {
                if constexpr (sizeof(E) == 4) out[lane + 32 * c] = acc[c] * inv;
                else out[lane + 32 * c] = __float2bfloat16(acc[c] * inv);
            }
        if (a.lse && lane == 0) a.lse[i] = top == -INFINITY ? -INFINITY : top + logf(sum);
    }
}

int tokens_per_tile(const CrossArgs& a) { return BQ / a.group; }

template <int NCH> int launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mo, const Args& a, cudaStream_t s) {
    FREE_CUDA_TRY(cudaFuncSetAttribute(cross_tc_kernel<NCH>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)Mem<NCH>::bytes));
    const int grid = (int)(a.items < kSms ? a.items : kSms);
    return free_launch(free_overlap_for_rows(a.rows / a.heads), cross_tc_kernel<NCH>, dim3(grid), dim3(kThreads), Mem<NCH>::bytes, s, mq, mk, mv, mo, a);
}

// Tiles per item and parts of the states.  Two tiles share the tiles of K and V that are loaded, but where that leaves SMs without an
// item, one is taken; and where that still does, the states are split, into parts of eight blocks at least.
void shape_of(const CrossArgs& a, int* tiles, int* pairs, int* parts) {
    const int tt = tokens_per_tile(a);
    const long long heads = (long long)a.n_seq * a.kv_heads, rows = (a.n_q + tt - 1) / tt;
    *tiles = heads * ((rows + 1) / 2) >= kSms ? 2 : 1;
    *pairs = (int)((rows + *tiles - 1) / *tiles);
    const long long items = heads * *pairs;
    const int most = (a.where.n_kv + 8 * BK - 1) / (8 * BK);
    long long want = items >= kSms ? 1 : (4 * kSms + items - 1) / items;
    if (want > most) want = most;
    *parts = want < 1 ? 1 : (int)want;
}

}  // namespace

bool cross_tc_supported(const CrossArgs& a) {
    if (a.group > BQ || a.where.n_kv < 1) return false;
    const bool packed = a.where.offsets != nullptr;
    const int enc = packed ? 1 : a.where.n_enc, rows = a.where.kv_rows;
    // several query heads in one box: they have to have a stride
    return mappable(a.q, a.n_seq, a.n_q, a.heads) && mappable(a.k, enc, rows, a.kv_heads) && mappable(a.v, enc, rows, a.kv_heads) &&
           mappable(a.o, a.n_seq, a.n_q, a.heads) && (a.group == 1 || a.q.head > 0);
}

CrossParts cross_tc_parts(const CrossArgs& a) {
    int tiles, pairs, parts;
    shape_of(a, &tiles, &pairs, &parts);
    return CrossParts{parts, nullptr, nullptr};
}

int cross_tc_forward(const CrossArgs& c, const CrossParts& parts, cudaStream_t s) {
    Args a{};
    a.where = c.where;
    a.n_q = c.n_q; a.heads = c.heads; a.kv_heads = c.kv_heads; a.d = c.d; a.group = c.group; a.tt = tokens_per_tile(c);
    int pairs, most;
    shape_of(c, &a.tiles, &pairs, &most);
    a.pairs = pairs; a.parts = parts.n;
    a.q_seq_mul = c.q.seq > 0; a.q_head_mul = c.q.head > 0;
    a.kv_head_mul = c.k.head > 0; a.kv_seq_mul = c.k.seq > 0; a.v_head_mul = c.v.head > 0; a.v_seq_mul = c.v.seq > 0;
    const long long items = (long long)c.n_seq * c.kv_heads * a.pairs * a.parts;
    if (items > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    a.items = (uint32_t)items;
    a.by_parts = div_by(a.parts); a.by_pairs = div_by(a.pairs); a.by_kv_heads = div_by(c.kv_heads); a.by_share = div_by(c.where.share);
    a.rows = (long long)c.n_seq * c.heads * c.n_q;
    a.scale = c.scale; a.c = c.scale * 1.4426950408889634f;
    a.lse = c.lse; a.part_out = parts.out; a.part_lse = parts.lse; a.err = c.err;
    const bool packed = c.where.offsets != nullptr;
    const int enc = packed ? 1 : c.where.n_enc, rows = c.where.kv_rows;
    CUtensorMap mq, mk, mv, mo;
    FREE_TRY(map_heads(&mq, c.q, c.n_seq, c.n_q, c.heads, c.d, c.group, a.tt));
    FREE_TRY(map_heads(&mk, c.k, enc, rows, c.kv_heads, c.d, 1, BK));
    FREE_TRY(map_heads(&mv, c.v, enc, rows, c.kv_heads, c.d, 1, BK));
    FREE_TRY(map_heads(&mo, c.o, c.n_seq, c.n_q, c.heads, c.d, c.group, a.tt));
    FREE_TRY(c.d <= 64 ? launch<1>(mq, mk, mv, mo, a, s) : launch<2>(mq, mk, mv, mo, a, s));
    return parts.n > 1 ? cross_join(FREE_BF16, c, parts, s) : FREE_OK;
}

int cross_join(int dtype, const CrossArgs& a, const CrossParts& parts, cudaStream_t s) {
    const long long rows = (long long)a.n_seq * a.heads * a.n_q, ctas = (rows + 7) / 8;
    const dim3 grid((unsigned)(ctas < kSms * 8 ? ctas : kSms * 8));
    const bool early = free_overlap_for_rows(rows);
    return dtype == FREE_FP32 ? free_launch(early, cross_join_kernel<float>, grid, dim3(256), 0, s, a, parts, rows)
                              : free_launch(early, cross_join_kernel<__nv_bfloat16>, grid, dim3(256), 0, s, a, parts, rows);
}
