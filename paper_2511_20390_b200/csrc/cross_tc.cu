// Attention to an encoder's states on the tensor cores (bf16 operands, fp32 softmax and accumulation), forward.
//
//   S = Q K^T (tcgen05, fp32 in tensor memory);  p = 2^(c S - m), c = scale log2 e;  O += p V;  out = O / sum p
//
// Persistent CTAs, one per SM.  An item is two tiles of 128 rows of one (sequence, key head), rows being (token, query head of the key
// head's group), so that shared key heads are read once.  Blocks of 64 states.  A warpgroup per tile does the softmax, a thread per
// row; one warp finds the items and loads tiles by TMA, four issue MMAs (per tile the scores, and O += p V), a warpgroup writes
// results while the softmax is at the next item.
//   - p goes back to tensor memory as the left operand of O += p V: it never passes shared memory.  Scores are free for the next block
//     as soon as they are in registers, so the two products and the softmax of a tile run beside one another.
//   - V is the right operand as it lies in memory (contraction along its rows), so nothing is transposed.
//   - The maximum that p is taken against moves only when it has grown by 2^8; then O is rescaled in tensor memory.
//   - Maxima leave NaN out, sums do not: a row without a state is one whose sum is zero, and a NaN that counts reaches out and lse.
//   - The last block of a sequence costs the 16-column steps that it has.  States that do not count: scores are replaced by -inf, and the
//     rows of V are zeroed in shared memory (0 x NaN would be NaN).
// Long states and few rows: the states are split into parts, each with its own softmax, joined by cross_join_kernel.
// What bounds it: a block's way through the softmax warps, some 1700 clocks for 64 states where the exponentials and conversions of its
// two warps per scheduler are 1050; the tensor cores work for 16% of the time, the exponentials' unit for 29%.  24 x 1024 tokens, 16 heads
// of 72, up to 300 states: 68 us in a graph, 71 as calls (0.32 PFLOP/s); 8 x 4096 tokens, 16 heads of 128, up to 512 states: 126 to 136 and 143 (0.64 to 0.73).
// Heads of a key head that do not divide 32 (three, five, six): results leave by single elements, 24 x 1024 tokens, 300 states, heads of 72, 12 on 4
// 276 us, 12 on 3 or 6 67.
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
// warps 0 - 7 softmax, 8 - 11 results, 12 loads, 13 tokens without a state, 14 and 15 idle, 16, 17 Q K^T of the tiles, 18, 19 p V
constexpr int kThreads = 640, kSms = 148;
// Registers: 640 x 96 at launch.
constexpr int kSoftmaxRegs = 152, kOtherRegs = 56;
static_assert(256 * kSoftmaxRegs + 384 * kOtherRegs <= kThreads * 96, "registers of the launch");
constexpr uint32_t kChunk = BQ * 128, kKvChunk = BK * 128;      // rows x 64 channels, 128-byte rows
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kCtrl = 3 * 1024;             // barriers, the queue of items, maxima and sums of the rows of both tiles
constexpr uint32_t kQueue = 8;
constexpr uint32_t kStage = 32 * 128;         // 32 rows x 64 channels on their way out
// State sequences up to this length take two sets of the tiles of Q: with nothing but a block or two per item, Q has to be on its way
// while the item before is worked on.  Longer ones take the room for K and V.
constexpr int kShort = 128;
// NCH: chunks of 64 channels; QB: sets of the two tiles of Q; SB, PB: buffers of a tile's scores and of its p in tensor memory.  Scores
// are free for the next block as soon as they are in registers, p when O += p V has read it.
template <int NCH, int QB, int SB, int PB> struct Mem {
    static constexpr uint32_t s_col = 0, p_col = 2 * SB * 64, o_col = p_col + 2 * PB * 32, o_width = (512 - o_col) / 2;    // columns, O per tile
    static constexpr uint32_t slots = NCH == 1 ? 12 : QB == 1 ? 6 : 4, stages = NCH == 2 && QB == 2 ? 1 : 2;    // stages: of every warp of results
    static constexpr uint32_t q = NCH * kChunk, kv = NCH * kKvChunk;
    static constexpr uint32_t bytes = 1024 + kCtrl + QB * 2 * q + slots * kv + 4 * stages * kStage;
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
    float c, scale;                           // c: scale * log2 e
    float *lse, *part_out, *part_lse;
    CrossMat o;
    bool boxed;
    uint32_t* err;
};

// One item: its place, and the blocks of states that it covers.  The warp that loads tiles finds them out, once for all.
struct alignas(16) Item {
    int s, kh, t0, part, tiles, nb;           // s < 0: no more items
    int left;                                 // states from the item's first on
    int enc, row;                             // its first state: encoder sequence and row
    int pad[3];
};
__device__ __forceinline__ Item item_of(const Args& a, uint32_t i) {
    Item it;
    if (i >= a.items) { it.s = -1; it.nb = 0; it.tiles = 0; return it; }
    const uint32_t k = a.by_parts(i), sh = a.by_pairs(k);
    it.part = (int)(i - k * a.parts);
    const int pair = (int)(k - sh * a.pairs);
    it.s = (int)a.by_kv_heads(sh); it.kh = (int)(sh - it.s * a.kv_heads);
    it.t0 = pair * a.tiles * a.tt;
    it.tiles = a.tiles == 2 && it.t0 + a.tt < a.n_q ? 2 : 1;
    const CrossSpan sp = cross_span_of_enc(a.where, a.where.seq_of ? __ldg(a.where.seq_of + it.s) : (int)a.by_share(it.s));
    const int blocks = (sp.len + BK - 1) / BK;
    int b0 = 0;
    it.nb = blocks;
    if (a.parts > 1) {
        b0 = (int)((long long)blocks * it.part / a.parts);
        it.nb = (int)((long long)blocks * (it.part + 1) / a.parts) - b0;
    }
    it.left = sp.len - b0 * BK; it.enc = sp.enc; it.row = sp.row0 + b0 * BK;
    return it;
}

template <int NCH, int QB, int SB, int PB>
__global__ void __launch_bounds__(kThreads, 1)
cross_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                const __grid_constant__ CUtensorMap mapO, const Args a) {
    using M = Mem<NCH, QB, SB, PB>;
    constexpr uint32_t NS = M::slots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* kv_empty = kv_full + NS;
    uint64_t* item_full = kv_empty + NS;
    uint64_t* item_free = item_full + kQueue;
    uint64_t* q_full = item_free + kQueue;    // [tile][set]
    uint64_t* q_empty = q_full + 4;
    uint64_t* s_full = q_empty + 4;           // [tile][buffer]
    uint64_t* s_free = s_full + 4;
    uint64_t* p_full = s_free + 4;
    uint64_t* pv_done = p_full + 4;           // O += p V is complete, p is free
    uint64_t* o_free = pv_done + 4;           // [tile]: results have been read from tensor memory
    uint64_t* o_full = o_free + 2;            // an item's last O += p V
    uint64_t* sums_full = o_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(sums_full + 2);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    Item* queue = reinterpret_cast<Item*>(smem + 640);
    float2* sums = reinterpret_cast<float2*>(smem + 1024);    // [tile][row]: maximum in use, sum
    static_assert((2 * NS + 2 * kQueue + 24 + 6 + 1) * 8 <= 640 && 640 + kQueue * sizeof(Item) <= 1024 && 1024 + 2 * BQ * 8 <= kCtrl, "control block");
    uint8_t* sQ = smem + kCtrl;
    uint8_t* ring = sQ + QB * 2 * M::q;
    uint8_t* staging = ring + NS * M::kv;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (uint32_t i = 0; i < NS; ++i) { tc::mbar_init(&kv_full[i], 1); tc::mbar_init(&kv_empty[i], 2); }
        for (uint32_t i = 0; i < kQueue; ++i) { tc::mbar_init(&item_full[i], 1); tc::mbar_init(&item_free[i], 16); }     // 8 softmax, 4 results, 4 MMA
        for (int i = 0; i < 4; ++i) { tc::mbar_init(&q_full[i], 1); tc::mbar_init(&q_empty[i], 1); tc::mbar_init(&s_full[i], 1); tc::mbar_init(&s_free[i], 4); tc::mbar_init(&p_full[i], 4); tc::mbar_init(&pv_done[i], 1); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&o_free[i], 4); tc::mbar_init(&o_full[i], 1); tc::mbar_init(&sums_full[i], 4); }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::fence_proxy_async();
    }
    if (warp == 12) { tc::tmem_alloc(tmem_slot, kTmemCols); tc::tmem_relinquish(); }
    if (const int used = a.tt * a.group; used < BQ) {
        // rows that whole tokens do not fill are zeros: their scores have a say in when a warp's rows move their maxima, which decides roundings
        const uint32_t pieces = (uint32_t)(BQ - used) * 8;
        for (uint32_t i = threadIdx.x; i < QB * 2 * NCH * pieces; i += kThreads)
            *reinterpret_cast<uint4*>(sQ + i / pieces * kChunk + used * 128 + i % pieces * 16) = make_uint4(0u, 0u, 0u, 0u);
        tc::fence_proxy_async();
    }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() { *abort_flag = 1; atomicOr(a.err, FREE_DEV_ERR_ATTN); };
    free_grid_dep_wait();                                // only this CTA's shared and tensor memory was touched so far
    free_grid_dep_launch();
    const int ks = (a.d + 15) / 16;                      // 16-channel steps
    auto see = [&](uint32_t n) { return cross_tc::wait(&item_full[n % kQueue], n / kQueue & 1u, abort_flag); };
    auto leave = [&](uint32_t n) {
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(&item_free[n % kQueue]);
    };

    if (warp < 8) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ------------------------------------------------------------------ softmax: a warpgroup per tile, a thread per row
        const int w = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16), to = lanes + M::o_col + w * M::o_width;
        uint32_t ns = 0, slot0 = 0, slot_ph = 0, free_ph = 1;    // blocks of this tile so far; ring position of the block's K
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            ok = see(n);
            if (!ok) break;
            const Item& it = queue[n % kQueue];
            if (it.s < 0) break;
            const int nb = it.nb, states = it.left, tiles = it.tiles;
            const uint8_t* mask = a.where.mask ? a.where.mask + (a.where.offsets ? 0 : (long long)it.enc * a.where.n_kv) + it.row : nullptr;
            leave(n);
            if (w >= tiles) {
                slot0 += 2u * nb;
                while (slot0 >= NS) { slot0 -= NS; slot_ph ^= 1u; }
                continue;
            }
            float top = -INFINITY, sum = 0.f;            // maximum in use
            bool early_s = false;
            for (int j = 0; j < nb; ++j, ++ns) {
                const uint32_t buf = 2 * w + ns % SB, pbuf = 2 * w + ns % PB;
                const bool whole = states - j * BK >= BK && !mask;
                ok = (j > 0 && __all_sync(0xffffffffu, early_s)) || cross_tc::wait(&s_full[buf], ns / SB & 1u, abort_flag);
                if (!ok) break;
                tc::tc_fence_after();
                uint32_t x[64], bits[2];
                tc::tmem_ld64(lanes + M::s_col + (w * SB + ns % SB) * 64u, x);
                tc::tmem_wait_ld();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&s_free[buf]);
                if (!whole) {
                    count_bits(bits, mask, j * BK, states, lane);
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
                        // the product before (the one before that is complete, or p of the last block could not have been stored)
                        ok = cross_tc::wait(&pv_done[2 * w + (ns - 1u) % PB], (ns - 1u) / PB & 1u, abort_flag);
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
                // (polled before the exponentials, and the next scores before p is stored: 115 clocks each that nothing waits for)
                const bool early_p = poll(&pv_done[pbuf], (ns / PB & 1u) ^ 1u);
                const uint64_t c2 = pair(a.c, a.c), b2 = pair(-base, -base);
                uint64_t s2[2] = {0ull, 0ull};
#pragma unroll
                for (int e = 0; e < 32; ++e) {
                    const uint64_t y = fma2(pair(__uint_as_float(x[2 * e]), __uint_as_float(x[2 * e + 1])), c2, b2);
                    const float p0 = ex2(low(y)), p1 = ex2(high(y));
                    s2[e & 1] = add2(s2[e & 1], pair(p0, p1));
                    x[e] = pack2(p0, p1);
                }
                ok = __all_sync(0xffffffffu, early_p) || cross_tc::wait(&pv_done[pbuf], (ns / PB & 1u) ^ 1u, abort_flag);
                early_s = poll(&s_full[2 * w + (ns + 1u) % SB], (ns + 1u) / SB & 1u);
                if (!ok) break;
                tc::tc_fence_after();
                tc::tmem_st32(lanes + M::p_col + (w * PB + ns % PB) * 32u, *reinterpret_cast<uint32_t (*)[32]>(x));
                const uint64_t s1 = add2(s2[0], s2[1]);
                sum += low(s1) + high(s1);
                if (!whole) {
                    // rows of V that do not count and that the product would read (both tiles' groups write the same zeros)
                    const int cols = states - j * BK >= BK ? BK : (states - j * BK + 15) & ~15;
                    const uint32_t out0 = ~bits[0] & low_bits(cols), out1 = ~bits[1] & low_bits(cols - 32);
                    if (out0 | out1) {
                        ok = cross_tc::wait(&kv_full[slot0 + 1], slot_ph, abort_flag);
                        if (!ok) break;
                        uint8_t* vt = ring + (slot0 + 1) * M::kv;
                        constexpr int PER = 8 * NCH;               // 16-byte pieces of a row
#pragma unroll
                        for (int u = 0; u < BK * PER / 128; ++u) {
                            const uint32_t i = u * 128u + r, k = i / PER, piece = i % PER;
                            if ((k < 32 ? out0 >> k : out1 >> (k - 32)) & 1u)
                                *reinterpret_cast<uint4*>(vt + (piece >> 3) * kKvChunk + k * 128 + (piece & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        }
                        tc::fence_proxy_async();
                    }
                }
                slot0 += 2;
                if (slot0 == NS) { slot0 = 0; slot_ph ^= 1u; }
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&p_full[pbuf]);
            }
            if (!ok) break;
            ok = cross_tc::wait(&o_free[w], free_ph, abort_flag);        // the last item's results are out: so are its sums
            free_ph ^= 1u;
            if (!ok) break;
            sums[w * BQ + r] = make_float2(top, sum);
            __syncwarp();
            if (lane == 0) tc::mbar_arrive(&sums_full[w]);
        }
        if (!ok && lane == 0) fail();
        __syncwarp();
    } else if (warp < 12) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        // ------------------------------------------------------------------ results, tile after tile, while the softmax is at the next item
        const int q = warp & 3, r = q * 32 + lane;
        const int row_t = r / a.group, row_h = r - row_t * a.group;
        uint8_t* mine = staging + (uint32_t)q * M::stages * kStage;
        uint32_t staged = 0, ph = 0;                 // ph: bit w, parity of tile w's barriers
        bool ok = true;
        for (uint32_t n = 0; ok; ++n) {
            ok = see(n);
            if (!ok) break;
            const Item it = queue[n % kQueue];
            leave(n);
            if (it.s < 0) break;
            for (int w = 0; w < it.tiles; ++w) {
                const uint32_t to = tmem + M::o_col + w * M::o_width + ((uint32_t)(q * 32) << 16);
                ok = cross_tc::wait(&sums_full[w], ph >> w & 1u, abort_flag);
                if (!ok) break;
                const float2 ts = sums[w * BQ + r];
                const float top = ts.x, sum = ts.y, inv = sum == 0.f ? 0.f : 1.f / sum;
                const int t = it.t0 + w * a.tt + row_t, h = it.kh * a.group + row_h;
                const bool row_ok = row_t < a.tt && t < a.n_q;
                const long long row = ((long long)it.s * a.heads + h) * a.n_q + t;
                if (row_ok && (a.parts > 1 || a.lse)) {
                    const float lse = top * a.scale + logf(sum);        // no state: both -inf
                    if (a.parts > 1) a.part_lse[it.part * a.rows + row] = lse;
                    else a.lse[row] = lse;
                }
                ok = cross_tc::wait(&o_full[w], ph >> w & 1u, abort_flag);
                if (!ok) break;
                ph ^= 1u << w;
                tc::tc_fence_after();
                if (a.parts == 1 && a.boxed) {
#pragma unroll 1
                    for (int ch = 0; ch < NCH; ++ch, ++staged) {
                        uint8_t* stage = mine + staged % M::stages * kStage;
                        if (lane == 0) tc::bulk_wait_read<(int)M::stages - 1>();      // the copy that last used this buffer has read it
                        __syncwarp();
#pragma unroll 1
                        for (int half = 0; half < 2 && 4 * ch + 2 * half < ks; ++half) {
                            uint32_t o[32];
                            tc::tmem_ld32(to + 64 * ch + 32 * half, o);
                            tc::tmem_wait_ld();
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                uint32_t pk[4];
#pragma unroll
                                for (int e = 0; e < 4; ++e)
                                    pk[e] = pack2(__uint_as_float(o[8 * c + 2 * e]) * inv, __uint_as_float(o[8 * c + 2 * e + 1]) * inv);
                                *reinterpret_cast<uint4*>(stage + lane * 128 + (((4 * half + c) ^ (lane & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                            }
                        }
                        if (ch == NCH - 1) {
                            tc::tc_fence_before();
                            __syncwarp();
                            if (lane == 0) tc::mbar_arrive(&o_free[w]);
                        }
                        tc::fence_proxy_async();
                        __syncwarp();
                        if (lane == 0) {
                            const int t_box = it.t0 + w * a.tt + q * 32 / a.group;
                            if (t_box < a.n_q) store_4d(&mapO, tc::smem_u32(stage), 64 * ch, it.kh * a.group, t_box, it.s);
                            tc::bulk_commit();
                        }
                    }
                } else {
                    float* part = a.part_out + (it.part * a.rows + row) * a.d;
                    __nv_bfloat16* out = reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(a.o.p)) + it.s * a.o.seq + t * a.o.tok + h * a.o.head;
#pragma unroll 1
                    for (int c = 0; c < ks; ++c) {
                        uint32_t o[16];
                        __syncwarp();
                        tc::tmem_ld16(to + 16 * c, o);
                        tc::tmem_wait_ld();
                        if (!row_ok) continue;
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (16 * c + e < a.d) {
                                const float v = __uint_as_float(o[e]) * inv;
                                if (a.parts == 1) out[16 * c + e] = __float2bfloat16(v);
                                else part[16 * c + e] = v;
                            }
                    }
                    tc::tc_fence_before();
                    __syncwarp();
                    if (lane == 0) tc::mbar_arrive(&o_free[w]);
                }
            }
            if (!ok) break;
        }
        if (!ok && lane == 0) fail();
        if (lane == 0) tc::bulk_wait<0>();           // every store complete before the CTA ends
        __syncwarp();
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 12) {
            // ------------------------------------------------------------------ items, and TMA loads
            if (lane == 0) { tc::tma_prefetch_desc(&mapQ); tc::tma_prefetch_desc(&mapK); tc::tma_prefetch_desc(&mapV); }
            const uint32_t q_bytes = (uint32_t)(a.tt * a.group) * 128u * NCH;
            uint32_t slot = 0, ph = 1, q_set[2] = {0, 0}, q_ph[2] = {1, 1};      // (parity of the first use's wait: passes at once)
            bool ok = true;
            uint32_t i = blockIdx.x;
            auto next_item = [&]() {                     // the next that has a state
                Item it = item_of(a, i);
                while (it.s >= 0) {
                    i = a.items - i > gridDim.x ? i + gridDim.x : a.items;
                    if (it.nb > 0) break;
                    it = item_of(a, i);
                }
                return it;
            };
            Item ahead = next_item();
            for (uint32_t n = 0; ok; ++n) {
                const Item it = ahead;
                ok = cross_tc::wait(&item_free[n % kQueue], (n / kQueue & 1u) ^ 1u, abort_flag);
                if (!ok) break;
                if (lane == 0) {
                    queue[n % kQueue] = it;
                    tc::mbar_arrive(&item_full[n % kQueue]);
                }
                __syncwarp();
                if (it.s < 0) break;
                ahead = next_item();
                for (int j = 0; ok && j < it.nb; ++j) {
#pragma unroll
                    for (int w = 0; w < 2; ++w) {
                        if (j > 0 || w >= it.tiles || !ok) break;
                        const uint32_t set = q_set[w], b = w * QB + set;
                        ok = cross_tc::wait(&q_empty[b], q_ph[w], abort_flag);
                        if (QB == 1 || set == 1) q_ph[w] ^= 1u;
                        if (QB == 2) q_set[w] ^= 1u;
                        if (ok && tc::elect_one()) {
                            tc::mbar_expect_tx(&q_full[b], q_bytes);
                            for (int ch = 0; ch < NCH; ++ch)
                                load_4d(tc::smem_u32(sQ + b * M::q + ch * kChunk), &mapQ, &q_full[b], 64 * ch, it.kh * a.group * a.q_head_mul, it.t0 + w * a.tt, it.s * a.q_seq_mul);
                        }
                        __syncwarp();
                    }
                    for (int kv = 0; ok && kv < 2; ++kv) {
                        ok = cross_tc::wait(&kv_empty[slot], ph, abort_flag);
                        if (ok && tc::elect_one()) {
                            tc::mbar_expect_tx(&kv_full[slot], M::kv);
                            for (int ch = 0; ch < NCH; ++ch)
                                load_4d(tc::smem_u32(ring + slot * M::kv + ch * kKvChunk), kv ? &mapV : &mapK, &kv_full[slot], 64 * ch,
                                        it.kh * (kv ? a.v_head_mul : a.kv_head_mul), it.row + j * BK, it.enc * (kv ? a.v_seq_mul : a.kv_seq_mul));
                        }
                        __syncwarp();
                        if (++slot == NS) { slot = 0; ph ^= 1u; }
                    }
                }
            }
            if (!ok) {
                if (lane == 0) fail();
                const long long t0 = clock64();          // loads in flight must land before the shared memory is given back
                while (clock64() - t0 < 400000ll) { }
            }
            __syncwarp();
        } else if (warp >= 16) {
            // ------------------------------------------------------------------ MMA issuers, one per tile for the scores and one for O += p V
            const bool scores = warp < 18;
            const int w = warp & 1;
            const uint32_t leader = tc::elect_one() ? 1u : 0u;
            const uint32_t idesc_o = tc::idesc_bf16(BQ, ks * 16) | kBMajorMN;
            const uint64_t q_desc = tc::smem_desc(tc::smem_u32(sQ + w * QB * M::q), 1024, 2), k_desc = tc::smem_desc(tc::smem_u32(ring), 1024, 2);
            const uint64_t v_desc = desc_mn(tc::smem_u32(ring), kKvChunk);
            const uint32_t d_s = tmem + M::s_col + w * SB * 64u, d_o = tmem + M::o_col + w * M::o_width, a_p = tmem + M::p_col + w * PB * 32u;
            uint32_t slot = scores ? 0 : 1, ph = 0;      // ring: K at even places, V at odd ones
            uint32_t b = 0, b_ph = 0, set = 0, item_ph = 0;    // buffer of scores or p; set of Q; parities
            bool ok = true;
            for (uint32_t n = 0; ok; ++n) {
                ok = see(n);
                if (!ok) break;
                const Item& it = queue[n % kQueue];
                const int s = it.s, nb = it.nb, tiles = it.tiles, states = it.left;
                leave(n);
                if (s < 0) break;
                const bool mine = w < tiles;
                if (mine) ok = scores ? cross_tc::wait(&q_full[w * QB + set], item_ph, abort_flag) : cross_tc::wait(&o_free[w], item_ph ^ 1u, abort_flag);
                for (int j = 0; ok && j < nb; ++j) {
                    ok = cross_tc::wait(&kv_full[slot], ph, abort_flag);
                    if (mine) {
                        const int left = states - j * BK, cols = left >= BK ? BK : (left + 15) & ~15;
                        if (ok) ok = scores ? cross_tc::wait(&s_free[2 * w + b], b_ph ^ 1u, abort_flag) : cross_tc::wait(&p_full[2 * w + b], b_ph, abort_flag);
                        if (!ok) break;
                        tc::tc_fence_after();
                        if (scores) {
                            const uint32_t idesc = tc::idesc_bf16(BQ, cols), d = d_s + b * 64u;
                            const uint64_t qd = q_desc + set * (M::q >> 4), kd = k_desc + slot * (M::kv >> 4);
#pragma unroll
                            for (int k = 0; k < 4 * NCH; ++k)
                                if (k < ks) tc::mma_bf16_if(leader, d, qd + ((k >> 2) * (kChunk >> 4) + (k & 3) * 2), kd + ((k >> 2) * (kKvChunk >> 4) + (k & 3) * 2), idesc, k != 0);
                            tc::mma_commit_if(leader, &s_full[2 * w + b]);
                        } else {
                            const uint32_t p = a_p + b * 32u;
                            const uint64_t vd = v_desc + slot * (M::kv >> 4);
#pragma unroll
                            for (int k = 0; k < BK / 16; ++k)
                                if (16 * k < cols) mma_ts_if(leader, d_o, p + 8u * k, vd + k * (2048u >> 4), idesc_o, j > 0 || k > 0);
                            tc::mma_commit_if(leader, &pv_done[2 * w + b]);
                        }
                        tc::mma_commit_if(leader, &kv_empty[slot]);
                        if (++b == (scores ? SB : PB)) { b = 0; b_ph ^= 1u; }
                    } else {
                        // a slot is free when both tiles are done with it: one that the item does not have is so as soon as it is full
                        // (not earlier, or it would count twice for one use of the slot)
                        if (ok && leader) tc::mbar_arrive(&kv_empty[slot]);
                    }
                    slot += 2;
                    if (slot >= NS) { slot -= NS; ph ^= 1u; }
                }
                if (ok && mine) {
                    tc::mma_commit_if(leader, scores ? &q_empty[w * QB + set] : &o_full[w]);
                    if (!scores || ++set == QB) { set = 0; item_ph ^= 1u; }
                }
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        } else if (warp == 13) {
            // ------------------------------------------------------------------ tokens without a state
            for (uint32_t i = blockIdx.x; i < a.items; i = a.items - i > gridDim.x ? i + gridDim.x : a.items) {
                const Item it = item_of(a, i);
                if (it.nb > 0) continue;
                const int last = it.t0 + it.tiles * a.tt < a.n_q ? it.t0 + it.tiles * a.tt : a.n_q;
                for (int h = it.kh * a.group; h < (it.kh + 1) * a.group; ++h) {
                    float* lse = a.parts > 1 ? a.part_lse + it.part * a.rows : a.lse;
                    for (int t = it.t0 + lane; lse && t < last; t += 32) lse[((long long)it.s * a.heads + h) * a.n_q + t] = -INFINITY;
                    if (a.parts == 1)
                        zero_rows(reinterpret_cast<__nv_bfloat16*>(const_cast<void*>(a.o.p)) + it.s * a.o.seq + it.t0 * a.o.tok + h * a.o.head, 2 * a.o.tok, last - it.t0, 2 * a.d, lane);
                }
            }
        }
    }
    // ---------------------------------------------------------------------- teardown
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 12) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, kTmemCols); }
}

// out, lse of a row from its parts' own (NaN where a part's lse is): a CTA per row, the parts' weights in shared memory, a slice of the parts per channel and 128 threads.
constexpr int kMaxParts = 2048;
template <typename E, int THREADS> __global__ void __launch_bounds__(THREADS) cross_join_kernel(const CrossArgs a, const CrossParts p, long long rows) {
    constexpr int SLICES = THREADS / 128, WARPS = THREADS / 32;
    __shared__ float weight[kMaxParts], part_of[SLICES][kCrossMaxD], reduce[WARPS];
    free_grid_dep_wait();
    free_grid_dep_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, ch = threadIdx.x & 127, slice = threadIdx.x >> 7;
    const long long i = blockIdx.x;
    float top = -INFINITY;
    for (int k = threadIdx.x; k < p.n; k += THREADS) {
        weight[k] = p.lse[k * rows + i];
        top = fmaxf(top, weight[k]);
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, o));
    if (lane == 0) reduce[warp] = top;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < WARPS; ++k) top = fmaxf(top, reduce[k]);
    __syncthreads();
    float sum = 0.f;
    for (int k = threadIdx.x; k < p.n; k += THREADS) {
        weight[k] = weight[k] == -INFINITY ? 0.f : expf(weight[k] - top);       // 0: a part without a state, which wrote nothing else
        sum += weight[k];
    }
    sum = free_warp_sum(sum);
    if (lane == 0) reduce[warp] = sum;
    __syncthreads();
    sum = 0.f;
#pragma unroll
    for (int k = 0; k < WARPS; ++k) sum += reduce[k];
    float acc = 0.f;
    if (ch < a.d) {
        const float* o = p.out + i * a.d + ch;
        const long long step = rows * a.d;
#pragma unroll 8
        for (int k = slice; k < p.n; k += SLICES) {
            const float f = weight[k], v = f != 0.f ? o[k * step] : 0.f;
            acc = fmaf(f, v, acc);
        }
    }
    part_of[slice][ch] = acc;
    __syncthreads();
    if (threadIdx.x < a.d) {
        float v = 0.f;
#pragma unroll
        for (int k = 0; k < SLICES; ++k) v += part_of[k][ch];
        v = sum == 0.f ? 0.f : v / sum;
        const int t = (int)(i % a.n_q), h = (int)(i / a.n_q % a.heads), s = (int)(i / a.n_q / a.heads);
        E* out = reinterpret_cast<E*>(const_cast<void*>(a.o.p)) + s * a.o.seq + t * a.o.tok + h * a.o.head;
        if constexpr (sizeof(E) == 4) out[ch] = v;
        else out[ch] = __float2bfloat16(v);
    }
    if (a.lse && threadIdx.x == 0) a.lse[i] = top + logf(sum);
}

int tokens_per_tile(const CrossArgs& a) { return BQ / a.group; }

template <int NCH, int QB, int SB, int PB> int launch(const CUtensorMap& mq, const CUtensorMap& mk, const CUtensorMap& mv, const CUtensorMap& mo, const Args& a, cudaStream_t s) {
    constexpr uint32_t bytes = Mem<NCH, QB, SB, PB>::bytes;
    FREE_CUDA_TRY(cudaFuncSetAttribute(cross_tc_kernel<NCH, QB, SB, PB>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
    const int grid = (int)(a.items < kSms ? a.items : kSms);
    return free_launch(free_overlap_for_rows(a.rows / a.heads), cross_tc_kernel<NCH, QB, SB, PB>, dim3(grid), dim3(kThreads), bytes, s, mq, mk, mv, mo, a);
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
    const int least = ((a.where.n_kv + BK - 1) / BK >> 20) + 1;      // a million blocks are a second's work: waits for an item give up after two
    *parts = want < least ? least : (int)want;
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

int cross_tc_parts(const CrossArgs& a) {
    int tiles, pairs, parts;
    shape_of(a, &tiles, &pairs, &parts);
    return parts;
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
    // results leave by tile copies of 32 rows, where these are whole tokens and heads end with a piece of 16 bytes (copies write whole ones)
    a.boxed = 32 % c.group == 0 && c.d % 8 == 0;
    a.o = c.o;
    FREE_TRY(map_heads(&mo, c.o, c.n_seq, c.n_q, c.heads, c.d, a.boxed ? c.group : 1, a.boxed ? 32 / c.group : 32));
    const bool brief = c.where.n_kv <= kShort;
    int code;
    if (c.d <= 64) code = launch<1, 2, 2, 2>(mq, mk, mv, mo, a, s);
    else if (c.d <= 96) code = brief ? launch<2, 2, 2, 1>(mq, mk, mv, mo, a, s) : launch<2, 1, 2, 1>(mq, mk, mv, mo, a, s);
    else code = brief ? launch<2, 2, 1, 2>(mq, mk, mv, mo, a, s) : launch<2, 1, 1, 2>(mq, mk, mv, mo, a, s);
    FREE_TRY(code);
    return parts.n > 1 ? cross_join(FREE_BF16, c, parts, s) : FREE_OK;
}

int cross_join(int dtype, const CrossArgs& a, const CrossParts& parts, cudaStream_t s) {
    const long long rows = (long long)a.n_seq * a.heads * a.n_q;
    if (parts.n > kMaxParts || rows > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    // many parts: more threads to read them (8 rows of 1184 parts, with the kernel before: 78 -> 54 us)
    const bool many = parts.n >= 128, exact = dtype == FREE_FP32;
    auto kernel = exact ? many ? cross_join_kernel<float, 1024> : cross_join_kernel<float, 256> : many ? cross_join_kernel<__nv_bfloat16, 1024> : cross_join_kernel<__nv_bfloat16, 256>;
    return free_launch(free_overlap_for_rows(rows), kernel, dim3((unsigned)rows), dim3(many ? 1024 : 256), 0, s, a, parts, rows);
}
