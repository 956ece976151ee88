// Attention to an encoder's states on the tensor cores (bf16 operands, fp32 softmax and accumulation), forward.
//
//   S = Q K^T (tcgen05, fp32 in tensor memory);  p = 2^(c S - m), c = scale log2 e;  O += p V;  out = O / sum p
//
// Persistent CTAs, one per SM.  An item is two tiles of 128 rows of one (sequence, key head), rows being (token, query head of the key
// head's group), so that shared key heads are read once.  A warpgroup per tile does the softmax, a thread per row; one warp
// loads tiles by TMA, one issues the MMAs.  While one tile's exponentials run, the tensor pipe does the other tile's products.
//   - p goes back to tensor memory, over its own scores, as the left operand of O += p V: it never passes shared memory.
//   - S of the next block of states (of the next item, too) is issued right behind O += p V; the pipe runs in order, so the
//     scores' columns are free by then.
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

constexpr int BQ = 128, BK = 128;
constexpr int kThreads = 384, kSms = 148;
// Registers: 384 x 168 at launch; the two softmax warpgroups take 216 (a row's 128 scores stay in them), the third keeps 72.
constexpr int kSoftmaxRegs = 216, kOtherRegs = 72;
static_assert(256 * kSoftmaxRegs + 128 * kOtherRegs <= 384 * 168, "registers of the launch");
constexpr uint32_t kChunk = 128 * 128;        // 128 rows x 64 channels, 128-byte rows
constexpr uint32_t kTmemCols = 512;           // scores of the two tiles: columns 0, 128; O: 256, 384
constexpr uint32_t kCtrl = 1024;
template <int NCH> struct Mem {               // NCH: chunks of 64 channels
    static constexpr int slots = NCH == 1 ? 8 : 4;
    static constexpr uint32_t tile = NCH * kChunk;
    static constexpr uint32_t bytes = 1024 + kCtrl + 2 * tile + slots * tile + 2 * kChunk;
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
};

struct Args {
    CrossWhere where;
    int n_q, heads, kv_heads, d, group, tt;   // tt: tokens of a tile
    int pairs, tiles, parts;                  // items per (sequence, key head), tiles per item, parts of the states
    int kv_head_mul, kv_seq_mul, v_head_mul, v_seq_mul, q_seq_mul, q_head_mul;      // 0 where one matrix serves all
    long long items, rows;                    // rows: n_seq * heads * n_q
    float c, ln2_over_c, scale;               // c: scale * log2 e
    float *lse, *part_out, *part_lse;
    uint32_t* err;
};

// One item: its place and the blocks of states that it covers.
struct Item {
    int s, kh, t0, part, tiles, b0, nb, limit;      // limit: tokens; blocks b0 .. b0 + nb - 1
    CrossSpan sp;
};
__device__ __forceinline__ Item item_of(const Args& a, long long i) {
    Item it;
    it.part = (int)(i % a.parts); i /= a.parts;
    const int pair = (int)(i % a.pairs); i /= a.pairs;
    it.kh = (int)(i % a.kv_heads); it.s = (int)(i / a.kv_heads);
    it.t0 = pair * a.tiles * a.tt;
    it.tiles = a.tiles == 2 && it.t0 + a.tt < a.n_q ? 2 : 1;
    it.sp = cross_span(a.where, it.s);
    const int blocks = (it.sp.len + BK - 1) / BK;
    it.b0 = (int)((long long)blocks * it.part / a.parts);
    it.nb = (int)((long long)blocks * (it.part + 1) / a.parts) - it.b0;
    return it;
}
__device__ __forceinline__ int columns_of(const Item& it, int j) {       // of scores, in steps of 16
    const int left = it.sp.len - (it.b0 + j) * BK;
    return left >= BK ? BK : (left + 15) & ~15;
}

__device__ __forceinline__ void group_sync(int w) {
    if (w == 0) asm volatile("bar.sync 1, 128;" ::: "memory");
    else asm volatile("bar.sync 2, 128;" ::: "memory");
}

// Walks over the blocks of all of a CTA's items that have any.
struct Steps {
    const Args& a;
    long long i, step;
    Item it;
    int j;
    bool live;
    __device__ __forceinline__ Steps(const Args& args, long long first, long long stride) : a(args), i(first - stride), step(stride), j(0), live(true) { next_item(); }
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

template <int NCH>
__global__ void __launch_bounds__(kThreads, 1)
cross_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                const __grid_constant__ CUtensorMap mapO, const Args a) {
    using M = Mem<NCH>;
    constexpr int NS = M::slots;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* kv_full = reinterpret_cast<uint64_t*>(smem);
    uint64_t* kv_empty = kv_full + NS;
    uint64_t* q_full = kv_empty + NS;
    uint64_t* q_empty = q_full + 2;
    uint64_t* s_full = q_empty + 2;
    uint64_t* p_full = s_full + 2;
    uint64_t* o_full = p_full + 2;
    uint64_t* o_free = o_full + 2;
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(o_free + 2);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    uint8_t* sQ = smem + kCtrl;
    uint8_t* ring = sQ + 2 * M::tile;
    uint8_t* staging = ring + NS * M::tile;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int i = 0; i < NS; ++i) { tc::mbar_init(&kv_full[i], 1); tc::mbar_init(&kv_empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            tc::mbar_init(&q_full[i], 1); tc::mbar_init(&q_empty[i], 1); tc::mbar_init(&s_full[i], 1);
            tc::mbar_init(&p_full[i], 4); tc::mbar_init(&o_full[i], 1); tc::mbar_init(&o_free[i], 4);
        }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::fence_proxy_async();
    }
    if (warp == 9) { tc::tmem_alloc(tmem_slot, kTmemCols); tc::tmem_relinquish(); }
    tc::tc_fence_before();
    __syncthreads();
    tc::tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    auto fail = [&]() { *abort_flag = 1; atomicOr(a.err, FREE_DEV_ERR_ATTN); };
    free_grid_dep_wait();                                // only this CTA's shared and tensor memory was touched so far
    free_grid_dep_launch();
    const int ks = (a.d + 15) / 16;                      // 16-channel steps

    if (warp >= 8) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == 8) {
            // ------------------------------------------------------------------ TMA producer
            if (lane == 0) { tc::tma_prefetch_desc(&mapQ); tc::tma_prefetch_desc(&mapK); tc::tma_prefetch_desc(&mapV); }
            const uint32_t q_bytes = (uint32_t)(a.tt * a.group) * 128u * NCH;
            uint32_t n = 0, q_ph = 0;                        // tiles loaded; bit w: parity of tile w's loads of Q
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
                                load_4d(tc::smem_u32(sQ + w * M::tile + ch * kChunk), &mapQ, &q_full[w], 64 * ch, it.kh * a.group * a.q_head_mul, it.t0 + w * a.tt, it.s * a.q_seq_mul);
                        }
                    }
                for (int kv = 0; ok && kv < 2; ++kv, ++n, __syncwarp()) {
                    const uint32_t slot = n % NS;
                    ok = tc::wait_uniform(&kv_empty[slot], ((n / NS) & 1u) ^ 1u, abort_flag);
                    if (ok && tc::elect_one()) {
                        tc::mbar_expect_tx(&kv_full[slot], M::tile);
                        for (int ch = 0; ch < NCH; ++ch)
                            load_4d(tc::smem_u32(ring + slot * M::tile + ch * kChunk), kv ? &mapV : &mapK, &kv_full[slot], 64 * ch,
                                    it.kh * (kv ? a.v_head_mul : a.kv_head_mul), it.sp.row0 + (it.b0 + st.j) * BK, it.sp.enc * (kv ? a.v_seq_mul : a.kv_seq_mul));
                    }
                }
            }
            if (!ok) {
                if (lane == 0) fail();
                const long long t0 = clock64();              // loads in flight must land before the shared memory is given back
                while (clock64() - t0 < 400000ll) { }
            }
            __syncwarp();
        } else if (warp == 9) {
            // ------------------------------------------------------------------ MMA issuer
            const uint32_t idesc_o = tc::idesc_bf16(BQ, ks * 16) | kBMajorMN;
            uint32_t n = 0, q_ph = 0, p_ph = 0, o_ph = 0;  // bit w: parity of tile w's barrier
            bool ok = true;
            // scores of tile w with the block of states in slot n; `head`: an item's first block, `tail`: its last
            auto scores = [&](const Item& it, int j, int w, uint32_t at) {
                if (j == 0) {
                    ok = tc::wait_uniform(&q_full[w], q_ph >> w & 1u, abort_flag);
                    q_ph ^= 1u << w;
                }
                if (ok) ok = tc::wait_uniform(&kv_full[at % NS], (at / NS) & 1u, abort_flag);
                if (!ok) return;
                tc::tc_fence_after();
                if (tc::elect_one()) {
                    const uint32_t qa = tc::smem_u32(sQ + w * M::tile), ka = tc::smem_u32(ring + (at % NS) * M::tile);
                    const uint32_t idesc = tc::idesc_bf16(BQ, columns_of(it, j));
                    for (int k = 0; k < ks; ++k) {
                        const uint32_t off = (k >> 2) * kChunk + (k & 3) * 32;
                        tc::mma_bf16(tmem + w * 128u, tc::smem_desc(qa + off, 1024, 2), tc::smem_desc(ka + off, 1024, 2), idesc, k != 0);
                    }
                    tc::mma_commit(&s_full[w]);
                    if (j == it.nb - 1) tc::mma_commit(&q_empty[w]);
                    if (w == it.tiles - 1) tc::mma_commit(&kv_empty[at % NS]);
                }
                __syncwarp();
            };
            Steps now(a, blockIdx.x, gridDim.x);
            if (now.live)
                for (int w = 0; ok && w < now.it.tiles; ++w) scores(now.it, now.j, w, n);
            while (ok && now.live) {
                Steps nx = now;
                nx.next();
                const uint32_t v = n + 1;
                for (int w = 0; ok && w < 2; ++w) {
                    if (w < now.it.tiles) {
                        if (now.j == 0) {
                            ok = tc::wait_uniform(&o_free[w], (o_ph >> w & 1u) ^ 1u, abort_flag);
                            o_ph ^= 1u << w;
                        }
                        if (ok) ok = tc::wait_uniform(&kv_full[v % NS], (v / NS) & 1u, abort_flag);
                        if (ok) ok = tc::wait_uniform(&p_full[w], p_ph >> w & 1u, abort_flag);
                        p_ph ^= 1u << w;
                        if (!ok) break;
                        tc::tc_fence_after();
                        if (tc::elect_one()) {
                            const uint32_t va = tc::smem_u32(ring + (v % NS) * M::tile);
                            const int steps = columns_of(now.it, now.j) / 16;
                            for (int k = 0; k < steps; ++k)
                                mma_ts(tmem + 256u + w * 128u, tmem + w * 128u + 8u * k, desc_mn(va + k * 2048, kChunk), idesc_o, now.j > 0 || k > 0);
                            if (now.last()) tc::mma_commit(&o_full[w]);
                            if (w == now.it.tiles - 1) tc::mma_commit(&kv_empty[v % NS]);
                        }
                        __syncwarp();
                    }
                    if (nx.live && w < nx.it.tiles) scores(nx.it, nx.j, w, n + 2);
                }
                now.i = nx.i; now.it = nx.it; now.j = nx.j; now.live = nx.live;
                n += 2;
            }
            if (!ok && lane == 0) fail();
            __syncwarp();
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        // ------------------------------------------------------------------ softmax and results: a warpgroup per tile, a thread per row
        const int w = warp >> 2, q = warp & 3, r = q * 32 + lane;
        const uint32_t ts = tmem + w * 128u + ((uint32_t)(q * 32) << 16), to = ts + 256u;
        const int row_t = r / a.group, row_h = r - row_t * a.group;
        uint8_t* mine = staging + w * kChunk;
        const bool writer = q == 0;                      // the warp that issues the tile's copies
        uint32_t n = 0, ns = 0, no = 0;                  // ring position of the block's K; scores and results seen
        bool ok = true;
        for (long long i = blockIdx.x; ok && i < a.items; i += gridDim.x) {
            const Item it = item_of(a, i);
            const uint32_t first = n;
            n += 2u * it.nb;
            if (w >= it.tiles) continue;
            const uint8_t* mask = cross_mask(a.where, it.sp);
            const int t = it.t0 + w * a.tt + row_t;
            const bool row_ok = row_t < a.tt && t < a.n_q;
            float top = -INFINITY, sum = 0.f;            // maximum in use
            for (int j = 0; j < it.nb; ++j) {
                const int cols = columns_of(it, j), nch = (cols + 31) / 32;
                uint32_t bits[4];
                count_bits(bits, mask, (it.b0 + j) * BK, it.sp.len, lane);
                ok = tc::wait_uniform(&s_full[w], ns & 1u, abort_flag);
                ++ns;
                if (!ok) break;
                tc::tc_fence_after();
                float x[128];
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c < nch) tc::tmem_ld32(ts + 32 * c, *reinterpret_cast<uint32_t (*)[32]>(&x[32 * c]));
                tc::tmem_wait_ld();
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c < nch) {
                        if (bits[c] != 0xffffffffu) {
#pragma unroll
                            for (int e = 0; e < 32; ++e) x[32 * c + e] = bits[c] >> e & 1u ? x[32 * c + e] : -INFINITY;
                        }
#pragma unroll
                        for (int e = 0; e < 32; ++e) m4[e & 3] = fmaxf(m4[e & 3], x[32 * c + e]);
                    }
                const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
                const bool grown = !((mx - top) * a.c <= 8.f) && mx > top;      // also the first block with a state that counts
                if (__any_sync(0xffffffffu, grown)) {
                    const float nt = fmaxf(top, mx);
                    const float alpha = nt == -INFINITY ? 1.f : ex2((top - nt) * a.c);
                    top = nt;
                    sum *= alpha;
                    if (j > 0) {
                        // the scores' commit covers every product issued before them, so O is at rest
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
                float s4[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (c < nch) {
                        uint32_t pk[16];
#pragma unroll
                        for (int e = 0; e < 16; ++e) {
                            const float p0 = ex2(fmaf(x[32 * c + 2 * e], a.c, -base)), p1 = ex2(fmaf(x[32 * c + 2 * e + 1], a.c, -base));
                            s4[e & 3] += p0;
                            s4[(e + 2) & 3] += p1;
                            pk[e] = pack2(p0, p1);
                        }
                        tc::tmem_st16(ts + 16 * c, pk);
                    }
                sum += (s4[0] + s4[1]) + (s4[2] + s4[3]);
                // rows of V that do not count and that the product would read
                if (w == 0) {
                    bool whole = true;
#pragma unroll
                    for (int c = 0; c < 4; ++c) whole = whole && (bits[c] | ~low_bits(cols - 32 * c)) == 0xffffffffu;
                    if (!whole) {
                        const uint32_t v = first + 2u * j + 1u;
                        ok = tc::wait_uniform(&kv_full[v % NS], (v / NS) & 1u, abort_flag);
                        if (!ok) break;
                        uint8_t* vt = ring + (v % NS) * M::tile;
                        for (int k = q; k < cols; k += 4)
                            if (!(bits[k >> 5] >> (k & 31) & 1u) && lane < 8 * NCH)
                                *reinterpret_cast<uint4*>(vt + (lane >> 3) * kChunk + k * 128 + (lane & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                        tc::fence_proxy_async();
                    }
                }
                tc::tmem_wait_st();
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&p_full[w]);
            }
            if (!ok) break;
            // ---- results
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const float lse = top == -INFINITY ? -INFINITY : top * a.scale + logf(sum);
            const long long row = ((long long)it.s * a.heads + it.kh * a.group + row_h) * a.n_q + t;
            if (it.nb > 0) {
                ok = tc::wait_uniform(&o_full[w], no & 1u, abort_flag);
                ++no;
                if (!ok) break;
                tc::tc_fence_after();
            }
            if (a.parts > 1) {
                if (row_ok) a.part_lse[it.part * a.rows + row] = lse;
                float* dst = a.part_out + (it.part * a.rows + row) * a.d;
                for (int c = 0; it.nb > 0 && c < ks; ++c) {
                    uint32_t o[16];
                    tc::tmem_ld16(to + 16 * c, o);
                    tc::tmem_wait_ld();
                    if (row_ok) {
#pragma unroll
                        for (int e = 0; e < 16; ++e)
                            if (16 * c + e < a.d) dst[16 * c + e] = __uint_as_float(o[e]) * inv;
                    }
                }
            } else {
                if (a.lse && row_ok) a.lse[row] = lse;
                for (int ch = 0; ch < NCH; ++ch) {
                    if (writer && lane == 0) tc::bulk_wait_read<0>();          // the copy that last used the staging tile has read it
                    group_sync(w);
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        if (ch * 4 + c >= ks) break;
                        uint32_t o[16], pk[8];
                        if (it.nb > 0) {
                            tc::tmem_ld16(to + 64 * ch + 16 * c, o);
                            tc::tmem_wait_ld();
                        }
#pragma unroll
                        for (int e = 0; e < 8; ++e)
                            pk[e] = it.nb > 0 ? pack2(__uint_as_float(o[2 * e]) * inv, __uint_as_float(o[2 * e + 1]) * inv) : 0u;
                        uint8_t* dst = mine + r * 128;
                        *reinterpret_cast<uint4*>(dst + (((2 * c) ^ (r & 7)) << 4)) = make_uint4(pk[0], pk[1], pk[2], pk[3]);
                        *reinterpret_cast<uint4*>(dst + (((2 * c + 1) ^ (r & 7)) << 4)) = make_uint4(pk[4], pk[5], pk[6], pk[7]);
                    }
                    tc::fence_proxy_async();
                    group_sync(w);
                    if (writer && lane == 0) {
                        store_4d(&mapO, tc::smem_u32(mine), 64 * ch, it.kh * a.group, it.t0 + w * a.tt, it.s);
                        tc::bulk_commit();
                    }
                }
            }
            if (it.nb > 0) {
                tc::tc_fence_before();
                __syncwarp();
                if (lane == 0) tc::mbar_arrive(&o_free[w]);
            }
        }
        if (!ok && lane == 0) fail();
        if (writer && lane == 0) tc::bulk_wait<0>();     // every store complete before the CTA ends
        __syncwarp();
    }
    // ---------------------------------------------------------------------- teardown
    tc::tc_fence_before();
    __syncthreads();
    if (warp == 9) { tc::tc_fence_after(); tc::tmem_dealloc(tmem, kTmemCols); }
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
// item, one is taken; and where that still does, the states are split, into parts of four blocks at least.
void shape_of(const CrossArgs& a, int* tiles, int* pairs, int* parts) {
    const int tt = tokens_per_tile(a);
    const long long heads = (long long)a.n_seq * a.kv_heads, rows = (a.n_q + tt - 1) / tt;
    *tiles = heads * ((rows + 1) / 2) >= kSms ? 2 : 1;
    *pairs = (int)((rows + *tiles - 1) / *tiles);
    const long long items = heads * *pairs;
    const int most = (a.where.n_kv + 4 * BK - 1) / (4 * BK);
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
    shape_of(c, &a.tiles, &a.pairs, &a.parts);
    a.parts = parts.n;
    a.q_seq_mul = c.q.seq > 0; a.q_head_mul = c.q.head > 0;
    a.kv_head_mul = c.k.head > 0; a.kv_seq_mul = c.k.seq > 0; a.v_head_mul = c.v.head > 0; a.v_seq_mul = c.v.seq > 0;
    a.items = (long long)c.n_seq * c.kv_heads * a.pairs * a.parts;
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
