// Tensor-core products of the gated linear layer (bf16 operands, fp32 accumulation), forward and backward.
//
//   GATED   z = x W^T + b, W = [gate rows; up rows] [2F, K];  h = act(z_gate) z_up          contraction over K
//   DX      dx = dz W,        dz [M, 2F]                                                    contraction over 2F
//   DW      dW = dz^T x                                                                     contraction over M
//
// One persistent kernel for all three, clusters of two CTAs (tcgen05 cta_group::2), one CTA per SM, 192 threads: warp 0 loads
// tiles by TMA into a ring of stages, warp 1 of the even CTA issues the MMAs, warps 2-5 of both CTAs are the epilogue on
// the other of two TMEM accumulators.  A cluster's tile is 256 rows x up to 256 accumulator columns; each CTA loads its own
// 128 rows of A and half of B (no multicast), 32 KB per 64-deep step.
//   - GATED pairs the projections inside a tile: the even CTA's half of B are 128 gate rows of W, the odd CTA's the matching
//     128 up rows, so an accumulator row holds z_gate and z_up side by side, and activation and product are the epilogue.
//     z leaves the SM only where the caller keeps it for the backward pass.
//   - DX and DW read W, dz and x as they lie: operands whose contraction runs along rows are MN-major tiles (64 x 64 boxes,
//     128-byte swizzle), so nothing is transposed in memory.
//   - Few tiles and a long contraction (DW over many rows of a small layer, DX over few rows) are split along the
//     contraction; the fp32 parts go to the workspace and are added in order, so repeats are bit-identical.
// Bound by the tensor pipe and the power cap except for few rows.  24576 rows, F = 4608, K = 1152 (0.52 TFLOP per product): forward
// without z 340 us in a burst, 395 to 413 under sustained load (1.32 to 1.26 PFLOP/s; a library product of that size 423), with z 406
// and 459 to 476 us (the 453 MB more to HBM are not hidden); DX and DW 350 us each in a burst.
#include "gated.h"
#include "tc_common.cuh"

namespace {

enum { GATED = 0, DX = 1, DW = 2 };

constexpr int BK = 64;
constexpr int kThreads = 192;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kABytes = 128 * BK * 2, kStageBytes = 2 * kABytes;
constexpr uint32_t kBoxBytes = 64 * BK * 2;             // one 64 x 64 box of an MN-major operand
constexpr uint32_t kCtrlBytes = 1024;
// Staging buffers per epilogue warp (GATED: of 32 rows x 64 bytes), and stages of operands: the loads are bound by their
// latency under load, a sixth stage is worth 4% (24576 rows, F = 4608, K = 1152).
template <int MODE> struct Mem {
    static constexpr int bufs = 4, stages = MODE == GATED ? 6 : 5;
    static constexpr uint32_t buf_bytes = MODE == GATED ? 2048 : 4096;
    static constexpr uint32_t bytes = 1024 + kCtrlBytes + 4 * bufs * buf_bytes + stages * kStageBytes;
    static_assert(bytes <= 227 * 1024, "shared memory of a CTA");
};
constexpr int kPairs = 74;                              // clusters of two on 148 SMs

struct Args {
    int M, N;                               // output rows and columns (GATED: N = F)
    int num_m, num_n, nk, splits;           // tiles, 64-deep steps of the contraction, parts of it
    int half, last_half;                    // B rows per CTA of a tile, and of a tile in the last column block
    long long plane_rows;                   // splits > 1: rows between the parts
    int F;
    const float* bias;                      // GATED: [2F] or nullptr, 16-byte aligned
    uint32_t* err;
};

// Operand tile whose contraction runs along the rows of memory: blocks of 64 columns (128 bytes, swizzled) kBoxBytes apart,
// groups of 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_mn(uint32_t saddr) {
    uint64_t d = 0;
    d |= (uint64_t)((saddr >> 4) & 0x3FFFu);
    d |= (uint64_t)(kBoxBytes >> 4) << 16;
    d |= (uint64_t)(1024u >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

__device__ __forceinline__ uint4 pack8(const float* v) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <int MODE, bool F32OUT, bool PRE, int ACT>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kThreads, 1)
gated_tc_kernel(const __grid_constant__ CUtensorMap mapA, const __grid_constant__ CUtensorMap mapB, const __grid_constant__ CUtensorMap mapO,
                const __grid_constant__ CUtensorMap mapG, const __grid_constant__ CUtensorMap mapU, const Args a) {
    constexpr int kStages = Mem<MODE>::stages, kBufs = Mem<MODE>::bufs;
    constexpr uint32_t kBufBytes = Mem<MODE>::buf_bytes;
    extern __shared__ uint8_t smem_raw[];
    uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
    uint64_t* full = reinterpret_cast<uint64_t*>(smem);  // used in the even CTA only
    uint64_t* empty = full + kStages;
    uint64_t* accf = empty + kStages;
    uint64_t* acce = accf + 2;                           // used in the even CTA only
    uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(acce + 2);
    volatile uint32_t* abort_flag = tmem_slot + 1;
    uint8_t* staging = smem + kCtrlBytes;
    uint8_t* tiles = staging + 4 * kBufs * kBufBytes;

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = tc::cluster_ctarank();
    const long long per_split = (long long)a.num_m * a.num_n, total = per_split * a.splits;
    const long long first = tc::cluster_id_x(), step = tc::num_clusters_x();

    // DX takes the last rows first: their dz is what the elementwise pass wrote last, and is still in the L2
    auto row_block = [&](long long t) {
        const int m = (int)(t % per_split / a.num_n);
        return MODE == DX ? a.num_m - 1 - m : m;
    };

    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) { tc::mbar_init(&full[s], 1); tc::mbar_init(&empty[s], 1); }
        for (int i = 0; i < 2; ++i) { tc::mbar_init(&accf[i], 1); tc::mbar_init(&acce[i], 8); }
        *abort_flag = 0;
        tc::fence_barrier_init();
        tc::fence_proxy_async();
    }
    if (warp == 1) { tc::tmem_alloc_pair(tmem_slot, kTmemCols); tc::tmem_relinquish_pair(); }
    tc::tc_fence_before();
    tc::cluster_sync_all();                              // barriers of both CTAs initialised before any remote use
    tc::tc_fence_after();
    const uint32_t tmem_base = *tmem_slot;
    auto fail = [&](uint32_t code) { *abort_flag = 1; atomicOr(a.err, code); };
    free_grid_dep_wait();                                // only this cluster's shared and tensor memory was touched so far
    free_grid_dep_launch();

    if (warp == 0) {
        // ------------------------------------------------------------------ TMA producer (both CTAs)
        if (lane == 0) { tc::tma_prefetch_desc(&mapA); tc::tma_prefetch_desc(&mapB); }
        const uint32_t full0 = tc::mapa(tc::smem_u32(&full[0]), 0);
        int s = 0;
        uint32_t ph = 0;
        bool ok = true;
        for (long long t = first; ok && t < total; t += step) {
            const int sp = (int)(t / per_split);
            const int m_blk = row_block(t), n_blk = (int)(t % a.num_n);
            const int half = n_blk == a.num_n - 1 ? a.last_half : a.half;
            const int m0 = m_blk * 256 + (int)rank * 128;
            // GATED: gate rows for the even CTA, up rows for the odd one
            const int n0 = MODE == GATED ? n_blk * a.half + (int)rank * a.F : n_blk * 2 * a.half + (int)rank * half;
            const int kb0 = (int)((long long)a.nk * sp / a.splits), kb1 = (int)((long long)a.nk * (sp + 1) / a.splits);
            const uint32_t tx = 2u * (kABytes + (uint32_t)half * BK * 2u);
            for (int kb = kb0; kb < kb1; ++kb) {
                ok = tc::wait_uniform(&empty[s], ph ^ 1u, abort_flag);
                if (!ok) { if (lane == 0) fail(FREE_DEV_ERR_EMPTY_WAIT); break; }
                if (tc::elect_one()) {
                    const uint32_t dst = tc::smem_u32(tiles + (size_t)s * kStageBytes), bar = full0 + 8u * s;
                    if (rank == 0) tc::mbar_expect_tx(&full[s], tx);
                    if (MODE == DW) {
                        tc::tma_load_2d_pair(dst, &mapA, bar, m0, kb * BK);
                        tc::tma_load_2d_pair(dst + kBoxBytes, &mapA, bar, m0 + 64, kb * BK);
                    } else {
                        tc::tma_load_2d_pair(dst, &mapA, bar, kb * BK, m0);
                    }
                    if (MODE == GATED) {
                        tc::tma_load_2d_pair(dst + kABytes, &mapB, bar, kb * BK, n0);
                    } else {
                        tc::tma_load_2d_pair(dst + kABytes, &mapB, bar, n0, kb * BK);
                        if (half > 64) tc::tma_load_2d_pair(dst + kABytes + kBoxBytes, &mapB, bar, n0 + 64, kb * BK);
                    }
                }
                __syncwarp();
                if (++s == kStages) { s = 0; ph ^= 1u; }
            }
        }
        if (!ok || *abort_flag) {
            // loads in flight must land before the shared memory is given back: they take microseconds
            const long long t0 = clock64();
            while (clock64() - t0 < 400000ll) { }
        }
        __syncwarp();
    } else if (warp == 1) {
        // ------------------------------------------------------------------ MMA issuer (even CTA only)
        if (rank == 0) {
            // bits 15, 16: A, B are MN-major
            const uint32_t major = (MODE == DW ? 1u << 15 : 0u) | (MODE != GATED ? 1u << 16 : 0u);
            const uint32_t idesc_full = tc::idesc_bf16(256, 2 * a.half) | major, idesc_last = tc::idesc_bf16(256, 2 * a.last_half) | major;
            uint32_t tl = 0, ph = 0;
            int s = 0;
            bool ok = true;
            for (long long t = first; ok && t < total; t += step, ++tl) {
                const int sp = (int)(t / per_split);
                const int kb0 = (int)((long long)a.nk * sp / a.splits), kb1 = (int)((long long)a.nk * (sp + 1) / a.splits);
                const uint32_t acc = tl & 1u, aph = (tl >> 1) & 1u;
                ok = tc::wait_uniform(&acce[acc], aph ^ 1u, abort_flag);
                if (!ok) { if (lane == 0) fail(FREE_DEV_ERR_ACC_EMPTY); break; }
                tc::tc_fence_after();
                const uint32_t d_tmem = tmem_base + acc * 256u;
                const uint32_t idesc = (int)(t % a.num_n) == a.num_n - 1 ? idesc_last : idesc_full;
                for (int kb = kb0; kb < kb1; ++kb) {
                    ok = tc::wait_uniform(&full[s], ph, abort_flag);
                    if (!ok) { if (lane == 0) fail(FREE_DEV_ERR_FULL_WAIT); break; }
                    tc::tc_fence_after();
                    if (tc::elect_one()) {
                        const uint32_t a_addr = tc::smem_u32(tiles + (size_t)s * kStageBytes), b_addr = a_addr + kABytes;
#pragma unroll
                        for (int k = 0; k < BK / 16; ++k) {
                            // 16 steps of the contraction: 32 bytes along a swizzled row, or two groups of 8 rows
                            const uint64_t da = MODE == DW ? smem_desc_mn(a_addr + k * 2048) : tc::smem_desc(a_addr + k * 32, 1024, 2);
                            const uint64_t db = MODE == GATED ? tc::smem_desc(b_addr + k * 32, 1024, 2) : smem_desc_mn(b_addr + k * 2048);
                            tc::mma_bf16_pair(d_tmem, da, db, idesc, (kb > kb0 || k > 0) ? 1u : 0u);
                        }
                        tc::mma_commit_pair(&empty[s]);
                    }
                    __syncwarp();
                    if (++s == kStages) { s = 0; ph ^= 1u; }
                }
                if (ok && tc::elect_one()) tc::mma_commit_pair(&accf[acc]);
                __syncwarp();
            }
        }
        __syncwarp();
    } else {
        // ------------------------------------------------------------------ epilogue (both CTAs)
        const int q = warp & 3;                          // TMEM lanes [32q, 32q + 32) belong to this warp
        const uint32_t acce0 = tc::mapa(tc::smem_u32(&acce[0]), 0);
        uint8_t* mine = staging + (size_t)q * kBufs * kBufBytes;
        uint32_t tl = 0, nst = 0;
        // 16-byte unit u of this lane's row in a staging buffer, rows of 128 bytes (GATED: 64), swizzled as the tensor maps expect
        auto unit = [&](uint8_t* buf, int u) {
            return reinterpret_cast<uint4*>(MODE == GATED ? buf + lane * 64 + ((u ^ ((lane >> 1) & 3)) << 4) : buf + lane * 128 + ((u ^ (lane & 7)) << 4));
        };
        for (long long t = first; t < total; t += step, ++tl) {
            const int sp = (int)(t / per_split);
            const int m_blk = row_block(t), n_blk = (int)(t % a.num_n);
            const int half = n_blk == a.num_n - 1 ? a.last_half : a.half;
            const uint32_t acc = tl & 1u, aph = (tl >> 1) & 1u;
            if (!tc::wait_uniform(&accf[acc], aph, abort_flag)) { if (lane == 0) fail(FREE_DEV_ERR_ACC_FULL); break; }
            tc::tc_fence_after();
            const int row0 = m_blk * 256 + (int)rank * 128 + q * 32;
            const uint32_t t_addr = tmem_base + ((uint32_t)(q * 32) << 16) + acc * 256u;
            if (MODE == GATED) {
                constexpr int NB = PRE ? 3 : 1;          // staging buffers of a chunk of 32 columns: h, z_gate, z_up
                const int n0 = n_blk * a.half;
#pragma unroll 1
                for (int c0 = 0; c0 < half && n0 + c0 < a.F; c0 += 32) {
                    uint32_t rg[32], ru[32];
                    tc::tmem_ld32(t_addr + (uint32_t)c0, rg);
                    tc::tmem_ld32(t_addr + (uint32_t)(half + c0), ru);
                    if (lane == 0) tc::bulk_wait_read<kBufs - NB>();   // the stores that last used these buffers have read them
                    __syncwarp();
                    uint8_t* bufs[NB];
#pragma unroll
                    for (int i = 0; i < NB; ++i) bufs[i] = mine + ((nst + i) % kBufs) * kBufBytes;
                    tc::tmem_wait_ld();
#pragma unroll
                    for (int g = 0; g < 4; ++g) {
                        const int n = n0 + c0 + 8 * g;
                        float zg[8], zu[8], hv[8];
#pragma unroll
                        for (int i = 0; i < 8; ++i) { zg[i] = __uint_as_float(rg[8 * g + i]); zu[i] = __uint_as_float(ru[8 * g + i]); }
                        if (a.bias && n < a.F) {         // F % 8 == 0: a group of 8 columns is inside or outside
#pragma unroll
                            for (int i = 0; i < 2; ++i) {
                                const float4 bg = __ldg(reinterpret_cast<const float4*>(a.bias + n) + i);
                                const float4 bu = __ldg(reinterpret_cast<const float4*>(a.bias + a.F + n) + i);
                                zg[4 * i] += bg.x; zg[4 * i + 1] += bg.y; zg[4 * i + 2] += bg.z; zg[4 * i + 3] += bg.w;
                                zu[4 * i] += bu.x; zu[4 * i + 1] += bu.y; zu[4 * i + 2] += bu.z; zu[4 * i + 3] += bu.w;
                            }
                        }
#pragma unroll
                        for (int i = 0; i < 8; ++i) hv[i] = free_gate_act_fast(ACT, zg[i]) * zu[i];
                        *unit(bufs[0], g) = pack8(hv);
                        if (PRE) { *unit(bufs[NB > 1 ? 1 : 0], g) = pack8(zg); *unit(bufs[NB > 2 ? 2 : 0], g) = pack8(zu); }
                    }
                    tc::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        const bool live = row0 < a.M;    // rows past M inside the box are clipped
                        if (live) tc::tma_store_2d(&mapO, tc::smem_u32(bufs[0]), n0 + c0, row0);
                        tc::bulk_commit();
                        if (PRE) {
                            if (live) tc::tma_store_2d(&mapG, tc::smem_u32(bufs[NB > 1 ? 1 : 0]), n0 + c0, row0);
                            tc::bulk_commit();
                            if (live) tc::tma_store_2d(&mapU, tc::smem_u32(bufs[NB > 2 ? 2 : 0]), n0 + c0, row0);
                            tc::bulk_commit();
                        }
                    }
                    nst += NB;
                }
            } else {
                constexpr int CH = F32OUT ? 32 : 64;     // columns of a staging buffer (128 bytes per row)
                const int n0 = n_blk * 2 * a.half;
                const int out_row = (int)(sp * a.plane_rows) + row0;
#pragma unroll 1
                for (int c0 = 0; c0 < 2 * half && n0 + c0 < a.N; c0 += CH) {
                    uint8_t* buf = mine + (nst % kBufs) * kBufBytes;
                    if (lane == 0) tc::bulk_wait_read<kBufs - 1>();
                    __syncwarp();
#pragma unroll
                    for (int h = 0; h < CH / 32; ++h) {
                        uint32_t r[32];
                        tc::tmem_ld32(t_addr + (uint32_t)(c0 + 32 * h), r);
                        tc::tmem_wait_ld();
                        if (F32OUT) {
#pragma unroll
                            for (int u = 0; u < 8; ++u) *unit(buf, u) = make_uint4(r[4 * u], r[4 * u + 1], r[4 * u + 2], r[4 * u + 3]);
                        } else {
#pragma unroll
                            for (int g = 0; g < 4; ++g) {
                                float v[8];
#pragma unroll
                                for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[8 * g + i]);
                                *unit(buf, 4 * h + g) = pack8(v);
                            }
                        }
                    }
                    tc::fence_proxy_async();
                    __syncwarp();
                    if (lane == 0) {
                        if (row0 < a.M) tc::tma_store_2d(&mapO, tc::smem_u32(buf), n0 + c0, out_row);
                        tc::bulk_commit();
                    }
                    ++nst;
                }
            }
            tc::tc_fence_before();
            __syncwarp();
            if (lane == 0) tc::mbar_arrive_cluster(acce0 + 8u * acc);
        }
        if (lane == 0) tc::bulk_wait<0>();               // every store of this warp complete before the CTA ends
        __syncwarp();
    }
    // ---------------------------------------------------------------------- teardown
    tc::tc_fence_before();
    tc::cluster_sync_all();                              // the peer may still read this CTA's shared memory until here
    if (warp == 1) { tc::tc_fence_after(); tc::tmem_dealloc_pair(tmem_base, kTmemCols); }
}

template <int MODE, bool F32OUT, bool PRE, int ACT = FREE_ACT_SILU>
int launch(const CUtensorMap& mA, const CUtensorMap& mB, const CUtensorMap& mO, const CUtensorMap& mG, const CUtensorMap& mU, const Args& a,
           long long rows, cudaStream_t s) {
    constexpr uint32_t kSmem = Mem<MODE>::bytes;
    auto kernel = gated_tc_kernel<MODE, F32OUT, PRE, ACT>;
    FREE_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmem));   // of the current device
    const long long tiles = (long long)a.num_m * a.num_n * a.splits;
    const int grid = 2 * (int)(tiles < kPairs ? tiles : kPairs);
    return free_launch(free_overlap_for_rows(rows), kernel, dim3(grid), dim3(kThreads), kSmem, s, mA, mB, mO, mG, mU, a);
}

// Width of the column blocks and parts of the contraction for a product of `rows` x K outputs over nk steps.  In units of a
// step of a 256-wide tile (64 deep, about 0.3 us on a full GPU, in which HBM moves 2 MB): a tile costs its steps plus about 6
// for filling the pipe, a step of a 128-wide tile 0.73 (it runs at the shared-memory bandwidth); parts cost a launch and 8
// bytes of traffic per output element and part.
GatedSplit choose_split(long long rows, int K, int nk) {
    GatedSplit g{1, (rows + 255) / 256 * 256, 128};              // the last row block of a part stays inside its own plane
    double best = 0;
    for (int half = 128; half >= 64; half -= 64) {
        const long long tiles = (rows + 255) / 256 * ((K + 2 * half - 1) / (2 * half));
        for (int s = 1; s <= 32 && s <= nk && (s == 1 || tiles * (s - 1) < 4 * kPairs); ++s) {     // beyond four waves: nothing to gain
            const long long waves = (tiles * s + kPairs - 1) / kPairs;
            const double cost = (double)waves * ((half == 64 ? 0.73 : 1.0) * ((nk + s - 1) / s) + 6.0) +
                                (s > 1 ? 10.0 + (double)s * (double)rows * K * 8.0 / 2.0e6 : 0.0);
            if ((half == 128 && s == 1) || cost < best) { best = cost; g.parts = s; g.half = half; }
        }
    }
    return g;
}

}  // namespace

bool gated_tc_supported(int F, int K) { return F % 8 == 0 && K % 8 == 0; }

int gated_tc_forward(int act, int M, int F, int K, const void* x, const void* w, const float* bias, void* h, void* preact, uint32_t* err, cudaStream_t s) {
    Args a{};
    a.M = M; a.N = F; a.F = F; a.bias = bias; a.err = err;
    // few rows: blocks of 64 columns put twice as many clusters on the weights
    a.num_m = (M + 255) / 256;
    a.half = (long long)a.num_m * ((F + 127) / 128) <= kPairs / 2 ? 64 : 128;
    a.last_half = a.half;
    a.num_n = (F + a.half - 1) / a.half; a.nk = (K + BK - 1) / BK; a.splits = 1;
    CUtensorMap mA, mB, mO, mG, mU;
    FREE_TRY(free_tensor_map_2d(&mA, x, (uint64_t)K, (uint64_t)M, (uint64_t)K * 2, BK, 128, 128));
    FREE_TRY(free_tensor_map_2d(&mB, w, (uint64_t)K, 2ull * F, (uint64_t)K * 2, BK, (uint32_t)a.half, 128));
    FREE_TRY(free_tensor_map_2d(&mO, h, (uint64_t)F, (uint64_t)M, (uint64_t)F * 2, 32, 32, 64));
    const bool silu = act == FREE_ACT_SILU;
    if (!preact)
        return silu ? launch<GATED, false, false, FREE_ACT_SILU>(mA, mB, mO, mO, mO, a, M, s)
                    : launch<GATED, false, false, FREE_ACT_GELU>(mA, mB, mO, mO, mO, a, M, s);
    // one map per half of z, so that a ragged last block of gate columns cannot reach into the up columns
    FREE_TRY(free_tensor_map_2d(&mG, preact, (uint64_t)F, (uint64_t)M, (uint64_t)F * 4, 32, 32, 64));
    FREE_TRY(free_tensor_map_2d(&mU, (const char*)preact + 2ull * F, (uint64_t)F, (uint64_t)M, (uint64_t)F * 4, 32, 32, 64));
    return silu ? launch<GATED, false, true, FREE_ACT_SILU>(mA, mB, mO, mG, mU, a, M, s)
                : launch<GATED, false, true, FREE_ACT_GELU>(mA, mB, mO, mG, mU, a, M, s);
}

GatedSplit gated_tc_split(bool dw, int M, int F, int K) {
    return choose_split(dw ? 2LL * F : M, K, ((dw ? M : 2 * F) + BK - 1) / BK);
}

int gated_tc_backward(bool dw, const GatedSplit& g, int M, int F, int K, const void* x, const void* w, const void* dz, void* out, float* parts, uint32_t* err, cudaStream_t s) {
    Args a{};
    a.M = dw ? 2 * F : M; a.N = K; a.F = F; a.err = err;
    a.half = g.half;
    a.num_m = (a.M + 255) / 256; a.num_n = (K + 2 * a.half - 1) / (2 * a.half); a.nk = ((dw ? M : 2 * F) + BK - 1) / BK;
    a.splits = g.parts; a.plane_rows = g.plane_rows;
    if (g.parts * g.plane_rows > 0x7fffffffLL) return FREE_ERR_UNSUPPORTED;
    a.last_half = K - (a.num_n - 1) * 2 * a.half <= 128 ? 64 : a.half;     // a ragged last column block is computed 128 wide where that holds it
    CUtensorMap mA, mB, mO;
    if (dw) {
        FREE_TRY(free_tensor_map_2d(&mA, dz, 2ull * F, (uint64_t)M, (uint64_t)F * 4, 64, BK, 128));
        FREE_TRY(free_tensor_map_2d(&mB, x, (uint64_t)K, (uint64_t)M, (uint64_t)K * 2, 64, BK, 128));
    } else {
        FREE_TRY(free_tensor_map_2d(&mA, dz, 2ull * F, (uint64_t)M, (uint64_t)F * 4, BK, 128, 128));
        FREE_TRY(free_tensor_map_2d(&mB, w, (uint64_t)K, 2ull * F, (uint64_t)K * 2, 64, BK, 128));
    }
    if (g.parts > 1) {
        FREE_TRY(free_tensor_map_2d_typed(&mO, 4, parts, (uint64_t)K, (uint64_t)(g.parts * g.plane_rows), (uint64_t)K * 4, 32, 32, 128));
        return dw ? launch<DW, true, false>(mA, mB, mO, mO, mO, a, M, s) : launch<DX, true, false>(mA, mB, mO, mO, mO, a, M, s);
    }
    FREE_TRY(free_tensor_map_2d(&mO, out, (uint64_t)K, (uint64_t)a.M, (uint64_t)K * 2, 64, 32, 128));
    return dw ? launch<DW, false, false>(mA, mB, mO, mO, mO, a, M, s) : launch<DX, false, false>(mA, mB, mO, mO, mO, a, M, s);
}
