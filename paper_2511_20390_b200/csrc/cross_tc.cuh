// What the tensor-core kernels of the attention to an encoder's states share: tile copies of heads and operands in tensor memory.
#pragma once
#include "cross.h"
#include "tc_common.cuh"

namespace cross_tc {

__device__ __forceinline__ float ex2(float x) { float y; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x)); return y; }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&v);
}
// Warp-uniform bounded wait as tc::wait_uniform; the abort flag and the clock are only looked at every 16 polls.
__device__ __forceinline__ bool wait(uint64_t* bar, uint32_t parity, volatile uint32_t* abort_flag) {
    bool r = tc::mbar_try_wait(bar, parity);
    if (!r) {
        const long long t0 = clock64();
        for (;;) {
#pragma unroll 1
            for (int i = 0; i < 16 && !r; ++i) r = tc::mbar_try_wait(bar, parity);
            if (r || *abort_flag || clock64() - t0 > 4000000000ll) break;
        }
    }
    return __all_sync(0xffffffffu, r);
}
// One poll, which does not wait.
__device__ __forceinline__ bool poll(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(ok) : "r"(tc::smem_u32(bar)), "r"(parity) : "memory");
    return ok != 0;
}
// Two of them, their first polls (some 115 clocks each) at once.
__device__ __forceinline__ bool wait2(uint64_t* bar1, uint32_t parity1, uint64_t* bar2, uint32_t parity2, volatile uint32_t* abort_flag) {
    const bool r1 = tc::mbar_try_wait(bar1, parity1), r2 = tc::mbar_try_wait(bar2, parity2);
    if (__all_sync(0xffffffffu, r1 && r2)) return true;
    return wait(bar1, parity1, abort_flag) && wait(bar2, parity2, abort_flag);
}
__device__ __forceinline__ void load_4d(uint32_t dst, const CUtensorMap* map, uint64_t* bar, int c, int head, int tok, int seq) {
    asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5, %6}], [%2];"
                 ::"r"(dst), "l"((uint64_t)map), "r"(tc::smem_u32(bar)), "r"(c), "r"(head), "r"(tok), "r"(seq) : "memory");
}
__device__ __forceinline__ void store_4d(const CUtensorMap* map, uint32_t src, int c, int head, int tok, int seq) {
    asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%2, %3, %4, %5}], [%1];"
                 ::"l"((uint64_t)map), "r"(src), "r"(c), "r"(head), "r"(tok), "r"(seq) : "memory");
}
// D[tmem] (+)= A[tmem] * B[smem], one step of 16, issued by the leader of a converged warp: lane m of A is row m, its 32-bit column c holds
// elements 2 c and 2 c + 1
__device__ __forceinline__ void mma_ts_if(uint32_t issue, uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate), "r"(issue) : "memory");
}
// Two fp32 numbers side by side: one instruction for both.
__device__ __forceinline__ uint64_t pair(float a, float b) { uint64_t v; asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(a), "f"(b)); return v; }
__device__ __forceinline__ float low(uint64_t v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float high(uint64_t v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) { uint64_t d; asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c)); return d; }
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) { uint64_t d; asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) { uint64_t d; asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b)); return d; }

// Operand whose contraction runs along the rows of memory: blocks of 64 columns (128 bytes, swizzled) `block` bytes apart, groups of
// 8 rows 1024 bytes apart.
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t block) {
    return (uint64_t)((saddr >> 4) & 0x3FFFu) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024u >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
constexpr uint32_t kBMajorMN = 1u << 16;      // instruction descriptor: B's contraction runs along rows

// The 32 * WORDS states from j0 on that count, one bit each.
__device__ __forceinline__ uint32_t low_bits(int n) { return n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u; }
template <int WORDS> __device__ __forceinline__ void count_bits(uint32_t (&w)[WORDS], const uint8_t* mask, int j0, int len, int lane) {   // whole warp
#pragma unroll
    for (int i = 0; i < WORDS; ++i) {
        w[i] = low_bits(len - j0 - 32 * i);
        if (mask) {
            const int j = j0 + 32 * i + lane;
            w[i] &= __ballot_sync(0xffffffffu, j < len && mask[j] != 0);
        }
    }
}

// Zeros into rows of `bytes` bytes, `apart` bytes from one to the next; whole warp.  Rows of whole pieces of 16 bytes are aligned to them.
__device__ __forceinline__ void zero_rows(void* p, long long apart, int rows, int bytes, int lane) {
    uint8_t* to = static_cast<uint8_t*>(p);
    const bool wide = bytes % 16 == 0;
    const int n = bytes / (wide ? 16 : 2);
    for (int r = lane / n, c = lane % n; r < rows;) {
        if (wide) *reinterpret_cast<uint4*>(to + r * apart + 16 * c) = make_uint4(0u, 0u, 0u, 0u);
        else *reinterpret_cast<uint16_t*>(to + r * apart + 2 * c) = 0;
        for (c += 32; c >= n; c -= n) ++r;
    }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
// bf16 heads [seq][tok][head][d] as a tensor map whose boxes are 64 channels x `heads_box` heads x `tok_box` tokens (128-byte
// swizzle; zero outside).  Dimensions of one element and strides of zero (a matrix that several share) become dimensions of one:
// their coordinates have to be 0.
bool mappable(const CrossMat& m, int n_seq, int n_tok, int heads);
int map_heads(CUtensorMap* map, const CrossMat& m, int n_seq, int n_tok, int heads, int d, int heads_box, int tok_box);

}  // namespace cross_tc
