// Internal interfaces of the attention to an encoder's states (cross_*.cu).
#pragma once
#include "internal.h"

constexpr int kCrossMaxD = 128, kCrossMaxLength = 0x7fff0000;

// A matrix of heads: element (s, t, h, c) at p[s * seq + t * tok + h * head + c].
struct CrossMat {
    const void* p;
    long long seq, tok, head;
};

// What every kernel needs to find the states of a sequence.
struct CrossWhere {
    const int32_t *lens, *offsets, *seq_of;
    const uint8_t* mask;
    int n_enc, n_kv, kv_rows, share;          // share: consecutive sequences that read one encoder sequence (seq_of == nullptr)
};

// States row0 .. row0 + len - 1 of encoder sequence `enc` (0 where packed); rows: those that it has, len of them at most can count
struct CrossSpan { int enc, row0, len, rows; };

__device__ __forceinline__ CrossSpan cross_span_of_enc(const CrossWhere& w, int e) {
    if ((unsigned)e >= (unsigned)w.n_enc) return CrossSpan{0, 0, 0, 0};
    if (w.offsets) {
        const int b = __ldg(w.offsets + e), n = __ldg(w.offsets + e + 1);
        const int lo = max(b, 0), hi = min(n, w.kv_rows);
        const int rows = lo < hi ? hi - lo : 0;
        return CrossSpan{0, lo, min(rows, w.n_kv), rows};
    }
    return CrossSpan{e, 0, w.lens ? min(max(__ldg(w.lens + e), 0), w.n_kv) : w.n_kv, w.n_kv};
}
__device__ __forceinline__ int cross_enc_of(const CrossWhere& w, int s) { return w.seq_of ? __ldg(w.seq_of + s) : s / w.share; }
__device__ __forceinline__ CrossSpan cross_span(const CrossWhere& w, int s) { return cross_span_of_enc(w, cross_enc_of(w, s)); }
// the mask's bytes of a span (nullptr: all states count)
__device__ __forceinline__ const uint8_t* cross_mask(const CrossWhere& w, const CrossSpan& sp) {
    return w.mask ? w.mask + (w.offsets ? (long long)sp.row0 : (long long)sp.enc * w.n_kv) : nullptr;
}

// dk, dv: blocks of B states of every encoder sequence and key head.  Either as many of every sequence, `per` for n_kv states, of which the
// last takes the rows of a packed sequence behind n_kv with it, whose gradients are zero; or (per = 0) of all its rows, packed ones only:
// a sequence's begin at number (its first row) / B + (its index), counted from the first sequence's, which leaves each the blocks that it needs
// (n rows from row a on are at most (a + n) / B - a / B + 1), so that there are n_enc + kv_rows / B of them however long a single one may be.
inline int cross_blocks_per(const CrossWhere& w, int B) {          // whichever are fewer
    const int per = w.n_kv > 0 ? (w.n_kv - 1) / B + 1 : 1;
    return w.offsets && w.n_enc + (long long)(w.kv_rows / B) < (long long)w.n_enc * per ? 0 : per;
}
inline long long cross_blocks(const CrossWhere& w, int B) {
    const int per = cross_blocks_per(w, B);
    return per ? (long long)w.n_enc * per : w.n_enc + (long long)(w.kv_rows / B);
}
struct CrossBlock {
    int e, head, row0;                        // encoder sequence, key head and the block's first of the sequence's rows; row0 < 0: no block
    bool more, last;                          // more = false: there are no blocks from this one on
};
// ROWS: per is 0.  (In a kernel of its own on the tensor cores: with the search beside the other way 512 sequences of 64 states took 5 to 12% longer.)
template <int B, bool ROWS> __device__ __forceinline__ CrossBlock cross_block(const CrossWhere& w, int kv_heads, int per, long long i) {     // whole warp, the same block
    if (!ROWS) {
        const int blk = (int)(i % per); i /= per;
        return CrossBlock{(int)(i / kv_heads), (int)(i % kv_heads), blk * B, true, blk + 1 == per};
    }
    const int head = (int)(i % kv_heads);
    i /= kv_heads;
    auto first = [&](int e) { return min(max(__ldg(w.offsets + e), 0), w.kv_rows) / B; };
    i += first(0);
    if (i >= (long long)first(w.n_enc) + w.n_enc) return CrossBlock{0, head, -1, false, false};
    // the last sequence that begins at i or before: a warp looks at 32 of those that are left
    int e = 0;
    for (int n = w.n_enc; n > 1;) {
        const int step = (n + 31) / 32, at = (int)(threadIdx.x & 31) * step;
        const unsigned before = __ballot_sync(0xffffffffu, at < n && first(e + min(at, n - 1)) + (long long)(e + at) <= i);
        const int skip = before ? (31 - __clz(before)) * step : 0;
        e += skip;
        n = min(step, n - skip);
    }
    const long long row0 = (i - e - first(e)) * B;                 // (offsets that decrease may leave none)
    return CrossBlock{e, head, row0 < w.kv_rows ? (int)max(row0, -1LL) : -1, true, false};
}

// Parts of the states of a call with few tokens (cross_join adds them): part p of row r = (sequence, head, token)
struct CrossParts {
    int n;                                    // parts; 1: results are written at once
    float* out;                               // [n][rows][d], each part's own softmax
    float* lse;                               // [n][rows]
};

struct CrossArgs {
    CrossMat q, k, v, o;                      // o: forward's result
    CrossMat g, dq, dk, dv;                   // backward: dout and the gradients
    CrossWhere where;
    int n_seq, n_q, heads, kv_heads, d, group;    // group: heads / kv_heads
    float scale;
    float* lse;                               // [n_seq, heads, n_q]
    float* delta;                             // backward: <dout, out>, laid out as lse
    unsigned long long* next;                 // backward: a counter that the kernel of delta sets to zero
    uint32_t* err;
};

// Parts of dk and dv that 64 MB hold: packed states may lie in many more rows than their sequences name
inline long long cross_parts_held(const CrossArgs& a) {
    const long long bytes = 8LL * (a.where.offsets ? 1 : a.where.n_enc) * a.where.kv_rows * a.kv_heads * a.d;
    return bytes > 0 && (64LL << 20) / bytes > 1 ? (64LL << 20) / bytes : 1;
}

// Tensor cores, bf16
bool cross_tc_supported(const CrossArgs& a);
int cross_tc_parts(const CrossArgs& a);
int cross_tc_forward(const CrossArgs& a, const CrossParts& parts, cudaStream_t s);
bool cross_bwd_tc_supported(const CrossArgs& a);
int cross_bwd_tc_parts(const CrossArgs& a);   // of the tokens, for dk and dv: fp32 [part][2][state rows][key heads][d] in the workspace where there are several
int cross_bwd_tc_dq(const CrossArgs& a, cudaStream_t s);
int cross_bwd_tc_dkv(const CrossArgs& a, int parts, float* part_out, cudaStream_t s);
int cross_join(int dtype, const CrossArgs& a, const CrossParts& parts, cudaStream_t s);
int cross_bwd_join(int dtype, const CrossArgs& a, int parts, const float* part_out, cudaStream_t s);      // dk and dv from their parts

// Few tokens, fp32 or bf16
bool cross_rows_supported(int dtype, const CrossArgs& a);
int cross_rows_parts(const CrossArgs& a);
int cross_rows_forward(int dtype, const CrossArgs& a, const CrossParts& parts, cudaStream_t s);

// CUDA cores, fp32 or bf16, any strides and alignment
int cross_simt_forward(int dtype, const CrossArgs& a, cudaStream_t s);
int cross_delta(int dtype, const CrossArgs& a, cudaStream_t s);
int cross_simt_dq(int dtype, const CrossArgs& a, cudaStream_t s);
int cross_simt_dkv_parts(const CrossArgs& a); // as cross_bwd_tc_parts
int cross_simt_dkv(int dtype, const CrossArgs& a, int parts, float* part_out, cudaStream_t s);
