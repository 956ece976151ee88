// Attention to an encoder's states: argument checks, choice of kernel and entry points.
#include "cross_tc.cuh"

namespace {

bool aligned(const void* p, int a) { return (reinterpret_cast<uintptr_t>(p) & (uintptr_t)(a - 1)) == 0; }

// FREE_OK and `empty` where nothing is to be done
int check(const free_cross_attn* c, bool* empty) {
    *empty = false;
    if (!c) return FREE_ERR_ARG;
    if (c->dtype != FREE_FP32 && c->dtype != FREE_BF16) return FREE_ERR_ARG;
    if (!(c->scale > 0.f) || c->scale > 2.3e38f) return FREE_ERR_ARG;      // (times log2 e it is finite)
    if (c->n_seq < 0 || c->n_q < 0 || c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads || c->d_head < 1) return FREE_ERR_SHAPE;
    if (c->n_enc < 0 || c->n_kv < 0 || c->kv_rows < 0) return FREE_ERR_SHAPE;
    if (c->kv_offsets && c->kv_lens) return FREE_ERR_ARG;
    if (c->n_enc == 0 ? c->n_seq != 0 : (!c->kv_seq && c->n_seq % c->n_enc)) return FREE_ERR_SHAPE;
    for (long long v : {c->q_seq, c->q_tok, c->q_head, c->k_seq, c->k_tok, c->k_head, c->v_seq, c->v_tok, c->v_head})
        if (v < 0) return FREE_ERR_SHAPE;
    if (c->d_head > kCrossMaxD) return FREE_ERR_UNSUPPORTED;
    // kernels count tokens, states and sequences in steps of up to 2048 behind the last one
    for (int n : {c->n_seq, c->n_q, c->n_enc, c->n_kv, c->kv_rows})
        if (n > kCrossMaxLength) return FREE_ERR_UNSUPPORTED;
    // rows of lse, tiles and tile copies' coordinates are counted in 31 bits
    long long blocks = (long long)c->n_enc * (c->n_kv / 64 + 1);
    if (c->kv_offsets && blocks > c->n_enc + (long long)(c->kv_rows / 64)) blocks = c->n_enc + (long long)(c->kv_rows / 64);
    if ((long long)c->n_seq * c->heads > 0x7fffffffLL / (c->n_q / 64 + 1) || blocks > 0x7fffffffLL / c->kv_heads) return FREE_ERR_UNSUPPORTED;
    *empty = c->n_seq == 0 || c->n_q == 0;
    return FREE_OK;
}
bool rows_of_states(const free_cross_attn* c) { return c->n_enc > 0 && (c->kv_offsets ? c->kv_rows : c->n_kv) > 0; }
bool states(const free_cross_attn* c) { return rows_of_states(c) && c->n_kv > 0; }

int pointers(const free_cross_attn* c, bool tokens) {              // (a call without tokens reads the states still: which of them count)
    const int e = c->dtype == FREE_FP32 ? 4 : 2;
    if ((tokens && !c->q) || (states(c) && (!c->k || !c->v))) return FREE_ERR_ARG;
    if ((tokens && !aligned(c->q, e)) || !aligned(c->k, e) || !aligned(c->v, e)) return FREE_ERR_ALIGN;
    if (!aligned(c->kv_lens, 4) || !aligned(c->kv_offsets, 4) || !aligned(c->kv_seq, 4)) return FREE_ERR_ALIGN;
    return FREE_OK;
}

CrossArgs args_of(const free_cross_attn* c) {
    CrossArgs a{};
    a.q = CrossMat{c->q, c->q_seq, c->q_tok, c->q_head};
    a.k = CrossMat{c->k, c->kv_offsets ? 0 : c->k_seq, c->k_tok, c->k_head};
    a.v = CrossMat{c->v, c->kv_offsets ? 0 : c->v_seq, c->v_tok, c->v_head};
    a.where = CrossWhere{c->kv_lens, c->kv_offsets, c->kv_seq, c->kv_mask, c->n_enc, states(c) ? c->n_kv : 0, c->kv_offsets ? c->kv_rows : c->n_kv, 1};
    if (!c->kv_seq && c->n_enc) a.where.share = c->n_seq / c->n_enc > 0 ? c->n_seq / c->n_enc : 1;
    a.n_seq = c->n_seq; a.n_q = c->n_q; a.heads = c->heads; a.kv_heads = c->kv_heads; a.d = c->d_head; a.group = c->heads / c->kv_heads;
    a.scale = c->scale;
    return a;
}

// heads and tokens of a result must not lie on one another
bool apart(long long seq, long long tok, long long head, int n_seq, int n_tok, int heads, int d) {
    const long long st[3] = {head, tok, seq};
    const int n[3] = {heads, n_tok, n_seq};
    int order[3] = {0, 1, 2};
    for (int i = 0; i < 3; ++i)
        for (int j = i + 1; j < 3; ++j)
            if (st[order[j]] < st[order[i]]) { const int t = order[i]; order[i] = order[j]; order[j] = t; }
    long long end = d;                                             // elements from the first to behind the last so far
    for (int i = 0; i < 3; ++i) {
        const int k = order[i];
        if (n[k] <= 1) continue;
        if (st[k] < end) return false;
        end += (n[k] - 1LL) * st[k];
    }
    return true;
}

int result(const void* p, int e, long long seq, long long tok, long long head, int n_seq, int n_tok, int heads, int d) {
    if (!p) return FREE_ERR_ARG;
    if (!aligned(p, e)) return FREE_ERR_ALIGN;
    if (seq < 0 || tok < 0 || head < 0 || !apart(seq, tok, head, n_seq, n_tok, heads, d)) return FREE_ERR_SHAPE;
    return FREE_OK;
}

size_t row_count(const free_cross_attn* c) { return (size_t)c->n_seq * c->heads * c->n_q; }

// Which kernel, and parts of the states: few rows on their own, bf16 on the tensor cores, the rest on CUDA cores.
enum Way { ROWS, TENSOR, SIMT };
Way way_of(const CrossArgs& a, int dtype, int* parts) {
    *parts = 1;
    if (cross_rows_supported(dtype, a)) { *parts = cross_rows_parts(a); return ROWS; }
    if (dtype == FREE_BF16 && cross_tc_supported(a)) { *parts = cross_tc_parts(a); return TENSOR; }
    return SIMT;
}
size_t part_bytes(const free_cross_attn* c, int parts) { return parts > 1 ? free_round_up(row_count(c) * parts * 4, 256) + row_count(c) * parts * c->d_head * 4 : 0; }

// parts of dk and dv
size_t sum_bytes(const free_cross_attn* c, int parts) {
    return parts > 1 ? (size_t)parts * 2 * (c->kv_offsets ? 1 : c->n_enc) * (c->kv_offsets ? c->kv_rows : c->n_kv) * c->kv_heads * c->d_head * 4 : 0;
}
constexpr size_t kNextBytes = 256;
size_t stat_bytes(const free_cross_attn* c) { return free_round_up((size_t)c->n_seq * c->heads * c->n_q * 4, 256); }

}  // namespace

extern "C" size_t free_op_cross_attention_workspace_bytes(const free_cross_attn* c) {
    bool empty;
    if (check(c, &empty) != FREE_OK || empty) return 0;
    // where the inputs turn out to be no matter for the tensor cores, less is used
    CrossArgs a = args_of(c);
    a.o = a.q;
    int parts;
    way_of(a, c->dtype, &parts);
    return part_bytes(c, parts);
}

extern "C" int free_op_cross_attention(const free_cross_attn* c, void* out, int64_t o_seq, int64_t o_tok, int64_t o_head, float* lse, void* ws,
                                       size_t ws_bytes, uint32_t* device_error, void* stream) {
    bool empty;
    FREE_TRY(check(c, &empty));
    if (empty) return FREE_OK;
    FREE_TRY(pointers(c, true));
    FREE_TRY(result(out, c->dtype == FREE_FP32 ? 4 : 2, o_seq, o_tok, o_head, c->n_seq, c->n_q, c->heads, c->d_head));
    if (!aligned(lse, 4)) return FREE_ERR_ALIGN;
    if (c->dtype == FREE_BF16 && !device_error) return FREE_ERR_ARG;
    CrossArgs a = args_of(c);
    a.o = CrossMat{out, o_seq, o_tok, o_head};
    a.lse = lse; a.err = device_error;
    CrossParts p{1, nullptr, nullptr};
    const Way way = way_of(a, c->dtype, &p.n);
    if (p.n > 1) {
        if (!ws || ws_bytes < part_bytes(c, p.n)) return FREE_ERR_WORKSPACE;
        if (!free_aligned16(ws)) return FREE_ERR_ALIGN;
        p.lse = (float*)ws;
        p.out = (float*)((char*)ws + free_round_up(row_count(c) * p.n * 4, 256));
    }
    if (way == ROWS) return cross_rows_forward(c->dtype, a, p, (cudaStream_t)stream);
    if (way == TENSOR) return cross_tc_forward(a, p, (cudaStream_t)stream);
    return cross_simt_forward(c->dtype, a, (cudaStream_t)stream);
}

extern "C" size_t free_op_cross_attention_bwd_workspace_bytes(const free_cross_attn* c) {
    bool empty;
    if (check(c, &empty) != FREE_OK || empty) return 0;
    CrossArgs a = args_of(c);
    a.g = a.q;
    const size_t simt = sum_bytes(c, cross_simt_dkv_parts(a)), tc = c->dtype == FREE_BF16 && cross_bwd_tc_supported(a) ? sum_bytes(c, cross_bwd_tc_parts(a)) : 0;
    return stat_bytes(c) + kNextBytes + (simt > tc ? simt : tc);
}

extern "C" int free_op_cross_attention_bwd(const free_cross_attn* c, const void* out, int64_t o_seq, int64_t o_tok, int64_t o_head, const float* lse,
                                           const void* dout, int64_t g_seq, int64_t g_tok, int64_t g_head,
                                           void* dq, int64_t dq_seq, int64_t dq_tok, int64_t dq_head,
                                           void* dk, int64_t dk_seq, int64_t dk_tok, int64_t dk_head,
                                           void* dv, int64_t dv_seq, int64_t dv_tok, int64_t dv_head,
                                           void* ws, size_t ws_bytes, uint32_t* device_error, void* stream) {
    bool empty;
    FREE_TRY(check(c, &empty));
    const cudaStream_t s = (cudaStream_t)stream;
    const int e = c->dtype == FREE_FP32 ? 4 : 2;
    if (!dk != !dv) return FREE_ERR_ARG;
    const int enc = c->kv_offsets ? 1 : c->n_enc, rows = c->kv_offsets ? c->kv_rows : c->n_kv;
    if (dk && rows_of_states(c)) {
        FREE_TRY(pointers(c, !empty));
        FREE_TRY(result(dk, e, c->kv_offsets ? 0 : dk_seq, dk_tok, dk_head, enc, rows, c->kv_heads, c->d_head));
        FREE_TRY(result(dv, e, c->kv_offsets ? 0 : dv_seq, dv_tok, dv_head, enc, rows, c->kv_heads, c->d_head));
    }
    if (!empty) {
        FREE_TRY(pointers(c, true));
        if (!out || !lse || !dout) return FREE_ERR_ARG;
        if (!aligned(out, e) || !aligned(dout, e) || !aligned(lse, 4)) return FREE_ERR_ALIGN;
        for (long long v : {o_seq, o_tok, o_head, g_seq, g_tok, g_head})
            if (v < 0) return FREE_ERR_SHAPE;
        if (dq) FREE_TRY(result(dq, e, dq_seq, dq_tok, dq_head, c->n_seq, c->n_q, c->heads, c->d_head));
        if (c->dtype == FREE_BF16 && !device_error) return FREE_ERR_ARG;
        if (!ws || ws_bytes < free_op_cross_attention_bwd_workspace_bytes(c)) return FREE_ERR_WORKSPACE;
        if (!free_aligned16(ws)) return FREE_ERR_ALIGN;
    }
    CrossArgs a = args_of(c);
    a.o = CrossMat{out, o_seq, o_tok, o_head};
    a.g = CrossMat{dout, g_seq, g_tok, g_head};
    a.dq = CrossMat{dq, dq_seq, dq_tok, dq_head};
    a.dk = CrossMat{dk, c->kv_offsets ? 0 : dk_seq, dk_tok, dk_head};
    a.dv = CrossMat{dv, c->kv_offsets ? 0 : dv_seq, dv_tok, dv_head};
    a.lse = const_cast<float*>(lse); a.delta = (float*)ws; a.next = (unsigned long long*)((char*)ws + stat_bytes(c)); a.err = device_error;
    if (!empty && (dq || dk)) FREE_TRY(cross_delta(c->dtype, a, s));
    // the tensor cores where the tile copies take every matrix (an empty call only writes zeros)
    const bool tc = c->dtype == FREE_BF16 && !empty && cross_bwd_tc_supported(a);
    // (more than a million tiles of states are over a second's work for an item, whose waits give up after two)
    if (!empty && dq)
        FREE_TRY(tc && c->n_kv >> 6 <= 1 << 20 && cross_tc::mappable(a.dq, c->n_seq, c->n_q, c->heads) ? cross_bwd_tc_dq(a, s) : cross_simt_dq(c->dtype, a, s));
    if (dk && rows_of_states(c)) {
        float* parts = empty ? nullptr : (float*)((char*)ws + stat_bytes(c) + kNextBytes);
        if (tc && cross_tc::mappable(a.dk, enc, rows, c->kv_heads) && cross_tc::mappable(a.dv, enc, rows, c->kv_heads))
            FREE_TRY(cross_bwd_tc_dkv(a, cross_bwd_tc_parts(a), parts, s));
        else
            FREE_TRY(cross_simt_dkv(c->dtype, a, empty ? 1 : cross_simt_dkv_parts(a), parts, s));
    }
    return FREE_OK;
}
