// Root-mean-square norm: argument checks and entry points.
#include "rms_norm.h"

namespace {

bool known(int dtype) { return dtype == FREE_FP32 || dtype == FREE_BF16; }
bool words(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3u) == 0; }
bool whole(const void* p, int dtype) { return (reinterpret_cast<uintptr_t>(p) & (dtype == FREE_FP32 ? 3u : dtype == FREE_BF16 ? 1u : 0u)) == 0; }
// an address counted in elements: what the accesses' width depends on is its low bits
long long place(const void* p, int dtype) { return (long long)(reinterpret_cast<uintptr_t>(p) / (dtype == FREE_FP32 ? 4 : dtype == FREE_BF16 ? 2 : 1)) & 7; }

// rows >= D apart: of the heads of a token, and of neighbouring tokens
bool apart(long long tok, long long head, int heads, int D) {
    if (heads == 1) return tok >= D;
    return head >= D && tok >= 0 && (tok >= (heads - 1LL) * head + D || (tok >= D && head >= tok));
}

}  // namespace

extern "C" int free_op_rms_norm(int x_dtype, int res_dtype, int y_dtype, int n_groups, int rows_per_group, int heads, int D,
                                const void* x, int64_t x_tok, int64_t x_head, const void* residual, int64_t res_stride,
                                void* res_out, int64_t res_out_stride, const float* weight, int64_t mod_stride, int unit_offset, float eps,
                                void* y, int64_t y_tok, int64_t y_head, float* scales, int64_t scale_stride, int scale_block, float* rstd, void* stream) {
    if (!known(x_dtype) || !(known(y_dtype) || y_dtype == FREE_E4M3) || (residual && !known(res_dtype)) || !(eps >= 0.f)) return FREE_ERR_ARG;
    if (n_groups < 0 || rows_per_group < 0 || heads < 1 || D < 1) return FREE_ERR_SHAPE;
    const long long M = (long long)n_groups * rows_per_group;
    if (M % heads) return FREE_ERR_SHAPE;
    if (y_dtype == FREE_E4M3 && (heads > 1 || (scale_block != 0 && scale_block != 128))) return FREE_ERR_ARG;
    if (heads > 1 && residual) return FREE_ERR_ARG;
    if (M == 0) return FREE_OK;
    if (!x || !y || (!residual && res_out) || (y_dtype == FREE_E4M3 && !scales)) return FREE_ERR_ARG;
    if (x_tok < 0 || x_head < 0 || !apart(y_tok, y_head, heads, D)) return FREE_ERR_SHAPE;
    if ((residual && res_stride < D) || (res_out && res_out_stride < D) || (weight && n_groups > 1 && mod_stride < 0)) return FREE_ERR_SHAPE;
    if (y_dtype == FREE_E4M3 && scale_stride < (scale_block ? (D + 127) / 128 : 1)) return FREE_ERR_SHAPE;
    if (!whole(x, x_dtype) || !whole(y, y_dtype) || !whole(residual, res_dtype) || !whole(res_out, res_dtype) || !words(weight) || !words(scales) || !words(rstd))
        return FREE_ERR_ALIGN;
    if (D > kRmsMaxD) return FREE_ERR_UNSUPPORTED;
    RmsArgs a{};
    a.M = M; a.D = D; a.heads = heads; a.rows_per_group = rows_per_group;
    a.x = x; a.x_tok = x_tok; a.x_head = x_head; a.res = residual; a.res_stride = res_stride; a.h = res_out; a.h_stride = res_out_stride;
    a.weight = weight; a.mod_stride = mod_stride; a.unit = unit_offset ? 1.f : 0.f; a.eps = eps;
    a.y = y; a.y_tok = y_tok; a.y_head = y_head; a.scales = scales; a.scale_stride = scale_stride; a.scale_block = scale_block; a.rstd = rstd;
    // four consecutive columns per access where everything is aligned to four elements
    const long long strides = x_tok | y_tok | (heads > 1 ? x_head | y_head : 0) | (residual ? res_stride : 0) | (res_out ? res_out_stride : 0) |
                              (weight && n_groups > 1 ? mod_stride : 0) | place(x, x_dtype) | place(y, y_dtype) |
                              (residual ? place(residual, res_dtype) : 0) | (res_out ? place(res_out, res_dtype) : 0);
    // (eight where every type has 16 bits or fewer, but for widths that have a kernel of whole blocks of 128 columns: 200 MB of bf16 rows in bf16
    // results take as long either way, 384 columns 87 and 88 us by eight, 768 80 and 80, or longer, 640 78 and 86, 1152 77 and 93.  Their
    // 8-bit results with scales per 128 columns halve the exchanges by eight, which pays where the row fills three quarters of that
    // kernel's 256, 512 or 1024 columns: 512 columns 86 us, by four 113, 384 116 and 121, 896 96 and 126, but 640 121 and 112, 128 205 and 179)
    int vw = D % 4 == 0 && strides % 4 == 0 && free_aligned16(weight) ? 4 : 1;
    const bool thin = x_dtype == FREE_BF16 && y_dtype != FREE_FP32 && (!residual || res_dtype == FREE_BF16);
    // heads that would leave lanes idle: 24 x 1024 tokens, 16 heads of 72, 25 us by four, 27 by eight; 12 of 96 20 and 21; 11 of 104 25 and 21;
    // 9 of 128 23 and 19
    const bool as_heads = !residual && y_dtype != FREE_E4M3 && D <= 128, idle = as_heads && D > 64 && D <= 96;
    const bool exact = !as_heads && D <= 1152 && D % 128 == 0, eight_bits = y_dtype == FREE_E4M3 && scale_block != 0;
    const int held = D <= 256 ? 256 : D <= 512 ? 512 : (D + 1023) / 1024 * 1024;
    if (vw == 4 && thin && D % 8 == 0 && strides % 8 == 0 && !idle && (!exact || (eight_bits && 4 * D >= 3 * held))) vw = 8;
    cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
    const bool rf = residual && res_dtype == FREE_FP32;            // without a residual its type does not matter
    if (x_dtype == FREE_FP32) return rf ? rms_norm_ff(a, vw, y_dtype, s) : rms_norm_fb(a, vw, y_dtype, s);
    return rf ? rms_norm_bf(a, vw, y_dtype, s) : rms_norm_bb(a, vw, y_dtype, s);
}

extern "C" size_t free_op_rms_norm_bwd_workspace_bytes(int n_groups, int rows_per_group, int D) {
    return n_groups < 1 || rows_per_group < 1 || D < 1 || D > kRmsMaxD ? 0 : rms_norm_bwd_bytes(n_groups, rows_per_group, D);
}

extern "C" int free_op_rms_norm_bwd(int x_dtype, int dy_dtype, int n_groups, int rows_per_group, int heads, int D,
                                    const void* h, int64_t h_tok, int64_t h_head, const void* dy, int64_t dy_tok, int64_t dy_head, const float* rstd,
                                    const float* weight, int64_t mod_stride, int unit_offset, const void* dres, int64_t dres_tok, int64_t dres_head,
                                    void* dx, int64_t dx_tok, int64_t dx_head, float* dweight, int64_t dmod_stride,
                                    void* ws, size_t ws_bytes, void* stream) {
    if (!known(x_dtype) || !known(dy_dtype)) return FREE_ERR_ARG;
    if (n_groups < 0 || rows_per_group < 0 || heads < 1 || D < 1) return FREE_ERR_SHAPE;
    const long long M = (long long)n_groups * rows_per_group;
    if (M % heads) return FREE_ERR_SHAPE;
    if (n_groups == 0) return FREE_OK;
    if (M > 0 && (!h || !dy || !rstd || !dx)) return FREE_ERR_ARG;
    if (M > 0 && (h_tok < 0 || h_head < 0 || dy_tok < 0 || dy_head < 0 || (dres && (dres_tok < 0 || dres_head < 0)) || !apart(dx_tok, dx_head, heads, D)))
        return FREE_ERR_SHAPE;
    if ((weight && n_groups > 1 && mod_stride < 0) || (dweight && n_groups > 1 && dmod_stride < D)) return FREE_ERR_SHAPE;
    if (!whole(h, x_dtype) || !whole(dy, dy_dtype) || !whole(dres, x_dtype) || !whole(dx, x_dtype) || !free_aligned16(ws) || !words(rstd) || !words(weight) ||
        !words(dweight)) return FREE_ERR_ALIGN;
    if (D > kRmsMaxD) return FREE_ERR_UNSUPPORTED;
    if (M == 0 && !dweight) return FREE_OK;
    if (heads > 1 && !rms_norm_bwd_takes_heads(D)) {
        auto even = [&](long long tok, long long head) { return tok == head * heads; };
        if (M > heads && (!even(h_tok, h_head) || !even(dy_tok, dy_head) || !even(dx_tok, dx_head) || (dres && !even(dres_tok, dres_head)))) return FREE_ERR_UNSUPPORTED;
        heads = 1; h_tok = h_head; dy_tok = dy_head; dx_tok = dx_head; dres_tok = dres_head;
    }
    RmsBwdArgs a{};
    a.x_dtype = x_dtype; a.dy_dtype = dy_dtype; a.D = D; a.heads = heads; a.groups = n_groups; a.rows_per_group = rows_per_group;
    a.x = h; a.x_tok = h_tok; a.x_head = h_head; a.dy = dy; a.dy_tok = dy_tok; a.dy_head = dy_head; a.rstd = rstd;
    a.weight = weight; a.mod_stride = mod_stride; a.unit = unit_offset ? 1.f : 0.f;
    a.dres = dres; a.dres_tok = dres_tok; a.dres_head = dres_head; a.dx = dx; a.dx_tok = dx_tok; a.dx_head = dx_head;
    a.dw = dweight; a.dmod_stride = dmod_stride; a.ws = (float*)ws; a.ws_bytes = ws_bytes;
    return rms_norm_bwd(a, reinterpret_cast<cudaStream_t>(stream));
}
