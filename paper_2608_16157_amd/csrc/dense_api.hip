// C ABI entry points of the dense 8-bit product, the 8-bit activation forms, the SwiGLU between two dense
// products and the router's balance loss: host-side validation, workspace carving, kernel enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "ftmoe_internal.h"

using namespace ftmoe;

namespace {

constexpr int kMaxDim = 65536;       // features
constexpr int kMaxTokens = 1048576;

bool dim_ok(int n) { return n >= 16 && n <= kMaxDim && n % 16 == 0; }
bool tokens_ok(int T) { return T >= 0 && T <= kMaxTokens; }
bool float_dtype(int d) { return d == FT_DT_F32 || d == FT_DT_BF16; }
bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }

ActForm form(const ft_act_codes_t *c, int R, int K) {
    if (!c) return ActForm{};
    return ActForm{c->codes, c->scales, R, pad128(K), pad128(R)};
}

// a form that the call reads or writes
ft_status_t form_status(const ft_act_codes_t *c) {
    if (!c || !c->codes || !c->scales) return FT_ERR_NULL;
    return aligned(c->codes) && aligned(c->scales) ? FT_OK : FT_ERR_SHAPE;
}
// one that may be left out
ft_status_t optional_status(const ft_act_codes_t *c) { return c ? form_status(c) : FT_OK; }

ft_status_t linear_status(const ft_linear_desc_t *d) {
    if (!d) return FT_ERR_NULL;
    if (!dim_ok(d->out_features) || !dim_ok(d->in_features)) return FT_ERR_SHAPE;
    if (!float_dtype(d->x_dtype) && d->x_dtype != FT_DT_FP8_ACT) return FT_ERR_DTYPE;
    return float_dtype(d->y_dtype) ? FT_OK : FT_ERR_DTYPE;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// ft_linear's workspace: the row form of x, and the parts of a split reduction (product_plan holds their
// bytes to kSplitBytes, and to kMaxParts outputs).  Grows with T.
struct LinearWs {
    size_t codes, scales, parts, total;
};
LinearWs linear_ws(const ft_linear_desc_t *d, int T) {
    const size_t Kp = pad128(d->in_features), Tp = pad128(std::max(T, 1));
    const bool packed = d->x_dtype == FT_DT_FP8_ACT;
    LinearWs w;
    w.codes = 0;
    w.scales = packed ? 0 : Tp * Kp;
    w.parts = w.scales + (packed ? 0 : round256(Tp * (Kp / 128)));
    w.total = w.parts + std::min(kSplitBytes, round256(static_cast<size_t>(kMaxParts) * std::max(T, 1) * d->out_features * 4));
    return w;
}

ft_status_t balance_status(const ft_balance_desc_t *d) {
    if (!d) return FT_ERR_NULL;
    if (d->n_experts < 1 || d->n_experts > kMaxExperts || d->top_k < 1 || d->top_k > d->n_experts || d->top_k > kMaxTopK)
        return FT_ERR_SHAPE;
    if (d->n_seq < 1 || d->n_seq > 65536) return FT_ERR_SHAPE;
    if (d->gating != FT_GATE_SOFTMAX_TOPK_RENORM && d->gating != FT_GATE_SIGMOID_TOPK_RENORM) return FT_ERR_DTYPE;
    return FT_OK;
}

int max_parts(int T) { return std::min(kBalMaxParts, (T + kBalMinPart - 1) / kBalMinPart); }

struct BalanceWs {
    size_t sums, tokens, total;
};
BalanceWs balance_ws(const ft_balance_desc_t *d, int T) {
    const size_t rows = static_cast<size_t>(max_parts(std::max(T, 1))) + d->n_seq;
    BalanceWs w;
    w.sums = 0;
    w.tokens = round256(rows * d->n_experts * 8);
    w.total = w.tokens + round256(rows * 4);
    return w;
}

BalanceArgs balance_args(const ft_balance_desc_t *d, const float *logits, const int32_t *topk_ids, const int32_t *seq_off,
                         const uint8_t *mask, int T, const ft_balance_t *b) {
    BalanceArgs a{};
    a.logits = logits;
    a.topk_ids = topk_ids;
    a.seq_off = seq_off;
    a.mask = mask;
    a.T = T;
    a.E = d->n_experts;
    a.k = d->top_k;
    a.gating = d->gating;
    a.n_seq = d->n_seq;
    a.frac_scale = static_cast<double>(d->coef) * d->n_experts / d->top_k;
    if (b) {
        a.counts = b->counts;
        a.tokens = b->tokens;
        a.prob = b->prob;
        a.frac = b->frac;
        a.loss = b->loss;
    }
    return a;
}

}  // namespace

extern "C" {

ft_status_t ft_act_quantize(const void *x, int32_t x_dtype, int32_t T, int32_t C, const ft_act_codes_t *row,
                            const ft_act_codes_t *col, void *stream) {
    if (!dim_ok(C) || !tokens_ok(T)) return FT_ERR_SHAPE;
    if (!float_dtype(x_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!x || (!row && !col)) return FT_ERR_NULL;
    if (ft_status_t s = optional_status(row); s != FT_OK) return s;
    if (ft_status_t s = optional_status(col); s != FT_OK) return s;
    if (!aligned(x)) return FT_ERR_SHAPE;
    const hipError_t e = launch_act_quantize(x, x_dtype == FT_DT_F32, T, C, form(row, T, C), form(col, C, T),
                                             static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FT_OK : FT_ERR_HIP;
}

size_t ft_linear_workspace_bytes(const ft_linear_desc_t *desc, int32_t max_tokens) {
    if (linear_status(desc) != FT_OK || !tokens_ok(max_tokens)) return 0;
    const LinearWs w = linear_ws(desc, max_tokens);
    return w.total;
}

ft_status_t ft_linear(const ft_linear_desc_t *desc, const uint8_t *w, const float *w_scales, const void *x,
                      const uint8_t *x_scales, int32_t T, void *y, void *ws, size_t ws_bytes, void *stream) {
    if (ft_status_t s = linear_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    if (T == 0) return FT_OK;
    const bool packed = desc->x_dtype == FT_DT_FP8_ACT;
    if (!w || !w_scales || !x || !y || (packed && !x_scales) || (!packed && !ws)) return FT_ERR_NULL;
    const LinearWs L = linear_ws(desc, T);
    if (ws && ws_bytes < L.total) return FT_ERR_CAPACITY;
    if (!aligned(w) || !aligned(x) || !aligned(y) || (packed && !aligned(x_scales)) || !aligned(ws) ||
        reinterpret_cast<uintptr_t>(w_scales) % 4)
        return FT_ERR_SHAPE;
    const hipStream_t s = static_cast<hipStream_t>(stream);
    uint8_t *base = static_cast<uint8_t *>(ws);
    ProductArgs p{};
    p.a = w;
    p.as = w_scales;
    p.out = y;
    p.M = desc->out_features;
    p.R = T;
    p.K = desc->in_features;
    p.Kp = pad128(p.K);
    p.bsr = pad128(T);
    int bx = 0;
    if (packed) {
        p.b = static_cast<const uint8_t *>(x);
        p.bs = x_scales;
    } else if (T <= kDirectTokens && T * p.Kp <= kDirectBytes) {
        p.x = x;
        bx = desc->x_dtype == FT_DT_BF16 ? 1 : 2;
    } else {
        const ft_act_codes_t q{base + L.codes, base + L.scales};
        if (launch_act_quantize(x, desc->x_dtype == FT_DT_F32, T, p.K, form(&q, T, p.K), ActForm{}, s) != hipSuccess)
            return FT_ERR_HIP;
        p.b = q.codes;
        p.bs = q.scales;
    }
    float *parts = ws ? reinterpret_cast<float *>(base + L.parts) : nullptr;
    return launch_product(p, false, bx, desc->y_dtype == FT_DT_F32 ? 1 : 0, parts, s) == hipSuccess ? FT_OK : FT_ERR_HIP;
}

ft_status_t ft_linear_transpose(int32_t out_features, int32_t in_features, const uint8_t *w, const float *w_scales,
                                uint8_t *wt, float *wt_scales, void *stream) {
    if (!dim_ok(out_features) || !dim_ok(in_features)) return FT_ERR_SHAPE;
    if (!w || !w_scales || !wt || !wt_scales) return FT_ERR_NULL;
    if (!aligned(w) || !aligned(wt) || reinterpret_cast<uintptr_t>(w_scales) % 4 || reinterpret_cast<uintptr_t>(wt_scales) % 4)
        return FT_ERR_SHAPE;
    return launch_weight_transpose(w, w_scales, wt, wt_scales, out_features, in_features, static_cast<hipStream_t>(stream)) ==
                   hipSuccess
               ? FT_OK
               : FT_ERR_HIP;
}

ft_status_t ft_linear_weight_grad(int32_t out_features, int32_t in_features, int32_t T, const ft_act_codes_t *dy_col,
                                  const ft_act_codes_t *x_col, void *dw, int32_t dw_dtype, int32_t accumulate, void *stream) {
    if (!dim_ok(out_features) || !dim_ok(in_features) || !tokens_ok(T) || (accumulate != 0 && accumulate != 1))
        return FT_ERR_SHAPE;
    if (!float_dtype(dw_dtype) || (accumulate && dw_dtype != FT_DT_F32)) return FT_ERR_DTYPE;
    if (!dw) return FT_ERR_NULL;
    if (!aligned(dw)) return FT_ERR_SHAPE;
    ProductArgs p{};
    if (T > 0) {
        if (ft_status_t s = form_status(dy_col); s != FT_OK) return s;
        if (ft_status_t s = form_status(x_col); s != FT_OK) return s;
        p.a = x_col->codes;
        p.as = x_col->scales;
        p.b = dy_col->codes;
        p.bs = dy_col->scales;
    } else if (accumulate) {
        return FT_OK;
    }
    p.out = dw;
    p.M = in_features;
    p.R = out_features;
    p.K = T;
    p.Kp = pad128(T);   // T = 0: no block to sum, zeros are stored
    p.asr = pad128(in_features);
    p.bsr = pad128(out_features);
    const int out = dw_dtype == FT_DT_BF16 ? 0 : accumulate ? 2 : 1;
    return launch_product(p, true, 0, out, nullptr, static_cast<hipStream_t>(stream)) == hipSuccess ? FT_OK : FT_ERR_HIP;
}

ft_status_t ft_swiglu_quantize(const void *gu, int32_t gu_dtype, int32_t T, int32_t inter, const ft_act_codes_t *h,
                               const ft_act_codes_t *saved, void *stream) {
    if (inter < 128 || inter > kMaxDim / 2 || inter % 128 || !tokens_ok(T)) return FT_ERR_SHAPE;
    if (!float_dtype(gu_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!gu) return FT_ERR_NULL;
    if (ft_status_t s = form_status(h); s != FT_OK) return s;
    if (ft_status_t s = optional_status(saved); s != FT_OK) return s;
    if (!aligned(gu)) return FT_ERR_SHAPE;
    const hipError_t e = launch_swiglu_quantize(gu, gu_dtype == FT_DT_F32, T, inter, form(h, T, inter),
                                                form(saved, T, 2 * inter), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FT_OK : FT_ERR_HIP;
}

ft_status_t ft_swiglu_backward(const ft_act_codes_t *saved, const void *dh, int32_t dh_dtype, int32_t T, int32_t inter,
                               const ft_act_codes_t *dgu_row, const ft_act_codes_t *dgu_col, const ft_act_codes_t *h_col,
                               void *stream) {
    if (inter < 128 || inter > kMaxDim / 2 || inter % 128 || !tokens_ok(T)) return FT_ERR_SHAPE;
    if (!float_dtype(dh_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!dh || (!dgu_row && !dgu_col && !h_col)) return FT_ERR_NULL;
    if (ft_status_t s = form_status(saved); s != FT_OK) return s;
    for (const ft_act_codes_t *c : {dgu_row, dgu_col, h_col})
        if (ft_status_t s = optional_status(c); s != FT_OK) return s;
    if (!aligned(dh)) return FT_ERR_SHAPE;
    const hipError_t e =
        launch_swiglu_backward(form(saved, T, 2 * inter), dh, dh_dtype == FT_DT_F32, T, inter, form(dgu_row, T, 2 * inter),
                               form(dgu_col, 2 * inter, T), form(h_col, inter, T), static_cast<hipStream_t>(stream));
    return e == hipSuccess ? FT_OK : FT_ERR_HIP;
}

size_t ft_balance_workspace_bytes(const ft_balance_desc_t *desc, int32_t max_tokens) {
    if (balance_status(desc) != FT_OK || !tokens_ok(max_tokens)) return 0;
    return balance_ws(desc, max_tokens).total;
}

ft_status_t ft_balance_loss(const ft_balance_desc_t *desc, const float *logits, const int32_t *topk_ids, int32_t T,
                            const int32_t *seq_off, const uint8_t *mask, const ft_balance_t *out, void *ws,
                            size_t ws_bytes, void *stream) {
    if (ft_status_t s = balance_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    if (!out || !out->counts || !out->tokens || !out->prob || !out->frac || !out->loss || !ws) return FT_ERR_NULL;
    if ((T > 0 && (!logits || !topk_ids)) || (desc->n_seq > 1 && !seq_off)) return FT_ERR_NULL;
    if (ws_bytes < ft_balance_workspace_bytes(desc, T)) return FT_ERR_CAPACITY;
    if (!aligned(ws)) return FT_ERR_SHAPE;
    BalanceArgs a = balance_args(desc, logits, topk_ids, seq_off, mask, T, out);
    if (T > kBalWholeTokens) {
        const BalanceWs w = balance_ws(desc, T);
        uint8_t *b = static_cast<uint8_t *>(ws);
        a.part_tokens = (T + max_parts(T) - 1) / max_parts(T);
        a.parts = (T + a.part_tokens - 1) / a.part_tokens;
        a.ws_sums = reinterpret_cast<float2 *>(b + w.sums);
        a.ws_tokens = reinterpret_cast<int32_t *>(b + w.tokens);
    }
    return launch_balance(a, static_cast<hipStream_t>(stream)) == hipSuccess ? FT_OK : FT_ERR_HIP;
}

ft_status_t ft_router_backward(const ft_balance_desc_t *desc, const float *logits, const int32_t *topk_ids, int32_t T,
                               const int32_t *seq_off, const uint8_t *mask, const ft_balance_t *balance,
                               const float *d_loss, const float *topk_w, const float *d_topk_w, float *d_logits,
                               void *stream) {
    if (ft_status_t s = balance_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    if (T == 0) return FT_OK;
    if (!logits || !d_logits || (!d_loss && !d_topk_w) || (desc->n_seq > 1 && !seq_off)) return FT_ERR_NULL;
    if (d_loss && (!balance || !balance->tokens || !balance->frac)) return FT_ERR_NULL;
    if (d_topk_w && (!topk_ids || !topk_w)) return FT_ERR_NULL;
    BalanceArgs a = balance_args(desc, logits, topk_ids, seq_off, mask, T, balance);
    a.topk_w = topk_w;
    a.d_topk_w = d_topk_w;
    a.d_loss = d_loss;
    a.d_logits = d_logits;
    return launch_router_backward(a, static_cast<hipStream_t>(stream)) == hipSuccess ? FT_OK : FT_ERR_HIP;
}

}  // extern "C"
