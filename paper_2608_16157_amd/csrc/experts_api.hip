// C ABI entry points of the routed experts in training (sorted pairs, rows of tokens, products over the groups) and of
// the norms around the block: host-side validation, workspace carving, kernel enqueue.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "ftmoe_internal.h"

using namespace ftmoe;

namespace {

constexpr int kMaxDim = 65536;       // features
constexpr int kMaxTokens = 1048576;
constexpr int kMaxRows = 1048576;

bool dim_ok(int n) { return n >= 16 && n <= kMaxDim && n % 16 == 0; }
bool tokens_ok(int T) { return T >= 0 && T <= kMaxTokens; }
bool float_dtype(int d) { return d == FT_DT_F32 || d == FT_DT_BF16; }
bool aligned(const void *p) { return reinterpret_cast<uintptr_t>(p) % 16 == 0; }
bool words(const void *p) { return reinterpret_cast<uintptr_t>(p) % 4 == 0; }

ActForm form(const ft_act_codes_t *c, int R, int K) {
    if (!c) return ActForm{};
    return ActForm{c->codes, c->scales, R, pad128(K), pad128(R)};
}
ft_status_t form_status(const ft_act_codes_t *c) {
    if (!c || !c->codes || !c->scales) return FT_ERR_NULL;
    return aligned(c->codes) && aligned(c->scales) ? FT_OK : FT_ERR_SHAPE;
}
ft_status_t optional_status(const ft_act_codes_t *c) { return c ? form_status(c) : FT_OK; }

// without the capacity
ft_status_t experts_status(const ft_sort_desc_t *d) {
    if (!d) return FT_ERR_NULL;
    if (d->n_experts < 1 || d->n_experts > kMaxExperts || d->top_k < 1 || d->top_k > d->n_experts || d->top_k > kMaxTopK)
        return FT_ERR_SHAPE;
    if (d->first < 0 || d->local < 1 || d->first > d->n_experts - d->local) return FT_ERR_SHAPE;
    return d->align == 16 || d->align == 128 ? FT_OK : FT_ERR_SHAPE;
}
ft_status_t sort_status(const ft_sort_desc_t *d) {
    if (ft_status_t s = experts_status(d); s != FT_OK) return s;
    return d->rows >= d->align && d->rows <= kMaxRows && d->rows % d->align == 0 ? FT_OK : FT_ERR_SHAPE;
}

size_t round256(size_t n) { return (n + 255) / 256 * 256; }

// Workgroups of the sort and the pairs of each.
struct SortPlan {
    int pairs, blocks, chunk;
};
SortPlan sort_plan(const ft_sort_desc_t *d, int T) {
    SortPlan p;
    p.pairs = T * d->top_k;   // at most 2^26
    const int held = (p.pairs + kSortPairs - 1) / kSortPairs;
    p.chunk = std::max(1, (held + kSortMaxBlocks - 1) / kSortMaxBlocks) * kSortPairs;
    p.blocks = std::max(1, (p.pairs + p.chunk - 1) / p.chunk);
    return p;
}

struct SortWs {
    size_t table, totals, total;
};
SortWs sort_ws(const ft_sort_desc_t *d, int T) {
    // blocks do not grow with every token past kSortMaxBlocks: room for as many as any smaller T takes
    const long held = (static_cast<long>(T) * d->top_k + kSortPairs - 1) / kSortPairs;
    SortWs w;
    w.table = 0;
    w.totals = round256(static_cast<size_t>(std::min<long>(std::max(held, 1L), kSortMaxBlocks)) * d->local * 4);
    w.total = w.totals + round256(static_cast<size_t>(d->local) * 4);
    return w;
}

RowsArgs rows_args(const ft_sort_desc_t *d, const ft_sort_t *t, int T, int C, const float *w) {
    // a pair's token: pairs are below 2^20 k and k at most 64, so that pair * k < 2^32 and the product's high word is exact
    const uint32_t over_k = d->top_k > 1 ? static_cast<uint32_t>((1ull << 32) / d->top_k + 1) : 0;
    return RowsArgs{t->row_pair, t->pair_row, t->off, w, T, d->top_k, d->local, d->rows, C, over_k};
}

GroupArgs group_args(const ft_sort_desc_t *d, const ft_sort_t *t) {
    return GroupArgs{t->off, t->count, d->local, d->align, d->rows, 0, 0};
}

ft_status_t norm_status(const ft_norm_desc_t *d) {
    if (!d) return FT_ERR_NULL;
    if (!dim_ok(d->channels) || (d->post_norm != 0 && d->post_norm != 1) || !(d->eps >= 0.0f) || !std::isfinite(d->eps) ||
        !std::isfinite(d->scale))
        return FT_ERR_SHAPE;
    return float_dtype(d->x_dtype) && float_dtype(d->y_dtype) && float_dtype(d->w_dtype) ? FT_OK : FT_ERR_DTYPE;
}

NormArgs norm_args(const ft_norm_desc_t *d, const ft_norm_params_t *p, int T) {
    NormArgs a{};
    a.pre = p->pre;
    a.post = p->post;
    a.gate = p->gate;
    a.tgate = p->token_gate;
    a.T = T;
    a.C = d->channels;
    a.post_norm = d->post_norm;
    a.eps = d->eps;
    a.scale = d->scale;
    return a;
}

ft_status_t params_status(const ft_norm_params_t *p) {
    if (!p) return FT_ERR_NULL;
    return aligned(p->pre) && aligned(p->post) && aligned(p->gate) && words(p->token_gate) ? FT_OK : FT_ERR_SHAPE;
}

ft_status_t done(hipError_t e) { return e == hipSuccess ? FT_OK : FT_ERR_HIP; }

}  // namespace

extern "C" {

int32_t ft_expert_sort_rows(const ft_sort_desc_t *desc, int32_t T) {
    if (experts_status(desc) != FT_OK || !tokens_ok(T)) return 0;
    const int64_t pairs = static_cast<int64_t>(T) * desc->top_k, a = desc->align;
    const int64_t rows = std::max(a, (pairs + std::min<int64_t>(desc->local, pairs) * (a - 1)) / a * a);
    return rows <= kMaxRows ? static_cast<int32_t>(rows) : 0;
}

size_t ft_expert_sort_workspace_bytes(const ft_sort_desc_t *desc, int32_t max_tokens) {
    if (sort_status(desc) != FT_OK || !tokens_ok(max_tokens)) return 0;
    return sort_ws(desc, max_tokens).total;
}

ft_status_t ft_expert_sort(const ft_sort_desc_t *desc, const int32_t *topk_ids, int32_t T, const uint8_t *mask,
                           const ft_sort_t *out, void *ws, size_t ws_bytes, void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    if (!out || !out->row_pair || !out->off || !out->count || !out->dropped || !ws) return FT_ERR_NULL;
    if (T > 0 && (!topk_ids || !out->pair_row)) return FT_ERR_NULL;
    const SortWs w = sort_ws(desc, T);
    if (ws_bytes < w.total) return FT_ERR_CAPACITY;
    if (!aligned(ws) || !words(topk_ids) || !words(out->row_pair) || !words(out->pair_row) || !words(out->off) ||
        !words(out->count) || !words(out->dropped))
        return FT_ERR_SHAPE;
    const SortPlan p = sort_plan(desc, T);
    uint8_t *base = static_cast<uint8_t *>(ws);
    SortArgs a{topk_ids, mask, p.pairs, desc->top_k, desc->first, desc->local, desc->align, desc->rows,
               out->row_pair, out->pair_row, out->off, out->count, out->dropped, p.chunk, p.blocks,
               reinterpret_cast<int32_t *>(base + w.table), reinterpret_cast<int32_t *>(base + w.totals)};
    return done(launch_sort(a, static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_gather(const ft_sort_desc_t *desc, const ft_sort_t *sort, const void *x, int32_t x_dtype, int32_t T,
                             int32_t C, const float *weights, void *plain, int32_t plain_dtype, const ft_act_codes_t *row,
                             const ft_act_codes_t *col, void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T) || !dim_ok(C)) return FT_ERR_SHAPE;
    if (!float_dtype(x_dtype) || (plain && !float_dtype(plain_dtype))) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!sort || !sort->row_pair || !sort->off || !x || (!plain && !row && !col)) return FT_ERR_NULL;
    if (ft_status_t s = optional_status(row); s != FT_OK) return s;
    if (ft_status_t s = optional_status(col); s != FT_OK) return s;
    if (!aligned(x) || !aligned(plain) || !words(weights) || !words(sort->row_pair) || !words(sort->off) ||
        (col && desc->align != 128))
        return FT_ERR_SHAPE;
    return done(launch_gather(rows_args(desc, sort, T, C, weights), x, x_dtype == FT_DT_F32, plain, plain_dtype == FT_DT_F32,
                              form(row, desc->rows, C), form(col, C, desc->rows), static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_combine(const ft_sort_desc_t *desc, const ft_sort_t *sort, const void *rows, int32_t rows_dtype,
                              int32_t T, int32_t C, const float *weights, const void *base, void *y, int32_t y_dtype,
                              void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T) || !dim_ok(C)) return FT_ERR_SHAPE;
    if (!float_dtype(rows_dtype) || !float_dtype(y_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!sort || !sort->pair_row || !rows || !y) return FT_ERR_NULL;
    if (!aligned(rows) || !aligned(y) || !aligned(base) || !words(weights) || !words(sort->pair_row)) return FT_ERR_SHAPE;
    return done(launch_combine(rows_args(desc, sort, T, C, weights), rows, rows_dtype == FT_DT_F32, base, y, y_dtype == FT_DT_F32,
                               static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_gate_grad(const ft_sort_desc_t *desc, const ft_sort_t *sort, const void *rows, int32_t rows_dtype,
                                const void *dy, int32_t dy_dtype, int32_t T, int32_t C, float *d_weights, void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T) || !dim_ok(C)) return FT_ERR_SHAPE;
    if (!float_dtype(rows_dtype) || !float_dtype(dy_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!sort || !sort->pair_row || !rows || !dy || !d_weights) return FT_ERR_NULL;
    if (!aligned(rows) || !aligned(dy) || !words(d_weights) || !words(sort->pair_row)) return FT_ERR_SHAPE;
    return done(launch_gate_grad(rows_args(desc, sort, T, C, nullptr), rows, rows_dtype == FT_DT_F32, dy, dy_dtype == FT_DT_F32,
                                 d_weights, static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_linear(const ft_sort_desc_t *desc, const ft_linear_desc_t *linear, const uint8_t *w,
                             const float *w_scales, const ft_act_codes_t *x, const ft_sort_t *sort, int32_t T, void *y,
                             void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!linear) return FT_ERR_NULL;
    if (!dim_ok(linear->out_features) || !dim_ok(linear->in_features) || !tokens_ok(T)) return FT_ERR_SHAPE;
    if (linear->x_dtype != FT_DT_FP8_ACT || !float_dtype(linear->y_dtype)) return FT_ERR_DTYPE;
    if (T == 0) return FT_OK;
    if (!w || !w_scales || !y || !sort || !sort->off || !sort->count) return FT_ERR_NULL;
    if (ft_status_t s = form_status(x); s != FT_OK) return s;
    if (!aligned(w) || !aligned(y) || !words(w_scales) || !words(sort->off) || !words(sort->count)) return FT_ERR_SHAPE;
    ProductArgs p{};
    p.a = w;
    p.as = w_scales;
    p.b = x->codes;
    p.bs = x->scales;
    p.out = y;
    p.M = linear->out_features;
    p.R = desc->rows;
    p.K = linear->in_features;
    p.Kp = pad128(p.K);
    p.bsr = pad128(desc->rows);
    GroupArgs g = group_args(desc, sort);
    g.a_stride = static_cast<size_t>(p.M) * p.Kp;
    g.as_stride = static_cast<size_t>(pad128(p.M) / 128) * (p.Kp / 128);
    const long pairs = static_cast<long>(T) * desc->top_k;
    return done(launch_expert_product(p, g, pairs, static_cast<float>(pairs) / desc->n_experts,
                                      linear->y_dtype == FT_DT_F32 ? 1 : 0, static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_linear_transpose(int32_t n, int32_t out_features, int32_t in_features, const uint8_t *w,
                                       const float *w_scales, uint8_t *wt, float *wt_scales, void *stream) {
    if (n < 1 || n > kMaxExperts || !dim_ok(out_features) || !dim_ok(in_features)) return FT_ERR_SHAPE;
    if (!w || !w_scales || !wt || !wt_scales) return FT_ERR_NULL;
    if (!aligned(w) || !aligned(wt) || !words(w_scales) || !words(wt_scales)) return FT_ERR_SHAPE;
    return done(launch_weight_transpose(w, w_scales, wt, wt_scales, n, out_features, in_features, static_cast<hipStream_t>(stream)));
}

ft_status_t ft_expert_weight_grad(const ft_sort_desc_t *desc, int32_t out_features, int32_t in_features,
                                  const ft_act_codes_t *dy_col, const ft_act_codes_t *x_col, const ft_sort_t *sort,
                                  int32_t T, void *dw, int32_t dw_dtype, int32_t accumulate, void *stream) {
    if (ft_status_t s = sort_status(desc); s != FT_OK) return s;
    if (!dim_ok(out_features) || !dim_ok(in_features) || !tokens_ok(T) || (accumulate != 0 && accumulate != 1) ||
        desc->align != 128)
        return FT_ERR_SHAPE;
    if (!float_dtype(dw_dtype) || (accumulate && dw_dtype != FT_DT_F32)) return FT_ERR_DTYPE;
    if (!dw) return FT_ERR_NULL;
    if (!aligned(dw)) return FT_ERR_SHAPE;
    if (T == 0 && accumulate) return FT_OK;
    ProductArgs p{};
    GroupArgs g{};
    g.n = desc->local;
    if (T > 0) {
        if (!sort || !sort->off || !sort->count) return FT_ERR_NULL;
        if (ft_status_t s = form_status(dy_col); s != FT_OK) return s;
        if (ft_status_t s = form_status(x_col); s != FT_OK) return s;
        if (!words(sort->off) || !words(sort->count)) return FT_ERR_SHAPE;
        g = group_args(desc, sort);
        p.a = x_col->codes;
        p.as = x_col->scales;
        p.b = dy_col->codes;
        p.bs = dy_col->scales;
    }
    p.out = dw;
    p.M = in_features;
    p.R = out_features;
    p.K = desc->rows;
    p.Kp = pad128(desc->rows);
    p.asr = pad128(in_features);
    p.bsr = pad128(out_features);
    const int out = dw_dtype == FT_DT_BF16 ? 0 : accumulate ? 2 : 1;
    const float mean = static_cast<float>(T) * desc->top_k / desc->n_experts;
    return done(launch_expert_weight_grad(p, g, mean, out, static_cast<hipStream_t>(stream)));
}

ft_status_t ft_block_norm(const ft_norm_desc_t *desc, const ft_norm_params_t *params, const void *x, const void *block,
                          int32_t T, void *r, void *n, const ft_act_codes_t *n_row, void *stream) {
    if (ft_status_t s = norm_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    if (T == 0) return FT_OK;
    if (!x || (!n && !n_row && (!r || !block))) return FT_ERR_NULL;
    if (ft_status_t s = params_status(params); s != FT_OK) return s;
    if (ft_status_t s = optional_status(n_row); s != FT_OK) return s;
    if (!aligned(x) || !aligned(block) || !aligned(r) || !aligned(n)) return FT_ERR_SHAPE;
    NormArgs a = norm_args(desc, params, T);
    a.x = x;
    a.b = block;
    a.r = r;
    a.nout = n;
    a.row = form(n_row, T, desc->channels);
    return done(launch_block_norm(a, desc->x_dtype == FT_DT_F32, desc->y_dtype == FT_DT_F32, desc->w_dtype == FT_DT_F32,
                                  static_cast<hipStream_t>(stream)));
}

size_t ft_block_norm_workspace_bytes(const ft_norm_desc_t *desc, int32_t max_tokens) {
    if (norm_status(desc) != FT_OK || !tokens_ok(max_tokens)) return 0;
    return round256(static_cast<size_t>(norm_parts(std::max(max_tokens, 1), desc->channels)) * 2 * desc->channels * 4);
}

ft_status_t ft_block_norm_backward(const ft_norm_desc_t *desc, const ft_norm_params_t *params, const void *r,
                                   const void *block, const void *dr, const void *dn, int32_t T, void *dx, void *d_block,
                                   const ft_norm_grads_t *grads, void *ws, size_t ws_bytes, void *stream) {
    if (ft_status_t s = norm_status(desc); s != FT_OK) return s;
    if (!tokens_ok(T)) return FT_ERR_SHAPE;
    const ft_norm_grads_t none{}, g = grads ? *grads : none;
    const bool sums = g.pre || g.post || g.gate;
    if (!dx && !d_block && !sums && !g.token_gate) return FT_ERR_NULL;
    if (T > 0 && (!r || (!dr && !dn) || (g.pre && !dn) || (!block && (d_block || g.post || g.gate || g.token_gate)))) return FT_ERR_NULL;
    if ((g.post && !desc->post_norm) || (sums && !ws)) return FT_ERR_NULL;
    if (ft_status_t s = params_status(params); s != FT_OK) return s;
    if (sums && ws_bytes < ft_block_norm_workspace_bytes(desc, T)) return FT_ERR_CAPACITY;
    if (!aligned(r) || !aligned(block) || !aligned(dr) || !aligned(dn) || !aligned(dx) || !aligned(d_block) || !aligned(ws) ||
        !words(g.pre) || !words(g.post) || !words(g.gate) || !words(g.token_gate))
        return FT_ERR_SHAPE;
    if (T == 0 && !sums) return FT_OK;
    NormArgs a = norm_args(desc, params, T);
    a.x = r;
    a.b = block;
    a.dr = dr;
    a.dn = dn;
    a.r = dx;
    a.nout = d_block;
    a.d_tgate = g.token_gate;
    a.parts = sums ? static_cast<float *>(ws) : nullptr;
    a.n_parts = T > 0 ? norm_parts(T, desc->channels) : 0;
    return done(launch_block_norm_backward(a, desc->x_dtype == FT_DT_F32, desc->y_dtype == FT_DT_F32, desc->w_dtype == FT_DT_F32,
                                           g.pre, g.post, g.gate, static_cast<hipStream_t>(stream)));
}

}  // extern "C"
