// C ABI of the EAT MoE-layer library: argument validation, workspace
// carve-up and the launch sequence.  Every check runs on the host before
// any HIP call; no exception leaves this file.
#include <math.h>
#include <string.h>

#include <algorithm>
#include <cstring>
#include <cmath>
#include <functional>
#include <initializer_list>
#include <new>

#include "eat_internal.h"

namespace {

constexpr int32_t kMaxTokens = 1 << 24;
constexpr int32_t kMaxCeTokens = 1 << 20, kMaxVocab = 1 << 24, kMaxCeWidth = 1 << 16;

bool finite(float v) { return isfinite(v) != 0; }
bool in01(float v) { return finite(v) && v >= 0.f && v <= 1.f; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) % a) == 0; }

eat_status_t check_params(const eat_params_t& p) {
    if (p.mode < EAT_MODE_EAT || p.mode > EAT_MODE_TOPP) return EAT_ERR_INVALID_ARG;
    if (p.E < 1 || p.d_model < 1 || p.d_ffn < 1 || p.d_shared < 0) return EAT_ERR_INVALID_ARG;
    if (p.top_k < 1 || p.top_k > p.E) return EAT_ERR_INVALID_ARG;
    if (p.mode == EAT_MODE_TOPP && !(finite(p.top_p) && p.top_p > 0.f && p.top_p <= 1.f))
        return EAT_ERR_INVALID_ARG;
    if (p.top_p_cap < 0 || p.top_p_cap > p.E) return EAT_ERR_INVALID_ARG;
    if (!in01(p.alpha) || !in01(p.beta)) return EAT_ERR_INVALID_ARG;
    const float fin[] = {p.w1, p.w2, p.w3, p.alpha1, p.alpha2, p.kappa1, p.kappa2,
                         p.ppl_up, p.ppl_down, p.eps, p.inv_temperature};
    for (float v : fin)
        if (!finite(v)) return EAT_ERR_INVALID_ARG;
    if (!in01(p.q_lo) || !in01(p.q_hi) || p.q_lo > p.q_hi) return EAT_ERR_INVALID_ARG;
    if (p.eps < 0.f || p.inv_temperature <= 0.f) return EAT_ERR_INVALID_ARG;
    if (p.cs_mode != 0 && p.cs_mode != 1) return EAT_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(p.expert_scale) % 4) return EAT_ERR_INVALID_ARG;
    if ((p.act_dtype != EAT_F32 && p.act_dtype != EAT_BF16) ||
        (p.expert_dtype != EAT_F32 && p.expert_dtype != EAT_BF16))
        return EAT_ERR_INVALID_ARG;
    // supported shapes and dtype pairs
    if (p.E > eat::kMaxExperts) return EAT_ERR_UNSUPPORTED;
    if (p.d_model % 64 || p.d_ffn % 64 || p.d_shared % 64) return EAT_ERR_UNSUPPORTED;
    // one expert matrix is addressed with 32-bit element offsets
    if (static_cast<int64_t>(p.d_model) * std::max(p.d_ffn, p.d_shared) >= (int64_t{1} << 31))
        return EAT_ERR_UNSUPPORTED;
    if (p.act_dtype != p.expert_dtype) return EAT_ERR_UNSUPPORTED;
    if (p.weight_layout != EAT_LAYOUT_ROWS && p.weight_layout != EAT_LAYOUT_PACKED) return EAT_ERR_INVALID_ARG;
    if (p.weight_layout == EAT_LAYOUT_PACKED && p.expert_dtype != EAT_BF16) return EAT_ERR_UNSUPPORTED;
    return EAT_OK;
}

// Whether two buffers (either may be null) share bytes.
struct Span {
    const void* p;
    size_t n;
};
bool overlap(Span u, Span v) {
    const uintptr_t a = reinterpret_cast<uintptr_t>(u.p), b = reinterpret_cast<uintptr_t>(v.p);
    return u.p && v.p && a < b + v.n && b < a + u.n;
}
// Whether a buffer that a call writes shares bytes with another of its buffers,
// the pairs apart for which `in_place` holds (same address, written read).
template <typename F>
bool clash(std::initializer_list<Span> out, std::initializer_list<Span> in, F in_place) {
    for (const Span* o = out.begin(); o != out.end(); ++o) {
        for (const Span* q = o + 1; q != out.end(); ++q)
            if (overlap(*o, *q)) return true;
        for (const Span& i : in)
            if (overlap(*o, i) && !(o->p == i.p && in_place(o->p, i.p))) return true;
    }
    return false;
}

size_t align256(size_t v) { return (v + 255) & ~size_t(255); }

}  // namespace

namespace eat {

Workspace plan_workspace(const eat_ctx& c, int32_t T) {
    const eat_params_t& p = c.p;
    Workspace w{};
    const size_t t = static_cast<size_t>(T), E = static_cast<size_t>(p.E);
    const size_t es = p.expert_dtype == EAT_BF16 ? 2 : 4;
    w.rows = static_cast<int64_t>(T) * c.kmax;
    w.splits = down_splits(p, T);
    w.up_splits = up_splits(p, T);
    const size_t rows = static_cast<size_t>(w.rows);
    size_t off = 0;
    auto take = [&](size_t bytes) { const size_t at = off; off += align256(bytes); return at; };
    w.lpart = take(static_cast<size_t>(T > 0 ? route_slices(p, T) : 1) * t * E * 4);
    w.route_total = off;
    w.prob = take(t * E * 4);
    w.gate = take(t * E * 4);
    w.mask = take(t * eat::mask_words(p.E) * 8);
    w.k = take(t * 4);
    w.offsets = take((E + 1) * 4);
    w.tok_idx = take(rows * 4);
    w.inv = take(t * E * 4);
    w.h = take(rows * p.d_ffn * es);
    // (the gate/up partials are added up before the down projection writes its slices)
    const size_t gu = w.up_splits > 1 ? 2 * static_cast<size_t>(w.up_splits) * rows * p.d_ffn * 4 : 0;
    w.gu = w.yp = take(std::max(gu, static_cast<size_t>(w.splits) * rows * p.d_model * 4));
    w.nrm = take(rows * static_cast<size_t>(norm_parts(p, T)) * 4);
    w.shared_splits = p.d_shared ? shared_splits(p, T) : 1;
    w.shared_up_splits = p.d_shared ? shared_up_splits(p, T) : 1;
    w.hs = take(p.d_shared ? t * p.d_shared * es : 0);
    w.ys = take(p.d_shared ? t * p.d_model * 4 : 0);
    w.gus = take(w.shared_up_splits > 1 ? 2 * static_cast<size_t>(w.shared_up_splits) * t * p.d_shared * 4 : 0);
    w.ysp = take(w.shared_splits > 1 ? static_cast<size_t>(w.shared_splits) * t * p.d_model * 4 : 0);
    w.sync = take(static_cast<size_t>(kSyncWords) * 4);
    w.total = off;
    return w;
}

}  // namespace eat

extern "C" {

eat_status_t eat_params_default(eat_params_t* out) {
    if (!out) return EAT_ERR_INVALID_ARG;
    memset(out, 0, sizeof(*out));
    out->mode = EAT_MODE_EAT;
    out->E = 8;
    out->d_model = 4096;
    out->d_ffn = 14336;
    out->top_k = 2;
    out->top_p = 0.6f;
    out->top_p_cap = 0;
    out->alpha = 0.95f;
    out->w1 = 0.3f; out->w2 = 0.3f; out->w3 = 0.4f;
    out->beta = 0.6f;
    out->alpha1 = 0.5f; out->alpha2 = 1.0f;
    out->kappa1 = 0.7f; out->kappa2 = 0.3f;
    out->ppl_up = 1.2f; out->ppl_down = 0.9f;
    out->q_lo = 0.1f; out->q_hi = 0.9f;
    out->eps = 1e-8f;
    out->inv_temperature = 1.0f;
    out->cs_mode = 0;
    out->act_dtype = EAT_BF16;
    out->expert_dtype = EAT_BF16;
    out->d_shared = 0;
    out->expert_scale = nullptr;
    out->weight_layout = EAT_LAYOUT_ROWS;
    return EAT_OK;
}

eat_status_t eat_create(const eat_params_t* params, int32_t max_tokens, eat_handle_t* out) {
    if (!params || !out) return EAT_ERR_INVALID_ARG;
    *out = nullptr;
    if (max_tokens < 1 || max_tokens > kMaxTokens) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_params(*params);
    if (st != EAT_OK) return st;
    // most (token, expert) rows a call can select: rows, segment offsets and
    // token indices are 32-bit
    int32_t kmax = params->E;
    if (params->mode == EAT_MODE_TOPK) kmax = params->top_k;
    else if (params->mode == EAT_MODE_TOPP && params->top_p_cap > 0) kmax = params->top_p_cap;
    if (static_cast<int64_t>(max_tokens) * kmax >= (int64_t{1} << 31)) return EAT_ERR_UNSUPPORTED;
    eat_ctx* c = new (std::nothrow) eat_ctx;
    if (!c) return EAT_ERR_INTERNAL;
    c->p = *params;
    c->max_tokens = max_tokens;
    c->kmax = kmax;
    *out = c;
    return EAT_OK;
}

eat_status_t eat_destroy(eat_handle_t h) {
    delete h;
    return EAT_OK;
}

eat_status_t eat_workspace_size(eat_handle_t h, int32_t T, size_t* bytes) {
    if (!h || !bytes || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    *bytes = eat::plan_workspace(*h, T).total;
    return EAT_OK;
}

eat_status_t eat_reset_accounts(eat_handle_t h, eat_accounts_t acc, hipStream_t stream) {
    if (!h || !acc.n || !acc.p_total || !acc.c_s) return EAT_ERR_INVALID_ARG;
    if (!aligned(acc.n, 8) || !aligned(acc.p_total, 4) || !aligned(acc.c_s, 4)) return EAT_ERR_INVALID_ARG;
    (void)hipGetLastError();
    return eat::launch_reset_accounts(h->p, acc, stream) == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

static eat_status_t check_accounts(const eat_ctx& c, const eat_accounts_t& acc) {
    if (c.p.mode != EAT_MODE_EAT) return EAT_OK;
    if (!acc.n || !acc.p_total || !acc.c_s) return EAT_ERR_INVALID_ARG;
    if (!aligned(acc.n, 8) || !aligned(acc.p_total, 4) || !aligned(acc.c_s, 4)) return EAT_ERR_INVALID_ARG;
    return EAT_OK;
}

eat_status_t eat_route_workspace_size(eat_handle_t h, int32_t T, size_t* bytes) {
    if (!h || !bytes || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    *bytes = eat::plan_workspace(*h, T).route_total;
    return EAT_OK;
}

eat_status_t eat_route(eat_handle_t h, const void* x, int32_t T, const float* w_router,
                       eat_accounts_t acc, const int8_t* ppl_trend, uint64_t* mask_out,
                       int32_t* k_out, float* gate_out, float* prob_out, void* ws, size_t ws_bytes,
                       hipStream_t stream) {
    if (!h || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    if (!x || !w_router || !mask_out || !k_out || !gate_out) return EAT_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(w_router, 16) || !aligned(mask_out, 8) || !aligned(k_out, 4) ||
        !aligned(gate_out, 4) || (prob_out && !aligned(prob_out, 4)))
        return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_accounts(*h, acc);
    if (st != EAT_OK) return st;
    const eat::Workspace w = eat::plan_workspace(*h, T);
    if (T > 0 && (!ws || ws_bytes < w.route_total)) return EAT_ERR_WORKSPACE;
    if (ws && !aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    if (T == 0) return EAT_OK;
    (void)hipGetLastError();
    const hipError_t e = eat::launch_route(h->p, x, T, w_router, acc, ppl_trend,
                                           reinterpret_cast<float*>(static_cast<char*>(ws) + w.lpart), mask_out,
                                           k_out, gate_out, prob_out, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

}  // extern "C"

namespace eat {

// Argument checks shared by the forward entry points (host only).
eat_status_t check_forward(const eat_ctx* h, const void* x, int32_t T, const float* w_router, const void* w1,
                           const void* w3, const void* w2, const void* ws1, const void* ws3, const void* ws2,
                           const eat_accounts_t& acc, const void* y, const uint64_t* mask_out,
                           const int32_t* expert_load_out) {
    if (!h || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    const eat_params_t& p = h->p;
    if (!x || !w_router || !w1 || !w3 || !w2 || !y) return EAT_ERR_INVALID_ARG;
    const void* a16[] = {x, w_router, w1, w3, w2, y};
    for (const void* q : a16)
        if (!aligned(q, 16)) return EAT_ERR_INVALID_ARG;
    if (p.d_shared > 0) {
        if (!ws1 || !ws3 || !ws2) return EAT_ERR_INVALID_ARG;
        if (!aligned(ws1, 16) || !aligned(ws3, 16) || !aligned(ws2, 16)) return EAT_ERR_INVALID_ARG;
    } else if (ws1 || ws3 || ws2) {
        return EAT_ERR_INVALID_ARG;
    }
    if ((mask_out && !aligned(mask_out, 8)) || (expert_load_out && !aligned(expert_load_out, 4)))
        return EAT_ERR_INVALID_ARG;
    return check_accounts(*h, acc);
}

// Enqueue one layer forward (arguments already checked, T > 0, workspace
// large enough).  `residual` (bf16 [T][d] or null) is added to y.
hipError_t forward_impl(const eat_ctx& h, const void* x, int32_t T, const float* w_router, const void* w1,
                        const void* w3, const void* w2, const void* ws1, const void* ws3, const void* ws2,
                        eat_accounts_t acc, const int8_t* ppl_trend, const uint16_t* residual, void* y,
                        uint64_t* mask_out, int32_t* expert_load_out, float* prob_out, void* ws,
                        hipStream_t stream, const hipEvent_t* events, int32_t n_events, AccountJob* defer) {
    const eat_params_t& p = h.p;
    const eat::Workspace w = eat::plan_workspace(h, T);
    char* base = static_cast<char*>(ws);
    eat::Buffers b;
    b.lpart = reinterpret_cast<float*>(base + w.lpart);
    b.prob = prob_out ? prob_out : reinterpret_cast<float*>(base + w.prob);
    b.gate = reinterpret_cast<float*>(base + w.gate);
    b.mask = mask_out ? mask_out : reinterpret_cast<uint64_t*>(base + w.mask);
    b.k = reinterpret_cast<int32_t*>(base + w.k);
    b.offsets = reinterpret_cast<int32_t*>(base + w.offsets);
    b.tok_idx = reinterpret_cast<int32_t*>(base + w.tok_idx);
    b.inv = reinterpret_cast<int32_t*>(base + w.inv);
    b.h = base + w.h;
    b.gu = reinterpret_cast<float*>(base + w.gu);
    b.yp = reinterpret_cast<float*>(base + w.yp);
    b.nrm2 = reinterpret_cast<float*>(base + w.nrm);
    b.hs = base + w.hs;
    b.ys = reinterpret_cast<float*>(base + w.ys);
    b.gus = reinterpret_cast<float*>(base + w.gus);
    b.ysp = reinterpret_cast<float*>(base + w.ysp);
    b.sync = reinterpret_cast<unsigned*>(base + w.sync);
    int32_t* const up_splits_dev = reinterpret_cast<int32_t*>(b.sync);
    int32_t* const down_splits_dev = reinterpret_cast<int32_t*>(b.sync + 1);

    hipError_t e = hipSuccess;
    auto mark = [&](int stage) {
        if (e == hipSuccess && stage < n_events && events[stage]) e = hipEventRecord(events[stage], stream);
    };
    mark(EAT_STAGE_BEGIN);
    if (e == hipSuccess)
        e = eat::launch_route(p, x, T, w_router, acc, ppl_trend, b.lpart, b.mask, b.k, b.gate, b.prob, stream);
    mark(EAT_STAGE_ROUTED);
    Segments seg{};
    if (eat::fuses_permutation(p, T))
        seg = Segments{b.mask, T, eat::mask_words(p.E), b.offsets, b.tok_idx, b.inv, expert_load_out};
    else if (e == hipSuccess)
        e = eat::launch_permute(p, T, b.mask, b.offsets, b.tok_idx, b.inv, expert_load_out, stream);
    mark(EAT_STAGE_PERMUTED);
    const bool bf16 = p.expert_dtype == EAT_BF16;
    if (e == hipSuccess) {
        if (bf16)
            e = eat::launch_experts_bf16(p, T, w.rows, static_cast<const uint16_t*>(x),
                                         static_cast<const uint16_t*>(w1), static_cast<const uint16_t*>(w3),
                                         static_cast<const uint16_t*>(w2), b.offsets, b.tok_idx, seg,
                                         static_cast<uint16_t*>(b.h), b.gu, b.yp, b.nrm2, up_splits_dev,
                                         down_splits_dev, stream, [&]() { mark(EAT_STAGE_UP); });
        else
            e = eat::launch_experts_f32(p, T, w.rows, static_cast<const float*>(x),
                                        static_cast<const float*>(w1), static_cast<const float*>(w3),
                                        static_cast<const float*>(w2), b.offsets, b.tok_idx, seg,
                                        static_cast<float*>(b.h), b.yp, stream, [&]() { mark(EAT_STAGE_UP); });
    }
    mark(EAT_STAGE_DOWN);
    const bool shared = p.d_shared > 0;
    if (e == hipSuccess && shared) {
        if (bf16)
            e = eat::launch_shared_bf16(p, T, static_cast<const uint16_t*>(x), static_cast<const uint16_t*>(ws1),
                                        static_cast<const uint16_t*>(ws3), static_cast<const uint16_t*>(ws2),
                                        static_cast<uint16_t*>(b.hs), b.ys, b.gus, b.ysp, stream);
        else
            e = eat::launch_shared_f32(p, T, static_cast<const float*>(x), static_cast<const float*>(ws1),
                                       static_cast<const float*>(ws3), static_cast<const float*>(ws2),
                                       static_cast<float*>(b.hs), b.ys, stream);
    }
    mark(EAT_STAGE_SHARED);
    // the down projection's slices: chosen on the device when it could take several
    const int32_t* splits_dev = bf16 && w.splits > 1 ? down_splits_dev : nullptr;
    const bool rows16 = bf16 && eat::rows_bf16(p, T);
    // (the hidden rows, at least 128 bytes each, are free once the down projection has read them)
    float2* const stats = rows16 ? static_cast<float2*>(b.h) : nullptr;
    if (e == hipSuccess)
        e = eat::launch_combine(p, T, b.mask, b.gate, b.inv, b.yp, shared ? b.ys : nullptr, residual, y, b.nrm2,
                                w.splits, w.rows * p.d_model, splits_dev, rows16, b.prob, stats, stream);
    mark(EAT_STAGE_COMBINED);
    if (defer) *defer = AccountJob{};
    if (e == hipSuccess && p.mode == EAT_MODE_EAT) {
        const AccountJob job{b.offsets, b.tok_idx, b.prob, b.nrm2, stats, eat::norm_parts(p, T), p.E, p.alpha, acc};
        if (defer) *defer = job;
        else e = eat::launch_update_accounts(job, T, stream);
    }
    mark(EAT_STAGE_END);
    return e;
}

}  // namespace eat

namespace {

using eat::check_forward;
using eat::forward_impl;

// Stacked-layer workspace: the largest layer workspace, then u, r and two
// h rows (bf16 [T][d] each), then the mixing GEMM's fp32 slices.
struct StackPlan {
    size_t layer, u, r, h0, h1, mix, total;
    int splits;
};

StackPlan plan_stack(const eat_stack_layer_t* layers, int32_t n, int32_t T) {
    StackPlan s{};
    auto up = [](size_t v) { return (v + 255) & ~static_cast<size_t>(255); };
    size_t lw = 0;
    for (int32_t l = 0; l < n; ++l) lw = std::max(lw, eat::plan_workspace(*layers[l].layer, T).total);
    const int d = layers[0].layer->p.d_model;
    const size_t row = up(static_cast<size_t>(T) * d * 2);
    s.splits = eat::dense_splits(d, d, T);
    s.layer = 0;
    s.u = up(lw);
    s.r = s.u + row;
    s.h0 = s.r + row;
    s.h1 = s.h0 + row;
    s.mix = s.h1 + row;
    s.total = s.mix + up(static_cast<size_t>(s.splits) * T * d * 4);
    return s;
}

eat_status_t check_stack(const eat_stack_layer_t* layers, int32_t n, int32_t T) {
    if (!layers || n < 1 || n > 1024 || T < 0) return EAT_ERR_INVALID_ARG;
    for (int32_t l = 0; l < n; ++l) {
        const eat_ctx* c = layers[l].layer;
        if (!c || T > c->max_tokens) return EAT_ERR_INVALID_ARG;
        if (c->p.act_dtype != EAT_BF16 || c->p.expert_dtype != EAT_BF16) return EAT_ERR_UNSUPPORTED;
        if (c->p.d_model != layers[0].layer->p.d_model) return EAT_ERR_INVALID_ARG;
        if (!layers[l].mix || !aligned(layers[l].mix, 16)) return EAT_ERR_INVALID_ARG;
    }
    if (!eat::mix_norm_fits(layers[0].layer->p.d_model)) return EAT_ERR_UNSUPPORTED;
    return EAT_OK;
}

}  // namespace

extern "C" {

eat_status_t eat_moe_forward_profiled(eat_handle_t h, const void* x, int32_t T, const float* w_router,
                                      const void* w1, const void* w3, const void* w2, const void* ws1,
                                      const void* ws3, const void* ws2, eat_accounts_t acc,
                                      const int8_t* ppl_trend, void* y, uint64_t* mask_out,
                                      int32_t* expert_load_out, void* ws, size_t ws_bytes, hipStream_t stream,
                                      const hipEvent_t* events, int32_t n_events) {
    if (n_events < 0 || n_events > EAT_NUM_STAGE_EVENTS || (n_events > 0 && !events)) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_forward(h, x, T, w_router, w1, w3, w2, ws1, ws3, ws2, acc, y, mask_out,
                                          expert_load_out);
    if (st != EAT_OK) return st;
    const eat::Workspace w = eat::plan_workspace(*h, T);
    if (T > 0 && (!ws || ws_bytes < w.total)) return EAT_ERR_WORKSPACE;
    if (ws && !aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    if (T == 0) return EAT_OK;
    (void)hipGetLastError();
    const hipError_t e = forward_impl(*h, x, T, w_router, w1, w3, w2, ws1, ws3, ws2, acc, ppl_trend, nullptr, y,
                                      mask_out, expert_load_out, nullptr, ws, stream, events, n_events);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_stack_workspace_size(const eat_stack_layer_t* layers, int32_t n_layers, int32_t T,
                                      size_t* bytes) {
    if (!bytes) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_stack(layers, n_layers, T);
    if (st != EAT_OK) return st;
    *bytes = plan_stack(layers, n_layers, T).total;
    return EAT_OK;
}

eat_status_t eat_stack_forward(const eat_stack_layer_t* layers, int32_t n_layers, const void* x, int32_t T,
                               const int8_t* ppl_trend, float rms_eps, void* h_out, uint64_t* masks_out,
                               float* probs_out, void* ws, size_t ws_bytes, hipStream_t stream) {
    eat_status_t st = check_stack(layers, n_layers, T);
    if (st != EAT_OK) return st;
    if (!x || !h_out || !aligned(x, 16) || !aligned(h_out, 16)) return EAT_ERR_INVALID_ARG;
    if ((masks_out && !aligned(masks_out, 8)) || (probs_out && !aligned(probs_out, 4))) return EAT_ERR_INVALID_ARG;
    if (!(rms_eps >= 0.0f) || !std::isfinite(rms_eps)) return EAT_ERR_INVALID_ARG;
    for (int32_t l = 0; l < n_layers; ++l) {
        const eat_stack_layer_t& L = layers[l];
        st = check_forward(L.layer, x, T, L.w_router, L.w1, L.w3, L.w2, L.ws1, L.ws3, L.ws2, L.acc, h_out,
                           masks_out, nullptr);
        if (st != EAT_OK) return st;
    }
    const StackPlan sp = plan_stack(layers, n_layers, T);
    if (T > 0 && (!ws || ws_bytes < sp.total)) return EAT_ERR_WORKSPACE;
    if (ws && !aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    if (T == 0) return EAT_OK;

    char* base = static_cast<char*>(ws);
    uint16_t* u = reinterpret_cast<uint16_t*>(base + sp.u);
    uint16_t* r = reinterpret_cast<uint16_t*>(base + sp.r);
    uint16_t* hb[2] = {reinterpret_cast<uint16_t*>(base + sp.h0), reinterpret_cast<uint16_t*>(base + sp.h1)};
    float* mix = reinterpret_cast<float*>(base + sp.mix);
    const int d = layers[0].layer->p.d_model;
    const int64_t stride = static_cast<int64_t>(T) * d;

    (void)hipGetLastError();
    size_t prob_off = 0;                      // layer l's probabilities start after T * E_j of the layers before
    size_t mask_off = 0;                      // and its masks after T * mask_words(E_j)
    // u_0 = bf16(RMSNorm(x))
    hipError_t e = eat::launch_mix_norm(nullptr, 0, 0, static_cast<const uint16_t*>(x), T, d, rms_eps, nullptr, u,
                                        nullptr, stream);
    const uint16_t* h = static_cast<const uint16_t*>(x);
    for (int32_t l = 0; l < n_layers && e == hipSuccess; ++l) {
        const eat_stack_layer_t& L = layers[l];
        // r = bf16(h + MoE_l(u)); the layer's account update rides on the
        // RMSNorm launch below (it reads the layer workspace, which the next
        // layer reuses only after that launch)
        eat::AccountJob job{};
        e = forward_impl(*L.layer, u, T, L.w_router, L.w1, L.w3, L.w2, L.ws1, L.ws3, L.ws2, L.acc, ppl_trend, h, r,
                         masks_out ? masks_out + mask_off : nullptr, nullptr,
                         probs_out ? probs_out + prob_off : nullptr, base + sp.layer, stream, nullptr, 0, &job);
        prob_off += static_cast<size_t>(T) * L.layer->p.E;
        mask_off += static_cast<size_t>(T) * eat::mask_words(L.layer->p.E);
        // h' = bf16(r M_l^T); u = bf16(RMSNorm(h')) for the next layer
        if (e == hipSuccess)
            e = eat::launch_dense_bf16(r, T, static_cast<const uint16_t*>(L.mix), d, d, mix, sp.splits, stride,
                                       stream);
        const bool last = l + 1 == n_layers;
        uint16_t* hn = last ? static_cast<uint16_t*>(h_out) : hb[l & 1];
        if (e == hipSuccess)
            e = eat::launch_mix_norm(mix, sp.splits, stride, nullptr, T, d, rms_eps, hn, last ? nullptr : u,
                                     job.experts > 0 ? &job : nullptr, stream);
        h = hn;
    }
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_moe_forward(eat_handle_t h, const void* x, int32_t T, const float* w_router,
                             const void* w1, const void* w3, const void* w2, const void* ws1,
                             const void* ws3, const void* ws2, eat_accounts_t acc,
                             const int8_t* ppl_trend, void* y, uint64_t* mask_out,
                             int32_t* expert_load_out, void* ws, size_t ws_bytes, hipStream_t stream) {
    return eat_moe_forward_profiled(h, x, T, w_router, w1, w3, w2, ws1, ws3, ws2, acc, ppl_trend, y, mask_out,
                                    expert_load_out, ws, ws_bytes, stream, nullptr, 0);
}

eat_status_t eat_pack_weights(const void* src, int32_t groups, int32_t M, int32_t K, void* dst,
                              hipStream_t stream) {
    if (!src || !dst || groups < 1 || M < 16 || K < 32 || M % 16 || K % 32) return EAT_ERR_INVALID_ARG;
    if (!aligned(src, 16) || !aligned(dst, 16)) return EAT_ERR_INVALID_ARG;
    const uintptr_t bytes = static_cast<uintptr_t>(groups) * M * K * 2;
    const uintptr_t s0 = reinterpret_cast<uintptr_t>(src), d0 = reinterpret_cast<uintptr_t>(dst);
    if (s0 < d0 + bytes && d0 < s0 + bytes) return EAT_ERR_INVALID_ARG;     // overlapping buffers
    (void)hipGetLastError();
    return eat::launch_pack(static_cast<const uint16_t*>(src), groups, M, K, static_cast<uint16_t*>(dst), stream) ==
                   hipSuccess
               ? EAT_OK
               : EAT_ERR_HIP;
}

eat_status_t eat_ppl_workspace_size(int32_t S, int32_t d, int32_t V, size_t* bytes) {
    if (!bytes || S < 0 || S > kMaxTokens || d < 64 || d % 64 || V < 64 || V % 64) return EAT_ERR_INVALID_ARG;
    if (static_cast<int64_t>(d) * V >= (int64_t{1} << 31)) return EAT_ERR_INVALID_ARG;
    *bytes = align256(static_cast<size_t>(eat::head_splits(V, d, S)) * S * V * 4);
    return EAT_OK;
}

eat_status_t eat_ppl_reset(int32_t S, double* nll_sum, int32_t* count, double* ppl_prev, hipStream_t stream) {
    if (S < 0 || (S > 0 && (!nll_sum || !count || !ppl_prev))) return EAT_ERR_INVALID_ARG;
    if (!aligned(nll_sum, 8) || !aligned(count, 4) || !aligned(ppl_prev, 8)) return EAT_ERR_INVALID_ARG;
    if (S == 0) return EAT_OK;
    (void)hipGetLastError();
    return eat::launch_ppl_reset(S, nll_sum, count, ppl_prev, stream) == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_ppl_trend(const void* h, int32_t S, int32_t d, const void* w_vocab, int32_t V,
                           const int32_t* target, double* nll_sum, int32_t* count, double* ppl_prev,
                           int8_t* trend_out, float* nll_out, void* ws, size_t ws_bytes, hipStream_t stream) {
    size_t need = 0;
    const eat_status_t st = eat_ppl_workspace_size(S, d, V, &need);
    if (st != EAT_OK) return st;
    if (S == 0) return EAT_OK;
    if (!h || !w_vocab || !target || !nll_sum || !count || !ppl_prev || !trend_out) return EAT_ERR_INVALID_ARG;
    if (!aligned(h, 16) || !aligned(w_vocab, 16) || !aligned(target, 4) || !aligned(nll_sum, 8) ||
        !aligned(count, 4) || !aligned(ppl_prev, 8) || (nll_out && !aligned(nll_out, 4)))
        return EAT_ERR_INVALID_ARG;
    if (!ws || ws_bytes < need) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    float* z = static_cast<float*>(ws);
    const int splits = eat::head_splits(V, d, S);
    const int64_t stride = static_cast<int64_t>(S) * V;
    (void)hipGetLastError();
    hipError_t e = eat::launch_head_bf16(static_cast<const uint16_t*>(h), S, static_cast<const uint16_t*>(w_vocab),
                                         V, d, z, splits, stride, stream);
    if (e == hipSuccess)
        e = eat::launch_ppl(z, splits, stride, S, V, static_cast<const uint16_t*>(h),
                            static_cast<const uint16_t*>(w_vocab), d, target, nll_sum, count, ppl_prev, trend_out, nll_out, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_ce_workspace_size(int32_t T, int32_t d, int32_t V, int32_t grads, size_t* bytes, size_t* min_bytes) {
    if (!bytes || T < 0 || T > kMaxCeTokens || d < 64 || d % 64 || V < 1 || V > kMaxVocab) return EAT_ERR_INVALID_ARG;
    if (grads < 0 || grads > (EAT_CE_DH | EAT_CE_DW)) return EAT_ERR_INVALID_ARG;
    if (d > kMaxCeWidth) return EAT_ERR_UNSUPPORTED;
    const bool dh = (grads & EAT_CE_DH) != 0, dw = (grads & EAT_CE_DW) != 0;
    *bytes = eat::plan_ce(T, d, V, dh, dw, SIZE_MAX).total;
    if (min_bytes) *min_bytes = eat::plan_ce(T, d, V, dh, dw, 0).total;
    return EAT_OK;
}

eat_status_t eat_ce_loss(const void* h, int32_t T, int32_t d, const void* w_vocab, int32_t V, const int32_t* target,
                         int32_t ignore, int32_t mean, float scale, float* loss_out, float* nll_out,
                         int32_t* count_out, void* dh, void* dw, void* ws, size_t ws_bytes, hipStream_t stream) {
    size_t most = 0;
    const eat_status_t st = eat_ce_workspace_size(T, d, V, (dh ? EAT_CE_DH : 0) | (dw ? EAT_CE_DW : 0), &most, nullptr);
    if (st != EAT_OK) return st;
    if ((mean != 0 && mean != 1) || !finite(scale)) return EAT_ERR_INVALID_ARG;
    if (!w_vocab || !loss_out || (T > 0 && (!h || !target))) return EAT_ERR_INVALID_ARG;
    if (!aligned(h, 16) || !aligned(w_vocab, 16) || !aligned(target, 4) || !aligned(loss_out, 4) ||
        !aligned(nll_out, 4) || !aligned(count_out, 4) || !aligned(dh, 16) || !aligned(dw, 16))
        return EAT_ERR_INVALID_ARG;
    const eat::CePlan p = eat::plan_ce(T, d, V, dh != nullptr, dw != nullptr, ws_bytes);
    if (!ws || ws_bytes < p.total) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const size_t hb = static_cast<size_t>(T) * d * 2, wb = static_cast<size_t>(V) * d * 2, tb = static_cast<size_t>(T) * 4;
    if (clash({{loss_out, 4}, {nll_out, tb}, {count_out, 4}, {dh, hb}, {dw, wb}, {ws, p.total}},
              {{h, hb}, {w_vocab, wb}, {target, tb}}, [&](const void* o, const void* i) { return o == dh && i == h; }))
        return EAT_ERR_INVALID_ARG;
    const eat::CeCall c{static_cast<const uint16_t*>(h), static_cast<const uint16_t*>(w_vocab), target, T, d, V, ignore,
                        mean, scale, loss_out, nll_out, count_out, static_cast<uint16_t*>(dh),
                        static_cast<uint16_t*>(dw)};
    (void)hipGetLastError();
    const hipError_t e = eat::launch_ce(p, c, static_cast<char*>(ws), stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_balance_workspace_size(eat_handle_t h, int32_t T, size_t* bytes) {
    if (!h || !bytes || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    *bytes = eat::plan_balance(h->p, T).total;
    return EAT_OK;
}

eat_status_t eat_balance_loss(eat_handle_t h, const void* x, int32_t T, const float* w_router, const float* prob,
                              const uint64_t* mask, const uint8_t* valid, float coef, float entropy_coef,
                              float* loss_out, int64_t* count_out, float* mean_prob_out, float* dlogits, void* dx,
                              float* dw_router, void* ws, size_t ws_bytes, hipStream_t stream) {
    if (!h || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    if (!finite(coef) || !finite(entropy_coef)) return EAT_ERR_INVALID_ARG;
    if (!loss_out || (T > 0 && (!prob || !mask))) return EAT_ERR_INVALID_ARG;
    if ((dx && !w_router) || (dw_router && T > 0 && !x)) return EAT_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(w_router, 16) || !aligned(prob, 4) || !aligned(mask, 8) || !aligned(loss_out, 4) ||
        !aligned(count_out, 8) || !aligned(mean_prob_out, 4) || !aligned(dlogits, 4) || !aligned(dx, 16) ||
        !aligned(dw_router, 16))
        return EAT_ERR_INVALID_ARG;
    const eat::BalancePlan b = eat::plan_balance(h->p, T);
    if (!ws || ws_bytes < b.total) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const size_t n = static_cast<size_t>(T), E = static_cast<size_t>(h->p.E), d = static_cast<size_t>(h->p.d_model);
    const size_t xb = n * d * (h->p.act_dtype == EAT_BF16 ? 2 : 4), rb = E * d * 4, pb = n * E * 4;
    if (clash({{loss_out, 4}, {count_out, E * 8}, {mean_prob_out, E * 4}, {dlogits, pb}, {dx, xb}, {dw_router, rb}, {ws, b.total}},
              {{x, xb}, {w_router, rb}, {prob, pb}, {mask, n * ((E + 63) / 64) * 8}, {valid, n}},
              [&](const void* o, const void* i) { return (o == dlogits && i == prob) || (o == dx && i == x && !dw_router); }))
        return EAT_ERR_INVALID_ARG;
    const eat::BalanceCall c{x, w_router, prob, mask, valid, T, coef, entropy_coef, loss_out, count_out, mean_prob_out,
                             dlogits, dx, dw_router};
    (void)hipGetLastError();
    const hipError_t e = eat::launch_balance(h->p, b, c, static_cast<char*>(ws), stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_sort_workspace_size(eat_handle_t h, int32_t T, size_t* bytes) {
    if (!h || !bytes || T < 0 || T > h->max_tokens) return EAT_ERR_INVALID_ARG;
    *bytes = align256(eat::sort_workspace(T, h->p.E));
    return EAT_OK;
}

// What the calls between tokens and sorted rows have in common: their sizes.
static eat_status_t check_sorted(const eat_ctx* h, int32_t T, int32_t cap, const uint64_t* mask, const int32_t* place) {
    if (!h || T < 0 || T > h->max_tokens || cap < 0) return EAT_ERR_INVALID_ARG;
    if (T > 0 && (!mask || !place)) return EAT_ERR_INVALID_ARG;
    return aligned(mask, 8) && aligned(place, 4) ? EAT_OK : EAT_ERR_INVALID_ARG;
}

namespace {

struct SortBytes {
    size_t x, rows, mask, pairs;
    SortBytes(const eat_ctx& h, int32_t T, int32_t cap) {
        const size_t n = static_cast<size_t>(T), row = static_cast<size_t>(h.p.d_model) * (h.p.act_dtype == EAT_BF16 ? 2 : 4);
        x = n * row;
        rows = static_cast<size_t>(cap) * row;
        mask = n * eat::mask_words(h.p.E) * 8;
        pairs = n * h.p.E * 4;
    }
};
eat::SortCall sort_call(const eat_ctx& h, const uint64_t* mask, const int32_t* place, const float* gate, int32_t T, int32_t cap) {
    return eat::SortCall{mask, place, gate, T, h.p.E, h.p.d_model, cap, h.p.act_dtype == EAT_BF16};
}
bool in_place_none(const void*, const void*) { return false; }

}  // namespace

eat_status_t eat_sort_tokens(eat_handle_t h, const void* x, int32_t T, const uint64_t* mask, int32_t cap, void* rows_out,
                             int32_t* offsets_out, int32_t* token_out, int32_t* place_out, void* ws, size_t ws_bytes,
                             hipStream_t stream) {
    const eat_status_t st = check_sorted(h, T, cap, mask, place_out);
    if (st != EAT_OK) return st;
    if (!offsets_out || (cap > 0 && !token_out) || (rows_out && T > 0 && !x) || (x && cap > 0 && !rows_out)) return EAT_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(rows_out, 16) || !aligned(offsets_out, 4) || !aligned(token_out, 4)) return EAT_ERR_INVALID_ARG;
    const size_t need = align256(eat::sort_workspace(T, h->p.E));
    if (need > 0 && (!ws || ws_bytes < need)) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const SortBytes b(*h, T, cap);
    if (clash({{rows_out, b.rows}, {offsets_out, (static_cast<size_t>(h->p.E) + 1) * 4}, {token_out, static_cast<size_t>(cap) * 4},
               {place_out, b.pairs}, {ws, need}}, {{x, b.x}, {mask, b.mask}}, in_place_none))
        return EAT_ERR_INVALID_ARG;
    (void)hipGetLastError();
    const hipError_t e = eat::launch_sort(sort_call(*h, mask, nullptr, nullptr, T, cap), x, cap > 0 ? rows_out : nullptr,
                                          offsets_out, token_out, place_out, ws, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_sort_backward(eat_handle_t h, const void* drows, int32_t cap, int32_t T, const uint64_t* mask,
                               const int32_t* place, void* dx, hipStream_t stream) {
    const eat_status_t st = check_sorted(h, T, cap, mask, place);
    if (st != EAT_OK) return st;
    if (T > 0 && (!dx || (cap > 0 && !drows))) return EAT_ERR_INVALID_ARG;
    if (!aligned(drows, 16) || !aligned(dx, 16)) return EAT_ERR_INVALID_ARG;
    const SortBytes b(*h, T, cap);
    if (clash({{dx, b.x}}, {{drows, b.rows}, {mask, b.mask}, {place, b.pairs}}, in_place_none)) return EAT_ERR_INVALID_ARG;
    if (T == 0) return EAT_OK;
    (void)hipGetLastError();
    return eat::launch_gather(sort_call(*h, mask, place, nullptr, T, cap), drows, dx, stream) == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_combine(eat_handle_t h, const void* rows, int32_t cap, int32_t T, const uint64_t* mask, const float* gate,
                         const int32_t* place, void* y, hipStream_t stream) {
    const eat_status_t st = check_sorted(h, T, cap, mask, place);
    if (st != EAT_OK) return st;
    if (T > 0 && (!y || !gate || (cap > 0 && !rows))) return EAT_ERR_INVALID_ARG;
    if (!aligned(rows, 16) || !aligned(y, 16) || !aligned(gate, 4)) return EAT_ERR_INVALID_ARG;
    const SortBytes b(*h, T, cap);
    if (clash({{y, b.x}}, {{rows, b.rows}, {mask, b.mask}, {place, b.pairs}, {gate, b.pairs}}, in_place_none))
        return EAT_ERR_INVALID_ARG;
    if (T == 0) return EAT_OK;
    (void)hipGetLastError();
    return eat::launch_gather(sort_call(*h, mask, place, gate, T, cap), rows, y, stream) == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_combine_backward(eat_handle_t h, const void* dy, const void* rows, int32_t cap, int32_t T,
                                  const uint64_t* mask, const float* gate, const int32_t* place, const float* prob,
                                  void* drows, float* dgate, float* dlogits, hipStream_t stream) {
    const eat_status_t st = check_sorted(h, T, cap, mask, place);
    if (st != EAT_OK) return st;
    if (T > 0 && (!dy || !gate || (dlogits && !prob) || ((dgate || dlogits) && cap > 0 && !rows))) return EAT_ERR_INVALID_ARG;
    if (!aligned(dy, 16) || !aligned(rows, 16) || !aligned(drows, 16) || !aligned(gate, 4) || !aligned(prob, 4) ||
        !aligned(dgate, 4) || !aligned(dlogits, 4))
        return EAT_ERR_INVALID_ARG;
    const SortBytes b(*h, T, cap);
    if (clash({{drows, b.rows}, {dgate, b.pairs}, {dlogits, b.pairs}},
              {{dy, b.x}, {rows, b.rows}, {mask, b.mask}, {place, b.pairs}, {gate, b.pairs}, {prob, b.pairs}},
              [&](const void* o, const void* i) {
                  return (o == drows && i == rows) || (o == dlogits && i == prob) || (o == dgate && i == gate);
              }))
        return EAT_ERR_INVALID_ARG;
    if (T == 0 || (!drows && !dgate && !dlogits)) return EAT_OK;
    (void)hipGetLastError();
    const hipError_t e = eat::launch_combine_grad(sort_call(*h, mask, place, gate, T, cap), dy, rows, prob, h->p.eps, drows,
                                                  dgate, dlogits, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

// ---- matrices in 8 bits

namespace {

constexpr int32_t kMaxFp8Width = 1 << 20, kMaxFp8Rows = 1 << 24;

eat_status_t check_fp8(int32_t groups, int32_t M, int32_t K) {
    if (groups < 1 || M < 1 || K < 1) return EAT_ERR_INVALID_ARG;
    if (groups > eat::kMaxExperts || M % 8 || K % 8 || M > kMaxFp8Width || K > kMaxFp8Width) return EAT_ERR_UNSUPPORTED;
    return static_cast<int64_t>(M) * eat::fp8::pad(K) < (int64_t{1} << 31) ? EAT_OK : EAT_ERR_UNSUPPORTED;
}

struct Carver {
    size_t off = 0;
    size_t take(size_t bytes) {
        const size_t at = off;
        off += align256(bytes);
        return at;
    }
};
size_t q_bytes(int32_t groups, int32_t M, int32_t Kp) { return static_cast<size_t>(groups) * M * Kp; }
size_t s_bytes(int32_t groups, int32_t M, int32_t lds) { return static_cast<size_t>(groups) * ((M + 127) / 128) * lds; }
eat::fp8::Matrix matrix_at(const void* q, const void* s, int32_t M, int32_t K) {
    return eat::fp8::Matrix{static_cast<uint8_t*>(const_cast<void*>(q)), static_cast<uint8_t*>(const_cast<void*>(s)), M,
                            eat::fp8::pad(K), eat::fp8::scale_bytes(K)};
}

// A product's workspace: the rows in 8 bits and, where the reduction is split, its slices.
struct ProductPlan {
    size_t q, s, part, total;
    int splits;
    ProductPlan(const eat::fp8::Rows& r, int32_t M, int32_t K) {
        Carver c;
        splits = eat::fp8::product_slices(r, M, eat::fp8::pad(K));
        q = c.take(static_cast<size_t>(r.src_rows) * eat::fp8::pad(K));
        s = c.take(static_cast<size_t>(r.src_rows) * eat::fp8::scale_bytes(K));
        part = c.take(splits > 1 ? static_cast<size_t>(splits) * r.cap * M * 4 : 0);
        total = c.off;
    }
};

// The experts' weights in their buffer.
struct ExpertsPlan {
    size_t w1, s1, w3, s3, w2, s2, w2t, s2t, w13t, s13t, total;
    ExpertsPlan(const eat_params_t& p, bool grads) {
        Carver c;
        const int E = p.E, d = p.d_model, F = p.d_ffn, dp = eat::fp8::pad(d), Fp = eat::fp8::pad(F);
        const int ld = eat::fp8::scale_bytes(d), lf = eat::fp8::scale_bytes(F), l2 = eat::fp8::scale_bytes(2 * Fp);
        w1 = c.take(q_bytes(E, F, dp));
        s1 = c.take(s_bytes(E, F, ld));
        w3 = c.take(q_bytes(E, F, dp));
        s3 = c.take(s_bytes(E, F, ld));
        w2 = c.take(q_bytes(E, d, Fp));
        s2 = c.take(s_bytes(E, d, lf));
        w2t = c.take(grads ? q_bytes(E, F, dp) : 0);
        s2t = c.take(grads ? s_bytes(E, F, ld) : 0);
        w13t = c.take(grads ? q_bytes(E, d, 2 * Fp) : 0);
        s13t = c.take(grads ? s_bytes(E, d, l2) : 0);
        total = c.off;
    }
};

// The workspace of one call over the experts.
struct ExpertsCall {
    size_t q, s, h, hs, part, total;
    int up, down;                // slices of the first and of the second product
    ExpertsCall(const eat_params_t& p, const eat::fp8::Rows& r, bool back) {
        Carver c;
        const int d = p.d_model, F = p.d_ffn, dp = eat::fp8::pad(d), Fp = eat::fp8::pad(F);
        const int K2 = back ? 2 * Fp : Fp;
        const size_t src = static_cast<size_t>(r.src_rows), n = static_cast<size_t>(r.cap);
        up = back ? eat::fp8::product_slices(r, F, dp) : eat::fp8::gated_slices(r, F, dp);
        down = eat::fp8::product_slices(r, d, K2);
        q = c.take(src * dp);
        s = c.take(src * eat::fp8::scale_bytes(d));
        h = c.take(n * K2);
        hs = c.take(n * eat::fp8::scale_bytes(K2));
        // (the first product's slices are used up before the second's are written)
        const size_t first = back ? (eat::fp8::back_in_one(r, F, up) ? 0 : up * n * F * 4) : up > 1 ? 2 * up * n * F * 4 : 0;
        part = c.take(std::max<size_t>(first, down > 1 ? down * n * d * 4 : 0));
        total = c.off;
    }
};

// `grads`: of the backward too, whose matrix [dg | du] -> dx has rows of both.
eat_status_t check_experts(const eat_ctx* h, int32_t T, int32_t rows, bool grads) {
    if (!h || T < 0 || T > h->max_tokens || rows < 0 || (rows > 0 && T == 0)) return EAT_ERR_INVALID_ARG;
    if (h->p.act_dtype != EAT_BF16 || rows > kMaxFp8Rows || T > kMaxFp8Rows) return EAT_ERR_UNSUPPORTED;
    const eat_status_t st = check_fp8(h->p.E, h->p.d_model, grads ? 2 * eat::fp8::pad(h->p.d_ffn) : h->p.d_ffn);
    return st != EAT_OK ? st : check_fp8(h->p.E, h->p.d_ffn, h->p.d_model);
}

}  // namespace

eat_status_t eat_fp8_size(int32_t groups, int32_t M, int32_t K, size_t* q_out, size_t* scale_out) {
    if (!q_out || !scale_out) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_fp8(groups, M, K);
    if (st != EAT_OK) return st;
    *q_out = q_bytes(groups, M, eat::fp8::pad(K));
    *scale_out = s_bytes(groups, M, eat::fp8::scale_bytes(K));
    return EAT_OK;
}

eat_status_t eat_fp8_quantize(const void* w, int32_t dtype, int32_t groups, int32_t M, int32_t K, int32_t transposed, void* q,
                              void* scale, hipStream_t stream) {
    if ((dtype != EAT_F32 && dtype != EAT_BF16) || (transposed != 0 && transposed != 1)) return EAT_ERR_INVALID_ARG;
    // (the matrix that is written; the limits of the one that is read follow but for its own padding)
    const eat_status_t st = transposed ? check_fp8(groups, K, M) : check_fp8(groups, M, K);
    if (st != EAT_OK) return st;
    if (!w || !q || !scale || !aligned(w, 16) || !aligned(q, 256) || !aligned(scale, 256)) return EAT_ERR_INVALID_ARG;
    const int32_t rows = transposed ? K : M, cols = transposed ? M : K;
    const eat::fp8::Matrix m = matrix_at(q, scale, rows, cols);
    if (clash({{q, q_bytes(groups, rows, m.Kp)}, {scale, s_bytes(groups, rows, m.lds)}},
              {{w, static_cast<size_t>(groups) * M * K * (dtype == EAT_BF16 ? 2 : 4)}}, in_place_none))
        return EAT_ERR_INVALID_ARG;
    (void)hipGetLastError();
    const hipError_t e = eat::fp8::launch_quantize_weights(w, dtype == EAT_BF16, groups, M, K, transposed ? nullptr : &m,
                                                           transposed ? &m : nullptr, 0, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

static eat_status_t check_product(int32_t src_rows, int32_t rows, int32_t groups, int32_t M, int32_t K) {
    if (src_rows < 0 || rows < 0 || (rows > 0 && src_rows == 0)) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_fp8(groups, M, K);
    if (st != EAT_OK) return st;
    return src_rows > kMaxFp8Rows || rows > kMaxFp8Rows ? EAT_ERR_UNSUPPORTED : EAT_OK;
}

eat_status_t eat_fp8_product_workspace_size(int32_t src_rows, int32_t rows, int32_t groups, int32_t M, int32_t K, size_t* bytes) {
    if (!bytes) return EAT_ERR_INVALID_ARG;
    const eat_status_t st = check_product(src_rows, rows, groups, M, K);
    if (st != EAT_OK) return st;
    // (with offsets there are more tiles, so fewer slices: the larger of the two)
    const int32_t dummy = 0;
    const ProductPlan all(eat::fp8::Rows{nullptr, nullptr, src_rows, rows, groups}, M, K);
    const ProductPlan cut(eat::fp8::Rows{nullptr, &dummy, src_rows, rows, groups}, M, K);
    *bytes = std::max(all.total, cut.total);
    return EAT_OK;
}

eat_status_t eat_fp8_product(const void* x, int32_t src_rows, const int32_t* token, const int32_t* offsets, int32_t rows,
                             const void* q, const void* scale, int32_t groups, int32_t M, int32_t K, void* out,
                             int32_t out_dtype, void* ws, size_t ws_bytes, hipStream_t stream) {
    const eat_status_t st = check_product(src_rows, rows, groups, M, K);
    if (st != EAT_OK) return st;
    if ((out_dtype != EAT_F32 && out_dtype != EAT_BF16) || (!offsets && groups != 1) || (!token && src_rows != rows)) return EAT_ERR_INVALID_ARG;
    if (!q || !scale || (rows > 0 && (!x || !out))) return EAT_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(token, 4) || !aligned(offsets, 4) || !aligned(q, 256) || !aligned(scale, 256) || !aligned(out, 16))
        return EAT_ERR_INVALID_ARG;
    const eat::fp8::Rows r{token, offsets, src_rows, rows, groups};
    const ProductPlan p(r, M, K);
    if (p.total > 0 && (!ws || ws_bytes < p.total)) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const eat::fp8::Matrix w = matrix_at(q, scale, M, K);
    const size_t n = static_cast<size_t>(rows), xb = static_cast<size_t>(src_rows) * K * 2;
    if (clash({{out, n * M * (out_dtype == EAT_BF16 ? 2 : 4)}, {ws, p.total}},
              {{x, xb}, {token, n * 4}, {offsets, (static_cast<size_t>(groups) + 1) * 4}, {q, q_bytes(groups, M, w.Kp)},
               {scale, s_bytes(groups, M, w.lds)}}, in_place_none))
        return EAT_ERR_INVALID_ARG;
    if (rows == 0) return EAT_OK;
    uint8_t* const base = static_cast<uint8_t*>(ws);
    (void)hipGetLastError();
    hipError_t e = eat::fp8::launch_quantize_rows(static_cast<const uint16_t*>(x), r, K, base + p.q, base + p.s, stream);
    if (e == hipSuccess)
        e = eat::fp8::launch_product(r, base + p.q, base + p.s, w.lds, w, out_dtype == EAT_BF16, out, p.splits,
                                     reinterpret_cast<float*>(base + p.part), stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_fp8_experts_size(eat_handle_t h, int32_t grads, size_t* bytes) {
    const eat_status_t st = check_experts(h, 0, 0, grads == 1);
    if (st != EAT_OK) return st;
    if (!bytes || (grads != 0 && grads != 1)) return EAT_ERR_INVALID_ARG;
    *bytes = ExpertsPlan(h->p, grads == 1).total;
    return EAT_OK;
}

eat_status_t eat_fp8_experts_quantize(eat_handle_t h, const void* w1, const void* w3, const void* w2, int32_t grads, void* buf,
                                      hipStream_t stream) {
    const eat_status_t st = check_experts(h, 0, 0, grads == 1);
    if (st != EAT_OK) return st;
    if (!w1 || !w3 || !w2 || !buf || (grads != 0 && grads != 1)) return EAT_ERR_INVALID_ARG;
    if (!aligned(w1, 16) || !aligned(w3, 16) || !aligned(w2, 16) || !aligned(buf, 256)) return EAT_ERR_INVALID_ARG;
    const eat_params_t& p = h->p;
    const ExpertsPlan x(p, grads == 1);
    const size_t wb = static_cast<size_t>(p.E) * p.d_model * p.d_ffn * 2;
    if (clash({{buf, x.total}}, {{w1, wb}, {w3, wb}, {w2, wb}}, in_place_none)) return EAT_ERR_INVALID_ARG;
    uint8_t* const b = static_cast<uint8_t*>(buf);
    const int E = p.E, d = p.d_model, F = p.d_ffn, Fp = eat::fp8::pad(F);
    const eat::fp8::Matrix m1 = matrix_at(b + x.w1, b + x.s1, F, d), m3 = matrix_at(b + x.w3, b + x.s3, F, d),
                           m2 = matrix_at(b + x.w2, b + x.s2, d, F), t2 = matrix_at(b + x.w2t, b + x.s2t, F, d),
                           t13 = matrix_at(b + x.w13t, b + x.s13t, d, 2 * Fp);
    (void)hipGetLastError();
    hipError_t e = eat::fp8::launch_quantize_weights(w1, true, E, F, d, &m1, grads ? &t13 : nullptr, 0, stream);
    if (e == hipSuccess) e = eat::fp8::launch_quantize_weights(w3, true, E, F, d, &m3, grads ? &t13 : nullptr, Fp, stream);
    if (e == hipSuccess) e = eat::fp8::launch_quantize_weights(w2, true, E, d, F, &m2, grads ? &t2 : nullptr, 0, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_fp8_experts_workspace_size(eat_handle_t h, int32_t T, int32_t rows, int32_t grads, size_t* bytes) {
    const eat_status_t st = check_experts(h, grads == 1 && rows > 0 ? 1 : T, rows, grads == 1);
    if (st != EAT_OK) return st;
    if (!bytes || (grads != 0 && grads != 1)) return EAT_ERR_INVALID_ARG;
    const int32_t dummy = 0;
    *bytes = ExpertsCall(h->p, eat::fp8::Rows{nullptr, &dummy, grads ? rows : T, rows, h->p.E}, grads == 1).total;
    return EAT_OK;
}

eat_status_t eat_fp8_experts_forward(eat_handle_t h, const void* x, int32_t T, const int32_t* token, const int32_t* offsets,
                                     int32_t rows, const void* buf, void* y, void* saved, void* ws, size_t ws_bytes,
                                     hipStream_t stream) {
    const eat_status_t st = check_experts(h, T, rows, false);
    if (st != EAT_OK) return st;
    if (!buf || !offsets || (rows > 0 && (!x || !token || !y))) return EAT_ERR_INVALID_ARG;
    if (!aligned(x, 16) || !aligned(token, 4) || !aligned(offsets, 4) || !aligned(buf, 256) || !aligned(y, 16) || !aligned(saved, 16))
        return EAT_ERR_INVALID_ARG;
    const eat_params_t& p = h->p;
    const eat::fp8::Rows r{token, offsets, T, rows, p.E};
    const ExpertsCall c(p, r, false);
    if (c.total > 0 && (!ws || ws_bytes < c.total)) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const ExpertsPlan w(p, false);            // (the transposes lie behind)
    const size_t n = static_cast<size_t>(rows), d = static_cast<size_t>(p.d_model);
    if (clash({{y, n * d * 2}, {saved, n * p.d_ffn * 4}, {ws, c.total}},
              {{x, T * d * 2}, {token, n * 4}, {offsets, (static_cast<size_t>(p.E) + 1) * 4}, {buf, w.total}}, in_place_none))
        return EAT_ERR_INVALID_ARG;
    if (rows == 0) return EAT_OK;
    const uint8_t* const b = static_cast<const uint8_t*>(buf);
    uint8_t* const base = static_cast<uint8_t*>(ws);
    const int F = p.d_ffn, ld = eat::fp8::scale_bytes(p.d_model);
    float* const part = reinterpret_cast<float*>(base + c.part);
    (void)hipGetLastError();
    hipError_t e = eat::fp8::launch_quantize_rows(static_cast<const uint16_t*>(x), r, p.d_model, base + c.q, base + c.s, stream);
    if (e == hipSuccess)
        e = eat::fp8::launch_gated(r, base + c.q, base + c.s, ld, matrix_at(b + w.w1, b + w.s1, F, p.d_model),
                                   matrix_at(b + w.w3, b + w.s3, F, p.d_model), base + c.h, base + c.hs,
                                   static_cast<uint16_t*>(saved), c.up, part, stream);
    if (e == hipSuccess)
        e = eat::fp8::launch_product(eat::fp8::Rows{nullptr, offsets, rows, rows, p.E}, base + c.h, base + c.hs, eat::fp8::scale_bytes(F),
                                     matrix_at(b + w.w2, b + w.s2, p.d_model, F), true, y, c.down, part, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

eat_status_t eat_fp8_experts_backward(eat_handle_t h, const void* dy, const int32_t* offsets, int32_t rows, const void* buf,
                                      const void* saved, void* dx, void* ws, size_t ws_bytes, hipStream_t stream) {
    const eat_status_t st = check_experts(h, rows > 0 ? 1 : 0, rows, true);
    if (st != EAT_OK) return st;
    if (!buf || !offsets || (rows > 0 && (!dy || !saved || !dx))) return EAT_ERR_INVALID_ARG;
    if (!aligned(dy, 16) || !aligned(offsets, 4) || !aligned(buf, 256) || !aligned(saved, 16) || !aligned(dx, 16)) return EAT_ERR_INVALID_ARG;
    const eat_params_t& p = h->p;
    const eat::fp8::Rows r{nullptr, offsets, rows, rows, p.E};
    const ExpertsCall c(p, r, true);
    if (c.total > 0 && (!ws || ws_bytes < c.total)) return EAT_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return EAT_ERR_INVALID_ARG;
    const ExpertsPlan w(p, true);
    const size_t n = static_cast<size_t>(rows), db = n * p.d_model * 2;
    if (clash({{dx, db}, {ws, c.total}},
              {{dy, db}, {offsets, (static_cast<size_t>(p.E) + 1) * 4}, {buf, w.total}, {saved, n * p.d_ffn * 4}},
              [&](const void* o, const void* i) { return o == dx && i == dy; }))
        return EAT_ERR_INVALID_ARG;
    if (rows == 0) return EAT_OK;
    const uint8_t* const b = static_cast<const uint8_t*>(buf);
    uint8_t* const base = static_cast<uint8_t*>(ws);
    const int F = p.d_ffn, Fp = eat::fp8::pad(F), ld = eat::fp8::scale_bytes(p.d_model), l2 = eat::fp8::scale_bytes(2 * Fp);
    float* const part = reinterpret_cast<float*>(base + c.part);
    (void)hipGetLastError();
    hipError_t e = eat::fp8::launch_quantize_rows(static_cast<const uint16_t*>(dy), r, p.d_model, base + c.q, base + c.s, stream);
    if (e == hipSuccess)
        e = eat::fp8::launch_gate_backward(r, base + c.q, base + c.s, ld, matrix_at(b + w.w2t, b + w.s2t, F, p.d_model), c.up, part,
                                           static_cast<const uint16_t*>(saved), base + c.h, base + c.hs, l2, stream);
    if (e == hipSuccess)
        e = eat::fp8::launch_product(r, base + c.h, base + c.hs, l2, matrix_at(b + w.w13t, b + w.s13t, p.d_model, 2 * Fp), true, dx,
                                     c.down, part, stream);
    return e == hipSuccess ? EAT_OK : EAT_ERR_HIP;
}

const char* eat_status_string(eat_status_t s) {
    // a C caller may pass any int: read the argument's bits, not the enum
    // (a C++ enum value outside its enumerators' range is undefined)
    int v;
    std::memcpy(&v, &s, sizeof v);
    switch (v) {
        case EAT_OK: return "ok";
        case EAT_ERR_INVALID_ARG: return "invalid argument";
        case EAT_ERR_UNSUPPORTED: return "unsupported shape or dtype";
        case EAT_ERR_WORKSPACE: return "workspace missing or too small";
        case EAT_ERR_HIP: return "HIP runtime error";
        case EAT_ERR_INTERNAL: return "internal error";
        case EAT_ERR_SCRATCH_LIMIT: return "call needs more than the allocation-free entry point's fixed scratch";
    }
    return "unknown status";
}

}  // extern "C"
