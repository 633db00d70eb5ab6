// C ABI of hh_train.h: argument validation, workspaces and the order in which the kernels are enqueued.
#include "../../include/hh_train.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ctx.h"
#include "kernels.h"

using namespace hh;

// ------------------------------------------------------------------ output projection and cross entropy
static int check_head(const hh_head_cfg* c) {
    if (!c) return fail(HH_ERR_INVALID_ARG, "cfg is NULL");
    if (c->dtype != HH_F32 && c->dtype != HH_BF16) return fail(HH_ERR_INVALID_ARG, "cfg.dtype %d is not HH_F32/HH_BF16", c->dtype);
    if (c->hidden <= 0 || c->vocab <= 0 || c->tokens <= 0) return fail(HH_ERR_INVALID_ARG, "cfg has a non-positive dimension");
    const int mult = c->dtype == HH_BF16 ? 64 : 8;
    if (c->hidden % mult) return fail(HH_ERR_UNSUPPORTED_SHAPE, "hidden (%d) must be a multiple of %d for this dtype", c->hidden, mult);
    if (c->hidden > 32768) return fail(HH_ERR_UNSUPPORTED_SHAPE, "hidden %d exceeds 32768", c->hidden);
    if (c->vocab > MAX_LD) return fail(HH_ERR_UNSUPPORTED_SHAPE, "vocab %d exceeds %d", c->vocab, MAX_LD);
    const long es = c->dtype == HH_BF16 ? 2 : 4;
    if ((long)c->tokens * c->hidden * es >= (1L << 31)) return fail(HH_ERR_UNSUPPORTED_SHAPE, "x of %d x %d elements reaches 2^31 bytes", c->tokens, c->hidden);
    if ((long)c->vocab * c->hidden * es >= (1L << 32) - (1L << 25))
        return fail(HH_ERR_UNSUPPORTED_SHAPE, "a weight of %d x %d elements reaches 2^32 bytes", c->vocab, c->hidden);
    return HH_OK;
}

// A pass over a block of tokens, and the block's pieces for which the scores are in the workspace.
struct HeadPlan {
    int dt, T, H, V, ld, slots;   // ld: a row of scores and of d
    int block, piece;             // tokens
    bool whole;                   // a row of scores fits the registers of a workgroup
    size_t stats, norm, z, d, xs, gemm_ws, total;
};
static int split_evenly(int n, int most) { const int parts = (n + most - 1) / most; return (n + parts - 1) / parts; }
// share: of a vocabulary that other devices have the rest of.
static HeadPlan head_plan(const hh_head_cfg* c, bool step, bool share) {
    HeadPlan p{};
    const bool bf = c->dtype == HH_BF16;
    p.dt = bf ? DT_BF16 : DT_F32;
    p.T = c->tokens; p.H = c->hidden; p.V = c->vocab;
    p.ld = (c->vocab + 63) & ~63;
    const int width = bf ? SCORE_SLOT : HEAD_F32_SLOT;
    p.slots = (c->vocab + width - 1) / width;
    // d is 4 bytes a score in both types, and below 2^31 bytes as an operand of 32-bit offsets; x's copy too, below 65536 rows of a grid
    const long most = std::min<long>(std::min<long>(((1L << 31) - 1) / (4L * p.ld), ((1L << 31) - 1) / (4L * p.H)), 32768);
    p.block = split_evenly(p.T, (int)std::max<long>(most, 1));
    p.piece = p.block;
    p.whole = p.ld <= head_row_most(p.dt) && (step || !bf) && !share;
    if (bf) {   // up to 512 MB of scores (a step of 4096 x 32000 in pieces of 256 MB: 10.77 -> 10.58 ms), 256 MB of statistics
        const long rows = step ? (1L << 29) / (4L * p.ld) : (1L << 28) / (8L * p.slots);
        p.piece = (int)std::min<long>(p.block, std::max<long>(256, rows / 256 * 256));
    }
    size_t off = 0;
    auto take = [&](size_t bytes) { size_t o = off; off += up256(bytes); return o; };
    if (!p.whole) p.stats = take((size_t)p.slots * p.piece * sizeof(float2) + (size_t)p.piece * sizeof(float));
    if (step && !p.whole && !share) p.norm = take((size_t)p.piece * sizeof(float2));
    if (step || !bf) p.z = take((size_t)p.piece * p.ld * 4);
    if (step) {
        p.d = bf ? take((size_t)p.block * p.ld * 4) : p.z;
        p.xs = take((size_t)p.block * p.H * 4);
    }
    p.gemm_ws = take(step ? GEMM_WS_BYTES : 0);
    p.total = off;
    return p;
}

extern "C" int hh_head_sizes(const hh_head_cfg* cfg, size_t* loss_workspace_bytes, size_t* step_workspace_bytes) {
    TRY(check_head(cfg));
    if (loss_workspace_bytes) *loss_workspace_bytes = std::max(head_plan(cfg, false, false).total, head_plan(cfg, false, true).total);
    if (step_workspace_bytes) *step_workspace_bytes = std::max(head_plan(cfg, true, false).total, head_plan(cfg, true, true).total);
    return HH_OK;
}

#define TRACED(kind, work, call)                          \
    do {                                                  \
        Traced t_(ctx, st, (kind), 1, (double)(work));    \
        HIP_TRY(call);                                    \
    } while (0)

// What a call is given and asked for, by token: of a step dx and dw; lse_in: the log-sum-exp over a vocabulary of which w is a share.
struct HeadCall {
    const void *x, *w;
    const int64_t* labels;
    int64_t first, limit;
    const float* dloss;
    float scale;
    float *loss, *lse, *picked;
    const float* lse_in;
    void* dx;
    float* dw;
    int accumulate;
};
static int head_run(hh_ctx* ctx, const HeadPlan& p, const HeadCall& c, void* ws, hipStream_t st) {
    const bool bf = p.dt == DT_BF16, step = c.dx != nullptr;
    const size_t es = dt_size(p.dt);
    const int H = p.H, V = p.V;
    ctx->gemm_ws = step ? at(ws, p.gemm_ws) : nullptr;
    ctx->gemm_room = 0;
    float2* const stats = p.whole || c.lse_in ? nullptr : (float2*)at(ws, p.stats);
    float* const z = step || !bf ? (float*)at(ws, p.z) : nullptr;
    for (int t0 = 0; t0 < p.T; t0 += p.block) {
        const int T = std::min(p.block, p.T - t0);
        for (int r0 = 0; r0 < T; r0 += p.piece) {
            const int M = std::min(p.piece, T - r0), at0 = t0 + r0;
            const void* const xr = at(c.x, (size_t)at0 * H * es);
            const HeadTokens t{c.labels + at0, c.first, c.limit, M, V, c.dloss ? c.dloss + at0 : nullptr, c.scale};
            auto from = [&](float* q) { return q ? q + at0 : nullptr; };
            GemmDesc g = desc(GEMM_NT, M, bf ? V : p.ld, H, xr, H, c.w, H, z, p.ld);
            const GemmScores scores{z, stats, t.labels, (int)c.first};
            if (bf) g.scores = &scores;
            else g.b_rows = V;
            HIP_TRY(tgemm(ctx, p.dt, g, st));
            void* const d = step ? at(ws, p.d + (size_t)r0 * p.ld * es) : nullptr;
            void* const xs = step ? at(ws, p.xs + (size_t)r0 * H * es) : nullptr;
            const double grad_bytes = 8.0 * M * V + (bf ? 6.0 : 8.0) * M * H;
            if (p.whole) {
                TRACED(HH_TRACE_ELEMENTWISE, step ? grad_bytes : 4.0 * M * V, head_row(p.dt, t, z, p.ld, from(c.loss), d, T, xr, xs, H, st));
                continue;
            }
            const float* const lse = c.lse_in ? c.lse_in + at0 : nullptr;
            float2* const norm = step && !lse ? (float2*)at(ws, p.norm) : nullptr;
            if (!lse) {
                if (!bf) TRACED(HH_TRACE_ELEMENTWISE, 4.0 * M * V, head_stats_f32(t, z, p.ld, stats, st));
                TRACED(HH_TRACE_ELEMENTWISE, 8.0 * M * p.slots, head_rows(t, stats, p.slots, from(c.loss), from(c.lse), norm, from(c.picked), st));
            }
            if (step) TRACED(HH_TRACE_ELEMENTWISE, grad_bytes, head_grad(p.dt, t, z, p.ld, norm, lse, d, T, xr, xs, H, st));
        }
        if (!step) continue;
        const void* const d = at(ws, p.d);
        const void* const xs = at(ws, p.xs);
        GemmDesc g[4];
        int n = 0;
        g[n] = desc(GEMM_NN, T, H, p.ld, d, p.ld, c.w, H, at(c.dx, (size_t)t0 * H * es), H);
        g[n++].b_rows = V;
        if (!bf && gemm_f32_long_k_better(T, H, p.ld)) {
            g[0].long_k = 1;
            HIP_TRY(tgemm(ctx, p.dt, g, n, st));
            n = 0;
        }
        // fp32 sums of 2^31 bytes and more in pieces of the vocabulary
        const int most = (int)std::min<long>(V, std::max<long>(256, ((1L << 31) - 1) / (4L * H) / 256 * 256));
        for (int v0 = 0; v0 < V; v0 += most) {
            if (n == 4) { HIP_TRY(tgemm(ctx, p.dt, g, n, st)); n = 0; }
            g[n++] = desc(GEMM_TN, std::min(most, V - v0), H, bf ? 2 * T : T, at(d, (size_t)v0 * es), p.ld, xs, H, c.dw + (size_t)v0 * H, H,
                          nullptr, 0, 1, c.accumulate || t0 > 0);
            g[n - 1].pair = bf;
        }
        HIP_TRY(tgemm(ctx, p.dt, g, n, st));
    }
    return HH_OK;
}

extern "C" int hh_head_loss(hh_ctx* ctx, const hh_head_cfg* cfg, const void* x, const void* w, const int64_t* labels, float* loss,
                            void* workspace, void* stream) {
    TRY(check_head(cfg));
    TRY(check_ptr(x, "x")); TRY(check_ptr(w, "w")); TRY(check_ptr(labels, "labels")); TRY(check_ptr(loss, "loss"));
    TRY(check_ptr(workspace, "workspace"));
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    HeadCall c{};
    c.x = x; c.w = w; c.labels = labels; c.limit = cfg->vocab; c.loss = loss;
    return head_run(ctx, head_plan(cfg, false, false), c, workspace, (hipStream_t)stream);
}

static int check_dloss(const float* dloss) {
    return (uintptr_t)dloss & 15 ? fail(HH_ERR_MISALIGNED, "dloss is not 16-byte aligned") : (int)HH_OK;
}

extern "C" int hh_head_step(hh_ctx* ctx, const hh_head_cfg* cfg, const void* x, const void* w, const int64_t* labels, const float* dloss,
                            float scale, float* loss, void* dx, float* dw, int accumulate, void* workspace, void* stream) {
    TRY(check_head(cfg));
    TRY(check_ptr(x, "x")); TRY(check_ptr(w, "w")); TRY(check_ptr(labels, "labels")); TRY(check_ptr(loss, "loss"));
    TRY(check_ptr(dx, "dx")); TRY(check_ptr(dw, "dw")); TRY(check_ptr(workspace, "workspace")); TRY(check_dloss(dloss));
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    HeadCall c{};
    c.x = x; c.w = w; c.labels = labels; c.limit = cfg->vocab; c.dloss = dloss; c.scale = scale;
    c.loss = loss; c.dx = dx; c.dw = dw; c.accumulate = accumulate;
    return head_run(ctx, head_plan(cfg, true, false), c, workspace, (hipStream_t)stream);
}

static int check_share(const hh_head_cfg* cfg, int32_t first) {
    TRY(check_head(cfg));
    if (first < 0 || first > INT32_MAX - cfg->vocab) return fail(HH_ERR_INVALID_ARG, "first (%d) is negative, or the share ends past 2^31 - 1", first);
    return HH_OK;
}

extern "C" int hh_head_share_fwd(hh_ctx* ctx, const hh_head_cfg* cfg, const void* x, const void* w, const int64_t* labels, int32_t first,
                                 float* lse, float* picked, void* workspace, void* stream) {
    TRY(check_share(cfg, first));
    TRY(check_ptr(x, "x")); TRY(check_ptr(w, "w")); TRY(check_ptr(labels, "labels")); TRY(check_ptr(lse, "lse"));
    TRY(check_ptr(picked, "picked")); TRY(check_ptr(workspace, "workspace"));
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    HeadCall c{};
    c.x = x; c.w = w; c.labels = labels; c.first = first; c.limit = INT64_MAX; c.lse = lse; c.picked = picked;
    return head_run(ctx, head_plan(cfg, false, true), c, workspace, (hipStream_t)stream);
}

extern "C" int hh_head_share_bwd(hh_ctx* ctx, const hh_head_cfg* cfg, const void* x, const void* w, const int64_t* labels, int32_t first,
                                 const float* lse, const float* dloss, float scale, void* dx, float* dw, int accumulate,
                                 void* workspace, void* stream) {
    TRY(check_share(cfg, first));
    TRY(check_ptr(x, "x")); TRY(check_ptr(w, "w")); TRY(check_ptr(labels, "labels")); TRY(check_ptr(lse, "lse"));
    TRY(check_ptr(dx, "dx")); TRY(check_ptr(dw, "dw")); TRY(check_ptr(workspace, "workspace")); TRY(check_dloss(dloss));
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    HeadCall c{};
    c.x = x; c.w = w; c.labels = labels; c.first = first; c.limit = INT64_MAX; c.dloss = dloss; c.scale = scale;
    c.lse_in = lse; c.dx = dx; c.dw = dw; c.accumulate = accumulate;
    return head_run(ctx, head_plan(cfg, true, true), c, workspace, (hipStream_t)stream);
}

// ------------------------------------------------------------------ lists of tensors
// Elements in front of the first one at which the pointers are all aligned for vectors of `vec` elements; -1: there is none.
struct Typed { const void* p; size_t es; };
static int lead(const Typed* p, int n, int vec) {
    for (int h = 0; h < vec; h++) {
        bool fits = true;
        for (int i = 0; i < n; i++) fits = fits && !(((uintptr_t)p[i].p + h * p[i].es) & (vec * p[i].es - 1));
        if (fits) return h;
    }
    return -1;
}
static long chunks_of(int64_t count, int head, int chunk) {
    const int64_t body = std::max<int64_t>(count - std::max(head, 0), 0);
    return std::max<long>(1, (long)((body + chunk - 1) / chunk));
}
static int check_item(int i, const char* name, const void* p, size_t es) {
    if (!p) return fail(HH_ERR_INVALID_ARG, "tensors[%d].%s is NULL", i, name);
    if ((uintptr_t)p & (es - 1)) return fail(HH_ERR_MISALIGNED, "tensors[%d].%s is not aligned to its type", i, name);
    return HH_OK;
}
static int check_list(int n, const void* tensors) {
    if (n < 0) return fail(HH_ERR_INVALID_ARG, "n is negative");
    if (n > 0 && !tensors) return fail(HH_ERR_INVALID_ARG, "tensors is NULL");
    return HH_OK;
}
static bool is_dtype(int d) { return d == HH_F32 || d == HH_BF16; }
static size_t size_of(int d) { return d == HH_BF16 ? 2 : 4; }
constexpr int64_t MAX_COUNT = (int64_t)1 << 34;
constexpr long MAX_CHUNKS = (1L << 24) - 8;        // 256 threads each, below 2^32 in a launch
static_assert(MAX_COUNT / ADAMW_CHUNK + 1 < MAX_CHUNKS && MAX_COUNT / CLIP_CHUNK + 1 < MAX_CHUNKS, "a tensor fits a launch");

// Fills lists of up to MAX tensors and hands each of them to `launch`.
template <typename List, int MAX, int CHUNK, typename Tensor, typename Fill, typename Launch>
static int for_lists(int n, const Tensor* tensors, Fill fill, Launch launch) {
    List l;
    l.n = l.chunks = 0;
    for (int i = 0; i < n; i++) {
        if (tensors[i].count == 0) continue;
        auto& t = l.t[l.n];
        fill(tensors[i], t);
        const long c = chunks_of(tensors[i].count, t.head, CHUNK);
        if (l.n && l.chunks + c > MAX_CHUNKS) {
            TRY(launch(l));
            l.t[0] = t;
            l.n = l.chunks = 0;
        }
        l.t[l.n].first = l.chunks;
        l.chunks += (int)c;
        if (++l.n == MAX) {
            TRY(launch(l));
            l.n = l.chunks = 0;
        }
    }
    return l.n ? launch(l) : HH_OK;
}

static void fill_clip(const hh_clip_tensor& q, ClipItem& t) {
    const size_t es = size_of(q.dtype);
    const Typed p[2] = {{q.g, es}, {q.out, es}};
    t = ClipItem{q.g, q.out, q.count, 0, (int16_t)lead(p, q.out ? 2 : 1, (int)(16 / es)), (int16_t)(q.dtype == HH_BF16)};
}

extern "C" int hh_grad_clip(hh_ctx* ctx, int n, const hh_clip_tensor* tensors, float max_norm, float* result, void* workspace, void* stream) {
    TRY(check_list(n, tensors));
    if (!(max_norm > 0.f)) return fail(HH_ERR_INVALID_ARG, "max_norm must be positive");
    TRY(check_ptr(result, "result")); TRY(check_ptr(workspace, "workspace"));
    bool copies = false;
    long most = 0;
    for (int i = 0; i < n; i++) {
        const hh_clip_tensor& t = tensors[i];
        if (!is_dtype(t.dtype)) return fail(HH_ERR_INVALID_ARG, "tensors[%d].dtype %d is not HH_F32/HH_BF16", i, t.dtype);
        if (t.count < 0 || t.count > MAX_COUNT) return fail(HH_ERR_INVALID_ARG, "tensors[%d].count is negative or exceeds 2^34", i);
        if (t.count == 0) continue;
        TRY(check_item(i, "g", t.g, size_of(t.dtype)));
        if (t.out) TRY(check_item(i, "out", t.out, size_of(t.dtype)));
        copies = copies || t.out;
    }
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    const hipStream_t st = (hipStream_t)stream;
    double* const slots = (double*)workspace;
    auto lists = [&](auto launch) { return for_lists<ClipList, CLIP_LIST, CLIP_CHUNK>(n, tensors, fill_clip, launch); };
    double bytes = 0.0;
    TRY(lists([&](const ClipList& l) -> int {
        most = std::max<long>(most, l.chunks);
        for (int i = 0; i < l.n; i++) bytes += (double)l.t[i].count * (l.t[i].bf16 ? 2 : 4);
        return HH_OK;
    }));
    // every launch has the same workgroups, so that each adds to a slot that the first one has written
    const int wgs = (int)std::max<long>(1, std::min<long>(most, CLIP_SLOTS));
    {
        Traced t_(ctx, st, HH_TRACE_ELEMENTWISE, 1, bytes);
        int add = 0;
        TRY(lists([&](const ClipList& l) -> int {
            HIP_TRY(clip_squares(l, slots, wgs, add, st));
            add = 1;
            return HH_OK;
        }));
        if (!add) {
            ClipList none{};
            HIP_TRY(clip_squares(none, slots, 1, 0, st));
        }
    }
    if (!copies) {
        HIP_TRY(clip_result(slots, wgs, max_norm, result, st));
        return HH_OK;
    }
    Traced t_(ctx, st, HH_TRACE_ELEMENTWISE, 1, 2.0 * bytes);
    float* told = result;
    return lists([&](const ClipList& l) -> int {
        HIP_TRY(clip_scale(l, slots, wgs, max_norm, told, st));
        told = nullptr;
        return HH_OK;
    });
}

static void fill_adamw(const hh_adamw_tensor& q, double lr, AdamwItem& t) {
    const bool pb = q.param_dtype == HH_BF16, gb = q.grad_dtype == HH_BF16;
    const Typed p[5] = {{q.m, 4}, {q.v, 4}, {q.g, size_of(q.grad_dtype)}, {q.param, size_of(q.param_dtype)}, {q.master, 4}};
    t = AdamwItem{q.param, q.master, q.m, q.v, q.g, q.count, (float)(1.0 - lr * q.decay), 0, (int16_t)lead(p, pb ? 5 : 4, 4), (int16_t)pb, (int16_t)gb, 0};
}

extern "C" int hh_adamw_step(hh_ctx* ctx, const hh_adamw_cfg* cfg, int n, const hh_adamw_tensor* tensors, const float* factor, void* stream) {
    if (!cfg) return fail(HH_ERR_INVALID_ARG, "cfg is NULL");
    auto below_one = [](double b) { return b >= 0.f && b < 1.f; };
    if (!below_one(cfg->beta1) || !below_one(cfg->beta2)) return fail(HH_ERR_INVALID_ARG, "beta1 and beta2 must be in [0, 1)");
    if (!(cfg->lr >= 0.f) || !(cfg->eps >= 0.f)) return fail(HH_ERR_INVALID_ARG, "lr and eps must be >= 0");
    if (cfg->step < 1) return fail(HH_ERR_INVALID_ARG, "step counts from 1");
    TRY(check_list(n, tensors));
    double bytes = 0.0;
    for (int i = 0; i < n; i++) {
        const hh_adamw_tensor& t = tensors[i];
        if (!is_dtype(t.param_dtype) || !is_dtype(t.grad_dtype)) return fail(HH_ERR_INVALID_ARG, "tensors[%d] has a dtype that is not HH_F32/HH_BF16", i);
        if (t.count < 0 || t.count > MAX_COUNT) return fail(HH_ERR_INVALID_ARG, "tensors[%d].count is negative or exceeds 2^34", i);
        if (!(t.decay >= 0.f)) return fail(HH_ERR_INVALID_ARG, "tensors[%d].decay must be >= 0", i);
        if (t.count == 0) continue;
        const bool pb = t.param_dtype == HH_BF16;
        TRY(check_item(i, "param", t.param, size_of(t.param_dtype)));
        TRY(check_item(i, "m", t.m, 4)); TRY(check_item(i, "v", t.v, 4)); TRY(check_item(i, "g", t.g, size_of(t.grad_dtype)));
        if (pb) TRY(check_item(i, "master", t.master, 4));
        else if (t.master) return fail(HH_ERR_INVALID_ARG, "tensors[%d]: an fp32 parameter is its own master copy (master must be NULL)", i);
        bytes += (double)t.count * (24.0 + size_of(t.grad_dtype) + (pb ? 2.0 : 0.0));
    }
    if ((uintptr_t)factor & 3) return fail(HH_ERR_MISALIGNED, "factor is not aligned to its type");
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    const hipStream_t st = (hipStream_t)stream;
    const double bc1 = 1.0 - std::pow(cfg->beta1, (double)cfg->step), bc2 = 1.0 - std::pow(cfg->beta2, (double)cfg->step);
    const AdamwHyper h{(float)cfg->beta1, (float)(1.0 - cfg->beta1), (float)cfg->beta2, (float)(1.0 - cfg->beta2), (float)cfg->eps,
                       (float)(cfg->lr / bc1), (float)(1.0 / std::sqrt(bc2))};
    auto fill = [&](const hh_adamw_tensor& q, AdamwItem& t) { fill_adamw(q, cfg->lr, t); };
    Traced t_(ctx, st, HH_TRACE_ELEMENTWISE, 1, bytes);
    return for_lists<AdamwList, ADAMW_LIST, ADAMW_CHUNK>(n, tensors, fill, [&](const AdamwList& l) -> int {
        HIP_TRY(adamw(l, h, factor, bytes > (double)LIST_CACHE, st));
        return HH_OK;
    });
}
