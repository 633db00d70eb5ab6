// C ABI of hh_mx.h: argument validation and the order in which the kernels are enqueued.
#include "../../include/hh_mx.h"

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "ctx.h"
#include "kernels.h"

using namespace hh;

static_assert(HH_MX_NONE == MX_NONE && HH_MX_E4M3 == MX_E4M3 && HH_MX_E2M1 == MX_E2M1 && HH_MX_PAD == MX_PAD, "the kernels' names for them");

static int check_dtype(int dtype) {
    return dtype == HH_F32 || dtype == HH_BF16 ? (int)HH_OK : fail(HH_ERR_INVALID_ARG, "dtype %d is not HH_F32/HH_BF16", dtype);
}
static int check_format(int format, const char* name, bool none = false) {
    if (format == HH_MX_E4M3 || format == HH_MX_E2M1 || (none && format == HH_MX_NONE)) return HH_OK;
    return fail(HH_ERR_INVALID_ARG, "%s %d is not HH_MX_E4M3/HH_MX_E2M1", name, format);
}
static int check_packed(const hh_mx_tensor* q, const char* name) {
    if (!q) return fail(HH_ERR_INVALID_ARG, "%s is NULL", name);
    if (!q->codes || !q->scales) return fail(HH_ERR_INVALID_ARG, "%s has a NULL pointer", name);
    if (((uintptr_t)q->codes | (uintptr_t)q->scales) & 15) return fail(HH_ERR_MISALIGNED, "%s is not 16-byte aligned", name);
    return HH_OK;
}
// Counts fit 32 bits, and groups of eight values in a row of `cols` do over all rows.
constexpr int64_t MOST_ROWS = INT32_MAX - MX_PAD, MOST_GROUPS = INT32_MAX;
static int check_matrix(int64_t rows, int64_t cols, int64_t padded) {
    if (rows <= 0 || cols <= 0) return fail(HH_ERR_INVALID_ARG, "rows and columns must be positive");
    if (rows > MOST_ROWS || cols > MOST_ROWS || rows * ((padded + 7) / 8) > MOST_GROUPS)
        return fail(HH_ERR_UNSUPPORTED_SHAPE, "%lld rows of %lld values reach 2^31 groups of eight", (long long)rows, (long long)cols);
    return HH_OK;
}
static int check_ld(int64_t ld, int64_t cols, const char* name) {
    if (ld < cols) return fail(HH_ERR_INVALID_ARG, "%s (%lld) is less than a row", name, (long long)ld);
    if (ld > (int64_t)1 << 40) return fail(HH_ERR_UNSUPPORTED_SHAPE, "%s exceeds 2^40", name);
    return HH_OK;
}
static int check_ctx(const hh_ctx* ctx) {
    if (!ctx) return fail(HH_ERR_INVALID_ARG, "ctx is NULL");
    int dev = 0;
    HIP_TRY(hipGetDevice(&dev));
    if (dev != ctx->device) return fail(HH_ERR_INVALID_ARG, "the context is of device %d, the current one is %d", ctx->device, dev);
    return HH_OK;
}
static int drop_of(const hh_dropout_cfg* c, Drop& d) {
    if (!(c->p >= 0.0 && c->p <= 1.0)) return fail(HH_ERR_INVALID_ARG, "drop.p must be from 0 to 1");
    if ((uintptr_t)c->step & 7) return fail(HH_ERR_MISALIGNED, "drop.step is not aligned to its type");
    const uint32_t t = (uint32_t)std::nearbyint(c->p * 65536.0);
    d = Drop{c->seed, c->offset, c->step, t, t == 65536 ? 0.f : (float)(65536.0 / (65536 - t))};
    return HH_OK;
}
static int dt_of(int dtype) { return dtype == HH_BF16 ? DT_BF16 : DT_F32; }
static MxRows rows_of(const hh_mx_tensor* q) { return q ? MxRows{(uint8_t*)q->codes, q->scales} : MxRows{nullptr, nullptr}; }
static double packed_bytes(int format, double rows, double k) { return rows * k * (format == HH_MX_E4M3 ? 1.0 : 0.5) * (1.0 + (format == HH_MX_E4M3 ? 1.0 : 2.0) / 32); }

#define TRACED(kind, work, call)                       \
    do {                                               \
        Traced t_(ctx, st, (kind), 1, (double)(work)); \
        HIP_TRY(call);                                 \
    } while (0)

// ------------------------------------------------------------------ dropout
extern "C" int hh_dropout(hh_ctx* ctx, const hh_dropout_cfg* drop, int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ldx, void* y,
                          int64_t ldy, void* stream) {
    if (!drop) return fail(HH_ERR_INVALID_ARG, "drop is NULL");
    Drop d;
    TRY(drop_of(drop, d));
    TRY(check_dtype(dtype)); TRY(check_matrix(rows, cols, cols));
    TRY(check_ld(ldx, cols, "ldx")); TRY(check_ld(ldy, cols, "ldy"));
    TRY(check_ptr(x, "x")); TRY(check_ptr(y, "y"));
    if (x == y && ldx != ldy) return fail(HH_ERR_INVALID_ARG, "y is x with another ld");
    TRY(check_ctx(ctx));
    const hipStream_t st = (hipStream_t)stream;
    TRACED(HH_TRACE_ELEMENTWISE, 2.0 * rows * cols * dt_size(dt_of(dtype)), dropout(dt_of(dtype), d, rows, cols, x, ldx, y, ldy, st));
    return HH_OK;
}

// ------------------------------------------------------------------ packing
extern "C" int hh_mx_sizes(int32_t format, int64_t rows, int64_t k, size_t* codes_bytes, size_t* scales_bytes) {
    TRY(check_format(format, "format"));
    if (rows <= 0 || k <= 0) return fail(HH_ERR_INVALID_ARG, "rows and k must be positive");
    TRY(check_matrix(rows, k, mx_width(std::min<int64_t>(k, MOST_ROWS))));
    const size_t n = (size_t)rows * mx_width(k);
    if (codes_bytes) *codes_bytes = format == HH_MX_E4M3 ? n : n / 2;
    if (scales_bytes) *scales_bytes = n / 32;
    return HH_OK;
}

extern "C" int hh_mx_quantise(hh_ctx* ctx, int64_t rows, int64_t cols, int32_t dtype, const void* x, int64_t ldx, int32_t format,
                              const hh_mx_tensor* by_row, const hh_mx_tensor* by_column, void* stream) {
    TRY(check_dtype(dtype)); TRY(check_format(format, "format"));
    TRY(check_matrix(rows, cols, mx_width(std::min<int64_t>(cols, MOST_ROWS))));
    if (by_column) TRY(check_matrix(cols, rows, mx_width(rows)));
    TRY(check_ld(ldx, cols, "ldx")); TRY(check_ptr(x, "x"));
    if (!by_row && !by_column) return fail(HH_ERR_INVALID_ARG, "by_row and by_column are NULL");
    if (by_row) TRY(check_packed(by_row, "by_row"));
    if (by_column) TRY(check_packed(by_column, "by_column"));
    TRY(check_ctx(ctx));
    const hipStream_t st = (hipStream_t)stream;
    const double out = packed_bytes(format, (double)rows, (double)cols) * ((by_row != nullptr) + (by_column != nullptr));
    TRACED(HH_TRACE_ELEMENTWISE, (double)rows * cols * dt_size(dt_of(dtype)) + out,
           mx_quantise(dt_of(dtype), rows, cols, x, ldx, format, rows_of(by_row), rows_of(by_column), st));
    return HH_OK;
}

extern "C" int hh_mx_values(hh_ctx* ctx, int64_t rows, int64_t k, int32_t format, const hh_mx_tensor* q, int32_t dtype, void* y, int64_t ldy,
                            void* stream) {
    TRY(check_dtype(dtype)); TRY(check_format(format, "format"));
    TRY(check_matrix(rows, k, mx_width(std::min<int64_t>(k, MOST_ROWS))));
    TRY(check_ld(ldy, k, "ldy")); TRY(check_packed(q, "q")); TRY(check_ptr(y, "y"));
    TRY(check_ctx(ctx));
    const hipStream_t st = (hipStream_t)stream;
    TRACED(HH_TRACE_ELEMENTWISE, (double)rows * k * dt_size(dt_of(dtype)) + packed_bytes(format, (double)rows, (double)k),
           mx_values(dt_of(dtype), rows, k, format, rows_of(q), y, ldy, st));
    return HH_OK;
}

// ------------------------------------------------------------------ residual and norm
static int check_add_norm(const hh_add_norm_cfg* c) {
    if (!c) return fail(HH_ERR_INVALID_ARG, "cfg is NULL");
    TRY(check_dtype(c->dtype)); TRY(check_format(c->format, "cfg.format", true));
    if (c->rows <= 0 || c->hidden <= 0) return fail(HH_ERR_INVALID_ARG, "cfg has a non-positive dimension");
    if (!(c->eps >= 0.f)) return fail(HH_ERR_INVALID_ARG, "eps must be >= 0");
    if (c->hidden > 32768) return fail(HH_ERR_UNSUPPORTED_SHAPE, "hidden %d exceeds 32768", c->hidden);
    if (c->rows > 1 << 24 || (int64_t)c->rows * mx_width(c->hidden) > (int64_t)1 << 34)
        return fail(HH_ERR_UNSUPPORTED_SHAPE, "%d rows of %d exceed 2^24 rows or 2^34 values", c->rows, c->hidden);
    return HH_OK;
}

extern "C" int hh_add_norm_fwd(hh_ctx* ctx, const hh_add_norm_cfg* cfg, const hh_dropout_cfg* drop, const void* x, const void* b, const void* g,
                               void* h, void* xn, const hh_mx_tensor* q, void* stream) {
    TRY(check_add_norm(cfg));
    Drop d{};
    if (drop) TRY(drop_of(drop, d));
    TRY(check_ptr(x, "x")); TRY(check_ptr(g, "g"));
    if (b) { TRY(check_ptr(b, "b")); TRY(check_ptr(h, "h")); }
    else if (h) return fail(HH_ERR_INVALID_ARG, "h is x where there is no b: it has to be NULL");
    if (xn) TRY(check_ptr(xn, "xn"));
    if (cfg->format != HH_MX_NONE) TRY(check_packed(q, "q"));
    else if (q) return fail(HH_ERR_INVALID_ARG, "q is given, but cfg.format is HH_MX_NONE");
    else if (!xn) return fail(HH_ERR_INVALID_ARG, "xn and q are NULL");
    TRY(check_ctx(ctx));
    const hipStream_t st = (hipStream_t)stream;
    const double n = (double)cfg->rows * cfg->hidden;
    const double bytes = n * dt_size(dt_of(cfg->dtype)) * (1 + 2 * (b != nullptr) + (xn != nullptr)) + (q ? packed_bytes(cfg->format, cfg->rows, cfg->hidden) : 0.0);
    TRACED(HH_TRACE_ELEMENTWISE, bytes,
           add_norm_fwd(dt_of(cfg->dtype), d, cfg->rows, cfg->hidden, cfg->eps, x, b, g, h, xn, cfg->format, rows_of(q), st));
    return HH_OK;
}

extern "C" int hh_add_norm_sizes(const hh_add_norm_cfg* cfg, size_t* workspace_bytes) {
    TRY(check_add_norm(cfg));
    if (workspace_bytes) *workspace_bytes = up256((size_t)add_norm_partial_rows(cfg->rows, cfg->hidden) * cfg->hidden * 4);
    return HH_OK;
}

extern "C" int hh_add_norm_bwd(hh_ctx* ctx, const hh_add_norm_cfg* cfg, const hh_dropout_cfg* drop, const void* h, const void* g, const void* dxn,
                               const void* dh, void* dx, void* db, float* dg, int accumulate, void* workspace, void* stream) {
    TRY(check_add_norm(cfg));
    Drop d{};
    if (drop) TRY(drop_of(drop, d));
    TRY(check_ptr(h, "h")); TRY(check_ptr(g, "g")); TRY(check_ptr(dxn, "dxn")); TRY(check_ptr(dx, "dx"));
    if (dh) TRY(check_ptr(dh, "dh"));
    if (db) TRY(check_ptr(db, "db"));
    if (db == dx) return fail(HH_ERR_INVALID_ARG, "db is dx");
    if (dg) { TRY(check_ptr(dg, "dg")); TRY(check_ptr(workspace, "workspace")); }
    TRY(check_ctx(ctx));
    const hipStream_t st = (hipStream_t)stream;
    const double n = (double)cfg->rows * cfg->hidden;
    TRACED(HH_TRACE_ELEMENTWISE, n * dt_size(dt_of(cfg->dtype)) * (3 + (dh != nullptr) + (db != nullptr)),
           add_norm_bwd(dt_of(cfg->dtype), d, cfg->rows, cfg->hidden, cfg->eps, h, g, dxn, dh, dx, db, dg, accumulate, (float*)workspace, st));
    return HH_OK;
}

// ------------------------------------------------------------------ product
static int check_product(const hh_mx_product_cfg* c, MxProduct& p) {
    if (!c) return fail(HH_ERR_INVALID_ARG, "cfg is NULL");
    TRY(check_dtype(c->dtype)); TRY(check_format(c->a_format, "cfg.a_format")); TRY(check_format(c->b_format, "cfg.b_format"));
    if (c->sums != HH_MX_SUMS_F32 && c->sums != HH_MX_SUMS_FAST) return fail(HH_ERR_INVALID_ARG, "cfg.sums %d is not HH_MX_SUMS_F32/HH_MX_SUMS_FAST", c->sums);
    if (c->m <= 0 || c->n <= 0 || c->k <= 0) return fail(HH_ERR_INVALID_ARG, "cfg has a non-positive dimension");
    TRY(check_ld(c->ldc, c->n, "cfg.ldc"));
    const int64_t width = mx_width(c->k), most = (1LL << 32) - (1LL << 25);
    if (c->m * width / (c->a_format == HH_MX_E4M3 ? 1 : 2) >= most || c->n * width / (c->b_format == HH_MX_E4M3 ? 1 : 2) >= most)
        return fail(HH_ERR_UNSUPPORTED_SHAPE, "an operand of %d or %d rows of %d values reaches 2^32 bytes", c->m, c->n, c->k);
    if ((int64_t)c->m * c->n > 1LL << 33) return fail(HH_ERR_UNSUPPORTED_SHAPE, "a result of %d x %d exceeds 2^33 elements", c->m, c->n);
    p = MxProduct{c->m, c->n, c->k, c->a_format, c->b_format, {}, {}, nullptr, c->ldc, c->dtype == HH_F32, 0, c->sums == HH_MX_SUMS_FAST};
    return HH_OK;
}

extern "C" int hh_mx_product_sizes(const hh_mx_product_cfg* cfg, size_t* workspace_bytes) {
    MxProduct p;
    TRY(check_product(cfg, p));
    if (workspace_bytes) *workspace_bytes = up256(mx_product_workspace(p));
    return HH_OK;
}

extern "C" int hh_mx_product(hh_ctx* ctx, const hh_mx_product_cfg* cfg, const hh_mx_tensor* a, const hh_mx_tensor* b, void* c, int accumulate,
                             void* workspace, void* stream) {
    MxProduct p;
    TRY(check_product(cfg, p));
    TRY(check_packed(a, "a")); TRY(check_packed(b, "b")); TRY(check_ptr(c, "c"));
    if (mx_product_workspace(p)) TRY(check_ptr(workspace, "workspace"));
    TRY(check_ctx(ctx));
    p.a = rows_of(a); p.b = rows_of(b); p.C = c; p.accumulate = accumulate != 0;
    const hipStream_t st = (hipStream_t)stream;
    TRACED(HH_TRACE_GEMM_NT, 2.0 * cfg->m * cfg->n * cfg->k, mx_product(p, workspace, st));
    return HH_OK;
}
