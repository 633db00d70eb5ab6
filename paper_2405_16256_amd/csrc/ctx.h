// What the C entry points share: the context, errors, checks of arguments, tracing.  (Internal to the library, host only.)
#pragma once
#include "../../include/hh.h"

#include <hip/hip_runtime.h>

#include <vector>

#include "kernels.h"

struct TraceRec {
    hipEvent_t a, b;
    int kind;
    double work;
    size_t events;  // the record whose events bracket the launch (its own, unless GEMMs share one)
    double share;   // of the time between them that is this family's
    int count;      // micro-batches that the launch takes side by side: it stands for a launch of each
};
struct hh_ctx {
    int device;
    float* rope_table;  // device: cos[S][d/2] then sin[S][d/2]
    int rope_seq, rope_dim;
    float rope_base;
    std::vector<TraceRec> trace;  // events created by hh_trace_begin
    size_t trace_used;
    bool trace_on;
    uint32_t trace_mask;          // families recorded while trace_on
    void* gemm_ws;                // k-split scratch inside the caller's workspace, set by each hot call
    size_t gemm_room;             // its bytes where several micro-batches go side by side, set by each such call
    std::vector<float*> retired_tables;   // rotary tables replaced by a larger one: freed with the context
};

namespace hh {

// ------------------------------------------------------------------ errors
int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int hip_fail(hipError_t e, const char* what);
int check_ptr(const void* p, const char* name);   // not null, 16-byte aligned

// ------------------------------------------------------------------ tracing
// When tracing is on, every kernel-family launch is bracketed by two events on the
// launch stream; hh_trace_end turns them into per-family time and work sums.
struct Traced {
    hipStream_t st; TraceRec* rec;
    Traced(hh_ctx* c, hipStream_t s, int kind, int count, double work) : st(s), rec(nullptr) {
        if (c->trace_on && ((c->trace_mask >> kind) & 1u) && c->trace_used < c->trace.size()) {
            rec = &c->trace[c->trace_used++];
            rec->kind = kind; rec->work = work * count; rec->events = c->trace_used - 1; rec->share = 1.0; rec->count = count;
            (void)hipEventRecord(rec->a, st);
        }
    }
    ~Traced() { if (rec) (void)hipEventRecord(rec->b, st); }
};
// A group of GEMMs in one call, traced.  Their scratch is ctx->gemm_ws.
hipError_t tgemm(hh_ctx* ctx, int dt, GemmDesc* g, int n, hipStream_t st);
inline hipError_t tgemm(hh_ctx* ctx, int dt, GemmDesc g, hipStream_t st) { return tgemm(ctx, dt, &g, 1, st); }
GemmDesc desc(int kind, int M, int N, int K, const void* A, int lda, const void* B, int ldb, void* C, int ldc,
              const void* R = nullptr, int ldr = 0, int out_f32 = 0, int acc = 0);

inline size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }
inline char* at(void* base, size_t off) { return (char*)base + off; }
inline const char* at(const void* base, size_t off) { return (const char*)base + off; }

}  // namespace hh

#define HIP_TRY(call)                                        \
    do {                                                     \
        hipError_t e_ = (call);                              \
        if (e_ != hipSuccess) return hh::hip_fail(e_, #call); \
    } while (0)
#define TRY(x)                \
    do {                      \
        int rc_ = (x);        \
        if (rc_ != HH_OK) return rc_; \
    } while (0)
