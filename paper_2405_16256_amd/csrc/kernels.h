// Host-side launchers of the gfx950 kernels (internal to the library).
// All pointers are device pointers; every launcher only enqueues on `st`.
#pragma once
#include <hip/hip_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace hh {

enum { DT_F32 = 0, DT_BF16 = 1 };
inline size_t dt_size(int dt) { return dt == DT_BF16 ? 2 : 4; }

// One operand of up to MICRO_MAX micro-batches that a launch takes side by side: its address in each of them.
constexpr int MICRO_MAX = 8;
struct Each { void* p[MICRO_MAX]; };

// C[M,N] (=|+=) op(A) op(B) (+ R), leading dimensions in elements.
//   GEMM_NT: A[M,K] row-major, B[N,K] row-major   (y = x W^T)
//   GEMM_NN: A[M,K] row-major, B[K,N] row-major   (dX = dY W)
//   GEMM_TN: A[K,M] row-major, B[K,N] row-major   (dW = dY^T X)
enum { GEMM_NT = 0, GEMM_NN = 1, GEMM_TN = 2 };
// The operands of a problem that the launch repeats for several micro-batches (weight gradients: C is the same in all of
// them and their products are added in the order of the micro-batches, each as a launch of its own would add it).
struct GemmMicro { Each A, B, C, R, X, Y; };
// What a GEMM (in bf16 the ring kernel) can do with a product before it is written, in place of a launch of its own:
//   FUSE_ROPE       NT, C = q|k|v rows or a part of them: the rotary embedding of the first `rot` columns, heads of `period`
//   FUSE_SWIGLU     NT, C = gate|up rows [M, period]: X [M, period/2] = silu(gate) * up
//   FUSE_SWIGLU_BWD NN, the product is dm [M, N]: with X = gate|up, C = m and Y = dgate|dup
// Each on the product rounded to the storage type, as the launch would read it.
enum { FUSE_NONE = 0, FUSE_ROPE, FUSE_SWIGLU, FUSE_SWIGLU_BWD };
// The largest tile (rows x columns) on which the ring kernel does it.
constexpr int fuse_tile(int kind) { return kind == FUSE_ROPE ? 192 * 128 : kind == FUSE_SWIGLU ? 128 * 128 : 64 * 128; }
struct GemmFuse {
    int kind;
    int period, rot;
    int seq, table_seq; const float* table;   // FUSE_ROPE: as for rope()
    void* X; void* Y;
};
// Partial sums of an NT or NN problem that its launch has left to the kernel that reads the result: fp32 tiles
// [tile][micro-batch][share][bm*bn], to be added in the order of the shares (then the residual) and rounded.
struct GemmSplit { const float* partial; int ksplit, bm, bn, tiles_n; };
// The launch leaves at most SPLIT_ROW of them for a row, in two shares or more: rows of at most SPLIT_COLUMNS columns.
constexpr int SPLIT_ROW = 16384, SPLIT_COLUMNS = SPLIT_ROW / 2;
// The RMSNorm of the rows of A on the way into an NT launch: xn and r (of each micro-batch) are written beside the product.
struct GemmNorm { Each xn, r; const void* gain; float eps; };
constexpr int NORM_K = 256;
// An NT launch (bf16) whose result is scores [M, N] over a vocabulary of any size N: fp32 in z (rows of ldc; null: not written),
// the largest score of a row and the sum of exp(score - largest) for each SCORE_SLOT columns in stats [slot][M], and behind
// those, [M] floats, the score of the row's label (of a label that is no column: nothing).  stats null: the scores alone.
constexpr int SCORE_SLOT = 64;
// Column c is word first + c of the vocabulary that the labels count in.
struct GemmScores { float* z; float2* stats; const int64_t* labels; int first; };
struct GemmDesc {
    int kind;
    int M, N, K;
    const void* A; int lda;
    const void* B; int ldb;
    int pair;                // TN (bf16): row K/2 + k of A is what row k lacks of its value, and row K/2 + k of B is row k again
    int long_k;              // fp32: gemm_f32_long_k takes it
    int b_rows;              // rows of B that are there (0: as many as the product has); the others read as zeros
    void* C; int ldc;
    const void* R; int ldr;  // optional residual in the storage dtype, added before rounding (NULL: none)
    int out_f32;             // 1: C is fp32 regardless of the storage dtype (parameter gradients)
    int accumulate;          // 1: C += result
    // B of an NN problem in up to three allocations: rows k1.. at B1, rows k2.. at B2 (0: no such segment)
    const void* B1; int k1;
    const void* B2; int k2;
    void* ws;                // optional scratch for k-split partial sums (bf16 path), may be NULL
    size_t ws_bytes;         // of one micro-batch: what a plan may use
    size_t ws_room;          // micro > 1: what there is for all of them
    GemmFuse fuse;
    GemmSplit* split;        // not null: the launch may leave its partial sums (ksplit > 1 then, else C is complete)
    const GemmNorm* norm;    // not null (bf16, where gemm_bf16_norms): A holds x, and xn takes its place; one for a launch
    const GemmScores* scores;   // not null (NT, bf16): C stays unused
    int micro;               // micro-batches; above 1 (bf16: where gemm_bf16_on_ring) their operands are in `each`
    const GemmMicro* each;
};
constexpr int MAX_LD = 1 << 18;   // elements of an operand's row, a vocabulary among them
constexpr size_t GEMM_WS_BYTES = (size_t)64 << 20;   // enough for 256 partial tiles of 256x256 fp32

// The library's own scratch array (one per GPU, held until the process ends) and its size.
constexpr size_t STATIC_SCRATCH_BYTES = (size_t)128 << 20;
hipError_t static_scratch_init(int device);   // `device` must be current; looks the array's address up once
void* static_scratch(int device);             // that address (null before a successful init)
// Up to 4 problems (8 weight gradients in bf16) of which none reads what another writes, either all NT or none; they share launches where that is
// predicted to be faster.
hipError_t gemm(int dtype, const GemmDesc* g, int n, hipStream_t st);
// One fp32 NN problem of a long k cut along it (gemm_f32_long_k.hip; needs `ws`, nothing added, no segments or micro-batches), and
// whether that is better.
hipError_t gemm_f32_long_k(const GemmDesc& g, hipStream_t st);
bool gemm_f32_long_k_better(int M, int N, int K);
// Whether all launches of these problems (bf16) are the ring kernel's, and if so: the bytes of partial sums that the largest of
// those launches keeps, its workgroups, and the largest tile.
struct RingUse { size_t partial; long workgroups; int tile; };
bool gemm_bf16_on_ring(const GemmDesc* g, int n, RingUse* use);
// Whether one launch of these problems (NT, one A) can norm the rows of A, and had better.
bool gemm_bf16_norms(const GemmDesc* g, int n);
// Whether they do; if not, gemm() on each of them alone launches the same.
bool gemm_shares_launch(int dtype, const GemmDesc* g, int n);

// xn = x * r * g, r = 1/sqrt(mean(x^2)+eps) per row.
// Here and below: micro-batches 0 .. n-1 side by side, an operand's address in each of them; the result of a micro-batch
// does not depend on n.
// split (bf16): x has yet to be summed (with the residual `res`) and written.
hipError_t rmsnorm_fwd(int dtype, const Each& x, const void* g, const Each& xn, const Each& r,
                       int n, int T, int H, float eps, hipStream_t st, const GemmSplit* split = nullptr, const Each* res = nullptr);
// dx = dres + r*(w - u*mean(w*u)), u = x*r, w = dxn*g; per-workgroup column sums of
// dxn*u go to partial[rmsnorm_bwd_blocks(T, H, partial_bytes)][H].
int rmsnorm_bwd_blocks(int T, int H, size_t partial_bytes);
hipError_t rmsnorm_bwd(int dtype, const Each& dxn, const Each& x, const Each& r, const void* g,
                       const Each& dres, const Each& dx, const Each& partial, size_t partial_bytes, int n, int T, int H, hipStream_t st,
                       const GemmSplit* split = nullptr,   // bf16: in place of dxn
                       float* gain = nullptr, int accumulate = 0);   // gain: gradient of g, written (+=) here; no partial sums then
// Whether rmsnorm_bwd had better write the gain's gradient itself (where nothing it reads is written by it).
bool rmsnorm_bwd_sums_gain(int T, int H, const GemmSplit* split);
// out[H] (=|+=) column sums of partial[rows][H], of one micro-batch after the other; one or two such sums in one launch
struct ColSum { Each partial; int rows; float* out; };
hipError_t colsum_reduce(const ColSum* jobs, int n_jobs, int n, int H, int accumulate, hipStream_t st);

// In-place rotary embedding of the first nrot heads (query heads, then key heads) of every row of a
// [T, ld] buffer.  table = cos[table_seq][d/2] followed by sin[table_seq][d/2], table_seq >= S.  (The backward rotation is
// part of attn_bwd.)
hipError_t rope(int dtype, const Each& qkv, int ld, int n, int T, int S, int nrot, int d, const float* table, int table_seq,
                hipStream_t st);

// gu[T,2F] = (gate | up);  m = silu(gate)*up
hipError_t swiglu_fwd(int dtype, const Each& gu, const Each& m, int n, int T, int F, hipStream_t st);
// dgu[T,2F] = (dgate | dup), and m recomputed
hipError_t swiglu_bwd(int dtype, const Each& dm, const Each& gu, const Each& dgu, const Each& m, int n, int T, int F, hipStream_t st);

// Causal attention over a [T, ld] buffer holding q | k | v column blocks of width nh*d, nkv*d, nkv*d;
// query head h uses key/value head h / (nh / nkv).  o [T, nh*d]; lse [B, nh, S] natural-log sum-exp of
// the scaled scores.
// micro.n micro-batches side by side, micro.saved bytes apart in qkv, o and lse, micro.ws bytes in dout, dvec, dqkv and
// scratch; how a micro-batch is split over workgroups does not depend on micro.n.
struct MicroStride { int n; size_t saved, ws; };
hipError_t attn_fwd(int dtype, const void* qkv, int ld, void* o, float* lse,
                    int B, int S, int nh, int nkv, int d, const MicroStride& micro, hipStream_t st);
// dqkv [T, ld] receives dq | dk | dv in the same layout.  dvec: scratch [B, nh, S] floats.  scratch: device
// memory of scratch_bytes, at least attn_bwd_scratch_bytes() (partial dK, dV sums when the query heads that share a
// key/value head are spread over several workgroups; may be null when it has no bytes; the fp32 path needs none and
// spreads the heads as far as what it is given reaches).  rope_table (as for rope(), rope_seq >= S;
// null: none): q and k were rotated before the forward call, and dq, dk are written as gradients of the
// unrotated q, k (the backward rotation applied before the one rounding to the storage type).
size_t attn_bwd_scratch_bytes(int dtype, int B, int S, int nh, int nkv, int d);
hipError_t attn_bwd(int dtype, const void* qkv, int ld, const void* o, const void* dout, const float* lse,
                    float* dvec, void* dqkv, void* scratch, size_t scratch_bytes, int B, int S, int nh, int nkv, int d,
                    const float* rope_table, int rope_seq, const MicroStride& micro, hipStream_t st);

// ---- output projection and softmax cross entropy (head.hip).  stats: [slot][M] (largest score, sum of exponentials) and behind them
// [M] floats, the labels' scores, as of GemmScores.
// What the calls below share: M tokens; the columns are words first .. first + N - 1, and a token counts whose label is from 0 to
// limit - 1.
struct HeadTokens { const int64_t* labels; int64_t first, limit; int M, N; const float* dloss; float scale; };
// The same of fp32 scores [M, N] in rows of ldz, slots of HEAD_F32_SLOT columns.
constexpr int HEAD_F32_SLOT = 1024;
hipError_t head_stats_f32(const HeadTokens& t, const float* z, int ldz, float2* stats, hipStream_t st);
// Whole rows of up to head_row_most() scores, of a whole vocabulary, at once: loss[M], and what head_grad writes where d is not null.
constexpr int head_row_most(int dtype) { return dtype == DT_BF16 ? 16384 : 32768; }
hipError_t head_row(int dtype, const HeadTokens& t, const float* z, int ldz, float* loss, void* d, int lo_rows, const void* x, void* xs, int H,
                    hipStream_t st);
// From the statistics of a row, each where it is not null: loss[M], lse[M] its log-sum-exp, norm[M] its largest score and one over its sum
// of exponentials, picked[M] its label's score, 0 where that is no column.
hipError_t head_rows(const HeadTokens& t, const float2* stats, int slots, float* loss, float* lse, float2* norm, float* picked, hipStream_t st);
// d from the scores z (rows of ldz both, the padding zeros) and their rows' norm, or log-sum-exp where norm is null, in bf16 as two
// matrices, the second lo_rows rows behind the first, in fp32 in place; and x [M, H] with zeros for the tokens that do not count, in
// bf16 a second time lo_rows rows behind.
hipError_t head_grad(int dtype, const HeadTokens& t, const float* z, int ldz, const float2* norm, const float* lse, void* d, int lo_rows, const void* x,
                     void* xs, int H, hipStream_t st);

// ---- lists of tensors (tensors.hip)
constexpr int CLIP_CHUNK = 8192, ADAMW_CHUNK = 2048;   // elements that a workgroup takes at a time
// What a launch reads and writes leaves nothing in the last-level cache for the next one where it is more than this.
constexpr size_t LIST_CACHE = (size_t)256 << 20;
constexpr int CLIP_LIST = 112, ADAMW_LIST = 56;   // tensors of a launch: what fits a kernel's arguments (4 KB), two for each lane of a wave at most
constexpr int CLIP_SLOTS = 1024;         // partial sums of squares
// `head` elements lie in front of the first one at which all pointers are aligned for vectors; -1: there is none.  Chunk c of the
// launch belongs to the last tensor with first <= c.
struct ClipItem { const void* g; void* out; int64_t count; int32_t first; int16_t head, bf16; };
struct ClipList { int n, chunks; ClipItem t[CLIP_LIST]; };
struct AdamwItem { void* param; float* master; float* m; float* v; const void* g; int64_t count; float keep; int32_t first; int16_t head, param_bf16, grad_bf16, pad; };
struct AdamwList { int n, chunks; AdamwItem t[ADAMW_LIST]; };
static_assert(sizeof(ClipList) + 32 <= 4096 && sizeof(AdamwList) + sizeof(float) * 16 <= 4096, "kernel arguments");
// keep: 1 - lr * decay
struct AdamwHyper { float beta1, rest1, beta2, rest2, eps, step_size, inv_sqrt_bc2; };   // rest: 1 - beta
// slots[0 .. wgs-1] (+)= sums of squares; wgs <= CLIP_SLOTS workgroups
hipError_t clip_squares(const ClipList& l, double* slots, int wgs, int add, hipStream_t st);
// result = (norm, factor) of the `slots` sums
hipError_t clip_result(const double* slots, int n_slots, float max_norm, float* result, hipStream_t st);
// the same (where `result` is not null), and the clipped copies
hipError_t clip_scale(const ClipList& l, const double* slots, int n_slots, float max_norm, float* result, hipStream_t st);
// stream: the tensors of all launches together are past LIST_CACHE
hipError_t adamw(const AdamwList& l, const AdamwHyper& h, const float* factor, bool stream, hipStream_t st);

// ---- residual path and microscaled formats (residual.hip, mx_pack.hip, mx_product.hip)
enum { MX_NONE = 0, MX_E4M3 = 1, MX_E2M1 = 2 };
constexpr int MX_PAD = 256;
inline long mx_width(long k) { return (k + MX_PAD - 1) / MX_PAD * MX_PAD; }
// dropped: of 65536 values, scale: of the others (nothing is dropped at 0)
struct Drop { uint64_t seed, offset; const uint64_t* step; uint32_t dropped; float scale; };
// A packed tensor of rows of `width` codes, a multiple of MX_PAD
struct MxRows { uint8_t* codes; uint8_t* scales; };
hipError_t dropout(int dtype, const Drop& d, long rows, long cols, const void* x, long ldx, void* y, long ldy, hipStream_t st);
hipError_t add_norm_fwd(int dtype, const Drop& d, int rows, int hidden, float eps, const void* x, const void* b, const void* g, void* h, void* xn,
                        int format, const MxRows& q, hipStream_t st);
// partial: add_norm_partial_rows() rows of `hidden` sums for dg, which is not written where it is null
int add_norm_partial_rows(int rows, int hidden);
hipError_t add_norm_bwd(int dtype, const Drop& d, int rows, int hidden, float eps, const void* h, const void* g, const void* dxn, const void* dh,
                        void* dx, void* db, float* dg, int accumulate, float* partial, hipStream_t st);
hipError_t mx_quantise(int dtype, long rows, long cols, const void* x, long ldx, int format, const MxRows& by_row, const MxRows& by_column,
                       hipStream_t st);
hipError_t mx_values(int dtype, long rows, long k, int format, const MxRows& q, void* y, long ldy, hipStream_t st);
// fast: sums may be of fewer bits than fp32's
struct MxProduct { int M, N, K; int fa, fb; MxRows a, b; void* C; long ldc; int f32, accumulate, fast; };
size_t mx_product_workspace(const MxProduct& p);
hipError_t mx_product(const MxProduct& p, void* ws, hipStream_t st);

}  // namespace hh
