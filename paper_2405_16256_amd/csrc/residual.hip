// Dropout, and the residual's addition with its norm: forward and backward.  All of them stream their tensors once.
#include <algorithm>

#include "mx.h"

namespace hh {

// ------------------------------------------------------------------ dropout
// Eight values a lane, which share a counter.  Bound by memory, with the generator in its shadow: 4096x12288 bf16 33 us (6.0 TB/s).
template <typename T, bool STREAM>
__global__ __launch_bounds__(256) void k_dropout(Drop d, int chunks, Divisor per_row, int cols, const T* x, long ldx, T* y, long ldy) {
    const int i = (int)(blockIdx.x * 256u + threadIdx.x);
    if (i >= chunks) return;
    int row = i;
    const int group = split_off(row, per_row), n = cols - 8 * group;
    const long at = 8L * group;
    Eight<T> e;
    e.template load<STREAM>(x + row * ldx + at, n);
    float v[8];
    e.widen(v);
    drop8(d, drop_offset(d), (uint32_t)group, (uint32_t)row, v);
    e.round(v);
    e.template store<STREAM>(y + row * ldy + at, n);
}

hipError_t dropout(int dtype, const Drop& d, long rows, long cols, const void* x, long ldx, void* y, long ldy, hipStream_t st) {
    const int per_row = (int)((cols + 7) / 8), chunks = (int)(rows * per_row);
    const unsigned grid = ((unsigned)chunks + 255u) / 256u;
    const bool stream = 2.0 * rows * cols * dt_size(dtype) > STREAM_BYTES;
    auto run = [&](auto kern, auto* from, auto* to) {
        kern<<<grid, 256, 0, st>>>(d, chunks, divisor(per_row), (int)cols, from, ldx, to, ldy);
        return hipGetLastError();
    };
    if (dtype == DT_BF16) return run(stream ? k_dropout<bf16_t, true> : k_dropout<bf16_t, false>, (const bf16_t*)x, (bf16_t*)y);
    return run(stream ? k_dropout<float, true> : k_dropout<float, false>, (const float*)x, (float*)y);
}

// ------------------------------------------------------------------ residual and norm
// h = x + dropout(b), r = 1 / sqrt(mean h^2 + eps), xn = h r g: a row stays in registers from its sum to its packed copy, so that each tensor
// is read or written once.  Bound by memory: 4096x12288 bf16 with dropout, h, xn and E4M3 written 77.8 us (5.8 TB/s); rows of 32768, 2048 of them,
// bf16 105 us, fp32 227 (5.1 and 4.7 TB/s); one row of 4096 3.2 us, a launch and a chain of loads, two barriers and stores.
// W waves a row, CH chunks of eight values a lane: chunk t + 64 W c.  Four rows to a workgroup where a wave takes one.
template <int W> constexpr int row_threads() { return W == 1 ? 256 : 64 * W; }
template <int W> constexpr int rows_each() { return W == 1 ? 4 : 1; }

// RAGGED: rows end inside a chunk.  The others are reached from a scalar address with a 32-bit distance, without a second path for the
// last chunk: a third of the registers of a row of 12288.
template <bool RAGGED> __device__ __forceinline__ int chunk_values(int hidden, int at) { return RAGGED ? hidden - at : at < hidden ? 8 : 0; }
template <typename T> __device__ __forceinline__ T* chunk_at(T* row, int at) { return (T*)((char*)row + (uint32_t)at * (uint32_t)sizeof(T)); }
template <typename T> __device__ __forceinline__ const T* chunk_at(const T* row, int at) { return (const T*)((const char*)row + (uint32_t)at * (uint32_t)sizeof(T)); }

// r = 1 / sqrt(ss / hidden + eps).  What a row's values have in common, the sums of eight squares each and r, is carried in 64 bits, r as the sum of two
// floats: a value of xn is rounded twice then, v r and the product with g.  4096x12288 bf16, of 1e6 values of xn 4.7 round otherwise than in 64 bits (7.5
// with fp32 sums and root), at the same time; rows of 512 lose most, 8192x512 8.9 -> 9.2 us.
template <int W>
__device__ __forceinline__ double lanes_sum(double s, double (&red)[W]) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, WAVE);
    if (W == 1) return s;
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
    __syncthreads();
    s = 0.0;
#pragma unroll
    for (int i = 0; i < W; i++) s += red[i];
    return s;
}
struct Root { float hi, lo; };
__device__ __forceinline__ Root split_inverse_root(double ss, double per_value, float eps) {
    const double a = fma(ss, per_value, (double)eps), x = __builtin_amdgcn_rsq(a), better = fma(0.5 * x, fma(-a * x, x, 1.0), x);
    const double r = better > 0.0 ? better : x;   // at 0 and at infinity, where Newton's step is NaN
    const float hi = (float)r;
    return Root{hi, hi < INFINITY ? (float)(r - hi) : 0.f};
}

// v r g for packing, near a border between two numbers of a format: on the side where the unrounded product lies, that is, with what is left of it behind
// the last bit as that bit.  Rounded to fp32 first, 9.5e-7 of the values that become E4M3 lie on a border, and half of them on its wrong side, which is
// a step of the format; so 44 of 1e8 were wrong, and 2 are.  4096x12288 with E4M3 79.5 -> 80.4 us, 256x4096 with E2M1 5.2 -> 5.5.
__device__ __forceinline__ float normed_odd(float v, const Root& r, float g) {
    const float y = v * r.hi, y_rest = fmaf(v, r.lo, fmaf(v, r.hi, -y)), u = y * g, u_rest = fmaf(y_rest, g, fmaf(y, g, -u));
    const float s = u + u_rest, rest = (u - s) + u_rest;
    constexpr int NORMAL_OR_DENORMAL = 0x198;   // of either sign
    if (!__builtin_amdgcn_classf(u_rest, NORMAL_OR_DENORMAL)) return u;   // an infinity, what is no number, and zeros with their sign
    if (fabsf(rest) <= fabsf(s) * 0x1p-40f) return s;   // s itself, but for the roundings in 64 bits
    const uint32_t w = __float_as_uint(s);
    return __uint_as_float((w - ((w ^ __float_as_uint(rest)) >> 31)) | 1u);
}

template <typename T, int W, int CH, bool RAGGED, bool STREAM>
__global__ __launch_bounds__(row_threads<W>()) void k_add_norm_fwd(Drop d, int rows, int hidden, int width, float eps, double per_value, const T* x, const T* b,
                                                                     const T* __restrict__ g, T* h, T* xn, int format, uint8_t* codes, uint8_t* scales) {
    __shared__ double red[W];
    const int t = (int)threadIdx.x & (64 * W - 1);
    const int row = (int)blockIdx.x * rows_each<W>() + (W == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0);
    if (row >= rows) return;   // one wave a row: no barrier follows
    const long base = (long)row * hidden;
    const T* const x_row = x + base;
    const T* const b_row = b + base;
    T* const h_row = h + base;
    T* const xn_row = xn + base;
    Eight<T> rx[CH], rb[CH], rg[CH];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int at = 8 * (t + 64 * W * c), n = chunk_values<RAGGED>(hidden, at);
        rx[c] = Eight<T>{};
        rb[c] = Eight<T>{};
        rg[c] = Eight<T>{};
        if (n > 0) {
            rx[c].template load<STREAM>(chunk_at(x_row, at), n);
            if (b) rb[c].template load<STREAM>(chunk_at(b_row, at), n);
            rg[c].load(chunk_at(g, at), n);
        }
    }
    const uint64_t offset = b && d.dropped ? drop_offset(d) : 0;
    float v[CH][8];
    double ss = 0.0;
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int group = t + 64 * W * c, n = chunk_values<RAGGED>(hidden, 8 * group);
        float squares = 0.f;
        rx[c].widen(v[c]);
        if (b && n > 0) {
            float u[8];
            rb[c].widen(u);
            if (d.dropped) drop8(d, offset, (uint32_t)group, (uint32_t)row, u);
#pragma unroll
            for (int i = 0; i < 8; i++) v[c][i] += u[i];
            rx[c].round(v[c]);
            rx[c].template store<STREAM>(chunk_at(h_row, 8 * group), n);
            rx[c].widen(v[c]);   // the norm is of the sum as it is kept
        }
#pragma unroll
        for (int i = 0; i < 8; i++) squares = fmaf(v[c][i], v[c][i], squares);
        ss += squares;
    }
    const Root r = split_inverse_root(lanes_sum<W>(ss, red), per_value, eps);
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int group = t + 64 * W * c, n = chunk_values<RAGGED>(hidden, 8 * group);
        float u[8];
        rg[c].widen(u);
#pragma unroll
        for (int i = 0; i < 8; i++) u[i] = i < n ? fmaf(v[c][i], r.hi, v[c][i] * r.lo) * u[i] : 0.f;   // past the end also where r is no number
        if (xn && n > 0) {
            Eight<T> e;
            e.round(u);
            e.template store<STREAM>(chunk_at(xn_row, 8 * group), n);
        }
        if (format != MX_NONE && 8 * group < width) {   // whole blocks of 32: the four lanes of one are here together
            // Borders (of normal numbers) end in 19 zeros at least, and two roundings are off by two last bits at most.
            uint32_t least = ~0u;
#pragma unroll
            for (int i = 0; i < 8; i++) least = min(least, (__float_as_uint(u[i]) + 2u) << 13);
            if (__builtin_expect(least <= 4u << 13, 0)) {
#pragma unroll
                for (int i = 0; i < 8; i++)
                    if ((__float_as_uint(u[i]) + 2u) << 13 <= 4u << 13 && i < n) u[i] = normed_odd(v[c][i], r, rg[c].at(i));
            }
            const uint32_t m = quad_max(magnitude8(u));
            const Pair<float> pairs[4] = {{u[0], u[1]}, {u[2], u[3]}, {u[4], u[5]}, {u[6], u[7]}};
            uint32_t byte;
            if (format == MX_E4M3) {
                const Packer<MX_E4M3> q(m);
                byte = q.byte;
                q.store8(pairs, codes + (size_t)row * width, group);
            } else {
                const Packer<MX_E2M1> q(m);
                byte = q.byte;
                q.store8(pairs, codes + (size_t)row * (width / 2), group);
            }
            store_scales(scales + (size_t)row * (width / MX_BLOCK) + (group >> 2), byte);
        }
    }
}

template <typename T>
static hipError_t fwd(const Drop& d, int rows, int hidden, float eps, const void* x, const void* b, const void* g, void* h, void* xn, int format,
                      const MxRows& q, hipStream_t st) {
    const int width = format == MX_NONE ? 0 : (int)mx_width(hidden), chunks = format == MX_NONE ? (hidden + 7) / 8 : width / 8;
    const bool stream = (double)rows * hidden * sizeof(T) * (1 + 2 * (b != nullptr) + (xn != nullptr)) > STREAM_BYTES;
    auto run = [&](auto kern, int each, int threads) {
        kern<<<(rows + each - 1) / each, threads, 0, st>>>(d, rows, hidden, width, eps, 1.0 / hidden, (const T*)x, (const T*)b, (const T*)g, (T*)h, (T*)xn, format,
                                                           q.codes, q.scales);
        return hipGetLastError();
    };
#define HH_SHAPE(W, CH) \
    if (chunks <= 64 * W * CH)                            \
        return run(hidden % 8 ? k_add_norm_fwd<T, W, CH, true, false> : stream ? k_add_norm_fwd<T, W, CH, false, true> : k_add_norm_fwd<T, W, CH, false, false>, \
                   rows_each<W>(), row_threads<W>())
    // Few rows take more waves each: the chip is not full, and a row's own chain is what they wait for (700x1003 fp32 5.6 -> 4.8 us, 2000x1024
    // bf16 the other way 4.8 -> 5.1; 200x8192 bf16 5.1 -> 4.7, 2048x4096 12.0 with 4 waves).
    HH_SHAPE(1, 1);
    if (rows >= 1024) HH_SHAPE(1, 2);
    HH_SHAPE(4, 1);
    if (rows < 256) HH_SHAPE(16, 1);
    HH_SHAPE(4, 2); HH_SHAPE(4, 3); HH_SHAPE(4, 4); HH_SHAPE(4, 6);
    HH_SHAPE(16, 2); HH_SHAPE(16, 4);
#undef HH_SHAPE
    return hipErrorInvalidValue;
}
hipError_t add_norm_fwd(int dtype, const Drop& d, int rows, int hidden, float eps, const void* x, const void* b, const void* g, void* h, void* xn,
                        int format, const MxRows& q, hipStream_t st) {
    return dtype == DT_BF16 ? fwd<bf16_t>(d, rows, hidden, eps, x, b, g, h, xn, format, q, st)
                            : fwd<float>(d, rows, hidden, eps, x, b, g, h, xn, format, q, st);
}

// ------------------------------------------------------------------ gradients
// The division of a root rounds twice; a step of Newton's, with a r's rounding carried along, leaves little more than half a step.  At 0 and at
// infinity, where the step is NaN, r stays.
__device__ __forceinline__ float inverse_root(float ss, int hidden, float eps) {
    const float a = ss / (float)hidden + eps, r = 1.0f / sqrtf(a), x = a * r;
    const float better = fmaf(0.5f * r, fmaf(-x, r, 1.0f) - fmaf(a, r, -x) * r, r);
    return better > 0.f ? better : r;
}
// One row's share of dx, db and dg: eight values of h (a), dxn (u), g (w) and dh (o, which becomes dx).
__device__ __forceinline__ void norm_grad8(const float* a, const float* u, const float* w, float* o, float* sum, float r, float k) {
#pragma unroll
    for (int i = 0; i < 8; i++) {
        sum[i] = fmaf(u[i], a[i] * r, sum[i]);
        o[i] = fmaf(r, fmaf(-a[i], k, u[i] * w[i]), o[i]);
    }
}
// The two sums of a row over the waves of a workgroup; `red` is taken in turn, so that a row needs one barrier.
template <int W>
__device__ __forceinline__ void row_sums(float& ss, float& dot, float (&red)[2][W]) {
    ss = wave_sum(ss);
    dot = wave_sum(dot);
    if (W > 1) {
        if ((threadIdx.x & 63) == 0) { red[0][threadIdx.x >> 6] = ss; red[1][threadIdx.x >> 6] = dot; }
        __syncthreads();
        ss = dot = 0.f;
#pragma unroll
        for (int i = 0; i < W; i++) { ss += red[0][i]; dot += red[1][i]; }
    }
}

// With u = dxn g: dx = dh + r (u - h r^2 mean(u h)), db = dropout(dx), dg = sum over rows of dxn h r.  Statistics are formed again from h, which
// the pass reads anyway.  Bound by memory: 4096x12288 bf16, three tensors read and two written, 96.1 us (5.2 TB/s) and 5.1 for the sums of dg.
// Workgroups walk rows p, p + parts, ... (four of them at once where a wave takes one) and keep their sums for dg in registers; partial[p].
// Registers of bf16 rows are held to what leaves four waves on a SIMD: a row's loads wait for no one but themselves, and the other waves'
// cover them.
template <typename T, int CH> constexpr int grad_waves() { return sizeof(T) == 2 && CH <= 3 ? 4 : 2; }
template <typename T, int W, int CH, bool RAGGED, bool STREAM>
__global__ __launch_bounds__(row_threads<W>(), (RAGGED ? 2 : grad_waves<T, CH>())) void k_add_norm_bwd(Drop d, int rows, int hidden, int parts, float eps, const T* h,
                                                                                          const T* __restrict__ g, const T* dxn, const T* dh, T* dx, T* db,
                                                                                          float* __restrict__ partial) {
    __shared__ float red[2][2][W];
    const int t = (int)threadIdx.x & (64 * W - 1), sub = W == 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6) : 0;
    const int p = (int)blockIdx.x;
    const uint64_t offset = db && d.dropped ? drop_offset(d) : 0;
    Eight<T> rg[CH];
    float sum[CH][8];
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int at = 8 * (t + 64 * W * c), n = chunk_values<RAGGED>(hidden, at);
        rg[c] = Eight<T>{};
        if (n > 0) rg[c].load(chunk_at(g, at), n);
#pragma unroll
        for (int i = 0; i < 8; i++) sum[c][i] = 0.f;
    }
    int turn = 0;
    for (int row = p * rows_each<W>() + sub; row < rows; row += parts * rows_each<W>(), turn ^= 1) {
        const long base = (long)row * hidden;
        const T* const h_row = h + base;
        const T* const dxn_row = dxn + base;
        const T* const dh_row = dh + base;
        T* const dx_row = dx + base;
        T* const db_row = db + base;
        Eight<T> rh[CH], ru[CH], rd[CH];
#pragma unroll
        for (int c = 0; c < CH; c++) {
            const int at = 8 * (t + 64 * W * c), n = chunk_values<RAGGED>(hidden, at);
            rh[c] = Eight<T>{};
            ru[c] = Eight<T>{};
            rd[c] = Eight<T>{};
            if (n > 0) {
                rh[c].template load<STREAM>(chunk_at(h_row, at), n);
                ru[c].template load<STREAM>(chunk_at(dxn_row, at), n);
                if (dh) rd[c].template load<STREAM>(chunk_at(dh_row, at), n);
            }
        }
        float ss = 0.f, dot = 0.f;
#pragma unroll
        for (int c = 0; c < CH; c++) {
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float a = rh[c].at(i);
                ss = fmaf(a, a, ss);
                dot = fmaf(ru[c].at(i) * rg[c].at(i), a, dot);
            }
        }
        row_sums<W>(ss, dot, red[turn]);
        const float r = inverse_root(ss, hidden, eps), k = r * (r * (dot / (float)hidden));   // r^2 may be past fp32
#pragma unroll
        for (int c = 0; c < CH; c++) {
            __builtin_amdgcn_sched_barrier(0);   // a chunk at a time
            rh[c].hide();                        // kept as they lie in memory, and widened a second time
            ru[c].hide();
            rg[c].hide();
            int group = t + 64 * W * c;
            asm("" : "+v"(group));   // what the generator makes of it is not kept from row to row
            const int n = chunk_values<RAGGED>(hidden, 8 * group);
            if (n <= 0) continue;
            float a[8], u[8], w[8], o[8];
            rh[c].widen(a);
            ru[c].widen(u);
            rg[c].widen(w);
            rd[c].widen(o);
            norm_grad8(a, u, w, o, sum[c], r, k);
            Eight<T> e;
            e.round(o);
            e.template store<STREAM>(chunk_at(dx_row, 8 * group), n);
            if (db) {
                if (d.dropped) drop8(d, offset, (uint32_t)group, (uint32_t)row, o);
                e.round(o);
                e.template store<STREAM>(chunk_at(db_row, 8 * group), n);
            }
        }
    }
    if (!partial) return;
    if constexpr (W == 1) {   // the four waves' sums as one
        __shared__ __attribute__((aligned(16))) float part[3][512 * CH];
        if (sub) {
#pragma unroll
            for (int c = 0; c < CH; c++)
#pragma unroll
                for (int i = 0; i < 8; i++) part[sub - 1][8 * (t + 64 * c) + i] = sum[c][i];
        }
        __syncthreads();
        if (sub) return;
#pragma unroll
        for (int c = 0; c < CH; c++)
#pragma unroll
            for (int i = 0; i < 8; i++)
                sum[c][i] = (sum[c][i] + part[0][8 * (t + 64 * c) + i]) + (part[1][8 * (t + 64 * c) + i] + part[2][8 * (t + 64 * c) + i]);
    }
#pragma unroll
    for (int c = 0; c < CH; c++) {
        const int at = 8 * (t + 64 * W * c), n = chunk_values<RAGGED>(hidden, at);
        Eight<float> e;
        e.round(sum[c]);
        if (n > 0) e.store(chunk_at(partial + (long)p * hidden, at), n);
    }
}

// Rows too long for a workgroup's registers: asked for a second time, which the caches answer, and dg's sums in LDS (up to 128 KB), so that a compute
// unit has one workgroup, whose loads nothing covers: 4096x16384 fp32 333 us, 2048x32768 bf16 188, fp32 359 (4.0, 3.6 and 3.7 TB/s).
template <typename T>
__global__ __launch_bounds__(1024) void k_add_norm_bwd_wide(Drop d, int rows, int hidden, int parts, float eps, const T* h, const T* __restrict__ g,
                                                             const T* dxn, const T* dh, T* dx, T* db, float* __restrict__ partial) {
    extern __shared__ __attribute__((aligned(16))) float sums[];   // a multiple of 8, each lane its own
    __shared__ float red[2][2][16];
    const int p = (int)blockIdx.x, chunks = (hidden + 7) / 8;
    const uint64_t offset = db && d.dropped ? drop_offset(d) : 0;
    for (int i = (int)threadIdx.x; i < chunks; i += 1024)
#pragma unroll
        for (int j = 0; j < 8; j++) sums[8 * i + j] = 0.f;
    int turn = 0;
    for (int row = p; row < rows; row += parts, turn ^= 1) {
        const long base = (long)row * hidden;
        float ss = 0.f, dot = 0.f;
        for (int c = (int)threadIdx.x; c < chunks; c += 1024) {
            const int at = 8 * c, n = hidden - at;
            Eight<T> rh, ru, rg;
            rh.load(h + base + at, n);
            ru.load(dxn + base + at, n);
            rg.load(g + at, n);
#pragma unroll
            for (int i = 0; i < 8; i++) {
                const float a = rh.at(i);
                ss = fmaf(a, a, ss);
                dot = fmaf(ru.at(i) * rg.at(i), a, dot);
            }
        }
        row_sums<16>(ss, dot, red[turn]);
        const float r = inverse_root(ss, hidden, eps), k = r * (r * (dot / (float)hidden));   // r^2 may be past fp32
        for (int c = (int)threadIdx.x; c < chunks; c += 1024) {
            const int at = 8 * c, n = hidden - at;
            Eight<T> e, rd{};
            float a[8], u[8], w[8], o[8], sum[8];
            e.load(h + base + at, n);
            e.widen(a);
            e.load(dxn + base + at, n);
            e.widen(u);
            e.load(g + at, n);
            e.widen(w);
            if (dh) rd.load(dh + base + at, n);
            rd.widen(o);
#pragma unroll
            for (int i = 0; i < 8; i++) sum[i] = sums[at + i];
            norm_grad8(a, u, w, o, sum, r, k);
#pragma unroll
            for (int i = 0; i < 8; i++) sums[at + i] = sum[i];
            e.round(o);
            e.store(dx + base + at, n);
            if (db) {
                if (d.dropped) drop8(d, offset, (uint32_t)c, (uint32_t)row, o);
                e.round(o);
                e.store(db + base + at, n);
            }
        }
    }
    if (!partial) return;
    for (int c = (int)threadIdx.x; c < chunks; c += 1024) {
        Eight<float> e;
        e.round(sums + 8 * c);
        e.store(partial + (long)p * hidden + 8 * c, hidden - 8 * c);
    }
}

// dg (+)= sum of the partial rows: 64 columns a workgroup, each of its 16 waves every sixteenth row, in a fixed order.  In 64 bits, of which the
// adds hide behind the loads: up to 47 roundings fewer.
__global__ __launch_bounds__(1024) void k_gain_sum(const float* __restrict__ partial, int parts, int hidden, float* dg, int accumulate) {
    __shared__ double part[16][64];
    const int share = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, col = (int)blockIdx.x * 64 + lane;
    double s = 0.0;
    if (col < hidden) {
        const float* at = partial + (long)share * hidden + col;
        const long step = 16L * hidden;
        int p = share;
        for (; p + 48 < parts; p += 64, at += 4 * step) {
            const double a = at[0], b = at[step], c = at[2 * step], d = at[3 * step];
            s += (a + b) + (c + d);
        }
        for (; p < parts; p += 16, at += step) s += *at;
    }
    part[share][lane] = s;
    __syncthreads();
    if (share == 0 && col < hidden) {
        s = accumulate ? dg[col] : 0.0;
#pragma unroll
        for (int i = 0; i < 16; i++) s += part[i][lane];
        dg[col] = (float)s;
    }
}

// Workgroups: two for each compute unit, with a row (four of them) each at least.  Fewer leave it waiting, more are more sums: of 256, 512 and
// 1024, 4096x12288 bf16 takes 103.9, 106.1, 115.4 us, 4096x8192 71.1, 69.1, 74.6, 8192x1003 37.1, 28.0, 27.1.
int add_norm_partial_rows(int rows, int hidden) { return std::min(hidden <= 1024 ? (rows + 3) / 4 : rows, 512); }

template <typename T>
static hipError_t bwd(const Drop& d, int rows, int hidden, float eps, const void* h, const void* g, const void* dxn, const void* dh, void* dx, void* db,
                      float* partial, hipStream_t st) {
    const int chunks = (hidden + 7) / 8, parts = add_norm_partial_rows(rows, hidden);
    const bool stream = (double)rows * hidden * sizeof(T) * (3 + (dh != nullptr) + (db != nullptr)) > STREAM_BYTES;
    auto run = [&](auto kern, int threads) {
        kern<<<parts, threads, 0, st>>>(d, rows, hidden, parts, eps, (const T*)h, (const T*)g, (const T*)dxn, (const T*)dh, (T*)dx, (T*)db, partial);
        return hipGetLastError();
    };
#define HH_SHAPE(W, CH) \
    if (chunks <= 64 * W * CH)                            \
        return run(hidden % 8 ? k_add_norm_bwd<T, W, CH, true, false> : stream ? k_add_norm_bwd<T, W, CH, false, true> : k_add_norm_bwd<T, W, CH, false, false>, \
                   row_threads<W>())
    HH_SHAPE(1, 1); HH_SHAPE(1, 2);
    HH_SHAPE(4, 1); HH_SHAPE(8, 1); HH_SHAPE(8, 2); HH_SHAPE(8, 3);
    if constexpr (sizeof(T) == 2) HH_SHAPE(8, 4);
#undef HH_SHAPE
    static std::atomic<uint64_t> lds_ok{0};
    const int lds = chunks * 32;
    const hipError_t e = allow_lds((const void*)&k_add_norm_bwd_wide<T>, 32768 * 4, lds_ok);
    if (e != hipSuccess) return e;
    k_add_norm_bwd_wide<T><<<parts, 1024, lds, st>>>(d, rows, hidden, parts, eps, (const T*)h, (const T*)g, (const T*)dxn, (const T*)dh, (T*)dx, (T*)db,
                                                     partial);
    return hipGetLastError();
}
hipError_t add_norm_bwd(int dtype, const Drop& d, int rows, int hidden, float eps, const void* h, const void* g, const void* dxn, const void* dh,
                        void* dx, void* db, float* dg, int accumulate, float* partial, hipStream_t st) {
    float* const to = dg ? partial : nullptr;
    const hipError_t e = dtype == DT_BF16 ? bwd<bf16_t>(d, rows, hidden, eps, h, g, dxn, dh, dx, db, to, st)
                                          : bwd<float>(d, rows, hidden, eps, h, g, dxn, dh, dx, db, to, st);
    if (e != hipSuccess || !dg) return e;
    k_gain_sum<<<(hidden + 63) / 64, 1024, 0, st>>>(partial, add_norm_partial_rows(rows, hidden), hidden, dg, accumulate);
    return hipGetLastError();
}

}  // namespace hh
