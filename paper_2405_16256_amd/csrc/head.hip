// Softmax cross entropy over a vocabulary: what comes between the product that forms the scores and the two that take their
// gradient.
//
// Row t of z has the statistics (largest score, sum of exponentials) of each slot of its columns.  k_head_rows puts them together,
//     m = max_s m_s,  S = sum_s S_s exp(m_s - m),  loss = log S + (m - z_t,label),
// and k_head_grad reads the scores once and writes d_tv = g_t (exp(z_tv - m) / S - [v = label(t)]).  All of it in fp32.  m and S stay
// two numbers: their one, m + log S, has the ulp of a score, which would be the relative error of all of a row's p and the
// absolute one of its loss (scores around 1000: 3e-5).  Shares of a vocabulary, which have only that one from outside, are off by it.
#include "common.h"
#include "kernels.h"

namespace hh {

constexpr float LOG2_E = 1.4426950408889634f;

// (m, s) and (m1, s1) as one; -inf with 0 is nothing
__device__ __forceinline__ void join(float& m, float& s, float m1, float s1) {
    const float top = fmaxf(m, m1), ref = top == -INFINITY ? 0.f : top;
    s = s * __builtin_amdgcn_exp2f((m - ref) * LOG2_E) + s1 * __builtin_amdgcn_exp2f((m1 - ref) * LOG2_E);
    m = top;
}

// d = hi + lo (bf16, two rows) or d itself (fp32) of 4 columns
__device__ __forceinline__ void put_d(bf16_t* hi_row, bf16_t* lo_row, uint32_t col, const float (&f)[4]) {
    const uint2 hi = make_uint2(pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3]));
    *reinterpret_cast<uint2*>(hi_row + col) = hi;
    *reinterpret_cast<uint2*>(lo_row + col) = make_uint2(pack_bf2(f[0] - lo_bf(hi.x), f[1] - hi_bf(hi.x)), pack_bf2(f[2] - lo_bf(hi.y), f[3] - hi_bf(hi.y)));
}
__device__ __forceinline__ void put_d(float* row, float*, uint32_t col, const float (&f)[4]) { Vec<float>::store(row + col, f); }
// A vector of a token's row of x, zeros where it does not count (zero times NaN would be NaN in dW): for bf16 beside lo as well, so that
// d^T x is one product over hi's rows and lo's.
template <typename T>
__device__ __forceinline__ void put_x(const T* __restrict__ x, T* __restrict__ xs, int row, int lo_rows, int H, int col, bool counts) {
    typename Vec<T>::Raw v{};
    if (counts) v = Vec<T>::raw(x + (size_t)row * H + col);
    *reinterpret_cast<typename Vec<T>::Raw*>(xs + (size_t)row * H + col) = v;
    if (sizeof(T) == 2) *reinterpret_cast<typename Vec<T>::Raw*>(xs + (size_t)(row + lo_rows) * H + col) = v;
}

// ------------------------------------------------------------------ whole rows
// All scores of a row in the registers of one workgroup: read once for the largest, the sum, the loss and d.  Bound by HBM
// (8 bytes a score in a step), by launches on small problems, of which it is one where the statistics and d apart are two, in fp32
// three (head steps of fp32 128 tokens, hidden 256, vocabulary 1000: 25.7 -> 18.1 us; 700, 1024, 8001: 317 -> 308; 700, 512, 30000: 598 -> 584;
// bf16 200, 512, 2000: 24.6 -> 22.0; 700, 512, 8191: 56.9 -> 53.7).  In bf16, whose statistics come with the product, it gains nothing
// between 8192 and 16384 columns (700 tokens, 512, 16384: 99.3 -> 99.0; 8192 tokens: 837 -> 864) and loses past that: a workgroup of 1024
// threads with 32 scores each has a CU to itself, and nothing is stored while it loads (2048 rows of 32000: 95 us apart, 114 whole).
template <typename T, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void k_head_row(HeadTokens t, const float* z, int ldz, float* __restrict__ loss, T* d, int lo_rows,
                                                      const T* __restrict__ x, T* __restrict__ xs, int H) {
    const int N = t.N;
    constexpr int NW = THREADS / WAVE;
    __shared__ float red[2 * NW];
    const int row = (int)blockIdx.x, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    const int64_t named = t.labels[row];
    const bool counts = named >= 0 && named < N;
    const int label = counts ? (int)named : -1;
    if (d)
        for (int col = (int)threadIdx.x * Vec<T>::N; col < H; col += THREADS * Vec<T>::N) put_x(x, xs, row, lo_rows, H, col, counts);
    T* const hi_row = d + (size_t)row * ldz;
    T* const lo_row = d + (size_t)(row + lo_rows) * ldz;
    z += (size_t)row * ldz;
    float f[NV][4];
    if (!counts) {
        if (threadIdx.x == 0) loss[row] = named < 0 ? 0.f : __builtin_nanf("");
        if (!d) return;
#pragma unroll
        for (int e = 0; e < 4; e++) f[0][e] = 0.f;
#pragma unroll
        for (int k = 0; k < NV; k++) {
            const int col = 4 * (k * THREADS + (int)threadIdx.x);
            if (col < ldz) put_d(hi_row, lo_row, (uint32_t)col, f[0]);
        }
        return;
    }
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < NV; k++) {
        const int col = 4 * (k * THREADS + (int)threadIdx.x);
#pragma unroll
        for (int e = 0; e < 4; e++) f[k][e] = -INFINITY;
        if (col < N) Vec<float>::load(z + (uint32_t)col, f[k]);   // rows are padded
    }
#pragma unroll
    for (int k = 0; k < NV; k++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if (4 * (k * THREADS + (int)threadIdx.x) + e >= N) f[k][e] = -INFINITY;
            top = fmaxf(top, f[k][e]);
        }
    top = wave_max(top);
    if (lane == 0) red[wave] = top;
    __syncthreads();
    top = red[0];
#pragma unroll
    for (int w = 1; w < NW; w++) top = fmaxf(top, red[w]);
    float sum = 0.f, mine = 0.f;
#pragma unroll
    for (int k = 0; k < NV; k++)
#pragma unroll
        for (int e = 0; e < 4; e++) {
            if (label == 4 * (k * THREADS + (int)threadIdx.x) + e) mine = f[k][e];
            f[k][e] = __builtin_amdgcn_exp2f((f[k][e] - top) * LOG2_E);
            sum += f[k][e];
        }
    sum = wave_sum(sum);
    if (lane == 0) red[NW + wave] = sum;
    __syncthreads();
    sum = red[NW];
#pragma unroll
    for (int w = 1; w < NW; w++) sum += red[NW + w];
    if ((int)threadIdx.x == (label >> 2) % THREADS) loss[row] = logf(sum) + (top - mine);
    if (!d) return;
    const float g = t.dloss ? t.scale * t.dloss[row] : t.scale, inv = 1.f / sum;
#pragma unroll
    for (int k = 0; k < NV; k++) {
        const int col = 4 * (k * THREADS + (int)threadIdx.x);
        if (col >= ldz) continue;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float p = f[k][e] * inv;
            f[k][e] = col + e < N ? g * (label == col + e ? p - 1.f : p) : 0.f;
        }
        put_d(hi_row, lo_row, (uint32_t)col, f[k]);
    }
}

template <typename T>
static void launch_row(const HeadTokens& t, const float* z, int ldz, float* loss, T* d, int lo_rows, const T* x, T* xs, int H, hipStream_t st) {
    if (ldz <= 1024) k_head_row<T, 256, 1><<<t.M, 256, 0, st>>>(t, z, ldz, loss, d, lo_rows, x, xs, H);
    else if (ldz <= 4096) k_head_row<T, 256, 4><<<t.M, 256, 0, st>>>(t, z, ldz, loss, d, lo_rows, x, xs, H);
    else if (ldz <= 8192) k_head_row<T, 512, 4><<<t.M, 512, 0, st>>>(t, z, ldz, loss, d, lo_rows, x, xs, H);
    else if (ldz <= 16384) k_head_row<T, 1024, 4><<<t.M, 1024, 0, st>>>(t, z, ldz, loss, d, lo_rows, x, xs, H);
    else if constexpr (sizeof(T) == 4) k_head_row<T, 1024, 8><<<t.M, 1024, 0, st>>>(t, z, ldz, loss, d, lo_rows, x, xs, H);
}
hipError_t head_row(int dtype, const HeadTokens& t, const float* z, int ldz, float* loss, void* d, int lo_rows, const void* x, void* xs, int H,
                    hipStream_t st) {
    if (ldz > head_row_most(dtype) || t.first || t.limit != t.N) return hipErrorInvalidValue;
    if (dtype == DT_BF16) launch_row(t, z, ldz, loss, (bf16_t*)d, lo_rows, (const bf16_t*)x, (bf16_t*)xs, H, st);
    else launch_row(t, z, ldz, loss, (float*)d, lo_rows, (const float*)x, (float*)xs, H, st);
    return hipGetLastError();
}

// ------------------------------------------------------------------ statistics of fp32 scores
// A workgroup reads HEAD_F32_SLOT columns of one row.  (In bf16 the product's own epilogue forms them.)
__global__ __launch_bounds__(256) void k_head_stats(HeadTokens t, const float* __restrict__ z, int ldz, float2* __restrict__ stats) {
    const int M = t.M, N = t.N;
    const int row = (int)blockIdx.y, slot = (int)blockIdx.x, col = slot * HEAD_F32_SLOT + 4 * (int)threadIdx.x;
    float f[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
    if (col < N) {
        Vec<float>::load(z + (size_t)row * ldz + col, f);   // rows are padded
#pragma unroll
        for (int e = 0; e < 4; e++)
            if (col + e >= N) f[e] = -INFINITY;
    }
    const int64_t label = t.labels[row] - t.first;
    if (label >= col && label < col + 4 && label < N)
        ((float*)(stats + (size_t)gridDim.x * M))[row] = label == col ? f[0] : label == col + 1 ? f[1] : label == col + 2 ? f[2] : f[3];
    __shared__ float red[8];
    float top = wave_max(fmaxf(fmaxf(f[0], f[1]), fmaxf(f[2], f[3])));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = top;
    __syncthreads();
    top = fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
    const float ref = top == -INFINITY ? 0.f : top;
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < 4; e++) sum += __builtin_amdgcn_exp2f((f[e] - ref) * LOG2_E);
    sum = block_sum<4>(sum, red + 4);
    if (threadIdx.x == 0) stats[(size_t)slot * M + row] = make_float2(top, sum);
}

hipError_t head_stats_f32(const HeadTokens& t, const float* z, int ldz, float2* stats, hipStream_t st) {
    k_head_stats<<<dim3((t.N + HEAD_F32_SLOT - 1) / HEAD_F32_SLOT, t.M), 256, 0, st>>>(t, z, ldz, stats);
    return hipGetLastError();
}

// ------------------------------------------------------------------ rows
// 4 rows a workgroup, 64 threads a row: the rows' statistics of a slot are 32 bytes, and there are workgroups for every CU from 1024
// tokens on.  Bound by latency: 700 tokens, 782 slots 5.9 us (8.9 with 16 rows of 64 threads), 333 tokens, 1563 slots 7.0 (13.8).
constexpr int ROWS_WG = 4;
__global__ __launch_bounds__(256) void k_head_rows(HeadTokens t, const float2* __restrict__ stats, int slots, float* __restrict__ loss,
                                                   float* __restrict__ lse_out, float2* __restrict__ norm_out, float* __restrict__ picked_out) {
    const int M = t.M;
    __shared__ float2 part[4][ROWS_WG];
    const int r = threadIdx.x & (ROWS_WG - 1), row = (int)blockIdx.x * ROWS_WG + r, from = threadIdx.x / ROWS_WG;
    float m = -INFINITY, s = 0.f;
    if (row < M) {
#pragma unroll 4
        for (int i = from; i < slots; i += 256 / ROWS_WG) {
            const float2 v = stats[(size_t)i * M + row];
            join(m, s, v.x, v.y);
        }
    }
#pragma unroll
    for (int o = ROWS_WG; o < 64; o <<= 1) {
        const float m1 = __shfl_xor(m, o, WAVE), s1 = __shfl_xor(s, o, WAVE);
        join(m, s, m1, s1);
    }
    if ((threadIdx.x & 63) < ROWS_WG) part[threadIdx.x >> 6][r] = make_float2(m, s);
    __syncthreads();
    if (threadIdx.x >= ROWS_WG || row >= M) return;
    m = part[0][r].x; s = part[0][r].y;
#pragma unroll
    for (int w = 1; w < 4; w++) join(m, s, part[w][r].x, part[w][r].y);
    const float log_s = logf(s);
    const int64_t label = t.labels[row], column = label - t.first;
    const float picked = column >= 0 && column < t.N ? ((const float*)(stats + (size_t)slots * M))[row] : 0.f;
    if (loss) loss[row] = label < 0 ? 0.f : label < t.limit ? log_s + (m - picked) : __builtin_nanf("");
    if (lse_out) lse_out[row] = m + log_s;
    if (norm_out) norm_out[row] = make_float2(m, 1.f / s);
    if (picked_out) picked_out[row] = label < 0 ? 0.f : picked;
}

hipError_t head_rows(const HeadTokens& t, const float2* stats, int slots, float* loss, float* lse, float2* norm, float* picked, hipStream_t st) {
    k_head_rows<<<(t.M + ROWS_WG - 1) / ROWS_WG, 256, 0, st>>>(t, stats, slots, loss, lse, norm, picked);
    return hipGetLastError();
}

// ------------------------------------------------------------------ gradient of the scores
// Of longer rows.  Bound by HBM: 2048 rows of 32000 86 us, 6.1 TB/s of scores in and d out.  A workgroup turns 1024 scores of a
// row into d; columns N .. ldz-1 become zeros, and so do rows that do not count, whatever their scores are.  The workgroups past
// those of the scores copy the row's x.  p = exp(z - m) / S from norm, exp(z - lse) where that is null.  The scores are asked for, 16
// bytes a lane, in front of what the row has in common: left to the compiler they wait for it, in three pieces (101 us).
template <typename T>
__global__ __launch_bounds__(256) void k_head_grad(HeadTokens t, const float* z, int ldz, const float2* __restrict__ norm, const float* __restrict__ lse,
                                                   T* d, int lo_rows, const T* __restrict__ x, T* __restrict__ xs, int H, int z_wgs) {
    constexpr int PER = 1024;
    const int row = (int)blockIdx.y;
    const int64_t label = t.labels[row];
    const bool counts = label >= 0 && label < t.limit;
    if ((int)blockIdx.x >= z_wgs) {
        constexpr int VN = Vec<T>::N;
        const int col = ((int)blockIdx.x - z_wgs) * (256 * VN) + VN * (int)threadIdx.x;
        if (col < H) put_x(x, xs, row, lo_rows, H, col, counts);
        return;
    }
    const int col = (int)blockIdx.x * PER + 4 * (int)threadIdx.x;
    if (col >= ldz) return;
    float f[4] = {0.f, 0.f, 0.f, 0.f};
    if (counts && col < t.N) {
        Vec<float>::load(z + (size_t)row * ldz + col, f);
        __builtin_amdgcn_sched_barrier(0);
        const float2 of = norm ? norm[row] : make_float2(lse[row], 1.f);
        const float g = t.dloss ? t.scale * t.dloss[row] : t.scale;
        const int64_t column = label - t.first;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const float p = __builtin_amdgcn_exp2f((f[e] - of.x) * LOG2_E) * of.y;
            f[e] = col + e < t.N ? g * (column == col + e ? p - 1.f : p) : 0.f;
        }
    }
    put_d(d + (size_t)row * ldz, d + (size_t)(row + lo_rows) * ldz, (uint32_t)col, f);
}

hipError_t head_grad(int dtype, const HeadTokens& t, const float* z, int ldz, const float2* norm, const float* lse, void* d, int lo_rows, const void* x,
                     void* xs, int H, hipStream_t st) {
    const int z_wgs = (ldz + 1023) / 1024;
    if (dtype == DT_BF16)
        k_head_grad<bf16_t><<<dim3(z_wgs + (H + 2047) / 2048, t.M), 256, 0, st>>>(t, z, ldz, norm, lse, (bf16_t*)d, lo_rows, (const bf16_t*)x,
                                                                                         (bf16_t*)xs, H, z_wgs);
    else
        k_head_grad<float><<<dim3(z_wgs + (H + 1023) / 1024, t.M), 256, 0, st>>>(t, z, ldz, norm, lse, (float*)d, lo_rows, (const float*)x, (float*)xs, H,
                                                                                        z_wgs);
    return hipGetLastError();
}

}  // namespace hh
