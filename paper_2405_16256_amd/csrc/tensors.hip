// Kernels over a list of tensors of any sizes: the global gradient norm, clipped copies, the optimizer's update.
//
// The list travels in the kernel's arguments, so a launch needs no table in device memory, and a graph that records it keeps its
// own.  Workgroups stride over chunks of LIST_CHUNK elements of all tensors; which tensor a chunk belongs to is one comparison in each lane
// and a count of the lanes.  Bound by HBM.
#include <climits>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace hh {

// The tensor of chunk c: `first` is the lane's own entry (INT_MAX past the last tensor).
__device__ __forceinline__ int tensor_of(int c, int first) {
    return __builtin_amdgcn_readfirstlane(__popcll(__ballot(first <= c)) - 1);
}

// The elements of a chunk: [beg, end) in vectors of VN, beg aligned, and [s0, s1), [s2, s3) one by one.
template <int VN>
struct Span {
    int64_t beg, end, s0, s1, s2, s3;
    __device__ __forceinline__ Span(int64_t count, int head, int64_t chunk) {
        const bool vectors = head >= 0;
        const int64_t lead = vectors ? (head < count ? head : count) : 0;
        const int64_t b = lead + chunk * LIST_CHUNK, e = b + LIST_CHUNK < count ? b + LIST_CHUNK : count;
        beg = b;
        end = vectors ? b + (e > b ? (e - b) / VN * VN : 0) : b;
        s0 = 0; s1 = chunk == 0 ? lead : 0;
        s2 = end; s3 = e;
    }
};

// ------------------------------------------------------------------ squares
template <typename T>
__device__ __forceinline__ float one(const T* p);
template <>
__device__ __forceinline__ float one(const float* p) { return *p; }
template <>
__device__ __forceinline__ float one(const bf16_t* p) { return bf2f(*p); }
__device__ __forceinline__ void put(float* p, float v) { *p = v; }
__device__ __forceinline__ void put(bf16_t* p, float v) { *p = f2bf(v); }

template <typename T>
__device__ __forceinline__ double squares(const T* g, const Span<Vec<T>::N>& s) {
    constexpr int VN = Vec<T>::N;
    double acc = 0.0;
    for (int64_t i = s.beg + (int)threadIdx.x * VN; i < s.end; i += 256 * VN) {
        float f[VN];
        Vec<T>::load(g + i, f);
#pragma unroll
        for (int e = 0; e < VN; e++) acc = fma((double)f[e], (double)f[e], acc);
    }
    for (int64_t i = s.s0 + (int)threadIdx.x; i < s.s1; i += 256) { const double v = one(g + i); acc = fma(v, v, acc); }
    for (int64_t i = s.s2 + (int)threadIdx.x; i < s.s3; i += 256) { const double v = one(g + i); acc = fma(v, v, acc); }
    return acc;
}

// sum over the workgroup's 4 waves, in every thread
__device__ __forceinline__ double block_sum_f64(double v, double* red) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, WAVE);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
    __syncthreads();
    return (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(256) void k_clip_squares(ClipList l, double* __restrict__ slots, int add) {
    __shared__ double red[4];
    const int lane = threadIdx.x & 63, first = lane < l.n ? l.t[lane].first : INT_MAX;
    double acc = 0.0;
    for (int c = (int)blockIdx.x; c < l.chunks; c += (int)gridDim.x) {
        const ClipItem& t = l.t[tensor_of(c, first)];
        if (t.bf16) acc += squares((const bf16_t*)t.g, Span<8>(t.count, t.head, c - t.first));
        else acc += squares((const float*)t.g, Span<4>(t.count, t.head, c - t.first));
    }
    acc = block_sum_f64(acc, red);
    if (threadIdx.x == 0) slots[blockIdx.x] = add ? slots[blockIdx.x] + acc : acc;
}

// Norm and factor from the sums of the slots, the same in every workgroup that forms them.
__device__ __forceinline__ float2 norm_and_factor(const double* __restrict__ slots, int n, float max_norm, double* red) {
    double acc = 0.0;
    for (int i = (int)threadIdx.x; i < n; i += 256) acc += slots[i];
    const float norm = (float)sqrt(block_sum_f64(acc, red));
    const float factor = max_norm / (norm + 1e-6f);
    return make_float2(norm, norm < INFINITY ? fminf(factor, 1.f) : __builtin_nanf(""));
}

__global__ __launch_bounds__(256) void k_clip_result(const double* __restrict__ slots, int n_slots, float max_norm, float* __restrict__ result) {
    __shared__ double red[4];
    const float2 r = norm_and_factor(slots, n_slots, max_norm, red);
    if (threadIdx.x == 0) { result[0] = r.x; result[1] = r.y; }
}

template <typename T>
__device__ __forceinline__ void scaled(const T* g, T* out, float f, const Span<Vec<T>::N>& s) {
    constexpr int VN = Vec<T>::N;
    for (int64_t i = s.beg + (int)threadIdx.x * VN; i < s.end; i += 256 * VN) {
        float v[VN];
        Vec<T>::load(g + i, v);
#pragma unroll
        for (int e = 0; e < VN; e++) v[e] *= f;
        Vec<T>::store(out + i, v);
    }
    for (int64_t i = s.s0 + (int)threadIdx.x; i < s.s1; i += 256) put(out + i, one(g + i) * f);
    for (int64_t i = s.s2 + (int)threadIdx.x; i < s.s3; i += 256) put(out + i, one(g + i) * f);
}

__global__ __launch_bounds__(256) void k_clip_scale(ClipList l, const double* __restrict__ slots, int n_slots, float max_norm, float* __restrict__ result) {
    __shared__ double red[4];
    const float2 r = norm_and_factor(slots, n_slots, max_norm, red);
    if (result && blockIdx.x == 0 && threadIdx.x == 0) { result[0] = r.x; result[1] = r.y; }
    const int lane = threadIdx.x & 63, first = lane < l.n ? l.t[lane].first : INT_MAX;
    for (int c = (int)blockIdx.x; c < l.chunks; c += (int)gridDim.x) {
        const ClipItem& t = l.t[tensor_of(c, first)];
        if (!t.out) continue;
        if (t.bf16) scaled((const bf16_t*)t.g, (bf16_t*)t.out, r.y, Span<8>(t.count, t.head, c - t.first));
        else scaled((const float*)t.g, (float*)t.out, r.y, Span<4>(t.count, t.head, c - t.first));
    }
}

hipError_t clip_squares(const ClipList& l, double* slots, int wgs, int add, hipStream_t st) {
    if (wgs < 1 || wgs > CLIP_SLOTS) return hipErrorInvalidValue;
    k_clip_squares<<<wgs, 256, 0, st>>>(l, slots, add);
    return hipGetLastError();
}
hipError_t clip_result(const double* slots, int n_slots, float max_norm, float* result, hipStream_t st) {
    k_clip_result<<<1, 256, 0, st>>>(slots, n_slots, max_norm, result);
    return hipGetLastError();
}
hipError_t clip_scale(const ClipList& l, const double* slots, int n_slots, float max_norm, float* result, hipStream_t st) {
    k_clip_scale<<<l.chunks < 2048 ? l.chunks : 2048, 256, 0, st>>>(l, slots, n_slots, max_norm, result);
    return hipGetLastError();
}

// ------------------------------------------------------------------ update
// One element.  Divisions and the root are IEEE ones: the kernel waits for memory all the same.
__device__ __forceinline__ void adamw_one(float g, float& p, float& m, float& v, const AdamwHyper& h, float keep) {
    m = fmaf(h.beta1, m, h.rest1 * g);
    v = fmaf(h.beta2, v, h.rest2 * g * g);
    p = fmaf(keep, p, -(h.step_size * m / (sqrtf(v) * h.inv_sqrt_bc2 + h.eps)));
}

template <bool PBF, bool GBF>
__device__ __forceinline__ void update(const AdamwItem& t, const AdamwHyper& h, float factor, int64_t chunk) {
    typedef typename std::conditional<GBF, bf16_t, float>::type G;
    const Span<4> s(t.count, t.head, chunk);
    float* const p = PBF ? t.master : (float*)t.param;
    bf16_t* const pb = (bf16_t*)t.param;
    const G* const g = (const G*)t.g;
    const float keep = t.keep;
    for (int64_t i = s.beg + (int)threadIdx.x * 4; i < s.end; i += 1024) {
        float pv[4], mv[4], vv[4], gv[4];
        if (GBF) {
            const uint2 u = *reinterpret_cast<const uint2*>(g + i);
            gv[0] = lo_bf(u.x); gv[1] = hi_bf(u.x); gv[2] = lo_bf(u.y); gv[3] = hi_bf(u.y);
        } else {
            Vec<float>::load((const float*)g + i, gv);
        }
        Vec<float>::load(p + i, pv); Vec<float>::load(t.m + i, mv); Vec<float>::load(t.v + i, vv);
#pragma unroll
        for (int e = 0; e < 4; e++) adamw_one(gv[e] * factor, pv[e], mv[e], vv[e], h, keep);
        Vec<float>::store(p + i, pv); Vec<float>::store(t.m + i, mv); Vec<float>::store(t.v + i, vv);
        if (PBF) *reinterpret_cast<uint2*>(pb + i) = make_uint2(pack_bf2(pv[0], pv[1]), pack_bf2(pv[2], pv[3]));
    }
    auto single = [&](int64_t i) {
        float pv = p[i], mv = t.m[i], vv = t.v[i];
        adamw_one(one(g + i) * factor, pv, mv, vv, h, keep);
        p[i] = pv; t.m[i] = mv; t.v[i] = vv;
        if (PBF) put(pb + i, pv);
    };
    for (int64_t i = s.s0 + (int)threadIdx.x; i < s.s1; i += 256) single(i);
    for (int64_t i = s.s2 + (int)threadIdx.x; i < s.s3; i += 256) single(i);
}

__global__ __launch_bounds__(256) void k_adamw(AdamwList l, AdamwHyper h, const float* __restrict__ factor) {
    const float f = factor ? *factor : 1.f;
    if (!(fabsf(f) < INFINITY)) return;   // gradients that are not finite: nothing changes
    const int lane = threadIdx.x & 63, first = lane < l.n ? l.t[lane].first : INT_MAX;
    for (int c = (int)blockIdx.x; c < l.chunks; c += (int)gridDim.x) {
        const AdamwItem& t = l.t[tensor_of(c, first)];
        const int64_t chunk = c - t.first;
        if (t.param_bf16) {
            if (t.grad_bf16) update<true, true>(t, h, f, chunk);
            else update<true, false>(t, h, f, chunk);
        } else {
            if (t.grad_bf16) update<false, true>(t, h, f, chunk);
            else update<false, false>(t, h, f, chunk);
        }
    }
}

hipError_t adamw(const AdamwList& l, const AdamwHyper& h, const float* factor, hipStream_t st) {
    k_adamw<<<l.chunks < 2048 ? l.chunks : 2048, 256, 0, st>>>(l, h, factor);
    return hipGetLastError();
}

}  // namespace hh
