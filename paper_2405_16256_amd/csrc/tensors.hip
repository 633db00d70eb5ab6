// Kernels over a list of tensors of any sizes: the global gradient norm, clipped copies, the optimizer's update.
//
// The list travels in the kernel's arguments, so a launch needs no table in device memory, and a graph that records it keeps its
// own.  A workgroup takes a chunk of one tensor; which tensor a chunk belongs to is one comparison in each lane and a count of the
// lanes.  Bound by HBM: all loads of a whole chunk are under way before the first one is used.
#include <climits>
#include <type_traits>

#include "common.h"
#include "kernels.h"

namespace hh {

// Where the tensors of a list begin: the lane's own entries (INT_MAX past the last one); the tensor of chunk c.
template <typename List, int MAX>
struct Begins {
    static_assert(MAX <= 2 * WAVE, "two entries a lane");
    int first[MAX > WAVE ? 2 : 1];
    __device__ __forceinline__ explicit Begins(const List& l) {
        const int lane = threadIdx.x & 63;
        first[0] = lane < l.n ? l.t[lane].first : INT_MAX;
        if constexpr (MAX > WAVE) first[1] = lane + WAVE < l.n ? l.t[lane + WAVE].first : INT_MAX;
    }
    __device__ __forceinline__ int tensor_of(int c) const {
        int n = __popcll(__ballot(first[0] <= c));
        if constexpr (MAX > WAVE) n += __popcll(__ballot(first[1] <= c));
        return __builtin_amdgcn_readfirstlane(n - 1);
    }
};

// The elements of a chunk of CHUNK: [beg, end) in vectors of VN, beg aligned, and [s0, s1), [s2, s3) one by one.
template <int VN, int CHUNK>
struct Span {
    int64_t beg, end, s0, s1, s2, s3;
    __device__ __forceinline__ Span(int64_t count, int head, int64_t chunk) {
        const bool vectors = head >= 0;
        const int64_t lead = vectors ? (head < count ? head : count) : 0;
        const int64_t b = lead + chunk * CHUNK, e = b + CHUNK < count ? b + CHUNK : count;
        beg = b;
        end = vectors ? b + (e > b ? (e - b) / VN * VN : 0) : b;
        s0 = 0; s1 = chunk == 0 ? lead : 0;
        s2 = end; s3 = e;
    }
    // vectors(i, whole): i = the thread's first element, whole: it has PER of them, 256 VN apart; one(i): a single element.
    static constexpr int PER = CHUNK / (256 * VN);
    template <typename V, typename S>
    __device__ __forceinline__ void walk(V vectors, S single) const {
        const int64_t i = beg + (int)threadIdx.x * VN;
        if (end - beg == CHUNK) vectors(i, std::integral_constant<int, PER>{});
        else
            for (int64_t j = i; j < end; j += 256 * VN) vectors(j, std::integral_constant<int, 1>{});
        for (int64_t j = s0 + (int)threadIdx.x; j < s1; j += 256) single(j);
        for (int64_t j = s2 + (int)threadIdx.x; j < s3; j += 256) single(j);
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
__device__ __forceinline__ double squares(const T* g, int64_t count, int head, int64_t chunk) {
    constexpr int VN = Vec<T>::N;
    double acc = 0.0;
    Span<VN, CLIP_CHUNK>(count, head, chunk).walk(
        [&](int64_t i, auto per) {
            typename Vec<T>::Raw raw[decltype(per)::value];
#pragma unroll
            for (int k = 0; k < decltype(per)::value; k++) raw[k] = Vec<T>::raw(g + i + k * 256 * VN);
#pragma unroll
            for (int k = 0; k < decltype(per)::value; k++) {
                float f[VN];
                Vec<T>::widen(raw[k], f);
#pragma unroll
                for (int e = 0; e < VN; e++) acc = fma((double)f[e], (double)f[e], acc);
            }
        },
        [&](int64_t i) { const double v = one(g + i); acc = fma(v, v, acc); });
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

// 1024 workgroups at most, each with a sum of its own, added in the order of the slots by whoever needs it.  202 million fp32 gradients: 127
// us, 6.4 TB/s.
__global__ __launch_bounds__(256) void k_clip_squares(ClipList l, double* __restrict__ slots, int add) {
    __shared__ double red[4];
    const Begins<ClipList, CLIP_LIST> begins(l);
    double acc = 0.0;
    for (int c = (int)blockIdx.x; c < l.chunks; c += (int)gridDim.x) {
        const ClipItem& t = l.t[begins.tensor_of(c)];
        if (t.bf16) acc += squares((const bf16_t*)t.g, t.count, t.head, c - t.first);
        else acc += squares((const float*)t.g, t.count, t.head, c - t.first);
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

// Past the caches: nothing reads these lines again soon, and what the stores would push out may still be read.
__device__ __forceinline__ void store_past(float* p, const float* f) { __builtin_nontemporal_store(f32x4{f[0], f[1], f[2], f[3]}, (f32x4*)p); }
__device__ __forceinline__ void store_past(bf16_t* p, const float* f) {
    const i32x4 v = {(int)pack_bf2(f[0], f[1]), (int)pack_bf2(f[2], f[3]), (int)pack_bf2(f[4], f[5]), (int)pack_bf2(f[6], f[7])};
    __builtin_nontemporal_store(v, (i32x4*)p);
}

template <typename T>
__device__ __forceinline__ void scaled(const T* g, T* out, float factor, int64_t count, int head, int64_t chunk) {
    constexpr int VN = Vec<T>::N;
    Span<VN, CLIP_CHUNK>(count, head, chunk).walk(
        [&](int64_t i, auto per) {
            typename Vec<T>::Raw raw[decltype(per)::value];
#pragma unroll
            for (int k = 0; k < decltype(per)::value; k++) raw[k] = Vec<T>::raw(g + i + k * 256 * VN);
#pragma unroll
            for (int k = 0; k < decltype(per)::value; k++) {
                float f[VN];
                Vec<T>::widen(raw[k], f);
#pragma unroll
                for (int e = 0; e < VN; e++) f[e] *= factor;
                store_past(out + i + k * 256 * VN, f);
            }
        },
        [&](int64_t i) { put(out + i, one(g + i) * factor); });
}

// A workgroup a chunk, in the opposite order of k_clip_squares: what that one read last is still in the last-level cache.  Eight
// neighbouring workgroups, which go to the eight XCDs in turn, keep their order, so that a chunk goes to the XCD whose L2 has
// read it.  202 million fp32 gradients, 455 us for both kernels before: with stores past the caches 434, in this order 420, a
// workgroup a chunk instead of 2048 workgroups 396.
__global__ __launch_bounds__(256) void k_clip_scale(ClipList l, const double* __restrict__ slots, int n_slots, float max_norm, float* __restrict__ result) {
    __shared__ double red[4];
    const float2 r = norm_and_factor(slots, n_slots, max_norm, red);
    if (result && blockIdx.x == 0 && threadIdx.x == 0) { result[0] = r.x; result[1] = r.y; }
    const Begins<ClipList, CLIP_LIST> begins(l);
    const int c = ((int)(gridDim.x >> 3) - 1 - (int)(blockIdx.x >> 3)) * 8 + (int)(blockIdx.x & 7);
    if (c >= l.chunks) return;
    const ClipItem& t = l.t[begins.tensor_of(c)];
    if (!t.out) return;
    if (t.bf16) scaled((const bf16_t*)t.g, (bf16_t*)t.out, r.y, t.count, t.head, c - t.first);
    else scaled((const float*)t.g, (float*)t.out, r.y, t.count, t.head, c - t.first);
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
    k_clip_scale<<<(l.chunks + 7) / 8 * 8, 256, 0, st>>>(l, slots, n_slots, max_norm, result);
    return hipGetLastError();
}

// ------------------------------------------------------------------ update
// One element.  Divisions and the root are IEEE ones: the kernel waits for memory all the same.
__device__ __forceinline__ void adamw_one(float g, float& p, float& m, float& v, const AdamwHyper& h, float keep) {
    m = fmaf(h.beta1, m, h.rest1 * g);
    v = fmaf(h.beta2, v, h.rest2 * g * g);
    p = fmaf(keep, p, -(h.step_size * m / (sqrtf(v) * h.inv_sqrt_bc2 + h.eps)));
}

template <bool PAST>
__device__ __forceinline__ void load4(const float* p, float (&f)[4]) {
    const f32x4 v = PAST ? __builtin_nontemporal_load((const f32x4*)p) : *(const f32x4*)p;
#pragma unroll
    for (int e = 0; e < 4; e++) f[e] = v[e];
}
template <bool PAST>
__device__ __forceinline__ void load4(const bf16_t* p, float (&f)[4]) {
    const i32x2 v = PAST ? __builtin_nontemporal_load((const i32x2*)p) : *(const i32x2*)p;
    f[0] = lo_bf((uint32_t)v[0]); f[1] = hi_bf((uint32_t)v[0]); f[2] = lo_bf((uint32_t)v[1]); f[3] = hi_bf((uint32_t)v[1]);
}
template <bool PAST>
__device__ __forceinline__ void store4(float* p, const float (&f)[4]) {
    const f32x4 v = {f[0], f[1], f[2], f[3]};
    if (PAST) __builtin_nontemporal_store(v, (f32x4*)p);
    else *(f32x4*)p = v;
}
template <bool PAST>
__device__ __forceinline__ void store4(bf16_t* p, const float (&f)[4]) {
    const i32x2 v = {(int)pack_bf2(f[0], f[1]), (int)pack_bf2(f[2], f[3])};
    if (PAST) __builtin_nontemporal_store(v, (i32x2*)p);
    else *(i32x2*)p = v;
}

template <bool PBF, bool GBF, bool PAST>
__device__ __forceinline__ void update(const AdamwItem& t, const AdamwHyper& h, float factor, int64_t chunk) {
    typedef typename std::conditional<GBF, bf16_t, float>::type G;
    float* const p = PBF ? t.master : (float*)t.param;
    bf16_t* const pb = (bf16_t*)t.param;
    float *const m = t.m, *const v = t.v;
    const G* const g = (const G*)t.g;
    const float keep = t.keep;
    Span<4, ADAMW_CHUNK>(t.count, t.head, chunk).walk(
        [&](int64_t i, auto per) {
            constexpr int PER = decltype(per)::value;
            float pv[PER][4], mv[PER][4], vv[PER][4], gv[PER][4];
#pragma unroll
            for (int k = 0; k < PER; k++) {
                const int64_t at = i + k * 1024;
                load4<PAST>(g + at, gv[k]); load4<PAST>(p + at, pv[k]); load4<PAST>(m + at, mv[k]); load4<PAST>(v + at, vv[k]);
            }
#pragma unroll
            for (int k = 0; k < PER; k++) {
                const int64_t at = i + k * 1024;
#pragma unroll
                for (int e = 0; e < 4; e++) adamw_one(gv[k][e] * factor, pv[k][e], mv[k][e], vv[k][e], h, keep);
                store4<PAST>(p + at, pv[k]); store4<PAST>(m + at, mv[k]); store4<PAST>(v + at, vv[k]);
                if (PBF) store4<PAST>(pb + at, pv[k]);
            }
        },
        [&](int64_t i) {
            float pv = p[i], mv = m[i], vv = v[i];
            adamw_one(one(g + i) * factor, pv, mv, vv, h, keep);
            p[i] = pv; m[i] = mv; v[i] = vv;
            if (PBF) put(pb + i, pv);
        });
}

// PAST: where the tensors do not fit the last-level cache, loads and stores go past the caches.  103 million elements 572 -> 485 us, 202
// million 1136 -> 1099 (5.6 TB/s); 3.2 million, which do fit, would take 18.7 instead of 16.3.
template <bool PAST>
__global__ __launch_bounds__(256) void k_adamw(AdamwList l, AdamwHyper h, const float* __restrict__ factor) {
    const float f = factor ? *factor : 1.f;
    if (!(fabsf(f) < INFINITY)) return;   // gradients that are not finite: nothing changes
    const Begins<AdamwList, ADAMW_LIST> begins(l);
    const int c = (int)blockIdx.x;
    const AdamwItem& t = l.t[begins.tensor_of(c)];
    const int64_t chunk = c - t.first;
    if (t.param_bf16) {
        if (t.grad_bf16) update<true, true, PAST>(t, h, f, chunk);
        else update<true, false, PAST>(t, h, f, chunk);
    } else {
        if (t.grad_bf16) update<false, true, PAST>(t, h, f, chunk);
        else update<false, false, PAST>(t, h, f, chunk);
    }
}

hipError_t adamw(const AdamwList& l, const AdamwHyper& h, const float* factor, bool stream, hipStream_t st) {
    if (stream) k_adamw<true><<<l.chunks, 256, 0, st>>>(l, h, factor);
    else k_adamw<false><<<l.chunks, 256, 0, st>>>(l, h, factor);
    return hipGetLastError();
}

}  // namespace hh
