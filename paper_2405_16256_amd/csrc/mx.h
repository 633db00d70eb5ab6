// Device helpers of the residual path and of the microscaled formats: the counter-based generator, packing of eight values, loads and
// stores of rows at any alignment.
#pragma once
#include "common.h"
#include "kernels.h"

namespace hh {

// ---- rows of the storage type, eight values at a time, at any alignment -------
// The memory unit takes 16-byte accesses at the alignment of their elements; where a row is aligned they cost no more for being written so.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef u32x4 u32x4_any __attribute__((aligned(2)));   // a bfloat16's alignment
// STREAM: the launch reads and writes more than the last-level cache keeps for the next one anyway (STREAM_BYTES).  Past the caches, cold
// tensors: dropout of 4096x12288 bf16 39.1 -> 36.6 us, residual addition with norm and packing 117 -> 105, 11008x4096 packed both ways
// and unpacked 88 -> 78.  Smaller ones are read by what follows while they are there.
constexpr double STREAM_BYTES = 96e6;
template <bool STREAM, typename V>
__device__ __forceinline__ V load_any(const V* p) { return STREAM ? __builtin_nontemporal_load(p) : *p; }
template <bool STREAM, typename V>
__device__ __forceinline__ void store_any(V* p, V v) {
    if constexpr (STREAM) __builtin_nontemporal_store(v, p);
    else *p = v;
}
template <bool STREAM = false> __device__ __forceinline__ u32x4 load16(const void* p) { return load_any<STREAM>(reinterpret_cast<const u32x4_any*>(p)); }
template <bool STREAM = false> __device__ __forceinline__ void store16(void* p, u32x4 v) { store_any<STREAM>(reinterpret_cast<u32x4_any*>(p), (u32x4_any)v); }
// N values of a row that has n more of them, as they lie in memory; what is behind its end is 0
template <typename T, int N> struct Few;
template <> struct Few<bf16_t, 8> {
    u32x4 w;
    __device__ __forceinline__ void hide() { asm volatile("" : "+v"(w)); }   // the compiler forgets what it has derived from them
    template <bool STREAM = false> __device__ __forceinline__ void load(const bf16_t* p, int n) {
        w = u32x4{0u, 0u, 0u, 0u};
        if (n >= 8) w = load16<STREAM>(p);
        else {
#pragma unroll
            for (int i = 0; i < 7; i++)
                if (i < n) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? hi_bf(w[i >> 1]) : lo_bf(w[i >> 1]); }
    __device__ __forceinline__ void widen(float* f) const {
#pragma unroll
        for (int i = 0; i < 8; i++) f[i] = at(i);
    }
    __device__ __forceinline__ void round(const float* f) {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = pack_bf2(f[2 * i], f[2 * i + 1]);
    }
    template <bool STREAM = false> __device__ __forceinline__ void store(bf16_t* p, int n) const {
        if (n >= 8) store16<STREAM>(p, w);
        else {
#pragma unroll
            for (int i = 0; i < 7; i++)
                if (i < n) p[i] = (bf16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
};
template <> struct Few<bf16_t, 4> {
    typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
    typedef u32x2 u32x2_any __attribute__((aligned(2)));
    u32x2 w;
    __device__ __forceinline__ void hide() { asm volatile("" : "+v"(w)); }
    template <bool STREAM = false> __device__ __forceinline__ void load(const bf16_t* p, int n) {
        w = u32x2{0u, 0u};
        if (n >= 4) w = load_any<STREAM>(reinterpret_cast<const u32x2_any*>(p));
        else {
#pragma unroll
            for (int i = 0; i < 3; i++)
                if (i < n) w[i >> 1] |= (uint32_t)p[i] << (16 * (i & 1));
        }
    }
    __device__ __forceinline__ float at(int i) const { return i & 1 ? hi_bf(w[i >> 1]) : lo_bf(w[i >> 1]); }
    __device__ __forceinline__ void round(const float* f) { w = u32x2{pack_bf2(f[0], f[1]), pack_bf2(f[2], f[3])}; }
    template <bool STREAM = false> __device__ __forceinline__ void store(bf16_t* p, int n) const {
        if (n >= 4) store_any<STREAM>(reinterpret_cast<u32x2_any*>(p), (u32x2_any)w);
        else {
#pragma unroll
            for (int i = 0; i < 3; i++)
                if (i < n) p[i] = (bf16_t)(w[i >> 1] >> (16 * (i & 1)));
        }
    }
};
template <int N> struct Few<float, N> {
    u32x4 w[N / 4];
    __device__ __forceinline__ void hide() {
#pragma unroll
        for (int i = 0; i < N / 4; i++) asm volatile("" : "+v"(w[i]));
    }
    template <bool STREAM = false> __device__ __forceinline__ void load(const float* p, int n) {
#pragma unroll
        for (int q = 0; q < N / 4; q++) {
            w[q] = u32x4{0u, 0u, 0u, 0u};
            if (n >= 4 * q + 4) w[q] = load16<STREAM>(p + 4 * q);
            else {
#pragma unroll
                for (int i = 0; i < 3; i++)
                    if (4 * q + i < n) w[q][i] = __float_as_uint(p[4 * q + i]);
            }
        }
    }
    __device__ __forceinline__ float at(int i) const { return __uint_as_float(w[i >> 2][i & 3]); }
    __device__ __forceinline__ void widen(float* f) const {
#pragma unroll
        for (int i = 0; i < N; i++) f[i] = at(i);
    }
    __device__ __forceinline__ void round(const float* f) {
#pragma unroll
        for (int i = 0; i < N; i++) w[i >> 2][i & 3] = __float_as_uint(f[i]);
    }
    template <bool STREAM = false> __device__ __forceinline__ void store(float* p, int n) const {
#pragma unroll
        for (int q = 0; q < N / 4; q++) {
            if (n >= 4 * q + 4) store16<STREAM>(p + 4 * q, w[q]);
            else {
#pragma unroll
                for (int i = 0; i < 3; i++)
                    if (4 * q + i < n) p[4 * q + i] = __uint_as_float(w[q][i]);
            }
        }
    }
};
template <typename T> using Eight = Few<T, 8>;

// ---- Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) --------------------------
// Eight elements share a counter, 16 bits each: half the generator's work of 32 bits each, whose twenty 32x32 -> 64 bit products a counter
// are at a quarter of the vector rate and bound a kernel that only streams (the share that is dropped is a multiple of 2^-16 then).
struct DropBits { uint32_t w[4]; };
__device__ __forceinline__ DropBits philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t seed) {
    uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
    for (int i = 0; i < 10; i++) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = (uint32_t)(b >> 32) ^ c1 ^ k0;
        c2 = (uint32_t)(a >> 32) ^ c3 ^ k1;
        c1 = (uint32_t)b;
        c3 = (uint32_t)a;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return DropBits{{c0, c1, c2, c3}};
}
__device__ __forceinline__ uint64_t drop_offset(const Drop& d) { return d.offset + (d.step ? *d.step : 0); }
// values 8 group .. of a row
__device__ __forceinline__ void drop8(const Drop& d, uint64_t offset, uint32_t group, uint32_t row, float* v) {
    const DropBits b = philox(group, row, offset, d.seed);
#pragma unroll
    for (int i = 0; i < 8; i++) {
        const uint32_t u = i & 1 ? b.w[i >> 1] >> 16 : b.w[i >> 1] & 0xFFFFu;
        v[i] = u >= d.dropped ? v[i] * d.scale : 0.f;   // chosen, not multiplied: a dropped NaN is 0
    }
}

// ---- microscaled formats ------------------------------------------------------
constexpr int MX_BLOCK = 32;
template <int F> struct Mx;
template <> struct Mx<MX_E4M3> { static constexpr int TOP = 8; static constexpr float MOST = 448.f; };
template <> struct Mx<MX_E2M1> { static constexpr int TOP = 2; static constexpr float MOST = 6.f; };

// The bits of the largest magnitude: compared as integers, so that infinities and NaNs come out on top.
__device__ __forceinline__ uint32_t magnitude8(const float* v) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; i++) m = max(m, __float_as_uint(v[i]) & 0x7FFFFFFFu);
    return m;
}
// Scale byte of a block from those bits; 255: it holds a NaN or an infinity.  (Below 2^-126 the exponent's bits are 0 and the scale is
// the least one, 2^-127, either way.)
template <int F>
__device__ __forceinline__ uint32_t scale_byte(uint32_t magnitude) {
    const int e = (int)(magnitude >> 23);
    return e == 255 ? 255u : (uint32_t)max(e - Mx<F>::TOP, 0);
}
// What a block's values are multiplied by: one over its scale, exactly.
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }
// A scale as a number: 2^(byte - 127), NaN for 255
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}
// Eight values, multiplied by `inv`, as codes in memory order.  The conversions round to nearest, ties to even; the one to four bits
// saturates by itself, the one to eight makes a NaN of what rounds past 448.
__device__ __forceinline__ uint32_t codes_e2m1(const float* v, float inv) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[0] * inv, v[1] * inv, 1.f, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[2] * inv, v[3] * inv, 1.f, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[4] * inv, v[5] * inv, 1.f, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, v[6] * inv, v[7] * inv, 1.f, 3);
    return c;
}
__device__ __forceinline__ uint32_t codes_e4m3(float a, float b, float c, float d, float inv) {
    auto clamp = [](float x) { return __builtin_amdgcn_fmed3f(x, -448.f, 448.f); };
    int r = __builtin_amdgcn_cvt_pk_fp8_f32(clamp(a * inv), clamp(b * inv), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(clamp(c * inv), clamp(d * inv), r, true);
}
constexpr uint32_t NAN_CODES_E2M1 = 0x77777777u, NAN_CODES_E4M3 = 0x7F7F7F7Fu;   // any value times the scale NaN
template <int F> struct Codes8;   // eight codes as they lie in memory
template <> struct Codes8<MX_E4M3> {
    uint2 w;
    __device__ __forceinline__ void set(const float* v, uint32_t byte) {
        const float inv = scale_inverse(byte);
        w = byte == 255u ? make_uint2(NAN_CODES_E4M3, NAN_CODES_E4M3)
                         : make_uint2(codes_e4m3(v[0], v[1], v[2], v[3], inv), codes_e4m3(v[4], v[5], v[6], v[7], inv));
    }
    __device__ __forceinline__ void store(uint8_t* row, size_t chunk) const { *reinterpret_cast<uint2*>(row + 8 * chunk) = w; }
};
template <> struct Codes8<MX_E2M1> {
    uint32_t w;
    __device__ __forceinline__ void set(const float* v, uint32_t byte) { w = byte == 255u ? NAN_CODES_E2M1 : codes_e2m1(v, scale_inverse(byte)); }
    __device__ __forceinline__ void store(uint8_t* row, size_t chunk) const { *reinterpret_cast<uint32_t*>(row + 4 * chunk) = w; }
};
// The largest of a value over the four neighbouring lanes that share a block
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

}  // namespace hh
