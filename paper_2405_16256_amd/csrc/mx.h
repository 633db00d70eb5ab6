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
// STREAM: a launch of more than STREAM_BYTES goes past the caches.  Cold tensors: dropout of 4096x12288 bf16 39.1 -> 36.6 us, residual addition
// with norm and packing 117 -> 105.  The last-level cache holds more than that, so it could cost a call that reads what the one before
// wrote; a residual connection with its E2M1 projection, forward and backward, takes 1103 us (4096 tokens, 12288 x 8192; 1133 through
// the caches), 688 (2048 tokens; 697), 531 (4096, 4096 x 11008; 539), 434 (8192, 4096 x 4096; 448).  Its forward half alone loses once in these
// four, 4096 tokens of 4096 x 11008, 149 us in place of 143.  Rows that end inside a chunk and the longest rows' gradients, which are read twice,
// go through the caches.
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
    // Through the caches whatever STREAM says: a store takes every other 16 bytes, and what goes past them goes out as these halves of lines
    // (8192x8192, dropout 160 us in place of 94, values of E4M3 125 of 60).
    template <bool STREAM = false> __device__ __forceinline__ void store(float* p, int n) const {
#pragma unroll
        for (int q = 0; q < N / 4; q++) {
            if (n >= 4 * q + 4) store16(p + 4 * q, w[q]);
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
// A scale as a number: 2^(byte - 127), NaN for 255
__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __uint_as_float(byte == 255u ? 0x7FC00000u : byte ? byte << 23 : 0x00400000u);
}
// Two neighbouring values of a block, as the conversions take them
template <typename T> struct Pair;
template <> struct Pair<float> { float a, b; };
template <> struct Pair<bf16_t> {
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    uint32_t w;
};
// Codes of a block's values.  The conversions divide by the scale, of which they take the exponent alone (0 is 2^-127), and round once, to
// nearest, ties to even.  The ones to four bits saturate by themselves, those to eight make a NaN of what rounds past 448.
template <int F>
struct Packer {
    uint32_t byte;
    __device__ __forceinline__ explicit Packer(uint32_t magnitude) : byte(scale_byte<F>(magnitude)) {}
    __device__ __forceinline__ float scale() const { return __uint_as_float(byte << 23); }
    // `into` with the codes of a pair in byte (E4M3: half word) AT
    template <int AT> __device__ __forceinline__ uint32_t put(uint32_t into, Pair<float> p) const {
        if constexpr (F == MX_E2M1) return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(into, p.a, p.b, scale(), AT);
        else {
            const float inv = __uint_as_float((254u - byte) << 23);
            return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(__builtin_amdgcn_fmed3f(p.a * inv, -448.f, 448.f),
                                                             __builtin_amdgcn_fmed3f(p.b * inv, -448.f, 448.f), (int)into, AT == 1);
        }
    }
    template <int AT> __device__ __forceinline__ uint32_t put(uint32_t into, Pair<bf16_t> p) const {
        Pair<bf16_t>::bf16x2 v;
        if constexpr (F == MX_E2M1) {
            __builtin_memcpy(&v, &p.w, 4);
            return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(into, v, scale(), AT);
        } else {   // 448 times the scale: the magnitudes' bits are in the order of the numbers
            const uint16_t most = (uint16_t)((byte + 8u) << 7 | 0x60u);
            typedef short s16x2 __attribute__((ext_vector_type(2)));
            Pair<bf16_t>::u16x2 m;
            s16x2 c;
            const uint32_t magnitudes = p.w & 0x7FFF7FFFu;
            __builtin_memcpy(&m, &magnitudes, 4);
            m = __builtin_elementwise_min(m, Pair<bf16_t>::u16x2{most, most});
            uint32_t w;
            __builtin_memcpy(&w, &m, 4);
            w |= p.w & 0x80008000u;
            __builtin_memcpy(&v, &w, 4);
            __builtin_memcpy(&c, &into, 4);
            c = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(c, v, scale(), AT == 1);
            __builtin_memcpy(&into, &c, 4);
            return into;
        }
    }
    // A block that holds a NaN or an infinity: any value times the scale NaN
    __device__ __forceinline__ uint32_t checked(uint32_t codes) const { return byte != 255u ? codes : F == MX_E2M1 ? 0x77777777u : 0x7F7F7F7Fu; }
    template <typename T> __device__ __forceinline__ uint32_t four(Pair<T> p, Pair<T> q) const { return checked(put<1>(put<0>(0u, p), q)); }   // E2M1: 16 bits of it
    // Eight values as they lie in memory
    template <typename T> __device__ __forceinline__ void eight(const Pair<T>* p, uint32_t* to) const {
        if constexpr (F == MX_E2M1) to[0] = checked(put<3>(put<2>(put<1>(put<0>(0u, p[0]), p[1]), p[2]), p[3]));
        else {
            to[0] = four(p[0], p[1]);
            to[1] = four(p[2], p[3]);
        }
    }
    template <bool STREAM = false, typename T> __device__ __forceinline__ void store8(const Pair<T>* p, uint8_t* row, size_t chunk) const {
        typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
        uint32_t w[2];
        eight(p, w);
        if constexpr (F == MX_E2M1) store_any<STREAM>(reinterpret_cast<uint32_t*>(row + 4 * chunk), w[0]);
        else store_any<STREAM>(reinterpret_cast<u32x2*>(row + 8 * chunk), u32x2{w[0], w[1]});
    }
};
template <int N> __device__ __forceinline__ Pair<bf16_t> pair_of(const Few<bf16_t, N>& v, int i) { return {v.w[i]}; }   // values 2 i, 2 i + 1
template <int N> __device__ __forceinline__ Pair<float> pair_of(const Few<float, N>& v, int i) { return {v.at(2 * i), v.at(2 * i + 1)}; }
// Value j of a and of b
template <int N> __device__ __forceinline__ Pair<bf16_t> pair_across(const Few<bf16_t, N>& a, const Few<bf16_t, N>& b, int j) {
    return {__builtin_amdgcn_perm(b.w[j >> 1], a.w[j >> 1], j & 1 ? 0x07060302u : 0x05040100u)};
}
template <int N> __device__ __forceinline__ Pair<float> pair_across(const Few<float, N>& a, const Few<float, N>& b, int j) { return {a.at(j), b.at(j)}; }

// Magnitudes of N values as they lie in memory, two bf16 to a word: their order as integers is that of the numbers, and two are compared at
// a time.
template <typename T, int N> struct Magnitudes;
template <int N> struct Magnitudes<bf16_t, N> {
    uint32_t w[N / 2];
    __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
        Pair<bf16_t>::u16x2 x, y;
        __builtin_memcpy(&x, &a, 4);
        __builtin_memcpy(&y, &b, 4);
        x = __builtin_elementwise_max(x, y);
        __builtin_memcpy(&a, &x, 4);
        return a;
    }
    __device__ __forceinline__ explicit Magnitudes(const Few<bf16_t, N>& v) {
#pragma unroll
        for (int i = 0; i < N / 2; i++) w[i] = v.w[i] & 0x7FFF7FFFu;
    }
    __device__ __forceinline__ void add(const Magnitudes& o) {
#pragma unroll
        for (int i = 0; i < N / 2; i++) w[i] = larger(w[i], o.w[i]);
    }
    __device__ __forceinline__ uint32_t column(int j) const { return (j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu) << 16; }   // as of fp32
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = w[0];
#pragma unroll
        for (int i = 1; i < N / 2; i++) m = larger(m, w[i]);
        return max(m >> 16, m & 0xFFFFu) << 16;
    }
};
template <int N> struct Magnitudes<float, N> {
    uint32_t w[N];
    __device__ __forceinline__ explicit Magnitudes(const Few<float, N>& v) {
#pragma unroll
        for (int i = 0; i < N; i++) w[i] = v.w[i >> 2][i & 3] & 0x7FFFFFFFu;
    }
    __device__ __forceinline__ void add(const Magnitudes& o) {
#pragma unroll
        for (int i = 0; i < N; i++) w[i] = max(w[i], o.w[i]);
    }
    __device__ __forceinline__ uint32_t column(int j) const { return w[j]; }
    __device__ __forceinline__ uint32_t largest() const {
        uint32_t m = w[0];
#pragma unroll
        for (int i = 1; i < N; i++) m = max(m, w[i]);
        return m;
    }
};
// The largest of a value over the four neighbouring lanes that share a block
__device__ __forceinline__ uint32_t quad_max(uint32_t m) {
    m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0xB1, 0xF, 0xF, true));   // lanes 1 0 3 2
    return max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x4E, 0xF, 0xF, true));   // lanes 2 3 0 1
}

// The scales of the four blocks of sixteen lanes, which are all here, as one word; `at`: where the first lane's goes.
__device__ __forceinline__ void store_scales(uint8_t* at, uint32_t byte) {
    uint32_t w = byte | (uint32_t)__builtin_amdgcn_update_dpp(0, (int)byte, 0x104, 0xF, 0xF, true) << 8;   // from four lanes on
    w |= (uint32_t)__builtin_amdgcn_update_dpp(0, (int)w, 0x108, 0xF, 0xF, true) << 16;                    // from eight
    if ((threadIdx.x & 15) == 0) *reinterpret_cast<uint32_t*>(at) = w;
}

}  // namespace hh
