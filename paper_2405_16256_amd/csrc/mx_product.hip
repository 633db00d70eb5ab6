// C (=|+=) A B^T of two microscaled operands on the matrix cores.
#include "mx.h"

namespace hh {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// What one lane holds of 32 rows x 64 k of an operand: row lane % 32 and, with h = lane / 32, of E2M1 the codes k = 32 h .. 32 h + 31, of E4M3
// the codes 16 h .. 16 h + 15 and 32 + 16 h .. 32 + 16 h + 15.  The scale of a lane is that of k = 32 h .. 32 h + 31 in both.
template <int F> __device__ __forceinline__ i32x8 fragment(const uint8_t* row, int k, int h);
template <> __device__ __forceinline__ i32x8 fragment<MX_E2M1>(const uint8_t* row, int k, int h) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(row + k / 2 + 16 * h);
    return i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0};
}
template <> __device__ __forceinline__ i32x8 fragment<MX_E4M3>(const uint8_t* row, int k, int h) {
    const i32x4 a = *reinterpret_cast<const i32x4*>(row + k + 16 * h), b = *reinterpret_cast<const i32x4*>(row + k + 32 + 16 * h);
    return i32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
template <int F> constexpr int FORMAT = F == MX_E4M3 ? 0 : 4;   // of the matrix instruction

// Widened to bfloat16 with their scale, exactly: 16 codes of a block, which this lane holds of 32 rows x 64 k twice, k = 32 q + 16 h .. + 15.
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
template <int F> __device__ __forceinline__ void widen16(const uint8_t* row, int k, int h, float scale, bf16x8& lo, bf16x8& hi);
template <> __device__ __forceinline__ void widen16<MX_E4M3>(const uint8_t* row, int k, int h, float scale, bf16x8& lo, bf16x8& hi) {
    const i32x4 codes = *reinterpret_cast<const i32x4*>(row + k + 16 * h);
    bf16x2v p[8];
#pragma unroll
    for (int i = 0; i < 4; i++) {
        p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], scale, false);
        p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((uint32_t)codes[i], scale, true);
    }
    lo = bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
    hi = bf16x8{p[4][0], p[4][1], p[5][0], p[5][1], p[6][0], p[6][1], p[7][0], p[7][1]};
}
template <> __device__ __forceinline__ void widen16<MX_E2M1>(const uint8_t* row, int k, int h, float scale, bf16x8& lo, bf16x8& hi) {
    const i32x2 codes = *reinterpret_cast<const i32x2*>(row + k / 2 + 8 * h);
    bf16x2v p[8];
#pragma unroll
    for (int i = 0; i < 2; i++) {
        p[4 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes[i], scale, 0);
        p[4 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes[i], scale, 1);
        p[4 * i + 2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes[i], scale, 2);
        p[4 * i + 3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4((uint32_t)codes[i], scale, 3);
    }
    lo = bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
    hi = bf16x8{p[4][0], p[4][1], p[5][0], p[5][1], p[6][0], p[6][1], p[7][0], p[7][1]};
}

// A workgroup of 4 waves forms 32x32 of C, each wave a quarter of k, straight from memory.  WIDE: on the bfloat16 instruction.
template <int FA, int FB, bool WIDE, typename TC>
__global__ __launch_bounds__(256) void k_product(MxProduct p, int width, int tiles_n) {
    __shared__ float part[3][64][17];
    const int wave = (int)threadIdx.x >> 6, lane = (int)threadIdx.x & 63, h = lane >> 5, l = lane & 31;
    const int m0 = ((int)blockIdx.x / tiles_n) * 32, n0 = ((int)blockIdx.x % tiles_n) * 32;
    const size_t ra = min(m0 + l, p.M - 1), rb = min(n0 + l, p.N - 1);   // rows past the end: any, their results are dropped
    const uint8_t* const a = p.a.codes + ra * (size_t)(FA == MX_E4M3 ? width : width / 2);
    const uint8_t* const b = p.b.codes + rb * (size_t)(FB == MX_E4M3 ? width : width / 2);
    const uint8_t* const sa = p.a.scales + ra * (size_t)(width / MX_BLOCK) + h;
    const uint8_t* const sb = p.b.scales + rb * (size_t)(width / MX_BLOCK) + h;
    f32x16 acc;
#pragma unroll
    for (int i = 0; i < 16; i++) acc[i] = 0.f;
    const int steps = (p.K + 63) / 64, from = steps * wave / 4, to = steps * (wave + 1) / 4;
    for (int s = from; s < to; s++) {
        if constexpr (WIDE) {
            const uint8_t* const ba = sa - h + 2 * s;
            const uint8_t* const bb = sb - h + 2 * s;
#pragma unroll
            for (int q = 0; q < 2; q++) {
                bf16x8 a0, a1, b0, b1;
                widen16<FA>(a, 64 * s + 32 * q, h, scale_value(ba[q]), a0, a1);
                widen16<FB>(b, 64 * s + 32 * q, h, scale_value(bb[q]), b0, b1);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b0, a0, acc, 0, 0, 0);
                acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b1, a1, acc, 0, 0, 0);
            }
        } else {
            const i32x8 fa = fragment<FA>(a, 64 * s, h), fb = fragment<FB>(b, 64 * s, h);
            acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(fb, fa, acc, FORMAT<FB>, FORMAT<FA>, 0, (int)sb[2 * s], 0, (int)sa[2 * s]);
        }
    }
    if (wave) {
#pragma unroll
        for (int i = 0; i < 16; i++) part[wave - 1][lane][i] = acc[i];
    }
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 0; w < 3; w++)
#pragma unroll
        for (int i = 0; i < 16; i++) acc[i] += part[w][lane][i];
    // a lane has row l of C and columns 8 q + 4 h .. + 3
    const int m = m0 + l;
    if (m >= p.M) return;
    TC* const c = (TC*)p.C + (long)m * p.ldc;
#pragma unroll
    for (int i = 0; i < 16; i++) {
        const int n = n0 + 8 * (i >> 2) + 4 * h + (i & 3);
        if (n >= p.N) continue;
        if constexpr (sizeof(TC) == 4) c[n] = p.accumulate ? c[n] + acc[i] : acc[i];
        else c[n] = f2bf(p.accumulate ? bf2f(c[n]) + acc[i] : acc[i]);
    }
}

size_t mx_product_workspace(const MxProduct&) { return 0; }

hipError_t mx_product(const MxProduct& p, void*, hipStream_t st) {
    const int width = (int)mx_width(p.K), tiles_n = (p.N + 31) / 32;
    const unsigned grid = (unsigned)(((p.M + 31) / 32) * (long)tiles_n);
    auto run = [&](auto kern) {
        kern<<<grid, 256, 0, st>>>(p, width, tiles_n);
        return hipGetLastError();
    };
    const bool a8 = p.fa == MX_E4M3, b8 = p.fb == MX_E4M3;
    if (p.f32) {
        if (a8 && b8) return run(k_product<MX_E4M3, MX_E4M3, true, float>);
        if (a8) return run(k_product<MX_E4M3, MX_E2M1, true, float>);
        if (b8) return run(k_product<MX_E2M1, MX_E4M3, true, float>);
        return run(k_product<MX_E2M1, MX_E2M1, false, float>);
    }
    if (a8 && b8) return run(k_product<MX_E4M3, MX_E4M3, false, bf16_t>);
    if (a8) return run(k_product<MX_E4M3, MX_E2M1, false, bf16_t>);
    if (b8) return run(k_product<MX_E2M1, MX_E4M3, false, bf16_t>);
    return run(k_product<MX_E2M1, MX_E2M1, false, bf16_t>);
}

}  // namespace hh
