// The way out of an NT product whose rows are scores over a vocabulary (GemmScores): what a softmax over a row needs, formed from
// the accumulators, and the scores themselves in fp32 where they are asked for.
//
// In the accumulators a lane owns one row and 32 of the wave's 64 columns, the other half wave the other 32: largest score and sum
// of exponentials of a slot are 32 values in registers and one exchange.  The running maximum and sum of a row's softmax are put
// together from its slots by the kernel that follows.  Without `stats` the scores alone are written.  Bound by the k loop:
// 2048x32000x4096 425 us without z (1.26 PFLOP/s), 465 with its 262 MB.
#pragma once
#include "gemm_tile.h"
#include "kernels.h"

namespace hh {

// rows row0 + 32 i + lane % 32, columns col0 + 32 j + 8 q + 4 (lane / 32) + e of [M, N]; z: null or rows of ldz >= N rounded up to 4.
// Column c is word first + c of the vocabulary that the labels count in.  patch: 4 KB of LDS that this wave alone uses.
template <int TM, int TN>
__device__ __forceinline__ void write_scores(f32x16 (&acc)[TM][TN], int row0, int col0, int M, int N, float* z, int ldz,
                                             const int64_t* __restrict__ labels, int first, float2* __restrict__ stats, char* patch) {
    static_assert(32 * TN == SCORE_SLOT, "a wave owns whole slots");
    constexpr float LOG2E = 1.4426950408889634f;
    if (col0 >= N) return;   // no column of the slot is there
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));   // what is derived from it is formed here and not kept through the k loop
    const int hf = lane >> 5, r_w = lane & 31, r_r = lane >> 3, c_r = lane & 7;
    const int slot = col0 / SCORE_SLOT;
    float* const picked = (float*)(stats + (size_t)((N + SCORE_SLOT - 1) / SCORE_SLOT) * M);
    int64_t label[TM];
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const int row = row0 + 32 * i + r_w;
        label[i] = stats && row < M ? labels[row] : (int64_t)first - 1;
    }
    const bool ragged = col0 + SCORE_SLOT > N;
    const __amdgpu_buffer_rsrc_t rsZ = make_rsrc(z, z ? (uint32_t)((size_t)M * ldz * 4u) : 0u);
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const int row = row0 + 32 * i + r_w;
        if (ragged) {
#pragma unroll
            for (int j = 0; j < TN; j++)
#pragma unroll
                for (int e = 0; e < 16; e++)
                    if (col0 + 32 * j + 8 * (e >> 2) + 4 * hf + (e & 3) >= N) acc[i][j][e] = -INFINITY;
        }
        if (stats) {
            float top = -INFINITY;
#pragma unroll
            for (int j = 0; j < TN; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) top = fmaxf(top, acc[i][j][e]);
            top = fmaxf(top, __shfl_xor(top, 32, WAVE));
            const float ref = top == -INFINITY ? 0.f : top;   // a slot of scores of -inf adds nothing, not NaN
            float sum = 0.f;
#pragma unroll
            for (int j = 0; j < TN; j++)
#pragma unroll
                for (int e = 0; e < 16; e++) sum += __builtin_amdgcn_exp2f((acc[i][j][e] - ref) * LOG2E);
            sum += __shfl_xor(sum, 32, WAVE);
            if (hf == 0 && row < M) stats[(size_t)slot * M + row] = make_float2(top, sum);
            const int64_t rel = label[i] - first - col0;
            const bool here = rel >= 0 && rel < SCORE_SLOT && col0 + rel < N;
            if (__any(here)) {   // few slots hold the label of one of their rows
                const int mine = here ? (int)rel - 4 * hf : -1;
                float v = 0.f;
#pragma unroll
                for (int j = 0; j < TN; j++)
#pragma unroll
                    for (int e = 0; e < 16; e++) v = mine == 32 * j + 8 * (e >> 2) + (e & 3) ? acc[i][j][e] : v;
                if (mine >= 0 && !(mine & 4)) picked[row] = v;   // of the two half waves the one that owns the column
            }
        }
        if (z) {
            const uint32_t zrow = (uint32_t)(row0 + 32 * i + r_r);
#pragma unroll
            for (int j = 0; j < TN; j++) {
                const int col = col0 + 32 * j + 4 * c_r;
#pragma unroll
                for (int q = 0; q < 4; q++)
                    *reinterpret_cast<float4*>(patch + r_w * 128 + (((2 * q + hf) ^ ((r_w >> 1) & 7)) << 4)) =
                        make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
#pragma unroll
                for (int t = 0; t < 4; t++) {
                    const int rr = 8 * t + r_r;
                    const i32x4 v = *reinterpret_cast<const i32x4*>(patch + rr * 128 + ((c_r ^ ((rr >> 1) & 7)) << 4));
                    __builtin_amdgcn_raw_buffer_store_b128(v, rsZ, col < N ? ((zrow + 8 * t) * (uint32_t)ldz + (uint32_t)col) * 4u : 0x80000000u, 0, 0);
                }
            }
        }
    }
}

}  // namespace hh
