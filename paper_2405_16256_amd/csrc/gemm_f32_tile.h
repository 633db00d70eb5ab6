// Operand tiles of the fp32 matrix-core GEMMs: filled straight from global memory into LDS, read back as MFMA fragments.
#pragma once
#include "gemm_tile.h"

namespace hh {

constexpr int FK = 32;   // k values per stage

// One operand's tile of ROWS rows of C's dimension x FK values of k.
//   KC (k contiguous): LDS [row][k], 128 bytes a row, 16-byte chunks XOR-swizzled by the row index.
//   otherwise:         LDS [k][row], bit 7 of the byte address flipped for k rows with bit 2 set, so that the two half
//                      waves of a fragment read (k and k + 4) fall into different banks.
template <bool KC, int ROWS>
struct FTile {
    static constexpr int BYTES = ROWS * FK * 4;
    static constexpr int PER_WAVE = BYTES / 1024 / 4;
    static constexpr int PITCH = ROWS * 4;
    struct Src { uint32_t off; int k; };   // byte offset at k tile 0; first k value the lane fetches there
    __device__ static __forceinline__ Src src(int wave, int i, int row0, int ld) {
        const int idx = wave * PER_WAVE + i, L = threadIdx.x & 63;
        if (KC) {
            const int r = 8 * idx + (L >> 3), c = (L & 7) ^ ((r >> 1) & 7);
            return {((uint32_t)(row0 + r) * (uint32_t)ld + (uint32_t)(4 * c)) * 4u, 4 * c};
        }
        const int p = idx * 1024 + L * 16;
        const int lb = p ^ ((((p / PITCH) >> 2) & 1) << 7);
        const int k = lb / PITCH;
        return {((uint32_t)k * (uint32_t)ld + (uint32_t)row0) * 4u + (uint32_t)(lb % PITCH), k};
    }
    __device__ static __forceinline__ uint32_t kstep_bytes(int ld) { return KC ? FK * 4u : (uint32_t)FK * (uint32_t)ld * 4u; }
    // the lane's 4 values of k step kk (8 k values): row rb + lane%32, k = 8kk + 4(lane/32) + e
    __device__ static __forceinline__ f32x4 frag(const char* lds, int rb, int kk) {
        const int l = threadIdx.x & 63, r = rb + (l & 31), hf = l >> 5;
        if (KC) return *reinterpret_cast<const f32x4*>(lds + r * 128 + (((2 * kk + hf) ^ ((r >> 1) & 7)) << 4));
        f32x4 v;
#pragma unroll
        for (int e = 0; e < 4; e++) {
            const int k = 8 * kk + 4 * hf + e;
            v[e] = *reinterpret_cast<const float*>(lds + ((k * PITCH + r * 4) ^ (hf << 7)));   // (k >> 2) & 1 == hf
        }
        return v;
    }
};

}  // namespace hh
