// C (=|+=) A B^T of two microscaled operands on the matrix cores.
#include <algorithm>
#include <type_traits>

#include "gemm_tile.h"
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

// ------------------------------------------------------------------ few rows
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


// ------------------------------------------------------------------ tiles
// BM x BN of C a workgroup, WR x WC waves, each 32 TM x 32 TN.  k advances KS at a time through two LDS stages that are filled straight from
// global memory; a row of a stage is 128 bytes of E4M3 (KS 128), or 64 beside that, or 128 of E2M1 on both sides (KS 256), and the scales of
// those k lie behind the tiles.  16-byte chunks are XOR-swizzled by the row so that a fragment's 16 lanes cover all banks.
template <int F, int KS> constexpr int ROW_BYTES = F == MX_E4M3 ? KS : KS / 2;
template <int RB> __device__ __forceinline__ int swizzled(int row, int chunk) {   // byte offset in the tile
    return row * RB + ((RB == 128 ? chunk ^ ((row >> 1) & 7) : chunk ^ ((row >> 2) & 3)) << 4);
}
template <int FA, int FB> constexpr int STAGE_K = FA == MX_E2M1 && FB == MX_E2M1 ? 256 : 128;

__device__ __forceinline__ void dma4(uint32_t lds_addr, uint32_t voff, i32x4 rs) {   // as dma16, four bytes a lane
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(voff), "s"(rs) : "memory");
}
__device__ __forceinline__ i32x4 rsrc_words(const void* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)p;
    return i32x4{(int)(uint32_t)a, (int)(uint32_t)(a >> 32), (int)bytes, 0x00020000};
}

// One operand's share of a stage: its tile and its scales.
template <int F, int KS, int ROWS, int NW>
struct MxTile {
    static constexpr int RB = ROW_BYTES<F, KS>, SB = KS / MX_BLOCK, BYTES = ROWS * RB, SCALES = ROWS * SB;
    static constexpr int PER_WAVE = BYTES / 1024 / NW;             // instructions of 1 KB
    static_assert(PER_WAVE * NW * 1024 == BYTES, "the tile splits evenly over the waves");
    static constexpr int SCALE_PARTS = SCALES / 256;               // instructions of 256 bytes, over all waves
    __device__ static __forceinline__ uint32_t voff(int wave, int i, int row0, uint32_t pitch) {
        constexpr int LPR = RB / 16;
        const int L = threadIdx.x & 63, r = (wave * PER_WAVE + i) * (64 / LPR) + L / LPR;
        const int logical = RB == 128 ? (L & 7) ^ ((r >> 1) & 7) : (L & 3) ^ ((r >> 2) & 3);
        return (uint32_t)(row0 + r) * pitch + (uint32_t)(logical * 16);
    }
    __device__ static __forceinline__ uint32_t scale_voff(int part, int row0, uint32_t pitch) {
        const int d = 64 * part + (int)(threadIdx.x & 63);
        return (uint32_t)(row0 + d / (SB / 4)) * pitch + (uint32_t)(4 * (d % (SB / 4)));
    }
    static constexpr int REGS = F == MX_E4M3 ? 2 : 1;
    struct Frag { i32x4 v[REGS]; };
    // rows rb .. rb + 31, k = 64 step ..; as the matrix instruction takes them, or (WIDE) as widen_piece does
    template <bool WIDE> __device__ static __forceinline__ Frag frag(const char* lds, int rb, int step) {
        const int l = threadIdx.x & 63, r = rb + (l & 31), h = l >> 5;
        Frag f;
        if constexpr (F == MX_E4M3) {
            f.v[0] = *reinterpret_cast<const i32x4*>(lds + swizzled<RB>(r, 4 * step + h));
            f.v[1] = *reinterpret_cast<const i32x4*>(lds + swizzled<RB>(r, 4 * step + 2 + h));
        } else if constexpr (WIDE) {
            const i32x2 a = *reinterpret_cast<const i32x2*>(lds + swizzled<RB>(r, 2 * step) + 8 * h);
            const i32x2 b = *reinterpret_cast<const i32x2*>(lds + swizzled<RB>(r, 2 * step + 1) + 8 * h);
            f.v[0] = i32x4{a[0], a[1], b[0], b[1]};
        } else {
            f.v[0] = *reinterpret_cast<const i32x4*>(lds + swizzled<RB>(r, 2 * step + h));
        }
        return f;
    }
    __device__ static __forceinline__ i32x8 operand(const Frag& f) {
        if constexpr (F == MX_E4M3) return i32x8{f.v[0][0], f.v[0][1], f.v[0][2], f.v[0][3], f.v[1][0], f.v[1][1], f.v[1][2], f.v[1][3]};
        else return i32x8{f.v[0][0], f.v[0][1], f.v[0][2], f.v[0][3], 0, 0, 0, 0};
    }
    // piece 2 q + p: codes 8 p .. of the lane's 16 of block q
    __device__ static __forceinline__ bf16x8 widen_piece(const Frag& f, int piece, float scale) {
        bf16x2v p[4];
        if constexpr (F == MX_E4M3) {
#pragma unroll
            for (int i = 0; i < 2; i++) {
                const uint32_t w = (uint32_t)f.v[piece >> 1][2 * (piece & 1) + i];
                p[2 * i] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
                p[2 * i + 1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
            }
        } else {
            const uint32_t w = (uint32_t)f.v[0][piece];
            p[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0);
            p[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1);
            p[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2);
            p[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3);
        }
        return bf16x8{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
    }
    // The scales of a stage for rows rb .. rb + 31: not WIDE, byte (KS 256: s, KS 128: 2 s) is that of step s for this lane's half; WIDE, bytes
    // 2 s and 2 s + 1 are those of step s.
    template <bool WIDE> __device__ static __forceinline__ int scales(const char* lds, int rb) {
        const int l = threadIdx.x & 63, r = rb + (l & 31), h = l >> 5;
        if constexpr (SB == 8) {
            const uint2 w = *reinterpret_cast<const uint2*>(lds + 8 * r);
            return (int)__builtin_amdgcn_perm(w.y, w.x, h ? 0x07050301u : 0x06040200u);
        } else {
            const uint32_t w = *reinterpret_cast<const uint32_t*>(lds + 4 * r);
            return (int)(WIDE ? w : w >> (8 * h));
        }
    }
};

template <int FA, int FB, int SA, int SB>
__device__ __forceinline__ f32x16 mfma_mx(i32x8 a, i32x8 b, f32x16 c, int sa, int sb) {
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, FORMAT<FA>, FORMAT<FB>, SA, sa, SB, sb);
}

struct MxProblem {
    const uint8_t *a, *b, *sa, *sb;
    uint32_t a_bytes, b_bytes, sa_bytes, sb_bytes;   // extents: rows past them read as zeros
    void* C;
    long ldc;
    int M, N, stages, accumulate, split;             // k stages; shares of them (grid's y)
    uint32_t pitch_a, pitch_b, pitch_s;
    float* partial;                                  // [share][M][N], where there are several
    TileMap map;
};

template <int FA, int FB, bool WIDE, typename TC, int BM, int BN, int WR, int WC>
__global__ __launch_bounds__(64 * WR * WC) void k_product_tiles(MxProblem p) {
    constexpr int KS = STAGE_K<FA, FB>, NW = WR * WC, TM = BM / WR / 32, TN = BN / WC / 32, STEPS = KS / 64, Q = STEPS * TM;
    using A = MxTile<FA, KS, BM, NW>;
    using B = MxTile<FB, KS, BN, NW>;
    constexpr int STAGE = A::BYTES + B::BYTES + A::SCALES + B::SCALES, AT_B = A::BYTES, AT_SA = AT_B + B::BYTES, AT_SB = AT_SA + A::SCALES;
    constexpr int PARTS = A::PER_WAVE + B::PER_WAVE, SCALE_PARTS = (A::SCALE_PARTS + B::SCALE_PARTS) / NW;
    static_assert(SCALE_PARTS * NW == A::SCALE_PARTS + B::SCALE_PARTS, "the scales split evenly over the waves");
    extern __shared__ __attribute__((aligned(1024))) char smem[];
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, h = lane >> 5;
    const int wm = (wave / WC) * 32 * TM, wn = (wave % WC) * 32 * TN;
    int tm, tn;
    p.map.tile((int)blockIdx.x, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN;
    const int first = p.stages * (int)blockIdx.y / p.split, nk = p.stages * ((int)blockIdx.y + 1) / p.split - first;
    i32x4 rsA = rsrc_words(p.a, p.a_bytes), rsB = rsrc_words(p.b, p.b_bytes), rsS[SCALE_PARTS];
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem);
    const int uwave = __builtin_amdgcn_readfirstlane(wave);
    uint32_t voA[A::PER_WAVE], voB[B::PER_WAVE], voS[SCALE_PARTS], toS[SCALE_PARTS];
#pragma unroll
    for (int i = 0; i < A::PER_WAVE; i++) voA[i] = A::voff(wave, i, m0, p.pitch_a) + first * A::RB;
#pragma unroll
    for (int i = 0; i < B::PER_WAVE; i++) voB[i] = B::voff(wave, i, n0, p.pitch_b) + first * B::RB;
#pragma unroll
    for (int i = 0; i < SCALE_PARTS; i++) {   // of A, then of B
        const int part = uwave + NW * i, of_b = part - A::SCALE_PARTS;
        rsS[i] = of_b < 0 ? rsrc_words(p.sa, p.sa_bytes) : rsrc_words(p.sb, p.sb_bytes);
        toS[i] = of_b < 0 ? AT_SA + part * 256 : AT_SB + of_b * 256;
        voS[i] = (of_b < 0 ? A::scale_voff(part, m0, p.pitch_s) : B::scale_voff(of_b, n0, p.pitch_s)) + first * A::SB;
    }
    auto dma_part = [&](int st, int i) {
        const uint32_t base = lds0 + st * STAGE;
        if (i < A::PER_WAVE) {
            dma16(base + (uwave * A::PER_WAVE + i) * 1024, voA[i], rsA);
            voA[i] += A::RB;
        } else if (i < PARTS) {
            const int j = i - A::PER_WAVE;
            dma16(base + AT_B + (uwave * B::PER_WAVE + j) * 1024, voB[j], rsB);
            voB[j] += B::RB;
        } else {
            dma4(base + toS[i - PARTS], voS[i - PARTS], rsS[i - PARTS]);
            voS[i - PARTS] += A::SB;
        }
    };
    constexpr int ALL = PARTS + SCALE_PARTS;
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
#pragma unroll
    for (int s = 0; s < 2; s++)
        if (s < nk) {
#pragma unroll
            for (int i = 0; i < ALL; i++) dma_part(s, i);
        }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();

    // Fragments of A are fetched AHEAD of their products, those of B a step ahead; scales with the first fragments of their stage.
    constexpr int AHEAD = 3, RING = 4;
    static_assert(Q % RING == 0 && STEPS % 2 == 0, "a stage ends where it began in both rings");
    typename A::Frag fa[RING];
    typename B::Frag fb[2][TN];
    int sa[TM], sb[TN], na[TM], nb[TN];
#pragma unroll
    for (int q = 0; q < AHEAD; q++) fa[q] = A::template frag<WIDE>(smem, wm + 32 * (q % TM), q / TM);
#pragma unroll
    for (int j = 0; j < TN; j++) fb[0][j] = B::template frag<WIDE>(smem + AT_B, wn + 32 * j, 0);
#pragma unroll
    for (int i = 0; i < TM; i++) sa[i] = A::template scales<WIDE>(smem + AT_SA, wm + 32 * i);
#pragma unroll
    for (int j = 0; j < TN; j++) sb[j] = B::template scales<WIDE>(smem + AT_SB, wn + 32 * j);
    for (int kt = 0; kt < nk; kt++) {
        const char* const cur = smem + (kt & 1) * STAGE;
        const char* const nxt = smem + ((kt + 1) & 1) * STAGE;
        // Behind the last stage nothing is there to be fetched.  The requests go out all the same, to buffers of no extent: with a branch around
        // them the compiler moves the matrix instructions in front of it behind it.
        if (kt + 2 >= nk) {
            rsA[2] = rsB[2] = 0;
#pragma unroll
            for (int x = 0; x < SCALE_PARTS; x++) rsS[x][2] = 0;
        }
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const int step = q / TM, i = q % TM;
            __builtin_amdgcn_sched_barrier(0);
            if (q == Q - AHEAD) {
                // Every wave has its last fragments of this stage, and the next stage has landed for all of them.
                asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < TM; x++) na[x] = A::template scales<WIDE>(nxt + AT_SA, wm + 32 * x);
#pragma unroll
                for (int x = 0; x < TN; x++) nb[x] = B::template scales<WIDE>(nxt + AT_SB, wn + 32 * x);
            }
            const int f = q + AHEAD;
            fa[f % RING] = f < Q ? A::template frag<WIDE>(cur, wm + 32 * (f % TM), f / TM) : A::template frag<WIDE>(nxt, wm + 32 * (f % TM), f / TM - STEPS);
            if (i == TM - 1) {
#pragma unroll
                for (int j = 0; j < TN; j++)
                    fb[(step + 1) & 1][j] = step + 1 < STEPS ? B::template frag<WIDE>(cur + AT_B, wn + 32 * j, step + 1) : B::template frag<WIDE>(nxt + AT_B, wn + 32 * j, 0);
            }
            if (q >= Q - AHEAD) {
#pragma unroll
                for (int x = 0; x < ALL; x++)
                    if (x * AHEAD / ALL == q - (Q - AHEAD)) dma_part(kt & 1, x);
            }
#pragma unroll
            for (int j = 0; j < TN; j++) {
                if constexpr (WIDE) {
#pragma unroll
                    for (int piece = 0; piece < 4; piece++) {
                        const int at = 8 * (2 * step + (piece >> 1));
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(
                            B::widen_piece(fb[step & 1][j], piece, scale_value((uint32_t)sb[j] >> at & 255u)),
                            A::widen_piece(fa[q % RING], piece, scale_value((uint32_t)sa[i] >> at & 255u)), acc[i][j], 0, 0, 0);
                    }
                } else {
                    const i32x8 x = B::operand(fb[step & 1][j]), y = A::operand(fa[q % RING]);
                    if (KS == 256) {
                        acc[i][j] = step == 0 ? mfma_mx<FB, FA, 0, 0>(x, y, acc[i][j], sb[j], sa[i]) : step == 1 ? mfma_mx<FB, FA, 1, 1>(x, y, acc[i][j], sb[j], sa[i])
                                  : step == 2 ? mfma_mx<FB, FA, 2, 2>(x, y, acc[i][j], sb[j], sa[i]) : mfma_mx<FB, FA, 3, 3>(x, y, acc[i][j], sb[j], sa[i]);
                    } else {
                        acc[i][j] = step == 0 ? mfma_mx<FB, FA, 0, 0>(x, y, acc[i][j], sb[j], sa[i]) : mfma_mx<FB, FA, 2, 2>(x, y, acc[i][j], sb[j], sa[i]);
                    }
                }
            }
        }
#pragma unroll
        for (int x = 0; x < TM; x++) sa[x] = na[x];
#pragma unroll
        for (int x = 0; x < TN; x++) sb[x] = nb[x];
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();   // the stages are free for the way out

    // A lane has row lane % 32 of a block and columns 8 g + 4 h .. + 3; through a patch of its own each wave's blocks come back with eight lanes
    // a row, so that stores cover 128-byte (fp32) or 64-byte segments.
    char* const patch = smem + wave * 4096;
    const int r_w = lane & 31, r_r = lane >> 3, c_r = lane & 7;
    const bool whole = p.split == 1;
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) {
#pragma unroll
            for (int g = 0; g < 4; g++)
                *reinterpret_cast<float4*>(patch + r_w * 128 + (((2 * g + h) ^ ((r_w >> 1) & 7)) << 4)) =
                    make_float4(acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]);
            const int col = n0 + wn + 32 * j + 4 * c_r, n = p.N - col;
#pragma unroll
            for (int t = 0; t < 4; t++) {
                const int rr = 8 * t + r_r, row = m0 + wm + 32 * i + rr;
                const float4 v4 = *reinterpret_cast<const float4*>(patch + rr * 128 + ((c_r ^ ((rr >> 1) & 7)) << 4));
                if (row >= p.M || n <= 0) continue;
                float v[4] = {v4.x, v4.y, v4.z, v4.w};
                if (!whole) {
                    Few<float, 4> e;
                    e.round(v);
                    e.store(p.partial + ((long)blockIdx.y * p.M + row) * p.N + col, n);
                } else if constexpr (sizeof(TC) == 4) {
                    float* const c = (float*)p.C + (long)row * p.ldc + col;
                    Few<float, 4> e;
                    if (p.accumulate) {
                        e.load(c, n);
#pragma unroll
                        for (int x = 0; x < 4; x++) v[x] += e.at(x);
                    }
                    e.round(v);
                    e.store(c, n);
                } else {
                    bf16_t* const c = (bf16_t*)p.C + (long)row * p.ldc + col;
                    Few<bf16_t, 4> e;
                    if (p.accumulate) {
                        e.load(c, n);
#pragma unroll
                        for (int x = 0; x < 4; x++) v[x] += e.at(x);
                    }
                    e.round(v);
                    e.store(c, n);
                }
            }
        }
}

template <int FA, int FB, bool WIDE, typename TC, int BM, int BN, int WR, int WC>
static hipError_t launch_tiles(const MxProduct& q, hipStream_t st) {
    constexpr int KS = STAGE_K<FA, FB>, NW = WR * WC;
    using A = MxTile<FA, KS, BM, NW>;
    using B = MxTile<FB, KS, BN, NW>;
    constexpr int LDS = std::max(2 * (A::BYTES + B::BYTES + A::SCALES + B::SCALES), NW * 4096);
    static std::atomic<uint64_t> lds_ok{0};
    auto kern = &k_product_tiles<FA, FB, WIDE, TC, BM, BN, WR, WC>;
    const hipError_t e = allow_lds((const void*)kern, LDS, lds_ok);
    if (e != hipSuccess) return e;
    const long width = mx_width(q.K);
    MxProblem p{};
    p.a = q.a.codes; p.b = q.b.codes; p.sa = q.a.scales; p.sb = q.b.scales;
    p.pitch_a = (uint32_t)(FA == MX_E4M3 ? width : width / 2); p.pitch_b = (uint32_t)(FB == MX_E4M3 ? width : width / 2);
    p.pitch_s = (uint32_t)(width / MX_BLOCK);
    p.a_bytes = (uint32_t)q.M * p.pitch_a; p.b_bytes = (uint32_t)q.N * p.pitch_b;
    p.sa_bytes = (uint32_t)q.M * p.pitch_s; p.sb_bytes = (uint32_t)q.N * p.pitch_s;
    p.C = q.C; p.ldc = q.ldc; p.M = q.M; p.N = q.N; p.accumulate = q.accumulate;
    p.stages = (q.K + KS - 1) / KS;
    p.split = 1;
    p.map = tile_map(q.M, q.N, BM, BN);
    kern<<<p.map.tiles(), 64 * NW, LDS, st>>>(p);
    return hipGetLastError();
}

size_t mx_product_workspace(const MxProduct&) { return 0; }

hipError_t mx_product(const MxProduct& p, void*, hipStream_t st) {
    if ((long)p.M * p.N >= 256 * 256) {
        auto tiles = [&](auto fa, auto fb) {
            constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;
            constexpr bool WIDE = FA == MX_E4M3 || FB == MX_E4M3;
            return p.f32 ? launch_tiles<FA, FB, WIDE, float, 256, 256, 2, 4>(p, st) : launch_tiles<FA, FB, false, bf16_t, 256, 256, 2, 4>(p, st);
        };
        std::integral_constant<int, MX_E4M3> e8;
        std::integral_constant<int, MX_E2M1> e4;
        return p.fa == MX_E4M3 ? (p.fb == MX_E4M3 ? tiles(e8, e8) : tiles(e8, e4)) : (p.fb == MX_E4M3 ? tiles(e4, e8) : tiles(e4, e4));
    }
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
