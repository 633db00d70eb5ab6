// C (=|+=) A B^T of two microscaled operands on the matrix cores.
#include <algorithm>
#include <type_traits>

#include "gemm_tile.h"
#include "mx.h"

namespace hh {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// ------------------------------------------------------------------ few rows
// C of up to 16 TM rows: 16 columns a workgroup, its waves take 256 k at a time in turn, straight from memory into registers, and their sums
// meet in LDS.  Bound by the one read of B: nothing of it is used twice, so it has no use for LDS, and what counts is that every wave of the
// chip has its whole share under way at once: 1x4096x11008 E4M3 by E2M1 7.6 us (24 MB, 3.2 TB/s; a launch that does nothing is 2 of them).  One
// after another, with B from memory, 8.6, E2M1 twice 7.8, E4M3 twice 14.5 (3.2 TB/s); of 32 rows 18.8, 13.0, 25.0: what else there is, and
// widening on either side.
//
// Of 16 rows x 128 k lane l holds row l % 16 and, with q = l / 16, the codes 32 q .. 32 q + 31 with their one scale: of E2M1 on both sides what the
// matrix instruction takes, otherwise (WIDE) eight at a time, widened, whatever k they are of, the same for both operands.
typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));
// The conversions take a scale's exponent alone, of which 0 is 2^-127 and 255 NaN to them.  What they make is exact where bfloat16 holds
// it, rounded to nearest below 2^-130 and infinite from 2^128 on.
__device__ __forceinline__ float scale_bits(uint32_t byte) { return __uint_as_float(byte << 23); }
template <int F> __device__ __forceinline__ bf16x8 widen8(uint32_t lo, uint32_t hi, float scale);   // 8 codes (E2M1: of lo) with their scale
template <> __device__ __forceinline__ bf16x8 widen8<MX_E4M3>(uint32_t lo, uint32_t hi, float scale) {
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
    const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
template <> __device__ __forceinline__ bf16x8 widen8<MX_E2M1>(uint32_t lo, uint32_t, float scale) {
    const bf16x2v a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(lo, scale, 0), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(lo, scale, 1);
    const bf16x2v c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(lo, scale, 2), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(lo, scale, 3);
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

template <int F>
struct RowUnit {   // 256 k of the lane's row
    i32x4 v[F == MX_E4M3 ? 4 : 2];
    uint2 s;
    __device__ __forceinline__ void load(const uint8_t* codes, const uint8_t* scales, int unit, int q) {
        constexpr int HALF = F == MX_E4M3 ? 2 : 1;   // loads
#pragma unroll
        for (int i = 0; i < 2 * HALF; i++)
            v[i] = *reinterpret_cast<const i32x4*>(codes + (128 * (long)unit + 64 * (i / HALF) + 16 * q) * HALF + 16 * (i % HALF));
        s = *reinterpret_cast<const uint2*>(scales + 8 * (long)unit);
    }
    __device__ __forceinline__ i32x8 operand(int half) const {   // E2M1, as the matrix instruction takes it
        const i32x4 a = v[half];
        return i32x8{a[0], a[1], a[2], a[3], 0, 0, 0, 0};
    }
    __device__ __forceinline__ uint32_t scale(int half, int q) const { return (half ? s.y : s.x) >> (8 * q); }
    // codes 8 eight .. of the 32
    __device__ __forceinline__ bf16x8 widened(int half, int eight, float scale) const {
        if constexpr (F == MX_E4M3) {
            const i32x4 a = v[2 * half + (eight >> 1)];
            return widen8<F>((uint32_t)a[2 * (eight & 1)], (uint32_t)a[2 * (eight & 1) + 1], scale);
        } else {
            return widen8<F>((uint32_t)v[half][eight], 0u, scale);
        }
    }
};

template <int F> constexpr int FORMAT = F == MX_E4M3 ? 0 : 4;   // of the matrix instruction
struct MxRowsProblem { const uint8_t *a, *b, *sa, *sb; void* C; long ldc; int M, N, units, accumulate; uint32_t pitch_a, pitch_b, pitch_s; };

template <int FA, int FB, typename TC, int TM, int NW>
__global__ __launch_bounds__(64 * NW) void k_product_rows(MxRowsProblem p) {
    constexpr bool WIDE = FA == MX_E4M3 || FB == MX_E4M3;
    __shared__ float part[NW][TM][256];
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63, q = lane >> 4, l = lane & 15;
    const int n0 = (int)blockIdx.x * 16;
    const uint32_t rb = (uint32_t)min(n0 + l, p.N - 1);   // rows past the end: any, their results are dropped
    const uint8_t* const b = p.b + (size_t)rb * p.pitch_b;
    const uint8_t* const sb = p.sb + (size_t)rb * p.pitch_s;
    const uint8_t *a[TM], *sa[TM];
    f32x4 acc[TM];
#pragma unroll
    for (int i = 0; i < TM; i++) {
        const uint32_t ra = (uint32_t)min(16 * i + l, p.M - 1);
        a[i] = p.a + (size_t)ra * p.pitch_a;
        sa[i] = p.sa + (size_t)ra * p.pitch_s;
        acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll 4
    for (int u = wave; u < p.units; u += NW) {
        RowUnit<FB> ub;
        RowUnit<FA> ua[TM];
        ub.load(b, sb, u, q);
#pragma unroll
        for (int i = 0; i < TM; i++) ua[i].load(a[i], sa[i], u, q);
#pragma unroll
        for (int half = 0; half < 2; half++) {
            if constexpr (WIDE) {
                const float xb = scale_bits(ub.scale(half, q) & 255u);
                float xa[TM];
#pragma unroll
                for (int i = 0; i < TM; i++) xa[i] = scale_bits(ua[i].scale(half, q) & 255u);
#pragma unroll
                for (int eight = 0; eight < 4; eight++) {
                    const bf16x8 w = ub.widened(half, eight, xb);
#pragma unroll
                    for (int i = 0; i < TM; i++) acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, ua[i].widened(half, eight, xa[i]), acc[i], 0, 0, 0);
                }
            } else {
#pragma unroll
                for (int i = 0; i < TM; i++)
                    acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(ub.operand(half), ua[i].operand(half), acc[i], FORMAT<FB>, FORMAT<FA>, 0,
                                                                            (int)ub.scale(half, q), 0, (int)ua[i].scale(half, q));
            }
        }
    }
    // a lane has row l of a block of C and columns 4 q .. 4 q + 3
#pragma unroll
    for (int i = 0; i < TM; i++) *reinterpret_cast<f32x4*>(&part[wave][i][16 * l + 4 * q]) = acc[i];
    __syncthreads();
    for (int e = (int)threadIdx.x; e < 256 * TM; e += 64 * NW) {
        const int m = e >> 4, n = n0 + (e & 15);
        if (m >= p.M || n >= p.N) continue;
        float v = 0.f;
#pragma unroll
        for (int w = 0; w < NW; w++) v += part[w][e >> 8][e & 255];
        if constexpr (sizeof(TC) == 4) {
            float* const c = (float*)p.C + (long)m * p.ldc + n;
            *c = p.accumulate ? *c + v : v;
        } else {
            bf16_t* const c = (bf16_t*)p.C + (long)m * p.ldc + n;
            *c = f2bf(p.accumulate ? bf2f(*c) + v : v);
        }
    }
}

// ------------------------------------------------------------------ tiles
// BM x BN of C a workgroup, WR x WC waves, each 32 TM x 32 TN.  k advances KS at a time through NS LDS stages that are filled straight from
// global memory; a row of a stage is KS bytes of E4M3 or KS / 2 of E2M1 (KS 128, or 256), and the scales of those k lie behind the
// tiles.  16-byte chunks are XOR-swizzled by the row so that a fragment's 16 lanes cover all banks.
//
// 4096x8192x12288 into bf16: E2M1 223 us (3.70 PFLOP/s; 214 to 223 from card to card), with fast sums E4M3 376 (2.19) and E4M3 by E2M1 318
// (2.60), widened 601 (1.37) and 574 (1.44), widened into fp32 595 (1.39).  The matrix cores alone, with random operands in registers, reach
// 6.8, 4.0 (both with an E4M3 operand) and (bf16) 1.8 PFLOP/s under the power limit.  Counters (E2M1, where it took 214): matrix
// cores busy 51 % of the cycles at 1.85 GHz, workgroups there 91 % (two tiles a compute unit, each with its start and end), waits 33 %,
// for LDS 3 %.  Without the loop's requests it takes 168 us, without the matrix instructions 165, with every request in L2 203: neither
// side is the limit by itself, and the two add up to more than either.  Four waves of 128x128, four stages of 128 k (268), fragments fetched
// earlier or later, requests spread wider and raised wave priorities changed nothing or cost time.
template <int F, int KS> constexpr int ROW_BYTES = F == MX_E4M3 ? KS : KS / 2;
template <int RB> __device__ __forceinline__ int turned(int row, int chunk) {
    return RB == 256 ? chunk ^ (row & 15) : RB == 128 ? chunk ^ ((row >> 1) & 7) : chunk ^ ((row >> 2) & 3);
}
template <int RB> __device__ __forceinline__ int swizzled(int row, int chunk) { return row * RB + (turned<RB>(row, chunk) << 4); }   // byte in the tile
template <int FA, int FB> constexpr int STAGE_K = FA == MX_E2M1 && FB == MX_E2M1 ? 256 : 128;

__device__ __forceinline__ void dma4(uint32_t lds_addr, uint32_t voff, i32x4 rs) {   // as dma16, four bytes a lane
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds_addr), "v"(voff), "s"(rs) : "memory");
}
__device__ __forceinline__ i32x4 rsrc_words(const void* p, uint32_t bytes) {
    const uint64_t a = (uint64_t)p;
    return i32x4{(int)(uint32_t)a, (int)(uint32_t)(a >> 32), (int)bytes, 0x00020000};
}

// One operand's share of a stage: its tile and its scales.  Of 32 rows x 64 k lane l holds row l % 32 and, with h = l / 32, of E2M1 the codes
// k = 32 h .. 32 h + 31, of E4M3 (and WIDE) 16 h .. 16 h + 15 and 32 + 16 h .. 32 + 16 h + 15; its scale is that of k = 32 h .. 32 h + 31.
template <int F, int KS, int ROWS, int NW>
struct MxTile {
    static constexpr int RB = ROW_BYTES<F, KS>, SB = KS / MX_BLOCK, BYTES = ROWS * RB, SCALES = ROWS * SB;
    static constexpr int PER_WAVE = BYTES / 1024 / NW;             // instructions of 1 KB
    static_assert(PER_WAVE * NW * 1024 == BYTES, "the tile splits evenly over the waves");
    static constexpr int SCALE_PARTS = SCALES / 256;               // instructions of 256 bytes, over all waves
    __device__ static __forceinline__ uint32_t voff(int wave, int i, int row0, uint32_t pitch) {
        constexpr int LPR = RB / 16;
        const int L = threadIdx.x & 63, r = (wave * PER_WAVE + i) * (64 / LPR) + L / LPR;
        return (uint32_t)(row0 + r) * pitch + (uint32_t)(turned<RB>(r, L % LPR) * 16);
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
        if constexpr (F == MX_E4M3) return widen8<F>((uint32_t)f.v[piece >> 1][2 * (piece & 1)], (uint32_t)f.v[piece >> 1][2 * (piece & 1) + 1], scale);
        else return widen8<F>((uint32_t)f.v[0][piece], 0u, scale);
    }
    // The scales of a stage for rows rb .. rb + 31, as they lie in LDS, and what the products take.  Not WIDE, byte (KS 256: s, KS 128: 2 s) is
    // that of step s for this lane's half; WIDE, those of step s are bytes 2 s and 2 s + 1.
    struct Scales {
        uint32_t w[SB / 4];
        __device__ __forceinline__ float of(int block) const { return scale_bits(w[block >> 2] >> (8 * (block & 3)) & 255u); }
    };
    __device__ static __forceinline__ Scales scales(const char* lds, int rb) {
        const int r = rb + (int)(threadIdx.x & 31);
        Scales s;
        if constexpr (SB == 8) {
            const uint2 w = *reinterpret_cast<const uint2*>(lds + 8 * r);
            s.w[0] = w.x;
            s.w[1] = w.y;
        } else {
            s.w[0] = *reinterpret_cast<const uint32_t*>(lds + 4 * r);
        }
        return s;
    }
    template <bool WIDE> __device__ static __forceinline__ Scales ordered(Scales s) {
        const int h = (int)(threadIdx.x & 63) >> 5;
        if constexpr (WIDE) return s;
        if constexpr (SB == 8) s.w[0] = __builtin_amdgcn_perm(s.w[1], s.w[0], h ? 0x07050301u : 0x06040200u);
        else s.w[0] >>= 8 * h;
        return s;
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

template <int FA, int FB, bool WIDE, typename TC, int KS, int BM, int BN, int WR, int WC, int NS>
__global__ __launch_bounds__(64 * WR * WC) void k_product_tiles(MxProblem p) {
    constexpr int NW = WR * WC, TM = BM / WR / 32, TN = BN / WC / 32, STEPS = KS / 64, Q = STEPS * TM;
    using A = MxTile<FA, KS, BM, NW>;
    using B = MxTile<FB, KS, BN, NW>;
    constexpr int STAGE = A::BYTES + B::BYTES + A::SCALES + B::SCALES, AT_B = A::BYTES, AT_SA = AT_B + B::BYTES, AT_SB = AT_SA + A::SCALES;
    constexpr int PARTS = A::PER_WAVE + B::PER_WAVE, SCALE_PARTS = (A::SCALE_PARTS + B::SCALE_PARTS + NW - 1) / NW;
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
    for (int i = 0; i < SCALE_PARTS; i++) {   // of A, then of B; where there are fewer than waves, some fetch the same
        const int part = (uwave + NW * i) % (A::SCALE_PARTS + B::SCALE_PARTS), of_b = part - A::SCALE_PARTS;
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
    // Behind the last stage nothing is there to be fetched.  The requests go out all the same, to buffers of no extent: with a branch around
    // them the compiler moves the matrix instructions in front of it behind it.
    auto past_the_end = [&](bool past) {
        if (past) {
            rsA[2] = rsB[2] = 0;
#pragma unroll
            for (int x = 0; x < SCALE_PARTS; x++) rsS[x][2] = 0;
        }
    };
#pragma unroll
    for (int s = 0; s < NS; s++) {
        past_the_end(s >= nk);
#pragma unroll
        for (int i = 0; i < ALL; i++) dma_part(s, i);
    }
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * ALL) : "memory");
    __syncthreads();

    // Fragments of A are fetched AHEAD of their products, those of B a step ahead; scales with the first fragments of their stage.
    // AHEAD is at most TM: the last fragments of B that a stage has are asked for in its last step but one, which has to be before the barrier.
    constexpr int AHEAD = TM >= 4 ? 3 : TM, RING = AHEAD == 1 ? 2 : 4;
    static_assert(AHEAD <= TM && AHEAD < RING, "see above");
    static_assert(Q % RING == 0 && STEPS % 2 == 0, "a stage ends where it began in both rings");
    typename A::Frag fa[RING];
    typename B::Frag fb[2][TN];
    typename A::Scales sa[TM], na[TM];
    typename B::Scales sb[TN], nb[TN];
#pragma unroll
    for (int q = 0; q < AHEAD; q++) fa[q] = A::template frag<WIDE>(smem, wm + 32 * (q % TM), q / TM);
#pragma unroll
    for (int j = 0; j < TN; j++) fb[0][j] = B::template frag<WIDE>(smem + AT_B, wn + 32 * j, 0);
#pragma unroll
    for (int i = 0; i < TM; i++) sa[i] = A::template ordered<WIDE>(A::scales(smem + AT_SA, wm + 32 * i));
#pragma unroll
    for (int j = 0; j < TN; j++) sb[j] = B::template ordered<WIDE>(B::scales(smem + AT_SB, wn + 32 * j));
    int slot = 0;
    for (int kt = 0; kt < nk; kt++) {
        const int next = slot + 1 == NS ? 0 : slot + 1;
        const char* const cur = smem + slot * STAGE;
        const char* const nxt = smem + next * STAGE;
        past_the_end(kt + NS >= nk);
#pragma unroll
        for (int q = 0; q < Q; q++) {
            const int step = q / TM, i = q % TM;
            __builtin_amdgcn_sched_barrier(0);
            if (q == Q - AHEAD) {
                // Every wave has its last fragments of this stage, and the next stage has landed for all of them.
                asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((NS - 2) * ALL) : "memory");
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
                __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                for (int x = 0; x < TM; x++) na[x] = A::scales(nxt + AT_SA, wm + 32 * x);
#pragma unroll
                for (int x = 0; x < TN; x++) nb[x] = B::scales(nxt + AT_SB, wn + 32 * x);
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
                    if (x * AHEAD / ALL == q - (Q - AHEAD)) dma_part(slot, x);
            }
#pragma unroll
            for (int j = 0; j < TN; j++) {
                if constexpr (WIDE) {
#pragma unroll
                    for (int piece = 0; piece < 4; piece++) {
                        const int block = 2 * step + (piece >> 1);
                        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(B::widen_piece(fb[step & 1][j], piece, sb[j].of(block)),
                                                                            A::widen_piece(fa[q % RING], piece, sa[i].of(block)), acc[i][j], 0, 0, 0);
                    }
                } else {
                    const i32x8 x = B::operand(fb[step & 1][j]), y = A::operand(fa[q % RING]);
                    const int ys = (int)sa[i].w[0], xs = (int)sb[j].w[0];
                    if (KS == 256) {
                        acc[i][j] = step == 0 ? mfma_mx<FB, FA, 0, 0>(x, y, acc[i][j], xs, ys) : step == 1 ? mfma_mx<FB, FA, 1, 1>(x, y, acc[i][j], xs, ys)
                                  : step == 2 ? mfma_mx<FB, FA, 2, 2>(x, y, acc[i][j], xs, ys) : mfma_mx<FB, FA, 3, 3>(x, y, acc[i][j], xs, ys);
                    } else {
                        acc[i][j] = step == 0 ? mfma_mx<FB, FA, 0, 0>(x, y, acc[i][j], xs, ys) : mfma_mx<FB, FA, 2, 2>(x, y, acc[i][j], xs, ys);
                    }
                }
            }
        }
        __builtin_amdgcn_sched_barrier(0);   // the scales have had the last products' time to arrive
#pragma unroll
        for (int x = 0; x < TM; x++) sa[x] = A::template ordered<WIDE>(na[x]);
#pragma unroll
        for (int x = 0; x < TN; x++) sb[x] = B::template ordered<WIDE>(nb[x]);
        slot = next;
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

// C (+)= sum of the shares of k, in their order
template <typename TC>
__global__ __launch_bounds__(256) void k_sum_shares(const float* __restrict__ partial, int shares, int groups, Divisor per_row, int M, int N, TC* C, long ldc,
                                                     int accumulate) {
    const int i = (int)(blockIdx.x * 256u + threadIdx.x);
    if (i >= groups) return;
    int row = i;
    const int col = 4 * split_off(row, per_row), n = N - col;
    float v[4] = {0.f, 0.f, 0.f, 0.f};
    for (int s = 0; s < shares; s++) {
        Few<float, 4> e;
        e.load(partial + ((long)s * M + row) * N + col, n);
#pragma unroll
        for (int x = 0; x < 4; x++) v[x] += e.at(x);
    }
    TC* const c = C + row * ldc + col;
    Few<TC, 4> e;
    if (accumulate) {
        e.load(c, n);
#pragma unroll
        for (int x = 0; x < 4; x++) v[x] += e.at(x);
    }
    e.round(v);
    e.store(c, n);
}

// Which kernel takes a product, and how many shares of k: the least predicted time.  A workgroup of tiles takes ENDS_US to start and to write
// its tile and STAGE_US a stage (256 k of E2M1, else 128), the same alone on its compute unit as beside another one; shares cost a second
// launch and the traffic of their sums.  Against the best of all plans, at 64 shapes and formats of 40 to 8192 rows, it is within 5 % in 59
// of them and 15 % off at worst; 1003x700x2050, E4M3 by E2M1 with fast sums and operands in the caches: tiles of 64 6.5 us, of 128 11.0, of 256
// 24; 2048x4096x4096 65, 43.5, 45; 4096x4096x4096 118, 87, 59.5.
enum { ROWS_16, ROWS_32, TILES_64, TILES_128, TILES_256 };
struct MxPlan { int kernel, split; };
// The instruction for E4M3 adds its products in fewer bits than fp32's: taken only where the caller allows it, the result has fewer still and it is
// faster, which it is not for few rows: 1, 16 and 32 x 4096 x 4096, E4M3 by E2M1, 4.8, 6.4 and 8.9 us widened, 5.1, 6.7 and 9.1 by that
// instruction; E4M3 twice 6.4, 7.8, 10.6 and 6.4, 7.7, 10.1.
static bool widened(const MxProduct& p) { return (p.fa == MX_E4M3 || p.fb == MX_E4M3) && (p.f32 || !p.fast || p.M <= 32); }
constexpr int CUS = 256;
static long tiles_of(const MxProduct& p, int b) { return (long)((p.M + b - 1) / b) * ((p.N + b - 1) / b); }
static MxPlan plan(const MxProduct& p) {
    if (p.M <= 16) return {ROWS_16, 1};
    if (p.M <= 32) return {ROWS_32, 1};
    const bool four = p.fa == MX_E2M1 && p.fb == MX_E2M1;
    constexpr float STAGE_US[3][3] = {{0.32f, 0.78f, 2.15f}, {0.26f, 0.65f, 1.85f}, {0.46f, 1.05f, 3.4f}};   // E2M1, E4M3, widened
    constexpr float ENDS_US[3] = {0.7f, 2.2f, 3.5f};
    const float* const us = STAGE_US[four ? 0 : widened(p) ? 2 : 1];
    const int stages = (p.K + (four ? 255 : 127)) / (four ? 256 : 128);
    MxPlan best{TILES_64, 1};
    float least = 0.f;
    for (int i = 0; i < 3; i++) {
        const long tiles = tiles_of(p, 64 << i);
        for (int split = 1; split <= 16 && (split == 1 || (stages >= 2 * split && tiles * split <= 2 * CUS)); split *= 2) {
            const long rounds = (tiles * split + CUS - 1) / CUS;
            float t = 2.f + (float)rounds * (ENDS_US[i] + (float)((stages + split - 1) / split) * us[i]);
            if (split > 1) t += 2.5f + (float)p.M * (float)p.N * (float)(4 * (split + 1)) / 2e6f;
            if (least == 0.f || t < least) { least = t; best = {TILES_64 + i, split}; }
        }
    }
    return best;
}

template <int FA, int FB, bool WIDE, typename TC, int KS, int BM, int BN, int WR, int WC, int NS>
static hipError_t launch_tiles(const MxProduct& q, int split, void* ws, hipStream_t st) {
    constexpr int NW = WR * WC;
    using A = MxTile<FA, KS, BM, NW>;
    using B = MxTile<FB, KS, BN, NW>;
    constexpr int LDS = std::max(NS * (A::BYTES + B::BYTES + A::SCALES + B::SCALES), NW * 4096);
    static std::atomic<uint64_t> lds_ok{0};
    auto kern = &k_product_tiles<FA, FB, WIDE, TC, KS, BM, BN, WR, WC, NS>;
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
    p.split = split;
    p.partial = (float*)ws;
    p.map = tile_map(q.M, q.N, BM, BN);
    kern<<<dim3(p.map.tiles(), split), 64 * NW, LDS, st>>>(p);
    if (split > 1) {
        const int per_row = (q.N + 3) / 4, groups = q.M * per_row;
        k_sum_shares<TC><<<(groups + 255) / 256, 256, 0, st>>>(p.partial, split, groups, divisor(per_row), q.M, q.N, (TC*)q.C, q.ldc, q.accumulate);
    }
    return hipGetLastError();
}
template <int FA, int FB, typename TC, int TM>
static hipError_t launch_rows(const MxProduct& q, hipStream_t st) {
    const long width = mx_width(q.K);
    const MxRowsProblem p{q.a.codes, q.b.codes, q.a.scales, q.b.scales, q.C, q.ldc, q.M, q.N, (int)(width / 256), q.accumulate,
                          (uint32_t)(FA == MX_E4M3 ? width : width / 2), (uint32_t)(FB == MX_E4M3 ? width : width / 2), (uint32_t)(width / MX_BLOCK)};
    const int grid = (q.N + 15) / 16;
    if (p.units <= 4) k_product_rows<FA, FB, TC, TM, 4><<<grid, 256, 0, st>>>(p);
    else if (p.units <= 8) k_product_rows<FA, FB, TC, TM, 8><<<grid, 512, 0, st>>>(p);
    else k_product_rows<FA, FB, TC, TM, 16><<<grid, 1024, 0, st>>>(p);
    return hipGetLastError();
}

// The kernel and the shares of k of a product, 100 kernel + shares: for tests, not in the public headers.
extern "C" int hh_internal_mx_plan(int m, int n, int k, int a_format, int b_format, int how) {
    const MxPlan l = plan(MxProduct{m, n, k, a_format, b_format, {}, {}, nullptr, n, how == 1, 0, how == 2});
    return 100 * l.kernel + l.split;
}

size_t mx_product_workspace(const MxProduct& p) {
    const MxPlan l = plan(p);
    return l.split > 1 ? (size_t)l.split * p.M * p.N * sizeof(float) : 0;
}

template <int FA, int FB, bool WIDE, typename TC>
static hipError_t run_product(const MxProduct& p, void* ws, hipStream_t st) {
    // Stages (operands in the caches, fast sums but where they are widened): three hide a request's way where LDS has room for them, which it has
    // where one side is half the bytes (4096x8192x12288 E4M3 by E2M1 5 % faster), for tiles of 64 (four are 2 % slower, two up to 30 %), and for one
    // workgroup of tiles of 128 on a compute unit (2048x2048x8192 E4M3 57.4 -> 45.0), where a second one does so too (2048x4096x4096, two of
    // them: 47.7, one at a time 50.3).  Tiles of 64 that are widened do better with two stages of 256 k, half as many ends of one (E4M3 by E2M1
    // 1024x1024x4096 18.5 -> 16.3 us, 1003x700x2050 11.2 -> 10.4); the others do not (11.2 and 12.1, 7.3 and 7.9).
    constexpr int NS = FA == FB ? 2 : 3, KS = STAGE_K<FA, FB>;
    const MxPlan l = plan(p);
    switch (l.kernel) {
        case ROWS_16: return launch_rows<FA, FB, TC, 1>(p, st);
        case ROWS_32: return launch_rows<FA, FB, TC, 2>(p, st);
        case TILES_64: return launch_tiles<FA, FB, WIDE, TC, WIDE ? 256 : KS, 64, 64, 2, 2, WIDE ? 2 : 3>(p, l.split, ws, st);
        case TILES_128:
            if constexpr (NS == 2)
                if (tiles_of(p, 128) * l.split > CUS) return launch_tiles<FA, FB, WIDE, TC, KS, 128, 128, 2, 2, 2>(p, l.split, ws, st);
            return launch_tiles<FA, FB, WIDE, TC, KS, 128, 128, 2, 2, 3>(p, l.split, ws, st);
        default: return launch_tiles<FA, FB, WIDE, TC, KS, 256, 256, 2, 4, NS>(p, l.split, ws, st);
    }
}
hipError_t mx_product(const MxProduct& p, void* ws, hipStream_t st) {
    auto run = [&](auto fa, auto fb) {
        constexpr int FA = decltype(fa)::value, FB = decltype(fb)::value;
        constexpr bool WIDE = FA == MX_E4M3 || FB == MX_E4M3;
        if (p.f32) return run_product<FA, FB, WIDE, float>(p, ws, st);
        return widened(p) ? run_product<FA, FB, WIDE, bf16_t>(p, ws, st) : run_product<FA, FB, false, bf16_t>(p, ws, st);
    };
    std::integral_constant<int, MX_E4M3> e8;
    std::integral_constant<int, MX_E2M1> e4;
    return p.fa == MX_E4M3 ? (p.fb == MX_E4M3 ? run(e8, e8) : run(e8, e4)) : (p.fb == MX_E4M3 ? run(e4, e8) : run(e4, e4));
}

}  // namespace hh
