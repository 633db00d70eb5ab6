// fp32 input gradient of an output projection, dx = d W with k over a vocabulary: an NN product of few tiles and hundreds of k stages,
// cut along k.
//
// v_mfma_f32_32x32x2_f32 on tiles of 64x128, a wave 1x2 blocks of 32x32, two stages of 32 k values, three workgroups a CU.  The
// shares' sums go to the workspace and are added in their order by a second kernel.  gemm_f32.hip walks all of k in one workgroup a tile
// (0.2 us a stage and more), which is the better way only where its 32x32 tiles fill the chip: see gemm_f32_long_k_better.
// Bound by latency on small problems (11x360x19739 40 us with the reduction), by the matrix cores on large ones (441x600x16837 98 us,
// 91 TFLOP/s).
#include <algorithm>

#include "gemm_f32_tile.h"
#include "kernels.h"

namespace hh {

constexpr int LBM = 64, LBN = 128;
struct F32LongK {
    const float *A, *B;
    float *C, *partial;        // partial: [share][tile][LBM * LBN]
    uint32_t a_bytes, b_bytes;
    int lda, ldb, ldc, M, N, K;
    TileMap map;
    Divisor tiles, ksplit;
};

__global__ __launch_bounds__(256, 2) void k_gemm_f32_long_k(F32LongK g) {
    constexpr int BM = LBM, BN = LBN;
    using TA = FTile<true, BM>;
    using TB = FTile<false, BN>;
    constexpr int TM = BM / 64, TN = BN / 64, STAGE = TA::BYTES + TB::BYTES;
    extern __shared__ __attribute__((aligned(1024))) char smem[];   // [stage][A | B]
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, hf = lane >> 5;
    const int wm = (wave >> 1) * (BM / 2), wn = (wave & 1) * (BN / 2);
    int share = (int)blockIdx.x;
    const int tix = split_off(share, g.tiles);
    int tm, tn;
    g.map.tile(tix, tm, tn);
    const int m0 = tm * BM, n0 = tn * BN, K = g.K;
    const int nk_all = (K + FK - 1) / FK;
    const int kbeg = quotient(share * nk_all, g.ksplit), nk = quotient((share + 1) * nk_all, g.ksplit) - kbeg;

    const uint64_t pa = (uint64_t)g.A, pb = (uint64_t)g.B;
    const i32x4 rsA = {(int)(uint32_t)pa, (int)(uint32_t)(pa >> 32), (int)g.a_bytes, 0x00020000};
    const i32x4 rsB = {(int)(uint32_t)pb, (int)(uint32_t)(pb >> 32), (int)g.b_bytes, 0x00020000};
    const uint32_t stepA = TA::kstep_bytes(g.lda), stepB = TB::kstep_bytes(g.ldb);
    typename TA::Src sa[TA::PER_WAVE];
    typename TB::Src sb[TB::PER_WAVE];
#pragma unroll
    for (int i = 0; i < TA::PER_WAVE; i++) { sa[i] = TA::src(wave, i, m0, g.lda); sa[i].off += (uint32_t)kbeg * stepA; }
#pragma unroll
    for (int i = 0; i < TB::PER_WAVE; i++) { sb[i] = TB::src(wave, i, n0, g.ldb); sb[i].off += (uint32_t)kbeg * stepB; }
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem);
    // k values at or past K read as zero, as in gemm_f32.hip
    auto issue = [&](int slot, int kt) {
        const uint32_t base = lds0 + slot * STAGE;
        const int k0 = (kbeg + kt) * FK;
#pragma unroll
        for (int i = 0; i < TA::PER_WAVE; i++) {
            dma16(base + (wave * TA::PER_WAVE + i) * 1024, k0 + sa[i].k >= K ? g.a_bytes : sa[i].off, rsA);
            sa[i].off += stepA;
        }
#pragma unroll
        for (int i = 0; i < TB::PER_WAVE; i++) {
            dma16(base + TA::BYTES + (wave * TB::PER_WAVE + i) * 1024, sb[i].off, rsB);
            sb[i].off += stepB;
        }
    };
    f32x16 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int r = 0; r < 16; r++) acc[i][j][r] = 0.f;
    issue(0, 0);
    for (int kt = 0; kt < nk; kt++) {
        // k tile kt has landed, and everyone has read k tile kt - 1, whose slot is filled next
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        if (kt + 1 < nk) issue((kt + 1) & 1, kt + 1);
        const char* cA = smem + (kt & 1) * STAGE;
        const char* cB = cA + TA::BYTES;
#pragma unroll
        for (int kk = 0; kk < FK / 8; kk++) {
            f32x4 fa[TM], fb[TN];
#pragma unroll
            for (int i = 0; i < TM; i++) fa[i] = TA::frag(cA, wm + 32 * i, kk);
#pragma unroll
            for (int j = 0; j < TN; j++) fb[j] = TB::frag(cB, wn + 32 * j, kk);
#pragma unroll
            for (int e = 0; e < 4; e++)
#pragma unroll
                for (int i = 0; i < TM; i++)
#pragma unroll
                    for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x2f32(fb[j][e], fa[i][e], acc[i][j], 0, 0, 0);
        }
    }
    float* pt = g.partial + ((size_t)share * g.tiles.d + tm * g.map.tiles_n + tn) * (BM * BN);
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++)
#pragma unroll
            for (int q = 0; q < 4; q++)
                *reinterpret_cast<float4*>(pt + (wm + 32 * i + (lane & 31)) * BN + wn + 32 * j + 8 * q + 4 * hf) =
                    make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
}

// The shares of a tile one after the other; a thread owns 4 columns of a row.
__global__ __launch_bounds__(256) void k_f32_long_k_reduce(F32LongK g) {
    constexpr int PER = LBM * LBN / 1024;
    const int tile = (int)blockIdx.x / PER, at = ((int)blockIdx.x % PER) * 1024 + (int)threadIdx.x * 4;
    const int tm = tile / g.map.tiles_n, tn = tile - tm * g.map.tiles_n;
    const int m = tm * LBM + at / LBN, n = tn * LBN + at % LBN;
    if (m >= g.M || n >= g.N) return;
    const float* p = g.partial + (size_t)tile * (LBM * LBN) + at;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int s = 0; s < g.ksplit.d; s++) {
        const float4 u = *reinterpret_cast<const float4*>(p + (size_t)s * g.tiles.d * (LBM * LBN));
        v.x += u.x; v.y += u.y; v.z += u.z; v.w += u.w;
    }
    *reinterpret_cast<float4*>(g.C + (size_t)m * g.ldc + n) = v;
}

// Where the product is better cut: 32x32 tiles that do not fill the chip, and a long k.  On 118 random steps (1 to 4000 tokens, hidden 64
// to 4096, vocabulary 500 to 32000) this choice is within 1 % of the better one of each; both gradients' products take 0.75 of the time
// they take where none is cut (11 tokens, hidden 360, vocabulary 19739: 235 -> 53 us; 441, 600, 16837: 249 -> 191), and longer
// outside: 333, 2048, 10000 243 -> 271, 1072, 584, 8410 212 -> 253, 630, 256, 2302 26 -> 34.
bool gemm_f32_long_k_better(int M, int N, int K) { return K >= 2500 && (long)((M + 31) / 32) * ((N + 31) / 32) <= 400; }

// Shares: the least work of the busiest CU, in multiply-adds of its tiles (they share its matrix cores) with 48 k values for the
// beginning and end of each, and 40 for a number of a share that is added.
static int shares(long tiles, int M, int N, int nk, size_t ws_bytes) {
    int best = 1;
    double least = 1e300;
    for (const int s : {1, 2, 3, 4, 5, 6, 8, 10, 12, 16, 20, 24, 32, 40, 48, 64}) {
        if ((size_t)tiles * s * LBM * LBN * 4 > ws_bytes || (s > 1 && nk / s < 4)) break;
        const double t = (double)((tiles * s + 255) / 256) * LBM * LBN * ((double)nk * FK / s + 48.0) + 40.0 * s * M * N / 256;
        if (t < least) { least = t; best = s; }
    }
    return best;
}

hipError_t gemm_f32_long_k(const GemmDesc& d, hipStream_t st) {
    if (d.kind != GEMM_NN || d.M <= 0 || d.N <= 0 || d.K <= 0 || d.k1 || d.micro > 1 || d.R || d.accumulate || d.fuse.kind) return hipErrorInvalidValue;
    const long a_bytes = ((long)(d.M - 1) * d.lda + d.K) * 4, b_bytes = ((long)((d.b_rows ? d.b_rows : d.K) - 1) * d.ldb + d.N) * 4;
    // 32-bit byte offsets, which run past the end by at most the 64 rows of a tile
    if (a_bytes >= (1L << 32) - (1L << 25) || b_bytes >= (1L << 32) - (1L << 25)) return hipErrorInvalidValue;
    if (d.lda > MAX_LD || d.ldb > MAX_LD || a_bytes + 256L * d.lda >= (1L << 32) || b_bytes + 256L * d.ldb >= (1L << 32)) return hipErrorInvalidValue;
    if (d.N % 4 || d.ldc % 4 || d.lda % 4 || d.ldb % 4 || d.K % 4) return hipErrorInvalidValue;
    F32LongK p{};
    p.A = (const float*)d.A; p.B = (const float*)d.B; p.C = (float*)d.C; p.partial = (float*)d.ws;
    p.a_bytes = (uint32_t)a_bytes; p.b_bytes = (uint32_t)b_bytes;
    p.lda = d.lda; p.ldb = d.ldb; p.ldc = d.ldc; p.M = d.M; p.N = d.N; p.K = d.K;
    p.map = tile_map(d.M, d.N, LBM, LBN);
    const int tiles = p.map.tiles();
    if (!d.ws || (size_t)tiles * LBM * LBN * 4 > d.ws_bytes) return hipErrorInvalidValue;
    p.tiles = divisor(tiles);
    p.ksplit = divisor(shares(tiles, d.M, d.N, (d.K + FK - 1) / FK, d.ws_bytes));
    constexpr int LDS = 2 * (LBM + LBN) * FK * 4;
    static_assert(LDS <= 48 * 1024, "no raised LDS limit");
    k_gemm_f32_long_k<<<tiles * p.ksplit.d, 256, LDS, st>>>(p);
    k_f32_long_k_reduce<<<tiles * (LBM * LBN / 1024), 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace hh
