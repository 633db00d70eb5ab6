// Packing to microscaled formats and back.
#include <type_traits>

#include "mx.h"

namespace hh {

// Packing.  A block's scale is the exponent of its largest magnitude, which is compared as an integer, and the conversions take values as they lie
// in memory, two at a time, with the scale: one read, one pass, one rounding.  Bound by memory.

// ------------------------------------------------------------------ by row
// Eight values a lane, four lanes a block; past the caches two such chunks a lane, with both loads under way, and codes that go past them too:
// 11008x4096 bf16 to E2M1 18.5 us (6.1 TB/s; one chunk 21.0, stores through the caches 19.3, both 22.7), to E4M3 22.4 (26.0).  Small tensors
// lose by the second chunk (333x2050 2.3 -> 2.6).
template <bool STREAM> constexpr int chunks_each() { return STREAM ? 2 : 1; }
template <typename T, int F, bool STREAM>
__global__ __launch_bounds__(256) void k_pack_rows(int chunks, Divisor per_row, int cols, const T* __restrict__ x, long ldx, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales) {
    constexpr int EACH = chunks_each<STREAM>();
    const unsigned first = blockIdx.x * (256u * EACH) + threadIdx.x;
    Eight<T> e[EACH];
#pragma unroll
    for (int c = 0; c < EACH; c++) {
        e[c] = Eight<T>{};
        if (first + 256u * c >= (unsigned)chunks) continue;   // whole rows of a multiple of 32 chunks
        int row = (int)(first + 256u * c);
        const int group = split_off(row, per_row), n = cols - 8 * group;
        if (n > 0) e[c].template load<STREAM>(x + row * ldx + 8L * group, n);
    }
#pragma unroll
    for (int c = 0; c < EACH; c++) {
        const unsigned i = first + 256u * c;
        if (i >= (unsigned)chunks) return;
        const Packer<F> q(quad_max(Magnitudes<T, 8>(e[c]).largest()));
        const Pair<T> pairs[4] = {pair_of(e[c], 0), pair_of(e[c], 1), pair_of(e[c], 2), pair_of(e[c], 3)};
        q.template store8<STREAM>(pairs, codes, i);
        store_scales(scales + (i >> 2), q.byte);
    }
}

// ------------------------------------------------------------------ by column, and both
// A workgroup takes 256 rows x 128 columns, a lane 4 columns of a block of 32 rows in registers: blocks along columns need no exchange at all,
// those along rows one of eight lanes, and x is read once for both.  Codes and scales go out through LDS, whole lines at a time.
// 11008x4096 bf16 from memory, both ways, to E2M1 32.3 us (4.3 TB/s; 35.8 straight from registers, 16 and 2 bytes a lane; packing twice 43), to E4M3
// 40.9; by column alone 21.6 and 26.2.  Without any store it is 22, of which the rows' part of the arithmetic is 8.
constexpr int PACK_ROWS = 256, PACK_COLS = 128;
template <typename T, int F, bool ROWS, bool STREAM>
__global__ __launch_bounds__(256) void k_pack_columns(long rows, int cols, const T* __restrict__ x, long ldx, int width, uint8_t* __restrict__ codes,
                                                       uint8_t* __restrict__ scales, long column_width, uint8_t* __restrict__ column_codes,
                                                       uint8_t* __restrict__ column_scales, Divisor tiles_in_line) {
    constexpr int BITS = F == MX_E4M3 ? 8 : 4, CODES = PACK_ROWS * PACK_COLS * BITS / 8, ROW = PACK_COLS * BITS / 8, COLUMN = PACK_ROWS * BITS / 8;
    constexpr int CHUNKS = COLUMN / 16;   // of a column in LDS, turned by it
    __shared__ __attribute__((aligned(16))) uint8_t smem[CODES + PACK_ROWS * PACK_COLS / MX_BLOCK];
    const int t = (int)threadIdx.x, lane = t & 63, block = 2 * (t >> 6) + (lane >> 5), c = 4 * (lane & 31);
    // Each die takes a run of tiles (workgroups go to the eight of them in turn), so that the tiles that share a line of what is written meet
    // in one L2.
    const int run = (int)gridDim.x >> 3, b = (int)blockIdx.x;
    int line = b < 8 * run ? (b & 7) * run + (b >> 3) : b;
    const int place = split_off(line, tiles_in_line), across = ROWS ? place : line, down = ROWS ? line : place;
    const int tile_col = across * PACK_COLS, col0 = tile_col + c;
    const long tile_row = (long)down * PACK_ROWS, row0 = tile_row + 32 * block;
    const int n = cols - col0, there = (int)min(rows - row0, 32L);   // rows of the block; none of a block of padding
    const T* const from = x + row0 * ldx + col0;
    Few<T, 4> raw[32];
    if (__all(n >= 4 && there == 32)) {
#pragma unroll
        for (int r = 0; r < 32; r++) raw[r].template load<STREAM>(from + r * ldx, 4);
    } else {
#pragma unroll
        for (int r = 0; r < 32; r++) {
            raw[r] = Few<T, 4>{};
            if (n > 0 && r < there) raw[r].template load<STREAM>(from + r * ldx, n);
        }
    }
    if (ROWS) {
#pragma unroll
        for (int r = 0; r < 32; r++) {
            uint32_t m = quad_max(Magnitudes<T, 4>(raw[r]).largest());
            m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));   // the other four of eight lanes
            const Packer<F> q(m);
            const uint32_t w = q.four(pair_of(raw[r], 0), pair_of(raw[r], 1));
            uint8_t* const to = smem + (32 * block + r) * ROW + c * BITS / 8;
            if constexpr (F == MX_E4M3) *reinterpret_cast<uint32_t*>(to) = w;
            else *reinterpret_cast<uint16_t*>(to) = (uint16_t)w;
            if ((lane & 7) == 0) smem[CODES + (32 * block + r) * (PACK_COLS / MX_BLOCK) + c / MX_BLOCK] = (uint8_t)q.byte;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < ROW / 16; i++) {
            const int at = i * 256 + t, r = at / (ROW / 16), piece = at % (ROW / 16);
            if (tile_row + r < rows)
                *reinterpret_cast<uint4*>(codes + ((size_t)(tile_row + r) * width * BITS / 8) + (tile_col * BITS / 8 + 16 * piece)) =
                    reinterpret_cast<const uint4*>(smem)[at];
        }
        if (tile_row + t < rows)
            *reinterpret_cast<uint32_t*>(scales + (size_t)(tile_row + t) * (width / MX_BLOCK) + tile_col / MX_BLOCK) =
                reinterpret_cast<const uint32_t*>(smem + CODES)[t];
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 32; r++) raw[r].hide();   // what was derived from them is formed again: half the registers
    }
    Magnitudes<T, 4> most(raw[0]);
#pragma unroll
    for (int r = 1; r < 32; r++) most.add(Magnitudes<T, 4>(raw[r]));
#pragma unroll
    for (int j = 0; j < 4; j++) {
        const Packer<F> q(most.column(j));
        uint32_t w[BITS];   // 32 codes
#pragma unroll
        for (int k = 0; k < 4; k++) {
            Pair<T> pairs[4];
#pragma unroll
            for (int i = 0; i < 4; i++) pairs[i] = pair_across(raw[8 * k + 2 * i], raw[8 * k + 2 * i + 1], j);
            q.eight(pairs, w + k * BITS / 4);
        }
#pragma unroll
        for (int i = 0; i < BITS / 4; i++)
            *reinterpret_cast<uint4*>(smem + (c + j) * COLUMN + 16 * ((block * (BITS / 4) + i) ^ (c / 4 & (CHUNKS - 1)))) =
                make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        smem[CODES + (c + j) * (PACK_ROWS / MX_BLOCK) + block] = (uint8_t)q.byte;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < COLUMN * PACK_COLS / 4096; i++) {
        const int at = i * 256 + t, col = at / CHUNKS, piece = (at % CHUNKS) ^ (col / 4 & (CHUNKS - 1));
        if (tile_col + col < cols)
            *reinterpret_cast<uint4*>(column_codes + ((size_t)(tile_col + col) * column_width * BITS / 8) + (tile_row * BITS / 8 + 16 * piece)) =
                reinterpret_cast<const uint4*>(smem)[at];
    }
    if (t < PACK_COLS && tile_col + t < cols)
        *reinterpret_cast<uint2*>(column_scales + (size_t)(tile_col + t) * (column_width / MX_BLOCK) + tile_row / MX_BLOCK) =
            reinterpret_cast<const uint2*>(smem + CODES)[t];
}

template <typename T, int F>
static hipError_t quantise(long rows, long cols, const void* x, long ldx, const MxRows& by_row, const MxRows& by_column, hipStream_t st) {
    const int width = (int)mx_width(cols);
    const bool stream = (double)rows * cols * (sizeof(T) + (F == MX_E4M3 ? 1.0 : 0.5) * ((by_row.codes != nullptr) + (by_column.codes != nullptr))) > STREAM_BYTES;
    if (!by_column.codes) {
        const int chunks = (int)(rows * (width / 8));
        auto kern = stream ? &k_pack_rows<T, F, true> : &k_pack_rows<T, F, false>;
        const unsigned each = 256u * (stream ? chunks_each<true>() : chunks_each<false>());
        kern<<<((unsigned)chunks + each - 1) / each, 256, 0, st>>>(chunks, divisor(width / 8), (int)cols, (const T*)x, ldx, by_row.codes, by_row.scales);
        return hipGetLastError();
    }
    const long column_width = mx_width(rows);
    const int across = by_row.codes ? width / PACK_COLS : ((int)cols + PACK_COLS - 1) / PACK_COLS, down = (int)(column_width / PACK_ROWS);
    auto run = [&](auto kern) {
        kern<<<(unsigned)(across * down), 256, 0, st>>>(rows, (int)cols, (const T*)x, ldx, width, by_row.codes, by_row.scales, column_width, by_column.codes,
                                                        by_column.scales, divisor(by_row.codes ? across : down));
        return hipGetLastError();
    };
    if (by_row.codes) return run(stream ? &k_pack_columns<T, F, true, true> : &k_pack_columns<T, F, true, false>);
    return run(stream ? &k_pack_columns<T, F, false, true> : &k_pack_columns<T, F, false, false>);
}
hipError_t mx_quantise(int dtype, long rows, long cols, const void* x, long ldx, int format, const MxRows& by_row, const MxRows& by_column,
                       hipStream_t st) {
    if (dtype == DT_BF16)
        return format == MX_E4M3 ? quantise<bf16_t, MX_E4M3>(rows, cols, x, ldx, by_row, by_column, st)
                                 : quantise<bf16_t, MX_E2M1>(rows, cols, x, ldx, by_row, by_column, st);
    return format == MX_E4M3 ? quantise<float, MX_E4M3>(rows, cols, x, ldx, by_row, by_column, st)
                             : quantise<float, MX_E2M1>(rows, cols, x, ldx, by_row, by_column, st);
}

// ------------------------------------------------------------------ values
// 4096x11008 of E2M1 to bf16 16.9 us (6.7 TB/s), 8192x8192 of E4M3 to fp32 60 (5.7).
template <typename T, int F, bool STREAM>
__global__ __launch_bounds__(256) void k_values(int chunks, Divisor per_row, int k, int width, const uint8_t* __restrict__ codes,
                                                 const uint8_t* __restrict__ scales, T* __restrict__ y, long ldy) {
    const int i = (int)(blockIdx.x * 256u + threadIdx.x);
    if (i >= chunks) return;
    int row = i;
    const int group = split_off(row, per_row);
    const size_t at = (size_t)row * (width / 8) + group;
    const float s = scale_value(scales[at >> 2]);
    typedef float f32x2v __attribute__((ext_vector_type(2)));
    float v[8];
    if constexpr (F == MX_E4M3) {
        const uint2 w = reinterpret_cast<const uint2*>(codes)[at];
#pragma unroll
        for (int q = 0; q < 2; q++) {
            const f32x2v a = __builtin_amdgcn_cvt_pk_f32_fp8((int)(q ? w.y : w.x), false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)(q ? w.y : w.x), true);
            v[4 * q] = a[0]; v[4 * q + 1] = a[1]; v[4 * q + 2] = b[0]; v[4 * q + 3] = b[1];
        }
    } else {
        const uint32_t w = reinterpret_cast<const uint32_t*>(codes)[at];
        const f32x2v a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 0), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 1);
        const f32x2v c = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 2), d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, 1.f, 3);
        v[0] = a[0]; v[1] = a[1]; v[2] = b[0]; v[3] = b[1]; v[4] = c[0]; v[5] = c[1]; v[6] = d[0]; v[7] = d[1];
    }
#pragma unroll
    for (int j = 0; j < 8; j++) v[j] *= s;
    Eight<T> e;
    e.round(v);
    e.template store<STREAM>(y + row * ldy + 8L * group, k - 8 * group);
}

hipError_t mx_values(int dtype, long rows, long k, int format, const MxRows& q, void* y, long ldy, hipStream_t st) {
    const int per_row = (int)((k + 7) / 8), chunks = (int)(rows * per_row), width = (int)mx_width(k);
    const unsigned grid = ((unsigned)chunks + 255u) / 256u;
    auto run = [&](auto kern, auto* to) {
        kern<<<grid, 256, 0, st>>>(chunks, divisor(per_row), (int)k, width, q.codes, q.scales, to, ldy);
        return hipGetLastError();
    };
    const bool stream = (double)rows * k * (dt_size(dtype) + (format == MX_E4M3 ? 1.0 : 0.5)) > STREAM_BYTES;
    auto pick = [&](auto* to, auto fmt) {
        typedef std::remove_pointer_t<decltype(to)> T;
        constexpr int F = decltype(fmt)::value;
        return run(stream ? &k_values<T, F, true> : &k_values<T, F, false>, to);
    };
    std::integral_constant<int, MX_E4M3> e8;
    std::integral_constant<int, MX_E2M1> e4;
    if (dtype == DT_BF16) return format == MX_E4M3 ? pick((bf16_t*)y, e8) : pick((bf16_t*)y, e4);
    return format == MX_E4M3 ? pick((float*)y, e8) : pick((float*)y, e4);
}

}  // namespace hh
