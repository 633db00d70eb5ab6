// Packing to microscaled formats and back.
#include <type_traits>

#include "mx.h"

namespace hh {

// Packing.  A block's scale is the exponent of its largest magnitude, which is compared as an integer, and every value is multiplied by one
// over the scale, exactly, before it is rounded: one read, one pass, no division.  Bound by memory.

// ------------------------------------------------------------------ by row
// Eight values a lane, four lanes a block.  11008x4096 bf16 to E2M1 18.9 us from the last-level cache (6.0 TB/s), 21.3 from memory.
template <typename T, int F, bool STREAM>
__global__ __launch_bounds__(256) void k_pack_rows(int chunks, Divisor per_row, int cols, const T* __restrict__ x, long ldx, uint8_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales) {
    const int i = (int)(blockIdx.x * 256u + threadIdx.x);
    if (i >= chunks) return;   // whole rows of a multiple of 32 chunks
    int row = i;
    const int group = split_off(row, per_row), n = cols - 8 * group;
    Eight<T> e{};
    if (n > 0) e.template load<STREAM>(x + row * ldx + 8L * group, n);
    float v[8];
    e.widen(v);
    const uint32_t byte = scale_byte<F>(quad_max(magnitude8(v)));
    Codes8<F> q;
    q.set(v, byte);
    q.store(codes, (size_t)i);
    if ((group & 3) == 0) scales[(size_t)i >> 2] = (uint8_t)byte;
}

// Magnitudes of four columns as they lie in memory, two bf16 to a word: their order as integers is that of the numbers, and two are compared at
// a time.
template <typename T> struct Magnitudes;
template <> struct Magnitudes<bf16_t> {
    typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
    uint32_t w[2];
    __device__ __forceinline__ static uint32_t larger(uint32_t a, uint32_t b) {
        u16x2 x, y;
        __builtin_memcpy(&x, &a, 4);
        __builtin_memcpy(&y, &b, 4);
        x = __builtin_elementwise_max(x, y);
        __builtin_memcpy(&a, &x, 4);
        return a;
    }
    __device__ __forceinline__ explicit Magnitudes(const Few<bf16_t, 4>& v) : w{v.w[0] & 0x7FFF7FFFu, v.w[1] & 0x7FFF7FFFu} {}
    __device__ __forceinline__ void add(const Magnitudes& o) { w[0] = larger(w[0], o.w[0]); w[1] = larger(w[1], o.w[1]); }
    __device__ __forceinline__ uint32_t column(int j) const { return (j & 1 ? w[j >> 1] >> 16 : w[j >> 1] & 0xFFFFu) << 16; }   // as of fp32
    __device__ __forceinline__ uint32_t largest() const { const uint32_t m = larger(w[0], w[1]); return max(m >> 16, m & 0xFFFFu) << 16; }
};
template <> struct Magnitudes<float> {
    uint32_t w[4];
    __device__ __forceinline__ explicit Magnitudes(const Few<float, 4>& v) {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = v.w[0][i] & 0x7FFFFFFFu;
    }
    __device__ __forceinline__ void add(const Magnitudes& o) {
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = max(w[i], o.w[i]);
    }
    __device__ __forceinline__ uint32_t column(int j) const { return w[j]; }
    __device__ __forceinline__ uint32_t largest() const { return max(max(w[0], w[1]), max(w[2], w[3])); }
};

// ------------------------------------------------------------------ by column, and both
// A lane takes 4 columns of a block of 32 rows in registers, ACROSS lanes the columns beside them and 64 / ACROSS the row blocks below: blocks
// along columns need no exchange at all, those along rows one of eight lanes, and x is read once for both.  11008x4096 bf16 to E2M1 both
// ways 38.8 us from memory (3.6 TB/s; 34 without the rows' codes, of which a lane has two bytes), packing twice 46.
template <typename T, int F, bool ROWS, int ACROSS, bool STREAM>
__global__ __launch_bounds__(256) void k_pack_columns(long rows, int cols, const T* __restrict__ x, long ldx, int width, uint8_t* __restrict__ codes,
                                                       uint8_t* __restrict__ scales, long column_width, uint8_t* __restrict__ column_codes,
                                                       uint8_t* __restrict__ column_scales, Divisor tiles_across) {
    constexpr int BITS = F == MX_E4M3 ? 8 : 4, DOWN = 64 / ACROSS;
    const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6;
    int down = (int)blockIdx.x;
    const int across = split_off(down, tiles_across);
    const int col0 = (across * 4 + wave) * (4 * ACROSS) + (lane % ACROSS) * 4;
    const long block = (long)down * DOWN + lane / ACROSS, row0 = block * 32;
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
    Magnitudes<T> most(raw[0]);
#pragma unroll
    for (int r = 1; r < 32; r++) most.add(Magnitudes<T>(raw[r]));
    if (ROWS && col0 < width) {
        uint8_t* to = codes + ((size_t)row0 * width + col0) * BITS / 8;
        uint8_t* scale = scales + (size_t)row0 * (width / MX_BLOCK) + (col0 >> 5);
#pragma unroll
        for (int r = 0; r < 32; r++) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = i < 4 ? raw[r].at(i) : 0.f;
            uint32_t m = quad_max(magnitude8(v));
            m = max(m, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)m, 0x141, 0xF, 0xF, true));   // the other four of eight lanes
            const uint32_t byte = scale_byte<F>(m);
            Codes8<F> q;
            q.set(v, byte);
            if (r < there) {
                if constexpr (F == MX_E4M3) *reinterpret_cast<uint32_t*>(to) = q.w.x;
                else *reinterpret_cast<uint16_t*>(to) = (uint16_t)q.w;
                if ((col0 & 31) == 0) *scale = (uint8_t)byte;
            }
            to += (size_t)width * BITS / 8;
            scale += width / MX_BLOCK;
        }
    }
#pragma unroll
    for (int j = 0; j < 4; j++) {
        if (j >= n) continue;
        const uint32_t byte = scale_byte<F>(most.column(j));
        uint32_t w[BITS];   // 32 codes
#pragma unroll
        for (int k = 0; k < 4; k++) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; i++) v[i] = raw[8 * k + i].at(j);
            Codes8<F> q;
            q.set(v, byte);
            if constexpr (F == MX_E4M3) { w[2 * k] = q.w.x; w[2 * k + 1] = q.w.y; }
            else w[k] = q.w;
        }
        uint4* const to = reinterpret_cast<uint4*>(column_codes + ((size_t)(col0 + j) * column_width + row0) * BITS / 8);
        if (row0 < column_width) {
            to[0] = make_uint4(w[0], w[1], w[2], w[3]);
            if constexpr (BITS == 8) to[1] = make_uint4(w[4], w[5], w[6], w[7]);
            column_scales[(size_t)(col0 + j) * (column_width / MX_BLOCK) + block] = (uint8_t)byte;
        }
    }
}

template <typename T, int F>
static hipError_t quantise(long rows, long cols, const void* x, long ldx, const MxRows& by_row, const MxRows& by_column, hipStream_t st) {
    const int width = (int)mx_width(cols);
    const bool stream = (double)rows * cols * (sizeof(T) + (F == MX_E4M3 ? 1.0 : 0.5) * ((by_row.codes != nullptr) + (by_column.codes != nullptr))) > STREAM_BYTES;
    if (!by_column.codes) {
        const int chunks = (int)(rows * (width / 8));
        auto kern = stream ? &k_pack_rows<T, F, true> : &k_pack_rows<T, F, false>;
        kern<<<((unsigned)chunks + 255u) / 256u, 256, 0, st>>>(chunks, divisor(width / 8), (int)cols, (const T*)x, ldx, by_row.codes, by_row.scales);
        return hipGetLastError();
    }
    const long column_width = mx_width(rows);
    // Wide tiles where rows are written too, tall ones where columns alone are: 11008x4096 bf16 to E2M1, past the caches, both ways with 16, 32
    // and 64 lanes across 41.7, 38.8 and 45.6 us, by column alone 24.7, 28.1 and 39.9.
    auto tiles = [&](auto kern, int lanes) {
        const int across = ((by_row.codes ? width : (int)cols) + 16 * lanes - 1) / (16 * lanes);
        const unsigned grid = (unsigned)(across * ((column_width + 2048 / lanes - 1) / (2048 / lanes)));
        kern<<<grid, 256, 0, st>>>(rows, (int)cols, (const T*)x, ldx, width, by_row.codes, by_row.scales, column_width, by_column.codes, by_column.scales,
                                   divisor(across));
        return hipGetLastError();
    };
    if (by_row.codes) return tiles(stream ? &k_pack_columns<T, F, true, 32, true> : &k_pack_columns<T, F, true, 32, false>, 32);
    return tiles(stream ? &k_pack_columns<T, F, false, 16, true> : &k_pack_columns<T, F, false, 16, false>, 16);
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
// 4096x11008 of E2M1 to bf16 16.9 us (6.7 TB/s).
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
