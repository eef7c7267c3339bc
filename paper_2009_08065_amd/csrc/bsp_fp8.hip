// Matrices in 8-bit floating point (e4m3) with a power of two for every 128 columns of a row, or for every 128 x 128 block
// (bsp_fp8_quant).
//
// The scale of a segment is the least power of two that brings its largest value to 448, e4m3's largest, or below.  It is held as
// a biased exponent in one byte, which the matrix instruction of the product takes as it is: no multiplication is spent on
// scales there, and a code times its scale has no rounding of its own.  Against a scale of largest / 448 it leaves at most one of the
// type's 18 binades unused.
//
// Bound by memory.  Row segments alone: 16 lanes to a segment.  Else a workgroup reads a 128 x 128 tile once, 4 x 8 values per thread, and has
// from it the row segments, the column segments (the rows of the transposed matrix) or the block, and the codes of either
// orientation; the transposed ones go through LDS.  Measured (MI355X, bf16, us): 16384 x 4096 by rows 33 (6.0 TB/s), 8192 x 1024 7.3; in both
// orientations 8192 x 4096 by rows 28 to 31 (4.4 TB/s), in blocks 23; 64 x 1024 by rows 2.5.  A width that is no multiple of 8 costs 10 to 25 % (loads
// that cross lines).
#include "bsp_common.h"
#include "bsp_fp8_device.h"

namespace bsp {
namespace {

constexpr int kThreads = 256;
constexpr int kPitch = 128 + 4;  // bytes of a column's codes in LDS

struct Quant {
    const void *X;
    uint8_t *Q, *S, *Qt, *St;
    int64_t rows, cols, tiles_c, pitch, pitch_t;  // pitches of Q and Qt: columns and rows, padded to 128
};

// Eight values of a row as they came.
template <int DT>
struct Piece {
    uint4 raw[DT == BSP_F32 ? 2 : 1];
    __device__ __forceinline__ void load(const void *X, int64_t at, int cols) {
        if (cols >= 8) {
            __builtin_memcpy(raw, (const uint8_t *)X + at * (DT == BSP_F32 ? 4 : 2), sizeof(raw));  // (loads need no alignment here)
        } else {
            typename elem<DT>::type v[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) v[j] = j < cols ? ((const typename elem<DT>::type *)X)[at + j] : typename elem<DT>::type(0);
            __builtin_memcpy(raw, v, sizeof(raw));
        }
    }
    __device__ __forceinline__ float operator[](int j) const {
        if constexpr (DT == BSP_F32) {
            const uint32_t w[8] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w, raw[1].x, raw[1].y, raw[1].z, raw[1].w};
            return __uint_as_float(w[j]);
        } else {
            const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
            const uint16_t h = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
            return elem<DT>::load(&h, 0);
        }
    }
};

// One row segment per 16 lanes, kRowsEach of them one below the other, all asked for at once.
constexpr int kRowsEach = 2;

template <int DT>
__global__ __launch_bounds__(kThreads) void quant_rows_kernel(Quant a) {
    const int c0 = 8 * (threadIdx.x & 15);
    const int64_t strip = blockIdx.x / a.tiles_c, tc = blockIdx.x - strip * a.tiles_c;  // (along the rows first)
    const int64_t row0 = strip * (kRowsEach * 16) + (threadIdx.x >> 4), col0 = 128 * tc + c0;
    const int cols = a.cols - col0 > 8 ? 8 : (int)(a.cols - col0);
    Piece<DT> raw[kRowsEach];
#pragma unroll
    for (int i = 0; i < kRowsEach; ++i) raw[i].load(a.X, (row0 + 16 * i) * a.cols + col0, row0 + 16 * i < a.rows ? cols : 0);
#pragma unroll
    for (int i = 0; i < kRowsEach; ++i) {
        const int64_t row = row0 + 16 * i;
        float v[8], m = 0.0f;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = raw[i][j], m = __builtin_fmaxf(m, magnitude(v[j]));
        if (DT != BSP_F16) keep_below<8>(v, m);
        m = max_of_16(m);
        if (row >= a.rows) continue;
        const uint32_t e = scale_exponent(m);
        const float s = inverse_scale(e);
        float y[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) y[j] = s * v[j];
        *reinterpret_cast<uint2 *>(a.Q + row * a.pitch + col0) = make_uint2(codes4(y), codes4(y + 4));
        if ((threadIdx.x & 15) == 0) a.S[row * a.tiles_c + tc] = (uint8_t)e;
    }
}

// The tile: kTileThreads threads of kEach rows x 8 columns each.  (With 8 x 8 values each, half the threads, the small matrices' chains of load,
// largest value and store were twice as long: 8192 x 1024 in both orientations 13.5 us.)
constexpr int kTileThreads = 512, kEach = 4, kTileWaves = kTileThreads / kWave;

template <int DT, bool BLOCK, bool TRANSPOSED>
__global__ __launch_bounds__(kTileThreads) void quant_kernel(Quant a) {
    __shared__ float top[TRANSPOSED && !BLOCK ? kTileWaves * 128 : kTileWaves];
    __shared__ __align__(16) uint8_t turned[TRANSPOSED ? 128 * kPitch : 16];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int64_t tr = blockIdx.x / a.tiles_c, tc = blockIdx.x - tr * a.tiles_c;
    const int r0 = kEach * (tid >> 4), c0 = 8 * (tid & 15);
    const int64_t row0 = 128 * tr + r0, col0 = 128 * tc + c0;
    const int rows = a.rows - row0 > kEach ? kEach : (int)(a.rows - row0), cols = a.cols - col0 > 8 ? 8 : (int)(a.cols - col0);  // (may be negative)

    Piece<DT> raw[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) raw[i].load(a.X, (row0 + i) * a.cols + col0, i < rows ? cols : 0);
    float v[kEach][8];
#pragma unroll
    for (int i = 0; i < kEach; ++i)
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = raw[i][j];

    float most = 0.0f;  // of this thread's magnitudes
    uint32_t e_row[kEach], e_col[8];  // biased exponents of the rows' and the columns' scales
    if constexpr (BLOCK) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < kEach; ++i)
#pragma unroll
            for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, magnitude(v[i][j]));
        most = m;
        m = max_of_16(m);
        m = __builtin_fmaxf(m, __shfl_xor(m, 16));
        m = __builtin_fmaxf(m, __shfl_xor(m, 32));
        if (lane == 0) top[wave] = m;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kTileWaves; ++w) m = __builtin_fmaxf(m, top[w]);
        const uint32_t e = scale_exponent(m);
#pragma unroll
        for (int i = 0; i < kEach; ++i) e_row[i] = e;
#pragma unroll
        for (int j = 0; j < 8; ++j) e_col[j] = e;
        if (tid == 0) {
            if (a.Q) a.S[tr * a.tiles_c + tc] = (uint8_t)e;
            if (TRANSPOSED) a.St[tc * (a.pitch_t / 128) + tr] = (uint8_t)e;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            float m = 0.0f;
#pragma unroll
            for (int j = 0; j < 8; ++j) m = __builtin_fmaxf(m, magnitude(v[i][j]));
            most = __builtin_fmaxf(most, m);
            m = max_of_16(m);
            e_row[i] = scale_exponent(m);
            if (a.Q && (tid & 15) == 0 && i < rows) a.S[(row0 + i) * a.tiles_c + tc] = (uint8_t)e_row[i];
        }
        if constexpr (TRANSPOSED) {
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                float m = 0.0f;
#pragma unroll
                for (int i = 0; i < kEach; ++i) m = __builtin_fmaxf(m, magnitude(v[i][j]));
                m = __builtin_fmaxf(m, __shfl_xor(m, 16));
                m = __builtin_fmaxf(m, __shfl_xor(m, 32));
                if (lane < 16) top[wave * 128 + c0 + j] = m;
            }
            __syncthreads();
            if (tid < 128) {  // a column's largest value, then its exponent in its place
                float m = top[tid];
#pragma unroll
                for (int w = 1; w < kTileWaves; ++w) m = __builtin_fmaxf(m, top[w * 128 + tid]);
                const uint32_t e = scale_exponent(m);
                top[tid] = __uint_as_float(e);
                if (128 * tc + tid < a.cols) a.St[(128 * tc + tid) * (a.pitch_t / 128) + tr] = (uint8_t)e;
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < 8; ++j) e_col[j] = __float_as_uint(top[c0 + j]);
        }
    }

    if (DT != BSP_F16) {  // (the scales are the same)
#pragma unroll
        for (int i = 0; i < kEach; ++i) keep_below<8>(v[i], most);
    }
    if (a.Q) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            if (i >= rows) break;
            const float s = inverse_scale(e_row[i]);
            float y[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) y[j] = s * v[i][j];
            *reinterpret_cast<uint2 *>(a.Q + (row0 + i) * a.pitch + col0) = make_uint2(codes4(y), codes4(y + 4));
        }
    }
    if constexpr (TRANSPOSED) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float s = inverse_scale(e_col[j]);
            float y[kEach];
#pragma unroll
            for (int i = 0; i < kEach; ++i) y[i] = s * v[i][j];
            *reinterpret_cast<uint32_t *>(turned + (c0 + j) * kPitch + r0) = codes4(y);
        }
        __syncthreads();
        for (int n = tid; n < 128 * 8; n += kTileThreads) {
            const int c = n >> 3, r = 16 * (n & 7);
            if (128 * tc + c < a.cols) {
                uint4 x;
                __builtin_memcpy(&x, turned + c * kPitch + r, 16);
                *reinterpret_cast<uint4 *>(a.Qt + (128 * tc + c) * a.pitch_t + 128 * tr + r) = x;
            }
        }
    }
}

template <int DT>
void launch(const Quant &a, unsigned grid, int64_t rows_grid, bool block, bool transposed, hipStream_t s) {
    if (block && transposed) quant_kernel<DT, true, true><<<grid, kTileThreads, 0, s>>>(a);
    else if (block) quant_kernel<DT, true, false><<<grid, kTileThreads, 0, s>>>(a);
    else if (transposed) quant_kernel<DT, false, true><<<grid, kTileThreads, 0, s>>>(a);
    else quant_rows_kernel<DT><<<(unsigned)rows_grid, kThreads, 0, s>>>(a);
}

}  // namespace
}  // namespace bsp

using namespace bsp;

extern "C" int bsp_fp8_quant(const void *X, int xdt, int64_t rows, int64_t cols, int layout, void *Q, uint8_t *S, void *Qt, uint8_t *St,
                             void *stream) {
    if (!valid_dtype(xdt) || (layout != BSP_FP8_ROW && layout != BSP_FP8_BLOCK)) return BSP_ERR_DTYPE;
    if (rows < 0 || cols <= 0 || cols >= ((int64_t)1 << 31) || rows >= ((int64_t)1 << 31)) return BSP_ERR_SHAPE;
    if (rows == 0 || (!Q && !Qt)) return BSP_OK;
    if (!X || (Q && !S) || (Qt && !St)) return BSP_ERR_NULL;
    if (!aligned(X, dtype_size(xdt)) || !aligned(Q, 16) || !aligned(Qt, 16)) return BSP_ERR_SHAPE;
    const int64_t tiles_r = (rows + 127) / 128, tiles_c = (cols + 127) / 128;
    const int64_t rows_grid = tiles_c * ((rows + kRowsEach * 16 - 1) / (kRowsEach * 16));
    // a launch has less than 2^32 threads: those of the kernel that runs (up to 64 rows a tile's are the more)
    const bool by_rows = layout == BSP_FP8_ROW && !Qt;
    if (by_rows ? rows_grid >= ((int64_t)1 << 32) / kThreads : tiles_r * tiles_c >= ((int64_t)1 << 32) / kTileThreads) return BSP_ERR_SHAPE;
    const Quant a = {X, (uint8_t *)Q, S, (uint8_t *)Qt, St, rows, cols, tiles_c, 128 * tiles_c, 128 * tiles_r};
    BSP_DISPATCH_DTYPE(xdt, DT, { launch<DT>(a, (unsigned)(tiles_r * tiles_c), rows_grid, layout == BSP_FP8_BLOCK, Qt != nullptr, (hipStream_t)stream); });
    return check_launch();
}
