// Device helpers of the 8-bit products: scales that are powers of two, codes of e4m3, the scaled matrix instructions.
#pragma once
#include "bsp_tile_device.h"

namespace bsp {
namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// |x|; 0 where x is not finite (its code is NaN whatever the scale).
__device__ __forceinline__ float magnitude(float x) {
    const uint32_t u = __float_as_uint(x) & 0x7fffffffu;
    return u < 0x7f800000u ? __uint_as_float(u) : 0.0f;
}

// The largest of 16 lanes' values (all >= 0), in every one of them: rotations within the row.
template <int CTRL>
__device__ __forceinline__ float max_turned(float x) {
    return __builtin_fmaxf(x, __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), CTRL, 0xf, 0xf, false)));
}
__device__ __forceinline__ float max_of_16(float x) { return max_turned<0x128>(max_turned<0x124>(max_turned<0x122>(max_turned<0x121>(x)))); }

// The biased exponent of the least power of two 2^e with largest / 2^e <= 448 = 1.75 2^8 (not below 2^-127; 2^0 for zero).
__device__ __forceinline__ uint32_t scale_exponent(float largest) {
    const uint32_t u = __float_as_uint(largest);
    const int e = (int)(u >> 23) - 8 + ((u & 0x7fffffu) > 0x600000u ? 1 : 0);
    return largest == 0.0f ? 127u : (e > 0 ? (uint32_t)e : 0u);
}
// 2^-e for a biased exponent of 0 to 253: exact, and so is a product with it unless the result is far below e4m3's least value.
__device__ __forceinline__ float inverse_scale(uint32_t e) { return __uint_as_float((254u - e) << 23); }

// From 1.9375 2^127 on (a type's lowest value, as a mask, is there) a value would go to the code 256 under the scale 2^120, and 2^128 is no number of fp32: it goes to 240,
// where 1.875 2^127 goes, under the same scale.  A thread whose largest magnitude says that it has such values puts that one in their place; for the others it
// is a comparison (8192 x 4096 in bf16 by rows 17.5 us as without; with every code held at or below a limit the kernels took up to 8 % longer).
constexpr float kBeyond = 1.9375f * 0x1p127f;
template <int N>
__device__ __forceinline__ void keep_below(float *v, float largest) {
    if (__builtin_expect(largest >= kBeyond, 0)) {
#pragma unroll
        for (int i = 0; i < N; ++i)
            if (magnitude(v[i]) >= kBeyond) v[i] = __builtin_copysignf(1.875f * 0x1p127f, v[i]);
    }
}

// Four values of at most 448 as codes, to the nearest (ties to even); NaN for what is not finite.
__device__ __forceinline__ uint32_t codes4(const float *y) {
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = (__float_as_uint(y[i]) & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : y[i];
    const int p = __builtin_amdgcn_cvt_pk_fp8_f32(x[0], x[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2], x[3], p, true);
}

// Eight 16-bit values.
template <int DT>
__device__ __forceinline__ void unpack8(uint4 p, float *v) {
    const uint32_t d[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint16_t lo = (uint16_t)d[j], hi = (uint16_t)(d[j] >> 16);
        v[2 * j] = elem<DT>::load(&lo, 0);
        v[2 * j + 1] = elem<DT>::load(&hi, 0);
    }
}

// Eight consecutive elements at any address (loads of 16 bytes need no alignment here).
template <int DT>
__device__ __forceinline__ void load8(const void *p, int64_t at, float *v) {
    if constexpr (DT == BSP_F32) {
        __builtin_memcpy(v, (const float *)p + at, 32);
    } else {
        uint4 x;
        __builtin_memcpy(&x, (const uint16_t *)p + at, 16);
        unpack8<DT>(x, v);
    }
}

// Eight consecutive outputs at y: the sums v with bias, activation and residual, in fp32, rounded once.  vec: y is a multiple of 8 elements
// from an aligned row; cols: how many there are.
template <int DT>
__device__ __forceinline__ void finish8(float (&v)[8], const float (&bias)[8], int act, const void *residual, void *Y, int64_t y, bool vec, int cols) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
        v[k] += bias[k];
        if (act == BSP_ACT_GELU) v[k] = gelu_fit(v[k]);
    }
    constexpr size_t size = DT == BSP_F32 ? 4 : 2;
    const uint8_t *r = (const uint8_t *)residual + y * size;
    uint8_t *o = (uint8_t *)Y + y * size;
    if (vec && ((reinterpret_cast<uintptr_t>(o) | reinterpret_cast<uintptr_t>(residual ? r : nullptr)) & 15) == 0) {
        if (residual) {
            float x[8];
            if constexpr (DT == BSP_F32) {
                const float4 a = *reinterpret_cast<const float4 *>(r), b = *reinterpret_cast<const float4 *>(r + 16);
                x[0] = a.x, x[1] = a.y, x[2] = a.z, x[3] = a.w, x[4] = b.x, x[5] = b.y, x[6] = b.z, x[7] = b.w;
            } else {
                unpack8<DT>(*reinterpret_cast<const uint4 *>(r), x);
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += x[k];
        }
        if constexpr (DT == BSP_F32) {
            store_y16(o, make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]), __float_as_uint(v[3])));
            store_y16(o + 16, make_uint4(__float_as_uint(v[4]), __float_as_uint(v[5]), __float_as_uint(v[6]), __float_as_uint(v[7])));
        } else {
            store_y16(o, make_uint4(cvt_pk<DT>(v[0], v[1]), cvt_pk<DT>(v[2], v[3]), cvt_pk<DT>(v[4], v[5]), cvt_pk<DT>(v[6], v[7])));
        }
    } else if (cols == 8) {  // (loads and stores need no alignment)
        if (residual) {
            float x[8];
            load8<DT>(r, 0, x);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += x[k];
        }
        if constexpr (DT == BSP_F32) {
            __builtin_memcpy(o, v, 32);
        } else {
            const uint4 x = make_uint4(cvt_pk<DT>(v[0], v[1]), cvt_pk<DT>(v[2], v[3]), cvt_pk<DT>(v[4], v[5]), cvt_pk<DT>(v[6], v[7]));
            __builtin_memcpy(o, &x, 16);
        }
    } else {
        if (residual) {  // all loads before the first store: a load waits for the stores before it, and seven of them in turn took 25 us where rows end here
            float x[8];
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = elem<DT>::load(r, k < cols ? k : 0);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] += x[k];
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
            if (k < cols) elem<DT>::store(o, k, v[k]);
    }
}

}  // namespace
}  // namespace bsp
