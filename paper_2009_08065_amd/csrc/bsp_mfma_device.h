// Device helpers shared by the matrix-core kernels of the layer: operand types, the 16x16x32 and 32x32x16
// matrix instructions, the transposing LDS read and the packed conversion to 16-bit floats.
#pragma once
#include <type_traits>

#include "bsp_common.h"

namespace bsp {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

template <int DT>
__device__ __forceinline__ f32x4 mfma16(uint4 a, uint4 b, f32x4 c) {
    if constexpr (DT == BSP_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

template <int DT>
__device__ __forceinline__ f32x16 mfma32(uint4 a, uint4 b, f32x16 c) {
    if constexpr (DT == BSP_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c,
                                                       0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0,
                                                      0, 0);
}

__device__ __forceinline__ uint2 tr_read(const uint8_t *lds_base, uint32_t off) {
    s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(lds_base + off));
    return __builtin_bit_cast(uint2, v);
}
// The same read at an LDS address given as an integer (the dynamic LDS block starts at 0 in kernels without
// static LDS variables; through its symbol every address costs an addition of that base).
__device__ __forceinline__ uint2 tr_read_at(uint32_t lds_addr) {
    s16x4 v = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4 *)(uintptr_t)lds_addr);
    return __builtin_bit_cast(uint2, v);
}

// Two fp32 -> two 16-bit floats (round-to-nearest-even, hardware conversion), packed.
template <int DT>
__device__ __forceinline__ uint32_t cvt_pk(float a, float b) {
    if constexpr (DT == BSP_BF16)
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, bf16x2));
    else
        return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{a, b}, f16x2));
}

// 64 lanes' 16 bytes at base + at to LDS at lds .. lds + 1023.  (Written out: for the builtin the compiler would wait for all such
// loads before any LDS read.  m0 is a reserved register, which can't be named as clobbered; nothing else in these kernels uses it.)
__device__ __forceinline__ void load_to_lds(uint32_t lds, const uint8_t *base, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n s_nop 0\n global_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(at), "s"(base));
}
// 64 lanes' bytes at base + at to LDS as 32-bit words at lds .. lds + 255.
__device__ __forceinline__ void load_bytes_to_lds(uint32_t lds, const uint8_t *base, uint32_t at) {
    asm volatile("s_mov_b32 m0, %0\n s_nop 0\n global_load_lds_ubyte %1, %2" ::"s"(lds), "v"(at), "s"(base));
}
template <int LEFT>
__device__ __forceinline__ void wait_loads() {  // until LEFT loads are on their way
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LEFT) : "memory");
}

extern __shared__ __attribute__((aligned(16))) uint8_t smem_x[];

// f(integral_constant<int, I>) for I = B .. E - 1: a loop whose index is a constant inside the body, so that
// register arrays indexed by it stay in registers.
template <int B, int E, typename F>
__device__ __forceinline__ void static_for(F &&f) {
    if constexpr (B < E) {
        f(std::integral_constant<int, B>{});
        static_for<B + 1, E>(f);
    }
}

}  // namespace
}  // namespace bsp
