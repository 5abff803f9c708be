// Device helpers of the latent operators: operands of v_mfma_f32_16x16x32_bf16 from LDS, results as bf16.
//
// Operand A: lane i holds row i % 16, elements 8 (i / 16) .. + 8 of it; operand B the same of a column; the result: column i % 16, rows
// 4 (i / 16) .. + 4.
#pragma once
#include "common.h"

namespace specv {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 lbf16x8;
typedef __bf16 lbf16x2 __attribute__((ext_vector_type(2)));
typedef short ls16x4 __attribute__((ext_vector_type(4)));
typedef float lf32x4 __attribute__((ext_vector_type(4)));
typedef float lf32x16 __attribute__((ext_vector_type(16)));

template <typename T>
__device__ __forceinline__ __attribute__((address_space(3))) T* lds_pointer(unsigned at) {
  return (__attribute__((address_space(3))) T*)static_cast<uintptr_t>(at);
}
__device__ __forceinline__ raw4 read_lds16(unsigned at) { return *lds_pointer<raw4>(at); }
// Of a 4 x 16 block of 16-bit elements, whose row i / 4, columns 4 (i % 4) .. + 4 lane i of 16 points at: the four elements of column i.
__device__ __forceinline__ ls16x4 read_columns(unsigned at) { return __builtin_amdgcn_ds_read_tr16_b64_v4i16(lds_pointer<ls16x4>(at)); }
__device__ __forceinline__ lbf16x8 join(ls16x4 a, ls16x4 b) {
  return __builtin_bit_cast(lbf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}
__device__ __forceinline__ lbf16x8 operand(const raw4& w) { return __builtin_bit_cast(lbf16x8, w); }
__device__ __forceinline__ lf32x4 multiply(lbf16x8 a, lbf16x8 b, lf32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ uint32_t pack2(float a, float b) {
  const lbf16x2 x = {static_cast<__bf16>(a), static_cast<__bf16>(b)};
  return __builtin_bit_cast(uint32_t, x);
}
__device__ __forceinline__ uint2 pack4(const lf32x4& x) { return make_uint2(pack2(x[0], x[1]), pack2(x[2], x[3])); }

}  // namespace specv
