// rows.h -- element conversions and row stores of the kernels of albireo_decode.h (norm.hip,
// matmul_w4.hip, adjust.hip).  Included inside `namespace {` after common.h.
#pragma once

// two fp32 values as two bf16 (a in the low half), rounded to nearest even
__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  f2 v;
  v.x = a;
  v.y = b;
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, b2));
}

template <class DT>
__device__ __forceinline__ void store1(unsigned char* row, int64_t i, float v) {
  if constexpr (DT::ES == 2) reinterpret_cast<uint16_t*>(row)[i] = (uint16_t)bf16_pair(v, v);
  else reinterpret_cast<float*>(row)[i] = v;
}
