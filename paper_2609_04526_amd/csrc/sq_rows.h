// Rows of a table or a head (bf16, or codes and scales) and of fp32 or bf16 data, 8
// values per lane.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "sq_device.h"
#include "sq_gemm_args.h"
#include "sq_launch.h"

namespace sq {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// An id or target of 4 or 8 bytes.
__device__ __forceinline__ int64_t id_at(const void* ids, int bytes, int64_t t) {
  return bytes == 8 ? static_cast<const int64_t*>(ids)[t] : (int64_t)static_cast<const int32_t*>(ids)[t];
}

__device__ __forceinline__ u32x4 bf16_of(const float (&v)[8]) {
  u32x4 w;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = bits_of(__builtin_convertvector((f32x2{v[2 * i], v[2 * i + 1]}), bf16x2));
  return w;
}

// 8 values of the table from value i (a multiple of 8) on.
template <int HEAD>
__device__ __forceinline__ void table8(const void* w, const uint8_t* scales, float ws2, int64_t i, float (&v)[8]) {
  if constexpr (HEAD == kCeBf16) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(w) + i);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(k & 1 ? q[k >> 1] & 0xFFFF0000u : q[k >> 1] << 16);
  } else {
    const uint32_t q = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(w) + (i >> 1));
    const uint32_t b = scales[i / ScaleOperand<HEAD>::kBlock];
    const float s = HEAD == kMX ? e8m0_to_f32(b) : e4m3_to_f32(b) * ws2;
    const f32x2 c[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                        __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[2 * k] = c[k].x * s;
      v[2 * k + 1] = c[k].y * s;
    }
  }
}

// 8 codes of one dword as fp32.
__device__ __forceinline__ void codes8(uint32_t q, float (&v)[8]) {
  const f32x2 c[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 1),
                      __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(q, 1.0f, 3)};
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    v[2 * k] = c[k].x;
    v[2 * k + 1] = c[k].y;
  }
}

template <bool BF16>
__device__ __forceinline__ void load8(const void* p, int64_t i, float (&v)[8]) {
  if constexpr (BF16) {
    const u32x4 q = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p) + i);
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = __uint_as_float(k & 1 ? q[k >> 1] & 0xFFFF0000u : q[k >> 1] << 16);
  } else {
    const f32x4* q = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + i);
    const f32x4 a = q[0], b = q[1];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = k < 4 ? a[k & 3] : b[k & 3];
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* p, int64_t i, const float (&v)[8]) {
  if constexpr (BF16) {
    *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p) + i) = bf16_of(v);
  } else {
    f32x4* q = reinterpret_cast<f32x4*>(static_cast<float*>(p) + i);
    q[0] = f32x4{v[0], v[1], v[2], v[3]};
    q[1] = f32x4{v[4], v[5], v[6], v[7]};
  }
}

// 8 values of a row as loaded.
template <bool BF16>
struct Raw8 {
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* p, int64_t i) {
    const u32x4* q = reinterpret_cast<const u32x4*>(static_cast<const uint8_t*>(p) + i * (BF16 ? 2 : 4));
#pragma unroll
    for (int k = 0; k < (BF16 ? 1 : 2); ++k) w[k] = q[k];
  }
  __device__ __forceinline__ float at(int k) const {
    if constexpr (BF16) return __uint_as_float(k & 1 ? w[0][k >> 1] & 0xFFFF0000u : w[0][k >> 1] << 16);
    else return __uint_as_float(w[k >> 2][k & 3]);
  }
};

}  // namespace sq
