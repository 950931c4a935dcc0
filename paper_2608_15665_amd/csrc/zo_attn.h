// Device pieces that the attention and rotary kernels share (not part of the ABI): 8-element rows in
// and out of registers, the 16 x 16 x 32 MFMA with its packed operands, transposed LDS reads.
#pragma once

#include "zo_internal.h"

namespace {

template <int DT>
__device__ __forceinline__ void load8(const void* X, size_t idx, float* v) {
  if constexpr (DT == ZO_F32) {
    const f32x4 a = *(const f32x4*)((const float*)X + idx);
    const f32x4 b = *(const f32x4*)((const float*)X + idx + 4);
    v[0] = a[0]; v[1] = a[1]; v[2] = a[2]; v[3] = a[3];
    v[4] = b[0]; v[5] = b[1]; v[6] = b[2]; v[7] = b[3];
  } else {
    const u32x4 u = *(const u32x4*)((const uint16_t*)X + idx);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (DT == ZO_BF16) {
        v[2 * e] = bf16_to_f32((bf16_t)u[e]);
        v[2 * e + 1] = bf16_to_f32((bf16_t)(u[e] >> 16));
      } else {
        v[2 * e] = f16_to_f32((uint16_t)u[e]);
        v[2 * e + 1] = f16_to_f32((uint16_t)(u[e] >> 16));
      }
    }
  }
}

template <int DT>
__device__ __forceinline__ void store8(void* Y, size_t idx, const float* v) {
  if constexpr (DT == ZO_F32) {
    *(f32x4*)((float*)Y + idx) = (f32x4){v[0], v[1], v[2], v[3]};
    *(f32x4*)((float*)Y + idx + 4) = (f32x4){v[4], v[5], v[6], v[7]};
  } else if constexpr (DT == ZO_BF16) {
    *(u32x4*)((uint16_t*)Y + idx) = (u32x4){pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]),
                                            pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7])};
  } else {
    *(u32x4*)((uint16_t*)Y + idx) = (u32x4){pack_f16x2(v[0], v[1]), pack_f16x2(v[2], v[3]),
                                            pack_f16x2(v[4], v[5]), pack_f16x2(v[6], v[7])};
  }
}

template <bool F16>
__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 c) {
  if constexpr (F16)
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                   __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  else
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// Two fp32 values rounded to nearest even into a packed pair of 16-bit values (one
// v_cvt_pk_bf16_f32 / v_cvt_pk_f16_f32), and back.
typedef _Float16 f16x2_t __attribute__((ext_vector_type(2)));
template <bool F16>
__device__ __forceinline__ uint32_t cvt_pk(float x, float y) {
  if constexpr (F16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){x, y}, f16x2_t));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2_t){x, y}, bf16x2_t));
}
template <bool F16>
__device__ __forceinline__ float unpk(uint32_t pk, int half) {
  const uint16_t h = (uint16_t)(half ? pk >> 16 : pk);
  if constexpr (F16)
    return f16_to_f32(h);
  else
    return bf16_to_f32(h);
}

typedef short i16x4_t __attribute__((ext_vector_type(4)));
// ds_read_b64_tr_b16: within each 16-lane group, lane i reads 4 consecutive 16-bit values
// D[i][0..3] at its own address, and lane j receives D[j/4 + 4e][j%4] for e = 0..3.  With
// lane i addressing row (r0 + i/4), columns c0 + 4 (i%4) of a row-major tile, lane j thus
// receives column c0 + j of rows r0 .. r0+3: a transposed fragment.
__device__ __forceinline__ u32x2 ds_read_tr(const uint16_t* p) {
  const i16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) i16x4_t*)(p));
  return __builtin_bit_cast(u32x2, v);
}

// The maximum over the four 16-lane groups.
__device__ __forceinline__ float max_groups(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto a = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t v = __float_as_uint(fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1])));
  const auto b = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return fmaxf(__uint_as_float(b[0]), __uint_as_float(b[1]));
}

}  // namespace
