// Operands of the 16 x 16 matrix instructions, the same for bf16 and fp32: a lane holds eight consecutive k of one row
// (of one column, for the right operand), lane & 15 its row, 8 (lane >> 4) its first k, so that a fragment spans 32 k.
// bf16 multiplies it in one v_mfma_f32_16x16x32_bf16, fp32 in eight v_mfma_f32_16x16x4_f32, whose step i takes element i
// of every lane: k = i, 8 + i, 16 + i, 24 + i, on both sides alike.  The product's lane holds rows 4 (lane >> 4) + 0..3 of
// column lane & 15.
#pragma once

#include "common.h"

namespace fb {

typedef float f32x8 __attribute__((ext_vector_type(8)));

template <typename T> struct FragOf;
template <> struct FragOf<bf16> { typedef bf16x8 type; };
template <> struct FragOf<float> { typedef f32x8 type; };
template <typename T> using Frag = typename FragOf<T>::type;

__device__ __forceinline__ f32x4 mma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x4 mma(f32x8 a, f32x8 b, f32x4 c) {
#pragma unroll
  for (int i = 0; i < 8; ++i) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a[i], b[i], c, 0, 0, 0);
  return c;
}

template <typename T> __device__ __forceinline__ Frag<T> zero_frag() {
  Frag<T> f;
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = (T)0.f;
  return f;
}
// eight elements at p, on 16 bytes (global memory or LDS)
__device__ __forceinline__ bf16x8 load_frag(const bf16 *p) { return *reinterpret_cast<const bf16x8 *>(p); }
__device__ __forceinline__ f32x8 load_frag(const float *p) {
  const f32x4 a = reinterpret_cast<const f32x4 *>(p)[0], b = reinterpret_cast<const f32x4 *>(p)[1];
  return f32x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ void store_frag(bf16 *p, bf16x8 v) { *reinterpret_cast<bf16x8 *>(p) = v; }
__device__ __forceinline__ void store_frag(float *p, f32x8 v) {
  reinterpret_cast<f32x4 *>(p)[0] = f32x4{v[0], v[1], v[2], v[3]};
  reinterpret_cast<f32x4 *>(p)[1] = f32x4{v[4], v[5], v[6], v[7]};
}

// Between a wave's writes to LDS that only it uses and its reads of them: LDS works off a wave's instructions in order.
__device__ __forceinline__ void own_lds() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
}

// Eight k of one column out of row-major LDS: column lane & 15 of the 16 at `col`, rows k0 + 0..3 and k1 + 0..3 of `pitch`
// elements.  bf16: gfx950's transposing LDS read; in each group of 16 lanes, lane j addresses four consecutive columns of
// row j >> 2, and lane l receives column l of the four rows.  8-byte alignment: pitch and col are multiples of four.
// Called by whole waves: each lane's result comes from addresses of its group's lanes.
__device__ __forceinline__ bf16x8 load_column_frag(const bf16 *lds, int pitch, int col, int k0, int k1) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  const int lane = threadIdx.x & 15, at = (lane >> 2) * pitch + col + 4 * (lane & 3);
  auto read = [&](int k) __attribute__((always_inline)) {
    return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4 *)(lds + k * pitch + at)));
  };
  const bf16x4 a = read(k0), b = read(k1);
  return bf16x8{a[0], a[1], a[2], a[3], b[0], b[1], b[2], b[3]};
}
__device__ __forceinline__ f32x8 load_column_frag(const float *lds, int pitch, int col, int k0, int k1) {
  const float *p = lds + col + (threadIdx.x & 15);
  f32x8 f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    f[i] = p[(k0 + i) * pitch];
    f[4 + i] = p[(k1 + i) * pitch];
  }
  return f;
}

}  // namespace fb
