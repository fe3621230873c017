// Numbers in e4m3 on the device: what the quantiser (dw_fp8_quant.hip) and the products that quantise on the way
// (dw_gemm_fp8.hip) share.
#pragma once

#include "dw_ops.h"

namespace dw {

// eight elements of a row as they are in memory
template <class E>
struct Raw8 {
  uint32_t w[8 / E::V][4];
  // elements e0 .. e0+7 of a row of n (zero past the end)
  __device__ __forceinline__ void load(const typename E::T* row, int64_t e0, int64_t n) {
#pragma unroll
    for (int h = 0; h < 8 / E::V; ++h) load16<E>(row, e0 + h * E::V, n, w[h]);
  }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int h = 0; h < 8 / E::V; ++h)
#pragma unroll
      for (int j = 0; j < 4; ++j) w[h][j] = 0u;
  }
  __device__ __forceinline__ void floats(float (&f)[8]) const {
#pragma unroll
    for (int h = 0; h < 8 / E::V; ++h) {
      float v[E::V];
      E::unpack(w[h], v);
#pragma unroll
      for (int j = 0; j < E::V; ++j) f[h * E::V + j] = v[j];
    }
  }
  __device__ __forceinline__ float one(int j) const {       // (j is a constant where this is used)
    const uint32_t u = w[j / E::V][E::V == 8 ? j / 2 : j % 4];
    return __uint_as_float(E::V == 4 ? u : j & 1 ? u & 0xFFFF0000u : u << 16);
  }
  // what it holds is unpacked anew where it is used next: registers hold it packed in between
  __device__ __forceinline__ void keep_packed() {
#pragma unroll
    for (int h = 0; h < 8 / E::V; ++h) asm volatile("" : "+v"(w[h][0]), "+v"(w[h][1]), "+v"(w[h][2]), "+v"(w[h][3]));
  }
};

__device__ __forceinline__ uint32_t magnitude(float f) { return __float_as_uint(f) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t larger(uint32_t a, uint32_t b) { return a > b ? a : b; }

// the largest of the 16 lanes of a row of lanes, to all of them: neighbours, pairs, halves of eight, eights
template <int CTRL>
__device__ __forceinline__ uint32_t lane_move(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true); }
__device__ __forceinline__ uint32_t largest_of_16(uint32_t v) {
  v = larger(v, lane_move<0xB1>(v));                        // quad_perm 1 0 3 2
  v = larger(v, lane_move<0x4E>(v));                        // quad_perm 2 3 0 1
  v = larger(v, lane_move<0x141>(v));                       // the eight reversed: the other four's
  return larger(v, lane_move<0x140>(v));                    // the sixteen reversed: the other eight's
}

struct Scale { uint32_t byte; float inverse; };
__device__ __forceinline__ Scale scale_of(uint32_t top) {
  if (top == 0u) return {127u, 1.f};
  if (top >= 0x7F800000u) return {127u, __uint_as_float(0x7FC00000u)};
  int e = (int)(top >> 23) - 127 - 8 + ((top & 0x7FFFFFu) > 0x600000u ? 1 : 0);
  e = e < -126 ? -126 : e;
  return {(uint32_t)(e + 127), __uint_as_float((uint32_t)(127 - e) << 23)};
}

__device__ __forceinline__ uint2 to_e4m3(const float (&f)[8], float inverse) {
  int lo = 0, hi = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[0] * inverse, f[1] * inverse, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(f[2] * inverse, f[3] * inverse, lo, true);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[4] * inverse, f[5] * inverse, hi, false);
  hi = __builtin_amdgcn_cvt_pk_fp8_f32(f[6] * inverse, f[7] * inverse, hi, true);
  return make_uint2((uint32_t)lo, (uint32_t)hi);
}

}  // namespace dw
