// The counter-based stream of the dropout masks on the device: what dw_dropout.hip and dw_rms.hip share.
//
// A 64-bit number of the stream (SplitMix64's output function on a counter, Steele, Lea & Flood 2014) serves four neighbours of
// a row with 16 bits each.  Its two 64-bit products are what a number costs: with one for each element the wide cases would be bound
// by them and not by memory.  Rows begin at a number of their own, so a piece of a row that starts at a multiple of
// four elements takes whole numbers, whatever n is.
#pragma once

#include "dw_ops.h"

namespace dw {

constexpr uint64_t kStreamGamma = 0x9E3779B97F4A7C15ull;

__device__ __forceinline__ uint64_t stream_mix(uint64_t x) {
  x ^= x >> 30; x *= 0xBF58476D1CE4E5B9ull;
  x ^= x >> 27; x *= 0x94D049BB133111EBull;
  x ^= x >> 31;
  return x;
}

struct DropKey {
  uint64_t key;                                            // that of number 1 with one GAMMA taken off
  uint32_t limit;
  float factor;
  __device__ __forceinline__ DropKey(const Drop& d, int w) : limit(d.limit), factor(d.factor) {
    const uint64_t step = d.step + (d.d_step ? *d.d_step : 0ull);
    key = stream_mix(stream_mix(d.seed + kStreamGamma * (uint64_t)(w + 1)) + kStreamGamma * (step + 1));
  }
  // the counter of the number of elements 4 g .. 4 g + 3 of row r (groups: numbers of a row)
  __device__ __forceinline__ uint64_t counter(int64_t r, int64_t groups, int64_t g) const {
    return key + kStreamGamma * (uint64_t)(r * groups + g + 1);
  }
  // x of four neighbours: kept and scaled, or zero
  __device__ __forceinline__ void apply(uint64_t counter, float* x) const {
    const uint64_t u = stream_mix(counter);
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = (uint32_t)(u >> (16 * j) & 0xFFFFu) < limit ? x[j] * factor : 0.f;
  }
  // the element in column e of row r
  __device__ __forceinline__ float one(int64_t r, int64_t groups, int64_t e, float x) const {
    const uint64_t u = stream_mix(counter(r, groups, e >> 2));
    return (uint32_t)(u >> (16 * (e & 3)) & 0xFFFFu) < limit ? x * factor : 0.f;
  }
  // the V elements from column e0 (a multiple of four) of row r
  template <int V>
  __device__ __forceinline__ void piece(int64_t r, int64_t groups, int64_t e0, float (&x)[V]) const {
    const uint64_t c = counter(r, groups, e0 >> 2);
#pragma unroll
    for (int h = 0; h < V / 4; ++h) apply(c + (uint64_t)h * kStreamGamma, x + 4 * h);
  }
};

// elements e0 .. e0+V-1 of a row of n, unpacked; zeros past the end
template <class E>
__device__ __forceinline__ void load_floats16(const typename E::T* row, int64_t e0, int64_t n, float (&f)[E::V]) {
  uint32_t r[4];
  load16<E>(row, e0, n, r);
  E::unpack(r, f);
}
// as they are in memory once they are stored
template <class E>
__device__ __forceinline__ void as_stored(float (&f)[E::V]) {
  if constexpr (E::V == 8) {
    uint32_t r[4];
    E::pack(f, r);
    E::unpack(r, f);
  }
}

}  // namespace dw
