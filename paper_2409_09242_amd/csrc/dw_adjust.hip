// Logits as a token is drawn from them: penalties for tokens of the request so far, a bias, a grammar's mask (gfx950, wave64).
//
//   seen: z / repetition where z > 0, else z repetition;   c > 0 times in the answer: - (frequency c + presence);   + bias;   mask -> -inf
//
// A block takes SPAN tokens of a row: it counts those of the history that lie there in LDS, in 31 bits and one for "seen in the
// prompt" (whole numbers: the order of the additions does not matter), and then goes over the logits.  Bound by memory, the logits in
// and out; the blocks of a row read its history from the caches.  8 x 64 rows of 131072, bf16, histories of up to 2048, bias and mask:
// 65 us = 4.3 TB/s (a copy 4.75; without a history 49 to 55: the two barriers around the counts are what is left of it); fp32 98.  Four rows
// of 32000 with histories of 300: 5.3 us, two trips to memory and the barriers.  Every block of a row goes over all of its history, a piece of four
// tokens a thread on its way at a time: 63 us with histories of up to 300 and of up to 2048, 76 of up to 8192 (fp32 98 and 120), 84 where all 8192 count.
#include "dw_ops.h"

namespace dw {

namespace {

constexpr int kThreads = 256;
constexpr uint32_t kSeen = 0x80000000u;

// The division is a product with the reciprocal, and both steps are one fused operation each: an exact division costs a dozen
// instructions, and almost every wave has an element of the history somewhere.  Roundings: the reciprocal's, those of the two
// operations.
struct Penalties {
  float repetition, inverse, presence, frequency;
  __device__ __forceinline__ Penalties(const AdjustArgs& a, int64_t at)
      : repetition(a.repetition ? a.repetition[at] : 1.f), inverse(1.f / repetition), presence(a.presence ? a.presence[at] : 0.f),
        frequency(a.frequency ? a.frequency[at] : 0.f) {}
  __device__ __forceinline__ float operator()(float z, uint32_t count) const {
    const uint32_t c = count & ~kSeen;
    const float less = c ? __builtin_fmaf(frequency, (float)c, presence) : 0.f;
    const float changed = __builtin_fmaf(z, z > 0.f ? inverse : repetition, -less);
    return count ? changed : z;
  }
};

// tokens i .. i+3 of a history's `length`, -1 past its end
__device__ __forceinline__ void load_tokens(const int32_t* history, int64_t i, int64_t length, int32_t (&v)[4]) {
  if (i + 4 <= length) {
    const Raw16a4 raw = *reinterpret_cast<const Raw16a4*>(history + i);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = (int32_t)raw.w[j];
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = i + j < length ? history[i + j] : -1;
  }
}

// The logits travel while the history is counted, so a block waits for memory twice and not once for every piece.
template <class E, bool BIAS, int SPAN>
__global__ __launch_bounds__(kThreads) void adjust_kernel(AdjustArgs a) {
  constexpr int V = E::V, ITEMS = SPAN / (kThreads * V);
  __shared__ __align__(16) uint32_t count[SPAN];
  const int w = blockIdx.z, vocab = (int)a.vocab, t = threadIdx.x;
  const int j0 = blockIdx.x * SPAN, j1 = j0 + SPAN < vocab ? j0 + SPAN : vocab;
  const int pieces = (j1 - j0) / V, odd = j0 + pieces * V + t;           // whole pieces, and this thread's element behind them
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const int64_t at = w * a.rows + r;
    const typename E::T* z = reinterpret_cast<const typename E::T*>(a.logits.p) + w * a.logits.stride + r * a.logits.ld;
    const float* bias = a.bias ? a.bias + w * a.bias_stride + r * a.bias_ld : nullptr;
    const uint32_t* mask = a.mask ? a.mask + w * a.mask_stride + r * a.mask_ld : nullptr;
    uint32_t raw[ITEMS][4], bits[ITEMS];
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int q = i * kThreads + t;
      bits[i] = ~0u;
      if (q < pieces) {
        load_piece_once<E>(at_piece<E>(z + j0, q), raw[i]);
        if (mask) bits[i] = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(mask + (j0 >> 5)) + (uint32_t)(q * V >> 5 << 2));
      }
    }
    float f_odd = odd < j1 ? E::one(z + odd) : 0.f;
    const Penalties change(a, at);
    if (a.history) {
      const int32_t* history = a.history + w * a.history_stride + r * a.history_ld;
      int32_t v[4];
      load_tokens(history, t * 4, a.length, v);            // (before it is known how many of them count)
      int64_t filled = a.length;
      if (a.filled && a.filled[at] < filled) filled = a.filled[at] > 0 ? a.filled[at] : 0;
      const int64_t answer = a.answer ? a.answer[at] : 0;
      for (int j = t * 4; j < j1 - j0; j += kThreads * 4) *reinterpret_cast<uint4*>(&count[j]) = make_uint4(0u, 0u, 0u, 0u);
      __syncthreads();
      for (int64_t i = t * 4; i < filled; i += kThreads * 4) {
        int32_t now[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) now[j] = v[j];
        load_tokens(history, i + kThreads * 4, filled, v);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (now[j] >= j0 && now[j] < j1 && i + j < filled) {
            if (i + j >= answer) atomicAdd(&count[now[j] - j0], 1u);
            else atomicOr(&count[now[j] - j0], kSeen);
          }
      }
      __syncthreads();
    }
    typename E::T* out = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride + r * a.out.ld;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i * kThreads + t >= pieces) continue;
      const uint32_t q0 = (uint32_t)(i * kThreads + t), allowed = bits[i] >> (q0 * V & 31);
      float f[V], add[V];
      if constexpr (BIAS) load_floats<V>(reinterpret_cast<const float*>(reinterpret_cast<const char*>(bias + j0) + q0 * V * 4), 0, V, 0.f, add);
      E::unpack(raw[i], f);
      if (a.history) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          const uint4 c = *reinterpret_cast<const uint4*>(&count[q0 * V + 4 * q]);
          if ((c.x | c.y | c.z | c.w) != 0u) {
            f[4 * q] = change(f[4 * q], c.x);
            f[4 * q + 1] = change(f[4 * q + 1], c.y);
            f[4 * q + 2] = change(f[4 * q + 2], c.z);
            f[4 * q + 3] = change(f[4 * q + 3], c.w);
          }
        }
      }
#pragma unroll
      for (int j = 0; j < V; ++j) {
        if constexpr (BIAS) f[j] += add[j];
        f[j] = allowed >> j & 1u ? f[j] : -__builtin_huge_valf();
      }
      store_piece<E>(at_piece<E>(out + j0, (int)q0), f);
    }
    if (odd < j1) {
      if (a.history) f_odd = change(f_odd, count[odd - j0]);
      if (bias) f_odd += bias[odd];
      if (mask && !(mask[odd >> 5] >> (odd & 31) & 1u)) f_odd = -__builtin_huge_valf();
      E::put(out + odd, f_odd);
    }
    if (gridDim.y < a.rows) __syncthreads();               // the next row's counts
  }
}

// In place and without a bias or a mask only the history's tokens change: a block counts a row's in a table of SLOTS places, at
// most half full, and each place that is taken changes its one element.
template <class E, int SLOTS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void adjust_history_kernel(AdjustArgs a) {
  __shared__ __align__(16) int32_t key[SLOTS];
  __shared__ __align__(16) uint32_t count[SLOTS];
  const int w = blockIdx.y, t = threadIdx.x;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const int64_t at = w * a.rows + r;
    const int32_t* history = a.history + w * a.history_stride + r * a.history_ld;
    const int length = (int)a.length, given = a.filled ? a.filled[at] : length, filled = given < length ? given : length;
    const int answer = a.answer ? a.answer[at] : 0;
    const Penalties change(a, at);
    for (int j = t * 4; j < SLOTS; j += BLOCK * 4) {
      *reinterpret_cast<int4*>(&key[j]) = make_int4(-1, -1, -1, -1);
      *reinterpret_cast<uint4*>(&count[j]) = make_uint4(0u, 0u, 0u, 0u);
    }
    __syncthreads();
    for (int i = t; i < length; i += BLOCK) {
      const int32_t v = history[i];
      if (i >= filled || (uint32_t)v >= (uint32_t)a.vocab) continue;
      uint32_t h = (uint32_t)v * 2654435769u / (uint32_t)(0x100000000ull / SLOTS);
      for (;;) {                                           // (ends: there are at most SLOTS / 2 tokens)
        const int32_t old = atomicCAS(&key[h], -1, v);
        if (old == -1 || old == v) break;
        h = (h + 1) & (SLOTS - 1);
      }
      if (i >= answer) atomicAdd(&count[h], 1u);
      else atomicOr(&count[h], kSeen);
    }
    __syncthreads();
    typename E::T* z = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride + r * a.out.ld;
    for (int j = t; j < SLOTS; j += BLOCK)
      if (key[j] >= 0) E::put(z + key[j], change(E::one(z + key[j]), count[j]));
    __syncthreads();                                       // the next row's table
  }
}

template <class E>
hipError_t adjust(const AdjustArgs& a, hipStream_t s) {
  if (a.out.p == a.logits.p && !a.bias && !a.mask && !a.history) return hipSuccess;
  // A token costs a line read and written, 128 bytes, a logit that is gone over 4 or 8.  512 rows of 131072, bf16, in place, by tokens
  // and by all logits (us): histories of 1024 random tokens 22 and 58, 2048 45 and 64, 8192 150 and 107; of 2048 as they come in text
  // 22 and 61
  if (a.out.p == a.logits.p && !a.bias && !a.mask && a.length <= a.vocab / 32 && a.length <= 8192) {
    const dim3 grid((unsigned)(a.rows < (1 << 20) ? a.rows : 1 << 20), (unsigned)a.k);
    if (a.length <= 1024) {
      hipLaunchKernelGGL((adjust_history_kernel<E, 2048, 256>), grid, dim3(256), 0, s, a);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((adjust_history_kernel<E, 16384, 1024>), grid, dim3(1024), 0, s, a);
    return hipGetLastError();
  }
  // four pieces a thread (512 rows of 131072, bf16, everything on, before other steps: 69 us; with spans of 4096 71, 2048 93, 16384 83)
  constexpr int SPAN = 4 * kThreads * E::V;
  const dim3 grid((unsigned)ceil_div(a.vocab, SPAN), (unsigned)(a.rows < 65535 ? a.rows : 65535), (unsigned)a.k);
  if (a.bias) hipLaunchKernelGGL((adjust_kernel<E, true, SPAN>), grid, dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((adjust_kernel<E, false, SPAN>), grid, dim3(kThreads), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust_logits(const AdjustArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? adjust<Bf16>(a, s) : adjust<F32>(a, s);
}

}  // namespace dw
