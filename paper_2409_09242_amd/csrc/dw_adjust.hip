// Logits as a token is drawn from them: penalties for tokens of the request so far, a bias, a grammar's mask (gfx950, wave64).
//
//   seen: z / repetition where z > 0, else z repetition;   c > 0 times in the answer: - (frequency c + presence);   + bias;   mask -> -inf
//
// A block takes kSpan tokens of a row: it counts those of the history that lie there in LDS, in 31 bits and one for "seen in the
// prompt" (whole numbers: the order of the additions does not matter), and then goes over the logits.  Bound by memory, the logits in
// and out; the blocks of a row read its history from the caches.
#include "dw_ops.h"

namespace dw {

namespace {

constexpr int kSpan = 8192;
constexpr uint32_t kSeen = 0x80000000u;

struct Penalties { float repetition, presence, frequency; };

__device__ __forceinline__ float penalised(float z, uint32_t count, const Penalties& p) {
  if (count == 0u) return z;
  z = z > 0.f ? z / p.repetition : z * p.repetition;
  const uint32_t c = count & ~kSeen;
  return c ? z - (p.frequency * (float)c + p.presence) : z;
}

template <class E>
__global__ __launch_bounds__(256) void adjust_kernel(AdjustArgs a) {
  constexpr int V = E::V;
  __shared__ uint32_t count[kSpan];
  const int w = blockIdx.z, vocab = (int)a.vocab;
  const int j0 = blockIdx.x * kSpan, j1 = j0 + kSpan < vocab ? j0 + kSpan : vocab;
  for (int64_t r = blockIdx.y; r < a.rows; r += gridDim.y) {
    const int64_t at = w * a.rows + r;
    int64_t filled = a.history ? a.length : 0;
    if (a.filled && a.filled[at] < filled) filled = a.filled[at] > 0 ? a.filled[at] : 0;
    const int64_t answer = a.answer ? a.answer[at] : 0;
    const int32_t* history = a.history + w * a.history_stride + r * a.history_ld;
    if (filled > 0) {                                      // (the same for the whole block)
      for (int j = threadIdx.x; j < kSpan; j += 256) count[j] = 0u;
      __syncthreads();
      for (int64_t i = threadIdx.x; i < filled; i += 256) {
        const int32_t v = history[i];
        if (v >= j0 && v < j1) {
          if (i >= answer) atomicAdd(&count[v - j0], 1u);
          else atomicOr(&count[v - j0], kSeen);
        }
      }
      __syncthreads();
    }
    const Penalties p = {a.repetition ? a.repetition[at] : 1.f, a.presence ? a.presence[at] : 0.f, a.frequency ? a.frequency[at] : 0.f};
    const typename E::T* z = reinterpret_cast<const typename E::T*>(a.logits.p) + w * a.logits.stride + r * a.logits.ld;
    typename E::T* out = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride + r * a.out.ld;
    const float* bias = a.bias ? a.bias + w * a.bias_stride + r * a.bias_ld : nullptr;
    const uint32_t* mask = a.mask ? a.mask + w * a.mask_stride + r * a.mask_ld : nullptr;
    for (int e0 = j0 + threadIdx.x * V; e0 < j1; e0 += 256 * V) {
      float f[V];
      uint32_t raw[4];
      load16<E>(z, e0, vocab, raw);
      E::unpack(raw, f);
      if (filled > 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = penalised(f[j], count[e0 - j0 + j], p);
      }
      if (bias) {
        float b[V];
        load_floats<V>(bias, e0, vocab, 0.f, b);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += b[j];
      }
      if (mask) {
        const uint32_t bits = mask[e0 >> 5] >> (e0 & 31);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = bits >> j & 1u ? f[j] : -__builtin_huge_valf();
      }
      store16<E>(out, e0, vocab, f);
    }
    if (gridDim.y < a.rows) __syncthreads();               // the next row's counts
  }
}

template <class E>
hipError_t adjust(const AdjustArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(a.vocab, kSpan), (unsigned)(a.rows < 65535 ? a.rows : 65535), (unsigned)a.k);
  hipLaunchKernelGGL(adjust_kernel<E>, grid, dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_adjust_logits(const AdjustArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? adjust<Bf16>(a, s) : adjust<F32>(a, s);
}

}  // namespace dw
