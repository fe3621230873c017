// Dropout with a mask that is stored nowhere, and the residual's addition behind it (gfx950, wave64).
//
//   y = residual + m x / q,   m and q from the counter-based stream of dw_dropout.h
//
// A group of threads takes a row at a time, 16 bytes of it a thread.
#include "dw_dropout.h"

namespace dw {

namespace {

template <class E>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int log_tpr) {
  constexpr int V = E::V;
  const int w = blockIdx.y, t = threadIdx.x & ((1 << log_tpr) - 1), g = threadIdx.x >> log_tpr;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* res = a.res.p ? reinterpret_cast<const typename E::T*>(a.res.p) + w * a.res.stride : nullptr;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.y.p) + w * a.y.stride;
  const DropKey key(a.drop, w);
  const int64_t n = a.n, groups = ceil_div(n, 4), step = (int64_t)gridDim.x * (256 >> log_tpr);
  for (int64_t r = (int64_t)blockIdx.x * (256 >> log_tpr) + g; r < a.rows; r += step) {
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += (int64_t)V << log_tpr) {
      float f[V];
      load_floats16<E>(x + r * a.x.ld, e0, n, f);
      key.piece<V>(r, groups, e0, f);
      if (res) {
        float b[V];
        load_floats16<E>(res + r * a.res.ld, e0, n, b);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += b[j];
      }
      store16<E>(y + r * a.y.ld, e0, n, f);
    }
  }
}

template <class E>
hipError_t dropout(const DropoutArgs& a, hipStream_t s) {
  const int64_t pieces = ceil_div(a.n, E::V);
  int log_tpr = 0;
  while (log_tpr < 8 && (1 << log_tpr) < pieces) ++log_tpr;
  int64_t blocks = ceil_div(a.rows, 256 >> log_tpr);
  const int64_t most = 16 * kCus / a.k > 1 ? 16 * kCus / a.k : 1;
  if (blocks > most) blocks = most;
  hipLaunchKernelGGL(dropout_kernel<E>, dim3((unsigned)blocks, (unsigned)a.k), dim3(256), 0, s, a, log_tpr);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? dropout<Bf16>(a, s) : dropout<F32>(a, s);
}

}  // namespace dw
