// Dropout with a mask that is stored nowhere, and the residual's addition behind it (gfx950, wave64).
//
//   y = residual + m x / q,   m and q from the counter-based stream of dw_dropout.h
//
// A group of threads takes a row at a time, 16 bytes of it a thread.  Bound by memory: 8 x 4096 rows of 4096, bf16, with a residual 139 us
// = 5.8 TB/s (outputs that the chip's cache holds from call to call: 120), the mask's arithmetic behind it; read without displacing what
// is read again (otherwise 150), and many blocks (16 a compute unit instead of 64: 4 to 7 % longer).  37 rows of 513, fp32, for four
// workers 2.8 us, about a launch.  A row is one block's at most: few rows are bound by its trips and not by memory (1 row of 16384, fp32, still about a
// launch, 4.9 us a call; 4 rows of 2^20, bf16, 256 us).
#include "dw_dropout.h"

namespace dw {

namespace {

// a thread takes every tpr-th piece of its group's row; the elements behind the row's whole pieces one each
template <class E, bool RES>
__global__ __launch_bounds__(256) void dropout_kernel(DropoutArgs a, int log_tpr) {
  constexpr int V = E::V;
  const int w = blockIdx.y, tpr = 1 << log_tpr, t = threadIdx.x & (tpr - 1), g = threadIdx.x >> log_tpr;
  const int n = (int)a.n, whole = n / V;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* res = reinterpret_cast<const typename E::T*>(a.res.p) + w * a.res.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.y.p) + w * a.y.stride;
  const DropKey key(a.drop, w);
  const int64_t groups = ceil_div(n, 4), step = (int64_t)gridDim.x * (256 >> log_tpr);
  for (int64_t r = (int64_t)blockIdx.x * (256 >> log_tpr) + g; r < a.rows; r += step) {
    const typename E::T* xr = x + r * a.x.ld;
    const typename E::T* rr = res + r * a.res.ld;
    typename E::T* yr = y + r * a.y.ld;
    for (int q = t; q < whole; q += tpr) {
      uint32_t raw[4], add[4];
      load_piece_once<E>(at_piece<E>(xr, q), raw);
      if constexpr (RES) load_piece_once<E>(at_piece<E>(rr, q), add);
      float f[V];
      E::unpack(raw, f);
      key.piece<V>(r, groups, (int64_t)q * V, f);
      if constexpr (RES) {
        float b[V];
        E::unpack(add, b);
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] += b[j];
      }
      store_piece<E>(at_piece<E>(yr, q), f);
    }
    for (int e = whole * V + t; e < n; e += tpr) {
      const float f = key.one(r, groups, e, E::one(xr + e));
      E::put(yr + e, RES ? f + E::one(rr + e) : f);
    }
  }
}

template <class E>
hipError_t dropout(const DropoutArgs& a, hipStream_t s) {
  const int64_t pieces = a.n / E::V;
  int log_tpr = 0;
  while (log_tpr < 8 && (1 << log_tpr) < pieces) ++log_tpr;
  int64_t blocks = ceil_div(a.rows, 256 >> log_tpr);
  const int64_t most = 64 * kCus / a.k;
  if (blocks > most) blocks = most;
  const dim3 grid((unsigned)blocks, (unsigned)a.k);
  if (a.res.p) hipLaunchKernelGGL((dropout_kernel<E, true>), grid, dim3(256), 0, s, a, log_tpr);
  else hipLaunchKernelGGL((dropout_kernel<E, false>), grid, dim3(256), 0, s, a, log_tpr);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? dropout<Bf16>(a, s) : dropout<F32>(a, s);
}

}  // namespace dw
