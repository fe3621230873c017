// Layer norm of the rows of k workers and its backward pass (gfx950, wave64).
//
//   y = (x - mu) r gamma + beta,   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps)      over a row of n
//   with h = (x - mu) r and a = dy gamma:
//   dx = r (a - mean(a) - h mean(a h)),   dgamma = sum over rows of dy h,   dbeta = sum over rows of dy
//
// TPR threads share a row and keep it in registers as ITEMS pieces of 16 bytes each, so x (and dy) are read once; sums
// over a row go through the lanes and, above a wave, through LDS.  The variance is the mean of squared differences from
// the mean that is already there, never a difference of two sums.  All sums are in fp32.
//
// Backward: a group of threads takes every strips-th row of one worker, and the column sums of its rows stay in the
// registers of the threads that own the columns; one row of partial sums per block goes to scratch, and a second
// kernel adds those up in their order, so results do not depend on the order in which blocks run.
#include "dw_ops.h"

namespace dw {

namespace {

// blocks of `groups` rows at a time: enough to fill the chip a few times over, shared among the workers
inline int64_t blocks_per_worker(int k, int64_t rows, int groups, int64_t target) {
  const int64_t most = ceil_div(rows, groups), share = ceil_div(target, k);
  return most < share ? most : share;
}

template <class E, int TPR, int ITEMS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void layer_norm_kernel(NormArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  const int64_t n = a.n;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float* beta = a.beta ? a.beta + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)n;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // every group of a block goes round the same number of times (the block's barriers are for TPR > 64, where it is one)
  for (int64_t r = (int64_t)blockIdx.x * GROUPS + g; r < a.rows; r += step) {
    const typename E::T* xr = x + r * a.x.ld;
    float v[ITEMS][V];
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      uint32_t raw[4];
      load16<E>(xr, (int64_t)(i * TPR + t) * V, n, raw);
      E::unpack(raw, v[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += v[i][j];
    }
    const float mean = row_sum<TPR>(sum, red, turn) * inv_n;
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int64_t e0 = (int64_t)(i * TPR + t) * V;
      if (e0 + V <= n) {
#pragma unroll
        for (int j = 0; j < V; ++j) { v[i][j] -= mean; sq += v[i][j] * v[i][j]; }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (e0 + j < n) { v[i][j] -= mean; sq += v[i][j] * v[i][j]; }
      }
    }
    const float var = row_sum<TPR>(sq, red, turn) * inv_n;
    const float rstd = 1.f / sqrtf(var + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[w * a.rows + r] = mean;
      if (a.rstd) a.rstd[w * a.rows + r] = rstd;
    }
    typename E::T* yr = y + r * a.out.ld;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int64_t e0 = (int64_t)(i * TPR + t) * V;
      if (e0 < n) {
        float ga[V], be[V], o[V];
#pragma unroll
        for (int j = 0; j < V; ++j) { ga[j] = 1.f; be[j] = 0.f; }
        if (gamma) load_floats<V>(gamma, e0, n, 1.f, ga);
        if (beta) load_floats<V>(beta, e0, n, 0.f, be);
#pragma unroll
        for (int j = 0; j < V; ++j) o[j] = v[i][j] * rstd * ga[j] + be[j];
        store16<E>(yr, e0, n, o);
      }
    }
  }
}

// rows too long for registers: a block goes over the row three times (the second and third from the caches)
template <class E>
__global__ __launch_bounds__(1024) void layer_norm_long_kernel(NormArgs a) {
  constexpr int V = E::V, TPR = 1024;
  __shared__ float red[2 * TPR / 64];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x;
  const int64_t n = a.n;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float* beta = a.beta ? a.beta + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)n;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const typename E::T* xr = x + r * a.x.ld;
    float sum = 0.f, sq = 0.f, v[V];
    uint32_t raw[4];
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      load16<E>(xr, e0, n, raw);
      E::unpack(raw, v);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += v[j];
    }
    const float mean = row_sum<TPR>(sum, red, turn) * inv_n;
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      load16<E>(xr, e0, n, raw);
      E::unpack(raw, v);
#pragma unroll
      for (int j = 0; j < V; ++j) { const float d = e0 + j < n ? v[j] - mean : 0.f; sq += d * d; }
    }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, red, turn) * inv_n + a.eps);
    if (t == 0) {
      if (a.mean) a.mean[w * a.rows + r] = mean;
      if (a.rstd) a.rstd[w * a.rows + r] = rstd;
    }
    typename E::T* yr = y + r * a.out.ld;
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      float ga[V], be[V];
      load16<E>(xr, e0, n, raw);
      E::unpack(raw, v);
#pragma unroll
      for (int j = 0; j < V; ++j) { ga[j] = 1.f; be[j] = 0.f; }
      if (gamma) load_floats<V>(gamma, e0, n, 1.f, ga);
      if (beta) load_floats<V>(beta, e0, n, 0.f, be);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = (v[j] - mean) * rstd * ga[j] + be[j];
      store16<E>(yr, e0, n, v);
    }
  }
}

template <class E, int TPR, int ITEMS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void layer_norm_grad_kernel(NormArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  constexpr int COLS = TPR * ITEMS * V;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  __shared__ float cols[GROUPS > 1 ? GROUPS * COLS : 1];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x % TPR, g = threadIdx.x / TPR;
  const int64_t n = a.n;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  typename E::T* dx = a.out.p ? reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride : nullptr;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)n;
  float dg[ITEMS][V], db[ITEMS][V], ga[ITEMS][V];
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) { dg[i][j] = 0.f; db[i][j] = 0.f; ga[i][j] = 1.f; }
    if (gamma) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 0.f, ga[i]);
  }
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  for (int64_t r = (int64_t)blockIdx.x * GROUPS + g; r < a.rows; r += step) {
    const float mean = a.mean[w * a.rows + r], rstd = a.rstd[w * a.rows + r];
    float h[ITEMS][V], v[ITEMS][V];
    float s1 = 0.f, s2 = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      uint32_t raw[4];
      const int64_t e0 = (int64_t)(i * TPR + t) * V;
      load16<E>(x + r * a.x.ld, e0, n, raw);
      E::unpack(raw, h[i]);
      load16<E>(dy + r * a.dy.ld, e0, n, raw);
      E::unpack(raw, v[i]);
      if (e0 < n) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[i][j] = (h[i][j] - mean) * rstd;
          dg[i][j] += v[i][j] * h[i][j];
          db[i][j] += v[i][j];
          v[i][j] *= ga[i][j];                             // past the end: dy reads as zero
          s1 += v[i][j];
          s2 += v[i][j] * h[i][j];
        }
      }
    }
    if (dx) {
      const float c1 = row_sum<TPR>(s1, red, turn) * inv_n, c2 = row_sum<TPR>(s2, red, turn) * inv_n;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int64_t e0 = (int64_t)(i * TPR + t) * V;
        if (e0 < n) {
          float o[V];
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = rstd * (v[i][j] - c1 - h[i][j] * c2);
          store16<E>(dx + r * a.out.ld, e0, n, o);
        }
      }
    }
  }
  if (!a.part) return;
  // the block's column sums: the groups' in order, dgamma's first and then dbeta's through the same LDS
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * 2 * n;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      const int64_t e0 = (int64_t)(i * TPR + t) * V;
#pragma unroll
      for (int j = 0; j < V; ++j)
        if (e0 + j < n) { out[e0 + j] = dg[i][j]; out[n + e0 + j] = db[i][j]; }
    }
  } else {
    for (int part = 0; part < 2; ++part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) cols[g * COLS + (i * TPR + t) * V + j] = part ? db[i][j] : dg[i][j];
      __syncthreads();
      for (int e = threadIdx.x; e < n; e += BLOCK) {
        float s = cols[e];
#pragma unroll
        for (int q = 1; q < GROUPS; ++q) s += cols[q * COLS + e];
        out[part * n + e] = s;
      }
    }
  }
}

// rows too long for registers: the sums over the row, then dx; the column sums are another kernel's
template <class E>
__global__ __launch_bounds__(1024) void layer_norm_grad_long_kernel(NormArgs a) {
  constexpr int V = E::V, TPR = 1024;
  __shared__ float red[2 * TPR / 64];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x;
  const int64_t n = a.n;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  typename E::T* dx = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)n;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mean = a.mean[w * a.rows + r], rstd = a.rstd[w * a.rows + r];
    float s1 = 0.f, s2 = 0.f, h[V], v[V], ga[V];
    uint32_t raw[4];
    auto read = [&](int64_t e0) {
      load16<E>(x + r * a.x.ld, e0, n, raw);
      E::unpack(raw, h);
      load16<E>(dy + r * a.dy.ld, e0, n, raw);
      E::unpack(raw, v);
#pragma unroll
      for (int j = 0; j < V; ++j) ga[j] = 1.f;
      if (gamma) load_floats<V>(gamma, e0, n, 0.f, ga);
#pragma unroll
      for (int j = 0; j < V; ++j) { h[j] = (h[j] - mean) * rstd; v[j] *= ga[j]; }
    };
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      read(e0);
#pragma unroll
      for (int j = 0; j < V; ++j) { s1 += v[j]; s2 += v[j] * h[j]; }
    }
    const float c1 = row_sum<TPR>(s1, red, turn) * inv_n, c2 = row_sum<TPR>(s2, red, turn) * inv_n;
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      read(e0);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = rstd * (v[j] - c1 - h[j] * c2);
      store16<E>(dx + r * a.out.ld, e0, n, v);
    }
  }
}

// column sums for long rows: a thread owns V columns, a block every strips-th row
template <class E>
__global__ __launch_bounds__(256) void layer_norm_cols_kernel(NormArgs a) {
  constexpr int V = E::V;
  const int w = blockIdx.z;
  const int64_t n = a.n, e0 = ((int64_t)blockIdx.y * 256 + threadIdx.x) * V;
  if (e0 >= n) return;
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  float dg[V], db[V], h[V], v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) dg[j] = db[j] = 0.f;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float mean = a.mean[w * a.rows + r], rstd = a.rstd[w * a.rows + r];
    uint32_t raw[4];
    load16<E>(x + r * a.x.ld, e0, n, raw);
    E::unpack(raw, h);
    load16<E>(dy + r * a.dy.ld, e0, n, raw);
    E::unpack(raw, v);
#pragma unroll
    for (int j = 0; j < V; ++j) { dg[j] += v[j] * ((h[j] - mean) * rstd); db[j] += v[j]; }
  }
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * 2 * n;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (e0 + j < n) { out[e0 + j] = dg[j]; out[n + e0 + j] = db[j]; }
}

// dgamma and dbeta from the blocks' partial sums: 64 columns a block, its 16 waves take every 16th strip each
__global__ __launch_bounds__(1024) void layer_norm_strips_kernel(NormArgs a) {
  __shared__ float lds[16][64];
  const int w = blockIdx.z, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int which = blockIdx.y;
  float* out = which ? a.dbeta : a.dgamma;
  if (!out) return;
  const int64_t n = a.n, e = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (e < n)
    for (int p = wave; p < a.strips; p += 16) s += a.part[(((int64_t)w * a.strips + p) * 2 + which) * n + e];
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && e < n) {
#pragma unroll
    for (int q = 1; q < 16; ++q) s += lds[q][lane];
    out[w * a.grad_stride + e] = s;
  }
}

// threads that share a row and 16-byte pieces a thread holds: the fewest threads whose registers take the row
struct NormShape { int tpr, items; };
NormShape norm_shape(int64_t n, int V) {
  const int64_t pieces = ceil_div(n, V);
  if (pieces <= 16) return {16, 1};
  if (pieces <= 64) return {64, 1};
  if (pieces <= 128) return {64, 2};
  if (pieces <= 256) return {256, 1};
  if (pieces <= 512) return {256, 2};
  if (pieces <= 1024) return {256, 4};
  if (pieces <= 2048) return {1024, 2};
  return {0, 0};
}

template <class E, int TPR, int ITEMS, int BLOCK>
hipError_t fwd(const NormArgs& a, hipStream_t s) {
  const dim3 grid((unsigned)blocks_per_worker(a.k, a.rows, BLOCK / TPR, 8 * kCus), (unsigned)a.k);
  hipLaunchKernelGGL((layer_norm_kernel<E, TPR, ITEMS, BLOCK>), grid, dim3(BLOCK), 0, s, a);
  return hipGetLastError();
}
template <class E>
hipError_t fwd_any(const NormArgs& a, hipStream_t s) {
  const NormShape c = norm_shape(a.n, E::V);
  if (c.tpr == 16) return fwd<E, 16, 1, 256>(a, s);
  if (c.tpr == 64) return c.items == 1 ? fwd<E, 64, 1, 256>(a, s) : fwd<E, 64, 2, 256>(a, s);
  if (c.tpr == 256) return c.items == 1 ? fwd<E, 256, 1, 256>(a, s) : c.items == 2 ? fwd<E, 256, 2, 256>(a, s) : fwd<E, 256, 4, 256>(a, s);
  if (c.tpr == 1024) return fwd<E, 1024, 2, 1024>(a, s);
  hipLaunchKernelGGL(layer_norm_long_kernel<E>, dim3((unsigned)blocks_per_worker(a.k, a.rows, 1, 4 * kCus), (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <class E, int TPR, int ITEMS, int BLOCK>
hipError_t bwd(const NormArgs& a, hipStream_t s) {
  hipLaunchKernelGGL((layer_norm_grad_kernel<E, TPR, ITEMS, BLOCK>), dim3((unsigned)a.strips, (unsigned)a.k), dim3(BLOCK), 0, s, a);
  return hipGetLastError();
}
template <class E>
hipError_t bwd_any(const NormArgs& a, hipStream_t s) {
  const NormShape c = norm_shape(a.n, E::V);
  if (c.tpr == 16) return bwd<E, 16, 1, 256>(a, s);
  if (c.tpr == 64) return c.items == 1 ? bwd<E, 64, 1, 256>(a, s) : bwd<E, 64, 2, 256>(a, s);
  if (c.tpr == 256) return c.items == 1 ? bwd<E, 256, 1, 256>(a, s) : c.items == 2 ? bwd<E, 256, 2, 256>(a, s) : bwd<E, 256, 4, 256>(a, s);
  if (c.tpr == 1024) return bwd<E, 1024, 2, 1024>(a, s);
  if (a.out.p) {
    hipLaunchKernelGGL(layer_norm_grad_long_kernel<E>, dim3((unsigned)blocks_per_worker(a.k, a.rows, 1, 4 * kCus), (unsigned)a.k), dim3(1024), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  if (!a.part) return hipSuccess;
  hipLaunchKernelGGL(layer_norm_cols_kernel<E>, dim3((unsigned)a.strips, (unsigned)ceil_div(a.n, 256 * E::V), (unsigned)a.k), dim3(256), 0, s, a);
  return hipGetLastError();
}

}  // namespace

int layer_norm_grad_strips(int k, int64_t rows, int64_t n, int dtype) {
  const NormShape c = norm_shape(n, dtype == DW_BF16 ? Bf16::V : F32::V);
  const int groups = c.tpr >= 256 || c.tpr == 0 ? 1 : 256 / c.tpr;
  return (int)blocks_per_worker(k, rows, groups, c.tpr == 1024 ? kCus : 2 * kCus);
}

hipError_t launch_layer_norm(const NormArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? fwd_any<Bf16>(a, s) : fwd_any<F32>(a, s);
}

hipError_t launch_layer_norm_grad(const NormArgs& a, bool sums, int dtype, hipStream_t s) {
  if (a.rows > 0) {
    const hipError_t e = dtype == DW_BF16 ? bwd_any<Bf16>(a, s) : bwd_any<F32>(a, s);
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;                            // (no rows: no strips, and the sums are zero)
  hipLaunchKernelGGL(layer_norm_strips_kernel, dim3((unsigned)ceil_div(a.n, 64), 2, (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace dw
