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
//
// Bound by memory: 16 x 512 rows of 4096, bf16, 23.5 us = 5.7 TB/s; the backward pass of 3 x 2731 rows of 5003, fp32, 82 us =
// 6.0 TB/s, and 6 for the columns' sums (on data that is in no cache 100 in all).  One row: 3.2 us, which is what a launch and
// two trips to memory take.
#include "dw_ops.h"

namespace dw {

namespace {

// blocks of `groups` rows at a time: `target` of them over all workers at most, so that they run all at once, and one a worker
inline int64_t blocks_per_worker(int k, int64_t rows, int groups, int64_t target) {
  const int64_t most = ceil_div(rows, groups), share = target > k ? target / k : 1;
  return most < share ? most : share;
}

// A row of n is its whole pieces of 16 bytes, piece i * TPR + t to thread t, and fewer than V elements more, one each to the
// first threads: every access is in bounds and no piece needs a mask of its own.  for_row sees to it that there are as many
// threads as odd elements.
template <class E, int TPR>
struct Split {
  int whole, tail;                                         // whole pieces; this thread's element behind them
  bool has_tail;
  __device__ __forceinline__ Split(int64_t n, int t) : whole((int)(n / E::V)), tail(whole * E::V + t), has_tail(tail < (int)n) {}
};

// ITEMS pieces of a row and its odd element, as they are in memory; what a thread has not reads as zero.  ONCE: with the
// policy of data that streams through
template <class E, int TPR, int ITEMS, bool ONCE>
struct RowRegs {
  uint32_t piece[ITEMS][4];
  float odd;
  __device__ __forceinline__ void load(const typename E::T* row, const Split<E, TPR>& s, int t) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i * TPR + t < s.whole) {
        if constexpr (ONCE) load_piece_once<E>(at_piece<E>(row, i * TPR + t), piece[i]);
        else load_piece<E>(at_piece<E>(row, i * TPR + t), piece[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) piece[i][j] = 0u;
      }
    }
    odd = s.has_tail ? E::one(row + s.tail) : 0.f;
  }
};

// FEW: gamma and beta of the thread's columns stay in registers over its rows
template <class E, int TPR, int ITEMS, int BLOCK, bool FEW>
__global__ __launch_bounds__(BLOCK) void layer_norm_kernel(NormArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  int turn = 0;
  const int w = blockIdx.y, t = GROUPS == 1 ? threadIdx.x : threadIdx.x % TPR, g = GROUPS == 1 ? 0 : threadIdx.x / TPR;
  const Split<E, TPR> split(a.n, t);
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float* beta = a.beta ? a.beta + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)a.n;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  // every group of a block goes round the same number of times (the block's barriers are for TPR > 64, where it is one)
  int64_t r = (int64_t)blockIdx.x * GROUPS + g;
  RowRegs<E, TPR, ITEMS, false> next;
  if (r < a.rows) next.load(x + r * a.x.ld, split, t);     // the first row travels along with gamma and beta
  float ga[ITEMS][V], be[ITEMS][V], ga_odd = 1.f, be_odd = 0.f;
  auto param = [&](const float* p, float fill, int i, float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = fill;
    if (p && i * TPR + t < split.whole) load_floats<V>(p, (int64_t)(i * TPR + t) * V, a.n, fill, f);
  };
  if constexpr (FEW) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) { param(gamma, 1.f, i, ga[i]); param(beta, 0.f, i, be[i]); }
  }
  if (split.has_tail) {
    if (gamma) ga_odd = gamma[split.tail];
    if (beta) be_odd = beta[split.tail];
  }
  for (; r < a.rows; r += step) {
    float v[ITEMS][V];
    float sum = next.odd;
    const float odd = next.odd;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      E::unpack(next.piece[i], v[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += v[i][j];
    }
    if (r + step < a.rows) next.load(x + (r + step) * a.x.ld, split, t);
    const float mean = row_sum<TPR>(sum, red, turn) * inv_n;
    const float odd_off = odd - mean;
    float sq = split.has_tail ? odd_off * odd_off : 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i * TPR + t < split.whole) {
#pragma unroll
        for (int j = 0; j < V; ++j) { v[i][j] -= mean; sq += v[i][j] * v[i][j]; }
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
      if (i * TPR + t < split.whole) {
        if constexpr (!FEW) { param(gamma, 1.f, i, ga[i]); param(beta, 0.f, i, be[i]); }
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * rstd * ga[i][j] + be[i][j];
        store_piece<E>(at_piece<E>(yr, i * TPR + t), v[i]);
      }
    }
    if (split.has_tail) E::put(yr + split.tail, odd_off * rstd * ga_odd + be_odd);
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

// Registers hold x, dy and the column sums of a thread's pieces, gamma, and the next row on its way; 1024 threads have half
// as many each, so there gamma comes from the caches and the next row is not fetched ahead.
template <class E, int TPR, int ITEMS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void layer_norm_grad_kernel(NormArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  constexpr bool AHEAD = TPR < 1024;
  constexpr int COLS = TPR * ITEMS * V;
  __shared__ float red[4 * (TPR > 64 ? TPR / 64 : 1)];
  __shared__ float cols[GROUPS > 1 ? GROUPS * (COLS + V) : 1];
  int turn = 0;
  const int w = blockIdx.y, t = GROUPS == 1 ? threadIdx.x : threadIdx.x % TPR, g = GROUPS == 1 ? 0 : threadIdx.x / TPR;
  const int64_t n = a.n;
  const Split<E, TPR> split(n, t);
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  typename E::T* dx = a.out.p ? reinterpret_cast<typename E::T*>(a.out.p) + w * a.out.stride : nullptr;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const float inv_n = 1.f / (float)n;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  int64_t r = (int64_t)blockIdx.x * GROUPS + g;
  // fp32 streams through (8192 x 4096: 74 us, otherwise 84); rows of bf16 share lines with their neighbours more often, which then
  // come twice (3 x 2731 x 5003: 133 against 113)
  RowRegs<E, TPR, ITEMS, E::V == 4> next_x, next_dy;
  float next_mean = 0.f, next_rstd = 0.f;
  auto fetch = [&](int64_t row) {
    next_x.load(x + row * a.x.ld, split, t);
    next_dy.load(dy + row * a.dy.ld, split, t);
    next_mean = a.mean[w * a.rows + row];
    next_rstd = a.rstd[w * a.rows + row];
  };
  if (AHEAD && r < a.rows) fetch(r);
  float dg[ITEMS][V], db[ITEMS][V], ga[ITEMS][V], dg_odd = 0.f, db_odd = 0.f, ga_odd = 1.f;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) { dg[i][j] = 0.f; db[i][j] = 0.f; ga[i][j] = 1.f; }
    if (AHEAD && gamma && i * TPR + t < split.whole) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 1.f, ga[i]);
  }
  if (gamma && split.has_tail) ga_odd = gamma[split.tail];
  for (; r < a.rows; r += step) {
    if constexpr (!AHEAD) fetch(r);
    const float mean = next_mean, rstd = next_rstd;
    float h[ITEMS][V], v[ITEMS][V];
    float s1 = 0.f, s2 = 0.f, h_odd = 0.f, v_odd = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      E::unpack(next_x.piece[i], h[i]);
      E::unpack(next_dy.piece[i], v[i]);
      if (i * TPR + t < split.whole) {
        float here[V];
        if (!AHEAD) {
#pragma unroll
          for (int j = 0; j < V; ++j) here[j] = 1.f;
          if (gamma) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 1.f, here);
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          h[i][j] = (h[i][j] - mean) * rstd;
          dg[i][j] += v[i][j] * h[i][j];
          db[i][j] += v[i][j];
          v[i][j] *= AHEAD ? ga[i][j] : here[j];
          s1 += v[i][j];
          s2 += v[i][j] * h[i][j];
        }
      }
    }
    if (split.has_tail) {
      h_odd = (next_x.odd - mean) * rstd;
      dg_odd += next_dy.odd * h_odd;
      db_odd += next_dy.odd;
      v_odd = next_dy.odd * ga_odd;
      s1 += v_odd;
      s2 += v_odd * h_odd;
    }
    if (AHEAD && r + step < a.rows) fetch(r + step);
    if (dx) {
      float c1, c2;
      row_sum2<TPR>(s1, s2, red, turn, c1, c2);
      c1 *= inv_n;
      c2 *= inv_n;
      typename E::T* out = dx + r * a.out.ld;
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        if (i * TPR + t < split.whole) {
          float o[V];
#pragma unroll
          for (int j = 0; j < V; ++j) o[j] = rstd * (v[i][j] - c1 - h[i][j] * c2);
          store_piece<E>(at_piece<E>(out, i * TPR + t), o);
        }
      }
      if (split.has_tail) E::put(out + split.tail, rstd * (v_odd - c1 - h_odd * c2));
    }
  }
  if (!a.part) return;
  // the block's column sums: the groups' in order, dgamma's first and then dbeta's through the same LDS
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * 2 * n;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i * TPR + t < split.whole) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          const int64_t e = (int64_t)(i * TPR + t) * V + 4 * q;
          const float fg[4] = {dg[i][4 * q], dg[i][4 * q + 1], dg[i][4 * q + 2], dg[i][4 * q + 3]};
          const float fb[4] = {db[i][4 * q], db[i][4 * q + 1], db[i][4 * q + 2], db[i][4 * q + 3]};
          store_piece<F32>(out + e, fg);
          store_piece<F32>(out + n + e, fb);
        }
      }
    if (split.has_tail) { out[split.tail] = dg_odd; out[n + split.tail] = db_odd; }
  } else {
    for (int part = 0; part < 2; ++part) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) cols[g * (COLS + V) + (i * TPR + t) * V + j] = part ? db[i][j] : dg[i][j];
      __syncthreads();                                     // (the odd elements' places may be those of a piece that is not there)
      if (split.has_tail) cols[g * (COLS + V) + split.tail] = part ? db_odd : dg_odd;
      __syncthreads();
      for (int e = threadIdx.x; e < n; e += BLOCK) {
        float s = cols[e];
#pragma unroll
        for (int q = 1; q < GROUPS; ++q) s += cols[q * (COLS + V) + e];
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

// f.template operator()<TPR, ITEMS>() for a row of n: the fewest threads whose registers take its whole pieces in up to two
// each, then up to four of 512 and (WIDE) of 1024, and at least as many as it has odd elements; false: too long.  In bf16 the
// shortest rows have up to seven of those, and four threads only where four will do (us, forward and backward, by four and by
// eight: 16 x 8192 x 32: 5.4 and 9.4, 6.8 and 11.1; 4 x 512 x 16 alike)
template <class E, bool WIDE, class F>
bool for_row(int64_t n, F f) {
  constexpr int FEWEST = 4;
  static_assert(E::V >= FEWEST && 16 >= E::V - 1, "every form but the first takes any number of odd elements");
  const int64_t pieces = n / E::V, odd = n % E::V;
  if (pieces <= 4 && odd <= FEWEST) f.template operator()<FEWEST, 1>();
  else if (pieces <= 4) f.template operator()<E::V, 1>();
  else if (pieces <= 16) f.template operator()<16, 1>();
  else if (pieces <= 32) f.template operator()<32, 1>();
  else if (pieces <= 64) f.template operator()<64, 1>();
  else if (pieces <= 128) f.template operator()<64, 2>();
  else if (pieces <= 256) f.template operator()<256, 1>();
  else if (pieces <= 512) f.template operator()<256, 2>();
  else if (pieces <= 1024) f.template operator()<512, 2>();
  else if (pieces <= 1536) f.template operator()<512, 3>();
  else if (pieces <= 2048) f.template operator()<512, 4>();
  else if constexpr (WIDE) {
    if (pieces > 4096) return false;
    f.template operator()<1024, 4>();
  } else return false;
  return true;
}
// the backward pass of bf16 has no registers for eight times as many columns in each of four arrays
template <class E> constexpr bool kWideGrad = E::V == 4;
constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <class E>
struct Forward {
  const NormArgs& a;
  hipStream_t s;
  template <int TPR, int ITEMS>
  void operator()() const {
    constexpr int BLOCK = block_of(TPR);
    constexpr bool FEW = ITEMS * E::V <= 16 && TPR < 1024;
    const dim3 grid((unsigned)blocks_per_worker(a.k, a.rows, BLOCK / TPR, 2048 * (int64_t)kCus / BLOCK), (unsigned)a.k);
    hipLaunchKernelGGL((layer_norm_kernel<E, TPR, ITEMS, BLOCK, FEW>), grid, dim3(BLOCK), 0, s, a);
  }
};
template <class E>
hipError_t fwd_any(const NormArgs& a, hipStream_t s) {
  if (!for_row<E, true>(a.n, Forward<E>{a, s}))
    hipLaunchKernelGGL(layer_norm_long_kernel<E>, dim3((unsigned)blocks_per_worker(a.k, a.rows, 1, 4 * kCus), (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

// blocks of the backward pass: two a compute unit from 256 threads on, so that there are few rows of partial sums (bf16,
// 8192 x 4096: 44 us, with four 56)
int64_t grad_blocks(int tpr) { return (tpr >= 1024 ? 1 : tpr >= 256 ? 2 : 4) * (int64_t)kCus; }

template <class E>
struct Backward {
  const NormArgs& a;
  hipStream_t s;
  template <int TPR, int ITEMS>
  void operator()() const {
    constexpr int BLOCK = block_of(TPR);
    hipLaunchKernelGGL((layer_norm_grad_kernel<E, TPR, ITEMS, BLOCK>), dim3((unsigned)a.strips, (unsigned)a.k), dim3(BLOCK), 0, s, a);
  }
};
struct Strips {
  int k; int64_t rows; int* strips;
  template <int TPR, int ITEMS>
  void operator()() const { *strips = (int)blocks_per_worker(k, rows, block_of(TPR) / TPR, grad_blocks(TPR)); }
};
template <class E>
hipError_t bwd_any(const NormArgs& a, hipStream_t s) {
  if (for_row<E, kWideGrad<E>>(a.n, Backward<E>{a, s})) return hipGetLastError();
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
  int strips = 0;
  const Strips count{k, rows, &strips};
  const bool fits = dtype == DW_BF16 ? for_row<Bf16, kWideGrad<Bf16>>(n, count) : for_row<F32, kWideGrad<F32>>(n, count);
  return fits ? strips : (int)blocks_per_worker(k, rows, 1, 2 * kCus);
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
