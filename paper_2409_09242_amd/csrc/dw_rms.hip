// Root-mean-square norm of the rows of k workers behind the residual's addition and a dropout, its output in 8 bits, and its
// backward pass (gfx950, wave64).
//
//   h = residual + dropout(x),   y = h r gamma,   r = 1 / sqrt(mean(h^2) + eps)            over a row of n
//   with t = h r and a = dy gamma:
//   dres = r (a - t mean(a t)) + dh,   dx = dropout(dres),   dgamma = sum over rows of dy t
//
// TPR threads share a row and keep it in registers as ITEMS pieces of 16 bytes each, so x and the residual are read once; h is
// rounded as it is stored before it is squared, so that the backward pass reads what the norm was taken of.  Sums over a row go
// through the lanes and, above a wave, through LDS, in fp32.
//
// In 8 bits a block of 128 columns lies in 16 (bf16) or 32 (fp32) neighbouring lanes: its largest magnitude is found by lane
// moves and the bytes leave from registers, without a trip of y through memory.  The transposed form needs 128 rows at once and is
// the quantiser's own kernel, which multiplies h by r and gamma as it loads it.
//
// Backward: a group of threads takes every strips-th row of one worker and keeps its column sums in registers; one row of partial
// sums per block goes to scratch, and a second kernel adds those up in their order.
//
// Bound by memory (a copy reaches 4.75 TB/s, two reads a write 5.9; what is still in the chip's cache comes on top): forward 16 x 512 rows
// of 4096, bf16, with a residual 43 us = 6.2 TB/s, its 8-bit form with dropout, 8 x 1024 x 4096, 43 us = 5.4 and 20 for the transposed
// form; backward 3 x 2731 rows of 5003, fp32, with a gradient from further on and a dropout's own output 157 us = 5.2 TB/s, and 5 for the
// columns' sums.  One row 3.7 us.  Registers hold rows of up to 4096 pieces of 16 bytes, in the backward pass of bf16 2048, and fewer elements
// behind them than a piece: bf16 forward to 32775 columns (32768 in 8 bits) and backward to 16391, fp32 both to 16387 (16384).  Of longer
// rows the forward pass reads h, or x, a second time (3.7 to 4.3 TB/s of the formulas' bytes), the backward pass dy and h three times (1.8 to 2.3).
#include "dw_dropout.h"
#include "dw_fp8.h"

namespace dw {

namespace {

inline int64_t blocks_per_worker(int k, int64_t rows, int groups, int64_t target) {
  const int64_t most = ceil_div(rows, groups), share = target > k ? target / k : 1;
  return most < share ? most : share;
}

// one piece of h: x, dropped, the residual added, rounded as it is stored
template <class E>
__device__ __forceinline__ void piece_of_h(const typename E::T* x, const typename E::T* res, const DropKey& key, bool drop, int64_t r,
                                           int64_t groups, int64_t e0, int64_t n, float (&f)[E::V]) {
  load_floats16<E>(x, e0, n, f);
  if (drop) key.piece<E::V>(r, groups, e0, f);
  if (res) {
    float b[E::V];
    load_floats16<E>(res, e0, n, b);
#pragma unroll
    for (int j = 0; j < E::V; ++j) f[j] += b[j];
  }
  if (drop || res) as_stored<E>(f);
}

// the largest magnitude of the lanes that share a block of 128 columns, to all of them
template <class E>
__device__ __forceinline__ uint32_t block_top(const float (&f)[E::V]) {
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < E::V; ++j) top = larger(top, magnitude(f[j]));
  top = largest_of_16(top);
  if constexpr (E::V == 4) top = larger(top, (uint32_t)__shfl_xor((int)top, 16));
  return top;
}

// y of one piece in 8 bits: numbers, and the block's scale by its first lane (and what fills the last word of scales)
template <class E>
__device__ __forceinline__ void put_eight(uint8_t* q, uint8_t* scale, int64_t e0, int64_t n, const float (&y)[E::V]) {
  const int64_t np = DW_FP8_ROW(n), ns = DW_FP8_SCALES(n);
  const Scale s = scale_of(block_top<E>(y));
  if (e0 >= np) return;
  int lo = 0;
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[0] * s.inverse, y[1] * s.inverse, lo, false);
  lo = __builtin_amdgcn_cvt_pk_fp8_f32(y[2] * s.inverse, y[3] * s.inverse, lo, true);
  if constexpr (E::V == 8) {
    int hi = 0;
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[4] * s.inverse, y[5] * s.inverse, hi, false);
    hi = __builtin_amdgcn_cvt_pk_fp8_f32(y[6] * s.inverse, y[7] * s.inverse, hi, true);
    *reinterpret_cast<uint2*>(q + e0) = make_uint2((uint32_t)lo, (uint32_t)hi);
  } else {
    *reinterpret_cast<uint32_t*>(q + e0) = (uint32_t)lo;
  }
  const int64_t b = e0 >> 7;
  if ((e0 & 127) == 0) {
    scale[b] = (uint8_t)s.byte;
    if (b == np / 128 - 1)
      for (int64_t i = b + 1; i < ns; ++i) scale[i] = 127;
  }
}

// A row of n is its whole pieces of 16 bytes, piece i * TPR + t to thread t, and fewer than V elements more, one each to the first
// threads: every access is in bounds and no piece needs a mask of its own.  for_row sees to it that there are as many threads as odd
// elements.
template <class E, int TPR>
struct Split {
  int whole, odd, t, column;                               // whole pieces; elements behind them; this thread, and its element of those
  bool has_odd;
  __device__ __forceinline__ Split(int64_t n, int t_) : whole((int)(n / E::V)), odd((int)(n % E::V)), t(t_), column(whole * E::V + t_), has_odd(t_ < odd) {}
};

// ITEMS pieces of a row and its odd element as they are in memory, so that nothing waits for them before they are used; what a thread
// has not reads as zero.  They stream through once: without displacing what is read again, they are read faster too (16384 x 4096, bf16,
// forward: 85 us and 105, backward, with more blocks, 95 and 108).
template <class E, int TPR, int ITEMS>
struct RowRegs {
  uint32_t piece[ITEMS][4], odd;
  __device__ __forceinline__ void load(const typename E::T* row, const Split<E, TPR>& s) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (i * TPR + s.t < s.whole) {
        load_piece_once<E>(at_piece<E>(row, i * TPR + s.t), piece[i]);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) piece[i][j] = 0u;
      }
    }
    odd = 0u;
    if (s.has_odd) odd = E::bits(row + s.column);
  }
};
template <class E, int TPR, int ITEMS>
__device__ __forceinline__ void store_row(typename E::T* row, const Split<E, TPR>& s, const float (&f)[ITEMS][E::V], float odd) {
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (i * TPR + s.t < s.whole) store_piece<E>(at_piece<E>(row, i * TPR + s.t), f[i]);
  if (s.has_odd) E::put(row + s.column, odd);
}
template <class E>
__device__ __forceinline__ float as_stored_one(float f) {
  return E::V == 8 ? __uint_as_float(pack_bf16(f, 0.f) << 16) : f;
}

// this thread's number, for the row at hand: what follows from it alone would otherwise be worked out once and take registers throughout
// (1024 threads with four pieces, fp32, backward: 66 of them in memory, so 32.  Forward in bf16 with four 27, backward with two 8, the others none)
__device__ __forceinline__ int anew(int t) {
  asm volatile("" : "+v"(t));
  return t;
}

// the elements behind the whole pieces, from the first threads of the group to the one whose next piece they begin, for the block of 128
// that they share with the pieces before them
template <class E, int TPR, int ITEMS>
__device__ __forceinline__ void gather_odd(float (&v)[ITEMS][E::V], float odd, const Split<E, TPR>& s, float* lds) {
  float f[E::V];
  if constexpr (TPR > 64) {
    __syncthreads();                                       // (what an earlier row left there has been read)
    if (s.has_odd) lds[s.t] = odd;
    __syncthreads();
  }
#pragma unroll
  for (int j = 0; j < E::V; ++j) {
    if constexpr (TPR > 64) f[j] = lds[j];
    else f[j] = __shfl(odd, j, TPR);
    f[j] = j < s.odd ? f[j] : 0.f;
  }
#pragma unroll
  for (int i = 0; i < ITEMS; ++i)
    if (i * TPR + s.t == s.whole)
#pragma unroll
      for (int j = 0; j < E::V; ++j) v[i][j] = f[j];
}

// FEW: gamma of the thread's columns stays in registers over its rows.  The next row travels while this one is worked on, except for
// the longest rows, for which 1024 threads have no registers left.
template <class E, int TPR, int ITEMS, int BLOCK, bool FEW>
__global__ __launch_bounds__(BLOCK) void rms_norm_kernel(RmsArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  constexpr bool AHEAD = TPR < 1024 || ITEMS <= 2;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)], odd_lds[8];
  int turn = 0;
  const int w = blockIdx.y, t = GROUPS == 1 ? threadIdx.x : threadIdx.x % TPR, g = GROUPS == 1 ? 0 : threadIdx.x / TPR;
  const int64_t n = a.n, groups = ceil_div(n, 4), np = DW_FP8_ROW(n), ns = DW_FP8_SCALES(n);
  const Split<E, TPR> split(n, t);
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* res = reinterpret_cast<const typename E::T*>(a.res.p) + w * a.res.stride;
  typename E::T* h = reinterpret_cast<typename E::T*>(a.h.p) + w * a.h.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.y.p) + w * a.y.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const bool drop = a.drop.limit < 65536u;
  const DropKey key(a.drop, w);
  const float inv_n = 1.f / (float)n;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  RowRegs<E, TPR, ITEMS> next, next_res;
  auto fetch = [&](int64_t r) {
    next.load(x + r * a.x.ld, split);
    if (a.res.p) next_res.load(res + r * a.res.ld, split);
  };
  int64_t r = (int64_t)blockIdx.x * GROUPS + g;
  if (AHEAD && r < a.rows) fetch(r);
  float ga[ITEMS][V], ga_odd = 1.f;
  auto param = [&](int i) {
#pragma unroll
    for (int j = 0; j < V; ++j) ga[i][j] = 1.f;
    if (gamma && i * TPR + t < split.whole) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 0.f, ga[i]);
  };
  if constexpr (FEW) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) param(i);
  }
  if (gamma && split.has_odd) ga_odd = gamma[split.column];
  for (; r < a.rows; r += step) {
    if constexpr (!AHEAD) fetch(r);
    const int tt = TPR * ITEMS >= 4096 ? anew(t) : t;
    float v[ITEMS][V], odd = E::value(next.odd);
    float sq = 0.f;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      E::unpack(next.piece[i], v[i]);
      if (drop) key.piece<V>(r, groups, (int64_t)(i * TPR + tt) * V, v[i]);
      if (a.res.p) {
        float b[V];
        E::unpack(next_res.piece[i], b);
#pragma unroll
        for (int j = 0; j < V; ++j) v[i][j] += b[j];
      }
      if (drop || a.res.p) as_stored<E>(v[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) sq += v[i][j] * v[i][j];
    }
    if (split.odd) {
      if (drop) odd = key.one(r, groups, split.column, odd);
      if (a.res.p) odd += E::value(next_res.odd);
      odd = as_stored_one<E>(odd);
      sq += odd * odd;                                     // (zero where there is none)
    }
    if (AHEAD && r + step < a.rows) fetch(r + step);
    if (a.h.p) store_row<E, TPR, ITEMS>(h + r * a.h.ld, split, v, odd);
    const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, red, turn) * inv_n + a.eps);
    if (t == 0 && a.rstd) a.rstd[w * a.rows + r] = rstd;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if constexpr (!FEW) param(i);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = v[i][j] * rstd * ga[i][j];
    }
    odd = odd * rstd * ga_odd;
    if (a.y.p) store_row<E, TPR, ITEMS>(y + r * a.y.ld, split, v, odd);
    if (a.q) {
      if (split.odd) gather_odd<E, TPR, ITEMS>(v, odd, split, odd_lds);
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        put_eight<E>(a.q + (w * a.rows + r) * np, a.scale + (w * a.rows + r) * ns, (int64_t)(i * TPR + t) * V, n, v[i]);
    }
  }
}

// rows too long for registers: a block goes over the row twice, the second time over h where that was stored (each thread what it
// wrote itself: h may be the residual or x)
template <class E>
__global__ __launch_bounds__(1024) void rms_norm_long_kernel(RmsArgs a) {
  constexpr int V = E::V, TPR = 1024;
  __shared__ float red[2 * TPR / 64];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x;
  const int64_t n = a.n, groups = ceil_div(n, 4), np = DW_FP8_ROW(n), ns = DW_FP8_SCALES(n);
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  const typename E::T* res = reinterpret_cast<const typename E::T*>(a.res.p) + w * a.res.stride;
  typename E::T* h = reinterpret_cast<typename E::T*>(a.h.p) + w * a.h.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.y.p) + w * a.y.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const bool drop = a.drop.limit < 65536u;
  const DropKey key(a.drop, w);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    float v[V], sq = 0.f;
    auto fresh = [&](int64_t e0) { piece_of_h<E>(x + r * a.x.ld, a.res.p ? res + r * a.res.ld : nullptr, key, drop, r, groups, e0, n, v); };
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      fresh(e0);
#pragma unroll
      for (int j = 0; j < V; ++j) sq += v[j] * v[j];
      if (a.h.p) store16<E>(h + r * a.h.ld, e0, n, v);
    }
    const float rstd = 1.f / sqrtf(row_sum<TPR>(sq, red, turn) * (1.f / (float)n) + a.eps);
    if (t == 0 && a.rstd) a.rstd[w * a.rows + r] = rstd;
    // (whole blocks of 128: the lanes that share one stay together, and a row in 8 bits is written to its end)
    for (int64_t e0 = (int64_t)t * V; e0 < np; e0 += TPR * V) {
      if (a.h.p) load_floats16<E>(h + r * a.h.ld, e0, n, v);
      else fresh(e0);
      float ga[V];
#pragma unroll
      for (int j = 0; j < V; ++j) ga[j] = 1.f;
      if (gamma) load_floats<V>(gamma, e0, n, 0.f, ga);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = v[j] * rstd * ga[j];
      if (a.y.p) store16<E>(y + r * a.y.ld, e0, n, v);
      if (a.q) put_eight<E>(a.q + (w * a.rows + r) * np, a.scale + (w * a.rows + r) * ns, e0, n, v);
    }
  }
}

// Registers hold the rows and the column sums of a thread's pieces, gamma, and the next rows on their way; 1024 threads have half as many
// each, so there, with more than eight columns a thread, gamma comes from the caches and the next rows are not fetched ahead.
template <class E, int TPR, int ITEMS, int BLOCK>
__global__ __launch_bounds__(BLOCK) void rms_norm_grad_kernel(RmsGradArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR, COLS = TPR * ITEMS * V;
  constexpr bool AHEAD = TPR < 1024 || ITEMS * V <= 8;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  __shared__ float cols[GROUPS > 1 ? GROUPS * (COLS + V) : 1];
  int turn = 0;
  const int w = blockIdx.y, t = GROUPS == 1 ? threadIdx.x : threadIdx.x % TPR, g = GROUPS == 1 ? 0 : threadIdx.x / TPR;
  const int64_t n = a.n, groups = ceil_div(n, 4);
  const Split<E, TPR> split(n, t);
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  const typename E::T* h = reinterpret_cast<const typename E::T*>(a.h.p) + w * a.h.stride;
  const typename E::T* dh = reinterpret_cast<const typename E::T*>(a.dh.p) + w * a.dh.stride;
  typename E::T* dres = reinterpret_cast<typename E::T*>(a.dres.p) + w * a.dres.stride;
  typename E::T* dx = reinterpret_cast<typename E::T*>(a.dx.p) + w * a.dx.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const DropKey key(a.drop, w);
  const bool wanted = a.dres.p || a.dx.p;
  const float inv_n = 1.f / (float)n;
  const int64_t step = (int64_t)gridDim.x * GROUPS;
  RowRegs<E, TPR, ITEMS> next_dy, next_h, next_dh;
  float next_rstd = 0.f;
  auto fetch = [&](int64_t r) {
    next_dy.load(dy + r * a.dy.ld, split);
    next_h.load(h + r * a.h.ld, split);
    if (AHEAD && a.dh.p && wanted) next_dh.load(dh + r * a.dh.ld, split);
    next_rstd = a.rstd[w * a.rows + r];
  };
  int64_t r = (int64_t)blockIdx.x * GROUPS + g;
  if (AHEAD && r < a.rows) fetch(r);
  float dg[ITEMS][V], ga[ITEMS][V], dg_odd = 0.f, ga_odd = 1.f;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
#pragma unroll
    for (int j = 0; j < V; ++j) { dg[i][j] = 0.f; ga[i][j] = 1.f; }
    if (AHEAD && gamma && i * TPR + t < split.whole) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 0.f, ga[i]);
  }
  if (gamma && split.has_odd) ga_odd = gamma[split.column];
  for (; r < a.rows; r += step) {
    if constexpr (!AHEAD) fetch(r);
    const int tt = TPR * ITEMS >= 4096 ? anew(t) : t;
    const float rstd = next_rstd;
    float v[ITEMS][V], u[ITEMS][V], sum = 0.f;             // a, and t
    uint32_t more[ITEMS][4], more_odd = 0u;                // dh as it is in memory
    float v_odd = E::value(next_dy.odd), u_odd = E::value(next_h.odd) * rstd;
    if (AHEAD && a.dh.p) more_odd = next_dh.odd;
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      E::unpack(next_dy.piece[i], v[i]);
      E::unpack(next_h.piece[i], u[i]);
      if constexpr (AHEAD)
#pragma unroll
        for (int j = 0; j < 4; ++j) more[i][j] = a.dh.p ? next_dh.piece[i][j] : 0u;
      if (!AHEAD && gamma && i * TPR + t < split.whole) load_floats<V>(gamma, (int64_t)(i * TPR + t) * V, n, 0.f, ga[i]);
#pragma unroll
      for (int j = 0; j < V; ++j) {
        u[i][j] *= rstd;
        dg[i][j] += v[i][j] * u[i][j];
        v[i][j] *= ga[i][j];
        sum += v[i][j] * u[i][j];
      }
    }
    dg_odd += v_odd * u_odd;                               // (zeros where there is none)
    v_odd *= ga_odd;
    sum += v_odd * u_odd;
    if (AHEAD && r + step < a.rows) fetch(r + step);
    if (!wanted) continue;
    const float c = row_sum<TPR>(sum, red, turn) * inv_n;
    if (!AHEAD && a.dh.p) { next_dh.load(dh + r * a.dh.ld, split); more_odd = next_dh.odd; }
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      float b[V];
      if constexpr (!AHEAD)
#pragma unroll
        for (int j = 0; j < 4; ++j) more[i][j] = a.dh.p ? next_dh.piece[i][j] : 0u;
      E::unpack(more[i], b);
#pragma unroll
      for (int j = 0; j < V; ++j) v[i][j] = rstd * (v[i][j] - u[i][j] * c) + b[j];
    }
    v_odd = rstd * (v_odd - u_odd * c) + E::value(more_odd);
    if (a.dres.p) store_row<E, TPR, ITEMS>(dres + r * a.dres.ld, split, v, v_odd);
    if (a.dx.p) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) key.piece<V>(r, groups, (int64_t)(i * TPR + tt) * V, v[i]);
      if (split.odd) v_odd = key.one(r, groups, split.column, v_odd);
      store_row<E, TPR, ITEMS>(dx + r * a.dx.ld, split, v, v_odd);
    }
  }
  if (!a.part) return;
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * n;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
      if (i * TPR + t < split.whole) {
#pragma unroll
        for (int q = 0; q < V / 4; ++q) {
          const float f[4] = {dg[i][4 * q], dg[i][4 * q + 1], dg[i][4 * q + 2], dg[i][4 * q + 3]};
          store_piece<F32>(out + (int64_t)(i * TPR + t) * V + 4 * q, f);
        }
      }
    if (split.has_odd) out[split.column] = dg_odd;
  } else {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i)
#pragma unroll
      for (int j = 0; j < V; ++j) cols[g * (COLS + V) + (i * TPR + t) * V + j] = dg[i][j];
    __syncthreads();                                       // (the odd elements' places may be those of a piece that is not there)
    if (split.has_odd) cols[g * (COLS + V) + split.column] = dg_odd;
    __syncthreads();
    for (int e = threadIdx.x; e < n; e += BLOCK) {
      float s = cols[e];
#pragma unroll
      for (int q = 1; q < GROUPS; ++q) s += cols[q * (COLS + V) + e];
      out[e] = s;
    }
  }
}

// column sums for rows too long for registers: a thread owns V columns, a block every strips-th row.  It runs first: the row
// kernel may write over dy
template <class E>
__global__ __launch_bounds__(256) void rms_norm_cols_kernel(RmsGradArgs a) {
  constexpr int V = E::V;
  const int w = blockIdx.z;
  const int64_t n = a.n, e0 = ((int64_t)blockIdx.y * 256 + threadIdx.x) * V;
  if (e0 >= n) return;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  const typename E::T* h = reinterpret_cast<const typename E::T*>(a.h.p) + w * a.h.stride;
  float dg[V], u[V], v[V];
#pragma unroll
  for (int j = 0; j < V; ++j) dg[j] = 0.f;
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float rstd = a.rstd[w * a.rows + r];
    load_floats16<E>(dy + r * a.dy.ld, e0, n, v);
    load_floats16<E>(h + r * a.h.ld, e0, n, u);
#pragma unroll
    for (int j = 0; j < V; ++j) dg[j] += v[j] * (u[j] * rstd);
  }
  float* out = a.part + ((int64_t)w * gridDim.x + blockIdx.x) * n;
#pragma unroll
  for (int j = 0; j < V; ++j)
    if (e0 + j < n) out[e0 + j] = dg[j];
}

template <class E>
__global__ __launch_bounds__(1024) void rms_norm_grad_long_kernel(RmsGradArgs a) {
  constexpr int V = E::V, TPR = 1024;
  __shared__ float red[2 * TPR / 64];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x;
  const int64_t n = a.n, groups = ceil_div(n, 4);
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  const typename E::T* h = reinterpret_cast<const typename E::T*>(a.h.p) + w * a.h.stride;
  const typename E::T* dh = reinterpret_cast<const typename E::T*>(a.dh.p) + w * a.dh.stride;
  typename E::T* dres = reinterpret_cast<typename E::T*>(a.dres.p) + w * a.dres.stride;
  typename E::T* dx = reinterpret_cast<typename E::T*>(a.dx.p) + w * a.dx.stride;
  const float* gamma = a.gamma ? a.gamma + w * a.param_stride : nullptr;
  const DropKey key(a.drop, w);
  for (int64_t r = blockIdx.x; r < a.rows; r += gridDim.x) {
    const float rstd = a.rstd[w * a.rows + r];
    float v[V], u[V], ga[V], sum = 0.f;
    auto read = [&](int64_t e0) {
      load_floats16<E>(dy + r * a.dy.ld, e0, n, v);
      load_floats16<E>(h + r * a.h.ld, e0, n, u);
#pragma unroll
      for (int j = 0; j < V; ++j) ga[j] = 1.f;
      if (gamma) load_floats<V>(gamma, e0, n, 0.f, ga);
#pragma unroll
      for (int j = 0; j < V; ++j) { u[j] *= rstd; v[j] *= ga[j]; }
    };
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      read(e0);
#pragma unroll
      for (int j = 0; j < V; ++j) sum += v[j] * u[j];
    }
    const float c = row_sum<TPR>(sum, red, turn) * (1.f / (float)n);
    for (int64_t e0 = (int64_t)t * V; e0 < n; e0 += TPR * V) {
      read(e0);
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = rstd * (v[j] - u[j] * c);
      if (a.dh.p) {
        load_floats16<E>(dh + r * a.dh.ld, e0, n, u);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] += u[j];
      }
      if (a.dres.p) store16<E>(dres + r * a.dres.ld, e0, n, v);
      if (a.dx.p) {
        key.piece<V>(r, groups, e0, v);
        store16<E>(dx + r * a.dx.ld, e0, n, v);
      }
    }
  }
}

// dgamma from the blocks' partial sums: 64 columns a block, its 16 waves take every 16th strip each, eight at a time (they are few
// columns, so that the trips to memory are what it takes)
__global__ __launch_bounds__(1024) void rms_norm_strips_kernel(RmsGradArgs a) {
  __shared__ float lds[16][64];
  const int w = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = a.n, e = (int64_t)blockIdx.x * 64 + lane;
  float s = 0.f;
  if (e < n) {
    const float* part = a.part + (int64_t)w * a.strips * n + e;
    for (int p = wave; p < a.strips; p += 128) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = p + 16 * j < a.strips ? part[(p + 16 * j) * n] : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) s += f[j];
    }
  }
  lds[wave][lane] = s;
  __syncthreads();
  if (wave == 0 && e < n) {
#pragma unroll
    for (int q = 1; q < 16; ++q) s += lds[q][lane];
    a.dgamma[w * a.grad_stride + e] = s;
  }
}

// f.template operator()<TPR, ITEMS>() for rows of so many pieces and odd elements; false: too long.  Above 1536 pieces 1024 threads take two each: with
// four of 512 threads the backward pass has no registers for a second block on the unit (4096 x 16384, bf16: 158 us and 114; fp32 with
// four of 1024: 287 and 214).  The lanes that share a block of 128 columns are
// in one group from 128 / V threads on, which is the fewest with an output in 8 bits (EIGHT)
template <class E, bool EIGHT, bool WIDE, class F>
bool for_row(int64_t n, F f) {
  const int64_t pieces = EIGHT ? DW_FP8_ROW(n) / E::V : n / E::V;
  if (!EIGHT && pieces <= 4 && n % E::V <= 4) f.template operator()<4, 1>();
  else if ((!EIGHT || E::V == 8) && pieces <= 16) f.template operator()<16, 1>();
  else if (pieces <= 32) f.template operator()<32, 1>();
  else if (pieces <= 64) f.template operator()<64, 1>();
  else if (pieces <= 128) f.template operator()<64, 2>();
  else if (pieces <= 256) f.template operator()<256, 1>();
  else if (pieces <= 512) f.template operator()<256, 2>();
  else if (pieces <= 1024) f.template operator()<512, 2>();
  else if (pieces <= 1536) f.template operator()<512, 3>();
  else if (pieces <= 2048) f.template operator()<1024, 2>();
  else if constexpr (WIDE) {
    if (pieces > 4096) return false;
    f.template operator()<1024, 4>();
  } else return false;
  return true;
}
constexpr int block_of(int tpr) { return tpr < 256 ? 256 : tpr; }

template <class E>
struct Forward {
  const RmsArgs& a;
  hipStream_t s;
  template <int TPR, int ITEMS>
  void operator()() const {
    constexpr int BLOCK = block_of(TPR);
    constexpr bool FEW = ITEMS * E::V <= 16 && TPR < 1024;
    // threads of a unit: as many as it holds, but in fp32, in blocks of 256, only as many as its registers have room for at once
    // (65536 x 1024, fp32, with a residual 199 us, with 2048 212; without 89 and 104; in 8 bits 166 and 185; bf16 within 3 us of each other)
    constexpr int THREADS = E::V == 4 && BLOCK == 256 ? 1024 : 2048;
    const dim3 grid((unsigned)blocks_per_worker(a.k, a.rows, BLOCK / TPR, THREADS * (int64_t)kCus / BLOCK), (unsigned)a.k);
    hipLaunchKernelGGL((rms_norm_kernel<E, TPR, ITEMS, BLOCK, FEW>), grid, dim3(BLOCK), 0, s, a);
  }
};
template <class E>
hipError_t forward(const RmsArgs& a, hipStream_t s) {
  const Forward<E> f{a, s};
  const bool fits = a.q ? for_row<E, true, true>(a.n, f) : for_row<E, false, true>(a.n, f);
  if (!fits)
    hipLaunchKernelGGL(rms_norm_long_kernel<E>, dim3((unsigned)blocks_per_worker(a.k, a.rows, 1, 4 * kCus), (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

template <class E> constexpr bool kWideGrad = E::V == 4;
// Blocks of the backward pass: a unit reads best with 8 KB or more of rows from each tensor at work, not many more, and fewer leave fewer rows of
// partial sums (us with 1, 2, 3 and 4 a unit: bf16, 65536 x 1024, 8 KB a block 88, 88, 93, 98; 1024 x 4096, 8 KB 14, 17, 19, 22;
// 13413 x 5003, 10 KB 128, 132, 134, 139; 32768 x 2048, 4 KB 126, 89, 92, 93; fp32, 129055 x 520, 2 KB 421, 248, 218, 227)
template <class E>
int64_t grad_blocks(int groups, int64_t n) {
  const int64_t bytes = groups * n * (int64_t)sizeof(typename E::T);
  return (bytes >= 8192 ? 1 : bytes >= 3000 ? 2 : 3) * (int64_t)kCus;
}

template <class E>
struct Backward {
  const RmsGradArgs& a;
  hipStream_t s;
  template <int TPR, int ITEMS>
  void operator()() const {
    constexpr int BLOCK = block_of(TPR);
    hipLaunchKernelGGL((rms_norm_grad_kernel<E, TPR, ITEMS, BLOCK>), dim3((unsigned)a.strips, (unsigned)a.k), dim3(BLOCK), 0, s, a);
  }
};
template <class E>
struct Strips {
  int k; int64_t rows, n; int* strips;
  template <int TPR, int ITEMS>
  void operator()() const { *strips = (int)blocks_per_worker(k, rows, block_of(TPR) / TPR, grad_blocks<E>(block_of(TPR) / TPR, n)); }
};
template <class E>
hipError_t backward(const RmsGradArgs& a, hipStream_t s) {
  if (for_row<E, false, kWideGrad<E>>(a.n, Backward<E>{a, s})) return hipGetLastError();
  if (a.part) {
    hipLaunchKernelGGL(rms_norm_cols_kernel<E>, dim3((unsigned)a.strips, (unsigned)ceil_div(a.n, 256 * E::V), (unsigned)a.k), dim3(256), 0, s, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || (!a.dres.p && !a.dx.p)) return e;
  }
  hipLaunchKernelGGL(rms_norm_grad_long_kernel<E>, dim3((unsigned)blocks_per_worker(a.k, a.rows, 1, 4 * kCus), (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rms_norm(const RmsArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? forward<Bf16>(a, s) : forward<F32>(a, s);
}

int rms_norm_grad_strips(int k, int64_t rows, int64_t n, int dtype) {
  int strips = 0;
  const bool fits = dtype == DW_BF16 ? for_row<Bf16, false, kWideGrad<Bf16>>(n, Strips<Bf16>{k, rows, n, &strips})
                                     : for_row<F32, false, kWideGrad<F32>>(n, Strips<F32>{k, rows, n, &strips});
  return fits ? strips : (int)blocks_per_worker(k, rows, 1, 2 * kCus);
}

hipError_t launch_rms_norm_grad(const RmsGradArgs& a, int dtype, hipStream_t s) {
  if (a.rows > 0) {
    const hipError_t e = dtype == DW_BF16 ? backward<Bf16>(a, s) : backward<F32>(a, s);
    if (e != hipSuccess) return e;
  }
  if (!a.dgamma) return hipSuccess;                        // (no rows: no strips, and the sums are zero)
  hipLaunchKernelGGL(rms_norm_strips_kernel, dim3((unsigned)ceil_div(a.n, 64), (unsigned)a.k), dim3(1024), 0, s, a);
  return hipGetLastError();
}

}  // namespace dw
