// Clipped policy loss with a KL term over the logits of chosen tokens, and its gradient (gfx950, wave64).
//
// For a row z of logits with target y:   lp = z_y - log sum_j exp(z_j),   q = exp(lp - old),
//   l  = -min(q A, clip(q, 1 - lo, 1 + hi) A) + beta (exp(ref - lp) - (ref - lp) - 1),     loss = sum over rows of w l
//   l' = (0 where the clipped term is the smaller, else -q A) + beta (1 - exp(ref - lp)),
//   dz_j = w l' ([j = y] - softmax(z)_j)
//
// TPR threads share a row, how many follows from the vocabulary alone.  One pass finds the maximum and the sum of exponentials
// together: a thread keeps both for the pieces (16 bytes) it has seen, the sum relative to its maximum, and the threads'
// are joined at the end.  For the gradient the pieces stay in registers as they came, so logits are read once; past 16 pieces
// of each of 1024 threads the rest of the row is read again, from the caches.  Log probabilities alone (no gradient) need no
// registers for the row, and are the same bits: the same pieces in the same order.  Bound by memory; with the whole row in the
// registers of one compute unit a block's loads and stores take turns, so rows are shared among as few threads as hold them.
// 8 x 1024 rows of 131072, bf16, with the gradient: 809 us = 5.3 TB/s; 4 x 100 rows of 5003, fp32: 6.8 us and 2.1 for the sums.
//
// Sums over a row are in fp32: a thread's pieces one after another (at most 16 up to 65536 logits in fp32 and 131072 in bf16,
// beyond that one for every 4096 or 8192 of the vocabulary), then a tree; the rows' losses go to scratch and a second kernel adds a
// worker's up in 64 bits in a fixed order.
#include "dw_ops.h"

namespace dw {

namespace {

__device__ __forceinline__ float exp_fast(float x) { return __builtin_amdgcn_exp2f(x * 1.44269504088896341f); }

template <int TPR>
__device__ __forceinline__ float row_max(float x, float* lds, int& turn) {
#pragma unroll
  for (int off = 1; off < (TPR < 64 ? TPR : 64); off <<= 1) x = fmaxf(x, __shfl_xor(x, off));
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = lds + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = at[0];
#pragma unroll
    for (int w = 1; w < W; ++w) x = fmaxf(x, at[w]);
  }
  return x;
}

// A piece is unpacked where it is worked on, once what came before it is done (`x`, `y`: what that left): all pieces' unpacked
// values at once, or kept for the second pass, would take twice the registers of the packed ones in bf16.
__device__ __forceinline__ void in_turn(uint32_t (&piece)[4], float& x, float& y) {
  asm volatile("" : "+v"(piece[0]), "+v"(piece[1]), "+v"(piece[2]), "+v"(piece[3]), "+v"(x), "+v"(y));
}

// a maximum to subtract: of -inf alone nothing, so that the sum stays zero (while a NaN, which no maximum takes, shows in it)
__device__ __forceinline__ float base_of(float m) { return m == -__builtin_huge_valf() ? 0.f : m; }

// the largest of what a thread has seen and the sum of exponentials relative to it
struct Running {
  float m = -__builtin_huge_valf(), s = 0.f;
  template <int V>
  __device__ __forceinline__ void add(const float (&f)[V]) {
    float top = f[0];
#pragma unroll
    for (int j = 1; j < V; ++j) top = fmaxf(top, f[j]);
    top = fmaxf(top, m);
    const float base = base_of(top);
    float e[V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = exp_fast(f[j] - base);
#pragma unroll
    for (int h = V / 2; h > 0; h /= 2)
#pragma unroll
      for (int j = 0; j < h; ++j) e[j] += e[j + h];
    s = __builtin_fmaf(s, exp_fast(m - base), e[0]);         // (nothing new: times 1 plus 0)
    m = top;
  }
};

template <class E, int TPR, int ITEMS, int BLOCK, bool LONG, bool GRAD>
__global__ __launch_bounds__(BLOCK, (GRAD && ITEMS >= 16 ? 4 : 1)) void policy_rows_kernel(PolicyArgs a) {      // (waves a SIMD)
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  int turn = 0;
  // (one group a block: everything about the row is uniform)
  const int w = blockIdx.y, t = GROUPS == 1 ? threadIdx.x : threadIdx.x % TPR, g = GROUPS == 1 ? 0 : threadIdx.x / TPR;
  const float ninf = -__builtin_huge_valf();
  // piece i of a thread is piece i * TPR + t of the row's whole ones; what is left of the row (fewer than V elements) goes
  // to the first threads, one each.  A thread without one holds -inf in its place, which changes neither maximum nor sum
  const int whole = (int)(a.vocab / V);
  const int tail = whole * V + t;
  const bool has_tail = tail < (int)a.vocab;
  for (int64_t r = (int64_t)blockIdx.x * GROUPS + g; r < a.rows; r += (int64_t)gridDim.x * GROUPS) {
    const int64_t at = w * a.rows + r;
    const typename E::T* z = reinterpret_cast<const typename E::T*>(a.logits.p) + w * a.logits.stride + r * a.logits.ld;
    typename E::T* out = GRAD ? reinterpret_cast<typename E::T*>(a.grad.p) + w * a.grad.stride + r * a.grad.ld : nullptr;
    const int y = a.target[at];
    const float weight = a.weight ? a.weight[at] : a.mean_weight;
    float loss = 0.f, logp = 0.f, slope = 0.f, scale = 0.f, top = 0.f, zy = 0.f, zt = ninf;
    uint32_t raw[ITEMS][4];
    if (y >= 0 && y < (int)a.vocab && weight != 0.f) {      // the same for all threads of the row
      zy = E::one(z + y);
      if (has_tail) zt = E::one(z + tail);
      Running run;
      auto take = [&](int i, int q) {                       // piece q into place i
        if (q < whole) {
          load_piece<E>(at_piece<E>(z, q), raw[i]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i][j] = E::kMinusInf;
        }
      };
      auto add = [&](const uint32_t (&piece)[4]) {
        float f[V];
        E::unpack(piece, f);
        run.add(f);
      };
      // the gradient's pieces, or (none is wanted) all of them, ITEMS at a time
      int q0 = t;
      do {
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) take(i, q0 + i * TPR);
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          in_turn(raw[i], run.m, run.s);
          add(raw[i]);
        }
        q0 += ITEMS * TPR;
      } while (!GRAD && q0 - t < whole);
      if constexpr (GRAD && LONG) {
        for (int q = q0; q < whole; q += TPR) {
          uint32_t more[4];
          load_piece<E>(at_piece<E>(z, q), more);
          add(more);
        }
      }
      const float one_more[1] = {zt};
      run.add(one_more);
      top = base_of(row_max<TPR>(run.m, red, turn));
      const float sum = row_sum<TPR>(run.s * exp_fast(run.m - top), red, turn);
      if (sum == 0.f) {                                     // nothing can be chosen: no loss and no gradient
        logp = ninf;
      } else {
        logp = (zy - top) - logf(sum);
        if (a.old_logp) {
          const float q = expf(logp - a.old_logp[at]), adv = a.advantage[at];
          const float freely = adv == 0.f ? 0.f : q * adv, held = fminf(fmaxf(q, a.q_min), a.q_max) * adv;
          const bool clipped = held < freely;
          loss = clipped ? -held : -freely;
          slope = clipped ? 0.f : -freely;
          if (a.kl_coef != 0.f) {
            const float gap = a.ref_logp[at] - logp, em1 = expm1f(gap);
            loss += a.kl_coef * (em1 - gap);
            slope -= a.kl_coef * em1;
          }
          loss *= weight;
          slope *= weight;
          scale = -slope / sum;
        }
      }
    }
    if (t == 0) {
      if (a.logp) a.logp[at] = logp;
      if (a.part) a.part[at] = loss;
    }
    if constexpr (GRAD) {
      if (scale != 0.f) {                                   // (NaN too)
        auto put = [&](const uint32_t (&piece)[4], int q) {
          float f[V];
          E::unpack(piece, f);
#pragma unroll
          for (int j = 0; j < V; ++j) f[j] = scale * exp_fast(f[j] - top);
          store_piece_once<E>(at_piece<E>(out, q), f);
        };
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          in_turn(raw[i], scale, top);
          if (i * TPR + t < whole) put(raw[i], i * TPR + t);
        }
        if constexpr (LONG) {
          for (int q = ITEMS * TPR + t; q < whole; q += TPR) {
            uint32_t more[4];
            load_piece<E>(at_piece<E>(z, q), more);
            put(more, q);
          }
        }
        if (has_tail) E::put(out + tail, scale * exp_fast(zt - top));
        // the target's element once more, by the thread that has just written it
        if (t == (y < whole * V ? y / V % TPR : y - whole * V)) E::put(out + y, slope + scale * exp_fast(zy - top));
      } else {
        float f[V];
#pragma unroll
        for (int j = 0; j < V; ++j) f[j] = 0.f;
        for (int q = t; q < whole; q += TPR) store_piece_once<E>(at_piece<E>(out, q), f);
        if (has_tail) E::put(out + tail, 0.f);
      }
    }
  }
}

__global__ __launch_bounds__(1024) void policy_sum_kernel(const float* part, float* loss, int64_t rows) {
  __shared__ double waves[16];
  const float* p = part + (int64_t)blockIdx.x * rows;
  double s = 0.0;
#pragma unroll 4
  for (int64_t r = threadIdx.x; r < rows; r += 1024) s += (double)p[r];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  s = threadIdx.x < 16 ? waves[threadIdx.x] : 0.0;
#pragma unroll
  for (int off = 1; off < 16; off <<= 1) s += __shfl_xor(s, off);
  if (threadIdx.x == 0) loss[blockIdx.x] = (float)s;
}

// ITEMS: pieces of a thread that the gradient keeps; log probabilities alone take up to eight at a time
template <class E, int TPR, int ITEMS, bool LONG>
hipError_t rows_of(const PolicyArgs& a, hipStream_t s) {
  constexpr int BLOCK = TPR < 256 ? 256 : TPR;
  int64_t blocks = ceil_div(a.rows, BLOCK / TPR);
  if (blocks > 65536) blocks = 65536;
  const dim3 grid((unsigned)blocks, (unsigned)a.k);
  if (a.grad.p) hipLaunchKernelGGL((policy_rows_kernel<E, TPR, ITEMS, BLOCK, LONG, true>), grid, dim3(BLOCK), 0, s, a);
  else hipLaunchKernelGGL((policy_rows_kernel<E, TPR, (ITEMS < 8 ? ITEMS : 8), BLOCK, false, false>), grid, dim3(BLOCK), 0, s, a);
  return hipGetLastError();
}

template <class E>
hipError_t rows_any(const PolicyArgs& a, hipStream_t s) {
  const int64_t pieces = a.vocab / E::V;
  if (pieces <= 64) return rows_of<E, 64, 1, false>(a, s);
  if (pieces <= 256) return rows_of<E, 64, 4, false>(a, s);
  if (pieces <= 1024) return rows_of<E, 256, 4, false>(a, s);
  if (pieces <= 2048) return rows_of<E, 256, 8, false>(a, s);
  if (pieces <= 4096) return rows_of<E, 512, 8, false>(a, s);
  if (pieces <= 8192) return rows_of<E, 512, 16, false>(a, s);
  if (pieces <= 16384) return rows_of<E, 1024, 16, false>(a, s);
  return rows_of<E, 1024, 16, true>(a, s);
}

}  // namespace

hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t s) {
  if (a.rows > 0) {
    const hipError_t e = dtype == DW_BF16 ? rows_any<Bf16>(a, s) : rows_any<F32>(a, s);
    if (e != hipSuccess || !a.loss) return e;
  }
  if (!a.loss) return hipSuccess;
  hipLaunchKernelGGL(policy_sum_kernel, dim3((unsigned)a.k), dim3(1024), 0, s, a.part, a.loss, a.rows);
  return hipGetLastError();
}

}  // namespace dw
