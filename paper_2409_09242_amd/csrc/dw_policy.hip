// Clipped policy loss with a KL term over the logits of chosen tokens, and its gradient (gfx950, wave64).
//
// For a row z of logits with target y:   lp = z_y - log sum_j exp(z_j),   q = exp(lp - old),
//   l  = -min(q A, clip(q, 1 - lo, 1 + hi) A) + beta (exp(ref - lp) - (ref - lp) - 1),     loss = sum over rows of w l
//   l' = (0 where the clipped term is the smaller, else -q A) + beta (1 - exp(ref - lp)),
//   dz_j = w l' ([j = y] - softmax(z)_j)
//
// TPR threads share a row and keep its logits in registers as they came (16-byte pieces, ITEMS a thread), so they are read
// once: the maximum, the sum of exponentials and the gradient all come from there.  Vocabularies beyond 16 pieces of each
// of 1024 threads read the rest of the row again, from the caches.  Sums over a row are in fp32 (at most 128 terms of a thread,
// then a tree); the rows' losses go to scratch and a second kernel adds a worker's up in 64 bits in a fixed order.
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

// the packed logits are what stays in registers from one pass over them to the next, not their unpacked values
template <int ITEMS>
__device__ __forceinline__ void unpack_anew(uint32_t (&raw)[ITEMS][4]) {
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) asm volatile("" : "+v"(raw[i][0]), "+v"(raw[i][1]), "+v"(raw[i][2]), "+v"(raw[i][3]));
}
// a thread with 16 pieces has registers for them and for a few values more: its pieces are worked on one at a time
template <int ITEMS>
__device__ __forceinline__ void keep_order() {
  if constexpr (ITEMS >= 16) __builtin_amdgcn_sched_barrier(0);
}

template <class E, int TPR, int ITEMS, int BLOCK, bool LONG, bool GRAD>
__global__ __launch_bounds__(BLOCK) void policy_rows_kernel(PolicyArgs a) {
  constexpr int V = E::V, GROUPS = BLOCK / TPR;
  __shared__ float red[2 * (TPR > 64 ? TPR / 64 : 1)];
  int turn = 0;
  const int w = blockIdx.y, t = threadIdx.x % TPR, g = threadIdx.x / TPR;
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
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        if (i * TPR + t < whole) {
          load_piece<E>(z + (int64_t)(i * TPR + t) * V, raw[i]);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j) raw[i][j] = E::kMinusInf;
        }
      }
      float m = zt;
      auto highest = [&](const uint32_t (&piece)[4]) {
        float f[V];
        E::unpack(piece, f);
#pragma unroll
        for (int j = 0; j < V; ++j) m = fmaxf(m, f[j]);
      };
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) { highest(raw[i]); keep_order<ITEMS>(); }
      if constexpr (LONG) {
        for (int q = ITEMS * TPR + t; q < whole; q += TPR) {
          uint32_t more[4];
          load_piece<E>(z + (int64_t)q * V, more);
          highest(more);
        }
      }
      m = row_max<TPR>(m, red, turn);
      unpack_anew(raw);
      top = m == ninf ? 0.f : m;                            // a row of -inf: the sum stays zero, while a NaN shows in it
      float sum = exp_fast(zt - top);
      auto add = [&](const uint32_t (&piece)[4]) {
        float f[V];
        E::unpack(piece, f);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += exp_fast(f[j] - top);
      };
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) { add(raw[i]); keep_order<ITEMS>(); }
      if constexpr (LONG) {
        for (int q = ITEMS * TPR + t; q < whole; q += TPR) {
          uint32_t more[4];
          load_piece<E>(z + (int64_t)q * V, more);
          add(more);
        }
      }
      sum = row_sum<TPR>(sum, red, turn);
      if constexpr (GRAD) unpack_anew(raw);
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
          store_piece_once<E>(out + (int64_t)q * V, f);
        };
#pragma unroll
        for (int i = 0; i < ITEMS; ++i) {
          if (i * TPR + t < whole) put(raw[i], i * TPR + t);
          keep_order<ITEMS>();
        }
        if constexpr (LONG) {
          for (int q = ITEMS * TPR + t; q < whole; q += TPR) {
            uint32_t more[4];
            load_piece<E>(z + (int64_t)q * V, more);
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
        for (int q = t; q < whole; q += TPR) store_piece_once<E>(out + (int64_t)q * V, f);
        if (has_tail) E::put(out + tail, 0.f);
      }
    }
  }
}

__global__ __launch_bounds__(256) void policy_sum_kernel(const float* part, float* loss, int64_t rows) {
  __shared__ double waves[4];
  const float* p = part + (int64_t)blockIdx.x * rows;
  double s = 0.0;
  for (int64_t r = threadIdx.x; r < rows; r += 256) s += (double)p[r];
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) waves[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) loss[blockIdx.x] = (float)((waves[0] + waves[1]) + (waves[2] + waves[3]));
}

template <class E, int TPR, int ITEMS, int BLOCK, bool LONG>
hipError_t rows_of(const PolicyArgs& a, hipStream_t s) {
  int64_t blocks = ceil_div(a.rows, BLOCK / TPR);
  if (blocks > 65536) blocks = 65536;
  const dim3 grid((unsigned)blocks, (unsigned)a.k);
  if (a.grad.p) hipLaunchKernelGGL((policy_rows_kernel<E, TPR, ITEMS, BLOCK, LONG, true>), grid, dim3(BLOCK), 0, s, a);
  else hipLaunchKernelGGL((policy_rows_kernel<E, TPR, ITEMS, BLOCK, LONG, false>), grid, dim3(BLOCK), 0, s, a);
  return hipGetLastError();
}

// the fewest threads a row that hold it in few pieces each
template <class E>
hipError_t rows_any(const PolicyArgs& a, hipStream_t s) {
  const int64_t pieces = a.vocab / E::V;
  if (pieces <= 64) return rows_of<E, 64, 1, 256, false>(a, s);
  if (pieces <= 256) return rows_of<E, 64, 4, 256, false>(a, s);
  if (pieces <= 1024) return rows_of<E, 256, 4, 256, false>(a, s);
  if (pieces <= 2048) return rows_of<E, 256, 8, 256, false>(a, s);
  if (pieces <= 4096) return rows_of<E, 1024, 4, 1024, false>(a, s);
  if (pieces <= 8192) return rows_of<E, 1024, 8, 1024, false>(a, s);
  if (pieces <= 16384) return rows_of<E, 1024, 16, 1024, false>(a, s);
  return rows_of<E, 1024, 16, 1024, true>(a, s);
}

}  // namespace

hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t s) {
  if (a.rows > 0) {
    const hipError_t e = dtype == DW_BF16 ? rows_any<Bf16>(a, s) : rows_any<F32>(a, s);
    if (e != hipSuccess || !a.loss) return e;
  }
  if (!a.loss) return hipSuccess;
  hipLaunchKernelGGL(policy_sum_kernel, dim3((unsigned)a.k), dim3(256), 0, s, a.part, a.loss, a.rows);
  return hipGetLastError();
}

}  // namespace dw
