// The gradient norm of every worker over all its tensors, and clipping (gfx950, wave64).
//
//   norm_w = sqrt(sum over the worker's tensors and elements of g^2),   c_w = min(1, max_norm / (norm_w + 1e-6)),  g' = c_w g
//
// Two passes: a block adds up the squares of a chunk of one tensor in 64 bits (no overflow, and the order of additions is
// fixed) and leaves one partial sum; the second pass adds a worker's partial sums, every block for itself and in the same
// order, and writes its chunk.  In place a worker that is not clipped is not touched again.
//
// The workers are replicas of one model, so tensor j has the same size for all of them: a launch carries, in its
// arguments, where the chunks and elements of its tensors begin (once) and their addresses (for each worker).
#include "dw_ops.h"

namespace dw {

namespace {

constexpr int kThreads = 256;

// what a block works on: elements [e0, e1) of tensor j of worker blockIdx.y
struct Chunk { int j; int64_t e0, e1; };

__device__ __forceinline__ Chunk find_chunk(const ClipTable& t, int b) {
  // the last tensor whose first chunk is at or before b: the lanes look at 64 tensors each turn
  int j = 0;
  const int lane = threadIdx.x & 63;
  for (int base = 0; base < t.n; base += 64) {
    const bool at = base + lane < t.n && t.chunk_of(base + lane) <= b;
    j += __popcll(__ballot(at));
  }
  j = __builtin_amdgcn_readfirstlane(j - 1);
  Chunk c;
  c.j = j;
  c.e0 = (int64_t)(b - t.chunk_of(j)) * t.chunk;
  const int64_t count = t.first_of(j + 1) - t.first_of(j);
  c.e1 = c.e0 + t.chunk < count ? c.e0 + t.chunk : count;
  return c;
}

// sum over the block, to all threads, in a fixed order
__device__ __forceinline__ double block_sum(double s, double* lds) {
#pragma unroll
  for (int off = 1; off < 64; off <<= 1) s += __shfl_xor(s, off);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = s;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);
}

template <class E>
__device__ __forceinline__ double squares(const void* base, const Chunk& c) {
  const typename E::T* p = reinterpret_cast<const typename E::T*>(base) + c.e0;
  const int n = (int)(c.e1 - c.e0), whole = n / E::V;
  double s = 0.0;
  for (int q = threadIdx.x; q < whole; q += kThreads) {
    uint32_t raw[4];
    float f[E::V];
    load_piece<E>(p + q * E::V, raw);
    E::unpack(raw, f);
#pragma unroll
    for (int j = 0; j < E::V; ++j) s = __builtin_fma((double)f[j], (double)f[j], s);
  }
  const int e = whole * E::V + threadIdx.x;
  if (e < n) { const double f = (double)E::one(p + e); s = __builtin_fma(f, f, s); }
  return s;
}

__global__ __launch_bounds__(kThreads) void grad_squares_kernel(ClipTable t) {
  __shared__ double lds[4];
  const Chunk c = find_chunk(t, blockIdx.x);
  const void* p = t.address(blockIdx.y, c.j);
  const double s = block_sum(t.is_bf16(c.j) ? squares<Bf16>(p, c) : squares<F32>(p, c), lds);
  if (threadIdx.x == 0) t.part[(int64_t)(t.worker0 + blockIdx.y) * t.parts + t.part0 + blockIdx.x] = s;
}

// the norm of worker w from its partial sums
__device__ __forceinline__ double worker_norm(const double* part, int parts, double* lds) {
  double s = 0.0;
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  return sqrt(block_sum(s, lds));
}

__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* part, int parts, float* norm) {
  __shared__ double lds[4];
  const double v = worker_norm(part + (int64_t)blockIdx.x * parts, parts, lds);
  if (threadIdx.x == 0) norm[blockIdx.x] = (float)v;
}

template <class E, bool PACK>
__device__ __forceinline__ void scale_chunk(void* base, float* out, const Chunk& c, float factor) {
  typename E::T* p = reinterpret_cast<typename E::T*>(base) + c.e0;
  const int n = (int)(c.e1 - c.e0), whole = n / E::V;
  for (int q = threadIdx.x; q < whole; q += kThreads) {
    uint32_t raw[4];
    float f[E::V];
    load_piece<E>(p + q * E::V, raw);
    E::unpack(raw, f);
#pragma unroll
    for (int j = 0; j < E::V; ++j) f[j] *= factor;
    if constexpr (PACK) {
#pragma unroll
      for (int h = 0; h < E::V / 4; ++h) {
        const float g[4] = {f[4 * h], f[4 * h + 1], f[4 * h + 2], f[4 * h + 3]};
        store_piece<F32>(out + q * E::V + 4 * h, g);
      }
    } else {
      store_piece<E>(p + q * E::V, f);
    }
  }
  const int e = whole * E::V + threadIdx.x;
  if (e < n) {
    const float f = E::one(p + e) * factor;
    if constexpr (PACK) out[e] = f; else E::put(p + e, f);
  }
}

template <bool PACK>
__global__ __launch_bounds__(kThreads) void clip_kernel(ClipTable t) {
  __shared__ double lds[4];
  const int w = t.worker0 + blockIdx.y;
  const double norm = worker_norm(t.part + (int64_t)w * t.parts, t.parts, lds);
  if (blockIdx.x == 0 && t.part0 == 0 && threadIdx.x == 0) t.norm[w] = (float)norm;
  // a norm that is not finite leaves the gradients as they are: the caller sees it and can leave the step out
  const double c = (double)t.max_norm / (norm + 1e-6);
  const float factor = c < 1.0 && norm <= 1.79769313486231571e308 ? (float)c : 1.f;
  if (!PACK && factor == 1.f) return;
  const Chunk ch = find_chunk(t, blockIdx.x);
  void* p = const_cast<void*>(t.address(blockIdx.y, ch.j));
  float* out = PACK ? t.out + (int64_t)w * t.out_stride + t.out0 + t.first_of(ch.j) + ch.e0 : nullptr;
  if (t.is_bf16(ch.j)) scale_chunk<Bf16, PACK>(p, out, ch, factor);
  else scale_chunk<F32, PACK>(p, out, ch, factor);
}

}  // namespace

// elements of a chunk: few enough partial sums that every block can add a worker's, many enough blocks to fill the chip
int64_t clip_chunk(int64_t elements_of_all_workers) {
  int64_t c = 4096;
  while (c * 4096 < elements_of_all_workers) c *= 2;
  return c;
}

// the tensors [j0, j0 + n) of the workers [w0, w0 + workers) that one launch carries
void clip_table_fill(ClipTable& t, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int dtype, int per_worker,
                     int j0, int w0) {
  int64_t first = 0, chunk = 0;
  for (int j = 0; j < t.n; ++j) {
    t.set_first(j, first);
    t.set_chunk(j, (int32_t)chunk);
    t.set_type(j, (dtypes ? dtypes[j0 + j] : dtype) == DW_BF16);
    first += counts[j0 + j];
    chunk += ceil_div(counts[j0 + j], t.chunk);
    for (int w = 0; w < t.workers; ++w) t.set_address(w, j, grads[(int64_t)(w0 + w) * per_worker + j0 + j]);
  }
  t.set_first(t.n, first);
  t.chunks = (int)chunk;
  t.elements = first;
}

hipError_t launch_grad_squares(const ClipTable& t, hipStream_t s) {
  if (t.chunks == 0) return hipSuccess;
  hipLaunchKernelGGL(grad_squares_kernel, dim3((unsigned)t.chunks, (unsigned)t.workers), dim3(kThreads), 0, s, t);
  return hipGetLastError();
}
hipError_t launch_grad_norm(const double* part, int parts, float* norm, int k, hipStream_t s) {
  hipLaunchKernelGGL(grad_norm_kernel, dim3((unsigned)k), dim3(kThreads), 0, s, part, parts, norm);
  return hipGetLastError();
}
hipError_t launch_clip(const ClipTable& t, hipStream_t s) {
  if (t.chunks == 0) return hipSuccess;
  const dim3 grid((unsigned)t.chunks, (unsigned)t.workers);
  if (t.out) hipLaunchKernelGGL(clip_kernel<true>, grid, dim3(kThreads), 0, s, t);
  else hipLaunchKernelGGL(clip_kernel<false>, grid, dim3(kThreads), 0, s, t);
  return hipGetLastError();
}

}  // namespace dw
