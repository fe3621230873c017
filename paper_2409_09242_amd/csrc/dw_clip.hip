// The gradient norm of every worker over all its tensors, and clipping (gfx950, wave64).
//
//   norm_w = sqrt(sum over the worker's tensors and elements of g^2),   c_w = min(1, max_norm / (norm_w + 1e-6)),  g' = c_w g
//
// Two passes: a block adds up the squares of a chunk of one tensor in 64 bits (no overflow, and the order of additions is
// fixed) and leaves one partial sum; the second pass adds a worker's partial sums, every block for itself and in the same
// order (many of them: a launch in between, once), and writes its chunk.  In place a worker that is not clipped is not touched again.
//
// The workers are replicas of one model, so tensor j has the same size for all of them: a launch carries, in its
// arguments, where the chunks and elements of its tensors begin (once) and their addresses (for each worker).
//
// Bound by memory: 8 workers of 50.4e6 elements in bf16 into a flat fp32 gradient: 138 us for the norms (5.9 TB/s), 511 for the
// packing (4.7 TB/s, twice as many bytes written as read); in place 454 for both, all clipped.  The second read is the price of a norm over all of it; the last
// 256 MB of the first pass are read first by the second, from the chip's cache.
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

constexpr int kAhead = 4;                                   // pieces of a thread in flight

template <class E>
__device__ __forceinline__ double squares(const void* base, const Chunk& c) {
  const typename E::T* p = reinterpret_cast<const typename E::T*>(base) + c.e0;
  const int n = (int)(c.e1 - c.e0), whole = n / E::V;
  double s = 0.0;
  auto add = [&](const uint32_t (&raw)[4]) {
    float f[E::V];
    E::unpack(raw, f);
#pragma unroll
    for (int j = 0; j < E::V; ++j) s = __builtin_fma((double)f[j], (double)f[j], s);
  };
  int q = threadIdx.x;
  for (; q + (kAhead - 1) * kThreads < whole; q += kAhead * kThreads) {
    uint32_t raw[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_piece<E>(p + (q + i * kThreads) * E::V, raw[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) add(raw[i]);
  }
  for (; q < whole; q += kThreads) {
    uint32_t raw[4];
    load_piece<E>(p + q * E::V, raw);
    add(raw);
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

// the norm of a worker from its partial sums
__device__ __forceinline__ double worker_norm(const double* part, int parts, double* lds) {
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < parts; i += kThreads) s += part[i];
  return sqrt(block_sum(s, lds));
}

// wide[w]: the norm in 64 bits for the second pass (nullptr: there is none, or its blocks add up for themselves)
__global__ __launch_bounds__(kThreads) void grad_norm_kernel(const double* part, int parts, float* norm, double* wide) {
  __shared__ double lds[4];
  const double v = worker_norm(part + (int64_t)blockIdx.x * parts, parts, lds);
  if (threadIdx.x == 0) {
    norm[blockIdx.x] = (float)v;
    if (wide) wide[blockIdx.x] = v;
  }
}

// four elements at a time into fp32, so that a wave's stores follow each other without gaps
template <class E>
__device__ __forceinline__ void pack_chunk(const void* base, float* out, const Chunk& c, float factor) {
  typedef uint32_t u32x2_a2 __attribute__((ext_vector_type(2), aligned(2)));
  const typename E::T* p = reinterpret_cast<const typename E::T*>(base) + c.e0;
  const int n = (int)(c.e1 - c.e0), whole = n / 4;
  struct Four { uint32_t w[E::V == 8 ? 2 : 4]; };
  auto get = [&](int q) {
    Four r;
    if constexpr (E::V == 8) {
      const u32x2_a2 v = *reinterpret_cast<const u32x2_a2*>(p + q * 4);
      r.w[0] = v.x; r.w[1] = v.y;
    } else {
      load_piece<E>(p + q * 4, r.w);
    }
    return r;
  };
  auto put = [&](const Four& r, int q) {
    float f[4];
    if constexpr (E::V == 8) {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(j & 1 ? r.w[j >> 1] & 0xFFFF0000u : r.w[j >> 1] << 16) * factor;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(r.w[j]) * factor;
    }
    store_piece_once<F32>(out + q * 4, f);
  };
  int q = threadIdx.x;
  for (; q + (kAhead - 1) * kThreads < whole; q += kAhead * kThreads) {
    Four r[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) r[i] = get(q + i * kThreads);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) put(r[i], q + i * kThreads);
  }
  for (; q < whole; q += kThreads) put(get(q), q);
  const int e = whole * 4 + threadIdx.x;
  if (e < n) out[e] = E::one(p + e) * factor;
}

template <class E>
__device__ __forceinline__ void scale_chunk(void* base, const Chunk& c, float factor) {
  typename E::T* p = reinterpret_cast<typename E::T*>(base) + c.e0;
  const int n = (int)(c.e1 - c.e0), whole = n / E::V;
  auto put = [&](const uint32_t (&raw)[4], int q) {
    float f[E::V];
    E::unpack(raw, f);
#pragma unroll
    for (int j = 0; j < E::V; ++j) f[j] *= factor;
    store_piece<E>(p + q * E::V, f);
  };
  int q = threadIdx.x;
  for (; q + (kAhead - 1) * kThreads < whole; q += kAhead * kThreads) {
    uint32_t raw[kAhead][4];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) load_piece<E>(p + (q + i * kThreads) * E::V, raw[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) put(raw[i], q + i * kThreads);
  }
  for (; q < whole; q += kThreads) {
    uint32_t raw[4];
    load_piece<E>(p + q * E::V, raw);
    put(raw, q);
  }
  const int e = whole * E::V + threadIdx.x;
  if (e < n) E::put(p + e, E::one(p + e) * factor);
}

template <bool PACK>
__global__ __launch_bounds__(kThreads) void clip_kernel(ClipTable t) {
  __shared__ double lds[4];
  // from the last chunk to the first: what the first pass read last is still in the chip's caches
  const int chunk = gridDim.x - 1 - blockIdx.x, worker = gridDim.y - 1 - blockIdx.y;
  const int w = t.worker0 + worker;
  double norm;
  if (t.wide) {
    norm = t.wide[w];
  } else {
    norm = worker_norm(t.part + (int64_t)w * t.parts, t.parts, lds);
    if (blockIdx.x == 0 && t.part0 == 0 && threadIdx.x == 0) t.norm[w] = (float)norm;
  }
  // a norm that is not finite leaves the gradients as they are: the caller sees it and can leave the step out
  const double c = (double)t.max_norm / (norm + 1e-6);
  const float factor = c < 1.0 && norm <= 1.79769313486231571e308 ? (float)c : 1.f;
  if (!PACK && factor == 1.f) return;
  const Chunk ch = find_chunk(t, chunk);
  void* p = const_cast<void*>(t.address(worker, ch.j));
  float* out = PACK ? t.out + (int64_t)w * t.out_stride + t.out0 + t.first_of(ch.j) + ch.e0 : nullptr;
  if constexpr (PACK) {
    if (t.is_bf16(ch.j)) pack_chunk<Bf16>(p, out, ch, factor);
    else pack_chunk<F32>(p, out, ch, factor);
  } else {
    if (t.is_bf16(ch.j)) scale_chunk<Bf16>(p, ch, factor);
    else scale_chunk<F32>(p, ch, factor);
  }
}

}  // namespace

// Elements of a chunk: blocks enough that the last of them do not leave the chip half empty (8 x 50.4e6 elements: 12400
// blocks 653 us, 3100 blocks 677), and chunks of 4096 at least.
int64_t clip_chunk(int64_t elements_of_all_workers) {
  int64_t c = 4096;
  while (c * 16384 < elements_of_all_workers) c *= 2;
  return c;
}
// Up to so many partial sums a worker every block of the second pass adds them up for itself; beyond, a launch between the
// passes does it once.
bool clip_adds_in_between(int parts) { return parts > 512; }

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
hipError_t launch_grad_norm(const double* part, int parts, float* norm, double* wide, int k, hipStream_t s) {
  hipLaunchKernelGGL(grad_norm_kernel, dim3((unsigned)k), dim3(kThreads), 0, s, part, parts, norm, wide);
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
