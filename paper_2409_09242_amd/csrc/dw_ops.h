// Internal declarations shared by the operators for training steps that the caller puts together (layer norm, 8-bit
// block products, policy loss, gradient clipping): loads and stores of rows, reductions, argument checks.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "dw_internal.h"

namespace dw {

constexpr int kCus = 256;             // compute units: grids are sized in multiples of it

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// 16 bytes at an address that is aligned to the element only: global memory takes such loads and stores whole, so a row
// that starts anywhere costs the lines it touches and no variant of its own
struct __attribute__((packed, aligned(2))) Raw16a2 { uint32_t w[4]; };
struct __attribute__((packed, aligned(4))) Raw16a4 { uint32_t w[4]; };

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {       // round to nearest even, NaN stays NaN
  const f32x2_t f = {lo, hi};
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2_t));
}

// a row element type: V elements fill 16 bytes
struct F32 {
  typedef float T;
  static constexpr int V = 4;
  static constexpr uint32_t kMinusInf = 0xFF800000u;
  __device__ static __forceinline__ void unpack(const uint32_t (&r)[4], float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = __uint_as_float(r[j]);
  }
  __device__ static __forceinline__ void pack(const float (&f)[V], uint32_t (&r)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = __float_as_uint(f[j]);
  }
  __device__ static __forceinline__ float one(const T* p) { return *p; }
  __device__ static __forceinline__ uint32_t bits(const T* p) { return *reinterpret_cast<const uint32_t*>(p); }      // as it is in memory
  __device__ static __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits); }
  __device__ static __forceinline__ void put(T* p, float f) { *p = f; }
  typedef Raw16a4 Raw;
};
struct Bf16 {
  typedef uint16_t T;
  static constexpr int V = 8;
  static constexpr uint32_t kMinusInf = 0xFF80FF80u;
  __device__ static __forceinline__ void unpack(const uint32_t (&r)[4], float (&f)[V]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f[2 * j] = __uint_as_float(r[j] << 16);
      f[2 * j + 1] = __uint_as_float(r[j] & 0xFFFF0000u);
    }
  }
  __device__ static __forceinline__ void pack(const float (&f)[V], uint32_t (&r)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = pack_bf16(f[2 * j], f[2 * j + 1]);
  }
  __device__ static __forceinline__ float one(const T* p) { return __uint_as_float((uint32_t)*p << 16); }
  __device__ static __forceinline__ uint32_t bits(const T* p) { return *p; }
  __device__ static __forceinline__ float value(uint32_t bits) { return __uint_as_float(bits << 16); }
  __device__ static __forceinline__ void put(T* p, float f) { *p = (uint16_t)pack_bf16(f, 0.f); }
  typedef Raw16a2 Raw;
};

// 16 bytes of whole elements
template <class E>
__device__ __forceinline__ void load_piece(const typename E::T* p, uint32_t (&r)[4]) {
  const typename E::Raw v = *reinterpret_cast<const typename E::Raw*>(p);
#pragma unroll
  for (int j = 0; j < 4; ++j) r[j] = v.w[j];
}
template <class E>
__device__ __forceinline__ void store_piece(typename E::T* p, const float (&f)[E::V]) {
  typename E::Raw v;
  E::pack(f, v.w);
  *reinterpret_cast<typename E::Raw*>(p) = v;
}
// piece q (16 bytes) of a row: a 32-bit offset from the row's address, which may be in scalar registers
template <class E, class T>
__device__ __forceinline__ T* at_piece(T* row, int q) {
  return reinterpret_cast<T*>(reinterpret_cast<uintptr_t>(row) + (uint32_t)q * 16u);
}
// the same for data that streams through once and must not displace what is read again
typedef uint32_t u32x4_a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef uint32_t u32x4_a4 __attribute__((ext_vector_type(4), aligned(4)));
template <class E> struct Streamed { typedef u32x4_a4 T; };
template <> struct Streamed<Bf16> { typedef u32x4_a2 T; };
template <class E>
__device__ __forceinline__ void load_piece_once(const typename E::T* p, uint32_t (&r)[4]) {
  const auto v = __builtin_nontemporal_load(reinterpret_cast<const typename Streamed<E>::T*>(p));
  r[0] = v.x; r[1] = v.y; r[2] = v.z; r[3] = v.w;
}
template <class E>
__device__ __forceinline__ void store_piece_once(typename E::T* p, const float (&f)[E::V]) {
  uint32_t r[4];
  E::pack(f, r);
  typename Streamed<E>::T v = {r[0], r[1], r[2], r[3]};
  __builtin_nontemporal_store(v, reinterpret_cast<typename Streamed<E>::T*>(p));
}
// the 16 bytes of elements e0 .. e0+V-1 of a row of n; elements at n and beyond read as zero
template <class E>
__device__ __forceinline__ void load16(const typename E::T* row, int64_t e0, int64_t n, uint32_t (&r)[4]) {
  if (e0 + E::V <= n) {
    const typename E::Raw v = *reinterpret_cast<const typename E::Raw*>(row + e0);
#pragma unroll
    for (int j = 0; j < 4; ++j) r[j] = v.w[j];
  } else {
    float f[E::V];
#pragma unroll
    for (int j = 0; j < E::V; ++j) f[j] = e0 + j < n ? E::one(row + e0 + j) : 0.f;
    E::pack(f, r);
  }
}
template <class E>
__device__ __forceinline__ void store16(typename E::T* row, int64_t e0, int64_t n, const float (&f)[E::V]) {
  if (e0 + E::V <= n) {
    typename E::Raw v;
    E::pack(f, v.w);
    *reinterpret_cast<typename E::Raw*>(row + e0) = v;
  } else {
#pragma unroll
    for (int j = 0; j < E::V; ++j)
      if (e0 + j < n) E::put(row + e0 + j, f[j]);
  }
}
// V floats of a parameter row (4-byte aligned)
template <int V>
__device__ __forceinline__ void load_floats(const float* row, int64_t e0, int64_t n, float fill, float (&f)[V]) {
  if (e0 + V <= n) {
#pragma unroll
    for (int q = 0; q < V / 4; ++q) {
      const Raw16a4 v = *reinterpret_cast<const Raw16a4*>(row + e0 + 4 * q);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[4 * q + j] = __uint_as_float(v.w[j]);
    }
  } else {
#pragma unroll
    for (int j = 0; j < V; ++j) f[j] = e0 + j < n ? row[e0 + j] : fill;
  }
}

// sum over the TPR consecutive threads that share a row, to all of them; TPR > 64: the whole block of TPR threads
// (`lds`: 2 * TPR/64 floats; `turn` alternates between calls so that one barrier a call is enough)
template <int TPR>
__device__ __forceinline__ float row_sum(float x, float* lds, int& turn) {
#pragma unroll
  for (int off = 1; off < (TPR < 64 ? TPR : 64); off <<= 1) x += __shfl_xor(x, off);
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = lds + turn * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = x;
    __syncthreads();
    x = at[0];
#pragma unroll
    for (int w = 1; w < W; ++w) x += at[w];
  }
  return x;
}

// two such sums with one barrier (`lds`: 4 * TPR/64 floats)
template <int TPR>
__device__ __forceinline__ void row_sum2(float x, float y, float* lds, int& turn, float& sx, float& sy) {
#pragma unroll
  for (int off = 1; off < (TPR < 64 ? TPR : 64); off <<= 1) { x += __shfl_xor(x, off); y += __shfl_xor(y, off); }
  if constexpr (TPR > 64) {
    constexpr int W = TPR / 64;
    float* at = lds + turn * 2 * W;
    turn ^= 1;
    if ((threadIdx.x & 63) == 0) { at[threadIdx.x >> 6] = x; at[W + (threadIdx.x >> 6)] = y; }
    __syncthreads();
    x = at[0];
    y = at[W];
#pragma unroll
    for (int w = 1; w < W; ++w) { x += at[w]; y += at[W + w]; }
  }
  sx = x;
  sy = y;
}

constexpr int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

// ---- layer norm (dw_norm.hip) ----------------------------------------------------------------------------------------
struct Rows { const void* p; int64_t ld, stride; };        // element (w, r, j) at p + w*stride + r*ld + j, in elements
struct RowsOut { void* p; int64_t ld, stride; };

struct NormArgs {
  Rows x, dy;
  RowsOut out;                                             // y, or dx
  const float* gamma; const float* beta; int64_t param_stride;
  float* mean; float* rstd;                                // [k][rows]
  float* dgamma; float* dbeta; int64_t grad_stride;
  float* part;                                             // backward: [k][strips][2][n]
  int k, strips;
  int64_t rows, n;
  float eps;
};
hipError_t launch_layer_norm(const NormArgs& a, int dtype, hipStream_t s);
hipError_t launch_layer_norm_grad(const NormArgs& a, bool sums, int dtype, hipStream_t s);
int layer_norm_grad_strips(int k, int64_t rows, int64_t n, int dtype);


// ---- policy loss (dw_policy.hip) -------------------------------------------------------------------------------------
struct PolicyArgs {
  Rows logits;
  RowsOut grad;                                            // p = nullptr: not wanted
  const int32_t* target;                                   // [k][rows], as the others
  const float* old_logp; const float* ref_logp; const float* advantage;      // old_logp = nullptr: log probabilities alone
  const float* weight; float mean_weight;                  // weight = nullptr: mean_weight for every row
  float q_min, q_max, kl_coef;
  float* logp; float* part;                                // part: a row's share of the loss
  float* loss;                                             // [k]
  int k;
  int64_t rows, vocab;
};
hipError_t launch_policy(const PolicyArgs& a, int dtype, hipStream_t s);

// ---- gradient norm and clipping (dw_clip.hip) ------------------------------------------------------------------------
// Arguments of one launch: tensors j < n of `workers` workers.  The table holds n + 1 places (in elements, from the launch's first
// tensor), the tensors' addresses (workers by n), then n first chunks and their types, two to a word.
struct ClipTable {
  static constexpr int kWords = 469;                       // 64-bit words; all arguments stay below 4 KB
  uint64_t word[kWords];
  int n, workers, chunks, worker0;
  int64_t chunk, elements;                                 // elements of a chunk, and of the launch's tensors (of one worker)
  double* part; int parts, part0;                          // partial sums [k][parts], this launch's first
  float* norm; float max_norm;
  const double* wide;                                      // [k] norms, or nullptr: every block adds the partial sums
  float* out; int64_t out_stride, out0;                    // nullptr: in place; out0: elements of a worker before this launch's
  // most tensors of one launch for so many workers
  static int tensors(int workers) { return (kWords - 2) * 2 / (2 * workers + 3); }
  __host__ __device__ int64_t first_of(int j) const { return (int64_t)word[j]; }
  __host__ __device__ const void* address(int w, int j) const { return reinterpret_cast<const void*>(word[n + 1 + w * n + j]); }
  __host__ __device__ int chunk_word(int j) const {
    const uint64_t v = word[n + 1 + workers * n + (j >> 1)];
    return (int)(uint32_t)(j & 1 ? v >> 32 : v);
  }
  __host__ __device__ int chunk_of(int j) const { return chunk_word(j) & 0x7FFFFFFF; }
  __host__ __device__ bool is_bf16(int j) const { return chunk_word(j) < 0; }
  void set_first(int j, int64_t v) { word[j] = (uint64_t)v; }
  void set_address(int w, int j, const void* p) { word[n + 1 + w * n + j] = reinterpret_cast<uint64_t>(p); }
  void set_chunk(int j, int32_t c) {
    uint64_t& v = word[n + 1 + workers * n + (j >> 1)];
    v = j & 1 ? (v & 0xFFFFFFFFull) | (uint64_t)(uint32_t)c << 32 : (uint64_t)(uint32_t)c;
  }
  void set_type(int j, bool bf16) {
    if (bf16) word[n + 1 + workers * n + (j >> 1)] |= j & 1 ? 1ull << 63 : 1ull << 31;
  }
};
static_assert(sizeof(ClipTable) <= 4096, "kernel arguments");
int64_t clip_chunk(int64_t elements_of_all_workers);
void clip_table_fill(ClipTable& t, const void* const* grads, const int64_t* counts, const int32_t* dtypes, int dtype, int per_worker,
                     int j0, int w0);
hipError_t launch_grad_squares(const ClipTable& t, hipStream_t s);
bool clip_adds_in_between(int parts);
hipError_t launch_grad_norm(const double* part, int parts, float* norm, double* wide, int k, hipStream_t s);
hipError_t launch_clip(const ClipTable& t, hipStream_t s);

// ---- 8-bit block products (dw_fp8_quant.hip, dw_gemm_fp8.hip) ----------------------------------------------------------
struct QuantArgs {
  Rows x;
  int k, square;
  int64_t rows, n;
  uint8_t* q; uint8_t* scale;                              // [k][rows][DW_FP8_ROW(n)], [k][rows][DW_FP8_SCALES(n)], or nullptr
  uint8_t* qt; uint8_t* scale_t;                           // [k][n][DW_FP8_ROW(rows)], [k][n][DW_FP8_SCALES(rows)], or nullptr
  const float* rstd;                                       // [k][rows]: the numbers are x rstd gamma (x alone where nullptr)
  const float* gamma; int64_t gamma_stride;                // [k] rows of n, or nullptr: 1
  uint32_t first;                                          // a launch's first block along the rows (0 from the caller)
};
hipError_t launch_fp8_quantize(const QuantArgs& a, int dtype, hipStream_t s);

struct Fp8Args {
  const uint8_t* a; const uint8_t* sa;                     // [k][m][kp], [k][m][ks]
  const uint8_t* b; const uint8_t* sb;                     // [k][n][kp], [k][n][ks]
  const float* bias; int64_t bias_stride;                  // [k] rows of n, or nullptr
  void* c; int64_t ldc, c_stride;
  int k, dtype;
  int64_t m, n, kp, ks;                                    // kp: padded contraction; ks: scale bytes of a row
  Rows x; int64_t contraction;                             // p != nullptr: operand a is x, to be quantised on the way (type: dtype)
  float* part; int slice_blocks;                           // slices of the contraction: [slices][k][m][n], blocks of 128 each
};
size_t fp8_scratch_bytes(int k, int64_t m, int64_t n, int64_t kp);
hipError_t launch_fp8_matmul(const Fp8Args& a, hipStream_t s);
bool fp8_linear_fused(int k, int64_t m, int64_t n, int64_t kp);
hipError_t launch_fp8_linear_fused(const Fp8Args& a, hipStream_t s);

// ---- dropout (dw_dropout.hip, dw_dropout.h) --------------------------------------------------------------------------
struct Drop {
  uint64_t seed, step;
  const uint64_t* d_step;                                  // nullptr, or what is added to step
  uint32_t limit;                                          // kept: a 16-bit number below it (65536: everything, no dropout)
  float factor;                                            // of what is kept
};
struct DropoutArgs {
  Rows x, res;                                             // res.p = nullptr: none
  RowsOut y;
  Drop drop;
  int k;
  int64_t rows, n;
};
hipError_t launch_dropout(const DropoutArgs& a, int dtype, hipStream_t s);

// ---- root-mean-square norm (dw_rms.hip) --------------------------------------------------------------------------------
struct RmsArgs {
  Rows x, res;                                             // res.p = nullptr: none
  Drop drop;
  const float* gamma; int64_t param_stride;
  RowsOut h, y;                                            // p = nullptr: not wanted
  uint8_t* q; uint8_t* scale;                              // y in 8 bits, or nullptr
  float* rstd;                                             // [k][rows], or nullptr
  int k;
  int64_t rows, n;
  float eps;
};
hipError_t launch_rms_norm(const RmsArgs& a, int dtype, hipStream_t s);

struct RmsGradArgs {
  Rows dy, h, dh;                                          // dh.p = nullptr: none
  Drop drop;
  const float* gamma; int64_t param_stride;
  const float* rstd;                                       // [k][rows]
  RowsOut dres, dx;                                        // p = nullptr: not wanted
  float* dgamma; int64_t grad_stride;                      // nullptr: not wanted
  float* part;                                             // [k][strips][n]
  int k, strips;
  int64_t rows, n;
};
int rms_norm_grad_strips(int k, int64_t rows, int64_t n, int dtype);
hipError_t launch_rms_norm_grad(const RmsGradArgs& a, int dtype, hipStream_t s);

// ---- embedding (dw_embed.hip) ------------------------------------------------------------------------------------------
struct EmbedArgs {
  const int32_t* token;                                    // [k][rows]
  Rows table;
  RowsOut y;
  int k;
  int64_t rows, vocab, n;
  float scale;
};
hipError_t launch_embedding(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t s);

struct EmbedGradArgs {
  const int32_t* token;                                    // [k][rows]
  Rows dy;
  float* grad; int64_t grad_ld, grad_stride;
  int k, accumulate;
  int64_t rows, vocab, n;
  float scale;
  char* scratch;
};
size_t embedding_grad_scratch(int k, int64_t rows, int64_t vocab, int64_t n);
hipError_t launch_embedding_grad(const EmbedGradArgs& a, int dtype, hipStream_t s);

// ---- logits before a token is drawn (dw_adjust.hip) --------------------------------------------------------------------
struct AdjustArgs {
  Rows logits;
  RowsOut out;
  const int32_t* history; int64_t history_ld, history_stride, length;
  const int32_t* filled; const int32_t* answer;            // [k][rows] each, or nullptr
  const float* repetition; const float* presence; const float* frequency;
  const float* bias; int64_t bias_ld, bias_stride;
  const uint32_t* mask; int64_t mask_ld, mask_stride;
  int k;
  int64_t rows, vocab;
};
hipError_t launch_adjust_logits(const AdjustArgs& a, int dtype, hipStream_t s);

}  // namespace dw
