// Rows of a table for tokens, and the gradient of the table by sorted tokens (gfx950, wave64).
//
//   y[r] = scale T[token[r]],     dT[v] = scale sum over r with token[r] = v of dy[r]
//
// The lookup is a copy of rows: bound by memory.
//
// The gradient without atomics: the rows' places are sorted by token, places of the same token in their order; a group of
// threads takes kChunk places in a row and adds the rows that share a token in registers.  A token whose places all lie in one
// chunk is written from there; of one that goes on into the next chunk each chunk leaves a partial sum, and a last kernel adds
// those in their order.  So every row of dy is read once, in fp32 sums whose order follows from the tokens alone, and a
// token that fills the whole batch costs no more than others.
//
// The sort: up to kRankRows places by counting (a place's rank is the number of smaller tokens, and of equal ones before it), which is
// n^2 comparisons but a single launch; longer lists digit by digit, eight bits at a time from the lowest, in blocks of kTile
// places whose counts of every digit are added up between the two passes over them.
#include "dw_ops.h"

namespace dw {

namespace {

// ---- lookup ----------------------------------------------------------------------------------------------------------

// U elements at any multiple of their size, as floats and back
template <class E, int U>
__device__ __forceinline__ void load_u(const typename E::T* p, float (&f)[U]) {
  if constexpr (E::V <= U) {
#pragma unroll
    for (int h = 0; h < U / E::V; ++h) {
      uint32_t r[4];
      float v[E::V];
      load_piece<E>(p + h * E::V, r);
      E::unpack(r, v);
#pragma unroll
      for (int j = 0; j < E::V; ++j) f[h * E::V + j] = v[j];
    }
  } else {                                                 // four of bf16
    struct __attribute__((packed, aligned(2))) Raw8a2 { uint32_t w[2]; };
    const Raw8a2 v = *reinterpret_cast<const Raw8a2*>(p);
#pragma unroll
    for (int j = 0; j < 2; ++j) { f[2 * j] = __uint_as_float(v.w[j] << 16); f[2 * j + 1] = __uint_as_float(v.w[j] & 0xFFFF0000u); }
  }
}
template <class E, int U>
__device__ __forceinline__ void store_u(typename E::T* p, const float (&f)[U]) {
  if constexpr (E::V <= U) {
#pragma unroll
    for (int h = 0; h < U / E::V; ++h) {
      float v[E::V];
#pragma unroll
      for (int j = 0; j < E::V; ++j) v[j] = f[h * E::V + j];
      store_piece<E>(p + h * E::V, v);
    }
  } else {
    struct __attribute__((packed, aligned(2))) Raw8a2 { uint32_t w[2]; };
    Raw8a2 v;
#pragma unroll
    for (int j = 0; j < 2; ++j) v.w[j] = pack_bf16(f[2 * j], f[2 * j + 1]);
    *reinterpret_cast<Raw8a2*>(p) = v;
  }
}

template <class ET, class E>
__global__ __launch_bounds__(256) void embedding_kernel(EmbedArgs a, int log_tpr) {
  constexpr int U = ET::V < E::V ? ET::V : E::V;
  const int w = blockIdx.y, t = threadIdx.x & ((1 << log_tpr) - 1), g = threadIdx.x >> log_tpr;
  const typename ET::T* table = reinterpret_cast<const typename ET::T*>(a.table.p) + w * a.table.stride;
  typename E::T* y = reinterpret_cast<typename E::T*>(a.y.p) + w * a.y.stride;
  const int n = (int)a.n;
  for (int64_t r = (int64_t)blockIdx.x * (256 >> log_tpr) + g; r < a.rows; r += (int64_t)gridDim.x * (256 >> log_tpr)) {
    const int32_t v = a.token[w * a.rows + r];
    const bool there = v >= 0 && v < a.vocab;
    const typename ET::T* from = table + (there ? v : 0) * a.table.ld;
    typename E::T* to = y + r * a.y.ld;
    for (int e0 = t * U; e0 < n; e0 += U << log_tpr) {
      if (e0 + U <= n) {
        float f[U];
#pragma unroll
        for (int j = 0; j < U; ++j) f[j] = 0.f;
        if (there) {
          load_u<ET, U>(from + e0, f);
#pragma unroll
          for (int j = 0; j < U; ++j) f[j] *= a.scale;
        }
        store_u<E, U>(to + e0, f);
      } else {
        for (int e = e0; e < n; ++e) E::put(to + e, there ? ET::one(from + e) * a.scale : 0.f);
      }
    }
  }
}

inline int log_threads(int64_t pieces) {                   // a power of two of threads for a row, at most a block
  int l = 0;
  while (l < 8 && (1 << l) < pieces) ++l;
  return l;
}
inline unsigned blocks_for(int64_t want, int k) {
  const int64_t most = 16 * kCus / k > 1 ? 16 * kCus / k : 1;
  return (unsigned)(want < most ? want : most);
}

template <class ET, class E>
hipError_t lookup(const EmbedArgs& a, hipStream_t s) {
  const int l = log_threads(ceil_div(a.n, ET::V < E::V ? ET::V : E::V));
  hipLaunchKernelGGL((embedding_kernel<ET, E>), dim3(blocks_for(ceil_div(a.rows, 256 >> l), a.k), (unsigned)a.k), dim3(256), 0, s, a, l);
  return hipGetLastError();
}

// ---- places by token -------------------------------------------------------------------------------------------------

constexpr int kRankRows = 8192;                            // up to here by counting
constexpr int kTile = 4096;                                // places of a block when sorting by digits, 1024 a wave
constexpr int kChunk = 32;                                 // places whose rows a group of threads adds up

// what is no token sorts behind all tokens
__device__ __forceinline__ int32_t key_of(int32_t token, int32_t vocab) { return (uint32_t)token < (uint32_t)vocab ? token : vocab; }

// 64 places a block, their keys against all of the worker's by 16 waves
__global__ __launch_bounds__(1024) void rank_kernel(const int32_t* token, int32_t* sorted, int32_t* place, int rows, int32_t vocab) {
  __shared__ int32_t part[16][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int32_t* tok = token + (int64_t)blockIdx.y * rows;
  const int r = blockIdx.x * 64 + lane;
  const int32_t mine = r < rows ? key_of(tok[r], vocab) : 0;
  const int per = (rows + 15) / 16, from = wave * per, to = from + per < rows ? from + per : rows;
  int rank = 0;
  for (int s = from; s < to; ++s) {
    const int32_t other = key_of(tok[s], vocab);
    rank += other < mine || (other == mine && s < r) ? 1 : 0;
  }
  part[wave][lane] = rank;
  __syncthreads();
  if (wave != 0 || r >= rows) return;
#pragma unroll
  for (int q = 1; q < 16; ++q) rank += part[q][lane];
  sorted[(int64_t)blockIdx.y * rows + rank] = mine;
  place[(int64_t)blockIdx.y * rows + rank] = r;
}

// the keys of a pass: the tokens themselves in the first, what the one before wrote in the others
struct Digits {
  const int32_t* token;                                    // first pass
  const int32_t* key_in; const int32_t* place_in;          // the others
  int32_t* key_out; int32_t* place_out;
  uint32_t* count;                                         // [k][256][tiles]
  int64_t rows;
  int32_t vocab, shift, tiles;
  __device__ __forceinline__ int32_t key(int w, int64_t r) const {
    return token ? key_of(token[w * rows + r], vocab) : key_in[w * rows + r];
  }
};

__global__ __launch_bounds__(256) void digit_count_kernel(Digits d) {
  __shared__ uint32_t count[256];
  const int w = blockIdx.y;
  count[threadIdx.x] = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < kTile; i += 256) {
    const int64_t r = (int64_t)blockIdx.x * kTile + i;
    if (r < d.rows) atomicAdd(&count[(uint32_t)d.key(w, r) >> d.shift & 255u], 1u);
  }
  __syncthreads();
  d.count[((int64_t)w * 256 + threadIdx.x) * d.tiles + blockIdx.x] = count[threadIdx.x];
}

// counts of all digits and tiles, digits first, to where each begins: one block a worker
__global__ __launch_bounds__(1024) void digit_scan_kernel(uint32_t* count, int64_t entries) {
  __shared__ uint32_t waves[16];
  uint32_t* c = count + (int64_t)blockIdx.x * entries;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint32_t before = 0;
  for (int64_t i0 = 0; i0 < entries; i0 += 4096) {
    const int64_t i = i0 + threadIdx.x * 4;
    uint32_t v[4], sum = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) { v[j] = i + j < entries ? c[i + j] : 0u; sum += v[j]; }
    uint32_t scan = sum;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const uint32_t u = (uint32_t)__shfl_up((int)scan, off);
      if (lane >= off) scan += u;
    }
    if (lane == 63) waves[wave] = scan;
    __syncthreads();
    uint32_t ahead = before, all = 0;
#pragma unroll
    for (int q = 0; q < 16; ++q) { ahead += q < wave ? waves[q] : 0u; all += waves[q]; }
    before += all;
    uint32_t at = ahead + scan - sum;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (i + j < entries) { c[i + j] = at; at += v[j]; }
    __syncthreads();
  }
}

// each place behind those of its tile's earlier places with the same digit: a wave takes 1024 places in their order
__global__ __launch_bounds__(256) void digit_place_kernel(Digits d) {
  __shared__ uint32_t next[4][256];
  const int w = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t r0 = (int64_t)blockIdx.x * kTile + wave * 1024;
#pragma unroll
  for (int q = 0; q < 4; ++q) next[q][threadIdx.x] = 0;
  __syncthreads();
  for (int i = 0; i < 16; ++i) {
    const int64_t r = r0 + i * 64 + lane;
    if (r < d.rows) atomicAdd(&next[wave][(uint32_t)d.key(w, r) >> d.shift & 255u], 1u);
  }
  __syncthreads();
  uint32_t at = d.count[((int64_t)w * 256 + threadIdx.x) * d.tiles + blockIdx.x];
#pragma unroll
  for (int q = 0; q < 4; ++q) { const uint32_t c = next[q][threadIdx.x]; next[q][threadIdx.x] = at; at += c; }
  __syncthreads();
  for (int i = 0; i < 16; ++i) {
    const int64_t r = r0 + i * 64 + lane;
    const bool there = r < d.rows;
    const int32_t key = there ? d.key(w, r) : 0;
    const uint32_t digit = (uint32_t)key >> d.shift & 255u;
    uint64_t same = __ballot(there);
#pragma unroll
    for (int b = 0; b < 8; ++b) {
      const uint64_t set = __ballot(digit >> b & 1u);
      same &= digit >> b & 1u ? set : ~set;
    }
    const uint32_t before = (uint32_t)__popcll(same & ((1ull << lane) - 1ull));
    // a wave's LDS accesses are done in their order: all lanes read, then the last of a digit's lanes moves its place on
    volatile uint32_t* mine = next[wave];
    const uint32_t to = there ? mine[digit] + before : 0u;
    __builtin_amdgcn_wave_barrier();
    if (there && (same >> lane) == 1ull) mine[digit] = to + 1u;
    __builtin_amdgcn_wave_barrier();
    if (there) {
      d.key_out[w * d.rows + to] = key;
      d.place_out[w * d.rows + to] = d.token ? (int32_t)r : d.place_in[w * d.rows + r];
    }
  }
}

// ---- sums ------------------------------------------------------------------------------------------------------------

struct SumArgs {
  EmbedGradArgs a;
  const int32_t* key; const int32_t* place;                // [k][rows], sorted
  float* part;                                             // [k][chunks][2][n]: of a token that came from the chunk before, and that goes on
  int64_t chunks;
};

__global__ __launch_bounds__(256) void embed_zero_kernel(EmbedGradArgs a) {
  const int w = blockIdx.y;
  float* grad = a.grad + w * a.grad_stride;
  if (a.grad_ld == a.n) {                                  // rows without gaps are one
    const int64_t all = a.vocab * a.n;
    for (int64_t e = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 4; e < all; e += (int64_t)gridDim.x * 1024) {
      const float zero[4] = {0.f, 0.f, 0.f, 0.f};
      store16<F32>(grad, e, all, zero);
    }
    return;
  }
  for (int64_t v = blockIdx.x; v < a.vocab; v += gridDim.x)
    for (int64_t e = threadIdx.x * 4; e < a.n; e += 1024) {
      const float zero[4] = {0.f, 0.f, 0.f, 0.f};
      store16<F32>(grad + v * a.grad_ld, e, a.n, zero);
    }
}

// the elements e0 .. e0+V-1 of a row of the gradient
template <int V>
__device__ __forceinline__ void put_sum(const EmbedGradArgs& a, int w, int32_t v, int64_t e0, float (&s)[V]) {
  float* row = a.grad + w * a.grad_stride + v * a.grad_ld;
#pragma unroll
  for (int q = 0; q < V / 4; ++q) {
    float f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = s[4 * q + j] * a.scale;
    if (a.accumulate) {
      float old[4];
      load_floats<4>(row, e0 + 4 * q, a.n, 0.f, old);
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] += old[j];
    }
    store16<F32>(row, e0 + 4 * q, a.n, f);
  }
}

template <class E>
__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs s, int log_tpr) {
  constexpr int V = E::V;
  const EmbedGradArgs& a = s.a;
  const int w = blockIdx.z, t = threadIdx.x & ((1 << log_tpr) - 1);
  const int64_t c = (int64_t)blockIdx.x * (256 >> log_tpr) + (threadIdx.x >> log_tpr);
  const int64_t e0 = (((int64_t)blockIdx.y << log_tpr) + t) * V;
  if (c >= s.chunks || e0 >= a.n) return;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride;
  const int32_t* key = s.key + w * a.rows;
  const int32_t* place = s.place + w * a.rows;
  const int64_t i0 = c * kChunk, i1 = i0 + kChunk < a.rows ? i0 + kChunk : a.rows;
  float* part = s.part + (w * s.chunks + c) * 2 * a.n;
  float sum[V];
#pragma unroll
  for (int j = 0; j < V; ++j) sum[j] = 0.f;
  int32_t now = key[i0];
  bool from_before = i0 > 0 && key[i0 - 1] == now;
  for (int64_t i = i0; i < i1; ++i) {
    if (now >= a.vocab) return;                            // nothing but what is no token from here on
    float f[V];
    uint32_t raw[4];
    load16<E>(dy + place[i] * a.dy.ld, e0, a.n, raw);
    E::unpack(raw, f);
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] += f[j];
    const int32_t next = i + 1 < a.rows ? key[i + 1] : -1;
    if (i + 1 == i1 || next != now) {
      const bool goes_on = i + 1 == i1 && next == now;
      if (from_before || goes_on) {
        float* to = part + (from_before ? 0 : a.n);
#pragma unroll
        for (int j = 0; j < V; ++j)
          if (e0 + j < a.n) to[e0 + j] = sum[j];
      } else {
        put_sum<V>(a, w, now, e0, sum);
      }
#pragma unroll
      for (int j = 0; j < V; ++j) sum[j] = 0.f;
      now = next;
      from_before = false;
    }
  }
}

// tokens that go on from the chunk they begin in: its partial sum and those of the chunks behind it
__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs s) {
  const EmbedGradArgs& a = s.a;
  const int w = blockIdx.z;
  const int32_t* key = s.key + w * a.rows;
  const int64_t c = blockIdx.x, i0 = c * kChunk, last = i0 + kChunk - 1;
  if (last + 1 >= a.rows) return;
  const int32_t v = key[last];
  if (v >= a.vocab || key[last + 1] != v) return;
  if (key[i0] == v && i0 > 0 && key[i0 - 1] == v) return;  // began before
  const int64_t e0 = ((int64_t)blockIdx.y * 256 + threadIdx.x) * 4;
  if (e0 >= a.n) return;
  const float* part = s.part + (w * s.chunks + c) * 2 * a.n;
  float sum[4];
  load_floats<4>(part + a.n, e0, a.n, 0.f, sum);
  for (int64_t q = 1; (c + q) * kChunk < a.rows && key[(c + q) * kChunk] == v; ++q) {
    float f[4];
    load_floats<4>(part + q * 2 * a.n, e0, a.n, 0.f, f);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += f[j];
  }
  put_sum<4>(a, w, v, e0, sum);
}

// scratch: sorted keys and places, then (digits) the others of the two, and counts, then the partial sums
struct GradLayout {
  size_t key, place, key2, place2, count, part, total;
  int64_t tiles, chunks;
  GradLayout(int k, int64_t rows, int64_t n) : tiles(ceil_div(rows, kTile)), chunks(ceil_div(rows, kChunk)) {
    size_t pos = 0;
    auto take = [&](size_t bytes) { const size_t at = pos; pos += (bytes + 255) / 256 * 256; return at; };
    const size_t list = (size_t)k * rows * 4;
    const bool digits = rows > kRankRows;
    key = take(list);
    place = take(list);
    key2 = take(digits ? list : 0);
    place2 = take(digits ? list : 0);
    count = take(digits ? (size_t)k * 256 * tiles * 4 : 0);
    part = take(chunks > 1 ? (size_t)k * chunks * 2 * n * 4 : 0);
    total = pos;
  }
};

template <class E>
hipError_t sums(const SumArgs& s, hipStream_t stream) {
  const int64_t pieces = ceil_div(s.a.n, E::V);
  const int l = log_threads(pieces);
  const dim3 grid((unsigned)ceil_div(s.chunks, 256 >> l), (unsigned)ceil_div(pieces, 1 << l), (unsigned)s.a.k);
  hipLaunchKernelGGL(embed_sum_kernel<E>, grid, dim3(256), 0, stream, s, l);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_embedding(const EmbedArgs& a, int table_dtype, int dtype, hipStream_t s) {
  if (table_dtype == DW_BF16) return dtype == DW_BF16 ? lookup<Bf16, Bf16>(a, s) : lookup<Bf16, F32>(a, s);
  return dtype == DW_BF16 ? lookup<F32, Bf16>(a, s) : lookup<F32, F32>(a, s);
}

size_t embedding_grad_scratch(int k, int64_t rows, int64_t vocab, int64_t n) { return GradLayout(k, rows, n).total; }

hipError_t launch_embedding_grad(const EmbedGradArgs& a, int dtype, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (!a.accumulate) {
    const int64_t want = ceil_div(a.vocab * a.n, 1024 * 4);
    hipLaunchKernelGGL(embed_zero_kernel, dim3((unsigned)(want < 8 * kCus ? want : 8 * kCus), (unsigned)a.k), dim3(256), 0, s, a);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (a.rows == 0) return e;
  const GradLayout lay(a.k, a.rows, a.n);
  int32_t* key = reinterpret_cast<int32_t*>(a.scratch + lay.key);
  int32_t* place = reinterpret_cast<int32_t*>(a.scratch + lay.place);
  if (a.rows <= kRankRows) {
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)ceil_div(a.rows, 64), (unsigned)a.k), dim3(1024), 0, s, a.token, key, place, (int)a.rows,
                       (int32_t)a.vocab);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    int32_t* key2 = reinterpret_cast<int32_t*>(a.scratch + lay.key2);
    int32_t* place2 = reinterpret_cast<int32_t*>(a.scratch + lay.place2);
    int passes = 1;
    while (passes < 4 && a.vocab >> (8 * passes)) ++passes;  // digits of the largest key, vocab
    Digits d = {};
    d.count = reinterpret_cast<uint32_t*>(a.scratch + lay.count);
    d.rows = a.rows;
    d.vocab = (int32_t)a.vocab;
    d.tiles = (int32_t)lay.tiles;
    const dim3 grid((unsigned)lay.tiles, (unsigned)a.k);
    for (int p = 0; p < passes; ++p) {
      d.token = p == 0 ? a.token : nullptr;
      d.shift = 8 * p;
      d.key_out = key; d.place_out = place;
      hipLaunchKernelGGL(digit_count_kernel, grid, dim3(256), 0, s, d);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(digit_scan_kernel, dim3((unsigned)a.k), dim3(1024), 0, s, d.count, (int64_t)256 * lay.tiles);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      hipLaunchKernelGGL(digit_place_kernel, grid, dim3(256), 0, s, d);
      if ((e = hipGetLastError()) != hipSuccess) return e;
      d.key_in = key; d.place_in = place;
      int32_t* t = key; key = key2; key2 = t;
      t = place; place = place2; place2 = t;
    }
    key = const_cast<int32_t*>(d.key_in);
    place = const_cast<int32_t*>(d.place_in);
  }
  SumArgs sum = {a, key, place, reinterpret_cast<float*>(a.scratch + lay.part), lay.chunks};
  if ((e = dtype == DW_BF16 ? sums<Bf16>(sum, s) : sums<F32>(sum, s)) != hipSuccess || lay.chunks == 1) return e;
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)(lay.chunks - 1), (unsigned)ceil_div(a.n, 1024), (unsigned)a.k), dim3(256), 0, s, sum);
  return hipGetLastError();
}

}  // namespace dw
