// Rows of a table for tokens, and the gradient of the table by sorted tokens (gfx950, wave64).
//
//   y[r] = scale T[token[r]],     dT[v] = scale sum over r with token[r] = v of dy[r]
//
// The lookup is a copy of rows, each by at most 256 threads: bound by memory where there are as many rows as the chip runs blocks, and otherwise by
// the trips of a row's block (1 row of 16384, fp32, still a launch, 4.6 us a call; 4 rows of 2^20, bf16, 185 us).
//
// The gradient without atomics: the rows' places are sorted by token, places of the same token in their order; a group of
// threads takes kChunk places in a row and adds the rows that share a token in registers.  A token whose places all lie in one
// chunk is written from there; of one that goes on into the next chunk each chunk leaves a partial sum, and a last kernel adds
// those in their order.  So every row of dy is read once, in fp32 sums whose order follows from the tokens and n alone.  The last kernel
// has a block for 1024 columns of a token, and above 512 columns a thread adds its columns' partial sums one after another: a token's time grows with
// its places.  16384 rows of 4096, bf16, over 32000 tokens, us a call: tokens as they come in text 181 (added to a gradient that is there
// 121), one token throughout 612 (355), of which the last kernel 549 (292); rows of 1024 columns 78 and 366 (72 and 354).
//
// The sort: few places by counting (a place's rank is the number of smaller tokens, and of equal ones before it), which is
// n^2 comparisons but a single launch; longer lists digit by digit, eight bits at a time from the lowest, in blocks of kTile
// places whose counts of every digit are added up between the two passes over them.
//
// Where the whole gradient is wanted, rows that no token has are filled with zeros beside the sort or beside the last sums.
// Bound by writing them: 4 x 4096 rows of 4096, bf16, over 32000 tokens 374 us a call, 2.4 GB at 6.4 TB/s (a fill alone reaches 6.8);
// added to a gradient that is there 99: sort 13, sums 75 (5.1 TB/s), joining 11.  3 x 333 rows of 1001, fp32, over 5003: 20.0, three launches.  Lookups: 8 x 1024 rows of 4096,
// fp32 to bf16, 31 us = 6.4 TB/s of what passes (common rows come from the caches); one row 2.0.
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
  const int64_t most = 16 * kCus / k;
  return (unsigned)(want < most ? want : most);
}

template <class ET, class E>
hipError_t lookup(const EmbedArgs& a, hipStream_t s) {
  const int l = log_threads(ceil_div(a.n, ET::V < E::V ? ET::V : E::V));
  hipLaunchKernelGGL((embedding_kernel<ET, E>), dim3(blocks_for(ceil_div(a.rows, 256 >> l), a.k), (unsigned)a.k), dim3(256), 0, s, a, l);
  return hipGetLastError();
}

// ---- places by token -------------------------------------------------------------------------------------------------

// Up to so many comparisons by counting, in one launch, else by digits, in three for each eight bits (with the sums of 64 columns, us: one
// worker's 8192 places 30 and 50, 16384 45 and 53, 32768 102 and 56; four workers' 8192 42 and 52, 16384 99 and 56; eight workers' 8192 63 and 56)
constexpr double kRankWork = 268435456.0;
// From so many bytes of zeros a worker's counting blocks are in front of its own zeros, below all workers' in front of all (us a call, own and
// all: 4 x 4096 rows over 32000 by 4096 392 and 401, 4 x 2048 by 2048 181 and 188, 2 x 2048 by 2048 100 and 103; 4 x 1024 over 8000 by
// 1024 33.1 and 31.9, 3 x 333 over 5003 by 1001 24.0 and 21.7; every 16th block of a row, which are all one die's: 445 for the first)
constexpr double kOwnRowBytes = 268435456.0;
constexpr int kRankPlaces = 16, kRankTile = 2048;          // places of a block, keys in its LDS
constexpr int kTile = 4096;                                // places of a block when sorting by digits, 1024 a wave
constexpr int kChunk = 16;                                 // places whose rows a group of threads adds up

// what is no token sorts behind all tokens
__device__ __forceinline__ int32_t key_of(int32_t token, int32_t vocab) { return (uint32_t)token < (uint32_t)vocab ? token : vocab; }

// n zeros by a wave, in whole pieces at multiples of 16 bytes
__device__ __forceinline__ void zero_floats(float* p, int64_t n) {
  const int lane = threadIdx.x & 63;
  const int64_t head = (0 - (reinterpret_cast<uintptr_t>(p) >> 2)) & 3, at = head < n ? head : n, pieces = (n - at) / 4;
  if (lane < at) p[lane] = 0.f;
  float4* q = reinterpret_cast<float4*>(p + at);
  for (int64_t i = lane; i < pieces; i += 64) q[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  const int64_t behind = at + pieces * 4 + lane;
  if (behind < n) p[behind] = 0.f;
}
// the gradient before anything is added up.  Without gaps between its rows a block writes one page of 4096 bytes, a thread 16 of them: the
// blocks that run at the same time then write next to each other, which is what memory takes fastest (2 GB: 6.8 TB/s; two pieces a
// thread 6.0, four 5.9, 64 KB a block 5.6, a row of 16 KB a wave 6.2 and of 6932 bytes 4.9)
constexpr int kPage = 4096;
constexpr int64_t kMostPages = 1 << 23;                    // of a worker (a launch has fewer than 2^32 threads a row); above by rows
struct ZeroArgs {
  float* grad; int64_t ld, stride, n;
  int block_rows;                                          // otherwise; 0: pages
  int64_t blocks;                                          // of a worker
};
__device__ __forceinline__ void zero_part(const ZeroArgs& a, int w, int64_t block, int64_t vocab) {
  float* grad = a.grad + w * a.stride;
  if (a.block_rows == 0) {
    const uintptr_t from = reinterpret_cast<uintptr_t>(grad), to = from + (uintptr_t)(vocab * a.n) * 4;
    const uintptr_t p = from / kPage * kPage + (uintptr_t)block * kPage + threadIdx.x * 16;
    if (p >= from && p + 16 <= to) {
      *reinterpret_cast<float4*>(p) = make_float4(0.f, 0.f, 0.f, 0.f);
    } else {
      for (uintptr_t q = p; q < p + 16; q += 4)
        if (q >= from && q < to) *reinterpret_cast<float*>(q) = 0.f;
    }
    return;
  }
  const int64_t v0 = block * a.block_rows, v1 = v0 + a.block_rows < vocab ? v0 + a.block_rows : vocab;
  for (int64_t v = v0 + (threadIdx.x >> 6); v < v1; v += 4) zero_floats(grad + v * a.ld, a.n);
}

// 16 places a block, each by 16 threads: the worker's keys go through LDS kRankTile at a time, and every thread compares its place's
// with a sixteenth of them, four to a read that a quarter of a wave shares.  Of keys before the block's an equal one counts, of
// those behind not; only a wave that has the block's own among its keys looks at where each stands.  The first blocks of a grid
// row are a worker's, or those of row 0 all workers' (in_first_row of them), the others write zeros.
__global__ __launch_bounds__(256) void rank_kernel(const int32_t* __restrict__ token, int32_t* __restrict__ sorted, int32_t* __restrict__ place, int rows,
                                                   int32_t vocab, int rank_blocks, int in_first_row, ZeroArgs zero) {
  __shared__ __align__(16) uint32_t keys[kRankTile];
  __shared__ int part[4][kRankPlaces];
  const uint32_t in_front = in_first_row == 0 ? (uint32_t)rank_blocks : blockIdx.y == 0 ? (uint32_t)in_first_row : 0u;
  if (blockIdx.x >= in_front) {
    if (blockIdx.x - in_front < zero.blocks) zero_part(zero, blockIdx.y, blockIdx.x - in_front, vocab);
    return;
  }
  const int w = in_first_row == 0 ? (int)blockIdx.y : (int)(blockIdx.x / (uint32_t)rank_blocks);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* tok = token + (int64_t)w * rows;
  const int r0 = ((int)blockIdx.x - (in_first_row == 0 ? 0 : w * rank_blocks)) * kRankPlaces, r = r0 + (lane & 15);
  const uint32_t last = (uint32_t)vocab;                   // (what is no token is behind it, also as an unsigned number below zero)
  auto key = [&](int s) {
    const uint32_t v = s < rows ? (uint32_t)tok[s] : ~0u;
    return s >= rows ? ~0u : v < last ? v : last;          // (none: above every key)
  };
  uint32_t next[kRankTile / 256];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < kRankTile / 256; ++i) next[i] = key(s0 + i * 256 + (int)threadIdx.x);
  };
  fetch(0);
  const uint32_t mine = r < rows ? key(r) : 0u;
  int rank = 0;
  for (int s0 = 0; s0 < rows; s0 += kRankTile) {
    __syncthreads();                                       // (the tile before has been read)
#pragma unroll
    for (int i = 0; i < kRankTile / 256; ++i) keys[i * 256 + threadIdx.x] = next[i];
    __syncthreads();
    if (s0 + kRankTile < rows) fetch(s0 + kRankTile);
    const int of_wave = s0 + wave * (kRankTile / 4), of_thread = wave * (kRankTile / 4) + (lane >> 4) * (kRankTile / 16);
    const uint4* four = reinterpret_cast<const uint4*>(keys + of_thread);
    if (r0 + kRankPlaces <= of_wave || r0 >= of_wave + kRankTile / 4) {
      const uint32_t limit = r0 > of_wave ? mine + 1u : mine;
#pragma unroll 8
      for (int i = 0; i < kRankTile / 64; ++i) {
        const uint4 k = four[i];
        rank += k.x < limit ? 1 : 0;
        rank += k.y < limit ? 1 : 0;
        rank += k.z < limit ? 1 : 0;
        rank += k.w < limit ? 1 : 0;
      }
    } else {
      const int before = r - (s0 + of_thread);             // of this thread's keys those below it stand before its place
#pragma unroll 4
      for (int i = 0; i < kRankTile / 64; ++i) {
        const uint4 k = four[i];
        rank += k.x < mine + (4 * i < before ? 1u : 0u) ? 1 : 0;
        rank += k.y < mine + (4 * i + 1 < before ? 1u : 0u) ? 1 : 0;
        rank += k.z < mine + (4 * i + 2 < before ? 1u : 0u) ? 1 : 0;
        rank += k.w < mine + (4 * i + 3 < before ? 1u : 0u) ? 1 : 0;
      }
    }
  }
  rank += __shfl_xor(rank, 16);
  rank += __shfl_xor(rank, 32);
  if (lane < kRankPlaces) part[wave][lane] = rank;
  __syncthreads();
  if (threadIdx.x >= kRankPlaces || r >= rows) return;
#pragma unroll
  for (int q = 1; q < 4; ++q) rank += part[q][lane];
  sorted[(int64_t)w * rows + rank] = (int32_t)mine;
  place[(int64_t)w * rows + rank] = r;
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
#pragma unroll
  for (int i = 0; i < kTile / 256; ++i) {
    const int64_t r = (int64_t)blockIdx.x * kTile + i * 256 + threadIdx.x;
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
  int32_t keys[16], places[16];                            // all on their way at once
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const int64_t r = r0 + i * 64 + lane;
    keys[i] = r < d.rows ? d.key(w, r) : 0;
    places[i] = d.token ? (int32_t)r : r < d.rows ? d.place_in[w * d.rows + r] : 0;
  }
#pragma unroll
  for (int q = 0; q < 4; ++q) next[q][threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i)
    if (r0 + i * 64 + lane < d.rows) atomicAdd(&next[wave][(uint32_t)keys[i] >> d.shift & 255u], 1u);
  __syncthreads();
  uint32_t at = d.count[((int64_t)w * 256 + threadIdx.x) * d.tiles + blockIdx.x];
#pragma unroll
  for (int q = 0; q < 4; ++q) { const uint32_t c = next[q][threadIdx.x]; next[q][threadIdx.x] = at; at += c; }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < 16; ++i) {
    const bool there = r0 + i * 64 + lane < d.rows;
    const int32_t key = keys[i];
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
      d.place_out[w * d.rows + to] = places[i];
    }
  }
}

// ---- sums ------------------------------------------------------------------------------------------------------------

struct SumArgs {
  EmbedGradArgs a;
  const int32_t* key; const int32_t* place;                // [k][rows], sorted
  float* part;                                             // [k][chunks][2][n]: of a token that came from the chunk before, and that goes on
  int64_t chunks;
  int log_tpr;                                             // threads of a chunk
  int slices;                                              // parts of a row by so many pieces
  int64_t piece_blocks;                                    // of a worker, for those; behind them the blocks for what is behind the whole pieces
  int log_join;                                            // threads of a row in the last kernel
  int64_t join_blocks;                                     // of a worker, in the last kernel; those behind them fill rows that no token has
  int fill_rows;                                           // of a block
};

// the sum of a token's rows in columns e0 .. e0+W-1, in the gradient or (part of it) in scratch
template <int W>
__device__ __forceinline__ void put_sum(const EmbedGradArgs& a, float* to, bool whole, const float (&s)[W]) {
  if constexpr (W == 1) {
    *to = whole ? (a.accumulate ? *to + s[0] * a.scale : s[0] * a.scale) : s[0];
  } else {
#pragma unroll
    for (int q = 0; q < W / 4; ++q) {
      float f[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) f[j] = whole ? s[4 * q + j] * a.scale : s[4 * q + j];
      if (whole && a.accumulate) {
        uint32_t old[4];
        load_piece<F32>(to + 4 * q, old);
#pragma unroll
        for (int j = 0; j < 4; ++j) f[j] += __uint_as_float(old[j]);
      }
      store_piece<F32>(to + 4 * q, f);
    }
  }
}

// A chunk's rows in columns e0 .. e0+W-1 (W: a piece, or one behind the whole pieces), `key` and `place` of it in LDS: key[-1] is the one
// before it, key[count] the one behind.  All rows are on their way before the first is added: memory operations of a wave are
// waited for in their order, so a load behind the write of a sum would wait for that too.
template <class E, int W>
__device__ __forceinline__ void sum_chunk(const SumArgs& s, int w, int64_t c, int count, const int32_t* key, const int32_t* place, int64_t e0) {
  const EmbedGradArgs& a = s.a;
  const typename E::T* dy = reinterpret_cast<const typename E::T*>(a.dy.p) + w * a.dy.stride + e0;
  float* grad = a.grad + w * a.grad_stride + e0;
  float* part = s.part + (w * s.chunks + c) * 2 * a.n + e0;
  if (key[0] >= a.vocab) return;                           // nothing but what is no token
  uint32_t raw[kChunk][W == 1 ? 1 : 4];
#pragma unroll
  for (int i = 0; i < kChunk; ++i) {
    const typename E::T* row = dy + place[i] * a.dy.ld;    // (behind the chunk's last the first row of all: in bounds, and not added)
    if constexpr (W == 1) raw[i][0] = __float_as_uint(E::one(row));
    else load_piece_once<E>(row, raw[i]);
  }
  float sum[W];
#pragma unroll
  for (int j = 0; j < W; ++j) sum[j] = 0.f;
  bool from_before = key[-1] == key[0];
#pragma unroll
  for (int i = 0; i < kChunk; ++i) {
    const int32_t now = key[i], next = key[i + 1];
    if (i >= count || now >= a.vocab) break;               // nothing but what is no token from here on
    if constexpr (W == 1) {
      sum[0] += __uint_as_float(raw[i][0]);
    } else {
      float f[W];
      E::unpack(raw[i], f);
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] += f[j];
    }
    if (i + 1 == count || next != now) {
      const bool whole = !from_before && next != now;
      put_sum<W>(a, whole ? grad + now * a.grad_ld : from_before ? part : part + a.n, whole, sum);
#pragma unroll
      for (int j = 0; j < W; ++j) sum[j] = 0.f;
      from_before = false;
    }
  }
}

// rows of the gradient that no token has: a thread looks for each among the sorted keys, then a wave writes it
__device__ __forceinline__ void fill_rows(const SumArgs& s, int w, int64_t v0, int32_t* present) {
  const EmbedGradArgs& a = s.a;
  const int32_t* key = s.key + w * a.rows;
  const int64_t v1 = v0 + s.fill_rows < a.vocab ? v0 + s.fill_rows : a.vocab;
  if (v0 + threadIdx.x < v1) {
    const int32_t v = (int32_t)(v0 + threadIdx.x);
    int64_t lo = 0, hi = a.rows;                           // the first key that is not below v lies in lo .. hi
    while (lo < hi) {
      const int64_t mid = (lo + hi) >> 1;
      if (key[mid] < v) lo = mid + 1;
      else hi = mid;
    }
    present[threadIdx.x] = lo < a.rows && key[lo] == v;
  }
  __syncthreads();
  for (int64_t v = v0 + (threadIdx.x >> 6); v < v1; v += 4)
    if (!present[v - v0]) zero_floats(a.grad + w * a.grad_stride + v * a.grad_ld, a.n);
}

constexpr int kLogFewest = 3, kFewestThreads = 1 << kLogFewest;                  // of a chunk, so that a block's places fit its LDS

template <class E>
__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs s) {
  constexpr int CHUNKS = 256 / kFewestThreads, KEYS = kChunk + 8;               // a key before and one behind, and whole pieces of LDS
  __shared__ __align__(16) int32_t key[CHUNKS * KEYS], place[CHUNKS * kChunk];
  const EmbedGradArgs& a = s.a;
  const int w = blockIdx.y;
  // the last blocks take the columns behind the whole pieces, fewest threads a chunk (4 x 16267 rows of 933, bf16: this
  // kernel 38 us, with as many as the others take 55; rows of 936 36)
  const bool behind = blockIdx.x >= s.piece_blocks;
  const int log_tpr = behind ? kLogFewest : s.log_tpr, slice = behind ? 0 : blockIdx.x % s.slices;
  const int t = threadIdx.x & ((1 << log_tpr) - 1), g = threadIdx.x >> log_tpr;
  const int64_t c = (int64_t)(behind ? blockIdx.x - s.piece_blocks : blockIdx.x / s.slices) * (256 >> log_tpr) + g, i0 = c * kChunk;
  const int count = i0 + kChunk < a.rows ? kChunk : (int)(a.rows - i0);         // (not positive: no chunk)
  int32_t* my_key = key + g * KEYS + 4;
  int32_t* my_place = place + g * kChunk;
  for (int i = t; i < kChunk + 2; i += 1 << log_tpr) {
    const int64_t at = i0 + i - 1;
    my_key[i - 1] = at >= 0 && at < a.rows ? s.key[w * a.rows + at] : -1;
    if (i < kChunk) my_place[i] = i < count ? s.place[w * a.rows + i0 + i] : 0;
  }
  __syncthreads();
  if (count <= 0) return;
  const int64_t whole = a.n / E::V;
  if (behind) {
    if (whole * E::V + t < a.n) sum_chunk<E, 1>(s, w, c, count, my_key, my_place, whole * E::V + t);
    return;
  }
  const int64_t q = ((int64_t)slice << s.log_tpr) + t;
  if (q < whole) sum_chunk<E, E::V>(s, w, c, count, my_key, my_place, q * E::V);
}

// tokens that go on from the chunk c they begin in, in 1024 columns: its partial sum and those of the chunks behind it.  Four columns a
// thread; where a row has fewer, several threads share them, each adds every so-manieth sum, and those are added in their order.
__device__ __forceinline__ void join(const SumArgs& s, int w, int64_t c, int64_t slice, float4* lds) {
  const EmbedGradArgs& a = s.a;
  const int32_t* key = s.key + w * a.rows;
  const int64_t i0 = c * kChunk, last = i0 + kChunk - 1;
  const int32_t v = key[last], behind = key[last + 1], first = key[i0], before = i0 > 0 ? key[i0 - 1] : -1;       // (a chunk follows)
  if (v >= a.vocab || behind != v || (first == v && before == v)) return;       // (or it began before)
  const int mine = threadIdx.x & ((1 << s.log_join) - 1), share = threadIdx.x >> s.log_join, shares = 256 >> s.log_join;
  const int64_t e0 = ((slice << s.log_join) + mine) * 4;
  const float* part = s.part + (w * s.chunks + c) * 2 * a.n;
  float sum[4] = {0.f, 0.f, 0.f, 0.f}, f[4];
  const int lane = threadIdx.x & 63;
  if (e0 < a.n && share == 0) load_floats<4>(part + a.n, e0, a.n, 0.f, sum);
  int64_t at = 1 + share;                                  // the next chunk (from c on) of this thread's
  for (int64_t q = 1; c + q < s.chunks; q += 64) {         // the next 64 chunks: in how many of them does it go on?
    const bool there = c + q + lane < s.chunks;
    const uint64_t not_mine = ~__ballot(there && key[(c + q + (there ? lane : 0)) * kChunk] == v);
    const int run = not_mine ? __builtin_ctzll(not_mine) : 64;
    if (e0 < a.n) {
#pragma unroll 4
      for (; at < q + run; at += shares) {
        load_floats<4>(part + at * 2 * a.n, e0, a.n, 0.f, f);
#pragma unroll
        for (int j = 0; j < 4; ++j) sum[j] += f[j];
      }
    }
    if (run < 64) break;
  }
  if (shares > 1) {                                        // (every thread of the block is here)
    lds[threadIdx.x] = make_float4(sum[0], sum[1], sum[2], sum[3]);
    __syncthreads();
    if (share > 0) return;
    for (int q = 1; q < shares; ++q) {
      const float4 more = lds[(q << s.log_join) + mine];
      sum[0] += more.x; sum[1] += more.y; sum[2] += more.z; sum[3] += more.w;
    }
  }
  if (e0 >= a.n) return;
  float* row = a.grad + w * a.grad_stride + v * a.grad_ld;
  if (e0 + 4 <= a.n) put_sum<4>(a, row + e0, true, sum);
  else
    for (int j = 0; j < 4; ++j) {
      const float one[1] = {sum[j]};
      if (e0 + j < a.n) put_sum<1>(a, row + e0 + j, true, one);
    }
}

__global__ __launch_bounds__(256) void embed_join_kernel(SumArgs s) {
  __shared__ float4 lds[256];
  const int w = blockIdx.y;
  const int64_t slices = ceil_div(s.a.n, 1024);
  if (blockIdx.x < s.join_blocks) join(s, w, blockIdx.x / slices, blockIdx.x % slices, lds);
  else fill_rows(s, w, (blockIdx.x - s.join_blocks) * s.fill_rows, reinterpret_cast<int32_t*>(lds));
}

// scratch: sorted keys and places, then (digits) the others of the two, and counts, then the partial sums
struct GradLayout {
  size_t key, place, key2, place2, count, part, total;
  int64_t tiles, chunks;
  bool digits;
  GradLayout(int k, int64_t rows, int64_t n) : tiles(ceil_div(rows, kTile)), chunks(ceil_div(rows, kChunk)) {
    size_t pos = 0;
    auto take = [&](size_t bytes) { const size_t at = pos; pos += (bytes + 255) / 256 * 256; return at; };
    const size_t list = (size_t)k * rows * 4;
    digits = (double)k * rows * rows > kRankWork;
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
hipError_t sums(SumArgs& s, hipStream_t stream) {
  const EmbedGradArgs& a = s.a;
  const int64_t whole = a.n / E::V;
  s.log_tpr = log_threads(whole);
  if (s.log_tpr < kLogFewest) s.log_tpr = kLogFewest;
  s.slices = (int)ceil_div(whole, 1 << s.log_tpr);
  s.piece_blocks = ceil_div(s.chunks, 256 >> s.log_tpr) * s.slices;
  const int64_t blocks = s.piece_blocks + (a.n % E::V ? ceil_div(s.chunks, 256 / kFewestThreads) : 0);
  hipLaunchKernelGGL(embed_sum_kernel<E>, dim3((unsigned)blocks, (unsigned)a.k), dim3(256), 0, stream, s);
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
  const GradLayout lay(a.k, a.rows, a.n);
  int32_t* key = reinterpret_cast<int32_t*>(a.scratch + lay.key);
  int32_t* place = reinterpret_cast<int32_t*>(a.scratch + lay.place);
  // The zeros: where at most a quarter of the rows can have a token, all rows beside the sort, page by page, and those few are written
  // once more; otherwise, where that would write up to all of them twice, at the end those that no token has, looked for one by one, at
  // most 256 KB a block, and four blocks a compute unit where there are as many rows (4 x 4096 rows of 4096 over 32000, the whole call: 374
  // us, the other way 434; 3 x 333 rows of 1001 over 5003: 20.0 and 20.8, and that 22.9 by 65 rows a block).
  const bool first = !a.accumulate && a.vocab / 4 >= a.rows, last = !a.accumulate && !first;
  const int64_t by_size = a.n >= 4096 ? 16 : a.n <= 256 ? 256 : 65536 / a.n, share = ceil_div(a.vocab * a.k, 4 * kCus);
  const int fill_rows = (int)(share < by_size ? share : by_size);
  const bool digits = lay.digits;
  const int rank_blocks = digits ? 0 : (int)ceil_div(a.rows, kRankPlaces);
  const int64_t pages = ceil_div(a.vocab * a.n * 4, kPage) + 1;                 // (one more: it may begin within one)
  const bool by_page = a.grad_ld == a.n && pages <= kMostPages;
  ZeroArgs zero = {a.grad, a.grad_ld, a.grad_stride, a.n, by_page ? 0 : fill_rows, 0};
  if (first) zero.blocks = by_page ? pages : ceil_div(a.vocab, fill_rows);
  const bool own_row = first && (double)a.k * a.vocab * a.n * 4.0 >= kOwnRowBytes;
  const int in_front = rank_blocks * (own_row ? 1 : a.k);
  if (in_front + zero.blocks > 0) {
    hipLaunchKernelGGL(rank_kernel, dim3((unsigned)(in_front + zero.blocks), (unsigned)(own_row || zero.blocks > 0 ? a.k : 1)), dim3(256), 0, s, a.token, key,
                       place, digits ? 0 : (int)a.rows, (int32_t)a.vocab, rank_blocks, own_row ? 0 : in_front, zero);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  if (digits) {
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
  SumArgs sum = {};
  sum.a = a;
  sum.key = key;
  sum.place = place;
  sum.part = reinterpret_cast<float*>(a.scratch + lay.part);
  sum.chunks = lay.chunks;
  if (a.rows > 0 && (e = dtype == DW_BF16 ? sums<Bf16>(sum, s) : sums<F32>(sum, s)) != hipSuccess) return e;
  sum.log_join = log_threads(ceil_div(a.n, 4));
  sum.join_blocks = lay.chunks > 1 ? (lay.chunks - 1) * ceil_div(a.n, 1024) : 0;
  sum.fill_rows = fill_rows;
  const int64_t blocks = sum.join_blocks + (last ? ceil_div(a.vocab, fill_rows) : 0);
  if (blocks == 0) return e;
  hipLaunchKernelGGL(embed_join_kernel, dim3((unsigned)blocks, (unsigned)a.k), dim3(256), 0, s, sum);
  return hipGetLastError();
}

}  // namespace dw
