// Numbers in e4m3 with one power-of-two scale per block of 128 (gfx950, wave64).
//
// A block of 128 along a row (square: of 128 x 128) with largest magnitude m gets the least e with m <= 448 2^e (448 is
// the largest number of e4m3), its elements are x 2^-e rounded to nearest, ties to even, and the scale is kept as the byte
// e + 127 (at least 1).  2^-e is a power of two, so the product is exact and the only rounding is that to e4m3; e follows
// from the bits of m: m = 1.f 2^E and 448 = 1.75 2^8, so e = E - 8, and one more where f > 0.75.  The largest magnitude is
// found on the bits as integers, where a NaN is above infinity and infinity above the rest: a block with one of them is all NaN.
//
// Rows alone: 16 lanes share a block, 8 elements each, one pass from registers.  With the transposed form or squares a
// block of 512 threads takes a tile of 128 x 128, 4 rows x 8 columns a thread; the transposed bytes leave through LDS so that
// both forms are written in whole lines while x is read once.  Bound by memory when there is much of it: 16 x 512 rows of 4096,
// bf16, 20.5 us = 4.9 TB/s; 4 x 2048 x 4096 in both forms 36 us = 3.7 TB/s, squares of 4 x 4096 x 4096 62 us = 4.3 TB/s.
#include "dw_fp8.h"

namespace dw {

namespace {

template <class E>
__global__ __launch_bounds__(256) void quantize_rows_kernel(QuantArgs a) {
  const int w = blockIdx.z, t = threadIdx.x & 15;
  const int64_t b = blockIdx.x;                             // block of 128 along the row
  const int64_t r = (int64_t)(a.first + blockIdx.y) * 16 + (threadIdx.x >> 4);
  const int64_t np = DW_FP8_ROW(a.n), ns = DW_FP8_SCALES(a.n);
  if (r >= a.rows) return;                                  // (16 lanes at once: those that exchange values stay together)
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride + r * a.x.ld;
  float f[8];
  Raw8<E> raw;
  raw.load(x, b * 128 + t * 8, a.n);
  raw.floats(f);
  uint32_t top = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) top = larger(top, magnitude(f[j]));
  const Scale s = scale_of(largest_of_16(top));
  const int64_t row = w * a.rows + r;
  *reinterpret_cast<uint2*>(a.q + row * np + b * 128 + t * 8) = to_e4m3(f, s.inverse);
  uint8_t* sc = a.scale + row * ns;
  if (t == 0) sc[b] = (uint8_t)s.byte;
  if (b == np / 128 - 1 && b + 1 + t < ns) sc[b + 1 + t] = 127;       // a row's scales fill whole words
}

constexpr int kTileThreads = 512, kRows = 4;                // rows of a thread

// NORM: the numbers are x rstd gamma, a root-mean-square norm whose rows' factors are known (multiplied anew where they are used
// next, like the unpacking), and the transposed form alone is wanted.  Four blocks on a unit then, within 64 registers: what one waits
// for the others fill (8 x 1024 x 4096 bf16: 21 us, with two 27).  In fp32 three, within 80, seven of which are in memory: 40 us, 4.2 TB/s
template <class E, bool SQUARE, bool NORM>
__global__ __launch_bounds__(kTileThreads, NORM ? (E::V == 8 ? 8 : 6) : 1) void quantize_tile_kernel(QuantArgs a) {
  constexpr int WAVES = kTileThreads / 64;
  __shared__ uint32_t tops[WAVES][128];
  __shared__ __align__(16) uint32_t tile[128][32];          // transposed bytes: [column][four rows, swizzled]
  int w = blockIdx.z;
  if ((int)gridDim.z > a.k) {                               // few tiles: one block for each form
    if (w >= a.k) { w -= a.k; a.q = nullptr; } else a.qt = nullptr;
  }
  const int64_t c0 = (int64_t)blockIdx.x * 128, r0 = (int64_t)(a.first + blockIdx.y) * 128;
  const int tc = threadIdx.x & 15, tr = threadIdx.x >> 4;   // this thread's 8 columns from 8 tc, 4 rows from 4 tr
  const int wave = threadIdx.x >> 6;
  const int64_t np = DW_FP8_ROW(a.n), ns = DW_FP8_SCALES(a.n), rp = DW_FP8_ROW(a.rows), rs = DW_FP8_SCALES(a.rows);
  const typename E::T* x = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
  Raw8<E> raw[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int64_t r = r0 + tr * kRows + i;
    if (r < a.rows) raw[i].load(x + r * a.x.ld, c0 + tc * 8, a.n);
    else raw[i].zero();
  }
  float by_row[kRows], by_col[8];
#pragma unroll
  for (int i = 0; i < kRows; ++i) by_row[i] = NORM && r0 + tr * kRows + i < a.rows ? a.rstd[w * a.rows + r0 + tr * kRows + i] : 1.f;
#pragma unroll
  for (int j = 0; j < 8; ++j) by_col[j] = 1.f;
  if constexpr (NORM)
    if (a.gamma) load_floats<8>(a.gamma + w * a.gamma_stride, c0 + tc * 8, a.n, 0.f, by_col);
  auto values = [&](int i, float (&f)[8]) {
    raw[i].floats(f);
    if constexpr (NORM) {
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = f[j] * by_row[i] * by_col[j];
    }
  };
  // (what fills the last block is +0 whatever gamma's sign)
  auto one = [&](int i, int j) {
    if constexpr (NORM) return r0 + tr * kRows + i < a.rows ? raw[i].one(j) * by_row[i] * by_col[j] : 0.f;
    else return raw[i].one(j);
  };
  uint32_t row_top[kRows], col_top[8];
#pragma unroll
  for (int i = 0; i < kRows; ++i) row_top[i] = 0;
#pragma unroll
  for (int j = 0; j < 8; ++j) col_top[j] = 0;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    float f[8];
    values(i, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t m = magnitude(f[j]);
      if constexpr (!NORM) row_top[i] = larger(row_top[i], m);
      col_top[j] = larger(col_top[j], m);
    }
    raw[i].keep_packed();
  }
  Scale all = {127u, 1.f};
  if constexpr (SQUARE) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < kRows; ++i) m = larger(m, row_top[i]);
    m = largest_of_16(m);
    if (tc == 0) tops[0][tr] = m;
    __syncthreads();
    m = 0;
#pragma unroll
    for (int q = 0; q < kTileThreads / 16; ++q) m = larger(m, tops[0][q]);
    all = scale_of(m);
  }
  if (!NORM && a.q) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const Scale s = SQUARE ? all : scale_of(largest_of_16(row_top[i]));
      const int64_t r = r0 + tr * kRows + i;
      if (r < a.rows) {
        const int64_t row = w * a.rows + r;
        float f[8];
        values(i, f);
        *reinterpret_cast<uint2*>(a.q + row * np + c0 + tc * 8) = to_e4m3(f, s.inverse);
        uint8_t* sc = a.scale + row * ns;
        if (tc == 0) sc[blockIdx.x] = (uint8_t)s.byte;
        if (blockIdx.x == gridDim.x - 1 && blockIdx.x + 1 + tc < ns) sc[blockIdx.x + 1 + tc] = 127;
      }
    }
  }
  if (!a.qt) return;
  __shared__ float inverse[128];
  Scale mine = all;                                         // of column threadIdx.x, for the first 128 threads
  if constexpr (!SQUARE) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {                           // over the wave's rows, then over the waves
      uint32_t m = col_top[j];
      m = larger(m, (uint32_t)__shfl_xor((int)m, 16));
      m = larger(m, (uint32_t)__shfl_xor((int)m, 32));
      if ((tr & 3) == 0) tops[wave][tc * 8 + j] = m;
    }
    __syncthreads();
    if (threadIdx.x < 128) {
      uint32_t m = 0;
#pragma unroll
      for (int q = 0; q < WAVES; ++q) m = larger(m, tops[q][threadIdx.x]);
      mine = scale_of(m);
      inverse[threadIdx.x] = mine.inverse;
    }
    __syncthreads();
  }
#pragma unroll
  for (int i = 0; i < kRows; ++i) raw[i].keep_packed();
  // Word tr of a column goes to place tr ^ 4 (tc mod 8): the lanes of a wave, 16 columns 8 apart and 4 words, then spread
  // over the banks, and pieces of 16 bytes stay whole.
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const float inv = SQUARE ? all.inverse : inverse[tc * 8 + j];
    int v = 0;
    v = __builtin_amdgcn_cvt_pk_fp8_f32(one(0, j) * inv, one(1, j) * inv, v, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(one(2, j) * inv, one(3, j) * inv, v, true);
    tile[tc * 8 + j][tr ^ ((tc & 7) << 2)] = (uint32_t)v;
  }
  __syncthreads();
#pragma unroll
  for (int p = 0; p < 128 * 8 / kTileThreads; ++p) {        // 8 threads a column, 16 rows each
    const int c = p * (kTileThreads / 8) + (threadIdx.x >> 3), at = threadIdx.x & 7;
    if (c0 + c < a.n)
      *reinterpret_cast<uint4*>(a.qt + (w * a.n + c0 + c) * rp + r0 + at * 16) =
          *reinterpret_cast<const uint4*>(&tile[c][(at ^ ((c >> 3) & 7)) * 4]);
  }
  if (threadIdx.x < 128 && c0 + threadIdx.x < a.n) {
    uint8_t* sc = a.scale_t + (w * a.n + c0 + threadIdx.x) * rs;
    const uint32_t b = a.first + blockIdx.y;
    sc[b] = (uint8_t)mine.byte;
    if (b == (uint32_t)(rp / 128) - 1)
      for (int64_t q = b + 1; q < rs; ++q) sc[q] = 127;
  }
}

// A grid has at most 65535 blocks along y: more blocks of `high` rows are several launches
template <class F>
hipError_t by_rows(QuantArgs a, int64_t high, F launch) {
  constexpr uint32_t kMost = 65535;
  const uint32_t blocks = (uint32_t)ceil_div(a.rows, high);
  for (a.first = 0; a.first < blocks; a.first += kMost) {
    launch(a, blocks - a.first < kMost ? blocks - a.first : kMost);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <class E>
hipError_t quantize(const QuantArgs& all, hipStream_t s) {
  const unsigned columns = (unsigned)(DW_FP8_ROW(all.n) / 128);
  if (!all.square && !all.qt)
    return by_rows(all, 16, [&](const QuantArgs& a, unsigned blocks) {
      hipLaunchKernelGGL(quantize_rows_kernel<E>, dim3(columns, blocks, (unsigned)a.k), dim3(256), 0, s, a);
    });
  // Both forms of at most a tile a compute unit: a block for each form, which shares the work among twice as many (us, one
  // block for both and a block for each; 3 x 333 x 784 fp32, 63 tiles: 6.1, 5.1; 3 x 1000 x 784, 168: 7.1, 6.6; 1 x 64 x 4096 bf16,
  // 32: 5.5, 4.5; 2 x 1500 x 1500, 288: 10.3, 9.0 and in fp32 10.7, 11.2; 1 x 2048 x 4096, 512: 10.7, 10.3 and 12.8, 16.3)
  const int64_t tiles = DW_FP8_ROW(all.n) / 128 * (DW_FP8_ROW(all.rows) / 128) * all.k;
  const int forms = all.q && all.qt && tiles <= kCus ? 2 : 1;
  return by_rows(all, 128, [&](const QuantArgs& a, unsigned blocks) {
    const dim3 grid(columns, blocks, (unsigned)(a.k * forms));
    if (a.rstd) hipLaunchKernelGGL((quantize_tile_kernel<E, false, true>), grid, dim3(kTileThreads), 0, s, a);
    else if (a.square) hipLaunchKernelGGL((quantize_tile_kernel<E, true, false>), grid, dim3(kTileThreads), 0, s, a);
    else hipLaunchKernelGGL((quantize_tile_kernel<E, false, false>), grid, dim3(kTileThreads), 0, s, a);
  });
}

}  // namespace

hipError_t launch_fp8_quantize(const QuantArgs& a, int dtype, hipStream_t s) {
  return dtype == DW_BF16 ? quantize<Bf16>(a, s) : quantize<F32>(a, s);
}

}  // namespace dw
