// Products of e4m3 matrices with a power-of-two scale per row and block of 128 along the contraction (gfx950, wave64).
//
//   C[m][n] = sum over blocks b of 2^(sa[m][b] + sb[n][b]) sum over k in b of a[m][k] b[n][k]   (+ bias[n])
//
// v_mfma_scale_f32_32x32x64_f8f6f4 multiplies 32 x 64 by 64 x 32 numbers of 8 bits and applies both scales (one byte per
// row and 32 numbers) by itself, so scaled blocks cost no more than unscaled ones and are accumulated in fp32 throughout.
// The contraction runs in blocks of 128, two steps of 64 each: a tile of BM + BN rows of 128 bytes, whole lines, goes from
// memory straight to LDS (global_load_lds, 16 bytes a lane), the next blocks are in flight, and every wave reads the operands
// of the next step from LDS while it multiplies the present one.  Rows lie back to back, so the 16-byte piece q of row r
// is kept in slot q ^ (r/2 mod 8): the 16 lanes that read at a time then touch all banks once.  A row's scales for 512
// numbers are one word; words go through LDS too, four blocks at a time.
//
// That instruction adds eight neighbouring products at a time and keeps their bits down to 2^-13 of the largest one's power
// (measured; all 8-bit matrix instructions of this chip do).  On normally distributed numbers the sums are then off by
// 1.4e-5 of their size, on numbers with one in a hundred a hundred times larger by 7e-5: a fraction of a percent of an
// output's rounding to bf16 (2e-3), but not fp32.  So outputs in fp32 take another way (EXACT): the same bytes are turned
// into bf16, scale and all, by one instruction for two numbers and multiplied by v_mfma_f32_32x32x16_bf16 at half the rate, whose
// sums are right to 24 bits.  The quantiser's largest number is 2^128 (what the lowest value of fp32 or bf16, a usual mask, is
// rounded to), which bf16 does not hold: both operands are widened at half their size, and the sums are multiplied by four at
// the end.  That is exact down to scales of 2^-123; below, numbers count in steps of 2^-132, which is twice bf16's smallest.
//
// Operand A of the instruction is the matrix b and operand B is a: a lane then holds one row of C and groups of four
// consecutive columns, which leave through a piece of LDS of the wave's own as whole row pieces of 16 bytes a lane.
// The accumulators start from the bias.  Rows past the end of a matrix repeat the last one; what they give is not written.
//
// 8192 cubed: 384 us = 2860 TFLOP/s (fp32 730 us = 1510); 4096 cubed: 56 us = 2480 (106 us = 1290).  16 x 512 x 4096 x 4096: 134 us =
// 2050, where b alone is 268 MB and comes from memory in pieces of 128 bytes (8 workers, b in the chip's cache: 55 us = 2520).
// What bounds a large product is power: of a block of 128 in a tile of 256 x 256 the matrix instructions take 0.85 us, with
// zeros for numbers the kernel takes 1.2 and with random ones 1.5, at a lower clock.  Tiles that load their successor while
// they are written, loads further ahead and shorter rows in more stages change nothing.
#include <type_traits>
#include <utility>

#include "dw_fp8.h"

namespace dw {

namespace fp8 {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) const char* lds_char;

constexpr int BK = 128, GROUP = 4;                          // bytes of a block, blocks per word of scales

// at most N vector-memory operations of this wave outstanding (N < 64), its LDS reads all returned
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (0x7 << 4) | (0x0 << 8));
}

// an index that the compiler takes as it is: it computes what follows from it where that is used and finds the constant parts
// of addresses, instead of keeping an address per use in registers
__device__ __forceinline__ int anew(int x) {
  asm volatile("" : "+v"(x));
  return x;
}

// Each lane's N bytes at base + offset go to LDS at `to` + N * lane; no register receives anything.  Written as assembly
// because behind the builtin the compiler waits for every load in flight before each read of LDS: it cannot tell that the
// read is of another stage.  The waits are the kernel's own (wait_vm before the barrier that precedes a stage's reads).
// m0 holds the place in LDS; nothing else in these kernels uses it.
template <int N>
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t offset, uint32_t to) {
#if defined(__HIP_DEVICE_COMPILE__)                          // (the host's pass does not know the constraint "s")
  if constexpr (N == 16) asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(to), "v"(offset), "s"(base));
  else asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(to), "v"(offset), "s"(base));
#endif
}

// f(0) .. f(N - 1) with the index as a constant: the products of a step and what is dealt out among them have to unroll
template <int FROM, int... I, class F>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) { (f(std::integral_constant<int, FROM + I>{}), ...); }
template <int FROM, int TO, class F>
__device__ __forceinline__ void each(F f) { each_of<FROM>(std::make_integer_sequence<int, (TO > FROM ? TO - FROM : 0)>{}, f); }

// an address that is the same in all lanes, in scalar registers
__device__ __forceinline__ const uint8_t* uniform(const uint8_t* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  return reinterpret_cast<const uint8_t*>((uint64_t)hi << 32 | lo);
}

template <int WTM_, int WTN_, int WM_, int WN_, int PER_CU_, int STAGES_, int LATE_8THS_>
struct Config {
  static constexpr int LATE_8THS = LATE_8THS_;              // eighths of a block's loads that are put off by a step
  static constexpr int WTM = WTM_, WTN = WTN_, WM = WM_, WN = WN_, PER_CU = PER_CU_, STAGES = STAGES_;
  static constexpr int NW = WM * WN, NT = NW * 64;
  static constexpr int BM = WM * WTM * 32, BN = WN * WTN * 32;
  static constexpr int A_B = BM * BK, STAGE_B = (BM + BN) * BK;
  static constexpr int CPW = STAGE_B / 1024 / NW;           // 1 KB pieces a wave moves per block
  static constexpr int OFF_S = STAGE_B * STAGES;            // two groups of scale words, (BM + BN) each
  static constexpr int LDS = OFF_S + 2 * (BM + BN) * 4;
  static_assert(STAGE_B % (1024 * NW) == 0 && BM % 64 == 0 && BN % 64 == 0, "whole pieces");
  static_assert(BM == BN && NW % 2 == 0, "half of the waves load A's tile, the others B's");
  static_assert(STAGES >= 2 && STAGES <= GROUP && (STAGES & (STAGES - 1)) == 0, "a group of scales is read before it is loaded anew");
};

__device__ __forceinline__ int swizzle(int row) { return (row >> 1) & 7; }

// eight numbers of 8 bits as bf16, times 2^(scale - 127)
__device__ __forceinline__ bf16x8 widen(int lo, int hi, float scale) {
  struct { bf16x2_t v[4]; } r;
  r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false);
  r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true);
  r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false);
  r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true);
  return __builtin_bit_cast(bf16x8, r);
}
// half of 2^(byte - 127), which is what a number is widened with, and what that makes of the product of two (the conversion
// takes the power from the exponent's bits: 2^-127 for a zero)
__device__ __forceinline__ float half_power(int byte) { return __uint_as_float(((unsigned)byte - 1u) << 23); }
constexpr float kWidened = 0.25f;

template <class C, bool EXACT, bool SLICE>
__global__ __launch_bounds__(C::NT, C::PER_CU) void gemm_fp8_kernel(Fp8Args a) {
  const int tiles_m = (int)((a.m + C::BM - 1) / C::BM), tiles_n = (int)((a.n + C::BN - 1) / C::BN);
  const int tiles = tiles_m * tiles_n;
  // consecutive blocks go to the eight dies in turn: each die gets a run of neighbouring tiles
  const int per_xcd = gridDim.x >> 3;
  const int logical = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
  const int w = logical / tiles, tile = logical - w * tiles;
  if (w >= a.k) return;
  // of a worker's tiles eight rows at a time: what a die works on is about as high as wide, and its L2 is read for fewer
  // rows of a and b (8192 cubed: 433 us with whole columns one after another, 394 so; 4096 x 512 x 4096: 22, 15.3)
  const int strip = tile / (8 * tiles_n), in_strip = tile - strip * 8 * tiles_n;
  const int high = tiles_m - strip * 8 < 8 ? tiles_m - strip * 8 : 8;
  const int64_t row0 = (int64_t)(strip * 8 + in_strip % high) * C::BM, col0 = (int64_t)(in_strip / high) * C::BN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave % C::WM) * C::WTM * 32, wn0 = (wave / C::WM) * C::WTN * 32;
  const int l32 = lane & 31, half = lane >> 5;

  extern __shared__ __attribute__((aligned(1024))) char smem[];

  const int64_t kp = a.kp;
  const uint8_t* A = a.a + w * a.m * kp;
  const uint8_t* Bm = a.b + w * a.n * kp;
  const uint8_t* sA = a.sa + w * a.m * a.ks;
  const uint8_t* sB = a.sb + w * a.n * a.ks;
  // blocks of 128 of this tile: all, or one slice of the contraction (slices begin at whole words of scales)
  const int all_blocks = (int)(kp / BK);
  const int block0 = SLICE ? (int)blockIdx.y * a.slice_blocks : 0;
  const int blocks = SLICE ? (all_blocks - block0 < a.slice_blocks ? all_blocks - block0 : a.slice_blocks) : all_blocks;

  // Workers begin at different blocks of the contraction (whole words of scales): the dies, each at a worker of its own, would
  // otherwise ask for the same columns of long rows at once, which lie in few channels of the memory.  (us, without and with:
  // 16 x 512 x 4096 x 4096: 146, 139; 16 x 256 x 4096 x 4096: 89, 80.  In tiles of 128 two of three shapes got slower by 3 and 8 %.)
  const int turn = SLICE || C::BM < 256 || blocks % GROUP ? 0 : w % (blocks / GROUP) * GROUP;
  auto place = [&](int b) { return b + turn < blocks ? b + turn : b + turn - blocks; };

  // The pieces this wave moves: the first half of the waves A's tile, the others B's; piece c holds rows 8c .. 8c+7.  A
  // uniform base that advances by a block, and a lane's offset from it (a tile's rows span less than 2^32 bytes).
  const bool of_a = wave < C::NW / 2;
  const int first = (of_a ? wave : wave - C::NW / 2) * C::CPW;
  const int64_t tile0 = of_a ? row0 : col0, behind = (of_a ? a.m : a.n) - 1 - tile0;
  const int last = behind < C::BM ? (int)behind : C::BM - 1;
  const uint8_t* base = (of_a ? A : Bm) + tile0 * kp + (int64_t)block0 * BK;
  uint32_t off[C::CPW];
#pragma unroll
  for (int c = 0; c < C::CPW; ++c) {
    const int row = (first + c) * 8 + (lane >> 3), q = (lane & 7) ^ swizzle(row);
    off[c] = (uint32_t)(row < last ? row : last) * (uint32_t)kp + (uint32_t)q * 16;
  }
  // scale words, 64 rows at a time: the same halves
  constexpr int SP = C::BM / 64, SPW = (SP + C::NW / 2 - 1) / (C::NW / 2);
  const int sfirst = of_a ? wave : wave - C::NW / 2;
  const uint8_t* sbase = (of_a ? sA : sB) + tile0 * a.ks + block0;
  uint32_t soff[SPW];
#pragma unroll
  for (int c = 0; c < SPW; ++c) {
    const int row = (sfirst + c * (C::NW / 2)) * 64 + lane;
    soff[c] = (uint32_t)(row < last ? row : last) * (uint32_t)a.ks;
  }
  const uint32_t lds0 = (uint32_t)(uintptr_t)(lds_char)smem;
  const uint32_t lds_tile = __builtin_amdgcn_readfirstlane(lds0 + (of_a ? 0 : C::A_B) + first * 1024);
  const uint32_t lds_scale = __builtin_amdgcn_readfirstlane(lds0 + C::OFF_S + (of_a ? 0 : C::BM * 4));
  auto issue = [&](const uint8_t* from, int b, int c) { load_to_lds<16>(from, off[c], lds_tile + (b & (C::STAGES - 1)) * C::STAGE_B + c * 1024); };
  auto issue_scales = [&](int g) {
    const uint8_t* from = uniform(sbase + place(g * GROUP));
#pragma unroll
    for (int c = 0; c < SPW; ++c)
      if (sfirst + c * (C::NW / 2) < SP)
        load_to_lds<4>(from, soff[c], lds_scale + (g & 1) * (C::BM + C::BN) * 4 + (sfirst + c * (C::NW / 2)) * 256);
  };

  f32x16 acc[C::WTM][C::WTN];
#pragma unroll
  for (int j = 0; j < C::WTN; ++j) {
    f32x16 start;
#pragma unroll
    for (int r = 0; r < 16; ++r) start[r] = 0.f;
    if (!SLICE && a.bias) {                                  // register r of a lane is column 8 (r/4) + 4 half + r%4 of the tile
      const float* bias = a.bias + w * a.bias_stride;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int64_t n = col0 + wn0 + j * 32 + (r >> 2) * 8 + half * 4 + (r & 3);
        start[r] = bias[n < a.n ? n : a.n - 1];
      }
    }
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) acc[i][j] = start;
  }

  // the 32 numbers of a lane's half of a step, for each row of the wave's tile; read in halves of 16
  struct Frags { uint4 x[C::WTM][2], y[C::WTN][2]; };
  constexpr int READS = 2 * (C::WTM + C::WTN);
  uint32_t at_x[4], at_y[4];                                 // where row 0 of the lane's rows lies in a stage, by step and half
#pragma unroll
  for (int u = 0; u < 4; ++u) {                              // (rows 32 apart are swizzled alike)
    const int q = (u >> 1) * 4 + half * 2 + (u & 1);
    at_x[u] = (wm0 + l32) * BK + ((q ^ swizzle(wm0 + l32)) << 4);
    at_y[u] = C::A_B + (wn0 + l32) * BK + ((q ^ swizzle(wn0 + l32)) << 4);
  }
  auto read_one = [&](Frags& f, int b, int sub, int r) {     // step `sub` of block b
    const char* stage = smem + (b & (C::STAGES - 1)) * C::STAGE_B;
    const int h = EXACT ? r / (READS / 2) : r & 1, i = EXACT ? r % (READS / 2) : r >> 1;    // (EXACT: what is widened first)
    if (i < C::WTM) f.x[i][h] = *reinterpret_cast<const uint4*>(stage + at_x[sub * 2 + h] + i * 32 * BK);
    else f.y[i - C::WTM][h] = *reinterpret_cast<const uint4*>(stage + at_y[sub * 2 + h] + (i - C::WTM) * 32 * BK);
  };
  int sx[C::WTM], sy[C::WTN], nx[C::WTM], ny[C::WTN];        // scale bytes: of the present block of 128, of the next
  auto read_scales = [&](int blk) {
    const uint8_t* bytes = reinterpret_cast<const uint8_t*>(smem) + C::OFF_S;
    const int group = ((blk / 4) & 1) * (C::BM + C::BN) * 4 + (blk & 3), lane4 = l32 * 4;
    const int ox = anew(group + wm0 * 4 + lane4), oy = anew(group + (C::BM + wn0) * 4 + lane4);
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) nx[i] = bytes[ox + i * 128];
#pragma unroll
    for (int j = 0; j < C::WTN; ++j) ny[j] = bytes[oy + j * 128];
  };
  auto take_scales = [&]() {
#pragma unroll
    for (int i = 0; i < C::WTM; ++i) sx[i] = nx[i];
#pragma unroll
    for (int j = 0; j < C::WTN; ++j) sy[j] = ny[j];
  };
  // what multiplies operand row i of a by row j of b: both halves at once, or (EXACT) eight numbers, q of four, widened before
  auto whole = [](const uint4 (&v)[2]) {
    const i32x8 r = {(int)v[0].x, (int)v[0].y, (int)v[0].z, (int)v[0].w, (int)v[1].x, (int)v[1].y, (int)v[1].z, (int)v[1].w};
    return r;
  };
  auto eight = [](const uint4 (&v)[2], int q, int scale) {
    const uint4 u = v[q >> 1];
    return q & 1 ? widen((int)u.z, (int)u.w, half_power(scale)) : widen((int)u.x, (int)u.y, half_power(scale));
  };
  struct Wide { bf16x8 x[C::WTM], y[C::WTN]; };
  auto widen_one = [&](Wide& d, const Frags& f, int q, int i, const int (&x)[C::WTM], const int (&y)[C::WTN]) {
    if (i < C::WTM) d.x[i] = eight(f.x[i], q, x[i]);
    else d.y[i - C::WTM] = eight(f.y[i - C::WTM], q, y[i - C::WTM]);
  };
  constexpr int Q = EXACT ? 4 : 1, PRODUCTS = C::WTM * C::WTN * Q, OPERANDS = C::WTM + C::WTN;
  Wide wide[2];                                              // EXACT: the present quarter of a step, and the next or the next step's first

  issue_scales(0);
#pragma unroll
  for (int b = 0; b < C::STAGES; ++b)
    if (b < blocks) {
      const uint8_t* from = uniform(base + (int64_t)place(b) * BK);
#pragma unroll
      for (int c = 0; c < C::CPW; ++c) issue(from, b, c);
    }
  if (blocks >= C::STAGES) wait_vm<C::CPW * (C::STAGES - 1)>();
  else wait_vm<0>();
  __syncthreads();
  Frags f0, f1;
  read_scales(0);
  take_scales();
#pragma unroll
  for (int r = 0; r < READS; ++r) read_one(f0, 0, 0, r);
  if constexpr (EXACT) {
    if (!SLICE && a.bias) {                                  // (not where it is read: that would wait for it before the first loads)
#pragma unroll
      for (int i = 0; i < C::WTM; ++i)
#pragma unroll
        for (int j = 0; j < C::WTN; ++j)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] *= kWidened;
    }
#pragma unroll
    for (int i = 0; i < OPERANDS; ++i) widen_one(wide[0], f0, 0, i, sx, sy);
  }

  // Step SUB of block b: its operands are in registers.  The second step opens with a barrier: every wave has then read all
  // of block b, whose stage is loaded anew, and block b + 1 has arrived (the counts leave the blocks behind it in flight;
  // loads of scale words, which are not counted, only make a wait longer).  Loads and reads are dealt out among the products
  // and kept there: the waves come from the barrier together, and a load put in front of the products would hold them all up.
  // The last LATE pieces of a block are loaded in the first half of the step behind the barrier's.
  constexpr int LATE = C::CPW * C::LATE_8THS / 8;
  auto step = [&](Frags& now, Frags& next, int b, auto more, auto sub) {
    constexpr bool MORE = decltype(more)::value;             // SUB 1: block b + STAGES exists; SUB 0: b - 1 + STAGES does, and b > 0
    constexpr int SUB = decltype(sub)::value;
    if constexpr (SUB == 1) {
      if constexpr (MORE) wait_vm<C::CPW * (C::STAGES - 2)>();
      else wait_vm<0>();
      __syncthreads();
      if constexpr (MORE) {
        if (((b + C::STAGES) & (GROUP - 1)) == 0) issue_scales((b + C::STAGES) / GROUP);
      }
    }
    const bool reads = SUB == 0 || MORE || b + 1 < blocks;
    const int loads = SUB == 1 ? b : b - 1;                  // whose stage is loaded anew
    const uint8_t* from = uniform(base + (int64_t)place(loads + C::STAGES) * BK);
    __builtin_amdgcn_sched_barrier(0);
    each<0, PRODUCTS>([&](auto p_) {
      constexpr int PN = C::WTM * C::WTN, p = decltype(p_)::value, q = p / PN, ij = p % PN, i = ij / C::WTN, j = ij % C::WTN;
      if constexpr (EXACT) {
        acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wide[q & 1].y[j], wide[q & 1].x[i], acc[i][j], 0, 0, 0);
        if constexpr (q + 1 < Q)
          each<ij * OPERANDS / PN, (ij + 1) * OPERANDS / PN>([&](auto o) { widen_one(wide[(q + 1) & 1], now, q + 1, o, sx, sy); });
      } else {
        acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(whole(now.y[j]), whole(now.x[i]), acc[i][j], 0, 0, 0, sy[j], 0, sx[i]);
      }
      if constexpr (MORE && SUB == 1) {
        each<p * (C::CPW - LATE) / PRODUCTS, (p + 1) * (C::CPW - LATE) / PRODUCTS>([&](auto c) { issue(from, loads, c); });
      } else if constexpr (MORE) {
        constexpr int HALF = PRODUCTS < 2 ? 1 : PRODUCTS / 2, at = p < HALF ? p : HALF, to = p + 1 < HALF ? p + 1 : HALF;
        each<C::CPW - LATE + at * LATE / HALF, C::CPW - LATE + to * LATE / HALF>([&](auto c) { issue(from, loads, c); });
      }
      if (reads) {
        each<p * READS / PRODUCTS, (p + 1) * READS / PRODUCTS>([&](auto r) { read_one(next, b + SUB, 1 - SUB, r); });
        if constexpr (SUB == 1 && p == (EXACT ? 0 : PRODUCTS / 2)) read_scales(b + 1);
        if constexpr (EXACT && q == Q - 1)
          each<ij * OPERANDS / PN, (ij + 1) * OPERANDS / PN>([&](auto o) {
            if constexpr (SUB == 1) widen_one(wide[0], next, 0, o, nx, ny);
            else widen_one(wide[0], next, 0, o, sx, sy);
          });
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    if constexpr (SUB == 1) take_scales();
  };
  using yes = std::true_type;
  using no = std::false_type;
  using first_step = std::integral_constant<int, 0>;
  using second_step = std::integral_constant<int, 1>;
  step(f0, f1, 0, no{}, first_step{});
  int b = 0;
  for (; b + C::STAGES < blocks; ++b) {
    step(f1, f0, b, yes{}, second_step{});
    step(f0, f1, b + 1, yes{}, first_step{});
  }
  for (; b < blocks; ++b) {
    step(f1, f0, b, no{}, second_step{});
    if (b + 1 < blocks) step(f0, f1, b + 1, no{}, first_step{});
  }

  __syncthreads();                                           // the stages are free: each wave stages its rows in its share
  const int64_t rows_left = a.m - row0 - wm0, cols_left = a.n - col0 - wn0;
  const int64_t ld = SLICE ? a.n : a.ldc;
  const int64_t at = SLICE ? (((int64_t)blockIdx.y * a.k + w) * a.m + row0 + wm0) * a.n + col0 + wn0
                           : w * a.c_stride + (row0 + wm0) * a.ldc + col0 + wn0;
  // 32 rows of one or two of the tile's 32s at a time: each wave turns them to whole lines in its piece of LDS.  A tile that
  // lies within C is written without a look at its ends.
  const bool within = rows_left >= C::WTM * 32 && cols_left >= C::WTN * 32;
  constexpr int OUT_B = 32 * (128 + 16);                     // of a wave: 32 rows of at most 128 bytes
  static_assert(C::NW * OUT_B <= C::OFF_S, "staging fits the stages");
  char* wl = smem + wave * OUT_B;
  auto write = [&](auto within_) {
    constexpr bool WITHIN = decltype(within_)::value;
    constexpr bool F = SLICE || EXACT;
    constexpr int JS = F || C::WTN < 2 ? 1 : 2, RS = JS * (F ? 128 : 64) + 16, LPR = JS * (F ? 8 : 4), RPP = 64 / LPR, V = F ? 4 : 8;
    using T = std::conditional_t<F, float, uint16_t>;
    using E = std::conditional_t<F, F32, Bf16>;
    const int r0 = lane / LPR, ch = lane % LPR;
    T* out = reinterpret_cast<T*>(SLICE ? reinterpret_cast<void*>(a.part) : a.c) + at + r0 * ld + ch * V;
#pragma unroll
    for (int i = 0; i < C::WTM; ++i)
#pragma unroll
      for (int j0 = 0; j0 < C::WTN; j0 += JS) {
#pragma unroll
        for (int j = 0; j < JS; ++j) {
          f32x16& v = acc[i][j0 + j];
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            char* to = wl + l32 * RS + (j * 32 + g * 8 + half * 4) * (int)sizeof(T);
            if constexpr (F) {
              constexpr float S = EXACT ? 1.f / kWidened : 1.f;
              *reinterpret_cast<float4*>(to) = make_float4(v[4 * g] * S, v[4 * g + 1] * S, v[4 * g + 2] * S, v[4 * g + 3] * S);
            }
            else *reinterpret_cast<uint2*>(to) = make_uint2(pack_bf16(v[4 * g], v[4 * g + 1]), pack_bf16(v[4 * g + 2], v[4 * g + 3]));
          }
        }
#pragma unroll
        for (int p = 0; p < 32 / RPP; ++p) {
          const uint4 v = *reinterpret_cast<const uint4*>(wl + (p * RPP + r0) * RS + ch * 16);
          T* o = out + (int64_t)(i * 32 + p * RPP) * ld + j0 * 32;
          if (WITHIN || (i * 32 + p * RPP + r0 < rows_left && (j0 * 32 + (ch + 1) * V <= cols_left))) {
            *reinterpret_cast<typename E::Raw*>(o) = typename E::Raw{{v.x, v.y, v.z, v.w}};
          } else if (i * 32 + p * RPP + r0 < rows_left) {
            const uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
            for (int e = 0; e < V; ++e)
              if (j0 * 32 + ch * V + e < cols_left) {
                if constexpr (F) o[e] = __uint_as_float(u[e]);
                else o[e] = (uint16_t)(u[e >> 1] >> (16 * (e & 1)));
              }
          }
        }
      }
  };
  if (within) write(std::true_type{});
  else write(std::false_type{});
}

// Few rows of a (a served model's tokens): the product is as fast as b can be read.  A block takes 16 rows of b and all of
// a, MT tiles of 16 rows; its waves deal the blocks of 128 out among themselves, each reading whole lines of b straight
// into registers, and add their sums up through LDS in order.  v_mfma_scale_f32_16x16x128_f8f6f4, b as operand A: a lane
// holds one row of a and four consecutive columns of C.  (EXACT: v_mfma_f32_16x16x32_bf16 on widened numbers, see above.)
// A lane reads 16 bytes at 16 (lane/16) and 16 at 64 + 16 (lane/16) of a row's 128: any division of the block among the
// lanes will do as long as it is the same for both operands.
typedef float f32x4 __attribute__((ext_vector_type(4)));

// E: a is not quantised yet (rows of a.x).  Every block does it for itself, into LDS, while its first loads of b are on their
// way: that costs less than a launch in front while the rows are few.  Rows in LDS are 16 bytes longer than their numbers, so
// that 16 of them lie over all banks.
constexpr int kRowWaves = 8;

template <int MT, bool EXACT, class E>
__global__ __launch_bounds__(kRowWaves * 64) void gemm_fp8_rows_kernel(Fp8Args a) {
  constexpr int WAVES = kRowWaves, AHEAD = 4 / MT < 2 ? 2 : 4 / MT;             // blocks of 128 a wave has in flight
  __shared__ float sums[WAVES][MT][16][17];
  const int w = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, part = lane >> 4;
  const int64_t n0 = (int64_t)blockIdx.x * 16;
  const int blocks = (int)(a.kp / BK);
  const int64_t nr = n0 + r16 < a.n ? n0 + r16 : a.n - 1;
  const uint8_t* pb = a.b + (w * a.n + nr) * a.kp + part * 16;
  const uint8_t* psb = a.sb + (w * a.n + nr) * a.ks;
  constexpr bool RAW = !std::is_void<E>::value;
  extern __shared__ __attribute__((aligned(16))) uint8_t rows8[];          // RAW: [m][kp + 16] numbers, then [m][blocks] scales
  uint8_t* scales8 = rows8 + a.m * (a.kp + 16);
  const uint8_t* pa[MT];
  const uint8_t* psa[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) {
    const int64_t mr = i * 16 + r16 < a.m ? i * 16 + r16 : a.m - 1;
    pa[i] = RAW ? rows8 + mr * (a.kp + 16) + part * 16 : a.a + (w * a.m + mr) * a.kp + part * 16;
    psa[i] = RAW ? scales8 + mr * blocks : a.sa + (w * a.m + mr) * a.ks;
  }
  struct Piece { uint4 lo, hi; int scale; };
  auto read = [](const uint8_t* row, const uint8_t* scales, int b) {
    return Piece{*reinterpret_cast<const uint4*>(row + (int64_t)b * BK), *reinterpret_cast<const uint4*>(row + (int64_t)b * BK + 64), scales[b]};
  };
  auto all = [](const Piece& p) {
    const i32x8 r = {(int)p.lo.x, (int)p.lo.y, (int)p.lo.z, (int)p.lo.w, (int)p.hi.x, (int)p.hi.y, (int)p.hi.z, (int)p.hi.w};
    return r;
  };
  f32x4 acc[MT];
#pragma unroll
  for (int i = 0; i < MT; ++i) acc[i] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto multiply = [&](const Piece& y, const Piece (&x)[MT]) {
    if constexpr (EXACT) {
      const float sy = half_power(y.scale);
      const bf16x8 y0 = widen((int)y.lo.x, (int)y.lo.y, sy), y1 = widen((int)y.lo.z, (int)y.lo.w, sy);
      const bf16x8 y2 = widen((int)y.hi.x, (int)y.hi.y, sy), y3 = widen((int)y.hi.z, (int)y.hi.w, sy);
#pragma unroll
      for (int i = 0; i < MT; ++i) {
        const float sx = half_power(x[i].scale);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y0, widen((int)x[i].lo.x, (int)x[i].lo.y, sx), acc[i], 0, 0, 0);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y1, widen((int)x[i].lo.z, (int)x[i].lo.w, sx), acc[i], 0, 0, 0);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y2, widen((int)x[i].hi.x, (int)x[i].hi.y, sx), acc[i], 0, 0, 0);
        acc[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(y3, widen((int)x[i].hi.z, (int)x[i].hi.w, sx), acc[i], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < MT; ++i)
        acc[i] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(all(y), all(x[i]), acc[i], 0, 0, 0, y.scale, 0, x[i].scale);
    }
  };
  // AHEAD blocks at a time, all of their loads before the first product: nothing else hides what a load takes
  for (int b = wave; b < blocks || (RAW && b == wave); b += AHEAD * WAVES) {
    Piece y[AHEAD], x[AHEAD][MT];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (b + u * WAVES < blocks) y[u] = read(pb, psb, b + u * WAVES);
    if constexpr (RAW) {
      if (b == wave) {                                       // once, and every wave comes by
        const typename E::T* rows = reinterpret_cast<const typename E::T*>(a.x.p) + w * a.x.stride;
        const int per_row = blocks * 16, all = (int)a.m * per_row, t = threadIdx.x & 15;
        for (int e = threadIdx.x; e < all; e += WAVES * 64) {               // 16 lanes a block of 128
          const int m = e / per_row, blk = (e - m * per_row) >> 4;
          Raw8<E> raw;
          float f[8];
          raw.load(rows + m * a.x.ld, (int64_t)blk * BK + t * 8, a.contraction);
          raw.floats(f);
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 8; ++j) top = larger(top, magnitude(f[j]));
          const Scale s = scale_of(largest_of_16(top));
          *reinterpret_cast<uint2*>(rows8 + m * (a.kp + 16) + blk * BK + t * 8) = to_e4m3(f, s.inverse);
          if (t == 0) scales8[m * blocks + blk] = (uint8_t)s.byte;
        }
        __syncthreads();
      }
    }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (b + u * WAVES < blocks) {
#pragma unroll
        for (int i = 0; i < MT; ++i) x[u][i] = read(pa[i], psa[i], b + u * WAVES);
      }
#pragma unroll
    for (int u = 0; u < AHEAD; ++u)
      if (b + u * WAVES < blocks) multiply(y[u], x[u]);
  }
#pragma unroll
  for (int i = 0; i < MT; ++i)
#pragma unroll
    for (int r = 0; r < 4; ++r) sums[wave][i][r16][part * 4 + r] = acc[i][r] * (EXACT ? 1.f / kWidened : 1.f);
  __syncthreads();
  for (int e = threadIdx.x; e < MT * 256; e += WAVES * 64) {
    const int m = e >> 4, c = e & 15;
    if (m >= a.m || n0 + c >= a.n) continue;
    float s = a.bias ? a.bias[w * a.bias_stride + n0 + c] : 0.f;
#pragma unroll
    for (int q = 0; q < WAVES; ++q) s += sums[q][m >> 4][m & 15][c];
    const int64_t at = w * a.c_stride + m * a.ldc + n0 + c;
    if constexpr (EXACT) F32::put(reinterpret_cast<float*>(a.c) + at, s);
    else Bf16::put(reinterpret_cast<uint16_t*>(a.c) + at, s);
  }
}

template <int MT>
hipError_t launch_rows(const Fp8Args& a, hipStream_t s) {
  const dim3 grid((unsigned)ceil_div(a.n, 16), (unsigned)a.k), block(kRowWaves * 64);
  if (a.dtype == DW_F32) hipLaunchKernelGGL((gemm_fp8_rows_kernel<MT, true, void>), grid, block, 0, s, a);
  else hipLaunchKernelGGL((gemm_fp8_rows_kernel<MT, false, void>), grid, block, 0, s, a);
  return hipGetLastError();
}

// Quantised on the way: up to 16 rows whose numbers fill at most 16 KB, as every block goes through all of them (us, against
// a launch of its own: 4096 x 4096, m = 1: 5.4, 7.7; m = 4: 7.0, 8.2; m = 8: 9.3, 8.5; 256 x 1024, m = 16: 4.4, 4.9)
constexpr int64_t kFusedRows = 16, kFusedBytes = 16384;
template <bool EXACT, class E>
hipError_t launch_fused(const Fp8Args& a, hipStream_t s) {
  const size_t lds = (size_t)(a.m * (a.kp + 16) + a.m * (a.kp / BK));
  hipLaunchKernelGGL((gemm_fp8_rows_kernel<1, EXACT, E>), dim3((unsigned)ceil_div(a.n, 16), (unsigned)a.k), dim3(kRowWaves * 64), lds, s, a);
  return hipGetLastError();
}

// an empty contraction: the bias, or zeros
__global__ __launch_bounds__(256) void bias_rows_kernel(Fp8Args a) {
  const int w = blockIdx.z;
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (n >= a.n) return;
  const float v = a.bias ? a.bias[w * a.bias_stride + n] : 0.f;
  for (int64_t m = blockIdx.y; m < a.m; m += gridDim.y) {
    const int64_t at = w * a.c_stride + m * a.ldc + n;
    if (a.dtype == DW_F32) F32::put(reinterpret_cast<float*>(a.c) + at, v);
    else Bf16::put(reinterpret_cast<uint16_t*>(a.c) + at, v);
  }
}

using Large = Config<4, 4, 2, 2, 1, 2, 3>;                      // 256 x 256, a wave 128 x 128
using Middle = Config<2, 2, 2, 2, 2, 2, 0>;                     // 128 x 128
using Small = Config<1, 1, 2, 2, 2, 4, 0>;                      // 64 x 64

// the slices' sums in their order, and the bias
template <class E>
__global__ __launch_bounds__(256) void add_slices_kernel(Fp8Args a, int slices) {
  const int w = blockIdx.z;
  const int64_t n = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)a.k * a.m * a.n;
  if (n >= a.n) return;
  const float bias = a.bias ? a.bias[w * a.bias_stride + n] : 0.f;
  for (int64_t m = blockIdx.y; m < a.m; m += gridDim.y) {
    const float* p = a.part + ((int64_t)w * a.m + m) * a.n + n;
    float s = bias;
#pragma unroll 4
    for (int i = 0; i < slices; ++i) s += p[i * step];
    E::put(reinterpret_cast<typename E::T*>(a.c) + w * a.c_stride + m * a.ldc + n, s);
  }
}

template <class C, bool EXACT, bool SLICE>
hipError_t launch_one(const Fp8Args& a, int slices, hipStream_t s) {
  const int64_t tiles = ceil_div(a.m, C::BM) * ceil_div(a.n, C::BN) * a.k;
  auto kern = gemm_fp8_kernel<C, EXACT, SLICE>;
  static LdsLimitOnce lds_limit;
  const hipError_t e = lds_limit.raise(reinterpret_cast<const void*>(kern), C::LDS);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(kern, dim3((unsigned)(ceil_div(tiles, 8) * 8), (unsigned)slices), dim3(C::NT), C::LDS, s, a);
  return hipGetLastError();
}

template <class C>
hipError_t launch(const Fp8Args& a, hipStream_t s) {
  return a.dtype == DW_F32 ? launch_one<C, true, false>(a, 1, s) : launch_one<C, false, false>(a, 1, s);
}

int64_t tiles_of(int k, int64_t m, int64_t n, int b) { return ceil_div(m, b) * ceil_div(n, b) * k; }

// Which kernel a product takes.  The rows kernel reads a anew for every 16 rows of b and is held by how fast a compute unit
// takes in rows of 64 bytes, so its time grows with m and with the contraction a wave goes through; the tiles read 64 rows of a
// whatever m is and are cut into slices where they are few.  Both sides, us, in bf16 (fp32 alike):
//   4096 x 4096            m = 1: 5.4, 7.0;  m = 16: 7.6, 7.8;  m = 32: 10.4, 8.5
//   four of 8192 x 2048    m = 1: 14.7, 16.6;  m = 8: 18, 16;   256 x 1024   m = 1: 2.4, 4.5;  m = 64: 4.8, 4.7
//   1024 x 8192            m = 1: 8.0, 7.2;  m = 16: 12, 7.6;   8192 x 8192  m = 1: 15, 15;  m = 16: 23, 16
bool rows_kernel(int k, int64_t m, int64_t n, int64_t kp) {
  if (kp > 4096 || m > 64 || m * kp > 65536) return false;
  return m <= 4 || tiles_of(k, m, n, 64) < kCus;
}

// Slices of the contraction (whole words of scales, 512 numbers) for products with fewer 64 x 64 tiles than compute units,
// by what they would take: 0.3 us a block of 128 (measured: bf16 0.25, fp32 0.45; one number, so that both results take the same
// scratch), and for slices 3.5 us and their sums, written and read, at 2 TB/s.  1024 x 8192, m = 64: 18 us whole, 8.5 in slices; 4096 x 4096, m = 128: 11 whole, 13.4 in two, 15.3 in four.
int slices_of(int k, int64_t m, int64_t n, int64_t blocks) {
  const int64_t tiles = tiles_of(k, m, n, 64), words = ceil_div(blocks, GROUP);
  int best = 1;
  double least = 0.3 * (double)blocks;
  for (int64_t s = 2; s <= 16 && s <= words && tiles * s <= 2 * kCus; ++s) {
    const int64_t per = ceil_div(words, s);
    if (ceil_div(words, per) != s) continue;                 // (a slice would be empty)
    const double t = 0.3 * (double)(per * GROUP) + 3.5 + (double)s * (double)(k * m * n) * 8.0 / 2e6;
    if (t < least) { least = t; best = (int)s; }
  }
  return best;
}

// Tiles of 256 or of 128 by the turns they take: one of 256 a compute unit, 10 units of time, against two of 128, 5.8, or at most
// one, 4 (us, 256s and 128s, in bf16; fp32 alike): 3000 cubed, 144 of 256: 43.7, 41.9; 3584 x 3584 x 512, 196: 14.1, 14.6;
// 4352 x 4096 x 4096, 272: 90, 82; 7168 x 4096 x 2048, 448: 53, 62; 8448 x 4096 x 1024, 528: 48, 44.5; 16384 x 4096 x 1024, 1024: 69, 73
bool large_tiles(int k, int64_t m, int64_t n) {
  const int64_t large = tiles_of(k, m, n, 256), middle = tiles_of(k, m, n, 128), rest = middle % (2 * kCus);
  const double last = rest == 0 ? 0 : rest <= kCus ? 4.0 : 5.8;
  return 10.0 * (double)ceil_div(large, kCus) <= 5.8 * (double)(middle / (2 * kCus)) + last;
}

}  // namespace fp8

size_t fp8_scratch_bytes(int k, int64_t m, int64_t n, int64_t kp) {
  const int s = fp8::rows_kernel(k, m, n, kp) ? 1 : fp8::slices_of(k, m, n, kp / fp8::BK);
  return s > 1 ? (size_t)s * k * m * n * sizeof(float) : 0;
}

bool fp8_linear_fused(int k, int64_t m, int64_t n, int64_t kp) {
  return kp > 0 && m <= fp8::kFusedRows && m * kp <= fp8::kFusedBytes && fp8::rows_kernel(k, m, n, kp);
}

hipError_t launch_fp8_linear_fused(const Fp8Args& a, hipStream_t s) {
  return a.dtype == DW_F32 ? fp8::launch_fused<true, F32>(a, s) : fp8::launch_fused<false, Bf16>(a, s);
}

hipError_t launch_fp8_matmul(const Fp8Args& a_, hipStream_t s) {
  Fp8Args a = a_;
  if (a.kp == 0) {
    const dim3 grid((unsigned)ceil_div(a.n, 256), (unsigned)(a.m < 1024 ? a.m : 1024), (unsigned)a.k);
    hipLaunchKernelGGL(fp8::bias_rows_kernel, grid, dim3(256), 0, s, a);
    return hipGetLastError();
  }
  if (fp8::rows_kernel(a.k, a.m, a.n, a.kp)) {
    if (a.m <= 16) return fp8::launch_rows<1>(a, s);
    return a.m <= 32 ? fp8::launch_rows<2>(a, s) : fp8::launch_rows<4>(a, s);
  }
  if (fp8::large_tiles(a.k, a.m, a.n)) return fp8::launch<fp8::Large>(a, s);
  // Small tiles while they run all at once, two a compute unit (us, 64s and 128s): 4096 x 512 x 4096, 512 of them: 15.0, 23.1 (fp32
  // 23.8, 28.4); 3 x 700 x 900 x 450, 495: 5.4, 7.1; 2 x 1500 x 700 x 5000, 528: 28.5, 30.4 (fp32 41.3, 36.0: the limit is where fp32
  // turns, which bf16 does a little later); 2048 cubed, 1024: 16.5, 12.6
  if (fp8::tiles_of(a.k, a.m, a.n, 64) > 2 * kCus) return fp8::launch<fp8::Middle>(a, s);
  const int slices = fp8::slices_of(a.k, a.m, a.n, a.kp / fp8::BK);
  if (slices == 1) return fp8::launch<fp8::Small>(a, s);
  const int words = (int)ceil_div(a.kp / fp8::BK, fp8::GROUP);
  a.slice_blocks = (int)ceil_div(words, slices) * fp8::GROUP;    // (the last slice may be shorter, none is empty)
  const hipError_t e = a.dtype == DW_F32 ? fp8::launch_one<fp8::Small, true, true>(a, slices, s) : fp8::launch_one<fp8::Small, false, true>(a, slices, s);
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)ceil_div(a.n, 256), (unsigned)(a.m < 1024 ? a.m : 1024), (unsigned)a.k);
  if (a.dtype == DW_F32) hipLaunchKernelGGL(fp8::add_slices_kernel<F32>, grid, dim3(256), 0, s, a, slices);
  else hipLaunchKernelGGL(fp8::add_slices_kernel<Bf16>, grid, dim3(256), 0, s, a, slices);
  return hipGetLastError();
}

}  // namespace dw
