// ops_product.hip -- the 8-bit block form and the product of two matrices in it.
//
// Form: codes q (e4m3) with one 32-bit scale for each 128 elements along the
// contraction (of one row, or of 128 rows).  Product: for each block of 128,
// the matrix cores sum the codes' products (v_mfma_f32_16x16x128_f8f6f4: one
// instruction is one block), and 32-bit VALU multiply-adds bring that sum to
// scale and add it up.
#include <type_traits>

#include "ops_common.h"

namespace hetsim {
namespace ops {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// ---------------------------------------------------------------- quantiser
// Rows only: 16 lanes hold the 128 elements of one (row, column block), eight
// each; the maximum crosses lanes, and each lane writes its eight codes.  One
// read and one write of the data, so memory bounds large ones: 8192 x 8192 in
// 33.6 us, 6.0 TB/s (the caches hold part of it from call to call).  1531 x 4096
// takes 5.1 us in a row of such calls and 6.9 between others, of which a launch
// of this kind takes 2.6 to 4.7 (17 x 8192).  Rows that are not whole multiples of eight
// elements, or misaligned, go one element at a time: 8192 x 8191 in 76 us.
template <typename T, bool kVec>
__global__ __launch_bounds__(256) void k_quant_rows(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                    uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ s,
                                                    int64_t lds) {
  const int64_t kb = (cols + kBlock - 1) / kBlock;
  const int64_t unit = ((int64_t)blockIdx.x * 256 + threadIdx.x) / 16;   // row-major: neighbouring blocks of a row
  if (unit >= rows * kb) return;                                          // (whole groups of 16 lanes)
  const int64_t row = unit / kb, b = unit % kb;
  const int64_t c = b * kBlock + (threadIdx.x & 15) * 8;
  float v[8];
  load8<T, kVec>(x + row * ld, c, cols - c, v);
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  m = fmaxf(max16(m), kAmaxFloor);
  const float f = kE4m3Max / m;
  *(u32x2*)(q + row * ldq + c) = u32x2{codes4(v[0], v[1], v[2], v[3], f), codes4(v[4], v[5], v[6], v[7], f)};
  if ((threadIdx.x & 15) == 0) s[b * lds + row] = m / kE4m3Max;
}

// Both forms, or the transpose alone, or blocks of 128 x 128: one workgroup
// reads a 128 x 128 tile once.  Thread (rg, cl) holds rows 8 rg .. 8 rg + 7 of
// the eight columns from 8 cl on, so that a row's maximum crosses the 16 lanes
// of one rg, a column's the 16 rgs, and the eight codes of one column are
// eight neighbours in the transpose, which goes through LDS so that 128-byte
// rows leave.  There the eight-byte piece rg of column k is at rg ^ (k / 8), so
// that the 16 columns that are written at a time lie in different banks.  One
// read and two writes of the data bound it: both forms of 8192 x 8192 in 53 us
// in a row of such calls, 62 between others, 4.4 TB/s (82 us with rows of LDS four
// banks apart and the elements kept as 32-bit floats).
template <typename T, bool kVec, int kRows>   // kRows: 1 or 128 rows to a scale
__global__ __launch_bounds__(256) void k_quant_tile(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld,
                                                    uint8_t* __restrict__ q, int64_t ldq, float* __restrict__ s,
                                                    int64_t lds, uint8_t* __restrict__ qt, int64_t ldqt,
                                                    float* __restrict__ st, int64_t ldst) {
  __shared__ __attribute__((aligned(16))) uint8_t tile[kBlock * kBlock];
  __shared__ float part[4][kBlock];
  const int t = threadIdx.x, rg = t / 16, cl = t % 16, wave = t / 64;
  const int64_t col_tiles = (cols + kBlock - 1) / kBlock;
  const int64_t bc = blockIdx.x % col_tiles, br = blockIdx.x / col_tiles;
  const int64_t c0 = bc * kBlock, r0 = br * kBlock;
  const int64_t c = c0 + cl * 8, r = r0 + rg * 8;
  // (kept as they are in memory, half the registers of their 32-bit values)
  Raw<T> raw[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) raw[i] = fetch8<T, kVec>(x + min(r + i, rows - 1) * ld, c, r + i < rows ? cols - c : 0);
  auto v = [&](int i, int j) { return kVec && (r + i >= rows || c >= cols) ? 0.0f : (float)raw[i].v[j]; };
  float rmax[8], cmax[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) cmax[j] = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    rmax[i] = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float a = fabsf(v(i, j));
      rmax[i] = fmaxf(rmax[i], a);
      cmax[j] = fmaxf(cmax[j], a);
    }
  }
  if constexpr (kRows == 1) {
    if (q) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float m = fmaxf(max16(rmax[i]), kAmaxFloor);
        const float f = kE4m3Max / m;
        if (r + i < rows) {
          *(u32x2*)(q + (r + i) * ldq + c) = u32x2{codes4(v(i, 0), v(i, 1), v(i, 2), v(i, 3), f),
                                                   codes4(v(i, 4), v(i, 5), v(i, 6), v(i, 7), f)};
          if (cl == 0) s[bc * lds + r + i] = m / kE4m3Max;
        }
      }
    }
    if (!qt) return;
    // column maxima over the wave's four rgs, then over the four waves
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 16));
      cmax[j] = fmaxf(cmax[j], __shfl_xor(cmax[j], 32));
      if ((t & 63) < 16) part[wave][cl * 8 + j] = cmax[j];
    }
    __syncthreads();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int k = cl * 8 + j;
      const float m = fmaxf(fmaxf(fmaxf(part[0][k], part[1][k]), fmaxf(part[2][k], part[3][k])), kAmaxFloor);
      const float f = kE4m3Max / m;
      *(u32x2*)(tile + k * kBlock + (rg ^ cl) * 8) = u32x2{codes4(v(0, j), v(1, j), v(2, j), v(3, j), f),
                                                    codes4(v(4, j), v(5, j), v(6, j), v(7, j), f)};
      if (rg == 0 && c0 + k < cols) st[br * ldst + c0 + k] = m / kE4m3Max;
    }
  } else {
    float m = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = fmaxf(m, rmax[i]);
    m = max16(m);
    m = fmaxf(m, __shfl_xor(m, 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    if ((t & 63) == 0) part[0][wave] = m;
    __syncthreads();
    m = fmaxf(fmaxf(fmaxf(part[0][0], part[0][1]), fmaxf(part[0][2], part[0][3])), kAmaxFloor);
    const float f = kE4m3Max / m;
    if (t == 0) {
      if (q) s[bc * lds + br] = m / kE4m3Max;
      if (qt) st[br * ldst + bc] = m / kE4m3Max;
    }
    if (q) {
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (r + i < rows)
          *(u32x2*)(q + (r + i) * ldq + c) = u32x2{codes4(v(i, 0), v(i, 1), v(i, 2), v(i, 3), f),
                                                   codes4(v(i, 4), v(i, 5), v(i, 6), v(i, 7), f)};
    }
    if (!qt) return;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      *(u32x2*)(tile + (cl * 8 + j) * kBlock + (rg ^ cl) * 8) = u32x2{codes4(v(0, j), v(1, j), v(2, j), v(3, j), f),
                                                              codes4(v(4, j), v(5, j), v(6, j), v(7, j), f)};
  }
  __syncthreads();
  // 128 columns of 128 codes: eight lanes write one column's 128 bytes
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int k = i * 32 + t / 8, piece = t % 8, sw = k / 8;
    const u32x4 a = *(const u32x4*)(tile + k * kBlock + (piece ^ (sw >> 1)) * 16);
    if (c0 + k < cols)
      *(u32x4*)(qt + (c0 + k) * ldqt + r0 + piece * 16) = sw & 1 ? u32x4{a[2], a[3], a[0], a[1]} : a;
  }
}

// Rows past what one launch takes go into further ones, whole tiles of 128 where
// it takes tiles.
template <typename T>
hipError_t quantize(const T* x, int64_t rows, int64_t cols, int64_t ld, const sim_blocks* q, const sim_blocks* qt,
                    hipStream_t st) {
  const bool vec = aligned(x, 8 * sizeof(T)) && cols % 8 == 0 && ld % 8 == 0;
  const int64_t block_rows = q ? q->block_rows : qt->block_rows, kb = cdiv(cols, kBlock);
  const bool units = block_rows == 1 && !qt;      // a group of 16 threads to a block of a row, or a workgroup to a tile
  const int64_t most = units ? most_groups(256) * 16 / kb : most_groups(256) / kb * kBlock;
  if (most == 0) return hipErrorInvalidValue;
  sim_blocks a = q ? *q : sim_blocks(), b = qt ? *qt : sim_blocks();
  for (int64_t r = 0; r < rows; r += most) {
    const int64_t n = rows - r < most ? rows - r : most;
    if (units) {
      auto k = vec ? k_quant_rows<T, true> : k_quant_rows<T, false>;
      k<<<dim3((uint32_t)cdiv(n * kb, 16)), 256, 0, st>>>(x, n, cols, ld, a.codes, a.ld, a.scales, a.ld_s);
    } else {
      auto k = block_rows == 1 ? (vec ? k_quant_tile<T, true, 1> : k_quant_tile<T, false, 1>)
                               : (vec ? k_quant_tile<T, true, kBlock> : k_quant_tile<T, false, kBlock>);
      k<<<dim3((uint32_t)(cdiv(n, kBlock) * kb)), 256, 0, st>>>(x, n, cols, ld, a.codes, a.ld, a.scales, a.ld_s, b.codes, b.ld,
                                                                b.scales, b.ld_s);
    }
    const hipError_t e = launched();
    if (e != hipSuccess) return e;
    x += n * ld;
    if (q) {
      a.codes += n * a.ld;
      a.scales += n / block_rows;
    }
    if (qt) {
      b.codes += n;
      b.scales += n / kBlock * b.ld_s;
    }
  }
  return hipSuccess;
}

hipError_t quantize_any(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, const sim_blocks* q,
                        const sim_blocks* qt, hipStream_t st) {
  switch (dtype) {
    case SIM_BF16: return quantize((const bf16*)x, rows, cols, ld, q, qt, st);
    case SIM_FP16: return quantize((const fp16*)x, rows, cols, ld, q, qt, st);
    default: return quantize((const float*)x, rows, cols, ld, q, qt, st);
  }
}

// ---------------------------------------------------------------- product
struct Product {
  const uint8_t* a;
  const uint8_t* b;
  const float* as;
  const float* bs;
  int64_t lda, ldb, las, lbs;
  int64_t m, n, k;
  int kb;               // blocks of 128 along k
  int a_shift, b_shift; // log2 of rows to a scale
  void* c;
  int64_t ldc;
  int c_dtype, accumulate;
  float* part;          // partial sums, a slot of a tile's size for each part of a split tile
  int whole, splits;    // tiles made by one workgroup each; parts of each of the others.  Of k_few: blocks
                        // along k to a part; parts
};

// Four neighbours of a row of C.
template <typename T>
__device__ inline void put4(T* c, int64_t have, bool vec, int accumulate, f32x4 v) {
  typedef T t4 __attribute__((ext_vector_type(4)));
  if (vec && have >= 4) {
    if (accumulate) {
      const t4 o = *(const t4*)c;
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += (float)o[i];
    }
    t4 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = (T)v[i];
    *(t4*)c = r;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < have) c[i] = (T)(accumulate ? v[i] + (float)c[i] : v[i]);
}

__device__ inline void put4_any(const Product& p, int64_t row, int64_t col, f32x4 v) {
  if (row >= p.m || col >= p.n) return;
  const int64_t at = row * p.ldc + col;
  const bool vec = ((((uintptr_t)p.c) | (uintptr_t)(p.ldc * 4)) & 15) == 0;   // (ldc a multiple of 4)
  if (p.c_dtype == SIM_BF16) put4((bf16*)p.c + at, p.n - col, vec, p.accumulate, v);
  else if (p.c_dtype == SIM_FP16) put4((fp16*)p.c + at, p.n - col, vec, p.accumulate, v);
  else put4((float*)p.c + at, p.n - col, vec, p.accumulate, v);
}

__device__ inline i32x8 join(i32x4 a, i32x4 b) {
  return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7);
}

// D[i][j] = sum over 128 codes of P[i] Q[j]: lane l gives row l % 16 of both
// operands, bytes 32 (l / 16) on, and gets rows 4 (l / 16) .. + 3 of column
// l % 16.  The instruction aligns a group of products to the largest of them, so
// this sum has less than 32 bits: on normal codes it is 1.33e-5 off (root of the
// mean square), the same with the 32-code form, where bf16 instructions on the
// same values are at 1e-8.  Taken all the same: those run at half the rate, behind
// a conversion of every code, and the codes themselves are 2.6 % off what was
// rounded to them.  Sums of blocks are in 32 bits.
__device__ inline f32x4 mfma128(i32x8 p, i32x8 q) {
  return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(p, q, f32x4{0.0f, 0.0f, 0.0f, 0.0f}, 0, 0, 0, 0, 0, 0);
}

// Tiled product: a workgroup makes kBM x kBN elements of C, wave (wm, wn) of
// its kWM x kWN waves a part of them.  Rows of A are the matrix instruction's
// columns, so that a lane has one scale of A for a tile and four neighbours of
// a row of C.  Both operands' blocks of 128 and their scales go from memory
// straight into LDS, one block ahead of the one being multiplied.  A lane of
// quarter q reads the 16-byte pieces q and q + 4 of its row, of both operands
// alike, and piece c of row r is stored at c ^ (r / 2 % 8): the 16 lanes that
// a read serves at a time then touch different banks.
// Order within a block, which scheduling barriers hold: while the matrix cores
// work on a tile, the VALU brings the one three before to scale, one piece of
// the next block is sent for, and the next 16 rows of B are read from LDS.
// kRowB: B has a scale for each row (else one for 128, the same for a whole
// wave), which costs a second VALU operation for each element.
// Eight waves of 128 x 64 fill the registers (226 to 240 of 256): fewer LDS
// reads for a product than with smaller ones, and two waves to a SIMD, so that
// one's VALU work hides in the other's matrix instructions.  Measured, 8192 x
// 8192 x 7168: 394 us in a row of such calls, 2.44 PFLOP/s (median between other
// kernels 477); 7168 x 8192 x 8192 with kRowB 501, 1.92 PFLOP/s (565).  No unit is
// full.  By the counters the matrix cores are busy 61 % of a SIMD's cycles and
// VALU instructions issue in 46 % (kRowB 46 and 58: 10 instructions for a matrix
// instruction, so 6), and the clock falls to 1.8 or 1.9 GHz by the card's power;
// without any fetching it takes 17 % less time, without the VALU work too 28 %.  Steps, at 7168 x 8192 x
// 8192: the compiler's order and conflicting LDS reads about 560 us, distinct
// banks and tiles in order 477, no branch and no wait within a block 445, pieces
// sent for one at a time 421.  Not faster: 32 x 32 x 64 instructions (5 %
// slower, for registers), rows padded apart, pieces sent for earlier, C through
// LDS.
template <int kBM, int kBN, int kWM, int kWN, bool kRowB>
__global__ __launch_bounds__(kWM * kWN * 64, 2) void k_product(Product p, int tiles_m, int tiles_n) {
  constexpr int kThreads = kWM * kWN * 64;
  constexpr int kTM = kBM / kWM / 16, kTN = kBN / kWN / 16;   // tiles of 16 of one wave
  constexpr int kCodes = (kBM + kBN) * kBlock, kStage = kCodes + (kBM + kBN) * 4;
  extern __shared__ __attribute__((aligned(128))) uint8_t lds[];
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t / 64);
  const int wm = wave % kWM, wn = wave / kWM;
  // Neighbouring workgroups go to different XCDs, each with its own L2: give
  // each XCD a run of neighbouring tiles, and runs of 8 tiles of A by all of
  // B's, so that what an XCD works on at a time shares rows and columns.
  int id = blockIdx.x, part = -1;
  if (id < p.whole) {
    const int per = p.whole / 8, extra = p.whole % 8, x = id % 8, y = id / 8;
    id = x * per + min(x, extra) + y;
  } else {
    part = id - p.whole;
    id = p.whole + part / p.splits;
  }
  const int group = 8 * tiles_n, g0 = id / group * 8, gm = min(8, tiles_m - g0);
  const int tm = g0 + id % group % gm, tn = id % group / gm;
  const int64_t m0 = (int64_t)tm * kBM, n0 = (int64_t)tn * kBN;
  const int z = part < 0 ? 0 : part % p.splits, zs = part < 0 ? 1 : p.splits;
  const int kb0 = (int)((int64_t)p.kb * z / zs), kb1 = (int)((int64_t)p.kb * (z + 1) / zs);
  // rows past the last are read as the last, and never stored
  const int last_m = (int)min((int64_t)kBM, p.m - m0) - 1, last_n = (int)min((int64_t)kBN, p.n - n0) - 1;

  // This thread's pieces of a stage: rows of A, then of B, as offsets from the
  // tile's first row (a tile spans less than 2^32 bytes).
  constexpr int kPieces = kCodes / 16 / kThreads, kPiecesA = kBM * 8 / kThreads;
  uint32_t off[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int piece = i * kThreads + t, row = piece / 8, at = (piece % 8) ^ ((row >> 1) & 7);
    off[i] = (i < kPiecesA ? (uint32_t)min(row, last_m) * (uint32_t)p.lda
                           : (uint32_t)min(row - kBM, last_n) * (uint32_t)p.ldb) + (uint32_t)at * 16;
    asm("" : "+v"(off[i]));   // (one register, not the lower half of a product's two)
  }
  constexpr int kScaleLoads = (kBM + kBN) / kThreads;
  static_assert((kBM + kBN) % kThreads == 0 && kBM % 64 == 0, "a wave's 64 scales are all of A or all of B");
  uint32_t soff[kScaleLoads];
#pragma unroll
  for (int i = 0; i < kScaleLoads; ++i) {
    const int row = i * kThreads + t;
    soff[i] = row < kBM ? (uint32_t)((m0 + min(row, last_m)) >> p.a_shift)
                        : (uint32_t)((n0 + min(row - kBM, last_n)) >> p.b_shift);
  }
  // (the descriptors' sizes are those of the tile's rows: what lies past them is not read)
  const __amdgpu_buffer_rsrc_t ra = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(p.a + m0 * p.lda), 0, (uint32_t)last_m * (uint32_t)p.lda + (uint32_t)p.kb * kBlock, 0x00027000);
  const __amdgpu_buffer_rsrc_t rb = __builtin_amdgcn_make_buffer_rsrc(
      (void*)(p.b + n0 * p.ldb), 0, (uint32_t)last_n * (uint32_t)p.ldb + (uint32_t)p.kb * kBlock, 0x00027000);
  // piece i of block kb on its way into a buffer; the scales after the last
  auto fetch = [&](int kb, int buf, int i) {
    if (i < kPieces) {
      __builtin_amdgcn_raw_ptr_buffer_load_lds(
          i < kPiecesA ? ra : rb, (__attribute__((address_space(3))) void*)(lds + buf * kStage + (i * kThreads + wave * 64) * 16),
          16, (int)off[i], kb * kBlock, 0, 0);
    } else {
      const int s = i - kPieces, row = s * kThreads + wave * 64;
      __builtin_amdgcn_global_load_lds(
          (const __attribute__((address_space(1))) void*)((row < kBM ? p.as + kb * p.las : p.bs + kb * p.lbs) + soff[s]),
          (__attribute__((address_space(3))) void*)(lds + buf * kStage + kCodes + row * 4), 4, 0, 0);
    }
  };
  constexpr int kFetches = kPieces + kScaleLoads;

  const int am = wm * (kBM / kWM), bn = wn * (kBN / kWN);
  const int quad = lane >> 4, r16 = lane & 15;
  // of a row r16 + a multiple of 16 the swizzle is the same
  const int sw = (r16 >> 1) & 7, at0 = (quad ^ sw) * 16, at1 = ((quad + 4) ^ sw) * 16;
  auto lds_read = [&](const uint8_t* row) { return join(*(const i32x4*)(row + at0), *(const i32x4*)(row + at1)); };

  // Tile n of a block is (n / kTM, n % kTM); its sum is in d[n % 4] until the
  // VALU adds it, kLag tiles later (the last of a block within the next).
  constexpr int kTiles = kTM * kTN, kLag = 3;
  static_assert(kTiles % 4 == 0 && kTM == 4 && kFetches <= kTiles, "the ring of sums goes on from block to block");
  f32x4 acc[kTN][kTM], d[4];
  float sa[kTM], next_sa[kTM];
  f32x4 sr = {0.0f, 0.0f, 0.0f, 0.0f}, next_sr = sr;
  i32x8 fa[kTM], fb[2];
#pragma unroll
  for (int j = 0; j < kTM; ++j) {
    sa[j] = 0.0f;
#pragma unroll
    for (int i = 0; i < kTN; ++i) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  }
  d[1] = d[2] = d[3] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};
  auto add = [&](int n) {
    const int i = n / kTM, j = n % kTM;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      if constexpr (kRowB) acc[i][j][r] += d[n % 4][r] * (sa[j] * sr[r]);
      else acc[i][j][r] += d[n % 4][r] * sa[j];
    }
  };
  // bases of a stage
  auto codes_a = [&](int buf) { return lds + buf * kStage + (am + r16) * kBlock; };
  auto codes_b = [&](int buf) { return lds + buf * kStage + (kBM + bn + r16) * kBlock; };
  auto scales = [&](int buf) { return (const float*)(lds + buf * kStage + kCodes); };
  float sb = 0.0f;
  auto read_scales = [&](int buf) {
    const float* S = scales(buf);
#pragma unroll
    for (int j = 0; j < kTM; ++j) next_sa[j] = S[am + j * 16 + r16];
    if constexpr (kRowB) next_sr = *(const f32x4*)(S + kBM + bn + quad * 4);
    else sb = S[kBM + bn];
  };

#pragma unroll
  for (int i = 0; i < kFetches; ++i) fetch(kb0, 0, i);
  __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's part of the stage has landed
  __syncthreads();                      // everybody's has
  read_scales(0);
  fb[0] = lds_read(codes_b(0));
#pragma unroll
  for (int j = 0; j < kTM; ++j) fa[j] = lds_read(codes_a(0) + j * 16 * kBlock);
  // (Straight-line code: at the end the last block is fetched and read again, for nothing.)
  for (int kb = kb0; kb < kb1; ++kb) {
    const int buf = (kb - kb0) & 1;
#pragma unroll
    for (int i = 0; i < kTN; ++i) {
      if (i + 1 == kTN) {
        // All of this block is in registers and the next has landed.  Once
        // that is so for everybody, this buffer can be filled again, and the
        // next block's operands are read behind the last group of this one.
        __builtin_amdgcn_s_waitcnt(0x0070);   // vmcnt(0) lgkmcnt(0)
        __syncthreads();
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < kTM; ++j) {
        const int n = i * kTM + j;
        d[n % 4] = mfma128(fb[i & 1], fa[j]);
        // (one at a time: a wave that issues them in a row waits for the others' to be taken)
        if (n < kFetches) fetch(min(kb + 1, kb1 - 1), buf ^ 1, n);
        // (behind the first tile: what is waited for there is this group's operands alone)
        if (j == 0 && i + 1 < kTN) fb[(i + 1) & 1] = lds_read(codes_b(buf) + (i + 1) * 16 * kBlock);
        if (j == 0 && i + 1 == kTN) fb[0] = lds_read(codes_b(buf ^ 1));
        if (i + 1 == kTN) fa[j] = lds_read(codes_a(buf ^ 1) + j * 16 * kBlock);
        if (n == kLag) {
#pragma unroll
          for (int q = 0; q < kTM; ++q) sa[q] = kRowB ? next_sa[q] : next_sa[q] * sb;
        }
        if constexpr (kRowB) {
          if (j == kLag) {
            sr = next_sr;
            if (i + 1 < kTN) next_sr = *(const f32x4*)(scales(buf) + kBM + bn + (i + 1) * 16 + quad * 4);
          }
        }
        add((n + kTiles - kLag) % kTiles);
        if (i + 1 == kTN && j == kTM - 1) read_scales(buf ^ 1);
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  }
  __builtin_amdgcn_s_waitcnt(0x0F70);   // nothing may land in LDS after this workgroup
#pragma unroll
  for (int n = kTiles - kLag; n < kTiles; ++n) add(n);
#pragma unroll
  for (int i = 0; i < kTN; ++i)
#pragma unroll
    for (int j = 0; j < kTM; ++j) {
      const int64_t row = m0 + am + j * 16 + r16, col = n0 + bn + i * 16 + quad * 4;
      if (part >= 0) {
        float* o = p.part + (int64_t)part * (kBM * kBN);
        *(f32x4*)(o + (am + j * 16 + r16) * kBN + bn + i * 16 + quad * 4) = acc[i][j];
      } else {
        put4_any(p, row, col, acc[i][j]);
      }
    }
}

// The split tiles: the sum of their parts, in their order.  Memory bounds it:
// 128 tiles in two parts 14 to 15 us, 5.8 TB/s of reads and writes.
template <int kBM, int kBN>
__global__ __launch_bounds__(256) void k_join(Product p, int tiles_m, int tiles_n) {
  constexpr int kWgs = kBM * kBN / 1024;   // workgroups to a tile, four neighbours to a thread
  const int s = blockIdx.x / kWgs, id = p.whole + s, e = (blockIdx.x % kWgs * 256 + threadIdx.x) * 4;
  const int group = 8 * tiles_n, g0 = id / group * 8, gm = min(8, tiles_m - g0);
  const int64_t row = (int64_t)(g0 + id % group % gm) * kBM + e / kBN, col = (int64_t)(id % group / gm) * kBN + e % kBN;
  if (row >= p.m || col >= p.n) return;
  const float* o = p.part + (int64_t)s * p.splits * (kBM * kBN) + e;
  f32x4 v = *(const f32x4*)o;
  for (int z = 1; z < p.splits; ++z) v += *(const f32x4*)(o + (int64_t)z * (kBM * kBN));
  put4_any(p, row, col, v);
}

__global__ __launch_bounds__(256) void k_zero(Product p) {
  const int64_t per_row = (p.n + 3) / 4;
  for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < p.m * per_row; at += (int64_t)gridDim.x * 256)
    put4_any(p, at / per_row, at % per_row * 4, f32x4{0.0f, 0.0f, 0.0f, 0.0f});
}

// The parts of a split k_few, [splits][m][n in whole fours], in their order.
__global__ __launch_bounds__(256) void k_join_few(Product p) {
  const int64_t per_row = (p.n + 3) / 4, at = (int64_t)blockIdx.x * 256 + threadIdx.x, size = p.m * per_row;
  if (at >= size) return;
  const f32x4* o = (const f32x4*)p.part + at;
  f32x4 v = *o;
  for (int z = 1; z < p.splits; ++z) v += o[z * size];
  put4_any(p, at / per_row, at % per_row * 4, v);
}

// ---------------------------------------------------------------- few tokens
// Up to 64 rows of A: the time is that of B's codes on their way from memory
// (one row of A, 7168 x 8192: 13.6 us, 4.3 TB/s; 17 rows 18, 64 rows 25, where
// the reads of A from the L2 count),
// so every wave streams 16 (or 32) rows of B straight into the matrix
// instruction's operand registers, up to eight blocks of 128 at a time.  The
// eight waves of a workgroup take every eighth block of the same rows, and add
// their sums up through LDS.  Rows of A are the instruction's columns, 16 to a
// tile; those past the last read the last one's, and are not stored.
// X: uint8_t, codes and scales as of any product; or the type of A before
// rounding, which every workgroup brings to 8 bits in LDS for itself while its
// first rows of B are on their way.
template <typename X>
struct Few {
  const X* x;
  int64_t ldx;
};
constexpr int kFewWaves = 8;

template <typename X, int kTM, int kTN, bool kRowB, bool kVec>
__global__ __launch_bounds__(kFewWaves * 64) void k_few(Product p, Few<X> few) {
  constexpr bool kCodes = sizeof(X) == 1;
  constexpr int kMost = kTM * kTN == 1 ? (kCodes ? 4 : 8) : kTM * kTN == 2 ? 4 : 2;   // blocks at a time, by the registers
  __shared__ f32x4 red[kFewWaves][kTM * kTN][64];
  extern __shared__ __attribute__((aligned(16))) uint8_t lds[];   // codes [m][128 kb], scales [kb][m]
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t / 64);
  const int quad = lane >> 4, r16 = lane & 15;
  const int64_t n0 = (int64_t)blockIdx.x * (16 * kTN);
  if (p.splits > 1) {
    const int64_t first = (int64_t)blockIdx.y * p.whole;
    p.kb = min(p.whole, p.kb - (int)first);
    p.k -= first * kBlock;
    p.b += first * kBlock;
    p.bs += first * p.lbs;
    if constexpr (kCodes) p.as += first * p.las;
    few.x += first * kBlock;
    p.ldc = (p.n + 3) / 4 * 4;
    p.c = p.part + blockIdx.y * p.m * p.ldc;
    p.c_dtype = SIM_FP32;
    p.accumulate = 0;
  }
  const int kp = p.kb * kBlock;
  float* lds_scales = (float*)(lds + (int)p.m * kp);
  const uint8_t* b[kTN];
  int64_t brow[kTN][4];
#pragma unroll
  for (int i = 0; i < kTN; ++i) {
    b[i] = p.b + min(n0 + i * 16 + r16, p.n - 1) * p.ldb + quad * 32;
#pragma unroll
    for (int r = 0; r < 4; ++r) brow[i][r] = min(n0 + i * 16 + quad * 4 + r, p.n - 1);
  }
  int arow[kTM];
  const uint8_t* a[kTM];
#pragma unroll
  for (int j = 0; j < kTM; ++j) {
    arow[j] = min(j * 16 + r16, (int)p.m - 1);
    if constexpr (kCodes) a[j] = few.x + arow[j] * few.ldx + quad * 32;
  }
  f32x4 acc[kTN][kTM];
#pragma unroll
  for (int i = 0; i < kTN; ++i)
#pragma unroll
    for (int j = 0; j < kTM; ++j) acc[i][j] = f32x4{0.0f, 0.0f, 0.0f, 0.0f};

  i32x8 fb[kMost][kTN];
  auto load_b = [&](int kb0, auto count) {
#pragma unroll
    for (int u = 0; u < decltype(count)::value; ++u)
#pragma unroll
      for (int i = 0; i < kTN; ++i) {
        const i32x4* s = (const i32x4*)(b[i] + (int64_t)(kb0 + u * kFewWaves) * kBlock);
        fb[u][i] = join(s[0], s[1]);
      }
  };
  auto work = [&](int kb0, auto count) {
    constexpr int kCount = decltype(count)::value;
    i32x8 fa[kCount][kTM];
    float sa[kCount][kTM], sb[kCount][kTN];
    f32x4 sr[kRowB ? kCount : 1][kTN];
#pragma unroll
    for (int u = 0; u < kCount; ++u) {
      const int kb = kb0 + u * kFewWaves;
#pragma unroll
      for (int i = 0; i < kTN; ++i) {
        if constexpr (kRowB) {
#pragma unroll
          for (int r = 0; r < 4; ++r) sr[u][i][r] = p.bs[kb * p.lbs + brow[i][r]];
        } else {
          sb[u][i] = p.bs[kb * p.lbs + ((n0 + i * 16) >> 7)];
        }
      }
#pragma unroll
      for (int j = 0; j < kTM; ++j) {
        if constexpr (kCodes) {
          const i32x4* s = (const i32x4*)(a[j] + (int64_t)kb * kBlock);
          fa[u][j] = join(s[0], s[1]);
          sa[u][j] = p.as[kb * p.las + (arow[j] >> p.a_shift)];
        } else {
          const i32x4* s = (const i32x4*)(lds + arow[j] * kp + kb * kBlock + quad * 32);
          fa[u][j] = join(s[0], s[1]);
          sa[u][j] = lds_scales[kb * (int)p.m + arow[j]];
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kCount; ++u)
#pragma unroll
      for (int i = 0; i < kTN; ++i)
#pragma unroll
        for (int j = 0; j < kTM; ++j) {
          const f32x4 d = mfma128(fb[u][i], fa[u][j]);
#pragma unroll
          for (int r = 0; r < 4; ++r) acc[i][j][r] += d[r] * (sa[u][j] * (kRowB ? sr[kRowB ? u : 0][i][r] : sb[u][i]));
        }
  };
  int kb = wave;
  bool loaded = false;
  typedef std::integral_constant<int, kMost> most;
  if (kb + (kMost - 1) * kFewWaves < p.kb) {
    load_b(kb, most());
    loaded = true;
  }
  if constexpr (!kCodes) {
    // 16 threads to a block of a row
    for (int unit = t / 16; unit < (int)p.m * p.kb; unit += kFewWaves * 4) {
      const int row = unit / p.kb, k = unit % p.kb, c = (t & 15) * 8;
      float v[8], m = 0.0f;
      load8<X, kVec>(few.x + row * few.ldx, k * kBlock + c, (int)p.k - k * kBlock - c, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
      m = fmaxf(max16(m), kAmaxFloor);
      const float f = kE4m3Max / m;
      *(u32x2*)(lds + row * kp + k * kBlock + c) = u32x2{codes4(v[0], v[1], v[2], v[3], f), codes4(v[4], v[5], v[6], v[7], f)};
      if (c == 0) lds_scales[k * (int)p.m + row] = m / kE4m3Max;
    }
    __syncthreads();
  }
  for (; kb + (kMost - 1) * kFewWaves < p.kb; kb += kMost * kFewWaves) {
    if (!loaded) load_b(kb, most());
    loaded = false;
    work(kb, most());
  }
  auto rest = [&](auto count) {
    constexpr int kCount = decltype(count)::value;
    if (kCount < kMost && kb + (kCount - 1) * kFewWaves < p.kb) {
      load_b(kb, count);
      work(kb, count);
      kb += kCount * kFewWaves;
    }
  };
  if constexpr (kMost > 4) rest(std::integral_constant<int, 4>());
  if constexpr (kMost > 2) rest(std::integral_constant<int, 2>());
  rest(std::integral_constant<int, 1>());
#pragma unroll
  for (int i = 0; i < kTN; ++i)
#pragma unroll
    for (int j = 0; j < kTM; ++j) red[wave][i * kTM + j][lane] = acc[i][j];
  __syncthreads();
  for (int e = t; e < kTN * kTM * 64; e += kFewWaves * 64) {
    const int s = e / 64, l = e % 64;
    f32x4 v = red[0][s][l];
#pragma unroll
    for (int w = 1; w < kFewWaves; ++w) v += red[w][s][l];
    put4_any(p, s % kTM * 16 + (l & 15), n0 + s / kTM * 16 + (l >> 4) * 4, v);
  }
}

// ---------------------------------------------------------------- launches
constexpr int64_t kFewRows = 64;     // most rows of A that k_few takes
constexpr int64_t kFewSlots = 256;   // workgroups of k_few that the card takes one to a CU
// A workgroup of k_few gets 35 GB/s of both operands (16 rows of B, those of A),
// its CU's reads under way being what bounds it.  With fewer workgroups than
// CUs, k is split over others, into parts of 32 KiB at least, and the parts
// joined, where that saves more than the 2.9 us that joining takes.  Measured,
// without and with: 1 x 1024 x 14336 10.8 and 7.7 us, 16 rows of it 15.4 and
// 9.0, 64 rows 34.8 and 14.1; 4 x 1024 x 8192 7.9 and 6.7; 64 x 768 x 4096 11.6
// and 8.0; about where it begins, 1 x 1024 x 8192 6.9 and 6.4, 16 x 1024 x 4096
// 6.0 and 6.6, 8 x 2048 x 8192 8.6 and 8.3.
// few_part: blocks along k to a part (all of them: no split).
int few_part(int64_t m, int64_t n, int64_t k) {
  const int64_t kb = cdiv(k, kBlock), slots = kFewSlots / cdiv(n, 16);
  const double bytes = (double)(m + 16) * (double)k;
  int64_t parts = (int64_t)(bytes / 32768.0);
  if (parts > slots) parts = slots;
  if (parts < 2 || (1.0 - 1.0 / (double)parts) * bytes < 35e3 * 2.9) return (int)kb;
  return (int)cdiv(kb, parts);
}
size_t few_bytes(int64_t m, int64_t n, int64_t k) {
  const int64_t parts = cdiv(cdiv(k, kBlock), few_part(m, n, k));
  return parts == 1 ? 0 : (size_t)(parts * m * cdiv(n, 4) * 16);
}
void split_few(Product& p) {
  p.whole = few_part(p.m, p.n, p.k);
  p.splits = (int)cdiv(p.kb, p.whole);
}
hipError_t join_few(const Product& p, hipStream_t st) {
  const hipError_t e = launched();
  if (e != hipSuccess || p.splits == 1) return e;
  k_join_few<<<dim3((uint32_t)cdiv(p.m * cdiv(p.n, 4), 256)), 256, 0, st>>>(p);
  return launched();
}

// k_few rounds A itself (one launch less) where that is little beside its part
// of B: every workgroup does it, and a CU takes two at a time.  Measured, with
// and without: 1 x 768 x 768 2.9 and 4.3 us, 16 rows of it 3.9 and 4.9, 2 x 7168
// x 8192 15.4 and 16.2, 2 x 11008 x 4096 13.4 and 13.2, 4 of it 15.7 and 13.7.
constexpr int64_t kRoundRows = 16, kRoundCodes = 16384;

bool rounds_itself(int64_t m, int64_t n, int64_t k) {
  return k > 0 && m <= kRoundRows && m * few_part(m, n, k) * kBlock * cdiv(n, 16 * 512) <= kRoundCodes;
}

hipError_t launch_few(Product p, hipStream_t st) {
  // more rows of B than one launch takes: several (they are not split along k)
  constexpr int64_t kMost = most_groups(kFewWaves * 64) / 8 * kBlock;
  while (p.n > kMost) {
    Product part = p;
    part.n = kMost;
    const hipError_t e = launch_few(part, st);
    if (e != hipSuccess) return e;
    p.n -= kMost;
    p.b += kMost * p.ldb;
    p.bs += kMost >> p.b_shift;
    p.c = (char*)p.c + kMost * type_bytes(p.c_dtype);
  }
  split_few(p);
  const Few<uint8_t> few = {p.a, p.lda};
  // 32 rows of B to a wave halve the reads of A; taken where 16 are more than a
  // workgroup to each CU.  Measured with 16 and with 32: 17 x 7168 x 8192 20.8
  // and 17.1 us, 64 x 5120 x 5120 26.3 and 18.0, 64 x 4096 x 4096 11.8 and 14.3,
  // 4 x 7168 x 8192 14.9 and 15.6.
  const bool wide = p.m > 4 && p.n > 16 * kFewSlots;
  const dim3 g((uint32_t)cdiv(p.n, wide ? 32 : 16), p.splits);
  auto go = [&](auto k) { k<<<g, kFewWaves * 64, 0, st>>>(p, few); };
  const bool rows = p.b_shift == 0;
  if (p.m <= 16 && wide) rows ? go(k_few<uint8_t, 1, 2, true, true>) : go(k_few<uint8_t, 1, 2, false, true>);
  else if (p.m <= 16) rows ? go(k_few<uint8_t, 1, 1, true, true>) : go(k_few<uint8_t, 1, 1, false, true>);
  else if (p.m <= 32 && wide) rows ? go(k_few<uint8_t, 2, 2, true, true>) : go(k_few<uint8_t, 2, 2, false, true>);
  else if (p.m <= 32) rows ? go(k_few<uint8_t, 2, 1, true, true>) : go(k_few<uint8_t, 2, 1, false, true>);
  else if (wide) rows ? go(k_few<uint8_t, 4, 2, true, true>) : go(k_few<uint8_t, 4, 2, false, true>);
  else rows ? go(k_few<uint8_t, 4, 1, true, true>) : go(k_few<uint8_t, 4, 1, false, true>);
  return join_few(p, st);
}

template <typename X>
hipError_t launch_few_round(Product p, const X* x, int64_t ldx, hipStream_t st) {
  split_few(p);
  const Few<X> few = {x, ldx};
  const bool vec = aligned(x, 16) && p.k % 8 == 0 && ldx * (int64_t)sizeof(X) % 16 == 0;
  const dim3 g((uint32_t)cdiv(p.n, 16), p.splits);
  const size_t lds = (size_t)(p.m * p.whole * (kBlock + 4));
  auto go = [&](auto k) { k<<<g, kFewWaves * 64, lds, st>>>(p, few); };
  if (p.b_shift == 0) vec ? go(k_few<X, 1, 1, true, true>) : go(k_few<X, 1, 1, true, false>);
  else vec ? go(k_few<X, 1, 1, false, true>) : go(k_few<X, 1, 1, false, false>);
  return join_few(p, st);
}

template <int kBM, int kBN, int kWM, int kWN>
hipError_t launch_product(const Product& p, hipStream_t st) {
  constexpr int kLds = 2 * (kBM + kBN) * (kBlock + 4);
  const int64_t tm = cdiv(p.m, kBM), tn = cdiv(p.n, kBN), split = tm * tn - p.whole;
  auto k = p.b_shift == 0 ? k_product<kBM, kBN, kWM, kWN, true> : k_product<kBM, kBN, kWM, kWN, false>;
  k<<<dim3((uint32_t)(p.whole + split * p.splits)), kWM * kWN * 64, kLds, st>>>(p, (int)tm, (int)tn);
  const hipError_t e = launched();
  if (e != hipSuccess || split == 0) return e;
  k_join<kBM, kBN><<<dim3((uint32_t)(split * (kBM * kBN / 1024))), 256, 0, st>>>(p, (int)tm, (int)tn);
  return launched();
}

// How a product is cut up, a function of the sizes alone.  The card takes 256
// tiles of 256 x 256 at a time, or 512 of 128 x 128.  Whole rounds of tiles are
// made by a workgroup each; the tiles of the last, unfilled round are split
// along k so that they fill it, and their parts joined.  Of the two tile sizes,
// each with and without the split, the one with the least estimated time is
// taken: a block of 128 along k takes a round 1.8 us (256 x 256) or 1.1 us
// (128 x 128: 18 % slower for the same work), a launch and the tile's begin and
// end 4 us, joining 3 us and the parts' way to memory and back at 4 TB/s.
struct Plan {
  int tile;     // 0: 256 x 256, 1: 128 x 128
  int whole, splits;
  double us;
};
Plan plan_of(int64_t m, int64_t n, int64_t k) {
  const int64_t kb = cdiv(k, kBlock);
  Plan best = {0, 0, 1, 0.0};
  for (int tile = 0; tile < 2; ++tile) {
    const int64_t side = tile == 0 ? 256 : 128, slots = tile == 0 ? 256 : 512;
    const double step = tile == 0 ? 1.8 : 1.1;
    const int64_t tiles = cdiv(m, side) * cdiv(n, side), rounds = tiles / slots, left = tiles % slots;
    if (tiles + slots > most_groups(tile == 0 ? 512 : 256)) continue;
    auto consider = [&](int64_t whole, int64_t splits, double us) {
      if (best.us == 0.0 || us < best.us) best = {tile, (int)whole, (int)splits, us};
    };
    consider(tiles, 1, 4.0 + step * (double)kb * (double)(rounds + (left > 0)));
    int64_t splits = left ? slots / left : 1;
    if (splits > kb / 4) splits = kb / 4;
    if (splits > 1)
      consider(rounds * slots, splits, 7.0 + step * ((double)(kb * rounds) + (double)cdiv(kb, splits)) +
                                           (double)(left * splits * side * side) * 8.0 / 4e6);
  }
  return best;
}
int64_t slots_bytes(const Plan& plan, int64_t m, int64_t n) {
  const int64_t side = plan.tile == 0 ? 256 : 128, tiles = cdiv(m, side) * cdiv(n, side);
  return plan.splits == 1 ? 0 : (tiles - plan.whole) * plan.splits * side * side * 4;
}

hipError_t product(Product p, hipStream_t st) {
  if (p.kb == 0) {
    if (p.accumulate) return hipSuccess;
    const int64_t grid = cdiv(p.m * cdiv(p.n, 4), 256);
    k_zero<<<dim3((uint32_t)(grid < 65536 ? grid : 65536)), 256, 0, st>>>(p);
    return launched();
  }
  if (p.m <= kFewRows) return launch_few(p, st);
  const Plan plan = plan_of(p.m, p.n, p.k);
  if (plan.us == 0.0) return hipErrorInvalidValue;
  p.whole = plan.whole;
  p.splits = plan.splits;
  return plan.tile == 0 ? launch_product<256, 256, 4, 2>(p, st) : launch_product<128, 128, 2, 2>(p, st);
}

Product make_product(const sim_blocks* a, const sim_blocks* b, int64_t m, int64_t n, int64_t k, void* c, int c_dtype,
                     int64_t ldc, int accumulate, void* ws) {
  Product p;
  p.a = a->codes; p.b = b->codes; p.as = a->scales; p.bs = b->scales;
  p.lda = a->ld; p.ldb = b->ld; p.las = a->ld_s; p.lbs = b->ld_s;
  p.m = m; p.n = n; p.k = k; p.kb = (int)cdiv(k, kBlock);
  p.a_shift = a->block_rows == 1 ? 0 : 7;
  p.b_shift = b->block_rows == 1 ? 0 : 7;
  p.c = c; p.ldc = ldc; p.c_dtype = c_dtype; p.accumulate = accumulate;
  p.part = (float*)ws; p.whole = 0; p.splits = 1;
  return p;
}

constexpr int64_t kMaxSize = (int64_t)1 << 31;   // of one side of a matrix
constexpr int64_t kMaxK = SIM_MATMUL_MAX_K;         // of the side that is summed over, and of a row of codes:
                                                 // 256 rows are less than 2^32 bytes

int code_of(hipError_t e) {
  return e == hipSuccess ? SIM_OK : e == hipErrorInvalidValue ? SIM_EINVAL : SIM_EHIP;
}

}  // namespace
}  // namespace ops
}  // namespace hetsim

using namespace hetsim::ops;

extern "C" int sim_op_quantize(const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, const sim_blocks* q,
                               const sim_blocks* qt, void* stream) {
  if (q && !q->codes) q = nullptr;
  if (qt && !qt->codes) qt = nullptr;
  if ((!q && !qt) || !type_bytes(dtype) || rows < 0 || cols < 0 || rows >= kMaxSize || cols >= kMaxSize || ld < cols)
    return SIM_EINVAL;
  if (q && !valid_blocks(q, rows, cols)) return SIM_EINVAL;
  if (qt && !valid_blocks(qt, cols, rows)) return SIM_EINVAL;
  if (q && qt && q->block_rows != qt->block_rows) return SIM_EINVAL;
  if (rows == 0 || cols == 0) return SIM_OK;
  if (!x || !aligned(x, (size_t)type_bytes(dtype))) return SIM_EINVAL;
  return code_of(quantize_any(x, dtype, rows, cols, ld, q, qt, (hipStream_t)stream));
}

extern "C" size_t sim_op_matmul_workspace(int64_t m, int64_t n, int64_t k) {
  if (m <= 0 || n <= 0 || k <= 0 || m >= kMaxSize || n >= kMaxSize || k > kMaxK) return 0;
  return m <= kFewRows ? few_bytes(m, n, k) : (size_t)slots_bytes(plan_of(m, n, k), m, n);
}

extern "C" int sim_op_matmul(const sim_blocks* a, const sim_blocks* b, int64_t m, int64_t n, int64_t k, void* c,
                             int c_dtype, int64_t ldc, int accumulate, void* workspace, size_t workspace_bytes,
                             void* stream) {
  if (m < 0 || n < 0 || k < 0 || m >= kMaxSize || n >= kMaxSize || k > kMaxK || ldc < n || !type_bytes(c_dtype))
    return SIM_EINVAL;
  if (!valid_blocks(a, m, k) || !valid_blocks(b, n, k) || a->ld > kMaxK || b->ld > kMaxK) return SIM_EINVAL;
  if (m == 0 || n == 0) return SIM_OK;
  if (!c || !aligned(c, (size_t)type_bytes(c_dtype))) return SIM_EINVAL;
  const size_t need = sim_op_matmul_workspace(m, n, k);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16)))) return SIM_EINVAL;
  return code_of(product(make_product(a, b, m, n, k, c, c_dtype, ldc, accumulate != 0, workspace), (hipStream_t)stream));
}

// Codes and scales of the activations, then the product's own workspace.
static size_t linear_codes(int64_t tokens, int64_t k) { return (size_t)(tokens * pad_block(k)); }
static size_t linear_scales(int64_t tokens, int64_t k) { return (size_t)((cdiv(k, kBlock) * tokens * 4 + 15) / 16 * 16); }

extern "C" size_t sim_op_linear_workspace(int64_t tokens, int64_t n, int64_t k) {
  if (tokens <= 0 || n <= 0 || k <= 0 || tokens >= kMaxSize || n >= kMaxSize || k > kMaxK) return 0;
  if (rounds_itself(tokens, n, k)) return few_bytes(tokens, n, k);
  return linear_codes(tokens, k) + linear_scales(tokens, k) + sim_op_matmul_workspace(tokens, n, k);
}

extern "C" int sim_op_linear(const void* x, int dtype, int64_t ldx, const sim_blocks* w, int64_t tokens, int64_t n,
                             int64_t k, void* y, int64_t ldy, void* workspace, size_t workspace_bytes, void* stream) {
  if (tokens < 0 || n < 0 || k < 0 || tokens >= kMaxSize || n >= kMaxSize || k > kMaxK || ldx < k || ldy < n ||
      !type_bytes(dtype) || !valid_blocks(w, n, k) || w->ld > kMaxK)
    return SIM_EINVAL;
  if (tokens == 0 || n == 0) return SIM_OK;
  if ((k && !x) || !y || !aligned(x, (size_t)type_bytes(dtype)) || !aligned(y, (size_t)type_bytes(dtype))) return SIM_EINVAL;
  const size_t need = sim_op_linear_workspace(tokens, n, k);
  if (workspace_bytes < need || (need && (!workspace || !aligned(workspace, 16)))) return SIM_EINVAL;
  if (rounds_itself(tokens, n, k)) {
    sim_blocks none = {};
    const Product p = make_product(&none, w, tokens, n, k, y, dtype, ldy, 0, workspace);
    const hipStream_t st = (hipStream_t)stream;
    return code_of(dtype == SIM_BF16   ? launch_few_round(p, (const bf16*)x, ldx, st)
                   : dtype == SIM_FP16 ? launch_few_round(p, (const fp16*)x, ldx, st)
                                       : launch_few_round(p, (const float*)x, ldx, st));
  }
  sim_blocks q;
  q.codes = (uint8_t*)workspace;
  q.ld = pad_block(k);
  q.scales = (float*)((uint8_t*)workspace + linear_codes(tokens, k));
  q.ld_s = tokens;
  q.block_rows = 1;
  if (k) {
    const hipError_t e = quantize_any(x, dtype, tokens, k, ldx, &q, nullptr, (hipStream_t)stream);
    if (e != hipSuccess) return code_of(e);
  }
  uint8_t* rest = (uint8_t*)q.scales + linear_scales(tokens, k);
  return code_of(product(make_product(&q, w, tokens, n, k, y, dtype, ldy, 0, rest), (hipStream_t)stream));
}
