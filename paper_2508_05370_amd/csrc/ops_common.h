// ops_common.h -- what the layer operators' kernels share: element types,
// vector loads and stores, reductions over lanes, argument checks.
#pragma once
#include <hip/hip_bf16.h>
#include <hip/hip_fp16.h>
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "hetsim_ops.h"

namespace hetsim {
namespace ops {

typedef __bf16 bf16;
typedef _Float16 fp16;
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kBlock = SIM_BLOCK;
constexpr float kE4m3Max = 448.0f;
constexpr float kAmaxFloor = 0x1p-110f;   // 448 / it is finite, it / 448 a normal number

inline int64_t cdiv(int64_t a, int64_t b) { return a / b + (a % b != 0); }
inline int64_t pad_block(int64_t a) { return cdiv(a, kBlock) * kBlock; }
inline bool aligned(const void* p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }
inline int type_bytes(int dtype) { return dtype == SIM_FP32 ? 4 : dtype == SIM_BF16 || dtype == SIM_FP16 ? 2 : 0; }

// Eight consecutive elements, as they are in memory, from column c of a row on.
// kVec: c is a multiple of eight, as are the row's length and alignment (a
// column past the row is read as the row's first ones: no branch, and no
// address outside); otherwise the first `have` (at most 8, may be <= 0) are
// read and the rest are zero.
template <typename T>
struct Raw {
  // (16 bytes are what callers make sure of, for 32-bit elements too)
  typedef T t8 __attribute__((ext_vector_type(8), aligned(16)));
  t8 v;
};
static_assert(alignof(Raw<float>::t8) == 16 && alignof(Raw<bf16>::t8) == 16, "an access of eight elements asks for 16 bytes' alignment");
// (a 32-bit column's place is a 32-bit number of bytes, so that the row's
// address stays in scalar registers)
template <typename T, typename I>
__device__ inline T* column(T* row, I c) {
  if constexpr (sizeof(I) == 4) return (T*)((std::conditional_t<std::is_const_v<T>, const char, char>*)row + (uint32_t)c * (uint32_t)sizeof(T));
  else return row + c;
}
template <typename T, bool kVec, typename I>
__device__ inline Raw<T> fetch8(const T* row, I c, I have) {
  Raw<T> r;
  if constexpr (kVec) {
    r.v = *(const typename Raw<T>::t8*)column(row, have > 0 ? c : 0);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) r.v[i] = i < have ? column(row, c)[i] : (T)0.0f;
  }
  return r;
}
// The same as 32-bit floats, zero past the row.
template <typename T, bool kVec, typename I>
__device__ inline void load8(const T* row, I c, I have, float v[8]) {
  const Raw<T> r = fetch8<T, kVec>(row, c, have);
#pragma unroll
  for (int i = 0; i < 8; ++i) v[i] = kVec && have <= 0 ? 0.0f : (float)r.v[i];
}

template <typename T, bool kVec, typename I>
__device__ inline void store8(T* row, I c, I have, const float v[8]) {
  T* p = column(row, c);
  if constexpr (kVec) {
    if (have <= 0) return;
    if constexpr (sizeof(T) == 4) {
      *(f32x4*)p = f32x4{v[0], v[1], v[2], v[3]};
      *((f32x4*)p + 1) = f32x4{v[4], v[5], v[6], v[7]};
    } else {
      typedef T t8 __attribute__((ext_vector_type(8)));
      t8 a;
#pragma unroll
      for (int i = 0; i < 8; ++i) a[i] = (T)v[i];
      *(t8*)p = a;
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) p[i] = (T)v[i];
  }
}

// Four codes of a block from four elements and the block's factor.
__device__ inline uint32_t codes4(float a, float b, float c, float d, float f) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a * f, b * f, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c * f, d * f, r, true);
}

// Lanes of a row of 16 combined without LDS: with the neighbour, the pair, the
// four and the eight beside; every lane gets the result.  All 16 must be active.
template <int kCtrl>
__device__ inline float row_move(float v) {
  return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), kCtrl, 0xF, 0xF, true));
}
__device__ inline float max16(float v) {
  v = fmaxf(v, row_move<0xB1>(v));    // quad_perm 1 0 3 2
  v = fmaxf(v, row_move<0x4E>(v));    // quad_perm 2 3 0 1
  v = fmaxf(v, row_move<0x141>(v));   // row_half_mirror
  return fmaxf(v, row_move<0x140>(v));   // row_mirror
}
__device__ inline float sum16(float v) {
  v += row_move<0xB1>(v);
  v += row_move<0x4E>(v);
  v += row_move<0x141>(v);
  return v + row_move<0x140>(v);
}
// Sum over the wave, the same in every lane.
__device__ inline float sum64(float v) {
  v = sum16(v);
  const auto lane = [&](int l) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), l)); };
  return (lane(0) + lane(16)) + (lane(32) + lane(48));
}

// Workgroups that one launch may have: it counts its threads in 32 bits.
constexpr int64_t most_groups(int threads) { return (((int64_t)1 << 32) - 1) / threads; }

inline hipError_t launched() { return hipGetLastError(); }

// A block form that a call reads or writes: rows x cols elements.
inline bool valid_blocks(const sim_blocks* b, int64_t rows, int64_t cols) {
  if (!b || (b->block_rows != 1 && b->block_rows != kBlock)) return false;
  if (rows == 0 || cols == 0) return true;
  if (!b->codes || !b->scales || !aligned(b->codes, 16) || !aligned(b->scales, 4)) return false;
  if (b->ld % 16 != 0 || b->ld < pad_block(cols)) return false;
  return b->ld_s >= cdiv(rows, b->block_rows);
}

}  // namespace ops
}  // namespace hetsim
