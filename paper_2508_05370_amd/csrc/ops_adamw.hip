// ops_adamw.hip -- one AdamW step over many tensors, moments in 32 or 8 bits.
//
// Every element is read and written once, so memory bounds it: 28 B for each
// parameter with 32-bit moments and gradients, 16 to 18 B with 8-bit moments,
// a 16-bit gradient and copy.  405M parameters with 8-bit moments take 1.21 ms,
// 5.4 TB/s; 125M with 32-bit ones 0.65 ms, 5.3 TB/s (a copy by the runtime
// reaches 4.7 to 4.9).  Tensors that do not start at 16 bytes go one element at a
// time: 125M 1.55 ms.  The 8-bit form was bound by the VALU at 115 operations an
// element, rounding by shifts and one quotient for each factor and scale: 1.33
// ms.  A workgroup takes one chunk of 2048 elements of
// one tensor; it finds the tensor by bisection over the chunk counts, which
// come with the launch.  Eight neighbours per thread: 16 threads hold one
// block of 128 moments, whose maximum crosses lanes.
#include <cmath>

#include "ops_common.h"

// No product is fused with a sum here: the moments' codes are reproducible only
// when every operation is rounded by itself.
#pragma clang fp contract(off)

namespace hetsim {
namespace ops {
namespace {

constexpr int kThreads = 256, kChunk = kThreads * 8;
constexpr int kTensors = 40;   // of one launch: the table is a kernel argument

struct Tensor {
  void* p;
  const void* grad;
  void* m;
  void* v;
  float* ms;
  float* vs;
  void* copy;
  int64_t n;
  uint64_t first;
  float keep;       // 1 - lr * weight_decay
  uint32_t vec;     // every pointer is a multiple of eight elements' size
};
struct Table {
  Tensor t[kTensors];
  uint32_t end[kTensors];   // chunks of tensors 0..i
  int n;
};
struct Step {
  float beta1, beta2, one_beta1, one_beta2, rate, power, eps;
  uint32_t key;
  const float* grad_scale;
  const uint32_t* skip;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0x9E3779B9u;
  x ^= x >> 15;
  x *= 0x85A308D3u;
  return x ^ (x >> 16);
}

// Rounding: an element's code is the value below or above it, up with the
// probability of the distance from the lower one; 16 bits r decide, up where
// r / 2^16 is at least what is missing to the upper value.  That is what
// v_cvt_sr_fp8_f32 does with r in the upper half of its random operand (equal
// to floor(x / spacing + r / 2^16) on 2^28 pairs of numbers, the range below
// 2^-6 with its constant spacing among them); NaN and infinities give NaN.

// The largest of a block; an infinity in it makes it one, a NaN does not count
// (its own code becomes one).
__device__ inline float block_max(const float v[8]) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
  return fmaxf(max16(m), kAmaxFloor);
}

template <bool kVec>
__device__ inline void load_codes(const uint8_t* p, int64_t have, float scale, float v[8]) {
  uint32_t w[2] = {0, 0};
  if constexpr (kVec) {
    if (have > 0) {
      const u32x2 a = *(const u32x2*)p;
      w[0] = a[0]; w[1] = a[1];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) w[i / 4] |= (uint32_t)p[i] << (8 * (i % 4));
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    v[4 * h + 0] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 0) * scale;
    v[4 * h + 1] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 1) * scale;
    v[4 * h + 2] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 2) * scale;
    v[4 * h + 3] = __builtin_amdgcn_cvt_f32_fp8((int)w[h], 3) * scale;
  }
}

template <bool kVec>
__device__ inline void store_codes(uint8_t* p, int64_t have, u32x2 c) {
  if constexpr (kVec) {
    if (have > 0) *(u32x2*)p = c;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < have) p[i] = (uint8_t)(c[i / 4] >> (8 * (i % 4)));
  }
}

// Byte i of the codes: x rounded with the upper half of r.
template <int i>
__device__ inline void put_code(u32x2& c, float x, uint32_t r) {
  c[i / 4] = (uint32_t)__builtin_amdgcn_cvt_sr_fp8_f32(x, (int)r, (int)c[i / 4], i % 4);
}
template <int i>
__device__ inline void put_codes(u32x2& cm, u32x2& cv, const float m[8], const float root[8], float fm, float fv, uint32_t key,
                                 uint32_t e) {
  if constexpr (i < 8) {
    const uint32_t r = mix(key ^ (e + i));
    put_code<i>(cm, m[i] * fm, r << 16);
    // (above zero, the smallest code at least; a NaN stays one)
    const float t = root[i] * fv;
    put_code<i>(cv, t > 0.0f ? fmaxf(t, 0x1p-9f) : t, r & 0xFFFF0000u);
    put_codes<i + 1>(cm, cv, m, root, fm, fv, key, e);
  }
}

// The bare instructions take numbers below 2^-126 for zero, which v and, with
// such an eps, the update's denominator can be.  So v is brought up by a power of
// four first where it is small; the denominator, where eps asks for it, by the
// caller's constants.  (sqrtf and a division, both rounded right: a layer of 1.8M
// parameters 9.05 us, so 8.65.)
__device__ inline float root_of(float v) {
  const bool small = v < 0x1p-96f;
  const float r = __builtin_amdgcn_sqrtf(small ? v * 0x1p32f : v);
  return small ? r * 0x1p-16f : r;
}

template <typename P, typename G, int kBits, bool kVec>
__device__ inline void chunk(const Tensor& t, const Step& s, int copy_dtype, int64_t at) {
  const int64_t have = t.n - at;
  float p[8], g[8], m[8], v[8], root[8];
  load8<P, kVec>((const P*)t.p, at, have, p);
  load8<G, kVec>((const G*)t.grad, at, have, g);
  if constexpr (kBits == 32) {
    load8<float, kVec>((const float*)t.m, at, have, m);
    load8<float, kVec>((const float*)t.v, at, have, v);
  } else {
    const bool any = have > 0;
    const float ms = any ? t.ms[at / kBlock] : 0.0f, vs = any ? t.vs[at / kBlock] : 0.0f;
    load_codes<kVec>((const uint8_t*)t.m + at, have, ms, m);
    load_codes<kVec>((const uint8_t*)t.v + at, have, vs, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = v[i] * v[i];
  }
  const float gs = s.grad_scale ? *s.grad_scale : 1.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float a = g[i] * gs;
    m[i] = s.beta1 * m[i] + s.one_beta1 * a;
    v[i] = s.beta2 * v[i] + s.one_beta2 * a * a;
    // (8-bit moments keep the root, so that one is rounded right; else, and in
    // the quotient, the last bit is lost beside the parameter's own)
    root[i] = kBits == 8 ? sqrtf(v[i]) : root_of(v[i]);
    p[i] = p[i] * t.keep - s.rate * m[i] * __builtin_amdgcn_rcpf(root[i] * s.power + s.eps);
  }
  store8<P, kVec>((P*)t.p, at, have, p);
  if (copy_dtype != SIM_NONE) {
    // the copy is of what p holds now
#pragma unroll
    for (int i = 0; i < 8; ++i) p[i] = (float)(P)p[i];
    if (copy_dtype == SIM_BF16) store8<bf16, kVec>((bf16*)t.copy, at, have, p);
    else if (copy_dtype == SIM_FP16) store8<fp16, kVec>((fp16*)t.copy, at, have, p);
    else store8<float, kVec>((float*)t.copy, at, have, p);
  }
  if constexpr (kBits == 32) {
    store8<float, kVec>((float*)t.m, at, have, m);
    store8<float, kVec>((float*)t.v, at, have, v);
  } else {
    // Both factors and both scales by one quotient: lane 0 of a quad makes the
    // first's, and so on.
    const float mm = block_max(m), mv = block_max(root);
    const bool second = threadIdx.x & 1, scale = threadIdx.x & 2;
    const float x = second ? mv : mm, quotient = (scale ? x : kE4m3Max) / (scale ? kE4m3Max : x);
    const float fm = row_move<0x00>(quotient), fv = row_move<0x55>(quotient);   // quad_perm 0 0 0 0, 1 1 1 1
    u32x2 cm = {0, 0}, cv = {0, 0};
    const uint64_t e = t.first + (uint64_t)at;   // (a multiple of eight)
    put_codes<0>(cm, cv, m, root, fm, fv, mix(s.key ^ (uint32_t)(e >> 32)), (uint32_t)e);
    store_codes<kVec>((uint8_t*)t.m + at, have, cm);
    store_codes<kVec>((uint8_t*)t.v + at, have, cv);
    const int lane = threadIdx.x & 15;
    if (lane == 2 || lane == 3) {
      const int64_t block = at / kBlock;      // (lane 0's: at is in the same block)
      if (block * kBlock < t.n) (lane == 2 ? t.ms : t.vs)[block] = quotient;
    }
  }
}

template <typename P, typename G, int kBits>
__global__ __launch_bounds__(kThreads) void k_adamw(Table tab, Step s, int copy_dtype) {
  if (s.skip && *s.skip) return;
  int lo = 0, hi = tab.n - 1;
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (blockIdx.x < tab.end[mid]) hi = mid;
    else lo = mid + 1;
  }
  const Tensor& t = tab.t[lo];
  const uint32_t c = blockIdx.x - (lo ? tab.end[lo - 1] : 0);
  const int64_t at = (int64_t)c * kChunk + threadIdx.x * 8;
  // a vector access needs all eight elements: the tensor's last few go one by one
  if (t.vec && (int64_t)(c + 1) * kChunk <= t.n) chunk<P, G, kBits, true>(t, s, copy_dtype, at);
  else chunk<P, G, kBits, false>(t, s, copy_dtype, at);
}

template <typename P, typename G>
hipError_t launch_pg(const Table& tab, const Step& s, int copy_dtype, int bits, hipStream_t st) {
  auto k = bits == 32 ? k_adamw<P, G, 32> : k_adamw<P, G, 8>;
  k<<<dim3(tab.end[tab.n - 1]), kThreads, 0, st>>>(tab, s, copy_dtype);
  return launched();
}
template <typename P>
hipError_t launch_p(const Table& tab, const Step& s, const sim_adamw_args& a, hipStream_t st) {
  switch (a.grad_dtype) {
    case SIM_BF16: return launch_pg<P, bf16>(tab, s, a.copy_dtype, a.state_bits, st);
    case SIM_FP16: return launch_pg<P, fp16>(tab, s, a.copy_dtype, a.state_bits, st);
    default: return launch_pg<P, float>(tab, s, a.copy_dtype, a.state_bits, st);
  }
}
hipError_t launch(const Table& tab, const Step& s, const sim_adamw_args& a, hipStream_t st) {
  switch (a.p_dtype) {
    case SIM_BF16: return launch_p<bf16>(tab, s, a, st);
    case SIM_FP16: return launch_p<fp16>(tab, s, a, st);
    default: return launch_p<float>(tab, s, a, st);
  }
}

}  // namespace
}  // namespace ops
}  // namespace hetsim

using namespace hetsim::ops;

extern "C" int sim_op_adamw(const sim_adamw_tensor* tensors, int64_t n, const sim_adamw_args* a, void* stream) {
  if (!a || n < 0 || (n && !tensors) || !type_bytes(a->p_dtype) || !type_bytes(a->grad_dtype)) return SIM_EINVAL;
  if (a->copy_dtype != SIM_NONE && !type_bytes(a->copy_dtype)) return SIM_EINVAL;
  if (a->state_bits != 8 && a->state_bits != 32) return SIM_EINVAL;
  // (written so that a NaN is refused)
  if (!(a->beta1 >= 0 && a->beta1 < 1 && a->beta2 >= 0 && a->beta2 < 1 && a->eps >= 0) || a->step < 1) return SIM_EINVAL;
  if (!(a->lr > -1e30 && a->lr < 1e30)) return SIM_EINVAL;
  if (!aligned(a->grad_scale, 4) || !aligned(a->skip, 4)) return SIM_EINVAL;
  const int pb = type_bytes(a->p_dtype), gb = type_bytes(a->grad_dtype), cb = type_bytes(a->copy_dtype);
  const int sb = a->state_bits / 8;
  for (int64_t i = 0; i < n; ++i) {
    const sim_adamw_tensor& t = tensors[i];
    if (t.n < 0 || t.n > ((int64_t)1 << 42) || t.first % kBlock != 0) return SIM_EINVAL;
    if (t.n == 0) continue;
    if (!t.p || !t.grad || !t.m || !t.v || !aligned(t.p, pb) || !aligned(t.grad, gb) || !aligned(t.m, sb) ||
        !aligned(t.v, sb))
      return SIM_EINVAL;
    if (a->state_bits == 8 && (!t.m_scale || !t.v_scale || !aligned(t.m_scale, 4) || !aligned(t.v_scale, 4)))
      return SIM_EINVAL;
    if (cb && (!t.copy || !aligned(t.copy, cb))) return SIM_EINVAL;
  }
  Step s;
  s.beta1 = (float)a->beta1;
  s.beta2 = (float)a->beta2;
  s.one_beta1 = (float)(1.0 - a->beta1);
  s.one_beta2 = (float)(1.0 - a->beta2);
  s.rate = (float)(a->lr / (1.0 - std::pow(a->beta1, (double)a->step)));
  s.power = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, (double)a->step)));
  s.eps = (float)a->eps;
  // (a root is zero or at least 2^-75: only eps makes a denominator below 2^-126;
  // both sides of the quotient times 2^24 then)
  if (s.eps > 0.0f && s.eps < 0x1p-126f)
    for (float* x : {&s.rate, &s.power, &s.eps}) *x *= 0x1p24f;
  s.key = mix(mix(mix((uint32_t)a->seed) ^ (uint32_t)(a->seed >> 32)) ^ (uint32_t)a->step);
  s.grad_scale = a->grad_scale;
  s.skip = a->skip;
  Table tab;
  tab.n = 0;
  int64_t chunks = 0;
  // as many tensors to a launch as its table and its grid hold; a tensor of
  // more chunks than a grid has goes in several pieces
  constexpr int64_t kGrid = most_groups(kThreads);
  for (int64_t i = 0; i < n; ++i) {
    int64_t done = 0;
    while (done < tensors[i].n) {
      const sim_adamw_tensor& t = tensors[i];
      const int64_t take = t.n - done < (kGrid - chunks) * kChunk ? t.n - done : (kGrid - chunks) * kChunk;
      Tensor& d = tab.t[tab.n];
      d.p = (char*)t.p + done * pb;
      d.grad = (const char*)t.grad + done * gb;
      d.m = (char*)t.m + done * sb;
      d.v = (char*)t.v + done * sb;
      d.ms = a->state_bits == 8 ? t.m_scale + done / kBlock : nullptr;
      d.vs = a->state_bits == 8 ? t.v_scale + done / kBlock : nullptr;
      d.copy = cb ? (char*)t.copy + done * cb : nullptr;
      d.n = take;
      d.first = t.first + (uint64_t)done;
      d.keep = (float)(1.0 - a->lr * (double)t.weight_decay);
      // 16 bytes at most are one access
      auto ok = [](const void* p, int bytes) { return aligned(p, bytes * 8 > 16 ? 16 : bytes * 8); };
      d.vec = ok(d.p, pb) && ok(d.grad, gb) && ok(d.m, sb) && ok(d.v, sb) && (!cb || ok(d.copy, cb));
      chunks += cdiv(take, kChunk);
      tab.end[tab.n++] = (uint32_t)chunks;
      done += take;
      if (tab.n == kTensors || chunks == kGrid) {
        if (launch(tab, s, *a, (hipStream_t)stream) != hipSuccess) return SIM_EHIP;
        tab.n = 0;
        chunks = 0;
      }
    }
  }
  if (tab.n && launch(tab, s, *a, (hipStream_t)stream) != hipSuccess) return SIM_EHIP;
  return SIM_OK;
}
