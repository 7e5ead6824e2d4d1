// ops_norm.hip -- the end of one block and the beginning of the next: norm of
// the block's output, gate and residual scale, norm of the sum; and their
// gradients.
//
// Every row is read once, stays in registers as 32-bit floats and leaves once,
// so memory bounds both passes: 8 B per element forward and 12 B backward with
// 16-bit data.  Thread t of a row's T threads holds the groups of eight
// neighbours t, t + T, ...: 16-byte accesses, and 16 neighbouring threads hold
// one block of 128 for the output in 8 bits.
//
// Two kinds of rows take several times what their bytes do.  Ones that are not
// whole multiples of eight elements, or do not start at 16 bytes, go one element
// at a time (kVec false): 8192 x 8191 forward 332 us and backward 458, where 8192 x
// 8192 take 115 and 169; 4096 x 4099 95 and 134, for 24.5 and 42.  And long ones,
// with more groups per thread than the registers hold, spill: backward from 8193
// channels on (layer norms a little from 4097 on), forward from 16385 on (with a
// stream in 32 bits a little from 12289 on).  By the
// compiler's report a lane of the backward pass keeps 15 to 112 registers in
// memory at up to 12288 channels (4096 rows, RMS: 167 us, 3.6 TB/s), 109 to 280 at
// up to 16384 (444 us, 1.8 TB/s) and 611 to 1329 beyond (2048 x 32768 1188 us, 0.7
// TB/s; forward, with up to 449, 336 us).
#include <type_traits>

#include "ops_common.h"

namespace hetsim {
namespace ops {
namespace {

// Sums of K values over a row's threads, which are `waves` whole waves from
// wave `first` on (all of a workgroup's rows sum at the same time).  `red` holds
// two sets of K floats for each of 16 waves, used in turn, so that one barrier
// for a sum is enough.
template <int K>
__device__ inline void row_sum(float v[K], float* red, int waves, int wave, int first, int& half) {
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = sum64(v[k]);
  if (waves == 1) return;
  float* r = red + half * 16 * K;
  half ^= 1;
  if ((threadIdx.x & 63) == 0) {
#pragma unroll
    for (int k = 0; k < K; ++k) r[k * 16 + wave] = v[k];
  }
  __syncthreads();
  const int l = threadIdx.x & 15;
#pragma unroll
  for (int k = 0; k < K; ++k) v[k] = sum16(l < waves ? r[k * 16 + first + l] : 0.0f);
}

// Parameters of a row, eight at a time; NULL: `other`.  Zero past the row.
template <bool kVec>
__device__ inline void param8(const float* p, int c, int have, float other, float v[8]) {
  if (p) {
    load8<float, kVec>(p, c, have, v);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = i < have ? other : 0.0f;
  }
}

constexpr int kThreads = 512;   // most of a row
// Groups of eight per thread up to which the weights stay in registers (8192 x
// 8192 forward 114 us, with one workgroup to a CU; reading them for every row,
// with two, 122).
constexpr int kHold = 2;

struct Fwd {
  int64_t rows, hidden, ld_h, ld_y, ld_ho, ld_x, rows_per_gate, ld_q, ld_s;
  int post, pre;
  float alpha, beta, eps;
  const void *h, *y, *gate;
  const float *pw, *pb, *qw, *qb;   // post weight and bias, pre weight and bias
  void *ho, *x;
  uint8_t* q;
  float *s, *post_stats, *pre_stats;
};

// Mean and reciprocal deviation of the row that v holds, which is left less its
// mean (elements past the row are zero, and stay so).
template <int kN>
__device__ inline void moments(float v[kN][8], const int have[kN], int kind, float inv, float eps, float* red,
                               int waves, int wave, int first, int& half, float& mean, float& rstd) {
  mean = 0.0f;
  if (kind == SIM_NORM_LAYER) {
    float a[1] = {0.0f};
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) a[0] += v[j][i];
    row_sum<1>(a, red, waves, wave, first, half);
    mean = a[0] * inv;
  }
  float a[1] = {0.0f};
  if (kind == SIM_NORM_LAYER) {
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        v[j][i] = i < have[j] ? v[j][i] - mean : 0.0f;
        a[0] += v[j][i] * v[j][i];
      }
  } else {
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) a[0] += v[j][i] * v[j][i];
  }
  row_sum<1>(a, red, waves, wave, first, half);
  rstd = 1.0f / sqrtf(a[0] * inv + eps);
}

// A workgroup takes rows_each rows one after another for each group of
// `per_row` threads, the next row on its way while one is worked on.  8192 x 8192
// in 16 bits: 115 us, 4.7 TB/s of 8 B per element, and with x in 8 bits 110, 4.3
// TB/s of 7 B (one row to a workgroup and branches around what is past the row:
// 136 to 159).
template <typename A, typename R, int kN, bool kVec>
__global__ __launch_bounds__(kThreads) void k_norm(Fwd p, int per_row, int rows_each) {
  __shared__ float red[32];
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64), waves = per_row / 64;
  const int mine = wave / waves, first = mine * waves, tr = threadIdx.x - first * 64, groups = blockDim.x / per_row;
  // rows mine, mine + groups, ... of the workgroup's (all threads meet the barriers)
  const int64_t row0 = (int64_t)blockIdx.x * groups * rows_each + mine;
  int half = 0;
  const float inv = 1.0f / (float)p.hidden;
  int c[kN], have[kN];
  Raw<R> nh[kN];
  Raw<A> ny[kN];
  auto fetch = [&](int64_t row) {
    row = min(row, p.rows - 1);
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      nh[j] = fetch8<R, kVec>((const R*)p.h + row * p.ld_h, c[j], have[j]);
      if (p.y) ny[j] = fetch8<A, kVec>((const A*)p.y + row * p.ld_y, c[j], have[j]);
    }
  };
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    c[j] = (j * per_row + tr) * 8;
    have[j] = (int)p.hidden - c[j];
  }
  fetch(row0);
  // The weights, zero past the row: beta gate post_weight, and the pre weight.
  // Up to kHold groups of eight per thread they stay in registers.
  constexpr int kKept = kN <= kHold ? kN : 1;
  float kept_gw[kKept][8], kept_qw[kKept][8];
  uint32_t gate_row = 0;
  auto load_gw = [&](int j, float gw[8]) {
    float w[8];
    param8<kVec>(p.pw, c[j], have[j], 1.0f, gw);
    if (p.gate) {
      load8<A, kVec>((const A*)p.gate + (int64_t)gate_row * p.hidden, c[j], have[j], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) gw[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) gw[i] *= p.beta;
  };
  auto keep_gw = [&]() {
    if constexpr (kN <= kHold) {
#pragma unroll
      for (int j = 0; j < kN; ++j) load_gw(j, kept_gw[j]);
    }
  };
  if constexpr (kN <= kHold) {
#pragma unroll
    for (int j = 0; j < kN; ++j) param8<kVec>(p.qw, c[j], have[j], 1.0f, kept_qw[j]);
  }
  keep_gw();
  for (int e = 0; e < rows_each; ++e) {
    const int64_t row_at = row0 + (int64_t)e * groups;
    if (row_at - mine >= p.rows) break;           // (the whole workgroup)
    const bool real = row_at < p.rows;
    const int64_t row = real ? row_at : p.rows - 1;
    float r[kN][8], v[kN][8];
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        r[j][i] = have[j] > 0 ? (float)nh[j].v[i] : 0.0f;
        v[j][i] = p.y && have[j] > 0 ? (float)ny[j].v[i] : 0.0f;
      }
    if (e + 1 < rows_each) fetch(row_at + groups);
    if (p.y) {
      if (p.gate && p.rows_per_gate < p.rows && (e == 0 || (uint32_t)row / (uint32_t)p.rows_per_gate != gate_row)) {
        gate_row = (uint32_t)row / (uint32_t)p.rows_per_gate;
        keep_gw();
      }
      float mean = 0.0f, rstd = 1.0f;
      if (p.post != SIM_NORM_NONE) {
        moments<kN>(v, have, p.post, inv, p.eps, red, waves, wave, first, half, mean, rstd);
        if (p.post_stats && tr == 0 && real) {
          p.post_stats[row] = mean;
          p.post_stats[p.rows + row] = rstd;
        }
      }
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float w[8];
        if constexpr (kN > kHold) load_gw(j, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[j][i] = p.alpha * r[j][i] + v[j][i] * (rstd * (kN > kHold ? w[i] : kept_gw[kN > kHold ? 0 : j][i]));
        if (p.pb) {
          float g[8];
          param8<kVec>(p.pb, c[j], have[j], 0.0f, w);
          if (p.gate) {
            load8<A, kVec>((const A*)p.gate + (int64_t)gate_row * p.hidden, c[j], have[j], g);
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] *= g[i];
          }
#pragma unroll
          for (int i = 0; i < 8; ++i) r[j][i] += p.beta * w[i];
        }
      }
    }
    if (p.ho && real) {
#pragma unroll
      for (int j = 0; j < kN; ++j) store8<R, kVec>((R*)p.ho + row * p.ld_ho, c[j], have[j], r[j]);
    }
    if (p.pre == SIM_NORM_NONE) continue;
    float mean, rstd;
    moments<kN>(r, have, p.pre, inv, p.eps, red, waves, wave, first, half, mean, rstd);
    if (!real) continue;
    if (p.pre_stats && tr == 0) {
      p.pre_stats[row] = mean;
      p.pre_stats[p.rows + row] = rstd;
    }
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      float w[8], b[8];
      if constexpr (kN > kHold) param8<kVec>(p.qw, c[j], have[j], 1.0f, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = r[j][i] * rstd * (kN > kHold ? w[i] : kept_qw[kN > kHold ? 0 : j][i]);
      if (p.qb) {
        load8<float, kVec>(p.qb, c[j], have[j], b);
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] += b[i];
      }
      if (p.q) {
        float m = 0.0f;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (!kVec && i >= have[j]) w[i] = 0.0f;
          m = fmaxf(m, fabsf(w[i]));
        }
        m = fmaxf(max16(m), kAmaxFloor);
        const float f = kE4m3Max / m;
        if (c[j] < ((int)p.hidden + kBlock - 1) / kBlock * kBlock) {
          // (zero past the row also where an infinite or NaN rstd has made NaN of its zeros)
          const uint32_t in = !kVec || have[j] > 0 ? ~0u : 0u;
          *(u32x2*)(p.q + row * p.ld_q + c[j]) =
              u32x2{codes4(w[0], w[1], w[2], w[3], f) & in, codes4(w[4], w[5], w[6], w[7], f) & in};
          if ((tr & 15) == 0) p.s[c[j] / kBlock * p.ld_s + row] = m / kE4m3Max;
        }
      } else {
        store8<A, kVec>((A*)p.x + row * p.ld_x, c[j], have[j], w);
      }
    }
  }
}

// ---------------------------------------------------------------- backward
// With D the gradient of r: n's is beta gate D.  For one row of the gate the
// sums Q = sum of beta D hat and P = sum of beta D over its tokens (hat: the
// normed y, or y) give all that depends on it: its own gradient is
// Q post_weight + P post_bias, and it adds gate Q and gate P to the post
// weight's and bias's.  So two column sums (Q and the pre weight's) are kept
// in registers, four with layer norms.
struct Bwd {
  int64_t rows, hidden, ld_dho, ld_dx, ld_h, ld_y, ld_dh, ld_dy, rows_per_gate;
  int post, pre;
  float alpha, beta;
  const void *dho, *dx, *h, *y, *gate;
  const float *pw, *pb, *qw, *post_stats, *pre_stats;
  void *dh, *dy;
  float* dgate;
  float* part;          // [chunks][kSums][hidden]
  int64_t chunks, rows_per_chunk, chunks_per_gate;   // chunks_per_gate 0: a chunk is whole rows of the gate
  uint32_t want;        // bit k: sum k is asked for
};
// column sums, in the order of the workspace (kQ, kP: gate times them, where a
// chunk holds whole rows of the gate)
enum { kDqw, kDqb, kQ, kP, kSums };

// One workgroup takes a chunk of rows, one after another, and keeps the chunk's
// column sums in registers; they leave once for a chunk, and k_norm_join adds
// the chunks up in their order.  A row's y is on its way while the pre norm is
// worked on, and the next row's other inputs while the post norm is.  Up to
// kHold groups of eight per thread the weights stay in registers too; beyond,
// they come from the caches for each row.  kLayer: some norm is a layer norm or
// has a bias; the two sums more that this takes are kept in LDS where registers
// would not hold them (every thread has its own places there).  kFull: both
// norms, and all inputs and outputs but the sums, are there.
// 8192 x 8192 in 16 bits: 165 us, 4.9 TB/s of 12 B per element; 2047 x 12288
// layer norms with the stream in 32 bits 135 us, 3.4 TB/s, where the registers
// do not hold a row ahead as well (with one, spilled: 178).
constexpr int kGradThreads = 512;

template <typename A, typename R, int kN, bool kVec, bool kLayer, bool kFull>
__global__ __launch_bounds__(kGradThreads) void k_norm_grad(Bwd p) {
  __shared__ float red[64];
  const int tr = threadIdx.x, per_row = blockDim.x, waves = per_row / 64;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const float inv = 1.0f / (float)p.hidden;
  int half = 0;
  int64_t r0, r1, gate_row;
  if (p.chunks_per_gate) {
    gate_row = blockIdx.x / (uint32_t)p.chunks_per_gate;
    r0 = gate_row * p.rows_per_gate + blockIdx.x % (uint32_t)p.chunks_per_gate * p.rows_per_chunk;
    r1 = min(min(r0 + p.rows_per_chunk, (gate_row + 1) * p.rows_per_gate), p.rows);
  } else {
    r0 = blockIdx.x * p.rows_per_chunk;
    r1 = min(r0 + p.rows_per_chunk, p.rows);
    gate_row = r0 / p.rows_per_gate;
  }
  const bool pre = kFull || p.pre != SIM_NORM_NONE, post = kFull || p.post != SIM_NORM_NONE;
  const bool has_y = kFull || p.y, has_dho = kFull || p.dho, has_dh = kFull || p.dh, has_dy = kFull || p.dy;
  constexpr int kKept = kN <= kHold ? kN : 1;
  int c[kN], have[kN];
  float dqw[kN][8], q[kN][8];
  // the pre bias's sum (0) and P (1)
  constexpr bool kInLds = kLayer && (kN == 3 || kN == 4);
  __shared__ f32x4 side_lds[kInLds ? 2 : 1][kInLds ? kN : 1][kInLds ? 2 : 1][kInLds ? kGradThreads : 1];
  float side[kLayer && !kInLds ? 2 : 1][kLayer && !kInLds ? kN : 1][8];
  auto side_get = [&](int k, int j, float v[8]) {
    if constexpr (kInLds) {
      const f32x4 a = side_lds[k][j][0][tr], b = side_lds[k][j][1][tr];
#pragma unroll
      for (int i = 0; i < 4; ++i) { v[i] = a[i]; v[4 + i] = b[i]; }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = side[k][j][i];
    }
  };
  auto side_set = [&](int k, int j, const float v[8]) {
    if constexpr (kInLds) {
      side_lds[k][j][0][tr] = f32x4{v[0], v[1], v[2], v[3]};
      side_lds[k][j][1][tr] = f32x4{v[4], v[5], v[6], v[7]};
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) side[k][j][i] = v[i];
    }
  };
  auto side_add = [&](int k, int j, const float x[8]) {
    if constexpr (kLayer) {
      float v[8];
      side_get(k, j, v);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] += x[i];
      side_set(k, j, v);
    }
  };
  auto side_clear = [&](int k, int j) {
    if constexpr (kLayer) {
      const float zero[8] = {0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f, 0.0f};
      side_set(k, j, zero);
    }
  };
  float kept_qw[kKept][8], kept_gw[kKept][8];   // the pre weight; beta gate post_weight
  auto load_gw = [&](int j, float gw[8]) {
    float w[8];
    param8<kVec>(post ? p.pw : nullptr, c[j], have[j], 1.0f, gw);
    if (p.gate) {
      load8<A, kVec>((const A*)p.gate + gate_row * p.hidden, c[j], have[j], w);
#pragma unroll
      for (int i = 0; i < 8; ++i) gw[i] *= w[i];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) gw[i] *= p.beta;
  };
  auto keep_gw = [&]() {
    if constexpr (kN <= kHold) {
#pragma unroll
      for (int j = 0; j < kN; ++j) load_gw(j, kept_gw[j]);
    }
  };
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    c[j] = (j * per_row + tr) * 8;
    have[j] = (int)p.hidden - c[j];
    if constexpr (kN <= kHold) param8<kVec>(p.qw, c[j], have[j], 1.0f, kept_qw[j]);
#pragma unroll
    for (int i = 0; i < 8; ++i) dqw[j][i] = q[j][i] = 0.0f;
    side_clear(0, j);
    side_clear(1, j);
  }
  if (has_y) keep_gw();

  Raw<R> ndh[kN], nh[kN];
  Raw<A> ndx[kN], ny[kN];
  float nqm = 0.0f, nqr = 1.0f;
  auto fetch = [&](int64_t row) {
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      if (pre) {
        ndx[j] = fetch8<A, kVec>((const A*)p.dx + row * p.ld_dx, c[j], have[j]);
        nh[j] = fetch8<R, kVec>((const R*)p.h + row * p.ld_h, c[j], have[j]);
      }
      if (has_dho) ndh[j] = fetch8<R, kVec>((const R*)p.dho + row * p.ld_dho, c[j], have[j]);
    }
    if (pre) { nqm = p.pre_stats[row]; nqr = p.pre_stats[p.rows + row]; }
  };
  // A group past the row holds the row's first elements, and its weights are zero:
  // it adds nothing to a sum, unless what it holds is not finite.
  auto only_in_row = [&](int j, float a[2], const float before[2]) {
    if (kVec && have[j] <= 0) {
      a[0] = before[0];
      a[1] = before[1];
    }
  };
  // (the last row of the gate may have fewer tokens than chunks for them)
  constexpr bool kAhead = !(kLayer && kN > kHold);   // registers for a row more
  if (kAhead && r0 < r1) fetch(r0);
  bool first_gate = true;
  for (int64_t row = r0; row < r1; ++row) {
    float pm = 0.0f, pr = 1.0f;
    if constexpr (!kAhead) fetch(row);
    if (has_y) {
#pragma unroll
      for (int j = 0; j < kN; ++j) ny[j] = fetch8<A, kVec>((const A*)p.y + row * p.ld_y, c[j], have[j]);
      if (post) { pm = p.post_stats[row]; pr = p.post_stats[p.rows + row]; }
    }
    float d[kN][8];
#pragma unroll
    for (int j = 0; j < kN; ++j)
#pragma unroll
      for (int i = 0; i < 8; ++i) d[j][i] = has_dho ? (float)ndh[j].v[i] : 0.0f;
    if (pre) {
      float u[kN][8], hat[kN][8], a[2] = {0.0f, 0.0f};
      const float qm = nqm, qr = nqr;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float w[8];
        if constexpr (kN > kHold) {
          __builtin_amdgcn_sched_barrier(0);   // (one group's weights at a time: registers)
          param8<kVec>(p.qw, c[j], have[j], 1.0f, w);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[j][i] = (float)ndx[j].v[i];
          hat[j][i] = (float)nh[j].v[i];
          if constexpr (kLayer) hat[j][i] -= qm;
          hat[j][i] *= qr;
          dqw[j][i] += u[j][i] * hat[j][i];
        }
        side_add(0, j, u[j]);
        const float before[2] = {a[0], a[1]};
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          u[j][i] *= kN > kHold ? w[i] : kept_qw[kN > kHold ? 0 : j][i];
          a[0] += u[j][i] * hat[j][i];
          if constexpr (kLayer) a[1] += u[j][i];
        }
        only_in_row(j, a, before);
      }
      row_sum<kLayer ? 2 : 1>(a, red, waves, wave, 0, half);
      const float a0 = a[0] * inv * qr, a1 = kLayer && p.pre == SIM_NORM_LAYER ? a[1] * inv : 0.0f;
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (kLayer) u[j][i] -= a1;
          d[j][i] += qr * u[j][i] - hat[j][i] * a0;
        }
    }
    if (kAhead && row + 1 < r1) fetch(row + 1);
    if (has_dh) {
      const float al = has_y ? p.alpha : 1.0f;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float o[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) o[i] = al * d[j][i];
        store8<R, kVec>((R*)p.dh + row * p.ld_dh, c[j], have[j], o);
      }
    }
    if (!has_y) continue;
    float y[kN][8], a[2] = {0.0f, 0.0f};
#pragma unroll
    for (int j = 0; j < kN; ++j) {
      float w[8];
      if constexpr (kN > kHold) {
        __builtin_amdgcn_sched_barrier(0);
        load_gw(j, w);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        y[j][i] = (float)ny[j].v[i];
        if constexpr (kLayer) y[j][i] -= pm;
        y[j][i] *= pr;                               // (pr is one without a norm)
        q[j][i] += d[j][i] * y[j][i];
      }
      side_add(1, j, d[j]);
      const float before[2] = {a[0], a[1]};
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        d[j][i] *= kN > kHold ? w[i] : kept_gw[kN > kHold ? 0 : j][i];
        a[0] += d[j][i] * y[j][i];
        if constexpr (kLayer) a[1] += d[j][i];
      }
      only_in_row(j, a, before);
    }
    if (post) {
      row_sum<kLayer ? 2 : 1>(a, red, waves, wave, 0, half);
      const float a0 = a[0] * inv * pr, a1 = kLayer && p.post == SIM_NORM_LAYER ? a[1] * inv : 0.0f;
#pragma unroll
      for (int j = 0; j < kN; ++j)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if constexpr (kLayer) d[j][i] -= a1;
          d[j][i] = pr * d[j][i] - y[j][i] * a0;
        }
    }
    if (has_dy) {
#pragma unroll
      for (int j = 0; j < kN; ++j) store8<A, kVec>((A*)p.dy + row * p.ld_dy, c[j], have[j], d[j]);
    }
    // The last token of a gate's row, in a chunk of whole rows of it: the
    // row's gradient leaves, and the chunk's own sums are kept in its part of
    // the workspace, where no other workgroup reads or writes.
    if (!p.chunks_per_gate && (row + 1 == r1 || row + 1 == (gate_row + 1) * p.rows_per_gate)) {
      float* part = p.part + (int64_t)blockIdx.x * kSums * p.hidden;
#pragma unroll
      for (int j = 0; j < kN; ++j) {
        float w[8], b[8], v[8], o[8], pp[8];
        if constexpr (kLayer) side_get(1, j, pp);
        param8<kVec>(post ? p.pw : nullptr, c[j], have[j], 1.0f, w);
        param8<kVec>(post ? p.pb : nullptr, c[j], have[j], 0.0f, b);
        if (p.gate) load8<A, kVec>((const A*)p.gate + gate_row * p.hidden, c[j], have[j], v);
        else param8<kVec>(nullptr, c[j], have[j], 1.0f, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          q[j][i] *= p.beta;
          o[i] = q[j][i] * w[i];
          if constexpr (kLayer) {
            pp[i] *= p.beta;
            o[i] += pp[i] * b[i];
          }
        }
        if (p.dgate) store8<float, kVec>(p.dgate + gate_row * p.hidden, c[j], have[j], o);
        if (p.want >> kQ & 1) {
          if (first_gate) param8<kVec>(nullptr, c[j], have[j], 0.0f, o);
          else load8<float, kVec>(part + kQ * p.hidden, c[j], have[j], o);
#pragma unroll
          for (int i = 0; i < 8; ++i) o[i] += v[i] * q[j][i];
          store8<float, kVec>(part + kQ * p.hidden, c[j], have[j], o);
        }
        if constexpr (kLayer) {
          if (p.want >> kP & 1) {
            if (first_gate) param8<kVec>(nullptr, c[j], have[j], 0.0f, o);
            else load8<float, kVec>(part + kP * p.hidden, c[j], have[j], o);
#pragma unroll
            for (int i = 0; i < 8; ++i) o[i] += v[i] * pp[i];
            store8<float, kVec>(part + kP * p.hidden, c[j], have[j], o);
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) q[j][i] = 0.0f;
        side_clear(1, j);
      }
      first_gate = false;
      if (row + 1 < r1) {
        ++gate_row;
        keep_gw();
      }
    }
  }
  float* part = p.part + (int64_t)blockIdx.x * kSums * p.hidden;
#pragma unroll
  for (int j = 0; j < kN; ++j) {
    if (p.want >> kDqw & 1) store8<float, kVec>(part + kDqw * p.hidden, c[j], have[j], dqw[j]);
    if (p.chunks_per_gate && (p.want >> kQ & 1)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) q[j][i] *= p.beta;
      store8<float, kVec>(part + kQ * p.hidden, c[j], have[j], q[j]);
    }
    if constexpr (kLayer) {
      float s[8];
      side_get(0, j, s);
      if (p.want >> kDqb & 1) store8<float, kVec>(part + kDqb * p.hidden, c[j], have[j], s);
      side_get(1, j, s);
#pragma unroll
      for (int i = 0; i < 8; ++i) s[i] *= p.beta;
      if (p.chunks_per_gate && (p.want >> kP & 1)) store8<float, kVec>(part + kP * p.hidden, c[j], have[j], s);
    }
  }
}

// Sums over chunks: a workgroup takes 64 columns of one run of chunks (those of
// one row of the gate, or all), wave w of its 16 every 16th chunk (256 chunks of
// 8192 columns: 6.7 to 7.6 us); with more workgroups than the card holds of 16 waves
// it has 8 (12288 columns, 4 runs of 64 chunks: 11.6 us, with 16 waves 15.6).
// The first pass, for each row of the gate, finishes that row's gradient and
// leaves the run's sums, times the gate, in the run's first chunk; the second
// adds the runs.  One run: one pass.
struct Join {
  float* part;
  float *dqw, *dqb, *dpw, *dpb, *dgate;
  const float *pw, *pb;
  const void* gate;
  int64_t hidden, runs, per_run, stride;   // chunks of a run; chunks between runs
  int act;
  bool whole;      // the runs' sums have been multiplied by the gate
  bool last;       // write the results
};
__global__ __launch_bounds__(1024) void k_norm_join(Join p) {
  __shared__ float red[16][kSums][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x / 64;
  const int waves = blockDim.x / 64;
  const int64_t groups = (p.hidden + 63) / 64, c = blockIdx.x % groups * 64 + lane, run = blockIdx.x / groups;
  const bool want[kSums] = {p.dqw != nullptr, p.dqb != nullptr, p.dpw || p.dgate, p.dpb || (p.dgate && p.pb)};
  float v[kSums] = {0.0f, 0.0f, 0.0f, 0.0f};
  if (c < p.hidden) {
    const float* s = p.part + run * p.per_run * p.stride * kSums * p.hidden + c;
#pragma unroll
    for (int k = 0; k < kSums; ++k)
      if (want[k]) {
        float a = 0.0f;
#pragma unroll 8
        for (int64_t i = wave; i < p.per_run; i += waves) a += s[(i * p.stride * kSums + k) * p.hidden];
        v[k] = a;
      }
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) red[wave][k][lane] = v[k];
  __syncthreads();
  if (wave != 0 || c >= p.hidden) return;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    v[k] = 0.0f;
    for (int w = 0; w < waves; ++w) v[k] += red[w][k][lane];
  }
  if (!p.whole) {
    if (p.dgate)
      p.dgate[run * p.hidden + c] = v[kQ] * (p.pw ? p.pw[c] : 1.0f) + (p.pb ? v[kP] * p.pb[c] : 0.0f);
    if (p.gate) {
      const int64_t at = run * p.hidden + c;
      const float g = p.act == SIM_BF16 ? (float)((const bf16*)p.gate)[at] : p.act == SIM_FP16 ? (float)((const fp16*)p.gate)[at]
                                                                                               : ((const float*)p.gate)[at];
      v[kQ] *= g;
      v[kP] *= g;
    }
  }
  if (p.last) {
    if (p.dqw) p.dqw[c] = v[kDqw];
    if (p.dqb) p.dqb[c] = v[kDqb];
    if (p.dpw) p.dpw[c] = v[kQ];
    if (p.dpb) p.dpb[c] = v[kP];
  } else {
    float* s = p.part + run * p.per_run * p.stride * kSums * p.hidden + c;
#pragma unroll
    for (int k = 0; k < kSums; ++k)
      if (want[k]) s[k * p.hidden] = v[k];
  }
}

// ---------------------------------------------------------------- launches
// Threads for a row and groups of eight per thread.
struct Shape {
  int threads, n;
};
Shape shape_of(int64_t hidden, int most) {
  const int64_t groups = cdiv(hidden, 8);
  int n = 1;
  while (groups > (int64_t)most * n) n = n < 4 ? n + 1 : 8;
  int64_t t = 64;
  while (t * n < groups) t += 64;
  return {(int)t, n};
}

template <typename A, typename R, int kN>
hipError_t launch_fwd(const Fwd& p, Shape s, bool vec, hipStream_t st) {
  // short rows: several to a workgroup, each on whole waves; and as many rows
  // one after another as leave the card full
  int rows = 1;
  while (rows * 2 * s.threads <= 256) rows *= 2;
  const int64_t waves = kN == 1 ? 16 : 8;   // that a CU holds, by their registers
  const int64_t fill = 256 * (waves * 64 / (s.threads * rows));
  const int64_t each = cdiv(p.rows, fill * rows);
  const int64_t grid = cdiv(p.rows, rows * each);
  if (grid > INT32_MAX) return hipErrorInvalidValue;
  auto k = vec ? k_norm<A, R, kN, true> : k_norm<A, R, kN, false>;
  k<<<dim3((uint32_t)grid), s.threads * rows, 0, st>>>(p, s.threads, (int)each);
  return launched();
}
template <typename A, typename R>
hipError_t launch_fwd_n(const Fwd& p, bool vec, hipStream_t st) {
  const Shape s = shape_of(p.hidden, kThreads);
  switch (s.n) {
    case 1: return launch_fwd<A, R, 1>(p, s, vec, st);
    case 2: return launch_fwd<A, R, 2>(p, s, vec, st);
    case 3: return launch_fwd<A, R, 3>(p, s, vec, st);
    case 4: return launch_fwd<A, R, 4>(p, s, vec, st);
    default: return launch_fwd<A, R, 8>(p, s, vec, st);
  }
}

template <typename A, typename R, int kN>
hipError_t launch_bwd(const Bwd& p, Shape s, bool vec, hipStream_t st) {
  const bool layer = p.pre == SIM_NORM_LAYER || p.post == SIM_NORM_LAYER || p.pb || (p.want >> kDqb & 1) || (p.want >> kP & 1);
  const bool full = p.pre != SIM_NORM_NONE && p.post != SIM_NORM_NONE && p.y && p.dho && p.dh && p.dy;
  auto k = !vec ? k_norm_grad<A, R, kN, false, true, false>
           : layer ? (full ? k_norm_grad<A, R, kN, true, true, true> : k_norm_grad<A, R, kN, true, true, false>)
                   : (full ? k_norm_grad<A, R, kN, true, false, true> : k_norm_grad<A, R, kN, true, false, false>);
  k<<<dim3((uint32_t)p.chunks), s.threads, 0, st>>>(p);
  return launched();
}
template <typename A, typename R>
hipError_t launch_bwd_n(const Bwd& p, bool vec, hipStream_t st) {
  const Shape s = shape_of(p.hidden, kGradThreads);
  switch (s.n) {
    case 1: return launch_bwd<A, R, 1>(p, s, vec, st);
    case 2: return launch_bwd<A, R, 2>(p, s, vec, st);
    case 3: return launch_bwd<A, R, 3>(p, s, vec, st);
    case 4: return launch_bwd<A, R, 4>(p, s, vec, st);
    default: return launch_bwd<A, R, 8>(p, s, vec, st);
  }
}

// act and res as template arguments
template <typename F>
hipError_t by_type(int act, int res, F f) {
  if (act == SIM_BF16) return res == SIM_FP32 ? f((bf16*)nullptr, (float*)nullptr) : f((bf16*)nullptr, (bf16*)nullptr);
  if (act == SIM_FP16) return res == SIM_FP32 ? f((fp16*)nullptr, (float*)nullptr) : f((fp16*)nullptr, (fp16*)nullptr);
  return f((float*)nullptr, (float*)nullptr);
}

// How the rows are cut into chunks: about as many as the card works on at a
// time (one workgroup to a CU with two groups of eight or more per thread, else
// two), none across two gate rows unless it holds whole ones.
struct Cut {
  int64_t chunks, rows_per_chunk, chunks_per_gate;
};
Cut cut_of(int64_t rows, int64_t hidden, int64_t rows_per_gate) {
  const int64_t kChunks = shape_of(hidden, kGradThreads).n > 1 ? 256 : 512;
  const int64_t per = rows_per_gate < rows ? rows_per_gate : rows, gates = cdiv(rows, per);
  const int64_t want = cdiv(rows, kChunks);
  if (per <= want) {
    const int64_t r = want / per * per;
    return {cdiv(rows, r), r, 0};
  }
  return {gates * cdiv(per, want), want, cdiv(per, want)};
}

bool valid_types(int act, int res) { return type_bytes(act) && (res == act || res == SIM_FP32); }
bool valid_kind(int k) { return k == SIM_NORM_NONE || k == SIM_NORM_RMS || k == SIM_NORM_LAYER; }
// 16-byte accesses of eight elements at a time
bool vec_rows(const void* p, int dtype, int64_t ld) {
  const int64_t bytes = type_bytes(dtype) * 8;
  return !p || (aligned(p, 16) && (ld * type_bytes(dtype)) % (bytes < 16 ? bytes : 16) == 0);
}
bool valid_rows(const void* p, int dtype, int64_t ld, int64_t hidden) {
  return ld >= hidden && aligned(p, (size_t)type_bytes(dtype));
}

}  // namespace
}  // namespace ops
}  // namespace hetsim

using namespace hetsim::ops;

extern "C" int sim_op_norm(const sim_norm_args* a, void* stream) {
  if (!a || a->rows < 0 || a->hidden < 1 || a->hidden > SIM_NORM_MAX_HIDDEN || a->rows > INT32_MAX ||
      !valid_types(a->act, a->res) || !valid_kind(a->post) || !valid_kind(a->pre))
    return SIM_EINVAL;
  if (!(a->eps >= 0.0f)) return SIM_EINVAL;
  if (a->rows == 0) return SIM_OK;
  const bool norm = a->pre != SIM_NORM_NONE;
  if (!a->h || !valid_rows(a->h, a->res, a->ld_h, a->hidden)) return SIM_EINVAL;
  if (a->y ? !valid_rows(a->y, a->act, a->ld_y, a->hidden) : a->post != SIM_NORM_NONE || a->gate) return SIM_EINVAL;
  if (a->gate && (a->rows_per_gate < 1 || !aligned(a->gate, (size_t)type_bytes(a->act)))) return SIM_EINVAL;
  if (a->h_out && !valid_rows(a->h_out, a->res, a->ld_h_out, a->hidden)) return SIM_EINVAL;
  if (norm && (a->x != nullptr) == (a->xq != nullptr)) return SIM_EINVAL;   // one of them
  if (!norm && (a->x || a->xq || a->pre_stats)) return SIM_EINVAL;
  if (a->x && !valid_rows(a->x, a->act, a->ld_x, a->hidden)) return SIM_EINVAL;
  if (a->xq && (!valid_blocks(a->xq, a->rows, a->hidden) || a->xq->block_rows != 1)) return SIM_EINVAL;
  if (a->post == SIM_NORM_NONE && (a->post_stats || a->post_weight || a->post_bias)) return SIM_EINVAL;
  for (const float* q : {a->post_weight, a->post_bias, a->pre_weight, a->pre_bias, (const float*)a->post_stats,
                         (const float*)a->pre_stats})
    if (!aligned(q, 4)) return SIM_EINVAL;
  Fwd p;
  p.rows = a->rows; p.hidden = a->hidden;
  p.ld_h = a->ld_h; p.ld_y = a->ld_y; p.ld_ho = a->ld_h_out; p.ld_x = a->ld_x;
  p.rows_per_gate = a->gate && a->rows_per_gate < a->rows ? a->rows_per_gate : a->rows;
  p.post = a->post; p.pre = a->pre;
  p.alpha = a->alpha; p.beta = a->beta; p.eps = a->eps;
  p.h = a->h; p.y = a->y; p.gate = a->gate;
  p.pw = a->post_weight; p.pb = a->post_bias; p.qw = a->pre_weight; p.qb = a->pre_bias;
  p.ho = a->h_out; p.x = a->x;
  p.q = a->xq ? a->xq->codes : nullptr;
  p.s = a->xq ? a->xq->scales : nullptr;
  p.ld_q = a->xq ? a->xq->ld : 0;
  p.ld_s = a->xq ? a->xq->ld_s : 0;
  p.post_stats = a->post_stats; p.pre_stats = a->pre_stats;
  const bool vec = a->hidden % 8 == 0 && vec_rows(a->h, a->res, a->ld_h) && vec_rows(a->y, a->act, a->ld_y) &&
                   vec_rows(a->h_out, a->res, a->ld_h_out) && vec_rows(a->x, a->act, a->ld_x) && aligned(a->gate, 16) &&
                   aligned(a->post_weight, 16) && aligned(a->post_bias, 16) && aligned(a->pre_weight, 16) &&
                   aligned(a->pre_bias, 16);
  const hipError_t e = by_type(a->act, a->res, [&](auto* x, auto* r) {
    return launch_fwd_n<std::remove_pointer_t<decltype(x)>, std::remove_pointer_t<decltype(r)>>(p, vec, (hipStream_t)stream);
  });
  return e == hipSuccess ? SIM_OK : e == hipErrorInvalidValue ? SIM_EINVAL : SIM_EHIP;
}

extern "C" size_t sim_op_norm_backward_workspace(int64_t rows, int64_t hidden, int64_t rows_per_gate) {
  if (rows <= 0 || hidden <= 0 || rows_per_gate <= 0) return 0;
  return (size_t)cut_of(rows, hidden, rows_per_gate).chunks * kSums * (size_t)hidden * 4;
}

extern "C" int sim_op_norm_backward(const sim_norm_grad_args* a, void* workspace, size_t workspace_bytes, void* stream) {
  if (!a || a->rows < 0 || a->hidden < 1 || a->hidden > SIM_NORM_MAX_HIDDEN || a->rows > INT32_MAX ||
      !valid_types(a->act, a->res) || !valid_kind(a->post) || !valid_kind(a->pre))
    return SIM_EINVAL;
  const bool pre = a->pre != SIM_NORM_NONE, post = a->post != SIM_NORM_NONE;
  if (!pre && (a->dpre_weight || a->dpre_bias)) return SIM_EINVAL;
  if (!post && (a->dpost_weight || a->dpost_bias || a->post_weight || a->post_bias)) return SIM_EINVAL;
  if (a->dgate && !a->gate) return SIM_EINVAL;
  if (a->gate && (a->rows_per_gate < 1 || !aligned(a->gate, (size_t)type_bytes(a->act)))) return SIM_EINVAL;
  for (const float* q : {a->post_weight, a->post_bias, a->pre_weight, a->post_stats, a->pre_stats, (const float*)a->dgate,
                         (const float*)a->dpost_weight, (const float*)a->dpost_bias, (const float*)a->dpre_weight,
                         (const float*)a->dpre_bias})
    if (!aligned(q, 4)) return SIM_EINVAL;
  const bool y = a->y != nullptr, gate = a->gate != nullptr;
  if (!y && (post || gate || a->dy)) return SIM_EINVAL;
  const int64_t per = gate && a->rows_per_gate < a->rows ? a->rows_per_gate : a->rows;
  Cut cut = {0, 0, 0};
  if (a->rows > 0) {
    if (a->dh_out && !valid_rows(a->dh_out, a->res, a->ld_dh_out, a->hidden)) return SIM_EINVAL;
    if (pre && (!a->dx || !valid_rows(a->dx, a->act, a->ld_dx, a->hidden) || !a->h ||
                !valid_rows(a->h, a->res, a->ld_h, a->hidden) || !a->pre_stats))
      return SIM_EINVAL;
    if (y && !valid_rows(a->y, a->act, a->ld_y, a->hidden)) return SIM_EINVAL;
    if (post && !a->post_stats) return SIM_EINVAL;
    if (a->dh && !valid_rows(a->dh, a->res, a->ld_dh, a->hidden)) return SIM_EINVAL;
    if (a->dy && !valid_rows(a->dy, a->act, a->ld_dy, a->hidden)) return SIM_EINVAL;
    cut = cut_of(a->rows, a->hidden, per);
    if (cut.chunks > INT32_MAX) return SIM_EINVAL;
    const size_t need = (size_t)cut.chunks * kSums * (size_t)a->hidden * 4;
    if (workspace_bytes < need || !workspace || !aligned(workspace, 16)) return SIM_EINVAL;
  }
  Bwd p;
  p.rows = a->rows; p.hidden = a->hidden;
  p.ld_dho = a->ld_dh_out; p.ld_dx = a->ld_dx; p.ld_h = a->ld_h; p.ld_y = a->ld_y; p.ld_dh = a->ld_dh; p.ld_dy = a->ld_dy;
  p.rows_per_gate = per > 0 ? per : 1;
  p.post = a->post; p.pre = a->pre;
  p.alpha = a->alpha; p.beta = a->beta;
  p.dho = a->dh_out; p.dx = a->dx; p.h = a->h; p.y = a->y; p.gate = a->gate;
  p.pw = a->post_weight; p.pb = a->post_bias; p.qw = a->pre_weight;
  p.post_stats = a->post_stats; p.pre_stats = a->pre_stats;
  p.dh = a->dh; p.dy = a->dy; p.dgate = a->dgate;
  p.part = (float*)workspace;
  p.chunks = cut.chunks; p.rows_per_chunk = cut.rows_per_chunk; p.chunks_per_gate = cut.chunks_per_gate;
  Join j;
  j.part = p.part;
  j.dqw = a->dpre_weight; j.dqb = a->dpre_bias; j.dpw = a->dpost_weight; j.dpb = a->dpost_bias;
  j.dgate = cut.chunks_per_gate ? a->dgate : nullptr;
  j.pw = a->post_weight; j.pb = a->post_bias; j.gate = a->gate;
  j.hidden = a->hidden; j.act = a->act;
  j.whole = cut.chunks_per_gate == 0; j.last = true;
  j.runs = 1; j.per_run = cut.chunks; j.stride = 1;
  p.want = (j.dqw ? 1u << kDqw : 0u) | (j.dqb ? 1u << kDqb : 0u) | (j.dpw || j.dgate ? 1u << kQ : 0u) |
           (j.dpb || (j.dgate && j.pb) ? 1u << kP : 0u);
  const hipStream_t st = (hipStream_t)stream;
  if (a->rows > 0) {
    const bool vec = a->hidden % 8 == 0 && vec_rows(a->dh_out, a->res, a->ld_dh_out) && vec_rows(a->dx, a->act, a->ld_dx) &&
                     vec_rows(a->h, a->res, a->ld_h) && vec_rows(a->y, a->act, a->ld_y) && vec_rows(a->dh, a->res, a->ld_dh) &&
                     vec_rows(a->dy, a->act, a->ld_dy) && aligned(a->gate, 16) && aligned(a->post_weight, 16) &&
                     aligned(a->post_bias, 16) && aligned(a->pre_weight, 16) && aligned(a->dgate, 16);
    const hipError_t e = by_type(a->act, a->res, [&](auto* x, auto* r) {
      return launch_bwd_n<std::remove_pointer_t<decltype(x)>, std::remove_pointer_t<decltype(r)>>(p, vec, st);
    });
    if (e != hipSuccess) return SIM_EHIP;
  }
  if (!p.want) return SIM_OK;
  const int64_t groups = cdiv(a->hidden, 64);
  if (cut.chunks_per_gate && cut.chunks > cut.chunks_per_gate) {
    j.runs = cdiv(a->rows, per);
    j.per_run = cut.chunks_per_gate;
    j.last = false;
    if (groups * j.runs > INT32_MAX) return SIM_EINVAL;
    k_norm_join<<<dim3((uint32_t)(groups * j.runs)), groups * j.runs > 512 ? 512 : 1024, 0, st>>>(j);
    if (launched() != hipSuccess) return SIM_EHIP;
    j.per_run = j.runs;
    j.runs = 1;
    j.stride = cut.chunks_per_gate;
    j.dgate = nullptr;
    j.whole = j.last = true;
    if (!j.dqw && !j.dqb && !j.dpw && !j.dpb) return SIM_OK;
  }
  k_norm_join<<<dim3((uint32_t)groups), 1024, 0, st>>>(j);
  return launched() == hipSuccess ? SIM_OK : SIM_EHIP;
}
