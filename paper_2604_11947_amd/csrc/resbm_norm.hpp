// resbm_norm.hpp -- the residual addition with its RMS norm, and that norm's backward, gfx950.
//
// Between two layers the residual stream is formed and normalised:
//     h = x + res + b I_{r x n}                     (the decoder's skip, Eq. 5, in the same pass)
//     y = h rstd gamma,   rstd = 1 / sqrt(mean_c h^2 + eps)
// and backwards, with xh = h rstd, w = g_y gamma, c = mean_c(w xh),
//     g_x = rstd (w - xh c) + g_h,   dgamma = sum_t g_y xh.
// Every op reads each operand once and writes each result once, so HBM bounds them (about one
// operation a byte).  A row has to be whole before any of its results, so a team of lanes owns a row
// and keeps it in registers, eight columns ("a chunk") a lane and CH chunks: 16, 32 or 64 lanes of a
// wave where n <= 128, 256 or 512 (four such waves a block), else a block of as many waves as the row
// needs.  Narrow rows that share a wave: 524288 x 128, no residual, 67 us (6.0 TB/s) against 186 us with a
// wave each.  The stream h is rounded once, to the activations' type, and the norm is that of the rounded
// h, whether h is written or not: then the backward pass, which reads h, is the adjoint of what the
// forward computed.
// A row that a wave or block has alone is addressed through a descriptor, so that columns behind the
// last and operands that are not there read as zeros and stores to them are dropped: every memory
// operation is unconditional, and the compiler counts exactly how many are in flight.
// Measured, with the passes' minimum bytes: 16384 x 4096 with residual and skip 90.8 us forward (5.9 TB/s)
// and 87.0 us backward (6.2 TB/s), 8-bit output at 32768 x 8192 319 us (5.9 TB/s); the card's own copy runs
// at 5.2 TB/s, its in-place sum of two tensors at 5.9.
// Included by resbm_matrix.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resbm.h"
#include "resbm_buffer.hpp"
#include "resbm_host.hpp"

#ifndef RESBM_IO_F32_BUILD
#define RESBM_IO_F32_BUILD 0
#endif

namespace resbm_nm {

using resbm::bld16;
using resbm::bld8;
using resbm::bst16;
using resbm::bst8;
using resbm::make_rsrc;
using resbm::rsrc_t;

// ---------------------------------------------------------------- eight activations
typedef uint32_t w2 __attribute__((ext_vector_type(2)));
typedef uint32_t w4 __attribute__((ext_vector_type(4)));
template <int POL>
__device__ __forceinline__ uint4 get16(const uint4* p) {
  if constexpr (POL != 0) return __builtin_bit_cast(uint4, __builtin_nontemporal_load((const w4*)p));
  return *p;
}
template <int POL>
__device__ __forceinline__ void put16(uint4 v, uint4* p) {
  if constexpr (POL != 0)
    __builtin_nontemporal_store(__builtin_bit_cast(w4, v), (w4*)p);
  else
    *p = v;
}
template <int POL>
__device__ __forceinline__ void put16(uint2 v, uint2* p) {
  if constexpr (POL != 0)
    __builtin_nontemporal_store(__builtin_bit_cast(w2, v), (w2*)p);
  else
    *p = v;
}
#if RESBM_IO_F32_BUILD
typedef float act_t;
struct Act8 {
  uint4 a, b;
};
template <int POL>
__device__ __forceinline__ Act8 load8(rsrc_t r, uint32_t o) {
  return {bld16<POL>(r, o * 4), bld16<POL>(r, o * 4 + 16)};
}
template <int POL>
__device__ __forceinline__ void store8(rsrc_t r, uint32_t o, const Act8& v) {
  bst16<POL>(r, o * 4, v.a);
  bst16<POL>(r, o * 4 + 16, v.b);
}
template <int POL>
__device__ __forceinline__ Act8 load8_at(const act_t* p) {
  return {get16<POL>((const uint4*)p), get16<POL>((const uint4*)p + 1)};
}
template <int POL>
__device__ __forceinline__ void store8_at(act_t* p, const Act8& v) {
  put16<POL>(v.a, (uint4*)p);
  put16<POL>(v.b, (uint4*)p + 1);
}
__device__ __forceinline__ Act8 load4_4(rsrc_t r, uint32_t o) { return load8<0>(r, o); }
__device__ __forceinline__ Act8 load4_4(const act_t* p, bool lo, bool hi) {
  const uint4 z = make_uint4(0, 0, 0, 0);
  return {lo ? ((const uint4*)p)[0] : z, hi ? ((const uint4*)p)[1] : z};
}
__device__ __forceinline__ void widen(const Act8& v, float (&f)[8]) {
  const uint32_t u[8] = {v.a.x, v.a.y, v.a.z, v.a.w, v.b.x, v.b.y, v.b.z, v.b.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(float, u[e]);
}
__device__ __forceinline__ Act8 narrow(const float (&f)[8]) {
  uint32_t u[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) u[e] = __builtin_bit_cast(uint32_t, f[e]);
  return {make_uint4(u[0], u[1], u[2], u[3]), make_uint4(u[4], u[5], u[6], u[7])};
}
#else
typedef __bf16 act_t;
typedef __bf16 nbf2 __attribute__((ext_vector_type(2)));
struct Act8 {
  uint4 v;
};
template <int POL>
__device__ __forceinline__ Act8 load8(rsrc_t r, uint32_t o) {
  return {bld16<POL>(r, o * 2)};
}
template <int POL>
__device__ __forceinline__ void store8(rsrc_t r, uint32_t o, const Act8& v) {
  bst16<POL>(r, o * 2, v.v);
}
template <int POL>
__device__ __forceinline__ Act8 load8_at(const act_t* p) {
  return {get16<POL>((const uint4*)p)};
}
template <int POL>
__device__ __forceinline__ void store8_at(act_t* p, const Act8& v) {
  put16<POL>(v.v, (uint4*)p);
}
// In two halves: a row of r = 4 mod 8 ends inside a chunk.
__device__ __forceinline__ Act8 load4_4(rsrc_t r, uint32_t o) {
  const uint2 a = bld8(r, o * 2), b = bld8(r, o * 2 + 8);
  return {make_uint4(a.x, a.y, b.x, b.y)};
}
__device__ __forceinline__ Act8 load4_4(const act_t* p, bool lo, bool hi) {
  const uint2 z = make_uint2(0, 0);
  const uint2 a = lo ? ((const uint2*)p)[0] : z, b = hi ? ((const uint2*)p)[1] : z;
  return {make_uint4(a.x, a.y, b.x, b.y)};
}
__device__ __forceinline__ float lo16(uint32_t u) { return __builtin_bit_cast(float, u << 16); }
__device__ __forceinline__ float hi16(uint32_t u) { return __builtin_bit_cast(float, u & 0xFFFF0000u); }
__device__ __forceinline__ void widen(const Act8& v, float (&f)[8]) {
  f[0] = lo16(v.v.x), f[1] = hi16(v.v.x), f[2] = lo16(v.v.y), f[3] = hi16(v.v.y);
  f[4] = lo16(v.v.z), f[5] = hi16(v.v.z), f[6] = lo16(v.v.w), f[7] = hi16(v.v.w);
}
__device__ __forceinline__ uint32_t pack2(float a, float b) {  // round to nearest even
  const nbf2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
__device__ __forceinline__ Act8 narrow(const float (&f)[8]) {
  return {make_uint4(pack2(f[0], f[1]), pack2(f[2], f[3]), pack2(f[4], f[5]), pack2(f[6], f[7]))};
}
#endif
constexpr size_t kActBytes = sizeof(act_t);

__device__ __forceinline__ void load_gain(rsrc_t r, int c, float (&f)[8]) {
  const uint4 a = bld16(r, (uint32_t)c * 4), b = bld16(r, (uint32_t)c * 4 + 16);
  const uint32_t u[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) f[e] = __builtin_bit_cast(float, u[e]);
}

// A lane's row t of a matrix of n columns.  Where a wave or block has one row (ONE), a descriptor over its
// columns: behind the last one, and where p is NULL, loads give zeros and stores are dropped.  Where a wave has
// several, the lane's own address, used where there is a column.
template <bool ONE, class E>
struct Row {
  rsrc_t r;
  E* p;
  int cols;
  __device__ __forceinline__ Row(E* base, int64_t t, int64_t T, int64_t ld, int n) {
    if constexpr (ONE) {
      r = make_rsrc(base + t * ld, base ? (int64_t)n * (int64_t)sizeof(E) : 0);  // (t < T here)
    } else {
      p = base && t < T ? base + t * ld : base;
      cols = base && t < T ? n : 0;
    }
  }
  template <int POL>
  __device__ __forceinline__ Act8 load(int c) const {
    if constexpr (ONE) return load8<POL>(r, (uint32_t)c);
    Act8 v = {};
    if (c < cols) v = load8_at<POL>(p + c);
    return v;
  }
  __device__ __forceinline__ Act8 load_by4(int c) const {
    if constexpr (ONE) return load4_4(r, (uint32_t)c);
    return load4_4(p + c, c < cols, c + 4 < cols);
  }
  template <int POL>
  __device__ __forceinline__ void store(int c, const Act8& v) const {
    if constexpr (ONE)
      store8<POL>(r, (uint32_t)c, v);
    else if (c < cols)
      store8_at<POL>(p + c, v);
  }
  template <int POL>
  __device__ __forceinline__ void store_codes(int c, uint2 v) const {
    if constexpr (ONE)
      bst8<POL>(r, (uint32_t)c, v);
    else if (c < cols)
      put16<POL>(v, (uint2*)(p + c));
  }
};

// The gain of a lane's chunks: kept in registers up to two chunks, read again at each use beyond
// (from L2; kept, they spilled).
template <int CH>
struct Gain {
  float w[CH <= 2 ? CH : 1][8];
  __device__ __forceinline__ void keep(rsrc_t r, int lanes, int lane) {
    if constexpr (CH <= 2)
#pragma unroll
      for (int k = 0; k < CH; ++k) load_gain(r, (k * lanes + lane) * 8, w[k]);
  }
  __device__ __forceinline__ void get(rsrc_t r, int k, int lanes, int lane, float (&f)[8]) const {
    if constexpr (CH <= 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = w[k][e];
    } else {
      load_gain(r, (k * lanes + lane) * 8, f);
    }
  }
};

// ---------------------------------------------------------------- sums and maxima over lanes
// Lane permutations within 16 lanes (DPP): after steps 1, 2, 4 and 8 every lane holds the result
// of its aligned group of 2, 4, 8 and 16 lanes.  The order of a sum is fixed by the lane alone.
template <int CTRL>
__device__ __forceinline__ uint32_t dpp(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
constexpr int kXor1 = 0xB1, kXor2 = 0x4E, kHalfMirror = 0x141, kMirror = 0x140;  // quad permutes, row mirrors

template <int CTRL>
__device__ __forceinline__ float add_step(float v) {
  return v + __builtin_bit_cast(float, dpp<CTRL>(__builtin_bit_cast(uint32_t, v)));
}
template <int CTRL>
__device__ __forceinline__ uint32_t max_step(uint32_t v) {
  const uint32_t o = dpp<CTRL>(v);
  return v > o ? v : o;
}
__device__ __forceinline__ float wave_sum(float v) {
  v = add_step<kMirror>(add_step<kHalfMirror>(add_step<kXor2>(add_step<kXor1>(v))));
  const int u = __builtin_bit_cast(int, v);
  const float a = __builtin_bit_cast(float, __builtin_amdgcn_readlane(u, 0));
  const float b = __builtin_bit_cast(float, __builtin_amdgcn_readlane(u, 16));
  const float c = __builtin_bit_cast(float, __builtin_amdgcn_readlane(u, 32));
  const float d = __builtin_bit_cast(float, __builtin_amdgcn_readlane(u, 48));
  return (a + b) + (c + d);
}
// Maxima are of magnitudes' bit patterns: as unsigned numbers they order like the values, with
// infinity above every finite one and NaN above infinity, so that neither is lost.
__device__ __forceinline__ uint32_t mag(float v) { return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t umax(uint32_t a, uint32_t b) { return a > b ? a : b; }
__device__ __forceinline__ uint32_t wave_max(uint32_t v) {
  v = max_step<kMirror>(max_step<kHalfMirror>(max_step<kXor2>(max_step<kXor1>(v))));
  const uint32_t a = __builtin_amdgcn_readlane(v, 0), b = __builtin_amdgcn_readlane(v, 16);
  const uint32_t c = __builtin_amdgcn_readlane(v, 32), d = __builtin_amdgcn_readlane(v, 48);
  return umax(umax(a, b), umax(c, d));
}

// Lanes that own a row: L = 16, 32 or 64 of a wave, 64 / L rows a wave, or (L = 0) the whole block.
constexpr int kMaxWaves = 16;
constexpr int kRowWaves = 4;  // waves of a block whose waves own rows
template <int L>
struct Shape {
  static constexpr int kRows = L ? 64 / L : 1;                      // a wave's or block's at a time
  static constexpr int kBlockRows = L ? kRows * kRowWaves : 1;
  static constexpr int kThreads = L ? 64 * kRowWaves : 64 * kMaxWaves;  // a block's, at most
  int lanes, lane, sub;  // a row's lanes, this one among them, and its row among the wave's
  int64_t first, step;   // the wave's first row, and the distance to its next ones
  // threads: the block's, from the arguments (blockDim would be read from memory again in the loop);
  // others: blocks before the first that owns rows
  __device__ __forceinline__ Shape(int threads, int others) {
    const int l = threadIdx.x & 63, block = (int)blockIdx.x - others;
    lanes = L ? L : threads;
    lane = L ? l % (L ? L : 1) : (int)threadIdx.x;
    sub = L ? l / (L ? L : 1) : 0;
    first = L ? (int64_t)block * kBlockRows + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) * kRows : (int64_t)block;
    step = (int64_t)((int)gridDim.x - others) * kBlockRows;
  }
  __device__ __forceinline__ int col(int k) const { return (k * lanes + lane) * 8; }
  template <class E>
  using Of = Row<kRows == 1, E>;
};

// The team's sum or maximum: of a row's lanes in their wave, or of the block.  One barrier: the slot
// alternates, and a slot is written again only behind the barrier of the call in between, which every
// reader of its old values has passed.  Every 16 lanes add the waves' values in the same order.
template <int L>
struct Team {
  uint32_t* lds;  // 2 * kMaxWaves words
  int waves, slot;
  __device__ __forceinline__ uint32_t others(uint32_t v) {
    uint32_t* s = lds + slot * kMaxWaves;
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    const int i = threadIdx.x & 15;
    return i < waves ? s[i] : 0;
  }
  __device__ __forceinline__ float sum(float v) {
    if constexpr (L == 16 || L == 32) {
      v = add_step<kMirror>(add_step<kHalfMirror>(add_step<kXor2>(add_step<kXor1>(v))));
      return L == 16 ? v : v + __shfl_xor(v, 16);
    }
    v = wave_sum(v);
    if constexpr (L == 64) return v;
    v = __builtin_bit_cast(float, others(__builtin_bit_cast(uint32_t, v)));
    return add_step<kMirror>(add_step<kHalfMirror>(add_step<kXor2>(add_step<kXor1>(v))));
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    if constexpr (L == 16 || L == 32) {
      v = max_step<kMirror>(max_step<kHalfMirror>(max_step<kXor2>(max_step<kXor1>(v))));
      return L == 16 ? v : umax(v, (uint32_t)__shfl_xor((int)v, 16));
    }
    v = wave_max(v);
    if constexpr (L == 64) return v;
    v = others(v);
    return max_step<kMirror>(max_step<kHalfMirror>(max_step<kXor2>(max_step<kXor1>(v))));
  }
};

// ---------------------------------------------------------------- 8-bit values
constexpr float kPerMax = 1.0f / 448.0f;  // of e4m3's largest value, rounded to float32
constexpr float kScaleFloor = 0x1p-126f;  // smallest normal: a group of zeros has a scale, and its reciprocal is finite

__device__ __forceinline__ float e4m3_scale(uint32_t amax_bits) {
  const float s = __builtin_bit_cast(float, amax_bits) * kPerMax;
  return s < kScaleFloor ? kScaleFloor : s;  // NaN stays
}
// Four values to e4m3, to nearest even; NaN stays NaN.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
  const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
}

// ---------------------------------------------------------------- forward
struct FwdArgs {
  int64_t T;
  int threads;  // a block's
  int n, r, group;  // group: columns per scale, n for one a row
  float eps;
  const act_t *x, *res, *b;
  int64_t ld_x, ld_res;
  const float* gamma;
  act_t* h;
  int64_t ld_h;
  void* y;
  int64_t ld_y;
  float *scale, *rstd;
};

template <int L, int CH, bool Q8, int POL>
__global__ __launch_bounds__(Shape<L>::kThreads) void k_norm_fwd(FwdArgs g) {
  __shared__ uint32_t s_red[2 * kMaxWaves];
  Team<L> team{s_red, g.threads >> 6, 0};
  const Shape<L> sh(g.threads, 0);
  using In = typename Shape<L>::template Of<const act_t>;
  using Out = typename Shape<L>::template Of<act_t>;
  const int lanes = sh.lanes, lane = sh.lane;
  const rsrc_t gain = make_rsrc(g.gamma, (int64_t)g.n * 4);
  // a wave or block goes through the loop as one: the barriers are uniform
  for (int64_t t0 = sh.first; t0 < g.T; t0 += sh.step) {
    const int64_t t = t0 + sh.sub;
    const In rx(g.x, t, g.T, g.ld_x, g.n), rr(g.res, t, g.T, g.ld_res, g.n), rb(g.b, t, g.T, g.r, g.r);
    const Out rh(g.h, t, g.T, g.ld_h, g.n);
    // 8-bit output with eight chunks a lane reads res and b where they are added (1024 x 65536: 119 us, with all loads
    // first it spilled, 150; 16-bit output does not: 96, and 102 the other way)
    constexpr int AB = Q8 && CH > 4 ? 1 : CH;
    Act8 h[CH], a[AB], b[AB];
    Gain<CH> w;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = sh.col(k);
      h[k] = rx.template load<POL>(c);
      if constexpr (AB == CH) {
        a[k] = rr.template load<POL>(c);
        b[k] = rb.load_by4(c);
      }
    }
    w.keep(gain, lanes, lane);
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float f[8], u[8], v[8];
      if constexpr (AB != CH) {
        a[0] = rr.template load<POL>(sh.col(k));
        b[0] = rb.load_by4(sh.col(k));
      }
      widen(h[k], f);
      widen(a[AB == CH ? k : 0], u);
      widen(b[AB == CH ? k : 0], v);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = f[e] + u[e] + v[e];
      h[k] = narrow(f);
      rh.template store<POL>(sh.col(k), h[k]);
      widen(h[k], f);
#pragma unroll
      for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
    }
    const float rstd = 1.0f / sqrtf(team.sum(ss) / (float)g.n + g.eps);
    const bool live = Shape<L>::kRows == 1 || t < g.T, leads = live && lane == 0;
    if (g.rstd && leads) g.rstd[t] = rstd;
    uint32_t row_max = 0;
    if constexpr (Q8) {
      if (g.group == g.n) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          float f[8], q[8];
          widen(h[k], f);
          w.get(gain, k, lanes, lane, q);
#pragma unroll
          for (int e = 0; e < 8; ++e) row_max = umax(row_max, mag(f[e] * rstd * q[e]));
        }
        row_max = team.max(row_max);
        if (leads) g.scale[t] = e4m3_scale(row_max);
      }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = sh.col(k);
      float f[8], q[8];
      widen(h[k], f);
      w.get(gain, k, lanes, lane, q);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = f[e] * rstd * q[e];
      if constexpr (Q8) {
        uint32_t m = row_max;
        if (g.group != g.n) {
          // groups of 32, 64, 128 or 256 columns: 4, 8, 16 or 32 aligned lanes, all of them in the row or none
          m = 0;
#pragma unroll
          for (int e = 0; e < 8; ++e) m = umax(m, mag(f[e]));
          m = max_step<kXor2>(max_step<kXor1>(m));
          if (g.group >= 64) m = max_step<kHalfMirror>(m);
          if (g.group >= 128) m = max_step<kMirror>(m);
          if (g.group >= 256) m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
        }
        const float s = e4m3_scale(m), inv = 1.0f / s;
        if (g.group != g.n && live && c < g.n && c % g.group == 0)
          g.scale[t * (g.n / g.group) + c / g.group] = s;
        const uint2 code = {to_e4m3(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv),
                            to_e4m3(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv)};
        typename Shape<L>::template Of<uint8_t>((uint8_t*)g.y, t, g.T, g.ld_y, g.n).template store_codes<POL>(c, code);
      } else {
        Out((act_t*)g.y, t, g.T, g.ld_y, g.n).template store<POL>(c, narrow(f));
      }
    }
  }
}

// ---------------------------------------------------------------- backward
struct BwdArgs {
  int64_t T;
  int threads, n;  // threads: a block's
  const act_t *h, *g_y, *g_h;
  int64_t ld_h, ld_gy, ld_gh;
  const float *gamma, *rstd;
  act_t* g_x;
  int64_t ld_gx;
  float* part;  // partial sums of dgamma, [blocks][n]
  float* dgamma;
  int accumulate;
  int strips;  // blocks that form dgamma of 64 columns each, before those that own rows
};

// With eight chunks a lane g_h is read only where it is added (1024 x 65536: 240 us; kept from the start it spilled, 275).
template <int CH>
struct BwdRow {
  static constexpr int kGh = CH <= 4 ? CH : 0;
  Act8 h[CH], gy[CH], gh[kGh ? kGh : 1];
  float rstd;
};
template <int POL, int L, int CH>
__device__ __forceinline__ void load_row(const BwdArgs& g, int64_t t0, const Shape<L>& sh, BwdRow<CH>& v) {
  using In = typename Shape<L>::template Of<const act_t>;
  const int n = t0 < g.T ? g.n : 0;  // rows behind the last have no columns
  const int64_t t = (t0 < g.T ? t0 : 0) + sh.sub;
  const In rh(g.h, t, g.T, g.ld_h, n), ry(g.g_y, t, g.T, g.ld_gy, n), rg(g.g_h, t, g.T, g.ld_gh, n);
#pragma unroll
  for (int k = 0; k < CH; ++k) {
    const int c = sh.col(k);
    v.h[k] = rh.template load<POL>(c);
    v.gy[k] = ry.template load<POL>(c);
    if constexpr (BwdRow<CH>::kGh > 0) v.gh[k] = rg.template load<POL>(c);
  }
  v.rstd = g.rstd[t < g.T ? t : g.T - 1];
}

// dgamma of 64 columns over all rows: eight lanes across, the block's others down, which add every
// (threads / 8)-th row each; their sums meet within a wave, then in wave order.
__device__ __forceinline__ void gain_strip(const BwdArgs& g, float (&s_sum)[kMaxWaves][64]) {
  const int q = threadIdx.x & 7, down = g.threads >> 3;
  const int c = (int)blockIdx.x * 64 + q * 8;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < g.n) {
#pragma unroll 4
    for (int64_t t = threadIdx.x >> 3; t < g.T; t += down) {
      float f[8], v[8];
      widen(load8_at<0>(g.h + t * g.ld_h + c), f);
      widen(load8_at<0>(g.g_y + t * g.ld_gy + c), v);
      const float rstd = g.rstd[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e] * (f[e] * rstd);
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma unroll
    for (int o = 8; o <= 32; o <<= 1) acc[e] += __shfl_xor(acc[e], o);
    if ((threadIdx.x & 63) < 8) s_sum[threadIdx.x >> 6][q * 8 + e] = acc[e];
  }
  __syncthreads();
  const int col = (int)blockIdx.x * 64 + (int)threadIdx.x;
  if (threadIdx.x < 64 && col < g.n) {
    float s = s_sum[0][threadIdx.x];
    for (int i = 1; i < g.threads >> 6; ++i) s += s_sum[i][threadIdx.x];
    g.dgamma[col] = g.accumulate ? g.dgamma[col] + s : s;
  }
}

// g_x and (GAIN) dgamma in one pass: a team takes every step-th row, with the next row's loads in
// flight, and adds its rows' dgamma in registers; a block writes one row of partial sums at the end,
// its waves' rows' (L != 0) added in their order.  Without GAIN: few rows, whose dgamma is formed beside
// them (gain_strip: it takes rstd and not the rows' means, so neither waits for the other), or rows too
// wide for sums in registers (k_norm_gain).
template <int L, int CH, bool GAIN, int POL>
__global__ __launch_bounds__(Shape<L>::kThreads) void k_norm_bwd(BwdArgs g) {
  __shared__ uint32_t s_red[2 * kMaxWaves];
  Team<L> team{s_red, g.threads >> 6, 0};
  const Shape<L> sh(g.threads, GAIN ? 0 : g.strips);
  constexpr int R = Shape<L>::kRows;
  const int lanes = sh.lanes, lane = sh.lane;
  if constexpr (!GAIN) {
    if ((int)blockIdx.x < g.strips) {
      __shared__ float s_gain[kMaxWaves][64];
      gain_strip(g, s_gain);
      return;
    }
  }
  const rsrc_t gain = make_rsrc(g.gamma, (int64_t)g.n * 4);
  Gain<CH> w;
  w.keep(gain, lanes, lane);
  float acc[GAIN ? CH : 1][8];
  if constexpr (GAIN)
#pragma unroll
    for (int k = 0; k < CH; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[k][e] = 0.0f;
  BwdRow<CH> row;
  int64_t t0 = sh.first;
  if constexpr (GAIN) load_row<POL>(g, t0, sh, row);
  for (; t0 < g.T; t0 += sh.step) {
    BwdRow<CH> next;
    if constexpr (GAIN)
      load_row<POL>(g, t0 + sh.step, sh, next);
    else
      load_row<POL>(g, t0, sh, row);
    float dot = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float f[8], v[8], a[8];
      widen(row.h[k], f);
      widen(row.gy[k], v);
      w.get(gain, k, lanes, lane, a);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float q = v[e] * (f[e] * row.rstd);  // g_y xh
        if constexpr (GAIN) acc[k][e] += q;
        dot += q * a[e];
      }
    }
    const float mean = team.sum(dot) / (float)g.n;
    const typename Shape<L>::template Of<act_t> ro(g.g_x, t0 + sh.sub, g.T, g.ld_gx, g.n);
    const typename Shape<L>::template Of<const act_t> rg(g.g_h, t0 + sh.sub, g.T, g.ld_gh, g.n);
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      float f[8], v[8], u[8], a[8];
      widen(row.h[k], f);
      widen(row.gy[k], v);
      if constexpr (BwdRow<CH>::kGh > 0)
        widen(row.gh[k], u);
      else
        widen(rg.template load<POL>(sh.col(k)), u);
      w.get(gain, k, lanes, lane, a);
#pragma unroll
      for (int e = 0; e < 8; ++e) f[e] = (v[e] * a[e] - f[e] * row.rstd * mean) * row.rstd + u[e];
      ro.template store<POL>(sh.col(k), narrow(f));
    }
    if constexpr (GAIN) row = next;
  }
  if constexpr (GAIN) {
    if constexpr (L != 0) {
      constexpr int S = Shape<L>::kBlockRows;  // rows that have sums of their own
      __shared__ float s_sum[S][L * 8];
      const int mine = (int)(threadIdx.x >> 6) * R + sh.sub;
#pragma unroll
      for (int e = 0; e < 8; ++e) s_sum[mine][lane * 8 + e] = acc[0][e];
      __syncthreads();
      for (int c = threadIdx.x; c < g.n; c += Shape<L>::kThreads) {
        float s = s_sum[0][c];
#pragma unroll
        for (int i = 1; i < S; ++i) s += s_sum[i][c];
        g.part[(int64_t)blockIdx.x * g.n + c] = s;
      }
    } else {
#pragma unroll
      for (int k = 0; k < CH; ++k) {
        const int c = (k * lanes + lane) * 8;
        if (c < g.n) {
          float* out = g.part + (int64_t)blockIdx.x * g.n + c;
          ((float4*)out)[0] = make_float4(acc[k][0], acc[k][1], acc[k][2], acc[k][3]);
          ((float4*)out)[1] = make_float4(acc[k][4], acc[k][5], acc[k][6], acc[k][7]);
        }
      }
    }
  }
}

// Partial sums of dgamma of wide rows: block (strip, group) adds the rows of its token group in 512
// columns, wave w the rows t = w mod 4 of it; the four waves' sums meet in LDS in wave order.
__global__ __launch_bounds__(256) void k_norm_gain(BwdArgs g, int64_t rows) {
  __shared__ float s_sum[4][512];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int c = (blockIdx.x * 64 + lane) * 8;
  const int64_t t0 = blockIdx.y * rows, t1 = t0 + rows < g.T ? t0 + rows : g.T;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll 4
  for (int64_t t = t0 + wave; t < t1; t += 4) {
    float f[8], v[8];
    widen(Row<true, const act_t>(g.h, t, g.T, g.ld_h, g.n).load<0>(c), f);
    widen(Row<true, const act_t>(g.g_y, t, g.T, g.ld_gy, g.n).load<0>(c), v);
    const float rstd = g.rstd[t];
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] += v[e] * (f[e] * rstd);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_sum[wave][lane * 8 + e] = acc[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int col = blockIdx.x * 512 + i;
    if (col < g.n) g.part[(int64_t)blockIdx.y * g.n + col] = (s_sum[0][i] + s_sum[1][i]) + (s_sum[2][i] + s_sum[3][i]);
  }
}

// dgamma (+)= the partial sums.  A block takes 32 columns: 64 threads down, eight loads each in
// flight (one after the other they took 6.9 us for 501 rows of 2112 sums), add every 64th row; the
// 64 sums of a column meet in two steps.  The order is fixed by the row's number alone.
__global__ __launch_bounds__(512) void k_norm_gain_sum(int n, int parts, const float* __restrict__ part,
                                                       float* __restrict__ dgamma, int accumulate) {
  __shared__ float s_sum[64][33], s_col[16][33];
  const int q = threadIdx.x & 7, row = threadIdx.x >> 3;
  const int c = blockIdx.x * 32 + q * 4;
  float4 a = make_float4(0, 0, 0, 0);
  if (c < n) {  // n is a multiple of 8
    for (int i0 = row; i0 < parts; i0 += 512) {
      float4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int i = i0 + 64 * u;
        v[u] = i < parts ? *(const float4*)(part + (int64_t)i * n + c) : make_float4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) a.x += v[u].x, a.y += v[u].y, a.z += v[u].z, a.w += v[u].w;
    }
  }
  s_sum[row][q * 4 + 0] = a.x;
  s_sum[row][q * 4 + 1] = a.y;
  s_sum[row][q * 4 + 2] = a.z;
  s_sum[row][q * 4 + 3] = a.w;
  __syncthreads();
  const int i = threadIdx.x & 31, k = threadIdx.x >> 5;
  s_col[k][i] = (s_sum[k][i] + s_sum[k + 16][i]) + (s_sum[k + 32][i] + s_sum[k + 48][i]);
  __syncthreads();
  const int col = blockIdx.x * 32 + i;
  if (k == 0 && col < n) {
    float s = 0.0f;
#pragma unroll
    for (int u = 0; u < 16; ++u) s += s_col[u][i];
    dgamma[col] = accumulate ? dgamma[col] + s : s;
  }
}

// ---------------------------------------------------------------- host
using resbm_host::aligned;
using resbm_host::extent;
using resbm_host::launch_status;
using resbm_host::ld_ok;
using resbm_host::overlap;

constexpr int kMaxWidth = 65536;
constexpr int64_t kMaxBlocks = 1 << 20;  // a launch's threads stay below 2^32; rows beyond take further turns

inline bool width_ok(int64_t T, int n) { return T >= 0 && T <= INT32_MAX && n >= 8 && n <= kMaxWidth && n % 8 == 0; }

inline int64_t blocks_for(int64_t T, int rpb) {
  const int64_t b = (T + rpb - 1) / rpb;
  return b < kMaxBlocks ? b : kMaxBlocks;
}

constexpr int kWaveWidth = 512;     // columns that a wave holds in one chunk a lane
constexpr int kGainWidth = 16384;   // the widest row whose dgamma sums stay in a block's registers
constexpr int kStream = 2;          // the cache policy "not to be used again soon"

// Loads and stores of tensors that the caches would not hold until their next use bypass them: the
// 256 MB behind the L2s keep what fits.  Forward at n = 4096, passes over three sets of tensors in turn:
// 67 MB each 11.7 us cached and 14.0 streaming, 134 MB 26.2 and 24.9, 538 MB 94.6 and 90.7.
inline bool streams_through(size_t bytes) { return bytes > ((size_t)120 << 20); }

// Lanes of a wave that own a row (0: a block does): several narrow rows share a wave.
inline int row_lanes(int n) { return n > kWaveWidth ? 0 : n <= 128 ? 16 : n <= 256 ? 32 : 64; }

// Blocks of the backward pass (GAIN: each writes a row of partial sums) and rows each takes, all nearly
// as many.  A multiple of the 256 compute units with about 2^20 columns in all, whose loads for two rows
// keep HBM busy; more blocks than that only add partial sums and contend: at 16384 x 4096, 256 blocks
// take 88.5 us, 512 98 us, 1024 107 us; at 32768 x 2048, 256 take 113, 512 93 and 1024 105 us.
struct GainPlan {
  int parts;
  int64_t rows;
};
inline GainPlan gain_plan(int64_t T, int n) {
  const int lanes = row_lanes(n);
  const int64_t unit = lanes ? 64 / lanes * kRowWaves : n <= kGainWidth ? 1 : 64;
  const int64_t fill = (4096 + n / 2) / n;
  const int64_t most = lanes ? 512 : 256 * (fill < 1 ? 1 : fill > 4 ? 4 : fill);
  const int64_t units = (T + unit - 1) / unit;
  const int64_t turns = (units + most - 1) / most;
  return {(int)((units + turns - 1) / turns), turns * unit};
}

// Chunks a lane.  16-bit output: one while eight waves hold the row (16384 x 4096: 90.7 us against 94.7 with
// two chunks and 93.2 with four), four beyond (16384 x 8192: 182 against 194 with two; 5120: 116 against 118).
// 8-bit output, with its maxima: two (16384 x 4096: 80.5 against 84 with one or four; 8192: 159 against 169
// with four).  Few rows leave compute units idle anyway and take a lane a chunk, to shorten each one's chain
// (on the device, one row: 16 bits n = 8192 3.1 us against 3.3, 8 bits n = 2048 2.6 against 2.9), except 8 bits
// above 4096, where sixteen waves meet twice (4.0 against 3.7).
inline int chunks_fwd(int64_t T, int n, bool q8) {
  if (n > 16384) return n <= 32768 ? 4 : 8;
  if (T <= 256 && n <= (q8 ? 4096 : 8192)) return 1;
  if (q8) return 2;
  return n <= 4096 ? 1 : 4;
}
inline int chunks_bwd(int n) { return n <= 4096 ? 1 : n <= 16384 ? 2 : n <= 32768 ? 4 : 8; }
inline int block_threads(int n, int ch) { return 64 * ((n + 512 * ch - 1) / (512 * ch)); }

template <bool Q8, int POL>
void run_fwd(FwdArgs g, hipStream_t s) {
  if (const int l = row_lanes(g.n)) {
    const dim3 few((uint32_t)blocks_for(g.T, 64 / l * kRowWaves)), four(64 * kRowWaves);
    g.threads = 64 * kRowWaves;
    if (l == 16)
      hipLaunchKernelGGL((k_norm_fwd<16, 1, Q8, POL>), few, four, 0, s, g);
    else if (l == 32)
      hipLaunchKernelGGL((k_norm_fwd<32, 1, Q8, POL>), few, four, 0, s, g);
    else
      hipLaunchKernelGGL((k_norm_fwd<64, 1, Q8, POL>), few, four, 0, s, g);
    return;
  }
  const int ch = chunks_fwd(g.T, g.n, Q8);
  const dim3 grid((uint32_t)blocks_for(g.T, 1)), blk(block_threads(g.n, ch));
  g.threads = (int)blk.x;
  switch (ch) {
    case 1: hipLaunchKernelGGL((k_norm_fwd<0, 1, Q8, POL>), grid, blk, 0, s, g); break;
    case 2: hipLaunchKernelGGL((k_norm_fwd<0, 2, Q8, POL>), grid, blk, 0, s, g); break;
    case 4: hipLaunchKernelGGL((k_norm_fwd<0, 4, Q8, POL>), grid, blk, 0, s, g); break;
    default: hipLaunchKernelGGL((k_norm_fwd<0, 8, Q8, POL>), grid, blk, 0, s, g); break;
  }
}

template <bool GAIN, int POL>
void launch_bwd(const BwdArgs& g, int l, int ch, dim3 grid, hipStream_t s) {
  const dim3 blk(g.threads);
  if (l == 16)
    hipLaunchKernelGGL((k_norm_bwd<16, 1, GAIN, POL>), grid, blk, 0, s, g);
  else if (l == 32)
    hipLaunchKernelGGL((k_norm_bwd<32, 1, GAIN, POL>), grid, blk, 0, s, g);
  else if (l == 64)
    hipLaunchKernelGGL((k_norm_bwd<64, 1, GAIN, POL>), grid, blk, 0, s, g);
  else if (ch == 1)
    hipLaunchKernelGGL((k_norm_bwd<0, 1, GAIN, POL>), grid, blk, 0, s, g);
  else
    hipLaunchKernelGGL((k_norm_bwd<0, 2, GAIN, POL>), grid, blk, 0, s, g);
}
inline void launch_wide(const BwdArgs& g, int ch, dim3 grid, hipStream_t s) {
  if (ch == 4)
    hipLaunchKernelGGL((k_norm_bwd<0, 4, false, 0>), grid, dim3(g.threads), 0, s, g);
  else
    hipLaunchKernelGGL((k_norm_bwd<0, 8, false, 0>), grid, dim3(g.threads), 0, s, g);
}

// Whether dgamma is formed beside the rows, in the same launch: up to eight rows a lane (a block's threads / 8
// rows go down at once), where that takes no longer than the second launch (n = 2048, 128 rows 4.5 us against
// 7.4, 256 rows 5.8 against 7.4, 512 rows 14 against 7.6; n = 1024, 128 rows 5.4 against 7.1, 256 rows 7.7
// against 7.1; n = 4096, 256 rows 6.5 against 7.6, 512 rows 10.7 against 8.5).
inline bool few_rows(int64_t T, int threads) { return T <= 256 && T <= threads; }

inline void run_bwd(BwdArgs g, float* ws, hipStream_t s) {
  const int l = row_lanes(g.n), ch = chunks_bwd(g.n);
  const bool wide = g.n > kGainWidth;
  const dim3 all((uint32_t)blocks_for(g.T, l ? 64 / l * kRowWaves : 1));
  g.threads = l ? 64 * kRowWaves : block_threads(g.n, ch);
  if (few_rows(g.T, g.threads)) {
    // one launch, or two where g_x takes the place of g_y, which dgamma reads
    const int strips = (g.n + 63) / 64;
    const bool place = g.g_x == g.g_y;
    for (int pass = place ? 0 : 1; pass < 2; ++pass) {
      g.strips = place && pass == 1 ? 0 : strips;
      const dim3 grid(g.strips + (place && pass == 0 ? 0 : all.x));
      wide ? launch_wide(g, ch, grid, s) : launch_bwd<false, 0>(g, l, ch, grid, s);
    }
    return;
  }
  const bool once = streams_through((3 + (g.g_h != nullptr)) * (size_t)g.T * g.n * kActBytes);
  const GainPlan p = gain_plan(g.T, g.n);
  g.part = ws;
  if (wide) {  // before g_x, which may take g_y's place
    hipLaunchKernelGGL(k_norm_gain, dim3((g.n + 511) / 512, p.parts), dim3(256), 0, s, g, p.rows);
    launch_wide(g, ch, all, s);
  } else {
    once ? launch_bwd<true, kStream>(g, l, ch, dim3(p.parts), s) : launch_bwd<true, 0>(g, l, ch, dim3(p.parts), s);
  }
  hipLaunchKernelGGL(k_norm_gain_sum, dim3((g.n + 31) / 32), dim3(512), 0, s, g.n, p.parts, (const float*)g.part, g.dgamma,
                     g.accumulate);
}

// Checks and arguments shared by the two forward ops; group == 0: 16-bit (or float32) output.
inline int32_t fwd(int64_t T, int32_t n, int32_t r, int32_t group, const void* x, int64_t ld_x, const void* res,
                   int64_t ld_res, const void* b, const float* gamma, float eps, void* h, int64_t ld_h, void* y,
                   int64_t ld_y, float* scale, float* rstd, void* stream) {
  if (!width_ok(T, n) || !(eps >= 0.0f) || eps > 3.0e38f) return RESBM_E_SHAPE;
  if (r < 0 || r > n || r % 4 != 0) return RESBM_E_SHAPE;
  const bool q8 = group != 0;
  if (q8 && group != n && ((group != 32 && group != 64 && group != 128 && group != 256) || n % group != 0))
    return RESBM_E_SHAPE;
  if (T == 0) return RESBM_OK;
  if (!x || !gamma || !y || (q8 && !scale) || (r > 0 && !b)) return RESBM_E_NULL;
  if (!ld_ok(ld_x, n) || (res && !ld_ok(ld_res, n)) || (h && !ld_ok(ld_h, n)) || !ld_ok(ld_y, n)) return RESBM_E_SHAPE;
  if (!aligned(x, 16) || !aligned(res, 16) || !aligned(h, 16) || !aligned(y, 16) || !aligned(gamma, 16) ||
      (r > 0 && !aligned(b, 16)) || !aligned(scale, 4) || !aligned(rstd, 4))
    return RESBM_E_ALIGN;
  const size_t bx = extent(T, n, ld_x, kActBytes), br = extent(T, n, ld_res, kActBytes);
  const size_t bh = extent(T, n, ld_h, kActBytes), by = extent(T, n, ld_y, q8 ? 1 : kActBytes);
  const size_t bb = (size_t)T * r * kActBytes, bg = (size_t)n * 4, bt = (size_t)T * 4;
  const size_t bs = q8 ? (size_t)T * (n / group) * 4 : 0;
  struct Range {
    const void* p;
    size_t n;
  };
  const Range in[4] = {{x, bx}, {res, br}, {r > 0 ? b : nullptr, bb}, {gamma, bg}};
  const Range out[4] = {{h, bh}, {y, by}, {scale, bs}, {rstd, bt}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 4; ++j) {
      // h may take the place of x or res, element for element: each is read before h is written there
      if (i == 0 && ((j == 0 && h == x && ld_h == ld_x) || (j == 1 && h == res && ld_h == ld_res))) continue;
      if (overlap(out[i].p, out[i].n, in[j].p, in[j].n)) return RESBM_E_ALIAS;
    }
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].n, out[j].p, out[j].n)) return RESBM_E_ALIAS;
  }
  FwdArgs g{};
  g.T = T, g.n = n, g.r = r, g.group = group, g.eps = eps;
  g.x = (const act_t*)x, g.ld_x = ld_x;
  g.res = (const act_t*)res, g.ld_res = ld_res;
  g.b = (const act_t*)b;
  g.gamma = gamma;
  g.h = (act_t*)h, g.ld_h = ld_h;
  g.y = y, g.ld_y = ld_y;
  g.scale = scale, g.rstd = rstd;
  const hipStream_t st = (hipStream_t)stream;
  const bool once = streams_through((1 + (res != nullptr) + (h != nullptr)) * (size_t)T * n * kActBytes + (size_t)T * n * (q8 ? 1 : kActBytes));
  if (q8)
    once ? run_fwd<true, kStream>(g, st) : run_fwd<true, 0>(g, st);
  else
    once ? run_fwd<false, kStream>(g, st) : run_fwd<false, 0>(g, st);
  return launch_status();
}

}  // namespace resbm_nm

extern "C" {

size_t resbm_norm_workspace_bytes(int64_t T, int32_t n) {
  if (!resbm_nm::width_ok(T, n)) return 0;
  if (T == 0) return 256;
  return ((size_t)resbm_nm::gain_plan(T, n).parts * n * 4 + 255) & ~(size_t)255;
}

int32_t resbm_skip_norm_fwd(int64_t T, int32_t n, int32_t r, const void* x, int64_t ld_x, const void* res,
                            int64_t ld_res, const void* b, const float* gamma, float eps, void* h, int64_t ld_h,
                            void* y, int64_t ld_y, float* rstd, void* stream) {
  return resbm_nm::fwd(T, n, r, 0, x, ld_x, res, ld_res, b, gamma, eps, h, ld_h, y, ld_y, nullptr, rstd, stream);
}

int32_t resbm_skip_norm_q8_fwd(int64_t T, int32_t n, int32_t r, int32_t group, const void* x, int64_t ld_x,
                               const void* res, int64_t ld_res, const void* b, const float* gamma, float eps, void* h,
                               int64_t ld_h, void* y, int64_t ld_y, float* scale, float* rstd, void* stream) {
  if (group <= 0) return RESBM_E_SHAPE;
  return resbm_nm::fwd(T, n, r, group, x, ld_x, res, ld_res, b, gamma, eps, h, ld_h, y, ld_y, scale, rstd, stream);
}

int32_t resbm_skip_norm_bwd(int64_t T, int32_t n, const void* h, int64_t ld_h, const float* gamma, const float* rstd,
                            const void* g_y, int64_t ld_gy, const void* g_h, int64_t ld_gh, void* g_x, int64_t ld_gx,
                            float* dgamma, int32_t accumulate, void* ws, size_t ws_bytes, void* stream) {
  using namespace resbm_nm;
  if (!width_ok(T, n)) return RESBM_E_SHAPE;
  if (T == 0) return RESBM_OK;
  if (!h || !gamma || !rstd || !g_y || !g_x || !dgamma || !ws) return RESBM_E_NULL;
  if (!ld_ok(ld_h, n) || !ld_ok(ld_gy, n) || (g_h && !ld_ok(ld_gh, n)) || !ld_ok(ld_gx, n)) return RESBM_E_SHAPE;
  if (!aligned(h, 16) || !aligned(g_y, 16) || !aligned(g_h, 16) || !aligned(g_x, 16) || !aligned(gamma, 16) ||
      !aligned(rstd, 4) || !aligned(dgamma, 16) || !aligned(ws, 256))
    return RESBM_E_ALIGN;
  const size_t need = resbm_norm_workspace_bytes(T, n);
  if (ws_bytes < need) return RESBM_E_WORKSPACE;
  const size_t bg = (size_t)n * 4, bt = (size_t)T * 4;
  const struct {
    const void* p;
    size_t n;
    bool place;  // g_x may take this input's place
  } in[5] = {{h, extent(T, n, ld_h, kActBytes), false},
             {g_y, extent(T, n, ld_gy, kActBytes), g_x == g_y && ld_gx == ld_gy},
             {g_h, extent(T, n, ld_gh, kActBytes), g_x == g_h && ld_gx == ld_gh},
             {gamma, bg, false},
             {rstd, bt, false}};
  const size_t bx = extent(T, n, ld_gx, kActBytes);
  for (const auto& i : in)
    if ((!i.place && overlap(g_x, bx, i.p, i.n)) || overlap(dgamma, bg, i.p, i.n) || overlap(ws, need, i.p, i.n))
      return RESBM_E_ALIAS;
  if (overlap(g_x, bx, dgamma, bg) || overlap(ws, need, g_x, bx) || overlap(ws, need, dgamma, bg)) return RESBM_E_ALIAS;
  BwdArgs g{};
  g.T = T, g.n = n;
  g.h = (const act_t*)h, g.ld_h = ld_h;
  g.g_y = (const act_t*)g_y, g.ld_gy = ld_gy;
  g.g_h = (const act_t*)g_h, g.ld_gh = ld_gh;
  g.gamma = gamma, g.rstd = rstd;
  g.g_x = (act_t*)g_x, g.ld_gx = ld_gx;
  g.dgamma = dgamma, g.accumulate = accumulate;
  run_bwd(g, (float*)ws, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"
