// resbm_norm.hpp -- the residual addition with its RMS norm, and that norm's backward, gfx950.
//
// Between two layers the residual stream is formed and normalised:
//     h = x + res + b I_{r x n}                     (the decoder's skip, Eq. 5, in the same pass)
//     y = h rstd gamma,   rstd = 1 / sqrt(mean_c h^2 + eps)
// and backwards, with xh = h rstd, w = g_y gamma, c = mean_c(w xh),
//     g_x = rstd (w - xh c) + g_h,   dgamma = sum_t g_y xh.
// Every op reads each operand once and writes each result once, so HBM bounds them (about one
// operation a byte); a row has to be whole before any of its results, so a team of TEAM lanes owns
// a row and keeps it in registers: one wave for narrow rows, a block for wide ones.  The stream h is
// rounded once, to the activations' type, and the norm is that of the rounded h, whether h is written
// or not: then the backward pass, which reads h, is the adjoint of what the forward computed.
// Included by resbm_matrix.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "resbm.h"
#include "resbm_host.hpp"

#ifndef RESBM_IO_F32_BUILD
#define RESBM_IO_F32_BUILD 0
#endif

namespace resbm_nm {

// ---------------------------------------------------------------- eight activations
#if RESBM_IO_F32_BUILD
typedef float act_t;
struct Act8 {
  float4 a, b;
};
__device__ __forceinline__ Act8 load8(const act_t* p) { return {((const float4*)p)[0], ((const float4*)p)[1]}; }
__device__ __forceinline__ void store8(act_t* p, const Act8& v) {
  ((float4*)p)[0] = v.a;
  ((float4*)p)[1] = v.b;
}
__device__ __forceinline__ Act8 zero8() { return {make_float4(0, 0, 0, 0), make_float4(0, 0, 0, 0)}; }
__device__ __forceinline__ void widen(const Act8& v, float (&f)[8]) {
  f[0] = v.a.x, f[1] = v.a.y, f[2] = v.a.z, f[3] = v.a.w;
  f[4] = v.b.x, f[5] = v.b.y, f[6] = v.b.z, f[7] = v.b.w;
}
__device__ __forceinline__ Act8 narrow(const float (&f)[8]) {
  return {make_float4(f[0], f[1], f[2], f[3]), make_float4(f[4], f[5], f[6], f[7])};
}
__device__ __forceinline__ void widen4(const act_t* p, float (&f)[4]) {
  const float4 v = *(const float4*)p;
  f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
}
#else
typedef __bf16 act_t;
typedef __bf16 nbf2 __attribute__((ext_vector_type(2)));
struct Act8 {
  uint4 v;
};
__device__ __forceinline__ Act8 load8(const act_t* p) { return {*(const uint4*)p}; }
__device__ __forceinline__ void store8(act_t* p, const Act8& v) { *(uint4*)p = v.v; }
__device__ __forceinline__ Act8 zero8() { return {make_uint4(0, 0, 0, 0)}; }
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
__device__ __forceinline__ void widen4(const act_t* p, float (&f)[4]) {
  const uint2 v = *(const uint2*)p;
  f[0] = lo16(v.x), f[1] = hi16(v.x), f[2] = lo16(v.y), f[3] = hi16(v.y);
}
#endif
constexpr size_t kActBytes = sizeof(act_t);

__device__ __forceinline__ void load_gain(const float* gamma, int c, float (&f)[8]) {
  const float4 a = ((const float4*)(gamma + c))[0], b = ((const float4*)(gamma + c))[1];
  f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
}

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

// The team's sum or maximum.  One barrier: the slot alternates, and a slot is written again only
// behind the barrier of the call in between, which every reader of its old values has passed.
template <int TEAM>
struct Team {
  float* lds;  // 2 * TEAM / 64 words (unused with TEAM == 64)
  int slot;
  __device__ __forceinline__ float sum(float v) {
    v = wave_sum(v);
    if constexpr (TEAM == 64) return v;
    float* s = lds + slot * (TEAM / 64);
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    float r = s[0];
#pragma unroll
    for (int i = 1; i < TEAM / 64; ++i) r += s[i];
    return r;
  }
  __device__ __forceinline__ uint32_t max(uint32_t v) {
    v = wave_max(v);
    if constexpr (TEAM == 64) return v;
    uint32_t* s = (uint32_t*)lds + slot * (TEAM / 64);
    slot ^= 1;
    if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = v;
    __syncthreads();
    uint32_t r = s[0];
#pragma unroll
    for (int i = 1; i < TEAM / 64; ++i) r = umax(r, s[i]);
    return r;
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

template <int TEAM>
constexpr int block_of() {
  return TEAM > 256 ? TEAM : 256;
}

template <int TEAM, int CH, bool Q8>
__global__ __launch_bounds__(block_of<TEAM>()) void k_norm_fwd(FwdArgs g) {
  constexpr int RPB = block_of<TEAM>() / TEAM;  // rows a block has at a time
  __shared__ float s_red[2 * (TEAM / 64)];
  Team<TEAM> team{s_red, 0};
  const int lane = threadIdx.x % TEAM;
  const int64_t step = (int64_t)gridDim.x * RPB;
  // a row's wave (TEAM == 64) or block goes through the loop as one: the barriers are uniform
  for (int64_t t = (int64_t)blockIdx.x * RPB + threadIdx.x / TEAM; t < g.T; t += step) {
    Act8 h[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      h[k] = c < g.n ? load8(g.x + t * g.ld_x + c) : zero8();
    }
    float ss = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      if (c < g.n) {
        float f[8];
        widen(h[k], f);
        if (g.res) {
          float v[8];
          widen(load8(g.res + t * g.ld_res + c), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += v[e];
        }
#pragma unroll
        for (int q = 0; q < 2; ++q)  // r is a multiple of 4
          if (c + 4 * q < g.r) {
            float v[4];
            widen4(g.b + t * g.r + c + 4 * q, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[4 * q + e] += v[e];
          }
        h[k] = narrow(f);
        if (g.h) store8(g.h + t * g.ld_h + c, h[k]);
        widen(h[k], f);
#pragma unroll
        for (int e = 0; e < 8; ++e) ss += f[e] * f[e];
      }
    }
    const float rstd = 1.0f / sqrtf(team.sum(ss) / (float)g.n + g.eps);
    if (g.rstd && lane == 0) g.rstd[t] = rstd;
    uint32_t row_max = 0;
    if constexpr (Q8) {
      if (g.group == g.n) {
#pragma unroll
        for (int k = 0; k < CH; ++k) {
          const int c = (k * TEAM + lane) * 8;
          if (c < g.n) {
            float f[8], w[8];
            widen(h[k], f);
            load_gain(g.gamma, c, w);
#pragma unroll
            for (int e = 0; e < 8; ++e) row_max = umax(row_max, mag(f[e] * rstd * w[e]));
          }
        }
        row_max = team.max(row_max);
        if (lane == 0) g.scale[t] = e4m3_scale(row_max);
      }
    }
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      const bool in = c < g.n;
      float f[8], w[8];
      if (in) {
        widen(h[k], f);
        load_gain(g.gamma, c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = f[e] * rstd * w[e];
      }
      if constexpr (Q8) {
        uint32_t m = row_max;
        if (g.group != g.n) {
          // groups of 32, 64, 128 or 256 columns: 4, 8, 16 or 32 aligned lanes; a lane without columns gives 0
          m = 0;
          if (in)
#pragma unroll
            for (int e = 0; e < 8; ++e) m = umax(m, mag(f[e]));
          m = max_step<kXor2>(max_step<kXor1>(m));
          if (g.group >= 64) m = max_step<kHalfMirror>(m);
          if (g.group >= 128) m = max_step<kMirror>(m);
          if (g.group >= 256) m = umax(m, (uint32_t)__shfl_xor((int)m, 16));
        }
        if (in) {
          const float s = e4m3_scale(m), inv = 1.0f / s;
          if (g.group != g.n && c % g.group == 0) g.scale[t * (g.n / g.group) + c / g.group] = s;
          uint2 q;
          q.x = to_e4m3(f[0] * inv, f[1] * inv, f[2] * inv, f[3] * inv);
          q.y = to_e4m3(f[4] * inv, f[5] * inv, f[6] * inv, f[7] * inv);
          *(uint2*)((uint8_t*)g.y + t * g.ld_y + c) = q;
        }
      } else {
        if (in) store8((act_t*)g.y + t * g.ld_y + c, narrow(f));
      }
    }
  }
}

// ---------------------------------------------------------------- backward
struct BwdArgs {
  int64_t T;
  int n;
  const act_t *h, *g_y, *g_h;
  int64_t ld_h, ld_gy, ld_gh;
  const float *gamma, *rstd;
  act_t* g_x;
  int64_t ld_gx;
};

// g_x, a row at a time.
template <int TEAM, int CH>
__global__ __launch_bounds__(block_of<TEAM>()) void k_norm_bwd(BwdArgs g) {
  constexpr int RPB = block_of<TEAM>() / TEAM;
  __shared__ float s_red[2 * (TEAM / 64)];
  Team<TEAM> team{s_red, 0};
  const int lane = threadIdx.x % TEAM;
  const int64_t step = (int64_t)gridDim.x * RPB;
  for (int64_t t = (int64_t)blockIdx.x * RPB + threadIdx.x / TEAM; t < g.T; t += step) {
    Act8 h[CH], gy[CH];
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      h[k] = c < g.n ? load8(g.h + t * g.ld_h + c) : zero8();
      gy[k] = c < g.n ? load8(g.g_y + t * g.ld_gy + c) : zero8();
    }
    const float rstd = g.rstd[t];
    float dot = 0.0f;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      if (c < g.n) {
        float f[8], v[8], w[8];
        widen(h[k], f);
        widen(gy[k], v);
        load_gain(g.gamma, c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) dot += v[e] * w[e] * (f[e] * rstd);
      }
    }
    const float mean = team.sum(dot) / (float)g.n;
#pragma unroll
    for (int k = 0; k < CH; ++k) {
      const int c = (k * TEAM + lane) * 8;
      if (c < g.n) {
        float f[8], v[8], w[8];
        widen(h[k], f);
        widen(gy[k], v);
        load_gain(g.gamma, c, w);
#pragma unroll
        for (int e = 0; e < 8; ++e) f[e] = (v[e] * w[e] - f[e] * rstd * mean) * rstd;
        if (g.g_h) {
          widen(load8(g.g_h + t * g.ld_gh + c), v);
#pragma unroll
          for (int e = 0; e < 8; ++e) f[e] += v[e];
        }
        store8(g.g_x + t * g.ld_gx + c, narrow(f));
      }
    }
  }
}

// Partial sums of dgamma: block (strip, group) adds the rows of its token group in 512 columns,
// wave w the rows t = w mod 4 of it; the four waves' sums meet in LDS in wave order.
__global__ __launch_bounds__(256) void k_norm_gain(BwdArgs g, int64_t rows, float* part) {
  __shared__ float s_sum[4][512];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = (blockIdx.x * 64 + lane) * 8;
  const int64_t t0 = blockIdx.y * rows, t1 = t0 + rows < g.T ? t0 + rows : g.T;
  float acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (c < g.n)
    for (int64_t t = t0 + wave; t < t1; t += 4) {
      float f[8], v[8];
      widen(load8(g.h + t * g.ld_h + c), f);
      widen(load8(g.g_y + t * g.ld_gy + c), v);
      const float rstd = g.rstd[t];
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[e] += v[e] * (f[e] * rstd);
    }
#pragma unroll
  for (int e = 0; e < 8; ++e) s_sum[wave][lane * 8 + e] = acc[e];
  __syncthreads();
  for (int i = threadIdx.x; i < 512; i += 256) {
    const int col = blockIdx.x * 512 + i;
    if (col < g.n) part[(int64_t)blockIdx.y * g.n + col] = (s_sum[0][i] + s_sum[1][i]) + (s_sum[2][i] + s_sum[3][i]);
  }
}

// dgamma (+)= the partial sums, added in the order of their rows modulo 32, then of the 32 sums.
__global__ __launch_bounds__(256) void k_norm_gain_sum(int n, int parts, const float* part, float* dgamma,
                                                       int accumulate) {
  __shared__ float s_sum[32][33];
  const int q = threadIdx.x & 7, row = threadIdx.x >> 3;
  const int c = blockIdx.x * 32 + q * 4;
  float4 a = make_float4(0, 0, 0, 0);
  if (c < n)  // n is a multiple of 8
    for (int i = row; i < parts; i += 32) {
      const float4 v = *(const float4*)(part + (int64_t)i * n + c);
      a.x += v.x, a.y += v.y, a.z += v.z, a.w += v.w;
    }
  s_sum[row][q * 4 + 0] = a.x;
  s_sum[row][q * 4 + 1] = a.y;
  s_sum[row][q * 4 + 2] = a.z;
  s_sum[row][q * 4 + 3] = a.w;
  __syncthreads();
  const int i = threadIdx.x, col = blockIdx.x * 32 + i;
  if (i < 32 && col < n) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 32; ++k) s += s_sum[k][i];
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

// Token groups of the dgamma sums: 64 rows each, at most 256.
struct GainPlan {
  int parts;
  int64_t rows;
};
inline GainPlan gain_plan(int64_t T) {
  int64_t p = (T + 63) / 64;
  p = p > 256 ? 256 : p;
  const int64_t rows = (T + p - 1) / p;
  return {(int)((T + rows - 1) / rows), rows};
}

inline int64_t blocks_for(int64_t T, int rpb) {
  const int64_t b = (T + rpb - 1) / rpb;
  return b < kMaxBlocks ? b : kMaxBlocks;
}

template <int TEAM, int CH, bool Q8>
void launch_fwd(const FwdArgs& g, hipStream_t s) {
  constexpr int BLK = block_of<TEAM>();
  hipLaunchKernelGGL((k_norm_fwd<TEAM, CH, Q8>), dim3((uint32_t)blocks_for(g.T, BLK / TEAM)), dim3(BLK), 0, s, g);
}
template <bool Q8>
void run_fwd(const FwdArgs& g, hipStream_t s) {
  if (g.n <= 512) return launch_fwd<64, 1, Q8>(g, s);
  if (g.n <= 2048) return launch_fwd<256, 1, Q8>(g, s);
  if (g.n <= 4096) return launch_fwd<256, 2, Q8>(g, s);
  if (g.n <= 8192) return launch_fwd<256, 4, Q8>(g, s);
  if (g.n <= 16384) return launch_fwd<512, 4, Q8>(g, s);
  if (g.n <= 32768) return launch_fwd<1024, 4, Q8>(g, s);
  return launch_fwd<1024, 8, Q8>(g, s);
}

template <int TEAM, int CH>
void launch_bwd(const BwdArgs& g, hipStream_t s) {
  constexpr int BLK = block_of<TEAM>();
  hipLaunchKernelGGL((k_norm_bwd<TEAM, CH>), dim3((uint32_t)blocks_for(g.T, BLK / TEAM)), dim3(BLK), 0, s, g);
}
inline void run_bwd(const BwdArgs& g, float* part, float* dgamma, int accumulate, hipStream_t s) {
  const GainPlan p = gain_plan(g.T);
  // before g_x, which may take g_y's place
  hipLaunchKernelGGL(k_norm_gain, dim3((g.n + 511) / 512, p.parts), dim3(256), 0, s, g, p.rows, part);
  hipLaunchKernelGGL(k_norm_gain_sum, dim3((g.n + 31) / 32), dim3(256), 0, s, g.n, p.parts, (const float*)part, dgamma,
                     accumulate);
  if (g.n <= 512) return launch_bwd<64, 1>(g, s);
  if (g.n <= 2048) return launch_bwd<256, 1>(g, s);
  if (g.n <= 4096) return launch_bwd<256, 2>(g, s);
  if (g.n <= 8192) return launch_bwd<256, 4>(g, s);
  if (g.n <= 16384) return launch_bwd<512, 4>(g, s);
  if (g.n <= 32768) return launch_bwd<1024, 4>(g, s);
  return launch_bwd<1024, 8>(g, s);
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
  if (q8)
    run_fwd<true>(g, (hipStream_t)stream);
  else
    run_fwd<false>(g, (hipStream_t)stream);
  return launch_status();
}

}  // namespace resbm_nm

extern "C" {

size_t resbm_norm_workspace_bytes(int64_t T, int32_t n) {
  if (!resbm_nm::width_ok(T, n)) return 0;
  if (T == 0) return 256;
  return ((size_t)resbm_nm::gain_plan(T).parts * n * 4 + 255) & ~(size_t)255;
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
  run_bwd(g, (float*)ws, dgamma, accumulate, (hipStream_t)stream);
  return launch_status();
}

}  // extern "C"
