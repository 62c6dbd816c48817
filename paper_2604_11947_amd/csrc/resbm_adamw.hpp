// resbm_adamw.hpp -- one AdamW step, and the gradients' norm, over many tensors at once, gfx950.
//
// Muon (resbm_muon_update) takes a stage's bottleneck weights; gains, projections and embeddings take
//     m <- b1 m + (1 - b1) g,   v <- b2 v + (1 - b2) g^2,
//     p <- p (1 - lr wd) - (lr / c1) m / (sqrt(v) / sqrt(c2) + eps),   ck = 1 - bk^step,
// element by element on 16 to 30 bytes an element and some 15 operations, so HBM bounds it, and launch
// latency where the tensors are small.  One launch therefore covers all tensors: a plan in device memory
// lists them and, for every chunk of one to four thousand elements, the tensor that it belongs to.  A block takes a chunk
// at a time; a lane takes four consecutive elements, 16 bytes of every float32 array.
// Arithmetic is float32 in the order written above, every operation rounded once (no contraction), so that
// results do not depend on the form a tensor is listed in.
//
// States in 8 bits: blocks of 256 elements, counted from the tensor's start, hold m and u = sqrt(v) as e4m3
// with one float32 scale each, s = max(amax (1 / 448), 2^-126).  A block is the 256 elements that a wave takes at
// once, so its maximum is one reduction over lanes.  u rather than v, because the square root halves the
// exponent's range: 2^-9 .. 448 covers u over five decades, v over ten.  A non-zero u never becomes zero (it
// rounds up to the smallest code): |m| is at most a few u (for b1^2 < b2), so m / u stays bounded where u is
// small beside the block's largest, while m / (0 + eps) would not.  The step itself uses the new m and v before their rounding.
// Nearest rounding takes no change below half a step, 3 to 6 % of a value: what a step changes by less only moves
// where the block's scale, which follows its largest element, moves the codes' borders.  A step moves u by
// 1 - sqrt(b2) at most downwards and m by 1 - b1.  Measured on half a block's gradients that become ten times
// smaller, the other half's as they were, both noisy: the median of u over the float32 states' one is 1.37 after
// 4 / (1 - b2) steps and 1.03 after 8 at b2 = 0.95; 2.0 and 1.5 at 0.97, 3.2 and 2.8 at 0.98, 4.9 and 7.2 at 0.99:
// it stands still.  m of elements whose gradients end beside steady ones stops at 4 of the smallest codes at
// b1 = 0.9 (0.01 lr a step at most), but anywhere at 0.95 (up to lr a step).  8-bit states are refused beyond.
// Included by resbm_matrix.hip.
#pragma once

#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>

#include "resbm.h"
#include "resbm_host.hpp"
#include "resbm_norm.hpp"

namespace resbm_aw {

using resbm_nm::e4m3_scale;
using resbm_nm::mag;
using resbm_nm::to_e4m3;
using resbm_nm::umax;
using resbm_nm::wave_max;

constexpr int kBlock = 256;            // elements per scale of an 8-bit state: 64 lanes x 4
constexpr int kThreads = 256;
constexpr int kTurn = kThreads * 4;    // elements that a block takes at once
// Turns of a chunk.  float32 states: one (a block's 218 M parameters: 1106 us, with two 1167); 8-bit states, half
// the bytes: two, with both turns' loads in flight (243 M parameters: 627 us, with one 663 and four 641);
// gradients alone: four.
constexpr int kTurns32 = 1, kTurns8 = 2, kTurnsGrad = 4;
constexpr int64_t kMaxBlocks = 1 << 20;
// Blocks, and partial sums, of the norm: 1024 with four loads a lane in flight read 6.4 to 6.6 TB/s; twice the
// blocks 5.9, or half 5.1, and so do twice or half the loads.
constexpr int kNormBlocks = 1024;
constexpr int kFewWaves = 16;
// Shared memory that a streaming step asks for and does not touch: five blocks to a compute unit instead of
// seven.  Five have enough loads in flight; with more the memory system serves them less evenly (218 M
// parameters 1056 us against 1082, 243 M in 8 bits 628 against 646; four: 1066 and 658).
constexpr int kFewerBlocks = 32000;
constexpr double kMostB1of8 = 0.9, kMostB2of8 = 0.95;  // the betas that 8-bit states follow
constexpr uint32_t kMagic = 0x57414452u;

// The plan, in host and device memory alike: Head, Entry[count], uint32 tensor[chunks].
struct Entry {
  float* p;
  const void* g;
  void *m, *v;
  float *m_scale, *v_scale;
  __bf16* copy;
  int64_t numel, first;  // first: the tensor's first chunk
  float wd;
  int32_t g16, q8, turns, unused;
};
struct Head {
  uint32_t magic;
  uint16_t grads_only, q8;  // q8: there are states in 8 bits
  int64_t count, chunks, bytes, traffic;  // traffic: bytes that a step reads and writes
  uintptr_t lo, hi;                       // the tensors lie between
};
static_assert(kThreads == 256, "block_sum adds four waves");
static_assert(sizeof(Head) == 56 && sizeof(Entry) == 96 && sizeof(resbm_adamw_tensor) == 80, "layouts");

struct Table {
  const Entry* entry;
  const uint32_t* tensor;
};

struct Hyper {
  double lr, b1, b2;
  float fb1, fb2, ob1, ob2, eps;  // bk and 1 - bk in float32
  float rate, rc2;                // lr / c1 and 1 / sqrt(c2)
  const double* lr_step;
  const float* grad_scale;
};

typedef float f2 __attribute__((ext_vector_type(2)));

__device__ __forceinline__ void from_e4m3(uint32_t q, float (&f)[4]) {
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)q, true);
  f[0] = a.x, f[1] = a.y, f[2] = b.x, f[3] = b.y;
}

// Four elements at any address that suits one: global memory takes wide accesses without their own alignment
// (50 M elements, float32 states: 241 us, from odd offsets 263 to 287, element by element 404; 8-bit states 146,
// 174 and 330).
typedef float f4 __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u1 __attribute__((aligned(1)));
typedef __bf16 b4 __attribute__((ext_vector_type(4), aligned(2)));

// Loads and stores of global memory (pointers that come from the plan would be taken for any memory),
// past the caches (NT) or not.
template <class V>
using Global = V __attribute__((address_space(1)));
template <bool NT = false, class V>
__device__ __forceinline__ auto get(const V* p) {
  const Global<const V>* q = (const Global<const V>*)p;
  if constexpr (NT) return __builtin_nontemporal_load(q);
  return *q;
}
template <bool NT = false, class U, class V>
__device__ __forceinline__ void put(U v, V* p) {
  Global<V>* q = (Global<V>*)p;
  if constexpr (NT)
    __builtin_nontemporal_store(v, q);
  else
    *q = v;
}

// Four elements from e on, of which `left` exist; those beyond are zero.
__device__ __forceinline__ void load_f32(const float* p, int64_t e, int left, float (&f)[4]) {
  if (left >= 4) {
    const f4 v = get((const f4*)(p + e));
    f[0] = v.x, f[1] = v.y, f[2] = v.z, f[3] = v.w;
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = i < left ? get(p + e + i) : 0.0f;
}
__device__ __forceinline__ void store_f32(float* p, int64_t e, int left, const float (&f)[4]) {
  if (left >= 4) {
    put(f4{f[0], f[1], f[2], f[3]}, (f4*)(p + e));
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) put(f[i], p + e + i);
}
__device__ __forceinline__ void load_grad(const Entry& t, int64_t e, int left, float (&f)[4]) {
  if (!t.g16) return load_f32((const float*)t.g, e, left, f);
  const uint16_t* g = (const uint16_t*)t.g;
  if (left >= 4) {
    const u2 v = get((const u2*)(g + e));
    f[0] = __builtin_bit_cast(float, v.x << 16), f[1] = __builtin_bit_cast(float, v.x & 0xFFFF0000u);
    f[2] = __builtin_bit_cast(float, v.y << 16), f[3] = __builtin_bit_cast(float, v.y & 0xFFFF0000u);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = i < left ? __builtin_bit_cast(float, (uint32_t)get(g + e + i) << 16) : 0.0f;
}
__device__ __forceinline__ uint32_t load_codes(const void* p, int64_t e, int left) {
  const uint8_t* q = (const uint8_t*)p + e;
  if (left >= 4) return get((const u1*)q);
  uint32_t v = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) v |= (uint32_t)get(q + i) << (8 * i);
  return v;
}
__device__ __forceinline__ void store_codes(void* p, int64_t e, int left, uint32_t v) {
  uint8_t* q = (uint8_t*)p + e;
  if (left >= 4) {
    put(v, (u1*)q);
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) put((uint8_t)(v >> (8 * i)), q + i);
}
__device__ __forceinline__ void store_copy(__bf16* p, int64_t e, int left, const float (&f)[4]) {
  const b4 v = {(__bf16)f[0], (__bf16)f[1], (__bf16)f[2], (__bf16)f[3]};
  if (left >= 4) {
    put(v, (b4*)(p + e));
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < left) put(v[i], p + e + i);
}

// b^n by squaring, in float64: the bias correction of a step that only the device knows.
__device__ __forceinline__ double power(double b, uint64_t n) {
  double r = 1.0;
  for (; n; n >>= 1) {
    if (n & 1) r *= b;
    b *= b;
  }
  return r;
}

// The step's constants, and the arithmetic of one element.
struct Step {
  float fb1, fb2, ob1, ob2, eps, rate, rc2, keep, gs;
  bool scaled;
};
__device__ __forceinline__ void step_element(const Step& s, float& p, float g, float& m, float& v, float& u) {
#pragma clang fp contract(off)
  if (s.scaled) g = g * s.gs;
  m = m * s.fb1 + g * s.ob1;
  v = v * s.fb2 + g * s.ob2 * g;
  u = sqrtf(v);
  p = p * s.keep - m / (u * s.rc2 + s.eps) * s.rate;
}
// m and v = u^2 from their codes.
__device__ __forceinline__ void decode4(uint32_t cm, uint32_t cu, float ms, float us, float (&m)[4], float (&v)[4]) {
#pragma clang fp contract(off)
  from_e4m3(cm, m);
  from_e4m3(cu, v);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = m[i] * ms;
    v[i] = v[i] * us;
    v[i] = v[i] * v[i];
  }
}
// Codes and scales of a wave's 256 elements.
__device__ __forceinline__ void encode4(const float (&m)[4], const float (&u)[4], uint32_t& cm, uint32_t& cu, float& ms,
                                        float& us) {
  uint32_t am = 0, au = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    am = umax(am, mag(m[i]));
    au = umax(au, mag(u[i]));
  }
  ms = e4m3_scale(wave_max(am)), us = e4m3_scale(wave_max(au));
  const float im = 1.0f / ms, iu = 1.0f / us;
  float q[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    q[i] = u[i] * iu;
    q[i] = u[i] > 0.0f && q[i] < 0x1p-9f ? 0x1p-9f : q[i];
  }
  cm = to_e4m3(m[0] * im, m[1] * im, m[2] * im, m[3] * im);
  cu = to_e4m3(q[0], q[1], q[2], q[3]);
}

// A whole chunk: every load of the chunk is issued before the first use.
template <bool Q8, bool G16, bool NT>
__device__ __forceinline__ void whole_chunk(const Entry& t, int64_t at, const Step& s) {
  const int lane = threadIdx.x & 63;
  constexpr int N = Q8 ? kTurns8 : kTurns32;
  f4 P[N], G[N], M[N], V[N];
  u2 H[N];
  uint32_t cm[N], cu[N];
  float ms[N], us[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t e = at + k * kTurn + threadIdx.x * 4;
    P[k] = get<NT>((const f4*)(t.p + e));
    if constexpr (G16)
      H[k] = get<NT>((const u2*)((const uint16_t*)t.g + e));
    else
      G[k] = get<NT>((const f4*)((const float*)t.g + e));
    if constexpr (Q8) {
      cm[k] = get<NT>((const u1*)((const uint8_t*)t.m + e));
      cu[k] = get<NT>((const u1*)((const uint8_t*)t.v + e));
      ms[k] = get(t.m_scale + e / kBlock);
      us[k] = get(t.v_scale + e / kBlock);
    } else {
      M[k] = get<NT>((const f4*)((const float*)t.m + e));
      V[k] = get<NT>((const f4*)((const float*)t.v + e));
    }
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t e = at + k * kTurn + threadIdx.x * 4;
    float m[4], v[4], u[4];
    if constexpr (Q8) {
      decode4(cm[k], cu[k], ms[k], us[k], m, v);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) m[i] = M[k][i], v[i] = V[k][i];
    }
    if constexpr (G16)
      G[k] = f4{__builtin_bit_cast(float, H[k][0] << 16), __builtin_bit_cast(float, H[k][0] & 0xFFFF0000u),
                __builtin_bit_cast(float, H[k][1] << 16), __builtin_bit_cast(float, H[k][1] & 0xFFFF0000u)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float p = P[k][i];
      step_element(s, p, G[k][i], m[i], v[i], u[i]);
      P[k][i] = p;
    }
    put<NT>(P[k], (f4*)(t.p + e));
    if (t.copy) put<NT>((b4{(__bf16)P[k][0], (__bf16)P[k][1], (__bf16)P[k][2], (__bf16)P[k][3]}), (b4*)(t.copy + e));
    if constexpr (Q8) {
      uint32_t qm, qu;
      float sm, su;
      encode4(m, u, qm, qu, sm, su);
      put<NT>(qm, (u1*)((uint8_t*)t.m + e));
      put<NT>(qu, (u1*)((uint8_t*)t.v + e));
      if (lane == 0) {
        put(sm, t.m_scale + e / kBlock);
        put(su, t.v_scale + e / kBlock);
      }
    } else {
      put<NT>((f4{m[0], m[1], m[2], m[3]}), (f4*)((float*)t.m + e));
      put<NT>((f4{v[0], v[1], v[2], v[3]}), (f4*)((float*)t.v + e));
    }
  }
}

// A tensor's last chunk, which ends inside: element by element there.
__device__ __forceinline__ void part_chunk(const Entry& t, int64_t at, const Step& s) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int k = 0; k < t.turns; ++k) {
    const int64_t w0 = at + k * kTurn + wave * kBlock;  // the wave's 256 elements
    if (w0 >= t.numel) break;
    const int64_t e = w0 + lane * 4, rest = t.numel - e;
    const int left = rest < 0 ? 0 : rest > 4 ? 4 : (int)rest;
    float p[4], g[4], m[4], v[4], u[4];
    load_f32(t.p, e, left, p);
    load_grad(t, e, left, g);
    if (t.q8) {
      decode4(load_codes(t.m, e, left), load_codes(t.v, e, left), get(t.m_scale + w0 / kBlock),
              get(t.v_scale + w0 / kBlock), m, v);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (i >= left) m[i] = v[i] = 0.0f;  // beside a scale that is not finite, no element is 0 times that
    } else {
      load_f32((const float*)t.m, e, left, m);
      load_f32((const float*)t.v, e, left, v);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) step_element(s, p[i], g[i], m[i], v[i], u[i]);
    store_f32(t.p, e, left, p);
    if (t.copy) store_copy(t.copy, e, left, p);
    if (t.q8) {
      uint32_t qm, qu;
      float sm, su;
      encode4(m, u, qm, qu, sm, su);
      store_codes(t.m, e, left, qm);
      store_codes(t.v, e, left, qu);
      if (lane == 0) {
        put(sm, t.m_scale + w0 / kBlock);
        put(su, t.v_scale + w0 / kBlock);
      }
    } else {
      store_f32((float*)t.m, e, left, m);
      store_f32((float*)t.v, e, left, v);
    }
  }
}

template <bool NT>
__global__ __launch_bounds__(kThreads) void k_adamw(const Entry* __restrict__ entry, const uint32_t* __restrict__ tensor,
                                                    int64_t chunks, Hyper hy) {
  Step s = {hy.fb1, hy.fb2, hy.ob1, hy.ob2, hy.eps, hy.rate, hy.rc2, 1.0f, 1.0f, hy.grad_scale != nullptr};
  if (hy.grad_scale) {
    s.gs = *hy.grad_scale;
    if (s.gs != s.gs) return;  // no norm, no step: everything stays as it is
  }
  double lr = hy.lr;
  if (hy.lr_step) {
    lr = hy.lr_step[0];
    const double step = hy.lr_step[1];
    const uint64_t n = step >= 1.0 ? (step < 1e18 ? (uint64_t)step : (uint64_t)1e18) : 1;
    s.rate = (float)(lr / (1.0 - power(hy.b1, n)));
    s.rc2 = (float)(1.0 / sqrt(1.0 - power(hy.b2, n)));
  }
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Entry t = entry[tensor[c]];
    const int64_t at = (c - t.first) * t.turns * kTurn;
    s.keep = (float)(1.0 - lr * (double)t.wd);
    if (at + t.turns * kTurn > t.numel)
      part_chunk(t, at, s);
    else if (t.q8)
      t.g16 ? whole_chunk<true, true, NT>(t, at, s) : whole_chunk<true, false, NT>(t, at, s);
    else
      t.g16 ? whole_chunk<false, true, NT>(t, at, s) : whole_chunk<false, false, NT>(t, at, s);
  }
}

// ---------------------------------------------------------------- gradient norm
// Sums are float64 from the first square on: any float32 gradient's square fits.
template <int CTRL>
__device__ __forceinline__ double add_step(double v) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = resbm_nm::dpp<CTRL>((uint32_t)u), hi = resbm_nm::dpp<CTRL>((uint32_t)(u >> 32));
  return v + __builtin_bit_cast(double, lo | hi << 32);
}
__device__ __forceinline__ double of_lane(double v, int lane) {
  const uint64_t u = __builtin_bit_cast(uint64_t, v);
  const uint64_t lo = (uint32_t)__builtin_amdgcn_readlane((int)u, lane);
  const uint64_t hi = (uint32_t)__builtin_amdgcn_readlane((int)(u >> 32), lane);
  return __builtin_bit_cast(double, lo | hi << 32);
}
__device__ __forceinline__ double wave_sum(double v) {
  v = add_step<resbm_nm::kXor2>(add_step<resbm_nm::kXor1>(v));
  v = add_step<resbm_nm::kMirror>(add_step<resbm_nm::kHalfMirror>(v));
  return (of_lane(v, 0) + of_lane(v, 16)) + (of_lane(v, 32) + of_lane(v, 48));
}
__device__ __forceinline__ double block_sum(double v, double* lds) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  return (lds[0] + lds[1]) + (lds[2] + lds[3]);  // kThreads / 64 waves
}

__device__ __forceinline__ void norm_out(double sum, double max_norm, float* out) {
  const double norm = sqrt(sum), f = max_norm / (norm + 1e-6);
  out[0] = (float)norm;
  out[1] = norm <= 1.7976931348623157e308 ? (float)(f < 1.0 ? f : 1.0) : __builtin_nanf("");
}

template <bool G16, int N>
__device__ __forceinline__ double whole_squares(const Entry& t, int64_t at, double s) {
  f4 g[N];
  u2 h[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    const int64_t e = at + k * kTurn + threadIdx.x * 4;
    if constexpr (G16)
      h[k] = get((const u2*)((const uint16_t*)t.g + e));
    else
      g[k] = get((const f4*)((const float*)t.g + e));
  }
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if constexpr (G16)
      g[k] = f4{__builtin_bit_cast(float, h[k][0] << 16), __builtin_bit_cast(float, h[k][0] & 0xFFFF0000u),
                __builtin_bit_cast(float, h[k][1] << 16), __builtin_bit_cast(float, h[k][1] & 0xFFFF0000u)};
#pragma unroll
    for (int i = 0; i < 4; ++i) s = fma((double)g[k][i], (double)g[k][i], s);
  }
  return s;
}

__global__ __launch_bounds__(kThreads) void k_grad_norm(const Entry* __restrict__ entry, const uint32_t* __restrict__ tensor,
                                                        int64_t chunks, double* __restrict__ part) {
  __shared__ double s_red[kThreads / 64];
  double s = 0.0;
  for (int64_t c = blockIdx.x; c < chunks; c += gridDim.x) {
    const Entry t = entry[tensor[c]];
    const int64_t at = (c - t.first) * t.turns * kTurn;
    if (t.turns == kTurnsGrad && at + kTurnsGrad * kTurn <= t.numel) {
      s = t.g16 ? whole_squares<true, kTurnsGrad>(t, at, s) : whole_squares<false, kTurnsGrad>(t, at, s);
      continue;
    }
    for (int k = 0; k < t.turns; ++k) {
      const int64_t e = at + k * kTurn + threadIdx.x * 4, rest = t.numel - e;
      const int left = rest < 0 ? 0 : rest > 4 ? 4 : (int)rest;
      float g[4];
      load_grad(t, e, left, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) s = fma((double)g[i], (double)g[i], s);
    }
  }
  s = block_sum(s, s_red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

// The partial sums of up to kNormBlocks blocks, all loads in flight at once.
__global__ __launch_bounds__(kThreads) void k_grad_norm_out(int parts, const double* __restrict__ part, double max_norm,
                                                            float* __restrict__ out) {
  __shared__ double s_red[kThreads / 64];
  double v[kNormBlocks / kThreads], s = 0.0;
#pragma unroll
  for (int k = 0; k < kNormBlocks / kThreads; ++k) {
    const int i = k * kThreads + threadIdx.x;
    v[k] = i < parts ? part[i] : 0.0;
  }
#pragma unroll
  for (int k = 0; k < kNormBlocks / kThreads; ++k) s += v[k];
  s = block_sum(s, s_red);
  if (threadIdx.x == 0) norm_out(s, max_norm, out);
}

// Up to a chunk for each of its waves in one launch (16 chunks of 4096 gradients: 4.9 us against 6.1 in two
// launches, 32: 7.3 against 5.9).
__global__ __launch_bounds__(64 * kFewWaves) void k_grad_norm_few(const Entry* __restrict__ entry,
                                                                  const uint32_t* __restrict__ tensor, int chunks,
                                                                  double max_norm, float* __restrict__ out) {
  __shared__ double s_red[kFewWaves];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  double s = 0.0;
  if (const int c = wave; c < chunks) {
    const Entry t = entry[tensor[c]];
    const int64_t at = (c - t.first) * t.turns * kTurn, end = at + t.turns * kTurn;
    const int64_t last = end < t.numel ? end : t.numel;
#pragma unroll 4
    for (int64_t w = at; w < last; w += 256) {
      const int64_t e = w + lane * 4, rest = last - e;
      float g[4];
      load_grad(t, e, rest < 0 ? 0 : rest > 4 ? 4 : (int)rest, g);
#pragma unroll
      for (int i = 0; i < 4; ++i) s = fma((double)g[i], (double)g[i], s);
    }
  }
  s = wave_sum(s);
  if (lane == 0) s_red[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = s_red[0];
#pragma unroll
    for (int i = 1; i < kFewWaves; ++i) s += s_red[i];
    norm_out(s, max_norm, out);
  }
}

// ---------------------------------------------------------------- host
using resbm_host::aligned;
using resbm_host::launch_status;
using resbm_host::overlap;

inline int turns_of(const resbm_adamw_tensor& a) {
  return !a.p ? kTurnsGrad : a.state == RESBM_STATE_E4M3 ? kTurns8 : kTurns32;
}
inline int64_t chunks_of(const resbm_adamw_tensor& a) {
  const int64_t k = (int64_t)turns_of(a) * kTurn;
  return (a.numel + k - 1) / k;
}
inline size_t plan_size(int64_t count, int64_t chunks) {
  return (sizeof(Head) + (size_t)count * sizeof(Entry) + (size_t)chunks * 4 + 255) & ~(size_t)255;
}

struct Range {
  uintptr_t at, end;
  int writes;
};

// The checks of a list; *chunks and *grads_only as the plan's head has them.
inline int32_t check_list(const resbm_adamw_tensor* t, int64_t count, int64_t* chunks, bool* grads_only) {
  if (count < 0 || count > (1 << 24)) return RESBM_E_SHAPE;
  if (count > 0 && !t) return RESBM_E_NULL;
  *chunks = 0;
  int64_t bare = 0, work = 0;
  for (int64_t i = 0; i < count; ++i) {
    const resbm_adamw_tensor& a = t[i];
    if (a.numel < 0 || a.numel > (int64_t)1 << 42) return RESBM_E_SHAPE;
    if (a.g_type != RESBM_TYPE_F32 && a.g_type != RESBM_TYPE_BF16) return RESBM_E_KIND;
    if (a.state != RESBM_STATE_F32 && a.state != RESBM_STATE_E4M3) return RESBM_E_KIND;
    if (!(a.weight_decay >= 0.0f && a.weight_decay < 3.0e38f)) return RESBM_E_SHAPE;
    const bool none = !a.p && !a.m && !a.v && !a.m_scale && !a.v_scale && !a.copy;
    if (a.numel == 0) continue;
    bare += none;
    work += 1;
    if (!a.g) return RESBM_E_NULL;
    const bool q8 = a.state == RESBM_STATE_E4M3;
    if (!none && (!a.p || !a.m || !a.v || (q8 && (!a.m_scale || !a.v_scale)))) return RESBM_E_NULL;
    const size_t sg = a.g_type == RESBM_TYPE_BF16 ? 2 : 4, ss = q8 ? 1 : 4;
    if (!aligned(a.p, 4) || !aligned(a.g, sg) || !aligned(a.m, ss) || !aligned(a.v, ss) || !aligned(a.copy, 2) ||
        (q8 && (!aligned(a.m_scale, 4) || !aligned(a.v_scale, 4))))
      return RESBM_E_ALIGN;
    *chunks += chunks_of(a);
  }
  if (*chunks > INT32_MAX) return RESBM_E_SHAPE;
  if (bare != 0 && bare != work) return RESBM_E_NULL;  // all with parameters and states, or none
  *grads_only = bare > 0;
  return RESBM_OK;
}

// Nothing that a step writes may overlap anything else in the list: all ranges by address, and
// the furthest end so far of those that are written, and of all, against the next one's start.
// *lo and *hi: the first address and the end of all.
inline int32_t check_overlap(const resbm_adamw_tensor* t, int64_t count, uintptr_t* lo, uintptr_t* hi) {
  Range* r = (Range*)malloc((size_t)count * 7 * sizeof(Range) + 1);
  if (!r) return RESBM_E_WORKSPACE;
  size_t k = 0;
  for (int64_t i = 0; i < count; ++i) {
    const resbm_adamw_tensor& a = t[i];
    const bool q8 = a.state == RESBM_STATE_E4M3;
    const size_t n = (size_t)a.numel, nb = (n + kBlock - 1) / kBlock * 4;
    const auto put = [&](const void* p, size_t bytes, int writes) {
      if (p && bytes) r[k++] = {(uintptr_t)p, (uintptr_t)p + bytes, writes};
    };
    put(a.p, n * 4, 1);
    put(a.g, n * (a.g_type == RESBM_TYPE_BF16 ? 2 : 4), 0);
    put(a.m, n * (q8 ? 1 : 4), 1);
    put(a.v, n * (q8 ? 1 : 4), 1);
    put(q8 ? a.m_scale : nullptr, nb, 1);
    put(q8 ? a.v_scale : nullptr, nb, 1);
    put(a.copy, n * 2, 1);
  }
  std::sort(r, r + k, [](const Range& a, const Range& b) { return a.at < b.at; });
  uintptr_t written = 0, any = 0;
  bool clash = false;
  for (size_t i = 0; i < k && !clash; ++i) {
    clash = r[i].at < (r[i].writes ? any : written);
    any = r[i].end > any ? r[i].end : any;
    if (r[i].writes) written = r[i].end > written ? r[i].end : written;
  }
  *lo = k ? r[0].at : 0, *hi = any;
  free(r);
  return clash ? RESBM_E_ALIAS : RESBM_OK;
}

// The head of the host's copy, if it is a plan.
inline const Head* head_of(const void* plan) {
  const Head* h = (const Head*)plan;
  return h && aligned(plan, 8) && h->magic == kMagic ? h : nullptr;
}
inline Table table_of(const Head* h, const void* dev) {
  const char* d = (const char*)dev;
  return {(const Entry*)(d + sizeof(Head)), (const uint32_t*)(d + sizeof(Head) + h->count * sizeof(Entry))};
}
// Whether an operand of a call meets what the call writes (a step: p, the states, the copies) or reads (a norm:
// the gradients) of the plan's tensors.  Most operands lie outside the span of all of them; for the others the
// entries are looked through (a norm's two operands among 400 tensors: 0.9 us of host time).
template <bool STEP>
inline bool meets(const Head* h, const void* p, size_t bytes) {
  if (!p || (uintptr_t)p >= h->hi || (uintptr_t)p + bytes <= h->lo) return false;
  const Entry* e = (const Entry*)(h + 1);
  for (const Entry* end = e + h->count; e < end; ++e) {
    const size_t n = (size_t)e->numel, ns = n * (e->q8 ? 1 : 4), nb = e->q8 ? (n + kBlock - 1) / kBlock * 4 : 0;
    if (!STEP) {
      if (overlap(p, bytes, e->g, n * (e->g16 ? 2 : 4))) return true;
    } else if (overlap(p, bytes, e->p, n * 4) || overlap(p, bytes, e->m, ns) || overlap(p, bytes, e->v, ns) ||
               overlap(p, bytes, e->copy, n * 2) || overlap(p, bytes, e->m_scale, nb) || overlap(p, bytes, e->v_scale, nb)) {
      return true;
    }
  }
  return false;
}
inline int norm_blocks(int64_t chunks) { return (int)(chunks < kNormBlocks ? chunks : kNormBlocks); }

}  // namespace resbm_aw

extern "C" {

size_t resbm_adamw_plan_bytes(const resbm_adamw_tensor* tensors, int64_t count) {
  int64_t chunks;
  bool grads_only;
  if (resbm_aw::check_list(tensors, count, &chunks, &grads_only) != RESBM_OK) return 0;
  return resbm_aw::plan_size(count, chunks);
}

int32_t resbm_adamw_plan(const resbm_adamw_tensor* tensors, int64_t count, void* plan, size_t plan_bytes) {
  using namespace resbm_aw;
  int64_t chunks;
  bool grads_only;
  int32_t st = check_list(tensors, count, &chunks, &grads_only);
  if (st != RESBM_OK) return st;
  if (!plan) return RESBM_E_NULL;
  if (!aligned(plan, 8)) return RESBM_E_ALIGN;
  const size_t bytes = plan_size(count, chunks);
  if (plan_bytes < bytes) return RESBM_E_WORKSPACE;
  uintptr_t lo, hi;
  st = check_overlap(tensors, count, &lo, &hi);
  if (st != RESBM_OK) return st;
  memset(plan, 0, bytes);
  Head* h = (Head*)plan;
  Entry* e = (Entry*)((char*)plan + sizeof(Head));
  uint32_t* at = (uint32_t*)(e + count);
  int64_t c = 0, traffic = 0;
  bool any8 = false;
  for (int64_t i = 0; i < count; ++i) {
    const resbm_adamw_tensor& a = tensors[i];
    const bool q8 = a.state == RESBM_STATE_E4M3, g16 = a.g_type == RESBM_TYPE_BF16;
    e[i] = {a.p, a.g, a.m, a.v, a.m_scale, a.v_scale, (__bf16*)a.copy, a.numel, c, a.weight_decay, g16, q8,
            turns_of(a), 0};
    any8 |= q8 && a.p && a.numel > 0;
    traffic += a.numel * ((g16 ? 2 : 4) + (!a.p ? 0 : 8 + (q8 ? 4 : 16) + (a.copy ? 2 : 0)));
    for (int64_t k = chunks_of(a); k > 0; --k) at[c++] = (uint32_t)i;
  }
  h->grads_only = grads_only;
  h->q8 = any8;
  h->count = count;
  h->chunks = chunks;
  h->bytes = (int64_t)bytes;
  h->traffic = traffic;
  h->lo = lo, h->hi = hi;
  h->magic = kMagic;
  return RESBM_OK;
}

int32_t resbm_adamw_update(const void* plan, const void* plan_dev, double lr, double beta1, double beta2, double eps,
                           int64_t step, const double* lr_step, const float* grad_scale, void* stream) {
  using namespace resbm_aw;
  if (!plan) return RESBM_E_NULL;
  const Head* h = head_of(plan);
  if (!h) return RESBM_E_KIND;
  if (!(beta1 >= 0.0 && beta1 < 1.0) || !(beta2 >= 0.0 && beta2 < 1.0) || !(eps >= 0.0 && eps < 3.0e38)) return RESBM_E_SHAPE;
  if (h->q8 && (beta1 > kMostB1of8 || beta2 > kMostB2of8)) return RESBM_E_SHAPE;
  if (!lr_step && (step < 1 || !isfinite(lr))) return RESBM_E_SHAPE;
  if (h->chunks == 0) return RESBM_OK;
  if (!plan_dev || h->grads_only) return RESBM_E_NULL;
  if (!aligned(plan_dev, 256) || !aligned(lr_step, 8) || !aligned(grad_scale, 4)) return RESBM_E_ALIGN;
  // every block reads these, some after others have written their tensors
  if (meets<true>(h, grad_scale, 4) || meets<true>(h, lr_step, 16) || meets<true>(h, plan_dev, h->bytes)) return RESBM_E_ALIAS;
  const double n = (double)(lr_step ? 1 : step);
  const Hyper hy = {lr, beta1, beta2, (float)beta1, (float)beta2, (float)(1.0 - beta1), (float)(1.0 - beta2), (float)eps,
                    (float)(lr / (1.0 - pow(beta1, n))), (float)(1.0 / sqrt(1.0 - pow(beta2, n))), lr_step, grad_scale};
  const int64_t blocks = h->chunks < kMaxBlocks ? h->chunks : kMaxBlocks;
  const Table tab = table_of(h, plan_dev);
  if (resbm_nm::streams_through((size_t)h->traffic))
    hipLaunchKernelGGL(k_adamw<true>, dim3((uint32_t)blocks), dim3(kThreads), kFewerBlocks, (hipStream_t)stream, tab.entry, tab.tensor,
                       h->chunks, hy);
  else
    hipLaunchKernelGGL(k_adamw<false>, dim3((uint32_t)blocks), dim3(kThreads), 0, (hipStream_t)stream, tab.entry,
                       tab.tensor, h->chunks, hy);
  return launch_status();
}

size_t resbm_grad_norm_workspace_bytes(const void* plan) {
  using namespace resbm_aw;
  const Head* h = head_of(plan);
  return h ? ((size_t)norm_blocks(h->chunks) * 8 + 256) & ~(size_t)255 : 0;
}

int32_t resbm_grad_norm(const void* plan, const void* plan_dev, double max_norm, float* out, void* ws, size_t ws_bytes,
                        void* stream) {
  using namespace resbm_aw;
  if (!plan) return RESBM_E_NULL;
  const Head* h = head_of(plan);
  if (!h) return RESBM_E_KIND;
  if (!(max_norm > 0.0)) return RESBM_E_SHAPE;
  if (!out || !ws || (!plan_dev && h->chunks > 0)) return RESBM_E_NULL;
  if (!aligned(plan_dev, 256) || !aligned(out, 4) || !aligned(ws, 256)) return RESBM_E_ALIGN;
  const size_t need = resbm_grad_norm_workspace_bytes(plan);
  if (ws_bytes < need) return RESBM_E_WORKSPACE;
  if (overlap(out, 8, ws, need) || overlap(out, 8, plan_dev, h->bytes) || overlap(ws, need, plan_dev, h->bytes) ||
      meets<false>(h, out, 8) || meets<false>(h, ws, need))
    return RESBM_E_ALIAS;
  const Table tab = table_of(h, plan_dev);
  if (h->chunks <= kFewWaves) {
    hipLaunchKernelGGL(k_grad_norm_few, dim3(1), dim3(64 * kFewWaves), 0, (hipStream_t)stream, tab.entry, tab.tensor,
                       (int)h->chunks, max_norm, out);
    return launch_status();
  }
  const int parts = norm_blocks(h->chunks);
  hipLaunchKernelGGL(k_grad_norm, dim3(parts), dim3(kThreads), 0, (hipStream_t)stream, tab.entry, tab.tensor, h->chunks,
                     (double*)ws);
  hipLaunchKernelGGL(k_grad_norm_out, dim3(1), dim3(kThreads), 0, (hipStream_t)stream, parts, (const double*)ws, max_norm,
                     out);
  return launch_status();
}

}  // extern "C"
