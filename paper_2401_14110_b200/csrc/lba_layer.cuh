// What a layer does with the finished contraction, in the kernel that forms it: scales and bias, activation, dropout, the
// product of a gated pair, residual, rounding to the output's type.
//
//   linear   z = fl(fl(y sa) sb) + bias          out = round(drop(act(z)) + residual)
//   gated    z, v: the two projections of a row  out = round(act(z) v)
//
// The two projections of a gated layer are contracted as one matrix of 2 N columns, column 2 j the gate's row j and column 2 j + 1
// the up projection's.  Every kernel's thread owns an even number of neighbouring columns from an even one on, so both halves of a
// pair meet in its registers whatever the tile, and a row of A is fetched and decoded once for both.
//
// All arithmetic is binary32, one rounding per operation; only the stores round to the output's type.  The epilogue of an element
// costs some tens of instructions where its chain costs 2 K, and saves the pass over z that a separate kernel would need.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lba_kernel.cuh"

namespace lba {

enum LayerType { LT_F32 = 0, LT_BF16 = 1, LT_F16 = 2, LT_CODES = 3, LT_COUNT = 4 };
enum LayerAct { ACT_NONE = 0, ACT_RELU = 1, ACT_GELU = 2, ACT_GELU_TANH = 3, ACT_SILU = 4, ACT_COUNT = 5 };

struct LinearProblem : Problem {
  int64_t n;                 // columns of the output: N, or N / 2 of a gated layer
  const uint8_t* B2;         // gated: the up projection (B, sb and bias are the gate's)
  const float *sb2, *bias2;
  const void* residual;
  void *dst, *pre;           // output; pre-activations, or null (gated: the gate's, then the up projection's)
  const float* out_scale;    // codes: what one unit of the code domain stands for
  const uint64_t* rng;       // seed, offset
  uint32_t drop_below;       // a word of the generator below this drops its element (0: no dropout)
  float keep_scale;          // 1 / (1 - p)
  int gated, act, residual_type, dst_type, pre_type;
};

// ------------------------------------------------------------------ B's rows as the loaders see them (plain problems: lba_kernel.cuh)
__device__ __forceinline__ const uint8_t* b_base(const LinearProblem& p, const uint8_t* b, int64_t n) { return p.gated && (n & 1) ? p.B2 : b; }
__device__ __forceinline__ int64_t b_row(const LinearProblem& p, int64_t n) { return p.gated ? n >> 1 : n; }
__device__ __forceinline__ int64_t b_rows(const LinearProblem& p) { return p.n; }

// ------------------------------------------------------------------ activations
// Both functions in binary32 from one exponential and one reciprocal each (hardware approximations, a few units in the last place),
// for two elements at a time:
//   gelu       z P(z), P the normal distribution: P(-x) = (c0 + c1 t + ... + c7 t^7) e^(-x^2/2), t = 1 / (1 + x/4), for 0 <= x <= 14.5, where
//              the exponential leaves binary32.  The sum stands for erfcx(x / sqrt 2) / 2, least maximum of the relative error over 1 + x^2 by
//              repeated least squares in 64 bits: off by 2.6e-8 (1 + x^2) of it.  P(z) is that below 0 and 1 minus it above, so the tail keeps
//              what was computed: a relative error of 5 (1 + x^2 / 20) 2^-21 at most (1/2 - (1/2 - P) had left 3e-8 steps of it, 5 % at z = -5,
//              nothing at -6; a form within 7.5e-8 of 1 is off by 0.4 % of P there).  The slope P + z P' has the same exponential in P'
//   gelu_tanh  1/2 (1 + tanh u) is the logistic function of 2 u
// The backward pass is bound by the instructions of its elementwise kernel where the activation takes some fifty an element, as it does
// from erff, expf and tanhf.
__device__ __forceinline__ float exp2_approx(float x) {
  float d;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
  return d;
}
__device__ __forceinline__ float rcp_approx(float x) {
  float d;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(x));
  return d;
}
__device__ __forceinline__ u64 exp2_approx(u64 x) {
  float lo, hi;
  unpack2(x, lo, hi);
  return pack2(exp2_approx(lo), exp2_approx(hi));
}
__device__ __forceinline__ u64 rcp_approx(u64 x) {
  float lo, hi;
  unpack2(x, lo, hi);
  return pack2(rcp_approx(lo), rcp_approx(hi));
}
__device__ __forceinline__ u64 both(float v) { return pack2(v, v); }
__device__ __forceinline__ u64 add2_rn(u64 a, u64 b) {
  u64 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
// 1 / (1 + 2^-x)
__device__ __forceinline__ u64 logistic2(u64 x) { return rcp_approx(add2_rn(exp2_approx(mul2_rn(x, both(-1.0f))), both(1.0f))); }

constexpr float LOG2E = 1.44269504088896f;
// values and slopes of a pair; either may be left unused
template <int ACT>
__device__ __forceinline__ void act_pair(u64 z, u64& value, u64& slope) {
  const u64 one = both(1.0f);
  float lo, hi;
  unpack2(z, lo, hi);
  if (ACT == ACT_RELU) {
    value = pack2(lo <= 0.0f ? 0.0f : lo, hi <= 0.0f ? 0.0f : hi);  // (a NaN passes)
    slope = pack2(lo > 0.0f ? 1.0f : 0.0f, hi > 0.0f ? 1.0f : 0.0f);
  } else if (ACT == ACT_GELU) {
    const u64 e = exp2_approx(mul2_rn(mul2_rn(z, z), both(-0.5f * LOG2E)));
    const u64 t = rcp_approx(fma2_rn(pack2(fabsf(lo), fabsf(hi)), both(0.25f), one));
    u64 q = fma2_rn(t, both(-0.0973319524f), both(0.369242488f));
    q = fma2_rn(t, q, both(-0.322637386f));
    q = fma2_rn(t, q, both(0.341565140f));
    q = fma2_rn(t, q, both(-0.0131597350f));
    q = fma2_rn(t, q, both(0.125920349f));
    q = fma2_rn(t, q, both(0.0962000110f));
    q = mul2_rn(fma2_rn(t, q, both(0.000201073912f)), e);     // P(-|z|)
    float below_lo, below_hi, above_lo, above_hi;
    unpack2(q, below_lo, below_hi);
    unpack2(fma2_rn(q, both(-1.0f), one), above_lo, above_hi);
    const u64 P = pack2(lo < 0.0f ? below_lo : above_lo, hi < 0.0f ? below_hi : above_hi);
    value = mul2_rn(z, P);
    slope = fma2_rn(z, mul2_rn(e, both(0.39894228040143268f)), P);
  } else if (ACT == ACT_GELU_TANH) {
    constexpr float C = 1.59576912160573f;                    // 2 sqrt(2 / pi)
    unpack2(mul2_rn(z, z), lo, hi);
    const u64 w = pack2(fminf(lo, 1e8f), fminf(hi, 1e8f));    // (far out, where the slope is 0 or 1 long since, z^2 may be infinite)
    const u64 s = logistic2(mul2_rn(z, fma2_rn(w, both(0.044715f * C * LOG2E), both(C * LOG2E))));
    const u64 curve = mul2_rn(s, fma2_rn(s, both(-1.0f), one));
    value = mul2_rn(z, s);
    slope = fma2_rn(mul2_rn(z, curve), fma2_rn(w, both(0.134145f * C), both(C)), s);
  } else if (ACT == ACT_SILU) {
    const u64 s = logistic2(mul2_rn(z, both(LOG2E)));
    value = mul2_rn(z, s);
    slope = mul2_rn(s, fma2_rn(z, fma2_rn(s, both(-1.0f), one), one));
  } else {
    value = z;
    slope = one;
  }
}
// f with the activation as a constant
template <typename F>
__device__ __forceinline__ void with_act(int act, F f) {
  switch (act) {
    case ACT_RELU: return f(std::integral_constant<int, ACT_RELU>());
    case ACT_GELU: return f(std::integral_constant<int, ACT_GELU>());
    case ACT_GELU_TANH: return f(std::integral_constant<int, ACT_GELU_TANH>());
    case ACT_SILU: return f(std::integral_constant<int, ACT_SILU>());
    default: return f(std::integral_constant<int, ACT_NONE>());
  }
}
// the values of W (2 or 4) elements, or of one
template <int W>
__device__ __forceinline__ void act_values(int act, float (&z)[W]) {
  with_act(act, [&](auto act_tag) {
#pragma unroll
    for (int j = 0; j < W; j += 2) {
      u64 value, slope;
      act_pair<decltype(act_tag)::value>(pack2(z[j], z[j + 1 < W ? j + 1 : j]), value, slope);
      float lo, hi;
      unpack2(value, lo, hi);
      z[j] = lo;
      if (j + 1 < W) z[j + 1] = hi;
    }
  });
}

// ------------------------------------------------------------------ dropout
// Philox4x32-10 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", SC 2011): ten rounds on the counter
// (j, m, offset low, offset high) under the key `seed` give the words of row m, columns 4 j to 4 j + 3.  A word belongs to an
// element, not to a thread, so every kernel and the backward pass draw the same mask and none is stored.
__device__ __forceinline__ uint4 philox(uint32_t c0, uint32_t c1, uint64_t offset, uint64_t seed) {
  uint32_t c2 = (uint32_t)offset, c3 = (uint32_t)(offset >> 32), k0 = (uint32_t)seed, k1 = (uint32_t)(seed >> 32);
#pragma unroll
  for (int r = 0; r < 10; ++r) {
    const uint64_t x = (uint64_t)0xD2511F53u * c0, y = (uint64_t)0xCD9E8D57u * c2;
    c0 = (uint32_t)(y >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)y;
    c2 = (uint32_t)(x >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)x;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return make_uint4(c0, c1, c2, c3);
}

// ------------------------------------------------------------------ loads and stores of W neighbouring elements
template <int W> struct Bytes;
template <> struct Bytes<1> { typedef uint8_t type; };
template <> struct Bytes<2> { typedef uint16_t type; };
template <> struct Bytes<4> { typedef uint32_t type; };
template <> struct Bytes<8> { typedef uint2 type; };
template <> struct Bytes<16> { typedef uint4 type; };

template <typename T> __device__ __forceinline__ float to_f32(T v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

// `valid` of the W elements at index i exist; all W go in one access where the address allows it
template <typename T, int W>
__device__ __forceinline__ void load_some(const void* base, int64_t i, int valid, float (&v)[W]) {
  const T* const src = static_cast<const T*>(base) + i;
  constexpr int SIZE = (int)sizeof(T) * W;
  if (valid == W && (reinterpret_cast<uintptr_t>(src) & (SIZE - 1)) == 0) {
    typename Bytes<SIZE>::type raw = *reinterpret_cast<const typename Bytes<SIZE>::type*>(src);
    const T* const e = reinterpret_cast<const T*>(&raw);
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = to_f32(e[j]);
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = j < valid ? to_f32(src[j]) : 0.0f;
  }
}
template <typename T, int W>
__device__ __forceinline__ void store_some(void* base, int64_t i, int valid, const T (&v)[W]) {
  T* const dst = static_cast<T*>(base) + i;
  constexpr int SIZE = (int)sizeof(T) * W;
  if (valid == W && (reinterpret_cast<uintptr_t>(dst) & (SIZE - 1)) == 0) {
    typename Bytes<SIZE>::type raw;
    T* const e = reinterpret_cast<T*>(&raw);
#pragma unroll
    for (int j = 0; j < W; ++j) e[j] = v[j];
    *reinterpret_cast<typename Bytes<SIZE>::type*>(dst) = raw;
  } else {
#pragma unroll
    for (int j = 0; j < W; ++j)
      if (j < valid) dst[j] = v[j];
  }
}
template <int W>
__device__ __forceinline__ void load_typed(const void* base, int type, int64_t i, int valid, float (&v)[W]) {
  if (type == LT_F32) load_some<float, W>(base, i, valid, v);
  else if (type == LT_BF16) load_some<__nv_bfloat16, W>(base, i, valid, v);
  else load_some<__half, W>(base, i, valid, v);
}
template <typename T, int W>
__device__ __forceinline__ void store_as(void* base, int64_t i, int valid, const float (&v)[W]) {
  T t[W];
#pragma unroll
  for (int j = 0; j < W; ++j) t[j] = from_f32<T>(v[j]);
  store_some<T, W>(base, i, valid, t);
}
template <int W>
__device__ __forceinline__ void store_typed(void* base, int type, int64_t i, int valid, const float (&v)[W]) {
  if (type == LT_F32) store_as<float, W>(base, i, valid, v);
  else if (type == LT_BF16) store_as<__nv_bfloat16, W>(base, i, valid, v);
  else store_as<__half, W>(base, i, valid, v);
}

// Nearest code of the operands' own format, ties to the even code, saturated.  E4M3: the conversion instruction (a NaN becomes
// the NaN code).  M4E3: its codes are consecutive from binary32 pattern 1.0 in steps of 2^19, but for code 0, which is zero; the
// smallest magnitude 1.0625 takes over halfway from it (0.53125 itself goes to the even code, zero).  A NaN saturates there.
__device__ __forceinline__ uint8_t encode_e4m3(float v) {
  uint16_t d;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(d) : "f"(0.0f), "f"(v));
  return (uint8_t)(d & 0xFF);
}
__device__ __forceinline__ uint8_t encode_m4e3(float v) {
  const float mag = fminf(fabsf(v), 248.0f);
  if (mag <= 0.53125f) return 0;
  const uint32_t u = __float_as_uint(fmaxf(mag, 1.0f));
  int code = (int)((u + 0x3FFFFu + ((u >> 19) & 1u)) >> 19) - (127 << 4);
  code = code < 1 ? 1 : code;  // 127 at most: 248 is on the grid
  return (uint8_t)(code | (v < 0.0f ? 0x80 : 0));
}

template <int W>
__device__ __forceinline__ void store_out(const LinearProblem& p, int64_t i, int valid, const float (&v)[W]) {
  if (p.dst_type == LT_CODES) {
    const float scale = *p.out_scale;
    uint8_t c[W];
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const float q = __fdiv_rn(v[j], scale);
      c[j] = p.in_m4e3 ? encode_m4e3(q) : encode_e4m3(q);
    }
    store_some<uint8_t, W>(p.dst, i, valid, c);
  } else {
    store_typed<W>(p.dst, p.dst_type, i, valid, v);
  }
}

// ------------------------------------------------------------------ the epilogue
__device__ __forceinline__ float scaled(float y, float sa, const float* sb, int per_col, const float* bias, int64_t n) {
  const float r = __fmul_rn(__fmul_rn(y, sa), sb[per_col ? n : 0]);
  return bias ? __fadd_rn(r, bias[n]) : r;
}

// W finished sums of row m (m < M), columns n to n + W - 1 (n a multiple of W; those from N on are not there); y: real values, every zero +0
template <int W>
__device__ __forceinline__ void layer_store(const LinearProblem& p, int64_t m, int64_t n, const float (&y)[W]) {
  static_assert(W == 2 || W == 4, "columns of a thread");
  if (n >= p.N) return;
  const float sa = p.sa[p.sa_per_row ? m : 0];
  if (p.gated) {
    constexpr int H = W / 2;
    const int64_t c = n >> 1, i = m * p.n + c;
    const int valid = p.n - c < H ? (int)(p.n - c) : H;
    float z[H], v[H], o[H];
#pragma unroll
    for (int j = 0; j < H; ++j) {
      z[j] = v[j] = 0.0f;
      if (j < valid) {
        z[j] = scaled(y[2 * j], sa, p.sb, p.sb_per_col, p.bias, c + j);
        v[j] = scaled(y[2 * j + 1], sa, p.sb2, p.sb_per_col, p.bias2, c + j);
      }
    }
    if (p.pre) {
      store_typed<H>(p.pre, p.pre_type, i, valid, z);
      store_typed<H>(p.pre, p.pre_type, i + p.M * p.n, valid, v);
    }
    act_values<H>(p.act, z);
#pragma unroll
    for (int j = 0; j < H; ++j) o[j] = __fmul_rn(z[j], v[j]);
    store_out<H>(p, i, valid, o);
    return;
  }
  const int64_t i = m * p.n + n;
  const int valid = p.n - n < W ? (int)(p.n - n) : W;
  float o[W];
#pragma unroll
  for (int j = 0; j < W; ++j) o[j] = j < valid ? scaled(y[j], sa, p.sb, p.sb_per_col, p.bias, n + j) : 0.0f;
  if (p.pre) store_typed<W>(p.pre, p.pre_type, i, valid, o);
  act_values<W>(p.act, o);
  if (p.drop_below) {
    const uint4 r = philox((uint32_t)(n >> 2), (uint32_t)m, p.rng[1], p.rng[0]);
    const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
    for (int j = 0; j < W; ++j) {
      const uint32_t word = W == 4 ? w[j] : (n & 2) ? w[2 + j] : w[j];
      o[j] = word >= p.drop_below ? __fmul_rn(o[j], p.keep_scale) : 0.0f;
    }
  }
  if (p.residual) {
    float r[W];
    load_typed<W>(p.residual, p.residual_type, i, valid, r);
#pragma unroll
    for (int j = 0; j < W; ++j) o[j] = __fadd_rn(o[j], r[j]);
  }
  store_out<W>(p, i, valid, o);
}

// The sums of a thread's TM x TN micro-tile of a BM x BN tile, still in carrier scaling, through layer_store.  The loops are
// rolled: sixteen copies of the epilogue would cost more in instruction fetches than the trip of the sums through local memory.
template <int BM, int BN, int TM, int TN>
__device__ __forceinline__ void layer_store_tile(const LinearProblem& p, int64_t m0, int64_t n0, int tx, int ty, const float (&s)[TM][TN]) {
#pragma unroll 1
  for (int i = 0; i < TM; ++i) {
    const int64_t m = m0 + (i / 4) * (BM / 2) + ty * 4 + (i % 4);
    if (m >= p.M) continue;
#pragma unroll 1
    for (int h = 0; h < TN / 4; ++h) {
      float y[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        y[j] = __fmul_rn(__fmul_rn(s[i][h * 4 + j], p.un1), p.un2);
        y[j] = (y[j] == 0.0f) ? 0.0f : y[j];
      }
      layer_store<4>(p, m, n0 + h * (BN / 2) + tx * 4, y);
    }
  }
}
// the same for one row piece
template <int W>
__device__ __forceinline__ void layer_store_sums(const LinearProblem& p, int64_t m, int64_t n, const float (&s)[W]) {
  float y[W];
#pragma unroll
  for (int j = 0; j < W; ++j) {
    y[j] = __fmul_rn(__fmul_rn(s[j], p.un1), p.un2);
    y[j] = (y[j] == 0.0f) ? 0.0f : y[j];
  }
  layer_store<W>(p, m, n, y);
}

}  // namespace lba
