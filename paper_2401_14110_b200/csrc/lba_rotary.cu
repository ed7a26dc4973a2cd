// Rotary positions: pair (x, y) of a head at position p and frequency f becomes (x cos pf - y sin pf, x sin pf + y cos pf) scale.
//
// Bound by memory: a value is read once and written once.  A block takes a few tokens: it forms their cosines and sines once in shared
// memory, then all heads of q and k use them.  Angles are formed in binary64 and reduced to a quarter turn there, which costs some 60
// instructions a pair of a token against 40 heads' loads and stores; in binary32 position 100000 would be off by 0.004.  A thread's first
// values are on their way while the table is formed: for single tokens that is one trip to memory instead of two.
#include <cmath>

#include "lba_entry.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

constexpr int ROT_THREADS = 256, ROT_AHEAD = 2, ROT_TABLE = 48 * 1024;

struct RotaryParams {
  const void *q, *k;
  void *q_out, *k_out;
  lba_strides q_at, k_at, q_out_at, k_out_at;
  const void* positions;
  const double* freqs;
  int64_t tokens;
  int heads, all_heads;       // of q; of both
  int pairs, rest;            // a head's pairs, and its values that pass
  int items, rot_items;       // pieces of work of a head: PV pairs each, then 2 PV passing values each
  int tile, block_heads;      // tokens and heads of a block
  int wide_positions, inverse;
  float scale;
};

template <typename T, int N, int ALIGN> struct alignas(ALIGN) Few { T v[N]; };

// one piece: where it comes from and goes to, and its values
template <typename T, int PV, bool INTER>
struct Piece {
  T* to;
  static constexpr int RUN = INTER ? 2 * PV : PV;
  Few<T, RUN, PV == 1 ? sizeof(T) : RUN * sizeof(T)> a, b;  // half layout: two runs
  int token, pair;                   // pair < 0: passes
  __device__ __forceinline__ void load(const RotaryParams& p, int i, int64_t t0, int h0, int hs) {
    const int c = i % p.items, r = i / p.items;
    const int h = h0 + r % hs;
    token = r / hs;
    const bool is_q = h < p.heads;
    const int head = is_q ? h : h - p.heads;
    const lba_strides from_at = is_q ? p.q_at : p.k_at, to_at = is_q ? p.q_out_at : p.k_out_at;
    const int64_t t = t0 + token;
    pair = c < p.rot_items ? c * PV : -1;
    const int first = c < p.rot_items ? (INTER ? 2 * c * PV : c * PV) : 2 * p.pairs + (c - p.rot_items) * 2 * PV;
    const T* const from = static_cast<const T*>(is_q ? p.q : p.k) + t * from_at.token + head * from_at.head + first;
    to = static_cast<T*>(is_q ? p.q_out : p.k_out) + t * to_at.token + head * to_at.head + first;
    a = *reinterpret_cast<const decltype(a)*>(from);
    if (!INTER) b = *reinterpret_cast<const decltype(b)*>(from + step(p));
  }
  __device__ __forceinline__ int step(const RotaryParams& p) const { return pair < 0 ? PV : p.pairs; }
  __device__ __forceinline__ void turn(const RotaryParams& p, const float2* table) {
    if (pair >= 0) {
      const float2* const w = table + token * p.pairs + pair;
#pragma unroll
      for (int j = 0; j < PV; ++j) {
        T& x = INTER ? a.v[2 * j] : a.v[j];
        T& y = INTER ? a.v[INTER ? 2 * j + 1 : j] : b.v[j];
        const float fx = to_f32(x), fy = to_f32(y), c = w[j].x, s = w[j].y;
        x = from_f32<T>(fx * c - fy * s);
        y = from_f32<T>(fx * s + fy * c);
      }
    }
    *reinterpret_cast<decltype(a)*>(to) = a;
    if (!INTER) *reinterpret_cast<decltype(b)*>(to + step(p)) = b;
  }
};

template <typename T, int PV, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS) rotary_kernel(const RotaryParams p) {
  extern __shared__ float2 table[];  // [tokens][pairs]: cosine, sine
  after_previous();
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int tokens = p.tokens - t0 < p.tile ? (int)(p.tokens - t0) : p.tile;
  const int h0 = blockIdx.y * p.block_heads, hs = p.all_heads - h0 < p.block_heads ? p.all_heads - h0 : p.block_heads;
  const int total = tokens * hs * p.items;
  Piece<T, PV, INTER> piece[ROT_AHEAD];
#pragma unroll
  for (int u = 0; u < ROT_AHEAD; ++u) {
    const int i = threadIdx.x + u * ROT_THREADS;
    if (i < total) piece[u].load(p, i, t0, h0, hs);
  }
  for (int i = threadIdx.x; i < tokens * p.pairs; i += ROT_THREADS) {
    const int t = i / p.pairs, j = i - t * p.pairs;
    const int64_t at = t0 + t;
    const double pos = p.wide_positions ? (double)static_cast<const int64_t*>(p.positions)[at] : (double)static_cast<const int32_t*>(p.positions)[at];
    const double quarters = pos * p.freqs[j] * 0.63661977236758134308;  // 2 / pi
    const double whole = rint(quarters);
    const int quadrant = (int)(whole - 4.0 * floor(whole * 0.25));
    float s, c;
    sincospif(0.5f * (float)(quarters - whole), &s, &c);
    float2 w = quadrant == 0 ? make_float2(c, s) : quadrant == 1 ? make_float2(-s, c) : quadrant == 2 ? make_float2(-c, -s) : make_float2(s, -c);
    if (p.inverse) w.y = -w.y;
    table[i] = make_float2(w.x * p.scale, w.y * p.scale);
  }
  __syncthreads();
  for (int i0 = threadIdx.x; i0 < total; i0 += ROT_AHEAD * ROT_THREADS) {
#pragma unroll
    for (int u = 0; u < ROT_AHEAD; ++u)
      if (i0 + u * ROT_THREADS < total) piece[u].turn(p, table);
#pragma unroll
    for (int u = 0; u < ROT_AHEAD; ++u) {
      const int i = i0 + (ROT_AHEAD + u) * ROT_THREADS;
      if (i < total) piece[u].load(p, i, t0, h0, hs);
    }
  }
}

// PV pairs at a time where sizes, strides and addresses allow it; else fewer
template <typename T, int PV, bool INTER>
cudaError_t run_rotary(RotaryParams p, cudaStream_t stream) {
  constexpr int BYTES = (int)sizeof(T) * PV * (INTER ? 2 : 1);
  if constexpr (PV > 1) {
    bool fits = p.pairs % PV == 0 && p.rest % (2 * PV) == 0;
    const auto good = [&](const void* a, const lba_strides& s) {
      return (reinterpret_cast<uintptr_t>(a) | (uintptr_t)(s.token * (int64_t)sizeof(T)) | (uintptr_t)(s.head * (int64_t)sizeof(T))) % BYTES == 0;
    };
    fits = fits && good(p.q, p.q_at) && good(p.q_out, p.q_out_at) && good(p.k, p.k_at) && good(p.k_out, p.k_out_at);
    if (!fits) return run_rotary<T, PV / 2, INTER>(p, stream);
  }
  p.rot_items = p.pairs / PV;
  p.items = p.rot_items + p.rest / (2 * PV);
  // Tokens of a block: as many as leave four blocks an SM, eight at most; with few tokens the heads are divided too
  const int sms = device_sms();
  const int64_t fair = p.tokens / (4 * sms);
  p.tile = (int)(fair < 1 ? 1 : fair > 8 ? 8 : fair);
  while (p.tile > 1 && (size_t)p.tile * p.pairs * sizeof(float2) > ROT_TABLE) --p.tile;
  const int64_t blocks = (p.tokens + p.tile - 1) / p.tile;
  int64_t parts = blocks >= 2 * sms ? 1 : (2 * sms + blocks - 1) / blocks;
  if (parts > p.all_heads) parts = p.all_heads;
  p.block_heads = (int)((p.all_heads + parts - 1) / parts);
  const dim3 grid((unsigned)blocks, (unsigned)((p.all_heads + p.block_heads - 1) / p.block_heads));
  return launch_after(rotary_kernel<T, PV, INTER>, grid, ROT_THREADS, (size_t)p.tile * p.pairs * sizeof(float2), stream, p);
}
template <typename T>
cudaError_t run_rotary(const RotaryParams& p, bool interleaved, cudaStream_t stream) {
  return interleaved ? run_rotary<T, 8 / (int)sizeof(T), true>(p, stream) : run_rotary<T, 16 / (int)sizeof(T), false>(p, stream);
}

}  // namespace
}  // namespace lba

using namespace lba;

extern "C" int lba_rotary(const void* q, lba_strides q_at, const void* k, lba_strides k_at, const lba_rotary_how* how, void* q_out,
                          lba_strides q_out_at, void* k_out, lba_strides k_out_at, void* stream) {
  if (!how) return LBA_ERR_NULL;
  if (how->type != LBA_TYPE_F32 && !half_type(how->type)) return LBA_ERR_LAYER;
  if (how->tokens < 0 || how->tokens > 2147483647LL || how->heads < 1 || how->kv_heads < 0 || how->heads > 65535 || how->kv_heads > 65535 - how->heads ||
      how->dim < 2 || how->dim > 1024 || how->dim % 2 || how->rotary_dim < 2 || how->rotary_dim > how->dim || how->rotary_dim % 2)
    return LBA_ERR_SHAPE;
  if (!std::isfinite(how->scale)) return LBA_ERR_LAYER;
  if (how->tokens == 0) return LBA_OK;
  if (!q || !q_out || (how->kv_heads && (!k || !k_out)) || !how->positions || !how->freqs) return LBA_ERR_NULL;
  RotaryParams p = {};
  p.q = q;
  p.q_out = q_out;
  p.q_at = q_at;
  p.q_out_at = q_out_at;
  if (how->kv_heads) {
    p.k = k;
    p.k_out = k_out;
    p.k_at = k_at;
    p.k_out_at = k_out_at;
  }
  p.positions = how->positions;
  p.freqs = how->freqs;
  p.tokens = how->tokens;
  p.heads = how->heads;
  p.all_heads = how->heads + how->kv_heads;
  p.pairs = how->rotary_dim / 2;
  p.rest = how->dim - how->rotary_dim;
  p.wide_positions = how->wide_positions != 0;
  p.inverse = how->inverse != 0;
  p.scale = how->scale;
  cudaStream_t s = (cudaStream_t)stream;
  return status_of(how->type == LBA_TYPE_F32    ? run_rotary<float>(p, how->interleaved != 0, s)
                   : how->type == LBA_TYPE_BF16 ? run_rotary<__nv_bfloat16>(p, how->interleaved != 0, s)
                                                : run_rotary<__half>(p, how->interleaved != 0, s));
}
