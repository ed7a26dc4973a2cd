// Rotary positions: pair (x, y) of a head at position p and frequency f becomes (x cos pf - y sin pf, x sin pf + y cos pf) scale.
//
// Bound by memory: a value is read once and written once.  A thread keeps a place in the row of a token, a head's pairs or some of its passing
// values, and walks over the tokens of its block, the next one's values on their way; cosines and sines of the block's tokens come from a table in
// shared memory that its threads form first, while the first values are on their way (for single tokens that is one trip to memory instead of
// two).  Angles are formed in binary64 and reduced to a quarter turn there, some 50 instructions a pair of a token against 40 heads' loads
// and stores; in binary32 position 100000 would be off by 0.004.  (With places and tokens found by division for every piece, 8191 tokens of
// 40 heads took 46 us, 270 instructions a piece.)
#include <cmath>

#include "lba_entry.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

constexpr int ROT_THREADS = 512, ROT_TABLE = 48 * 1024;

struct RotaryParams {
  const void *q, *k;
  void *q_out, *k_out;
  lba_strides q_at, k_at, q_out_at, k_out_at;
  const void* positions;
  const double* freqs;
  int64_t tokens;
  int heads, all_heads;       // of q; of both
  int pairs, rest;            // a head's pairs, and its values that pass
  int items, rot_items;       // pieces of a head: PV pairs each, then 2 PV passing values each
  int tile;                   // tokens of a block
  int wide_positions, inverse;
  float scale;
};

template <typename T, int N, int ALIGN> struct alignas(ALIGN) Few { T v[N]; };

template <typename T, int PV, bool INTER>
__global__ void __launch_bounds__(ROT_THREADS, 3) rotary_kernel(const RotaryParams p) {
  constexpr int RUN = INTER ? 2 * PV : PV;
  typedef Few<T, RUN, PV == 1 ? sizeof(T) : RUN * sizeof(T)> Vec;
  extern __shared__ float2 table[];  // [tokens][pairs]: cosine, sine
  after_previous();
  const int64_t t0 = (int64_t)blockIdx.x * p.tile;
  const int tokens = p.tokens - t0 < p.tile ? (int)(p.tokens - t0) : p.tile;
  const int place = blockIdx.y * blockDim.x + threadIdx.x;
  const bool mine = place < p.all_heads * p.items;
  const int h = place / p.items, c = place - h * p.items;
  const bool is_q = h < p.heads, turns = c < p.rot_items;
  const int head = is_q ? h : h - p.heads;
  const lba_strides from_at = is_q ? p.q_at : p.k_at, to_at = is_q ? p.q_out_at : p.k_out_at;
  const int first = turns ? (INTER ? 2 * c * PV : c * PV) : 2 * p.pairs + (c - p.rot_items) * 2 * PV, step = turns ? p.pairs : PV;
  const T* from = static_cast<const T*>(is_q ? p.q : p.k) + t0 * from_at.token + head * from_at.head + first;
  T* to = static_cast<T*>(is_q ? p.q_out : p.k_out) + t0 * to_at.token + head * to_at.head + first;
  Vec a, b;  // half layout, and what passes: two runs
  const auto load = [&] {
    a = *reinterpret_cast<const Vec*>(from);
    if (!INTER) b = *reinterpret_cast<const Vec*>(from + step);
    from += from_at.token;
  };
  if (mine) load();
  for (int i = threadIdx.x; i < tokens * p.pairs; i += blockDim.x) {
    const int t = i / p.pairs, j = i - t * p.pairs;
    const int64_t at = t0 + t;
    const double pos = p.wide_positions ? (double)static_cast<const int64_t*>(p.positions)[at] : (double)static_cast<const int32_t*>(p.positions)[at];
    const double quarters = pos * p.freqs[j] * 0.63661977236758134308;  // 2 / pi
    const double whole = rint(quarters);
    const int quadrant = (int)__double2ll_rn(whole) & 3;
    // sine and cosine of at most an eighth of a turn: their series, what is left out below 2^-28 of them
    const float x = (float)(quarters - whole) * 1.57079632679f, x2 = x * x;
    const float s = fmaf(x * x2, fmaf(x2, fmaf(x2, fmaf(x2, 1.0f / 362880, -1.0f / 5040), 1.0f / 120), -1.0f / 6), x);
    const float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -1.0f / 3628800, 1.0f / 40320), -1.0f / 720), 1.0f / 24), -0.5f), 1.0f);
    float2 w = quadrant & 1 ? make_float2(-s, c) : make_float2(c, s);
    if (quadrant & 2) w = make_float2(-w.x, -w.y);
    if (p.inverse) w.y = -w.y;
    // (a thread's PV pairs lie a row of pieces apart, two and two, so that neighbouring threads' 16 bytes are neighbours)
    const int piece = PV == 1 ? j : 2 * (((j % PV) / 2) * p.rot_items + j / PV) + j % 2;
    table[t * p.pairs + piece] = make_float2(w.x * p.scale, w.y * p.scale);
  }
  __syncthreads();
  if (!mine) return;
  const float2* w = table + (turns ? (PV == 1 ? c : 2 * c) : 0);
#pragma unroll 1
  for (int t = 0; t < tokens; ++t) {
    Vec x = a, y = b;
    if (t + 1 < tokens) load();
    if (turns) {
#pragma unroll
      for (int j = 0; j < PV; ++j) {
        T& first_of = INTER ? x.v[2 * j] : x.v[j];
        T& second_of = INTER ? x.v[INTER ? 2 * j + 1 : j] : y.v[j];
        const float2 cs = PV == 1 ? w[0] : w[2 * (j / 2) * p.rot_items + j % 2];
        const float fx = to_f32(first_of), fy = to_f32(second_of);
        first_of = from_f32<T>(fx * cs.x - fy * cs.y);
        second_of = from_f32<T>(fx * cs.y + fy * cs.x);
      }
    }
    *reinterpret_cast<Vec*>(to) = x;
    if (!INTER) *reinterpret_cast<Vec*>(to + step) = y;
    to += to_at.token;
    w += p.pairs;
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
  // Places in equal blocks of whole warps.  Tokens of a block: five, or as many as leave four blocks an SM.  Blocks form their tables while others
  // move values: 8191 tokens of 40 heads took 46 us with all blocks in one round of twelve tokens, 37 with eight tokens, 35 with five, 52 with one.
  const int64_t places = (int64_t)p.all_heads * p.items;
  const int64_t parts = (places + ROT_THREADS - 1) / ROT_THREADS, threads = ((places + parts - 1) / parts + 31) / 32 * 32;
  const int64_t fair = p.tokens / (4 * device_sms());
  p.tile = (int)(fair < 1 ? 1 : fair > 5 ? 5 : fair);
  while (p.tile > 1 && (size_t)p.tile * p.pairs * sizeof(float2) > ROT_TABLE) --p.tile;
  const dim3 grid((unsigned)((p.tokens + p.tile - 1) / p.tile), (unsigned)((places + threads - 1) / threads));
  return launch_after(rotary_kernel<T, PV, INTER>, grid, (int)threads, (size_t)p.tile * p.pairs * sizeof(float2), stream, p);
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
