// Gradients of attention.  With dp_ij = g[i] v[j] and delta[i] = g[i] out[i]:
//
//   p_ij = exp(scale q[i] k[j] - lse[i])     ds_ij = p_ij (dp_ij - delta[i])
//   grad_q[i] = scale sum_j ds_ij k[j]       grad_k[j] = scale sum_i ds_ij q[i]       grad_v[j] = sum_i p_ij g[i]
//
// Two launches.  attention_delta_kernel forms delta and turns lse into powers of two, reading grad_out and out once.  Then
// attention_grad_kernel: a CTA takes 128 rows that stay, of q (for grad_q) or of k and v (for grad_k and grad_v, over all query heads of
// the group), and walks over 128 rows of the others at a time:
//   T1 = X1 Y1^T (scores), T2 = X2 Y2^T (dp)       X: q, g or k, v: shared memory for the whole CTA; Y: the other two, from two rings
//   p from T1, then ds from T2                     two warpgroups, 64 columns each, a row a thread
//   acc1 += ds Y1, and for keys acc2 += p Y2       p and ds lie in tensor memory over T2, sums in 128 more columns each
// Scores and dp are so formed twice, seven products where five would do; in return every sum is formed by one CTA in a fixed order, and no
// 32-bit gradient of q goes through memory or atomics.
//
// Bound by the matrix instructions, 512 clocks each (four for keys, three for queries), and by the 1024 clocks of exponentials and what goes
// with them, which they hide only in part: 2600 clocks a tile for keys, 2100 for queries.  p waits in registers until T2 has been read: so T1(n+1) is formed
// as soon as T1(n) is in registers, and scores are there before the warpgroups want them.  Where the sums leave room in tensor memory (queries; heads
// of up to 64) there is a second T2, and T2(n+1) is formed ahead too; else it follows acc1(n) and acc2(n) while the warpgroups form p of tile n+1.  (With
// p over T1, T1(n+1) came after acc2(n): 3500 clocks a tile.  With p in shared memory there is room for two tiles of Y1 only, and their copies came late: 4200.)
// 2 x 4096 tokens, 16 heads and 4 key-value heads of 128, causal, both launches: 470 us in a steady run, under the power limit (0.73 PFLOP/s of the
// five products), 408 in a burst.  binary16, whose maxima the first launch forms as well: 435.
// (Tiles of 64 rows, two of them in flight, a warpgroup each: with 64 columns a product wants 192 bytes of shared memory a clock, or 128 of
// tensor memory, and took 57 clocks a step instead of 32; 2 x 4096 tokens of 16 heads took 515 us.)
//
// p and ds are rounded to the inputs' type on their way into the products, which leaves gradients off by 1.4 times what their own rounding
// costs; where a CTA walks over one or two tiles of a head, and a few terms may cancel, they have a second piece (over T1, which is then formed late).
// delta comes from an output of 16 bits; where few keys are seen, that would add as much again (1.6 times with four keys), so rows
// of up to 32 keys get theirs from p and dp.  binary16 has few exponents: p is held times 2^8, and ds times a power of two chosen from the
// largest finite |grad_out| and |v| so that it cannot overflow: for grad_q of the row's own g and the values up to its block's last key, for the
// others of the rows from the block's first on that go with its keys.  So neither other sequences nor rows and keys that a mask hides cost it bits.
#include <algorithm>
#include <cmath>

#include "lba_tile.cuh"

namespace lba {
namespace {

constexpr int XT = 128, YT = 128, YC = 64, GRAD_THREADS = 384, Y1_SLOTS = 3, Y2_SLOTS = 2, CUTS = 4, DELTA_THREADS = 256;  // YC: columns of a warpgroup
constexpr int FINE_TILES = 2;  // of a head: walks in which p and ds have two pieces
constexpr float P_UP = 256.0f;
constexpr int P_BITS = 8;

struct GradParams {
  CUtensorMap q, k, v, g;    // boxes of 128 rows
  const int32_t *cu_q, *cu_k;
  int64_t q_rows, k_rows, key_blocks;
  int sequences, heads, kv_heads, group, dim, causal, bf;
  float to_log2, scale;
  const float2* stats;       // [heads][q_rows]: lse in powers of two, delta
  const uint32_t *most_g, *most_v;  // see DeltaParams
  const uint8_t* row_most;
  const void* g_raw;
  void *grad_q, *grad_k, *grad_v;
};
struct DeltaParams {
  const void *g, *out, *q, *k, *v;
  lba_strides q_at, k_at, v_at;
  const float* lse;
  const int32_t *cu_q, *cu_k;
  int64_t q_rows, k_rows;
  int few_parts;             // blocks that share a sequence's rows of few keys in one head
  uint32_t few_blocks, value_blocks;  // of rows of few keys; of 128 rows of v in one head (binary16)
  int sequences, heads, kv_heads, dim, causal;
  float to_log2;
  float2* stats;
  // binary16 only: largest finite |grad_out|, |v| of blocks of 128 rows as bits, [block_at][kv_heads]; the exponent byte of a row's |grad_out|, [heads][q_rows]
  uint32_t *most_g, *most_v;
  uint8_t* row_most;
  void *grad_q, *grad_k, *grad_v;
};
// the place of block t of sequence b, which begins at row `first`, among all sequences' blocks of 128 rows: sequences leave one free at most
__device__ __forceinline__ int64_t block_at(int first, int b, int t) { return (int64_t)(first / XT) + b + t; }

// ------------------------------------------------------------------ delta
// A warp takes 8 or 16 heads of a row, 16 lanes each, or 8 where a head has up to 64 values; they and the sequences' ends are on their way at once.  Rows
// of no sequence get gradients of 0.
constexpr int FEW_KEYS = 32, DELTA_AHEAD = 4;
template <typename T>
__device__ __forceinline__ void widen8(const T* src, float (&v)[8]) {  // at a 16-byte boundary
  const uint4 raw = *reinterpret_cast<const uint4*>(src);
  const T* const e = reinterpret_cast<const T*>(&raw);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
}
template <typename T>
__device__ __forceinline__ void load_half8(const T* src, float (&v)[8]) {
  const uint4 raw = __ldg(reinterpret_cast<const uint4*>(src));
  widen8(reinterpret_cast<const T*>(&raw), v);
}
// The rows of a sequence that see few keys, for one head: sum p dp / sum p.  Keys, values and 8 rows at a time lie in shared memory; a warp a row, a key
// a lane.  Four blocks share the rows, which are 32 at most under a causal mask, and come before the others.  (One block behind them, with rows read as they
// were wanted, kept 2 x 4096 rows of 16 heads at 31 us instead of 19.)  Without a mask they are all rows of a sequence of few keys: so there are as many
// blocks as leave one eight turns of eight rows, where sequences are of one length, and 64 at most (with four, 8192 rows of 16 heads over 32 keys
// took 627 us instead of 218, and 65536 took 6800 instead of 1760; over 33 keys, which have none of these blocks, 110 and 820).
constexpr int FEW_ROWS = DELTA_THREADS / 32, FEW_PARTS = 4, FEW_PARTS_MOST = 64, FEW_TURNS = 8, FEW_PITCH = 128 / 8 + 1;  // pieces of 16 bytes from row to row: lanes' pieces lie in different banks
struct FewShared {
  uint4 k[FEW_KEYS * FEW_PITCH], v[FEW_KEYS * FEW_PITCH], q[FEW_ROWS * FEW_PITCH], g[FEW_ROWS * FEW_PITCH];
  float lse[FEW_ROWS];
};
template <typename T>
__device__ void delta_of_few(const DeltaParams& p, int b, int h, int part, FewShared& sh) {
  int q_first, q_count, k_first, k_count;
  rows_of(p.cu_q, p.q_rows, b, &q_first, &q_count);
  rows_of(p.cu_k, p.k_rows, b, &k_first, &k_count);
  const int off = k_count - q_count, lane = threadIdx.x & 31, pieces = p.dim / 8;
  const int first = (p.causal ? max(0, -off) : 0) + part * FEW_ROWS, last = p.causal ? min(q_count, FEW_KEYS - off) : k_count <= FEW_KEYS ? q_count : 0;
  const int most = min(k_count, FEW_KEYS);
  if (first >= last || most == 0) return;
  const int kv = h / (p.heads / p.kv_heads);
  const auto bring = [&](uint4* to, const void* from, int64_t row, int rows, int head, const lba_strides& at) {
    for (int i = threadIdx.x; i < rows * pieces; i += DELTA_THREADS) {
      const int j = i / pieces, c = i - j * pieces;
      to[j * FEW_PITCH + c] = __ldg(reinterpret_cast<const uint4*>(static_cast<const T*>(from) + (row + j) * at.token + head * at.head) + c);
    }
  };
  const lba_strides g_at = {(int64_t)p.heads * p.dim, p.dim};
  for (int i0 = first; i0 < last; i0 += p.few_parts * FEW_ROWS) {
    const int rows = min(FEW_ROWS, last - i0), i = threadIdx.x >> 5;
    const int64_t row0 = q_first + i0;
    if (i0 == first) {
      bring(sh.k, p.k, k_first, most, kv, p.k_at);
      bring(sh.v, p.v, k_first, most, kv, p.v_at);
    } else {
      __syncthreads();  // (the rows before are no longer read)
    }
    bring(sh.q, p.q, row0, rows, h, p.q_at);
    bring(sh.g, p.g, row0, rows, h, g_at);
    if (threadIdx.x < rows) sh.lse[threadIdx.x] = __ldg(p.lse + h * p.q_rows + row0 + threadIdx.x);
    __syncthreads();
    if (i < rows) {
      const int keys = p.causal ? min(k_count, i0 + i + off + 1) : k_count, mine = min(lane, most - 1) * FEW_PITCH;
      const float lse = sh.lse[i];
      float s = 0.0f, dp = 0.0f;
#pragma unroll 2
      for (int c = 0; c < pieces; ++c) {
        float a[8], x[8];
        widen8(reinterpret_cast<const T*>(sh.q + i * FEW_PITCH + c), a);
        widen8(reinterpret_cast<const T*>(sh.k + mine + c), x);
#pragma unroll
        for (int f = 0; f < 8; ++f) s = fmaf(a[f], x[f], s);
        widen8(reinterpret_cast<const T*>(sh.g + i * FEW_PITCH + c), a);
        widen8(reinterpret_cast<const T*>(sh.v + mine + c), x);
#pragma unroll
        for (int f = 0; f < 8; ++f) dp = fmaf(a[f], x[f], dp);
      }
      float weight = lane < keys ? exp2_approx(fmaf(s, p.to_log2, -lse * LOG2E)) : 0.0f, sum = lane < keys ? weight * dp : 0.0f;
#pragma unroll
      for (int x = 16; x > 0; x /= 2) {
        sum += __shfl_xor_sync(0xFFFFFFFFu, sum, x);
        weight += __shfl_xor_sync(0xFFFFFFFFu, weight, x);
      }
      if (lane == 0) p.stats[h * p.q_rows + row0 + i] = make_float2(lse * LOG2E, __fdividef(sum, weight));  // (weights add up to 1, but for rounding)
    }
  }
}

// The sequence of a row, or -1.  A warp, every lane the same arguments and results, here and in ends_of.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int sequences, int64_t row, int lane) {
  if (!cu) return 0;
  const auto holds = [&](int x) { return cu[x] <= row && row < cu[x + 1]; };
  if (sequences >= 32) {
    int b = 0, hi = sequences - 1;  // the last sequence that begins at or before the row
    while (b < hi) {
      const int mid = (b + hi + 1) / 2;
      if (cu[mid] <= row) b = mid;
      else hi = mid - 1;
    }
    if (holds(b)) return b;
  }
  // (that is another one where offsets descend: a sequence that ends before it starts)
  for (int b0 = 0; b0 < sequences; b0 += 32) {
    const unsigned has = __ballot_sync(0xFFFFFFFFu, b0 + lane < sequences && holds(b0 + lane));
    if (has) return b0 + __ffs(has) - 1;
  }
  return -1;
}
// Of `row`'s sequence, which is returned (-1: none), the first row in q and the counts
__device__ __forceinline__ int ends_of(const DeltaParams& p, int64_t row, int lane, int* q_first, int* q_count, int* k_count) {
  if (p.cu_q && p.sequences < 32) {  // one trip to memory
    const int at = min(lane, p.sequences), q = __ldg(p.cu_q + at), k = p.cu_k ? __ldg(p.cu_k + at) : 0, q_next = __shfl_down_sync(0xFFFFFFFFu, q, 1);
    const unsigned has = __ballot_sync(0xFFFFFFFFu, lane < p.sequences && q <= row && row < q_next);
    const int b = max(__ffs(has) - 1, 0);
    const int q_top = (int)p.q_rows, k_top = (int)p.k_rows;
    *q_first = min(max(__shfl_sync(0xFFFFFFFFu, q, b), 0), q_top);
    *q_count = max(min(max(__shfl_sync(0xFFFFFFFFu, q, b + 1), 0), q_top) - *q_first, 0);
    const int lo = min(max(__shfl_sync(0xFFFFFFFFu, k, b), 0), k_top), hi = min(max(__shfl_sync(0xFFFFFFFFu, k, b + 1), 0), k_top);
    *k_count = p.cu_k ? max(hi - lo, 0) : k_top;
    return has ? b : -1;
  }
  const int b = sequence_of(p.cu_q, p.sequences, row, lane);
  int k_first;
  rows_of(p.cu_q, p.q_rows, max(b, 0), q_first, q_count);
  rows_of(p.cu_k, p.k_rows, max(b, 0), &k_first, k_count);
  return b;
}

// the largest finite magnitude of eight values, as bits
__device__ __forceinline__ uint32_t largest(const float (&x)[8], uint32_t most) {
#pragma unroll
  for (int e = 0; e < 8; ++e) most = fabsf(x[e]) < INFINITY ? max(most, __float_as_uint(fabsf(x[e]))) : most;
  return most;
}
// 128 rows of v in one head
template <typename T>
__device__ void most_of_values(const DeltaParams& p, uint32_t block) {
  __shared__ uint32_t warps[DELTA_THREADS / 32];
  const int h = (int)(block % p.kv_heads), pieces = p.dim / 8;
  const Place place = find_place(p.cu_q, p.q_rows, p.cu_k, p.k_rows, p.sequences, true, XT, block / p.kv_heads);
  if (!place.found) return;
  const int first = place.level * XT, rows = min(XT, place.k_count - first);
  const T* const src = static_cast<const T*>(p.v) + (int64_t)(place.k_first + first) * p.v_at.token + h * p.v_at.head;
  uint32_t most = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < rows * pieces; i += DELTA_THREADS) {
    float v[8];
    load_half8(src + i / pieces * p.v_at.token + i % pieces * 8, v);
    most = largest(v, most);
  }
  most = __reduce_max_sync(0xFFFFFFFFu, most);
  if ((threadIdx.x & 31) == 0) warps[threadIdx.x >> 5] = most;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < DELTA_THREADS / 32; ++i) most = max(most, warps[i]);
    p.most_v[block_at(place.k_first, place.sequence, place.level) * p.kv_heads + h] = most;
  }
}

template <typename T, int LANES>  // of a head
__global__ void __launch_bounds__(DELTA_THREADS, 5) attention_delta_kernel(const DeltaParams p) {
  constexpr int HEADS = 32 / LANES, SLOTS = DELTA_AHEAD * HEADS;  // heads at a time, of a block
  constexpr bool HALF = std::is_same<T, __half>::value;
  __shared__ FewShared few;
  __shared__ uint32_t most[DELTA_THREADS / 32][HALF ? SLOTS : 1];
  __shared__ int64_t most_at[DELTA_THREADS / 32];
  after_previous();
  if (blockIdx.x < p.few_blocks) {
    const uint32_t line = blockIdx.x / p.few_parts;
    if (blockIdx.y == 0) delta_of_few<T>(p, (int)(line / p.heads), (int)(line % p.heads), blockIdx.x % p.few_parts, few);
    return;
  }
  if (HALF && blockIdx.x < p.few_blocks + p.value_blocks) {
    if (blockIdx.y == 0) most_of_values<T>(p, blockIdx.x - p.few_blocks);
    return;
  }
  const int lane = threadIdx.x & 31, d = lane % LANES * 8, h0 = blockIdx.y * DELTA_AHEAD * HEADS + lane / LANES;
  const int64_t row = (int64_t)(blockIdx.x - p.few_blocks - p.value_blocks) * (DELTA_THREADS / 32) + (threadIdx.x >> 5);
  if (row < p.q_rows) {
    const T *const g_row = static_cast<const T*>(p.g) + row * p.heads * p.dim, *const o_row = static_cast<const T*>(p.out) + row * p.heads * p.dim;
    uint4 g[DELTA_AHEAD], o[DELTA_AHEAD];
    float lse[DELTA_AHEAD];
#pragma unroll
    for (int u = 0; u < DELTA_AHEAD; ++u) {
      const int h = h0 + u * HEADS;
      const bool there = h < p.heads && d < p.dim;
      g[u] = there ? __ldg(reinterpret_cast<const uint4*>(g_row + h * p.dim + d)) : make_uint4(0u, 0u, 0u, 0u);
      o[u] = there ? __ldg(reinterpret_cast<const uint4*>(o_row + h * p.dim + d)) : make_uint4(0u, 0u, 0u, 0u);
      lse[u] = h < p.heads ? __ldg(p.lse + h * p.q_rows + row) : 0.0f;
    }
    int q_first, q_count, k_count;
    const int b = ends_of(p, row, lane, &q_first, &q_count, &k_count);
    const bool inside = b >= 0;
    if (HALF && lane == 0) most_at[threadIdx.x >> 5] = inside ? block_at(q_first, b, ((int)row - q_first) / XT) : -1;
    const int keys = p.causal ? min(k_count, (int)row - q_first + k_count - q_count + 1) : k_count;
#pragma unroll
    for (int u = 0; u < DELTA_AHEAD; ++u) {
      const int h = h0 + u * HEADS;
      if (!inside) {
        if (h < p.heads && d < p.dim) *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_q) + (row * p.heads + h) * p.dim + d) = make_uint4(0u, 0u, 0u, 0u);
        continue;
      }
      float x[8], y[8], sum = 0.0f;
      widen8(reinterpret_cast<const T*>(&g[u]), x);
      widen8(reinterpret_cast<const T*>(&o[u]), y);
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(x[e], y[e], sum);
      if constexpr (HALF) {
        uint32_t m = largest(x, 0);
#pragma unroll
        for (int e = LANES / 2; e > 0; e /= 2) m = max(m, __shfl_xor_sync(0xFFFFFFFFu, m, e));
        if (d == 0) most[threadIdx.x >> 5][u * HEADS + lane / LANES] = m;
        if (d == 0 && h < p.heads) p.row_most[h * p.q_rows + row] = (uint8_t)(m >> 23);
      }
#pragma unroll
      for (int e = LANES / 2; e > 0; e /= 2) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, e);
      if (d == 0 && h < p.heads && !(keys > 0 && keys <= FEW_KEYS))
        p.stats[h * p.q_rows + row] = make_float2(lse[u] == -INFINITY ? INFINITY : lse[u] * LOG2E, sum);
    }
  }
  if (row < p.k_rows && blockIdx.y == 0) {
    const int64_t n = (int64_t)p.kv_heads * p.dim;
    if (p.cu_k && (row < p.cu_k[0] || row >= p.cu_k[p.sequences])) {
      for (int64_t i = lane * 8; i < n; i += 256) {
        *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_k) + row * n + i) = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_v) + row * n + i) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
  }
  if constexpr (HALF) {  // the rows' largest together, head by head of the key-value heads (a maximum does not depend on the order)
    if (row >= p.q_rows && lane == 0) most_at[threadIdx.x >> 5] = -1;
    __syncthreads();
    const int slot = threadIdx.x, h = blockIdx.y * SLOTS + slot, group = p.heads / p.kv_heads;
    if (slot < SLOTS && h < p.heads && (slot == 0 || h % group == 0)) {
      const int heads = min(min(group - h % group, SLOTS - slot), p.heads - h);
      uint32_t m = 0;
      for (int w = 0; w < DELTA_THREADS / 32; ++w) {
        if (most_at[w] < 0) continue;
        for (int i = 0; i < heads; ++i) m = max(m, most[w][slot + i]);
        if (w + 1 < DELTA_THREADS / 32 && most_at[w + 1] == most_at[w]) continue;
        uint32_t* const to = p.most_g + most_at[w] * p.kv_heads + h / group;
        if (m > __ldcg(to)) atomicMax(to, m);
        m = 0;
      }
    }
  }
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// what the rounding of a pair has cut off, rounded itself
template <typename T>
__device__ __forceinline__ uint32_t rest_of(float lo, float hi, uint32_t pair) {
  const T* const t = reinterpret_cast<const T*>(&pair);
  return pack_pair<T>(lo - to_f32(t[0]), hi - to_f32(t[1]));
}
// the power of two that ds is multiplied by, from the exponent bytes of the largest |g| and |v|: |ds| <= 2 dim |g| |v| stays below 2^15
__device__ __forceinline__ int ds_bits(uint32_t g, uint32_t v, int dim) {
  if (g == 0 || v == 0) return 0;
  return 15 - ((int)g - 126) - ((int)v - 126) - (33 - __clz(dim - 1));
}

// ------------------------------------------------------------------ gradients
template <int DT> constexpr int kGradTile = 128 * DT * 2;  // bytes of 128 rows

struct GradShared {
  uint64_t x_full, full1[Y1_SLOTS], empty1[Y1_SLOTS], full2[Y2_SLOTS], empty2[Y2_SLOTS];
  uint64_t cut1[CUTS], clean1[CUTS], cut2[CUTS], clean2[CUTS];  // copies that a mask cuts, and their cleaning
  uint64_t t1, t1_read, t2[2], ds_there, done;
  uint32_t tmem;
  int dead;
  int odd;                   // values of g that are not finite were taken out of a cut tile
  Place place;
  alignas(16) float minus[2][2][YC], delta[2][2][YC];  // [tile's parity][warpgroup]
};

template <int DT> constexpr size_t kGradTiles = (size_t)kGradTile<DT> * (2 + Y1_SLOTS + Y2_SLOTS);
template <int DT> constexpr size_t kGradSmem = kGradTiles<DT> + sizeof(GradShared);
static_assert(kGradSmem<128> <= 227 * 1024, "shared memory of a CTA");

// what a CTA walks over: tiles first..last - 1 of `heads` heads in turn
struct Walk {
  int heads, first, last;
  int low, high;             // tiles t with t < low or t >= high are cut by a mask
  __device__ __forceinline__ int count() const { return heads * max(0, last - first); }
  __device__ __forceinline__ bool cut(int t) const { return t < low || t >= high; }
};

template <typename T, int DT, bool KEYS>
__device__ void attention_grad(const GradParams& p, GradShared& sh, uint8_t* raw_smem, uint32_t base, int head, uint32_t tmem) {
  constexpr int BLOCKS = DT / 64, TILE = kGradTile<DT>, BLOCK = 128 * 128;
  // Tensor memory: T1, T2, acc1, acc2, 128 columns each; where the sums leave room, a second T2, which every other tile has
  constexpr bool TWO = !KEYS || DT == 64;
  constexpr int ACC1 = 256, ACC2 = TWO ? 320 : 384, OTHER = TWO ? 256 : 0;
  const int warp = threadIdx.x >> 5;
  const uint32_t ring1 = base + 2 * TILE, ring2 = ring1 + Y1_SLOTS * TILE;
  volatile int* const dead = &sh.dead;
  const Place place = sh.place;
  const int q_first = place.q_first, q_count = place.q_count, k_first = place.k_first, k_count = place.k_count;
  const int off = k_count - q_count;
  const int x_first = KEYS ? k_first : q_first, x_count = KEYS ? k_count : q_count, y_first = KEYS ? q_first : k_first, y_count = KEYS ? q_count : k_count;
  const int block = KEYS ? place.blocks - 1 - place.level : place.level;  // (with a causal mask the first keys and the last queries have most to do)
  const int x0 = block * XT;
  Walk walk;
  walk.heads = KEYS ? p.group : 1;
  walk.first = 0;
  walk.last = (y_count + YT - 1) / YT;
  walk.low = 0;
  walk.high = y_count / YT;
  if (p.causal && KEYS) {  // query i sees key j from i >= j - off on
    walk.first = max(0, x0 - off) / YT;
    walk.low = (max(0, min(x0 + XT, x_count) - 1 - off) + YT - 1) / YT;
  } else if (p.causal) {
    walk.last = (max(0, min(y_count, min(x0 + XT, x_count) + off)) + YT - 1) / YT;
    walk.high = min(walk.high, max(0, x0 + off + 1) / YT);
  }
  const int all = walk.count();
  const bool fine = walk.last - walk.first <= FINE_TILES;

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8) {
      if (elected() && all) {
        const auto load = [&](uint32_t dst, const CUtensorMap* map, int h, int row, uint32_t bar) {
          mbar_arrive_expect(bar, TILE);
#pragma unroll
          for (int x = 0; x < BLOCKS; ++x) tile_load(dst + x * BLOCK, map, x * 64, h, row, bar);
        };
        mbar_arrive_expect(smem_u32(&sh.x_full), 2 * TILE);
        for (int i = 0; i < 2; ++i)
          for (int x = 0; x < BLOCKS; ++x)
            tile_load(base + i * TILE + x * BLOCK, KEYS ? (i ? &p.v : &p.k) : (i ? &p.g : &p.q), x * 64, head, x_first + x0, smem_u32(&sh.x_full));
        int cuts = 0, h = 0, t = walk.first;
        for (int n = 0; n < all; ++n) {
          const int slot1 = n % Y1_SLOTS, slot2 = n % Y2_SLOTS, y_head = KEYS ? head * p.group + h : head / p.group, row = y_first + t * YT;
          // (of a cut tile, those who want it wait for its own barriers; the slot's phases count copies.  Fewer tiles than there are cut barriers
          // are under way, so the last use of each is over)
          const bool cut = walk.cut(t);
          if (!mbar_wait(smem_u32(&sh.empty1[slot1]), ((n / Y1_SLOTS) & 1) ^ 1, dead)) break;
          if (cut) mbar_arrive(smem_u32(&sh.full1[slot1]));
          load(ring1 + slot1 * TILE, KEYS ? &p.q : &p.k, y_head, row, smem_u32(cut ? &sh.cut1[cuts % CUTS] : &sh.full1[slot1]));
          if (!mbar_wait(smem_u32(&sh.empty2[slot2]), ((n / Y2_SLOTS) & 1) ^ 1, dead)) break;
          const bool cut2 = KEYS && cut;
          if (cut2) mbar_arrive(smem_u32(&sh.full2[slot2]));
          load(ring2 + slot2 * TILE, KEYS ? &p.g : &p.v, y_head, row, smem_u32(cut2 ? &sh.cut2[cuts % CUTS] : &sh.full2[slot2]));
          cuts += cut;
          if (++t == walk.last) {
            t = walk.first;
            ++h;
          }
        }
      }
    } else if (warp == 9) {
      if (elected()) {
        const int steps = (p.dim + 15) / 16;
        const uint32_t kind_t = tile_kind(p.bf, YT, false), kind_a = tile_kind(p.bf, steps * 16, true);
        const uint64_t rows = tile_operand(0, 16, 1024), lines = tile_operand(0, BLOCK, 1024);
        bool ok = all == 0 || mbar_wait(smem_u32(&sh.x_full), 0, dead);
        int cuts1 = 0, cuts2 = 0, t1 = walk.first, t2 = walk.first;  // of the next tile whose T1, T2 is formed
        const auto product = [&](uint32_t d, uint32_t x, uint32_t y, uint64_t& bar) {
          const uint64_t a = rows + (x >> 4), b = rows + (y >> 4);
#pragma unroll
          for (int s = 0; s < DT / 16; ++s) {
            if (s >= steps) break;
            const int at = ((s >> 2) * BLOCK + (s & 3) * 32) >> 4;
            mma_shared(d, a + at, b + at, kind_t, s != 0);
          }
          mma_arrive(smem_u32(&bar));
        };
        const auto form1 = [&](int n) {
          if (walk.cut(t1)) {
            ok = ok && mbar_wait(smem_u32(&sh.clean1[cuts1 % CUTS]), (cuts1 / CUTS) & 1, dead);
            ++cuts1;
          } else {
            ok = ok && mbar_wait(smem_u32(&sh.full1[n % Y1_SLOTS]), (n / Y1_SLOTS) & 1, dead);
          }
          if (++t1 == walk.last) t1 = walk.first;
          if (ok) product(tmem, base, ring1 + (n % Y1_SLOTS) * TILE, sh.t1);
        };
        const auto form2 = [&](int n) {
          if (KEYS && walk.cut(t2)) {
            ok = ok && mbar_wait(smem_u32(&sh.clean2[cuts2 % CUTS]), (cuts2 / CUTS) & 1, dead);
            ++cuts2;
          } else {
            ok = ok && mbar_wait(smem_u32(&sh.full2[n % Y2_SLOTS]), (n / Y2_SLOTS) & 1, dead);
          }
          if (++t2 == walk.last) t2 = walk.first;
          if (!ok) return;
          product(tmem + 128 + (n & 1) * OTHER, base + TILE, ring2 + (n % Y2_SLOTS) * TILE, sh.t2[n & 1]);
          if (!KEYS) mma_arrive(smem_u32(&sh.empty2[n % Y2_SLOTS]));
        };
        if (all && ok) {
          form1(0);
          form2(0);
        }
        for (int n = 0; n < all && ok; ++n) {
          if (n + 1 < all && !fine) {
            ok = mbar_wait(smem_u32(&sh.t1_read), n & 1, dead);
            tmem_after();
            form1(n + 1);
            if (TWO && ok) form2(n + 1);
          }
          ok = ok && mbar_wait(smem_u32(&sh.ds_there), n & 1, dead);
          if (!ok) break;
          tmem_after();
          // in T2, of each warpgroup's 64 columns: the pairs of ds, then those of p; in T1 their second pieces
          const auto add = [&](uint32_t acc, uint32_t a, uint32_t y, bool more) {
            const uint64_t b = lines + (y >> 4);
#pragma unroll
            for (int s = 0; s < YT / 16; ++s) mma_tensor(acc, a + (s >> 2) * YC + (s & 3) * 8, b + s * (2048 >> 4), kind_a, more || s != 0);
          };
          const uint32_t of = tmem + 128 + (n & 1) * OTHER;
          add(tmem + ACC1, of, ring1 + (n % Y1_SLOTS) * TILE, n != 0);
          if (fine) add(tmem + ACC1, tmem, ring1 + (n % Y1_SLOTS) * TILE, true);
          mma_arrive(smem_u32(&sh.empty1[n % Y1_SLOTS]));
          if (KEYS) {
            add(tmem + ACC2, of + YC / 2, ring2 + (n % Y2_SLOTS) * TILE, n != 0);
            if (fine) add(tmem + ACC2, tmem + YC / 2, ring2 + (n % Y2_SLOTS) * TILE, true);
            mma_arrive(smem_u32(&sh.empty2[n % Y2_SLOTS]));
          }
          if (n + 1 < all && fine) form1(n + 1);
          if (n + 1 < all && (fine || !TWO)) form2(n + 1);
        }
        mma_arrive(smem_u32(&sh.done));
      }
    } else {
      // Cut tiles.  Rows behind the sequence become 0 where they are summed over (0 times a neighbour's infinity would be NaN), and so do values of Y1
      // that are not finite: rows that see them have an lse that is NaN.  Rows of g that hold such values have a delta that is not finite; where a tile is
      // cut by the causal mask they are taken out too, and added to the sums of the keys that the row sees at the end.
      int cuts = 0, t = walk.first, h = 0;
      bool ok = true;
      const auto clean = [&](uint32_t tile_at, int at_t, const bool (&values)[YT / 64], uint64_t& there, uint64_t& clean) {
        bool odd = false;
        ok = ok && mbar_wait(smem_u32(&there), (cuts / CUTS) & 1, dead);
        if (!ok) return;
        uint8_t* const tile = raw_smem + (tile_at - smem_u32(raw_smem));
#pragma unroll
        for (int i = 0; i < YT / 64; ++i) {
          const int row = threadIdx.x - 10 * 32 + 64 * i;
          if (at_t * YT + row >= y_count) clear_row<BLOCKS>(tile, row);
          else if (values[i]) odd |= keep_finite<T, BLOCKS>(tile, row);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        if (KEYS && odd) sh.odd = 1;
        mbar_arrive(smem_u32(&clean));
      };
      for (int n = 0; n < all && ok; ++n) {
        const int at_t = t, at_h = h;
        if (++t == walk.last) {
          t = walk.first;
          ++h;
        }
        if (!walk.cut(at_t)) continue;
        bool values[YT / 64], bad_g[YT / 64];
#pragma unroll
        for (int i = 0; i < YT / 64; ++i) {
          const int row = at_t * YT + threadIdx.x - 10 * 32 + 64 * i;
          values[i] = p.causal;
          bad_g[i] = KEYS && at_t < walk.low && row < y_count &&
                     !isfinite(__ldg(p.stats + (int64_t)(head * p.group + at_h) * p.q_rows + y_first + row).y);
        }
        clean(ring1 + (n % Y1_SLOTS) * TILE, at_t, values, sh.cut1[cuts % CUTS], sh.clean1[cuts % CUTS]);
        if (KEYS) clean(ring2 + (n % Y2_SLOTS) * TILE, at_t, bad_g, sh.cut2[cuts % CUTS], sh.clean2[cuts % CUTS]);
        ++cuts;
      }
    }
    return;
  }

  asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
  const int w = warp >> 2, thread = threadIdx.x & 127, x = x0 + thread;  // the thread's row of X
  const uint32_t lanes = (uint32_t)(warp & 3) << 21, t1 = tmem + w * YC + lanes;
  const u64 c = both(p.to_log2);
  bool ok = true;
  int bits = 0;
  if constexpr (std::is_same<T, __half>::value) {
    const int kv = KEYS ? head : head / p.group;
    const auto most_of = [&](const uint32_t* most, int first, int from, int to) {
      uint32_t x = 0;
      for (int t = from + (threadIdx.x & 31); t < to; t += 32) x = max(x, __ldg(most + block_at(first, place.sequence, t) * p.kv_heads + kv));
      return __reduce_max_sync(0xFFFFFFFFu, x) >> 23;
    };
    // (rows from walk.first on see the keys up to the last)
    const uint32_t v = most_of(p.most_v, k_first, 0, KEYS ? (k_count + YT - 1) / YT : walk.last);
    const uint32_t g = KEYS ? most_of(p.most_g, q_first, walk.first, walk.last) : x < x_count ? __ldg(p.row_most + (int64_t)head * p.q_rows + x_first + x) : 0u;
    bits = ds_bits(g, v, p.dim);
  }
  const float up = power_of_two(bits - P_BITS);  // of ds, beside the 2^8 of p
  const u64 up2 = both(up);
  float2 mine = make_float2(0.0f, 0.0f);  // queries: this row's; keys: a column's of the next tile
  int h_ahead = 0, t_ahead = walk.first;  // of the next tile whose statistics are fetched
  const auto stats_ahead = [&] {
    const int i = t_ahead * YT + w * YC + thread;
    mine = make_float2(0.0f, 0.0f);
    if (h_ahead < walk.heads && thread < YC && i < y_count) mine = __ldg(p.stats + (int64_t)(head * p.group + h_ahead) * p.q_rows + y_first + i);
    if (++t_ahead >= walk.last) {
      t_ahead = walk.first;
      ++h_ahead;
    }
  };
  const auto hand_over = [&](int n) {
    if (thread < YC) {
      sh.minus[n & 1][w][thread] = P_BITS - mine.x;
      sh.delta[n & 1][w][thread] = -mine.y * up;
    }
    stats_ahead();
  };
  if (KEYS) {
    stats_ahead();
    hand_over(0);
  } else if (x < x_count) {
    mine = __ldg(p.stats + (int64_t)head * p.q_rows + x_first + x);
  }
  const u64 row_minus = both(P_BITS - mine.x), row_delta = both(-mine.y * up);
  int t = walk.first;
  for (int n = 0; n < all; ++n) {
    const int at_t = t;
    if (++t == walk.last) t = walk.first;
    ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.t1), n & 1, dead));
    tmem_after();
    int lo = 0, hi = YC;  // of the warpgroup's columns, those that the row goes with
    const bool cut = walk.cut(at_t);
    if (cut) {
      const int first = at_t * YT + w * YC;
      if (KEYS) {
        hi = y_count - first;
        if (p.causal) lo = x - off - first;
      } else {
        hi = (p.causal ? min(y_count, x + off + 1) : y_count) - first;
      }
    }
    uint32_t s[YC];  // scores, then weights
    if (ok) {
#pragma unroll
      for (int e = 0; e < YC; e += 32) tmem_load32(t1 + e, s + e);
      tmem_wait_ld();
      tmem_before();
      mbar_arrive(smem_u32(&sh.t1_read));
    }
    // The columns' statistics are there, and those of the last tile are read no more.  The warpgroup's own, so the barrier is its own too; warps whose
    // wait ran out meet the others here all the same.
    if (KEYS) asm volatile("bar.sync %0, 128;" ::"r"(1 + w) : "memory");
    if (!ok) continue;
    uint32_t pw[KEYS ? YC / 2 : 1];
    const auto weights = [&](auto masked) {  // (a test per element, even of a value that is the same for all, doubled the instructions)
#pragma unroll
      for (int e = 0; e < YC; e += 4) {
        const float4 m = KEYS ? *reinterpret_cast<const float4*>(&sh.minus[n & 1][w][e]) : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int f = 0; f < 4; f += 2) {
          float p0, p1;
          unpack2(fma2_rn(pack2u(s[e + f], s[e + f + 1]), c, KEYS ? (f ? pack2(m.z, m.w) : pack2(m.x, m.y)) : row_minus), p0, p1);
          p0 = exp2_approx(p0);
          p1 = exp2_approx(p1);
          if constexpr (decltype(masked)::value) {
            if (e + f < lo || e + f >= hi) p0 = 0.0f;
            if (e + f + 1 < lo || e + f + 1 >= hi) p1 = 0.0f;
          }
          s[e + f] = __float_as_uint(p0);
          s[e + f + 1] = __float_as_uint(p1);
          if (KEYS) pw[(e + f) / 2] = pack_pair<T>(p0, p1);
        }
      }
    };
    if (cut) weights(std::true_type());
    else weights(std::false_type());
    if (KEYS) hand_over(n + 1);
    ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.t2[n & 1]), (n >> 1) & 1, dead));
    if (!ok) continue;
    tmem_after();
    const uint32_t t2 = t1 + 128 + (n & 1) * OTHER;
    // the upper half first: p goes over it while the lower one is formed
    uint32_t dw[YC / 2];
    const auto slopes = [&](auto masked, auto two) {
#pragma unroll
      for (int half = YC - 32; half >= 0; half -= 32) {
        uint32_t dp[32];
        tmem_load32(t2 + half, dp);
        float4 m[KEYS ? 8 : 1];
        if (KEYS) {
#pragma unroll
          for (int e = 0; e < 8; ++e) m[e] = *reinterpret_cast<const float4*>(&sh.delta[n & 1][w][half + 4 * e]);
        }
        tmem_wait_ld();
        if (KEYS && half) tmem_store32(t2 + YC / 2, pw);
        uint32_t rest[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
          const float4& four = m[KEYS ? e / 4 : 0];
          float d0, d1;
          unpack2(mul2_rn(fma2_rn(pack2u(dp[e], dp[e + 1]), up2, KEYS ? (e & 2 ? pack2(four.z, four.w) : pack2(four.x, four.y)) : row_delta),
                          pack2u(s[half + e], s[half + e + 1])), d0, d1);
          if constexpr (decltype(masked)::value) {  // (0 times what a mask hides may be NaN)
            if (half + e < lo || half + e >= hi) d0 = 0.0f;
            if (half + e + 1 < lo || half + e + 1 >= hi) d1 = 0.0f;
          }
          dw[(half + e) / 2] = pack_pair<T>(d0, d1);
          if constexpr (decltype(two)::value) rest[e / 2] = rest_of<T>(d0, d1, dw[(half + e) / 2]);
        }
        if constexpr (decltype(two)::value) {
          tmem_st16(t1 + half / 2, rest);
          if constexpr (KEYS) {
#pragma unroll
            for (int e = 0; e < 32; e += 2) rest[e / 2] = rest_of<T>(__uint_as_float(s[half + e]), __uint_as_float(s[half + e + 1]), pw[(half + e) / 2]);
            tmem_st16(t1 + YC / 2 + half / 2, rest);
          }
        }
      }
    };
    if (fine) slopes(std::true_type(), std::true_type());
    else if (cut) slopes(std::true_type(), std::false_type());
    else slopes(std::false_type(), std::false_type());
    tmem_store32(t2, dw);
    tmem_wait_st();
    tmem_before();
    mbar_arrive(smem_u32(&sh.ds_there));
  }
  // both warpgroups bring the sums out, each half of the columns
  ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.done), 0, dead)) && ok && !*dead;
  tmem_after();
  const int lane = threadIdx.x & 31, out_heads = KEYS ? p.kv_heads : p.heads, there = min(32, x_count - (x - lane));  // rows of the warp
  const float by1 = p.scale * power_of_two(-bits), by2 = 1.0f / P_UP;
  // 32 values a row at a time, through shared memory (X is no longer read), four lanes a row side by side
  uint8_t* const stage = raw_smem + (base - smem_u32(raw_smem)) + warp * 2048;
  const auto piece_of = [&](int r, int c) { return reinterpret_cast<uint4*>(stage + r * 64 + ((c ^ ((r >> 1) & 3)) << 4)); };
#pragma unroll 1
  for (int which = 0; which < (KEYS ? 2 : 1); ++which) {
    T* const dst = static_cast<T*>(KEYS ? (which ? p.grad_v : p.grad_k) : p.grad_q);
    const float by = which ? by2 : by1;
#pragma unroll 1
    for (int d = w * (DT / 2); d < (w + 1) * (DT / 2) && d < p.dim; d += 32) {
      uint32_t o[32];
      if (all) {
        tmem_load32(tmem + (which ? ACC2 : ACC1) + lanes + d, o);
        tmem_wait_ld();
      } else {
#pragma unroll
        for (int e = 0; e < 32; ++e) o[e] = 0u;
      }
      if (KEYS && which && sh.odd && x < x_count) {  // what was taken out of g
        for (int h = 0; h < walk.heads; ++h) {
          for (int i = max(walk.first * YT, x - off); i < min(walk.low * YT, y_count); ++i) {
            const int64_t h_at = head * p.group + h;
            if (isfinite(__ldg(p.stats + h_at * p.q_rows + y_first + i).y)) continue;
            const T* const src = static_cast<const T*>(p.g_raw) + ((int64_t)(y_first + i) * p.heads + h_at) * p.dim + d;
#pragma unroll
            for (int e = 0; e < 32; ++e) {
              const float v = d + e < p.dim ? to_f32(src[e]) : 0.0f;
              if (!isfinite(v)) o[e] = __float_as_uint(__uint_as_float(o[e]) + v);
            }
          }
        }
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = pack_pair<T>(__uint_as_float(o[8 * e + 2 * u]) * by, __uint_as_float(o[8 * e + 2 * u + 1]) * by);
        *piece_of(lane, e) = make_uint4(v[0], v[1], v[2], v[3]);
      }
      __syncwarp();
      const int c = lane & 3;
#pragma unroll
      for (int r = lane >> 2; r < 32; r += 8) {
        if (r >= there || d + c * 8 >= p.dim) break;
        uint4 v = *piece_of(r, c);
        if (!ok) v = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);  // NaN
        *reinterpret_cast<uint4*>(dst + ((int64_t)(x_first + x - lane + r) * out_heads + head) * p.dim + d + c * 8) = v;
      }
      __syncwarp();
    }
  }
  tmem_before();
}

template <typename T, int DT>
__global__ void __launch_bounds__(GRAD_THREADS, 1) attention_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ __align__(1024) uint8_t raw_smem[];  // (1024: the swizzle's period.  There is no room to find a boundary in)
  GradShared& sh = *reinterpret_cast<GradShared*>(raw_smem + kGradTiles<DT>);
  const int warp = threadIdx.x >> 5;
  const uint32_t base = smem_u32(raw_smem);
  if (threadIdx.x == 8 * 32) {
    map_ahead(&p.q);
    map_ahead(&p.k);
    map_ahead(&p.v);
    map_ahead(&p.g);
  }
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&sh.x_full), 1);
    mbar_init(smem_u32(&sh.done), 1);
    for (int i = 0; i < Y1_SLOTS; ++i) {
      mbar_init(smem_u32(&sh.full1[i]), 1);
      mbar_init(smem_u32(&sh.empty1[i]), 1);
    }
    for (int i = 0; i < Y2_SLOTS; ++i) {
      mbar_init(smem_u32(&sh.full2[i]), 1);
      mbar_init(smem_u32(&sh.empty2[i]), 1);
    }
    for (int i = 0; i < CUTS; ++i) {
      mbar_init(smem_u32(&sh.cut1[i]), 1);
      mbar_init(smem_u32(&sh.cut2[i]), 1);
      mbar_init(smem_u32(&sh.clean1[i]), 64);
      mbar_init(smem_u32(&sh.clean2[i]), 64);
    }
    mbar_init(smem_u32(&sh.t1), 1);
    for (int i = 0; i < 2; ++i) mbar_init(smem_u32(&sh.t2[i]), 1);
    mbar_init(smem_u32(&sh.t1_read), 256);
    mbar_init(smem_u32(&sh.ds_there), 256);
    mbar_init_fence();
    sh.dead = 0;
    sh.odd = 0;
  }
  after_previous();
  if (warp == 9) tmem_alloc(smem_u32(&sh.tmem), 512);
  const bool keys = (int64_t)blockIdx.x < p.key_blocks;
  const int64_t index = keys ? blockIdx.x : blockIdx.x - p.key_blocks;
  const int heads = keys ? p.kv_heads : p.heads, head = (int)(index % heads);
  if (warp == 8) {
    const Place place = find_place(p.cu_q, p.q_rows, p.cu_k, p.k_rows, p.sequences, keys, XT, index / heads);
    if ((threadIdx.x & 31) == 0) sh.place = place;
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = sh.tmem;
  const bool found = sh.place.found != 0;
  if (found) {
    if (keys) attention_grad<T, DT, true>(p, sh, raw_smem, base, head, tmem);
    else attention_grad<T, DT, false>(p, sh, raw_smem, base, head, tmem);
  }
  __syncthreads();
  if (warp == 9) {
    if (sh.dead) let_copies_land();
    else if (found) mbar_wait(smem_u32(&sh.done), 0, &sh.dead);
    tmem_after();
    __syncwarp();
    tmem_free(tmem, 512);
  }
}

template <typename T, int DT>
cudaError_t launch_grad(const GradParams& p, int64_t blocks, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(attention_grad_kernel<T, DT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kGradSmem<DT>);
  if (e != cudaSuccess) return e;
  return launch_after(attention_grad_kernel<T, DT>, dim3((unsigned)blocks), GRAD_THREADS, kGradSmem<DT>, stream, p);
}

template <typename T, int LANES>
cudaError_t launch_delta(const DeltaParams& d, int64_t blocks, cudaStream_t stream) {
  constexpr int HEADS = DELTA_AHEAD * 32 / LANES;
  return launch_after(attention_delta_kernel<T, LANES>, dim3((unsigned)blocks, (unsigned)((d.heads + HEADS - 1) / HEADS)), DELTA_THREADS, 0, stream, d);
}

size_t stats_bytes(const lba_attention_how* h) { return (size_t)h->heads * h->q_rows * sizeof(float2); }
// blocks of 128 rows as block_at counts them, and bytes of the largest magnitudes of q's and k's
int64_t blocks_of(const lba_attention_how* h, int64_t rows) { return rows / XT + h->sequences; }
size_t most_bytes(const lba_attention_how* h) {
  return h->type == LBA_TYPE_BF16 ? 0 : (size_t)(blocks_of(h, h->q_rows) + blocks_of(h, h->k_rows)) * h->kv_heads * sizeof(uint32_t);
}
size_t stats_offset(const lba_attention_how* h) { return (most_bytes(h) + 255) / 256 * 256; }
size_t row_bytes(const lba_attention_how* h) { return h->type == LBA_TYPE_BF16 ? 0 : (size_t)h->heads * h->q_rows; }

}  // namespace
}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_backward_workspace_bytes(const lba_attention_how* how) {
  return check_attention(how) == LBA_OK && how->sequences ? stats_offset(how) + stats_bytes(how) + row_bytes(how) : 0;
}

int lba_attention_backward(const void* grad_out, const void* q, const void* k, const void* v, const void* out, const float* lse,
                           const lba_attention_how* how, void* grad_q, void* grad_k, void* grad_v, void* workspace, size_t workspace_bytes, void* stream) {
  const int st = check_attention(how);
  if (st != LBA_OK) return st;
  const cudaStream_t s = (cudaStream_t)stream;
  if ((how->q_rows > 0 && (!grad_out || !q || !out || !lse || !grad_q)) || (how->k_rows > 0 && (!k || !v || !grad_k || !grad_v))) return LBA_ERR_NULL;
  for (const void* t : {grad_out, q, k, v, out, (const void*)grad_q, (const void*)grad_k, (const void*)grad_v})
    if (!aligned16(t)) return LBA_ERR_ALIGN;
  const size_t q_bytes = (size_t)how->q_rows * how->heads * how->dim * 2, k_bytes = (size_t)how->k_rows * how->kv_heads * how->dim * 2;
  if (how->sequences == 0 || how->q_rows == 0 || how->k_rows == 0) {  // no pair at all
    cudaError_t e = q_bytes ? cudaMemsetAsync(grad_q, 0, q_bytes, s) : cudaSuccess;
    if (e == cudaSuccess && k_bytes) e = cudaMemsetAsync(grad_k, 0, k_bytes, s);
    if (e == cudaSuccess && k_bytes) e = cudaMemsetAsync(grad_v, 0, k_bytes, s);
    return status_of(e);
  }
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < lba_attention_backward_workspace_bytes(how)) return LBA_ERR_WORKSPACE;
  GradParams p;
  p.bf = how->type == LBA_TYPE_BF16;
  const lba_strides g_at = {(int64_t)how->heads * how->dim, how->dim};
  if (!head_map(&p.q, p.bf, q, how->q_rows, how->heads, how->dim, how->q_at, YT) || !head_map(&p.g, p.bf, grad_out, how->q_rows, how->heads, how->dim, g_at, YT) ||
      !head_map(&p.k, p.bf, k, how->k_rows, how->kv_heads, how->dim, how->k_at, YT) ||
      !head_map(&p.v, p.bf, v, how->k_rows, how->kv_heads, how->dim, how->v_at, YT))
    return cuda_fail(cudaErrorInvalidValue);
  uint32_t *const most_g = p.bf ? nullptr : static_cast<uint32_t*>(workspace), *const most_v = p.bf ? nullptr : most_g + blocks_of(how, how->q_rows) * how->kv_heads;
  float2* const stats = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + stats_offset(how));
  DeltaParams d = {};
  d.g = grad_out;
  d.out = out;
  d.q = q;
  d.k = k;
  d.v = v;
  d.q_at = how->q_at;
  d.k_at = how->k_at;
  d.v_at = how->v_at;
  d.causal = how->causal != 0;
  d.to_log2 = how->scale * LOG2E;
  d.lse = lse;
  d.cu_q = p.cu_q = how->cu_q;
  d.cu_k = p.cu_k = how->cu_k;
  d.q_rows = p.q_rows = how->q_rows;
  d.k_rows = p.k_rows = how->k_rows;
  d.sequences = p.sequences = how->sequences;
  d.heads = p.heads = how->heads;
  d.kv_heads = p.kv_heads = how->kv_heads;
  d.dim = p.dim = how->dim;
  d.stats = stats;
  d.most_g = most_g;
  d.most_v = most_v;
  d.row_most = reinterpret_cast<uint8_t*>(stats) + stats_bytes(how);
  p.row_most = d.row_most;
  d.grad_q = p.grad_q = grad_q;
  d.grad_k = p.grad_k = grad_k;
  d.grad_v = p.grad_v = grad_v;
  p.stats = stats;
  p.g_raw = grad_out;
  p.most_g = most_g;
  p.most_v = most_v;
  p.group = how->heads / how->kv_heads;
  p.causal = how->causal != 0;
  p.to_log2 = how->scale * LOG2E;
  p.scale = how->scale;
  p.key_blocks = (how->k_rows / XT + how->sequences) * how->kv_heads;
  const int64_t blocks = p.key_blocks + (how->q_rows / XT + how->sequences) * how->heads;
  const int64_t most_rows = how->q_rows > how->k_rows ? how->q_rows : how->k_rows, row_blocks = (most_rows + DELTA_THREADS / 32 - 1) / (DELTA_THREADS / 32);
  const int64_t turns = how->causal ? 0 : how->q_rows / how->sequences / FEW_ROWS;
  d.few_parts = (int)std::min<int64_t>(std::max<int64_t>(turns / FEW_TURNS, FEW_PARTS), FEW_PARTS_MOST);
  const int64_t few_blocks = (int64_t)how->sequences * how->heads * d.few_parts, value_blocks = p.bf ? 0 : blocks_of(how, how->k_rows) * how->kv_heads;
  const int64_t delta_blocks = row_blocks + few_blocks + value_blocks;
  if (delta_blocks > 2147483647LL || blocks > 2147483647LL) return LBA_ERR_SHAPE;
  d.few_blocks = (uint32_t)few_blocks;
  d.value_blocks = (uint32_t)value_blocks;
  cudaError_t e = most_g ? cudaMemsetAsync(most_g, 0, blocks_of(how, how->q_rows) * how->kv_heads * sizeof(uint32_t), s) : cudaSuccess;
  if (e != cudaSuccess) return status_of(e);
  e = how->dim <= 64 ? (p.bf ? launch_delta<__nv_bfloat16, 8>(d, delta_blocks, s) : launch_delta<__half, 8>(d, delta_blocks, s))
                     : (p.bf ? launch_delta<__nv_bfloat16, 16>(d, delta_blocks, s) : launch_delta<__half, 16>(d, delta_blocks, s));
  if (e != cudaSuccess) return status_of(e);
  if (how->dim <= 64) return status_of(p.bf ? launch_grad<__nv_bfloat16, 64>(p, blocks, s) : launch_grad<__half, 64>(p, blocks, s));
  return status_of(p.bf ? launch_grad<__nv_bfloat16, 128>(p, blocks, s) : launch_grad<__half, 128>(p, blocks, s));
}

}  // extern "C"
