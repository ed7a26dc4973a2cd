// Gradients of attention.  With dp_ij = g[i] v[j] and delta[i] = g[i] out[i]:
//
//   p_ij = exp(scale q[i] k[j] - lse[i])     ds_ij = p_ij (dp_ij - delta[i])
//   grad_q[i] = scale sum_j ds_ij k[j]       grad_k[j] = scale sum_i ds_ij q[i]       grad_v[j] = sum_i p_ij g[i]
//
// Two launches.  attention_delta_kernel forms delta and turns lse into powers of two, reading grad_out and out once.  Then
// attention_grad_kernel: a CTA takes 128 rows that stay, of q (for grad_q) or of k and v (for grad_k and grad_v, over all query heads of
// the group), and walks over 64 rows of the others at a time:
//   T1 = X1 Y1^T (scores), T2 = X2 Y2^T (dp)       X: q, g or k, v: shared memory for the whole CTA; Y: the other two, from a ring
//   p and ds from T1 and T2, in registers          two warpgroups, each every second tile, a row a thread
//   acc1 += ds Y1, and for keys acc2 += p Y2       p and ds lie in tensor memory over T1 and T2, sums in 128 more columns each
// Scores and dp are so formed twice, seven products where five would do; in return every sum is formed by one CTA in a fixed order, and no
// 32-bit gradient of q goes through memory or atomics.
//
// p is rounded to the inputs' type on its way into the product, and ds held as two pieces of it: delta comes from an output of 16 bits, and one
// rounding more of ds would leave grad_q and grad_k off by 1.5 times what their own rounding costs (with two pieces by 1.1 times).  binary16
// has few exponents: p is held times 2^8, and ds times a power of two chosen from the largest |grad_out| and |v| so that it cannot overflow.
//
// Bound by the matrix instructions.  128 x 64 scores with both operands in shared memory want 192 bytes a clock where 128 are there, 384 clocks
// instead of 256, so a query block's X lies in tensor memory (1024 clocks a tile); a key block has no columns left for that (1536).
#include <cmath>

#include "lba_tile.cuh"

namespace lba {
namespace {

constexpr int XT = 128, YT = 64, GRAD_THREADS = 384, GRAD_STAGES = 4, DELTA_THREADS = 256;
constexpr float P_UP = 256.0f;
constexpr int P_BITS = 8;

struct GradParams {
  CUtensorMap q, k, v, g;    // boxes of 64 rows
  const int32_t *cu_q, *cu_k;
  int64_t q_rows, k_rows, key_blocks;
  int sequences, heads, kv_heads, group, dim, causal, bf;
  float to_log2, scale;
  const void *q_raw, *g_raw; // contiguous grad_out
  lba_strides q_at;
  const float2* stats;       // [heads][q_rows]: lse in powers of two, delta
  const uint32_t* most;      // largest |grad_out|, |v| as bits (binary16), or null
  void *grad_q, *grad_k, *grad_v;
};
struct DeltaParams {
  const void *g, *out, *v;
  lba_strides v_at;
  const float* lse;
  const int32_t *cu_q, *cu_k;
  int64_t q_rows, k_rows;
  int sequences, heads, kv_heads, dim;
  float2* stats;
  uint32_t* most;
  void *grad_q, *grad_k, *grad_v;
};

// ------------------------------------------------------------------ delta
// A group of 16 lanes takes a row's head.  Rows of no sequence get gradients of 0.
template <typename T>
__global__ void __launch_bounds__(DELTA_THREADS) attention_delta_kernel(const DeltaParams p) {
  after_previous();
  const int sub = threadIdx.x & 15, d = sub * 8;
  const int64_t n = p.q_rows * p.heads, m = p.k_rows * p.kv_heads;
  const int64_t at = (int64_t)blockIdx.x * (DELTA_THREADS / 16) + (threadIdx.x >> 4);
  uint32_t most_g = 0, most_v = 0;
  if (at < n) {
    const int64_t row = at / p.heads;
    const int head = (int)(at - row * p.heads);
    const bool inside = !p.cu_q || (row >= p.cu_q[0] && row < p.cu_q[p.sequences]);
    float sum = 0.0f;
    if (d < p.dim) {
      const int64_t i = at * p.dim + d;
      if (inside) {
        float g[8], o[8];
        load_some<T, 8>(p.g, i, 8, g);
        load_some<T, 8>(p.out, i, 8, o);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          sum = fmaf(g[e], o[e], sum);
          most_g = max(most_g, __float_as_uint(g[e]) & 0x7FFFFFFFu);
        }
      } else {
        *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_q) + i) = make_uint4(0u, 0u, 0u, 0u);
      }
    }
#pragma unroll
    for (int x = 8; x > 0; x /= 2) sum += __shfl_xor_sync(0xFFFFu << (threadIdx.x & 16), sum, x);
    if (sub == 0) {
      const float lse = inside ? p.lse[head * p.q_rows + row] : 0.0f;
      p.stats[head * p.q_rows + row] = make_float2(lse == -INFINITY ? INFINITY : lse * LOG2E, sum);
    }
  }
  if (at < m && d < p.dim) {
    const int64_t row = at / p.kv_heads;
    const bool inside = !p.cu_k || (row >= p.cu_k[0] && row < p.cu_k[p.sequences]);
    if (!inside) {
      *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_k) + at * p.dim + d) = make_uint4(0u, 0u, 0u, 0u);
      *reinterpret_cast<uint4*>(static_cast<T*>(p.grad_v) + at * p.dim + d) = make_uint4(0u, 0u, 0u, 0u);
    } else if (p.most) {
      float v[8];
      load_some<T, 8>(static_cast<const T*>(p.v) + row * p.v_at.token + (at - row * p.kv_heads) * p.v_at.head, d, 8, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) most_v = max(most_v, __float_as_uint(v[e]) & 0x7FFFFFFFu);
    }
  }
  if (p.most) {  // (a maximum does not depend on the order)
    most_g = __reduce_max_sync(0xFFFFFFFFu, most_g);
    most_v = __reduce_max_sync(0xFFFFFFFFu, most_v);
    if ((threadIdx.x & 31) == 0) {
      if (most_g > __ldcg(p.most)) atomicMax(p.most, most_g);
      if (most_v > __ldcg(p.most + 1)) atomicMax(p.most + 1, most_v);
    }
  }
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(127 + e) << 23); }
// the power of two that ds is multiplied by: |ds| <= 2 dim |g| |v| stays below 2^15
__device__ __forceinline__ int ds_bits(const GradParams& p) {
  if (!p.most) return 0;
  const uint32_t g = p.most[0], v = p.most[1];
  if (g >= 0x7F800000u || v >= 0x7F800000u || g == 0 || v == 0) return 0;
  return 15 - ((int)(g >> 23) - 126) - ((int)(v >> 23) - 126) - (33 - __clz(p.dim - 1));
}

// ------------------------------------------------------------------ gradients
template <int DT> constexpr int kX = XT * DT * 2;  // bytes of a tile
template <int DT> constexpr int kY = YT * DT * 2;
template <int DT> constexpr size_t kGradSmem = 1024 + 2 * (size_t)kX<DT> + 2 * (size_t)kY<DT> * GRAD_STAGES;

struct GradShared {
  uint64_t x_full, x_there, full[GRAD_STAGES], empty[GRAD_STAGES], cut_full[4], clean[4], products[2], weights[2], done;
  uint32_t tmem;
  int dead, seq, block, found;
  alignas(16) float2 stats[2][YT];
};

// what a CTA walks over: tiles first..last - 1 of `heads` heads in turn
struct Walk {
  int heads, first, last;
  int low, high;             // tiles t with t < low or t >= high are cut by a mask
  __device__ __forceinline__ int count() const { return heads * max(0, last - first); }
  __device__ __forceinline__ bool cut(int t) const { return t < low || t >= high; }
};

template <typename T>
__device__ __forceinline__ float2 pair_values(uint32_t w) {
  if constexpr (std::is_same<T, __nv_bfloat16>::value) return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

template <typename T, int DT, bool KEYS>
__device__ void attention_grad(const GradParams& p, GradShared& sh, uint8_t* raw_smem, uint32_t base, int head, uint32_t tmem) {
  constexpr int BLOCKS = DT / 64, X = kX<DT>, Y = kY<DT>, X_BLOCK = XT * 128, Y_BLOCK = YT * 128;
  const int warp = threadIdx.x >> 5;
  const uint32_t ring = base + 2 * X;
  volatile int* const dead = &sh.dead;
  int q_first, q_count, k_first, k_count;
  rows_of(p.cu_q, p.q_rows, sh.seq, &q_first, &q_count);
  rows_of(p.cu_k, p.k_rows, sh.seq, &k_first, &k_count);
  const int off = k_count - q_count;
  const int x_first = KEYS ? k_first : q_first, x_count = KEYS ? k_count : q_count, y_first = KEYS ? q_first : k_first, y_count = KEYS ? q_count : k_count;
  // longest first: the last queries, the first keys
  const int block = !KEYS && p.causal ? (x_count + XT - 1) / XT - 1 - sh.block : sh.block;
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
  const int tiles = max(0, walk.last - walk.first), all = walk.count();

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 8) {
      if (elected() && all) {
        if (KEYS) {
          mbar_arrive_expect(smem_u32(&sh.x_full), 2 * X);
          for (int i = 0; i < 2; ++i)
            for (int x = 0; x < BLOCKS; ++x)
              for (int r = 0; r < 2; ++r)
                tile_load(base + i * X + x * X_BLOCK + r * Y_BLOCK, i ? &p.v : &p.k, x * 64, head, x_first + x0 + r * YT, smem_u32(&sh.x_full));
        }
        int cuts = 0;
        for (int n = 0; n < all; ++n) {
          const int stage = n % GRAD_STAGES, h = n / tiles, t = walk.first + n - h * tiles;
          if (!mbar_wait(smem_u32(&sh.empty[stage]), ((n / GRAD_STAGES) & 1) ^ 1, dead)) break;
          const bool cut = walk.cut(t);
          // (at most four tiles are under way, so the fourth cut tile before this one is done with)
          const uint32_t bar = smem_u32(cut ? &sh.cut_full[cuts % 4] : &sh.full[stage]), dst = ring + stage * 2 * Y;
          if (cut) {
            mbar_arrive(smem_u32(&sh.full[stage]));
            ++cuts;
          }
          mbar_arrive_expect(bar, 2 * Y);
          const int y_head = KEYS ? head * p.group + h : head / p.group;
          for (int i = 0; i < 2; ++i)
            for (int x = 0; x < BLOCKS; ++x)
              tile_load(dst + i * Y + x * Y_BLOCK, KEYS ? (i ? &p.g : &p.q) : (i ? &p.v : &p.k), x * 64, y_head, y_first + t * YT, bar);
        }
      }
    } else if (warp == 9) {
      if (elected()) {
        const int steps = (p.dim + 15) / 16;
        const uint32_t kind_t = tile_kind(p.bf, YT, false), kind_a = tile_kind(p.bf, steps * 16, true);
        const uint64_t rows = tile_operand(0, 16, 1024), lines = tile_operand(0, Y_BLOCK, 1024);
        bool ok = all == 0 || mbar_wait(smem_u32(KEYS ? &sh.x_full : &sh.x_there), 0, dead);
        tmem_after();
        int cuts = 0;
        const auto products = [&](int n) {  // T1 and T2 of tile n
          const int stage = n % GRAD_STAGES, h = n / tiles, t = walk.first + n - h * tiles;
          if (walk.cut(t)) {
            ok = ok && mbar_wait(smem_u32(&sh.clean[cuts % 4]), (cuts / 4) & 1, dead);
            ++cuts;
          } else {
            ok = ok && mbar_wait(smem_u32(&sh.full[stage]), (n / GRAD_STAGES) & 1, dead);
          }
          if (!ok) return;
          for (int i = 0; i < 2; ++i) {
            const uint64_t a = rows + ((base + i * X) >> 4), b = rows + ((ring + (stage * 2 + i) * Y) >> 4);
            for (int s = 0; s < steps; ++s) {
              const uint32_t d = tmem + i * 128 + (n & 1) * YT;
              const uint64_t y = b + (((s >> 2) * Y_BLOCK + (s & 3) * 32) >> 4);
              if (KEYS) mma_shared(d, a + (((s >> 2) * X_BLOCK + (s & 3) * 32) >> 4), y, kind_t, s != 0);
              else mma_tensor(d, tmem + 384 + i * 64 + s * 8, y, kind_t, s != 0);
            }
          }
          mma_arrive(smem_u32(&sh.products[n & 1]));
        };
        for (int n = 0; n < 2 && n < all; ++n) products(n);
        for (int n = 0; n < all && ok; ++n) {
          ok = mbar_wait(smem_u32(&sh.weights[n & 1]), (n >> 1) & 1, dead);
          if (!ok) break;
          tmem_after();
          const int stage = n % GRAD_STAGES;
          const uint64_t y1 = lines + ((ring + stage * 2 * Y) >> 4);
          for (int s = 0; s < 2 * YT / 16; ++s)  // both pieces of ds
            mma_tensor(tmem + 256, tmem + 128 + (n & 1) * YT + s * 8, y1 + (s % (YT / 16)) * (2048 >> 4), kind_a, n != 0 || s != 0);
          if (KEYS) {
            const uint64_t y2 = y1 + (Y >> 4);
            for (int s = 0; s < YT / 16; ++s) mma_tensor(tmem + 384, tmem + (n & 1) * YT + s * 8, y2 + s * (2048 >> 4), kind_a, n != 0 || s != 0);
          }
          mma_arrive(smem_u32(&sh.empty[stage]));
          if (n + 2 < all) products(n + 2);
        }
        mma_arrive(smem_u32(&sh.done));
      }
    } else {
      // Cut tiles: a thread a row.  Rows behind the sequence become 0 where they are summed over (0 times a neighbour's infinity would be
      // NaN), and so do values of Y1 that are not finite: rows that see them have an lse that is NaN.
      const int row = threadIdx.x - 10 * 32;
      int cuts = 0;
      for (int n = 0; n < all; ++n) {
        const int stage = n % GRAD_STAGES, h = n / tiles, t = walk.first + n - h * tiles;
        if (!walk.cut(t)) continue;
        if (!mbar_wait(smem_u32(&sh.cut_full[cuts % 4]), (cuts / 4) & 1, dead)) break;
        uint8_t* const tile = raw_smem + (ring - smem_u32(raw_smem)) + stage * 2 * Y;
        const bool behind = t * YT + row >= y_count;
        for (int x = 0; x < BLOCKS; ++x) {
#pragma unroll
          for (int piece = 0; piece < 8; ++piece) {
            uint4* const at = reinterpret_cast<uint4*>(tile + x * Y_BLOCK + swizzled(row, piece));
            if (behind) {
              *at = make_uint4(0u, 0u, 0u, 0u);
              if (KEYS) *reinterpret_cast<uint4*>(reinterpret_cast<uint8_t*>(at) + Y) = make_uint4(0u, 0u, 0u, 0u);
            } else if (p.causal) {
              uint4 v = *at;
              uint32_t* const u = &v.x;
              constexpr uint32_t EXP = std::is_same<T, __nv_bfloat16>::value ? 0x7F80u : 0x7C00u;
              bool here = false;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                if ((u[e] & EXP) == EXP) u[e] &= 0xFFFF0000u, here = true;
                if ((u[e] & (EXP << 16)) == EXP << 16) u[e] &= 0x0000FFFFu, here = true;
              }
              if (here) *at = v;
            }
          }
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        mbar_arrive(smem_u32(&sh.clean[cuts % 4]));
        ++cuts;
      }
    }
    return;
  }

  asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
  const int w = warp >> 2, thread = threadIdx.x & 127, x = x0 + thread;  // the thread's row of X
  const uint32_t lanes = (uint32_t)(warp & 3) << 21, t1 = tmem + w * YT + lanes, t2 = t1 + 128;
  const u64 c = both(p.to_log2);
  const int bits = ds_bits(p);
  const u64 up = both(power_of_two(bits - P_BITS));  // of ds, beside the 2^8 of p
  bool ok = true;
  float2 mine = make_float2(0.0f, 0.0f);  // queries: this row's; keys: a column's of the next tile
  const auto stats_of = [&](int n) {
    const int h = n / max(tiles, 1), i = (walk.first + n - h * tiles) * YT + thread;
    mine = make_float2(0.0f, 0.0f);
    if (n < all && thread < YT && i < y_count) mine = __ldg(p.stats + (int64_t)(head * p.group + h) * p.q_rows + y_first + i);
  };
  if (!KEYS) {  // this warpgroup's operand of all first products: a row a thread, in tensor memory beside the sums
    const T* const row = w ? static_cast<const T*>(p.g_raw) + ((int64_t)(x_first + x) * p.heads + head) * p.dim
                           : static_cast<const T*>(p.q_raw) + (int64_t)(x_first + x) * p.q_at.token + head * p.q_at.head;
    for (int d = 0; d < p.dim; d += 32) {
      uint32_t v[16];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint4 four = x < x_count && d + 8 * e < p.dim ? __ldg(reinterpret_cast<const uint4*>(row + d + 8 * e)) : make_uint4(0u, 0u, 0u, 0u);
        v[4 * e] = four.x, v[4 * e + 1] = four.y, v[4 * e + 2] = four.z, v[4 * e + 3] = four.w;
      }
      __syncwarp();
      tmem_st16(tmem + 384 + w * 64 + lanes + d / 2, v);
    }
    tmem_wait_st();
    tmem_before();
    mbar_arrive(smem_u32(&sh.x_there));
  }
  if (KEYS) stats_of(w);
  else if (x < x_count) mine = __ldg(p.stats + (int64_t)head * p.q_rows + x_first + x);
  for (int n = w; n < all; n += 2) {
    if (KEYS) {  // the columns' statistics; the warpgroup's own, so the barrier is its own too
      asm volatile("bar.sync %0, 128;" ::"r"(1 + w) : "memory");
      if (thread < YT) sh.stats[w][thread] = make_float2(mine.x - P_BITS, mine.y);
      asm volatile("bar.sync %0, 128;" ::"r"(1 + w) : "memory");
      stats_of(n + 2);
    }
    ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.products[w]), (n >> 1) & 1, dead));
    if (!ok) continue;  // (the warpgroup's other warps wait at its barrier)
    tmem_after();
    const int t = walk.first + n % tiles;
    int lo = 0, hi = YT;  // columns that the row goes with
    if (walk.cut(t)) {
      if (KEYS) {
        hi = y_count - t * YT;
        if (p.causal) lo = x - off - t * YT;
      } else {
        hi = (p.causal ? min(y_count, x + off + 1) : y_count) - t * YT;
      }
    }
    const bool masked = walk.cut(t);
    uint32_t s[YT], dp[YT];
#pragma unroll
    for (int half = 0; half < YT; half += 32) {
      tmem_load32(t1 + half, s + half);
      tmem_load32(t2 + half, dp + half);
    }
    tmem_wait_ld();
#pragma unroll
    for (int half = 0; half < YT; half += 32) {
      uint32_t pw[16], dw[16], low[16];
#pragma unroll
      for (int e = half; e < half + 32; e += 2) {
        u64 minus, delta;
        if (KEYS) {
          const float4 st = *reinterpret_cast<const float4*>(&sh.stats[w][e]);
          minus = pack2(-st.x, -st.z);
          delta = pack2(-st.y, -st.w);
        } else {
          minus = both(P_BITS - mine.x);
          delta = both(-mine.y);
        }
        float p0, p1;
        unpack2(fma2_rn(pack2u(s[e], s[e + 1]), c, minus), p0, p1);
        p0 = exp2_approx(p0);
        p1 = exp2_approx(p1);
        float d0, d1;
        unpack2(mul2_rn(mul2_rn(add2_rn(pack2u(dp[e], dp[e + 1]), delta), up), pack2(p0, p1)), d0, d1);
        if (masked) {
          if (e < lo || e >= hi) p0 = d0 = 0.0f;
          if (e + 1 < lo || e + 1 >= hi) p1 = d1 = 0.0f;
        }
        const int at = (e - half) / 2;
        if (KEYS) pw[at] = pack_pair<T>(p0, p1);
        dw[at] = pack_pair<T>(d0, d1);
        const float2 held = pair_values<T>(dw[at]);
        low[at] = pack_pair<T>(d0 - held.x, d1 - held.y);
      }
      // over columns that have been read: p's 32, ds' first pieces' 32 and second pieces' 32
      if (KEYS) tmem_st16(t1 + half / 2, pw);
      tmem_st16(t2 + half / 2, dw);
      tmem_st16(t2 + YT / 2 + half / 2, low);
    }
    tmem_wait_st();
    tmem_before();
    mbar_arrive(smem_u32(&sh.weights[w]));
  }
  // both warpgroups bring the sums out, each half of the columns
  ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.done), 0, dead)) && ok && !*dead;
  tmem_after();
  const bool there = x < x_count;
  const int out_heads = KEYS ? p.kv_heads : p.heads;
  const int64_t at = ((int64_t)(x_first + x) * out_heads + head) * p.dim;
  const float by1 = p.scale * power_of_two(-bits), by2 = 1.0f / P_UP;
#pragma unroll 1
  for (int which = 0; which < (KEYS ? 2 : 1); ++which) {
    T* const dst = static_cast<T*>(KEYS ? (which ? p.grad_v : p.grad_k) : p.grad_q) + at;
    const float by = which ? by2 : by1;
#pragma unroll 1
    for (int d = w * (DT / 2); d < (w + 1) * (DT / 2) && d < p.dim; d += 32) {
      uint32_t o[32];
      __syncwarp();
      if (all) {
        tmem_load32(tmem + 256 + which * 128 + lanes + d, o);
        tmem_wait_ld();
      }
      if (!there) continue;
#pragma unroll
      for (int e = 0; e < 32; e += 8) {
        if (d + e >= p.dim) break;
        uint32_t v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          float lo = all ? __uint_as_float(o[e + 2 * u]) * by : 0.0f, hi = all ? __uint_as_float(o[e + 2 * u + 1]) * by : 0.0f;
          if (!ok) lo = hi = __uint_as_float(0x7FC00000u);
          v[u] = pack_pair<T>(lo, hi);
        }
        *reinterpret_cast<uint4*>(dst + d + e) = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
  }
  tmem_before();
}

template <typename T, int DT>
__global__ void __launch_bounds__(GRAD_THREADS, 1) attention_grad_kernel(const __grid_constant__ GradParams p) {
  extern __shared__ uint8_t raw_smem[];
  __shared__ GradShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(raw_smem) + 1023) & ~1023u;
  if (threadIdx.x == 0) {
    mbar_init(smem_u32(&sh.x_full), 1);
    mbar_init(smem_u32(&sh.x_there), 256);
    mbar_init(smem_u32(&sh.done), 1);
    for (int i = 0; i < GRAD_STAGES; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 4; ++i) {
      mbar_init(smem_u32(&sh.cut_full[i]), 1);
      mbar_init(smem_u32(&sh.clean[i]), 64);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.products[i]), 1);
      mbar_init(smem_u32(&sh.weights[i]), 128);
    }
    mbar_init_fence();
    sh.dead = 0;
  }
  after_previous();
  if (warp == 9) tmem_alloc(smem_u32(&sh.tmem), 512);
  const bool keys = (int64_t)blockIdx.x < p.key_blocks;
  const int64_t index = keys ? blockIdx.x : blockIdx.x - p.key_blocks;
  const int heads = keys ? p.kv_heads : p.heads, head = (int)(index % heads);
  if (warp == 8) {
    int seq = 0, block = 0;
    const bool found = find_block(keys ? p.cu_k : p.cu_q, keys ? p.k_rows : p.q_rows, p.sequences, XT, index / heads, &seq, &block);
    if (lane == 0) {
      sh.found = found;
      sh.seq = seq;
      sh.block = block;
    }
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = sh.tmem;
  const bool found = sh.found != 0;
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

size_t stats_bytes(const lba_attention_how* h) { return (size_t)h->heads * h->q_rows * sizeof(float2); }

}  // namespace
}  // namespace lba

using namespace lba;

extern "C" {

size_t lba_attention_backward_workspace_bytes(const lba_attention_how* how) {
  return check_attention(how) == LBA_OK && how->sequences ? 256 + stats_bytes(how) : 0;
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
  p.q_raw = q;
  p.g_raw = grad_out;
  p.q_at = how->q_at;
  const lba_strides g_at = {(int64_t)how->heads * how->dim, how->dim};
  if (!head_map(&p.q, p.bf, q, how->q_rows, how->heads, how->dim, how->q_at, YT) || !head_map(&p.g, p.bf, grad_out, how->q_rows, how->heads, how->dim, g_at, YT) ||
      !head_map(&p.k, p.bf, k, how->k_rows, how->kv_heads, how->dim, how->k_at, YT) ||
      !head_map(&p.v, p.bf, v, how->k_rows, how->kv_heads, how->dim, how->v_at, YT))
    return cuda_fail(cudaErrorInvalidValue);
  uint32_t* const most = p.bf ? nullptr : static_cast<uint32_t*>(workspace);
  float2* const stats = reinterpret_cast<float2*>(static_cast<uint8_t*>(workspace) + 256);
  DeltaParams d = {};
  d.g = grad_out;
  d.out = out;
  d.v = v;
  d.v_at = how->v_at;
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
  d.most = most;
  d.grad_q = p.grad_q = grad_q;
  d.grad_k = p.grad_k = grad_k;
  d.grad_v = p.grad_v = grad_v;
  p.stats = stats;
  p.most = most;
  p.group = how->heads / how->kv_heads;
  p.causal = how->causal != 0;
  p.to_log2 = how->scale * LOG2E;
  p.scale = how->scale;
  p.key_blocks = (how->k_rows / XT + how->sequences) * how->kv_heads;
  const int64_t blocks = p.key_blocks + (how->q_rows / XT + how->sequences) * how->heads;
  const int64_t vectors = how->q_rows * how->heads > how->k_rows * how->kv_heads ? how->q_rows * how->heads : how->k_rows * how->kv_heads;
  const int64_t delta_blocks = (vectors + DELTA_THREADS / 16 - 1) / (DELTA_THREADS / 16);
  if (delta_blocks > 2147483647LL || blocks > 2147483647LL) return LBA_ERR_SHAPE;
  cudaError_t e = most ? cudaMemsetAsync(most, 0, 8, s) : cudaSuccess;
  if (e != cudaSuccess) return status_of(e);
  e = p.bf ? launch_after(attention_delta_kernel<__nv_bfloat16>, dim3((unsigned)delta_blocks), DELTA_THREADS, 0, s, d)
           : launch_after(attention_delta_kernel<__half>, dim3((unsigned)delta_blocks), DELTA_THREADS, 0, s, d);
  if (e != cudaSuccess) return status_of(e);
  if (how->dim <= 64) return status_of(p.bf ? launch_grad<__nv_bfloat16, 64>(p, blocks, s) : launch_grad<__half, 64>(p, blocks, s));
  return status_of(p.bf ? launch_grad<__nv_bfloat16, 128>(p, blocks, s) : launch_grad<__half, 128>(p, blocks, s));
}

}  // extern "C"
