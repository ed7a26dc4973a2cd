// Attention over whole prompts: out[i] = sum_j softmax_j(scale q[i] k[j]) v[j] for packed sequences, causal or not, grouped heads.
//
// One pass over the keys with the running maximum and sum of a softmax; scores and weights never leave the SM.  Bound by the tensor cores
// and the exponential units together: 128 x 128 scores of 128 dimensions are 1024 clocks of matrix instructions (two products) and 1024 clocks of
// exponentials (16 a clock).  So an SM holds two tiles of 128 queries: while the tensor cores work on one tile's products, a warpgroup forms the
// other's weights.  The tiles are two of one head in one CTA, which share their keys' copies (W = 2), or two CTAs with a tile each, whose
// starts and ends hide behind each other (W = 1; for 128 dimensions they have room for one K and one V tile each).
//   4 warps a tile   its softmax, a query row a thread: scores from tensor memory to registers, weights back over them as the second
//                    product's operand; its output stays in tensor memory to the end.  The maximum that weights are relative to is raised only
//                    when a score exceeds it by 2^8, and the output is rescaled only then (in 32 bits nothing is lost by weights of up to 256)
//   a warp           tensor copies of K and V tiles into a ring
//   a warp           one thread issues all products
//   two warps        clean tiles of V that the mask cuts: rows behind the sequence become 0 (0 times a neighbour's infinity would be NaN),
//                    and values that are not finite, which rows before them must not see, are taken out and added to the others' results
// A prompt of 8192 tokens, 32 heads of 128, takes 530 us in a steady run, under the power limit (1.04 PFLOP/s), and 461 us in a burst
// (1.19, 70% of the matrix peak);
// short sequences are bound by what a CTA does once: some 9 us for its place, its first copies and products, and its rows' way out.
// Weights are rounded to the inputs' type (2^-9 or 2^-12 of each, at random; the result is rounded to that type once more); sums of weights
// are of the unrounded ones.  binary16 has few exponents: weights are held 2^7 above the maximum's, so that with the 2^8 by which a score may exceed it
// they end at 2^15, and those below 2^-21 of the maximum's have fewer bits, those below 2^-32 none.
#include <cmath>

#include "lba_tile.cuh"

namespace lba {
namespace {

constexpr int QT = 128, KT = 128, MAX_STAGES = 10, CUT_TILES = 4;
constexpr float LAZY = 8.0f;  // binades
// binades that weights are held above the maximum's, and what takes them from their sum
template <typename T> constexpr float kUp = std::is_same<T, __half>::value ? 7.0f : 0.0f;
template <typename T> constexpr float kDown = std::is_same<T, __half>::value ? 0x1p-7f : 1.0f;

struct ForwardParams {
  CUtensorMap q, k, v;
  const int32_t *cu_q, *cu_k;
  int64_t q_rows, k_rows;
  int sequences, heads, group, dim, causal, bf, in_m4e3, codes;
  float to_log2;             // scale log2(e)
  const float* out_scale;
  const void* v_raw;
  lba_strides v_at;
  void* out;
  float* lse;
};

template <int DT> constexpr int kTile = 128 * DT * 2;                       // bytes of a tile of 128 rows
template <int DT, int W> constexpr int kStages = W == 1 ? (DT == 128 ? 2 : 5) : (DT == 128 ? 5 : 10);
template <int DT, int W> constexpr size_t kForwardSmem = 1024 + (size_t)kTile<DT> * (W + kStages<DT, W>);

struct ForwardShared {
  uint64_t q_full[2], full[MAX_STAGES], empty[MAX_STAGES], scores[2], weights[2][2], done;  // weights: of the first 96 keys of a tile, of the others
  uint64_t cut_full[CUT_TILES], clean[CUT_TILES];  // copies of V that the mask cuts, and their cleaning: once each
  uint32_t cut[CUT_TILES][4];  // rows of the masked tiles of V that hold values that are not finite
  uint32_t tmem;
  int dead;
  Place place;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}
// weights of 32 scores, relative to the maximum: packed, and their sum.  (A quarter of the exponentials as polynomials on the FMA units was slower:
// a prompt of 8192 took 540 us instead of 520 in a steady run, 481 instead of 461 in a burst.)
template <typename T>
__device__ __forceinline__ void weigh32(const uint32_t* s, uint32_t* out, u64 by, u64 minus, u64 (&sum)[4]) {
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    float lo, hi;
    unpack2(fma2_rn(pack2u(s[i], s[i + 1]), by, minus), lo, hi);
    lo = exp2_approx(lo);
    hi = exp2_approx(hi);
    sum[i / 2 % 4] = add2_rn(sum[i / 2 % 4], pack2(lo, hi));
    out[i / 2] = pack_pair<T>(lo, hi);
  }
}

// Codes of quotients, nearest and saturated as encode_e4m3 and encode_m4e3 of the rounded quotient.  Both ends of an interval around v times the
// reciprocal that holds the quotient have the same code almost always, codes being monotone; only else is there a division (which branches, and
// took 117 clocks an element).
struct Quotients {
  float scale, low, high;  // reciprocals less and plus 2^-21 of themselves; 0 where they have no such precision
  __device__ __forceinline__ explicit Quotients(float s) : scale(s) {
    const bool normal = s > 0x1p-100f && s < 0x1p100f;
    const float r = normal ? 1.0f / s : 0.0f;
    low = r * (1.0f - 0x1p-21f);
    high = r * (1.0f + 0x1p-21f);
  }
  __device__ __forceinline__ static uint32_t four(float a, float b, float c, float d, bool m4e3) {
    if (m4e3) return encode_m4e3(a) | (uint32_t)encode_m4e3(b) << 8 | (uint32_t)encode_m4e3(c) << 16 | (uint32_t)encode_m4e3(d) << 24;
    uint32_t x;
    asm("{\n\t.reg .b16 l, h;\n\tcvt.rn.satfinite.e4m3x2.f32 l, %2, %1;\n\tcvt.rn.satfinite.e4m3x2.f32 h, %4, %3;\n\tmov.b32 %0, {l, h};\n\t}"
        : "=r"(x) : "f"(a), "f"(b), "f"(c), "f"(d));
    return x;
  }
  __device__ __noinline__ static uint32_t divided(float a, float b, float c, float d, float s, bool m4e3) {
    return four(__fdiv_rn(a, s), __fdiv_rn(b, s), __fdiv_rn(c, s), __fdiv_rn(d, s), m4e3);
  }
  __device__ __forceinline__ uint32_t codes(const float4& v, bool m4e3) const {
    const uint32_t x = four(v.x * low, v.y * low, v.z * low, v.w * low, m4e3), y = four(v.x * high, v.y * high, v.z * high, v.w * high, m4e3);
    return x == y && low != 0.0f ? x : divided(v.x, v.y, v.z, v.w, scale, m4e3);
  }
};

// W: tiles of queries of a CTA
template <typename T, int DT, int W>
__global__ void __launch_bounds__(128 * (W + 1), 3 - W) attention_kernel(const __grid_constant__ ForwardParams p) {
  constexpr int BLOCKS = DT / 64, TILE = kTile<DT>, HALF = 128 * 128, STAGES = kStages<DT, W>, COLUMNS = 256 * W;
  constexpr int COPIES = 4 * W, PRODUCTS = COPIES + 1, CLEAN = COPIES + 2;  // warps
  extern __shared__ uint8_t raw_smem[];
  __shared__ ForwardShared sh;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t base = (smem_u32(raw_smem) + 1023) & ~1023u, q_smem = base, ring = base + W * TILE;
  volatile int* const dead = &sh.dead;

  const int head = blockIdx.x % p.heads;
  if (warp == COPIES && lane == 0) {
    map_ahead(&p.q);
    map_ahead(&p.k);
    map_ahead(&p.v);
  }
  if (warp == 0) {
    if (lane == 0) {
      for (int i = 0; i < W; ++i) {
        mbar_init(smem_u32(&sh.q_full[i]), 1);
        mbar_init(smem_u32(&sh.scores[i]), 1);
        mbar_init(smem_u32(&sh.weights[i][0]), 128);
        mbar_init(smem_u32(&sh.weights[i][1]), 128);
      }
      for (int i = 0; i < STAGES; ++i) {
        mbar_init(smem_u32(&sh.full[i]), 1);
        mbar_init(smem_u32(&sh.empty[i]), 1);
      }
      for (int i = 0; i < CUT_TILES; ++i) {
        mbar_init(smem_u32(&sh.cut_full[i]), 1);
        mbar_init(smem_u32(&sh.clean[i]), 64);
      }
      mbar_init(smem_u32(&sh.done), 1);
      mbar_init_fence();
      for (int i = 0; i < CUT_TILES * 4; ++i) sh.cut[i / 4][i % 4] = 0;
      sh.dead = 0;
    }
  }
  after_previous();
  if (warp == PRODUCTS) tmem_alloc(smem_u32(&sh.tmem), COLUMNS);  // (not before: a CTA of the kernel before this one could still want it)
  if (warp == COPIES) {
    const Place place = find_place(p.cu_q, p.q_rows, p.cu_k, p.k_rows, p.sequences, false, W * QT, blockIdx.x / p.heads);
    if (lane == 0) sh.place = place;
  }
  tmem_before();
  __syncthreads();
  tmem_after();
  const uint32_t tmem = sh.tmem;
  const Place place = sh.place;
  const bool alive = place.found != 0;
  if (alive) {
    // (with a causal mask the last blocks, which have the most keys, are of the highest levels)
    const int q_first = place.q_first, q_count = place.q_count, k_first = place.k_first, k_count = place.k_count, off = k_count - q_count, block = place.level;
    const int i0 = block * W * QT;
    // tiles of keys of either query tile, and the first that a mask cuts
    int tiles[W], whole[W];
#pragma unroll
    for (int w = 0; w < W; ++w) {
      const int lo = i0 + w * QT, hi = min(lo + QT, q_count) - 1;
      const int keys = lo >= q_count ? 0 : p.causal ? max(0, min(k_count, hi + off + 1)) : k_count;
      tiles[w] = (keys + KT - 1) / KT;
      whole[w] = (p.causal ? max(0, min(k_count, lo + off + 1)) : k_count) / KT;
    }
    const int all = max(tiles[0], tiles[W - 1]);
    // the first tile of V to be cleaned: behind it, masks cut every tile of some query tile that is not empty
    const int dirty = min(tiles[0] ? whole[0] : all, tiles[W - 1] ? whole[W - 1] : all);
    const int kv = head / p.group;

    if (warp >= COPIES) {
      // (168 or 128 registers a thread are there from the launch; the softmax threads take 208 or 192)
      if constexpr (W == 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
      else asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
      if (warp == COPIES) {
        if (elected()) {
#pragma unroll
          for (int w = 0; w < W; ++w) {
            if (!tiles[w]) continue;
            mbar_arrive_expect(smem_u32(&sh.q_full[w]), TILE);
            for (int x = 0; x < BLOCKS; ++x) tile_load(q_smem + w * TILE + x * HALF, &p.q, x * 64, head, q_first + i0 + w * QT, smem_u32(&sh.q_full[w]));
          }
          int stage = 0;
          uint32_t phase = 1;
          for (int n = 0; n < 2 * all; ++n) {  // K and V of a tile in turn
            if (!mbar_wait(smem_u32(&sh.empty[stage]), phase, dead)) break;
            const bool cut = (n & 1) && (n >> 1) >= dirty;
            const uint32_t dst = ring + stage * TILE, bar = smem_u32(cut ? &sh.cut_full[(n >> 1) - dirty] : &sh.full[stage]);
            if (cut) mbar_arrive(smem_u32(&sh.full[stage]));  // (its phases count copies; those who want this one wait for its own barriers)
            mbar_arrive_expect(bar, TILE);
            for (int x = 0; x < BLOCKS; ++x) tile_load(dst + x * HALF, n & 1 ? &p.v : &p.k, x * 64, kv, k_first + (n >> 1) * KT, bar);
            if (++stage == STAGES) {
              stage = 0;
              phase ^= 1;
            }
          }
        }
      } else if (warp == PRODUCTS) {
        if (elected()) {
          const int steps = (p.dim + 15) / 16;
          const uint32_t kind_s = tile_kind(p.bf, KT, false), kind_o = tile_kind(p.bf, steps * 16, true);
          const uint64_t rows = tile_operand(0, 16, 1024), lines = tile_operand(0, HALF, 1024);
          bool ok = true;
          // K of tile j is copy 2 j, V 2 j + 1
          const auto full = [&](int copy) { ok = ok && mbar_wait(smem_u32(&sh.full[copy % STAGES]), (copy / STAGES) & 1, dead); };
          const auto scores = [&](int w, int j) {
            full(2 * j);
            if (!ok) return;
            const uint64_t a = rows + ((q_smem + w * TILE) >> 4), b = rows + ((ring + (2 * j % STAGES) * TILE) >> 4);
#pragma unroll
            for (int s = 0; s < DT / 16; ++s) {
              if (s >= steps) break;
              const int at = ((s >> 2) * HALF + (s & 3) * 32) >> 4;
              mma_shared(tmem + w * KT, a + at, b + at, kind_s, s != 0);
            }
            mma_arrive(smem_u32(&sh.scores[w]));
          };
#pragma unroll
          for (int w = 0; w < W; ++w) {
            if (!tiles[w]) continue;
            ok = ok && mbar_wait(smem_u32(&sh.q_full[w]), 0, dead);
            scores(w, 0);
          }
          if (ok && all) mma_arrive(smem_u32(&sh.empty[0]));
          for (int j = 0; j < all && ok; ++j) {
            const int vs = (2 * j + 1) % STAGES;
            if (j >= dirty) ok = ok && mbar_wait(smem_u32(&sh.clean[j - dirty]), 0, dead);
            else full(2 * j + 1);
#pragma unroll
            for (int w = 0; w < W; ++w) {
              if (j >= tiles[w]) continue;
              const uint64_t b = lines + ((ring + vs * TILE) >> 4);
#pragma unroll
              for (int s = 0; s < KT / 16; ++s) {
                if (s == 0 || s == 6) {
                  ok = ok && mbar_wait(smem_u32(&sh.weights[w][s / 6]), j & 1, dead);
                  if (!ok) break;
                  tmem_after();
                }
                mma_tensor(tmem + (W + w) * 128, tmem + w * KT + s * 8, b + s * (2048 >> 4), kind_o, j != 0 || s != 0);
              }
              if (!ok) break;
              if (j + 1 < tiles[w]) scores(w, j + 1);
              else mma_arrive(smem_u32(&sh.scores[w]));  // the output is complete
            }
            if (ok) {
              mma_arrive(smem_u32(&sh.empty[vs]));
              if (j + 1 < all) mma_arrive(smem_u32(&sh.empty[(2 * j + 2) % STAGES]));
            }
          }
          mma_arrive(smem_u32(&sh.done));
        }
      } else {
        for (int j = dirty; j < all; ++j) {
          const int stage = (2 * j + 1) % STAGES;
          if (!mbar_wait(smem_u32(&sh.cut_full[j - dirty]), 0, dead)) break;
          uint8_t* const tile = raw_smem + (ring - smem_u32(raw_smem)) + stage * TILE;
          for (int row = threadIdx.x - CLEAN * 32; row < KT; row += 64) {
            bool odd = false;
            if (j * KT + row >= k_count) clear_row<BLOCKS>(tile, row);
            else if (p.causal) odd = keep_finite<T, BLOCKS>(tile, row);
            if (odd) atomicOr(&sh.cut[j - dirty][row >> 5], 1u << (row & 31));
          }
          asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
          mbar_arrive(smem_u32(&sh.clean[j - dirty]));
        }
      }
    } else {
      if constexpr (W == 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
      else asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
      const int w = warp >> 2, mine = tiles[w], row = threadIdx.x & 127, i = i0 + w * QT + row;
      const uint32_t lanes = (uint32_t)(warp & 3) << 21, s_at = tmem + w * KT + lanes, o_at = tmem + (W + w) * 128 + lanes;
      const float c = p.to_log2, out_scale = p.codes ? __ldg(p.out_scale) : 1.0f;  // (fetched here: at the end every block would wait for it)
      const bool there = i < q_count;
      float top = there ? -INFINITY : INFINITY;  // (rows behind the sequence, the next one's, never raise: bits do not depend on what is packed beside it)
      u64 total[4] = {};  // chains of their own
      bool ok = true;
      for (int j = 0; j < mine; ++j) {
        ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.scores[w]), j & 1, dead));
        if (!ok) break;
        tmem_after();
        uint32_t s[KT];
#pragma unroll
        for (int x = 0; x < KT; x += 32) tmem_load32(s_at + x, s + x);
        tmem_wait_ld();
        if (j >= whole[w]) {
          const int limit = (p.causal ? min(k_count, i + off + 1) : k_count) - j * KT;  // keys of this tile that the row sees
#pragma unroll
          for (int x = 0; x < KT; ++x)
            if (x >= limit) s[x] = 0xFF800000u;
        }
        // (three operands an instruction, eight chains: one chain of 127 took 450 clocks)
        float top8[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) top8[x] = __uint_as_float(s[x]);
#pragma unroll
        for (int x = 8; x < KT; x += 16) {
#pragma unroll
          for (int e = 0; e < 8; ++e) top8[e] = x + 8 + e < KT ? max3(top8[e], __uint_as_float(s[x + e]), __uint_as_float(s[x + 8 + e])) : fmaxf(top8[e], __uint_as_float(s[x + e]));
        }
        const float most = max3(max3(top8[0], top8[1], top8[2]), max3(top8[3], top8[4], top8[5]), fmaxf(top8[6], top8[7]));
        const bool raise = most * c > top * c + LAZY;  // (true whenever there is no maximum yet, and some score)
        if (__any_sync(0xFFFFFFFFu, raise)) {
          const float next = fmaxf(top, most);
          if (j > 0) {
            const float by = next == -INFINITY ? 1.0f : exp2_approx((top - next) * c);
            const u64 by2 = both(by);
#pragma unroll
            for (int x = 0; x < 4; ++x) total[x] = mul2_rn(total[x], by2);
            for (int x = 0; x < p.dim; x += 32) {
              uint32_t o[32];
              tmem_load32(o_at + x, o);
              tmem_wait_ld();
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * by);
              tmem_store32(o_at + x, o);
            }
          }
          top = next;
        }
        const u64 by = both(c), minus = both(top == -INFINITY ? 0.0f : kUp<T> - top * c);
        uint32_t packed[KT / 2];
        // (the first products start while the last quarter is formed)
#pragma unroll
        for (int x = 0; x < 96; x += 32) weigh32<T>(s + x, packed + x / 2, by, minus, total);
        tmem_store32(s_at, packed);
        tmem_st16(s_at + 32, *reinterpret_cast<const uint32_t(*)[16]>(packed + 32));
        tmem_wait_st();
        tmem_before();
        mbar_arrive(smem_u32(&sh.weights[w][0]));
        weigh32<T>(s + 96, packed + 48, by, minus, total);
        tmem_st16(s_at + 48, *reinterpret_cast<const uint32_t(*)[16]>(packed + 48));
        tmem_wait_st();
        tmem_before();
        mbar_arrive(smem_u32(&sh.weights[w][1]));
      }
      if (mine && ok) ok = __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(&sh.scores[w]), mine & 1, dead));
      tmem_after();
      float lo, hi;
      unpack2(add2_rn(add2_rn(total[0], total[1]), add2_rn(total[2], total[3])), lo, hi);
      const float sum = lo + hi;
      if (there && p.lse)
        p.lse[(int64_t)head * p.q_rows + q_first + i] =
            !ok ? __uint_as_float(0x7FC00000u) : sum == 0.0f ? -INFINITY : (top * c + log2f(sum * kDown<T>)) * 0.69314718055994531f;
      const float inv = !ok ? __uint_as_float(0x7FC00000u) : sum == 0.0f ? 0.0f : __fdiv_rn(1.0f, sum);
      uint32_t poison = 0;  // of the cut tiles, as one word: any at all?
      if (p.causal) {
        for (int x = 0; x < CUT_TILES; ++x)
          for (int e = 0; e < 4; ++e) poison |= sh.cut[x][e];
      }
      const Quotients quotients(out_scale);
      // 32 values a row at a time go out through shared memory (the tile of Q is no longer read), four lanes a row side by side.  The code is kept
      // short: it runs once a CTA and is fetched as it runs (unrolled over a row's values, codes took 10000 clocks).
      uint8_t* const stage = raw_smem + (q_smem - smem_u32(raw_smem)) + w * TILE + (warp & 3) * 4096;
      const int rows = min(32, q_count - (i - lane));
#pragma unroll 1
      for (int x = 0; x < p.dim && rows > 0; x += 32) {
        uint32_t o[32];
        if (mine) {
          tmem_load32(o_at + x, o);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) o[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 32; e += 4)
          *reinterpret_cast<float4*>(stage + swizzled(lane, e / 4)) =
              make_float4(__uint_as_float(o[e]) * inv, __uint_as_float(o[e + 1]) * inv, __uint_as_float(o[e + 2]) * inv, __uint_as_float(o[e + 3]) * inv);
        if (poison && there) {
          for (int t = 0; t < CUT_TILES * 128; ++t) {
            const int key = dirty * KT + t;
            if (!((sh.cut[t >> 7][(t >> 5) & 3] >> (t & 31)) & 1u) || key > i + off) continue;
            const T* const src = static_cast<const T*>(p.v_raw) + (int64_t)(k_first + key) * p.v_at.token + kv * p.v_at.head + x;
#pragma unroll 1
            for (int e = 0; e < 32 && x + e < p.dim; ++e) {
              const float v = to_f32(src[e]);
              if (!isfinite(v)) *reinterpret_cast<float*>(stage + swizzled(lane, e >> 2) + (e & 3) * 4) += v;
            }
          }
        }
        __syncwarp();
        const int c = lane & 3, col = x + c * 8;
#pragma unroll
        for (int r = lane >> 2; r < 32; r += 8) {
          if (r >= rows || col >= p.dim) break;
          float4 a = *reinterpret_cast<const float4*>(stage + swizzled(r, 2 * c)), b = *reinterpret_cast<const float4*>(stage + swizzled(r, 2 * c + 1));
          if (!ok) a = b = make_float4(inv, inv, inv, inv);  // (a late copy of Q could still land here)
          const int64_t at = ((int64_t)(q_first + i - lane + r) * p.heads + head) * p.dim + col;
          if (p.codes) {
            *reinterpret_cast<uint2*>(static_cast<uint8_t*>(p.out) + at) = make_uint2(quotients.codes(a, p.in_m4e3), quotients.codes(b, p.in_m4e3));
          } else {
            *reinterpret_cast<uint4*>(static_cast<T*>(p.out) + at) = make_uint4(pack_pair<T>(a.x, a.y), pack_pair<T>(a.z, a.w), pack_pair<T>(b.x, b.y), pack_pair<T>(b.z, b.w));
          }
        }
        __syncwarp();
      }
      tmem_before();
    }
  }
  __syncthreads();
  if (warp == PRODUCTS) {
    if (*dead) {
      let_copies_land();
    } else if (alive) {
      mbar_wait(smem_u32(&sh.done), 0, dead);
    }
    tmem_after();
    __syncwarp();
    tmem_free(tmem, COLUMNS);
  }
}

template <typename T, int DT, int W>
cudaError_t launch_forward(const ForwardParams& p, cudaStream_t stream) {
  const cudaError_t e = cudaFuncSetAttribute(attention_kernel<T, DT, W>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kForwardSmem<DT, W>);
  if (e != cudaSuccess) return e;
  const int64_t blocks = (p.q_rows / (W * QT) + p.sequences) * p.heads;
  return launch_after(attention_kernel<T, DT, W>, dim3((unsigned)blocks), 128 * (W + 1), kForwardSmem<DT, W>, stream, p);
}
// One tile a CTA for short sequences: they leave fewer halves of a CTA empty, and start and end more often.  Longer ones want their keys copied
// once for two tiles, the more of 128 dimensions (those copies would come near what L2 can give).  A mask of the future halves a row's keys.
// One against two, us, bfloat16: 12 heads of 64, 32 x 128 tokens 13.6 19.4, 4 x 1024 33.2 36.7, 4 x 2048 97 92; causal, 4 x 2048 56.5 59.4,
// 8192 163 161.  32 heads of 128, 32 x 128 tokens 36 60, 12 x 384 53 71, 8 x 700 113 109; causal, 12 x 384 70 88, 24 of 1 to 1024 185 210, 4 x 1024
// 87 82.  16 heads of 80, causal, 7 of 1 to 2003: 45 52.
template <typename T>
cudaError_t launch_forward(const ForwardParams& p, cudaStream_t stream) {
  const int64_t limit = (p.dim <= 64 ? 1024 : 384) * (p.causal ? 2 : 1);
  const bool one = p.q_rows <= limit * p.sequences;
  if (p.dim <= 64) return one ? launch_forward<T, 64, 1>(p, stream) : launch_forward<T, 64, 2>(p, stream);
  return one ? launch_forward<T, 128, 1>(p, stream) : launch_forward<T, 128, 2>(p, stream);
}

}  // namespace

// what both passes ask of their arguments
int check_attention(const lba_attention_how* h) {
  if (!h) return LBA_ERR_NULL;
  if (!half_type(h->type) || !(h->scale > 0.0f) || !std::isfinite(h->scale)) return LBA_ERR_LAYER;
  if (h->heads < 1 || h->kv_heads < 1 || h->heads % h->kv_heads || h->heads > 65535 || h->dim < 8 || h->dim > 128 || h->dim % 8 || h->q_rows < 0 ||
      h->k_rows < 0 || h->q_rows > 2147483647LL - 1024 || h->k_rows > 2147483647LL - 1024 || h->sequences < 0)
    return LBA_ERR_SHAPE;
  if ((!h->cu_q || !h->cu_k) && h->sequences != 1) return LBA_ERR_SHAPE;
  const auto bad = [&](const lba_strides& s, int heads, int64_t rows) {  // tensor copies want strides of whole 16 bytes, below 2^40
    const auto off = [](int64_t v) { return v < 8 || v % 8 || v >= (1LL << 39); };
    return (heads > 1 && off(s.head)) || (rows > 1 && off(s.token));
  };
  if (bad(h->q_at, h->heads, h->q_rows) || bad(h->k_at, h->kv_heads, h->k_rows) || bad(h->v_at, h->kv_heads, h->k_rows)) return LBA_ERR_ALIGN;
  // a CTA for every block of rows of every sequence and head, sequences at most a block more than their rows fill
  if ((h->q_rows / 128 + h->k_rows / 128 + h->sequences + 2) > 2147483647LL / h->heads) return LBA_ERR_SHAPE;
  return LBA_OK;
}

}  // namespace lba

using namespace lba;

extern "C" int lba_attention(const void* q, const void* k, const void* v, const lba_attention_how* how, int out_type, const float* out_scale,
                             int out_flags, void* out, float* lse, void* stream) {
  const int st = check_attention(how);
  if (st != LBA_OK) return st;
  if ((out_type != how->type && out_type != LBA_TYPE_CODES) || (out_flags & ~LBA_FLAG_INPUT_M4E3)) return LBA_ERR_LAYER;
  if (how->q_rows == 0 || how->sequences == 0) return LBA_OK;
  if (!q || !out || (how->k_rows > 0 && (!k || !v)) || (out_type == LBA_TYPE_CODES && !out_scale)) return LBA_ERR_NULL;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out)) return LBA_ERR_ALIGN;
  ForwardParams p;
  p.bf = how->type == LBA_TYPE_BF16;
  // (without keys nothing is copied, but a map needs an address and a row)
  if (!head_map(&p.q, p.bf, q, how->q_rows, how->heads, how->dim, how->q_at, 128) ||
      !head_map(&p.k, p.bf, how->k_rows ? k : q, how->k_rows ? how->k_rows : 1, how->kv_heads, how->dim, how->k_rows ? how->k_at : how->q_at, 128) ||
      !head_map(&p.v, p.bf, how->k_rows ? v : q, how->k_rows ? how->k_rows : 1, how->kv_heads, how->dim, how->k_rows ? how->v_at : how->q_at, 128))
    return cuda_fail(cudaErrorInvalidValue);
  p.cu_q = how->cu_q;
  p.cu_k = how->cu_k;
  p.q_rows = how->q_rows;
  p.k_rows = how->k_rows;
  p.sequences = how->sequences;
  p.heads = how->heads;
  p.group = how->heads / how->kv_heads;
  p.dim = how->dim;
  p.causal = how->causal != 0;
  p.in_m4e3 = out_flags & LBA_FLAG_INPUT_M4E3;
  p.codes = out_type == LBA_TYPE_CODES;
  p.to_log2 = how->scale * LOG2E;
  p.out_scale = out_scale;
  p.v_raw = v;
  p.v_at = how->v_at;
  p.out = out;
  p.lse = lse;
  return status_of(p.bf ? launch_forward<__nv_bfloat16>(p, (cudaStream_t)stream) : launch_forward<__half>(p, (cudaStream_t)stream));
}
