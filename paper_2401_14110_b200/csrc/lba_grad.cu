// Backward pass of the linear and gated layers under the straight-through estimator: the quantisers pass the gradient, so
//
//   dz = drop(g) act'(z)                              linear
//   dz = g v act'(z), dv = g act(z)                   gated (z, v the two projections; both stand side by side below)
//   grad_a[m][k] = sum_n dz[m][n] sb[n] B[n][k]       grad_b[n][k] = sum_m dz[m][n] sa[m] A[m][k]       grad_bias[n] = sum_m dz[m][n]
//
// Nothing rounds between additions here, so the products run on the tensor cores.  Codes of either operand format have at most
// five significant bits: bfloat16 holds them exactly, and only dz is rounded.  One bfloat16 piece of it goes with bfloat16
// gradients (a rounding of 2^-9 beside the result's own), two with binary16 ones (2^-15 at most), three with binary32 ones (dz exactly); fewer
// where dz itself has no more bits (see pieces()).  Every piece costs one more pass of the matrix instruction.
//
// Scales that differ by row or column belong to the summed index of one of the products: dz is multiplied by both before it is
// rounded, and the other product divides its rows by the one that it does not want.  So both read the same pieces.
//
// Two launches:
//   grad_prepare_kernel   reads g and z once; writes the pieces of scaled dz, the sums of dz over blocks of rows (for the bias) and both
//                         operands' codes as bfloat16.  Bound by memory.
//   grad_product_kernel   both products as one list of 256 x 256 tiles, a pair of CTAs each (tcgen05, TMA), cut into equal shares of work;
//                         and the bias sums' last step.
#include "lba_grad.cuh"

#include "lba_async.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

constexpr int PREP_ROWS = 32, PREP_COLS = 256, PREP_THREADS = 256, PREP_EACH = PREP_ROWS * PREP_COLS / (8 * PREP_THREADS);
typedef __nv_bfloat16 bf16;

struct PrepParams {
  const void *grad, *pre;
  const uint8_t *A, *B, *B2;
  const float *sa, *sb, *sb2;  // factors of dz: by row; by column or by half (null: none)
  const uint64_t* rng;
  bf16 *z, *aw, *bw;         // pieces of dz (planes of `plane` elements), codes of A and B
  float* partial;            // [row blocks][nz] sums of dz
  uint32_t* flags;           // words that the second kernel wants at zero
  int64_t M, N, K, np, nz, kp, plane;
  int pieces;                // 0: no product is wanted
  int act, in_m4e3, sb_per_col, flag_words;
  uint32_t drop_below;
  int64_t z_blocks, col_blocks, a_blocks;  // blocks of dz, then of A's codes, then of B's
};

template <typename T> struct Raw8;  // eight elements as they lie in memory
template <> struct Raw8<float> { float4 v[2]; };
template <> struct Raw8<bf16> { uint4 v; };
template <> struct Raw8<__half> { uint4 v; };
// eight neighbouring elements from i on, `valid` of which exist
template <typename T>
__device__ __forceinline__ Raw8<T> load8(const void* base, int64_t i, int valid) {
  Raw8<T> r;
  const T* const src = static_cast<const T*>(base) + i;
  if (valid == 8 && (reinterpret_cast<uintptr_t>(src) & 15) == 0) {
    if constexpr (sizeof(T) == 4) {
      r.v[0] = __ldcs(reinterpret_cast<const float4*>(src));
      r.v[1] = __ldcs(reinterpret_cast<const float4*>(src) + 1);
    } else {
      r.v = __ldcs(reinterpret_cast<const uint4*>(src));
    }
  } else {
    T* const e = reinterpret_cast<T*>(&r);
#pragma unroll
    for (int j = 0; j < 8; ++j) e[j] = j < valid ? src[j] : from_f32<T>(0.0f);
  }
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, float (&v)[8]) {
  const T* const e = reinterpret_cast<const T*>(&r);
#pragma unroll
  for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
}

// v as the sum of bfloat16 pieces, all but the last cut toward zero (which cannot overflow and leaves an exact remainder)
__device__ __forceinline__ void store_pieces(bf16* dst, int64_t plane, int pieces, const float (&v)[8]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) rest[j] = v[j];
#pragma unroll 1
  for (int q = 0; q < pieces; ++q) {
    uint4 out;
    uint32_t* const w = &out.x;
    const bool last = q + 1 == pieces;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      uint32_t h[2];
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const float r = rest[j + e];
        if (last) {
          h[e] = (uint32_t)__bfloat16_as_ushort(__float2bfloat16_rn(r));
        } else {
          const float head = __uint_as_float(__float_as_uint(r) & 0xFFFF0000u);
          h[e] = __float_as_uint(r) >> 16;
          rest[j + e] = isfinite(r) ? r - head : 0.0f;
          if (r != r) h[e] = 0x7FC0u;  // a NaN whose payload the cut would lose
        }
      }
      w[j / 2] = h[0] | (h[1] << 16);
    }
    *reinterpret_cast<uint4*>(dst + q * plane) = out;
  }
}

__device__ __forceinline__ void expand_codes(const PrepParams& p, const uint8_t* row, bf16* dst, int64_t k) {
  uint4 out = make_uint4(0u, 0u, 0u, 0u);
  if (row) {
    __align__(8) uint8_t c[8];
    const int valid = p.K - k < 8 ? (int)(p.K - k) : 8;
    const uint8_t* const src = row + k;
    if (valid == 8 && (reinterpret_cast<uintptr_t>(src) & 7) == 0) {
      *reinterpret_cast<uint2*>(c) = __ldg(reinterpret_cast<const uint2*>(src));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = j < valid ? __ldg(src + j) : (uint8_t)0;
    }
    uint32_t* const w = &out.x;
    const uint32_t* const c4 = reinterpret_cast<const uint32_t*>(c);
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      u64 v[2];
      if (p.in_m4e3) decode4<true>(c4[q], v[0], v[1]);
      else decode4<false>(c4[q], v[0], v[1]);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float lo, hi;
        unpack2(v[e], lo, hi);
        w[2 * q + e] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);  // exact: the low halves are zero
      }
    }
  }
  *reinterpret_cast<uint4*>(dst + k) = out;
}

template <typename G, typename Z, bool GATED>
__global__ void __launch_bounds__(PREP_THREADS) grad_prepare_kernel(const PrepParams p) {
  constexpr int HALVES = GATED ? 2 : 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  after_previous();
  int64_t b = blockIdx.x;
  if (b == 0)
    for (int i = threadIdx.x; i < p.flag_words; i += PREP_THREADS) p.flags[i] = 0u;
  if (b >= p.z_blocks) {  // codes: a warp takes a row at a time
    b -= p.z_blocks;
    const bool is_a = b < p.a_blocks;
    const int64_t row = (is_a ? b : b - p.a_blocks) * 8 + warp;
    const uint8_t* src = nullptr;
    bf16* dst;
    if (is_a) {
      if (row >= p.M) return;
      src = p.A + row * p.K;
      dst = p.aw + row * p.kp;
    } else {
      if (row >= p.nz) return;
      if (row < p.N) src = p.B + row * p.K;
      else if (row >= p.np && row < p.np + p.N) src = p.B2 + (row - p.np) * p.K;
      dst = p.bw + row * p.kp;  // (rows of the padding: zeros)
    }
    for (int64_t k = lane * 8; k < p.kp; k += 256) expand_codes(p, src, dst, k);
    return;
  }

  __shared__ float sums[HALVES][PREP_THREADS / 32][PREP_COLS];
  const int64_t n = (b % p.col_blocks) * PREP_COLS + lane * 8, m0 = (b / p.col_blocks) * PREP_ROWS + warp;
  const int valid = n >= p.N ? 0 : p.N - n < 8 ? (int)(p.N - n) : 8;
  float total[HALVES][8];
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) total[h][j] = 0.0f;
  if (n < p.np) {
    // all of a thread's loads before its first store: four rows of sixteen bytes and more are on their way at a time
    Raw8<G> g[PREP_EACH];
    Raw8<Z> z[PREP_EACH][HALVES];
    const bool reads_z = GATED || p.act != ACT_NONE;
#pragma unroll
    for (int i = 0; i < PREP_EACH; ++i) {
      const int64_t m = m0 + i * (PREP_THREADS / 32);
      if (m >= p.M) break;
      g[i] = load8<G>(p.grad, m * p.N + n, valid);
      if (reads_z) {
#pragma unroll
        for (int h = 0; h < HALVES; ++h) z[i][h] = load8<Z>(p.pre, (h * p.M + m) * p.N + n, valid);
      }
    }
    float scale[HALVES][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      scale[0][j] = !p.sb ? 1.0f : p.sb_per_col ? (j < valid ? p.sb[n + j] : 0.0f) : p.sb[0];
      if (GATED) scale[HALVES - 1][j] = p.sb_per_col ? (j < valid ? p.sb2[n + j] : 0.0f) : p.sb2[0];
    }
    with_act(p.act, [&](auto act_tag) {
      constexpr int ACT = decltype(act_tag)::value;
#pragma unroll
      for (int i = 0; i < PREP_EACH; ++i) {
        const int64_t m = m0 + i * (PREP_THREADS / 32);
        if (m >= p.M) break;
        float gv[8], zv[8], d[HALVES][8];
        widen8(g[i], gv);
        if (GATED || ACT != ACT_NONE) widen8(z[i][0], zv);
        if (!GATED && p.drop_below) {
          const uint64_t seed = p.rng[0], offset = p.rng[1];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 r = philox((uint32_t)(n >> 2) + h, (uint32_t)m, offset, seed);
            const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (w[j] < p.drop_below) gv[4 * h + j] = 0.0f;
          }
        }
        if constexpr (GATED) {
          float v[8];
          widen8(z[i][1], v);
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            d[0][j] = gv[j] * v[j] * act_slope_of<ACT>(zv[j]);
            d[1][j] = gv[j] * act_value_of<ACT>(zv[j]);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j)
            d[0][j] = ACT == ACT_NONE ? gv[j] : ACT == ACT_RELU ? (zv[j] > 0.0f ? gv[j] : 0.0f) : gv[j] * act_slope_of<ACT>(zv[j]);
        }
        const float by = p.sa ? p.sa[m] : 1.0f;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          float s[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            d[h][j] = j < valid ? d[h][j] : 0.0f;  // the padding of a row
            total[h][j] += d[h][j];
            s[j] = d[h][j] * (scale[h][j] * by);
          }
          if (p.pieces) store_pieces(p.z + m * p.nz + h * p.np + n, p.plane, p.pieces, s);
        }
      }
    });
  }
  if (!p.partial) return;
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[h][warp][lane * 8 + j] = total[h][j];
  __syncthreads();
  const int64_t col = (b % p.col_blocks) * PREP_COLS + threadIdx.x;
  if (col >= p.np) return;
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < PREP_THREADS / 32; ++w) s += sums[h][w][threadIdx.x];
    p.partial[(b / p.col_blocks) * p.nz + h * p.np + col] = s;
  }
}

// ------------------------------------------------------------------ products
// out[r][s] = alpha sum_l X[r][l] Y[l][s] over the pieces of X.
//   grad_a: r = m, l = n, s = k; X's rows are contiguous in l (K-major)
//   grad_b: r = n, l = m, s = k; X is read from the same layout, contiguous in r (MN-major); so is Y, contiguous in s, in both
// A cluster of two CTAs forms a 256 x 256 tile: each CTA holds 128 rows of X, half of Y's columns and the accumulators of its rows, and
// one thread of the first issues the matrix instructions of both (cta_group::2).  What bounds such a product is what the L2 can
// deliver: a CTA alone with 128 x 256 outputs fetched 48 KB per 64 l where this takes 32 (4096 x 4096 x 1024: 82 us alone).
// Six warps a CTA: one thread loads, one multiplies into one of two accumulators of 256 columns of tensor memory, four bring the
// other one out.
//
// Equal shares.  The tiles' steps of 64 l stand in one row, cut into shares of equal length; a cluster walks its own from the end.  A
// tile that a border cuts is begun by lower shares, which leave binary32 sums in the workspace, and finished by the share with its last
// step, which adds them in order.  A cluster takes the number of its share when it starts, from a counter, so it only ever waits for
// clusters that run already or have ended, and what it waits for is the first thing that those do.  Where whole tiles divide as well, they stay whole.
constexpr int BM = 128, BN = 256, BL = 64, GRAD_THREADS = 192;  // of a CTA: rows, columns, step
constexpr int X_BYTES = BM * BL * 2, STAGE = 2 * X_BYTES, STAGES = 6;
constexpr size_t PRODUCT_SMEM = 1024 + (size_t)STAGE * STAGES + 256;
constexpr int PART_FLOATS = BM * BN;  // a CTA's part of a begun tile

struct Job {
  int64_t rows, cols;       // of one half's output
  int64_t r_tiles, s_tiles; // r_tiles: of one half
  int64_t half;             // X's coordinate r of the second half
  int x_mn, pieces, steps;  // steps: blocks of l times pieces
  int div_stride;
  void* out[2];
  const float *alpha[2], *div[2];  // factors of a half, divisors of its rows (or null)
};
struct ProductParams {
  CUtensorMap x[2], y[2];
  Job job[2];
  int64_t tiles0, tiles;    // of the first job, of both
  int64_t units0, units;    // their steps
  int64_t share;            // steps of a cluster; 0: whole tiles
  int out_type;
  float factor;
  uint32_t* flags;          // shares: the counter, then a word per CTA's part
  float* parts;
  const float* partial;     // bias: [row blocks][nz]
  float* bias[2];
  int64_t row_blocks, N, np, nz;
};

__device__ __forceinline__ uint32_t mapa(uint32_t addr, int rank) {
  uint32_t d;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
  return d;
}
// a box of a three-dimensional map into this CTA's memory, counted by a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}
// Shared-memory operand of a matrix instruction, 128-byte swizzle: 1024-byte groups of eight 128-byte lines.  K-major: a line is
// a row's 64 values of l, `stride` the step between groups of eight rows.  MN-major: a line is 64 rows at one l, `stride` the
// step between groups of eight l and `lead` the one between blocks of 64 rows.
__device__ __forceinline__ uint64_t operand(uint32_t addr, int lead, int stride) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
__device__ __forceinline__ void mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
      "r"(idesc), "r"((uint32_t)add) : "memory");
}
// the barrier at this address in both CTAs
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar), "h"((uint16_t)3)
               : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(addr));
  tmem_wait_ld();
}

// a cluster's work, piece by piece: a tile and some of its steps
struct Work {
  int job, half, k0, k1;
  int64_t r, s, start;  // first row (of the half) and column, the tile's first step among all
};
struct Walk {
  int64_t at, end, by;  // shares: steps [end, at) are left; whole tiles: the next tile, their number
  __device__ __forceinline__ Walk(const ProductParams& p, int64_t c, int64_t clusters) {
    by = clusters;
    if (p.share) {
      end = c * p.share;
      at = end + p.share < p.units ? end + p.share : p.units;
    } else {
      at = c;
      end = p.tiles;
    }
  }
  __device__ __forceinline__ bool next(const ProductParams& p, Work& w) {
    int64_t t;
    if (p.share) {
      if (at <= end) return false;
      w.job = at - 1 >= p.units0;
      const int steps = p.job[w.job].steps;
      const int64_t base = w.job ? p.units0 : 0;
      t = (at - 1 - base) / steps;
      w.start = base + t * steps;
      w.k1 = (int)(at - w.start);
      w.k0 = end > w.start ? (int)(end - w.start) : 0;
      at = w.start + w.k0;
    } else {
      if (at >= end) return false;
      w.job = at >= p.tiles0;
      t = w.job ? at - p.tiles0 : at;
      w.k0 = 0;
      w.k1 = p.job[w.job].steps;
      w.start = 0;
      at += by;
    }
    const Job& j = p.job[w.job];
    w.s = (t % j.s_tiles) * BN;
    t /= j.s_tiles;
    w.half = t >= j.r_tiles;
    w.r = (w.half ? t - j.r_tiles : t) * (2 * BM);
    return true;
  }
};

// the bias' gradient: sums of the row blocks' sums, in their order; a warp adds every fourth of 32 columns
__device__ __forceinline__ void bias_sums(const ProductParams& p, float (*part)[32], int warp, int lane) {
  for (int64_t c0 = (int64_t)blockIdx.x * 32; c0 < p.nz; c0 += (int64_t)gridDim.x * 32) {
    const int64_t c = c0 + lane;
    float s = 0.0f;
    if (c < p.nz)
      for (int64_t r = warp; r < p.row_blocks; r += 4) s += p.partial[r * p.nz + c];
    part[warp][lane] = s;
    asm volatile("bar.sync 1, 128;" ::: "memory");
    const int64_t half = c >= p.np, n = half ? c - p.np : c;
    if (warp == 0 && c < p.nz && n < p.N && p.bias[half])
      p.bias[half][n] = (part[0][lane] + part[1][lane] + (part[2][lane] + part[3][lane])) * p.factor;
    asm volatile("bar.sync 1, 128;" ::: "memory");
  }
}

template <typename T>
__device__ __forceinline__ void store32(T* dst, int64_t valid, const float (&r)[32], float alpha) {
  constexpr int W = 16 / (int)sizeof(T);
  if (valid >= 32 && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
#pragma unroll
    for (int q = 0; q < 32 / W; ++q) {
      uint4 raw;
      T* const e = reinterpret_cast<T*>(&raw);
#pragma unroll
      for (int j = 0; j < W; ++j) e[j] = from_f32<T>(r[q * W + j] * alpha);
      *reinterpret_cast<uint4*>(dst + q * W) = raw;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < valid) dst[j] = from_f32<T>(r[j] * alpha);
  }
}

__global__ void __launch_bounds__(GRAD_THREADS, 1) grad_product_kernel(const __grid_constant__ ProductParams p) {
  extern __shared__ unsigned char product_raw[];
  unsigned char* const base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(product_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(base + STAGES * STAGE);  // full, empty per stage; done, free per accumulator
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4);
  volatile int* const dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* const share_slot = tmem_slot + 2;
  __shared__ float part[4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1;  // in the cluster
  const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_done = empty + 8 * STAGES, acc_free = acc_done + 16;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + 8 * i, 1);   // the first CTA's counts both CTAs' bytes
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_done + 8 * i, 1);
      mbar_init(acc_free + 8 * i, 256);  // the first CTA's: both CTAs' readers
    }
    *dead = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  __syncwarp();
  cluster_sync();  // the other CTA runs: its memory may be written
  after_previous();
  if (p.share && rank == 0 && threadIdx.x == 0) {
    const uint32_t c = atomicAdd(p.flags, 1u);
    *share_slot = c;
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(mapa(smem_u32(share_slot), 1)), "r"(c) : "memory");
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cluster_sync();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  const int64_t share = p.share ? *share_slot : blockIdx.x >> 1;
  Walk walk(p, share, gridDim.x >> 1);
  Work w;

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      while (walk.next(p, w)) {
        const Job& j = p.job[w.job];
        const int r = (int)(w.r + (w.half ? j.half : 0)) + rank * BM, s = (int)w.s + rank * (BN / 2);
        int l = w.k0 / j.pieces, q = w.k0 % j.pieces;
        for (int k = w.k0; k < w.k1; ++k) {
          mbar_wait(empty + 8 * stage, phase ^ 1, dead);
          if (*dead) goto loaded;
          const uint32_t x = smem_u32(base + stage * STAGE), y = x + X_BYTES, bar = mapa(full + 8 * stage, 0);
          if (rank == 0) mbar_arrive_expect(full + 8 * stage, 2 * STAGE);
          if (j.x_mn) {
            tma_load(x, &p.x[w.job], r, l * BL, q, bar);
            tma_load(x + X_BYTES / 2, &p.x[w.job], r + 64, l * BL, q, bar);
          } else {
            tma_load(x, &p.x[w.job], l * BL, r, q, bar);
          }
          tma_load(y, &p.y[w.job], s, l * BL, 0, bar);
          tma_load(y + X_BYTES / 2, &p.y[w.job], s + 64, l * BL, 0, bar);
          if (++q == j.pieces) {
            q = 0;
            ++l;
          }
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
    loaded:;
    }
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      while (walk.next(p, w)) {
        const int x_mn = p.job[w.job].x_mn;
        // binary32 sums of bfloat16 products; which operand is MN-major; sizes
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)x_mn << 15) | (1u << 16) | ((BN / 8) << 17) | ((2 * BM / 16) << 24);
        mbar_wait_cluster(acc_free + 8 * acc, acc_phase ^ 1, dead);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int b = w.k0; b < w.k1; ++b) {
          mbar_wait_cluster(full + 8 * stage, phase, dead);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t x = smem_u32(base + stage * STAGE), y = x + X_BYTES;
          if (!*dead) {
#pragma unroll
            for (int k = 0; k < BL / 16; ++k)
              mma(tmem + acc * BN, x_mn ? operand(x + k * 2048, X_BYTES / 2, 1024) : operand(x + k * 32, 16, 1024),
                  operand(y + k * 2048, X_BYTES / 2, 1024), idesc, b > w.k0 || k > 0);
          }
          mma_commit(empty + 8 * stage);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
          }
        }
        mma_commit(acc_done + 8 * acc);
        if (++acc == 2) {
          acc = 0;
          acc_phase ^= 1;
        }
      }
    }
  } else {
    const int quarter = warp & 3;  // the lanes of tensor memory that this warp may read
    const int row = quarter * 32 + lane;
    if (p.partial) bias_sums(p, part, quarter, lane);
    int acc = 0;
    uint32_t phase = 0;
    while (walk.next(p, w)) {
      const Job& j = p.job[w.job];
      const bool begins = w.k1 < j.steps, ends = w.k0 > 0 && !begins;
      const int64_t first = ends ? w.start / p.share : share;  // the shares that began this tile: first to share - 1
      if (ends) {
        if (row == 0)
          for (int64_t c = first; c < share; ++c) wait_flag(p.flags + 1 + 2 * c + rank, dead);
        asm volatile("bar.sync 1, 128;" ::: "memory");
      }
      mbar_wait(acc_done + 8 * acc, phase, dead);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int64_t r = w.r + rank * BM + row;
      float alpha = p.factor * (j.alpha[w.half] ? *j.alpha[w.half] : 1.0f);
      if (j.div[w.half] && r < j.rows) alpha = __fdiv_rn(alpha, j.div[w.half][r * j.div_stride]);
      if (*dead) alpha = __uint_as_float(0x7FC00000u);
      float4* const mine = reinterpret_cast<float4*>(p.parts + (2 * share + rank) * PART_FLOATS) + row;  // [four columns][row]
#pragma unroll 1
      for (int c = 0; c < BN; c += 32) {
        uint32_t t[32];
        float v[32];
        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + c, t);
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(t[i]);
        if (begins) {
#pragma unroll
          for (int i = 0; i < 8; ++i) mine[(c / 4 + i) * BM] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
          continue;
        }
        for (int64_t o = first; o < share; ++o) {
          const float4* const theirs = reinterpret_cast<const float4*>(p.parts + (2 * o + rank) * PART_FLOATS) + row;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            const float4 f = __ldcg(theirs + (c / 4 + i) * BM);
            v[4 * i] += f.x;
            v[4 * i + 1] += f.y;
            v[4 * i + 2] += f.z;
            v[4 * i + 3] += f.w;
          }
        }
        const int64_t valid = j.cols - (w.s + c), at = r * j.cols + w.s + c;
        if (r < j.rows && valid > 0) {
          if (p.out_type == LT_F32) store32(static_cast<float*>(j.out[w.half]) + at, valid, v, alpha);
          else if (p.out_type == LT_BF16) store32(static_cast<bf16*>(j.out[w.half]) + at, valid, v, alpha);
          else store32(static_cast<__half*>(j.out[w.half]) + at, valid, v, alpha);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      mbar_arrive_cluster(mapa(acc_free + 8 * acc, 0));
      if (begins) {
        __threadfence();
        asm volatile("bar.sync 1, 128;" ::: "memory");
        if (row == 0) asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p.flags + 1 + 2 * share + rank), "r"(1u) : "memory");
      }
      if (++acc == 2) {
        acc = 0;
        phase ^= 1;
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  cluster_sync();  // nothing of the other CTA's is on its way here any more
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
}

// ------------------------------------------------------------------ host
int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// bfloat16 pieces that dz takes beside a result of the given type; dz that is g itself or zero has no more bits than g, and a
// common scale is applied to the finished product
int pieces(const GradCall& c) {
  const auto of = [](int type) { return type == LT_BF16 ? 1 : type == LT_F16 ? 2 : 3; };
  const bool plain = !c.gated && (c.act == ACT_NONE || c.act == ACT_RELU) && !c.sa_per_row && !c.sb_per_col;
  return plain && of(c.grad_type) < of(c.out_type) ? of(c.grad_type) : of(c.out_type);
}

int clusters_of_the_device() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n < 2) return 74;
  return n / 2;
}

struct Layout {
  int64_t np, nz, kp, row_blocks;
  int pieces, flag_words;
  // tiles of the products and their division (see the product kernel)
  int64_t tiles[2], units[2], share;
  int steps[2], clusters;
  size_t z, aw, bw, partial, flags, parts, total;
};
Layout layout(const GradCall& c) {
  Layout l = {};
  const int halves = c.gated ? 2 : 1;
  const bool a = c.grad_a && c.K > 0, b = c.grad_b && c.K > 0;
  l.np = up(c.N, 8);
  l.nz = l.np * halves;
  l.kp = up(c.K, 8);
  l.row_blocks = (c.M + PREP_ROWS - 1) / PREP_ROWS;
  l.pieces = a || b ? pieces(c) : 0;
  const auto blocks = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
  if (a) {
    l.steps[0] = (int)(blocks(l.nz, BL) * l.pieces);
    l.tiles[0] = blocks(c.M, 2 * BM) * blocks(c.K, BN);
  }
  if (b) {
    l.steps[1] = (int)(blocks(c.M, BL) * l.pieces);
    l.tiles[1] = halves * blocks(c.N, 2 * BM) * blocks(c.K, BN);
  }
  for (int i = 0; i < 2; ++i) l.units[i] = l.tiles[i] * l.steps[i];
  // Whole tiles, in turn, or equal shares: a cut costs about ten steps (a part written and read again), and a share has at least four
  const int64_t all = l.tiles[0] + l.tiles[1], units = l.units[0] + l.units[1], most = clusters_of_the_device();
  if (all > 0) {
    const int64_t n = all < most ? all : most;
    int64_t whole = 0;  // steps of the busiest cluster: cluster c takes the tiles c, c + n, ...
    for (int64_t x = 0; x < n; ++x) {
      const int64_t first = x < l.tiles[0] ? (l.tiles[0] - 1 - x) / n + 1 : 0, both = (all - 1 - x) / n + 1;
      const int64_t load = first * l.steps[0] + (both - first) * l.steps[1];
      whole = load > whole ? load : whole;
    }
    const int64_t even = blocks(units, most) < 4 ? 4 : blocks(units, most);
    l.share = even + 10 < whole ? even : 0;
    l.clusters = (int)(l.share ? blocks(units, l.share) : n);
  }
  l.flag_words = l.share ? 1 + 2 * l.clusters : 0;
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  l.z = take((size_t)c.M * l.nz * 2 * l.pieces);
  l.aw = take(b ? (size_t)c.M * l.kp * 2 : 0);
  l.bw = take(a ? (size_t)l.nz * l.kp * 2 : 0);
  l.partial = take(c.grad_bias ? (size_t)l.row_blocks * l.nz * 4 : 0);
  l.flags = take((size_t)l.flag_words * 4);
  l.parts = take(l.share ? (size_t)l.clusters * 2 * PART_FLOATS * 4 : 0);
  l.total = at;
  return l;
}

// planes x rows x cols of bfloat16, rows `pitch` elements apart; boxes of 64 columns and `box_rows` rows, 128-byte swizzle
bool make_map(CUtensorMap* map, const void* base, int64_t cols, int64_t rows, int64_t planes, int64_t pitch, int64_t plane, int box_rows) {
  const EncodeTiled encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes}, strides[2] = {(cuuint64_t)pitch * 2, (cuuint64_t)plane * 2};
  const cuuint32_t box[3] = {64, (cuuint32_t)box_rows, 1}, step[3] = {1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename G, typename Z>
cudaError_t launch_prepare(const PrepParams& q, bool gated, unsigned blocks, cudaStream_t stream) {
  return gated ? launch_after(grad_prepare_kernel<G, Z, true>, dim3(blocks), PREP_THREADS, 0, stream, q)
               : launch_after(grad_prepare_kernel<G, Z, false>, dim3(blocks), PREP_THREADS, 0, stream, q);
}
template <typename G>
cudaError_t launch_prepare(const PrepParams& q, const GradCall& c, unsigned blocks, cudaStream_t stream) {
  return c.pre_type == LT_F32 ? launch_prepare<G, float>(q, c.gated, blocks, stream)
         : c.pre_type == LT_BF16 ? launch_prepare<G, bf16>(q, c.gated, blocks, stream) : launch_prepare<G, __half>(q, c.gated, blocks, stream);
}

}  // namespace

size_t backward_workspace(const GradCall& c) { return c.M > 0 && c.N > 0 ? layout(c).total : 0; }

cudaError_t launch_backward(const GradCall& c, void* workspace, cudaStream_t stream) {
  const size_t size = c.out_type == LT_F32 ? 4 : 2;
  cudaError_t e = cudaSuccess;
  const auto zero = [&](void* dst, size_t bytes) {
    if (dst && bytes && e == cudaSuccess) e = cudaMemsetAsync(dst, 0, bytes, stream);
  };
  if (c.M == 0 || c.N == 0) {  // empty sums
    zero(c.grad_a, c.M * c.K * size);
    zero(c.grad_b, c.N * c.K * size);
    zero(c.grad_b2, c.N * c.K * size);
    zero(c.grad_bias, c.N * 4);
    zero(c.grad_bias2, c.N * 4);
    return e;
  }
  const Layout l = layout(c);
  const bool a = l.tiles[0] > 0, b = l.tiles[1] > 0;
  if (!a && !b && !c.grad_bias) return cudaSuccess;
  unsigned char* const ws = static_cast<unsigned char*>(workspace);

  PrepParams q = {};
  q.grad = c.grad; q.pre = c.pre; q.A = c.A; q.B = c.B; q.B2 = c.B2;
  q.sa = c.sa_per_row ? c.sa : nullptr;
  q.sb = c.sb_per_col || c.gated ? c.sb : nullptr;
  q.sb2 = c.sb2;
  q.rng = c.rng;
  q.z = reinterpret_cast<bf16*>(ws + l.z);
  q.aw = reinterpret_cast<bf16*>(ws + l.aw);
  q.bw = reinterpret_cast<bf16*>(ws + l.bw);
  q.partial = c.grad_bias ? reinterpret_cast<float*>(ws + l.partial) : nullptr;
  q.flags = reinterpret_cast<uint32_t*>(ws + l.flags);
  q.flag_words = l.flag_words;
  q.M = c.M; q.N = c.N; q.K = c.K; q.np = l.np; q.nz = l.nz; q.kp = l.kp;
  q.plane = c.M * l.nz;
  q.pieces = l.pieces;
  q.act = c.act; q.in_m4e3 = c.in_m4e3; q.sb_per_col = c.sb_per_col;
  q.drop_below = c.drop_below;
  q.col_blocks = (l.np + PREP_COLS - 1) / PREP_COLS;
  q.z_blocks = q.col_blocks * l.row_blocks;
  q.a_blocks = b ? (c.M + 7) / 8 : 0;
  const int64_t b_blocks = a ? (l.nz + 7) / 8 : 0, blocks = q.z_blocks + q.a_blocks + b_blocks;
  if (blocks > 2147483647LL) return cudaErrorInvalidValue;
  e = c.grad_type == LT_F32 ? launch_prepare<float>(q, c, (unsigned)blocks, stream)
      : c.grad_type == LT_BF16 ? launch_prepare<bf16>(q, c, (unsigned)blocks, stream) : launch_prepare<__half>(q, c, (unsigned)blocks, stream);
  if (e != cudaSuccess) return e;

  ProductParams p = {};
  p.out_type = c.out_type;
  p.factor = c.keep_scale;
  p.partial = q.partial;
  p.bias[0] = c.grad_bias; p.bias[1] = c.grad_bias2;
  p.row_blocks = l.row_blocks; p.N = c.N; p.np = l.np; p.nz = l.nz;
  p.flags = q.flags;
  p.parts = reinterpret_cast<float*>(ws + l.parts);
  p.share = l.share;
  p.tiles0 = p.tiles = l.tiles[0];
  p.units0 = p.units = l.units[0];
  p.tiles += l.tiles[1];
  p.units += l.units[1];
  // (a job without tiles is never looked at: the first one's borders are both 0 then)
  const auto add = [&](int i, bool x_mn, const void* y, int64_t y_rows, int64_t rows) -> Job& {
    if (!make_map(&p.x[i], q.z, l.nz, c.M, l.pieces, l.nz, q.plane, x_mn ? BL : BM) ||
        !make_map(&p.y[i], y, c.K, y_rows, 1, l.kp, y_rows * l.kp, BL))
      e = cudaErrorInvalidValue;
    Job& j = p.job[i];
    j.x_mn = x_mn;
    j.pieces = l.pieces;
    j.steps = l.steps[i];
    j.rows = rows;
    j.cols = c.K;
    j.r_tiles = (rows + 2 * BM - 1) / (2 * BM);
    j.s_tiles = (c.K + BN - 1) / BN;
    return j;
  };
  if (a) {
    Job& j = add(0, false, q.bw, l.nz, c.M);
    j.out[0] = c.grad_a;
    j.alpha[0] = q.sb ? nullptr : c.sb;
    j.div[0] = q.sa;
    j.div_stride = 1;
  }
  if (b) {
    Job& j = add(1, true, q.aw, c.M, c.N);
    j.out[0] = c.grad_b;
    j.out[1] = c.grad_b2;
    j.alpha[0] = j.alpha[1] = q.sa ? nullptr : c.sa;
    j.div[0] = q.sb;
    j.div[1] = c.sb2;
    j.div_stride = c.sb_per_col;
    j.half = l.np;
  }
  if (e != cudaSuccess) return e;
  e = cudaFuncSetAttribute(grad_product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PRODUCT_SMEM);
  if (e != cudaSuccess) return e;
  int64_t clusters = l.clusters;
  if (!p.share && c.grad_bias) {  // more CTAs for the bias: they find no tile
    const int64_t wanted = (l.nz + 63) / 64, most = clusters_of_the_device();
    if (clusters < wanted) clusters = wanted < most ? wanted : most;
  }
  return launch_after(grad_product_kernel, dim3((unsigned)(2 * clusters)), GRAD_THREADS, PRODUCT_SMEM, stream, p, 2);
}

}  // namespace lba
