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
// Two launches:
//   grad_prepare_kernel   reads g and z once; writes the pieces of dz, dz sb where the scale differs by column, the sums of its rows
//                         per column (for the bias), and both operands' codes as bfloat16.  Bound by memory.
//   grad_product_kernel   both products as one list of 128 x BN tiles (tcgen05, TMA), and the bias sums' last step.
#include "lba_grad.cuh"

#include "lba_async.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

constexpr int PREP_ROWS = 32, PREP_COLS = 256, PREP_THREADS = 256;
typedef __nv_bfloat16 bf16;

struct PrepParams {
  const void *grad, *pre;
  const uint8_t *A, *B, *B2;
  const float *sa, *sb, *sb2;
  const uint64_t* rng;
  bf16 *za, *zb, *aw, *bw;   // pieces of dz for grad_a and for grad_b (planes of `plane` elements), codes of A and B
  float* partial;            // [row blocks][nz] sums of dz
  int64_t M, N, K, np, nz, kp, plane;
  int pieces_a, pieces_b;    // 0: not wanted
  int grad_type, pre_type, act, gated, in_m4e3, sa_per_row, sb_per_col;
  uint32_t drop_below;
  int shared;                // grad_a reads grad_b's pieces
  int64_t z_blocks, col_blocks, a_blocks;  // blocks of dz, then of A's codes, then of B's
};

// eight neighbouring elements from i on, `valid` of which exist
__device__ __forceinline__ void load8(const void* base, int type, int64_t i, int valid, float (&v)[8]) {
  if (type == LT_F32) {
    float lo[4], hi[4];
    load_some<float, 4>(base, i, valid < 4 ? valid : 4, lo);
    load_some<float, 4>(base, i + 4, valid > 4 ? valid - 4 : 0, hi);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      v[j] = lo[j];
      v[4 + j] = hi[j];
    }
  } else if (type == LT_BF16) {
    load_some<bf16, 8>(base, i, valid, v);
  } else {
    load_some<__half, 8>(base, i, valid, v);
  }
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
    uint8_t c[8];
    const int valid = p.K - k < 8 ? (int)(p.K - k) : 8;
    const uint8_t* const src = row + k;
    if (valid == 8 && (reinterpret_cast<uintptr_t>(src) & 7) == 0) {
      *reinterpret_cast<uint2*>(c) = __ldg(reinterpret_cast<const uint2*>(src));
    } else {
#pragma unroll
      for (int j = 0; j < 8; ++j) c[j] = j < valid ? __ldg(src + j) : (uint8_t)0;
    }
    uint32_t* const w = &out.x;
#pragma unroll
    for (int j = 0; j < 8; j += 2) {
      const float lo = p.in_m4e3 ? decode_m4e3_top((uint32_t)c[j] << 24) : decode_e4m3_top((uint32_t)c[j] << 24, 0x1p120f);
      const float hi = p.in_m4e3 ? decode_m4e3_top((uint32_t)c[j + 1] << 24) : decode_e4m3_top((uint32_t)c[j + 1] << 24, 0x1p120f);
      w[j / 2] = (__float_as_uint(lo) >> 16) | (__float_as_uint(hi) & 0xFFFF0000u);  // exact
    }
  }
  *reinterpret_cast<uint4*>(dst + k) = out;
}

__global__ void __launch_bounds__(PREP_THREADS) grad_prepare_kernel(const PrepParams p) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  after_previous();
  int64_t b = blockIdx.x;
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

  __shared__ float sums[2][PREP_THREADS / 32][PREP_COLS];
  const int64_t n = (b % p.col_blocks) * PREP_COLS + lane * 8, m0 = (b / p.col_blocks) * PREP_ROWS;
  const int valid = n >= p.N ? 0 : p.N - n < 8 ? (int)(p.N - n) : 8;
  const int halves = p.gated ? 2 : 1;
  float total[2][8];
#pragma unroll
  for (int j = 0; j < 8; ++j) total[0][j] = total[1][j] = 0.0f;
  if (n < p.np) {
    float scale[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      // (a linear layer's common scale is applied to the finished product)
      scale[0][j] = p.sb_per_col ? (j < valid ? p.sb[n + j] : 0.0f) : p.gated ? p.sb[0] : 1.0f;
      scale[1][j] = !p.gated ? 0.0f : p.sb_per_col ? (j < valid ? p.sb2[n + j] : 0.0f) : p.sb2[0];
    }
#pragma unroll 1
    for (int i = 0; i < PREP_ROWS / 8; ++i) {
      const int64_t m = m0 + i * 8 + warp;
      if (m >= p.M) break;
      float g[8], z[8], d[2][8];
      load8(p.grad, p.grad_type, m * p.N + n, valid, g);
      if (p.drop_below) {
        const uint64_t seed = p.rng[0], offset = p.rng[1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint4 r = philox((uint32_t)(n >> 2) + h, (uint32_t)m, offset, seed);
          const uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (w[j] < p.drop_below) g[4 * h + j] = 0.0f;
        }
      }
      if (p.gated) {
        float v[8];
        load8(p.pre, p.pre_type, m * p.N + n, valid, z);
        load8(p.pre, p.pre_type, (p.M + m) * p.N + n, valid, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          d[0][j] = g[j] * v[j] * act_slope(p.act, z[j]);
          d[1][j] = g[j] * act_value(p.act, z[j]);
        }
      } else if (p.act == ACT_NONE) {
#pragma unroll
        for (int j = 0; j < 8; ++j) d[0][j] = g[j];
      } else {
        load8(p.pre, p.pre_type, m * p.N + n, valid, z);
#pragma unroll
        for (int j = 0; j < 8; ++j) d[0][j] = p.act == ACT_RELU ? (z[j] > 0.0f ? g[j] : 0.0f) : g[j] * act_slope(p.act, z[j]);
      }
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        if (h >= halves) break;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          d[h][j] = j < valid ? d[h][j] : 0.0f;  // the padding of a row
          total[h][j] += d[h][j];
        }
        const int64_t at = m * p.nz + h * p.np + n;
        if (p.pieces_b) {
          float s[8];
          const float by = p.sa_per_row ? p.sa[m] : 1.0f;
#pragma unroll
          for (int j = 0; j < 8; ++j) s[j] = d[h][j] * by;
          store_pieces(p.zb + at, p.plane, p.pieces_b, s);
        }
        if (p.pieces_a && !p.shared) {
          float s[8];
#pragma unroll
          for (int j = 0; j < 8; ++j) s[j] = d[h][j] * scale[h][j];
          store_pieces(p.za + at, p.plane, p.pieces_a, s);
        }
      }
    }
  }
  if (!p.partial) return;
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int j = 0; j < 8; ++j) sums[h][warp][lane * 8 + j] = total[h][j];
  __syncthreads();
  const int64_t col = (b % p.col_blocks) * PREP_COLS + threadIdx.x;
  if (col >= p.np) return;
  for (int h = 0; h < halves; ++h) {
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
// Persistent CTAs of six warps: one thread loads (TMA, 128-byte swizzle), one issues tcgen05.mma into one of two accumulators of
// BN columns of tensor memory, four warps bring the other one out.
constexpr int BM = 128, BL = 64, GRAD_THREADS = 192;
constexpr int X_BYTES = BM * BL * 2;
template <int BN> constexpr int STAGE_BYTES = X_BYTES + BN * BL * 2;
template <int BN> constexpr int STAGE_COUNT = BN == 256 ? 4 : BN == 128 ? 6 : 8;
template <int BN> constexpr size_t PRODUCT_SMEM = 1024 + (size_t)STAGE_BYTES<BN> * STAGE_COUNT<BN> + 256;

struct Job {
  int64_t rows, cols;       // of one half's output
  int64_t r_tiles, s_tiles; // r_tiles: of one half
  int64_t half;             // X's coordinate r of the second half
  int x_mn, pieces, l_blocks, halves;
  void* out[2];
  const float *alpha[2];    // device factors of each half (null: 1)
};
struct ProductParams {
  CUtensorMap x[2], y[2];
  Job job[2];
  int64_t tiles0, tiles;    // of the first job, of both
  int out_type;
  float factor;
  const float* partial;     // bias: [row blocks][nz]
  float* bias[2];
  int64_t row_blocks, N, np, nz;
};

__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int x, int y, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
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
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b),
      "r"(idesc), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
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

struct Tile {
  int job, half;
  int64_t r, s;  // first row (of the half) and column
};
template <int BN>
__device__ __forceinline__ Tile tile_of(const ProductParams& p, int64_t t) {
  Tile v;
  v.job = t >= p.tiles0;
  const Job& j = p.job[v.job];
  if (v.job) t -= p.tiles0;
  v.s = (t % j.s_tiles) * BN;
  t /= j.s_tiles;
  v.half = t >= j.r_tiles;
  v.r = (v.half ? t - j.r_tiles : t) * BM;
  return v;
}

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
__device__ __forceinline__ void store32(T* dst, int64_t valid, const uint32_t (&r)[32], float alpha) {
  constexpr int W = 16 / (int)sizeof(T);
  if (valid >= 32 && (reinterpret_cast<uintptr_t>(dst) & 15) == 0) {
#pragma unroll
    for (int q = 0; q < 32 / W; ++q) {
      uint4 raw;
      T* const e = reinterpret_cast<T*>(&raw);
#pragma unroll
      for (int j = 0; j < W; ++j) e[j] = from_f32<T>(__uint_as_float(r[q * W + j]) * alpha);
      *reinterpret_cast<uint4*>(dst + q * W) = raw;
    }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j < valid) dst[j] = from_f32<T>(__uint_as_float(r[j]) * alpha);
  }
}

template <int BN>
__global__ void __launch_bounds__(GRAD_THREADS, 1) grad_product_kernel(const __grid_constant__ ProductParams p) {
  constexpr int STAGES = STAGE_COUNT<BN>, STAGE = STAGE_BYTES<BN>;
  constexpr uint32_t COLS = 2 * BN;  // of tensor memory: 128, 256 or 512
  extern __shared__ unsigned char smem_raw[];
  unsigned char* const base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(base + STAGES * STAGE);  // full, empty per stage; done, free per accumulator
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 4);
  volatile int* const dead = reinterpret_cast<volatile int*>(tmem_slot + 1);
  __shared__ float part[4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_done = empty + 8 * STAGES, acc_free = acc_done + 16;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + 8 * i, 1);
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_done + 8 * i, 1);
      mbar_init(acc_free + 8 * i, 128);
    }
    *dead = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(COLS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
  const uint32_t tmem = *tmem_slot;
  after_previous();

  if (warp == 0) {
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
        const Tile v = tile_of<BN>(p, t);
        const Job& j = p.job[v.job];
        const int r = (int)(v.r + (v.half ? j.half : 0)), s = (int)v.s;
        for (int b = 0; b < j.l_blocks; ++b)
          for (int q = 0; q < j.pieces; ++q) {
            mbar_wait(empty + 8 * stage, phase ^ 1, dead);
            if (*dead) goto loaded;
            const uint32_t x = smem_u32(base + stage * STAGE), y = x + X_BYTES, bar = full + 8 * stage;
            mbar_arrive_expect(bar, STAGE);
            if (j.x_mn) {
              tma_load(x, &p.x[v.job], r, b * BL, q, bar);
              tma_load(x + X_BYTES / 2, &p.x[v.job], r + 64, b * BL, q, bar);
            } else {
              tma_load(x, &p.x[v.job], b * BL, r, q, bar);
            }
#pragma unroll
            for (int i = 0; i < BN / 64; ++i) tma_load(y + i * 64 * BL * 2, &p.y[v.job], s + 64 * i, b * BL, 0, bar);
            if (++stage == STAGES) {
              stage = 0;
              phase ^= 1;
            }
          }
      }
    loaded:;
    }
  } else if (warp == 1) {
    if (lane == 0) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 0;
      for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
        const Job& j = p.job[tile_of<BN>(p, t).job];
        const int x_mn = j.x_mn, steps = j.l_blocks * j.pieces;
        // binary32 sums of bfloat16 products; which operand is MN-major; sizes
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)x_mn << 15) | (1u << 16) | ((BN / 8) << 17) | ((BM / 16) << 24);
        mbar_wait(acc_free + 8 * acc, acc_phase ^ 1, dead);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        for (int b = 0; b < steps; ++b) {
          mbar_wait(full + 8 * stage, phase, dead);
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t x = smem_u32(base + stage * STAGE), y = x + X_BYTES;
          if (!*dead) {
#pragma unroll
            for (int k = 0; k < BL / 16; ++k)
              mma(tmem + acc * BN, x_mn ? operand(x + k * 2048, X_BYTES / 2, 1024) : operand(x + k * 32, 16, 1024),
                  operand(y + k * 2048, 64 * BL * 2, 1024), idesc, b > 0 || k > 0);
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
    if (p.partial) bias_sums(p, part, quarter, lane);
    int acc = 0;
    uint32_t phase = 0;
    for (int64_t t = blockIdx.x; t < p.tiles; t += gridDim.x) {
      const Tile v = tile_of<BN>(p, t);
      const Job& j = p.job[v.job];
      mbar_wait(acc_done + 8 * acc, phase, dead);
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      const int64_t r = v.r + quarter * 32 + lane;
      const float alpha = *dead ? __uint_as_float(0x7FC00000u) : p.factor * (j.alpha[v.half] ? *j.alpha[v.half] : 1.0f);
#pragma unroll 1
      for (int c = 0; c < BN; c += 32) {
        uint32_t w[32];
        tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + c, w);
        const int64_t valid = j.cols - (v.s + c), at = r * j.cols + v.s + c;
        if (r < j.rows && valid > 0) {
          if (p.out_type == LT_F32) store32(static_cast<float*>(j.out[v.half]) + at, valid, w, alpha);
          else if (p.out_type == LT_BF16) store32(static_cast<bf16*>(j.out[v.half]) + at, valid, w, alpha);
          else store32(static_cast<__half*>(j.out[v.half]) + at, valid, w, alpha);
        }
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      mbar_arrive(acc_free + 8 * acc);
      if (++acc == 2) {
        acc = 0;
        phase ^= 1;
      }
    }
  }
  __syncwarp();
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
  __syncthreads();
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(COLS) : "memory");
}

// ------------------------------------------------------------------ host
int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// bfloat16 pieces that dz takes beside a result of the given type; dz that is g itself or zero has no more bits than g, and a
// common scale is applied to the finished product
int pieces(const GradCall& c, bool scaled) {
  const auto of = [](int type) { return type == LT_BF16 ? 1 : type == LT_F16 ? 2 : 3; };
  const bool plain = !c.gated && (c.act == ACT_NONE || c.act == ACT_RELU) && !scaled;
  return plain && of(c.grad_type) < of(c.out_type) ? of(c.grad_type) : of(c.out_type);
}

struct Layout {
  int64_t np, nz, kp, row_blocks;
  int pieces_a, pieces_b;
  bool shared;  // both products read the same pieces of dz
  size_t za, zb, aw, bw, partial, total;
};
Layout layout(const GradCall& c) {
  Layout l;
  const int halves = c.gated ? 2 : 1;
  l.np = up(c.N, 8);
  l.nz = l.np * halves;
  l.kp = up(c.K, 8);
  l.row_blocks = (c.M + PREP_ROWS - 1) / PREP_ROWS;
  l.pieces_a = c.grad_a ? pieces(c, c.sb_per_col) : 0;
  l.pieces_b = c.grad_b || c.grad_b2 ? pieces(c, c.sa_per_row) : 0;
  // A gated layer's halves have scales of their own, so grad_a needs them inside dz
  l.shared = l.pieces_a && l.pieces_b && l.pieces_a == l.pieces_b && !c.sb_per_col && !c.sa_per_row && !c.gated;
  const size_t plane = (size_t)c.M * l.nz * 2;
  size_t at = 0;
  const auto take = [&at](size_t bytes) {
    const size_t was = at;
    at += up256(bytes);
    return was;
  };
  l.zb = take(plane * l.pieces_b);
  l.za = l.shared ? l.zb : take(plane * l.pieces_a);
  l.aw = take(l.pieces_b ? (size_t)c.M * l.kp * 2 : 0);
  l.bw = take(l.pieces_a ? (size_t)l.nz * l.kp * 2 : 0);
  l.partial = take(c.grad_bias || c.grad_bias2 ? (size_t)l.row_blocks * l.nz * 4 : 0);
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

int multiprocessors() {
  int dev = 0, n = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || n <= 0) return 148;
  return n;
}

template <int BN>
cudaError_t launch_products(const ProductParams& p, int sms, cudaStream_t stream) {
  auto kernel = grad_product_kernel<BN>;
  constexpr size_t smem = PRODUCT_SMEM<BN>;
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  int64_t grid = p.tiles;
  if (p.partial && (p.nz + 31) / 32 > grid) grid = (p.nz + 31) / 32;
  if (grid > sms) grid = sms;
  return launch_after(kernel, dim3((unsigned)grid), GRAD_THREADS, smem, stream, p);
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
  GradCall w = c;
  if (c.K == 0) w.grad_a = w.grad_b = w.grad_b2 = nullptr;  // nothing to write
  const Layout l = layout(w);
  if (!l.pieces_a && !l.pieces_b && !w.grad_bias && !w.grad_bias2) return cudaSuccess;
  unsigned char* const ws = static_cast<unsigned char*>(workspace);
  const int halves = c.gated ? 2 : 1;

  PrepParams q = {};
  q.grad = c.grad; q.pre = c.pre; q.A = c.A; q.B = c.B; q.B2 = c.B2;
  q.sa = c.sa; q.sb = c.sb; q.sb2 = c.sb2; q.rng = c.rng;
  q.za = reinterpret_cast<bf16*>(ws + l.za);
  q.zb = reinterpret_cast<bf16*>(ws + l.zb);
  q.aw = reinterpret_cast<bf16*>(ws + l.aw);
  q.bw = reinterpret_cast<bf16*>(ws + l.bw);
  q.partial = w.grad_bias || w.grad_bias2 ? reinterpret_cast<float*>(ws + l.partial) : nullptr;
  q.M = c.M; q.N = c.N; q.K = c.K; q.np = l.np; q.nz = l.nz; q.kp = l.kp;
  q.plane = c.M * l.nz;
  q.pieces_a = l.pieces_a; q.pieces_b = l.pieces_b; q.shared = l.shared;
  q.grad_type = c.grad_type; q.pre_type = c.pre_type; q.act = c.act; q.gated = c.gated; q.in_m4e3 = c.in_m4e3;
  q.sa_per_row = c.sa_per_row; q.sb_per_col = c.sb_per_col;
  q.drop_below = c.drop_below;
  q.col_blocks = (l.np + PREP_COLS - 1) / PREP_COLS;
  q.z_blocks = q.col_blocks * l.row_blocks;
  q.a_blocks = l.pieces_b ? (c.M + 7) / 8 : 0;
  const int64_t b_blocks = l.pieces_a ? (l.nz + 7) / 8 : 0, blocks = q.z_blocks + q.a_blocks + b_blocks;
  if (blocks > 2147483647LL) return cudaErrorInvalidValue;
  if ((e = launch_after(grad_prepare_kernel, dim3((unsigned)blocks), PREP_THREADS, 0, stream, q)) != cudaSuccess) return e;

  ProductParams p = {};
  p.out_type = c.out_type;
  p.factor = c.keep_scale;
  p.partial = q.partial;
  p.bias[0] = w.grad_bias; p.bias[1] = w.grad_bias2;
  p.row_blocks = l.row_blocks; p.N = c.N; p.np = l.np; p.nz = l.nz;
  int jobs = 0;
  const auto add = [&](const void* x, bool x_mn, int np, const void* y, int64_t y_rows, int64_t rows, int64_t length) -> Job& {
    if (!make_map(&p.x[jobs], x, l.nz, c.M, np, l.nz, q.plane, x_mn ? BL : BM) || !make_map(&p.y[jobs], y, c.K, y_rows, 1, l.kp, y_rows * l.kp, BL))
      e = cudaErrorInvalidValue;
    Job& j = p.job[jobs++];
    j.x_mn = x_mn;
    j.pieces = np;
    j.rows = rows;
    j.cols = c.K;
    j.l_blocks = (int)((length + BL - 1) / BL);
    j.r_tiles = (rows + BM - 1) / BM;
    j.halves = 1;
    return j;
  };
  if (l.pieces_a) {
    Job& j = add(q.za, false, l.pieces_a, q.bw, l.nz, c.M, l.nz);
    j.out[0] = c.grad_a;
    j.alpha[0] = c.sb_per_col || c.gated ? nullptr : c.sb;
  }
  if (l.pieces_b) {
    Job& j = add(q.zb, true, l.pieces_b, q.aw, c.M, c.N, c.M);
    j.out[0] = c.grad_b;
    j.out[1] = c.grad_b2;
    j.alpha[0] = j.alpha[1] = c.sa_per_row ? nullptr : c.sa;
    j.halves = halves;
    j.half = l.np;
  }
  if (e != cudaSuccess) return e;

  // Tile width: the fewest rounds of tiles over the SMs, each round weighted by what a step of such a tile takes
  const int sms = multiprocessors();
  const auto tiles = [&](int bn) {
    p.tiles = p.tiles0 = 0;
    for (int i = 0; i < jobs; ++i) {
      p.job[i].s_tiles = (c.K + bn - 1) / bn;
      p.tiles += p.job[i].s_tiles * p.job[i].r_tiles * p.job[i].halves;
      if (i == 0) p.tiles0 = p.tiles;
    }
    return p.tiles;
  };
  const int widths[3] = {256, 128, 64};
  const double cost[3] = {1.0, 0.58, 0.4};
  int best = 0;
  double least = 1e300;
  for (int i = 0; i < 3; ++i) {
    const double t = (double)((tiles(widths[i]) + sms - 1) / sms) * cost[i];
    if (t < least) {
      least = t;
      best = i;
    }
  }
  tiles(widths[best]);
  return best == 0 ? launch_products<256>(p, sms, stream) : best == 1 ? launch_products<128>(p, sms, stream) : launch_products<64>(p, sms, stream);
}

}  // namespace lba
