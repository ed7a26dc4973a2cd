// Backward pass of the linear and gated layers under the straight-through estimator: the quantisers pass the gradient, so
//
//   dz = drop(g) act'(z)                              linear
//   dz = g v act'(z), dv = g act(z)                   gated (z, v the two projections; both stand side by side below)
//   grad_a[m][k] = sum_n dz[m][n] sb[n] B[n][k]       grad_b[n][k] = sum_m dz[m][n] sa[m] A[m][k]       grad_bias[n] = sum_m dz[m][n]
//
// Nothing rounds between additions here, so the products run on the tensor cores.  Codes of either operand format have at most
// five significant bits: bfloat16 holds them exactly, and only dz is rounded, to at least twice the result's significant bits: two
// bfloat16 pieces beside bfloat16 gradients (off by 2^-15 of it at most), three beside binary16 and binary32 ones (dz exactly); fewer
// where dz itself has no more bits (see pieces()).  Every piece costs one more pass of the matrix instruction.
//
// Scales that differ by row or column belong to the summed index of one of the products: dz is multiplied by both scales' fractions
// in [1, 2) before it is rounded, and the other product divides its rows by the one that it does not want.  So both read the same pieces.
// The powers of two go into the codes' bfloat16 forms, which stay exact: dz keeps its range (the scale of a row of zeros is often the
// smallest normal number, whose product with dz would have no bits left), and a scale of 0 gives zeros.
//
// Two launches (few rows: one, in lba_grad_few.cu):
//   grad_prepare_kernel   reads g and z once; writes the pieces of scaled dz, the sums of dz over blocks of rows (for the bias) and both
//                         operands' codes as bfloat16.  Bound by memory.
//   grad_product_kernel   both products as one list of 256 x 256 tiles, a pair of CTAs each (tcgen05, TMA), cut into equal shares of work;
//                         and the bias sums' last step.
#include "lba_grad.cuh"

#include <cstring>

#include "lba_async.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

constexpr int PREP_COLS = 256, PREP_THREADS = 256, PREP_SIDE = 8 * PREP_THREADS / PREP_COLS;  // PREP_SIDE: rows beside each other in a block
// A thread takes eight columns of every eighth row of its block.  The bytes of its next rows are on their way to shared memory while it
// computes one: under load a fetch takes 2000 clocks, so an SM wants 50 KB and more in flight (4096 x 4096 in bfloat16 took 21 us with a
// row ahead in registers).  Blocks are as tall as makes them one wave, so that what a block does but once (indexes, scales, the sums'
// last step, a third of all instructions with four rows a thread) weighs little.
__host__ __device__ constexpr int prep_depth(int bytes) { return 4 * PREP_THREADS * bytes <= 48 * 1024 ? 4 : 2; }
constexpr int PREP_RESIDENT = 4;  // blocks that an SM holds, as a rule
typedef __nv_bfloat16 bf16;

struct PrepParams {
  const void *grad, *pre;
  const uint8_t *A, *B, *B2;
  const float *sa, *sb, *sb2;  // scales in dz and the codes: by row; by column or by half (null: none)
  const uint64_t* rng;
  bf16 *z, *aw, *bw;         // pieces of dz (planes of `plane` elements), codes of A and B
  float* partial;            // [row blocks][nz] sums of dz
  uint32_t* flags;           // words that the second kernel wants at zero
  int64_t M, N, K, np, nz, kp, plane;
  int pieces;                // 0: no product is wanted
  int act, in_m4e3, sb_per_col, flag_words, each;
  uint32_t drop_below;
  int z_blocks, col_blocks, a_blocks;  // blocks of dz, then of A's codes, then of B's
};

template <typename T> struct Raw8;  // eight elements as they lie in memory
template <> struct Raw8<float> { float4 v[2]; };
template <> struct Raw8<bf16> { uint4 v; };
template <> struct Raw8<__half> { uint4 v; };
// sends for eight neighbouring elements, `valid` of which exist; they arrive in this thread's slot (one in every PREP_THREADS sixteen
// bytes).  whole: all eight, at a 16-byte boundary
template <typename T>
__device__ __forceinline__ void send_for8(uint4* slot, const T* src, bool whole, int valid) {
  if (whole) {
#pragma unroll
    for (int q = 0; q < (int)sizeof(T) / 2; ++q)
      asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_u32(slot + q * PREP_THREADS)), "l"(reinterpret_cast<const uint4*>(src) + q) : "memory");
  } else {
    constexpr int PER = 16 / (int)sizeof(T);
#pragma unroll
    for (int q = 0; q < 8 / PER; ++q) {
      T* const dst = reinterpret_cast<T*>(slot + q * PREP_THREADS);
#pragma unroll
      for (int j = 0; j < PER; ++j) dst[j] = q * PER + j < valid ? src[q * PER + j] : from_f32<T>(0.0f);
    }
  }
}
template <typename T>
__device__ __forceinline__ bool whole8(const void* base, int64_t pitch, int valid) {
  return valid == 8 && ((reinterpret_cast<uintptr_t>(base) | (uintptr_t)(pitch * sizeof(T))) & 15) == 0;
}
template <typename T>
__device__ __forceinline__ Raw8<T> arrived8(const uint4* slot) {
  Raw8<T> r;
  uint4* const v = reinterpret_cast<uint4*>(&r);
#pragma unroll
  for (int q = 0; q < (int)sizeof(T) / 2; ++q) v[q] = slot[q * PREP_THREADS];
  return r;
}
template <typename T>
__device__ __forceinline__ void widen8(const Raw8<T>& r, u64 (&v)[4]) {
  if constexpr (std::is_same<T, bf16>::value) {
    const uint32_t* const w = reinterpret_cast<const uint32_t*>(&r);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack2u(w[j] << 16, w[j] & 0xFFFF0000u);
  } else {
    const T* const e = reinterpret_cast<const T*>(&r);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack2(to_f32(e[2 * j]), to_f32(e[2 * j + 1]));
  }
}

// a scale s > 0 as 2^e f, 1 <= f < 2 (0 and subnormal numbers: 0 f)
__device__ __forceinline__ float fraction_of(float s) { return __uint_as_float((__float_as_uint(s) & 0x007FFFFFu) | 0x3F800000u); }
__device__ __forceinline__ float power_of(float s) { return __uint_as_float(__float_as_uint(s) & 0x7F800000u); }

// v as the sum of bfloat16 pieces, all but the last cut toward zero (which cannot overflow and leaves an exact remainder)
__device__ __forceinline__ void store_pieces(bf16* dst, int64_t plane, int pieces, const u64 (&v)[4]) {
  uint4 out;
  uint32_t* const w = &out.x;
  if (pieces > 1) {
    float rest[8];
#pragma unroll
    for (int j = 0; j < 4; ++j) unpack2(v[j], rest[2 * j], rest[2 * j + 1]);
#pragma unroll 1
    for (int q = 0; q + 1 < pieces; ++q) {
#pragma unroll
      for (int j = 0; j < 8; j += 2) {
        uint32_t h[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const float r = rest[j + e];
          h[e] = r != r ? 0x7FC00000u : __float_as_uint(r) & 0xFFFF0000u;  // (a NaN's payload may lie in what is cut)
          rest[j + e] = isfinite(r) ? r - __uint_as_float(h[e]) : 0.0f;
        }
        w[j / 2] = __byte_perm(h[0], h[1], 0x7632);
      }
      *reinterpret_cast<uint4*>(dst + q * plane) = out;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(rest[2 * j], rest[2 * j + 1]);
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      float lo, hi;
      unpack2(v[j], lo, hi);
      const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
      w[j] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  *reinterpret_cast<uint4*>(dst + (pieces - 1) * plane) = out;
}

__device__ __forceinline__ void expand_codes(const PrepParams& p, const uint8_t* row, bf16* dst, int64_t k, u64 power) {
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
        unpack2(mul2_rn(v[e], power), lo, hi);
        w[2 * q + e] = __byte_perm(__float_as_uint(lo), __float_as_uint(hi), 0x7632);  // exact: the low halves are zero
      }
    }
  }
  *reinterpret_cast<uint4*>(dst + k) = out;
}

template <typename G, typename Z, bool GATED>
__global__ void __launch_bounds__(PREP_THREADS, GATED ? 3 : 4) grad_prepare_kernel(const PrepParams p) {
  constexpr int HALVES = GATED ? 2 : 1;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  // The second kernel's CTAs may be set up as SMs run out of these: they are let in when the last of these has started, and wait for
  // the end of all (its shared memory does not fit beside these)
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  after_previous();
  int b = blockIdx.x;
  if (b == 0)
    for (int i = threadIdx.x; i < p.flag_words; i += PREP_THREADS) p.flags[i] = 0u;
  if (b >= p.z_blocks) {  // codes: a warp takes a row at a time
    b -= p.z_blocks;
    const bool is_a = b < p.a_blocks;
    const int64_t row = (int64_t)(is_a ? b : b - p.a_blocks) * 8 + warp;
    const uint8_t* src = nullptr;
    const float* scale = nullptr;
    bf16* dst;
    if (is_a) {
      if (row >= p.M) return;
      src = p.A + row * p.K;
      if (p.sa) scale = p.sa + row;
      dst = p.aw + row * p.kp;
    } else {
      if (row >= p.nz) return;
      const int64_t n = row < p.np ? row : row - p.np;
      if (n < p.N) {
        src = (row < p.np ? p.B : p.B2) + n * p.K;
        scale = row < p.np ? p.sb : p.sb2;
        if (scale && p.sb_per_col) scale += n;
      }
      dst = p.bw + row * p.kp;  // (rows of the padding: zeros)
    }
    const u64 power = both(scale ? power_of(*scale) : 1.0f);
    for (int64_t k = lane * 8; k < p.kp; k += 256) expand_codes(p, src, dst, k, power);
    return;
  }

  constexpr int G_SLOTS = sizeof(G) / 2, Z_SLOTS = sizeof(Z) / 2, ROW_SLOTS = (G_SLOTS + HALVES * Z_SLOTS) * PREP_THREADS;
  constexpr int DEPTH = prep_depth(16 * ROW_SLOTS / PREP_THREADS);
  __shared__ uint4 store[DEPTH * ROW_SLOTS];
  static_assert(sizeof(store) >= HALVES * PREP_THREADS * 8 * 4 && sizeof(store) <= 48 * 1024, "the sums of the rows take its place");
  const int row_block = b / p.col_blocks, col_block = b - row_block * p.col_blocks;  // (64-bit divisions here had been a third of all instructions)
  const int64_t n = (int64_t)col_block * PREP_COLS + lane * 8, m0 = (int64_t)row_block * (PREP_SIDE * p.each) + warp;
  const int valid = n >= p.N ? 0 : p.N - n < 8 ? (int)(p.N - n) : 8;
  u64 total[HALVES][4];
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < 4; ++j) total[h][j] = 0ull;
  if (n < p.np && m0 < p.M) {
    const bool reads_z = GATED || p.act != ACT_NONE;
    const int64_t left = (p.M - m0 + PREP_SIDE - 1) / PREP_SIDE;
    const int rows = left < p.each ? (int)left : p.each;
    const int64_t pitch = PREP_SIDE * p.N;
    const G* gp = static_cast<const G*>(p.grad) + m0 * p.N + n;
    const Z* zp = static_cast<const Z*>(p.pre) + m0 * p.N + n;
    const bool g_whole = whole8<G>(p.grad, p.N, valid), z_whole = whole8<Z>(p.pre, p.N, valid) && (!GATED || p.M * p.N * sizeof(Z) % 16 == 0);
    uint4* slot = store + threadIdx.x;
    const auto send = [&](bool there) {  // for the next row, into the current slot
      if (there) {
        send_for8(slot, gp, g_whole, valid);
        if (reads_z) {
#pragma unroll
          for (int h = 0; h < HALVES; ++h) send_for8(slot + (G_SLOTS + h * Z_SLOTS) * PREP_THREADS, zp + h * p.M * p.N, z_whole, valid);
        }
        gp += pitch;
        zp += pitch;
      }
      asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < DEPTH; ++i, slot += ROW_SLOTS) send(i < rows);
    slot = store + threadIdx.x;
    u64 scale[HALVES][4];
#pragma unroll
    for (int h = 0; h < HALVES; ++h) {
      const float* const sb = h ? p.sb2 : p.sb;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        scale[h][j] = !sb ? both(1.0f)
                      : !p.sb_per_col ? both(fraction_of(sb[0]))
                                      : pack2(2 * j < valid ? fraction_of(sb[n + 2 * j]) : 0.0f, 2 * j + 1 < valid ? fraction_of(sb[n + 2 * j + 1]) : 0.0f);
    }
    with_act(p.act, [&](auto act_tag) {
      constexpr int ACT = decltype(act_tag)::value;
      constexpr bool READS_Z = GATED || ACT != ACT_NONE;
      bf16* out = p.z + m0 * p.nz + n;
      int64_t m = m0;
      // (a rolled loop: a straight run of four rows is 3000 instructions that each warp fetches once; 32 x 512 took 18 us)
#pragma unroll 1
      for (int i = 0; i < rows; ++i, m += PREP_SIDE, out += PREP_SIDE * p.nz) {
        asm volatile("cp.async.wait_group %0;" ::"n"(DEPTH - 1) : "memory");
        u64 gv[4], zv[4], d[HALVES][4];
        widen8(arrived8<G>(slot), gv);
        if (READS_Z) widen8(arrived8<Z>(slot + G_SLOTS * PREP_THREADS), zv);
        if (!GATED && p.drop_below) {
          const uint64_t seed = p.rng[0], offset = p.rng[1];
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint4 r = philox((uint32_t)(n >> 2) + h, (uint32_t)m, offset, seed);
            float lo, hi;
            unpack2(gv[2 * h], lo, hi);
            gv[2 * h] = pack2(r.x < p.drop_below ? 0.0f : lo, r.y < p.drop_below ? 0.0f : hi);
            unpack2(gv[2 * h + 1], lo, hi);
            gv[2 * h + 1] = pack2(r.z < p.drop_below ? 0.0f : lo, r.w < p.drop_below ? 0.0f : hi);
          }
        }
        [[maybe_unused]] u64 other[4];
        if constexpr (GATED) widen8(arrived8<Z>(slot + (G_SLOTS + Z_SLOTS) * PREP_THREADS), other);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          u64 value, slope;
          if (READS_Z) act_pair<ACT>(zv[j], value, slope);
          if constexpr (GATED) {
            d[0][j] = mul2_rn(mul2_rn(gv[j], other[j]), slope);
            d[HALVES - 1][j] = mul2_rn(gv[j], value);
          } else if (ACT == ACT_RELU) {  // (an infinite gradient stays out where the slope is 0)
            float glo, ghi, slo, shi;
            unpack2(gv[j], glo, ghi);
            unpack2(slope, slo, shi);
            d[0][j] = pack2(slo != 0.0f ? glo : 0.0f, shi != 0.0f ? ghi : 0.0f);
          } else {
            d[0][j] = ACT == ACT_NONE ? gv[j] : mul2_rn(gv[j], slope);
          }
        }
        // (the padding of a row: g is 0 there, z too, and every slope finite)
        const u64 by = both(p.sa ? fraction_of(p.sa[m]) : 1.0f);
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          u64 s[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            total[h][j] = add2_rn(total[h][j], d[h][j]);
            s[j] = mul2_rn(d[h][j], scale[h][j]);
          }
          if (p.sa) {
#pragma unroll
            for (int j = 0; j < 4; ++j) s[j] = mul2_rn(s[j], by);
          }
          if (p.pieces) store_pieces(out + h * p.np, p.plane, p.pieces, s);
        }
        send(i + DEPTH < rows);
        slot += ROW_SLOTS;
        if (slot >= store + DEPTH * ROW_SLOTS) slot -= DEPTH * ROW_SLOTS;
      }
    });
  }
  if (!p.partial) return;
  __syncthreads();  // `store` is free
  float* const sums = reinterpret_cast<float*>(store);  // [half][warp][column]
#pragma unroll
  for (int h = 0; h < HALVES; ++h)
#pragma unroll
    for (int j = 0; j < 4; j += 2)
      *reinterpret_cast<ulonglong2*>(&sums[(h * (PREP_THREADS / 32) + warp) * PREP_COLS + lane * 8 + 2 * j]) = make_ulonglong2(total[h][j], total[h][j + 1]);
  __syncthreads();
  const int64_t col = (int64_t)col_block * PREP_COLS + threadIdx.x;
  if (col >= p.np) return;
#pragma unroll
  for (int h = 0; h < HALVES; ++h) {
    float s = 0.0f;
#pragma unroll
    for (int w = 0; w < PREP_THREADS / 32; ++w) s += sums[(h * (PREP_THREADS / 32) + w) * PREP_COLS + threadIdx.x];
    p.partial[row_block * p.nz + h * p.np + col] = s;
  }
}

// ------------------------------------------------------------------ products
// out[r][s] = alpha sum_l X[r][l] Y[l][s] over the pieces of X.
//   grad_a: r = m, l = n, s = k; X's rows are contiguous in l (K-major)
//   grad_b: r = n, l = m, s = k; X is read from the same layout, contiguous in r (MN-major); so is Y, contiguous in s, in both
// A cluster of two CTAs forms a 256 x 256 tile: each CTA holds 128 rows of X, half of Y's columns and the accumulators of its rows, and
// one thread of the first issues the matrix instructions of both (cta_group::2).  What bounds such a product is what the L2 can
// deliver: a CTA alone with 128 x 256 outputs fetched 48 KB per 64 l where this takes 32 (4096 x 4096 x 1024, one piece of dz: 82 us
// alone against 53; two pieces 92, 87 % of the tensor pipe).
// Ten warps a CTA: one thread loads, one multiplies into one of two accumulators of 256 columns of tensor memory, eight warps bring the
// other one out.  A step is 512 clocks of the tensor cores, so its loads must take the one thread less: two copies with three- and
// four-dimensional boxes and no arithmetic but the coordinates' (three copies and 64-bit divisions in a lane chosen by its number had
// taken 725).
//
// Clusters take whole tiles in turn, side by side in l, so that what one fetches its neighbours find in L2.  The last tiles of the list
// are divided where that saves time (layout() says when): their steps of 64 l stand in one row, cut into equal shares, one per
// cluster.  A tile that a border cuts is begun by lower shares, which leave binary32 sums in the workspace, and finished by the share with
// its last step, which adds them in order.  A cluster walks its share from the end and before its whole tiles, and takes the share's number
// from a counter when it starts: it only ever waits for clusters that run already or have ended, for the first thing that those do.
// `longest`: binary32 results of long sums would lose precision to the matrix instructions, which cut a sum at each addition (8192
// terms were off by 2.8e-6, where 1000 are by 8e-7).  Their tiles are formed in stretches, added up in binary32.
// A wait that runs out ends in NaN, never in sums that miss a step.  Inside a pair it stops the copies and products of both CTAs (`dead`, set
// in both): what either brings out from there on is NaN, and parts of tiles that it hands over are marked as lost.  A tile with a lost part, or
// with one that was not handed over in time (`missed`), becomes NaN.
constexpr int BM = 128, BN = 256, BL = 64, GRAD_THREADS = 320, OUT_THREADS = 256;  // of a CTA: rows, columns, step
constexpr int X_BYTES = BM * BL * 2, STAGE = 2 * X_BYTES, STAGES = 5;
constexpr int OUT_PITCH = 36;         // floats from row to row of a warp's outputs in shared memory: 128 bytes, 16-byte accesses on all banks
constexpr size_t PRODUCT_SMEM = 1024 + (size_t)STAGE * STAGES + 256 + OUT_THREADS * OUT_PITCH * 4;
constexpr int PART_FLOATS = BM * BN;  // a CTA's part of a begun tile
enum PartFlag : uint32_t { PART_THERE = 1, PART_LOST = 2 };
enum WaitOverride { WAIT_AS_IT_IS = 0, WAIT_NO_PART = 1, WAIT_NO_OPERANDS = 2, WAIT_NO_SUMS = 3 };  // lba_set_wait_override

struct Job {
  int64_t rows, cols;       // of one half's output
  int r_tiles, s_tiles;     // r_tiles: of one half
  int half;                 // blocks of 64 before the second half's first in X
  int x_mn, pieces, blocks, steps;  // blocks of l, and these times pieces
  int div_stride;
  void* out[2];
  const float *alpha[2], *div[2];  // factors of a half, scales whose fractions divide its rows (or null)
};
struct ProductParams {
  CUtensorMap x[2], y[2];
  Job job[2];
  int tiles0, tiles;        // of the first job, of both
  int whole;                // tiles that stay whole, the first ones
  int units0, units, first; // with shares: steps of the first job, of both, those before the divided ones
  int share;                // steps of a cluster's share; 0: there are none
  int longest;              // steps that the matrix instructions add up before binary32 additions take over (all, if none is meant)
  int out_type;
  int wait_override;
  float factor;
  uint32_t* flags;          // shares: the counter, then a word per CTA's part
  float *parts, *sums;      // parts of begun tiles, and sums of a CTA's steps so far: PART_FLOATS each per CTA
  const float* partial;     // bias: [row blocks][nz]
  float* bias[2];
  int64_t row_blocks, N, np, nz;
};

__device__ __forceinline__ uint32_t mapa(uint32_t addr, int rank) {
  uint32_t d;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
  return d;
}
// a box of blocks of 64 columns: columns of block b, rows from y on, plane z; counted by a barrier of either CTA of the pair
__device__ __forceinline__ void tma_load(uint32_t dst, const CUtensorMap* map, int y, int b, int z, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(dst), "l"(map), "r"(0), "r"(y), "r"(b), "r"(z), "r"(bar) : "memory");
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
// (orders nothing but the arrival: what it follows, reads of tensor memory, has its own fence, and a release would wait for the
// outputs' stores)
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// a wait of this pair ran out: both CTAs know
__device__ __forceinline__ void give_up(volatile int* dead, int rank) {
  *dead = 1;
  asm volatile("st.relaxed.cluster.shared::cluster.u32 [%0], %1;" ::"r"(mapa(smem_u32(const_cast<int*>(dead)), rank ^ 1)), "r"(1) : "memory");
}
// waits for another CTA's part of a tile; false where it is lost, or not there in time
__device__ __forceinline__ bool part_there(const uint32_t* flag, volatile int* missed) {
  uint32_t v = 0;
  wait_until([&] {
    asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(flag) : "memory");
    if (!v) __nanosleep(64);
    return v != 0;
  }, missed);
  return v == PART_THERE;
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
  int r, s, start;  // first row tile (of the half) and column tile, the tile's first step among all
  bool goes_on, last;  // k0 to k1 are not the first, are the last steps of this piece
  int from, to;        // its steps
};
struct Walk {
  int at, end, tile, by;  // steps [end, at) of the share are left; the next whole tile, the number of clusters
  __device__ __forceinline__ Walk(const ProductParams& p, int c, int clusters) {
    tile = c;
    by = clusters;
    end = at = 0;
    if (p.share) {
      end = p.first + c * p.share;
      at = end + p.share < p.units ? end + p.share : p.units;
    }
  }
  __device__ __forceinline__ void stretch(const ProductParams& p, Work& w) {
    w.last = w.to - w.k0 <= p.longest;
    w.k1 = w.last ? w.to : w.k0 + p.longest;
  }
  __device__ __forceinline__ bool next(const ProductParams& p, Work& w) {
    if (!w.last) {  // more of the same piece
      w.k0 = w.k1;
      w.goes_on = true;
      stretch(p, w);
      return true;
    }
    int t;
    if (at > end) {
      w.job = at - 1 >= p.units0;
      const int steps = p.job[w.job].steps, base = w.job ? p.units0 : 0;
      t = (at - 1 - base) / steps;
      w.start = base + t * steps;
      w.to = at - w.start;
      w.from = end > w.start ? end - w.start : 0;
      at = w.start + w.from;
    } else {
      if (tile >= p.whole) return false;
      w.job = tile >= p.tiles0;
      t = w.job ? tile - p.tiles0 : tile;
      w.from = 0;
      w.to = p.job[w.job].steps;
      w.start = 0;
      tile += by;
    }
    const Job& j = p.job[w.job];
    const int row = t / j.s_tiles;
    w.s = t - row * j.s_tiles;
    w.half = row >= j.r_tiles;
    w.r = w.half ? row - j.r_tiles : row;
    w.k0 = w.from;
    w.goes_on = false;
    stretch(p, w);
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

// Outputs leave through shared memory, 128 bytes of a row at a time: a warp's 32 rows, a row per lane there, four rows per store of
// the warp to memory.  (A row per lane straight to memory had each store touch 32 rows: with rows of 1203 floats, where nothing is
// aligned, 1000 x 777 x 1203 took 42 us for its products.)
template <typename T> constexpr int OUT_COLS = 128 / (int)sizeof(T);
// 32 columns of this lane's row, from column 32 `half` of the 128 bytes on
template <typename T>
__device__ __forceinline__ void stage_row(float* row, int half, const float (&v)[32], float alpha) {
  if constexpr (sizeof(T) == 4) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      reinterpret_cast<float4*>(row)[i] = make_float4(v[4 * i] * alpha, v[4 * i + 1] * alpha, v[4 * i + 2] * alpha, v[4 * i + 3] * alpha);
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      T t[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) t[q] = from_f32<T>(v[8 * i + q] * alpha);
      uint4 raw;
      memcpy(&raw, t, 16);
      reinterpret_cast<uint4*>(row)[4 * half + i] = raw;
    }
  }
}
// `rows` and `cols` of them to rows of `pitch` elements
template <typename T>
__device__ __forceinline__ void store_rows(T* out, int64_t pitch, int rows, int cols, const float* sm, int lane) {
  if (pitch * sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0 && cols == OUT_COLS<T>) {
    uint4* dst = reinterpret_cast<uint4*>(out + (lane / 8) * pitch) + lane % 8;
    const uint4* src = reinterpret_cast<const uint4*>(sm + (lane / 8) * OUT_PITCH) + lane % 8;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const uint4 raw = src[i * OUT_PITCH];  // four rows on: 4 OUT_PITCH floats
      if (i * 4 + lane / 8 < rows) *dst = raw;
      dst += pitch * sizeof(T) / 4;
    }
  } else {
#pragma unroll 1
    for (int c = lane; c < cols; c += 32) {
      T* dst = out + c;
#pragma unroll 8
      for (int i = 0; i < rows; ++i) {
        *dst = reinterpret_cast<const T*>(sm + i * OUT_PITCH)[c];
        dst += pitch;
      }
    }
  }
}

__global__ void __launch_bounds__(GRAD_THREADS, 1) grad_product_kernel(const __grid_constant__ ProductParams p) {
  extern __shared__ unsigned char product_raw[];
  unsigned char* const base = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(product_raw) + 1023) & ~(uintptr_t)1023);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(base + STAGES * STAGE);  // full, empty per stage; done, free per accumulator; the last products
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * STAGES + 5);
  volatile int *const dead = reinterpret_cast<volatile int*>(tmem_slot + 1), *const missed = dead + 1;
  uint32_t* const share_slot = tmem_slot + 3;
  float* const outs = reinterpret_cast<float*>(base + STAGES * STAGE + 256);  // 32 x 32 of each warp that brings outputs out
  __shared__ float part[4][32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = blockIdx.x & 1;  // in the cluster
  const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, acc_done = empty + 8 * STAGES, acc_free = acc_done + 16,
                 last_done = acc_free + 16;

  if (threadIdx.x == 0) {
    for (int i = 0; i < STAGES; ++i) {
      mbar_init(full + 8 * i, 1);   // the first CTA's counts both CTAs' bytes
      mbar_init(empty + 8 * i, 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(acc_done + 8 * i, 1);
      mbar_init(acc_free + 8 * i, 2 * OUT_THREADS / 32);  // the first CTA's: both CTAs' reading warps
    }
    mbar_init(last_done, 1);
    *dead = *missed = 0;
    mbar_init_fence();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(2 * BN) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  if (warp == 2 && lane < 4) {
    const CUtensorMap* const map = lane < 2 ? &p.x[lane] : &p.y[lane - 2];
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
  }
  __syncwarp();
  if (p.share) cluster_sync();  // the other CTA runs: its memory may be written
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
  const int share = p.share ? (int)*share_slot : blockIdx.x >> 1;
  Walk walk(p, share, gridDim.x >> 1);
  const int runs_out = p.wait_override == WAIT_NO_PART || (blockIdx.x >> 1) % 3 == 1 ? p.wait_override : WAIT_AS_IT_IS;
  Work w;
  w.last = true;

  if (warp == 0) {
    if (elected()) {
      int stage = 0;
      uint32_t phase = 1;
      bool alive = true;
      const uint32_t stages = smem_u32(base), bars0 = mapa(full, 0);  // the first CTA's
      while (alive && walk.next(p, w)) {
        const Job& j = p.job[w.job];
        const CUtensorMap *const xm = &p.x[w.job], *const ym = &p.y[w.job];
        const int x_mn = j.x_mn, blocks = j.blocks;
        const int r = w.r * (2 * BM) + rank * BM, rb = r / 64 + (w.half ? j.half : 0), sb = w.s * (BN / 64) + rank * (BN / 128);
        // the last piece first: the matrix instructions cut their sums, so what is small is added up before what is large (all pieces of
        // a step together had tripled the error of binary32 results)
        int q = w.k0 / blocks, l = w.k0 - q * blocks;
        q = j.pieces - 1 - q;
#pragma unroll 1
        for (int k = w.k0; k < w.k1; ++k) {
          if (!mbar_wait(empty + 8 * stage, phase, dead)) {
            give_up(dead, rank);
            alive = false;
            break;
          }
          const uint32_t x = stages + stage * STAGE, bar = bars0 + 8 * stage;
          if (rank == 0) mbar_arrive_expect(full + 8 * stage, 2 * STAGE);
          if (x_mn) tma_load(x, xm, l * BL, rb, q, bar);
          else tma_load(x, xm, r, l, q, bar);
          tma_load(x + X_BYTES, ym, l * BL, sb, 0, bar);
          if (++l == blocks) {
            l = 0;
            --q;
          }
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
          }
        }
      }
    }
  } else if (warp == 1) {
    if (rank == 0 && elected()) {
      int stage = 0, acc = 0;
      uint32_t phase = 0, acc_phase = 1;
      bool alive = true;
      const uint32_t stages = smem_u32(base);
      while (alive && walk.next(p, w)) {
        const int x_mn = p.job[w.job].x_mn;
        // binary32 sums of bfloat16 products; which operand is MN-major; sizes
        const uint32_t idesc = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)x_mn << 15) | (1u << 16) | ((BN / 8) << 17) | ((2 * BM / 16) << 24);
        // operands of a stage at address 0; a step of 16 l is 2048 bytes on where l counts lines, 32 where it counts within one
        const uint64_t x0 = x_mn ? operand(0, X_BYTES / 2, 1024) : operand(0, 16, 1024), y0 = operand(0, X_BYTES / 2, 1024);
        const uint32_t xk = x_mn ? 2048 >> 4 : 32 >> 4;
        alive = mbar_wait_cluster(acc_free + 8 * acc, acc_phase, dead);
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        bool add = false;
#pragma unroll 1
        for (int b = w.k0; alive && b < w.k1; ++b) {
          if (!mbar_wait_cluster(full + 8 * stage, phase, dead) || runs_out == WAIT_NO_OPERANDS) {
            alive = false;
            break;
          }
          asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
          const uint32_t x = (stages + stage * STAGE) >> 4, y = x + (X_BYTES >> 4);
#pragma unroll
          for (int k = 0; k < BL / 16; ++k) {
            mma(tmem + acc * BN, x0 + x + k * xk, y0 + y + k * (2048 >> 4), idesc, add);
            add = true;
          }
          mma_commit(empty + 8 * stage);
          if (++stage == STAGES) {
            stage = 0;
            phase ^= 1;
          }
        }
        if (!alive) {  // (the sums never count as done: whoever waits for them gives up too)
          give_up(dead, rank);
          break;
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
    const int row = quarter * 32 + lane, c_first = warp < 6 ? 0 : BN / 2;
    const bool leader = threadIdx.x == 64;
    float* const sm = outs + (warp - 2) * (32 * OUT_PITCH);
    if (p.partial && warp < 6) bias_sums(p, part, quarter, lane);
    int acc = 0;
    uint32_t phase = 0;
    while (walk.next(p, w)) {
      const Job& j = p.job[w.job];
      const bool begins = w.last && w.to < j.steps, ends = w.last && w.from > 0 && !begins;
      const int first = ends ? (w.start - p.first) / p.share : share;  // the shares that began this tile: first to share - 1
      if (ends) {
        if (leader)  // (one tile of a cluster's walk at most: `missed` is about that one)
          for (int c = first; c < share; ++c)
            if (runs_out == WAIT_NO_PART || !part_there(p.flags + 1 + 2 * c + rank, missed)) *missed = 1;
        asm volatile("bar.sync 2, 256;" ::: "memory");
      }
      const int64_t r0 = (int64_t)w.r * (2 * BM) + rank * BM + quarter * 32, r = r0 + lane;
      float alpha = p.factor * (j.alpha[w.half] ? *j.alpha[w.half] : 1.0f);
      if (j.div[w.half] && r < j.rows) alpha = __fdiv_rn(alpha, fraction_of(j.div[w.half][r * j.div_stride]));
      if (runs_out == WAIT_NO_SUMS || !mbar_wait(acc_done + 8 * acc, phase, dead)) give_up(dead, rank);
      __syncwarp();
      asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
      if (*dead || (ends && *missed)) alpha = __uint_as_float(0x7FC00000u);
      float4* const mine = reinterpret_cast<float4*>(p.parts + (2 * (int64_t)share + rank) * PART_FLOATS) + row;  // [four columns][row]
      float4* const sums = reinterpret_cast<float4*>(p.sums + (int64_t)blockIdx.x * PART_FLOATS) + row;
      const int rows = j.rows - r0 < 32 ? (int)(j.rows - r0 > 0 ? j.rows - r0 : 0) : 32;
      const int64_t s0 = (int64_t)w.s * BN, pitch = j.cols;
      void* const out = j.out[w.half];
      const bool mine_too = lane < rows;  // (rows behind the last one are never read)
      const auto add = [&](float (&v)[32], const float4* from, int c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float4 f = __ldcg(from + (c / 4 + i) * BM);
          v[4 * i] += f.x;
          v[4 * i + 1] += f.y;
          v[4 * i + 2] += f.z;
          v[4 * i + 3] += f.w;
        }
      };
      const auto keep = [&](const float (&v)[32], float4* to, int c) {
#pragma unroll
        for (int i = 0; i < 8; ++i) __stcg(to + (c / 4 + i) * BM, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
      };
      const auto bring_out = [&](auto type_tag) {
        typedef decltype(type_tag) T;
#pragma unroll 1
        for (int c0 = c_first; c0 < c_first + BN / 2; c0 += OUT_COLS<T>) {
          if (s0 + c0 >= pitch) break;
#pragma unroll
          for (int half = 0; half < OUT_COLS<T> / 32; ++half) {
            const int c = c0 + 32 * half;
            uint32_t t[32];
            float v[32];
            tmem_ld32(tmem + ((uint32_t)(quarter * 32) << 16) + acc * BN + c, t);
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(t[i]);
            if (w.goes_on && mine_too) add(v, sums, c);
            if (!w.last) {  // (read by this thread alone)
              if (mine_too) keep(v, sums, c);
            } else if (begins) {
              if (mine_too) keep(v, mine, c);
            } else {
              if (mine_too) {
#pragma unroll 2  // (two shares' sums on their way at a time)
                for (int o = first; o < share; ++o) add(v, reinterpret_cast<const float4*>(p.parts + (2 * (int64_t)o + rank) * PART_FLOATS) + row, c);
              }
              stage_row<T>(sm + lane * OUT_PITCH, half, v, alpha);
            }
          }
          if (w.last && !begins) {
            __syncwarp();
            const int64_t left = pitch - (s0 + c0);
            store_rows(static_cast<T*>(out) + r0 * pitch + s0 + c0, pitch, rows, left < OUT_COLS<T> ? (int)left : OUT_COLS<T>, sm, lane);
            __syncwarp();
          }
        }
      };
      if (rows > 0) {
        if (p.out_type == LT_F32) bring_out(float());
        else if (p.out_type == LT_BF16) bring_out(bf16());
        else bring_out(__half());
      }
      asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive_cluster(mapa(acc_free + 8 * acc, 0));
      if (begins) {
        __threadfence();
        asm volatile("bar.sync 2, 256;" ::: "memory");
        if (leader)
          asm volatile("st.release.gpu.global.u32 [%0], %1;" ::"l"(p.flags + 1 + 2 * share + rank), "r"((uint32_t)(*dead ? PART_LOST : PART_THERE)) : "memory");
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
  if (*dead) {     // (the same in both CTAs) ... but what was sent before a wait ran out
    if (warp == 1 && rank == 0 && elected()) {
      asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(last_done) : "memory");
      *missed = 0;
      mbar_wait(last_done, 0, missed);
    }
    if (warp == 0) let_copies_land();
    __syncwarp();
    cluster_sync();
  }
  if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(2 * BN) : "memory");
}

// ------------------------------------------------------------------ host
int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }
size_t up256(size_t v) { return (v + 255) / 256 * 256; }

// bfloat16 pieces that dz takes beside a result of the given type: at least twice the result's significant bits, 8 and 11, whatever the
// sizes.  With as many bits as the result's own, dz's rounding is as large as the result's in sums of any length (terms of either sign grow
// and their errors grow alike): gradients in bfloat16 were off by 1.41 times as much as with dz in binary32, single ones by twice.  dz that is
// g itself or zero has no more bits than g, and a common scale is applied to the finished product.
int pieces(const GradCall& c) {
  const bool plain = !c.gated && (c.act == ACT_NONE || c.act == ACT_RELU) && !c.sa_per_row && !c.sb_per_col;
  const int wanted = c.out_type == LT_BF16 ? 2 : 3, held = c.grad_type == LT_BF16 ? 1 : c.grad_type == LT_F16 ? 2 : 3;
  return plain && held < wanted ? held : wanted;
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
  int64_t tiles[2], units[2], whole, share, first;
  int steps[2], at_a, at_b, clusters, each, longest;  // at_a, at_b: each product's place in the list
  size_t z, aw, bw, partial, flags, parts, sums, total;
};
Layout layout(const GradCall& c) {
  Layout l = {};
  const int halves = c.gated ? 2 : 1;
  const bool a = c.grad_a && c.K > 0, b = c.grad_b && c.K > 0;
  l.np = up(c.N, 64);  // whole blocks of the copies' 64 columns
  l.nz = l.np * halves;
  l.kp = up(c.K, 64);
  l.pieces = a || b ? pieces(c) : 0;
  const auto blocks = [](int64_t n, int64_t by) { return (n + by - 1) / by; };
  const int64_t most = clusters_of_the_device();
  l.each = (int)blocks(blocks(c.M, PREP_SIDE) * blocks(l.np, PREP_COLS), 2 * most * PREP_RESIDENT);
  l.each = l.each < 1 ? 1 : l.each > 64 ? 64 : l.each;
  l.row_blocks = blocks(c.M, PREP_SIDE * l.each);
  // the product with shorter sums first: long tiles are the ones to divide
  const int64_t steps_a = blocks(l.nz, BL) * l.pieces, steps_b = blocks(c.M, BL) * l.pieces;
  l.at_a = !a ? -1 : b && steps_b < steps_a ? 1 : 0;
  l.at_b = !b ? -1 : l.at_a == 0 ? 1 : 0;
  if (a) {
    l.steps[l.at_a] = (int)steps_a;
    l.tiles[l.at_a] = blocks(c.M, 2 * BM) * blocks(c.K, BN);
  }
  if (b) {
    l.steps[l.at_b] = (int)steps_b;
    l.tiles[l.at_b] = halves * blocks(c.N, 2 * BM) * blocks(c.K, BN);
  }
  for (int i = 0; i < 2; ++i) l.units[i] = l.tiles[i] * l.steps[i];
  // How many tiles stay whole: all, or some, the others in equal shares.  In steps, a tile takes at least EPILOGUE (bringing it out hides
  // behind the next one's steps), so shorter tiles are never divided (1 x 4096 x 4096 89 us otherwise, 45 like this).  A share costs beside
  // its own steps what its begun sums take to be written and waited for, less where whole tiles follow, and the finishing cluster
  // JOIN for each share that it adds: a tile must not be cut too often.  All tiles whole and like this, us (dz in one piece): 256 x 8192 x 512 gated
  // 91.5 and 55.3 (94 with 26 shares a tile), 8192 x 512 x 512 51.2 and 35.8, 6000 x 4096 x 1024 106.7 and 98.6, 4096 x 4096 x 1024
  // 71.2 and 70.9.
  constexpr int64_t EPILOGUE = 16, CUT = 30, CUT_BEFORE_WHOLE = 14, JOIN = 5;
  const int64_t all = l.tiles[0] + l.tiles[1], units = l.units[0] + l.units[1];
  const auto steps_of = [&](int64_t tile) { return (int64_t)(tile < l.tiles[0] ? l.steps[0] : l.steps[1]); };
  const auto steps_before = [&](int64_t tile) { return tile < l.tiles[0] ? tile * l.steps[0] : l.units[0] + (tile - l.tiles[0]) * l.steps[1]; };
  if (all > 0) {
    const auto cost_of = [&](int64_t tile) { return steps_of(tile) > EPILOGUE ? steps_of(tile) : EPILOGUE; };
    const auto load = [&](int64_t whole) {  // of the busiest cluster, whose tile is the last of every round
      if (whole == 0) return (int64_t)0;
      const int64_t rounds = blocks(whole, most), in_first = (whole < l.tiles[0] ? whole : l.tiles[0]) / most;
      return in_first * cost_of(0) + (rounds > in_first ? (rounds - in_first - 1) * cost_of(all - 1) + cost_of(whole - 1) : 0);
    };
    const int64_t longest = steps_of(all - 1), fewest = l.steps[0] < EPILOGUE ? l.tiles[0] : 0;  // whole tiles, at least
    l.whole = all;
    int64_t least = load(all);
    const auto consider = [&](int64_t whole) {
      if (whole < fewest || whole >= all || longest < EPILOGUE || units >= (1ll << 31)) return;
      int64_t even = blocks(units - steps_before(whole), most);
      while (even < 8 || even * even < JOIN * longest) ++even;
      const int64_t time = load(whole) + even + (whole > 0 ? CUT_BEFORE_WHOLE : CUT) + JOIN * blocks(longest, even);
      if (time < least) {
        least = time;
        l.whole = whole;
        l.share = even;
      }
    };
    for (int64_t whole = all / most * most, tries = 0; whole >= 0 && tries < 8; whole -= most, ++tries) consider(whole);
    consider(fewest);
    l.first = steps_before(l.whole);
    // every cluster has a share or a whole tile
    const int64_t shares = l.share ? blocks(units - l.first, l.share) : 0, wholes = l.whole < most ? l.whole : most;
    l.clusters = (int)(shares > wholes ? shares : wholes);
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
  const int most_steps = l.steps[0] > l.steps[1] ? l.steps[0] : l.steps[1];
  constexpr int LONGEST = 16;
  l.longest = c.out_type == LT_F32 && most_steps > LONGEST ? LONGEST : 2147483647;
  l.sums = take(l.longest < most_steps ? (size_t)l.clusters * 2 * PART_FLOATS * 4 : 0);
  l.total = at;
  return l;
}

// planes x rows x pitch / 64 blocks of 64 columns of bfloat16; boxes of `box_blocks` blocks of `box_rows` rows, 128-byte swizzle
bool make_map(CUtensorMap* map, const void* base, int64_t rows, int64_t planes, int64_t pitch, int64_t plane, int box_rows, int box_blocks) {
  const EncodeTiled encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)pitch / 64, (cuuint64_t)planes};
  const cuuint64_t strides[3] = {(cuuint64_t)pitch * 2, 128, (cuuint64_t)plane * 2};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, (cuuint32_t)box_blocks, 1}, step[4] = {1, 1, 1, 1};
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
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

size_t backward_workspace(const GradCall& c) { return c.M > 0 && c.N > 0 && !few_rows(c, pieces(c)) ? layout(c).total : 0; }

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
  if (few_rows(c, pieces(c))) return launch_backward_few(c, pieces(c), stream);
  const Layout l = layout(c);
  const bool a = l.at_a >= 0, b = l.at_b >= 0;
  if (!a && !b && !c.grad_bias) return cudaSuccess;
  if (l.tiles[0] + l.tiles[1] > 2147483647LL) return cudaErrorInvalidValue;
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
  q.each = l.each;
  q.M = c.M; q.N = c.N; q.K = c.K; q.np = l.np; q.nz = l.nz; q.kp = l.kp;
  q.plane = c.M * l.nz;
  q.pieces = l.pieces;
  q.act = c.act; q.in_m4e3 = c.in_m4e3; q.sb_per_col = c.sb_per_col;
  q.drop_below = c.drop_below;
  const int64_t col_blocks = (l.np + PREP_COLS - 1) / PREP_COLS, z_blocks = col_blocks * l.row_blocks, a_blocks = b ? (c.M + 7) / 8 : 0;
  const int64_t blocks = z_blocks + a_blocks + (a ? (l.nz + 7) / 8 : 0);
  if (blocks > 2147483647LL) return cudaErrorInvalidValue;
  q.col_blocks = (int)col_blocks;
  q.z_blocks = (int)z_blocks;
  q.a_blocks = (int)a_blocks;

  ProductParams p = {};
  p.out_type = c.out_type;
  p.wait_override = c.wait_override;
  p.factor = c.keep_scale;
  p.partial = q.partial;
  p.bias[0] = c.grad_bias; p.bias[1] = c.grad_bias2;
  p.row_blocks = l.row_blocks; p.N = c.N; p.np = l.np; p.nz = l.nz;
  p.flags = q.flags;
  p.parts = reinterpret_cast<float*>(ws + l.parts);
  p.sums = reinterpret_cast<float*>(ws + l.sums);
  p.longest = l.longest;
  p.whole = (int)l.whole;
  p.share = (int)l.share;
  p.tiles0 = (int)l.tiles[0];
  p.tiles = (int)(l.tiles[0] + l.tiles[1]);
  p.units0 = (int)l.units[0];
  p.units = (int)(l.units[0] + l.units[1]);
  p.first = (int)l.first;
  // (a job without tiles is never looked at: the first one's borders are both 0 then)
  const auto add = [&](int i, bool x_mn, const void* y, int64_t y_rows, int64_t rows) -> Job& {
    if (!make_map(&p.x[i], q.z, c.M, l.pieces, l.nz, q.plane, x_mn ? BL : BM, x_mn ? BM / 64 : 1) ||
        !make_map(&p.y[i], y, y_rows, 1, l.kp, y_rows * l.kp, BL, BN / 128))
      e = cudaErrorInvalidValue;
    Job& j = p.job[i];
    j.x_mn = x_mn;
    j.pieces = l.pieces;
    j.blocks = l.steps[i] / l.pieces;
    j.steps = l.steps[i];
    j.rows = rows;
    j.cols = c.K;
    j.r_tiles = (int)((rows + 2 * BM - 1) / (2 * BM));
    j.s_tiles = (int)((c.K + BN - 1) / BN);
    return j;
  };
  if (a) {
    Job& j = add(l.at_a, false, q.bw, l.nz, c.M);
    j.out[0] = c.grad_a;
    j.alpha[0] = q.sb ? nullptr : c.sb;
    j.div[0] = q.sa;
    j.div_stride = 1;
  }
  if (b) {
    Job& j = add(l.at_b, true, q.aw, c.M, c.N);
    j.out[0] = c.grad_b;
    j.out[1] = c.grad_b2;
    j.alpha[0] = j.alpha[1] = q.sa ? nullptr : c.sa;
    j.div[0] = q.sb;
    j.div[1] = c.sb2;
    j.div_stride = c.sb_per_col;
    j.half = (int)(l.np / 64);
  }
  if (e != cudaSuccess) return e;
  e = cudaFuncSetAttribute(grad_product_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)PRODUCT_SMEM);
  if (e != cudaSuccess) return e;
  e = c.grad_type == LT_F32 ? launch_prepare<float>(q, c, (unsigned)blocks, stream)
      : c.grad_type == LT_BF16 ? launch_prepare<bf16>(q, c, (unsigned)blocks, stream) : launch_prepare<__half>(q, c, (unsigned)blocks, stream);
  if (e != cudaSuccess) return e;
  int64_t clusters = l.clusters;
  if (!p.share && c.grad_bias) {  // more CTAs for the bias: they find no tile
    const int64_t wanted = (l.nz + 63) / 64, most = clusters_of_the_device();
    if (clusters < wanted) clusters = wanted < most ? wanted : most;
  }
  return launch_after(grad_product_kernel, dim3((unsigned)(2 * clusters)), GRAD_THREADS, PRODUCT_SMEM, stream, p, 2);
}

}  // namespace lba
