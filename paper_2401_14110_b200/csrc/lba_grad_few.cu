// Backward pass of the layers for few rows (the formulas are lba_grad.cu's), in one launch without a workspace.
//
// With M rows of activations the weights are read once and their gradients written once: N K bytes and 2 or 4 N K.  Products of M
// columns are too thin for 256 x 256 tiles, and bringing the weights to bfloat16 in memory first is 4 bytes more for each (one row,
// 4096 x 4096, bfloat16: 44 us in two launches).  Here a weight goes from memory to a register, becomes bfloat16 there and is an
// operand of mma.m16n8k16, whose 16 rows are the activations'; dz is formed again by every CTA for the block of columns that it
// needs, M elements per column, and kept in shared memory.  Three kinds of CTAs, by their number:
//   A  grad_a: 16 rows m and 128 columns k, several times; the eight CTAs of a cluster and their eight warps share out the sum over n, 16 at a time and
//      warp; the 64 sums are added in a fixed order, through shared memory and then through the cluster's.
//   B  grad_b: 128 to 1024 rows n and 64 to 512 columns k, the activations' codes brought to bfloat16 in shared memory.
//   C  grad_bias: 128 n.
// The order in which a fragment's rows and columns are numbered is free as long as both operands agree, so a lane's share of a fragment is
// made of neighbours in memory: 16 bytes of four weight rows, 16 columns of grad_a, eight of grad_b.  Loops stay rolled where they can: a
// launch this short meets each instruction for the first time (with both products' loops unrolled 32 x 8192 x 2048 took 88 us).
#include "lba_grad.cuh"

#include "lba_async.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

typedef __nv_bfloat16 bf16;
constexpr int FEW_THREADS = 256, BLOCK = 128, CLUSTER = 8, MOST_BLOCKS = 8;  // columns n of dz: in blocks; B: up to MOST_BLOCKS times tiles in a CTA
constexpr int RED_PITCH = 132;                // floats from row to row of a warp's sums: 16-byte accesses on all banks
constexpr int RED_FLOATS = 8 * 8 * RED_PITCH;  // eight warps' sums of eight rows
constexpr int OUT_PITCH = 36;                 // of a warp's 16 x 32 outputs
constexpr int FEW_ROWS = 64;
constexpr size_t MOST_SMEM = 220 * 1024, SUMS_BYTES = (RED_FLOATS + 16 * 128) * 4;
enum Kind { GRAD_A, GRAD_B, GRAD_BIAS };
// elements from row to row of dz or of activations in shared memory: an odd number of 16-byte words
__host__ __device__ constexpr int pitch_of(int cols) { return cols + 8; }

struct FewParams {
  const void *grad, *pre;
  const uint8_t *A, *B[2];
  const float *sa, *sb[2];          // scales by row, by column or half: multiplied into dz (null: they are `alpha`)
  const float *alpha_a, *alpha_b;   // common scales of the finished products (or null)
  const uint64_t* rng;
  void *out_a, *out_b[2];
  float* bias[2];
  int64_t M, N, K;
  int grad_type, pre_type, out_type, act, gated, in_m4e3, sb_per_col, pieces;
  uint32_t drop_below;
  float factor;
  int blocks, all, tiles;              // blocks of n in a half, in all; tiles of 16 rows
  int a_ctas, b_ctas, a_each, b_each;  // CTAs; blocks of n of a CTA (A: of a cluster's)
  int a_times, red_at;                 // A: groups of 128 columns of a CTA, one after the other; where the warps' sums lie (bytes)
  int b_width, b_cols;                 // B: columns k of a CTA, CTAs side by side
  int n_whole;                         // eight elements of a row always lie whole at a 16-byte boundary
};

struct Raw { uint4 v[2]; };  // eight elements as they lie in memory
// Loads that a launch can tell to be whole stand in a path of their own, side by side: behind a branch for each of them every load waited
// for the one before (1 x 8192 x 512: 25 us for grad_a)
__device__ __forceinline__ void load8_whole(Raw& r, const void* base, int type, int64_t at) {
  const uint4* const src = reinterpret_cast<const uint4*>(static_cast<const unsigned char*>(base) + at * (type == LT_F32 ? 4 : 2));
  r.v[0] = __ldg(src);
  if (type == LT_F32) r.v[1] = __ldg(src + 1);
}
__device__ __forceinline__ void load8(Raw& r, const void* base, int type, int64_t at, int valid) {
  uint32_t* const w = &r.v[0].x;
  if (type == LT_F32) {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) w[j] = __ldg(static_cast<const uint32_t*>(base) + at + j);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < valid) w[j / 2] |= (uint32_t)__ldg(static_cast<const uint16_t*>(base) + at + j) << (16 * (j & 1));
  }
}
__device__ __forceinline__ void widen(const Raw& r, int type, u64 (&v)[4]) {
  const uint32_t* const w = &r.v[0].x;
  if (type == LT_BF16) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack2u(w[j] << 16, w[j] & 0xFFFF0000u);
  } else if (type == LT_F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = pack2u(w[2 * j], w[2 * j + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w[j]));
      v[j] = pack2(f.x, f.y);
    }
  }
}

// What a thread reads for eight neighbouring elements of dz
struct Inputs {
  Raw g, z, v, by;
  int64_t n;
  int m, half, valid;
};
__device__ __forceinline__ Inputs fetch(const FewParams& p, Kind kind, int block, int m, int n8) {
  Inputs in;
  in.half = block >= p.blocks;
  in.n = (int64_t)(block - (in.half ? p.blocks : 0)) * BLOCK + 8 * n8;
  in.m = m;
  in.valid = in.n >= p.N ? 0 : p.N - in.n < 8 ? (int)(p.N - in.n) : 8;
  in.g = in.z = in.v = in.by = Raw{make_uint4(0u, 0u, 0u, 0u), make_uint4(0u, 0u, 0u, 0u)};
  if (in.valid) {
    const int64_t at = m * p.N + in.n;
    const bool reads_z = p.gated || p.act != ACT_NONE, reads_by = kind == GRAD_A && p.sb_per_col;
    if (p.n_whole) {
      load8_whole(in.g, p.grad, p.grad_type, at);
      if (reads_z) load8_whole(in.z, p.pre, p.pre_type, at);
      if (p.gated) load8_whole(in.v, p.pre, p.pre_type, p.M * p.N + at);
      if (reads_by) load8_whole(in.by, p.sb[in.half], LT_F32, in.n);
    } else {
      load8(in.g, p.grad, p.grad_type, at, in.valid);
      if (reads_z) load8(in.z, p.pre, p.pre_type, at, in.valid);
      if (p.gated) load8(in.v, p.pre, p.pre_type, p.M * p.N + at, in.valid);
      if (reads_by) load8(in.by, p.sb[in.half], LT_F32, in.n, in.valid);
    }
  }
  return in;
}
__device__ __forceinline__ void slopes(const FewParams& p, const Inputs& in, u64 (&d)[4]) {
  u64 g[4], z[4], v[4];
  widen(in.g, p.grad_type, g);
  widen(in.z, p.pre_type, z);
  widen(in.v, p.pre_type, v);
  if (p.drop_below) {
    const uint64_t seed = p.rng[0], offset = p.rng[1];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint4 r = philox((uint32_t)(in.n >> 2) + h, (uint32_t)in.m, offset, seed);
      float lo, hi;
      unpack2(g[2 * h], lo, hi);
      g[2 * h] = pack2(r.x < p.drop_below ? 0.0f : lo, r.y < p.drop_below ? 0.0f : hi);
      unpack2(g[2 * h + 1], lo, hi);
      g[2 * h + 1] = pack2(r.z < p.drop_below ? 0.0f : lo, r.w < p.drop_below ? 0.0f : hi);
    }
  }
  with_act(p.act, [&](auto act_tag) {
    constexpr int ACT = decltype(act_tag)::value;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      u64 value, slope;
      act_pair<ACT>(z[j], value, slope);
      if (p.gated) {
        d[j] = in.half ? mul2_rn(g[j], value) : mul2_rn(mul2_rn(g[j], v[j]), slope);
      } else if (ACT == ACT_RELU) {  // (an infinite gradient stays out where the slope is 0)
        float glo, ghi, slo, shi;
        unpack2(g[j], glo, ghi);
        unpack2(slope, slo, shi);
        d[j] = pack2(slo != 0.0f ? glo : 0.0f, shi != 0.0f ? ghi : 0.0f);
      } else {
        d[j] = ACT == ACT_NONE ? g[j] : mul2_rn(g[j], slope);
      }
    }
  });
}
// d as the sum of bfloat16 pieces, all but the last cut toward zero (which cannot overflow and leaves an exact remainder); pieces are
// `plane` elements apart
__device__ __forceinline__ void put_pieces(bf16* dst, int plane, int pieces, const u64 (&d)[4]) {
  float rest[8];
#pragma unroll
  for (int j = 0; j < 4; ++j) unpack2(d[j], rest[2 * j], rest[2 * j + 1]);
  uint4 out;
  uint32_t* const w = &out.x;
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
  *reinterpret_cast<uint4*>(dst + (pieces - 1) * plane) = out;
}

// Two codes in the upper bytes of two halves as bfloat16 (the lower bytes: anything).  E4M3: the bits in bfloat16's places are the value
// times 2^-120.  M4E3: every exponent is a normal one, and no magnitude bits mean 0.
template <bool M4E3>
__device__ __forceinline__ uint32_t decode_pair(uint32_t y) {
  if (M4E3) {
    const uint32_t mag = (y >> 5) & 0x03F803F8u, some = ((mag + 0x7FFF7FFFu) >> 15) & 0x00010001u;
    return ((mag + 0x3F803F80u) & (some * 0xFFFFu)) | (y & 0x80008000u);
  }
  uint32_t out;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(out) : "r"(((y >> 4) & 0x07F007F0u) | (y & 0x80008000u)), "r"(0x7B807B80u));  // 2^120
  return out;
}
// pairs of column c of four columns in two rows (lower half: r0)
template <bool M4E3, int C>
__device__ __forceinline__ uint32_t decode_rows(uint32_t r0, uint32_t r1) {
  return decode_pair<M4E3>(__byte_perm(r0, r1, C == 0 ? 0x4400 : C == 1 ? 0x5511 : C == 2 ? 0x6622 : 0x7733));
}
__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void load_fragment(uint32_t addr, uint32_t (&a)[4]) {
  if (TRANS)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr) : "memory");
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(a[0]), "=r"(a[1]), "=r"(a[2]), "=r"(a[3]) : "r"(addr) : "memory");
}
// 16 bytes of a row from byte k on, whatever lies behind the row's end at `end`
__device__ __forceinline__ uint4 row_bytes16(const uint8_t* row, int64_t k, int64_t end) {
  uint4 out = make_uint4(0u, 0u, 0u, 0u);
  if (k >= end) return out;
  const uint8_t* const src = row + k;
  const uint32_t* const at = reinterpret_cast<const uint32_t*>(reinterpret_cast<uintptr_t>(src) & ~(uintptr_t)3);
  const uint32_t shift = (reinterpret_cast<uintptr_t>(src) & 3) * 8;
  uint32_t w[5];
#pragma unroll
  for (int i = 0; i < 5; ++i) w[i] = reinterpret_cast<const uint8_t*>(at + i) < row + end ? __ldg(at + i) : 0u;  // (words with a byte of the row)
  uint32_t* const o = &out.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) o[i] = __funnelshift_r(w[i], w[i + 1], shift);
  return out;
}
__device__ __forceinline__ void store_one(void* out, int type, int64_t at, float v) {
  if (type == LT_F32) static_cast<float*>(out)[at] = v;
  else if (type == LT_BF16) static_cast<bf16*>(out)[at] = from_f32<bf16>(v);
  else static_cast<__half*>(out)[at] = from_f32<__half>(v);
}
__device__ __forceinline__ void few_cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 peer_float4(uint32_t addr, int rank) {
  uint32_t d;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(d) : "r"(addr), "r"(rank));
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(d) : "memory");
  return v;
}

// dz of `count` blocks, rows m from m0 on, into shared memory: pieces of it times the scales of n or m, or (for the bias) itself
__device__ __forceinline__ void put_blocks(const FewParams& p, Kind kind, int block, int count, int m0, int rows, int pitch, int plane, unsigned char* dst) {
  // (sixteen threads side by side; the others go down the rows of block after block, without a division per step)
  const int n8 = threadIdx.x % (BLOCK / 8), first = threadIdx.x / (BLOCK / 8), by_blocks = 16 / rows, by_rows = 16 - by_blocks * rows;
  static_assert(FEW_THREADS / (BLOCK / 8) == 16, "steps of 16 rows");
  int b = first / rows, row = first - b * rows;
  if (b >= count) return;
  Inputs in = fetch(p, kind, block + b, m0 + row, n8);
#pragma unroll 1
  while (true) {
    const int here = row, col = b * (BLOCK / 8) + n8;
    b += by_blocks;
    row += by_rows;
    if (row >= rows) {
      row -= rows;
      ++b;
    }
    const bool more = b < count;
    Inputs next = in;
    if (more) next = fetch(p, kind, block + b, m0 + row, n8);
    u64 d[4] = {0ull, 0ull, 0ull, 0ull};
    if (in.valid) {
      slopes(p, in, d);
      if (kind == GRAD_A && p.sb[in.half]) {
        u64 by[4];
        widen(in.by, LT_F32, by);
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = mul2_rn(d[j], p.sb_per_col ? by[j] : both(p.sb[in.half][0]));
      }
      if (kind == GRAD_B && p.sa) {
        const u64 by = both(p.sa[in.m]);
#pragma unroll
        for (int j = 0; j < 4; ++j) d[j] = mul2_rn(d[j], by);
      }
    }
    if (kind == GRAD_BIAS) {
      ulonglong2* const to = reinterpret_cast<ulonglong2*>(reinterpret_cast<float*>(dst) + here * RED_PITCH + 8 * col);
      to[0] = make_ulonglong2(d[0], d[1]);
      to[1] = make_ulonglong2(d[2], d[3]);
    } else {
      put_pieces(reinterpret_cast<bf16*>(dst) + here * pitch + 8 * col, plane, p.pieces, d);
    }
    if (!more) return;
    in = next;
  }
}

// B: the codes of columns k0 to k0 + width - 1 of all rows as bfloat16; column 8 u + 2 i + e of each 32 stands at 8 i + 2 u + e
template <bool M4E3, bool WHOLE>
__device__ __forceinline__ void put_activations(const FewParams& p, int64_t k0, bf16* to) {
  const int across = p.b_width / 16;
#pragma unroll 2
  for (int o = threadIdx.x; o < p.tiles * 16 * across; o += FEW_THREADS) {
    const int m = o / across, c = (o - m * across) * 16;
    uint4 raw = make_uint4(0u, 0u, 0u, 0u);
    if (WHOLE) {
      if (m < p.M && k0 + c < p.K) raw = __ldg(reinterpret_cast<const uint4*>(p.A + m * p.K + k0 + c));
    } else if (m < p.M) {
      raw = row_bytes16(p.A + m * p.K, k0 + c, p.K);
    }
    uint32_t* const dst = reinterpret_cast<uint32_t*>(to + m * pitch_of(p.b_width) + (c & ~31)) + (c & 16) / 8;
#pragma unroll
    for (int q = 0; q < 4; ++q) {  // four columns: half of u = (c % 32) / 8 + q / 2
      const uint32_t w = (&raw.x)[q];
      dst[4 * (2 * (q & 1)) + q / 2] = decode_pair<M4E3>(__byte_perm(w, 0u, 0x1100));
      dst[4 * (2 * (q & 1) + 1) + q / 2] = decode_pair<M4E3>(__byte_perm(w, 0u, 0x3322));
    }
  }
}

// B: this warp's 16 x 32 outputs, row by row
template <typename T>
__device__ __forceinline__ void store_staged(T* out, int64_t pitch, int rows, int64_t cols, const float* sm, int lane) {
  if (lane >= cols) return;
#pragma unroll 8
  for (int r = 0; r < rows; ++r) out[r * pitch + lane] = from_f32<T>(sm[r * OUT_PITCH + lane]);
}
template <typename T>
__device__ __forceinline__ void bring_out(T* out, const FewParams& p, int64_t n, int64_t k, const float (&sum)[4][4], float alpha, float* sm, int lane) {
  const int g = lane >> 2, t = lane & 3;
  const bool whole = k + 32 <= p.K && p.K * sizeof(T) % 16 == 0 && (reinterpret_cast<uintptr_t>(out) & 15) == 0;
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = sum[q / 2][2 * r + (q & 1)] * alpha;
    if (whole) {
      constexpr int WORDS = (int)sizeof(T) / 2;
      uint4 raw[WORDS];
      if constexpr (std::is_same<T, bf16>::value) {  // (two a conversion)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * j], v[2 * j + 1]);
          (&raw[0].x)[j] = *reinterpret_cast<const uint32_t*>(&b);
        }
      } else {
        T* const e = reinterpret_cast<T*>(raw);
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = from_f32<T>(v[j]);
      }
      uint4* const dst = reinterpret_cast<uint4*>(out + (n + g + 8 * r) * p.K + k + 8 * t);
      if (n + g + 8 * r < p.N) {
#pragma unroll
        for (int q = 0; q < WORDS; ++q) dst[q] = raw[q];
      }
    } else {
      float4* const dst = reinterpret_cast<float4*>(sm + (g + 8 * r) * OUT_PITCH + 8 * t);
      dst[0] = make_float4(v[0], v[1], v[2], v[3]);
      dst[1] = make_float4(v[4], v[5], v[6], v[7]);
    }
  }
  if (!whole) {  // (a lane's eight columns straight to memory: 8 x 1001 x 777 took 34 us)
    __syncwarp();
    store_staged(out + n * p.K + k, p.K, p.N - n < 16 ? (int)(p.N - n) : 16, p.K - k, sm, lane);
    __syncwarp();
  }
}

// WHOLE: 16 codes of a row always lie whole at a 16-byte boundary
template <bool M4E3, bool WHOLE>
__global__ void __launch_bounds__(FEW_THREADS, 2) grad_few_kernel(const __grid_constant__ FewParams p) {
  extern __shared__ __align__(16) unsigned char smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, t = lane & 3, rank = blockIdx.x % CLUSTER;
  const Kind kind = (int)blockIdx.x < p.a_ctas ? GRAD_A : (int)blockIdx.x < p.a_ctas + p.b_ctas ? GRAD_B : GRAD_BIAS;  // (whole clusters)
  after_previous();
  // what this CTA forms: blocks of n from `c` to `end`, columns k from k0 on, rows m from m0 on
  int c, end, m0 = 0, tiles = p.tiles;
  int64_t k0 = 0;
  if (kind == GRAD_A) {
    const int cluster = blockIdx.x / CLUSTER, cols = p.a_ctas / (CLUSTER * p.tiles), tile = cluster / cols;
    k0 = (int64_t)(cluster - tile * cols) * (128 * p.a_times);
    m0 = tile * 16;
    tiles = 1;
    c = rank * p.a_each;
    end = c + p.a_each;
  } else if (kind == GRAD_B) {
    const int id = blockIdx.x - p.a_ctas, down = id / p.b_cols;
    c = down * p.b_each;
    end = c + p.b_each;
    k0 = (int64_t)(id - down * p.b_cols) * p.b_width;
  } else {
    c = blockIdx.x - p.a_ctas - p.b_ctas;
    end = c + 1;
  }
  end = end < p.all ? end : p.all;
  const int rows = p.M - m0 < tiles * 16 ? (int)p.M - m0 : tiles * 16;
  const int pitch = pitch_of((kind == GRAD_A ? p.a_each : p.b_each) * BLOCK), plane = tiles * 16 * pitch;
  bf16* const z = reinterpret_cast<bf16*>(smem);
  bf16* const activations = z + plane * p.pieces;

  if (kind == GRAD_B) {
    if (c >= end) return;  // (the last cluster's rest)
    put_activations<M4E3, WHOLE>(p, k0, activations);
    for (int row = rows + warp; row < tiles * 16; row += FEW_THREADS / 32)  // (zeros behind the last row, which are summed)
      for (int piece = 0; piece < p.pieces; ++piece)
        for (int o = lane; o < pitch / 8; o += 32) reinterpret_cast<uint4*>(z + piece * plane + row * pitch)[o] = make_uint4(0u, 0u, 0u, 0u);
    put_blocks(p, kind, c, end - c, 0, rows, pitch, plane, smem);
    __syncthreads();
    const float alpha = p.factor * (p.alpha_b ? *p.alpha_b : 1.0f);
    const int k_pitch = pitch_of(p.b_width), across = p.b_width / 32, bits = __ffs(across) - 1;  // (a power of two)
    const int units = (end - c) * (BLOCK / 16) << bits;
    float* const staged = reinterpret_cast<float*>(activations + tiles * 16 * k_pitch) + warp * 16 * OUT_PITCH;
    // matrices of a fragment, transposed: n 0-7 and 8-15 at m 0-7, the same at m 8-15; columns 0-7 at m 0-7 and 8-15, columns 8-15
    const uint32_t from = smem_u32(z) + 2 * (((lane & 7) + (lane >> 4) * 8) * pitch + (lane & 8));
    const uint32_t from_y = smem_u32(activations) + 2 * ((lane & 15) * k_pitch + (lane >> 4) * 8);
#pragma unroll 1
    for (int o = warp; o < units; o += FEW_THREADS / 32) {  // 16 n and 32 k
      const int s = o >> bits, j = o & (across - 1), block = c + s / (BLOCK / 16), half = block >= p.blocks;
      const int64_t n = (int64_t)(block - (half ? p.blocks : 0)) * BLOCK + s % (BLOCK / 16) * 16, k = k0 + 32 * j;
      if (n >= p.N || k >= p.K) continue;
      float sum[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[i][e] = 0.0f;
#pragma unroll 1
      for (int piece = p.pieces - 1; piece >= 0; --piece) {  // what is small is added up first
#pragma unroll 1
        for (int i = 0; i < tiles; ++i) {
          uint32_t a[4], y[2][4];
          load_fragment<true>(from + 2 * (piece * plane + i * 16 * pitch + 16 * s), a);
#pragma unroll
          for (int h = 0; h < 2; ++h) load_fragment<true>(from_y + 2 * (i * 16 * k_pitch + 32 * j + 16 * h), y[h]);
#pragma unroll
          for (int q = 0; q < 4; ++q) mma16816(sum[q], a, y[q / 2][2 * (q & 1)], y[q / 2][2 * (q & 1) + 1]);
        }
      }
      if (p.out_type == LT_F32) bring_out(static_cast<float*>(p.out_b[half]), p, n, k, sum, alpha, staged, lane);
      else if (p.out_type == LT_BF16) bring_out(static_cast<bf16*>(p.out_b[half]), p, n, k, sum, alpha, staged, lane);
      else bring_out(static_cast<__half*>(p.out_b[half]), p, n, k, sum, alpha, staged, lane);
    }
    return;
  }
  if (kind == GRAD_BIAS) {
    if (c >= end) return;
    put_blocks(p, kind, c, 1, 0, rows, 0, 0, smem);
    __syncthreads();
    const int half = c >= p.blocks;
    const int64_t n = (int64_t)(c - (half ? p.blocks : 0)) * BLOCK + threadIdx.x;
    if (threadIdx.x < BLOCK && n < p.N && p.bias[half]) {
      const float* const sums = reinterpret_cast<const float*>(smem);
      float sum = 0.0f;
      for (int m = 0; m < rows; ++m) sum += sums[m * RED_PITCH + threadIdx.x];
      p.bias[half][n] = sum * p.factor;
    }
    return;
  }

  uint4 next[4];
  const auto fetch_codes = [&](int block, int64_t k0) {
    const int half = block >= p.blocks;
    const int64_t n0 = (int64_t)(block - (half ? p.blocks : 0)) * BLOCK + 16 * warp + 2 * t;
    const uint8_t* const from = p.B[half] + n0 * p.K;
    const int64_t k = k0 + 16 * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) next[i] = make_uint4(0u, 0u, 0u, 0u);
    if (WHOLE) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int down = (i & 1) + 8 * (i >> 1);
        if (block < end && n0 + down < p.N && k < p.K) next[i] = __ldg(reinterpret_cast<const uint4*>(from + down * p.K + k));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int down = (i & 1) + 8 * (i >> 1);
        if (block < end && n0 + down < p.N) next[i] = row_bytes16(from + down * p.K, k, p.K);
      }
    }
  };
  fetch_codes(c, k0);
  if (c < end) put_blocks(p, kind, c, end - c, m0, rows, pitch, plane, smem);  // (rows behind the last one: anything, they meet no other)
  __syncthreads();
  float* const red = reinterpret_cast<float*>(smem + p.red_at);  // (in dz's place where no other group reads that)
  float* const sums = red + RED_FLOATS;  // [16][128]
  const float alpha = p.factor * (p.alpha_a ? *p.alpha_a : 1.0f);
#pragma unroll 1
  for (const int64_t k_end = k0 + 128 * p.a_times < p.K ? k0 + 128 * p.a_times : p.K; k0 < k_end; k0 += 128) {
    float acc[16][4];
#pragma unroll
    for (int j = 0; j < 16; ++j)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[j][e] = 0.0f;
    // matrices of a fragment: rows m 0-7 and 8-15 at n 0-7, the same at n 8-15
    uint32_t from = smem_u32(z) + 2 * (((lane & 7) + (lane & 8)) * pitch + 16 * warp + (lane >> 4) * 8);
#pragma unroll 1
    for (int b = c; b < end; ++b, from += 2 * BLOCK) {
      uint4 now[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) now[i] = next[i];
      if (b + 1 < end) fetch_codes(b + 1, k0);
      else if (k0 + 128 < k_end) fetch_codes(c, k0 + 128);
      uint32_t only[4];
      load_fragment<false>(from, only);
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const uint32_t r0 = (&now[0].x)[q], r1 = (&now[1].x)[q], r2 = (&now[2].x)[q], r3 = (&now[3].x)[q];
        const uint32_t b0[4] = {decode_rows<M4E3, 0>(r0, r1), decode_rows<M4E3, 1>(r0, r1), decode_rows<M4E3, 2>(r0, r1),
                                decode_rows<M4E3, 3>(r0, r1)};
        const uint32_t b1[4] = {decode_rows<M4E3, 0>(r2, r3), decode_rows<M4E3, 1>(r2, r3), decode_rows<M4E3, 2>(r2, r3),
                                decode_rows<M4E3, 3>(r2, r3)};
        if (p.pieces == 1) {
#pragma unroll
          for (int j = 0; j < 4; ++j) mma16816(acc[4 * q + j], only, b0[j], b1[j]);
        } else {
#pragma unroll 1
          for (int piece = p.pieces - 1; piece >= 0; --piece) {
            uint32_t a[4];
            load_fragment<false>(from + 2 * piece * plane, a);
#pragma unroll
            for (int j = 0; j < 4; ++j) mma16816(acc[4 * q + j], a, b0[j], b1[j]);
          }
        }
      }
    }

    // The warps' sums: lane (g, t) holds columns 32 t to 32 t + 31 of rows g and g + 8.  16-byte words are exchanged within eight, so that
    // lanes meet no bank twice
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      if (8 * r >= rows) break;
      __syncthreads();
      if (g + 8 * r < rows) {
#pragma unroll
        for (int s = 0; s < 8; ++s) {
          const int j = 4 * (s & 3), e = 2 * r + (s >> 2);
          *reinterpret_cast<float4*>(red + (warp * 8 + g) * RED_PITCH + 32 * t + 4 * (s ^ (2 * t))) = make_float4(acc[j][e], acc[j + 1][e], acc[j + 2][e], acc[j + 3][e]);
        }
      }
      __syncthreads();
      const int row = threadIdx.x >> 5, s = threadIdx.x & 31, at = (s & 24) + ((s & 7) ^ (2 * (s >> 3)));
      if (row + 8 * r < rows) {
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
        for (int w = 0; w < 8; ++w) {
          const float4 f = *reinterpret_cast<const float4*>(red + (w * 8 + row) * RED_PITCH + 4 * at);
          v.x += f.x;
          v.y += f.y;
          v.z += f.z;
          v.w += f.w;
        }
        reinterpret_cast<float4*>(sums)[(row + 8 * r) * 32 + s] = v;
      }
    }
    few_cluster_sync();
    // the cluster's: a CTA takes every eighth row
    if (warp < 2 && warp * CLUSTER + rank < rows) {
      const int row = warp * CLUSTER + rank;
      const uint32_t from = smem_u32(sums + row * 128 + 4 * lane);
      float4 f[CLUSTER];
#pragma unroll
      for (int r = 0; r < CLUSTER; ++r) f[r] = peer_float4(from, r);
      float v[4] = {f[0].x, f[0].y, f[0].z, f[0].w};
#pragma unroll
      for (int r = 1; r < CLUSTER; ++r) {
        v[0] += f[r].x;
        v[1] += f[r].y;
        v[2] += f[r].z;
        v[3] += f[r].w;
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (k0 + 4 * lane + j < p.K) store_one(p.out_a, p.out_type, (m0 + row) * p.K + k0 + 4 * lane + j, v[j] * alpha);
    }
    few_cluster_sync();  // the others have read this CTA's sums
  }
}

// of a cluster's CTA: dz of 16 rows and an eighth of all n
size_t dz_bytes(const GradCall& c, int pieces) {
  const int64_t all = (c.N + BLOCK - 1) / BLOCK * (c.gated ? 2 : 1), each = (all + CLUSTER - 1) / CLUSTER;
  return each > 1024 ? MOST_SMEM + 1 : (size_t)32 * pitch_of((int)each * BLOCK) * pieces;
}

}  // namespace

// Every 16 rows bring the weights and every 128 columns k the elementwise work of all rows once more, in more CTAs than run at a time where
// there are many of both; and dz of many columns n leaves room for one group of 128 k a CTA.  Both sides on 305 sizes of 16 to 64 rows, 512 to
// 8192 n and 256 to 4096 k, linear and gated, bfloat16 and binary32: the rule's choice takes 0.5 % more than the better side on
// average, 35 % at most (48 x 8192 x 256, gated: 54 us instead of 40; without the limit on n it is 81 %).  All gradients in bfloat16, GELU, scales per channel, us
// here and in two launches: 1 x 512 x 512 5.5 and 11.6, 4 x 8192 x 8192 89 and 153, 17 x 4096 x 4096 42 and 57, 32 x 2048 x 2048 18.8 and 27.7,
// 32 x 1024 x 4096 20.2 and 26.1, 48 x 4096 x 1024 25.0 and 30.2, 64 x 1024 x 1024 16.2 and 17.0, 64 x 4096 x 1024 29.6 and 30.9,
// 48 x 1024 x 2048 19.1 and 18.1, 64 x 2048 x 4096 46 and 32, 64 x 8192 x 1024 47.4 and 44.4, 64 x 4096 x 4096 130 and 55.
bool few_rows(const GradCall& c, int pieces) {
  if (c.M <= 0 || c.M > FEW_ROWS || c.N <= 0 || c.K <= 0) return false;
  const int64_t tiles = (c.M + 15) / 16;
  if (tiles > 1 && (tiles * tiles * c.K > 16384 || tiles * c.N * (c.gated ? 2 : 1) > 32768)) return false;
  return c.grad_a ? dz_bytes(c, pieces) <= MOST_SMEM : c.grad_b != nullptr;
}

cudaError_t launch_backward_few(const GradCall& c, int pieces, cudaStream_t stream) {
  FewParams p = {};
  p.grad = c.grad; p.pre = c.pre; p.A = c.A; p.B[0] = c.B; p.B[1] = c.B2;
  p.sa = c.sa_per_row ? c.sa : nullptr;
  p.sb[0] = c.sb_per_col || c.gated ? c.sb : nullptr;
  p.sb[1] = c.sb2;
  p.alpha_a = p.sb[0] ? nullptr : c.sb;
  p.alpha_b = p.sa ? nullptr : c.sa;
  p.rng = c.rng;
  p.out_a = c.grad_a; p.out_b[0] = c.grad_b; p.out_b[1] = c.grad_b2;
  p.bias[0] = c.grad_bias; p.bias[1] = c.grad_bias2;
  p.M = c.M; p.N = c.N; p.K = c.K;
  p.grad_type = c.grad_type; p.pre_type = c.pre_type; p.out_type = c.out_type;
  p.act = c.act; p.gated = c.gated; p.in_m4e3 = c.in_m4e3; p.sb_per_col = c.sb_per_col;
  p.pieces = pieces;
  p.drop_below = c.drop_below;
  p.factor = c.keep_scale;
  const auto up8 = [](int64_t v) { return (v + CLUSTER - 1) / CLUSTER * CLUSTER; };
  const int64_t blocks = (c.N + BLOCK - 1) / BLOCK, all = c.gated ? 2 * blocks : blocks;
  const int64_t tiles = (c.M + 15) / 16, a_cols = (c.K + 127) / 128;
  // A: no more clusters than run at a time, two CTAs an SM, so that dz is formed once by each (16 x 8192 x 8192, grad_a alone: 47 us
  // with 64 clusters), where dz can stay beside the sums
  const size_t dz = dz_bytes(c, pieces);
  const int64_t times = dz + SUMS_BYTES <= 112 * 1024 ? (a_cols * tiles + 35) / 36 : 1;
  const int64_t a_ctas = c.grad_a ? (a_cols + times - 1) / times * CLUSTER * tiles : 0;
  p.red_at = times > 1 ? (int)dz : 0;
  // B: wide CTAs, which form less of dz again, where there are enough of them; several blocks each where there are many
  int width = 512;
  const auto cols = [&] { return (c.K + width - 1) / width; };
  while (width > 64 && all * cols() < 148) width /= 2;
  int64_t each = all * cols() / (4 * 148);
  each = each < 1 ? 1 : each > MOST_BLOCKS / tiles ? MOST_BLOCKS / tiles : each;
  const int64_t b_ctas = c.grad_b ? up8((all + each - 1) / each * cols()) : 0;
  const int64_t ctas = a_ctas + b_ctas + (c.grad_bias ? up8(all) : 0);
  if (ctas > 2147483647LL) return cudaErrorInvalidValue;
  p.blocks = (int)blocks;
  p.all = (int)all;
  p.tiles = (int)tiles;
  p.a_ctas = (int)a_ctas;
  p.b_ctas = (int)b_ctas;
  p.a_times = (int)times;
  p.a_each = (int)((all + CLUSTER - 1) / CLUSTER);
  p.b_each = (int)each;
  p.b_width = width;
  p.b_cols = (int)cols();
  const auto aligned = [](const void* a) { return (reinterpret_cast<uintptr_t>(a) & 15) == 0; };  // (so is a null pointer)
  p.n_whole = c.N % 8 == 0 && aligned(c.grad) && aligned(c.pre) && aligned(c.sb) && aligned(c.sb2);
  const bool k_whole = c.K % 16 == 0 && aligned(c.A) && aligned(c.B) && aligned(c.B2);
  size_t smem = 0;
  const auto wants = [&smem](size_t bytes) { smem = smem > bytes ? smem : bytes; };
  if (a_ctas) {
    wants(p.red_at + SUMS_BYTES);
    wants(dz);
  }
  if (b_ctas) wants(tiles * 32 * ((size_t)pitch_of(BLOCK * (int)each) * pieces + pitch_of(width)) + FEW_THREADS / 32 * 16 * OUT_PITCH * 4);
  if (c.grad_bias) wants((size_t)tiles * 16 * RED_PITCH * 4);
  const auto launch = [&](auto kernel) {
    // (the same limit in every call: another thread's may lie between these two lines)
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)MOST_SMEM);
    return e != cudaSuccess ? e : launch_after(kernel, dim3((unsigned)ctas), FEW_THREADS, smem, stream, p, CLUSTER);
  };
  if (c.in_m4e3) return k_whole ? launch(grad_few_kernel<true, true>) : launch(grad_few_kernel<true, false>);
  return k_whole ? launch(grad_few_kernel<false, true>) : launch(grad_few_kernel<false, false>);
}

}  // namespace lba
