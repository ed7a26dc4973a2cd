// A key-value cache in 4 bits: what is appended is rounded to E2M1 values under a power of two per 32 (include/lba.h has the layout), and
// the attention of single tokens reads it as it lies.
//
// Attention wants 136 bytes of memory and 256 g multiply-adds, 512 g operations, for a (token, head) of 128 dimensions, g being the query heads that
// share it.  Eight heads together are 190 TFLOP/s at 6.4 TB/s, out of reach of the CUDA cores, so both products run on the tensor cores, and a warp
// feeds them from registers: m16n8k16 with 16 tokens (keys) or 16 dimensions (values) as rows and eight query heads as columns.  tcgen05
// would have a tile of 128 rows and operands in shared memory, where 4-bit values would have to be widened first.
//   S = K Q^T   E2M1 values are exact in binary16 (one conversion instruction for two).  The bytes of a key row stand so that a lane's 16
//               bytes are its operands of all k-steps, and both k-steps of a group of 32 lie in it: the group's power of two multiplies a
//               finished 32-term sum, in binary32
//   softmax     one pass; a running maximum per head that is raised only when a score exceeds it by 2^5, so that a vote replaces the
//               reduction of most steps
//   O = V^T P   P goes from accumulator to operand layout by the matrix transpose, with 9 bits of headroom below; the values' powers of two
//               differ by token and group, so P is multiplied by them, relative to one that the warp's first steps with a line have set.  16
//               binades around it are binary16's to tell apart (2^-12 of a weight); once any token's power of two lies outside (of a
//               group that is not all zeros), weights and values of that line are multiplied in binary32, token by token (740 us instead
//               of 107 for the 48 requests below)
// A query head is brought to [1, 2) by a power of two first and is then exact in binary16 but for what lies 2^-17 (binary16 queries: 2^-14) below
// its largest value.
// A warp has two units of 64 tokens in shared memory, one that it computes and one on its way by bulk copies, and meets no other warp.  What
// bounds it now is the latency of a warp's own chain from load to second product, with three warps a scheduler to hide it: some 290 instructions for
// 16 tokens of 128 dimensions and four heads, issue slots 55% busy, the busiest pipe 51% (conversions, byte moves), while the copies are waited for
// in 4% of the time.  48 requests of up to 16384 tokens, 8 heads of 128, 4 query heads each: 106 us, 4.0 TB/s.  (With loads straight to registers, two
// steps ahead, 140 us; 8 or 16 warps instead of 12, units of 32 tokens, three units or steps one by one: 109 to 130 us.)
#include <cmath>

#include "lba_async.cuh"
#include "lba_entry.cuh"
#include "lba_layer.cuh"

namespace lba {
namespace {

struct CacheView {
  uint8_t* pages;
  const int32_t* table;
  int64_t page_count;
  int heads, page, sequences, width;
  __host__ __device__ __forceinline__ int64_t run(int dim) const { return (int64_t)page * (dim + dim / 16); }  // bytes of a (page, head)
};
// the planes of a run: key codes, value codes, key exponents, value exponents
template <int D>
__device__ __forceinline__ uint8_t* plane(const CacheView& c, int64_t page, int head, int which) {
  return c.pages + (page * c.heads + head) * c.run(D) + (int64_t)c.page * (which == 0 ? 0 : which == 1 ? D / 2 : which == 2 ? D : D + D / 32);
}

// ------------------------------------------------------------------ append and read
constexpr int ROW_THREADS = 256, MAX_CU = 1024;

struct RowsParams {
  CacheView c;
  const void *k, *v;          // append: from; read: to
  lba_strides k_at, v_at;
  int64_t tokens;
  const int32_t *start, *cu;
  int block_heads;
};

// The (page, row) of token row t, or false.  `cu` was brought to shared memory where it fits.
template <typename P>
__device__ __forceinline__ bool locate(const P& p, const int32_t* cu_shared, int64_t t, int64_t* page, int* row) {
  int b;
  int64_t first;
  const int n = p.c.sequences;
  if (!p.cu) {
    if (t >= n) return false;
    b = (int)t;
    first = t;
  } else {  // the last sequence that begins at or before t
    const int32_t* const cu = n < MAX_CU ? cu_shared : p.cu;
    int lo = 0, hi = n;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (cu[mid] <= t) lo = mid;
      else hi = mid - 1;
    }
    b = lo;
    if (b >= n || cu[b] > t) return false;
    first = cu[b];
  }
  const int64_t pos = (int64_t)p.start[b] + (t - first);
  if (pos < 0 || pos >= (int64_t)p.c.width * p.c.page) return false;
  const int block = (int)(pos / p.c.page);
  *row = (int)(pos - (int64_t)block * p.c.page);
  *page = p.c.table[(int64_t)b * p.c.width + block];
  return *page >= 0 && *page < p.c.page_count;
}

// A lane takes eight neighbouring values, a quarter of a group; a warp a few tokens (those of 32 / (D / 8) rows), whose places it looks up once, and
// walks over heads, a key and a value row of each token at a time and the next head's on their way.  Bound by rounding's instructions (issue
// slots 74% busy): 12000 tokens of 8 heads of 128 are appended and read back, 111 MB, in 34 us, half the memory's rate.  (With a block of 16
// tokens for each head that looked up its own tokens 41 us, three quarters of it issue slots.)
template <int D> constexpr int kRowSplit = D / 8;
template <int D> constexpr int kWarpRows = 32 / kRowSplit<D>;

__device__ __forceinline__ uint32_t encode8(const float (&x)[8]) {  // eight values as 4-bit codes, the first in the lowest bits
  uint32_t d;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\tcvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\tcvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\tmov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(d) : "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]));
  return d;
}
// the pairs of a word's four bytes in binary16
__device__ __forceinline__ void decode8(uint32_t w, uint32_t (&h)[4]) {
  asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\tcvt.rn.f16x2.e2m1x2 %2, c;\n\tcvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
}
__device__ __forceinline__ float2 widen(uint32_t h) { return __half22float2(*reinterpret_cast<const __half2*>(&h)); }

// eight neighbouring values, in accesses of 16 bytes where the address allows them
template <typename T>
__device__ __forceinline__ void load8(const T* src, float (&x)[8]) {
  constexpr int W = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 8; i += W) {
    float v[W];
    load_some<T, W>(src, i, W, v);
#pragma unroll
    for (int j = 0; j < W; ++j) x[i + j] = v[j];
  }
}
template <typename T>
__device__ __forceinline__ void store8(T* dst, const float (&x)[8]) {
  constexpr int W = 16 / (int)sizeof(T);
#pragma unroll
  for (int i = 0; i < 8; i += W) {
    float v[W];
#pragma unroll
    for (int j = 0; j < W; ++j) v[j] = x[i + j];
    store_as<T, W>(dst, i, W, v);
  }
}

// what a lane reads and writes of one row, and their change from head to head
template <typename T>
struct Walk8 {
  T* number;
  uint8_t *codes, *exps;
  __device__ __forceinline__ void next(int64_t stride, int64_t run) {
    number += stride;
    codes += run;
    exps += run;
  }
};

// 2^-e of a group from its largest magnitude's bits, and its exponent byte (255: not a number)
__device__ __forceinline__ float group_scale(uint32_t top, int* byte) {
  int e = (int)(top >> 23) - 129 + ((top & 0x7FFFFFu) > 0x400000u);  // 1.f 2^E <= 1.5 2^(e+2)
  e = e < -126 ? -126 : e > 125 ? 125 : e;                            // (6 2^126 is no binary32 number)
  *byte = top >= 0x7F800000u ? 255 : e + 127;
  return __uint_as_float((uint32_t)(127 - e) << 23);
}

template <typename T, int D, bool READ>
__global__ void __launch_bounds__(ROW_THREADS) cache_rows_kernel(const RowsParams p) {
  constexpr int SPLIT = kRowSplit<D>, ROWS = kWarpRows<D>;
  __shared__ int32_t cu[MAX_CU];
  __shared__ __align__(16) uint8_t stage[ROW_THREADS / 32][ROWS * D / 2];
  after_previous();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane / SPLIT, q = lane % SPLIT;  // row of the warp, eighth values q
  const int64_t t = ((int64_t)blockIdx.x * (ROW_THREADS / 32) + warp) * ROWS + r;
  const int h0 = blockIdx.y * p.block_heads, h1 = min(h0 + p.block_heads, p.c.heads);
  if (p.cu && p.c.sequences < MAX_CU) {
    for (int i = threadIdx.x; i <= p.c.sequences; i += ROW_THREADS) cu[i] = p.cu[i];
    __syncthreads();
  }
  const bool there = r < ROWS && t < p.tokens;
  int64_t page = -1;
  int row = 0;
  bool stored = there, in_sequence = there;  // stored: has a place in the cache
  if (there) {
    stored = locate(p, cu, t, &page, &row);
    if (READ && p.cu) {  // (a row of a sequence whose token is not there reads as 0; one of no sequence is left)
      const int32_t* const all = p.c.sequences < MAX_CU ? cu : p.cu;
      in_sequence = stored || (t >= all[0] && t < all[p.c.sequences]);
    } else if (READ) {
      in_sequence = t < p.c.sequences;
    }
  }
  const int64_t run = p.c.run(D);
  // a key row's eighth q = 4 g + c is the word at c D/8 + 4 g; a value row's q = 2 i + h are bytes (4 h + j) D/16 + i
  Walk8<T> k, v;
  k.number = static_cast<T*>(const_cast<void*>(p.k)) + t * p.k_at.token + h0 * p.k_at.head + q * 8;
  v.number = static_cast<T*>(const_cast<void*>(p.v)) + t * p.v_at.token + h0 * p.v_at.head + q * 8;
  if (!stored) page = 0;
  k.codes = plane<D>(p.c, page, h0, 0) + row * (D / 2) + (q & 3) * (D / 8) + (q >> 2) * 4;
  v.codes = plane<D>(p.c, page, h0, 1) + row * (D / 2) + 4 * q;
  k.exps = plane<D>(p.c, page, h0, 2) + row * (D / 32) + (q >> 2);
  v.exps = plane<D>(p.c, page, h0, 3) + row * (D / 32) + (q >> 2);
  uint8_t* const line = stage[warp] + min(r, ROWS - 1) * (D / 2);
  if constexpr (!READ) {
    float x[8], y[8];
    if (there && h0 < h1) {
      load8<T>(k.number, x);
      load8<T>(v.number, y);
    }
#pragma unroll 1
    for (int h = h0; h < h1; ++h) {
      uint32_t top_x = 0, top_y = 0;
      if (there) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          top_x = max(top_x, __float_as_uint(x[j]) & 0x7FFFFFFFu);
          top_y = max(top_y, __float_as_uint(y[j]) & 0x7FFFFFFFu);
        }
      }
      // the four lanes of a group (lanes beyond the last row reduce zeros)
#pragma unroll
      for (int d = 1; d < 4; d *= 2) {
        top_x = max(top_x, __shfl_xor_sync(0xFFFFFFFFu, top_x, d));
        top_y = max(top_y, __shfl_xor_sync(0xFFFFFFFFu, top_y, d));
      }
      int byte_x, byte_y;
      const float by_x = group_scale(top_x, &byte_x), by_y = group_scale(top_y, &byte_y);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        x[j] *= by_x;
        y[j] *= by_y;
      }
      const uint32_t wx = byte_x == 255 ? 0u : encode8(x), wy = byte_y == 255 ? 0u : encode8(y);
      Walk8<T> to_k = k, to_v = v;
      k.next(p.k_at.head, run);
      v.next(p.v_at.head, run);
      if (there && h + 1 < h1) {
        load8<T>(k.number, x);
        load8<T>(v.number, y);
      }
      if (r < ROWS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) line[((q & 1) * 4 + j) * (D / 16) + (q >> 1)] = (uint8_t)(wy >> (8 * j));
      }
      __syncwarp();
      if (stored) {
        *reinterpret_cast<uint32_t*>(to_k.codes) = wx;
        *reinterpret_cast<uint32_t*>(to_v.codes) = *reinterpret_cast<const uint32_t*>(line + 4 * q);
        if ((q & 3) == 0) {
          *to_k.exps = (uint8_t)byte_x;
          *to_v.exps = (uint8_t)byte_y;
        }
      }
      __syncwarp();
    }
  } else {
    uint32_t wk = 0, wv = 0, ek = 0, ev = 0;
    const auto fetch = [&] {
      if (stored) {
        wk = *reinterpret_cast<const uint32_t*>(k.codes);
        wv = *reinterpret_cast<const uint32_t*>(v.codes);
        ek = *k.exps;
        ev = *v.exps;
      }
    };
    if (h0 < h1) fetch();
#pragma unroll 1
    for (int h = h0; h < h1; ++h) {
      if (r < ROWS) *reinterpret_cast<uint32_t*>(line + 4 * q) = wv;
      __syncwarp();
      uint32_t w = 0;
      if (r < ROWS) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= (uint32_t)line[((q & 1) * 4 + j) * (D / 16) + (q >> 1)] << (8 * j);
      }
      __syncwarp();
      const auto write = [&](uint32_t word, uint32_t exp, T* to) {
        uint32_t h2[4];
        decode8(word, h2);
        const float by = exp == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(exp << 23);
        float x[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 f = widen(h2[j]);
          x[2 * j] = f.x * by;
          x[2 * j + 1] = f.y * by;
        }
        if (in_sequence) store8<T>(to, x);
      };
      const uint32_t word = wk, exp_k = ek, exp_v = ev;
      T *const to_k = k.number, *const to_v = v.number;
      k.next(p.k_at.head, run);
      v.next(p.v_at.head, run);
      if (h + 1 < h1) fetch();
      write(word, exp_k, to_k);
      write(w, exp_v, to_v);
    }
  }
}

template <bool READ, typename T>
cudaError_t launch_rows(RowsParams p, int dim, cudaStream_t stream) {
  const auto go = [&](auto d) {
    constexpr int D = decltype(d)::value, ROWS = kWarpRows<D> * (ROW_THREADS / 32);
    // heads of a block: all, or as few as bring eight blocks to every SM
    const int64_t blocks = (p.tokens + ROWS - 1) / ROWS, parts = (8LL * device_sms() + blocks - 1) / blocks;
    p.block_heads = (int)((p.c.heads + parts - 1) / parts);
    return launch_after(cache_rows_kernel<T, D, READ>, dim3((unsigned)blocks, (unsigned)((p.c.heads + p.block_heads - 1) / p.block_heads)), ROW_THREADS, 0,
                        stream, p);
  };
  switch (dim) {
    case 32: return go(std::integral_constant<int, 32>());
    case 64: return go(std::integral_constant<int, 64>());
    case 96: return go(std::integral_constant<int, 96>());
    default: return go(std::integral_constant<int, 128>());
  }
}
template <bool READ>
cudaError_t launch_rows(const RowsParams& p, int dim, int type, cudaStream_t stream) {
  return type == LBA_TYPE_F32 ? launch_rows<READ, float>(p, dim, stream)
         : type == LBA_TYPE_BF16 ? launch_rows<READ, __nv_bfloat16>(p, dim, stream) : launch_rows<READ, __half>(p, dim, stream);
}

// ------------------------------------------------------------------ attention of single tokens
// Work is counted in units of 64 tokens of a line: a piece of up to HT query heads of a key-value head of a sequence.  All units of all
// lines, sequence by sequence, stand in one row, cut into equal shares, one for each warp (a share may take in many lines, and a line
// many shares), so no warp waits for another.  A warp leaves a part for every line that it meets: sums, maximum and outputs relative to
// it.  Warp w's part of line i is number w + i: one of the two grows from each part to the next.  cache_combine_kernel adds up the parts
// of each line.  (With CTAs that merged their eight warps' parts, each for a stretch of one line, 48 requests of up to 16384 tokens took
// 135 us at the best length of a stretch: a CTA's start and end cost 5 us.)
constexpr int UNIT = 64, STEP = 16, DEC_STAGES = 2, DEC_WARPS = 12, DEC_THREADS = 32 * DEC_WARPS;
constexpr int KNOWN = 128, GROUPS = 65536 / KNOWN;  // sequences of which a warp knows the lengths at a time
constexpr float HEADROOM = 5.0f;     // binades by which a score may exceed its head's running maximum
constexpr float P_BITS = 9.0f;       // weights in binary16: at most 2^(9 + 5), and twice that times the power of two of their values
constexpr float NO_MAX = -1e30f;
constexpr int EDGE_ABOVE = 3;        // binades that a line's values may grow by above its first ones' largest; 12 are left below

struct DecodeParams {
  CacheView c;
  const void* q;
  lba_strides q_at;
  const int32_t* lengths;
  int heads, group, pieces;           // query heads; of a key-value head; pieces of a group
  int warps;                          // that there are shares for, at most
  float scale;
  int out_type, in_m4e3;
  const float* out_scale;
  void* out;
  int* before;                        // [sequences + 1]: units of a line in all sequences before
  float* parts;                       // [warps + lines][HT][D + 2]
  __host__ __device__ int lines() const { return c.heads * pieces; }  // of a sequence
};
__device__ __forceinline__ int share_of(const DecodeParams& p, int all_units) { return max((int)(((unsigned)(all_units * p.lines()) + p.warps - 1) / p.warps), 1); }

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma16816_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {  // sums from 0 on
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};"
      : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ uint32_t transposed(uint32_t m) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(m));
  return d;
}
__device__ __forceinline__ uint32_t half_pair(float lo, float hi) {
  const __half2 h = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t mul_halves(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// largest of the bytes at each of four places
__device__ __forceinline__ uint32_t max_bytes(uint32_t a, uint32_t b) {
  constexpr uint32_t EVEN = 0x00FF00FFu;
  return __vmaxu2(a & EVEN, b & EVEN) | (__vmaxu2((a >> 8) & EVEN, (b >> 8) & EVEN) << 8);
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, int bytes, uint32_t bar) {
  asm volatile("cp.async.bulk.shared::cta.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar) : "memory");
}

// A unit in shared memory: the four planes of a run, 64 tokens of each
template <int NG>
struct Unit {
  static constexpr int D = 32 * NG, VALUES = UNIT * D / 2, KEY_EXP = UNIT * D, VALUE_EXP = UNIT * (D + NG), BYTES = UNIT * (D + 2 * NG);
};
template <int NG>
__device__ __forceinline__ uint32_t exponents(const uint8_t* p) {
  if constexpr (NG == 4) return *reinterpret_cast<const uint32_t*>(p);
  if constexpr (NG == 2) return *reinterpret_cast<const uint16_t*>(p);
  if constexpr (NG == 1) return *p;
  return (uint32_t)p[0] | ((uint32_t)p[1] << 8) | ((uint32_t)p[2] << 16);
}

template <int D>
__device__ __forceinline__ void store_decoded(const DecodeParams& p, int64_t i, float v) {
  if (p.out_type == LBA_TYPE_CODES) {
    const float z = __fdiv_rn(v, *p.out_scale);
    static_cast<uint8_t*>(p.out)[i] = p.in_m4e3 ? encode_m4e3(z) : encode_e4m3(z);
  } else if (p.out_type == LBA_TYPE_BF16) {
    static_cast<__nv_bfloat16*>(p.out)[i] = __float2bfloat16_rn(v);
  } else {
    static_cast<__half*>(p.out)[i] = __float2half_rn(v);
  }
}

// of a sequence: what its length and its row of the table allow (below 2^31 - 64: view_of)
__device__ __forceinline__ int tokens_of(const DecodeParams& p, int b) { return max(0, min(p.lengths[b], p.c.width * p.c.page)); }
__device__ __forceinline__ int units_of(int tokens) { return (tokens + UNIT - 1) / UNIT; }

struct WarpState {  // what a warp needs from line to line
  int before[KNOWN + 1], tokens[KNOWN];  // units of a line before each of the sequences that are known, and their tokens
};
template <int NG> constexpr size_t kDecodeSmem = (size_t)DEC_WARPS * (DEC_STAGES * (Unit<NG>::BYTES + 8) + sizeof(WarpState)) + 128;

// HT: query heads of a line.  Columns of the scores are heads, eight at a time; with four heads they are there twice.
template <typename T, int NG, int HT>
__global__ void __launch_bounds__(DEC_THREADS, 1) cache_attention_kernel(const DecodeParams p) {
  typedef Unit<NG> U;
  constexpr int D = 32 * NG, NT = HT <= 8 ? 1 : HT / 8, OT = HT / 4, PART = D + 2;  // tiles of eight columns, of four heads' outputs
  constexpr int BATCH = HT <= 8 ? 2 : 1;                                            // steps of 16 tokens side by side: independent chains
  constexpr bool TWICE = HT == 4;
  extern __shared__ __align__(128) uint8_t units[];  // [warp][stage], then each warp's barriers and state
  __shared__ int groups[GROUPS + 1];                 // units of a line in all sequences before each KNOWN of them
  __shared__ int dead_flag;
  volatile int* const dead = &dead_flag;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
  uint8_t* const mine = units + warp * (DEC_STAGES * U::BYTES);
  uint64_t* const full = reinterpret_cast<uint64_t*>(units + DEC_WARPS * DEC_STAGES * U::BYTES) + warp * DEC_STAGES;
  WarpState& state = reinterpret_cast<WarpState*>(units + DEC_WARPS * DEC_STAGES * (U::BYTES + 8))[warp];
  if (threadIdx.x == 0) dead_flag = 0;
  if (lane == 0) {
    for (int i = 0; i < DEC_STAGES; ++i) mbar_init(smem_u32(full + i), 1);
    mbar_init_fence();
  }
  after_previous();
  const int group_count = (p.c.sequences + KNOWN - 1) / KNOWN;
  // the tokens of group g's sequences, four neighbours a lane; returns the group's units
  const auto know = [&](int g, int units_before) -> int {
    __syncwarp();  // (what was known is no longer read)
    int n[4], sum = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int b = g * KNOWN + lane * 4 + i, t = b < p.c.sequences ? tokens_of(p, b) : 0;
      state.tokens[lane * 4 + i] = t;
      n[i] = sum;
      sum += units_of(t);
    }
    int upto = sum;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int u = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += u;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) state.before[lane * 4 + i] = units_before + upto - sum + n[i];
    const int all = __shfl_sync(0xFFFFFFFFu, upto, 31);
    if (lane == 0) state.before[KNOWN] = units_before + all;
    __syncwarp();
    return all;
  };
  const int lines = p.lines();
  int known = 0, all;
  if (group_count <= 1) {
    all = know(0, 0);
    __syncthreads();  // (of what the first threads have set up)
  } else {
    for (int g = warp; g < group_count; g += DEC_WARPS) {
      const int n = know(g, 0);
      if (lane == 0) groups[g + 1] = n;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      int sum = 0;
      groups[0] = 0;
      for (int g = 1; g <= group_count; ++g) groups[g] = sum += groups[g];
    }
    __syncthreads();
    all = groups[group_count];
  }
  if (blockIdx.x == 0) {  // for the second kernel
    for (int g = warp; g < group_count; g += DEC_WARPS) {
      if (group_count > 1) know(g, groups[g]);
      for (int i = lane; i < KNOWN && g * KNOWN + i < p.c.sequences; i += 32) p.before[g * KNOWN + i] = state.before[i];
      __syncwarp();
    }
    if (threadIdx.x == 0) p.before[p.c.sequences] = all;
  }
  const int share = share_of(p, all), total = all * lines;
  // (first the first warp of every CTA: few units spread over the SMs)
  const int me = warp * (int)gridDim.x + (int)blockIdx.x;
  int at = (int)min((unsigned)me * (unsigned)share, (unsigned)total);
  const int end = (int)min((unsigned)at + (unsigned)share, (unsigned)total);
  if (group_count > 1 && at < end) {  // the group of the first unit: the last that begins at or before it
    int lo = 0, hi = group_count - 1;
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (groups[mid] <= at / lines) lo = mid;
      else hi = mid - 1;
    }
    known = lo;
    know(lo, groups[lo]);
  }
  int filled = 0;  // units that were sent for so far: their number says which stage and phase
  bool ok = true;
#pragma unroll 1
  while (at < end) {
    int seq;
    while (true) {  // the last of the known sequences that begins at or before this unit, and is not empty
      const int place = at / lines;
      int n = 0;
#pragma unroll
      for (int i = 0; i < KNOWN; i += 32) n += __popc(__ballot_sync(0xFFFFFFFFu, state.before[i + lane] <= place));
      if (place < state.before[KNOWN]) {  // (of several that begin there, all but the last are empty)
        seq = n - 1;
        break;
      }
      ++known;
      know(known, groups[known]);
    }
    const int tokens = state.tokens[seq], n_units = units_of(tokens), inside = at - state.before[seq] * lines;
    const int b = known * KNOWN + seq, line = inside / n_units, kvh = line / p.pieces, piece = line - kvh * p.pieces;
    const int u0 = inside - line * n_units, u1 = min(n_units, u0 + end - at);
    at += u1 - u0;

    // A unit comes in runs of tokens that lie in one page: all 64, or 32 or 16 where pages are no multiples of 64.  The lanes hold the next 32 runs'
    // pages (-1: not there) and first rows.  (The copies are an elected lane's with the same operands in every lane: where four lanes each
    // sent for a run, a unit cost 200 instructions.)
    const int run = p.c.page % 64 == 0 ? 64 : p.c.page % 32 == 0 ? 32 : 16, runs = UNIT / run;
    int window = u0 * runs, pages, rows;
    const auto look_up = [&] {
      const int t = (window + lane) * run, number = t / p.c.page;
      rows = t - number * p.c.page;
      pages = t < tokens ? __ldg(p.c.table + (int64_t)b * p.c.width + number) : -1;
      if (pages >= p.c.page_count) pages = -1;
    };
    look_up();
    const auto fill = [&](int u, int stage) -> uint32_t {  // one unit after another; the mask says which of its four steps are there
      if (u * runs - window >= 32) {
        window = u * runs;
        look_up();
      }
      uint32_t there = 0;
      const int left = min(tokens - u * UNIT, UNIT);
      const uint32_t bar = smem_u32(full + stage), dst = smem_u32(mine + stage * U::BYTES);
      int page[4], row[4], up[4], bytes = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (i >= runs) break;
        page[i] = __shfl_sync(0xFFFFFFFFu, pages, u * runs + i - window);
        row[i] = __shfl_sync(0xFFFFFFFFu, rows, u * runs + i - window);
        up[i] = page[i] < 0 ? 0 : (min(left - i * run, run) + STEP - 1) / STEP * STEP;  // whole steps: sizes are multiples of 16 bytes
        there |= ((1u << (up[i] / STEP)) - 1u) << (i * run / STEP);
        bytes += up[i] * (D + 2 * NG);
      }
      if (there && elected()) {
        mbar_arrive_expect(bar, bytes);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (i >= runs) break;
          if (!up[i]) continue;
          const uint8_t* const src = p.c.pages + ((int64_t)page[i] * p.c.heads + kvh) * p.c.run(D);
          const int first = i * run;
          bulk_load(dst + first * (D / 2), src + row[i] * (D / 2), up[i] * (D / 2), bar);
          bulk_load(dst + U::VALUES + first * (D / 2), src + (p.c.page + row[i]) * (D / 2), up[i] * (D / 2), bar);
          bulk_load(dst + U::KEY_EXP + first * NG, src + p.c.page * D + row[i] * NG, up[i] * NG, bar);
          bulk_load(dst + U::VALUE_EXP + first * NG, src + p.c.page * (D + NG) + row[i] * NG, up[i] * NG, bar);
        }
      }
      __syncwarp();
      return there;
    };
    uint32_t there[DEC_STAGES];
    int order[DEC_STAGES];  // of the fills: which stage and phase
#pragma unroll
    for (int i = 0; i < DEC_STAGES; ++i) {
      there[i] = 0;
      order[i] = filled;
      if (u0 + i < u1) there[i] = fill(u0 + i, filled % DEC_STAGES);
      if (there[i]) ++filled;
    }

    // query heads: column r of a tile; values 32 g + 8 c to + 7
    uint32_t q[NT][NG][4];
    float to_log2[NT][2];  // of columns 2 c and 2 c + 1
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int h = piece * HT + (TWICE ? r & 3 : n * 8 + r);
      float x[NG][8], top = 0.0f;
      const bool has = h < p.group;
      const T* const src = static_cast<const T*>(p.q) + (int64_t)b * p.q_at.token + (int64_t)(kvh * p.group + h) * p.q_at.head + c * 8;
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        load_some<T, 8>(src, g * 32, has ? 8 : 0, x[g]);
#pragma unroll
        for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[g][j]));
      }
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      int e = (int)(__float_as_uint(top) >> 23) - 127;  // (infinities stay what they are under any factor)
      e = e < -126 ? -126 : e > 126 ? 126 : e;
      const float down = __uint_as_float((uint32_t)(127 - e) << 23);
      const float up = fmaxf(__uint_as_float((uint32_t)(127 + e) << 23) * (p.scale * LOG2E), 0x1p-149f);  // (0 times the -inf of what is not there is no number)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) q[n][g][j] = half_pair(x[g][2 * j] * down, x[g][2 * j + 1] * down);
#pragma unroll
      for (int j = 0; j < 2; ++j) to_log2[n][j] = __shfl_sync(0xFFFFFFFFu, up, (2 * c + j) * 4);
    }

    // m: the maximum that weights are relative to, less 9 binades; limit: the score from which on it is raised.
    // edge: for each group the highest exponent byte of the 16 that weights can be brought to, in 16..254 (0: no token yet): outputs are relative to
    // the power of two below it.  A byte of edge - (exponents) is in 0..15 where the exponent is among the 16; an exponent above gives 17 to 255
    // there, and a borrow only comes from such a byte: no high half of a byte set means that all are among them.
    float o[OT][NG][4], m[NT][2], limit[NT][2], l[NT][2];
    uint32_t edge = 0, base = 0;  // base + 4 e: bytes 0x40 - 4 (edge - e), the high byte of 2^(1 - (edge - e)) in binary16
    bool by_token = false;        // some token was outside: from then on products are formed in binary32
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = limit[n][0] = limit[n][1] = NO_MAX;
      l[n][0] = l[n][1] = 0.0f;
    }
#pragma unroll
    for (int t = 0; t < OT; ++t)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < 4; ++j) o[t][g][j] = 0.0f;

    // Bytes (0, 2^-d) as the half of a pair that a column's weights are in: of place g, by selector place_of + g place_step.  Values of tokens
    // 2 c and 2 c + 1 (and 8 on) are taken in the other order where c is odd: so the four rows of a load lie in both halves of the banks.
    const uint32_t place_of = r < 4 ? 0x4404u : 0x0444u, place_step = r < 4 ? 0x0010u : 0x1000u;
    const int swap = c & 1;
    const uint32_t pick0 = swap ? 0x3232u : 0x1010u, pick1 = swap ? 0x1010u : 0x3232u;

    // The same sums token by token in binary32: a weight comes from the lane that holds it, a lane's outputs are those of the matrix instructions
    const auto add_by_token = [&](const uint8_t* unit, int first, int left, uint32_t steps, const float (&z)[BATCH][NT][4]) {
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {
        const int here = (steps >> x) & 1 ? left - x * STEP : 0;
        float e[NT][4];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[n][j] = exp2_approx(fmaf(z[x][n][j], to_log2[n][j & 1], -m[n][j & 1]));
            l[n][j & 1] += e[n][j];
          }
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll 1
          for (int i = 0; i < 8 && half * 8 + i < here; ++i) {
            float w[OT][2];  // of heads 4 t + 2 (c & 1) and the next
#pragma unroll
            for (int t = 0; t < OT; ++t)
#pragma unroll
              for (int j = 0; j < 2; ++j)
                w[t][j] = __shfl_sync(0xFFFFFFFFu, e[t * NT / OT][2 * half + j], i * 4 + (TWICE ? 0 : 2 * (t & 1)) + (c & 1));
            const int row = first + x * STEP + half * 8 + i;
            const uint32_t exps = exponents<NG>(unit + U::VALUE_EXP + row * NG);
            const uint8_t* const codes = unit + U::VALUES + row * (D / 2) + r * (D / 16);
#pragma unroll
            for (int g = 0; g < NG; ++g) {
              // (an exponent byte of 0 holds nothing but zeros; 2^-126 below the outputs' power of two values count as 0)
              const int power = (int)((exps >> (8 * g)) & 255u), d = power - (int)((edge >> (8 * g)) & 255u) + 1;
              const float by = power == 255 ? __uint_as_float(0x7FC00000u) : power == 0 || d < -126 ? 0.0f : __uint_as_float((uint32_t)(127 + d) << 23);
#pragma unroll
              for (int k = 0; k < 2; ++k) {
                const uint32_t code = codes[2 * g + k] >> (c >> 1) * 4;
                // as a binary32 number 2^126 below, 1/2 among those without a leading 1
                const float v = __uint_as_float((code & 8u) << 28 | (code & 7u) << 22) * 0x1p126f * by;
#pragma unroll
                for (int t = 0; t < OT; ++t)
#pragma unroll
                  for (int j = 0; j < 2; ++j) o[t][g][2 * k + j] = fmaf(w[t][j], v, o[t][g][2 * k + j]);
              }
            }
          }
      }
    };

    // BATCH steps from token `first` of a unit on, of which `left` tokens exist and `steps` (bits) are there
    const auto compute = [&](const uint8_t* unit, int first, int left, uint32_t steps) {
      float z[BATCH][NT][4];  // tokens r (0, 1) and r + 8 (2, 3); columns 2 c (0, 2) and 2 c + 1 (1, 3)
      uint32_t ve[BATCH][4];
      const uint8_t* const keys = unit + (first + r) * (D / 2) + c * (D / 8);
      const uint8_t* const key_exps = unit + U::KEY_EXP + (first + r) * NG;
      const uint8_t* const value_exps = unit + U::VALUE_EXP + (first + 2 * c) * NG;
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {
        uint32_t k[2][NG], ke[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint8_t* const src = keys + (x * STEP + 8 * i) * (D / 2);
          if constexpr (NG == 4) {
            const uint4 w = *reinterpret_cast<const uint4*>(src);
            k[i][0] = w.x, k[i][1] = w.y, k[i][2] = w.z, k[i][3] = w.w;
          } else if constexpr (NG == 2) {
            const uint2 w = *reinterpret_cast<const uint2*>(src);
            k[i][0] = w.x, k[i][1] = w.y;
          } else {
#pragma unroll
            for (int g = 0; g < NG; ++g) k[i][g] = reinterpret_cast<const uint32_t*>(src)[g];
          }
          ke[i] = exponents<NG>(key_exps + (x * STEP + 8 * i) * NG);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) ve[x][i] = exponents<NG>(value_exps + (x * STEP + ((i & 1) ^ swap) + (i >> 1) * 8) * NG);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t lo[4], hi[4];
          decode8(k[0][g], lo);
          decode8(k[1][g], hi);
          const int up = 23 - 8 * g;
          float by[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) by[i] = __uint_as_float((up >= 0 ? ke[i] << (up & 31) : ke[i] >> (-up & 31)) & 0x7F800000u);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            float sum[4];
            const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
            mma16816_first(sum, a0, q[n][g][0], q[n][g][1]);
            mma16816(sum, a1, q[n][g][2], q[n][g][3]);
#pragma unroll
            for (int j = 0; j < 4; ++j) z[x][n][j] = g == 0 ? sum[j] * by[j >> 1] : fmaf(sum[j], by[j >> 1], z[x][n][j]);
          }
        }
      }
      if (left < BATCH * STEP || steps != (1u << BATCH) - 1u) {  // what does not exist, or was not copied, may be anything
#pragma unroll
        for (int x = 0; x < BATCH; ++x) {
          const int here = (steps >> x) & 1 ? left - x * STEP : 0;
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j)
              if (r + (j >> 1) * 8 >= here) z[x][n][j] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (2 * c + ((i & 1) ^ swap) + (i >> 1) * 8 >= here) ve[x][i] = edge;
        }
      }
      uint32_t wide = 0;
      bool raise = false;
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {
#pragma unroll
        for (int i = 0; i < 4; ++i) wide |= edge - ve[x][i];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) raise |= z[x][n][j] > limit[n][j & 1];
      }
      raise |= edge == 0 || (wide & 0xF0F0F0F0u) != 0;
      if (__any_sync(0xFFFFFFFFu, raise)) {
        // (a byte of 255, no number, has no binade.  Tokens that are not there have bytes of edge: 0 before there is one)
        uint32_t top = 0;
#pragma unroll
        for (int x = 0; x < BATCH; ++x)
#pragma unroll
          for (int i = 0; i < 4; ++i) top = max_bytes(top, ve[x][i] & ~__vcmpeq4(ve[x][i], 0xFFFFFFFFu));
        top = max_bytes(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
        top = max_bytes(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
        uint32_t by = 0;  // binades by which the edge rises, and outputs with it
        constexpr uint32_t GROUP_BYTES = 0xFFFFFFFFu >> (8 * (4 - NG));
        if (edge == 0) {
          edge = __vminu4(__vmaxu4(__vaddus4(top, 0x01010101u * EDGE_ABOVE), 0x10101010u), 0xFEFEFEFEu) & GROUP_BYTES;
          base = (0x40404040u & GROUP_BYTES) - 4u * edge;
          wide = 0;
#pragma unroll
          for (int x = 0; x < BATCH; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int here = (steps >> x) & 1 ? left - x * STEP : 0;
              if (2 * c + ((i & 1) ^ swap) + (i >> 1) * 8 >= here) ve[x][i] = edge;
              wide |= edge - ve[x][i];
            }
        }
        if (!by_token && __any_sync(0xFFFFFFFFu, (wide & 0xF0F0F0F0u) != 0)) {
          // groups of zeros (exponent byte 1, or 0 where nothing was written) go with any power of two
          wide = 0;
#pragma unroll
          for (int x = 0; x < BATCH; ++x)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint8_t* const codes = unit + U::VALUES + (first + x * STEP + 2 * c + ((i & 1) ^ swap) + (i >> 1) * 8) * (D / 2) + r * (D / 16);
              uint32_t used = 0;
#pragma unroll
              for (int g = 0; g < NG; ++g)
                if ((codes[2 * g] | codes[2 * g + 1]) & 0x77u) used |= 255u << (8 * g);
#pragma unroll
              for (int d = 4; d < 32; d *= 2) used |= __shfl_xor_sync(0xFFFFFFFFu, used, d);
              const uint32_t zero = __vcmpleu4(ve[x][i], 0x01010101u) & ~used & GROUP_BYTES;
              ve[x][i] = (ve[x][i] & ~zero) | (edge & zero);
              wide |= edge - ve[x][i];
            }
          by_token = __any_sync(0xFFFFFFFFu, (wide & 0xF0F0F0F0u) != 0);
        }
        if (by_token) {
          top = max_bytes(top, edge);
          by = top - edge;
          edge = top;
        }
        float a[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float t = fmaxf(z[0][n][j], z[0][n][j + 2]);
            if (BATCH == 2) t = fmaxf(t, fmaxf(z[BATCH - 1][n][j], z[BATCH - 1][n][j + 2]));
            t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
            t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
            t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
            t = fmaxf(m[n][j], t * to_log2[n][j] - P_BITS);
            a[n][j] = exp2_approx(m[n][j] - t);
            m[n][j] = t;
            limit[n][j] = t == NO_MAX ? NO_MAX : (t + P_BITS + HEADROOM) / to_log2[n][j];
            l[n][j] *= a[n][j];
          }
#pragma unroll
        for (int t = 0; t < OT; ++t) {
          float f[2];  // of heads 4 t + 2 (c & 1) and the next
#pragma unroll
          for (int j = 0; j < 2; ++j) f[j] = TWICE ? a[0][j] : __shfl_sync(0xFFFFFFFFu, a[t / 2][j], (lane & 28) + 2 * (t & 1) + (c & 1));
#pragma unroll
          for (int g = 0; g < NG; ++g) {
            const int d = (by >> (8 * g)) & 255;
            const float down = d > 126 ? 0.0f : __uint_as_float((uint32_t)(127 - d) << 23);
#pragma unroll
            for (int j = 0; j < 4; ++j) o[t][g][j] *= f[j & 1] * down;
          }
        }
      }
      if (by_token) {
        add_by_token(unit, first, left, steps, z);
        return;
      }
#pragma unroll
      for (int x = 0; x < BATCH; ++x) {
        // weights as operands: rows of the transposed 8 x 8 blocks are columns of the scores, columns tokens 2 c, 2 c + 1 and 2 c + 8, 2 c + 9
        uint32_t both4[OT][4], high[4];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float e[4];
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            e[j] = exp2_approx(fmaf(z[x][n][j], to_log2[n][j & 1], -m[n][j & 1]));
            l[n][j & 1] += e[j];
          }
          const uint32_t w0 = transposed(half_pair(e[0], e[1])), w1 = transposed(half_pair(e[2], e[3]));
#pragma unroll
          for (int t = n * OT / NT; t < (n + 1) * OT / NT; ++t) {
            const int from_lane = (r & 3) * 4 + 16 * (t & 1) + c;
            const uint32_t x0 = TWICE ? w0 : __shfl_sync(0xFFFFFFFFu, w0, from_lane), x1 = TWICE ? w1 : __shfl_sync(0xFFFFFFFFu, w1, from_lane);
            both4[t][0] = __byte_perm(x0, x0, pick0);
            both4[t][1] = __byte_perm(x0, x0, pick1);
            both4[t][2] = __byte_perm(x1, x1, pick0);
            both4[t][3] = __byte_perm(x1, x1, pick1);
          }
        }
        uint32_t v[4][(NG + 1) / 2];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          high[i] = base + 4u * ve[x][i];
          const uint8_t* const src = unit + U::VALUES + (first + x * STEP + 2 * c + ((i & 1) ^ swap) + (i >> 1) * 8) * (D / 2) + r * (D / 16);
          if constexpr (NG == 4) {
            const uint2 w = *reinterpret_cast<const uint2*>(src);
            v[i][0] = w.x, v[i][1] = w.y;
          } else if constexpr (NG == 2) {
            v[i][0] = *reinterpret_cast<const uint32_t*>(src);
          } else {
            // (both halves of a word are filled: from a 16-bit load alone, nvcc 12.9 had the conversions of its bytes give 0)
            const uint16_t* const h = reinterpret_cast<const uint16_t*>(src);
            v[i][0] = h[0] | (uint32_t)h[NG == 3] << 16;
            if constexpr (NG == 3) v[i][1] = h[2] | (uint32_t)h[2] << 16;
          }
        }
        // A byte's conversion gives two dimensions of a token.  They are two k-steps of the product, and its columns are four heads twice: the first
        // four columns' weights are 0 for the second dimension, the others' for the first.  So are the factors that bring a weight to its group.
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          uint32_t h[4][2], f[4];  // [token][rows r and r + 8: bytes 16 g + r and 16 g + 8 + r]
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            f[i] = __byte_perm(high[i], 0u, place_of + g * place_step);
            const uint32_t word = v[i][g / 2];
            if (g & 1)
              asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %2;\n\tcvt.rn.f16x2.e2m1x2 %0, c;\n\tcvt.rn.f16x2.e2m1x2 %1, d;\n\t}" : "=r"(h[i][0]), "=r"(h[i][1]) : "r"(word));
            else
              asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %2;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\tcvt.rn.f16x2.e2m1x2 %1, b;\n\t}" : "=r"(h[i][0]), "=r"(h[i][1]) : "r"(word));
          }
          const uint32_t a0[4] = {h[0][0], h[0][1], h[1][0], h[1][1]}, a1[4] = {h[2][0], h[2][1], h[3][0], h[3][1]};
#pragma unroll
          for (int t = 0; t < OT; ++t) {
            mma16816(o[t][g], a0, mul_halves(both4[t][0], f[0]), mul_halves(both4[t][1], f[1]));
            mma16816(o[t][g], a1, mul_halves(both4[t][2], f[2]), mul_halves(both4[t][3], f[3]));
          }
        }
      }
    };

#pragma unroll 1
    for (int u = u0; u < u1; u += DEC_STAGES) {
#pragma unroll
      for (int i = 0; i < DEC_STAGES; ++i) {
        if (there[i]) {
          const int stage = order[i] % DEC_STAGES;
          ok = ok && __all_sync(0xFFFFFFFFu, mbar_wait(smem_u32(full + stage), (order[i] / DEC_STAGES) & 1, dead));
          if (ok) {
            const uint8_t* const unit = mine + stage * U::BYTES;
            const int left = tokens - (u + i) * UNIT;
#pragma unroll 1
            for (int first = 0; first < UNIT; first += BATCH * STEP) {
              const uint32_t steps = (there[i] >> (first / STEP)) & ((1u << BATCH) - 1u);
              if (steps) compute(unit, first, left - first, steps);
            }
          }
          __syncwarp();
        }
        const int next = u + i + DEC_STAGES;
        order[i] = filled;
        there[i] = ok && next < u1 ? fill(next, filled % DEC_STAGES) : 0;
        if (there[i]) ++filled;
      }
    }

    // The part.  It is brought to a sum of weights in 1/4..1/2, so that its outputs, which are at most that times the largest value, are in range.
    float* const part = p.parts + (me + (int64_t)b * lines + line) * (HT * PART);
    float to_range[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float t = l[n][j];
        t += __shfl_xor_sync(0xFFFFFFFFu, t, 4);
        t += __shfl_xor_sync(0xFFFFFFFFu, t, 8);
        t += __shfl_xor_sync(0xFFFFFFFFu, t, 16);
        if (!ok) t = __uint_as_float(0x7FC00000u);
        const int e = t > 0.0f && t < INFINITY ? (int)(__float_as_uint(t) >> 23) - 125 : 0;  // (a sum that is not 0 is 2^-126 or more)
        to_range[n][j] = __uint_as_float((uint32_t)(127 - e) << 23);
        const int h = n * 8 + 2 * c + j;
        if (r == 0 && h < HT) *reinterpret_cast<float2*>(part + h * PART + D) = make_float2(m[n][j] + (float)e, t * to_range[n][j]);
      }
#pragma unroll
    for (int t = 0; t < OT; ++t) {
      float f[2];  // of heads 4 t + 2 (c & 1) and the next
#pragma unroll
      for (int j = 0; j < 2; ++j) f[j] = TWICE ? to_range[0][j] : __shfl_sync(0xFFFFFFFFu, to_range[t / 2][j], (lane & 28) + 2 * (t & 1) + (c & 1));
#pragma unroll
      for (int g = 0; g < NG; ++g) {
        const uint32_t e = (edge >> (8 * g)) & 255u;
        const float by = __uint_as_float((e == 0 ? 0u : e - 1) << 23);  // (0: no token was there)
#pragma unroll
        for (int j = 0; j < 4; ++j) part[(4 * t + 2 * (c & 1) + (j & 1)) * PART + 2 * (16 * g + r + 8 * (j >> 1)) + (c >> 1)] = o[t][g][j] * f[j & 1] * by;
      }
    }
  }
  if (!ok) let_copies_land();
}

// a line's parts together: a block per head
constexpr int PARTS_AT_ONCE = 256;
template <int NG, int HT>
__global__ void __launch_bounds__(32 * NG) cache_combine_kernel(const DecodeParams p) {
  constexpr int D = 32 * NG, PART = D + 2;
  __shared__ float2 weight[PARTS_AT_ONCE];  // of a part: its maximum and sum; then the factor of its outputs, and its sum times that
  __shared__ float tops[NG];
  after_previous();
  const int b = blockIdx.y, h = blockIdx.x, d = threadIdx.x, lines = p.lines();
  const int kvh = h / p.group, in_group = h - kvh * p.group, piece = in_group / HT, line = kvh * p.pieces + piece, col = in_group - piece * HT;
  const int begin = p.before[b], units = p.before[b + 1] - begin, share = share_of(p, p.before[p.c.sequences]), first = begin * lines + line * units;
  const int w0 = first / share, n = units > 0 ? (first + units - 1) / share - w0 + 1 : 0;
  const float* const part = p.parts + (w0 + (int64_t)b * lines + line) * (HT * PART) + col * PART;
  constexpr int AHEAD = 16;
  const float down = n > 1 ? (float)(32 - __clz(n - 1)) : 0.0f;  // binades that n parts' sums may be above one's
  float top = NO_MAX, sum = 0.0f, v = 0.0f, ahead[AHEAD];  // ahead: of the first parts, beside their weights
#pragma unroll
  for (int i = 0; i < AHEAD; ++i) ahead[i] = i < n ? __ldg(part + (int64_t)i * HT * PART + d) : 0.0f;
  for (int i0 = 0; i0 < n; i0 += PARTS_AT_ONCE) {  // (two trips to memory for 256 parts, one for the first sixteen; one after the other they cost one each four)
    const int here = min(n - i0, PARTS_AT_ONCE);
    float most = top;
    for (int i = d; i < here; i += D) {
      const float2 ml = __ldg(reinterpret_cast<const float2*>(part + (int64_t)(i0 + i) * HT * PART + D));
      weight[i] = ml;
      most = fmaxf(most, ml.x);
    }
#pragma unroll
    for (int x = 16; x > 0; x /= 2) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, x));
    if ((d & 31) == 0) tops[d >> 5] = most;
    __syncthreads();
#pragma unroll
    for (int x = 0; x < NG; ++x) most = fmaxf(most, tops[x]);
    const float was = exp2_approx(top - most);
    top = most;
    sum *= was;
    v *= was;
    const auto add = [&](int i, float vi) {
      const float by = exp2_approx(weight[i].x - top - down);
      sum = fmaf(weight[i].y, by, sum);
      if (weight[i].y != 0.0f) v = fmaf(vi, by, v);  // (tokens that are not there leave nothing)
    };
    if (i0 == 0) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i)
        if (i < here) add(i, ahead[i]);
    }
#pragma unroll 8
    for (int i = i0 == 0 ? AHEAD : 0; i < here; ++i) add(i, __ldg(part + (int64_t)(i0 + i) * HT * PART + d));
    __syncthreads();
  }
  store_decoded<D>(p, ((int64_t)b * p.heads + h) * D + d, sum == 0.0f ? 0.0f : __fdiv_rn(v, sum));
}

struct DecodePlan {
  int cols, pieces, blocks;
  size_t before_bytes, bytes;
};
// A CTA on every SM, or as many as there can be units for.  Units are counted in 31 bits.
bool plan_decode(const CacheView& c, int dim, int heads, DecodePlan* d) {
  const int group = heads / c.heads;
  d->cols = group > 8 ? 16 : group > 4 ? 8 : 4;
  d->pieces = (group + d->cols - 1) / d->cols;
  const double lines = (double)c.sequences * c.heads * d->pieces, most = std::ceil((double)c.width * c.page / UNIT);
  if (most * lines > 2147483647.0 - 65536.0) return false;
  const double resident = device_sms(), useful = most * lines;
  d->blocks = useful < 1 ? 1 : (int)(useful < resident ? useful : resident);
  d->before_bytes = ((size_t)(c.sequences + 1) * sizeof(int) + 255) / 256 * 256;
  d->bytes = d->before_bytes + ((size_t)d->blocks * DEC_WARPS + (size_t)lines) * d->cols * (dim + 2) * sizeof(float);
  return true;
}

template <typename T, int NG, int HT>
cudaError_t launch_decode(const DecodeParams& p, cudaStream_t stream) {
  cudaError_t e = cudaFuncSetAttribute(cache_attention_kernel<T, NG, HT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kDecodeSmem<NG>);
  if (e != cudaSuccess) return e;
  e = launch_after(cache_attention_kernel<T, NG, HT>, dim3((unsigned)(p.warps / DEC_WARPS)), DEC_THREADS, kDecodeSmem<NG>, stream, p);
  if (e != cudaSuccess) return e;
  return launch_after(cache_combine_kernel<NG, HT>, dim3((unsigned)p.heads, (unsigned)p.c.sequences), 32 * NG, 0, stream, p);
}
template <typename T>
cudaError_t launch_decode(const DecodeParams& p, int dim, int cols, cudaStream_t stream) {
  const auto go = [&](auto ng) {
    constexpr int NG = decltype(ng)::value;
    return cols == 4 ? launch_decode<T, NG, 4>(p, stream) : cols == 8 ? launch_decode<T, NG, 8>(p, stream) : launch_decode<T, NG, 16>(p, stream);
  };
  switch (dim) {
    case 32: return go(std::integral_constant<int, 1>());
    case 64: return go(std::integral_constant<int, 2>());
    case 96: return go(std::integral_constant<int, 3>());
    default: return go(std::integral_constant<int, 4>());
  }
}

// LBA_OK and the view, or why not
int view_of(const lba_cache* c, CacheView* v) {
  if (!c) return LBA_ERR_NULL;
  if (c->page_count < 0 || c->page_count > 2147483647LL || c->kv_heads < 1 || c->kv_heads > 4095 || c->dim < 32 || c->dim > 128 || c->dim % 32 ||
      c->page < 16 || c->page > 1024 || c->page % 16 || c->sequences < 0 || c->sequences > 65535 || c->table_width < 0 ||
      c->table_width > (2147483647 - 8192) / c->page)
    return LBA_ERR_SHAPE;
  if (reinterpret_cast<uintptr_t>(c->pages) & 15) return LBA_ERR_ALIGN;
  v->pages = static_cast<uint8_t*>(c->pages);
  v->table = c->table;
  v->page_count = c->page_count;
  v->heads = c->kv_heads;
  v->page = c->page;
  v->sequences = c->sequences;
  v->width = c->table_width;
  return LBA_OK;
}

int rows_params(RowsParams* p, const lba_cache* cache, int type, int64_t tokens, const int32_t* start, const int32_t* cu, const void* k, const void* v) {
  const int st = view_of(cache, &p->c);
  if (st != LBA_OK) return st;
  if (type != LBA_TYPE_F32 && !half_type(type)) return LBA_ERR_LAYER;
  if (tokens < 0 || tokens > 2147483647LL) return LBA_ERR_SHAPE;
  if (tokens > 0 && cache->sequences > 0) {
    if (!start || !k || !v || (cache->page_count > 0 && !cache->pages) || (cache->table_width > 0 && !cache->table)) return LBA_ERR_NULL;
  }
  p->k = k;
  p->v = v;
  p->tokens = tokens;
  p->start = start;
  p->cu = cu;
  return LBA_OK;
}

}  // namespace
}  // namespace lba

using namespace lba;

extern "C" {

int lba_cache_append(const lba_cache* cache, const void* k, lba_strides k_at, const void* v, lba_strides v_at, int type, int64_t tokens,
                     const int32_t* start, const int32_t* cu, void* stream) {
  RowsParams p = {};
  const int st = rows_params(&p, cache, type, tokens, start, cu, k, v);
  if (st != LBA_OK) return st;
  if (tokens == 0 || cache->sequences == 0) return LBA_OK;
  p.k_at = k_at;
  p.v_at = v_at;
  return status_of(launch_rows<false>(p, cache->dim, type, (cudaStream_t)stream));
}

int lba_cache_read(const lba_cache* cache, const int32_t* start, const int32_t* cu, int64_t tokens, int type, void* k, void* v, void* stream) {
  RowsParams p = {};
  const int st = rows_params(&p, cache, type, tokens, start, cu, k, v);
  if (st != LBA_OK) return st;
  if (tokens == 0 || cache->sequences == 0) return LBA_OK;
  p.k_at.token = p.v_at.token = (int64_t)cache->kv_heads * cache->dim;
  p.k_at.head = p.v_at.head = cache->dim;
  return status_of(launch_rows<true>(p, cache->dim, type, (cudaStream_t)stream));
}

size_t lba_cache_attention_workspace_bytes(const lba_cache* cache, int heads) {
  CacheView c;
  if (view_of(cache, &c) != LBA_OK || heads < 1 || heads > 65535 || heads % c.heads) return 0;
  DecodePlan plan;
  return plan_decode(c, cache->dim, heads, &plan) ? plan.bytes : 0;
}

int lba_cache_attention(const void* q, lba_strides q_at, int type, int heads, const lba_cache* cache, const int32_t* lengths, float scale,
                        int out_type, const float* out_scale, int out_flags, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  DecodeParams p = {};
  const int st = view_of(cache, &p.c);
  if (st != LBA_OK) return st;
  if (heads < 1 || heads > 65535 || heads % cache->kv_heads) return LBA_ERR_SHAPE;
  if (!half_type(type) || (out_type != type && out_type != LBA_TYPE_CODES) || (out_flags & ~LBA_FLAG_INPUT_M4E3) || !(scale > 0.0f) || !std::isfinite(scale))
    return LBA_ERR_LAYER;
  if (cache->sequences == 0) return LBA_OK;
  if (!q || !out || !lengths || (cache->page_count > 0 && !cache->pages) || (cache->table_width > 0 && !cache->table)) return LBA_ERR_NULL;
  if (out_type == LBA_TYPE_CODES && !out_scale) return LBA_ERR_NULL;
  DecodePlan plan;
  if (!plan_decode(p.c, cache->dim, heads, &plan)) return LBA_ERR_SHAPE;
  if ((!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < plan.bytes)) return LBA_ERR_WORKSPACE;
  p.q = q;
  p.q_at = q_at;
  p.lengths = lengths;
  p.heads = heads;
  p.group = heads / cache->kv_heads;
  p.pieces = plan.pieces;
  p.warps = plan.blocks * DEC_WARPS;
  p.scale = scale;
  p.out_type = out_type;
  p.in_m4e3 = out_flags & LBA_FLAG_INPUT_M4E3;
  p.out_scale = out_scale;
  p.out = out;
  p.before = static_cast<int*>(workspace);
  p.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + plan.before_bytes);
  return status_of(type == LBA_TYPE_BF16 ? launch_decode<__nv_bfloat16>(p, cache->dim, plan.cols, (cudaStream_t)stream)
                                         : launch_decode<__half>(p, cache->dim, plan.cols, (cudaStream_t)stream));
}

}  // extern "C"
