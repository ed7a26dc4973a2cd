// A key-value cache in 4 bits: what is appended is rounded to E2M1 values under a power of two per 32 (include/lba.h has the layout), and
// the attention of single tokens reads it as it lies.
//
// Attention is bound by memory: a (token, head) of 128 dimensions is 136 bytes and 512 g multiply-adds for the g query heads that share it.
// Eight heads together want 190 TFLOP/s at 6.4 TB/s, out of reach of the CUDA cores, so both products run on the tensor cores, and a warp
// feeds them from registers: m16n8k16 with 16 tokens (keys) or 16 dimensions (values) as rows and eight query heads as columns.  tcgen05
// would have a tile of 128 rows and operands in shared memory, where 4-bit values would have to be widened first.
//   S = K Q^T   E2M1 values are exact in binary16 (one conversion instruction for two).  The bytes of a key row stand so that a lane's 16
//               bytes are its operands of all k-steps, and both k-steps of a group of 32 lie in it: the group's power of two multiplies a
//               finished 32-term sum, in binary32
//   softmax     one pass; a running maximum per head that is raised only when a score exceeds it by 2^5, so that a vote replaces the
//               reduction of most steps
//   O = V^T P   P goes from accumulator to operand layout by the matrix transpose, with 10 bits of headroom below; the values' powers of two
//               differ by token and group, so P is multiplied by them, relative to the largest that the warp has met in the group (15 and
//               more binades below it they count as 0: 2^-15 of the largest value).  binary16: 2^-12 of a weight
// A query head is brought to [1, 2) by a power of two first and is then exact in binary16 but for what lies 2^-14 below its largest value.
// Loads go straight to registers, two steps of 16 tokens ahead of the one computed; no shared memory, no barriers until the end.
#include <cmath>

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

// A thread takes eight neighbouring values: a quarter of a group.  Blocks are rows (tokens) of one head's keys or values.
template <int D> constexpr int kRowSplit = D / 8;
template <int D> constexpr int kBlockRows = ROW_THREADS / kRowSplit<D>;

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

template <typename T, int D, bool READ>
__global__ void __launch_bounds__(ROW_THREADS) cache_rows_kernel(const RowsParams p) {
  constexpr int SPLIT = kRowSplit<D>, ROWS = kBlockRows<D>;
  __shared__ int32_t cu[MAX_CU];
  __shared__ __align__(16) uint8_t stage[ROWS * D / 2];
  after_previous();
  const bool values = blockIdx.y >= (unsigned)p.c.heads;
  const int head = blockIdx.y - (values ? p.c.heads : 0);
  const int r = threadIdx.x / SPLIT, q = threadIdx.x % SPLIT;  // row of the block, eighth values q
  const int64_t t = (int64_t)blockIdx.x * ROWS + r;
  const bool there = r < ROWS && t < p.tokens;
  const lba_strides at = values ? p.v_at : p.k_at;
  T* const mine = static_cast<T*>(const_cast<void*>(values ? p.v : p.k)) + t * at.token + head * at.head + q * 8;
  float x[8];
  if (!READ && there) load8<T>(mine, x);   // on its way while the token's place is looked up
  if (p.cu && p.c.sequences < MAX_CU) {
    for (int i = threadIdx.x; i <= p.c.sequences; i += ROW_THREADS) cu[i] = p.cu[i];
    __syncthreads();
  }
  int64_t page = -1;
  int row = 0;
  bool in_sequence = there;
  if (there) {
    const bool found = locate(p, cu, t, &page, &row);
    if (!found) page = -1;
    if (READ && p.cu) {  // (a row of a sequence whose token is not there reads as 0; one of no sequence is left)
      in_sequence = found || (t >= (p.c.sequences < MAX_CU ? cu[0] : p.cu[0]) && t < (p.c.sequences < MAX_CU ? cu[p.c.sequences] : p.cu[p.c.sequences]));
    } else if (READ) {
      in_sequence = t < p.c.sequences;
    }
  }
  uint8_t* const codes = page < 0 ? nullptr : plane<D>(p.c, page, head, values ? 1 : 0) + (int64_t)row * (D / 2);
  uint8_t* const exps = page < 0 ? nullptr : plane<D>(p.c, page, head, values ? 3 : 2) + (int64_t)row * (D / 32);
  uint8_t* const line = stage + r * (D / 2);
  // a key row's eighth q = 4 g + c is the word at c D/8 + 4 g; a value row's q = 2 i + h are bytes (4 h + j) D/16 + i
  const int word_at = (q & 3) * (D / 8) + (q >> 2) * 4;
  if constexpr (!READ) {
    uint32_t top = 0;
    if (there) {
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, __float_as_uint(x[j]) & 0x7FFFFFFFu);
    }
    // the four lanes of a group (SPLIT is a multiple of four; rows that are not there reduce zeros)
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = max(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    const bool lost = top >= 0x7F800000u;
    int e = (int)(top >> 23) - 129 + ((top & 0x7FFFFFu) > 0x400000u);  // 1.f 2^E <= 1.5 2^(e+2)
    e = e < -126 ? -126 : e > 125 ? 125 : e;  // (6 2^126 is no binary32 number)
    const float by = __uint_as_float((uint32_t)(127 - e) << 23);
    if (there && page >= 0) {
      uint32_t w = 0;
      if (!lost) {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= by;
        w = encode8(x);
      }
      if (values) {
#pragma unroll
        for (int j = 0; j < 4; ++j) line[((q & 1) * 4 + j) * (D / 16) + (q >> 1)] = (uint8_t)(w >> (8 * j));
      } else {
        *reinterpret_cast<uint32_t*>(codes + word_at) = w;
      }
      if ((q & 3) == 0) exps[q >> 2] = lost ? 255 : (uint8_t)(e + 127);
    }
    if (!values) return;
    __syncthreads();
    if (there && page >= 0) *reinterpret_cast<uint32_t*>(codes + 4 * q) = *reinterpret_cast<const uint32_t*>(line + 4 * q);
  } else {
    uint32_t w = 0, exp = 0;
    if (page >= 0) {
      w = *reinterpret_cast<const uint32_t*>(codes + (values ? 4 * q : word_at));
      exp = exps[q >> 2];
    }
    if (values) {
      if (there) *reinterpret_cast<uint32_t*>(line + 4 * q) = w;
      __syncthreads();
      w = 0;
      if (there) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w |= (uint32_t)line[((q & 1) * 4 + j) * (D / 16) + (q >> 1)] << (8 * j);
      }
    }
    if (!in_sequence) return;
    uint32_t h[4];
    decode8(w, h);
    const float by = exp == 255 ? __uint_as_float(0x7FC00000u) : __uint_as_float(exp << 23);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float2 f = widen(h[j]);
      x[2 * j] = f.x * by;
      x[2 * j + 1] = f.y * by;
    }
    store8<T>(mine, x);
  }
}

template <bool READ, typename T>
cudaError_t launch_rows(const RowsParams& p, int dim, cudaStream_t stream) {
  const auto go = [&](auto d) {
    constexpr int D = decltype(d)::value;
    return launch_after(cache_rows_kernel<T, D, READ>, dim3((unsigned)((p.tokens + kBlockRows<D> - 1) / kBlockRows<D>), (unsigned)(2 * p.c.heads)),
                        ROW_THREADS, 0, stream, p);
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
constexpr int DEC_WARPS = 8, DEC_THREADS = 32 * DEC_WARPS, STEP = 16;
constexpr float HEADROOM = 5.0f;     // binades by which a score may exceed its head's running maximum
constexpr float P_SCALE = 1024.0f;   // weights in binary16: at most 2^(10 + 5)
constexpr float NO_MAX = -1e30f;

struct DecodeParams {
  CacheView c;
  const void* q;
  lba_strides q_at;
  const int32_t* lengths;
  int heads, group, blocks_of_heads;  // query heads; of a key-value head; pieces of 8 NT of a group
  int chunk, chunks;                  // tokens of a CTA, most CTAs of a sequence's head
  float scale;
  int out_type, in_m4e3;
  const float* out_scale;
  void* out;
  float* parts;                       // [sequence][key-value head][piece][chunk][8 NT heads][D + 2]
};

__device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
template <int N>
__device__ __forceinline__ uint32_t load_exponents(const uint8_t* p) {
  if constexpr (N == 4) return __ldg(reinterpret_cast<const uint32_t*>(p));
  if constexpr (N == 2) return __ldg(reinterpret_cast<const uint16_t*>(p));
  if constexpr (N == 1) return __ldg(p);
  return (uint32_t)__ldg(p) | ((uint32_t)__ldg(p + 1) << 8) | ((uint32_t)__ldg(p + 2) << 16);
}

// what a lane needs of 16 tokens: rows r and r + 8 of the keys (r = lane / 4), tokens 2 c, 2 c + 1, 2 c + 8, 2 c + 9 of the values (c = lane % 4)
template <int NG>
struct Step16 {
  uint32_t k[2][NG], ke[2], v[4][(NG + 1) / 2], ve[4];
  __device__ __forceinline__ void load(const CacheView& cache, int64_t page, int head, int row, int r, int c) {
    constexpr int D = 32 * NG;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const uint8_t* const src = plane<D>(cache, page, head, 0) + (int64_t)(row + r + 8 * i) * (D / 2) + c * (D / 8);
      if constexpr (NG == 4) {
        const uint4 w = __ldg(reinterpret_cast<const uint4*>(src));
        k[i][0] = w.x, k[i][1] = w.y, k[i][2] = w.z, k[i][3] = w.w;
      } else if constexpr (NG == 2) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(src));
        k[i][0] = w.x, k[i][1] = w.y;
      } else {
#pragma unroll
        for (int g = 0; g < NG; ++g) k[i][g] = __ldg(reinterpret_cast<const uint32_t*>(src) + g);
      }
      ke[i] = load_exponents<NG>(plane<D>(cache, page, head, 2) + (int64_t)(row + r + 8 * i) * NG);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int t = row + 2 * c + (i & 1) + (i >> 1) * 8;
      const uint8_t* const src = plane<D>(cache, page, head, 1) + (int64_t)t * (D / 2) + r * (D / 16);
      if constexpr (NG == 4) {
        const uint2 w = __ldg(reinterpret_cast<const uint2*>(src));
        v[i][0] = w.x, v[i][1] = w.y;
      } else if constexpr (NG == 2) {
        v[i][0] = __ldg(reinterpret_cast<const uint32_t*>(src));
      } else {
        const uint16_t* const s = reinterpret_cast<const uint16_t*>(src);
        v[i][0] = __ldg(s);
        if constexpr (NG == 3) {
          v[i][0] |= (uint32_t)__ldg(s + 1) << 16;
          v[i][1] = __ldg(s + 2);
        }
      }
      ve[i] = load_exponents<NG>(plane<D>(cache, page, head, 3) + (int64_t)t * NG);
    }
  }
};

// Eight columns' worth of outputs of one head of the batch, from parts in turn: their maxima, sums and unscaled outputs
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

// of a sequence: what its length and its row of the table allow (below 2^31 - 2 chunk: view_of)
__device__ __forceinline__ int tokens_of(const DecodeParams& p, int b) { return max(0, min(p.lengths[b], p.c.width * p.c.page)); }

template <typename T, int NG, int NT>
__global__ void __launch_bounds__(DEC_THREADS, NT == 1 ? 2 : 1) cache_attention_kernel(const DecodeParams p) {
  constexpr int D = 32 * NG, COLS = 8 * NT, PART = D + 2;
  extern __shared__ float merge[];  // [warp][COLS][D + 2]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = lane >> 2, c = lane & 3;
  after_previous();
  const int b = blockIdx.z, piece = blockIdx.y % p.blocks_of_heads, kvh = blockIdx.y / p.blocks_of_heads;
  const int length = tokens_of(p, b), first = blockIdx.x * p.chunk;
  if (first >= length && p.chunks != 1) return;  // (with a single chunk the outputs of empty sequences are written here)
  const int tokens = min(p.chunk, length - first), steps = tokens > 0 ? (tokens + STEP - 1) / STEP : 0;  // 16-token steps, cut among the warps
  const int s0 = steps * warp / DEC_WARPS, s1 = steps * (warp + 1) / DEC_WARPS;
  const int32_t* const table = p.c.table + (int64_t)b * p.c.width;

  const auto page_of = [&](int s) -> int {  // of step s of this CTA; -1: not there
    if (s >= s1) return -1;
    const int pg = __ldg(table + (first + s * STEP) / p.c.page);
    return pg >= 0 && pg < p.c.page_count ? pg : -1;
  };
  // pages of the next 32 steps, one a lane
  int window = s0, pages = page_of(s0 + lane);
  const auto next_page = [&](int s) -> int {  // warp-uniform, s ascending
    if (s - window >= 32) {
      window = s;
      pages = page_of(s + lane);
    }
    return __shfl_sync(0xFFFFFFFFu, pages, s - window);
  };
  Step16<NG> ahead[2];
  int at[2], row = (first + s0 * STEP) % p.c.page;
  const auto fetch = [&](int u, int s) {  // of one step after another
    at[u] = s < s1 ? next_page(s) : -1;
    if (at[u] >= 0) ahead[u].load(p.c, at[u], kvh, row, r, c);
    row = row + STEP == p.c.page ? 0 : row + STEP;
  };
  fetch(0, s0);
  fetch(1, s0 + 1);

  // query heads: column r of a tile; values 32 g + 8 c to + 7
  uint32_t q[NT][NG][4];
  float to_log2[NT][2];  // of columns 2 c and 2 c + 1
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int h = piece * COLS + n * 8 + r;
    float x[NG][8], top = 0.0f;
    const bool there = h < p.group;
    const T* const src = static_cast<const T*>(p.q) + (int64_t)b * p.q_at.token + (int64_t)(kvh * p.group + h) * p.q_at.head + c * 8;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      load_some<T, 8>(src, g * 32, there ? 8 : 0, x[g]);
#pragma unroll
      for (int j = 0; j < 8; ++j) top = fmaxf(top, fabsf(x[g][j]));
    }
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
    top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
    int e = (int)(__float_as_uint(top) >> 23) - 127;  // (infinities stay what they are under any factor)
    e = e < -126 ? -126 : e > 126 ? 126 : e;
    const float down = __uint_as_float((uint32_t)(127 - e) << 23), up = __uint_as_float((uint32_t)(127 + e) << 23) * (p.scale * LOG2E);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
      for (int j = 0; j < 4; ++j) q[n][g][j] = half_pair(x[g][2 * j] * down, x[g][2 * j + 1] * down);
#pragma unroll
    for (int j = 0; j < 2; ++j) to_log2[n][j] = __shfl_sync(0xFFFFFFFFu, up, (2 * c + j) * 4);
  }

  float o[NT][2 * NG][4], m[NT][2], l[NT][2];
  uint32_t ref = 0;  // the largest exponent byte of each group so far
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int i = 0; i < 2 * NG; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) o[n][i][j] = 0.0f;
    m[n][0] = m[n][1] = NO_MAX;
    l[n][0] = l[n][1] = 0.0f;
  }

  const auto compute = [&](Step16<NG>& w, int s) {
    const int left = tokens - s * STEP;  // tokens of this step that exist
    float z[NT][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[n][j] = 0.0f;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      uint32_t lo[4], hi[4];
      decode8(w.k[0][g], lo);
      decode8(w.k[1][g], hi);
      const int up = 23 - 8 * g;
      float by[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) by[i] = __uint_as_float((up >= 0 ? w.ke[i] << (up & 31) : w.ke[i] >> (-up & 31)) & 0x7F800000u);
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]}, a1[4] = {lo[2], hi[2], lo[3], hi[3]};
        mma16816(sum, a0, q[n][g][0], q[n][g][1]);
        mma16816(sum, a1, q[n][g][2], q[n][g][3]);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[n][j] = fmaf(sum[j], by[j >> 1], z[n][j]);
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) z[n][j] *= to_log2[n][j & 1];
    if (left < STEP) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (r + (j >> 1) * 8 >= left) z[n][j] = -INFINITY;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (2 * c + (i & 1) + (i >> 1) * 8 >= left) w.ve[i] = 0;
    }
    uint32_t top = max_bytes(max_bytes(w.ve[0], w.ve[1]), max_bytes(w.ve[2], w.ve[3]));
    bool raise = max_bytes(top, ref) != ref;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) raise |= z[n][j] > m[n][j & 1] + HEADROOM;
    if (__any_sync(0xFFFFFFFFu, raise)) {
      top = max_bytes(top, __shfl_xor_sync(0xFFFFFFFFu, top, 1));
      top = max_bytes(top, __shfl_xor_sync(0xFFFFFFFFu, top, 2));
      const uint32_t old = ref;
      ref = max_bytes(ref, top);
      const uint32_t by = ref - old;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float a[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          float t = fmaxf(fmaxf(z[n][j], z[n][j + 2]), m[n][j]);
          t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 4));
          t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 8));
          t = fmaxf(t, __shfl_xor_sync(0xFFFFFFFFu, t, 16));
          a[j] = exp2_approx(m[n][j] - t);
          m[n][j] = t;
          l[n][j] *= a[j];
        }
#pragma unroll
        for (int i = 0; i < 2 * NG; ++i) {
          const int d = (by >> (8 * (i >> 1))) & 255;
          const float down = d > 126 ? 0.0f : __uint_as_float((uint32_t)(127 - d) << 23);
#pragma unroll
          for (int j = 0; j < 4; ++j) o[n][i][j] *= a[j & 1] * down;
        }
      }
    }
    // weights as operands: rows of the transposed 8 x 8 blocks are heads, columns tokens
    uint32_t w0[NT], w1[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float e[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        e[j] = exp2_approx(z[n][j] - m[n][j & 1]);
        l[n][j & 1] += e[j];
      }
      w0[n] = transposed(half_pair(e[0] * P_SCALE, e[1] * P_SCALE));
      w1[n] = transposed(half_pair(e[2] * P_SCALE, e[3] * P_SCALE));
    }
    uint32_t below[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) below[i] = ref - w.ve[i];  // (no byte borrows)
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      // 2^-d of two tokens in binary16, 0 from d = 15 on
      uint32_t f[2];
#pragma unroll
      for (int i = 0; i < 2; ++i)
        f[i] = 0x3C003C00u - (__vminu2(__byte_perm(below[2 * i], below[2 * i + 1], 0x0400 | (g << 8) | g) & 0x00FF00FFu, 0x000F000Fu) << 10);
      uint32_t b0[NT], b1[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        b0[n] = mul_halves(w0[n], f[0]);
        b1[n] = mul_halves(w1[n], f[1]);
      }
#pragma unroll
      for (int u = 0; u < 2; ++u) {
        const int i = 2 * g + u;
        uint32_t h[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const uint32_t word = w.v[t][i / 4] >> (8 * (i % 4));
          asm("{\n\t.reg .b8 a, b, c, d;\n\tmov.b32 {a, b, c, d}, %1;\n\tcvt.rn.f16x2.e2m1x2 %0, a;\n\t}" : "=r"(h[t]) : "r"(word));
        }
        const uint32_t a[4] = {__byte_perm(h[0], h[1], 0x5410), __byte_perm(h[0], h[1], 0x7632), __byte_perm(h[2], h[3], 0x5410),
                               __byte_perm(h[2], h[3], 0x7632)};
#pragma unroll
        for (int n = 0; n < NT; ++n) mma16816(o[n][i], a, b0[n], b1[n]);
      }
    }
  };
#pragma unroll 1
  for (int s = s0; s < s1; s += 2) {
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      Step16<NG> now = ahead[u];
      const bool there = at[u] >= 0;
      fetch(u, s + 2 + u);
      if (there) compute(now, s + u);
    }
  }

  // ---- the warps' sums together
  float* const mine = merge + warp * COLS * PART;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      float t = l[n][j];
      t += __shfl_xor_sync(0xFFFFFFFFu, t, 4);
      t += __shfl_xor_sync(0xFFFFFFFFu, t, 8);
      t += __shfl_xor_sync(0xFFFFFFFFu, t, 16);
      const int col = n * 8 + 2 * c + j;
      if (r == 0) {
        mine[col * PART + D] = m[n][j];
        mine[col * PART + D + 1] = t;
      }
#pragma unroll
      for (int i = 0; i < 2 * NG; ++i) {
        const uint32_t e = (ref >> (8 * (i >> 1))) & 255u;
        const float by = e == 255u ? __uint_as_float(0x7FC00000u) : __uint_as_float(e << 23);
        *reinterpret_cast<float2*>(mine + col * PART + 16 * i + 2 * r) =
            make_float2(o[n][i][j] * (1.0f / P_SCALE) * by, o[n][i][2 + j] * (1.0f / P_SCALE) * by);
      }
    }
  }
  __syncthreads();
  const int cols = p.group - piece * COLS < COLS ? p.group - piece * COLS : COLS;
  float* const part = p.parts + ((((int64_t)b * gridDim.y + blockIdx.y) * p.chunks + blockIdx.x) * COLS) * PART;
  for (int i = threadIdx.x; i < cols * D; i += DEC_THREADS) {
    const int col = i / D, d = i - col * D;
    float top = NO_MAX, sum = 0.0f, v = 0.0f;
#pragma unroll
    for (int w = 0; w < DEC_WARPS; ++w) top = fmaxf(top, merge[(w * COLS + col) * PART + D]);
#pragma unroll
    for (int w = 0; w < DEC_WARPS; ++w) {
      const float* const src = merge + (w * COLS + col) * PART;
      const float by = exp2_approx(src[D] - top);
      sum = fmaf(src[D + 1], by, sum);
      if (src[D + 1] != 0.0f) v = fmaf(src[d], by, v);  // (a warp without tokens has nothing to add)
    }
    if (p.chunks == 1) {
      const int64_t at_out = ((int64_t)b * p.heads + kvh * p.group + piece * COLS + col) * D + d;
      store_decoded<D>(p, at_out, sum == 0.0f ? 0.0f : __fdiv_rn(v, sum));
    } else {
      part[col * PART + d] = v;
      if (d == 0) {
        part[col * PART + D] = top;
        part[col * PART + D + 1] = sum;
      }
    }
  }
}

// the chunks' sums together: a block per head
template <int NG, int NT>
__global__ void __launch_bounds__(128) cache_combine_kernel(const DecodeParams p) {
  constexpr int D = 32 * NG, COLS = 8 * NT, PART = D + 2;
  after_previous();
  const int b = blockIdx.y, h = blockIdx.x, kvh = h / p.group, in_group = h - kvh * p.group, piece = in_group / COLS, col = in_group - piece * COLS;
  const int d = threadIdx.x;
  if (d >= D) return;
  const int n = (tokens_of(p, b) + p.chunk - 1) / p.chunk;
  const float* const part = p.parts + (((int64_t)b * p.c.heads * p.blocks_of_heads + kvh * p.blocks_of_heads + piece) * p.chunks) * COLS * PART + col * PART;
  float top = NO_MAX, sum = 0.0f, v = 0.0f;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const float* const src = part + (int64_t)i * COLS * PART;
    const float mx = __ldg(src + D), li = __ldg(src + D + 1), vi = __ldg(src + d);
    const float t = fmaxf(top, mx), was = exp2_approx(top - t), by = exp2_approx(mx - t);
    sum = sum * was + li * by;
    v = v * was;
    if (li != 0.0f) v = fmaf(vi, by, v);
    top = t;
  }
  store_decoded<D>(p, ((int64_t)b * p.heads + h) * D + d, sum == 0.0f ? 0.0f : __fdiv_rn(v, sum));
}

struct DecodePlan {
  int cols, pieces, chunk, chunks;
  size_t bytes;
};
// Tokens of a CTA: enough CTAs at full length for eight rounds over the SMs (lengths differ, and the host does not know them), 128 tokens at
// least, a step of every warp, and 4096 at most.
DecodePlan plan_decode(const CacheView& c, int dim, int heads) {
  DecodePlan d = {};
  const int group = heads / c.heads;
  d.cols = group > 8 ? 16 : 8;
  d.pieces = (group + d.cols - 1) / d.cols;
  const int64_t most = (int64_t)c.width * c.page, lines = (int64_t)c.sequences * c.heads * d.pieces;
  int64_t chunk = (int64_t)((double)most * (double)lines / (16.0 * device_sms()));
  chunk = (chunk + 127) / 128 * 128;
  chunk = chunk < 128 ? 128 : chunk > 4096 ? 4096 : chunk;
  d.chunk = (int)chunk;
  d.chunks = (int)(most <= chunk ? 1 : (most + chunk - 1) / chunk);
  d.bytes = d.chunks == 1 ? 0 : (size_t)lines * d.chunks * d.cols * (dim + 2) * sizeof(float);
  return d;
}

template <typename T, int NG, int NT>
cudaError_t launch_decode(const DecodeParams& p, cudaStream_t stream) {
  constexpr int D = 32 * NG;
  constexpr size_t smem = (size_t)DEC_WARPS * 8 * NT * (D + 2) * sizeof(float);
  cudaError_t e = cudaFuncSetAttribute(cache_attention_kernel<T, NG, NT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  e = launch_after(cache_attention_kernel<T, NG, NT>, dim3((unsigned)p.chunks, (unsigned)(p.c.heads * p.blocks_of_heads), (unsigned)p.c.sequences),
                   DEC_THREADS, smem, stream, p);
  if (e != cudaSuccess || p.chunks == 1) return e;
  return launch_after(cache_combine_kernel<NG, NT>, dim3((unsigned)p.heads, (unsigned)p.c.sequences), 128, 0, stream, p);
}
template <typename T>
cudaError_t launch_decode(const DecodeParams& p, int dim, int cols, cudaStream_t stream) {
  const auto go = [&](auto ng) {
    constexpr int NG = decltype(ng)::value;
    return cols == 8 ? launch_decode<T, NG, 1>(p, stream) : launch_decode<T, NG, 2>(p, stream);
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
  return plan_decode(c, cache->dim, heads).bytes;
}

int lba_cache_attention(const void* q, lba_strides q_at, int type, int heads, const lba_cache* cache, const int32_t* lengths, float scale,
                        int out_type, const float* out_scale, int out_flags, void* out, void* workspace, size_t workspace_bytes, void* stream) {
  DecodeParams p = {};
  const int st = view_of(cache, &p.c);
  if (st != LBA_OK) return st;
  if (heads < 1 || heads > 65535 || heads % cache->kv_heads) return LBA_ERR_SHAPE;
  if (!half_type(type) || (out_type != type && out_type != LBA_TYPE_CODES) || (out_flags & ~LBA_FLAG_INPUT_M4E3) || !std::isfinite(scale)) return LBA_ERR_LAYER;
  if (cache->sequences == 0) return LBA_OK;
  if (!q || !out || !lengths || (cache->page_count > 0 && !cache->pages) || (cache->table_width > 0 && !cache->table)) return LBA_ERR_NULL;
  if (out_type == LBA_TYPE_CODES && !out_scale) return LBA_ERR_NULL;
  const DecodePlan plan = plan_decode(p.c, cache->dim, heads);
  if (plan.bytes && (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) || workspace_bytes < plan.bytes)) return LBA_ERR_WORKSPACE;
  p.q = q;
  p.q_at = q_at;
  p.lengths = lengths;
  p.heads = heads;
  p.group = heads / cache->kv_heads;
  p.blocks_of_heads = plan.pieces;
  p.chunk = plan.chunk;
  p.chunks = plan.chunks;
  p.scale = scale;
  p.out_type = out_type;
  p.in_m4e3 = out_flags & LBA_FLAG_INPUT_M4E3;
  p.out_scale = out_scale;
  p.out = out;
  p.parts = static_cast<float*>(workspace);
  return status_of(type == LBA_TYPE_BF16 ? launch_decode<__nv_bfloat16>(p, cache->dim, plan.cols, (cudaStream_t)stream)
                                         : launch_decode<__half>(p, cache->dim, plan.cols, (cudaStream_t)stream));
}

}  // extern "C"
