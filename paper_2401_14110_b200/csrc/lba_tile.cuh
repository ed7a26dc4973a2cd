// Matrix instructions of one CTA (tcgen05, cta_group::1) on operands in shared and tensor memory, for the attention kernels.
//
// Tiles lie as tensor copies leave them under the 128-byte swizzle: blocks of 64 values of the head's dimension, each [rows][128 bytes].
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "lba_async.cuh"
#include "lba_entry.cuh"
#include "lba_layer.cuh"

namespace lba {

// ------------------------------------------------------------------ tensor memory
__device__ __forceinline__ void tmem_alloc(uint32_t slot, int columns) {  // one warp; the address comes back in shared memory
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(uint32_t tmem, int columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(columns) : "memory");
}
__device__ __forceinline__ void tmem_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// 32 columns of this warp's lanes
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
        "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
        "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
        "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, %17, %18, %19, "
      "%20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}

// ------------------------------------------------------------------ products
// Shared-memory operand of a matrix instruction.  Values of the summed index side by side (128-byte lines of 64): `stride` is the step between
// groups of eight rows.  The other index side by side: a line is 64 rows at one summed index, `stride` the step between groups of eight lines,
// `lead` the one between blocks of 64 rows.
__device__ __forceinline__ uint64_t tile_operand(uint32_t addr, int lead, int stride) {
  return (uint64_t)((addr >> 4) & 0x3FFF) | ((uint64_t)(lead >> 4) << 16) | ((uint64_t)(stride >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// binary32 sums of 128 x n products of bfloat16 or binary16 values; b_mn: B's rows side by side
__device__ __forceinline__ uint32_t tile_kind(bool bf, int n, bool b_mn) {
  return (1u << 4) | (bf ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) | ((uint32_t)(n / 8) << 17) | ((128u / 16) << 24);
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t kind, bool add) {  // A in shared memory
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a),
               "l"(b), "r"(kind), "r"((uint32_t)add) : "memory");
}
__device__ __forceinline__ void mma_tensor(uint32_t d, uint32_t a, uint64_t b, uint32_t kind, bool add) {  // A in tensor memory, two values a column
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d), "r"(a),
               "l"(b), "r"(kind), "r"((uint32_t)add) : "memory");
}
// arrives when everything that this thread has issued is done
__device__ __forceinline__ void mma_arrive(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void map_ahead(const CUtensorMap* map) { asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory"); }
// rows y.. of head h, values x to x + 63, as a block of a tile
__device__ __forceinline__ void tile_load(uint32_t dst, const CUtensorMap* map, int x, int h, int y, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst), "l"(map),
               "r"(x), "r"(h), "r"(y), "r"(bar) : "memory");
}
// the byte of (row, 16-byte piece) in a block under the swizzle
__device__ __forceinline__ int swizzled(int row, int piece) { return row * 128 + ((piece ^ (row & 7)) << 4); }

template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {
  uint32_t d;
  if constexpr (std::is_same<T, __nv_bfloat16>::value) asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  else asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(d) : "f"(hi), "f"(lo));
  return d;
}

// [rows][heads][dim] with these strides, in boxes of 64 values of one head and `box` rows; what lies past the head's values or the last row is 0
inline bool head_map(CUtensorMap* map, bool bf, const void* base, int64_t rows, int heads, int dim, lba_strides at, int box) {
  const EncodeTiled encode = tensor_map_encoder();
  if (!encode) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)dim, (cuuint64_t)heads, (cuuint64_t)rows};
  // (the stride of an index that is always 0 may be anything, and is often 1 or 0)
  const cuuint64_t strides[2] = {(cuuint64_t)(heads > 1 ? at.head * 2 : 16), (cuuint64_t)(rows > 1 ? at.token * 2 : 16)};
  const cuuint32_t boxes[3] = {64, 1, (cuuint32_t)box}, step[3] = {1, 1, 1};
  return encode(map, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, boxes, step,
                CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A tile's row: to 0; or rid of values that are not finite, true if it had any.  (A line's eight loads come first, then a sum that carries into a sign
// bit from exponents of ones only: with loads and tests in turn a tile took one warp 5000 clocks.)
template <int BLOCKS>
__device__ __forceinline__ void clear_row(uint8_t* tile, int row) {
#pragma unroll
  for (int x = 0; x < BLOCKS; ++x)
#pragma unroll
    for (int piece = 0; piece < 8; ++piece) *reinterpret_cast<uint4*>(tile + x * 128 * 128 + swizzled(row, piece)) = make_uint4(0u, 0u, 0u, 0u);
}
template <typename T, int BLOCKS>
__device__ __forceinline__ bool keep_finite(uint8_t* tile, int row) {
  constexpr uint32_t EXP = std::is_same<T, __nv_bfloat16>::value ? 0x7F807F80u : 0x7C007C00u, ONE = std::is_same<T, __nv_bfloat16>::value ? 0x00800080u : 0x04000400u;
  constexpr uint32_t SIGNS = 0x80008000u;
  bool any = false;
#pragma unroll 1
  for (int x = 0; x < BLOCKS; ++x) {
    uint4 v[8];
#pragma unroll
    for (int piece = 0; piece < 8; ++piece) v[piece] = *reinterpret_cast<const uint4*>(tile + x * 128 * 128 + swizzled(row, piece));
    uint32_t here = 0;
#pragma unroll
    for (int piece = 0; piece < 8; ++piece)
      here |= ((v[piece].x & EXP) + ONE) | ((v[piece].y & EXP) + ONE) | ((v[piece].z & EXP) + ONE) | ((v[piece].w & EXP) + ONE);
    if (!(here & SIGNS)) continue;
    any = true;
#pragma unroll 1
    for (int piece = 0; piece < 8; ++piece) {
      uint32_t* const u = reinterpret_cast<uint32_t*>(tile + x * 128 * 128 + swizzled(row, piece));
#pragma unroll 1
      for (int e = 0; e < 4; ++e) {
        const uint32_t bad = ((u[e] & EXP) + ONE) & SIGNS;  // a value's sign bit, where all of the value goes
        u[e] &= ~(bad | (bad - (bad >> 15)));
      }
    }
  }
  return any;
}

// ------------------------------------------------------------------ packed sequences
// the rows of sequence b: from first on, `count` of them
__device__ __forceinline__ void rows_of(const int32_t* cu, int64_t rows, int b, int* first, int* count) {
  if (!cu) {
    *first = 0;
    *count = (int)rows;
    return;
  }
  const int top = (int)rows, lo = min(max(cu[b], 0), top), hi = min(max(cu[b + 1], 0), top);
  *first = lo;
  *count = max(hi - lo, 0);
}
// Where a block of `size` rows lies: of a sequence with `blocks` of them, the one with `level` blocks that have less to do (or as much).
struct Place {
  int found, level, blocks, q_first, q_count, k_first, k_count, sequence;
};
// Block `index` of all sequences' blocks of their rows of q, or of k; a warp, every lane the same arguments and results.  With up to 128
// sequences, blocks of high levels come first, whatever their sequence: a launch ends with short ones (seven sequences of 1 to 2003 rows, the
// longest one last, took 52 us in the sequences' order).  With more, sequence by sequence.  One trip to memory for both kinds of rows.
__device__ __forceinline__ Place find_place(const int32_t* cu_q, int64_t q_rows, const int32_t* cu_k, int64_t k_rows, int sequences, bool by_keys, int size,
                                            int64_t index) {
  const int lane = threadIdx.x & 31;
  Place p = {};
  const auto blocks_of = [&](int b, Place& x) -> int {
    x.q_count = x.k_count = 0;
    if (b >= sequences) return 0;
    rows_of(cu_q, q_rows, b, &x.q_first, &x.q_count);
    rows_of(cu_k, k_rows, b, &x.k_first, &x.k_count);
    return ((by_keys ? x.k_count : x.q_count) + size - 1) / size;
  };
  const auto take = [&](const Place& x, int from) {
    p.found = 1;
    p.q_first = __shfl_sync(0xFFFFFFFFu, x.q_first, from);
    p.q_count = __shfl_sync(0xFFFFFFFFu, x.q_count, from);
    p.k_first = __shfl_sync(0xFFFFFFFFu, x.k_first, from);
    p.k_count = __shfl_sync(0xFFFFFFFFu, x.k_count, from);
    p.blocks = ((by_keys ? p.k_count : p.q_count) + size - 1) / size;
  };
  constexpr int MANY = 4;
  if (sequences <= 32 * MANY) {
    Place x[MANY];
    int n[MANY], most = 0;
#pragma unroll
    for (int i = 0; i < MANY; ++i) n[i] = 32 * i < sequences ? blocks_of(32 * i + lane, x[i]) : 0;
#pragma unroll
    for (int i = 0; i < MANY; ++i) most = max(most, n[i]);
    most = __reduce_max_sync(0xFFFFFFFFu, most);
    const auto from_level = [&](int t) -> int64_t {  // blocks of level t and above
      int64_t sum = 0;
#pragma unroll
      for (int i = 0; i < MANY; ++i)
        if (32 * i < sequences) sum += __reduce_add_sync(0xFFFFFFFFu, max(0, n[i] - t));
      return sum;
    };
    if (index >= from_level(0)) return p;
    int lo = 0, hi = most - 1;  // the highest level that index has reached
    while (lo < hi) {
      const int mid = (lo + hi + 1) / 2;
      if (from_level(mid) > index) lo = mid;
      else hi = mid - 1;
    }
    int rank = (int)(index - from_level(lo + 1));
#pragma unroll
    for (int i = 0; i < MANY; ++i) {
      if (32 * i >= sequences || p.found) continue;
      const unsigned has = __ballot_sync(0xFFFFFFFFu, n[i] > lo);
      if (rank < __popc(has)) {
        const int l = __fns(has, 0, rank + 1);
        take(x[i], l);
        p.sequence = 32 * i + l;
      } else {
        rank -= __popc(has);
      }
    }
    p.level = lo;
    return p;
  }
  for (int b0 = 0; b0 < sequences; b0 += 32) {
    Place x;
    const int n = blocks_of(b0 + lane, x);
    int upto = n;
#pragma unroll
    for (int d = 1; d < 32; d *= 2) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, upto, d);
      if (lane >= d) upto += v;
    }
    const unsigned hit = __ballot_sync(0xFFFFFFFFu, index < upto);
    if (hit) {
      const int l = __ffs(hit) - 1;
      take(x, l);
      p.sequence = b0 + l;
      p.level = __shfl_sync(0xFFFFFFFFu, upto, l) - 1 - (int)index;
      return p;
    }
    index -= __shfl_sync(0xFFFFFFFFu, upto, 31);
  }
  return p;
}

int check_attention(const lba_attention_how* how);  // lba_attention.cu

}  // namespace lba
