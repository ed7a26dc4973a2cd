// Layers on few rows (a token, or the tokens of a few sequences that decode together), in chunks of 16.
//
// With one row every byte of the weights is read once and used once: the layer takes as long as its weights take to arrive (4096 x
// 4096: 16.8 MB, 2.6 us at the copy rate), if decoding and the chains keep up.  Tiles cannot: a 16x16 tile spends sixteen rows of work on one.
// Here a lane takes one chunk of one pair of columns (the two halves of a packed instruction) and walks its sixteen steps for
// every row, so nothing is computed that no output needs, a warp's lanes read 512 consecutive bytes of a row of weights, and
// the chunk sums of a column, which do not depend on each other, spread over the lanes.  What stays sequential is the second
// hierarchy, T <- Q_acc(C_j + T) in chunk order: one addition in sixteen, done by warps of their own a round behind.
//
//   rounds of 32 chunks (512 k).  Producer warps bring the round's weights into a ring of stages (one bulk copy per row) and decode
//   its activations into the same stage; compute warps take (round, pair) tasks in turn and leave the chunk sums in a second ring;
//   fold warps keep T of every (row, pair) in registers.  Barriers count tasks, so no warp waits for a whole round.
// A CTA owns as many pairs as fit, so that one wave of CTAs covers the columns where it can: the fold of a CTA's last round and the
// first load of the next would otherwise show.
// Steps and folds are those of the packed kernel, bit for bit; a chunk or eight folds run without the clamp of Eq. 2 where
// sum |a_k| max |b| (or |T| + sum |C_j|) shows that it cannot act.
#pragma once
#include "lba_async.cuh"
#include "lba_kernel_small.cuh"

namespace lba {

constexpr int ROWS_MAX = 16;                 // rows at most
constexpr int ROWS_CHUNKS = 32;              // chunks of a round: one per lane
constexpr int ROWS_COMPUTE = 16, ROWS_PRODUCE = 2, ROWS_FOLD = 4;  // warps
constexpr int ROWS_THREADS = 32 * (ROWS_COMPUTE + ROWS_PRODUCE + ROWS_FOLD);
constexpr int ROWS_CHAINS = 2;               // (row, pair) chains per lane of a fold warp, at most
constexpr int ROWS_SUM_RING = 3;
constexpr int ROWS_MAX_STAGES = 8;
constexpr int ROWS_PITCH = ROWS_CHUNKS + 2;  // pairs of sums from one chain to the next: 16-byte aligned, lanes on different banks

struct RowsProblem : LinearProblem {
  int pairs, stages;  // pairs of columns of a CTA
};
inline __host__ __device__ int rows_a_bytes(int M) { return M * (ROWS_CHUNKS * BK * 4 + ROWS_CHUNKS * 4); }
inline __host__ __device__ int rows_b_bytes(int pairs) { return 2 * pairs * ROWS_CHUNKS * BK; }
inline __host__ __device__ int rows_sum_bytes(int M, int pairs) { return M * pairs * ROWS_PITCH * 8; }
inline __host__ __device__ int rows_smem(int M, int pairs, int stages) {
  return stages * (rows_a_bytes(M) + rows_b_bytes(pairs)) + ROWS_SUM_RING * rows_sum_bytes(M, pairs) + 8 * 2 * (ROWS_MAX_STAGES + ROWS_SUM_RING) + 16;
}

template <bool SAT, int RNE, bool M4E3>
__global__ void __launch_bounds__(ROWS_THREADS, 1) lba_rows_kernel(const RowsProblem p) {
  extern __shared__ __align__(16) unsigned char smem_raw[];
  const int M = (int)p.M, pairs = p.pairs, stages = p.stages;
  const int a_bytes = rows_a_bytes(M), b_bytes = rows_b_bytes(pairs), s_bytes = rows_sum_bytes(M, pairs);
  unsigned char* const sums = smem_raw + stages * (a_bytes + b_bytes);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sums + ROWS_SUM_RING * s_bytes);
  volatile int* const dead = reinterpret_cast<volatile int*>(bars + 2 * (ROWS_MAX_STAGES + ROWS_SUM_RING));
  const uint32_t full = smem_u32(bars), empty = full + 8 * ROWS_MAX_STAGES, sum_full = empty + 8 * ROWS_MAX_STAGES,
                 sum_free = sum_full + 8 * ROWS_SUM_RING;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n0 = (int64_t)blockIdx.x * (2 * pairs);
  const int mine = (int)((p.N - n0 + 1) / 2 < pairs ? (p.N - n0 + 1) / 2 : pairs);  // pairs of this CTA
  const int chunks = (int)(p.K / BK), rounds = (chunks + ROWS_CHUNKS - 1) / ROWS_CHUNKS;

  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(full + 8 * i, 32 * ROWS_PRODUCE);
      mbar_init(empty + 8 * i, mine);
    }
    for (int i = 0; i < ROWS_SUM_RING; ++i) {
      mbar_init(sum_full + 8 * i, mine);
      mbar_init(sum_free + 8 * i, ROWS_FOLD);
    }
    *dead = 0;
    mbar_init_fence();
  }
  __syncthreads();
  after_previous();

  if (warp < ROWS_COMPUTE) {
    const PairSteps<SAT, RNE> steps(p);
    const u64 mul_b = pack2(p.pk_b, p.pk_b);
    // Tasks in turn.  A warp's next round is at most one trip around either ring ahead: a barrier tells two phases apart, not three.
    const int ring = stages < ROWS_SUM_RING ? stages : ROWS_SUM_RING;
    const int workers = ring * mine < ROWS_COMPUTE ? ring * mine : ROWS_COMPUTE;
    int r = warp / mine, pair = warp % mine, stage = r, buf = r;  // (below both rings' sizes)
    uint32_t phase = 0, sum_phase = 0;
    while (warp < workers && r < rounds) {
      mbar_wait(full + 8 * stage, phase, dead);
      mbar_wait(sum_free + 8 * buf, sum_phase ^ 1, dead);
      const unsigned char* const st = smem_raw + stage * (a_bytes + b_bytes);
      const float4* const a = reinterpret_cast<const float4*>(st) + lane;                       // [m][quarter of a chunk][chunk]
      const float* const l1 = reinterpret_cast<const float*>(st + M * (ROWS_CHUNKS * BK * 4)) + lane;  // [m][chunk]
      const uint4* const b = reinterpret_cast<const uint4*>(st + a_bytes) + 2 * pair * ROWS_CHUNKS + lane;
      const bool there = r * ROWS_CHUNKS + lane < chunks;
      u64 w[BK];
      {
        const uint4 x = b[0], y = b[ROWS_CHUNKS];
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // bytes of the two columns in turn, so that each pair decodes into one
          decode4<M4E3>(__byte_perm(xs[q], ys[q], 0x5140), w[4 * q], w[4 * q + 1]);
          decode4<M4E3>(__byte_perm(xs[q], ys[q], 0x7362), w[4 * q + 2], w[4 * q + 3]);
        }
#pragma unroll
        for (int k = 0; k < BK; ++k) w[k] = mul2_rn(w[k], mul_b);
      }
      u64* const out = reinterpret_cast<u64*>(sums + buf * s_bytes) + pair * ROWS_PITCH + lane;
      const int out_pitch = pairs * ROWS_PITCH;
      auto rows = [&](auto count_tag, int m) {
        constexpr int R = decltype(count_tag)::value;
        float av[R][BK];
        bool fast = true;
#pragma unroll
        for (int i = 0; i < R; ++i) {
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 v = a[((m + i) * 4 + q) * ROWS_CHUNKS];
            av[i][4 * q] = v.x;
            av[i][4 * q + 1] = v.y;
            av[i][4 * q + 2] = v.z;
            av[i][4 * q + 3] = v.w;
          }
          fast = fast && l1[(m + i) * ROWS_CHUNKS] < p.clamp_lim;
        }
        u64 acc[R];
#pragma unroll
        for (int i = 0; i < R; ++i) acc[i] = 0ull;
        auto chain = [&](auto clamp_tag) {
          constexpr bool CLAMP = decltype(clamp_tag)::value;
#pragma unroll
          for (int k = 0; k < BK; ++k)
#pragma unroll
            for (int i = 0; i < R; ++i) acc[i] = steps.template step<CLAMP>(pack2(av[i][k], av[i][k]), w[k], acc[i]);
        };
        if (__all_sync(0xFFFFFFFFu, fast || !there)) chain(std::false_type());
        else chain(std::true_type());
#pragma unroll
        for (int i = 0; i < R; ++i) out[(m + i) * out_pitch] = acc[i];
      };
      int m = 0;
#pragma unroll 1
      for (; m + 1 < M; m += 2) rows(std::integral_constant<int, 2>(), m);
      if (m < M) rows(std::integral_constant<int, 1>(), m);
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(empty + 8 * stage);
        mbar_arrive(sum_full + 8 * buf);
      }
      pair += workers;
      while (pair >= mine) {
        pair -= mine;
        ++r;
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
        if (++buf == ROWS_SUM_RING) {
          buf = 0;
          sum_phase ^= 1;
        }
      }
    }
  } else if (warp < ROWS_COMPUTE + ROWS_PRODUCE) {
    const int t = threadIdx.x - 32 * ROWS_COMPUTE;
    const u64 mul_a = pack2(p.pk_a, p.pk_a);
    const float bound = (p.in_m4e3 ? 248.0f : 448.0f) * 1.01f * p.slab_factor;
    const float norm = p.nrm_scale;
    int stage = 0;
    uint32_t phase = 0;
    for (int r = 0; r < rounds; ++r) {
      mbar_wait(empty + 8 * stage, phase ^ 1, dead);
      if (*dead) break;
      unsigned char* const st = smem_raw + stage * (a_bytes + b_bytes);
      const uint32_t bar = full + 8 * stage;
      const int have = chunks - r * ROWS_CHUNKS < ROWS_CHUNKS ? chunks - r * ROWS_CHUNKS : ROWS_CHUNKS;
      if (warp == ROWS_COMPUTE) {
        const int rows = (int)(p.N - n0 < 2 * pairs ? p.N - n0 : 2 * pairs);
        if (lane == 0) mbar_expect(bar, rows * have * BK);
        __syncwarp();
        for (int i = lane; i < rows; i += 32)
          bulk_load(smem_u32(st + a_bytes) + i * (ROWS_CHUNKS * BK),
                    b_base(p, p.B, n0 + i) + b_row(p, n0 + i) * p.K + (int64_t)r * (ROWS_CHUNKS * BK), have * BK, bar);
      }
      for (int i = t; i < M * ROWS_CHUNKS; i += 32 * ROWS_PRODUCE) {
        const int m = i / ROWS_CHUNKS, c = i % ROWS_CHUNKS;
        if (c >= have) continue;
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(p.A + m * p.K + ((int64_t)r * ROWS_CHUNKS + c) * BK));
        const uint32_t w4[4] = {v.x, v.y, v.z, v.w};
        float l1 = 0.0f;
        float4* const dst = reinterpret_cast<float4*>(st) + m * (4 * ROWS_CHUNKS) + c;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          u64 lo, hi;
          decode4<M4E3>(w4[q], lo, hi);
          float4 f;
          unpack2(lo, f.x, f.y);
          unpack2(hi, f.z, f.w);
          l1 += (fabsf(f.x) + fabsf(f.y)) + (fabsf(f.z) + fabsf(f.w));
          unpack2(mul2_rn(lo, mul_a), f.x, f.y);
          unpack2(mul2_rn(hi, mul_a), f.z, f.w);
          dst[q * ROWS_CHUNKS] = f;
        }
        // |S_i| <= sum |a_k| max |b|, as a fraction of 2^(e_max + 1) (see the packed kernel; the scale may be infinite)
        reinterpret_cast<float*>(st + M * (ROWS_CHUNKS * BK * 4))[i] = l1 == 0.0f ? 0.0f : l1 * bound * norm;
      }
      mbar_arrive(bar);
      if (++stage == stages) {
        stage = 0;
        phase ^= 1;
      }
    }
  } else {
    const PairSteps<SAT, RNE> steps(p);
    const int f = threadIdx.x - 32 * (ROWS_COMPUTE + ROWS_PRODUCE);
    const int total = M * mine;  // chains of this CTA
    const bool can_skip = p.nrm_scale < INFINITY;
    u64 T[ROWS_CHAINS];
    int at[ROWS_CHAINS];
#pragma unroll
    for (int i = 0; i < ROWS_CHAINS; ++i) {
      const int c = f + i * 32 * ROWS_FOLD;
      T[i] = 0ull;
      at[i] = c < total ? ((c / mine) * pairs + c % mine) * ROWS_PITCH : -1;
    }
    int buf = 0;
    uint32_t phase = 0;
    for (int r = 0; r < rounds; ++r) {
      mbar_wait(sum_full + 8 * buf, phase, dead);
      const u64* const s = reinterpret_cast<const u64*>(sums + buf * s_bytes);
      const int have = chunks - r * ROWS_CHUNKS < ROWS_CHUNKS ? chunks - r * ROWS_CHUNKS : ROWS_CHUNKS;
#pragma unroll
      for (int i = 0; i < ROWS_CHAINS; ++i) {
        if (at[i] < 0) continue;
        constexpr int G = 8;
#pragma unroll 1
        for (int c = 0; c < have; c += G) {
          u64 v[G];
#pragma unroll
          for (int j = 0; j < G; j += 2) {
            const ulonglong2 q = *reinterpret_cast<const ulonglong2*>(s + at[i] + c + j);
            v[j] = c + j < have ? q.x : 0ull;      // a zero changes no sum
            v[j + 1] = c + j + 1 < have ? q.y : 0ull;
          }
          float lo, hi, bl, bh;
          unpack2(T[i], lo, hi);
          bl = fabsf(lo);
          bh = fabsf(hi);
#pragma unroll
          for (int j = 0; j < G; ++j) {
            unpack2(v[j], lo, hi);
            bl += fabsf(lo);
            bh += fabsf(hi);
          }
          if (can_skip && fmaxf(bl, bh) * p.inv_top * p.slab_factor < p.clamp_lim) {
#pragma unroll
            for (int j = 0; j < G; ++j) T[i] = steps.template fold_as<false>(v[j], T[i]);
          } else {
#pragma unroll
            for (int j = 0; j < G; ++j) T[i] = steps.fold(v[j], T[i]);
          }
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sum_free + 8 * buf);
      if (++buf == ROWS_SUM_RING) {
        buf = 0;
        phase ^= 1;
      }
    }
#pragma unroll
    for (int i = 0; i < ROWS_CHAINS; ++i) {
      const int c = f + i * 32 * ROWS_FOLD;
      if (c >= total) continue;
      float o[2];
      unpack2(T[i], o[0], o[1]);
      if (*dead) o[0] = o[1] = __uint_as_float(0x7FC00000u);
      layer_store_sums<2>(p, c / mine, n0 + 2 * (c % mine), o);
    }
  }
}

cudaError_t launch_rows(int rne, const LinearProblem& p, int pairs, int stages, cudaStream_t stream);

}  // namespace lba
