// Layers on few rows (a token, or the tokens of a few sequences that decode together), in chunks of 16.
//
// With one row every byte of the weights is read once and used once: the layer takes as long as its weights take to arrive (4096 x
// 4096: 16.8 MB, 2.6 us at the copy rate), if decoding and the chains keep up.  Tiles cannot: a 16x16 tile spends sixteen rows of work on one.
// Here a lane takes one chunk of one pair of columns (the two halves of a packed instruction) and walks its sixteen steps for
// every row, so nothing is computed that no output needs, a warp's lanes read 512 consecutive bytes of a row of weights, and
// the chunk sums of a column, which do not depend on each other, spread over the lanes.  What stays sequential is the second
// hierarchy, T <- Q_acc(C_j + T) in chunk order: one addition in sixteen, done by warps of their own a round behind.
//
//   rounds of 32 chunks (512 k).  Producer warps bring the round's weights into a ring of stages (one tensor copy per operand; a bulk
//   copy per row had cost 85 clocks of issue each, 2400 a round) and decode its activations into the same stage; compute warps take (round, pair) tasks in turn and leave the chunk sums in a second ring;
//   fold warps keep T of every (row, pair) in registers.  Barriers count tasks, so no warp waits for a whole round.
// A CTA owns as many pairs as fit, so that one wave of CTAs covers the columns where it can: the fold of a CTA's last round and the
// first load of the next would otherwise show.
// Steps and folds are those of the packed kernel, bit for bit; a chunk runs without the clamp of Eq. 2 where sum |a_k| max |b|
// shows that it cannot act.
#pragma once
#include <cuda.h>

#include "lba_async.cuh"
#include "lba_kernel_small.cuh"

namespace lba {

constexpr int ROWS_MAX = 16;                 // rows at most
constexpr int ROWS_CHUNKS = 32;              // chunks of a round: one per lane
constexpr int ROWS_FOLD = 4, ROWS_DECODE = 3, ROWS_COMPUTE = 12;  // warps, in this order, and one that issues the copies
constexpr int ROWS_COPY_WARP = ROWS_FOLD + ROWS_DECODE, ROWS_FIRST_COMPUTE = ROWS_COPY_WARP + 1;
constexpr int ROWS_WARPS = ROWS_FIRST_COMPUTE + ROWS_COMPUTE, ROWS_THREADS = 32 * ROWS_WARPS;
constexpr int ROWS_MIN_STAGES = 3;           // at least as many as warps that take rounds in turn
constexpr int ROWS_CHAINS = 4;               // (row, column) chains per lane of a fold warp, at most (one where there is one row)
constexpr int ROWS_SUM_RING = 3;             // rounds of sums kept; two where a third would cost a wave of CTAs
constexpr int ROWS_MAX_STAGES = 8;
constexpr int ROWS_ROOM = 227 * 1024;        // bytes of shared memory
constexpr int ROWS_PITCH = ROWS_CHUNKS + 4;  // sums from one chain to the next: 16-byte aligned, lanes on different banks

struct RowsProblem : LinearProblem {
  CUtensorMap b[2];   // the operands as [N][K / 8] 64-bit words, boxes of a round's 64 words of a CTA's rows
  int pairs, stages, ring;  // pairs of columns of a CTA, rounds of operands and of sums that it holds
  // Scales of the operands.  E4M3 bytes are widened by an FMA whose other factor is a half: 2^-14 there leaves B's scaling to A and
  // saves its multiplication, where A then stays normal (`halves` is 1.0 twice, and both scales the usual ones, where it does not).
  uint32_t halves;
  float scale_a, scale_b;
};
inline __host__ __device__ int rows_a_bytes(int M) { return M * (ROWS_CHUNKS * BK * 4 + ROWS_CHUNKS * 4); }
inline __host__ __device__ int rows_b_bytes(int pairs) { return 2 * pairs * ROWS_CHUNKS * BK; }
inline __host__ __device__ int rows_sum_bytes(int M, int pairs) { return M * 2 * pairs * ROWS_PITCH * 4; }
inline __host__ __device__ int rows_smem(int M, int pairs, int stages, int ring) {
  return stages * (rows_a_bytes(M) + rows_b_bytes(pairs)) + ring * rows_sum_bytes(M, pairs) + 8 * 2 * (ROWS_MAX_STAGES + ROWS_SUM_RING) + 16;
}

// T <- Q_acc(C + T) of one output
template <int RNE>
struct FoldStep {
  uint32_t mask;
  float sat, k1, k2;
  __device__ __forceinline__ explicit FoldStep(const Problem& p) : mask(p.qa.mask), sat(p.qa.sat), k1(p.acc_k1), k2(p.acc_k2) {}
  __device__ __forceinline__ float operator()(float c, float t) const {
    float v;
    if (RNE == 0) {
      asm("add.rz.ftz.f32 %0, %1, %2;" : "=f"(v) : "f"(c), "f"(t));
      v = and_bits(v, mask);
    } else {
      asm("add.rn.ftz.f32 %0, %1, %2;" : "=f"(v) : "f"(c), "f"(t));
      v = RNE == 1 ? __fmaf_rn(v, k2, __fmul_rn(v, k1)) : __bfloat162float(__float2bfloat16_rn(v));
    }
    return clamp_mag(v, sat);
  }
};

// SCALED: B's scaling is in `halves`.  ONE: a single row; a task is then two pairs, so that two chains run beside each other as they
// do for two rows (a step waits 12.5 clocks for the one before it and issues four instructions).
template <bool SAT, int RNE, bool M4E3, bool SCALED, bool ONE>
__global__ void __launch_bounds__(ROWS_THREADS, 1) lba_rows_kernel(const __grid_constant__ RowsProblem p) {
  extern __shared__ __align__(128) unsigned char rows_raw[];
  unsigned char* const smem_raw = rows_raw;
  const int M = ONE ? 1 : (int)p.M, pairs = p.pairs, stages = p.stages;
  const int a_bytes = rows_a_bytes(M), b_bytes = rows_b_bytes(pairs), s_bytes = rows_sum_bytes(M, pairs);
  unsigned char* const sums = smem_raw + stages * (a_bytes + b_bytes);
  uint64_t* const bars = reinterpret_cast<uint64_t*>(sums + p.ring * s_bytes);
  volatile int* const dead = reinterpret_cast<volatile int*>(bars + 2 * (ROWS_MAX_STAGES + ROWS_SUM_RING));
  const uint32_t full = smem_u32(bars), empty = full + 8 * ROWS_MAX_STAGES, sum_full = empty + 8 * ROWS_MAX_STAGES,
                 sum_free = sum_full + 8 * ROWS_SUM_RING;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t n0 = (int64_t)blockIdx.x * (2 * pairs);
  const int mine = (int)((p.N - n0 + 1) / 2 < pairs ? (p.N - n0 + 1) / 2 : pairs);  // pairs of this CTA
  // Tasks of a round: two pairs, or a pair and some of the rows where pairs alone would leave compute warps without one
  const int groups = ONE || mine >= ROWS_COMPUTE || M < 4 ? 1 : (ROWS_COMPUTE + mine - 1) / mine < M / 2 ? (ROWS_COMPUTE + mine - 1) / mine : M / 2;
  const int group_rows = ((M + groups - 1) / groups + 1) & ~1;  // even: two rows run beside each other
  const int tasks = ONE ? (mine + 1) / 2 : mine * ((M + group_rows - 1) / group_rows);
  const bool by_rows = M >= ROWS_DECODE;  // the decoding warps share a round, or take rounds in turn
  const int fold_warps = (M * 2 * mine + 31) / 32 < ROWS_FOLD ? (M * 2 * mine + 31) / 32 : ROWS_FOLD;
  const int chunks = (int)(p.K / BK), rounds = (chunks + ROWS_CHUNKS - 1) / ROWS_CHUNKS;

  if (threadIdx.x == 0) {
    for (int i = 0; i < stages; ++i) {
      mbar_init(full + 8 * i, 1 + (by_rows ? ROWS_DECODE : 1));
      mbar_init(empty + 8 * i, tasks);
    }
    for (int i = 0; i < p.ring; ++i) {
      mbar_init(sum_full + 8 * i, tasks);
      mbar_init(sum_free + 8 * i, fold_warps);
    }
    *dead = 0;
    mbar_init_fence();
  }
  __syncthreads();
  after_previous();

  // chunk `c` of a row, if there is one, to its place in a stage
  auto fetch = [&](int m, int c) {
    return __ldg(reinterpret_cast<const uint4*>(p.A + m * p.K) + (c < chunks ? c : 0));
  };
  auto decode = [&](const uint4& raw, unsigned char* st, int m) {
    const u64 mul_a = pack2(p.scale_a, p.scale_a);
    const uint32_t w4[4] = {raw.x, raw.y, raw.z, raw.w};
    float l1 = 0.0f;
    float4* const dst = reinterpret_cast<float4*>(st) + m * (4 * ROWS_CHUNKS) + lane;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      u64 lo, hi;
      decode4<M4E3>(w4[e], lo, hi);
      float4 f;
      unpack2(lo, f.x, f.y);
      unpack2(hi, f.z, f.w);
      l1 += (fabsf(f.x) + fabsf(f.y)) + (fabsf(f.z) + fabsf(f.w));
      unpack2(mul2_rn(lo, mul_a), f.x, f.y);
      unpack2(mul2_rn(hi, mul_a), f.z, f.w);
      dst[e * ROWS_CHUNKS] = f;
    }
    // |S_i| <= sum |a_k| max |b|, as a fraction of 2^(e_max + 1) (see the packed kernel; the scale may be infinite)
    const float bound = (M4E3 ? 248.0f : 448.0f) * 1.01f * p.slab_factor;
    reinterpret_cast<float*>(st + M * (ROWS_CHUNKS * BK * 4))[m * ROWS_CHUNKS + lane] = l1 == 0.0f ? 0.0f : l1 * bound * p.nrm_scale;
  };
  // the weights of round r; what lies behind the last row or the last k arrives as zeros
  auto copy = [&](int r, int stage) {
    const uint32_t dst = smem_u32(smem_raw + stage * (a_bytes + b_bytes) + a_bytes), bar = full + 8 * stage;
    mbar_arrive_expect(bar, b_bytes);
    if (p.gated) {
      tensor_load(dst, &p.b[0], r * 64, (int)(n0 >> 1), bar);
      tensor_load(dst + b_bytes / 2, &p.b[1], r * 64, (int)(n0 >> 1), bar);
    } else {
      tensor_load(dst, &p.b[0], r * 64, (int)n0, bar);
    }
  };

  // every warp helps with the first round's activations, for which there is nothing else to do yet
  if (warp == ROWS_COPY_WARP && elected()) copy(0, 0);
  __syncwarp();
  for (int m = warp; m < M; m += ROWS_WARPS) decode(fetch(m, lane), smem_raw, m);
  __syncthreads();

  if (warp >= ROWS_FIRST_COMPUTE) {
    const PairSteps<SAT, RNE> steps(p);
    const u64 mul_b = pack2(p.scale_b, p.scale_b);
    const uint32_t halves = p.halves;
    // Tasks in turn.  A warp's next round is at most one trip around either ring ahead: a barrier tells two phases apart, not three.
    const int ring = stages < p.ring ? stages : p.ring;
    const int workers = ring * tasks < ROWS_COMPUTE ? ring * tasks : ROWS_COMPUTE;
    const int me = warp - ROWS_FIRST_COMPUTE;
    int r = me / tasks, task = me % tasks, stage = r, buf = r;  // (below both rings' sizes)
    uint32_t phase = 0, sum_phase = 0;
    while (me < workers && r < rounds) {
      mbar_wait(full + 8 * stage, phase, dead);
      mbar_wait(sum_free + 8 * buf, sum_phase ^ 1, dead);
      const unsigned char* const st = smem_raw + stage * (a_bytes + b_bytes);
      const float4* const a = reinterpret_cast<const float4*>(st) + lane;                       // [m][quarter of a chunk][chunk]
      const float* const l1 = reinterpret_cast<const float*>(st + M * (ROWS_CHUNKS * BK * 4)) + lane;  // [m][chunk]
      const uint4* const b = reinterpret_cast<const uint4*>(st + a_bytes) + lane;
      float* const out = reinterpret_cast<float*>(sums + buf * s_bytes) + lane;                 // [m][column][chunk]
      const int out_pitch = 2 * pairs * ROWS_PITCH;
      const bool there = r * ROWS_CHUNKS + lane < chunks;
      // a pair's two columns: rows next to each other, or the same row of both operands
      auto weights = [&](int pair, u64 (&w)[BK]) {
        const uint4 x = b[(p.gated ? pair : 2 * pair) * ROWS_CHUNKS], y = b[(p.gated ? pairs + pair : 2 * pair + 1) * ROWS_CHUNKS];
        const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int q = 0; q < 4; ++q) {  // bytes of the two columns in turn, so that each pair decodes into one
          decode4<M4E3>(__byte_perm(xs[q], ys[q], 0x5140), w[4 * q], w[4 * q + 1], halves);
          decode4<M4E3>(__byte_perm(xs[q], ys[q], 0x7362), w[4 * q + 2], w[4 * q + 3], halves);
        }
        if (!SCALED) {
#pragma unroll
          for (int k = 0; k < BK; ++k) w[k] = mul2_rn(w[k], mul_b);
        }
      };
      auto load_row = [&](int m, float (&v)[BK]) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float4 f = a[(m * 4 + q) * ROWS_CHUNKS];
          v[4 * q] = f.x;
          v[4 * q + 1] = f.y;
          v[4 * q + 2] = f.z;
          v[4 * q + 3] = f.w;
        }
      };
      auto store = [&](int m, int pair, u64 acc) {
        float* const dst = out + m * out_pitch + 2 * pair * ROWS_PITCH;
        unpack2(acc, dst[0], dst[ROWS_PITCH]);
      };
      if constexpr (ONE) {
        const int p0 = 2 * task, p1 = 2 * task + 1 < mine ? 2 * task + 1 : p0;
        u64 w[2][BK], acc[2] = {0ull, 0ull};
        float v[BK];
        weights(p0, w[0]);
        weights(p1, w[1]);
        load_row(0, v);
        auto chain = [&](auto clamp_tag) {
          constexpr bool CLAMP = decltype(clamp_tag)::value;
#pragma unroll
          for (int k = 0; k < BK; ++k)
#pragma unroll
            for (int i = 0; i < 2; ++i) acc[i] = steps.template step<CLAMP>(pack2(v[k], v[k]), w[i][k], acc[i]);
        };
        if (__all_sync(0xFFFFFFFFu, l1[0] < p.clamp_lim || !there)) chain(std::false_type());
        else chain(std::true_type());
        store(0, p0, acc[0]);
        store(0, p1, acc[1]);
      } else {
        const int pair = task % mine, m0 = task / mine * group_rows, m1 = m0 + group_rows < M ? m0 + group_rows : M;
        u64 w[BK];
        weights(pair, w);
        auto rows = [&](auto count_tag, int m) {
          constexpr int R = decltype(count_tag)::value;
          float v[R][BK];
          u64 acc[R];
          bool fast = true;
#pragma unroll
          for (int i = 0; i < R; ++i) {
            load_row(m + i, v[i]);
            acc[i] = 0ull;
            fast = fast && l1[(m + i) * ROWS_CHUNKS] < p.clamp_lim;
          }
          auto chain = [&](auto clamp_tag) {
            constexpr bool CLAMP = decltype(clamp_tag)::value;
#pragma unroll
            for (int k = 0; k < BK; ++k)
#pragma unroll
              for (int i = 0; i < R; ++i) acc[i] = steps.template step<CLAMP>(pack2(v[i][k], v[i][k]), w[k], acc[i]);
          };
          if (__all_sync(0xFFFFFFFFu, fast || !there)) chain(std::false_type());
          else chain(std::true_type());
#pragma unroll
          for (int i = 0; i < R; ++i) store(m + i, pair, acc[i]);
        };
        int m = m0;
#pragma unroll 1
        for (; m + 1 < m1; m += 2) rows(std::integral_constant<int, 2>(), m);
        if (m < m1) rows(std::integral_constant<int, 1>(), m);
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(empty + 8 * stage);
        mbar_arrive(sum_full + 8 * buf);
      }
      task += workers;
      while (task >= tasks) {
        task -= tasks;
        ++r;
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
        if (++buf == p.ring) {
          buf = 0;
          sum_phase ^= 1;
        }
      }
    }
  } else if (warp == ROWS_COPY_WARP) {
    if (elected()) {
      int stage = 1;
      uint32_t phase = 0;
      for (int r = 1; r < rounds; ++r) {
        mbar_wait(empty + 8 * stage, phase ^ 1, dead);
        if (*dead) break;  // (the others' waits end for it)
        copy(r, stage);
        if (++stage == stages) {
          stage = 0;
          phase ^= 1;
        }
      }
    }
  } else if (warp >= ROWS_FOLD) {
    // the other rounds' activations, fetched two rows ahead
    const int d = warp - ROWS_FOLD, step_r = by_rows ? 1 : ROWS_DECODE, m_first = by_rows ? d : 0, m_step = by_rows ? ROWS_DECODE : 1;
    if (lane == 0 && (by_rows || d == 0)) mbar_arrive(full);  // the first round's are there
    int r = by_rows || d == 0 ? step_r : d, stage = r;
    uint32_t phase = 0;
    for (; r < rounds; r += step_r) {
      if (stage >= stages) {
        stage -= stages;
        phase ^= 1;
      }
      const int c = r * ROWS_CHUNKS + lane;
      uint4 next = fetch(m_first, c), after = fetch(m_first + m_step < M ? m_first + m_step : m_first, c);
      mbar_wait(empty + 8 * stage, phase ^ 1, dead);
      unsigned char* const st = smem_raw + stage * (a_bytes + b_bytes);
#pragma unroll 1
      for (int m = m_first; m < M; m += m_step) {
        const uint4 now = next;
        next = after;
        if (m + 2 * m_step < M) after = fetch(m + 2 * m_step, c);
        decode(now, st, m);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(full + 8 * stage);
      stage += step_r;
    }
  } else if (warp < fold_warps) {
    constexpr int CHAINS = ONE ? 1 : ROWS_CHAINS;
    const FoldStep<RNE> step(p);
    const int f = threadIdx.x, columns = 2 * mine;
    const int total = M * columns;  // chains of this CTA
    float T[CHAINS];
#pragma unroll
    for (int i = 0; i < CHAINS; ++i) T[i] = 0.0f;
    int buf = 0;
    uint32_t phase = 0;
    for (int r = 0; r < rounds; ++r) {
      mbar_wait(sum_full + 8 * buf, phase, dead);
      const int have = chunks - r * ROWS_CHUNKS < ROWS_CHUNKS ? chunks - r * ROWS_CHUNKS : ROWS_CHUNKS;
#pragma unroll
      for (int i = 0; i < CHAINS; ++i) {
        const int c = f + i * 32 * ROWS_FOLD;
        if (c >= total) break;
        const float* const s = reinterpret_cast<const float*>(sums + buf * s_bytes) + ((c / columns) * 2 * pairs + c % columns) * ROWS_PITCH;
        if (have == ROWS_CHUNKS) {
#pragma unroll
          for (int j = 0; j < ROWS_CHUNKS; j += 4) {
            const float4 v = *reinterpret_cast<const float4*>(s + j);
            T[i] = step(v.w, step(v.z, step(v.y, step(v.x, T[i]))));
          }
        } else {
#pragma unroll 1
          for (int j = 0; j < have; ++j) T[i] = step(s[j], T[i]);
        }
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(sum_free + 8 * buf);
      if (++buf == p.ring) {
        buf = 0;
        phase ^= 1;
      }
    }
    // a column's neighbour in its pair sits in the next lane
#pragma unroll
    for (int i = 0; i < CHAINS; ++i) {
      const int c = f + i * 32 * ROWS_FOLD;
      float o[2] = {T[i], __shfl_down_sync(0xFFFFFFFFu, T[i], 1)};
      if (c >= total || (c & 1)) continue;
      if (*dead) o[0] = o[1] = __uint_as_float(0x7FC00000u);
      layer_store_sums<2>(p, c / columns, n0 + c % columns, o);
    }
  }
  if (*dead) let_copies_land();  // (a warp whose wait ran out sees it, and it was that warp's to wait for a copy)
}

struct RowsShape { int pairs, stages, ring; };  // no stages: the kernel does not apply
cudaError_t launch_rows(int rne, const LinearProblem& p, const RowsShape& shape, cudaStream_t stream);

}  // namespace lba
