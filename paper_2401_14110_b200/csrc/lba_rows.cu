// Launch of the few-row kernel.
#include "lba_kernel_rows.cuh"

namespace lba {
namespace {

template <bool SAT, int RNE, bool M4E3, bool SCALED>
cudaError_t launch(const RowsProblem& p, cudaStream_t stream) {
  auto kernel = p.M == 1 ? lba_rows_kernel<SAT, RNE, M4E3, SCALED, true> : lba_rows_kernel<SAT, RNE, M4E3, SCALED, false>;
  const size_t smem = rows_smem((int)p.M, p.pairs, p.stages, p.ring);
  // (the same limit in every call: another thread's may lie between this line and the launch)
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, ROWS_ROOM);
  if (e != cudaSuccess) return e;
  const int64_t pairs = (p.N + 1) / 2;
  return launch_after(kernel, dim3((unsigned)((pairs + p.pairs - 1) / p.pairs)), ROWS_THREADS, smem, stream, p);
}
template <bool SAT, int RNE>
cudaError_t by_bytes(const RowsProblem& p, cudaStream_t stream) {
  if (p.in_m4e3) return launch<SAT, RNE, true, false>(p, stream);
  return p.halves != 0x3C003C00u ? launch<SAT, RNE, false, true>(p, stream) : launch<SAT, RNE, false, false>(p, stream);
}
template <int RNE>
cudaError_t by_product(const RowsProblem& p, cudaStream_t stream) {
  return p.pq == PQ_NONE ? by_bytes<false, RNE>(p, stream) : by_bytes<true, RNE>(p, stream);
}

}  // namespace

cudaError_t launch_rows(int rne, const LinearProblem& p, const RowsShape& shape, cudaStream_t stream) {
  RowsProblem q;
  static_cast<LinearProblem&>(q) = p;
  q.pairs = shape.pairs;
  q.stages = shape.stages;
  q.ring = shape.ring;
  // all of the product's scaling but 2^-14 in A: its smallest and largest magnitudes, 2^-9 and 448, must stay normal
  const float all = p.pk_a * 16384.0f * p.pk_b;
  const bool scaled = !p.in_m4e3 && all * 0x1p-9f >= 0x1p-126f && all <= 0x1p118f;
  q.halves = scaled ? 0x04000400u : 0x3C003C00u;
  q.scale_a = scaled ? all : p.pk_a;
  q.scale_b = scaled ? 1.0f : p.pk_b;
  const EncodeTiled encode = tensor_map_encoder();
  if (!encode) return cudaErrorNotSupported;
  for (int i = 0; i <= p.gated; ++i) {
    const cuuint64_t dims[2] = {(cuuint64_t)p.K / 8, (cuuint64_t)p.n}, stride = (cuuint64_t)p.K;
    const cuuint32_t box[2] = {ROWS_CHUNKS * BK / 8, (cuuint32_t)(p.gated ? q.pairs : 2 * q.pairs)}, step[2] = {1, 1};
    if (encode(&q.b[i], CU_TENSOR_MAP_DATA_TYPE_UINT64, 2, const_cast<uint8_t*>(i ? p.B2 : p.B), dims, &stride, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
               CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  }
  return rne == 0 ? by_product<0>(q, stream) : rne == 1 ? by_product<1>(q, stream) : by_product<2>(q, stream);
}

}  // namespace lba
