// Launch of the few-row kernel.
#include "lba_kernel_rows.cuh"

namespace lba {
namespace {

template <bool SAT, int RNE, bool M4E3>
cudaError_t launch(const RowsProblem& p, cudaStream_t stream) {
  auto kernel = lba_rows_kernel<SAT, RNE, M4E3>;
  const size_t smem = rows_smem((int)p.M, p.pairs, p.stages);
  const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return e;
  const int64_t pairs = (p.N + 1) / 2;
  return launch_after(kernel, dim3((unsigned)((pairs + p.pairs - 1) / p.pairs)), ROWS_THREADS, smem, stream, p);
}
template <bool SAT, int RNE>
cudaError_t by_bytes(const RowsProblem& p, cudaStream_t stream) {
  return p.in_m4e3 ? launch<SAT, RNE, true>(p, stream) : launch<SAT, RNE, false>(p, stream);
}
template <int RNE>
cudaError_t by_product(const RowsProblem& p, cudaStream_t stream) {
  return p.pq == PQ_NONE ? by_bytes<false, RNE>(p, stream) : by_bytes<true, RNE>(p, stream);
}

}  // namespace

cudaError_t launch_rows(int rne, const LinearProblem& p, int pairs, int stages, cudaStream_t stream) {
  RowsProblem q;
  static_cast<LinearProblem&>(q) = p;
  q.pairs = pairs;
  q.stages = stages;
  return rne == 0 ? by_product<0>(q, stream) : rne == 1 ? by_product<1>(q, stream) : by_product<2>(q, stream);
}

}  // namespace lba
