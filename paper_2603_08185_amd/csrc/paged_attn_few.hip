// serq_paged_attn's kernel for sequences with few rows (paged_attn_few.h) and its launch.
#include "paged_attn_few.h"

namespace serq {
namespace {

template <int DT, bool F8, int D, int NB>
__global__ __launch_bounds__(256, 2) void paged_attn_few_kernel(AttnParams p) {
  __shared__ __align__(16) char lds[few::kLds<F8, D, NB>];
  few::work<DT, F8, D, NB>(p, blockIdx.x, gridDim.x, lds);
}

template <int DT, bool F8, int D>
int launch(const AttnParams& p, int nb, int workgroups, hipStream_t st) {
  const dim3 grid((unsigned)workgroups);
  if (nb == 1) hipLaunchKernelGGL((paged_attn_few_kernel<DT, F8, D, 1>), grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL((paged_attn_few_kernel<DT, F8, D, 2>), grid, dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

}  // namespace

size_t paged_attn_few_slot_floats(int nb, int D) { return (size_t)16 * nb * (D + 2); }
int paged_attn_few_resident(int nb, bool f8, int D) { return D == 64 && f8 && nb == 1 ? 3 : 2; }

int launch_paged_attn_few(const AttnParams& p, int dtype, bool f8, int D, int nb, int workgroups, hipStream_t st) {
  const bool bf = dtype == SERQ_BF16;
  if (D == 128) {
    if (bf) return f8 ? launch<SERQ_BF16, true, 128>(p, nb, workgroups, st) : launch<SERQ_BF16, false, 128>(p, nb, workgroups, st);
    return f8 ? launch<SERQ_F16, true, 128>(p, nb, workgroups, st) : launch<SERQ_F16, false, 128>(p, nb, workgroups, st);
  }
  if (bf) return f8 ? launch<SERQ_BF16, true, 64>(p, nb, workgroups, st) : launch<SERQ_BF16, false, 64>(p, nb, workgroups, st);
  return f8 ? launch<SERQ_F16, true, 64>(p, nb, workgroups, st) : launch<SERQ_F16, false, 64>(p, nb, workgroups, st);
}

}  // namespace serq
