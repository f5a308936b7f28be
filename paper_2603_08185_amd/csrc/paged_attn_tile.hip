// serq_paged_attn's kernel for sequences with many rows (paged_attn_tile.h) and its launch.
#include "paged_attn_tile.h"

namespace serq {
namespace {

template <int DT, bool F8, int D>
__global__ __launch_bounds__(256, 2) void paged_attn_tile_kernel(AttnParams p) {
  __shared__ __align__(16) char lds[tile::kLds<D>];
  tile::work<DT, F8, D>(p, blockIdx.x, lds);
}

template <int DT, bool F8, int D>
int launch(const AttnParams& p, int blocks, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_tile_kernel<DT, F8, D>), dim3((unsigned)(blocks * p.slices * p.c.heads)), dim3(256), 0, st, p);
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

}  // namespace

size_t paged_attn_tile_slot_floats(int D) { return (size_t)kTileRows * (D + 2); }

int launch_paged_attn_tile(const AttnParams& p, int dtype, bool f8, int D, int blocks, hipStream_t st) {
  const bool bf = dtype == SERQ_BF16;
  if (D == 128) {
    if (bf) return f8 ? launch<SERQ_BF16, true, 128>(p, blocks, st) : launch<SERQ_BF16, false, 128>(p, blocks, st);
    return f8 ? launch<SERQ_F16, true, 128>(p, blocks, st) : launch<SERQ_F16, false, 128>(p, blocks, st);
  }
  if (bf) return f8 ? launch<SERQ_BF16, true, 64>(p, blocks, st) : launch<SERQ_BF16, false, 64>(p, blocks, st);
  return f8 ? launch<SERQ_F16, true, 64>(p, blocks, st) : launch<SERQ_F16, false, 64>(p, blocks, st);
}

}  // namespace serq
