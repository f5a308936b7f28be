// serq_paged_attn for batches that hold both chunks and single tokens: one launch in which some workgroups do the work of paged_attn_tile.h, bound by the
// matrix instructions, and the others, beside them on the same compute units, that of paged_attn_few.h, bound by memory.  The first take
// longest and start first.
// Measured (us, one launch after the other / together): a chunk of 384 after 3500 beside 7 single tokens, E4M3 cache, 67.6 / 53.8; 512 after up to 4000
// beside 30 single tokens 108 / 86; 2000 after 4000 beside 6 170 / 157.
#include "paged_attn_few.h"
#include "paged_attn_tile.h"

namespace serq {
namespace {

template <int DT, bool F8, int D>
__global__ __launch_bounds__(256, 2) void paged_attn_mixed_kernel(AttnParams many, AttnParams few, int tiles) {
  constexpr int LDS = tile::kLds<D> > few::kLds<F8, D, 1> ? tile::kLds<D> : few::kLds<F8, D, 1>;
  __shared__ __align__(16) char lds[LDS];
  if ((int)blockIdx.x < tiles) tile::work<DT, F8, D>(many, blockIdx.x, lds);
  else few::work<DT, F8, D, 1>(few, blockIdx.x - tiles, gridDim.x - tiles, lds);
}

template <int DT, bool F8, int D>
int launch(const AttnParams& many, const AttnParams& few, int tiles, int shares, hipStream_t st) {
  hipLaunchKernelGGL((paged_attn_mixed_kernel<DT, F8, D>), dim3((unsigned)(tiles + shares)), dim3(256), 0, st, many, few, tiles);
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

}  // namespace

int launch_paged_attn_mixed(const AttnParams& many, const AttnParams& few, int dtype, bool f8, int D, int blocks, int shares, hipStream_t st) {
  const bool bf = dtype == SERQ_BF16;
  const int tiles = blocks * many.slices * many.c.heads;
  if (D == 128) {
    if (bf) return f8 ? launch<SERQ_BF16, true, 128>(many, few, tiles, shares, st) : launch<SERQ_BF16, false, 128>(many, few, tiles, shares, st);
    return f8 ? launch<SERQ_F16, true, 128>(many, few, tiles, shares, st) : launch<SERQ_F16, false, 128>(many, few, tiles, shares, st);
  }
  if (bf) return f8 ? launch<SERQ_BF16, true, 64>(many, few, tiles, shares, st) : launch<SERQ_BF16, false, 64>(many, few, tiles, shares, st);
  return f8 ? launch<SERQ_F16, true, 64>(many, few, tiles, shares, st) : launch<SERQ_F16, false, 64>(many, few, tiles, shares, st);
}

}  // namespace serq
