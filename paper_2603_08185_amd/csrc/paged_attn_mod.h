// The kernels of serq_paged_attn_mod: those of serq_paged_attn with what stands between the scores and the softmax (Mod), each compiled in a
// source of its own (paged_attn_ranges.hip, paged_attn_capped.hip, paged_attn_biased.hip), and a call's launch.
//
// Few rows are bound by memory with or without them: 40 tokens over up to 8000 keys 85 us plain, 88 capped; one over 65000, 16 heads of 64 channels, 51 plain, 52
// with a bias.  Many rows, 32 query and 8 key heads of 128 channels, a prompt of 8192 tokens: plain 484, with a bias 548 (two instructions a score before the products),
// capped 603 (four a score, two of them an exponential and a reciprocal, between the products with V; E4M3 636, 64 channels 436); with a prefix
// of 5531 of them seen both ways 710 for 1.46 times the work.  12000 tokens of packed documents, 8.5 tiles a row block: 158 to 166, of which row blocks without
// a key (their beginnings and ends, q read and the result stored) take 47.
#pragma once

#include "paged_attn_few.h"
#include "paged_attn_tile.h"

namespace serq {
namespace {

template <int DT, bool F8, int D, int NB, int MOD>
__global__ __launch_bounds__(256, 2) void paged_attn_mod_few_kernel(AttnModParams p) {
  __shared__ __align__(16) char lds[few::kLds<F8, D, NB>];
  few::work<DT, F8, D, NB, MOD>(p, blockIdx.x, gridDim.x, lds);
}

template <int DT, bool F8, int D, int MOD>
__global__ __launch_bounds__(256, 2) void paged_attn_mod_tile_kernel(AttnModParams p) {
  __shared__ __align__(16) char lds[tile::kLds<D>];
  tile::work<DT, F8, D, MOD>(p, blockIdx.x, lds);
}

template <int DT, bool F8, int D, int MOD>
__global__ __launch_bounds__(256, 2) void paged_attn_mod_mixed_kernel(AttnModParams many, AttnModParams few, int tiles) {
  constexpr int LDS = tile::kLds<D> > few::kLds<F8, D, 1> ? tile::kLds<D> : few::kLds<F8, D, 1>;
  __shared__ __align__(16) char lds[LDS];
  if ((int)blockIdx.x < tiles) tile::work<DT, F8, D, MOD>(many, blockIdx.x, lds);
  else few::work<DT, F8, D, 1, MOD>(few, blockIdx.x - tiles, gridDim.x - tiles, lds);
}

template <int DT, int MOD>
__global__ __launch_bounds__(256, 2) void paged_attn_mod_few_pairs_kernel(AttnModParams p, PairPlan n) {
  __shared__ __align__(16) char lds[few::kLds<false, 128, 1>];
  few::work_pairs<DT, MOD>(p, n, blockIdx.x, lds);
}

template <int MOD, int DT, bool F8, int D>
int launch_mod_of(const ModLaunch& a, hipStream_t st) {
  const int tiles = a.many ? a.blocks * a.many->slices * a.many->c.heads : 0;
  if (a.many && a.few && a.nb == 1) {
    hipLaunchKernelGGL((paged_attn_mod_mixed_kernel<DT, F8, D, MOD>), dim3((unsigned)(tiles + a.shares)), dim3(256), 0, st, *a.many, *a.few, tiles);
  } else {
    if (a.many) hipLaunchKernelGGL((paged_attn_mod_tile_kernel<DT, F8, D, MOD>), dim3((unsigned)tiles), dim3(256), 0, st, *a.many);
    if (a.few && a.nb == 1) hipLaunchKernelGGL((paged_attn_mod_few_kernel<DT, F8, D, 1, MOD>), dim3((unsigned)a.shares), dim3(256), 0, st, *a.few);
    else if (a.few) hipLaunchKernelGGL((paged_attn_mod_few_kernel<DT, F8, D, 2, MOD>), dim3((unsigned)a.shares), dim3(256), 0, st, *a.few);
  }
  return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
}

template <int MOD>
int launch_mod(const ModLaunch& a, hipStream_t st) {
  const bool bf = a.dtype == SERQ_BF16;
  if (a.pairs.two) {
    const dim3 grid((unsigned)(a.pairs.one > a.pairs.two ? a.pairs.one : a.pairs.two));
    if (bf) hipLaunchKernelGGL((paged_attn_mod_few_pairs_kernel<SERQ_BF16, MOD>), grid, dim3(256), 0, st, *a.few, a.pairs);
    else hipLaunchKernelGGL((paged_attn_mod_few_pairs_kernel<SERQ_F16, MOD>), grid, dim3(256), 0, st, *a.few, a.pairs);
    return hipGetLastError() == hipSuccess ? SERQ_OK : SERQ_EHIP;
  }
  if (a.D == 128) {
    if (bf) return a.f8 ? launch_mod_of<MOD, SERQ_BF16, true, 128>(a, st) : launch_mod_of<MOD, SERQ_BF16, false, 128>(a, st);
    return a.f8 ? launch_mod_of<MOD, SERQ_F16, true, 128>(a, st) : launch_mod_of<MOD, SERQ_F16, false, 128>(a, st);
  }
  if (bf) return a.f8 ? launch_mod_of<MOD, SERQ_BF16, true, 64>(a, st) : launch_mod_of<MOD, SERQ_BF16, false, 64>(a, st);
  return a.f8 ? launch_mod_of<MOD, SERQ_F16, true, 64>(a, st) : launch_mod_of<MOD, SERQ_F16, false, 64>(a, st);
}

}  // namespace
}  // namespace serq
