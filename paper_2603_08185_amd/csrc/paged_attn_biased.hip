// serq_paged_attn_mod's kernels (paged_attn_mod.h): scores less a slope times the distance.
#include "paged_attn_mod.h"

namespace serq {
int launch_paged_attn_biased(const ModLaunch& a, hipStream_t st) { return launch_mod<kBiased>(a, st); }
}  // namespace serq
