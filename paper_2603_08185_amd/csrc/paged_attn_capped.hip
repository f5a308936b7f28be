// serq_paged_attn_mod's kernels (paged_attn_mod.h): scores capped by a tanh.
#include "paged_attn_mod.h"

namespace serq {
int launch_paged_attn_capped(const ModLaunch& a, hipStream_t st) { return launch_mod<kCapped>(a, st); }
}  // namespace serq
