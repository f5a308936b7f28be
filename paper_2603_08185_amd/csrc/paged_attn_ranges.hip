// serq_paged_attn_mod's kernels (paged_attn_mod.h): rows that see a range of keys of their own.
#include "paged_attn_mod.h"

namespace serq {
int launch_paged_attn_ranges(const ModLaunch& a, hipStream_t st) { return launch_mod<kRanges>(a, st); }
}  // namespace serq
