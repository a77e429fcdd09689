// Attention over the FP8 cache for the rows of a pass: how a call's work is split, and its launch
// (the kernel: attention8.h).
#include "attention8.h"

namespace specdec {

bool attention8_fits(int rps, int batch, int n_heads, int n_kv_heads) {
  return batch <= kF8MaxBatch && (long)n_kv_heads * tiles_of(rps * (n_heads / n_kv_heads)) <= kF8MaxUnits;
}

int attention8_parts(int rps, int batch, int n_heads, int n_kv_heads, int head_dim, int max_ctx) {
  return plan_of(rps, batch, n_heads, n_kv_heads, head_dim, max_ctx).parts;
}

hipError_t launch_attention8(const AttnArgs& a, hipStream_t s) {
  const int B = a.M / a.rps;
  const Plan p = plan_of(a.rps, B, a.n_heads, a.n_kv_heads, a.head_dim, a.max_ctx);
  if (p.parts > a.n_split || p.n_tiles > kF8TilesPerSlot * a.f8.ring.capacity ||
      !attention8_fits(a.rps, B, a.n_heads, a.n_kv_heads))
    return hipErrorInvalidValue;  // (the callers have checked)
  return launch_plan(a, p, B, Alone{}, s);
}

}  // namespace specdec
