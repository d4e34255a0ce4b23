// Launch of the bf16 attention over a context cache that is read in part (a
// window and its first keys) or held in 4 bits: the kernel of attn_bf16.h with
// those reads compiled in.
#include "attn_bf16.h"

namespace glance {
namespace {

template <int D, bool TREE>
void launch(const AttnParams& p, bool kv4, hipStream_t s) {
  const dim3 grid(grid_blocks(p)), block(512);
  const bool wide = p.tiles_rg > 4;
  if (kv4 && wide) hipLaunchKernelGGL((attn_bf16<D, TREE, true, true, true>), grid, block, 0, s, p);
  else if (kv4) hipLaunchKernelGGL((attn_bf16<D, TREE, false, true, true>), grid, block, 0, s, p);
  else if (wide) hipLaunchKernelGGL((attn_bf16<D, TREE, true, false, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((attn_bf16<D, TREE, false, false, true>), grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_attn_cache_bf16(const AttnParams& p, bool kv4, bool tree, hipStream_t s, hipEvent_t ev0,
                                  hipEvent_t ev1) {
  // A dense cache without a window is the plain call's case and runs its kernel, so
  // that both entry points give the same bits.  (The plan is the same.  The windowed
  // kernel moves a row's reference at other scores; of the same inputs, 28/4 heads
  // of 128, it took for 64 rows over 4 x 16384 keys 78.4 us against 75.5, over 16
  // ragged contexts 315 against 297; for 16 rows over 4 x 16384 keys 36.3 against
  // 39.9; for 1 and 16 rows over the ragged contexts the same.)
  if (!kv4 && p.window == kNoWindow) return launch_attn_bf16(p, tree, s, ev0, ev1);
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.d == 128) {
    if (tree) launch<128, true>(p, kv4, s);
    else launch<128, false>(p, kv4, s);
  } else {
    if (tree) launch<64, true>(p, kv4, s);
    else launch<64, false>(p, kv4, s);
  }
  const hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
