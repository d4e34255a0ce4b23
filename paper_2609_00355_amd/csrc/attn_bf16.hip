// Launch of the bf16 attention over a dense cache read in whole (attn_bf16.h).
#include "attn_bf16.h"

namespace glance {
namespace {

template <int D, bool TREE>
void launch(const AttnParams& p, dim3 grid, dim3 block, hipStream_t s) {
  if (p.tiles_rg > 4) hipLaunchKernelGGL((attn_bf16<D, TREE, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((attn_bf16<D, TREE, false>), grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_attn_bf16(const AttnParams& p, bool tree, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  const dim3 grid(grid_blocks(p)), block(512);
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.d == 128) {
    if (tree) launch<128, true>(p, grid, block, s);
    else launch<128, false>(p, grid, block, s);
  } else {
    if (tree) launch<64, true>(p, grid, block, s);
    else launch<64, false>(p, grid, block, s);
  }
  hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
