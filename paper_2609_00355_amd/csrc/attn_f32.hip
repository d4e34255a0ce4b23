// Launch of the fp32 attention over a dense cache read in whole (attn_f32.h).
#include "attn_f32.h"

namespace glance {
namespace {

template <int D, bool TREE>
void launch(const AttnParams& p, dim3 grid, hipStream_t s) {
  if (p.rows_rg == 16) hipLaunchKernelGGL((attn_f32<D, TREE, 1, 8>), grid, dim3(512), 0, s, p);
  else hipLaunchKernelGGL((attn_f32<D, TREE, 2, 4>), grid, dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_attn_f32(const AttnParams& p, bool tree, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  const int items = p.nsplit * p.batch * p.hkv * p.row_groups;
  const dim3 grid((items + 7) / 8 * 8);
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.d == 128) {
    if (tree) launch<128, true>(p, grid, s);
    else launch<128, false>(p, grid, s);
  } else {
    if (tree) launch<64, true>(p, grid, s);
    else launch<64, false>(p, grid, s);
  }
  hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
