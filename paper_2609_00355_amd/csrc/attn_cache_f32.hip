// Launch of the fp32 attention over a context cache that is read in part (a
// window and its first keys) or held in 4 bits: the kernel of attn_f32.h with
// those reads compiled in.
#include "attn_f32.h"

namespace glance {
namespace {

template <int D, bool TREE, bool KV4>
void launch_rows(const AttnParams& p, dim3 grid, hipStream_t s) {
  if (p.rows_rg == 16) hipLaunchKernelGGL((attn_f32<D, TREE, 1, 8, KV4, true>), grid, dim3(512), 0, s, p);
  else hipLaunchKernelGGL((attn_f32<D, TREE, 2, 4, KV4, true>), grid, dim3(256), 0, s, p);
}

template <int D, bool TREE>
void launch(const AttnParams& p, bool kv4, hipStream_t s) {
  const int items = p.nsplit * p.batch * p.hkv * p.row_groups;
  const dim3 grid((items + 7) / 8 * 8);
  if (kv4) launch_rows<D, TREE, true>(p, grid, s);
  else launch_rows<D, TREE, false>(p, grid, s);
}

}  // namespace

hipError_t launch_attn_cache_f32(const AttnParams& p, bool kv4, bool tree, hipStream_t s, hipEvent_t ev0,
                                  hipEvent_t ev1) {
  // A dense cache without a window: the plain call's kernel, for the same bits (and
  // 48.2 us instead of 55.1 for 64 rows of 28/4 heads of 128 over 4096 keys).
  if (!kv4 && p.window == kNoWindow) return launch_attn_f32(p, tree, s, ev0, ev1);
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
