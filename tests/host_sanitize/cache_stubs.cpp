// Host-only stand-ins for the launchers of the context-cache operators, beside
// stubs.cpp: each checks the parameters that the kernels index with.
#include <stdio.h>
#include <stdlib.h>

#include "glance_internal.h"
#include "stubs.h"

int g_cache_launches = 0;

namespace {
void must(bool ok, const char* what) {
  if (!ok) {
    fprintf(stderr, "STUB FAIL: %s\n", what);
    abort();
  }
}
void in_ws(const void* p, size_t bytes, const char* what) {
  const char* a = static_cast<const char*>(p);
  const char* w = static_cast<const char*>(g_stub.ws);
  must(w && a >= w && a + bytes <= w + g_stub.ws_bytes, what);
}
}  // namespace

namespace glance {

hipError_t launch_attn_cache_bf16(const AttnParams& p, bool kv4, bool, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  const size_t wslots = (size_t)p.slots_per_g * p.hkv * p.row_groups;
  in_ws(p.plan, (size_t)p.batch * sizeof(int2), "piece table");
  in_ws(p.part_ml, wslots * p.rows_rg * sizeof(float2), "(max, sum) partials");
  in_ws(p.part_o, wslots * p.tiles_rg * (size_t)(p.d / 8) * 64 * 8, "output partials");
  must(p.window >= 1 && p.n_sinks >= 0, "reach");
  must(!kv4 || p.cap == 0 || (p.k_scale && p.v_scale), "scales");
  return hipSuccess;
}

hipError_t launch_attn_cache_f32(const AttnParams& p, bool kv4, bool, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  const size_t slots = (size_t)p.batch * p.hkv * p.nsplit * p.rows_pad;
  in_ws(p.part_ml, slots * sizeof(float2), "(max, sum) partials");
  in_ws(p.part_o, slots * p.d * sizeof(float), "output partials");
  must(p.window >= 1 && p.n_sinks >= 0, "reach");
  must(!kv4 || p.cap == 0 || (p.k_scale && p.v_scale), "scales");
  // the splits hold every key that a sequence of any length reads: the sinks'
  // blocks of 16 and the blocks from the one that row 0's window begins in
  for (long long ctx = 0; ctx <= p.cap; ctx += ctx < 200 ? 1 : 37) {
    const long long lo = ctx - p.window + 1 > 0 ? ctx - p.window + 1 : 0;
    const long long sinks = ((p.n_sinks < ctx ? p.n_sinks : ctx) + 15) / 16 * 16;
    long long first = lo / 16 * 16 > sinks ? lo / 16 * 16 : sinks;
    if (first > ctx) first = ctx;
    const long long keys = (sinks < ctx ? sinks : ctx) + (lo < ctx ? ctx - first : 0);
    must(keys <= (long long)p.nsplit * p.split_keys, "splits");
  }
  return hipSuccess;
}

hipError_t launch_cache_convert(const CacheParams& p, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  must(p.src.kv4 != p.dst.kv4, "formats");
  return hipSuccess;
}

hipError_t launch_commit_kv4(const CommitKv4Params& p, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  must(p.dst.kv4 && p.n >= 1 && p.n <= 64, "commit");
  return hipSuccess;
}

hipError_t launch_weigh(const WeighParams& p, bool, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  must(p.group >= 1 && p.group * p.hkv == p.hq && p.window >= 1, "weigh");
  return hipSuccess;
}

hipError_t launch_evict(const EvictParams& p, hipStream_t, hipEvent_t, hipEvent_t) {
  ++g_cache_launches;
  must(p.budget >= 1 && p.budget <= p.dst.cap && p.n_sinks + p.n_recent <= p.budget, "evict");
  return hipSuccess;
}

}  // namespace glance
