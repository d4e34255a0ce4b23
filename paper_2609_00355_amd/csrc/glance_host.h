// What the host layer's files share: error reporting, argument checks and the
// attention plan.
#pragma once

#include "glance.h"
#include "glance_internal.h"

namespace glance {

// Records the calling thread's error message; returns st.
glance_status fail(glance_status st, const char* fmt, ...) __attribute__((format(printf, 2, 3)));

inline bool aligned16(const void* ptr) { return (reinterpret_cast<uintptr_t>(ptr) & 15u) == 0; }

bool dtype_ok(const glance_dtype& d);

glance_status check_hip(hipError_t e, const char* what);

// The pending profiling events, which the next call takes.
void take_events(hipEvent_t* a, hipEvent_t* b);

// Attention workspace: [piece table][(max, sum) partials][O partials].
struct Plan {
  AttnParams p;
  size_t counter_bytes;  // the bf16 path's per-sequence piece table
  size_t part_ml_bytes;
  size_t part_o_bytes;
  size_t total;
};

// window 0: the kernels that read a dense cache in whole.
glance_status make_plan(const glance_attn_shape* s, int n_sinks, int window, Plan* out);

// The checks of an attention call's own arguments that both kinds of cache
// share, and the plan's pointers set up in p.
glance_status bind_attn(const glance_attn_shape* s, const Plan& pl, bool tree, const void* q, const void* k_ctx,
                        const void* v_ctx, const void* k_new, const void* v_new, const int32_t* ctx_lens,
                        const int32_t* parents, void* out, float* lse, void* workspace, size_t workspace_bytes,
                        AttnParams* p);

}  // namespace glance
