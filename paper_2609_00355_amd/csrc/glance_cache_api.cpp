// C-ABI host layer of the operators on a context cache: argument checks and
// kernel launches (see include/glance.h).
#include "glance.h"

#include <string.h>

#include "glance_host.h"

namespace glance {
namespace {

glance_status ok() { return GLANCE_OK; }

// The format as the integer the caller stored (any int may be in the field).
int format_bits(const glance_cache& c) {
  int v;
  memcpy(&v, &c.format, sizeof v);
  return v;
}

bool is_kv4(const glance_cache& c) { return format_bits(c) == GLANCE_CACHE_KV4; }

size_t row_bytes(const glance_cache& c) {
  return is_kv4(c) ? (size_t)c.head_dim / 2 : (size_t)c.head_dim * (c.dtype == GLANCE_BF16 ? 2 : 4);
}

struct Need {
  const void* ptr;
  const char* name;
  bool need;
  size_t align;
};

// `owner` (or "") names the struct whose fields these are.
template <size_t N>
glance_status check_pointers(const Need (&req)[N], const char* owner) {
  const char* sep = owner[0] ? ": " : "";
  for (auto& r : req) {
    if (r.need && !r.ptr) return fail(GLANCE_ERR_INVALID_ARG, "%s%s%s is NULL", owner, sep, r.name);
    if (r.ptr && (reinterpret_cast<uintptr_t>(r.ptr) & (r.align - 1)))
      return fail(GLANCE_ERR_INVALID_ARG, "%s%s%s is not %zu-byte aligned", owner, sep, r.name, r.align);
  }
  return ok();
}

// Sizes, format and pointers of one cache; `name` names it in messages.
glance_status check_cache(const glance_cache* c, const char* name) {
  if (!c) return fail(GLANCE_ERR_INVALID_ARG, "%s is NULL", name);
  if (c->batch < 1) return fail(GLANCE_ERR_INVALID_ARG, "%s: batch must be >= 1 (got %d)", name, c->batch);
  if (c->n_kv_heads < 1) return fail(GLANCE_ERR_INVALID_ARG, "%s: n_kv_heads must be >= 1", name);
  if (c->batch > 32767 || c->n_kv_heads > 65535)  // grid dimensions
    return fail(GLANCE_ERR_UNSUPPORTED, "%s: batch must be <= 32767 and n_kv_heads <= 65535", name);
  if (c->head_dim != 64 && c->head_dim != 128)
    return fail(GLANCE_ERR_UNSUPPORTED, "%s: head_dim must be 64 or 128 (got %d)", name, c->head_dim);
  if (c->capacity < 0) return fail(GLANCE_ERR_INVALID_ARG, "%s: capacity must be >= 0", name);
  if (c->capacity > 1 << 25) return fail(GLANCE_ERR_UNSUPPORTED, "%s: capacity must be <= 2^25", name);
  const int f = format_bits(*c);
  if (f != GLANCE_CACHE_DENSE && f != GLANCE_CACHE_KV4)
    return fail(GLANCE_ERR_UNSUPPORTED, "%s: format must be GLANCE_CACHE_DENSE or GLANCE_CACHE_KV4", name);
  if (f == GLANCE_CACHE_DENSE && !dtype_ok(c->dtype))
    return fail(GLANCE_ERR_UNSUPPORTED, "%s: dtype must be GLANCE_F32 or GLANCE_BF16", name);
  const bool scales = f == GLANCE_CACHE_KV4 && c->capacity > 0;
  const Need req[] = {{c->k, "k", c->capacity > 0, 16},     {c->v, "v", c->capacity > 0, 16},
                      {c->k_scale, "k_scale", scales, 16},  {c->v_scale, "v_scale", scales, 16},
                      {c->ctx_lens, "ctx_lens", true, 4},   {c->weights, "weights", false, 4}};
  return check_pointers(req, name);
}

CacheView view(const glance_cache& c) {
  CacheView v = {};
  v.k = static_cast<unsigned char*>(c.k);
  v.v = static_cast<unsigned char*>(c.v);
  v.k_scale = static_cast<unsigned char*>(c.k_scale);
  v.v_scale = static_cast<unsigned char*>(c.v_scale);
  v.lens = c.ctx_lens;
  v.weights = c.weights;
  v.cap = c.capacity;
  v.row_bytes = (int)row_bytes(c);
  v.kv4 = is_kv4(c);
  return v;
}

glance_status check_reach(int32_t n_sinks, int32_t window) {
  if (n_sinks < 0) return fail(GLANCE_ERR_INVALID_ARG, "n_sinks must be >= 0 (got %d)", n_sinks);
  if (window < 0) return fail(GLANCE_ERR_INVALID_ARG, "window must be >= 0 (got %d)", window);
  return ok();
}

// Shape, reach and cache of a call that reads the cache, and its plan.
glance_status check_read(const glance_attn_shape* s, const glance_cache* c, int32_t n_sinks, int32_t window,
                         Plan* pl) {
  glance_status st = check_reach(n_sinks, window);
  if (st == GLANCE_OK) st = make_plan(s, n_sinks, window ? window : kNoWindow, pl);
  if (st == GLANCE_OK) st = check_cache(c, "cache");
  if (st != GLANCE_OK) return st;
  if (c->batch != s->batch || c->n_kv_heads != s->n_kv_heads || c->head_dim != s->head_dim ||
      c->capacity != s->ctx_capacity)
    return fail(GLANCE_ERR_INVALID_ARG, "the cache's batch, n_kv_heads, head_dim and capacity must be the shape's");
  if (!is_kv4(*c) && c->dtype != s->dtype)
    return fail(GLANCE_ERR_INVALID_ARG, "a dense cache's dtype must be the shape's");
  return ok();
}

// Whether two buffers share a byte.
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && x < y + b_bytes && y < x + a_bytes;
}

// The caches of a call that copies from one into the other: the same heads,
// and no buffer of the one in a buffer of the other (the lengths may be shared).
glance_status check_pair(const glance_cache* src, const glance_cache* dst) {
  glance_status st = check_cache(src, "src");
  if (st == GLANCE_OK) st = check_cache(dst, "dst");
  if (st != GLANCE_OK) return st;
  if (src->batch != dst->batch || src->n_kv_heads != dst->n_kv_heads || src->head_dim != dst->head_dim)
    return fail(GLANCE_ERR_INVALID_ARG, "src and dst must have the same batch, n_kv_heads and head_dim");
  struct Buf {
    const void* ptr;
    size_t bytes;
  };
  auto bufs = [](const glance_cache& c, Buf (&out)[5]) {
    const size_t rows = (size_t)c.batch * c.n_kv_heads * c.capacity;
    const size_t scales = is_kv4(c) ? rows * (c.head_dim / 32) : 0;
    out[0] = {c.k, rows * row_bytes(c)};
    out[1] = {c.v, rows * row_bytes(c)};
    out[2] = {scales ? c.k_scale : nullptr, scales};
    out[3] = {scales ? c.v_scale : nullptr, scales};
    out[4] = {c.weights, rows * sizeof(float)};
  };
  Buf a[5], b[5];
  bufs(*src, a);
  bufs(*dst, b);
  for (auto& x : a)
    for (auto& y : b)
      if (overlap(x.ptr, x.bytes, y.ptr, y.bytes))
        return fail(GLANCE_ERR_INVALID_ARG, "src and dst must not overlap");
  const size_t lens = (size_t)src->batch * sizeof(int32_t);
  if (src->ctx_lens != dst->ctx_lens && overlap(src->ctx_lens, lens, dst->ctx_lens, lens))
    return fail(GLANCE_ERR_INVALID_ARG, "src's and dst's ctx_lens must be one array or apart");
  return ok();
}

glance_status cache_attn(bool tree, const glance_attn_shape* s, const glance_cache* cache, int32_t n_sinks,
                         int32_t window, const void* q, const void* k_new, const void* v_new,
                         const int32_t* parents, void* out, float* lse, void* workspace, size_t workspace_bytes,
                         hipStream_t stream) {
  Plan pl;
  AttnParams p;
  glance_status st = check_read(s, cache, n_sinks, window, &pl);
  if (st == GLANCE_OK)
    st = bind_attn(s, pl, tree, q, cache->k, cache->v, k_new, v_new, cache->ctx_lens, parents, out, lse, workspace,
                   workspace_bytes, &p);
  if (st != GLANCE_OK) return st;
  const bool kv4 = is_kv4(*cache), bf16 = s->dtype == GLANCE_BF16;
  p.k_scale = static_cast<const unsigned char*>(cache->k_scale);
  p.v_scale = static_cast<const unsigned char*>(cache->v_scale);
  hipEvent_t e0, e1;
  take_events(&e0, &e1);
  hipError_t e = bf16 ? launch_attn_cache_bf16(p, kv4, tree, stream, e0, e1)
                      : launch_attn_cache_f32(p, kv4, tree, stream, e0, e1);
  if ((st = check_hip(e, "attention kernel launch")) != GLANCE_OK) return st;
  if (!bf16 && p.nsplit == 1) return ok();  // every workgroup wrote its rows' output
  e = bf16 ? launch_attn_merge_pieces(p, stream) : launch_attn_merge(p, stream);
  return check_hip(e, "merge kernel launch");
}

}  // namespace
}  // namespace glance

using namespace glance;

extern "C" {

glance_status glance_cache_block_draft_attn(const glance_attn_shape* s, const glance_cache* cache, int32_t n_sinks,
                                            int32_t window, const void* q, const void* k_new, const void* v_new,
                                            void* out, float* lse, void* workspace, size_t workspace_bytes,
                                            hipStream_t stream) {
  return cache_attn(false, s, cache, n_sinks, window, q, k_new, v_new, nullptr, out, lse, workspace,
                    workspace_bytes, stream);
}

glance_status glance_cache_tree_verify_attn(const glance_attn_shape* s, const glance_cache* cache, int32_t n_sinks,
                                            int32_t window, const void* q, const void* k_new, const void* v_new,
                                            const int32_t* parents, void* out, float* lse, void* workspace,
                                            size_t workspace_bytes, hipStream_t stream) {
  return cache_attn(true, s, cache, n_sinks, window, q, k_new, v_new, parents, out, lse, workspace,
                    workspace_bytes, stream);
}

size_t glance_cache_attn_workspace_size(const glance_attn_shape* s, int32_t n_sinks, int32_t window) {
  Plan pl;
  if (check_reach(n_sinks, window) != GLANCE_OK) return 0;
  if (make_plan(s, n_sinks, window ? window : kNoWindow, &pl) != GLANCE_OK) return 0;
  return pl.total;
}

glance_status glance_cache_convert(const glance_cache* src, const glance_cache* dst, hipStream_t stream) {
  glance_status st = check_pair(src, dst);
  if (st != GLANCE_OK) return st;
  if (is_kv4(*src) == is_kv4(*dst))
    return fail(GLANCE_ERR_INVALID_ARG, "one of src and dst must be dense and the other in 4 bits");
  CacheParams p = {};
  p.src = view(*src);
  p.dst = view(*dst);
  p.batch = src->batch;
  p.hkv = src->n_kv_heads;
  p.d = src->head_dim;
  p.bf16 = (is_kv4(*src) ? dst : src)->dtype == GLANCE_BF16;
  hipEvent_t e0, e1;
  take_events(&e0, &e1);
  return check_hip(launch_cache_convert(p, stream, e0, e1), "conversion kernel launch");
}

glance_status glance_cache_commit_path(const glance_cache* cache, int32_t n_nodes, glance_dtype dtype,
                                       const void* k_new, const void* v_new, const int32_t* accept_len,
                                       const int32_t* accept_path, int32_t path_stride, hipStream_t stream) {
  glance_status st = check_cache(cache, "cache");
  if (st != GLANCE_OK) return st;
  if (!dtype_ok(dtype)) return fail(GLANCE_ERR_UNSUPPORTED, "dtype must be GLANCE_F32 or GLANCE_BF16");
  if (!is_kv4(*cache)) {
    if (cache->dtype != dtype) return fail(GLANCE_ERR_INVALID_ARG, "a dense cache's dtype must be the new rows'");
    return glance_commit_path(cache->batch, n_nodes, cache->n_kv_heads, cache->head_dim, cache->capacity, dtype, k_new,
                              v_new, accept_len, accept_path, path_stride, cache->k, cache->v, cache->ctx_lens,
                              stream);
  }
  if (n_nodes < 1 || n_nodes > 64)
    return fail(GLANCE_ERR_UNSUPPORTED, "n_nodes must be in 1..64 (got %d)", n_nodes);
  if (cache->capacity < 1) return fail(GLANCE_ERR_INVALID_ARG, "cache: capacity must be >= 1");
  if (path_stride < 1) return fail(GLANCE_ERR_INVALID_ARG, "path_stride must be >= 1");
  const Need req[] = {{k_new, "k_new", true, 16},
                      {v_new, "v_new", true, 16},
                      {accept_len, "accept_len", true, 4},
                      {accept_path, "accept_path", true, 4}};
  if ((st = check_pointers(req, "")) != GLANCE_OK) return st;
  CommitKv4Params p = {};
  p.dst = view(*cache);
  p.k_new = k_new;
  p.v_new = v_new;
  p.accept_len = accept_len;
  p.accept_path = accept_path;
  p.batch = cache->batch;
  p.hkv = cache->n_kv_heads;
  p.d = cache->head_dim;
  p.n = n_nodes;
  p.path_stride = path_stride;
  p.bf16 = dtype == GLANCE_BF16;
  hipEvent_t e0, e1;
  take_events(&e0, &e1);
  return check_hip(launch_commit_kv4(p, stream, e0, e1), "commit kernel launch");
}

glance_status glance_cache_weigh(const glance_attn_shape* s, const glance_cache* cache, int32_t n_sinks,
                                 int32_t window, const void* q, const float* lse, const void* k_new,
                                 const int32_t* accept_len, const int32_t* accept_path, int32_t path_stride,
                                 float decay, float* weights_out, hipStream_t stream) {
  Plan pl;
  glance_status st = check_read(s, cache, n_sinks, window, &pl);
  if (st != GLANCE_OK) return st;
  if (cache->capacity < 1) return fail(GLANCE_ERR_INVALID_ARG, "cache: capacity must be >= 1");
  if (!(decay >= 0.f && decay <= 1.f))
    return fail(GLANCE_ERR_INVALID_ARG, "decay must be in [0, 1] (got %g)", (double)decay);
  const bool path = accept_path != nullptr;
  if (path != (accept_len != nullptr) || path != (k_new != nullptr))
    return fail(GLANCE_ERR_INVALID_ARG, "a path needs k_new, accept_len and accept_path, and no path none of them");
  if (path && path_stride < 1) return fail(GLANCE_ERR_INVALID_ARG, "path_stride must be >= 1");
  if (decay > 0.f && !cache->weights) return fail(GLANCE_ERR_INVALID_ARG, "cache: weights is NULL");
  const Need req[] = {{q, "q", true, 16},
                      {lse, "lse", true, 4},
                      {weights_out, "weights_out", true, 4},
                      {k_new, "k_new", path, 16},
                      {accept_len, "accept_len", path, 4},
                      {accept_path, "accept_path", path, 4}};
  if ((st = check_pointers(req, "")) != GLANCE_OK) return st;
  const size_t bytes = (size_t)s->batch * s->n_kv_heads * s->ctx_capacity * sizeof(float);
  if (weights_out != cache->weights && overlap(weights_out, bytes, cache->weights, bytes))
    return fail(GLANCE_ERR_INVALID_ARG, "weights_out must be the cache's weights or apart from them");
  WeighParams p = {};
  p.cache = view(*cache);
  p.q = q;
  p.lse = lse;
  p.k_new = k_new;
  p.accept_len = accept_len;
  p.accept_path = accept_path;
  p.out = weights_out;
  p.batch = s->batch;
  p.n = s->n_new;
  p.hq = s->n_q_heads;
  p.hkv = s->n_kv_heads;
  p.group = pl.p.group;
  p.d = s->head_dim;
  p.path_stride = path_stride;
  p.n_sinks = n_sinks;
  p.window = pl.p.window;
  p.scale_log2 = pl.p.scale_log2;
  p.decay = decay;
  hipEvent_t e0, e1;
  take_events(&e0, &e1);
  return check_hip(launch_weigh(p, s->dtype == GLANCE_BF16, stream, e0, e1), "weights kernel launch");
}

glance_status glance_cache_evict(const glance_cache* src, const glance_cache* dst, int32_t budget, int32_t n_sinks,
                                 int32_t n_recent, int32_t* kept, hipStream_t stream) {
  glance_status st = check_pair(src, dst);
  if (st != GLANCE_OK) return st;
  if (is_kv4(*src) != is_kv4(*dst) || (!is_kv4(*src) && src->dtype != dst->dtype))
    return fail(GLANCE_ERR_INVALID_ARG, "src and dst must have the same format and dtype");
  if ((long long)src->batch * src->n_kv_heads > 65535)  // a grid dimension
    return fail(GLANCE_ERR_UNSUPPORTED, "batch * n_kv_heads must be <= 65535");
  if (!src->weights || !dst->weights)
    return fail(GLANCE_ERR_INVALID_ARG, "%s: weights is NULL", src->weights ? "dst" : "src");
  if (src->capacity < 1) return fail(GLANCE_ERR_INVALID_ARG, "src: capacity must be >= 1");
  if (budget < 1) return fail(GLANCE_ERR_INVALID_ARG, "budget must be >= 1 (got %d)", budget);
  if (dst->capacity < budget)
    return fail(GLANCE_ERR_INVALID_ARG, "dst's capacity (%d) must be >= budget (%d)", dst->capacity, budget);
  if (n_sinks < 0 || n_recent < 0)
    return fail(GLANCE_ERR_INVALID_ARG, "n_sinks and n_recent must be >= 0 (got %d, %d)", n_sinks, n_recent);
  if ((long long)n_sinks + n_recent > budget)
    return fail(GLANCE_ERR_INVALID_ARG, "n_sinks + n_recent (%d + %d) must be <= budget (%d)", n_sinks, n_recent,
                budget);
  const Need req[] = {{kept, "kept", true, 4}};
  if ((st = check_pointers(req, "")) != GLANCE_OK) return st;
  EvictParams p = {};
  p.src = view(*src);
  p.dst = view(*dst);
  p.kept = kept;
  p.batch = src->batch;
  p.hkv = src->n_kv_heads;
  p.d = src->head_dim;
  p.budget = budget;
  p.n_sinks = n_sinks;
  p.n_recent = n_recent;
  hipEvent_t e0, e1;
  take_events(&e0, &e1);
  return check_hip(launch_evict(p, stream, e0, e1), "eviction kernel launch");
}

}  // extern "C"
