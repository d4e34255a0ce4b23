// Drives the entry points of the context-cache operators (glance_cache_api.cpp)
// with the launchers stubbed, under AddressSanitizer and
// UndefinedBehaviorSanitizer.  Placeholder device pointers are never read.
#include <stdio.h>
#include <stdlib.h>

#include <vector>

#include "glance.h"
#include "stubs.h"

extern int g_cache_launches;
static int g_checks = 0;
#define CHECK(cond)                                                                                    \
  do {                                                                                                 \
    ++g_checks;                                                                                        \
    if (!(cond)) {                                                                                     \
      fprintf(stderr, "CHECK failed at line %d: %s (%s)\n", __LINE__, #cond, glance_last_error());     \
      exit(1);                                                                                         \
    }                                                                                                  \
  } while (0)

static void* fake(uintptr_t k) { return reinterpret_cast<void*>(k << 40); }

static glance_cache cache(int batch, int hkv, int d, int cap, glance_cache_format f, glance_dtype dt, uintptr_t at) {
  glance_cache c = {batch, hkv, d, cap, f, dt, fake(at), fake(at + 1), nullptr, nullptr,
                    static_cast<int32_t*>(fake(at + 4)), static_cast<float*>(fake(at + 5))};
  if (f == GLANCE_CACHE_KV4) c.k_scale = fake(at + 2), c.v_scale = fake(at + 3);
  return c;
}

int main() {
  std::vector<char> buf;
  const int shapes[][6] = {{1, 16, 4, 1, 64, 256}, {16, 64, 28, 4, 128, 32768}, {16, 1, 28, 4, 128, 32768}, {3, 37, 8, 2, 64, 11003},
                           {1, 1, 4, 4, 64, 0},    {40, 64, 16, 1, 128, 720},   {1, 64, 64, 4, 128, 5}};
  const int reach[][2] = {{0, 0}, {0, 1}, {4, 64}, {1000, 3}, {2147483647, 2147483647}, {17, 4096}, {5, 2500}};
  for (int dt = 0; dt < 2; ++dt)
    for (int f = 0; f < 2; ++f)
      for (auto& sh : shapes)
        for (auto& r : reach) {
          glance_attn_shape s = {sh[0], sh[1], sh[2], sh[3], sh[4], sh[5], 0.f, (glance_dtype)dt};
          glance_cache c = cache(sh[0], sh[3], sh[4], sh[5], (glance_cache_format)f, (glance_dtype)dt, 16);
          const size_t need = glance_cache_attn_workspace_size(&s, r[0], r[1]);
          CHECK(need > 0);
          buf.assign(need + 256, 0);
          char* ws = buf.data() + ((256 - (reinterpret_cast<uintptr_t>(buf.data()) & 255)) & 255);
          g_stub.ws = ws;
          g_stub.ws_bytes = need;
          const int before = g_cache_launches;
          CHECK(glance_cache_block_draft_attn(&s, &c, r[0], r[1], fake(1), fake(2), fake(3), fake(4), nullptr, ws, need,
                                              nullptr) == GLANCE_OK);
          CHECK(glance_cache_tree_verify_attn(&s, &c, r[0], r[1], fake(1), fake(2), fake(3), (const int32_t*)fake(5), fake(4),
                                              (float*)fake(6), ws, need, nullptr) == GLANCE_OK);
          CHECK(glance_cache_tree_verify_attn(&s, &c, r[0], r[1], fake(1), fake(2), fake(3), (const int32_t*)fake(5), fake(4),
                                              (float*)fake(6), ws, need - 1, nullptr) == GLANCE_ERR_WORKSPACE);
          CHECK(g_cache_launches == before + 2);
          const glance_status st = glance_cache_weigh(&s, &c, r[0], r[1], fake(1), (const float*)fake(6), nullptr, nullptr,
                                                      nullptr, 0, 0.5f, c.weights, nullptr);
          CHECK(st == (sh[5] ? GLANCE_OK : GLANCE_ERR_INVALID_ARG));
        }
  glance_cache dense = cache(2, 2, 64, 100, GLANCE_CACHE_DENSE, GLANCE_BF16, 16);
  glance_cache packed = cache(2, 2, 64, 80, GLANCE_CACHE_KV4, GLANCE_F32, 32);
  CHECK(glance_cache_convert(&dense, &packed, nullptr) == GLANCE_OK);
  CHECK(glance_cache_convert(&packed, &dense, nullptr) == GLANCE_OK);
  CHECK(glance_cache_convert(&dense, &dense, nullptr) == GLANCE_ERR_INVALID_ARG);
  CHECK(glance_cache_commit_path(&packed, 8, GLANCE_BF16, fake(1), fake(2), (const int32_t*)fake(3), (const int32_t*)fake(4), 8,
                                 nullptr) == GLANCE_OK);
  CHECK(glance_cache_commit_path(&dense, 8, GLANCE_BF16, fake(1), fake(2), (const int32_t*)fake(3), (const int32_t*)fake(4), 8,
                                 nullptr) == GLANCE_OK);
  glance_cache to = cache(2, 2, 64, 50, GLANCE_CACHE_DENSE, GLANCE_BF16, 48);
  CHECK(glance_cache_evict(&dense, &to, 50, 4, 46, (int32_t*)fake(1), nullptr) == GLANCE_OK);
  CHECK(glance_cache_evict(&dense, &to, 51, 4, 46, (int32_t*)fake(1), nullptr) == GLANCE_ERR_INVALID_ARG);
  // a buffer of the one inside a buffer of the other, and just behind it
  to.k = static_cast<char*>(dense.v) + 2 * 2 * 100 * 128 - 16;
  CHECK(glance_cache_evict(&dense, &to, 50, 4, 4, (int32_t*)fake(1), nullptr) == GLANCE_ERR_INVALID_ARG);
  to.k = static_cast<char*>(dense.v) + 2 * 2 * 100 * 128;
  CHECK(glance_cache_evict(&dense, &to, 50, 4, 4, (int32_t*)fake(1), nullptr) == GLANCE_OK);
  // fields that hold no value of their enum
  int bad = 9;
  glance_cache odd = dense;
  __builtin_memcpy(&odd.format, &bad, sizeof bad);
  CHECK(glance_cache_convert(&odd, &packed, nullptr) == GLANCE_ERR_UNSUPPORTED);
  odd = dense;
  __builtin_memcpy(&odd.dtype, &bad, sizeof bad);
  CHECK(glance_cache_convert(&odd, &packed, nullptr) == GLANCE_ERR_UNSUPPORTED);
  odd = packed;
  __builtin_memcpy(&odd.dtype, &bad, sizeof bad);  // not read in a 4-bit cache
  CHECK(glance_cache_convert(&dense, &odd, nullptr) == GLANCE_OK);
  printf("%d checks passed\n", g_checks);
  return 0;
}
