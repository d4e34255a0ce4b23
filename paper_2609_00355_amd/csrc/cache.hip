// A context cache in 4 bits: conversion from and into a dense one, and the
// commit of a round's accepted path into it.
//
// Format.  32 consecutive dims of a key or value share a power of two 2^e; each
// is held as the nearest of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times 2^e (one sign, two
// exponent and one fraction bit), ties to the even code, at most 6.  With a the
// largest magnitude, e is two below the exponent of a rounded to two
// significant bits: a 2^-e lies in [3.5, 7), so clipping to 6 loses at most one
// of 7 and no block gives up its last bit to a maximum just above 6.  e >= -125
// keeps every nonzero value a normal number, e <= 125 every value finite.  A byte holds e + 127, and 255
// (every value reads NaN) where the block has a NaN or an infinity.
//
// On the GPU: the exponent byte is (bits(a) + 2^21) >> 23, less two (2^21 is
// half a unit of the second significant bit), a's bits being the integer
// maximum of the magnitudes' bits, which NaN and infinity win.  The codes come
// from the scaled conversion instruction, which rounds to nearest even and
// clips.  Bound by memory: a lane takes eight values, four lanes a block, so that
// loads are 16 bytes a lane and a block's maximum two exchanges within a quad.
// 4 caches of 16384 slots, 4 heads of 128 in bf16 (134 MB and 36 MB of codes and
// scales): into 4 bits 39 us, 4.4 TB/s, and back 26, 6.5 TB/s.
#include "glance_internal.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;

__device__ __forceinline__ int clamp_len(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }

// Eight values of a row at element `at` (a multiple of 8) as floats.
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, size_t at, float (&x)[8]) {
  if constexpr (BF16) {
    const u32x4 w = *reinterpret_cast<const u32x4*>(static_cast<const unsigned short*>(base) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __builtin_bit_cast(float, w[i] << 16);
      x[2 * i + 1] = __builtin_bit_cast(float, w[i] & 0xffff0000u);
    }
  } else {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + at);
    const f32x4 a = p[0], b = p[1];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[i] = a[i];
      x[4 + i] = b[i];
    }
  }
}

// The larger of a lane's value and its neighbour's; the four lanes of a block
// are one quad.
template <int CTRL>
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}

// Codes of a lane's eight values and the block's exponent byte (every lane of
// the quad takes part).
__device__ __forceinline__ unsigned encode8(const float (&x)[8], unsigned& scale) {
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const unsigned a = __builtin_bit_cast(unsigned, x[i]) & 0x7fffffffu;
    m = m > a ? m : a;
  }
  m = quad_max<0xb1>(m);  // quad_perm [1,0,3,2]
  m = quad_max<0x4e>(m);  // quad_perm [2,3,0,1]
  const unsigned e = (m + 0x200000u) >> 23;
  scale = m >= 0x7f800000u ? 255u : min(max(e, 4u), 254u) - 2u;
  const float s = __builtin_bit_cast(float, scale << 23);
  unsigned c = 0;
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
  c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
  return c;
}

constexpr int kConvertThreads = 256;

// Grid (chunks of a head's rows, KV heads, 2 batch: keys and values).
template <bool BF16, bool PACK>
__global__ __launch_bounds__(kConvertThreads) void convert_kernel(CacheParams p) {
  const int b = blockIdx.z >> 1, g = blockIdx.y;
  const bool v_side = blockIdx.z & 1;
  const int len = min(clamp_len(p.src.lens[b], p.src.cap), p.dst.cap);
  if (blockIdx.x == 0 && g == 0 && !v_side && threadIdx.x == 0) p.dst.lens[b] = len;
  const int per_row = p.d / 8;  // 8 or 16 lanes: a row's quads stay in one wave
  const int u = blockIdx.x * kConvertThreads + threadIdx.x;
  const int row = u / per_row, part = u % per_row;
  if (row >= len) return;
  const size_t head = (size_t)b * p.hkv + g;
  const size_t from = head * p.src.cap + row, to = head * p.dst.cap + row;
  const unsigned char* src = v_side ? p.src.v : p.src.k;
  unsigned char* dst = v_side ? p.dst.v : p.dst.k;
  if constexpr (PACK) {
    float x[8];
    load8<BF16>(src, from * p.d + 8 * part, x);
    unsigned scale;
    const unsigned c = encode8(x, scale);
    *reinterpret_cast<unsigned*>(dst + to * (p.d / 2) + 4 * part) = c;
    if (part % 4 == 0) (v_side ? p.dst.v_scale : p.dst.k_scale)[to * (p.d / 32) + part / 4] = (unsigned char)scale;
  } else {
    const unsigned c = *reinterpret_cast<const unsigned*>(src + from * (p.d / 2) + 4 * part);
    const unsigned e = (v_side ? p.src.v_scale : p.src.k_scale)[from * (p.d / 32) + part / 4];
    const float s = __builtin_bit_cast(float, e << 23);
    if constexpr (BF16) {
      const u32x4 w = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 0)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 1)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 2)),
                       __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c, s, 3))};
      *reinterpret_cast<u32x4*>(dst + (to * p.d + 8 * part) * 2) = w;
    } else {
      const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 0), b2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 1);
      const f32x2 d = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 2), f = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c, s, 3);
      f32x4* o = reinterpret_cast<f32x4*>(dst + (to * p.d + 8 * part) * 4);
      o[0] = f32x4{a[0], a[1], b2[0], b2[1]};
      o[1] = f32x4{d[0], d[1], f[0], f[1]};
    }
  }
}

constexpr int kCommitThreads = 512;

// Commit of an accepted path, one workgroup a sequence (as commit.hip, whose
// clamps these are): slot ctx + i takes the codes of path node i's rows, and
// the length is advanced behind a barrier.
template <bool BF16>
__global__ __launch_bounds__(kCommitThreads) void commit_kv4_kernel(CommitKv4Params p) {
  __shared__ int s_node[64];
  __shared__ int s_rows, s_ctx;
  const int b = blockIdx.x, tid = threadIdx.x;
  if (tid == 0) {
    const int want = max(0, min(min(p.accept_len[b] >= 64 ? 64 : p.accept_len[b] + 1, p.path_stride), p.n));
    int r = 0;
    for (; r < want; ++r) {
      const int node = p.accept_path[(size_t)b * p.path_stride + r];
      if (node < 0 || node >= p.n) break;
      s_node[r] = node;
    }
    s_rows = r;
    s_ctx = clamp_len(p.dst.lens[b], p.dst.cap);
  }
  __syncthreads();
  const int rows = s_rows, ctx = s_ctx;
  const int writable = max(0, min(rows, p.dst.cap - ctx));
  const int per_row = p.d / 8;
  const int per = writable * p.hkv * per_row;  // a multiple of 4: quads are whole
  for (int u = tid; u < 2 * per; u += kCommitThreads) {
    const bool v_side = u >= per;
    const int w = v_side ? u - per : u;
    const int part = w % per_row, g = (w / per_row) % p.hkv, i = w / (per_row * p.hkv);
    float x[8];
    load8<BF16>(v_side ? p.v_new : p.k_new, (((size_t)b * p.n + s_node[i]) * p.hkv + g) * p.d + 8 * part, x);
    unsigned scale;
    const unsigned c = encode8(x, scale);
    const size_t to = ((size_t)b * p.hkv + g) * p.dst.cap + ctx + i;
    *reinterpret_cast<unsigned*>((v_side ? p.dst.v : p.dst.k) + to * (p.d / 2) + 4 * part) = c;
    if (part % 4 == 0) (v_side ? p.dst.v_scale : p.dst.k_scale)[to * (p.d / 32) + part / 4] = (unsigned char)scale;
  }
  __syncthreads();
  if (tid == 0) p.dst.lens[b] = min(ctx + rows, p.dst.cap);
}

}  // namespace

hipError_t launch_cache_convert(const CacheParams& p, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  const int rows = p.src.cap < p.dst.cap ? p.src.cap : p.dst.cap;
  const long long units = (long long)rows * (p.d / 8);
  const long long chunks = (units + kConvertThreads - 1) / kConvertThreads;
  const dim3 grid((unsigned)(chunks > 0 ? chunks : 1), (unsigned)p.hkv, (unsigned)(2 * p.batch)), block(kConvertThreads);
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.dst.kv4) {
    if (p.bf16) hipLaunchKernelGGL((convert_kernel<true, true>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((convert_kernel<false, true>), grid, block, 0, s, p);
  } else {
    if (p.bf16) hipLaunchKernelGGL((convert_kernel<true, false>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((convert_kernel<false, false>), grid, block, 0, s, p);
  }
  const hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

hipError_t launch_commit_kv4(const CommitKv4Params& p, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.bf16) hipLaunchKernelGGL(commit_kv4_kernel<true>, dim3((unsigned)p.batch), dim3(kCommitThreads), 0, s, p);
  else hipLaunchKernelGGL(commit_kv4_kernel<false>, dim3((unsigned)p.batch), dim3(kCommitThreads), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
