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
// scales): into 4 bits 38.5 us, 4.4 TB/s, and back 25.5, 6.7 TB/s.
#include "glance_internal.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(2))) unsigned short u16x2;

__device__ __forceinline__ int clamp_len(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }

// Eight values of a row, as they lie in memory.
template <bool BF16>
struct Eight {
  u32x4 w[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* at) {
#pragma unroll
    for (int i = 0; i < (BF16 ? 1 : 2); ++i) w[i] = static_cast<const u32x4*>(at)[i];
  }
  // Bits (as fp32) of the largest magnitude; NaN and infinity are larger than any.
  __device__ __forceinline__ unsigned largest() const {
    if constexpr (BF16) {
      u16x2 m = {};
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w[0][i] & 0x7fff7fffu));
      return (unsigned)(m[0] > m[1] ? m[0] : m[1]) << 16;
    } else {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned a = w[i / 4][i % 4] & 0x7fffffffu;
        m = m > a ? m : a;
      }
      return m;
    }
  }
  // Their codes at a scale.  (The words are copied first: a bit cast of a vector's
  // element is built as one of its first element.)
  __device__ __forceinline__ unsigned codes(float s) const {
    unsigned c = 0;
    if constexpr (BF16) {
      const unsigned v0 = w[0][0], v1 = w[0][1], v2 = w[0][2], v3 = w[0][3];
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v0), s, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v1), s, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v2), s, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2, v3), s, 3);
    } else {
      float f[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned v = w[i / 4][i % 4];
        f[i] = __builtin_bit_cast(float, v);
      }
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[0], f[1], s, 0);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[2], f[3], s, 1);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[4], f[5], s, 2);
      c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, f[6], f[7], s, 3);
    }
    return c;
  }
};

// The larger of a lane's value and its neighbour's; the four lanes of a block
// are one quad.
template <int CTRL>
__device__ __forceinline__ unsigned quad_max(unsigned v) {
  const unsigned o = (unsigned)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xf, 0xf, false);
  return v > o ? v : o;
}

// Codes of a lane's eight values and the block's exponent byte (every lane of
// the quad takes part).
template <bool BF16>
__device__ __forceinline__ unsigned encode8(const Eight<BF16>& x, unsigned& scale) {
  unsigned m = x.largest();
  m = quad_max<0xb1>(m);  // quad_perm [1,0,3,2]
  m = quad_max<0x4e>(m);  // quad_perm [2,3,0,1]
  const unsigned e = (m + 0x200000u) >> 23;
  scale = m >= 0x7f800000u ? 255u : min(max(e, 4u), 254u) - 2u;
  return x.codes(__builtin_bit_cast(float, scale << 23));
}

constexpr int kConvertThreads = 256;
constexpr int kConvertUnits = 4;  // groups of eight values of a thread, in flight at once

// Grid (chunks of a head's rows, KV heads, 2 batch: keys and values).  A chunk's
// rows follow one another, so a group's place is its number within the chunk
// behind a uniform address (one group a thread and addresses of 64 bits a lane:
// both ways below together 65.6 us instead of 64.2).
template <bool BF16, bool PACK>
__global__ __launch_bounds__(kConvertThreads) void convert_kernel(CacheParams p) {
  const int b = blockIdx.z >> 1, g = blockIdx.y;
  const bool v_side = blockIdx.z & 1;
  const int len = min(clamp_len(p.src.lens[b], p.src.cap), p.dst.cap);
  if (blockIdx.x == 0 && g == 0 && !v_side && threadIdx.x == 0) p.dst.lens[b] = len;
  const int shift = __builtin_ctz((unsigned)p.d / 8);  // groups of a row, 8 or 16: a row's quads stay in one wave
  const int row0 = (int)(blockIdx.x * (kConvertUnits * kConvertThreads)) >> shift;
  if (row0 >= len) return;
  const int units = (len - row0) << shift;  // groups from here on (fewer than 2^30)
  const size_t head = (size_t)b * p.hkv + g;
  const size_t from = (head * p.src.cap + row0) * p.d, to = (head * p.dst.cap + row0) * p.d;  // values
  const unsigned char* src = v_side ? p.src.v : p.src.k;
  unsigned char* dst = v_side ? p.dst.v : p.dst.k;
  // (groups past the last repeat it and are not stored)
  if constexpr (PACK) {
    constexpr int kBytes = BF16 ? 16 : 32;
    const unsigned char* in = src + from * (kBytes / 8);
    unsigned* out = reinterpret_cast<unsigned*>(dst + to / 2);
    unsigned char* scales = (v_side ? p.dst.v_scale : p.dst.k_scale) + to / 32;
    Eight<BF16> x[kConvertUnits];
#pragma unroll
    for (int i = 0; i < kConvertUnits; ++i) {
      const unsigned u = (unsigned)min(i * kConvertThreads + (int)threadIdx.x, units - 1);
      x[i].load(in + u * kBytes);
    }
#pragma unroll
    for (int i = 0; i < kConvertUnits; ++i) {
      const unsigned u = i * kConvertThreads + threadIdx.x;
      unsigned scale;
      const unsigned c = encode8(x[i], scale);
      if ((int)u >= units) continue;
      out[u] = c;
      if (u % 4 == 0) scales[u / 4] = (unsigned char)scale;
    }
  } else {
    const unsigned* in = reinterpret_cast<const unsigned*>(src + from / 2);
    const unsigned char* scales = (v_side ? p.src.v_scale : p.src.k_scale) + from / 32;
    unsigned c[kConvertUnits], e[kConvertUnits];
#pragma unroll
    for (int i = 0; i < kConvertUnits; ++i) {
      const unsigned u = (unsigned)min(i * kConvertThreads + (int)threadIdx.x, units - 1);
      c[i] = in[u];
      e[i] = scales[u / 4];
    }
#pragma unroll
    for (int i = 0; i < kConvertUnits; ++i) {
      const unsigned u = i * kConvertThreads + threadIdx.x;
      if ((int)u >= units) continue;
      const float s = __builtin_bit_cast(float, e[i] << 23);
      if constexpr (BF16) {
        const u32x4 w = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 0)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 1)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 2)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(c[i], s, 3))};
        *reinterpret_cast<u32x4*>(dst + to * 2 + u * 16) = w;
      } else {
        f32x4* o = reinterpret_cast<f32x4*>(dst + to * 4 + u * 32);
        const f32x2 v0 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 0), v1 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 1);
        const f32x2 v2 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 2), v3 = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(c[i], s, 3);
        o[0] = f32x4{v0[0], v0[1], v1[0], v1[1]};
        o[1] = f32x4{v2[0], v2[1], v3[0], v3[1]};
      }
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
    Eight<BF16> x;
    x.load(static_cast<const char*>(v_side ? p.v_new : p.k_new) +
           ((((size_t)b * p.n + s_node[i]) * p.hkv + g) * p.d + 8 * part) * (BF16 ? 2 : 4));
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
  const int rows_wg = kConvertUnits * kConvertThreads / (p.d / 8);
  const int chunks = (rows + rows_wg - 1) / rows_wg;
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
