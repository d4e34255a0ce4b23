// Attention weight accumulated per context slot.
//
// For slot j of a (sequence, KV head)
//   out[j] = decay w[j] + sum over the rows r that see j of exp(scale q_r . k_j - lse_r),
// rows being (new row, query head of the group) pairs: all of a block's, or those
// of an accepted path.  The scores are formed again from the queries, the keys
// and the call's log-sum-exps; with those known a slot's sum needs no other
// slot, so every tile of keys belongs to one wave, which walks all rows: no
// second pass, no atomics, the same bits every time.
//
// A wave holds 32 KB keys as matrix operand A and takes the rows in tiles of 32
// as B, S^T[key][row] = K . Q^T: a lane's results are 16 keys of one row, so
// the row's log-sum-exp is one register and the sums over rows stay in 16 KB
// registers, folded across lanes once at the end.
#include "glance_internal.h"

#include <type_traits>

#include "attn_plan.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kWeighWaves = 4;

// Matrix operands of a 32-row tile (keys or queries), a lane's half of one row.
// bf16: D / 16 steps of 8 dims; fp32: D / 8 quads of dims.  Of a 4-bit cache a
// lane takes D / 2 consecutive dims (so do the queries), otherwise the dims
// alternate between the halves: the two lanes of a row read neighbouring bytes.
template <int D, bool BF16, bool KV4>
struct Operand {
  static constexpr int N = BF16 ? D / 16 : D / 8;
  using Part = std::conditional_t<BF16, bf16x8, f32x4>;
  Part x[N];
  static constexpr int W = BF16 ? 8 : 4;  // dims of a part
  static __device__ __forceinline__ int dim(int h, int i) { return KV4 ? h * (D / 2) + W * i : 2 * W * i + W * h; }
  __device__ __forceinline__ void load(const void* base, size_t row, int h) {
    using T = std::conditional_t<BF16, __bf16, float>;
    const T* p = static_cast<const T*>(base) + row * D;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = *reinterpret_cast<const Part*>(p + dim(h, i));
  }
  __device__ __forceinline__ void load_codes(const unsigned char* codes, const unsigned char* scales, size_t row, int h) {
    const unsigned* c = reinterpret_cast<const unsigned*>(codes + row * (D / 2) + h * (D / 4));
    const unsigned char* s = scales + row * (D / 32) + h * (D / 64);
#pragma unroll
    for (int w = 0; w < D / 16; ++w) {  // eight dims
      const unsigned code = c[w];
      const float f = __builtin_bit_cast(float, (unsigned)s[w / 4] << 23);
      if constexpr (BF16) {
        const u32x4 v = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 0)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 1)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 2)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 3))};
        x[w] = __builtin_bit_cast(bf16x8, v);
      } else {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 1);
        const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 2);
        const f32x2 g = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 3);
        x[2 * w] = f32x4{a[0], a[1], b[0], b[1]};
        x[2 * w + 1] = f32x4{e[0], e[1], g[0], g[1]};
      }
    }
  }
};

template <int D, bool BF16, bool KV4>
__device__ __forceinline__ f32x16 scores(const Operand<D, BF16, KV4>& k, const Operand<D, BF16, KV4>& q) {
  f32x16 s = {};
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.x[i], q.x[i], s, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(k.x[i][u], q.x[i][u], s, 0, 0, 0);
  }
  return s;
}

// Grid (key tiles of a head's capacity, KV heads, sequences); with a path, one
// more workgroup for the path's own keys, whose slots follow the context.
template <int D, bool BF16, bool KV4>
__global__ __launch_bounds__(64 * kWeighWaves) void weigh_kernel(WeighParams p) {
  constexpr int KB = BF16 ? 2 : 1;     // 32-key blocks of a wave
  constexpr int KEYS = 32 * KB;        // keys of a wave
  constexpr int NV = 16 * KB;
  constexpr float kLog2e = 1.4426950408889634f;
  using Op = Operand<D, BF16, KV4>;
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.z, g = blockIdx.y;
  const int ctx = clamp_ctx(p.cache.lens[b], p.cache.cap);
  const bool path = p.accept_path != nullptr;
  const bool is_new = path && blockIdx.x == gridDim.x - 1;
  const int key0 = ((is_new ? 0 : (int)blockIdx.x * kWeighWaves) + wave) * KEYS;  // slot, or path row

  // the rows: all new rows, or the path's nodes up to the first invalid entry
  int rows = p.n, node = lane;
  if (path) {
    const int a = p.accept_len[b];
    const int want = max(0, min(min(a >= 64 ? 64 : a + 1, p.path_stride), p.n));
    node = lane < want ? p.accept_path[(size_t)b * p.path_stride + lane] : -1;
    const unsigned long long bad = __ballot(node < 0 || node >= p.n);
    rows = bad ? (int)__builtin_ctzll(bad) : 64;
  }
  const int end = is_new ? rows : ctx;
  if (key0 >= end) return;

  const int r32 = lane & 31, h = lane >> 5;
  const size_t head = (size_t)b * p.hkv + g;
  // context keys that no row sees (outside row 0's window and the sinks) only fade
  const int lo = max(0, ctx - p.window + 1);
  const bool seen = is_new || key0 < min(p.n_sinks, ctx) || key0 + KEYS > lo;
  float sum[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) sum[i] = 0.f;
  if (seen) {
    Op k[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int key = min(key0 + 32 * kb + r32, end - 1);  // past the end: any valid row
      if (is_new) k[kb].load(p.k_new, ((size_t)b * p.n + __shfl(node, key)) * p.hkv + g, h);
      else if constexpr (KV4) k[kb].load_codes(p.cache.k, p.cache.k_scale, head * p.cache.cap + key, h);
      else k[kb].load(p.cache.k, head * p.cache.cap + key, h);
    }
    const int total = rows * p.group;
    for (int r0 = 0; r0 < total; r0 += 32) {
      const int r = min(r0 + r32, total - 1);
      const int i = r / p.group;  // the row's place: position ctx + i
      const size_t at = ((size_t)b * p.n + (path ? __shfl(node, i) : i)) * p.hq + (size_t)g * p.group + (r - i * p.group);
      const float off = r0 + r32 < total ? -p.lse[at] * kLog2e : -__builtin_inff();
      Op q;
      q.load(p.q, at, h);
      // bit x: the row sees key0 + x
      unsigned long long vis = ~0ull;
      if (is_new) vis = bits_below(i + 1 - key0) & (window_word(p.n_sinks - ctx, i - p.window + 1, key0));
      else if (key0 + KEYS > p.n_sinks && key0 < ctx + rows - p.window)
        vis = window_word(p.n_sinks, ctx + i - p.window + 1, key0);
      vis >>= 4 * h;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const f32x16 s = scores<D, BF16, KV4>(k[kb], q);
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const float e = __builtin_amdgcn_exp2f(fmaf(s[x], p.scale_log2, off));
          sum[16 * kb + x] += (vis >> (32 * kb + 8 * (x >> 2) + (x & 3))) & 1ull ? e : 0.f;
        }
      }
    }
  }
  // Fold over the 32 lanes of a half: in each step a lane keeps the half of its
  // sums that its lane bit names and gets the partner's, until one is left (for
  // one block of 32 keys the last step adds pairs).
  int mine = 0, left = NV;
#pragma unroll
  for (int bit = 16; bit >= 1; bit >>= 1) {
    if (left > 1) {
      left /= 2;
      const bool up = r32 & bit;
#pragma unroll
      for (int x = 0; x < NV / 2; ++x)
        if (x < left) {
          const float keep = up ? sum[x + left] : sum[x], give = up ? sum[x] : sum[x + left];
          sum[x] = keep + __shfl_xor(give, bit);
        }
      mine += up ? left : 0;
    } else {
      sum[0] += __shfl_xor(sum[0], bit);
    }
  }
  const int key = key0 + 32 * (mine >> 4) + 8 * ((mine & 15) >> 2) + 4 * h + (mine & 3);
  if (key >= end || (KB == 1 && (r32 & 1))) return;
  float* out = p.out + head * p.cache.cap;
  if (is_new) {
    if (ctx + key < p.cache.cap) out[ctx + key] = sum[0];
  } else {
    const float old = p.decay > 0.f ? p.decay * p.cache.weights[head * p.cache.cap + key] : 0.f;
    out[key] = old + sum[0];
  }
}

template <int D, bool BF16>
void launch(const WeighParams& p, hipStream_t s) {
  const int keys = kWeighWaves * (BF16 ? 64 : 32);
  const int tiles = (p.cache.cap + keys - 1) / keys + (p.accept_path ? 1 : 0);
  const dim3 grid((unsigned)tiles, (unsigned)p.hkv, (unsigned)p.batch), block(64 * kWeighWaves);
  if (p.cache.kv4) hipLaunchKernelGGL((weigh_kernel<D, BF16, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((weigh_kernel<D, BF16, false>), grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_weigh(const WeighParams& p, bool bf16, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  if (ev0) (void)hipEventRecord(ev0, s);
  if (p.d == 128) {
    if (bf16) launch<128, true>(p, s);
    else launch<128, false>(p, s);
  } else {
    if (bf16) launch<64, true>(p, s);
    else launch<64, false>(p, s);
  }
  const hipError_t e = hipGetLastError();
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
