// Attention weight accumulated per context slot.
//
// For slot j of a (sequence, KV head)
//   out[j] = decay w[j] + sum over the rows r that see j of exp(scale q_r . k_j - lse_r),
// rows being (new row, query head of the group) pairs: all of a block's, or those
// of an accepted path.  The scores are formed again from the queries, the keys
// and the call's log-sum-exps; with those known a slot's sum needs no other
// slot, so every tile of 32 KB keys belongs to one wave, which walks all rows:
// no second pass, no atomics, the same bits every time.
//
// Work.  The context tiles of 64 keys that some row sees are cut into pieces of
// equal size by the attention's plan (attn_plan.h), a workgroup each, whose waves
// take its tiles in turn; slots that no row sees only fade, and the pieces of
// their sequence share them.  The queries of up to kRows rows are staged in LDS
// once a workgroup (more rows: in turn, the sums added up in the output), a
// tile's keys are loaded into registers while the tile before is computed.
//
// S[row][key] = Q . K^T with the rows as matrix operand A: a lane's results are
// 16 rows of one key, so the sums over rows are sums over a lane's registers
// (with the keys as A they would be sums over lanes, 31 exchanges a tile).
#include "glance_internal.h"

#include <type_traits>

#include "attn_plan.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) int i32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kWeighWaves = 4;
constexpr float kLog2e = 1.4426950408889634f;

// A lane's half of one row (a key or a query) as matrix operands: bf16 D / 16
// steps of 8 dims, fp32 D / 8 quads of dims.  Of a 4-bit cache a lane takes D / 2
// consecutive dims (the queries alike), otherwise the dims alternate between
// the halves, so that the two lanes of a row read neighbouring bytes.
template <int D, bool BF16, bool KV4>
struct Operand {
  using T = std::conditional_t<BF16, __bf16, float>;
  using Part = std::conditional_t<BF16, bf16x8, f32x4>;  // 16 bytes
  static constexpr int W = BF16 ? 8 : 4;                 // dims of a part
  static constexpr int N = D / (2 * W);                  // parts of a lane
  Part x[N];
  static __device__ __forceinline__ int part(int h, int i) { return KV4 ? h * N + i : 2 * i + h; }
  __device__ __forceinline__ void load(const void* row, int h) {
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = static_cast<const Part*>(row)[part(h, i)];
  }
};

// A lane's codes of a key's half: D / 4 bytes, and the scales of its D / 64 blocks.
template <int D>
struct Codes {
  u32x4 c[D / 64];
  unsigned scale[D / 64];
  __device__ __forceinline__ void load(const unsigned char* codes, const unsigned char* scales, size_t row, int h) {
    const u32x4* p = reinterpret_cast<const u32x4*>(codes + row * (D / 2) + h * (D / 4));
    const unsigned char* s = scales + row * (D / 32) + h * (D / 64);
#pragma unroll
    for (int i = 0; i < D / 64; ++i) {
      c[i] = p[i];
      scale[i] = s[i];
    }
  }
  template <bool BF16>
  __device__ __forceinline__ void values(Operand<D, BF16, true>& k) const {
#pragma unroll
    for (int w = 0; w < D / 16; ++w) {  // eight dims
      const unsigned code = c[w / 4][w % 4];
      const float f = __builtin_bit_cast(float, scale[w / 4] << 23);
      if constexpr (BF16) {
        const u32x4 v = {__builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 0)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 1)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 2)),
                         __builtin_bit_cast(unsigned, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(code, f, 3))};
        k.x[w] = __builtin_bit_cast(bf16x8, v);
      } else {
        const f32x2 a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 0);
        const f32x2 b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 1);
        const f32x2 e = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 2);
        const f32x2 g = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, f, 3);
        k.x[2 * w] = f32x4{a[0], a[1], b[0], b[1]};
        k.x[2 * w + 1] = f32x4{e[0], e[1], g[0], g[1]};
      }
    }
  }
};

template <int D, bool BF16, bool KV4>
__device__ __forceinline__ f32x16 scores(const Operand<D, BF16, KV4>& q, const Operand<D, BF16, KV4>& k) {
  f32x16 s = {};
  if constexpr (BF16) {
#pragma unroll
    for (int i = 0; i < D / 16; ++i) s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q.x[i], k.x[i], s, 0, 0, 0);
  } else {
#pragma unroll
    for (int i = 0; i < D / 8; ++i)
#pragma unroll
      for (int u = 0; u < 4; ++u) s = __builtin_amdgcn_mfma_f32_32x32x2f32(q.x[i][u], k.x[i][u], s, 0, 0, 0);
  }
  return s;
}

template <int D, bool BF16, bool KV4>
__global__ __launch_bounds__(64 * kWeighWaves, 2) void weigh_kernel(WeighParams p) {
  using Op = Operand<D, BF16, KV4>;
  constexpr int KB = BF16 ? 2 : 1;                         // 32-key blocks of a wave at a time
  constexpr int RB = D * (BF16 ? 2 : 4), CH = RB / 16;     // bytes and 16-byte chunks of a query
  constexpr int kRows = 65536 / RB < 256 ? 65536 / RB : 256;  // queries in LDS
  __shared__ __attribute__((aligned(16))) u32x4 sQ[kRows * CH];
  __shared__ __attribute__((aligned(16))) float sOff[kRows];  // -lse in log2 units, -inf for padding rows
  __shared__ __attribute__((aligned(16))) int sPlace[kRows];  // the row's place: position ctx + place
  __shared__ int sNode[64];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const AttnParams& plan = p.plan;
  const int g = blockIdx.x / plan.slots_per_g;
  Piece pc;
  if (!find_piece<true>(plan, blockIdx.x - g * plan.slots_per_g, lane, pc)) return;
  const int b = pc.b, ctx = pc.ctx;
  const TileMap tm = tile_map<64>(plan, ctx);
  const size_t head = (size_t)b * p.hkv + g;
  const float* old = p.cache.weights + head * p.cache.cap;  // (not read where decay is 0)
  float* out = p.out + head * p.cache.cap;
  const bool path = p.accept_path != nullptr;

  // the rows: all new rows, or the path's nodes up to the first invalid entry
  int rows = p.n, node = lane;
  if (path) {
    const int a = p.accept_len[b];
    const int want = max(0, min(min(a >= 64 ? 64 : a + 1, p.path_stride), p.n));
    node = lane < want ? p.accept_path[(size_t)b * p.path_stride + lane] : -1;
    const unsigned long long bad = __ballot(node < 0 || node >= p.n);
    rows = bad ? (int)__builtin_ctzll(bad) : 64;
  }
  if (wave == 0) sNode[lane] = node;

  // slots that no row sees, the pieces of the sequence a share each
  {
    const int first = min(ctx, 64 * tm.head), gap = min(ctx, 64 * (tm.head + tm.skip)) - first;
    const int from = first + (int)((long long)gap * pc.index / pc.count);
    const int to = first + (int)((long long)gap * (pc.index + 1) / pc.count);
    for (int j = from + tid; j < to; j += 64 * kWeighWaves) out[j] = p.decay > 0.f ? p.decay * old[j] : 0.f;
  }

  // This wave's steps: blocks of 32 KB keys of the piece, in turn.  A step's keys are
  // context slots, or in the tile behind them the path's own rows.
  constexpr int KEYS = 32 * KB, SPT = 64 / KEYS;  // steps of a tile
  const int r32 = lane & 31, h = lane >> 5;
  struct Step {
    bool is_new;
    int key0, end;  // first key and the keys there are
  };
  const int n_steps = pc.n_tiles * SPT;
  auto step_at = [&](int s) __attribute__((always_inline)) {
    const int j = pc.t_begin + s / SPT;
    Step o;
    o.is_new = j == tm.n;
    o.key0 = (o.is_new ? 0 : 64 * tm.at(j)) + (s % SPT) * KEYS;
    o.end = o.is_new ? (path ? rows : 0) : ctx;
    return o;
  };
  // The next step's keys, or their codes (with codes the path's own keys are
  // loaded where they are used).
  std::conditional_t<KV4, Codes<D>, Op> next[KB];
  auto key_row = [&](const Step& s, int kb) __attribute__((always_inline)) {  // past the end: any valid row
    return min(s.key0 + 32 * kb + r32, s.end - 1);
  };
  auto new_key = [&](const Step& s, int kb) __attribute__((always_inline)) {
    const int n = __shfl(node, key_row(s, kb));
    return static_cast<const char*>(p.k_new) + (((size_t)b * p.n + n) * p.hkv + g) * RB;
  };
  auto load = [&](const Step& s) __attribute__((always_inline)) {
    if (s.key0 >= s.end || (KV4 && s.is_new)) return;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const size_t row = head * p.cache.cap + key_row(s, kb);
      if constexpr (KV4) next[kb].load(p.cache.k, p.cache.k_scale, row, h);
      else if (s.is_new) next[kb].load(new_key(s, kb), h);
      else next[kb].load(p.cache.k + row * RB, h);
    }
  };
  if (wave < n_steps) load(step_at(wave));

  const int total = rows * p.group;
  // 16-byte chunk c of query r in LDS: rows 16 apart share banks
  auto chunk = [](int r, int c) __attribute__((always_inline)) {
    return r * CH + (CH >= 16 ? c ^ (r & 15) : c ^ ((r >> 1) & 7));
  };
  for (int r0 = 0; r0 == 0 || r0 < total; r0 += kRows) {
    const int n_rows = min(kRows, total - r0);
    const int padded = (n_rows + 31) / 32 * 32;
    __syncthreads();  // sNode is written; the queries before are no longer read
    for (int u = tid; u < padded * CH; u += 64 * kWeighWaves) {
      const int r = u / CH, c = u % CH;
      u32x4 v = {};
      if (r < n_rows) {
        const int i = (r0 + r) / p.group;
        const size_t at = ((size_t)b * p.n + sNode[i]) * p.hq + (size_t)g * p.group + (r0 + r - i * p.group);
        v = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.q) + at * RB + 16 * c);
        if (c == 0) {
          sOff[r] = -p.lse[at] * kLog2e;
          sPlace[r] = i;
        }
      } else if (c == 0) {
        sOff[r] = -__builtin_inff();
        sPlace[r] = 0;
      }
      sQ[chunk(r, c)] = v;
    }
    __syncthreads();
    for (int s = wave; s < n_steps; s += kWeighWaves) {
      const Step st = step_at(s);
      Op k[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if constexpr (KV4) {
          if (!st.is_new) next[kb].template values<BF16>(k[kb]);
          else if (st.key0 < st.end) k[kb].load(new_key(st, kb), h);
        } else {
          k[kb] = next[kb];
        }
      }
      // the next step's keys, past the last one the first's for the next rows
      if (s + kWeighWaves < n_steps) load(step_at(s + kWeighWaves));
      else if (r0 + kRows < total) load(step_at(wave));
      if (st.key0 >= st.end) continue;
      // the places of the rows that see the lane's key of each block
      int from[KB], to[KB];
      bool all = !st.is_new;
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        const int key = st.key0 + 32 * kb + r32;
        const int slot = st.is_new ? ctx + key : key;
        from[kb] = st.is_new ? key : 0;
        const long long last = (long long)slot - ctx + p.plan.window - 1;
        to[kb] = slot < p.plan.n_sinks || last > 64 ? 64 : (int)last;
      }
      all = all && (st.key0 + KEYS <= p.plan.n_sinks || st.key0 >= ctx + rows - p.plan.window);
      float sum[KB][2] = {};
      for (int rt = 0; rt < padded; rt += 32) {
        Op q;
#pragma unroll
        for (int i = 0; i < Op::N; ++i) q.x[i] = __builtin_bit_cast(typename Op::Part, sQ[chunk(rt + r32, Op::part(h, i))]);
        f32x4 off[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) off[x] = *reinterpret_cast<const f32x4*>(&sOff[rt + 8 * x + 4 * h]);
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
          const f32x16 z = scores<D, BF16, KV4>(q, k[kb]);
          if (all) {
#pragma unroll
            for (int x = 0; x < 16; ++x)
              sum[kb][x & 1] += __builtin_amdgcn_exp2f(fmaf(z[x], p.scale_log2, off[x >> 2][x & 3]));
          } else {
#pragma unroll
            for (int x = 0; x < 16; ++x) {
              const int place = sPlace[rt + 8 * (x >> 2) + 4 * h + (x & 3)];
              const float e = __builtin_amdgcn_exp2f(fmaf(z[x], p.scale_log2, off[x >> 2][x & 3]));
              sum[kb][x & 1] += place >= from[kb] && place <= to[kb] ? e : 0.f;
            }
          }
        }
      }
      // both halves of a key's rows; with two blocks each half stores one
      float w;
      int key = st.key0 + r32;
      if constexpr (KB == 2) {
        const float a = sum[0][0] + sum[0][1], c = sum[1][0] + sum[1][1];
        w = (h ? c : a) + __shfl_xor(h ? a : c, 32);
        key += 32 * h;
      } else {
        w = sum[0][0] + sum[0][1];
        w += __shfl_xor(w, 32);
        if (h) continue;
      }
      if (key >= st.end) continue;
      const int slot = st.is_new ? ctx + key : key;
      if (slot >= p.cache.cap) continue;
      if (r0 > 0) w += out[slot];
      else if (!st.is_new && p.decay > 0.f) w = fmaf(p.decay, old[slot], w);
      out[slot] = w;
    }
  }
}

template <int D, bool BF16>
void launch(const WeighParams& p, hipStream_t s) {
  const dim3 grid((unsigned)(p.plan.slots_per_g * p.hkv)), block(64 * kWeighWaves);
  if (p.cache.kv4) hipLaunchKernelGGL((weigh_kernel<D, BF16, true>), grid, block, 0, s, p);
  else hipLaunchKernelGGL((weigh_kernel<D, BF16, false>), grid, block, 0, s, p);
}

}  // namespace

hipError_t launch_weigh(const WeighParams& params, bool bf16, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  // two workgroups a compute unit, a tile a wave at least
  WeighParams p = params;
  p.plan = {};
  p.plan.batch = p.batch;
  p.plan.cap = p.cache.cap;
  p.plan.ctx_lens = p.cache.lens;
  p.plan.n_sinks = p.n_sinks;
  p.plan.window = p.window;
  const int per_g = 512 / p.hkv;
  p.plan.slots_per_g = per_g > p.batch ? per_g : p.batch;
  p.plan.min_tiles = kWeighWaves;
  p.plan.tiles_rg = 5;  // (least_piece: no more than four)
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
