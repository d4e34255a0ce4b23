// Attention weight accumulated per context slot.
//
// For slot j of a (sequence, KV head)
//   out[j] = decay w[j] + sum over the rows r that see j of exp(scale q_r . k_j - lse_r),
// rows being (new row, query head of the group) pairs: all of a block's, or those
// of an accepted path.  The scores are formed again from the queries, the keys
// and the call's log-sum-exps; with those known a slot's sum needs no other
// slot, so every tile of 32 KB keys belongs to one wave, which walks the rows: no
// atomics, the same bits every time, and one pass over the keys where the rows
// fit LDS (below).
//
// Work.  The context tiles of 64 keys that some row sees are cut into pieces by
// the attention's plan (attn_plan.h; equal within a sequence, and over 16 ragged
// contexts of 2048 to 32768 keys at most 78 tiles, 70 on average), a workgroup
// each, about one a compute unit; its waves take the piece's tiles as they become
// free (a wave that shares its SIMD with an older one gets two thirds of its
// turns).  Slots that no row sees only fade, and the pieces of their sequence share
// them.  The queries of up to kRows rows, 256 or, in fp32 with 128 dims, 128, are
// staged in LDS; more rows come in turn, for which the keys are read, converted
// and the sums read back again (64 rows of 7 heads over 4 x 16384 bf16 keys: two
// turns, 50 us; over 4-bit keys 38).  A tile's keys are loaded into registers while
// the tile before is computed.
//
// S[row][key] = Q . K^T with the rows as matrix operand A: a lane's results are
// 16 rows of one key, so the sums over rows are sums over a lane's registers
// (with the keys as A they would be sums over lanes, 31 exchanges a tile).
//
// fp32 products, exponentials and sums; of bf16 and 4-bit caches the products are
// exact and summed in fp32 by the matrix unit.
//
// Bound by the read of the keys where the rows are few: about 10 path nodes of 7
// heads over 4 caches of 16384 bf16 keys and 4 heads of 128 (67 MB) take 21.5 us,
// 13.8 at the rate of a large copy, of which 4 are the chain of loads from the
// lengths to the first key (asked for only once the path was known, and with a
// dozen spilled addresses: 24.7).  With
// more rows by vector instructions, an exponential, a multiply-add and an addition
// a score: 16 rows of 7 heads over 16 ragged caches of 2048 to 32768 4-bit keys
// take 47 to 50 us, 26 at the rate of a large matrix product.
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

constexpr int kWeighWaves = 8;
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
  static constexpr int kRow = D * (BF16 ? 2 : 4);  // bytes of a row
  static __device__ __forceinline__ unsigned lane_offset(int row, int h) { return row * kRow + 16 * part(h, 0); }
  // from a uniform address and lane_offset()
  __device__ __forceinline__ void load(const void* base, unsigned off) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      x[i] = *reinterpret_cast<const Part*>(static_cast<const char*>(base) + off + 16 * (KV4 ? i : 2 * i));
  }
};

// A lane's codes of a key's half: D / 4 bytes, and the scales of its D / 64 blocks.
template <int D>
struct Codes {
  u32x4 c[D / 64];
  unsigned scale;
  static __device__ __forceinline__ unsigned lane_offset(int row, int h) { return row * (D / 2) + h * (D / 4); }
  static __device__ __forceinline__ unsigned lane_scale(int row, int h) { return row * (D / 32) + h * (D / 64); }
  __device__ __forceinline__ void load(const unsigned char* codes, const unsigned char* scales, unsigned off, unsigned soff) {
#pragma unroll
    for (int i = 0; i < D / 64; ++i) c[i] = *reinterpret_cast<const u32x4*>(codes + off + 16 * i);
    if constexpr (D == 128) scale = *reinterpret_cast<const unsigned short*>(scales + soff);
    else scale = scales[soff];
  }
  template <bool BF16>
  __device__ __forceinline__ void values(Operand<D, BF16, true>& k) const {
#pragma unroll
    for (int w = 0; w < D / 16; ++w) {  // eight dims
      const unsigned code = c[w / 4][w % 4];
      const float f = __builtin_bit_cast(float, (scale >> (8 * (w / 4)) & 255u) << 23);
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
  using Next = std::conditional_t<KV4, Codes<D>, Op>;
  constexpr int KB = BF16 ? 2 : 1;                     // 32-key blocks of a wave at a time
  constexpr int RB = Op::kRow, CH = RB / 16;           // bytes and 16-byte chunks of a query
  constexpr int LB = RB + 16;  // ... and its stride in LDS: 16 rows at one chunk lie in 16 different bank groups
  constexpr int kRows = 65536 / RB < 256 ? 65536 / RB : 256;  // queries in LDS
  __shared__ __attribute__((aligned(16))) char sQ[kRows * LB];
  __shared__ __attribute__((aligned(16))) float sOff[kRows];  // -lse in log2 units, -inf for padding rows
  __shared__ __attribute__((aligned(16))) int sPlace[kRows];  // the row's place: position ctx + place
  __shared__ int sRow[kRows];                                 // its query, -1 for padding rows
  __shared__ int sTicket;
  __shared__ float sPart[64 * kWeighWaves];  // sums of a step's parts

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
  // Steps: blocks of 32 KB keys of the piece.  A step's keys are context slots,
  // or in the tile behind them the path's own rows.
  constexpr int KEYS = 32 * KB, SPT = 64 / KEYS;  // steps of a tile
  const int r32 = lane & 31, h = lane >> 5;
  struct Step {
    bool is_new;
    int key0, end;  // first key and the keys there are
  };
  const int n_steps = pc.n_tiles * SPT;
  // fp32, whose products take eight times as long: with fewer steps than half the
  // waves `parts` waves share one, a part of the row tiles each, and their sums
  // are added up in order at the end.  64 rows of 12/1 heads over 542 4-bit keys
  // 61.8 -> 41 us, 36 rows of 28/4 heads over a window of 545 24.6 -> 16.9.  (In
  // bf16 the registers do not go round: 47.9 -> 50.4 in the largest calls.)
  const int parts = BF16 || n_steps > 4 ? 1 : n_steps == 1 ? 8 : n_steps == 2 ? 4 : 2;
  const int part = wave % parts, own_step = wave / parts;
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
  Next next[KB];
  auto new_key = [&](const Step& s, int kb, Op& k) __attribute__((always_inline)) {
    const int n = __shfl(node, min(s.key0 + 32 * kb + r32, s.end - 1));
    const char* row = static_cast<const char*>(p.k_new) + (((size_t)b * p.n + n) * p.hkv + g) * RB;
    k.load(row, Op::lane_offset(0, h));
  };
  auto load_context = [&](const Step& s) __attribute__((always_inline)) {
    const size_t row = head * p.cache.cap + s.key0;
    const int last = min(KEYS, s.end - s.key0) - 1;  // >= 0; keys past it are its copies
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      const int r = min(32 * kb + r32, last);
      if constexpr (KV4)
        next[kb].load(p.cache.k + row * (D / 2), p.cache.k_scale + row * (D / 32), Next::lane_offset(r, h), Next::lane_scale(r, h));
      else
        next[kb].load(p.cache.k + row * RB, Next::lane_offset(r, h));
    }
  };
  auto load = [&](const Step& s) __attribute__((always_inline)) {
    if (s.key0 >= s.end) return;
    if (!s.is_new) return load_context(s);
    if constexpr (!KV4) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) new_key(s, kb, next[kb]);
    }
  };

  // Loads go out before the words that only decide what is done with them have
  // come: the path's with its length, then the first step's keys (any valid row
  // where that step has none of the context).
  const int most = min(p.path_stride, p.n);
  int accepted = 0;
  if (path) {
    accepted = p.accept_len[b];
    node = lane < most ? p.accept_path[(size_t)b * p.path_stride + lane] : -1;
  }
  const Step first_step = step_at(min(own_step, n_steps - 1));
  const bool first_held = !first_step.is_new && first_step.key0 < first_step.end;
  load_context(first_held ? first_step : Step{false, 0, 1});
  if (path) {
    const int want = max(0, min(accepted >= 64 ? 64 : accepted + 1, most));
    const unsigned long long bad = __ballot(lane >= want || node < 0 || node >= p.n);
    rows = bad ? (int)__builtin_ctzll(bad) : 64;
  }

  // slots that no row sees, the pieces of the sequence a share each
  constexpr int kThreads = 64 * kWeighWaves;
  {
    const int first = min(ctx, 64 * tm.head), gap = min(ctx, 64 * (tm.head + tm.skip)) - first;
    const int from = first + (int)((long long)gap * pc.index / pc.count);
    const int to = first + (int)((long long)gap * (pc.index + 1) / pc.count);
    for (int j = from + tid; j < to; j += kThreads) out[j] = p.decay > 0.f ? p.decay * old[j] : 0.f;
  }

  const int total = rows * p.group;
  constexpr int kBatch = 4;
  for (int r0 = 0; r0 == 0 || r0 < total; r0 += kRows) {
    const int n_rows = min(kRows, total - r0);
    const int padded = (n_rows + 31) / 32 * 32;
    if (r0 > 0) __syncthreads();  // the queries before are no longer read
    // The rows' places, a row a thread; then their queries, kBatch 16-byte chunks
    // a thread in flight at once, and behind the first of these (loads arrive in
    // order) the first step's keys, where they are not there yet.
    static_assert(kRows <= kThreads, "a row a thread");
    int t = tid;
    asm volatile("" : "+v"(t));  // addresses made from it here are not kept, spilled, for another turn
    float lse = __builtin_inff();
    {
      const int i = min(r0 + t, max(total - 1, 0)) / p.group;
      const int node_i = path ? __shfl(node, i) : i;
      const int at = (b * p.n + node_i) * p.hq + g * p.group + (r0 + t - i * p.group);
      if (t < n_rows) lse = p.lse[at];
      if (t < kRows) {
        sPlace[t] = i;
        sRow[t] = t < n_rows ? at : -1;
      }
      if (t == 0) sTicket = kWeighWaves;
    }
    __syncthreads();
    int s = own_step;  // the first step; the others by ticket
    for (int u0 = 0; u0 < padded * CH || u0 == 0; u0 += kBatch * kThreads) {
      int row[kBatch];
      u32x4 v[kBatch];
#pragma unroll
      for (int x = 0; x < kBatch; ++x) row[x] = sRow[min((u0 + x * kThreads + t) / CH, kRows - 1)];
#pragma unroll
      for (int x = 0; x < kBatch; ++x)  // (for padding rows any query)
        v[x] = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.q) + (size_t)max(row[x], 0) * RB + 16 * (t % CH));
      if (u0 == 0 && s < n_steps && !(r0 == 0 && first_held)) load(step_at(s));
#pragma unroll
      for (int x = 0; x < kBatch; ++x) {
        const int r = (u0 + x * kThreads + t) / CH;
        if (r < padded) *reinterpret_cast<u32x4*>(sQ + r * LB + 16 * (t % CH)) = row[x] >= 0 ? v[x] : u32x4{};
      }
    }
    static_assert(kThreads % CH == 0, "a thread's chunk of a query is one and the same");
    if (t < kRows) sOff[t] = -lse * kLog2e;
    __syncthreads();
    while (s < n_steps) {
      const Step st = step_at(s);
      Op k[KB];
#pragma unroll
      for (int kb = 0; kb < KB; ++kb) {
        if constexpr (KV4) {
          if (!st.is_new) {
            next[kb].template values<BF16>(k[kb]);
          } else if (st.key0 < st.end) {
            new_key(st, kb, k[kb]);
            // waited for here: otherwise the compiler waits for every load, the
            // next step's too, wherever the keys are used
            __builtin_amdgcn_s_waitcnt(0xf70);  // vmcnt(0)
          }
        } else {
          k[kb] = next[kb];
        }
      }
      // The slot that this lane writes and its old weight (or the sum over the
      // rows before), read ahead of the next step's keys, since loads arrive in
      // order, and by every lane, since a wait stands behind a conditional one.
      const int mine = st.key0 + r32 + (KB == 2 ? 32 * h : 0);
      const int slot = st.is_new ? ctx + mine : mine;
      const bool writes = mine < st.end && slot < p.cache.cap && (KB == 2 || h == 0);
      const float keep = r0 > 0 ? 1.f : st.is_new ? 0.f : p.decay;
      const float before = (r0 > 0 || p.decay == 0.f ? out : old)[min(slot, p.cache.cap - 1)];
      s = n_steps;
      if (parts == 1) {
        int ticket = 0;
        if (lane == 0) ticket = atomicAdd(&sTicket, 1);
        s = __builtin_amdgcn_readfirstlane(ticket);
      }
      if (s < n_steps) load(step_at(s));
      if (st.key0 >= st.end) continue;
      float sum[KB][2] = {};
      // a step whose keys every row sees needs no places
      const bool all = !st.is_new && (st.key0 + KEYS <= p.plan.n_sinks || st.key0 >= ctx + rows - p.plan.window);
      const int rt0 = 32 * part, stride = 32 * parts;  // this wave's row tiles
      auto walk = [&](auto ALL_) __attribute__((always_inline)) {
        constexpr bool ALL = decltype(ALL_)::value;
        int from[KB], to[KB];  // the places of the rows that see the lane's key of each block
        if (!ALL) {
#pragma unroll
          for (int kb = 0; kb < KB; ++kb) {
            const int key = st.key0 + 32 * kb + r32;
            const int at = st.is_new ? ctx + key : key;
            from[kb] = st.is_new ? key : 0;
            const long long last = (long long)at - ctx + p.plan.window - 1;
            to[kb] = at < p.plan.n_sinks || last > 64 ? 64 : (int)last;
          }
        }
        Op q;
        f32x4 off[4];
        const unsigned lane_q = r32 * LB + 16 * Op::part(h, 0);
        auto query = [&](int rt, int i) __attribute__((always_inline)) {
          q.x[i] = *reinterpret_cast<const typename Op::Part*>(sQ + rt * LB + lane_q + 16 * (KV4 ? i : 2 * i));
        };
        auto offset = [&](int rt, int x) __attribute__((always_inline)) {
          off[x] = *reinterpret_cast<const f32x4*>(&sOff[rt + 8 * x + 4 * h]);
        };
        auto add = [&](const f32x16& z, int rt, int kb, int x) __attribute__((always_inline)) {
          float e = __builtin_amdgcn_exp2f(fmaf(z[x], p.scale_log2, off[x >> 2][x & 3]));
          if (!ALL) {
            const int place = sPlace[rt + 8 * (x >> 2) + 4 * h + (x & 3)];
            e = place >= from[kb] && place <= to[kb] ? e : 0.f;
          }
          sum[kb][x & 1] += e;
        };
#pragma unroll
        for (int i = 0; i < Op::N; ++i) query(rt0, i);
#pragma unroll
        for (int x = 0; x < 4; ++x) offset(rt0, x);
        if constexpr (KB == 2) {
          // Matrix and vector instructions in turn: the products of one block
          // between the exponentials of the other, operands reloaded as soon as
          // they are used.  (With the products first and the exponentials behind
          // them the two took turns on the SIMD as well: 62 us instead of 50 for 16
          // rows over 16 ragged caches in 4 bits.)
          constexpr int E = 16 / Op::N;  // exponentials a product
          f32x16 z0 = scores<D, BF16, KV4>(q, k[0]), z1;
          for (int rt = rt0; rt < padded; rt += stride) {
            const int nt = rt + stride < padded ? rt + stride : rt0;
#pragma unroll
            for (int i = 0; i < Op::N; ++i) {
              z1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q.x[i], k[1].x[i], i == 0 ? f32x16{} : z1, 0, 0, 0);
              query(nt, i);
#pragma unroll
              for (int x = E * i; x < E * i + E; ++x) add(z0, rt, 0, x);
              __builtin_amdgcn_sched_barrier(0);
            }
#pragma unroll
            for (int i = 0; i < Op::N; ++i) {
              z0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(q.x[i], k[0].x[i], i == 0 ? f32x16{} : z0, 0, 0, 0);
#pragma unroll
              for (int x = E * i; x < E * i + E; ++x) add(z1, rt, 1, x);
              if (E * i % 4 + E >= 4) offset(nt, E * i / 4);
              __builtin_amdgcn_sched_barrier(0);
            }
          }
        } else {
          for (int rt = rt0; rt < padded; rt += stride) {
            const int nt = rt + stride < padded ? rt + stride : rt0;
            const f32x16 z = scores<D, BF16, KV4>(q, k[0]);
#pragma unroll
            for (int i = 0; i < Op::N; ++i) query(nt, i);
#pragma unroll
            for (int x = 0; x < 16; ++x) add(z, rt, 0, x);
#pragma unroll
            for (int x = 0; x < 4; ++x) offset(nt, x);
          }
        }
      };
      if (rt0 < padded) {
        if (all) walk(std::true_type{});
        else walk(std::false_type{});
      }
      // both halves of a key's rows; with two blocks each half stores one
      float w;
      if constexpr (KB == 2) {
        const float a = sum[0][0] + sum[0][1], c = sum[1][0] + sum[1][1];
        w = (h ? c : a) + __shfl_xor(h ? a : c, 32);
      } else {
        w = sum[0][0] + sum[0][1];
        w += __shfl_xor(w, 32);
      }
      if (parts > 1) sPart[tid] = w;
      else if (writes) out[slot] = keep > 0.f ? fmaf(keep, before, w) : w;
    }
    if (parts > 1) {
      __syncthreads();
      if (part != 0 || own_step >= n_steps) continue;
      const Step st = step_at(own_step);
      const int mine = st.key0 + r32 + (KB == 2 ? 32 * h : 0);
      const int slot = st.is_new ? ctx + mine : mine;
      if (mine >= st.end || slot >= p.cache.cap || (KB == 1 && h != 0)) continue;
      float w = sPart[tid];
      for (int i = 1; i < parts; ++i) w += sPart[tid + 64 * i];
      const float keep = r0 > 0 ? 1.f : st.is_new ? 0.f : p.decay;
      out[slot] = keep > 0.f ? fmaf(keep, (r0 > 0 ? out : old)[slot], w) : w;
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
  // a workgroup a compute unit
  WeighParams p = params;
  p.plan = {};
  p.plan.batch = p.batch;
  p.plan.cap = p.cache.cap;
  p.plan.ctx_lens = p.cache.lens;
  p.plan.n_sinks = p.n_sinks;
  p.plan.window = p.window;
  const int per_g = 256 / p.hkv;
  p.plan.slots_per_g = per_g > p.batch ? per_g : p.batch;
  // The least piece is the attention's rule (least_piece(), here up to four tiles),
  // which is one of its merge; there is none here.  It costs where workgroups would
  // be left over, above all in fp32, whose waves share a step only in pieces of one
  // or two tiles: with the rule, and with pieces of one tile, 64 rows of 12/1 heads
  // of 128 over 4096 fp32 keys take 122 and 60 us, 16 rows of 28/4 heads 23.7 and
  // 16.3; in bf16 24.9 and 23.0, 9.2 and 9.2; full calls the same.
  p.plan.min_tiles = 1;
  p.plan.tiles_rg = 5;
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
