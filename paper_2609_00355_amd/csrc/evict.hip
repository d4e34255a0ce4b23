// Eviction from a context cache by accumulated attention weight.
//
// Of every (sequence, KV head) with more than `budget` slots the first n_sinks,
// the last n_recent and the budget - n_sinks - n_recent of greatest weight
// among the others are kept, in their order; ties go to the lowest slot and a
// NaN counts as larger than every number.
//
// Selection, by a workgroup of a (sequence, KV head): the least kept weight by
// counts of order-preserving keys, then the kept slots in order by prefix sums.
// Bound by the instructions of some five passes over a workgroup's keys and a dozen
// barriers.  Then the kept rows of K, V, scales and weights are copied, 16 bytes a
// lane, bound by memory.
//
// Where LDS holds every key of the cache, the workgroups of a head (as many as
// fill the compute units) all select, which costs no more time than one doing so,
// and each copies its share of the rows: one launch.  The lengths are not known
// when the launch is chosen, so the capacity decides.  Caches of larger capacity:
// one workgroup a head selects, reading the weights past the held ones in
// every pass, and a second launch copies.  4096 of 16384 slots of 16 heads of 128 in
// bf16 (33 MB kept): 21.3 us in one launch, the selection 10 of it (13.7 at the rate
// of a large copy), 23.7 in two; 5001 of up to 11003 slots of 10 fp32 heads of 64:
// 16.0 and 19.9 (9.7).  Beyond, the selection grows with the length: a quarter of
// 65536, 131072 and 262144 slots of 4 bf16 heads of 128 takes 41, 82 and 157 us
// (13.7, 27.4 and 54.8), of 16 such heads 85, 159 and 310 (55, 110 and 219).
#include "glance_internal.h"

#include "attn_plan.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;
constexpr int kChunk = 4 * kSelectThreads;  // slots the workgroup reads with one load a lane
constexpr int kChunks = 4;                  // chunks in flight
constexpr int kBinBits = 11, kBins = 1 << kBinBits;
constexpr int kHeld = 32768;                // keys held in LDS: those of the first slots
constexpr int kListed = 4096;               // ... and those still in question
constexpr unsigned kRanked = 128;           // ... when they are ranked directly

// Keys: the unsigned order of weights, -0 and +0 equal and every NaN the largest,
// between one for slots there are not and one for slots kept whatever they weigh.
constexpr unsigned kNever = 0, kAlways = 0xffffffffu;
__device__ __forceinline__ unsigned order_key(unsigned bits) {
  const float w = __builtin_bit_cast(float, bits);
  const int u = __builtin_bit_cast(int, w + 0.f);  // -0 becomes +0
  const unsigned k = (unsigned)(u ^ (u >> 31 | (int)0x80000000));
  return w != w ? kAlways - 1 : k - 1;
}

__device__ __forceinline__ int clamp_len(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }

// Inclusive prefix sum within each row of 16 lanes, all lanes active: with a
// wave's count in lane `wave` of every row, what the waves before it counted.
__device__ __forceinline__ int row_incl_sum(int v) {
  v += plan_dpp<0x111, 0xf, 0>(v);  // row_shr:1
  v += plan_dpp<0x112, 0xf, 0>(v);  // row_shr:2
  v += plan_dpp<0x114, 0xf, 0>(v);  // row_shr:4
  v += plan_dpp<0x118, 0xf, 0>(v);  // row_shr:8
  return v;
}
// Largest value of each row of 16 lanes, and of the wave, in every lane.
__device__ __forceinline__ unsigned row_umax(unsigned v) {
  v = max(v, (unsigned)plan_dpp<0xb1, 0xf, 0>((int)v));   // quad_perm [1,0,3,2]
  v = max(v, (unsigned)plan_dpp<0x4e, 0xf, 0>((int)v));   // quad_perm [2,3,0,1]
  v = max(v, (unsigned)plan_dpp<0x141, 0xf, 0>((int)v));  // row_half_mirror
  return max(v, (unsigned)plan_dpp<0x140, 0xf, 0>((int)v));  // row_mirror
}
__device__ __forceinline__ unsigned wave_umax(unsigned v) {
  v = row_umax(v);
  v = max(v, (unsigned)plan_dpp<0x142, 0xa, 0>((int)v));  // row_bcast:15
  v = max(v, (unsigned)plan_dpp<0x143, 0xc, 0>((int)v));  // row_bcast:31
  return (unsigned)__builtin_amdgcn_readlane((int)v, 63);
}
// Sum of each aligned run of eight lanes, in all of them (whole runs active).
__device__ __forceinline__ int eight_sum(int v) {
  v += plan_dpp<0xb1, 0xf, 0>(v);         // quad_perm [1,0,3,2]
  v += plan_dpp<0x4e, 0xf, 0>(v);         // quad_perm [2,3,0,1]
  return v + plan_dpp<0x141, 0xf, 0>(v);  // row_half_mirror
}
static_assert(kSelectWaves == 16, "a row of lanes holds the waves' counts");

// The rows r0 .. r1 - 1 of a head's destination, by a workgroup of
// kSelectThreads; slot_of(r) is the source slot of row r.
template <class Slot>
__device__ __forceinline__ void gather_rows(const EvictParams& p, int head, int r0, int r1, Slot slot_of) {
  constexpr int kBatch = 4;  // 16-byte pieces of a thread in flight
  const int tid = threadIdx.x;
  const int shift = __builtin_ctz((unsigned)p.src.row_bytes / 16);  // pieces of a row: a power of two
  const int units = r1 > r0 ? (r1 - r0) << shift : 0;
  const size_t from = (size_t)head * p.src.cap, to = (size_t)head * p.dst.cap;
  for (int u0 = 0; u0 < 2 * units; u0 += kBatch * kSelectThreads) {
    u32x4 v[kBatch];
    u32x4* at[kBatch];
#pragma unroll
    for (int x = 0; x < kBatch; ++x) {
      const int u = min(u0 + x * kSelectThreads + tid, 2 * units - 1);
      const bool v_side = u >= units;
      const int w = v_side ? u - units : u;
      const int row = r0 + (w >> shift), piece = w & ((1 << shift) - 1);
      const u32x4* src = reinterpret_cast<const u32x4*>(v_side ? p.src.v : p.src.k);
      u32x4* dst = reinterpret_cast<u32x4*>(v_side ? p.dst.v : p.dst.k);
      v[x] = src[((from + slot_of(row)) << shift) + piece];
      at[x] = dst + ((to + row) << shift) + piece;
    }
#pragma unroll
    for (int x = 0; x < kBatch; ++x)
      if (u0 + x * kSelectThreads + tid < 2 * units) *at[x] = v[x];
  }
  for (int r = r0 + tid; r < r1; r += kSelectThreads) {
    const size_t f = from + slot_of(r), t = to + r;
    const float w = p.src.weights[f];
    if (p.src.kv4) {
      if (p.d == 128) {  // 4 or 2 bytes of scales
        const unsigned k = reinterpret_cast<const unsigned*>(p.src.k_scale)[f], v = reinterpret_cast<const unsigned*>(p.src.v_scale)[f];
        reinterpret_cast<unsigned*>(p.dst.k_scale)[t] = k;
        reinterpret_cast<unsigned*>(p.dst.v_scale)[t] = v;
      } else {
        const unsigned short k = reinterpret_cast<const unsigned short*>(p.src.k_scale)[f], v = reinterpret_cast<const unsigned short*>(p.src.v_scale)[f];
        reinterpret_cast<unsigned short*>(p.dst.k_scale)[t] = k;
        reinterpret_cast<unsigned short*>(p.dst.v_scale)[t] = v;
      }
    }
    p.dst.weights[t] = w;
  }
}

template <bool GATHER>
__global__ __launch_bounds__(kSelectThreads) void evict_select(EvictParams p) {
  __shared__ u32x4 s_keys[kHeld / 4];
  __shared__ unsigned s_hist[kBins];
  __shared__ unsigned s_list[kListed];
  __shared__ unsigned s_sum[kSelectWaves], s_found[3], s_rank[3], s_n;
  __shared__ uint2 s_range[kSelectWaves];
  __shared__ int2 s_count[2][kSelectWaves];
  const int head = blockIdx.x, b = head / p.hkv;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int len = clamp_len(p.src.lens[b], p.src.cap);
  // the places that this workgroup fills
  const int r0 = GATHER ? (int)((long long)p.budget * blockIdx.y / gridDim.y) : 0;
  const int r1 = GATHER ? (int)((long long)p.budget * (blockIdx.y + 1) / gridDim.y) : p.budget;
  int* kept = p.kept + (size_t)head * p.budget;
  int* s_kept = reinterpret_cast<int*>(s_keys);  // GATHER: the slots at those places
  if (GATHER && head % p.hkv == 0 && blockIdx.y == 0 && tid == 0) p.dst.lens[b] = min(len, p.budget);
  if (len <= p.budget) {
    for (int j = r0 + tid; j < r1; j += kSelectThreads) kept[j] = j < len ? j : -1;
    if (GATHER) {
      const int from = (int)((long long)len * blockIdx.y / gridDim.y), to = (int)((long long)len * (blockIdx.y + 1) / gridDim.y);
      gather_rows(p, head, from, to, [&](int r) { return r; });
    }
    return;
  }
  const float* w = p.src.weights + (size_t)head * p.src.cap;
  const int lo = p.n_sinks, hi = len - p.n_recent;  // slots that have to earn their place
  unsigned need = (unsigned)(p.budget - p.n_sinks - p.n_recent);

  // The keys of slots j0 + kChunk c + 4 tid + i.  A thread's slots are its own in
  // every pass, so it finds its keys in LDS without a barrier; only longer
  // sequences' are read again.
  auto fetch = [&](int j0, u32x4 (&k)[kChunks]) __attribute__((always_inline)) {
    typedef u32x4 __attribute__((aligned(4))) loose;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int j = j0 + kChunk * c + 4 * tid;
      k[c] = u32x4{};
      if (len >= 4) k[c] = *reinterpret_cast<const loose*>(w + min(j, len - 4));
    }
    unsigned top = 0;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int j = j0 + kChunk * c + 4 * tid;
      if (j > len - 4) {  // the last slots, one by one
#pragma unroll
        for (int i = 0; i < 4; ++i) k[c][i] = __builtin_bit_cast(unsigned, w[min(j + i, len - 1)]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) top = max(top, k[c][i]);
    }
    // (weights are sums of exponentials: all of a wave's are mostly 0 or more)
    if (__builtin_amdgcn_ballot_w64(top > 0x7f800000u) == 0) {
#pragma unroll
      for (int c = 0; c < kChunks; ++c) k[c] += 0x7fffffffu;  // order_key() of these
    } else {
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) k[c][i] = order_key(k[c][i]);
    }
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int first = j0 + kChunk * c, j = first + 4 * tid;
      if (first < lo || first + kChunk > hi) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          k[c][i] = j + i >= lo && j + i < hi ? k[c][i] : j + i < len ? kAlways : kNever;
      }
      if (j0 < kHeld) s_keys[j / 4] = k[c];
    }
  };
  auto read = [&](int j0, u32x4 (&k)[kChunks]) __attribute__((always_inline)) {
    if (j0 >= kHeld) return fetch(j0, k);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) k[c] = s_keys[(j0 + kChunk * c) / 4 + tid];
  };
  static_assert(kHeld % (kChunks * kChunk) == 0, "a read is held in whole or not at all");

  // The need-th largest key, by counts in kBins bins: of the keys from the least
  // to the largest, then of those in the bin where the count from the top reaches
  // `need`, until a bin is one key.  Bins of the keys' own range, not of fixed
  // bits, spread them over more bins, so that fewer lanes add to one at a time,
  // and leave few keys in each.  Bin 0 is never counted: it has what the others
  // leave (weights of 0, often many, are there).  Keys of the last bin are listed
  // once they fit, and ranked one against the other once they are few.
  //
  // Four waves share a SIMD, so an instruction a key costs 256 cycles here.
  unsigned base = kAlways, equal = 0;
  if (need > 0) {
    unsigned most = 0, least = 0;  // largest key plus 1, least key's complement plus 1 (kNever, kAlways: 1, 0 and 0, 1)
    for (int j0 = 0; j0 < len; j0 += kChunks * kChunk) {
      u32x4 k[kChunks];
      fetch(j0, k);
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          most = max(most, k[c][i] + 1);
          least = max(least, 0u - k[c][i]);
        }
    }
    for (int i = tid; i < kBins; i += kSelectThreads) s_hist[i] = 0;
    if (tid == 0) s_n = 0;
    most = wave_umax(most);
    least = wave_umax(least);
    if (lane == 0) s_range[wave] = make_uint2(most, least);
    __syncthreads();
    const uint2 range = s_range[lane & 15];
    most = (unsigned)__builtin_amdgcn_readfirstlane((int)row_umax(range.x)) - 1;
    base = 0u - (unsigned)__builtin_amdgcn_readfirstlane((int)row_umax(range.y));
    unsigned span = most - base;   // the keys in question: base .. base + span
    equal = (unsigned)(hi - lo);   // how many they are
    int n_list = 0;                // keys listed, 0 before
    for (bool first = true;; first = false) {
      const int shift = span >> kBinBits ? 32 - kBinBits - __builtin_clz(span) : 0;
      const unsigned step = 1u << shift;
      if (!first) {
        for (int i = tid; i < kBins; i += kSelectThreads) s_hist[i] = 0;
        __syncthreads();
      }
      // of the keys from bin 1 on (all others, kNever and kAlways too, wrap past them)
      auto count = [&](unsigned k) __attribute__((always_inline)) {
        const unsigned d = k - (base + step);
        if (d <= span - step) atomicAdd(&s_hist[1 + (d >> shift)], 1u);
      };
      if (span == 0) {
      } else if (n_list) {
        for (int i = tid; i < n_list; i += kSelectThreads) count(s_list[i]);
      } else {
        for (int j0 = 0; j0 < len; j0 += kChunks * kChunk) {
          u32x4 k[kChunks];
          read(j0, k);
#pragma unroll
          for (int c = 0; c < kChunks; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i) count(k[c][i]);
        }
      }
      __syncthreads();
      // the bin in which the count from the top reaches `need`: every wave sums
      // its 128 bins, and the one with the crossing finds it
      const int bin = kBins - 2 - 128 * wave - 2 * lane;  // and the one above it
      const unsigned hi_bin = s_hist[bin + 1], lo_count = s_hist[bin];
      const unsigned incl = (unsigned)wave_incl_sum((int)(hi_bin + lo_count));
      if (lane == 63) s_sum[wave] = incl;
      __syncthreads();
      const int sum = (int)s_sum[lane & 15], sums = row_incl_sum(sum);
      const unsigned before = (unsigned)__builtin_amdgcn_readlane(sums - sum, wave);
      const unsigned at_hi = before + incl - hi_bin - lo_count, at_lo = at_hi + hi_bin;
      const unsigned lo_bin = bin == 0 ? equal - at_lo : lo_count;
      const bool in_hi = at_hi < need && need <= at_lo, in_lo = at_lo < need && need <= at_lo + lo_bin;
      if (in_hi || in_lo) {  // one lane of the workgroup
        s_found[0] = (unsigned)(in_lo ? bin : bin + 1);
        s_found[1] = need - (in_lo ? at_lo : at_hi);
        s_found[2] = in_lo ? lo_bin : hi_bin;
      }
      __syncthreads();
      base += (unsigned)__builtin_amdgcn_readfirstlane((int)s_found[0]) << shift;
      need = (unsigned)__builtin_amdgcn_readfirstlane((int)s_found[1]);
      equal = (unsigned)__builtin_amdgcn_readfirstlane((int)s_found[2]);
      span = min(step - 1, most - base);
      if (shift == 0) break;
      if (n_list == 0 && equal <= kListed) {
        for (int j0 = 0; j0 < len; j0 += kChunks * kChunk) {
          u32x4 k[kChunks];
          read(j0, k);
          unsigned long long in[4 * kChunks];
          int n = 0;
#pragma unroll
          for (int x = 0; x < 4 * kChunks; ++x) {
            in[x] = __builtin_amdgcn_ballot_w64(k[x / 4][x % 4] - base <= span);
            n += __popcll(in[x]);
          }
          if (n == 0) continue;
          int at = 0;
          if (lane == 0) at = (int)atomicAdd(&s_n, (unsigned)n);
          at = __builtin_amdgcn_readfirstlane(at);
#pragma unroll
          for (int x = 0; x < 4 * kChunks; ++x) {
            if (in[x] == 0) continue;
            if (in[x] >> lane & 1u)
              s_list[at + __builtin_amdgcn_mbcnt_hi((unsigned)(in[x] >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)in[x], 0))] = k[x / 4][x % 4];
            at += __popcll(in[x]);
          }
        }
        n_list = (int)equal;
        __syncthreads();
        if (equal <= kRanked) {
          // eight lanes a key, each with an eighth of the others
          const int mine = tid / 8;
          if (mine < (int)equal) {
            const unsigned key = s_list[mine];
            int above = 0, same = 0;
            for (int i = tid % 8; i < (int)equal; i += 8) {
              const unsigned k = s_list[i];
              above += k > key ? 1 : 0;
              same += k == key ? 1 : 0;
            }
            above = eight_sum(above);
            same = eight_sum(same);
            if (above < (int)need && (int)need <= above + same) {  // one key, perhaps of several slots
              s_rank[0] = key;
              s_rank[1] = need - above;
              s_rank[2] = same;
            }
          }
          __syncthreads();
          base = s_rank[0];
          need = s_rank[1];
          equal = s_rank[2];
          break;
        }
      }
    }
  }
  // Kept slots in order: those above the least kept key and the first `need` of
  // the `equal` ones that are it.  A slot's place is the number kept before it:
  // counts of two chunks share a word (at most 4096 each).
  int out = 0, ties = 0;  // kept, and equal ones, in the chunks before
  int turn = 0;
  // exclusive sums over the workgroup of each chunk's counts, and their totals
  auto scan = [&](int2 mine, int2& total) __attribute__((always_inline)) {
    const int2 incl = make_int2(wave_incl_sum(mine.x), wave_incl_sum(mine.y));
    int2* slot = s_count[turn];
    turn ^= 1;  // (a barrier lies between two uses of a buffer)
    if (lane == 63) slot[wave] = incl;
    __syncthreads();
    const int2 o = slot[lane & 15], sums = make_int2(row_incl_sum(o.x), row_incl_sum(o.y));
    total = make_int2(__builtin_amdgcn_readlane(sums.x, 15), __builtin_amdgcn_readlane(sums.y, 15));
    return make_int2(incl.x - mine.x + __builtin_amdgcn_readlane(sums.x - o.x, wave),
                     incl.y - mine.y + __builtin_amdgcn_readlane(sums.y - o.y, wave));
  };
  auto half = [](int2 v, int c) __attribute__((always_inline)) { return ((c & 2 ? v.y : v.x) >> (c & 1 ? 16 : 0)) & 0xffff; };
  auto add = [](int2& v, int c, int n) __attribute__((always_inline)) { (c & 2 ? v.y : v.x) += n << (c & 1 ? 16 : 0); };
  const bool some = need < equal;  // not all of the equal ones are kept
  const bool none = p.budget == p.n_sinks + p.n_recent;
  for (int j0 = 0; j0 < len; j0 += kChunks * kChunk) {
    u32x4 k[kChunks];
    if (none) fetch(j0, k);  // nothing was read before
    else read(j0, k);
    int2 total;
    if (some) {
      int2 mine = make_int2(0, 0);
#pragma unroll
      for (int c = 0; c < kChunks; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) add(mine, c, k[c][i] == base ? 1 : 0);
      const int2 at = scan(mine, total);
#pragma unroll
      for (int c = 0; c < kChunks; ++c) {
        int rank = ties + half(at, c);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (k[c][i] == base && rank++ >= (int)need) k[c][i] = kNever;
        ties += half(total, c);
      }
    }
    int2 mine = make_int2(0, 0);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      int n = 0;
#pragma unroll
      for (int i = 0; i < 4; ++i) n += k[c][i] >= base ? 1 : 0;
      add(mine, c, n);
    }
    const int2 at = scan(mine, total);
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
      const int j = j0 + kChunk * c + 4 * tid;
      int place = out + half(at, c);
      out += half(total, c);
      if (GATHER && (place >= r1 || place + 4 <= r0)) continue;
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (k[c][i] >= base) {
          // (a place is at most its slot, and the barrier in scan() lies behind
          // every read of the keys up to this chunk's: none is overwritten unread)
          if (!GATHER) kept[place] = j + i;
          else if (place >= r0 && place < r1) s_kept[place - r0] = j + i;
          ++place;
        }
    }
  }
  if (GATHER) {
    __syncthreads();
    for (int r = r0 + tid; r < r1; r += kSelectThreads) kept[r] = s_kept[r - r0];
    gather_rows(p, head, r0, r1, [&](int r) { return s_kept[r - r0]; });
  }
}

constexpr int kGatherThreads = 256;

// Grid (chunks of a head's 16-byte pieces, heads, 2: keys and values).
__global__ __launch_bounds__(kGatherThreads) void evict_gather(EvictParams p) {
  const int head = blockIdx.y;
  const bool v_side = blockIdx.z;
  const int pieces = p.src.row_bytes / 16;
  const int u = blockIdx.x * kGatherThreads + threadIdx.x;
  const int row = u / pieces, piece = u % pieces;
  if (u == 0 && !v_side && head % p.hkv == 0) {
    // (only this thread reads the length here: the destination's may be the same)
    const int b = head / p.hkv;
    p.dst.lens[b] = min(clamp_len(p.src.lens[b], p.src.cap), p.budget);
  }
  if (row >= p.budget) return;
  const int slot = p.kept[(size_t)head * p.budget + row];
  if (slot < 0) return;
  const size_t from = (size_t)head * p.src.cap + slot, to = (size_t)head * p.dst.cap + row;
  const u32x4* src = reinterpret_cast<const u32x4*>(v_side ? p.src.v : p.src.k);
  u32x4* dst = reinterpret_cast<u32x4*>(v_side ? p.dst.v : p.dst.k);
  dst[to * pieces + piece] = src[from * pieces + piece];
  if (piece != 0) return;
  if (p.src.kv4) {
    const int n = p.d / 32;  // 2 or 4 bytes
    const unsigned char* s = (v_side ? p.src.v_scale : p.src.k_scale) + from * n;
    unsigned char* d = (v_side ? p.dst.v_scale : p.dst.k_scale) + to * n;
    if (n == 4) *reinterpret_cast<unsigned*>(d) = *reinterpret_cast<const unsigned*>(s);
    else *reinterpret_cast<unsigned short*>(d) = *reinterpret_cast<const unsigned short*>(s);
  }
  if (!v_side) p.dst.weights[to] = p.src.weights[from];
}

}  // namespace

hipError_t launch_evict(const EvictParams& p, hipStream_t s, hipEvent_t ev0, hipEvent_t ev1) {
  const int heads = p.batch * p.hkv;
  const long long units = (long long)p.budget * (p.src.row_bytes / 16);
  const dim3 grid((unsigned)((units + kGatherThreads - 1) / kGatherThreads), (unsigned)heads, 2);
  if (ev0) (void)hipEventRecord(ev0, s);
  // (with shared lengths other workgroups of the one launch would still read what it writes)
  if (p.src.cap <= kHeld && p.src.lens != p.dst.lens) {
    const int parts = heads < 256 ? 256 / heads : 1;
    hipLaunchKernelGGL(evict_select<true>, dim3((unsigned)heads, (unsigned)parts), dim3(kSelectThreads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (ev1) (void)hipEventRecord(ev1, s);
    return e;
  }
  hipLaunchKernelGGL(evict_select<false>, dim3((unsigned)heads), dim3(kSelectThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(evict_gather, grid, dim3(kGatherThreads), 0, s, p);
    e = hipGetLastError();
  }
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
