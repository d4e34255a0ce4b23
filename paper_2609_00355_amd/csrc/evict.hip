// Eviction from a context cache by accumulated attention weight.
//
// Of every (sequence, KV head) with more than `budget` slots the first n_sinks,
// the last n_recent and the budget - n_sinks - n_recent of greatest weight
// among the others are kept, in their order; ties go to the lowest slot and a
// NaN counts as larger than every number.  Two launches:
//
// 1. evict_select, one workgroup per (sequence, KV head): the least kept weight
//    by radix selection on order-preserving keys (four passes of eight bits over
//    the weights, counted in LDS), then the kept slots in order by a prefix sum.
// 2. evict_gather: the kept rows of K, V, scales and weights, 16 bytes a lane
//    where rows are that wide.  Bound by memory.
#include "glance_internal.h"

namespace glance {
namespace {

typedef __attribute__((ext_vector_type(4))) unsigned int u32x4;

constexpr int kSelectThreads = 1024;
constexpr int kSelectWaves = kSelectThreads / 64;

// Unsigned order of weights: -0 and +0 are equal, every NaN is the largest.
__device__ __forceinline__ unsigned order_key(float w) {
  unsigned u = __builtin_bit_cast(unsigned, w);
  if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
  if (u == 0x80000000u) u = 0;
  return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int clamp_len(int len, int cap) { return len < 0 ? 0 : (len > cap ? cap : len); }

__global__ __launch_bounds__(kSelectThreads) void evict_select(EvictParams p) {
  __shared__ unsigned s_hist[256];
  __shared__ unsigned s_prefix, s_need;
  __shared__ int s_count[2][kSelectWaves];
  const int head = blockIdx.x, b = head / p.hkv;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int len = clamp_len(p.src.lens[b], p.src.cap);
  int* kept = p.kept + (size_t)head * p.budget;
  if (len <= p.budget) {
    for (int j = tid; j < p.budget; j += kSelectThreads) kept[j] = j < len ? j : -1;
    return;
  }
  const float* w = p.src.weights + (size_t)head * p.src.cap;
  const int lo = p.n_sinks, hi = len - p.n_recent;  // slots that have to earn their place
  const unsigned take = (unsigned)(p.budget - p.n_sinks - p.n_recent);
  // the take-th largest key: its bits from the top, eight at a time; `need` of
  // the keys that agree with the bits found so far are still to be counted
  unsigned prefix = 0, need = take;
  if (take > 0) {
    for (int shift = 24; shift >= 0; shift -= 8) {
      if (tid < 256) s_hist[tid] = 0;
      __syncthreads();
      for (int j = lo + tid; j < hi; j += kSelectThreads) {
        const unsigned k = order_key(w[j]);
        if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&s_hist[(k >> shift) & 255u], 1u);
      }
      __syncthreads();
      if (wave == 0) {
        // lane l holds bins 255 - 4 l .. 252 - 4 l: counts from the largest bin on
        unsigned c[4], mine = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          c[i] = s_hist[255 - 4 * lane - i];
          mine += c[i];
        }
        unsigned incl = mine;
#pragma unroll
        for (int off = 1; off < 64; off <<= 1) {
          const unsigned o = __shfl_up(incl, off);
          if (lane >= off) incl += o;
        }
        unsigned before = incl - mine;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if (before < need && need <= before + c[i]) {  // one lane, one bin
            s_prefix = prefix | (unsigned)(255 - 4 * lane - i) << shift;
            s_need = need - before;
          }
          before += c[i];
        }
      }
      __syncthreads();
      prefix = s_prefix;
      need = s_need;
    }
  }
  // kept slots in order: those above the least kept key and the first `need`
  // that equal it; a chunk of slots at a time
  int out = 0, ties = 0;
  for (int j0 = 0; j0 < len; j0 += kSelectThreads) {
    const int j = j0 + tid;
    const bool mid = j >= lo && j < hi;
    const unsigned k = mid && take > 0 ? order_key(w[j]) : 0;
    const bool tie = mid && take > 0 && k == prefix;
    const unsigned long long tb = __ballot(tie);
    if (lane == 0) s_count[0][wave] = __popcll(tb);
    __syncthreads();
    int tie_rank = ties + __popcll(tb & ((1ull << lane) - 1));
    for (int x = 0; x < kSelectWaves; ++x) {
      tie_rank += x < wave ? s_count[0][x] : 0;
      ties += s_count[0][x];
    }
    const bool keep = j < len && (!mid || (take > 0 && (k > prefix || (tie && tie_rank < (int)need))));
    const unsigned long long kb = __ballot(keep);
    if (lane == 0) s_count[1][wave] = __popcll(kb);
    __syncthreads();
    int at = out + __popcll(kb & ((1ull << lane) - 1));
    for (int x = 0; x < kSelectWaves; ++x) {
      at += x < wave ? s_count[1][x] : 0;
      out += s_count[1][x];
    }
    if (keep) kept[at] = j;
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
  hipLaunchKernelGGL(evict_select, dim3((unsigned)heads), dim3(kSelectThreads), 0, s, p);
  hipError_t e = hipGetLastError();
  if (e == hipSuccess) {
    hipLaunchKernelGGL(evict_gather, grid, dim3(kGatherThreads), 0, s, p);
    e = hipGetLastError();
  }
  if (ev1) (void)hipEventRecord(ev1, s);
  return e;
}

}  // namespace glance
