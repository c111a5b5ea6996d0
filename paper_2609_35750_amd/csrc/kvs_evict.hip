// gfx950 kernel of the eviction by attention weight: of every sequence of a
// paged cache, the entries of lowest weight leave until `keep` are left.  The
// first tokens (positions below `sinks`) and the newest (above the newest
// position - recent) are never taken; equal weights leave in the table's order.
//
// One workgroup a sequence.  The n-th lowest weight is found by narrowing the
// range of weights: as integers that order like the floats, the range is cut
// into 1,024 equal bins, the bin that holds the n-th is the next range, until
// nothing is left to tell apart (the whole bin leaves, or it is one value): two
// or three counts of all entries instead of a sort.  Equal steps of these
// integers are equal steps of a weight's exponent and leading bits, so weights
// that span many powers of two spread over the bins, and the counts (atomics on
// integers in LDS) rarely meet.  Bound by latency: 8 bytes a slot are read.
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>

namespace kvs {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave, kEvictBins = 1024;

// Integers that order like the floats; -0 like +0, and NaN above everything.
__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 0xffffffffu;
  const unsigned b = w == 0.f ? 0u : __float_as_uint(w);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}

// Entries a thread keeps in registers: KEEP strips of 64 a wave; 0: read again for every count (longer tables).
template <int KEEP>
__global__ void __launch_bounds__(kEvictThreads) paged_evict_lowest_kernel(PagedEvictLowest a) {
  __shared__ int hist[kEvictBins];
  __shared__ int red[4][kEvictWaves];
  __shared__ int pick[2];   // bin of the n-th, entries below it
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int BS = a.block_size;
  const int n = min(max(a.seq_blocks[s], 0), a.max_blocks) * BS;   // slots of the sequence
  const int* trow = a.block_table + (size_t)s * a.max_blocks;
  int32_t* out = a.positions + (size_t)s * a.max_out;

  // wave w has the places [w per, (w + 1) per) of the table, in strips of 64
  const int strips = KEEP ? KEEP : (n + kEvictThreads - 1) / kEvictThreads;
  const int c0 = wave * strips * kWave;
  auto slot_at = [&](int c) __attribute__((always_inline)) {   // -1: no slot
    if (c >= n) return -1;
    const int blk = trow[c / BS];
    return (unsigned)blk < (unsigned)a.num_blocks ? blk * BS + c % BS : -1;
  };
  int pos_r[KEEP ? KEEP : 1];        // position of the entry; -1: none
  unsigned key_r[KEEP ? KEEP : 1];
  int slot_r[KEEP ? KEEP : 1];
  int live = 0, last = -1;
#pragma unroll
  for (int k = 0; k < (KEEP ? KEEP : 0); ++k) {
    slot_r[k] = slot_at(c0 + k * kWave + lane);
    pos_r[k] = slot_r[k] >= 0 ? a.slot_pos[slot_r[k]] : -1;
    key_r[k] = slot_r[k] >= 0 ? weight_key(a.slot_weight[slot_r[k]]) : 0u;
  }
  // f(strip, position, key, slot) for every strip; position -1 where the lane has no entry
  auto each = [&](auto f) __attribute__((always_inline)) {
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < (KEEP ? KEEP : 1); ++k) f(pos_r[k], key_r[k], slot_r[k]);
    } else {
#pragma unroll 4
      for (int k = 0; k < strips; ++k) {
        const int slot = slot_at(c0 + k * kWave + lane);
        f(slot >= 0 ? a.slot_pos[slot] : -1, slot >= 0 ? weight_key(a.slot_weight[slot]) : 0u, slot);
      }
    }
  };
  each([&](int pos, unsigned, int) __attribute__((always_inline)) {
    live += __builtin_popcountll(__ballot(pos >= 0));
    last = max(last, pos);
  });
  last = wave_max(last);
  if (lane == 0) {
    red[0][wave] = live;
    red[1][wave] = last;
  }
  __syncthreads();
  live = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    live += red[0][w];
    last = max(last, red[1][w]);
  }
  const int newest = last - a.recent;   // positions above it stay (last >= -1, recent >= 0)
  auto is_free = [&](int pos) { return pos >= 0 && pos >= a.sinks && pos <= newest; };
  // the entries that may leave: how many, and the range of their keys
  int nfree = 0;
  unsigned lo = 0xffffffffu, hi = 0u;
  each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
    const bool f = is_free(pos);
    nfree += __builtin_popcountll(__ballot(f));
    lo = f ? min(lo, key) : lo;
    hi = f ? max(hi, key) : hi;
  });
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    lo = min(lo, (unsigned)__shfl_xor((int)lo, off));
    hi = max(hi, (unsigned)__shfl_xor((int)hi, off));
  }
  __syncthreads();   // red is read
  if (lane == 0) {
    red[0][wave] = nfree;
    red[1][wave] = (int)lo;
    red[2][wave] = (int)hi;
  }
  __syncthreads();
  nfree = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    nfree += red[0][w];
    lo = min(lo, (unsigned)red[1][w]);
    hi = max(hi, (unsigned)red[2][w]);
  }
  const int go = min(min(max(live - max(a.keep[s], 0), 0), nfree), a.max_out);   // entries that leave
  for (int i = go + tid; i < a.max_out; i += kEvictThreads) out[i] = -1;
  if (tid == 0) a.counts[s] = go;
  if (go == 0) return;

  // Narrow [lo, hi] to the key of the go-th lowest: `rank` of the entries in the range leave (1 <= rank <= entries in
  // the range), and all below it.
  int rank = go, inside = nfree;
  while (rank < inside && lo < hi) {
    const unsigned width = hi - lo;
    const int shift = max(22 - (int)__builtin_clz(width), 0);   // width >> shift < 1,024
    hist[tid] = 0;
    __syncthreads();
    each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
      if (is_free(pos) && key >= lo && key <= hi) atomicAdd(&hist[(key - lo) >> shift], 1);
    });
    __syncthreads();
    const int cnt = hist[tid], incl = wave_scan(cnt);
    if (lane == kWave - 1) red[3][wave] = incl;
    __syncthreads();
    int below = incl - cnt;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) below += w < wave ? red[3][w] : 0;
    if (below < rank && rank <= below + cnt) {   // one thread
      pick[0] = tid;
      pick[1] = below;
    }
    __syncthreads();
    const int bin = pick[0];
    rank -= pick[1];
    inside = hist[bin];
    lo += (unsigned)bin << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1u);
    __syncthreads();   // hist and pick are read
  }

  // All entries below lo leave, and of those in [lo, hi] the first `rank` in the table's order (all of them, or
  // all equal).
  int nbelow = 0, nin = 0;
  each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
    const bool f = is_free(pos);
    nbelow += __builtin_popcountll(__ballot(f && key < lo));
    nin += __builtin_popcountll(__ballot(f && key >= lo && key <= hi));
  });
  if (lane == 0) {
    red[0][wave] = nbelow;
    red[1][wave] = nin;
  }
  __syncthreads();
  int at = 0, in = 0;   // entries in front of this wave's that leave for certain, that lie in the range
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    at += w < wave ? red[0][w] : 0;
    in += w < wave ? red[1][w] : 0;
  }
  at += min(in, rank);
  const unsigned long long before = (1ull << lane) - 1ull;
  each([&](int pos, unsigned key, int slot) __attribute__((always_inline)) {
    const bool f = is_free(pos), in_range = f && key >= lo && key <= hi;
    const unsigned long long range = __ballot(in_range);
    const bool gone = (f && key < lo) || (in_range && in + __builtin_popcountll(range & before) < rank);
    const unsigned long long leave = __ballot(gone);
    if (gone) {
      out[at + __builtin_popcountll(leave & before)] = pos;
      a.slot_pos[slot] = -1;
    }
    in += __builtin_popcountll(range);
    at += __builtin_popcountll(leave);
  });
}

template __global__ void paged_evict_lowest_kernel<4>(PagedEvictLowest);
template __global__ void paged_evict_lowest_kernel<16>(PagedEvictLowest);
template __global__ void paged_evict_lowest_kernel<0>(PagedEvictLowest);

hipError_t launch_paged_evict_lowest(const PagedEvictLowest& p) {
  const long long width = (long long)p.max_blocks * p.block_size;
  const auto kernel = width <= 4 * kEvictThreads    ? paged_evict_lowest_kernel<4>
                      : width <= 16 * kEvictThreads ? paged_evict_lowest_kernel<16>
                                                    : paged_evict_lowest_kernel<0>;
  prof_begin("paged_evict_lowest", p.stream);
  hipLaunchKernelGGL(kernel, dim3((unsigned)p.S), dim3(kEvictThreads), 0, p.stream, p);
  prof_end(p.stream);
  return hipGetLastError();
}

}  // namespace kvs
