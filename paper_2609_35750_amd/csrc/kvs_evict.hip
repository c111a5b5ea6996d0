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

// Places of the table a lane looks at, 64 apart: one division, then additions.
struct Places {
  int c, blk, row, BS, dblk, drow;
  __device__ __forceinline__ Places(int first, int bs) : c(first), blk(first / bs), row(first % bs), BS(bs) {
    dblk = kWave / bs;
    drow = kWave % bs;
  }
  __device__ __forceinline__ void next() {
    c += kWave;
    blk += dblk;
    row += drow;
    if (row >= BS) {
      row -= BS;
      ++blk;
    }
  }
};

// Entries a thread keeps in registers: KEEP strips of 64 a wave; 0: read again for every count (longer tables).
template <int KEEP>
__global__ void __launch_bounds__(kEvictThreads) paged_evict_lowest_kernel(PagedEvictLowest a) {
  constexpr int N = KEEP ? KEEP : 1;
  __shared__ int hist[kEvictBins];
  __shared__ int red[2][4][kEvictWaves];   // by turns, so that one barrier stands between two exchanges
  __shared__ int pick[2][2];               // bin of the n-th, entries below it
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.seq_blocks[s], 0), a.max_blocks) * a.block_size;   // slots of the sequence
  const int* trow = a.block_table + (size_t)s * a.max_blocks;
  int32_t* out = a.positions + (size_t)s * a.max_out;
  const int keep = max(a.keep[s], 0);

  // wave w has the places [w strips 64, (w + 1) strips 64) of the table, in strips of 64
  const int strips = (n + kEvictThreads - 1) / kEvictThreads, c0 = wave * strips * kWave + lane;
  // an entry: its position (-1: none), the key of its weight, its slot
  int pos_r[N], slot_r[N];
  unsigned key_r[N];
  auto slot_of = [&](int entry, const Places& p) __attribute__((always_inline)) {
    return p.c < n && (unsigned)entry < (unsigned)a.num_blocks ? entry * a.block_size + p.row : -1;
  };
  if (KEEP) {
    Places p(c0, a.block_size);
#pragma unroll
    for (int k = 0; k < N; ++k, p.next()) slot_r[k] = k < strips && p.c < n ? trow[p.blk] : -1;
    p = Places(c0, a.block_size);
#pragma unroll
    for (int k = 0; k < N; ++k, p.next()) slot_r[k] = k < strips ? slot_of(slot_r[k], p) : -1;
    float w[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      pos_r[k] = slot_r[k] >= 0 ? a.slot_pos[slot_r[k]] : -1;
      w[k] = slot_r[k] >= 0 ? a.slot_weight[slot_r[k]] : 0.f;
    }
#pragma unroll
    for (int k = 0; k < N; ++k) key_r[k] = weight_key(w[k]);
  }
  // f(position, key, slot) for every strip
  auto each = [&](auto f) __attribute__((always_inline)) {
    if (KEEP) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (k < strips) f(pos_r[k], key_r[k], slot_r[k]);
    } else {
      Places p(c0, a.block_size);
#pragma unroll 8
      for (int k = 0; k < strips; ++k, p.next()) {
        const int slot = slot_of(p.c < n ? trow[p.blk] : -1, p);
        f(slot >= 0 ? a.slot_pos[slot] : -1, slot >= 0 ? weight_key(a.slot_weight[slot]) : 0u, slot);
      }
    }
  };

  // live entries, the newest position, the range of the keys (of all but the sinks: the newest are not known yet)
  int live = 0, last = -1;
  unsigned lo = 0xffffffffu, hi = 0u;
  each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
    live += __builtin_popcountll(__ballot(pos >= 0));
    last = max(last, pos);
    const bool f = pos >= a.sinks && pos >= 0;
    lo = f ? min(lo, key) : lo;
    hi = f ? max(hi, key) : hi;
  });
  last = wave_max(last);
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) {
    lo = min(lo, (unsigned)__shfl_xor((int)lo, off));
    hi = max(hi, (unsigned)__shfl_xor((int)hi, off));
  }
  if (lane == 0) {
    red[0][0][wave] = live;
    red[0][1][wave] = last;
    red[0][2][wave] = (int)lo;
    red[0][3][wave] = (int)hi;
  }
  hist[tid] = 0;
  __syncthreads();
  live = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    live += red[0][0][w];
    last = max(last, red[0][1][w]);
    lo = min(lo, (unsigned)red[0][2][w]);
    hi = max(hi, (unsigned)red[0][3][w]);
  }
  const int newest = last - a.recent;   // positions above it stay (last >= -1, recent >= 0)
  auto is_free = [&](int pos) { return pos >= 0 && pos >= a.sinks && pos <= newest; };

  // Narrow [lo, hi] to the key of the go-th lowest: `rank` of the free entries in the range leave (1 <= rank <= inside,
  // how many those are), and all below it.  The first count also says how many free entries there are.
  int go = min(max(live - keep, 0), a.max_out), rank = go, inside = INT_MAX;   // entries that leave
  bool first = true;
  int turn = 1;
  while (rank > 0 && rank < inside && (first || lo < hi)) {
    const unsigned width = hi >= lo ? hi - lo : 0u;
    const int shift = max(22 - (width ? (int)__builtin_clz(width) : 32), 0);   // width >> shift < 1,024
    each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
      if (is_free(pos) && key >= lo && key <= hi) atomicAdd(&hist[(key - lo) >> shift], 1);
    });
    __syncthreads();
    const int cnt = hist[tid], incl = wave_scan(cnt);
    if (lane == kWave - 1) red[turn][0][wave] = incl;
    __syncthreads();
    int below = incl - cnt, all = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
      const int x = red[turn][0][w];
      below += w < wave ? x : 0;
      all += x;
    }
    if (first) rank = go = min(go, all);
    first = false;
    if (below < rank && rank <= below + cnt) {   // one thread, if any entry leaves
      pick[turn][0] = tid;
      pick[turn][1] = below;
    }
    hist[tid] = 0;
    if (below < rank && rank <= below + cnt) red[turn][1][0] = cnt;
    __syncthreads();
    if (rank == 0) break;
    rank -= pick[turn][1];
    inside = red[turn][1][0];
    lo += (unsigned)pick[turn][0] << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1u);
    turn ^= 1;
  }
  for (int i = go + tid; i < a.max_out; i += kEvictThreads) out[i] = -1;
  if (tid == 0) a.counts[s] = go;
  if (go == 0) return;

  // All entries below lo leave, and of those in [lo, hi] the first `rank` in the table's order (all of them, or
  // all equal).
  int nbelow = 0, nin = 0;
  each([&](int pos, unsigned key, int) __attribute__((always_inline)) {
    const bool f = is_free(pos);
    nbelow += __builtin_popcountll(__ballot(f && key < lo));
    nin += __builtin_popcountll(__ballot(f && key >= lo && key <= hi));
  });
  if (lane == 0) {
    red[turn][2][wave] = nbelow;
    red[turn][3][wave] = nin;
  }
  __syncthreads();
  int at = 0, in = 0;   // entries in front of this wave's that leave for certain, that lie in the range
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    at += w < wave ? red[turn][2][w] : 0;
    in += w < wave ? red[turn][3][w] : 0;
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
