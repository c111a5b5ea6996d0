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
//
// One CU asks for one line of memory a clock or two, so where a table's slots
// lie apart (blocks of fewer than four), reading them is what costs: 64
// sequences of 2,000 to 16,000 single slots took 54 us that way.  There, and
// where a sequence's places do not fit the workgroup's registers, a kernel on
// all CUs first brings positions and weights into the table's order (11 + 25 us;
// 10 of the 25 are the marks, one scattered word an evicted slot).  Eight
// sequences of 4,096 in blocks of 16: 14 us, 24 before the range of the keys,
// the counts and the prefix sums shared barriers.
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>

namespace kvs {

constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / kWave, kEvictBins = 1024;

// Integers that order like the floats; -0 like +0, and NaN above everything but kStays.
__device__ __forceinline__ unsigned weight_key(float w) {
  if (w != w) return 0xfffffffeu;
  const unsigned b = w == 0.f ? 0u : __float_as_uint(w);
  return b ^ ((b >> 31) ? 0xffffffffu : 0x80000000u);
}
constexpr unsigned kStays = 0xffffffffu;   // no entry, or one that is not taken: outside every range of keys

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

// Position and weight's key of every place of the tables, in their order: (-1, 0) where there is no slot.
constexpr int kGatherThreads = 256;
__global__ void __launch_bounds__(kGatherThreads) paged_gather_kernel(PagedEvictLowest a) {
  const int s = blockIdx.y, c = blockIdx.x * kGatherThreads + threadIdx.x;
  const int n = min(max(a.seq_blocks[s], 0), a.max_blocks) * a.block_size;
  if (c >= n) return;
  const int entry = a.block_table[(size_t)s * a.max_blocks + c / a.block_size];
  int2 v = make_int2(-1, 0);
  if ((unsigned)entry < (unsigned)a.num_blocks) {
    const int slot = entry * a.block_size + c % a.block_size;
    v = make_int2(a.slot_pos[slot], (int)weight_key(a.slot_weight[slot]));
  }
  a.gathered[(size_t)s * a.max_blocks * a.block_size + c] = v;
}

// Entries a thread keeps in registers: KEEP strips of 64 a wave; 0: read again for every count (longer tables).
// GATHERED: from what paged_gather_kernel wrote.
template <int KEEP, bool GATHERED>
__global__ void __launch_bounds__(kEvictThreads) paged_evict_lowest_kernel(PagedEvictLowest a) {
  constexpr int N = KEEP ? KEEP : 1;
  __shared__ int hist[kEvictBins];
  __shared__ int red[2][4][kEvictWaves];   // by turns, so that one barrier stands between two exchanges
  __shared__ int pick[2][3];               // bin of the n-th, entries below it, in it
  const int s = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n = min(max(a.seq_blocks[s], 0), a.max_blocks) * a.block_size;   // slots of the sequence
  const int* trow = a.block_table + (size_t)s * a.max_blocks;
  int32_t* out = a.positions + (size_t)s * a.max_out;
  const int keep = max(a.keep[s], 0);

  // wave w has the places [w strips 64, (w + 1) strips 64) of the table, in strips of 64
  const int strips = (n + kEvictThreads - 1) / kEvictThreads, c0 = wave * strips * kWave + lane;
  const int2* gathered = GATHERED ? a.gathered + (size_t)s * a.max_blocks * a.block_size : nullptr;
  // an entry: its position (-1: none), the key of its weight, its slot (GATHERED: its place)
  int pos_r[N], slot_r[N];
  unsigned key_r[N];
  auto slot_of = [&](int entry, const Places& p) __attribute__((always_inline)) {
    return p.c < n && (unsigned)entry < (unsigned)a.num_blocks ? entry * a.block_size + p.row : -1;
  };
  if (KEEP && GATHERED) {
    int2 v[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      slot_r[k] = c0 + k * kWave;
      v[k] = k < strips && slot_r[k] < n ? gathered[slot_r[k]] : make_int2(-1, 0);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) {
      pos_r[k] = v[k].x;
      key_r[k] = (unsigned)v[k].y;
    }
  } else if (KEEP) {
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
#pragma unroll 8
      for (int k = 0; k < strips; ++k) {
        const int c = c0 + k * kWave;
        const int2 v = c < n ? gathered[c] : make_int2(-1, 0);
        f(v.x, (unsigned)v.y, c);
      }
    }
  };

  // live entries, the newest position
  int live = 0, last = -1;
  each([&](int pos, unsigned, int) __attribute__((always_inline)) {
    live += __builtin_popcountll(__ballot(pos >= 0));
    last = max(last, pos);
  });
  last = wave_max(last);
  if (lane == 0) {
    red[0][0][wave] = live;
    red[0][1][wave] = last;
  }
  hist[tid] = 0;
  __syncthreads();
  live = 0;
#pragma unroll
  for (int w = 0; w < kEvictWaves; ++w) {
    live += red[0][0][w];
    last = max(last, red[0][1][w]);
  }
  // positions in [sinks, newest] may leave (last >= -1, recent >= 0; none do if newest < sinks)
  const int newest = last - a.recent;
  const unsigned span = newest >= a.sinks ? (unsigned)(newest - a.sinks) : 0u;
  const bool none = newest < a.sinks;
  auto key_of = [&](int pos, unsigned key) __attribute__((always_inline)) {
    return pos >= 0 && (unsigned)(pos - a.sinks) <= span && !none ? key : kStays;
  };
  if (KEEP) {
#pragma unroll
    for (int k = 0; k < N; ++k) key_r[k] = key_of(pos_r[k], key_r[k]);
  }
  // f(position, key or kStays, slot)
  auto each_key = [&](auto f) __attribute__((always_inline)) {
    each([&](int pos, unsigned key, int slot) __attribute__((always_inline)) { f(pos, KEEP ? key : key_of(pos, key), slot); });
  };

  // Narrow [lo, hi] to the key of the go-th lowest: `rank` of the entries in the range leave (1 <= rank <= inside, how
  // many those are), and all below it.  Every turn first finds the range of the keys that are there (one value,
  // however many entries, ends the search); the first one also says how many entries may leave.
  int go = min(max(live - keep, 0), a.max_out), rank = go, inside = INT_MAX, turn = 1;   // go: entries that leave
  unsigned lo = 0u, hi = 0xfffffffeu;
  while (rank > 0 && rank < inside) {
    unsigned mn = kStays, mx = 0u;
    int cnt = 0;
    each_key([&](int, unsigned key, int) __attribute__((always_inline)) {
      const bool f = key - lo <= hi - lo;
      mn = f ? min(mn, key) : mn;
      mx = f ? max(mx, key) : mx;
      if (inside == INT_MAX) cnt += __builtin_popcountll(__ballot(f));
    });
    mn = (unsigned)wave_min((int)(mn ^ 0x80000000u)) ^ 0x80000000u;
    mx = (unsigned)wave_max((int)(mx ^ 0x80000000u)) ^ 0x80000000u;
    if (lane == 0) {
      red[turn][1][wave] = cnt;
      red[turn][2][wave] = (int)mn;
      red[turn][3][wave] = (int)mx;
    }
    __syncthreads();
    cnt = 0;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) {
      cnt += red[turn][1][w];
      mn = min(mn, (unsigned)red[turn][2][w]);
      mx = max(mx, (unsigned)red[turn][3][w]);
    }
    if (inside == INT_MAX) rank = go = min(go, inside = cnt);
    lo = mn;
    hi = mx;
    if (rank == 0 || rank == inside || lo == hi) break;
    const unsigned width = hi - lo;
    const int shift = max(22 - (int)__builtin_clz(width), 0);   // width >> shift < 1,024
    each_key([&](int, unsigned key, int) __attribute__((always_inline)) {
      const unsigned d = key - lo;
      if (d <= width) atomicAdd(&hist[d >> shift], 1);
    });
    __syncthreads();
    const int n_bin = hist[tid], incl = wave_scan(n_bin);
    if (lane == kWave - 1) red[turn][0][wave] = incl;
    hist[tid] = 0;
    __syncthreads();
    int below = incl - n_bin;
#pragma unroll
    for (int w = 0; w < kEvictWaves; ++w) below += w < wave ? red[turn][0][w] : 0;
    if (below < rank && rank <= below + n_bin) {   // one thread
      pick[turn][0] = tid;
      pick[turn][1] = below;
      pick[turn][2] = n_bin;
    }
    __syncthreads();
    rank -= pick[turn][1];
    inside = pick[turn][2];
    lo += (unsigned)pick[turn][0] << shift;
    hi = lo + min(hi - lo, (1u << shift) - 1u);
    turn ^= 1;
  }
  for (long long i = (long long)go + tid; i < a.max_out; i += kEvictThreads) out[i] = -1;   // max_out: up to INT32_MAX
  if (tid == 0) a.counts[s] = go;
  if (go == 0) return;

  // All entries below lo leave, and of those in [lo, hi] the first `rank` in the table's order (all of them, or
  // all equal).
  int nbelow = 0, nin = 0;
  const unsigned width = hi - lo;
  each_key([&](int, unsigned key, int) __attribute__((always_inline)) {
    nbelow += __builtin_popcountll(__ballot(key < lo));
    nin += __builtin_popcountll(__ballot(key - lo <= width));
  });
  turn ^= 1;   // of red: the other one's values may still be read
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
  unsigned gone_r = 0;   // strips whose entry leaves
  int k_at = 0;
  each_key([&](int pos, unsigned key, int slot) __attribute__((always_inline)) {
    const bool in_range = key - lo <= width;
    const unsigned long long range = __ballot(in_range);
    const bool gone = key < lo || (in_range && in + __builtin_popcountll(range & before) < rank);
    const unsigned long long leave = __ballot(gone);
    if (gone) {
      out[at + __builtin_popcountll(leave & before)] = pos;
      if (!KEEP) a.slot_pos[trow[slot / a.block_size] * a.block_size + slot % a.block_size] = -1;
    }
    if (KEEP) gone_r |= (unsigned)gone << k_at++;
    in += __builtin_popcountll(range);
    at += __builtin_popcountll(leave);
  });
  if (KEEP && GATHERED) {   // all table entries at once: one latency, not one a strip
    int blk[N];
#pragma unroll
    for (int k = 0; k < N; ++k) blk[k] = (gone_r >> k) & 1u ? trow[slot_r[k] / a.block_size] : 0;
#pragma unroll
    for (int k = 0; k < N; ++k) slot_r[k] = blk[k] * a.block_size + slot_r[k] % a.block_size;
  }
  if (KEEP) {
#pragma unroll
    for (int k = 0; k < N; ++k)
      if ((gone_r >> k) & 1u) a.slot_pos[slot_r[k]] = -1;
  }
}

template __global__ void paged_evict_lowest_kernel<4, false>(PagedEvictLowest);
template __global__ void paged_evict_lowest_kernel<16, false>(PagedEvictLowest);
template __global__ void paged_evict_lowest_kernel<16, true>(PagedEvictLowest);
template __global__ void paged_evict_lowest_kernel<0, true>(PagedEvictLowest);

static bool gathers(long long width, int block_size) { return width > 16 * kEvictThreads || (block_size < 4 && width > kEvictThreads); }

size_t paged_evict_ws_bytes(int S, int max_blocks, int block_size) {
  const long long width = (long long)max_blocks * block_size;
  return gathers(width, block_size) ? ((size_t)S * width * sizeof(int2) + 255) & ~(size_t)255 : 0;
}

hipError_t launch_paged_evict_lowest(const PagedEvictLowest& p) {
  const long long width = (long long)p.max_blocks * p.block_size;
  prof_begin("paged_evict_lowest", p.stream);
  if (gathers(width, p.block_size)) {
    const dim3 grid((unsigned)((width + kGatherThreads - 1) / kGatherThreads), (unsigned)p.S);
    hipLaunchKernelGGL(paged_gather_kernel, grid, dim3(kGatherThreads), 0, p.stream, p);
    hipLaunchKernelGGL((width <= 16 * kEvictThreads ? paged_evict_lowest_kernel<16, true> : paged_evict_lowest_kernel<0, true>),
                       dim3((unsigned)p.S), dim3(kEvictThreads), 0, p.stream, p);
  } else {
    hipLaunchKernelGGL((width <= 4 * kEvictThreads ? paged_evict_lowest_kernel<4, false> : paged_evict_lowest_kernel<16, false>),
                       dim3((unsigned)p.S), dim3(kEvictThreads), 0, p.stream, p);
  }
  prof_end(p.stream);
  return hipGetLastError();
}

}  // namespace kvs
