// gfx950 kernels of the attention of many query rows over the streamed paged
// cache: one token a sequence where sequences share the first blocks of their
// tables (rollouts of one prompt, Section 2, "KV-streams": retained entries
// stay where they are), and several new tokens a sequence (tool observations,
// drafted tokens) that see the live entries up to their own positions.  Copies
// of cache slots, for blocks that stop being shared and for compaction.
//
// For one KV head the rows of a piece of work (a job) are tokens x the G q-heads
// of the head's group; all of them see the same run of a block table, so a tile
// of its keys and values serves up to 128 rows:
//   shared prefix   rows of all the group's members, the table's first blocks
//   own part        rows of one sequence, the blocks behind its prefix
//   new tokens      rows of one sequence's tokens, its whole table
// A job is cut into row blocks of 128 and runs of tiles (units, one workgroup
// each).  A unit leaves for each row the largest score m, l = sum exp(s - m) and
// o = sum exp(s - m) V; the merge joins what belongs to a row: m = max m_i, l =
// sum l_i exp(m_i - m), o likewise, O = o / l, LSE = m + ln l.
#include "kvs_decode_plan.h"
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>

namespace kvs {

// ---------------------------------------------------------------- copies
// Slot dst[i] takes the K and V rows of slot src[i], its position and its weight; MOVE: slot src[i] is empty then.
// 16-byte pieces, one of K and one of V a thread and turn; bound by HBM: 16,000 entries of 8 KV heads at D = 128 (131 MB
// read and written) in 28 us, 4.6 TB/s where a large copy reaches 5.0.  (Several pieces a thread, asked for together, were
// slower, and pieces head by head the same.)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int D>
__global__ void __launch_bounds__(256) paged_copy_kernel(PagedCopy a) {
  const long long per = (long long)a.Hkv * (D / 8), pieces = a.n * per;
  const int num_slots = a.num_blocks * a.block_size;
  uint16_t* kc = (uint16_t*)a.k_cache;
  uint16_t* vc = (uint16_t*)a.v_cache;
  for (long long c = (long long)blockIdx.x * 256 + threadIdx.x; c < pieces; c += (long long)gridDim.x * 256) {
    const long long i = c / per;
    const int r = (int)(c - i * per), h = r / (D / 8), d8 = r - h * (D / 8);
    const int from = a.src[i], to = a.dst[i];
    if ((unsigned)from >= (unsigned)num_slots || (unsigned)to >= (unsigned)num_slots) continue;
    auto at = [&](int slot) {
      return (((long long)(slot / a.block_size) * a.Hkv + h) * a.block_size + slot % a.block_size) * D + 8 * d8;
    };
    const long long x = at(from), y = at(to);
    const u32x4 k = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kc + x));
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vc + x));
    __builtin_nontemporal_store(k, reinterpret_cast<u32x4*>(kc + y));
    __builtin_nontemporal_store(v, reinterpret_cast<u32x4*>(vc + y));
    if (r == 0) {
      if (a.slot_pos) {
        a.slot_pos[to] = a.slot_pos[from];
        if (a.move) a.slot_pos[from] = -1;
      }
      if (a.slot_weight) a.slot_weight[to] = a.slot_weight[from];
    }
  }
}

hipError_t launch_paged_copy(const PagedCopy& p) {
  if (p.n == 0) return hipSuccess;
  const long long pieces = (long long)p.n * p.Hkv * (p.D / 8);
  const unsigned grid = (unsigned)std::min<long long>((pieces + 255) / 256, 1 << 20);
  hipLaunchKernelGGL(p.D == 128 ? paged_copy_kernel<128> : paged_copy_kernel<64>, dim3(grid), dim3(256), 0, p.stream, p);
  return hipGetLastError();
}

// ---------------------------------------------------------------- the plan
// Jobs of more than 64 rows (D = 64: 32) have units of 128 rows, four waves that share a tile of keys and values, and are
// cut into equal runs; smaller ones have units of one wave.  Those are bound by HBM, so what counts is that all waves end
// together: the smaller jobs' chunks, one job's behind the other's, are dealt to the waves in equal parts, and a wave whose
// part spans jobs has a unit in each of them.  The two kinds run one after the other, each so that it fills the chip.
constexpr int kWideRows = 128;
constexpr int narrow_rows(int D) { return D == 128 ? 64 : 32; }   // most rows of a narrow job
template <int D>
constexpr int rows_bn() { return D == 128 ? 32 : 64; }   // keys of a tile of wide units
constexpr int kLeastTiles = 4;    // of a wide unit, in 32-key tiles
constexpr int kStartChunks = 2;   // what beginning a narrow job costs a wave (the latency of six reads), as chunks
constexpr int kPlanSmall = 256, kPlanGroups = 64;   // sequences and groups that one wave plans, in LDS
// A group's rows are narrow jobs, by row blocks, up to this many: reading the prefix twice, from the caches, costs less than
// a launch for wide units (40 sequences behind 114 entries, D = 64, 34 -> 26 us); four blocks of a long one more (64
// sequences behind 16,384 144 -> 165).
constexpr int kPrefixBlocks = 2;

// What the plan weighs for wide units: 128 rows of partial results, written and read, cost as much as these tiles (16
// ragged chunks are the same with 40; 64 sequences behind 16,384 entries 145 -> 149 us), and a round that fills a third or two of
// the places takes these parts of a full one, whose workgroups share their CU by threes (against parts of a half and
// three quarters, or two thirds and 0.8 as here: 2,048 tokens behind 8,192 entries, D = 64, 231 and 225 us).
constexpr float kSplitTiles = 20.f, kOneOfThree = 0.65f, kTwoOfThree = 0.8f;
constexpr int kChunk = 64;        // places of a table that are skipped or looked at together

// What a unit is, as its waves read it: the chunks k, k + n, k + 2 n, ... of the places [c0, c1) of a table, so that a run
// of places that its rows do not see falls on all units of the job alike.
struct Unit {
  int s;          // sequence whose table is read; -1: no such unit
  int c0, c1;
  int split;      // k | n << 16
  int rows;       // of the job (a group's narrow one: of its row block; a cut one: of the row blocks that are cut)
  int tok;        // first token of the job, or of its members' list
  int row0;       // first row of the unit, counted from token `tok`; | 1: token i is list[tok + i], else tok + i; | 2: other
                  // units read the same entries
  int part;       // first row of its partial results (KV head 0); -1: O and LSE are written
};
static_assert(sizeof(Unit) == 32, "two 16-byte loads");

// Partial results of a job, of its first `rows` rows: row r of KV head g and split k at part + (k Hkv + g) rows + r.
struct Parts {
  int part, rows, n;   // n: splits; 0: no partial results
};

struct RowsArgs {
  const uint16_t* q;
  const uint16_t* kc;
  const uint16_t* vc;
  const int* slot_pos;
  const int* table;
  const int* nblk;
  const int* prefix_group;    // SHARED
  const int* prefix_blocks;
  const int* q_pos;           // else
  const int* cu;
  uint16_t* o;
  float* lse;
  int S, groups, ntok, Hq, Hkv, G, max_blocks, BS, num_blocks, window, sinks;
  int shift;                  // BS = 1 << shift; -1: BS is no power of two
  int narrow;                 // narrow_rows(D)
  float scale_log2;
  // workspace
  int* rank;        // [S] SHARED: of a sequence among its group's members
  int* list;        // [S] members, group by group
  int* count;       // [groups] members, and
  int* base;        // [groups] the first of them in `list` (more than kPlanSmall sequences or groups)
  int* jobs;        // [6][jobs] tiles, rows, first wide and narrow unit, first chunk, first row block (the same)
  Parts* own;       // [S] of each sequence
  Parts* prefix;    // [groups][kPrefixBlocks] of each group's row blocks; the first one has all rows if they are wide
  Unit* units;      // [max_units[0] + max_units[1]]: wide, narrow
  int* waves;       // [max_waves + 1] first narrow unit of each wave
  float* part;      // [max_part][D]
  float2* part_ml;  // [max_part]: m (log2 units), l
  int* parts;       // [1] whether there are partial rows
  int2* stats;      // [S][ceil(max_blocks BS / kChunk)] least and greatest position in each chunk of a table (window > 0)
  long long max_part, max_split;   // rows of partial results; of those of wide jobs cut into several units
  int max_units[2], max_waves;
  int want[2];      // wide units, and waves of narrow ones, per KV head that fill the chip
};

struct Job {
  int s, c0, c1, rows, tok, row0;   // row0: with the flags of Unit
};
__device__ __forceinline__ int block_of(const RowsArgs& a, int place) { return a.shift >= 0 ? place >> a.shift : place / a.BS; }
__device__ __forceinline__ bool is_wide(const RowsArgs& a, int rows) { return rows > a.narrow; }
__device__ __forceinline__ int row_blocks(int rows) { return (rows + kWideRows - 1) / kWideRows; }   // of a wide job
// Splits of a wide job of `tiles` (at most kTileCap) under runs of c tiles.  New tokens that see nothing still have rows
// to write.
template <bool SHARED>
__device__ __forceinline__ int job_splits(const RowsArgs& a, int tiles, int rows, int c, float rc) {
  return !is_wide(a, rows) || (SHARED && tiles == 0) ? 0 : unit_count(tiles, c, rc);
}
// Chunks of a narrow job that are dealt.
template <bool SHARED>
__device__ __forceinline__ int job_chunks(const RowsArgs& a, int tiles, int rows) {
  const int n = (tiles + 1) / 2;
  return is_wide(a, rows) || rows == 0 ? 0 : SHARED ? n : max(n, 1);
}

// Prefix sums over the workgroup's NT threads, without the own value, on top of `from`, which moves on by their total.
template <int NT>
__device__ __forceinline__ long long block_scan(int x, long long& from, int* buf) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, incl = wave_scan(x);
  long long before = from + incl - x;
  if (NT == kWave) {
    from += wave_last(incl);
    return before;
  }
  __syncthreads();   // buf is read
  if (lane == kWave - 1) buf[wave] = incl;
  __syncthreads();
  for (int w = 0; w < NT / kWave; ++w) {
    before += w < wave ? buf[w] : 0;
    from += buf[w];
  }
  return before;
}

__device__ __forceinline__ int chunks_of(int places) { return (int)(((unsigned)places + kChunk - 1) / kChunk); }

// Positions in the chunks of the tables, a wave a chunk at a time: (least, greatest), of none (INT_MAX, -1).
__device__ __forceinline__ void chunk_stats(const RowsArgs& a, int first, int waves) {
  const int lane = threadIdx.x & 63, each = chunks_of(a.max_blocks * a.BS);
  for (long long i = first; i < (long long)a.S * each; i += waves) {
    const int s = (int)(i / each), c = (int)(i - (long long)s * each) * kChunk + lane;
    const int n = min(max(a.nblk[s], 0), a.max_blocks) * a.BS, b = block_of(a, c);
    const int e = c < n ? a.table[(size_t)s * a.max_blocks + b] : -1;
    const int p = (unsigned)e < (unsigned)a.num_blocks ? a.slot_pos[e * a.BS + (c - b * a.BS)] : -1;
    const int lo = wave_min(p < 0 ? INT_MAX : p), hi = wave_max(p);
    if (lane == 0) a.stats[i] = make_int2(lo, hi);
  }
}

// The plan, by workgroup 0: for up to 256 sequences and groups one wave makes it, with what it knows of them in LDS, and
// all of them try the sizes of wide jobs' runs and write the units.  Bound by latency: 5 us for 4 sequences, 11 for 64 of
// one group, 30 for 256 of 64 groups.  Beyond that the counts are in global memory, and each group among 64 sequences is a
// round trip there: 104 us for 512 shuffled sequences of 64 groups, 224 for 1,024 of 128.  Under a window the other workgroups take the positions of the tables' chunks.
template <bool SHARED, bool SMALL>
__global__ void __launch_bounds__(SMALL ? 512 : 1024) rows_plan_kernel(RowsArgs a) {
  constexpr int NT = SMALL ? 512 : 1024, PT = SMALL ? kWave : NT;   // threads; those that plan
  constexpr int CAP = SMALL ? kPlanSmall : 1, JOBS = SHARED && SMALL ? kPrefixBlocks * kPlanGroups + CAP : CAP;
  __shared__ int sJobs[6 * JOBS], sGroup[SHARED ? 6 * CAP + kPlanGroups : 1], sPart[JOBS], sSplits[JOBS];
  __shared__ Job sJob[JOBS];
  constexpr int NW = NT / kWave, TRIES = SHARED ? 16 : 24;
  __shared__ int buf[PT / kWave], sTop[PT / kWave], sTopWide, sUnits[2], sSize[TRIES], sWhole[TRIES];
  __shared__ long long sLeast, sWork, sChunks;
  __shared__ float sCost[TRIES];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, GJ = SHARED ? kPrefixBlocks * a.groups : 0, J = GJ + a.S;
  if (blockIdx.x > 0) {
    chunk_stats(a, (blockIdx.x - 1) * (NT / kWave) + wave, (gridDim.x - 1) * (NT / kWave));
    return;
  }
  int* tiles = SMALL ? sJobs : a.jobs;
  int* rows = SMALL ? sJobs + JOBS : a.jobs + J;
  // units of the jobs in front of each, wide and narrow ones counted apart
  int* first[2] = {SMALL ? sJobs + 2 * JOBS : a.jobs + 2 * J, SMALL ? sJobs + 3 * JOBS : a.jobs + 3 * J};
  // where each narrow job's first chunk lies among all that is dealt
  int* chunk = SMALL ? sJobs + 4 * JOBS : a.jobs + 4 * J;
  int* block = SMALL ? sJobs + 5 * JOBS : a.jobs + 5 * J;   // row blocks of the wide jobs in front of each
  int* count = SMALL ? sGroup : a.count;
  int* base = SMALL ? sGroup + CAP : a.base;
  int* rank = SMALL ? sGroup + 2 * CAP : a.rank;
  int* list = SMALL ? sGroup + 3 * CAP : a.list;
  int* sBlocks = sGroup + 4 * CAP;   // SMALL: a sequence's blocks and group, read once
  int* sOf = sGroup + 5 * CAP;
  int* sCommon = sGroup + 6 * CAP;   // SMALL: prefix_blocks
  auto sync = [&]() {
    if (SMALL) {   // one wave, whose accesses to LDS take place in order
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    } else {
      __syncthreads();
    }
  };
  auto blocks_of = [&](int s) { return SMALL && SHARED ? sBlocks[s] : min(max(a.nblk[s], 0), a.max_blocks); };
  auto group_of = [&](int s) { return SMALL ? sOf[s] : a.prefix_group[s]; };
  // blocks of group g's prefix
  auto prefix_of = [&](int g) {
    return count[g] < 2 ? 0 : min(max(SMALL ? sCommon[g] : a.prefix_blocks[g], 0), blocks_of(list[base[g]]));
  };
  // job j: the groups first, then the sequences
  auto job_of = [&](int j) {
    if (SHARED && j < GJ) {
      const int g = j / kPrefixBlocks, rb = j % kPrefixBlocks, b = prefix_of(g), all = b ? count[g] * a.G : 0;
      const bool wide = all > kPrefixBlocks * a.narrow;
      const int r = wide ? (rb == 0 ? all : 0) : min(max(all - rb * a.narrow, 0), a.narrow);
      if (r == 0) return Job{0, 0, rb == 0 ? b * a.BS : 0, 0, 0, 0};
      return Job{list[base[g]], 0, b * a.BS, r, base[g], rb * a.narrow | 1 | (all > a.narrow ? 2 : 0)};
    }
    const int s = j - GJ, blocks = blocks_of(s);
    if (SHARED) {
      const int g = group_of(s);
      int b = 0;
      if ((unsigned)g < (unsigned)a.groups) b = min(SMALL ? sJob[kPrefixBlocks * g].c1 / a.BS : prefix_of(g), blocks);
      return Job{s, b * a.BS, blocks * a.BS, a.G, s, 0};
    }
    const int t0 = min(max(a.cu[s], 0), a.ntok), t1 = min(max(a.cu[s + 1], t0), a.ntok);
    return Job{s, 0, blocks * a.BS, (t1 - t0) * a.G, t0, 0};
  };
  if (!SMALL || wave == 0) {
    if (SHARED) {
      for (int g = tid; g < a.groups; g += PT) count[g] = 0;
      if (SMALL) {
        constexpr int N = SMALL ? CAP / PT : 1;
        int nb[N], gr[N];   // all reads at once
        const int common = tid < a.groups ? a.prefix_blocks[tid] : 0;
#pragma unroll
        for (int k = 0; k < N; ++k) {
          nb[k] = k * PT + tid < a.S ? a.nblk[k * PT + tid] : 0;
          gr[k] = k * PT + tid < a.S ? a.prefix_group[k * PT + tid] : -1;
        }
#pragma unroll
        for (int k = 0; k < N; ++k) {
          sBlocks[k * PT + tid] = min(max(nb[k], 0), a.max_blocks);
          sOf[k * PT + tid] = gr[k];
        }
        sCommon[tid] = common;
      }
      sync();
      if (wave == 0)   // ranks in the sequences' order: 64 of them at a time, group by group of those among them
        for (int s0 = 0; s0 < a.S; s0 += kWave) {
          const int s = s0 + lane, g = s < a.S ? group_of(s) : -1;
          unsigned long long todo = __ballot((unsigned)g < (unsigned)a.groups);
          while (todo) {
            const int g1 = __builtin_amdgcn_readlane(g, __builtin_ctzll(todo));
            const unsigned long long same = __ballot(g == g1);
            const int before = count[g1];
            if (g == g1) rank[s] = before + __builtin_popcountll(same & ((1ull << lane) - 1ull));
            if (lane == 0) count[g1] = before + __builtin_popcountll(same);
            if (SMALL) sync();
            else __threadfence_block();
            todo &= ~same;
          }
        }
      sync();
      long long from = 0;
      for (int g0 = 0; g0 < a.groups; g0 += PT) {
        const int g = g0 + tid;
        const int x = (int)block_scan<PT>(g < a.groups ? count[g] : 0, from, buf);
        if (g < a.groups) base[g] = x;
      }
      sync();
      for (int s = tid; s < a.S; s += PT) {
        const int g = group_of(s);
        if ((unsigned)g < (unsigned)a.groups) {
          const int i = base[g] + rank[s];
          list[i] = s;
        }
      }
      sync();
    }
    int top = 1;
    long long least = 0, work = 0, chunks = 0;   // row blocks and tiles of all wide jobs; chunks of all narrow ones
    // the groups in turns of their own: the sequences' jobs begin where they end
    for (int j0 = 0; j0 < J; j0 += PT) {
      const int ends = j0 < GJ ? min(GJ, j0 + PT) : min(J, j0 + PT), j = j0 + tid;
      const bool mine = j < ends;
      const Job x = mine ? job_of(j) : Job{0, 0, 0, 0, 0, 0};
      const bool wide = is_wide(a, x.rows);
      int places = x.rows ? x.c1 - x.c0 : 0;
      // by all the job's tokens: by a row block's own, eight windowed chunks are cut less, and 110 us become 119
      if (!SHARED && a.window > 0) places = (int)min((long long)places, (long long)a.window + a.sinks + x.rows / a.G);
      const int t = wide ? plan_tiles(places) : (int)(((unsigned)places + 31) / 32);
      if (mine) {
        tiles[j] = t;
        rows[j] = x.rows;
        if (SMALL) sJob[j] = x;
      }
      top = max(top, wide ? t : 0);
      const long long rb0 = block_scan<PT>(wide ? row_blocks(x.rows) : 0, least, buf);
      block_scan<PT>(wide ? (int)min((long long)row_blocks(x.rows) * t, 1ll << 24) : 0, work, buf);
      const int m = job_chunks<SHARED>(a, t, x.rows), begin = m > 0 ? kStartChunks : 0;
      const long long c0 = block_scan<PT>(m + begin, chunks, buf) + begin;
      if (mine) {
        chunk[j] = (int)min(c0, (long long)INT_MAX);
        block[j] = (int)min(rb0, (long long)INT_MAX);
      }
      if (j0 < GJ) {
        j0 = ends - PT;
        sync();
      }
    }
    top = wave_max(top);
    if (lane == 0) sTop[wave] = top;
    sync();
    for (int w = 0; w < PT / kWave; ++w) top = max(top, sTop[w]);
    if (tid == 0) {
      sTopWide = top;
      sLeast = least;
      sWork = work;
      sChunks = chunks;
    }
  }
  __syncthreads();
  // How wide jobs are cut, in tiles of the time that a place on the chip has: all of them into runs of one size, the whole
  // of the longest, which always fits, or a part of it; or, for new tokens, the row blocks that fill whole rounds left
  // whole and those behind them cut, so that few rows have partial results and yet the last round is short.  Units of one
  // size end by rounds, and where they are smaller than the largest the last ones half of what they lack later.  (By the
  // work's share and half a unit more: 4 chunks of 500 to 900 tokens 144 -> 162 us, 2,048 tokens at D = 64 225 -> 250, 16
  // ragged chunks 543 -> 558.)  A wave a cut at a time.
  int C = sTopWide, whole = 0;   // row blocks left whole
  // of a wide job: its row blocks that are cut (the first ones: a causal row block's last rows see most), and into how many
  auto cut_of = [&](int j, int c, float rc, int front, int& n) {
    const int r = rows[j], nb = is_wide(a, r) ? row_blocks(r) : 0, b = nb - min(max(front - block[j], 0), nb);
    n = b ? job_splits<SHARED>(a, tiles[j], r, c, rc) : 0;
    return b;
  };
  if (sLeast > 0) {
    const long long rounds = sLeast / a.want[0];
    for (int i = wave; i < (rounds > 0 ? TRIES : 16); i += NW) {
      const int k = i < 16 ? i : i - 15;
      const int n = k < 4 ? k + 1 : k & 1 ? 4 << ((k - 3) >> 1) : 6 << ((k - 4) >> 1);   // 1 .. 4, 6, 8, 12, 16, 24, ...
      const int c = (sTopWide + n - 1) / n, front = i < 16 ? 0 : (int)min(rounds * a.want[0], (long long)INT_MAX);
      const float rc = __builtin_amdgcn_rcpf((float)c), place = 1.f / (float)a.want[0];
      long long units = 0, split = 0, left = 0;   // behind those left whole; rows of partial results; tiles of those left whole
      for (int j0 = 0; j0 < J; j0 += kWave) {
        const int j = j0 + lane;
        int m = 0;
        const int b = j < J ? cut_of(j, c, rc, front, m) : 0;
        units += wave_last(wave_scan((int)min((long long)m * b, 1ll << 24)));   // more than there may be at any rate
        if (!SHARED && front > 0) {
          const int nb = j < J && is_wide(a, rows[j]) ? row_blocks(rows[j]) - b : 0;
          left += wave_last(wave_scan(nb > 0 ? (int)min((long long)nb * tiles[j], 1ll << 24) : 0));
        }
        split += wave_last(wave_scan(m > 1 ? (int)min((long long)m * min(rows[j], b * kWideRows), 1ll << 24) : 0));
      }
      if (lane == 0) {
        const float u = (float)units * place, full = floorf(u + 1e-3f), rest = u - full;   // rounds
        const float last = rest < 1e-3f ? 0.f : rest < 0.334f ? kOneOfThree : rest < 0.667f ? kTwoOfThree : 1.f;
        const float mean = units > 0 ? (float)(sWork - left) * __builtin_amdgcn_rcpf((float)units) : 0.f;
        const float least = (full > 0.f ? 1.f : last) * (float)c;
        const float ends = (float)left * place + fmaxf(least, (full + last) * mean + 0.5f * ((float)c - mean));
        sSize[i] = c;
        sWhole[i] = front;
        const bool fits = front + units <= a.max_units[0] && split <= a.max_split;
        sCost[i] = !fits || (n > 1 && c < kLeastTiles) || (i >= 16 && front == sLeast)
                       ? INFINITY
                       : ends + (float)split * (kSplitTiles / kWideRows) * place;
      }
    }
    __syncthreads();
    float best = INFINITY;
    for (int i = 0; i < (rounds > 0 ? TRIES : 16); ++i)
      if (sCost[i] < best) {
        best = sCost[i];
        C = sSize[i];
        whole = sWhole[i];
      }
  }
  const float rC = __builtin_amdgcn_rcpf((float)C);
  const int per = (int)max(1ll, (sChunks + a.want[1] - 1) / a.want[1]);   // of a wave
  auto wave_of = [&](int x) { return (int)((unsigned)x / (unsigned)per); };   // of all that is dealt, less than 2^31
  if (!SMALL || wave == 0) {
    // first units of the jobs, wide and narrow ones counted apart, and their first partial rows
    long long units0[2] = {0, 0}, part0 = 0;
    for (int j0 = 0; j0 < J; j0 += PT) {
      const int j = j0 + tid, r = j < J ? rows[j] : 0, t = j < J ? tiles[j] : 0, m = job_chunks<SHARED>(a, t, r);
      int nw = 0;
      const int b = j < J ? cut_of(j, C, rC, whole, nw) : 0, nb = is_wide(a, r) ? row_blocks(r) : 0;
      const int nn = m > 0 ? wave_of(chunk[j] + m - 1) - wave_of(chunk[j]) + 1 : 0, n = nw + nn;
      const int cut_rows = nb ? min(r, b * kWideRows) : r;
      const long long uw = block_scan<PT>(nb - b + nw * b, units0[0], buf);
      const long long un = block_scan<PT>(nn, units0[1], buf);
      const long long pn = block_scan<PT>(SHARED || n > 1 ? n * cut_rows : 0, part0, buf);
      if (j < J) {
        first[0][j] = (int)min(uw, (long long)INT_MAX);
        first[1][j] = (int)min(un, (long long)INT_MAX);
        const Parts parts = {(int)(pn * a.Hkv), cut_rows, SHARED || n > 1 ? n : 0};
        if (SMALL) {   // stored below
          sPart[j] = parts.part;
          sSplits[j] = parts.n;
        } else {
          (j < GJ ? a.prefix[j] : a.own[j - GJ]) = parts;
        }
      }
    }
    // offsets that overlap (only where cu_seqlens decreases) may ask for more than there is: nothing is computed then
    const bool fit = units0[0] <= a.max_units[0] && units0[1] <= a.max_units[1] && part0 * a.Hkv <= a.max_part;
    if (tid == 0) {
      a.parts[0] = fit && part0 > 0;
      sUnits[0] = fit ? (int)units0[0] : 0;
      sUnits[1] = fit ? (int)units0[1] : 0;
    }
  }
  __syncthreads();
  if (SMALL) {   // what the merge reads
    for (int j = tid; j < J; j += NT) {
      int n;
      const int b = cut_of(j, C, rC, whole, n), r = rows[j];
      (j < GJ ? a.prefix[j] : a.own[j - GJ]) = {sPart[j], is_wide(a, r) ? min(r, b * kWideRows) : r, sSplits[j]};
    }
    for (int s = tid; SHARED && s < a.S; s += NT) {
      const int g = group_of(s);
      if ((unsigned)g < (unsigned)a.groups) {
        a.list[base[g] + rank[s]] = s;
        a.rank[s] = rank[s];
      }
    }
  }
  // the last job that begins at or before x: those without one of these begin where the next one does
  auto search = [&](const int* begin, int x) {
    int j = 0;
    for (int step = 1 << (31 - __builtin_clz(J)); step > 0; step >>= 1)
      if (j + step < J && begin[j + step] <= x) j += step;
    return j;
  };
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int all = sUnits[k];
    Unit* out = a.units + (k == 0 ? 0 : a.max_units[0]);
    for (int u = tid; u < a.max_units[k]; u += NT) {
      if (u >= all) {
        out[u].s = -1;
        continue;
      }
      const int j = search(first[k], u), i = u - first[k][j];
      const Job b = SMALL ? sJob[j] : job_of(j);
      const int part = SMALL ? sPart[j] : j < GJ ? a.prefix[j].part : a.own[j - GJ].part;
      int c0 = b.c0, c1 = b.c1, sp = 0, n, row0 = b.row0, job_rows = b.rows;
      if (k == 0) {   // the last rows first: they see most
        const int nb = row_blocks(b.rows), cut = cut_of(j, C, rC, whole, n), x = i - (nb - cut);
        if (x < 0) {
          n = 1;
          row0 |= (nb - 1 - i) * kWideRows;
        } else {
          sp = cut == 1 ? x : x / cut;
          row0 |= (cut - 1 - (x - sp * cut)) * kWideRows;
          job_rows = min(job_rows, cut * kWideRows);
        }
      } else {
        const int m = job_chunks<SHARED>(a, tiles[j], b.rows), w = wave_of(chunk[j]);
        n = wave_of(chunk[j] + m - 1) - w + 1;
        sp = i;
      }
      const int split = k == 1 && (SHARED || a.window == 0) ? 1 << 16 : sp | n << 16;
      if (k == 1 && (SHARED || a.window == 0)) {   // the part of wave w + i; under a window an equal part of the chunks
        const long long x = (long long)(wave_of(chunk[j]) + i) * per - chunk[j];
        c1 = (int)min((long long)c1, c0 + (x + per) * kChunk);
        c0 = (int)min((long long)c1, c0 + max(x, 0ll) * kChunk);
      }
      out[u] = {b.s, c0, c1, split, job_rows, b.tok, row0, SHARED || n > 1 ? part + sp * a.Hkv * job_rows : -1};
    }
  }
  for (int w = tid; w <= a.max_waves; w += NT) {
    const long long x = (long long)w * per;
    int u = sUnits[1];
    if (u > 0 && x < sChunks) {
      const int j = search(chunk, (int)x);
      const int m = job_chunks<SHARED>(a, tiles[j], rows[j]);
      u = first[1][j];
      if (m > 0 && chunk[j] <= x)   // within the job, or behind it, where the next one begins
        u += min(w, wave_of(chunk[j] + m - 1) + 1) - wave_of(chunk[j]);
    }
    a.waves[w] = u;
  }
}

// ---------------------------------------------------------------- the units
// A row of a unit (lane % 32 of a wave) and what it sees: the entry at position p iff p <= at and (at - p < window or
// p < sinks); SHARED: every live entry.
struct RowLane {
  int tok, h, at;
  bool ok;
};
template <bool SHARED>
__device__ __forceinline__ RowLane row_of(const RowsArgs& a, const Unit& un, int g, int row, int last) {
  const int r = min(row, last), i = r / a.G;   // lanes past the last row repeat it
  RowLane x;
  x.tok = un.row0 & 1 ? a.list[un.tok + i] : un.tok + i;
  x.h = g * a.G + r - i * a.G;
  x.at = SHARED ? INT_MAX - 1 : min(max(a.q_pos[x.tok], -1), INT_MAX - 1);   // INT_MAX is nobody's
  x.ok = row <= last;
  return x;
}
template <bool SHARED>
__device__ __forceinline__ bool seen(const RowsArgs& a, int p, int at) {
  return p <= at && (SHARED || a.window == 0 || at - p < a.window || p < a.sinks);
}
// Whether some row at a position in [lo, hi] may see the entry at p (-1: there is none).
template <bool SHARED>
__device__ __forceinline__ bool seen_by_some(const RowsArgs& a, int p, int lo, int hi) {
  return p >= 0 && (SHARED || (p <= hi && (a.window == 0 || lo - p < a.window || p < a.sinks)));
}

// The chunks of a unit that its rows (at positions in [lo, hi]) may see something of, 64 of the unit's at a time as a
// mask; wave-uniform.
template <bool SHARED>
struct ChunkWalker {
  unsigned long long mask;
  int ord, ords, at, k, n;   // next of the unit's chunks; their number; the mask's first one
  __device__ __forceinline__ void init(const Unit& un) {
    k = un.split & 0xffff;
    n = un.split >> 16;
    const int chunks = chunks_of(un.c1 - un.c0);
    ords = chunks > k ? (chunks - k + n - 1) / n : 0;
    ord = at = 0;
    mask = 0;
  }
  // the next 64
  __device__ __forceinline__ void look(const RowsArgs& a, const Unit& un, int lo, int hi, int lane) {
    at = ord;
    bool see = ord + lane < ords;
    if (!SHARED && a.window > 0 && see) {
      const int2 p = a.stats[(size_t)un.s * chunks_of(a.max_blocks * a.BS) + (ord + lane) * n + k];
      see = p.x <= hi && (p.y > lo - a.window || p.x < a.sinks);
    }
    mask = __ballot(see);
    ord += 64;
  }
  // whether there is another one
  __device__ __forceinline__ bool more(const RowsArgs& a, const Unit& un, int lo, int hi, int lane) {
    while (mask == 0 && ord < ords) look(a, un, lo, hi, lane);
    return mask != 0;
  }
  // the place of the table that the next one begins at; past the unit's last place if there is none
  __device__ __forceinline__ int next(const Unit& un) {
    const int c = un.c0 + ((at + __builtin_ctzll(mask | 1ull << 63)) * n + k) * kChunk;
    const bool some = mask != 0;
    mask &= mask - 1ull;
    return some ? c : un.c1;
  }
};

// The running softmax of 32 rows (a lane's column) and their sums of V, relative to 2^m.  The probabilities are bf16 in
// the products.  OWN: each tile's are relative to its largest score, times a power of two, so that the largest ones, which
// weigh most, are exact; m then moves with every tile, within half a step of the row's maximum.  Narrow units, bound by
// HBM, do that: O of 16 rollouts behind 4,096 entries is 2.30e-3 -> 2.03e-3 off the 64-bit result, as the decode of one
// sequence's, for 37.4 -> 38.8 us; wide ones, whose vector units are as busy as their matrix cores, do not.
template <int D, bool OWN>
struct RowState {
  static constexpr int DB = D / 32;
  f32x16 acc[DB];
  float m, l;   // reference (log2 units), sum
  float top;    // OWN: the row's maximum
  __device__ __forceinline__ void init() {
#pragma unroll
    for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
    m = top = -INFINITY;
    l = 0.f;
  }
  // NKB blocks of 32 keys: masked scores become their exponentials.  Not OWN: m moves only when a score exceeds it by
  // more than 8 (log2 units): probabilities are at most 2^8 then, and bf16 keeps their relative precision.
  template <int NKB>
  __device__ __forceinline__ void weigh(f32x16 (&s)[NKB], float scale_log2) {
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    if (OWN || __ballot(mx * scale_log2 > m + 8.f)) {
      float m_new = fmaxf(mx, wave_xor32(mx)) * scale_log2;
      if (OWN) {
        top = fmaxf(top, m_new);
        m_new = m_new == -INFINITY ? m : m_new + rintf(top - m_new);
      } else {
        m_new = fmaxf(m, m_new);
      }
      const float alpha = m_new == m ? 1.f : __builtin_amdgcn_exp2f(m - m_new);
      l *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
      m = m_new;
    }
    const float use = m == -INFINITY ? 0.f : m;   // 0 until the row has seen an entry
    float ls = 0.f;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], scale_log2, -use));
        s[kb][r] = e;
        ls += e;
      }
    l += ls;
  }
  // O and LSE, or the partial results, of row `row`.
  __device__ __forceinline__ void finish(const RowsArgs& a, const Unit& un, const RowLane& rw, int g, int row, int half) {
    const float sum = halves_sum(l);
    if (!rw.ok) return;
    if (un.part < 0) {
      const float inv = sum <= 0.f ? 0.f : 1.f / sum;
      uint16_t* orow = a.o + ((size_t)rw.tok * a.Hq + rw.h) * D;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<uint2*>(orow + 32 * d + 8 * q4 + 4 * half) = pack4_bf16(
              acc[d][4 * q4] * inv, acc[d][4 * q4 + 1] * inv, acc[d][4 * q4 + 2] * inv, acc[d][4 * q4 + 3] * inv);
      if (half == 0)
        a.lse[(size_t)rw.tok * a.Hq + rw.h] = sum <= 0.f ? -INFINITY : (m + __log2f(sum)) * 0.6931471805599453f;
      return;
    }
    const size_t pidx = (size_t)un.part + (size_t)g * un.rows + row;
    float* dst = a.part + pidx * D;
    if (!(sum <= 0.f)) {   // else O is left unwritten (the merge skips it)
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4)
          *reinterpret_cast<float4*>(dst + 32 * d + 8 * q4 + 4 * half) =
              make_float4(acc[d][4 * q4], acc[d][4 * q4 + 1], acc[d][4 * q4 + 2], acc[d][4 * q4 + 3]);
    }
    if (half == 0) a.part_ml[pidx] = make_float2(m, sum);
  }
};

constexpr int kWidePick = 512;   // places of the table that a wide unit looks at together (more, and its loop spills registers)

// A wide unit walks its chunks of the table 512 places at a time: the slots that some row of it sees go to a list in LDS
// (two dependent reads, for all places at once), and the keys and values of the listed slots are gathered tile by tile,
// double-buffered, each tile read by the four waves.  Scores are S^T = K Q^T (keys on M, rows on N), so that a lane holds 16
// scores of one row; softmax and the products with V as in the forward of the eviction mask.  Three workgroups a CU, whose
// registers just do without spills.  Bound by the matrix cores at the clock their power leaves, as that forward: 4,096
// tokens of 32 q-heads over 20,480 entries (D = 128) 1.21 ms, 993 TFLOP/s, 0.91 of that forward's rate over a trace of 16,384
// in turns with it, matrix cores busy 52% at 1.85 GHz.  Asking for
// the next 512 places while the tiles of the last ones are computed, by copies to LDS, made that 5% slower.
// FAR: caches of 4 GiB or more, whose rows need 64-bit addresses of their own; else a copy takes one addition.
template <int D, bool SHARED, bool FAR>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3))) rows_wide_kernel(RowsArgs a) {
  using LY = Lay<D, true>;
  constexpr int KS = D / 16, BN = rows_bn<D>(), NKB = BN / 32, PITCH = LY::PITCH, TILE = BN * PITCH;
  constexpr int PIECES = BN * LY::CPRP / kWave, PW = (PIECES + 3) / 4, PICK = kWidePick, LOOK = PICK / 256;
  static_assert(BN * LY::CPRP % kWave == 0, "tile must fill whole 64-slot pieces");
  __shared__ __attribute__((aligned(1024))) uint16_t sK0[TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sK1[TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV0[TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV1[TILE];
  // rows [block][KV head][row] of the listed slots (not FAR: in bytes), and their positions; INT_MAX: nothing there
  __shared__ __attribute__((aligned(16))) uint32_t sRow[PICK];
  __shared__ __attribute__((aligned(16))) int sPos[PICK];
  __shared__ int sCnt[LOOK * 4], sAll[4], sMin[4], sMax[4];

  const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5, col = lane & 31;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int uidx = blockIdx.x / a.Hkv, g = blockIdx.x - uidx * a.Hkv;
  const Unit un = a.units[uidx];
  if (un.s < 0) return;
  const auto rl = LY::row_lane(lane);
  const int tl = LY::tr_lo(lane), th = LY::tr_hi(lane);
  const int row0 = (un.row0 & ~3) + 32 * wave, row = row0 + col;
  const bool wave_ok = row0 < un.rows;
  int at;   // this lane's row sees entries up to there
  bf16x8 qreg[KS];
  {
    const RowLane rw = row_of<SHARED>(a, un, g, row, un.rows - 1);
    at = rw.at;
    const uint16_t* qrow = a.q + ((size_t)rw.tok * a.Hq + rw.h) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + 16 * ks));
  }
  const int wlo = SHARED ? at : wave_min(at), whi = SHARED ? at : wave_max(at);
  int lo = wlo, hi = whi;
  if (!SHARED) {
    if (lane == 0) {
      sMin[wave] = wlo;
      sMax[wave] = whi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if ((un.row0 & ~3) + 32 * w < un.rows) {
        lo = min(lo, sMin[w]);
        hi = max(hi, sMax[w]);
      }
    lo = __builtin_amdgcn_readfirstlane(lo);
    hi = __builtin_amdgcn_readfirstlane(hi);
  }
  RowState<D, false> st;
  st.init();
  const int* trow = uniform_ptr(a.table + (size_t)un.s * a.max_blocks);

  // Copies of tile t: this lane's 16-byte slots of it are (wave + 4 i) 64 + lane.  Their tile rows (times 4) and byte
  // offsets in the source rows, packed: a register more and the loop spills, whose reloads wait for the copies.
  uint32_t piece[PW];
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int qs = (wave + 4 * i) * kWave + lane, r = min(qs / LY::CPRP, BN - 1), pc = qs - qs / LY::CPRP * LY::CPRP;
    piece[i] = 4u * r | (pc < LY::CPR ? 16u * (pc ^ LY::flip(r)) : 0u) << 16;
  }
  auto stage = [&](uint16_t* sK, uint16_t* sV, int t) __attribute__((always_inline)) {
    const uint32_t lk = lds_addr(sK) + wave * kWave * 16, lv = lds_addr(sV) + wave * kWave * 16;
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int n = wave + 4 * i;
      if (i < PW - 1 || PIECES % 4 == 0 || n < PIECES) {
        const uint32_t r = *reinterpret_cast<const uint32_t*>(reinterpret_cast<const char*>(sRow + t * BN) + (piece[i] & 0xffffu));
        if (FAR) {
          const size_t off = (size_t)r * (2 * D) + (piece[i] >> 16);
          dma_b128_cached((const char*)a.kc + off, lk + i * 4 * kWave * 16);
          dma_b128_cached((const char*)a.vc + off, lv + i * 4 * kWave * 16);
        } else {
          const uint32_t off = r + (piece[i] >> 16);
          dma_b128(a.kc, off, lk + i * 4 * kWave * 16);
          dma_b128(a.vc, off, lv + i * 4 * kWave * 16);
        }
      }
    }
  };
  // `all`: every row of the workgroup sees every entry of the tile
  auto compute = [&](const uint16_t* cK, const uint16_t* cV, int t, bool all) __attribute__((always_inline)) {
    f32x16 s[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      s[kb] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[kb] = mfma32(lds_read_b128(cK + 32 * kb * PITCH + LY::row_at(rl, ks)), qreg[ks], s[kb]);
    }
    if (!all) {
      const int p = sPos[t * BN + (BN == 64 ? lane : col)];
      if (__ballot(seen<SHARED>(a, p, wlo) && seen<SHARED>(a, p, whi)) != ~0ull) {
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int q4 = 0; q4 < 4; ++q4) {
            const int4 e = *reinterpret_cast<const int4*>(&sPos[t * BN + 32 * kb + 8 * q4 + 4 * half]);
            if (!seen<SHARED>(a, e.x, at)) s[kb][4 * q4] = -INFINITY;
            if (!seen<SHARED>(a, e.y, at)) s[kb][4 * q4 + 1] = -INFINITY;
            if (!seen<SHARED>(a, e.z, at)) s[kb][4 * q4 + 2] = -INFINITY;
            if (!seen<SHARED>(a, e.w, at)) s[kb][4 * q4 + 3] = -INFINITY;
          }
      }
    }
    st.template weigh<NKB>(s, a.scale_log2);
    __builtin_amdgcn_s_setprio(3);   // the products with V run back to back while other waves weigh
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const bf16x8 pb = pack8(s[kb], 8 * t2);
#pragma unroll
        for (int d = 0; d < D / 32; ++d)
          st.acc[d] = mfma32(tr_operand<D, true>(cV, 32 * kb + 16 * t2, 32 * d, tl, th), pb, st.acc[d]);
      }
    __builtin_amdgcn_s_setprio(0);
  };

  ChunkWalker<SHARED> walk;
  walk.init(un);
  bool again = false;
  while (walk.ord < walk.ords) {
    walk.look(a, un, lo, hi, lane);
    for (; walk.mask; again = true) {
      // the slots of the next places that some row sees, in the table's order
      int slot[LOOK], pos[LOOK], blk[LOOK];
      unsigned long long vis[LOOK];
#pragma unroll
      for (int k = 0; k < LOOK; ++k) {
        int c = un.c1;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int x = walk.next(un);
          if (w == wave) c = x;
        }
        c += lane;
        const int b = block_of(a, c);
        blk[k] = c < un.c1 ? trow[b] : -1;
        slot[k] = (unsigned)blk[k] < (unsigned)a.num_blocks ? blk[k] * a.BS + (c - b * a.BS) : -1;
      }
#pragma unroll
      for (int k = 0; k < LOOK; ++k) pos[k] = slot[k] >= 0 ? a.slot_pos[slot[k]] : -1;
      if (again) __syncthreads();   // the lists are read
      int all = 0;
#pragma unroll
      for (int k = 0; k < LOOK; ++k) {
        vis[k] = __ballot(seen_by_some<SHARED>(a, pos[k], lo, hi));
        if (!SHARED) all += __builtin_popcountll(vis[k] & __ballot(seen<SHARED>(a, pos[k], lo) && seen<SHARED>(a, pos[k], hi)));
        if (lane == 0) sCnt[k * 4 + wave] = __builtin_popcountll(vis[k]);
      }
      if (!SHARED && lane == 0) sAll[wave] = all;
      __syncthreads();
      int cnt = 0, mine[LOOK];
#pragma unroll
      for (int k = 0; k < LOOK; ++k)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          if (w == wave) mine[k] = cnt;
          cnt += sCnt[k * 4 + w];
        }
      cnt = __builtin_amdgcn_readfirstlane(cnt);
      if (cnt == 0) continue;
      const bool full = SHARED || __builtin_amdgcn_readfirstlane(sAll[0] + sAll[1] + sAll[2] + sAll[3]) == cnt;
      const int ntile = (cnt + BN - 1) / BN, last = cnt % BN ? ntile - 1 : ntile;   // the tile that is not full
#pragma unroll
      for (int k = 0; k < LOOK; ++k)
        if ((vis[k] >> lane) & 1ull) {
          const int i = mine[k] + __builtin_popcountll(vis[k] & ((1ull << lane) - 1ull));
          const uint32_t r = (((uint32_t)blk[k] * a.Hkv + g) * a.BS + (slot[k] - blk[k] * a.BS)) * (FAR ? 1u : 2u * D);
          sRow[i] = r;
          sPos[i] = SHARED ? 0 : pos[k];
          if (i == cnt - 1)   // the last tile's places behind it repeat it, and nobody sees them
            for (int x = cnt; x < ntile * BN; ++x) {
              sRow[x] = r;
              sPos[x] = INT_MAX;
            }
        }
      __syncthreads();
      auto step = [&](uint16_t* cK, uint16_t* cV, uint16_t* nK, uint16_t* nV, int t) __attribute__((always_inline)) {
        wait_vm();
        __syncthreads();   // tile t is there, and nobody reads tile t - 1 any more
        if (t + 1 < ntile) stage(nK, nV, t + 1);
        if (t == last) {   // V of the places behind the last entry: their factor is 0, and must stay it
          const int n = cnt - t * BN;
          for (int x = tid; x < (BN - n) * (PITCH / 2); x += 256) reinterpret_cast<uint32_t*>(cV + n * PITCH)[x] = 0u;
          __syncthreads();
        }
        if (wave_ok) compute(cK, cV, t, full && t != last);
      };
      stage(sK0, sV0, 0);
      for (int t = 0;;) {
        step(sK0, sV0, sK1, sV1, t);
        if (++t >= ntile) break;
        step(sK1, sV1, sK0, sV0, t);
        if (++t >= ntile) break;
      }
    }
  }
  st.finish(a, un, row_of<SHARED>(a, un, g, row, un.rows - 1), g, row, half);
}

// A narrow unit, 64 rows at most (D = 64: 32, where two columns' registers would leave half the waves a CU), is one wave,
// with its own tiles of 32 entries (double-buffered; D = 128: 40 KB of LDS, so that four share a CU, one a SIMD).  Every
// global read of its loop is a copy to LDS, so all of them complete in
// issue order under one counter: step n issues the K and V copies of tile n + 1, waits until only these are
// outstanding, asks for the next piece of what the tiles after it need, and computes tile n.  That is, for 192 places
// of the table at a time, in consecutive steps: their table entries; the positions of the slots these name; and, when
// the list of slots to gather runs short, the slots that some row sees are added to it (a ring of 256).  Bound by HBM where
// jobs are long: 4 tokens of each of 64 sequences behind 1,000 to 8,000 entries (1.14 GB) 190 us, 6.0 TB/s; 16 rollouts
// behind 4,096 common entries (80 MB) 28 us, half of it the dependent reads in front of the first tile.
constexpr int kNarrowPick = 192, kNarrowRing = 256;
template <int D>
struct NarrowSpace {
  static constexpr int TILE = 32 * Lay<D, true>::PITCH;
  uint16_t *k, *v;   // [2][TILE]
  int *tab, *slot;   // [kNarrowPick]
  uint32_t* row;     // [kNarrowRing]
  int* pos;
};
// A unit of up to 32 NC rows: operands of K and V are read once for all of them.
template <int D, bool SHARED, int NC>
__device__ __forceinline__ void narrow_unit(const RowsArgs& a, const Unit& un, int g, const NarrowSpace<D>& x) {
  using LY = Lay<D, true>;
  constexpr int KS = D / 16, BN = 32, PITCH = LY::PITCH, TILE = BN * PITCH, NP = kNarrowPick / kWave;
  constexpr int SLOTS = BN * LY::CPRP, NI = (SLOTS + kWave - 1) / kWave, OPS = 2 * NI;   // copies of a tile
  uint16_t *const sK = x.k, *const sV = x.v;
  int *const sTab = x.tab, *const sSlot = x.slot, *const sPos = x.pos;
  uint32_t* const sRow = x.row;
  const int lane = threadIdx.x, half = lane >> 5, col = lane & 31;
  const auto rl = LY::row_lane(lane);
  const int tl = LY::tr_lo(lane), th = LY::tr_hi(lane);
  const int* trow = a.table + (size_t)un.s * a.max_blocks;
  ChunkWalker<SHARED> walk;
  walk.init(un);
  RowState<D, true> st[NC];
  bf16x8 qreg[NC][KS];
  const int row0 = un.row0 & ~3;
  int at[NC], lo = INT_MAX, hi = -1;
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    const RowLane rw = row_of<SHARED>(a, un, g, row0 + 32 * c + col, row0 + un.rows - 1);
    at[c] = rw.at;
    const uint16_t* qrow = a.q + ((size_t)rw.tok * a.Hq + rw.h) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qreg[c][ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + 16 * ks));
    lo = min(lo, SHARED ? rw.at : wave_min(rw.at));
    hi = max(hi, SHARED ? rw.at : wave_max(rw.at));
    st[c].init();
  }

  int prow[NI], pcol[NI];   // this lane's 16-byte slots of a tile: row (-1: none), source element
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int qs = i * kWave + lane, r = qs / LY::CPRP, pc = qs - r * LY::CPRP;
    prow[i] = qs < SLOTS ? r : -1;
    pcol[i] = qs < SLOTS && pc < LY::CPR ? 8 * (pc ^ LY::flip(r)) : 0;
  }
  unsigned tail = 0;   // entries listed so far
  int place[NP];       // first places of the chunks in work
  int stage = 0;       // of these: 0 none, 1 table entries asked for, 2 positions asked for, 3 there
  auto ask_table = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      place[k] = walk.next(un);
      dma_b32_global(trow + block_of(a, min(place[k] + lane, un.c1 - 1)), lds_addr(&sTab[k * kWave]));
    }
    stage = 1;
  };
  // the slot of a place, by its landed table entry (-1: an entry outside the cache)
  auto slot_of = [&](int k, int& blk) __attribute__((always_inline)) {
    const int c = min(place[k] + lane, un.c1 - 1);
    blk = sTab[k * kWave + lane];
    return (unsigned)blk < (unsigned)a.num_blocks ? blk * a.BS + (c - block_of(a, c) * a.BS) : -1;
  };
  auto ask_pos = [&]() __attribute__((always_inline)) {
    int blk, slot[NP];
#pragma unroll
    for (int k = 0; k < NP; ++k) slot[k] = slot_of(k, blk);
#pragma unroll
    for (int k = 0; k < NP; ++k) dma_b32_global(a.slot_pos + max(slot[k], 0), lds_addr(&sSlot[k * kWave]));
    stage = 2;
  };
  auto enlist = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < NP; ++k) {
      int blk;
      const int slot = slot_of(k, blk), pos = sSlot[k * kWave + lane];
      const bool vis = place[k] + lane < un.c1 && slot >= 0 && seen_by_some<SHARED>(a, pos, lo, hi);
      const unsigned long long m = __ballot(vis);
      if (vis) {
        const unsigned i = (tail + __builtin_popcountll(m & ((1ull << lane) - 1ull))) % kNarrowRing;
        sRow[i] = ((uint32_t)blk * a.Hkv + g) * a.BS + (slot - blk * a.BS);
        if (!SHARED) sPos[i] = pos;
      }
      tail = __builtin_amdgcn_readfirstlane(tail + __builtin_popcountll(m));
    }
    stage = 0;
  };
  // Entries from `head` on that make the next tile; lists more where they are short of one.
  auto ready = [&](unsigned head) __attribute__((always_inline)) {
    while (tail - head < BN && (stage > 0 || walk.more(a, un, lo, hi, lane))) {
      // what has not been asked for ahead: at the start, and where places show few entries
      if (stage == 0) ask_table();
      if (stage == 1) {
        wait_vm_le<0>();
        ask_pos();
      }
      if (stage == 2) wait_vm_le<0>();
      enlist();
    }
    return min(tail - head, (unsigned)BN);
  };
  auto gather = [&](int b, unsigned head, int n) __attribute__((always_inline)) {
    uint32_t r[NI];
#pragma unroll
    for (int i = 0; i < NI; ++i) r[i] = sRow[(head + min(max(prow[i], 0), n - 1)) % kNarrowRing];   // past the last: it again
#pragma unroll
    for (int i = 0; i < NI; ++i)
      if (i * kWave + kWave <= SLOTS || prow[i] >= 0) {
        const size_t off = (size_t)r[i] * D + pcol[i];
        if (SHARED && (un.row0 & 2)) {
          dma_b128_cached(a.kc + off, lds_addr(sK + b * TILE) + i * kWave * 16);
          dma_b128_cached(a.vc + off, lds_addr(sV + b * TILE) + i * kWave * 16);
        } else {
          dma_b128_global(a.kc + off, lds_addr(sK + b * TILE) + i * kWave * 16);
          dma_b128_global(a.vc + off, lds_addr(sV + b * TILE) + i * kWave * 16);
        }
      }
  };

  wait_vm_le<0>();   // Q is in: no compiler-visible load stays pending in the loop
  unsigned head = -BN;   // of the tile in work, n entries; the first turn has none
  int n = 0, b = 1;
  for (bool more = true; more;) {
    const int n1 = n == 0 || n == BN ? (int)ready(head + BN) : 0;   // a tile that is not full is the last
    if (n1 > 0) {
      gather(b ^ 1, head + BN, n1);
      wait_vm_le<OPS>();
    } else {
      wait_vm_le<0>();
    }
    more = n1 > 0;
    if (stage == 0 && walk.more(a, un, lo, hi, lane)) ask_table();
    else if (stage == 1) ask_pos();
    else if (stage == 2) stage = 3;
    if (n > 0) {
      const uint16_t* cK = sK + b * TILE;
      uint16_t* cV = sV + b * TILE;
      f32x16 s[NC][1];
#pragma unroll
      for (int c = 0; c < NC; ++c) s[c][0] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        const bf16x8 ka = lds_read_b128(cK + LY::row_at(rl, ks));
#pragma unroll
        for (int c = 0; c < NC; ++c) s[c][0] = mfma32(ka, qreg[c][ks], s[c][0]);
      }
      if (n < BN) {   // V of the places behind the last entry: their factor is 0, and must stay it
        for (int i = lane; i < (BN - n) * (PITCH / 8); i += kWave)
          *reinterpret_cast<uint4*>(&cV[n * PITCH + 8 * i]) = make_uint4(0u, 0u, 0u, 0u);
      }
      const int p = SHARED ? 0 : sPos[(head + col) % kNarrowRing];
      if (__ballot(col < n && (SHARED || (seen<SHARED>(a, p, lo) && seen<SHARED>(a, p, hi)))) != ~0ull) {
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int i = 8 * q4 + 4 * half;
          int4 e = make_int4(0, 0, 0, 0);
          if (!SHARED) e = *reinterpret_cast<const int4*>(&sPos[(head + i) % kNarrowRing]);   // head: a multiple of 32
#pragma unroll
          for (int c = 0; c < NC; ++c) {
            if (!(i < n && seen<SHARED>(a, e.x, at[c]))) s[c][0][4 * q4] = -INFINITY;
            if (!(i + 1 < n && seen<SHARED>(a, e.y, at[c]))) s[c][0][4 * q4 + 1] = -INFINITY;
            if (!(i + 2 < n && seen<SHARED>(a, e.z, at[c]))) s[c][0][4 * q4 + 2] = -INFINITY;
            if (!(i + 3 < n && seen<SHARED>(a, e.w, at[c]))) s[c][0][4 * q4 + 3] = -INFINITY;
          }
        }
      }
      bf16x8 pb[NC][2];
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        st[c].template weigh<1>(s[c], a.scale_log2);
#pragma unroll
        for (int t = 0; t < 2; ++t) pb[c][t] = pack8(s[c][0], 8 * t);
      }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int d = 0; d < D / 32; ++d) {
          const bf16x8 va = tr_operand<D, true>(cV, 16 * t, 32 * d, tl, th);
#pragma unroll
          for (int c = 0; c < NC; ++c) st[c].acc[d] = mfma32(va, pb[c][t], st[c].acc[d]);
        }
    }
    head += BN;
    n = n1;
    b ^= 1;
  }
#pragma unroll
  for (int c = 0; c < NC; ++c)
    st[c].finish(a, un, row_of<SHARED>(a, un, g, row0 + 32 * c + col, row0 + un.rows - 1), g, 32 * c + col, half);
}

template <int D, bool SHARED>
__global__ void __launch_bounds__(64) rows_narrow_kernel(RowsArgs a) {
  constexpr int TILE = NarrowSpace<D>::TILE;
  __shared__ __attribute__((aligned(1024))) uint16_t sK[2 * TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV[2 * TILE];
  __shared__ __attribute__((aligned(256))) int sTab[kNarrowPick];
  __shared__ __attribute__((aligned(256))) int sSlot[kNarrowPick];
  __shared__ __attribute__((aligned(16))) uint32_t sRow[kNarrowRing];
  __shared__ __attribute__((aligned(16))) int sPos[SHARED ? 4 : kNarrowRing];
  static_assert(kNarrowRing >= kNarrowPick + 2 * 32, "what is left of the last places, the tile in work, new ones");
  const int widx = blockIdx.x / a.Hkv, g = blockIdx.x - widx * a.Hkv, last = a.waves[widx + 1];
  for (int uidx = a.waves[widx]; uidx < last; ++uidx) {
    const Unit un = a.units[a.max_units[0] + uidx];
    const NarrowSpace<D> x{sK, sV, sTab, sSlot, sRow, sPos};
    if (un.rows <= 32) narrow_unit<D, SHARED, 1>(a, un, g, x);
    else if (D == 128) narrow_unit<D, SHARED, narrow_rows(D) / 32>(a, un, g, x);
  }
}

// ---------------------------------------------------------------- the merge
// A partial result joined to what there is: m, l and four of the sums of V.
struct Joined {
  float m, l;
  float4 x;
  __device__ __forceinline__ void add(float2 ml, const float4& y) {
    if (ml.y <= 0.f) return;   // a part without an entry: its sums are unwritten
    const float top = fmaxf(m, ml.x), f = m == top ? 1.f : __builtin_amdgcn_exp2f(m - top), e = __builtin_amdgcn_exp2f(ml.x - top);
    m = top;
    l = l * f + ml.y * e;
    x.x = x.x * f + y.x * e;
    x.y = x.y * f + y.y * e;
    x.z = x.z * f + y.z * e;
    x.w = x.w * f + y.w * e;
  }
};

// The partial results of a row: the group's prefix and the sequence's own part, or a sequence's splits.  BLOCK: a
// workgroup a row, whose groups of D / 4 lanes take the parts in turn (one long sequence has hundreds); else, for many
// rows of new tokens, which have few parts each, a wave a token and KV head, whose halves (D = 64: quarters) take the
// head's rows in turn, so that the token is looked up once.  Bound by the latency of its reads: four parts are asked for
// at a time.  4 us for few rows, 10 for 64 sequences with 39 MB of parts, 17 for 4,096 tokens with 54 MB.  A workgroup a row
// against a wave a token: one token over 32,000 entries 36 and 83 us.
template <int D, bool SHARED, bool BLOCK>
__global__ void __launch_bounds__(256) rows_merge_kernel(RowsArgs a) {
  constexpr int LPS = D / 4, PER = kWave / LPS, UNROLL = 4;
  __shared__ float2 sML[BLOCK ? 4 : 1];
  __shared__ float4 sX[BLOCK ? 4 * LPS : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, sub = lane / LPS, d4 = lane & (LPS - 1);
  if (!SHARED && a.parts[0] == 0) return;   // every row is written by its unit
  const int per_tok = BLOCK ? a.Hq : a.Hkv;
  const long long all = (long long)a.ntok * per_tok;
  for (long long i = BLOCK ? blockIdx.x : blockIdx.x * 4ll + wave; i < all; i += BLOCK ? gridDim.x : gridDim.x * 4ll) {
    const int tok = (int)(i / per_tok), at = (int)(i - (long long)tok * per_tok), g = BLOCK ? at / a.G : at;
    Parts set[2] = {};
    long long row[2] = {};   // of the first q-head of the KV head
    int first = 0;
    if (!SHARED) {   // the sequence of the token: the last one that begins at or before it
      int s = 0;
      for (int step = 1 << (31 - __builtin_clz(a.S)); step > 0; step >>= 1)
        if (s + step < a.S && a.cu[s + step] <= tok) s += step;
      const int t0 = min(max(a.cu[s], 0), a.ntok), t1 = min(max(a.cu[s + 1], t0), a.ntok);
      if (tok < t0 || tok >= t1) continue;
      set[0] = a.own[s];
      first = (tok - t0) * a.G;
      if (set[0].n == 0 || first >= set[0].rows) continue;   // written by its unit
      row[0] = first;
    } else {
      set[0] = a.own[tok];
      const int grp = a.prefix_group[tok];
      if ((unsigned)grp < (unsigned)a.groups) {
        int mine = a.rank[tok] * a.G + at - g * a.G;   // among the group's rows
        set[1] = a.prefix[kPrefixBlocks * (long long)grp];
        if (set[1].n > 0 && set[1].rows <= a.narrow) {
          const int rb = mine / a.narrow;
          set[1] = a.prefix[kPrefixBlocks * (long long)grp + rb];
          mine -= rb * a.narrow;
        }
        row[1] = mine - (at - g * a.G);
      }
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) row[k] += set[k].part + (long long)g * set[k].rows;
    const int n = set[0].n + set[1].n;
    for (int r = BLOCK ? at - g * a.G : sub; r < a.G; r += BLOCK ? a.G : PER) {
      if (!SHARED && first + r >= set[0].rows) continue;
      auto where = [&](int p) {
        return r + (p < set[0].n ? row[0] + (long long)p * a.Hkv * set[0].rows
                                 : row[1] + (long long)(p - set[0].n) * a.Hkv * set[1].rows);
      };
      constexpr int STEP = BLOCK ? 4 * PER : 1;
      Joined x = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
      for (int p0 = BLOCK ? wave * PER + sub : 0; p0 < n; p0 += UNROLL * STEP) {
        float2 v[UNROLL];
        float4 y[UNROLL];
#pragma unroll
        for (int k = 0; k < UNROLL; ++k) {   // the last one again behind the end
          const long long w = where(min(p0 + k * STEP, n - 1));
          v[k] = a.part_ml[w];
          y[k] = reinterpret_cast<const float4*>(a.part + w * D)[d4];
        }
#pragma unroll
        for (int k = 0; k < UNROLL; ++k)
          if (p0 + k * STEP < n) x.add(v[k], y[k]);
      }
      if (BLOCK) {
#pragma unroll
        for (int off = LPS; off < kWave; off <<= 1) {
          const float2 v = make_float2(__shfl_xor(x.m, off), __shfl_xor(x.l, off));
          const float4 y = make_float4(__shfl_xor(x.x.x, off), __shfl_xor(x.x.y, off), __shfl_xor(x.x.z, off), __shfl_xor(x.x.w, off));
          x.add(v, y);
        }
        if (sub == 0) {
          if (d4 == 0) sML[wave] = make_float2(x.m, x.l);
          sX[wave * LPS + d4] = x.x;
        }
        __syncthreads();
        if (wave == 0)
#pragma unroll
          for (int w = 1; w < 4; ++w) x.add(sML[w], sX[w * LPS + d4]);
        __syncthreads();
      }
      if (!BLOCK || (wave == 0 && sub == 0)) {
        const float inv = x.l <= 0.f ? 0.f : 1.f / x.l;
        const size_t out = (size_t)tok * a.Hq + g * a.G + r;
        reinterpret_cast<uint2*>(a.o + out * D)[d4] = pack4_bf16(x.x.x * inv, x.x.y * inv, x.x.z * inv, x.x.w * inv);
        if (d4 == 0) a.lse[out] = x.l <= 0.f ? -INFINITY : (x.m + __log2f(x.l)) * 0.6931471805599453f;
      }
    }
  }
}

// ---------------------------------------------------------------- launchers
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Units per KV head that fill the chip: three wide ones a CU, four narrow ones (D = 64: seven).
static int rows_want(const PagedRows& p, bool wide) {
  return ((wide ? 3 : p.D == 128 ? 4 : 7) * 256 + p.Hkv - 1) / p.Hkv;
}
constexpr long long kBlockRows = 4096;   // rows of new tokens that are merged by a workgroup each
// Sizes of a call's workspace, in this order.
struct RowsSpace {
  long long units[2], waves, split, part;   // units per KV head, wide and narrow; waves of narrow ones; partial rows of cut
                                            // wide jobs per KV head, and of all
  size_t parts, rank, list, count, base, jobs, own, prefix, unit, wave, stats, rows, ml;
  size_t bytes() const { return parts + rank + list + count + base + jobs + own + prefix + unit + wave + stats + rows + ml; }
};
static size_t stats_chunks(const PagedRows& p) { return ((size_t)p.max_blocks * p.block_size + kChunk - 1) / kChunk; }
static bool plans_small(const PagedRows& p) { return p.S <= kPlanSmall && p.groups <= kPlanGroups; }
// Row blocks of wide jobs: one for every 128 rows, and one more a job (SHARED: groups, and sequences by themselves if they
// have so many q-heads).  A job has no splits of fewer than kLeastTiles tiles; those of wide jobs add no more units than
// four rounds of them and than three times the row blocks (or one round).  Narrow jobs: a unit each, and one more for
// every wave's end.  Partial rows: of wide jobs 128 a unit (new tokens: only what is cut has any, and the plan cuts no more
// than twice the units that may be added); of narrow ones those of every job once and of the units that are added, for
// new tokens, where only jobs of several units have any, twice the latter.
static RowsSpace rows_space(const PagedRows& p) {
  RowsSpace x{};
  const long long G = p.Hq / p.Hkv, tokens = p.shared ? p.S : p.ntok, all = tokens * G;
  const long long narrow = narrow_rows(p.D), width = (long long)p.max_blocks * p.block_size;
  const long long jobs = (p.shared ? (long long)p.groups * kPrefixBlocks : 0) + p.S;
  const long long most = p.shared ? kPrefixBlocks * narrow : narrow;   // rows of a narrow job, or of a group's
  const long long wide_jobs = std::min<long long>(p.shared ? p.groups : p.S, all / most) + (p.shared && G > narrow ? p.S : 0);
  const long long blocks = all > most || (p.shared && G > narrow) ? all / kWideRows + wide_jobs : 0, want = rows_want(p, true);
  const long long more = std::min(std::max(want, 3 * blocks), 4 * want);
  x.units[0] = std::min(blocks * ((width + 32 * kLeastTiles - 1) / (32 * kLeastTiles)), blocks + more);
  x.waves = std::min<long long>(rows_want(p, false), jobs * ((width + kChunk - 1) / kChunk + kStartChunks));
  x.units[1] = jobs + x.waves;
  x.split = (p.shared ? x.units[0] : 2 * std::min(more, x.units[0])) * kWideRows;
  x.part = (x.split + (p.shared ? 2 * all + x.waves * narrow : 2 * x.waves * narrow)) * p.Hkv;
  x.parts = 256;
  if (p.shared) {
    x.rank = x.list = round256((size_t)p.S * sizeof(int));
    x.prefix = round256((size_t)p.groups * kPrefixBlocks * sizeof(Parts));
  }
  if (!plans_small(p)) {
    if (p.shared) x.count = x.base = round256((size_t)p.groups * sizeof(int));
    x.jobs = round256(6 * (size_t)jobs * sizeof(int));
  }
  x.own = round256((size_t)p.S * sizeof(Parts));
  x.unit = round256((size_t)(x.units[0] + x.units[1]) * sizeof(Unit));
  x.wave = round256((size_t)(x.waves + 1) * sizeof(int));
  if (!p.shared) x.stats = round256((size_t)p.S * stats_chunks(p) * sizeof(int2));
  x.rows = round256((size_t)x.part * p.D * sizeof(float));
  x.ml = round256((size_t)x.part * sizeof(float2));
  return x;
}
size_t paged_rows_ws_bytes(const PagedRows& p) { return rows_space(p).bytes(); }
bool paged_rows_fit(const PagedRows& p) {
  const RowsSpace x = rows_space(p);
  const long long rows = (long long)(p.shared ? p.S : p.ntok) * p.Hq;
  return std::max(x.units[0], x.units[1]) * p.Hkv <= 0x7fffffffll / 256 && x.part <= 0x7fffffffll && rows <= (1ll << 26) - 4 &&
         ((long long)p.S + kPrefixBlocks * (long long)p.groups) * ((long long)stats_chunks(p) + kStartChunks) <= 0x7fffffffll;
}

template <int D, bool SHARED>
static hipError_t launch_rows(const PagedRows& p, const RowsArgs& a) {
  // under a window also the tables' chunks, 16 waves of them a CU
  const bool small = plans_small(p);
  const unsigned looks = !SHARED && p.window > 0 ? (unsigned)std::min((p.S * stats_chunks(p) + 7) / 8, (size_t)512) : 0;
  if (small) hipLaunchKernelGGL((rows_plan_kernel<SHARED, true>), dim3(1 + looks), dim3(512), 0, p.stream, a);
  else hipLaunchKernelGGL((rows_plan_kernel<SHARED, false>), dim3(1 + looks), dim3(1024), 0, p.stream, a);
  const bool far = (long long)p.num_blocks * p.block_size * p.Hkv * (2 * D) >= 1ll << 32;
  prof_begin(SHARED ? "paged_decode_shared" : "paged_extend", p.stream);
  if (a.max_units[0])
    hipLaunchKernelGGL((far ? rows_wide_kernel<D, SHARED, true> : rows_wide_kernel<D, SHARED, false>),
                       dim3((unsigned)((long long)a.max_units[0] * a.Hkv)), dim3(256), 0, p.stream, a);
  hipLaunchKernelGGL((rows_narrow_kernel<D, SHARED>), dim3((unsigned)((long long)a.max_waves * a.Hkv)), dim3(64), 0,
                     p.stream, a);
  prof_end(p.stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long rows = (long long)a.ntok * a.Hq;
  if (SHARED || rows <= kBlockRows)
    hipLaunchKernelGGL((rows_merge_kernel<D, SHARED, true>), dim3((unsigned)std::min(rows, 16384ll)), dim3(256), 0, p.stream, a);
  else
    hipLaunchKernelGGL((rows_merge_kernel<D, SHARED, SHARED>), dim3((unsigned)std::min((rows / a.G + 3) / 4, 4096ll)), dim3(256),
                       0, p.stream, a);
  return hipGetLastError();
}

hipError_t launch_paged_rows(const PagedRows& p) {
  const RowsSpace x = rows_space(p);
  RowsArgs a{};
  a.q = (const uint16_t*)p.q;
  a.kc = (const uint16_t*)p.k_cache;
  a.vc = (const uint16_t*)p.v_cache;
  a.slot_pos = p.slot_pos;
  a.table = p.block_table;
  a.nblk = p.seq_blocks;
  a.prefix_group = p.prefix_group;
  a.prefix_blocks = p.prefix_blocks;
  a.q_pos = p.q_pos;
  a.cu = p.cu;
  a.o = (uint16_t*)p.o;
  a.lse = p.lse;
  a.S = p.S;
  a.groups = p.groups;
  a.ntok = p.shared ? p.S : p.ntok;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.Hq / p.Hkv;
  a.max_blocks = p.max_blocks;
  a.BS = p.block_size;
  a.num_blocks = p.num_blocks;
  a.shift = p.block_size & (p.block_size - 1) ? -1 : __builtin_ctz((unsigned)p.block_size);
  a.window = p.window;
  a.sinks = p.sinks;
  a.scale_log2 = p.scale * 1.4426950408889634f;
  char* w = (char*)p.ws;
  auto take = [&](size_t bytes) {
    char* at = w;
    w += bytes;
    return at;
  };
  a.parts = (int*)take(x.parts);
  a.rank = (int*)take(x.rank);
  a.list = (int*)take(x.list);
  a.count = (int*)take(x.count);
  a.base = (int*)take(x.base);
  a.jobs = (int*)take(x.jobs);
  a.own = (Parts*)take(x.own);
  a.prefix = (Parts*)take(x.prefix);
  a.units = (Unit*)take(x.unit);
  a.waves = (int*)take(x.wave);
  a.stats = (int2*)take(x.stats);
  a.part = (float*)take(x.rows);
  a.part_ml = (float2*)take(x.ml);
  a.max_part = x.part;
  a.max_split = x.split;
  for (int k = 0; k < 2; ++k) {
    a.max_units[k] = (int)x.units[k];
    a.want[k] = rows_want(p, k == 0);
  }
  a.max_waves = (int)x.waves;
  a.narrow = narrow_rows(p.D);
  if (p.shared) return p.D == 128 ? launch_rows<128, true>(p, a) : launch_rows<64, true>(p, a);
  return p.D == 128 ? launch_rows<128, false>(p, a) : launch_rows<64, false>(p, a);
}

}  // namespace kvs
