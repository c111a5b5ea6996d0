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
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>

namespace kvs {

// ---------------------------------------------------------------- copies
// Slot dst[i] takes the K and V rows of slot src[i], its position and its weight; MOVE: slot src[i] is empty then.
// 16-byte pieces, one of K and one of V a thread and turn; bound by HBM.
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
    const uint4 k = *reinterpret_cast<const uint4*>(kc + x), v = *reinterpret_cast<const uint4*>(vc + x);
    *reinterpret_cast<uint4*>(kc + y) = k;
    *reinterpret_cast<uint4*>(vc + y) = v;
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
constexpr int kRowBlock = 128;   // rows of a unit: 32 a wave
template <int D>
constexpr int rows_bn() { return D == 128 ? 32 : 64; }   // keys of a tile
constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / kWave;
constexpr int kLeastTiles = 4;   // of a unit, in 32-key tiles

// What a unit is, as its workgroups read it.
struct Unit {
  int s;          // sequence whose table is read; -1: no such unit
  int c0, c1;     // places of the table
  int rows;       // of the job
  int tok;        // first token of the job, or of its members' list
  int row0;       // first row of the unit
  int part;       // first row of its partial results (KV head 0); -1: O and LSE are written
  int listed;     // whether token i of the job is list[tok + i], else tok + i
};
static_assert(sizeof(Unit) == 32, "two 16-byte loads");

// Partial results of a job: row r of KV head g and split k at part + (k Hkv + g) rows + r.
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
  float scale_log2;
  // workspace
  int* rank;        // [S] SHARED: of a sequence among its group's members
  int* count;       // [groups] members
  int* base;        // [groups] first member in `list`
  int* list;        // [S] members, group by group
  int* first;       // [jobs + 1] first unit of each job
  Parts* own;       // [S] of each sequence
  Parts* prefix;    // [S] of its group
  Unit* units;      // [max_units]
  float* part;      // [max_part][D]
  float2* part_ml;  // [max_part]: m (log2 units), l
  int max_units;
  long long max_part;
  int want;         // units per KV head that fill the chip
};

struct Job {
  int s, c0, c1, rows, tok, listed;
};

// Job j: the groups first, then the sequences.
template <bool SHARED>
__device__ __forceinline__ int prefix_of(const RowsArgs& a, int g) {   // blocks of group g's prefix
  const int m = a.count[g];
  if (m < 2) return 0;
  const int s = a.list[a.base[g]];
  return max(0, min(min(a.prefix_blocks[g], a.nblk[s]), a.max_blocks));
}
template <bool SHARED>
__device__ __forceinline__ Job job_of(const RowsArgs& a, int j) {
  if (SHARED && j < a.groups) {
    const int n = a.count[j], b = prefix_of<SHARED>(a, j);
    if (b == 0) return {0, 0, 0, 0, 0, 1};
    return {a.list[a.base[j]], 0, b * a.BS, n * a.G, a.base[j], 1};
  }
  const int s = SHARED ? j - a.groups : j;
  const int blocks = min(max(a.nblk[s], 0), a.max_blocks);
  if (SHARED) {
    const int g = a.prefix_group[s], b = (unsigned)g < (unsigned)a.groups ? min(prefix_of<SHARED>(a, g), blocks) : 0;
    return {s, b * a.BS, blocks * a.BS, a.G, s, 0};
  }
  const int t0 = min(max(a.cu[s], 0), a.ntok), t1 = min(max(a.cu[s + 1], t0), a.ntok);
  return {s, 0, blocks * a.BS, (t1 - t0) * a.G, t0, 0};
}
__device__ __forceinline__ int job_tiles(const Job& j) { return (int)(((unsigned)(j.c1 - j.c0) + 31) / 32); }
__device__ __forceinline__ int job_blocks(const Job& j) { return (j.rows + kRowBlock - 1) / kRowBlock; }
// Splits of a job under runs of c tiles.  New tokens that see nothing still have rows to write.
template <bool SHARED>
__device__ __forceinline__ int job_splits(const Job& j, int c) {
  if (j.rows == 0) return 0;
  const int n = (job_tiles(j) + c - 1) / c;
  return SHARED ? n : max(n, 1);
}

// One workgroup.  The size of the runs, the same for all jobs, is the smallest for which units and partial results fit.
template <bool SHARED>
__global__ void __launch_bounds__(kPlanThreads) rows_plan_kernel(RowsArgs a) {
  __shared__ long long su[kPlanWaves], sp[kPlanWaves];
  __shared__ int st[kPlanWaves], pick[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, J = SHARED ? a.groups + a.S : a.S;
  if (SHARED) {
    for (int g = tid; g < a.groups; g += kPlanThreads) a.count[g] = 0;
    __syncthreads();
    if (wave == 0)   // ranks in the sequences' order: 64 of them at a time, group by group of those among them
      for (int s0 = 0; s0 < a.S; s0 += kWave) {
        const int s = s0 + lane, g = s < a.S ? a.prefix_group[s] : -1;
        unsigned long long todo = __ballot((unsigned)g < (unsigned)a.groups);
        while (todo) {
          const int g1 = __builtin_amdgcn_readlane(g, __builtin_ctzll(todo));
          const unsigned long long same = __ballot(g == g1);
          const int before = a.count[g1];
          if (g == g1) a.rank[s] = before + __builtin_popcountll(same & ((1ull << lane) - 1ull));
          if (lane == 0) a.count[g1] = before + __builtin_popcountll(same);
          __threadfence_block();
          todo &= ~same;
        }
      }
    __syncthreads();
    int from = 0;
    for (int g0 = 0; g0 < a.groups; g0 += kPlanThreads) {
      const int g = g0 + tid, n = g < a.groups ? a.count[g] : 0, incl = wave_scan(n);
      if (lane == kWave - 1) st[wave] = incl;
      __syncthreads();
      int x = from + incl - n;
      for (int w = 0; w < kPlanWaves; ++w) {
        x += w < wave ? st[w] : 0;
        from += st[w];
      }
      if (g < a.groups) a.base[g] = x;
      __syncthreads();
    }
    for (int s = tid; s < a.S; s += kPlanThreads) {
      const int g = a.prefix_group[s];
      if ((unsigned)g < (unsigned)a.groups) a.list[a.base[g] + a.rank[s]] = s;
    }
    __syncthreads();
  }
  // units and partial rows for runs of c tiles, by one wave
  auto need = [&](int c, long long& units, long long& rows) {
    units = rows = 0;
    for (int j = lane; j < J; j += kWave) {
      const Job x = job_of<SHARED>(a, j);
      const int n = job_splits<SHARED>(x, c);
      units += (long long)n * job_blocks(x);
      if (SHARED || n > 1) rows += (long long)n * x.rows * a.Hkv;
    }
    for (int off = 32; off > 0; off >>= 1) {
      units += __shfl_xor(units, off);
      rows += __shfl_xor(rows, off);
    }
  };
  int top = 1;
  long long least = 0;
  for (int j = tid; j < J; j += kPlanThreads) {
    const Job x = job_of<SHARED>(a, j);
    top = max(top, job_tiles(x));
    least += job_blocks(x);
  }
  for (int off = 32; off > 0; off >>= 1) least += __shfl_xor(least, off);
  top = wave_max(top);
  if (lane == 0) {
    st[wave] = top;
    su[wave] = least;
  }
  __syncthreads();
  least = 0;
  for (int w = 0; w < kPlanWaves; ++w) {
    top = max(top, st[w]);
    least += su[w];
  }
  // as many units as fill the chip, and half as many on top where the row blocks alone do
  const long long most = min((long long)a.max_units, max((long long)a.want, least + a.want / 2));
  __syncthreads();
  // 16 sizes at a time: first in equal ratios from the least to the whole of the longest job, then between two of these
  int lo = min(kLeastTiles, top), hi = top;
  for (int turn = 0; turn < 2; ++turn) {
    int c = lo + (int)((long long)(hi - lo) * (wave + 1) / kPlanWaves);
    if (turn == 0) c = min(hi, max(lo, (int)(lo * __builtin_amdgcn_exp2f(__log2f((float)hi / (float)lo) * ((float)wave / (kPlanWaves - 1))))));
    if (turn == 0 && wave == kPlanWaves - 1) c = hi;
    long long units, rows;
    need(c, units, rows);
    if (lane == 0) {
      su[wave] = units <= most && rows <= a.max_part;
      st[wave] = c;
    }
    __syncthreads();
    if (tid == 0) {
      int w = 0;
      while (w < kPlanWaves - 1 && !su[w]) ++w;
      pick[0] = w > 0 ? st[w - 1] : lo;
      pick[1] = st[w];
    }
    __syncthreads();
    lo = pick[0];
    hi = pick[1];
    if (turn == 0 && lo == hi) break;
  }
  const int C = hi;
  // first units and first partial rows
  long long unit0 = 0, part0 = 0;
  for (int j0 = 0; j0 < J; j0 += kPlanThreads) {
    const int j = j0 + tid;
    const Job x = j < J ? job_of<SHARED>(a, j) : Job{0, 0, 0, 0, 0, 0};
    const int n = job_splits<SHARED>(x, C);
    const long long mu = (long long)n * job_blocks(x), mp = SHARED || n > 1 ? (long long)n * x.rows * a.Hkv : 0;
    long long u = mu, p = mp;
    for (int off = 1; off < kWave; off <<= 1) {
      const long long du = __shfl_up(u, off), dp = __shfl_up(p, off);
      if (lane >= off) {
        u += du;
        p += dp;
      }
    }
    if (lane == kWave - 1) {
      su[wave] = u;
      sp[wave] = p;
    }
    __syncthreads();
    u += unit0 - mu;
    p += part0 - mp;
    for (int w = 0; w < kPlanWaves; ++w) {
      if (w < wave) {
        u += su[w];
        p += sp[w];
      }
      unit0 += su[w];
      part0 += sp[w];
    }
    if (j < J) {
      a.first[j] = (int)min(u, (long long)a.max_units);
      const Parts parts = {(int)p, x.rows, mp ? n : 0};
      if (SHARED && j < a.groups) a.prefix[j] = parts;
      else a.own[SHARED ? j - a.groups : j] = parts;
    }
    __syncthreads();
  }
  // offsets that overlap (only where cu_seqlens decreases) may ask for more than there is: nothing is computed then
  const bool fits = unit0 <= a.max_units && part0 <= a.max_part;
  const int total = fits ? (int)unit0 : 0;
  if (!fits)
    for (int s = tid; s < a.S; s += kPlanThreads) a.own[s].n = 0;
  for (int u = tid; u < a.max_units; u += kPlanThreads) {
    Unit x{};
    x.s = -1;
    if (u < total) {
      int j = 0;   // the last job that begins at or before u
      for (int step = 1 << (31 - __builtin_clz(J)); step > 0; step >>= 1)
        if (j + step < J && a.first[j + step] <= u) j += step;
      const Job b = job_of<SHARED>(a, j);
      const Parts parts = SHARED ? (j < a.groups ? a.prefix[j] : a.own[j - a.groups]) : a.own[j];
      const int nb = job_blocks(b), tiles = job_tiles(b), n = max(job_splits<SHARED>(b, C), 1);
      const int k = (u - a.first[j]) / nb, rb = nb - 1 - (u - a.first[j] - k * nb);   // the last rows see most: first
      const int per = (tiles + n - 1) / n;
      x = {b.s,   (int)min((long long)b.c0 + 32ll * per * k, (long long)b.c1),
           (int)min((long long)b.c0 + 32ll * per * (k + 1), (long long)b.c1),
           b.rows, b.tok, rb * kRowBlock, parts.n ? parts.part + k * a.Hkv * b.rows : -1, b.listed};
    }
    a.units[u] = x;
  }
}

// ---------------------------------------------------------------- the units
constexpr int kRowsPick = 1024;   // places of the table that are looked at together

// A unit walks its run of the table 1,024 places at a time: the slots that some
// row of it sees go to a list in LDS (two dependent reads, for all places at
// once), and the keys and values of the listed slots are gathered tile by tile,
// double-buffered, each tile read by the four waves.  Scores are S^T = K Q^T
// (keys on M, rows on N), so that a lane holds 16 scores of one row; softmax and
// the products with V as in the forward of the eviction mask.
template <int D, bool SHARED>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(3, 3))) rows_kernel(RowsArgs a) {
  using LY = Lay<D, true>;
  constexpr int KS = D / 16, DB = D / 32, BN = rows_bn<D>(), NKB = BN / 32, PITCH = LY::PITCH, TILE = BN * PITCH;
  constexpr int PIECES = BN * LY::CPRP / kWave, PW = (PIECES + 3) / 4, LOOK = kRowsPick / 256;
  static_assert(BN * LY::CPRP % kWave == 0, "tile must fill whole 64-slot pieces");
  __shared__ __attribute__((aligned(1024))) uint16_t sK[2][TILE];
  __shared__ __attribute__((aligned(1024))) uint16_t sV[2][TILE];
  __shared__ __attribute__((aligned(16))) uint32_t sRow[kRowsPick];   // rows [block][KV head][row] of the listed slots
  __shared__ __attribute__((aligned(16))) int sPos[kRowsPick];        // and their positions; INT_MAX: nothing there
  __shared__ int sCnt[LOOK * 4], sMin[4], sMax[4];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5, col = lane & 31;
  const int uidx = blockIdx.x / a.Hkv, g = blockIdx.x - uidx * a.Hkv;
  const Unit un = a.units[uidx];
  if (un.s < 0) return;
  const auto rl = LY::row_lane(lane);
  const int tl = LY::tr_lo(lane), th = LY::tr_hi(lane);

  // this lane's row: its token and q-head
  const int row = un.row0 + 32 * wave + col, rr = min(row, un.rows - 1);
  const bool row_ok = row < un.rows, wave_ok = un.row0 + 32 * wave < un.rows;
  const int ti = rr / a.G, tok = un.listed ? a.list[un.tok + ti] : un.tok + ti, h = g * a.G + rr - ti * a.G;
  bf16x8 qreg[KS];
  {
    const uint16_t* qrow = a.q + ((size_t)tok * a.Hq + h) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qreg[ks] = as_bf16x8(*reinterpret_cast<const uint4*>(qrow + 16 * ks));
  }
  const int at = SHARED ? INT_MAX - 1 : max(a.q_pos[tok], -1);
  const int wlo = wave_min(at), whi = wave_max(at);   // lanes past the last row repeat it
  int lo = wlo, hi = whi;
  if (!SHARED) {
    if (lane == 0) {
      sMin[wave] = wlo;
      sMax[wave] = whi;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 4; ++w)
      if (un.row0 + 32 * w < un.rows) {
        lo = min(lo, sMin[w]);
        hi = max(hi, sMax[w]);
      }
  }
  // p is seen by the row at position i iff p <= i and (i - p < window or p < sinks)
  auto seen = [&](int p, int i) __attribute__((always_inline)) {
    return p <= i && (SHARED || a.window == 0 || i - p < a.window || p < a.sinks);
  };

  f32x16 acc[DB];
#pragma unroll
  for (int d = 0; d < DB; ++d) acc[d] = f32x16{};
  // running maximum (log2 units), the offset of the exponentials (0 until the row has seen an entry), and the raw score
  // above which the maximum moves
  float m_run = -INFINITY, l_run = 0.f, m_use = 0.f, thr = -INFINITY;
  const float inv_scale_log2 = 1.f / a.scale_log2;
  const int* trow = a.table + (size_t)un.s * a.max_blocks;

  // this lane's 16-byte slots of a tile: row and source element
  int prow[PW], pcol[PW];
#pragma unroll
  for (int i = 0; i < PW; ++i) {
    const int qs = (wave + 4 * i) * kWave + lane, r = qs / LY::CPRP, pc = qs - r * LY::CPRP;
    prow[i] = min(r, BN - 1);
    pcol[i] = pc < LY::CPR ? 8 * (pc ^ LY::flip(r)) : 0;
  }
  auto stage = [&](int t) __attribute__((always_inline)) {
    const int b = t & 1;
#pragma unroll
    for (int i = 0; i < PW; ++i) {
      const int n = wave + 4 * i;
      if (i < PW - 1 || PIECES % 4 == 0 || n < PIECES) {
        const size_t off = (size_t)sRow[t * BN + prow[i]] * D + pcol[i];
        dma_b128_global(a.kc + off, lds_addr(sK[b]) + n * kWave * 16);
        dma_b128_global(a.vc + off, lds_addr(sV[b]) + n * kWave * 16);
      }
    }
  };

  auto compute = [&](int t, int cnt) __attribute__((always_inline)) {
    const uint16_t* cK = sK[t & 1];
    const uint16_t* cV = sV[t & 1];
    f32x16 s[NKB];
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb) {
      s[kb] = f32x16{};
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) s[kb] = mfma32(lds_read_b128(cK + 32 * kb * PITCH + LY::row_at(rl, ks)), qreg[ks], s[kb]);
    }
    // whether every row of the wave sees every entry of the tile
    const int p = sPos[t * BN + (BN == 64 ? lane : col)];
    const bool full = __ballot(seen(p, wlo) && seen(p, whi)) == ~0ull;
    if (!full) {
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int q4 = 0; q4 < 4; ++q4) {
          const int4 e = *reinterpret_cast<const int4*>(&sPos[t * BN + 32 * kb + 8 * q4 + 4 * half]);
          if (!seen(e.x, at)) s[kb][4 * q4] = -INFINITY;
          if (!seen(e.y, at)) s[kb][4 * q4 + 1] = -INFINITY;
          if (!seen(e.z, at)) s[kb][4 * q4 + 2] = -INFINITY;
          if (!seen(e.w, at)) s[kb][4 * q4 + 3] = -INFINITY;
        }
    }
    float mx = -INFINITY;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[kb][r]);
    if (__ballot(mx > thr)) {
      const float m_new = fmaxf(m_run, fmaxf(mx, wave_xor32(mx)) * a.scale_log2);
      const float alpha = m_new == m_run ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) acc[d][r] *= alpha;
      m_run = m_new;
      m_use = m_run == -INFINITY ? 0.f : m_run;
      thr = (m_run + 8.f) * inv_scale_log2;
    }
    float ls = 0.f;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][r], a.scale_log2, -m_use));
        s[kb][r] = e;
        ls += e;
      }
    l_run += ls;
#pragma unroll
    for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
      for (int t2 = 0; t2 < 2; ++t2) {
        const bf16x8 pb = pack8(s[kb], 8 * t2);
#pragma unroll
        for (int d = 0; d < DB; ++d) acc[d] = mfma32(tr_operand<D, true>(cV, 32 * kb + 16 * t2, 32 * d, tl, th), pb, acc[d]);
      }
  };

  for (long long base = un.c0; base < un.c1; base += kRowsPick) {
    // the slots of the next 1,024 places that some row sees, in the table's order
    int slot[LOOK], pos[LOOK];
    unsigned long long vis[LOOK];
#pragma unroll
    for (int k = 0; k < LOOK; ++k) {
      const long long c = base + k * 256 + tid;
      const int blk = (int)(c / a.BS), e = c < un.c1 ? trow[blk] : -1;
      slot[k] = (unsigned)e < (unsigned)a.num_blocks ? e * a.BS + (int)(c - (long long)blk * a.BS) : -1;
    }
#pragma unroll
    for (int k = 0; k < LOOK; ++k) pos[k] = slot[k] >= 0 ? a.slot_pos[slot[k]] : -1;
    if (base != un.c0) __syncthreads();   // the lists are read
#pragma unroll
    for (int k = 0; k < LOOK; ++k) {
      vis[k] = __ballot(pos[k] >= 0 && (SHARED || (pos[k] <= hi && (a.window == 0 || lo - pos[k] < a.window || pos[k] < a.sinks))));
      if (lane == 0) sCnt[k * 4 + wave] = __builtin_popcountll(vis[k]);
    }
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
    const int ntile = (cnt + BN - 1) / BN;
#pragma unroll
    for (int k = 0; k < LOOK; ++k)
      if ((vis[k] >> lane) & 1ull) {
        const int i = mine[k] + __builtin_popcountll(vis[k] & ((1ull << lane) - 1ull)), blk = slot[k] / a.BS;
        const uint32_t r = ((uint32_t)blk * a.Hkv + g) * a.BS + (slot[k] - blk * a.BS);
        sRow[i] = r;
        sPos[i] = SHARED ? 0 : pos[k];
        if (i == cnt - 1)   // the last tile's places behind it repeat it, and nobody sees them
          for (int x = cnt; x < ntile * BN; ++x) {
            sRow[x] = r;
            sPos[x] = INT_MAX;
          }
      }
    __syncthreads();
    stage(0);
    for (int t = 0; t < ntile; ++t) {
      wait_vm();
      __syncthreads();   // tile t is there, and nobody reads tile t - 1 any more
      if (t + 1 < ntile) stage(t + 1);
      if (t == ntile - 1 && cnt % BN) {   // V of the places behind the last entry: their factor is 0, and must stay it
        for (int x = tid; x < (ntile * BN - cnt) * (PITCH / 8); x += 256)
          *reinterpret_cast<uint4*>(&sV[t & 1][(BN - (ntile * BN - cnt)) * PITCH + 8 * x]) = make_uint4(0u, 0u, 0u, 0u);
        __syncthreads();
      }
      if (wave_ok) compute(t, cnt);
    }
  }

  const float l_tot = halves_sum(l_run);
  if (!row_ok) return;
  if (un.part < 0) {
    const float inv = l_tot <= 0.f ? 0.f : 1.f / l_tot;
    uint16_t* orow = a.o + ((size_t)tok * a.Hq + h) * D;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<uint2*>(orow + 32 * d + 8 * q4 + 4 * half) =
            pack4_bf16(acc[d][4 * q4] * inv, acc[d][4 * q4 + 1] * inv, acc[d][4 * q4 + 2] * inv, acc[d][4 * q4 + 3] * inv);
    if (half == 0) a.lse[(size_t)tok * a.Hq + h] = l_tot <= 0.f ? -INFINITY : (m_run + __log2f(l_tot)) * 0.6931471805599453f;
    return;
  }
  const size_t pidx = (size_t)un.part + (size_t)g * un.rows + row;
  float* dst = a.part + pidx * D;
  if (!(l_tot <= 0.f)) {   // else O is left unwritten (the merge skips it)
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
      for (int q4 = 0; q4 < 4; ++q4)
        *reinterpret_cast<float4*>(dst + 32 * d + 8 * q4 + 4 * half) =
            make_float4(acc[d][4 * q4], acc[d][4 * q4 + 1], acc[d][4 * q4 + 2], acc[d][4 * q4 + 3]);
  }
  if (half == 0) a.part_ml[pidx] = make_float2(m_run, l_tot);
}

// ---------------------------------------------------------------- the merge
// One wave a (token, q-head): the partial results of the group's prefix and of the sequence's own part, or of a
// sequence's splits.  D / 4 lanes read one partial result as float4.
template <int D, bool SHARED>
__global__ void __launch_bounds__(256) rows_merge_kernel(RowsArgs a) {
  constexpr int LPS = D / 4, PER = kWave / LPS;
  const int lane = threadIdx.x & 63;
  const long long r = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (r >= (long long)a.ntok * a.Hq) return;
  const int tok = (int)(r / a.Hq), h = (int)(r - (long long)tok * a.Hq), g = h / a.G;
  Parts set[2] = {};
  long long at[2] = {};
  int s = tok;
  if (!SHARED) {   // the sequence of the token: the last one that begins at or before it
    s = 0;
    for (int step = 1 << (31 - __builtin_clz(a.S)); step > 0; step >>= 1)
      if (s + step < a.S && a.cu[s + step] <= tok) s += step;
    const int t0 = min(max(a.cu[s], 0), a.ntok), t1 = min(max(a.cu[s + 1], t0), a.ntok);
    if (tok < t0 || tok >= t1) return;
    set[0] = a.own[s];
    if (set[0].n == 0) return;   // written by its unit
    at[0] = (long long)(tok - t0) * a.G;
  } else {
    set[0] = a.own[s];
    const int grp = a.prefix_group[s];
    if ((unsigned)grp < (unsigned)a.groups) {
      set[1] = a.prefix[grp];
      at[1] = (long long)a.rank[s] * a.G;
    }
  }
#pragma unroll
  for (int k = 0; k < 2; ++k) at[k] += set[k].part + (long long)g * set[k].rows + (h - g * a.G);
  const int n = set[0].n + set[1].n;
  auto where = [&](int i) {
    return i < set[0].n ? at[0] + (long long)i * a.Hkv * set[0].rows : at[1] + (long long)(i - set[0].n) * a.Hkv * set[1].rows;
  };
  float M = -INFINITY;
  for (int i = lane; i < n; i += kWave) {
    const float2 v = a.part_ml[where(i)];
    if (!(v.y <= 0.f)) M = fmaxf(M, v.x);
  }
#pragma unroll
  for (int off = 32; off > 0; off >>= 1) M = fmaxf(M, __shfl_xor(M, off));
  float L = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int i = lane / LPS; i < n; i += PER) {
    const long long w = where(i);
    const float2 v = a.part_ml[w];
    if (!(v.y <= 0.f)) {
      const float f = __builtin_amdgcn_exp2f(v.x - M);
      const float4 y = reinterpret_cast<const float4*>(a.part + w * D)[lane & (LPS - 1)];
      L += v.y * f;
      x.x += y.x * f;
      x.y += y.y * f;
      x.z += y.z * f;
      x.w += y.w * f;
    }
  }
#pragma unroll
  for (int off = LPS; off < kWave; off <<= 1) {
    L += __shfl_xor(L, off);
    x.x += __shfl_xor(x.x, off);
    x.y += __shfl_xor(x.y, off);
    x.z += __shfl_xor(x.z, off);
    x.w += __shfl_xor(x.w, off);
  }
  if (lane < LPS) {
    const float inv = L <= 0.f ? 0.f : 1.f / L;
    reinterpret_cast<uint2*>(a.o + r * D)[lane] = pack4_bf16(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (lane == 0) a.lse[r] = L <= 0.f ? -INFINITY : (M + __log2f(L)) * 0.6931471805599453f;
  }
}

// ---------------------------------------------------------------- launchers
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Units per KV head that fill the chip: three workgroups a CU.
static int rows_want(int Hkv) { return (3 * 256 + Hkv - 1) / Hkv; }
// Sizes of a call's workspace, in this order.
struct RowsSpace {
  long long units, part;   // units per KV head; partial rows
  size_t rank, count, base, list, first, own, prefix, unit, rows, ml;
  size_t bytes() const { return rank + count + base + list + first + own + prefix + unit + rows + ml; }
};
// Row blocks: at most one a job beside the full ones.  Partial rows: one for every row of every job, and what the splits
// of half a round of units take.
static RowsSpace rows_space(const PagedRows& p) {
  RowsSpace x{};
  const long long G = p.Hq / p.Hkv, want = rows_want(p.Hkv);
  const long long tokens = p.shared ? p.S : p.ntok, jobs = (long long)p.S + p.groups;
  const long long blocks = (p.shared ? p.S : 0) + tokens * G / kRowBlock + (p.shared ? p.groups : p.S);
  x.units = std::max(want, blocks + want / 2);
  x.part = ((p.shared ? 2 : 1) * tokens * G + want * kRowBlock) * p.Hkv;
  if (p.shared) {
    x.rank = x.list = round256((size_t)p.S * sizeof(int));
    x.count = x.base = round256((size_t)p.groups * sizeof(int));
    x.prefix = round256((size_t)p.groups * sizeof(Parts));
  }
  x.first = round256((size_t)(jobs + 1) * sizeof(int));
  x.own = round256((size_t)p.S * sizeof(Parts));
  x.unit = round256((size_t)x.units * sizeof(Unit));
  x.rows = round256((size_t)x.part * p.D * sizeof(float));
  x.ml = round256((size_t)x.part * sizeof(float2));
  return x;
}
size_t paged_rows_ws_bytes(const PagedRows& p) { return rows_space(p).bytes(); }
bool paged_rows_fit(const PagedRows& p) {
  const RowsSpace x = rows_space(p);
  const long long rows = (long long)(p.shared ? p.S : p.ntok) * p.Hq;
  return x.units * p.Hkv <= 0x7fffffffll / 256 && x.part <= 0x7fffffffll && rows <= (1ll << 26) - 4;
}

template <int D, bool SHARED>
static hipError_t launch_rows(const PagedRows& p, const RowsArgs& a) {
  hipLaunchKernelGGL(rows_plan_kernel<SHARED>, dim3(1), dim3(kPlanThreads), 0, p.stream, a);
  prof_begin(SHARED ? "paged_decode_shared" : "paged_extend", p.stream);
  hipLaunchKernelGGL((rows_kernel<D, SHARED>), dim3((unsigned)(a.max_units * a.Hkv)), dim3(256), 0, p.stream, a);
  prof_end(p.stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const long long rows = (long long)a.ntok * a.Hq;
  hipLaunchKernelGGL((rows_merge_kernel<D, SHARED>), dim3((unsigned)((rows + 3) / 4)), dim3(256), 0, p.stream, a);
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
  a.window = p.window;
  a.sinks = p.sinks;
  a.scale_log2 = p.scale * 1.4426950408889634f;
  char* w = (char*)p.ws;
  auto take = [&](size_t bytes) {
    char* at = w;
    w += bytes;
    return at;
  };
  a.rank = (int*)take(x.rank);
  a.count = (int*)take(x.count);
  a.base = (int*)take(x.base);
  a.list = (int*)take(x.list);
  a.first = (int*)take(x.first);
  a.own = (Parts*)take(x.own);
  a.prefix = (Parts*)take(x.prefix);
  a.units = (Unit*)take(x.unit);
  a.part = (float*)take(x.rows);
  a.part_ml = (float2*)take(x.ml);
  a.max_units = (int)x.units;
  a.max_part = x.part;
  a.want = rows_want(p.Hkv);
  if (p.shared) return p.D == 128 ? launch_rows<128, true>(p, a) : launch_rows<64, true>(p, a);
  return p.D == 128 ? launch_rows<128, false>(p, a) : launch_rows<64, false>(p, a);
}

}  // namespace kvs
