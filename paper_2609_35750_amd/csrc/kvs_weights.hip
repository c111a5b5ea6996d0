// gfx950 kernels of the attention weight every key of a trace has received:
//
//   W_j = sum_{h} sum_{i sees j} exp(s_ij^h - LSE_i^h),   s_ij^h = scale <Q_i^h, K_j^g>
//
// the column sums of the softmax matrix over all q-heads (or over the last
// queries of each trace only), which is what an eviction by accumulated
// attention weight starts from when a prompt or a replayed trace enters the
// cache.  LSE is the forward's, so there is neither a running maximum nor a
// second pass: one product, one exponential and one addition per score.
//
// Work: a workgroup takes 256 keys of one KV head and a chunk of query rows,
// all q-heads of the group or some of them, in steps of 64 rows of one q-head.
// K stays in registers as the B operand (lane <-> key), Q and LSE of a step are
// staged in LDS, so a lane sums its own key's column and no score is ever
// exchanged.  A wave takes 64 of the keys: every Q operand read from LDS serves
// two products (with one, the four SIMDs would ask for all of the LDS
// bandwidth), and the products of the two are the two chains that keep the
// matrix core fed.  Chunks cut long columns into items of about equal length
// without a plan (by the trace's length: under a window the block with the
// sinks, which all rows see, has far longer items than the others); their sums
// are added, heads and chunks in order, by a second kernel, so the result does
// not depend on the order in which the workgroups run.
//
// 16 products and 96 vector operations of a wave for every 32 rows x 64 keys.
// 16k trace with evicted segments (32/8 heads, D = 128): 498 us of a call of
// 506, 966 TFLOP/s, where a large matrix product reaches 1,336. Bound by the
// sum of its parts, which do not hide each other: the matrix core is busy for
// 44% of the time and the vector unit for 56%, at 2.0 GHz, and of 528 us
// (passes without pause) the call loses 73 without the exponentials, 45
// without the copies and 181 without seven in eight of the products. Other
// forms, each measured beside the one of its time (the last of those 542): two
// waves a SIMD that hold two pairs of accumulators, the exponentials of one
// between the products of the other, 559, no faster than these three; 128 keys
// a workgroup, twice the copies, 590; class and addresses found for every step
// and LSE scaled on the way to LDS 757.
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>
#include <type_traits>

namespace kvs {

constexpr int kWeightKeys = 256;   // keys of a workgroup
constexpr int kWeightStep = 64;    // query rows of a step

struct WeightArgs {
  const uint16_t* q;
  const uint16_t* k;
  const float* lse;
  float* lse2;          // LSE * log2(e), in LSE's layout (rows that count)
  const int* evict;     // NULL: nothing is evicted
  int* until;           // last query's index + 1 of every key (evict_at under the window)
  const int* cu;
  int2* kstats;
  float* part;          // [nchunk][Hkv][nhp][ntok]: sums of a chunk's rows over a part of the group's q-heads
  float* w;             // [ntok]
  int B, T, Hq, Hkv, G, ntok, nkb, nchunk, chunk_rows, last_rows;
  int nhp, part_heads;  // parts of the group's q-heads, q-heads of a part
  int varlen, window, sinks;
  float scale_log2;
};

// Key-tile statistics in the first nks workgroups; LSE in the form the products use it in the others, one thread a value
// (a launch for both, and the main kernel copies the values to LDS as they are).
__global__ void __launch_bounds__(256) key_weights_pre_kernel(WeightArgs a, int nks) {
  if ((int)blockIdx.x < nks) {
    kstats_group(a.evict, a.cu, a.T, a.ntok, blockIdx.x, kstats_groups(a.T), a.kstats, {a.window, a.sinks, a.until});
    return;
  }
  const int rows = (a.last_rows + 255) / 256;   // groups of 256 rows, counted from the end of the trace
  int wg = blockIdx.x - nks;
  const int r = wg % rows * 256 + threadIdx.x;
  wg /= rows;
  const int h = wg % a.Hq, b = wg / a.Hq;
  const Trace tr = trace_of(a.cu, b, a.T, a.ntok);
  const int i = tr.L - 1 - r;
  if (i < 0 || r >= a.last_rows) return;
  const long long li = a.varlen ? (long long)h * a.ntok + tr.tok0 + i : ((long long)b * a.Hq + h) * a.T + i;
  a.lse2[li] = a.lse[li] * 1.4426950408889634f;
}

// Rows of a trace that count, and the chunks of them that see any of the kWeightKeys keys from j0 on.
struct WeightRange {
  int r0;        // first row that counts
  int lo, hi;    // rows [lo, hi) counted from r0 see some key
  int c_lo, c_hi;
};
__device__ __forceinline__ WeightRange weight_range(const WeightArgs& a, const Trace& tr, int b, int j0) {
  const int t0 = j0 / kKeyTile, nt = (tr.L + kKeyTile - 1) / kKeyTile;
  int emax = 0;
#pragma unroll
  for (int t = 0; t < kWeightKeys / kKeyTile; ++t)
    emax = max(emax, a.kstats[kstat_index(b, tr.tok0, min(t0 + t, nt - 1), kKeyTile)].y);
  WeightRange r;
  r.r0 = max(tr.L - a.last_rows, 0);
  r.lo = max(j0 - r.r0, 0);
  r.hi = emax - r.r0;
  r.c_lo = r.lo / a.chunk_rows;
  r.c_hi = r.hi > r.lo ? (r.hi + a.chunk_rows - 1) / a.chunk_rows : r.c_lo;
  return r;
}

template <int D>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(D == 128 ? 3 : 4, D == 128 ? 3 : 4)))
key_weights_kernel(WeightArgs a) {
  constexpr int KS = D / 16, PITCH = Lay<D, true>::PITCH, TILE = kWeightStep * PITCH;
  __shared__ __attribute__((aligned(1024))) uint16_t sQ[2 * TILE];                  // two tiles of Q rows,
  __shared__ __attribute__((aligned(256))) float sL[2 * kWeightStep];              // and their LSE * log2(e)

  int wg = blockIdx.x;
  const int g = wg % a.Hkv;
  wg /= a.Hkv;
  const int hp = wg % a.nhp;
  wg /= a.nhp;
  const int kb = wg % a.nkb;
  wg /= a.nkb;
  const int h0 = g * a.G + hp * a.part_heads, nh = min(a.part_heads, a.G - hp * a.part_heads);   // the item's q-heads
  const int c = a.nchunk - 1 - wg % a.nchunk, b = wg / a.nchunk;   // the last rows, which see the most keys, first
  const Trace tr = trace_of(a.cu, b, a.T, a.ntok);
  const int j0 = kb * kWeightKeys;
  if (j0 >= min(max(tr.L - a.last_rows, 0) + (c + 1) * a.chunk_rows, tr.L)) return;   // all rows above the diagonal
  const WeightRange rg = weight_range(a, tr, b, j0);
  if (c < rg.c_lo || c >= rg.c_hi) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int kw = j0 + 64 * wave;   // the wave's first key
  const auto rl = Lay<D, true>::row_lane(lane);

  // this lane's two keys
  bf16x8 kreg[2][KS];
  int key[2], until[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int j = kw + 32 * n + col, jc = min(j, tr.L - 1);
    key[n] = j;
    until[n] = a.until[tr.tok0 + jc];
    const uint16_t* src = a.k + ((size_t)(tr.tok0 + jc) * a.Hkv + g) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kreg[n][ks] = as_bf16x8(*reinterpret_cast<const uint4*>(src + 16 * ks));
  }
  float acc[2] = {0.f, 0.f};

  // the item's rows [i_lo, i_hi), a step 64 of them and one q-head, heads fastest
  const int i_lo = rg.r0 + max(c * a.chunk_rows, rg.lo / kWeightStep * kWeightStep);
  const int i_hi = rg.r0 + min((c + 1) * a.chunk_rows, rg.hi);
  RowStager<D, kWeightStep, 4, true> qst;
  qst.init(wave, lane, (long long)a.Hq * D);
  const uint32_t tile_lds = lds_addr(sQ), word_lds = lds_addr(sL);
  // what is staged next: first row, q-head, and the addresses of its first row of Q and its first LSE, advanced step
  // by step (from the step they are two 64-bit products of every wave, ahead of the copies)
  const long long word_step = a.varlen ? a.ntok : a.T;
  int next_i = i_lo, next_h = 0;
  const uint16_t* next_q = a.q + ((size_t)(tr.tok0 + i_lo) * a.Hq + h0) * D;
  const float* next_l = a.lse2 + (a.varlen ? (long long)h0 * a.ntok + tr.tok0 : ((long long)b * a.Hq + h0) * a.T) + i_lo;
  auto stage = [&](int buf) __attribute__((always_inline)) {
    const int dr = tr.L - 1 - next_i;
    qst.issue_at(tile_lds + 2 * buf * TILE, uniform_ptr(next_q), qst.limit(dr, (long long)a.Hq * D), wave);
    if (wave == 3) stage_words_at(word_lds + 4 * buf * kWeightStep, uniform_ptr(next_l), dr, lane);
    const bool wrap = ++next_h == nh;
    next_h = wrap ? 0 : next_h;
    next_i += wrap ? kWeightStep : 0;
    next_q += D + (wrap ? (long long)kWeightStep * a.Hq * D - nh * D : 0ll);
    next_l += word_step + (wrap ? kWeightStep - nh * word_step : 0ll);
  };

  // The 32 rows from ib on (row m of the tile) x the wave's two groups of 32 keys.  C layout: lane <-> key, element r
  // <-> row 8 (r / 4) + 4 half + r % 4.
  unsigned span[2];   // rows j .. j + span - 1 see key j
  auto rows32 = [&](int buf, int m, int ib, auto masked) __attribute__((always_inline)) {
    constexpr int AHEAD = 3;   // operands in flight
    const uint16_t* tile = sQ + buf * TILE + m * PITCH;
    const float* words = sL + buf * kWeightStep + m + 4 * half;
    f32x16 x[2];
    bf16x8 qa[AHEAD];
    float4 l4[4];
#pragma unroll
    for (int ks = 0; ks < AHEAD; ++ks) qa[ks] = lds_read_b128(tile + Lay<D, true>::row_at(rl, ks));
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
      for (int n = 0; n < 2; ++n) x[n] = mfma32(qa[ks % AHEAD], kreg[n][ks], ks == 0 ? f32x16{} : x[n]);
      if (ks + AHEAD < KS) qa[ks % AHEAD] = lds_read_b128(tile + Lay<D, true>::row_at(rl, ks + AHEAD));
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) l4[q4] = *reinterpret_cast<const float4*>(words + 8 * q4);
    float s[2][4] = {};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const float l[4] = {l4[r >> 2].x, l4[r >> 2].y, l4[r >> 2].z, l4[r >> 2].w};
#pragma unroll
      for (int n = 0; n < 2; ++n) {
        float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], a.scale_log2, -l[r & 3]));
        if (decltype(masked)::value) {   // whatever a masked place holds
          const bool vis = (unsigned)(ib + 8 * (r >> 2) + 4 * half + (r & 3) - key[n]) < span[n];
          p = vis ? p : 0.f;
        }
        s[n][r & 3] += p;
      }
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) acc[n] += (s[n][0] + s[n][1]) + (s[n][2] + s[n][3]);
  };

  stage(0);
  wait_vm();   // and K: no load the compiler counts stays pending in the loop
  int emin = INT_MAX, emax = INT_MIN;   // over the wave's 64 keys
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int e = min(until[n], tr.L);
    const bool ok = key[n] < tr.L;
    span[n] = ok ? (unsigned)max(e - key[n], 0) : 0u;
    emin = min(emin, ok ? e : INT_MIN);   // keys past the trace: never FULL
    emax = max(emax, ok ? e : INT_MIN);
  }
  emin = wave_min(emin);
  emax = wave_max(emax);
  __syncthreads();
  int buf = 0;
  for (int i0 = i_lo; i0 < i_hi; i0 += kWeightStep) {
    const bool any = i0 + kWeightStep - 1 >= kw && i0 < emax;                         // some of the 64 x 64 visible
    const bool full = i0 >= kw + 63 && i0 + kWeightStep <= min(emin, tr.L);            // all of it
    for (int h = 0; h < nh; ++h) {
      if (h + 1 < nh || i0 + kWeightStep < i_hi) stage(buf ^ 1);
      if (any) {
#pragma unroll 1
        for (int m = 0; m < kWeightStep; m += 32) {
          if (full) rows32(buf, m, i0 + m, std::false_type{});
          else rows32(buf, m, i0 + m, std::true_type{});
        }
      }
      wait_vm();
      __syncthreads();
      buf ^= 1;
    }
  }

#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const float t = halves_sum(acc[n]);   // the rows of the other lane half
    if (half == 0 && key[n] < tr.L) a.part[(((size_t)c * a.Hkv + g) * a.nhp + hp) * a.ntok + tr.tok0 + key[n]] = t;
  }
}

// W of a trace's keys: the sums of all heads and of the chunks that see the key's block, in order.
__global__ void __launch_bounds__(kWeightKeys) key_weights_reduce_kernel(WeightArgs a) {
  const int kb = blockIdx.x % a.nkb, b = blockIdx.x / a.nkb;
  const Trace tr = trace_of(a.cu, b, a.T, a.ntok);
  const int j0 = kb * kWeightKeys, j = j0 + threadIdx.x;
  if (j >= tr.L) return;
  const WeightRange rg = weight_range(a, tr, b, j0);
  float s = 0.f;
  for (int c = rg.c_lo; c < min(rg.c_hi, a.nchunk); ++c)
#pragma unroll 8
    for (int g = 0; g < a.Hkv * a.nhp; ++g) s += a.part[((size_t)c * a.Hkv * a.nhp + g) * a.ntok + tr.tok0 + j];
  a.w[tr.tok0 + j] = s;
}

template __global__ void key_weights_kernel<64>(WeightArgs);
template __global__ void key_weights_kernel<128>(WeightArgs);

// ---------------------------------------------------------------- launcher
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// How the rows are cut: about kWeightItems items (half of them above the diagonal, empty), of whole steps; where those
// of one chunk do not start a workgroup on every CU, by q-heads too (24 traces of 100 to 1,500 tokens, the last 64
// queries, 16/2 heads: 26.0 us whole groups, 18.5 two heads a part, 22.1 one).  16k trace: 8,192 items 567 us in all, 16,384 575, 32,768 603.
struct WeightCut {
  int nkb, nchunk, chunk_rows, nhp, part_heads;
};
constexpr long long kWeightItems = 8192, kWeightLeast = 1024;
static WeightCut weight_cut(int B, int T, int Hkv, int G, int last_rows) {
  const long long rows = std::min(T, last_rows), nkb = (T + kWeightKeys - 1) / kWeightKeys, blocks = B * nkb * Hkv;
  const long long want = std::max(1ll, kWeightItems / blocks);
  WeightCut c;
  c.nkb = (int)nkb;
  c.chunk_rows = (int)(((rows + want - 1) / want + kWeightStep - 1) / kWeightStep * kWeightStep);
  c.nchunk = (int)((rows + c.chunk_rows - 1) / c.chunk_rows);
  c.part_heads = (int)std::max(1ll, std::min((long long)G, G * blocks * c.nchunk / kWeightLeast));
  c.nhp = (G + c.part_heads - 1) / c.part_heads;
  return c;
}
static size_t lse2_bytes(int ntok, int Hq) { return round256((size_t)ntok * Hq * sizeof(float)); }
size_t ws_weights_bytes(int B, int T, int ntok, int Hq, int Hkv, int last_rows) {
  const WeightCut c = weight_cut(B, T, Hkv, Hq / Hkv, last_rows);
  return lse2_bytes(ntok, Hq) + round256((size_t)c.nchunk * Hkv * c.nhp * ntok * sizeof(float));
}

static long long weights_main_grid(const WeightCut& c, int B, int Hkv) { return (long long)B * c.nchunk * c.nkb * Hkv * c.nhp; }
static long long weights_pre_grid(int B, int T, int Hq, int last_rows) {
  return (long long)B * (kstats_groups(T) + (long long)((std::min(T, last_rows) + 255) / 256) * Hq);
}
long long weights_grid(int B, int T, int Hq, int Hkv, int last_rows) {
  return std::max(weights_main_grid(weight_cut(B, T, Hkv, Hq / Hkv, last_rows), B, Hkv),
                  weights_pre_grid(B, T, Hq, last_rows));
}

hipError_t launch_key_weights(const Problem& p, int2* kstats, int last_rows, void* ws, float* w) {
  WeightArgs a{};
  a.q = (const uint16_t*)p.q;
  a.k = (const uint16_t*)p.k;
  a.lse = p.lse_in;
  a.lse2 = (float*)ws;
  a.evict = p.evict;
  a.until = p.until;
  a.window = p.window;
  a.sinks = p.sinks;
  a.cu = p.cu;
  a.kstats = kstats;
  a.part = (float*)((char*)ws + lse2_bytes(p.ntok, p.Hq));
  a.w = w;
  a.B = p.B;
  a.T = p.T;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.G;
  a.ntok = p.ntok;
  const WeightCut cut = weight_cut(p.B, p.T, p.Hkv, p.G, last_rows);
  a.nkb = cut.nkb;
  a.last_rows = std::min(last_rows, p.T);
  a.chunk_rows = cut.chunk_rows;
  a.nchunk = cut.nchunk;
  a.nhp = cut.nhp;
  a.part_heads = cut.part_heads;
  a.varlen = p.cu != nullptr;
  a.scale_log2 = p.scale * 1.4426950408889634f;
  hipLaunchKernelGGL(key_weights_pre_kernel, dim3((unsigned)weights_pre_grid(p.B, p.T, p.Hq, a.last_rows)), dim3(256), 0,
                     p.stream, a, kstats_groups(p.T) * p.B);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const dim3 grid((unsigned)weights_main_grid(cut, p.B, p.Hkv));
  prof_begin("key_weights", p.stream);
  if (p.D == 128) hipLaunchKernelGGL(key_weights_kernel<128>, grid, dim3(256), 0, p.stream, a);
  else hipLaunchKernelGGL(key_weights_kernel<64>, grid, dim3(256), 0, p.stream, a);
  prof_end(p.stream);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(key_weights_reduce_kernel, dim3((unsigned)(p.B * a.nkb)), dim3(kWeightKeys), 0, p.stream, a);
  return hipGetLastError();
}

}  // namespace kvs
