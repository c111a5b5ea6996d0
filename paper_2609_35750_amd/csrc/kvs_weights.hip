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
// Work: a workgroup takes 128 keys of one KV head and a chunk of query rows,
// all q-heads of the group, in steps of 64 rows of one q-head.  K stays in
// registers as the B operand (lane <-> key), Q and LSE of a step are staged in
// LDS, so a lane sums its own key's column and no score is ever exchanged.  A
// wave takes 64 keys x 32 rows: every Q operand read from LDS serves two
// products (with one, the four SIMDs would ask for all of the LDS bandwidth).
// Chunks cut long columns into items of about equal length without a plan;
// their sums are added, heads and chunks in order, by a second kernel, so the
// result does not depend on the order in which the workgroups run.
#include "kvs_device.h"
#include "kvs_launch.h"

#include <algorithm>
#include <climits>

namespace kvs {

constexpr int kWeightKeys = 128;   // keys of a workgroup
constexpr int kWeightStep = 64;    // query rows of a step

struct WeightArgs {
  const uint16_t* q;
  const uint16_t* k;
  const float* lse;
  const int* until;     // last query's index + 1 of every key (evict_at under the window)
  const int* cu;
  const int2* kstats;
  float* part;          // [nchunk][Hkv][ntok]: sums of a chunk's rows
  float* w;             // [ntok]
  int B, T, Hq, Hkv, G, ntok, nkb, nchunk, chunk_rows, last_rows;
  int varlen;
  float scale_log2;
};

// Rows of a trace that count, and the chunks of them that see any of the 128 keys from j0 on.
struct WeightRange {
  int r0;        // first row that counts
  int lo, hi;    // rows [lo, hi) counted from r0 see some key
  int c_lo, c_hi;
};
__device__ __forceinline__ WeightRange weight_range(const WeightArgs& a, const Trace& tr, int b, int j0) {
  const int t0 = j0 / kKeyTile, nt = (tr.L + kKeyTile - 1) / kKeyTile;
  int emax = a.kstats[kstat_index(b, tr.tok0, t0, kKeyTile)].y;
  if (t0 + 1 < nt) emax = max(emax, a.kstats[kstat_index(b, tr.tok0, t0 + 1, kKeyTile)].y);
  WeightRange r;
  r.r0 = max(tr.L - a.last_rows, 0);
  r.lo = max(j0 - r.r0, 0);
  r.hi = emax - r.r0;
  r.c_lo = r.lo / a.chunk_rows;
  r.c_hi = r.hi > r.lo ? (r.hi + a.chunk_rows - 1) / a.chunk_rows : r.c_lo;
  return r;
}

template <int D>
__global__ void __launch_bounds__(256) key_weights_kernel(WeightArgs a) {
  constexpr int KS = D / 16, PITCH = Lay<D, true>::PITCH;
  __shared__ __attribute__((aligned(1024))) uint16_t sQ0[kWeightStep * PITCH];
  __shared__ __attribute__((aligned(1024))) uint16_t sQ1[kWeightStep * PITCH];
  __shared__ __attribute__((aligned(16))) float sL[2][kWeightStep];   // LSE * log2(e)
  __shared__ float sum[2][kWeightKeys];

  int wg = blockIdx.x;
  const int g = wg % a.Hkv;
  wg /= a.Hkv;
  const int kb = wg % a.nkb;
  wg /= a.nkb;
  const int c = a.nchunk - 1 - wg % a.nchunk, b = wg / a.nchunk;   // the last rows, which see the most keys, first
  const Trace tr = trace_of(a.cu, b, a.T, a.ntok);
  const int j0 = kb * kWeightKeys;
  if (j0 >= tr.L) return;
  const WeightRange rg = weight_range(a, tr, b, j0);
  if (c < rg.c_lo || c >= rg.c_hi) return;

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int half = lane >> 5, col = lane & 31;
  const int rb = 32 * (wave >> 1), kw = j0 + 64 * (wave & 1);   // the wave's rows of a step, its first key
  const auto rl = Lay<D, true>::row_lane(lane);

  // this lane's two keys
  bf16x8 kreg[2][KS];
  int key[2], emin[2], emax[2];
  unsigned span[2];
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const int j = kw + 32 * n + col, jc = min(j, tr.L - 1);
    const int e = min(a.until[tr.tok0 + jc], tr.L);
    key[n] = j;
    span[n] = j < tr.L ? (unsigned)max(e - j, 0) : 0u;   // rows j .. e - 1 see the key
    emin[n] = wave_min(j < tr.L ? e : INT_MAX);
    emax[n] = wave_max(j < tr.L ? e : INT_MIN);
    const uint16_t* src = a.k + ((size_t)(tr.tok0 + jc) * a.Hkv + g) * D + 8 * half;
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) kreg[n][ks] = as_bf16x8(*reinterpret_cast<const uint4*>(src + 16 * ks));
  }
  float acc[2] = {0.f, 0.f};

  // steps of the item: (64 rows, q-head of the group), heads fastest; rows counted from r0
  const int row_lo = max(c * a.chunk_rows, rg.lo / kWeightStep * kWeightStep);
  const int row_hi = min((c + 1) * a.chunk_rows, rg.hi);
  const int steps = (row_hi - row_lo + kWeightStep - 1) / kWeightStep * a.G;
  RowStager<D, kWeightStep, 4, true> qst;
  qst.init(wave, lane, (long long)a.Hq * D);
  struct Pos {
    int i0, hh;
  };
  auto advance = [&](Pos& p) __attribute__((always_inline)) {
    const bool wrap = ++p.hh == a.G;
    p.hh = wrap ? 0 : p.hh;
    p.i0 += wrap ? kWeightStep : 0;
  };
  Pos next = {rg.r0 + row_lo, 0}, cur = next;
  auto stage = [&](uint16_t* tile, float* words) __attribute__((always_inline)) {
    const int h = g * a.G + next.hh;
    qst.issue(lds_addr(tile), a.q + ((size_t)tr.tok0 * a.Hq + h) * D, (long long)a.Hq * D, next.i0, tr.L - 1, wave);
    if (wave == 3) {
      const int i = min(next.i0 + lane, tr.L - 1);
      const long long li = a.varlen ? (long long)h * a.ntok + tr.tok0 + i : ((long long)b * a.Hq + h) * a.T + i;
      words[lane] = a.lse[li] * 1.4426950408889634f;
    }
    advance(next);
  };
  auto compute = [&](const uint16_t* tile, const float* words) __attribute__((always_inline)) {
    const int ib = cur.i0 + rb;
    int cls[2];
#pragma unroll
    for (int n = 0; n < 2; ++n) cls[n] = tile_class(ib, ib + 32, kw + 32 * n, kw + 32 * n + 32, tr.L, emin[n], emax[n]);
    advance(cur);
    if (cls[0] == kEmpty && cls[1] == kEmpty) return;
    f32x16 x[2] = {};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const bf16x8 qa = lds_read_b128(tile + rb * PITCH + Lay<D, true>::row_at(rl, ks));
#pragma unroll
      for (int n = 0; n < 2; ++n) x[n] = mfma32(qa, kreg[n][ks], x[n]);
    }
    float l2[16];
#pragma unroll
    for (int q4 = 0; q4 < 4; ++q4) {
      const float4 l4 = *reinterpret_cast<const float4*>(words + rb + 8 * q4 + 4 * half);
      l2[4 * q4] = l4.x, l2[4 * q4 + 1] = l4.y, l2[4 * q4 + 2] = l4.z, l2[4 * q4 + 3] = l4.w;
    }
#pragma unroll
    for (int n = 0; n < 2; ++n) {
      if (cls[n] == kEmpty) continue;
      float s[4] = {0.f, 0.f, 0.f, 0.f};
      if (cls[n] == kFull) {
#pragma unroll
        for (int r = 0; r < 16; ++r) s[r & 3] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], a.scale_log2, -l2[r]));
      } else {
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(x[n][r], a.scale_log2, -l2[r]));
          const bool vis = (unsigned)(ib + 8 * (r >> 2) + 4 * half + (r & 3) - key[n]) < span[n];
          s[r & 3] += vis ? p : 0.f;   // whatever a masked place holds
        }
      }
      acc[n] += (s[0] + s[1]) + (s[2] + s[3]);
    }
  };

  stage(sQ0, sL[0]);
  wait_vm();
  __syncthreads();
  for (int step = 0; step < steps; step += 2) {
    if (step + 1 < steps) stage(sQ1, sL[1]);
    compute(sQ0, sL[0]);
    wait_vm();
    __syncthreads();
    if (step + 1 >= steps) break;
    if (step + 2 < steps) stage(sQ0, sL[0]);
    compute(sQ1, sL[1]);
    wait_vm();
    __syncthreads();
  }

  // the rows of the other lane half and of the other wave with these keys
#pragma unroll
  for (int n = 0; n < 2; ++n) {
    const float t = halves_sum(acc[n]);
    if (half == 0) sum[wave >> 1][64 * (wave & 1) + 32 * n + col] = t;
  }
  __syncthreads();
  const int j = j0 + tid;
  if (tid < kWeightKeys && j < tr.L)
    a.part[((size_t)c * a.Hkv + g) * a.ntok + tr.tok0 + j] = sum[0][tid] + sum[1][tid];
}

// W of a trace's keys: the sums of all heads and of the chunks that see the key's block, in order.
__global__ void __launch_bounds__(128) key_weights_reduce_kernel(WeightArgs a) {
  const int kb = blockIdx.x % a.nkb, b = blockIdx.x / a.nkb;
  const Trace tr = trace_of(a.cu, b, a.T, a.ntok);
  const int j0 = kb * kWeightKeys, j = j0 + threadIdx.x;
  if (j >= tr.L) return;
  const WeightRange rg = weight_range(a, tr, b, j0);
  float s = 0.f;
  for (int c = rg.c_lo; c < min(rg.c_hi, a.nchunk); ++c)
#pragma unroll 8
    for (int g = 0; g < a.Hkv; ++g) s += a.part[((size_t)c * a.Hkv + g) * a.ntok + tr.tok0 + j];
  a.w[tr.tok0 + j] = s;
}

template __global__ void key_weights_kernel<64>(WeightArgs);
template __global__ void key_weights_kernel<128>(WeightArgs);

// ---------------------------------------------------------------- launcher
static size_t round256(size_t n) { return (n + 255) & ~(size_t)255; }

// Items of about kWeightItems in all (half of them above the diagonal, empty), of whole steps.
constexpr long long kWeightItems = 32768;
static int weight_chunk_rows(int B, int T, int Hkv, int last_rows) {
  const long long rows = std::min(T, last_rows), nkb = (T + kWeightKeys - 1) / kWeightKeys;
  const long long want = std::max(1ll, kWeightItems / (B * nkb * Hkv));
  return (int)(((rows + want - 1) / want + kWeightStep - 1) / kWeightStep * kWeightStep);
}
static int weight_chunks(int B, int T, int Hkv, int last_rows) {
  const int per = weight_chunk_rows(B, T, Hkv, last_rows);
  return (std::min(T, last_rows) + per - 1) / per;
}
long long weights_grid(int B, int T, int Hkv, int last_rows) {
  return (long long)B * weight_chunks(B, T, Hkv, last_rows) * ((T + kWeightKeys - 1) / kWeightKeys) * Hkv;
}
size_t ws_weights_bytes(int B, int T, int ntok, int Hkv, int last_rows) {
  return round256((size_t)weight_chunks(B, T, Hkv, last_rows) * Hkv * ntok * sizeof(float));
}

hipError_t launch_key_weights(const Problem& p, const int2* kstats, int last_rows, float* part, float* w) {
  WeightArgs a{};
  a.q = (const uint16_t*)p.q;
  a.k = (const uint16_t*)p.k;
  a.lse = p.lse_in;
  a.until = p.until;
  a.cu = p.cu;
  a.kstats = kstats;
  a.part = part;
  a.w = w;
  a.B = p.B;
  a.T = p.T;
  a.Hq = p.Hq;
  a.Hkv = p.Hkv;
  a.G = p.G;
  a.ntok = p.ntok;
  a.nkb = (p.T + kWeightKeys - 1) / kWeightKeys;
  a.last_rows = std::min(last_rows, p.T);
  a.chunk_rows = weight_chunk_rows(p.B, p.T, p.Hkv, last_rows);
  a.nchunk = weight_chunks(p.B, p.T, p.Hkv, last_rows);
  a.varlen = p.cu != nullptr;
  a.scale_log2 = p.scale * 1.4426950408889634f;
  const dim3 grid((unsigned)weights_grid(p.B, p.T, p.Hkv, last_rows));
  prof_begin("key_weights", p.stream);
  if (p.D == 128) hipLaunchKernelGGL(key_weights_kernel<128>, grid, dim3(256), 0, p.stream, a);
  else hipLaunchKernelGGL(key_weights_kernel<64>, grid, dim3(256), 0, p.stream, a);
  prof_end(p.stream);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(key_weights_reduce_kernel, dim3((unsigned)(p.B * a.nkb)), dim3(kWeightKeys), 0, p.stream, a);
  return hipGetLastError();
}

}  // namespace kvs
