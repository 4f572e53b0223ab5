// rows_common.cuh -- what the few-token attentions share: sequences as a call sees
// them, the cut of all units' tiles into runs, and the joining of cut units.
#pragma once
#include <math.h>

#include "common.cuh"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kJoinThreads = 128;
constexpr int kErrCount = 4, kErrTimeout = 8, kErrPage = 32;  // KVK_DEVERR_*
constexpr int kWholeCtx = 512;
constexpr uint32_t kWaits = 1u << 20;  // polls of up to 2 us each
constexpr uint32_t kAll = 0xffffffffu;

// (M, L, x) += (m, l, y): sums relative to 2^M; m = -inf: nothing
__device__ __forceinline__ void join(float &M, float &L, float4 &x, float m, float l, float4 y) {
  const float n = fmaxf(M, m);
  const float f = M == -INFINITY ? 0.f : fast_exp2(M - n), h = m == -INFINITY ? 0.f : fast_exp2(m - n);
  M = n;
  L = L * f + l * h;
  x.x = x.x * f + y.x * h;
  x.y = x.y * f + y.y * h;
  x.z = x.z * f + y.z * h;
  x.w = x.w * f + y.w * h;
}

// One sequence of the batch as the call sees it.
struct Seq {
  int q0, n, len;  // first token, tokens, positions held
};
__device__ __forceinline__ Seq load_seq(const PagedView &v, int b, int max_new) {
  Seq s;
  const int e0 = v.cu[b], e1 = v.cu[b + 1], len = v.lens[b];
  const int c0 = min(max(e0, 0), v.n_tokens);
  s.n = min(max(e1, c0), v.n_tokens) - c0;
  s.q0 = c0;
  s.len = max(len, 0);
  const int64_t cap = (int64_t)v.max_pages << v.page_shift;
  if (s.n > 0 && (s.n > max_new || s.len > cap)) {
    set_err(v.err, kErrCount);
    s.n = min(s.n, max_new);
    s.len = (int)min((int64_t)s.len, cap);
  }
  return s;
}
// Positions from lo (a multiple of the tile) in nt tiles that the new tokens see;
// at least one tile, so that rows that see nothing get their zeros.
__device__ __forceinline__ void seq_range(const Seq &s, const AttnArgs &a, int &lo, int &nt) {
  const int sh = a.pt_shift;
  lo = max(0, s.len - s.n - a.window + 1) >> sh << sh;
  nt = max(1, (s.len - 1 + (1 << sh) - lo) >> sh);
}

// A place in the list of tiles.
struct At {
  int b, h, t;       // sequence, unit of KV heads, tile of the unit
  int lo, nt;        // the unit's first position and tiles
  Seq s;
};

// The unit behind x's.
__device__ __forceinline__ void next_unit(const AttnArgs &a, int units, At &x) {
  x.t = 0;
  if (++x.h < units) return;
  x.h = 0;
  do {
    if (++x.b >= a.pv.B) return;  // behind the last unit: not used again
    x.s = load_seq(a.pv, x.b, a.max_new);
  } while (x.s.n == 0);
  seq_range(x.s, a, x.lo, x.nt);
}

// One warp: the run of this CTA, `mine` tiles from `at` on, of `share` tiles (units,
// where they are never cut) a CTA, `least` at least.
__device__ __forceinline__ void find_run(const AttnArgs &a, int units, int least, int lane, At &at_out, int &mine_out,
                                         int &share_out) {
  const PagedView &pv = a.pv;
  int64_t before = 0, total = 0;  // tiles of the sequences before this lane's chunk
  Seq sq = {0, 0, 0};
  int per = 0;
  auto chunk = [&](int b0) {
    const bool in = b0 + lane < pv.B;
    if (in) sq = load_seq(pv, b0 + lane, a.max_new);
    int lo = 0, nt = 0;
    if (in && sq.n > 0) seq_range(sq, a, lo, nt);
    per = a.whole && nt > 0 ? 1 : nt;
    uint32_t x = per;  // 32 sequences of at most 2^22 tiles
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t y = __shfl_up_sync(kAll, x, o);
      if (lane >= o) x += y;
    }
    return (int64_t)units * x;  // up to and with this lane's sequence
  };
  int64_t upto = 0;
  for (int b0 = 0; b0 < pv.B; b0 += 32) {
    upto = chunk(b0);
    total += __shfl_sync(kAll, upto, 31);
  }
  const int64_t share = max(div_pos(total + gridDim.x - 1, gridDim.x), (int64_t)(a.whole ? 1 : least));
  const int64_t w0 = share * blockIdx.x;
  if (lane == 0) mine_out = 0;
  __syncwarp();
  if (w0 < total) {
    for (int b0 = 0; b0 < pv.B; b0 += 32) {
      if (pv.B > 32) upto = chunk(b0);
      const uint32_t past = __ballot_sync(kAll, before + upto > w0);
      if (past) {
        if (lane == __ffs(past) - 1) {
          At x;
          x.b = b0 + lane;
          x.s = sq;
          const int64_t off = w0 - (before + upto - (int64_t)units * per);
          x.h = (int)div_pos(off, per);
          x.t = (int)(off - (int64_t)x.h * per);
          seq_range(x.s, a, x.lo, x.nt);
          at_out = x;
          mine_out = (int)min(share, total - w0);
          if (a.whole) {  // units to tiles
            int tiles = x.nt;
            for (int u = 1; u < (int)min(share, total - w0); ++u) {
              next_unit(a, units, x);
              tiles += x.nt;
            }
            mine_out = tiles;
          }
        }
        break;
      }
      before += __shfl_sync(kAll, upto, 31);
    }
  }
  if (lane == 0) share_out = (int)min(share, (int64_t)1 << 30);
}

// 4 channels (v-th four) of row r of a (sequence, KV head), divided by its sum.
// A row before position 0 sees nothing and gives zeros.
template <int D, bool BF16>
__device__ __forceinline__ void store_row(const AttnArgs &a, int q0, int p_base, int head, int r, int v, float4 x, float L) {
  const int j = r / a.G;
  const bool sees = p_base + j >= 0;
  const float inv = sees ? 1.f / L : 0.f;
  if (!sees) x = make_float4(0.f, 0.f, 0.f, 0.f);
  uint8_t *dst = static_cast<uint8_t *>(a.out) + 2 * (((int64_t)(q0 + j) * a.Hq + head * a.G + (r - j * a.G)) * D + 4 * v);
  *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<BF16>(x.x * inv, x.y * inv), pack2<BF16>(x.z * inv, x.w * inv));
}

// Joins the pieces of the units that the first kernel cut.  A thread takes 4
// channels of a row; a CTA has one row, its groups of threads every
// `groups`-th piece and meeting in shared memory, where there are rows for no
// more (long contexts of few sequences), else a row per group.  The last CTA
// clears the list for the next call.
template <int D, bool BF16>
__global__ void __launch_bounds__(kJoinThreads) attn_join_kernel(const AttnArgs a) {
  constexpr int V = D / 4, groups = kJoinThreads / V, U = 8;
  __shared__ float4 sx[kJoinThreads];
  __shared__ float2 sl[kJoinThreads];
  const int tid = threadIdx.x, v = tid % V, grp = tid / V;
  const int rows = a.hc * a.rows;
  pdl_wait();
  const int n = min(*reinterpret_cast<volatile int *>(&a.list->n), kRowsMaxCtas) * rows;
  const bool wide = n <= (int)gridDim.x;
  const int step = wide ? groups : 1;
  for (int item = wide ? blockIdx.x : blockIdx.x * groups + grp; item < n; item += gridDim.x * (wide ? 1 : groups)) {
    const RowsSplit u = a.list->unit[item / rows];
    const int y = item % rows, c0 = u.first, hd = y / u.rows, r = y - hd * u.rows;
    if (y >= a.hc * u.rows) continue;
    float M = -INFINITY, L = 0.f;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p0 = c0 + (wide ? grp : 0); p0 <= u.last; p0 += U * step) {
      float4 z[U];
      float pm[U], pl[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int p = p0 + i * step;
        const float *src = a.part + ((int64_t)(2 * p + (p == c0)) * kRowsMaxHeads + hd) * rows_part(D);
        const bool in = p <= u.last;
        z[i] = in ? __ldcg(reinterpret_cast<const float4 *>(src + r * D + 4 * v)) : make_float4(0.f, 0.f, 0.f, 0.f);
        pm[i] = in ? __ldcg(src + kRowsPerUnit * D + r) : -INFINITY;
        pl[i] = in ? __ldcg(src + kRowsPerUnit * (D + 1) + r) : 0.f;
      }
#pragma unroll
      for (int i = 0; i < U; ++i) join(M, L, x, pm[i], pl[i], z[i]);
    }
    if (wide) {
      sx[tid] = x;
      sl[tid] = make_float2(M, L);
      __syncthreads();
      if (grp > 0) break;
#pragma unroll
      for (int i = 1; i < groups; ++i) join(M, L, x, sl[tid + i * V].x, sl[tid + i * V].y, sx[tid + i * V]);
    }
    store_row<D, BF16>(a, u.q0, u.p_base, u.head + hd, r, v, x, L);
  }
  pdl_trigger();
  // every CTA has read n before it counts itself
  __syncthreads();
  if (tid == 0) {
    __threadfence();
    if (atomicInc(&a.list->done, gridDim.x - 1) == gridDim.x - 1) a.list->n = 0;
  }
}

}  // namespace
}  // namespace kvk
