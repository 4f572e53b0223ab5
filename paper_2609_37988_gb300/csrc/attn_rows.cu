// attn_rows.cu -- attention of a few new tokens per sequence over a paged
// cache (single tokens, drafted ones): bound by the cache's bytes.
//
// Query j of sequence b sits at position p = len_b - n_b + j and sees
// positions max(0, p - window + 1) .. p; head h reads KV head h / G.  Rows
// r = j G + (head in its group), at most 8 or 16 of a (sequence, KV head), make a
// unit, so that a key or value byte is read once for all of them; with small
// pages a unit takes HC = 2 or 4 KV heads side by side, whose parts of a page
// adjoin, so that a copy is 16 KB either way.  A unit's positions go in tiles of
// 64 / HC; the tiles of all units, one behind another, are cut into equal runs,
// one per CTA (two CTAs per SM are resident), whatever the sequences' lengths
// are.  A unit that a run covers whole is written at once; the pieces of the
// others go to the workspace, with a note of where they lie, and a second kernel
// joins them, a CTA per row (one CTA per unit that did it behind its own run
// took 50 us for 152 pieces of 20 rows).  Where no sequence can have more than
// kWholeCtx positions, CTAs take whole units of one KV head and nothing has to
// be joined: the second launch costs the caller more than the longer runs do.
//
// A CTA: 4 warps, 16 positions of one head's tile each, and a warp that looks
// up pages and copies key and value tiles by TMA through a ring (96 KB; each
// half of a tile is refilled as soon as the four warps have read it).  Scores
// and results are computed transposed, S^T = K Q^T and O^T += V^T P^T on
// mma.m16n8k16 (positions and channels in the 16, query rows in the 8: few rows
// waste little), fp32 accumulation, the softmax online in base 2, each warp with
// its own maxima and sums; P enters as hi + lo halves (f16: 2^14 times as large, so
// that small weights stay normal).  Measured: a 14B-shaped step over 32 x 8192
// positions in pages of 16, 165 us (6.5 TB/s, 96 % of the copy bandwidth); 8 x 8192
// 51 us, 1 x 8192 15 us, of which 10 are start and joining.
//
// Non-finite values: weight 0 times an infinite value would be NaN, so tiles
// that some row does not see in full are looked through first, and a warp whose
// 16 positions have such a value adds them by plain arithmetic, row by row.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"
#include "umma.cuh"

namespace kvk {
namespace {

constexpr int kT = 64;        // positions x KV heads of a tile
constexpr int kThreads = 128;  // that compute; a warp beside them copies
constexpr int kErrCount = 4, kErrTimeout = 8, kErrPage = 32;  // KVK_DEVERR_*
constexpr int kMinShare = 4;   // tiles of a run at least
constexpr int kWholeCtx = 512;
constexpr uint32_t kWaits = 1u << 20;  // polls of up to 2 us each
constexpr uint32_t kAll = 0xffffffffu;

template <bool BF16>
__device__ __forceinline__ bool pair_finite(uint32_t w) {
  constexpr uint32_t m = BF16 ? 0x7F80u : 0x7C00u;
  return (w & m) != m && (w >> 16 & m) != m;
}

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

struct RowsArgs {
  CUtensorMap mk, mv;
  AttnArgs a;
};

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
__global__ void __launch_bounds__(kThreads) attn_join_kernel(const AttnArgs a) {
  constexpr int V = D / 4, groups = kThreads / V, U = 8;
  __shared__ float4 sx[kThreads];
  __shared__ float2 sl[kThreads];
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

template <int D>
constexpr int rows_stages() { return D == 128 ? 6 : 12; }  // key and value tiles in turn

// NB: query rows of a unit in blocks of 8
template <int D, int NB, bool BF16>
__global__ void __launch_bounds__(kThreads + 32, 2) attn_rows_kernel(const __grid_constant__ RowsArgs ra) {
  constexpr int RB = D * 2;            // bytes of a row
  constexpr int kTile = kT * RB;       // bytes of a key (or value) tile
  constexpr int KS = D / 16, NS = rows_stages<D>(), RU = 8 * NB;
  // Weights are at most 1: the reference is the largest score so far.  In f16 those
  // below 2^-14 would lose bits to the type's subnormals and those below 2^-25 all of
  // them, while the row's sum has them whole.  Kept 2^14 times as large (the sum too:
  // the quotient is the same) they are off by 2^-39 of the largest at most.
  constexpr float kShift = BF16 ? 0.f : 14.f;
  const AttnArgs &a = ra.a;
  extern __shared__ uint8_t sm_raw[];
  uint8_t *sm = sm_raw + ((1024u - (smem_u32(sm_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_full[NS], s_free[NS];
  __shared__ int s_abort, s_mine, s_share;
  __shared__ At s_at;
  __shared__ float2 s_ml[4][RU];
  const PagedView &pv = a.pv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, c = lane & 3;
  const int HC = a.hc, units = pv.Hkv / HC;
  const int per_head = 4 / HC, hh = warp / per_head, sub = warp % per_head;  // the warp's head and positions
  if (tid == 128) {
    prefetch_tensor_map(&ra.mk);
    prefetch_tensor_map(&ra.mv);
  }
  if (tid == 64) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], kThreads / 32);
    }
    s_abort = 0;
    fence_mbar_init();
  }
  pdl_wait();

  auto next_unit = [&](At &x) {
    x.t = 0;
    if (++x.h < units) return;
    x.h = 0;
    do {
      if (++x.b >= pv.B) return;  // behind the last unit: not used again
      x.s = load_seq(pv, x.b, a.max_new);
    } while (x.s.n == 0);
    seq_range(x.s, a, x.lo, x.nt);
  };

  // the run of this CTA: `mine` tiles from s_at on
  if (warp == 0) {
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
    const int64_t share = max(div_pos(total + gridDim.x - 1, gridDim.x), (int64_t)(a.whole ? 1 : kMinShare));
    const int64_t w0 = share * blockIdx.x;
    if (lane == 0) s_mine = 0;
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
            s_at = x;
            s_mine = (int)min(share, total - w0);
            if (a.whole) {  // units to tiles
              int tiles = x.nt;
              for (int u = 1; u < (int)min(share, total - w0); ++u) {
                next_unit(x);
                tiles += x.nt;
              }
              s_mine = tiles;
            }
          }
          break;
        }
        before += __shfl_sync(kAll, upto, 31);
      }
    }
    if (lane == 0) s_share = (int)min(share, (int64_t)1 << 30);
  }
  __syncthreads();
  const int mine = s_mine;
  if (mine == 0) {
    pdl_trigger();
    return;
  }
  At at = s_at;

  volatile int *abort_flag = &s_abort;
  auto wait = [&](uint64_t *bar, uint32_t parity) {
    if (mbar_wait_or_abort(bar, parity, kWaits, abort_flag)) return true;
    *abort_flag = 1;
    return false;
  };
  int stage = 0;  // place in the ring and its round's parity
  uint32_t par = 0;
  auto next_stage = [&]() {
    if (++stage == NS) stage = 0, par ^= 1;
  };

  // a tile in shared memory: per part (the positions of one page, at most 64)
  // and KV head boxes of 64 channels, 128-byte-swizzled rows
  const int pt = 1 << a.pt_shift, shift = a.part_shift, parts = pt >> shift, box = 128 << shift;
  auto row_at = [&](int r) { return ((r >> shift) * HC + hh) * (RB << shift) + (r & ((1 << shift) - 1)) * 128; };

  if (warp == kThreads / 32) {
    // -- copies: a lane per part of a tile, its page looked up a tile ahead;
    // outside the pool reads as zeros.  Parts that no query sees (a window may
    // begin inside a tile) have no page: their entries may be stale.
    auto seen = [&](const At &x) {
      const int t = x.lo + x.t * pt + (lane << shift);
      return lane < parts && t < x.s.len && t + (1 << shift) > x.s.len - x.s.n - a.window + 1;
    };
    auto look_up = [&](const At &x) {
      const int t = x.lo + x.t * pt + (lane << shift);
      return seen(x) ? pv.table[(int64_t)x.b * pv.max_pages + (t >> pv.page_shift)] : pv.n_pages;
    };
    int page = look_up(at);
    // (asked once: a limit from the arguments in the loop's waits cost 1.3 %)
    bool ok = !a.give_up;
    if (!ok && lane == 0) *abort_flag = 1;
    for (int w = 0; w < mine && ok; ++w) {
      const int t = at.lo + at.t * pt + (lane << shift);
      const int y = t & ((1 << pv.page_shift) - 1), h = at.h * HC;
      int now = page;
      if ((unsigned)now >= (unsigned)pv.n_pages) {
        if (seen(at)) set_err(pv.err, kErrPage);
        now = pv.n_pages;
      }
      if (w + 1 < mine) {
        if (++at.t >= at.nt) next_unit(at);
        page = look_up(at);
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        int got = 1;
        if (lane == 0) {
          got = wait(&s_free[stage], par ^ 1);
          if (got) mbar_expect_tx(&s_full[stage], kTile);
        }
        ok = __shfl_sync(kAll, got, 0) != 0;
        if (!ok) break;
        if (lane < parts)
          tma_load_5d(sm + stage * kTile + (lane << shift) * RB * HC, kv ? &ra.mv : &ra.mk, 0, y, 0, h, now, &s_full[stage]);
        next_stage();
      }
    }
    pdl_trigger();
    // the copies in flight land before the CTA ends, whoever waits for them: the
    // other warps may give up after this one is through
    if (lane == 0) {
      for (int i = 0; i < NS; ++i) {
        if (par == 0 && i >= stage) break;
        mbar_wait(&s_full[i], i < stage ? par : par ^ 1, kWaits);
      }
      if (*abort_flag) set_err(pv.err, kErrTimeout);
    }
    return;
  }

  auto bar_sync = [&]() { asm volatile("bar.sync 1, %0;" ::"n"(kThreads) : "memory"); };
  auto any_of_all = [&](bool x) {  // a bar_sync too
    uint32_t r;
    asm volatile("{\n .reg .pred p, q;\n setp.ne.u32 q, %1, 0;\n bar.red.or.pred p, 1, %2, q;\n selp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(r)
                 : "r"(x ? 1u : 0u), "n"(kThreads)
                 : "memory");
    return r != 0;
  };
  auto release = [&](int at_stage) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&s_free[at_stage]);
  };
  // lanes' rows of a 16-position tile: of the keys as the A operand, of the
  // values as its transpose
  const int rk = sub * 16 + (lane & 15), xk = lane >> 4, at_k = row_at(rk);
  const int rv = sub * 16 + (lane & 7) + ((lane & 16) >> 1), xv = (lane >> 3) & 1, at_v = row_at(rv);
  for (int w = 0; w < mine;) {
    // a piece: tiles [t_begin, t_end) of one unit
    const int t_begin = at.t, t_end = min(at.nt, at.t + (mine - w)), w_begin = w;
    const int R = at.s.n * a.G;
    const int p_base = at.s.len - at.s.n;
    // Q^T as the B operand (row 8 nb + g), and the positions that rows
    // 8 nb + 2 c + e see
    uint32_t qf[KS][NB][2];
    int lim[2 * NB], low[2 * NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = 8 * nb + g, j = r / a.G;
      const bool real = r < R;
      const uint8_t *src = a.q.p + 2 * ((int64_t)(at.s.q0 + (real ? j : 0)) * a.q.ts +
                                        (int64_t)((at.h * HC + hh) * a.G + (real ? r - j * a.G : 0)) * a.q.hs);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          qf[k][nb][x] = real ? *reinterpret_cast<const uint32_t *>(src + 32 * k + 16 * x + 4 * c) : 0u;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * nb + 2 * c + e;
        lim[2 * nb + e] = rr < R ? p_base + rr / a.G : -1;
        low[2 * nb + e] = lim[2 * nb + e] - a.window + 1;
      }
    }
    const int lim_min = p_base, low_max = at.s.len - a.window;  // of the first and the last token
    float o[NB][KS][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < KS; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
    float m[2 * NB], l[2 * NB];
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) m[i] = -INFINITY, l[i] = 0.f;

    int k_stage = 0, v_stage = 0;
    for (; at.t < t_end; ++at.t, ++w) {
      if (!wait(&s_full[stage], par)) break;
      k_stage = stage;
      const uint8_t *ks = sm + stage * kTile + at_k;
      next_stage();
      const int t0 = at.lo + at.t * pt + sub * 16;  // the warp's positions
      // two chains of products (even and odd k-steps): one is latency
      float s[NB][4] = {}, s1[NB][4] = {};
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        uint32_t a0, a1, a2, a3;
        ldmatrix_x4(a0, a1, a2, a3, ks + (k >> 2) * box + (((2 * (k & 3) + xk) ^ (rk & 7)) << 4));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) mma<BF16>(k & 1 ? s1[nb] : s[nb], a0, a1, a2, a3, qf[k][nb][0], qf[k][nb][1]);
      }
      // the last tile's stages are kept: the warps' states meet there
      const bool last = at.t + 1 == t_end;
      if (!last) release(k_stage);
      const bool partial = t0 + 15 > lim_min || t0 < low_max;
      float mx[2 * NB];
      bool more = false;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int i = 2 * nb + e;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const int t = t0 + g + 8 * y;
            float x = (s[nb][2 * y + e] + s1[nb][2 * y + e]) * a.sig_log2;
            if (partial && (t > lim[i] || t < low[i])) x = -INFINITY;
            s[nb][2 * y + e] = x;
          }
          mx[i] = fmaxf(s[nb][e], s[nb][2 + e]);
          more = more || mx[i] > m[i];
        }
      if (__any_sync(kAll, more)) {
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
#pragma unroll
          for (int y = 4; y < 32; y <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(kAll, mx[i], y));
          const float mn = fmaxf(m[i], mx[i]);
          const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - mn);
          if (m[i] != mn) {
            l[i] *= f;
#pragma unroll
            for (int k = 0; k < KS; ++k) o[i >> 1][k][i & 1] *= f, o[i >> 1][k][2 + (i & 1)] *= f;
          }
          m[i] = mn;
        }
      }
      // P^T as the B operand, hi and lo
      uint32_t ph[NB][2], pl[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float ref = m[2 * nb + (e & 1)];
          s[nb][e] -= ref == -INFINITY ? 0.f : ref;
          if constexpr (kShift != 0.f) s[nb][e] += kShift;  // (adding 0 would cost 1 %)
          s[nb][e] = fast_exp2(s[nb][e]);
          l[2 * nb + (e & 1)] += s[nb][e];
        }
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          uint32_t h, lo;
          split2<BF16>(s[nb][2 * y], s[nb][2 * y + 1], h, lo);
          ph[nb][y] = movmatrix_t(h);
          pl[nb][y] = movmatrix_t(lo);
        }
      }
      if (!wait(&s_full[stage], par)) break;
      v_stage = stage;
      const uint8_t *vs = sm + stage * kTile;
      next_stage();
      bool plain = false;
      if (partial) {
        bool ok = true;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 u = *reinterpret_cast<const uint4 *>(vs + at_k + (k >> 2) * box + (((2 * (k & 3) + xk) ^ (rk & 7)) << 4));
          ok = ok && pair_finite<BF16>(u.x) && pair_finite<BF16>(u.y) && pair_finite<BF16>(u.z) && pair_finite<BF16>(u.w);
        }
        plain = __any_sync(kAll, !ok);
      }
      if (!plain) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t a0, a1, a2, a3;
          ldmatrix_x4_t(a0, a1, a2, a3, vs + at_v + (k >> 2) * box + (((2 * (k & 3) + xv) ^ (rv & 7)) << 4));
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            mma<BF16>(o[nb][k], a0, a1, a2, a3, ph[nb][0], ph[nb][1]);
            mma<BF16>(o[nb][k], a0, a1, a2, a3, pl[nb][0], pl[nb][1]);
          }
        }
      } else {
#pragma unroll 1
        for (int y = 0; y < 16; ++y) {
          const int rr = sub * 16 + y, t = t0 + y;
          const uint8_t *row = vs + row_at(rr);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float p0 = __shfl_sync(kAll, s[nb][e], (y & 7) * 4 + c), p1 = __shfl_sync(kAll, s[nb][2 + e], (y & 7) * 4 + c);
              const float p = y & 8 ? p1 : p0;
              if (t <= lim[2 * nb + e] && t >= low[2 * nb + e]) {
#pragma unroll
                for (int k = 0; k < KS; ++k)
#pragma unroll
                  for (int z = 0; z < 2; ++z) {
                    const uint16_t u = *reinterpret_cast<const uint16_t *>(
                        row + (k >> 2) * box + (((2 * (k & 3) + z) ^ (rr & 7)) << 4) + 2 * g);
                    o[nb][k][2 * z + e] += p * unpack2<BF16>(u).x;
                  }
              }
            }
        }
      }
      if (!last) release(v_stage);
    }

    // The warps' states meet in the two stages just read (keys in an even one,
    // values in the next), channels of row r turned by 8 (r / 2) against bank
    // conflicts.
    float *mg = reinterpret_cast<float *>(sm + k_stage * kTile);  // [4][RU][D]
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
#pragma unroll
      for (int y = 4; y < 32; y <<= 1) l[i] += __shfl_xor_sync(kAll, l[i], y);
      if (g == 0) s_ml[warp][8 * (i >> 1) + 2 * c + (i & 1)] = make_float2(m[i], l[i]);
    }
    if (any_of_all(*abort_flag != 0)) break;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
      const int r = 8 * (i >> 1) + 2 * c + (i & 1);
      float M = m[i];
      for (int y = 0; y < per_head; ++y) M = fmaxf(M, s_ml[hh * per_head + y][r].x);
      // a warp that saw nothing has zeros, and 0 * f stays 0; NaN sums stay NaN
      const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - M);
      float *dst = mg + (warp * RU + r) * D;
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int z = 0; z < 2; ++z) dst[(16 * k + 8 * z + g + 8 * (r >> 1)) & (D - 1)] = o[i >> 1][k][2 * z + (i & 1)] * f;
    }
    const bool whole = t_begin == 0 && t_end == at.nt;
    float *part = a.part + ((int64_t)(2 * blockIdx.x + (t_begin == 0)) * kRowsMaxHeads + hh) * rows_part(D);
    // lane r: row r's sum and where it goes
    float inv = 0.f;
    uint32_t row_off = 0;
    if (lane < R) {
      float M = s_ml[hh * per_head][lane].x, L = 0.f;
      for (int i = 1; i < per_head; ++i) M = fmaxf(M, s_ml[hh * per_head + i][lane].x);
      for (int i = 0; i < per_head; ++i) {
        const float2 ml = s_ml[hh * per_head + i][lane];
        L += ml.y * (ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - M));
      }
      const int j = lane / a.G;
      row_off = (uint32_t)((at.s.q0 + j) * a.Hq + (at.h * HC + hh) * a.G + (lane - j * a.G));
      // a row before position 0 sees nothing and gives zeros
      inv = p_base + j >= 0 ? 1.f / L : -1.f;
      if (!whole && sub == 0) {
        __stcg(part + kRowsPerUnit * D + lane, M);
        __stcg(part + kRowsPerUnit * (D + 1) + lane, L);
      }
    }
    bar_sync();
    // the warps of a head share its rows, 4 channels a lane
    constexpr int V = D / 4, RW = 32 / V;  // rows of a warp at a time
    const int v = lane % V;
#pragma unroll 4
    for (int i = 0; i < RU; i += RW * per_head) {
      const int r = i + sub * RW + lane / V;
      const float f = __shfl_sync(kAll, inv, r & 31);
      const uint32_t off = __shfl_sync(kAll, row_off, r & 31);
      if (r < R) {
        const float *src = mg + ((hh * per_head) * RU + r) * D + ((4 * v + 8 * (r >> 1)) & (D - 1));
        float4 x = *reinterpret_cast<const float4 *>(src);
        for (int y = 1; y < per_head; ++y) {
          const float4 z = *reinterpret_cast<const float4 *>(src + y * RU * D);
          x.x += z.x, x.y += z.y, x.z += z.z, x.w += z.w;
        }
        if (!whole) {
          __stcg(reinterpret_cast<float4 *>(part + r * D + 4 * v), x);
        } else {
          if (f < 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
          *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.out) + ((uint64_t)off * D + 4 * v) * 2) =
              make_uint2(pack2<BF16>(x.x * f, x.y * f), pack2<BF16>(x.z * f, x.w * f));
        }
      }
    }
    if (!whole && t_begin == 0 && tid == 0) {
      const int at_list = atomicAdd(&a.list->n, 1);  // a CTA adds one at most
      const int last = min((int)blockIdx.x + (w_begin + at.nt - 1) / s_share, (int)gridDim.x - 1);
      if ((unsigned)at_list < (unsigned)kRowsMaxCtas) a.list->unit[at_list] = RowsSplit{(int)blockIdx.x, last, at.s.q0, p_base, at.h * HC, R};
    }
    if (w < mine) {
      fence_proxy_async();
      bar_sync();
      release(k_stage);
      release(v_stage);
      if (at.t >= at.nt) next_unit(at);
    }
  }
  if (*abort_flag && lane == 0) set_err(pv.err, kErrTimeout);
  pdl_trigger();
}

template <int D, int NB, bool BF16>
cudaError_t launch_t(const AttnArgs &a, cudaStream_t st) {
  constexpr int smem = rows_stages<D>() * kT * D * 2 + 1024;
  RowsArgs ra;
  memcpy(&ra.mk, a.whole ? a.ok : a.wk, sizeof ra.mk);
  memcpy(&ra.mv, a.whole ? a.ov : a.wv, sizeof ra.mv);
  ra.a = a;
  ra.a.rows = std::min(8 * NB, a.max_new * a.G);
  cudaError_t e = allow_smem<&attn_rows_kernel<D, NB, BF16>>(smem, a.device);
  if (e != cudaSuccess) return e;
  // two CTAs per SM, no more of them than runs that there can be
  const int64_t cap = ((int64_t)a.pv.max_pages << a.pv.page_shift) / (kT / a.hc) + 2;
  const int64_t tiles = (int64_t)a.pv.B * (a.pv.Hkv / a.hc) * cap;
  const int64_t runs = a.whole ? tiles / cap : (tiles + kMinShare - 1) / kMinShare;
  const int grid = (int)std::min<int64_t>(std::min(2 * a.sms, kRowsMaxCtas), runs);
  e = launch_pdl(attn_rows_kernel<D, NB, BF16>, dim3(grid), dim3(kThreads + 32), smem, st, ra);
  if (e != cudaSuccess || a.whole) return e;
  // a unit cut in pieces starts in a CTA of its own; eight of the joining CTAs
  // fit an SM
  return launch_pdl(attn_join_kernel<D, BF16>, dim3(std::min(grid * a.hc * ra.a.rows, 8 * a.sms)), dim3(kThreads), 0, st, ra.a);
}
template <int D, bool BF16>
cudaError_t launch_rows(const AttnArgs &a, cudaStream_t st) {
  return a.max_new * a.G <= 8 ? launch_t<D, 1, BF16>(a, st) : launch_t<D, 2, BF16>(a, st);
}

}  // namespace

cudaError_t launch_attn_rows(const AttnArgs &in, int dtype, cudaStream_t st) {
  if (in.pv.B == 0 || in.pv.n_tokens == 0) return cudaSuccess;
  AttnArgs a = in;
  a.whole = ((int64_t)a.pv.max_pages << a.pv.page_shift) <= kWholeCtx;
  a.hc = a.whole ? 1 : rows_heads(1 << a.pv.page_shift, a.pv.Hkv);
  a.part_shift = std::min(a.pv.page_shift, 6);
  a.pt_shift = a.hc == 4 ? 4 : a.hc == 2 ? 5 : 6;
  const bool bf = dtype == kSrvBf16;
  switch (a.pv.D) {
    case 128: return bf ? launch_rows<128, true>(a, st) : launch_rows<128, false>(a, st);
    case 64: return bf ? launch_rows<64, true>(a, st) : launch_rows<64, false>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
