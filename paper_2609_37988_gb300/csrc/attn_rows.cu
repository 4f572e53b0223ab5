// attn_rows.cu -- attention of a few new tokens per sequence over a paged
// cache (single tokens, drafted ones): bound by the cache's bytes.
//
// Query j of sequence b sits at position p = len_b - n_b + j and sees
// positions max(0, p - window + 1) .. p; head h reads KV head h / G.  Rows
// r = j G + (head in its group) of a (sequence, KV head) go in units of 16, so
// that a key or value byte is read once for all of them.  A unit's positions
// go in tiles of 64; the tiles of all units, one behind another, are cut into
// equal runs, one per CTA (two CTAs per SM are resident), whatever the
// sequences' lengths are.  A unit that a run covers whole is written at once;
// the pieces of the others go to the workspace, and the CTA that adds the last
// one joins them (fixed order, so results do not depend on who is last).
//
// A CTA: 4 warps, 16 positions of a tile each, and a warp that looks up pages
// and copies key and value tiles by TMA through a ring (96 KB; each half of a
// tile is refilled as soon as the four warps have read it).  S = Q K^T and
// O += P V on mma.m16n8k16 with fp32 accumulation, the softmax online in base
// 2, each warp with its own maxima and sums; P enters as hi + lo halves, whose
// products are free beside the copies.
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

constexpr int kT = 64;        // positions per tile
constexpr int kThreads = 128;  // that compute; a warp beside them copies
constexpr int kErrCount = 4, kErrTimeout = 8, kErrPage = 32;  // KVK_DEVERR_*
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
  const int c0 = min(max(v.cu[b], 0), v.n_tokens);
  s.n = min(max(v.cu[b + 1], c0), v.n_tokens) - c0;
  s.q0 = c0;
  s.len = max(v.lens[b], 0);
  const int64_t cap = (int64_t)v.max_pages << v.page_shift;
  if (s.n > max_new || s.len > cap) {
    set_err(v.err, kErrCount);
    s.n = min(s.n, max_new);
    s.len = (int)min((int64_t)s.len, cap);
  }
  return s;
}
// Positions [lo, hi) that the rows of unit block rb see (lo a multiple of the
// tile; at least one tile, so that rows that see nothing get their zeros).
__device__ __forceinline__ void block_range(const Seq &s, int G, int window, int rb, int &lo, int &nt) {
  const int first = s.len - s.n + rb * kRowsPerUnit / G;
  const int last = s.len - s.n + min(s.n * G - 1, rb * kRowsPerUnit + kRowsPerUnit - 1) / G;
  lo = max(0, first - window + 1) / kT * kT;
  nt = max(1, (last + kT - lo) / kT);
}
__device__ __forceinline__ int row_blocks(const Seq &s, int G) { return (s.n * G + kRowsPerUnit - 1) / kRowsPerUnit; }
__device__ __forceinline__ int seq_tiles(const Seq &s, int G, int window) {
  int sum = 0;
  for (int rb = 0; rb < row_blocks(s, G); ++rb) {
    int lo, nt;
    block_range(s, G, window, rb, lo, nt);
    sum += nt;
  }
  return sum;
}

// A place in the list of tiles.
struct At {
  int b, h, rb, t;   // sequence, KV head, row block, tile of the unit
  int lo, nt;        // the unit's first position and tiles
  Seq s;
};

struct RowsArgs {
  CUtensorMap mk, mv;
  AttnArgs a;
};

template <int D>
constexpr int rows_stages() { return D == 128 ? 6 : 12; }  // key and value tiles in turn

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads + 32, 2) attn_rows_kernel(const __grid_constant__ RowsArgs ra) {
  constexpr int RB = D * 2;            // bytes of a row
  constexpr int kTile = kT * RB;       // bytes of a key (or value) tile: boxes of 64 channels
  constexpr int KS = D / 16, NS = rows_stages<D>();
  const AttnArgs &a = ra.a;
  extern __shared__ uint8_t sm_raw[];
  uint8_t *sm = sm_raw + ((1024u - (smem_u32(sm_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_full[NS], s_free[NS];
  __shared__ int s_abort;
  __shared__ int64_t s_total, s_start;
  __shared__ int s_b, s_last;
  __shared__ float2 s_ml[4][kRowsPerUnit];
  const PagedView &pv = a.pv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, c = lane & 3;
  if (tid == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], kThreads / 32);
    }
    s_abort = 0;
    fence_mbar_init();
  }
  pdl_wait();

  // the run of this CTA: tiles [w0, w1) of all
  if (warp == 0) {
    int64_t total = 0;
    for (int b = lane; b < pv.B; b += 32) total += (int64_t)pv.Hkv * seq_tiles(load_seq(pv, b, a.max_new), a.G, a.window);
    for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
    const int64_t share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)1);
    const int64_t w0 = share * blockIdx.x;
    int64_t before = 0;
    int found = -1;
    if (w0 < total) {
      for (int b0 = 0; b0 < pv.B && found < 0; b0 += 32) {
        int64_t x = 0;
        if (b0 + lane < pv.B) x = (int64_t)pv.Hkv * seq_tiles(load_seq(pv, b0 + lane, a.max_new), a.G, a.window);
        int64_t sum = x;
        for (int o = 1; o < 32; o <<= 1) {
          const int64_t y = __shfl_up_sync(kAll, sum, o);
          if (lane >= o) sum += y;
        }
        const uint32_t past = __ballot_sync(kAll, before + sum > w0);
        if (past) {
          const int f = __ffs(past) - 1;
          found = b0 + f;
          before += __shfl_sync(kAll, sum - x, f);
        } else {
          before += __shfl_sync(kAll, sum, 31);
        }
      }
    }
    if (lane == 0) {
      s_total = total;
      s_b = found;
      s_start = before;
    }
  }
  __syncthreads();
  const int64_t total = s_total;
  const int64_t share = max((total + gridDim.x - 1) / gridDim.x, (int64_t)1);
  const int64_t w0 = share * blockIdx.x, w1 = min(total, w0 + share);
  if (w0 >= w1) {
    pdl_trigger();
    return;
  }

  auto settle = [&](At &x) { block_range(x.s, a.G, a.window, x.rb, x.lo, x.nt); };
  auto next_unit = [&](At &x) {
    x.t = 0;
    if (++x.rb >= row_blocks(x.s, a.G)) {
      x.rb = 0;
      if (++x.h >= pv.Hkv) {
        x.h = 0;
        do {
          if (++x.b >= pv.B) return;  // behind the last unit: not used again
          x.s = load_seq(pv, x.b, a.max_new);
        } while (x.s.n == 0);
      }
    }
    settle(x);
  };
  At at;
  {
    at.b = s_b;
    at.s = load_seq(pv, at.b, a.max_new);
    int64_t off = w0 - s_start;
    const int per = seq_tiles(at.s, a.G, a.window);
    at.h = (int)(off / per);
    int r = (int)(off - (int64_t)at.h * per);
    at.rb = 0;
    settle(at);
    while (r >= at.nt) {
      r -= at.nt;
      ++at.rb;
      settle(at);
    }
    at.t = r;
  }

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
  // boxes of 64 channels, 128-byte-swizzled rows
  const int shift = min(pv.page_shift, 6), parts = kT >> shift, box = 128 << shift;
  auto row_at = [&](int r) { return ((r >> shift) << shift) * RB + (r & ((1 << shift) - 1)) * 128; };

  if (warp == kThreads / 32) {
    // -- copies: a lane per part of a tile (the positions of one page), its
    // page looked up a tile ahead; outside the pool reads as zeros
    auto look_up = [&](const At &x) {
      const int t = x.lo + x.t * kT + (lane << shift);
      return lane < parts && t < x.s.len ? pv.table[(int64_t)x.b * pv.max_pages + (t >> pv.page_shift)] : pv.n_pages;
    };
    int page = look_up(at);
    bool ok = true;
    for (int64_t w = w0; w < w1 && ok; ++w) {
      const int t = at.lo + at.t * kT + (lane << shift);
      const int y = t & ((1 << pv.page_shift) - 1), h = at.h;
      int now = page;
      if ((unsigned)now >= (unsigned)pv.n_pages) {
        if (lane < parts && t < at.s.len) set_err(pv.err, kErrPage);
        now = pv.n_pages;
      }
      if (w + 1 < w1) {
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
          tma_load_5d(sm + stage * kTile + (lane << shift) * RB, kv ? &ra.mv : &ra.mk, 0, y, 0, h, now, &s_full[stage]);
        next_stage();
      }
    }
    if (*abort_flag && lane == 0) {  // the copies in flight land before the CTA ends
      for (int i = 0; i < NS; ++i) {
        if (par == 0 && i >= stage) break;
        mbar_wait(&s_full[i], i < stage ? par : par ^ 1, kWaits);
      }
    }
    if (*abort_flag && lane == 0) set_err(pv.err, kErrTimeout);
    pdl_trigger();
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
  for (int64_t w = w0; w < w1;) {
    // a piece: tiles [t_begin, t_end) of one unit
    const int t_begin = at.t, t_end = (int)min((int64_t)at.nt, at.t + (w1 - w));
    const int R = min(kRowsPerUnit, at.s.n * a.G - at.rb * kRowsPerUnit);
    const int p_base = at.s.len - at.s.n;
    uint32_t qf[KS][4];
    int lim[2], low[2];
    bool real[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = at.rb * kRowsPerUnit + g + 8 * i, j = r / a.G;
      real[i] = g + 8 * i < R;
      lim[i] = real[i] ? p_base + j : -1;
      low[i] = lim[i] - a.window + 1;
      const uint8_t *src = a.q.p + 2 * ((int64_t)(at.s.q0 + (real[i] ? j : 0)) * a.q.ts +
                                        (int64_t)(at.h * a.G + (real[i] ? r - j * a.G : 0)) * a.q.hs);
#pragma unroll
      for (int k = 0; k < KS; ++k)
#pragma unroll
        for (int x = 0; x < 2; ++x)
          qf[k][2 * x + i] = real[i] ? *reinterpret_cast<const uint32_t *>(src + 32 * k + 16 * x + 4 * c) : 0u;
    }
    const int lim_min = p_base + at.rb * kRowsPerUnit / a.G;                     // of the first row
    const int low_max = p_base + (at.rb * kRowsPerUnit + R - 1) / a.G - a.window + 1;  // of the last
    float o[D / 8][4];
#pragma unroll
    for (int i = 0; i < D / 8; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};

    int k_stage = 0, v_stage = 0;
    for (; at.t < t_end; ++at.t, ++w) {
      if (!wait(&s_full[stage], par)) break;
      k_stage = stage;
      const uint8_t *ks = sm + stage * kTile;
      next_stage();
      const int t0 = at.lo + at.t * kT + warp * 16;  // the warp's positions
      float s[2][4] = {};
      {
        const int r = warp * 16 + (lane & 7) + ((lane & 16) >> 1), x = (lane >> 3) & 1, at_r = row_at(r);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t b0, b1, b2, b3;
          ldmatrix_x4(b0, b1, b2, b3, ks + at_r + (k >> 2) * box + (((2 * (k & 3) + x) ^ (r & 7)) << 4));
          mma<BF16>(s[0], qf[k][0], qf[k][1], qf[k][2], qf[k][3], b0, b1);
          mma<BF16>(s[1], qf[k][0], qf[k][1], qf[k][2], qf[k][3], b2, b3);
        }
      }
      // the last tile's stages are kept: the warps' states meet there
      const bool last = at.t + 1 == t_end;
      if (!last) release(k_stage);
      const bool partial = t0 + 15 > lim_min || t0 < low_max;
      float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = e >> 1, t = t0 + 8 * nb + 2 * c + (e & 1);
          float x = s[nb][e] * a.sig_log2;
          if (partial && (t > lim[i] || t < low[i])) x = -INFINITY;
          s[nb][e] = x;
          mx[i] = fmaxf(mx[i], x);
        }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(kAll, mx[i], 1));
        mx[i] = fmaxf(mx[i], __shfl_xor_sync(kAll, mx[i], 2));
      }
      if (__any_sync(kAll, mx[0] > m[0] || mx[1] > m[1])) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const float mn = fmaxf(m[i], mx[i]);
          const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - mn);
          if (m[i] != mn) {
            l[i] *= f;
#pragma unroll
            for (int k = 0; k < D / 8; ++k) o[k][2 * i] *= f, o[k][2 * i + 1] *= f;
          }
          m[i] = mn;
        }
      }
      const float ref[2] = {m[0] == -INFINITY ? 0.f : m[0], m[1] == -INFINITY ? 0.f : m[1]};
#pragma unroll
      for (int nb = 0; nb < 2; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[nb][e] = fast_exp2(s[nb][e] - ref[e >> 1]);
          l[e >> 1] += s[nb][e];
        }
      // P as the A operand: rows g, g + 8; positions 2c.. of either half
      uint32_t ph[4], pl[4];
      split2<BF16>(s[0][0], s[0][1], ph[0], pl[0]);
      split2<BF16>(s[0][2], s[0][3], ph[1], pl[1]);
      split2<BF16>(s[1][0], s[1][1], ph[2], pl[2]);
      split2<BF16>(s[1][2], s[1][3], ph[3], pl[3]);
      if (!wait(&s_full[stage], par)) break;
      v_stage = stage;
      const uint8_t *vs = sm + stage * kTile;
      next_stage();
      const int r = warp * 16 + (lane & 15), x = lane >> 4, at_r = row_at(r);
      bool plain = false;
      if (partial) {
        bool ok = true;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint4 u = *reinterpret_cast<const uint4 *>(vs + at_r + (k >> 2) * box + (((2 * (k & 3) + x) ^ (r & 7)) << 4));
          ok = ok && pair_finite<BF16>(u.x) && pair_finite<BF16>(u.y) && pair_finite<BF16>(u.z) && pair_finite<BF16>(u.w);
        }
        plain = __any_sync(kAll, !ok);
      }
      if (!plain) {
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          uint32_t b0, b1, b2, b3;
          ldmatrix_x4_t(b0, b1, b2, b3, vs + at_r + (k >> 2) * box + (((2 * (k & 3) + x) ^ (r & 7)) << 4));
          mma<BF16>(o[2 * k], ph[0], ph[1], ph[2], ph[3], b0, b1);
          mma<BF16>(o[2 * k + 1], ph[0], ph[1], ph[2], ph[3], b2, b3);
          mma<BF16>(o[2 * k], pl[0], pl[1], pl[2], pl[3], b0, b1);
          mma<BF16>(o[2 * k + 1], pl[0], pl[1], pl[2], pl[3], b2, b3);
        }
      } else {
        for (int y = 0; y < 16; ++y) {
          const int from = (lane & ~3) | ((y & 7) >> 1), t = t0 + y;
          float p[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float e0 = __shfl_sync(kAll, s[0][2 * i], from), e1 = __shfl_sync(kAll, s[0][2 * i + 1], from);
            const float f0 = __shfl_sync(kAll, s[1][2 * i], from), f1 = __shfl_sync(kAll, s[1][2 * i + 1], from);
            p[i] = y & 8 ? (y & 1 ? f1 : f0) : (y & 1 ? e1 : e0);
          }
          const int rr = warp * 16 + y, at_rr = row_at(rr);
#pragma unroll
          for (int k = 0; k < D / 8; ++k) {
            const uint32_t u = *reinterpret_cast<const uint32_t *>(vs + at_rr + (k >> 3) * box + (((k & 7) ^ (rr & 7)) << 4) + 4 * c);
            const float2 f = unpack2<BF16>(u);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              if (t <= lim[i] && t >= low[i]) {
                o[k][2 * i] += p[i] * f.x;
                o[k][2 * i + 1] += p[i] * f.y;
              }
          }
        }
      }
      if (!last) release(v_stage);
    }

    // the four warps' states are joined in the two stages just read (keys in an
    // even one, values in the next)
    float *mg = reinterpret_cast<float *>(sm + k_stage * kTile);  // [4][16][D]
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      l[i] += __shfl_xor_sync(kAll, l[i], 1);
      l[i] += __shfl_xor_sync(kAll, l[i], 2);
      if (c == 0) s_ml[warp][g + 8 * i] = make_float2(m[i], l[i]);
    }
    if (any_of_all(*abort_flag != 0)) break;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int r = g + 8 * i;
      const float M = fmaxf(fmaxf(s_ml[0][r].x, s_ml[1][r].x), fmaxf(s_ml[2][r].x, s_ml[3][r].x));
      const float f = m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - M);
      // a warp that saw nothing has zeros, and 0 * f stays 0; NaN sums stay NaN
#pragma unroll
      for (int k = 0; k < D / 8; ++k)
        *reinterpret_cast<float2 *>(mg + ((warp * 16 + r) * D + 8 * k + 2 * c)) = make_float2(o[k][2 * i] * f, o[k][2 * i + 1] * f);
    }
    bar_sync();
    const bool whole = t_begin == 0 && t_end == at.nt;
    // where the unit's tiles lie: the CTA that starts it and the last one
    const int64_t u0 = w - t_end;
    const int c0 = (int)(u0 / share), c1 = (int)((u0 + at.nt - 1) / share);
    float *part = a.part + (int64_t)(2 * blockIdx.x + (blockIdx.x == c0)) * rows_part(D);
    auto store = [&](int r, int v, float4 x, float L) {
      const int rr = at.rb * kRowsPerUnit + r, j = rr / a.G;
      // a row before position 0 sees nothing and gives zeros
      const bool sees = p_base + j >= 0;
      const float inv = sees ? 1.f / L : 0.f;
      if (!sees) x = make_float4(0.f, 0.f, 0.f, 0.f);
      uint8_t *dst = static_cast<uint8_t *>(a.out) +
                     2 * (((int64_t)(at.s.q0 + j) * a.Hq + at.h * a.G + (rr - j * a.G)) * D + 4 * v);
      *reinterpret_cast<uint2 *>(dst) = make_uint2(pack2<BF16>(x.x * inv, x.y * inv), pack2<BF16>(x.z * inv, x.w * inv));
    };
    for (int e = tid; e < R * (D / 4); e += kThreads) {
      const int r = e / (D / 4), v = e % (D / 4);
      const float M = fmaxf(fmaxf(s_ml[0][r].x, s_ml[1][r].x), fmaxf(s_ml[2][r].x, s_ml[3][r].x));
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      float L = 0.f;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float4 y = *reinterpret_cast<const float4 *>(mg + (i * 16 + r) * D + 4 * v);
        x.x += y.x, x.y += y.y, x.z += y.z, x.w += y.w;
        const float2 ml = s_ml[i][r];
        L += ml.y * (ml.x == -INFINITY ? 0.f : fast_exp2(ml.x - M));
      }
      if (whole) {
        store(r, v, x, L);
      } else {
        __stcg(reinterpret_cast<float4 *>(part + r * D + 4 * v), x);
        if (v == 0) {
          __stcg(part + kRowsPerUnit * D + r, M);
          __stcg(part + kRowsPerUnit * (D + 1) + r, L);
        }
      }
    }
    if (!whole) {
      __threadfence();
      bar_sync();
      if (tid == 0) {
        const bool last = atomicAdd(a.counter + c0, 1) == c1 - c0;
        if (last) a.counter[c0] = 0;  // as the next call expects it
        s_last = last;
      }
      bar_sync();
      if (s_last) {
        __threadfence();
        // thread (group, row, 4 channels): the pieces group, group + n, ...;
        // the groups meet in shared memory
        const int vecs = R * (D / 4), groups = max(1, kThreads / vecs);
        for (int e0 = 0; e0 < vecs; e0 += kThreads) {
          const int e = e0 + tid % min(vecs, kThreads), grp = vecs < kThreads ? tid / vecs : 0;
          const int r = e / (D / 4), v = e % (D / 4);
          const bool on = e < vecs && grp < groups;
          float M = -INFINITY, L = 0.f;
          float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
          if (on) {
            constexpr int U = 8;
            for (int p0 = c0 + grp; p0 <= c1; p0 += U * groups) {
              float4 y[U];
              float pm[U], pl[U];
#pragma unroll
              for (int u = 0; u < U; ++u) {
                const int p = p0 + u * groups;
                const float *src = a.part + (int64_t)(2 * p + (p == c0)) * rows_part(D);
                const bool in = p <= c1;
                y[u] = in ? __ldcg(reinterpret_cast<const float4 *>(src + r * D + 4 * v)) : make_float4(0.f, 0.f, 0.f, 0.f);
                pm[u] = in ? __ldcg(src + kRowsPerUnit * D + r) : -INFINITY;
                pl[u] = in ? __ldcg(src + kRowsPerUnit * (D + 1) + r) : 0.f;
              }
#pragma unroll
              for (int u = 0; u < U; ++u) join(M, L, x, pm[u], pl[u], y[u]);
            }
          }
          if (groups > 1) {
            float4 *sx = reinterpret_cast<float4 *>(mg);
            float2 *sl = reinterpret_cast<float2 *>(sx + kThreads);
            bar_sync();  // mg has been read
            sx[tid] = x;
            sl[tid] = make_float2(M, L);
            bar_sync();
            if (tid < vecs)
              for (int i = 1; i < groups; ++i) join(M, L, x, sl[tid + i * vecs].x, sl[tid + i * vecs].y, sx[tid + i * vecs]);
          }
          if (on && grp == 0) store(r, v, x, L);
        }
      }
    }
    fence_proxy_async();
    bar_sync();
    release(k_stage);
    release(v_stage);
    if (w < w1 && at.t >= at.nt) next_unit(at);
  }
  if (*abort_flag && lane == 0) set_err(pv.err, kErrTimeout);
  pdl_trigger();
}

template <int D, bool BF16>
cudaError_t launch_t(const AttnArgs &a, cudaStream_t st) {
  constexpr int smem = rows_stages<D>() * kT * D * 2 + 1024;
  RowsArgs ra;
  memcpy(&ra.mk, a.wk, sizeof ra.mk);
  memcpy(&ra.mv, a.wv, sizeof ra.mv);
  ra.a = a;
  static std::atomic<bool> ready{false};
  if (!ready.load(std::memory_order_relaxed)) {
    const cudaError_t e =
        cudaFuncSetAttribute(attn_rows_kernel<D, BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    ready.store(true, std::memory_order_relaxed);
  }
  // two CTAs per SM, no more of them than tiles that there can be
  const int64_t cap = ((int64_t)a.pv.max_pages << a.pv.page_shift) / kT + 2;
  const int64_t tiles = (int64_t)a.pv.B * a.pv.Hkv * ((a.max_new * a.G + kRowsPerUnit - 1) / kRowsPerUnit) * cap;
  const int grid = (int)std::min<int64_t>(std::min(2 * a.sms, kRowsMaxCtas), tiles);
  return launch_pdl(attn_rows_kernel<D, BF16>, dim3(grid), dim3(kThreads + 32), smem, st, ra);
}

}  // namespace

cudaError_t launch_attn_rows(const AttnArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.B == 0 || a.pv.n_tokens == 0) return cudaSuccess;
  const bool bf = dtype == kSrvBf16;
  switch (a.pv.D) {
    case 128: return bf ? launch_t<128, true>(a, st) : launch_t<128, false>(a, st);
    case 64: return bf ? launch_t<64, true>(a, st) : launch_t<64, false>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
