// attn_codes_rows.cu -- attention of a few new tokens per sequence over a paged
// cache in 8 bits: bound by the cache's bytes.
//
// Units, runs and the joining of cut units are those of the 16-bit form
// (rows_common.cuh).  A tile is 128 positions x KV heads of codes, 16 KB; a unit has
// up to 4 KV heads, so that a copy is 8 or 16 KB where pages are small.  A CTA: 4
// warps, 32 positions of one head's tile each, in two blocks of 16 that lie in one
// page and so have one power of two, and a warp that looks up pages and powers and
// copies the tiles by TMA through a ring of 64 KB (96 KB leave the L1 too little for
// what 16 rows spill: three tokens of 32 sequences 122 us, 114 with 64).  (8 warps of one block each took
// 426 instructions a block, a third of them around the products: 100 us where
// two blocks take 93.)
//
// Codes are exact in f16 and go to the tensor cores as they are: S^T = K Q^T and
// O^T += V^T P^T on mma.m16n8k16.  The keys' power multiplies the scores.  The
// values' power enters the weights: a warp's sums O are kept relative to 2^E, E the
// largest power so far among the pages that the unit's rows see, the weights p 2^(e - E)
// are rounded to f16 (half a step: 2^-11 of a weight; kept 2^14 times as large, what the
// type's subnormals cut off is 2^-39 of the row's largest, times 2^(E - e)).  Queries are f16 too: bf16 ones, a row times the power
// of two that brings its largest to [2^13, 2^14), which is exact but for numbers
// below 2^-28 of that.
//
// Fragments: a product's 16 channels (of keys) or rows (of values) may stand in any
// order, so lanes take neighbouring bytes.  Keys: ldmatrix gives lane (g, c) the codes
// of channels 4c .. 4c + 3 of position g, two pairs for the products' slots 2c, 2c + 1
// and 2c + 8, 2c + 9.  Values: transposed, channels 2g and 2g + 1 of positions 2c and
// 2c + 1, one byte permutation away from a pair of positions per channel.
//
// Measured (40 / 8 heads of 128, bf16, pages of 16): single tokens of 32 sequences over
// 8192 positions 91 us, 0.86 of the bandwidth (in 16 bits 166), three tokens each 112 us.
#include <cuda.h>
#include <math.h>
#include <string.h>

#include <algorithm>

#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"
#include "rows_common.cuh"
#include "serve.h"
#include "umma.cuh"

namespace kvk {
namespace {

constexpr int kT = 128;         // positions x KV heads of a tile
constexpr int kWarps = 4;       // that compute; one beside them copies
constexpr int kThreads = 32 * kWarps;
constexpr int kBlocks = 2;      // of 16 positions, a warp's of a tile
constexpr int kMinShare = 2;    // tiles of a run at least
constexpr float kShift = 14.f;  // weights are 2^14 as large

struct RowsArgs {
  CUtensorMap mk, mv;
  AttnArgs a;
};

// an even number: keys and values in turn
template <int D>
constexpr int rows_stages() { return 512 / D; }

__device__ __forceinline__ void ldm(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at));
}
__device__ __forceinline__ void ldm_t(uint32_t (&r)[4], uint32_t at) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(at));
}

// NB: query rows of a unit in blocks of 8
template <int D, int NB, bool BF16>
__global__ void __launch_bounds__(kThreads + 32, 2) attn_codes_rows_kernel(const __grid_constant__ RowsArgs ra) {
  constexpr int kTile = kT * D;        // bytes of a key (or value) tile
  constexpr int KS = D / 16, NS = rows_stages<D>(), RU = 8 * NB;
  const AttnArgs &a = ra.a;
  extern __shared__ uint8_t sm_raw[];
  uint8_t *sm = sm_raw + ((1024u - (smem_u32(sm_raw) & 1023u)) & 1023u);
  __shared__ uint64_t s_full[NS], s_free[NS];
  __shared__ int s_abort, s_mine, s_share;
  __shared__ At s_at;
  __shared__ float2 s_ml[kWarps][RU];
  __shared__ int s_e[kWarps];
  // powers of a tile's parts and heads, keys' and values'
  __shared__ alignas(16) int8_t s_pow[NS / 2][2][8][kRowsMaxHeads];
  const PagedView &pv = a.pv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int g = lane >> 2, c = lane & 3;
  const int HC = a.hc, units = pv.Hkv / HC;
  const int per_head = kWarps / HC, hh = warp / per_head, sub = warp % per_head;  // the warp's head and positions
  if (tid == kThreads) {
    prefetch_tensor_map(&ra.mk);
    prefetch_tensor_map(&ra.mv);
  }
  if (tid == 64) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&s_full[i], 1);
      mbar_init(&s_free[i], kWarps);
    }
    s_abort = 0;
    fence_mbar_init();
  }
  pdl_wait();
  if (warp == 0) find_run(a, units, kMinShare, lane, s_at, s_mine, s_share);
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

  // a tile in shared memory: per part (the positions of one page) and KV head its
  // rows of D bytes, 16-byte pieces swizzled
  const int pt = 1 << a.pt_shift, shift = a.part_shift, parts = pt >> shift;
  auto row_at = [&](int r) { return (((r >> shift) * HC + hh) << shift) * D + (r & ((1 << shift) - 1)) * D; };
  auto swz = [&](int r) { return D == 128 ? r & 7 : r >> 1 & 3; };

  if (warp == kWarps) {
    // -- copies: a lane per part of a tile, its page looked up two tiles ahead and its
    // powers one; what is read is not touched before the next turn, as a look at it
    // would wait for it.  Outside the pool reads as zeros.  Parts that no query sees
    // (a window may begin inside a tile) have no page: their entries may be stale.
    struct Next {
      int page, y, h;  // as found: -1 where no query sees it
      bool seen;
    };
    auto look_up = [&](const At &x) {
      const int t = x.lo + x.t * pt + (lane << shift);
      Next n = {-1, t & ((1 << pv.page_shift) - 1), x.h * HC, lane < parts && t < x.s.len && t + (1 << shift) > x.s.len - x.s.n - a.window + 1};
      n.page = load_if(pv.table + (int64_t)x.b * pv.max_pages + (t >> pv.page_shift), n.seen, -1);
      return n;
    };
    auto checked = [&](Next n) {
      if ((unsigned)n.page >= (unsigned)pv.n_pages) {
        if (n.seen) set_err(pv.err, kErrPage);
        n.page = pv.n_pages;
      }
      return n;
    };
    // (no page: the least power, so that its zeros do not move the sums' 2^E)
    auto powers = [&](const Next &n, const int8_t *e) {
      const int8_t *p = e + (int64_t)n.page * pv.Hkv + n.h;
      const bool in = n.page < pv.n_pages;
      if (HC == 4) return (uint32_t)load_if(reinterpret_cast<const int32_t *>(p), in, (int)0x80808080u);
      if (HC == 2) return (uint32_t)load_if(reinterpret_cast<const uint16_t *>(p), in, 0x8080);
      return (uint32_t)load_if(reinterpret_cast<const uint8_t *>(p), in, 0x80);
    };
    auto step = [&]() {
      if (++at.t >= at.nt) next_unit(a, units, at);
      return look_up(at);
    };
    Next now = look_up(at), found = now;
    if (mine > 1) found = step();
    now = checked(now);
    uint32_t ek = powers(now, pv.ke), ev = powers(now, pv.ve);
    // (asked once: a limit from the arguments in the loop's waits cost 1.3 % in the 16-bit form)
    bool ok = !a.give_up;
    if (!ok && lane == 0) *abort_flag = 1;
    for (int w = 0; w < mine && ok; ++w) {
      uint32_t ek_next = 0, ev_next = 0;
      Next next = now;
      if (w + 1 < mine) {
        next = checked(found);
        ek_next = powers(next, pv.ke), ev_next = powers(next, pv.ve);
        if (w + 2 < mine) found = step();
      }
#pragma unroll
      for (int kv = 0; kv < 2; ++kv) {
        int got = 1;
        if (lane == 0) got = wait(&s_free[stage], par ^ 1);
        ok = __shfl_sync(kAll, got, 0) != 0;
        if (!ok) break;
        if (kv == 0) {  // the warps have read both of the place's last powers with its keys
          if (lane < parts) {
            *reinterpret_cast<uint32_t *>(s_pow[stage >> 1][0][lane]) = ek;
            *reinterpret_cast<uint32_t *>(s_pow[stage >> 1][1][lane]) = ev;
          }
          __syncwarp();
        }
        if (lane == 0) mbar_expect_tx(&s_full[stage], kTile);
        __syncwarp();
        if (lane < parts)
          tma_load_4d(sm + stage * kTile + ((lane * HC) << shift) * D, kv ? &ra.mv : &ra.mk, 0, now.y, now.h, now.page, &s_full[stage]);
        next_stage();
      }
      now = next, ek = ek_next, ev = ev_next;
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
  // this lane's row of either block, as ldmatrix wants its address: of its first 16
  // codes, the swizzle in place (what a row starts on leaves those bits alone)
  constexpr int PB = kBlocks;
  const int r_lane = sub * 16 * PB + (lane & 15);
  uint32_t at_row[PB];
  int my_part[PB];
#pragma unroll
  for (int b = 0; b < PB; ++b) {
    at_row[b] = smem_u32(sm) + row_at(r_lane + 16 * b) + (((lane >> 4) ^ swz(r_lane)) << 4);
    my_part[b] = (sub * PB + b) * 16 >> shift;
  }
  for (int w = 0; w < mine;) {
    // a piece: tiles [t_begin, t_end) of one unit
    const int t_begin = at.t, t_end = min(at.nt, at.t + (mine - w)), w_begin = w;
    const int R = at.s.n * a.G;
    const int p_base = at.s.len - at.s.n;
    // Q^T as the B operand (row 8 nb + g); of rows 8 nb + 2 c + e their tokens, a byte
    // each (255: none), and the scores' factor
    uint32_t qf[KS][NB][2], tok = 0;
    float sig[2 * NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = 8 * nb + g, j = r / a.G;
      const bool real = r < R;
      const uint8_t *src = a.q.p + 2 * ((int64_t)(at.s.q0 + (real ? j : 0)) * a.q.ts +
                                        (int64_t)((at.h * HC + hh) * a.G + (real ? r - j * a.G : 0)) * a.q.hs);
      float top = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const uint2 x = real ? *reinterpret_cast<const uint2 *>(src + 32 * k + 8 * c) : make_uint2(0u, 0u);
        qf[k][nb][0] = x.x, qf[k][nb][1] = x.y;
        if constexpr (BF16) {
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 f = unpack2<true>(qf[k][nb][y] & 0x7fff7fffu);
            top = fmaxf(top, fmaxf(f.x, f.y));
          }
        }
      }
      float back = 1.f;
      if constexpr (BF16) {
        top = fmaxf(top, __shfl_xor_sync(kAll, top, 1));
        top = fmaxf(top, __shfl_xor_sync(kAll, top, 2));
        const int e = min(max(13 - ((int)(__float_as_uint(top) >> 23) - 127), -115), 115);
        const float f = pow2f(e);
        back = pow2f(-e);
#pragma unroll
        for (int k = 0; k < KS; ++k)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const float2 x = unpack2<true>(qf[k][nb][y]);
            qf[k][nb][y] = pack_f16(x.x * f, x.y * f);
          }
      }
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * nb + 2 * c + e;
        tok |= (rr < R ? (uint32_t)(rr / a.G) : 255u) << (8 * (2 * nb + e));
        sig[2 * nb + e] = a.sig_log2 * __shfl_sync(kAll, back, 4 * (2 * c + e));
      }
    }
    // whether row i sees position t
    auto sees = [&](int i, int t) {
      const int j = tok >> (8 * i) & 255;
      return j != 255 && t <= p_base + j && t > p_base + j - a.window;
    };
    const int lim_min = p_base, low_max = at.s.len - a.window;  // of the first and the last token
    float o[NB][KS][4];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int i = 0; i < KS; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.f;
    float m[2 * NB], l[2 * NB];
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) m[i] = -INFINITY, l[i] = 0.f;
    int E = pv.e_lo;  // o is relative to 2^E

    int k_stage = 0, v_stage = 0;
    for (; at.t < t_end; ++at.t, ++w) {
      if (!wait(&s_full[stage], par)) break;
      k_stage = stage;
      float fk[PB];
      int ev[PB];
#pragma unroll
      for (int b = 0; b < PB; ++b) {
        fk[b] = pow2f(min(max((int)s_pow[stage >> 1][0][my_part[b]][hh], pv.e_lo), pv.e_hi));
        ev[b] = min(max((int)s_pow[stage >> 1][1][my_part[b]][hh], pv.e_lo), pv.e_hi);
      }
      const int t0 = at.lo + at.t * pt + sub * 16 * PB;  // the warp's positions
      float s[PB][NB][4] = {};
#pragma unroll
      for (int k = 0; k < KS; k += 2)
#pragma unroll
        for (int b = 0; b < PB; ++b) {
          uint32_t r[4];
          ldm(r, (at_row[b] + k_stage * kTile) ^ (k << 4));
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint32_t a0 = code2_f16(r[2 * y]), a1 = code2_f16(r[2 * y + 1]);
            const uint32_t a2 = code2_f16(r[2 * y] >> 16), a3 = code2_f16(r[2 * y + 1] >> 16);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma<false>(s[b][nb], a0, a1, a2, a3, qf[k + y][nb][0], qf[k + y][nb][1]);
          }
        }
      next_stage();
      // the last tile's stages are kept: the warps' states meet there
      const bool last = at.t + 1 == t_end;
      if (!last) release(k_stage);
      const bool partial = t0 + 16 * PB - 1 > lim_min || t0 < low_max;
      float mx[2 * NB];
      bool more = false;
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) {
        mx[i] = -INFINITY;
#pragma unroll
        for (int b = 0; b < PB; ++b) {
          // (finite: powers past binary32 times a score of 0 are 0)
          const float f = fminf(sig[i] * fk[b], 3.4028234e38f);
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            float &x = s[b][i >> 1][2 * y + (i & 1)];
            x *= f;
            mx[i] = fmaxf(mx[i], x);
          }
        }
      }
      if (partial) {
#pragma unroll
        for (int i = 0; i < 2 * NB; ++i) {
          mx[i] = -INFINITY;
#pragma unroll
          for (int b = 0; b < PB; ++b)
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              float &x = s[b][i >> 1][2 * y + (i & 1)];
              if (!sees(i, t0 + 16 * b + 8 * y + g)) x = -INFINITY;
              mx[i] = fmaxf(mx[i], x);
            }
        }
      }
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) more = more || mx[i] > m[i];
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
      int top = ev[0];
#pragma unroll
      for (int b = 1; b < PB; ++b) top = max(top, ev[b]);
      if (top > E) {
        const float f = pow2f(max(E - top, -126));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int k = 0; k < KS; ++k) o[nb][k][0] *= f, o[nb][k][1] *= f, o[nb][k][2] *= f, o[nb][k][3] *= f;
        E = top;
      }
      // P^T as the B operand
      uint32_t ph[PB][NB][2];
#pragma unroll
      for (int b = 0; b < PB; ++b) {
        const float fv = pow2f(max(ev[b] - E, -126));
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float ref = m[2 * nb + (e & 1)];
            float &x = s[b][nb][e];
            x = fast_exp2(x - ((ref == -INFINITY ? 0.f : ref) - kShift));
            l[2 * nb + (e & 1)] += x;
            x *= fv;
          }
#pragma unroll
          for (int y = 0; y < 2; ++y) ph[b][nb][y] = movmatrix_t(pack_f16(s[b][nb][2 * y], s[b][nb][2 * y + 1]));
        }
      }
      if (!wait(&s_full[stage], par)) break;
      v_stage = stage;
      next_stage();
      bool plain = false;
      if (partial) {
        // weight 0 times a NaN would be NaN
        uint32_t any = 0;
#pragma unroll
        for (int b = 0; b < PB; ++b)
#pragma unroll
          for (int k = 0; k < KS; k += 2) {
            uint32_t r[4];
            ldm(r, (at_row[b] + v_stage * kTile) ^ (k << 4));
#pragma unroll
            for (int y = 0; y < 4; ++y) any |= (r[y] & 0x7f7f7f7fu) + 0x01010101u;
          }
        plain = __any_sync(kAll, (any & 0x80808080u) != 0);
      }
      if (!plain) {
#pragma unroll
        for (int k = 0; k < KS; k += 2)
#pragma unroll
          for (int b = 0; b < PB; ++b) {
            uint32_t r[4];
            ldm_t(r, (at_row[b] + v_stage * kTile) ^ (k << 4));
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              // bytes of either channel side by side
              const uint32_t u = __byte_perm(r[2 * y], 0, 0x3120), v = __byte_perm(r[2 * y + 1], 0, 0x3120);
              const uint32_t a0 = code2_f16(u), a1 = code2_f16(u >> 16), a2 = code2_f16(v), a3 = code2_f16(v >> 16);
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma<false>(o[nb][k + y], a0, a1, a2, a3, ph[b][nb][0], ph[b][nb][1]);
            }
          }
      } else {
#pragma unroll 1
        for (int y = 0; y < 16 * PB; ++y) {
          const int rr = sub * 16 * PB + y, t = t0 + y;
          const uint8_t *row = sm + v_stage * kTile + row_at(rr);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              // the weight, from the lane that has it in the operand
              uint32_t w2 = 0;
#pragma unroll
              for (int b = 0; b < PB; ++b)
#pragma unroll
                for (int z = 0; z < 2; ++z) {
                  const uint32_t x = __shfl_sync(kAll, ph[b][nb][z], 4 * (2 * c + e) + (y >> 1 & 3));
                  w2 = y >> 3 == 2 * b + z ? x : w2;
                }
              const float2 pair = unpack2<false>(w2);
              const float p = y & 1 ? pair.y : pair.x;
              if (sees(2 * nb + e, t)) {
#pragma unroll
                for (int k = 0; k < KS; ++k) {
                  const float2 x = unpack2<false>(code2_f16(*reinterpret_cast<const uint16_t *>(row + ((k ^ swz(rr)) << 4) + 2 * g)));
                  o[nb][k][e] += p * x.x;
                  o[nb][k][2 + e] += p * x.y;
                }
              }
            }
        }
      }
      if (!last) release(v_stage);
    }

    // The warps' states meet in the two stages just read (keys in an even one,
    // values in the next), relative to the head's largest power.
    float *mg = reinterpret_cast<float *>(sm + k_stage * kTile);  // [kWarps][RU][D]
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
#pragma unroll
      for (int y = 4; y < 32; y <<= 1) l[i] += __shfl_xor_sync(kAll, l[i], y);
      if (g == 0) s_ml[warp][8 * (i >> 1) + 2 * c + (i & 1)] = make_float2(m[i], l[i]);
    }
    if (lane == 0) s_e[warp] = E;
    if (any_of_all(*abort_flag != 0)) break;
    int Eh = E;
    for (int y = 0; y < per_head; ++y) Eh = max(Eh, s_e[hh * per_head + y]);
    const bool whole = t_begin == 0 && t_end == at.nt;
    float *part = a.part + ((int64_t)(2 * blockIdx.x + (t_begin == 0)) * kRowsMaxHeads + hh) * rows_part(D);
    // A piece's sums are in the values' own units; a large power is taken from all
    // of it, the reference put up by as much, so that they stay finite.
    const int down = whole || Eh < 0 ? 0 : 40;
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
        __stcg(part + kRowsPerUnit * D + lane, M + (float)down);
        __stcg(part + kRowsPerUnit * (D + 1) + lane, L * pow2f(-down));
      }
    }
    const float unit = pow2f(Eh - down), rel = pow2f(max(E - Eh, -126));
    constexpr int V = D / 4, RW = 32 / V;  // lanes of a row, rows of a warp at a time
    const int v = lane % V;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
      const int r = 8 * (i >> 1) + 2 * c + (i & 1);
      float M = m[i];
      for (int y = 0; y < per_head; ++y) M = fmaxf(M, s_ml[hh * per_head + y][r].x);
      // a warp that saw nothing has zeros, and 0 * f stays 0; NaN sums stay NaN
      const float f = (m[i] == -INFINITY ? 0.f : fast_exp2(m[i] - M)) * rel;
      float *dst = mg + (warp * RU + r) * D;
#pragma unroll
      for (int k = 0; k < KS; ++k)
        *reinterpret_cast<float2 *>(dst + ((16 * k + 2 * g + 16 * c) & (D - 1))) =
            make_float2(o[i >> 1][k][i & 1] * f, o[i >> 1][k][2 + (i & 1)] * f);
    }
    bar_sync();
    // the warps of a head share its rows, 4 channels a lane
#pragma unroll 2
    for (int i = sub * RW; i < RU; i += RW * per_head) {
      const int r = i + lane / V;
      const float f = __shfl_sync(kAll, inv, r & 31);
      const uint32_t off = __shfl_sync(kAll, row_off, r & 31);
      if (r < R) {
        const float *src = mg + ((hh * per_head) * RU + r) * D + ((4 * v + 16 * (r >> 1 & 3)) & (D - 1));
        float4 x = *reinterpret_cast<const float4 *>(src);
        for (int y = 1; y < per_head; ++y) {
          const float4 z = *reinterpret_cast<const float4 *>(src + y * RU * D);
          x.x += z.x, x.y += z.y, x.z += z.z, x.w += z.w;
        }
        if (!whole) {
          __stcg(reinterpret_cast<float4 *>(part + r * D + 4 * v), make_float4(x.x * unit, x.y * unit, x.z * unit, x.w * unit));
        } else {
          if (f < 0.f) x = make_float4(0.f, 0.f, 0.f, 0.f);
          *reinterpret_cast<uint2 *>(static_cast<uint8_t *>(a.out) + ((uint64_t)off * D + 4 * v) * 2) =
              make_uint2(pack2<BF16>(x.x * f * unit, x.y * f * unit), pack2<BF16>(x.z * f * unit, x.w * f * unit));
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
      if (at.t >= at.nt) next_unit(a, units, at);
    }
  }
  if (*abort_flag && lane == 0) set_err(pv.err, kErrTimeout);
  pdl_trigger();
}

template <int D, int NB, bool BF16>
cudaError_t launch_t(const AttnArgs &a, cudaStream_t st) {
  constexpr int smem = rows_stages<D>() * kT * D + 1024;
  RowsArgs ra;
  memcpy(&ra.mk, a.whole ? a.ok : a.wk, sizeof ra.mk);
  memcpy(&ra.mv, a.whole ? a.ov : a.wv, sizeof ra.mv);
  ra.a = a;
  ra.a.rows = std::min(8 * NB, a.max_new * a.G);
  cudaError_t e = allow_smem<&attn_codes_rows_kernel<D, NB, BF16>>(smem, a.device);
  if (e != cudaSuccess) return e;
  // no more CTAs than are resident, or than runs that there can be
  const int64_t cap = ((int64_t)a.pv.max_pages << a.pv.page_shift) / (kT / a.hc) + 2;
  const int64_t tiles = (int64_t)a.pv.B * (a.pv.Hkv / a.hc) * cap;
  const int64_t runs = a.whole ? tiles / cap : (tiles + kMinShare - 1) / kMinShare;
  const int grid = (int)std::min<int64_t>(std::min(2 * a.sms, kRowsMaxCtas), runs);
  e = launch_pdl(attn_codes_rows_kernel<D, NB, BF16>, dim3(grid), dim3(kThreads + 32), smem, st, ra);
  if (e != cudaSuccess || a.whole) return e;
  // a unit cut in pieces starts in a CTA of its own; eight of the joining CTAs
  // fit an SM
  return launch_pdl(attn_join_kernel<D, BF16>, dim3(std::min(grid * a.hc * ra.a.rows, 8 * a.sms)), dim3(kJoinThreads), 0, st, ra.a);
}
template <int D, bool BF16>
cudaError_t launch_rows(const AttnArgs &a, cudaStream_t st) {
  return a.max_new * a.G <= 8 ? launch_t<D, 1, BF16>(a, st) : launch_t<D, 2, BF16>(a, st);
}

}  // namespace

// [pages, KV heads, slots, D] codes in boxes of a page's slots x `heads` heads
cudaError_t make_codes_map(void *out, void *pool, int D, int page, int Hkv, int n_pages, int heads) {
  const uint64_t d = (uint64_t)D, P = (uint64_t)page, H = (uint64_t)Hkv, N = (uint64_t)n_pages;
  const uint64_t dims[4] = {d, P, H, N}, strides[3] = {d, d * P, d * P * H};
  const uint32_t box[4] = {(uint32_t)D, (uint32_t)page, (uint32_t)heads, 1}, one[4] = {1, 1, 1, 1};
  return encode_tensor_map_tiled(out, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, pool, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                                 D == 128 ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_64B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

cudaError_t launch_attn_codes_rows(const AttnArgs &in, int dtype, cudaStream_t st) {
  if (in.pv.B == 0 || in.pv.n_tokens == 0) return cudaSuccess;
  AttnArgs a = in;
  a.whole = ((int64_t)a.pv.max_pages << a.pv.page_shift) <= kWholeCtx;
  a.hc = a.whole ? 1 : code_heads(1 << a.pv.page_shift, a.pv.Hkv);
  a.part_shift = a.pv.page_shift;
  a.pt_shift = a.hc == 4 ? 5 : a.hc == 2 ? 6 : 7;
  const bool bf = dtype == kSrvBf16;
  switch (a.pv.D) {
    case 128: return bf ? launch_rows<128, true>(a, st) : launch_rows<128, false>(a, st);
    case 64: return bf ? launch_rows<64, true>(a, st) : launch_rows<64, false>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
