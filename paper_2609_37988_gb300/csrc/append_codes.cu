// append_codes.cu -- new tokens into the pages of a cache in 8 bits.
//
// A page's keys of one KV head (and its values) share a power of two: a number x is
// held as the e4m3 code nearest to x 2^-e (ties to even).  e is the least in the
// dtype's range with max |x| <= 448 2^e over the page's finite numbers, so that with
// e4m3's own exponents every code times 2^e is a number of the dtype and attention
// loses nothing more.  A page that was begun before keeps at least its e; where new
// tokens raise it, the codes that are there go to the nearest of code 2^(old - new):
// exact but for those that become subnormal.  What is not finite is held as NaN and
// does not count for e.
//
// Memory-bound: 2 bytes read and 1 written a number.  A group of threads takes one
// page's new tokens of one KV head, keys or values, up to 64 numbers a thread in
// registers: read once, their largest magnitude found, coded and written.  (A group
// smaller than the page's tokens, which the host takes where most sequences have few,
// goes over them twice.)  Magnitudes are compared as 16-bit integers, two at a time;
// what is not finite stands above them all and sends its thread another way.
// Measured, 40 / 8 heads of 128: 4 x 4096 tokens 20.5 us (floor 14.8; compared
// and checked one by one as floats 25.2); a step of 32 3.0.  With keys turned on the way
// 61 us in pages of 16 and 162 in pages of 128 (in 16 bits 31), a step 5.0 (3.5): every
// CTA finds its page's sines for itself, those with values alone too, and a channel's
// partner is a load of its own.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kThreads = 256;
constexpr int kChunks = 8;                         // of 8 channels, a thread's
constexpr int kErrCapacity = 2, kErrPage = 32;     // KVK_DEVERR_*
constexpr uint32_t kAll = 0xffffffffu;

// The new tokens that go to one page.
struct Unit {
  int page;            // < 0: nothing to do
  int s0, s1;          // their slots
  int tok;             // token of slot s0
  int pos;             // position of slot s0
};

// One warp: unit number `u` of the batch.
__device__ Unit find_unit(const PagedView &v, int u, int lane) {
  Unit r = {-1, 0, 0, 0, 0};
  int before = 0;
  for (int b0 = 0; b0 < v.B; b0 += 32) {
    const int b = b0 + lane;
    int c0 = 0, n = 0, len = 0, first = 0, last = -1;
    if (b < v.B) {
      const int e0 = v.cu[b], e1 = v.cu[b + 1];
      len = max(v.lens[b], 0);
      c0 = min(max(e0, 0), v.n_tokens);
      n = min(max(e1, c0), v.n_tokens) - c0;
      const int cap = v.max_pages << v.page_shift;
      first = max(len - n, 0);
      last = min(len, cap) - 1;
      if (n == 0) last = first - 1;
    }
    const int mine = last >= first ? (last >> v.page_shift) - (first >> v.page_shift) + 1 : 0;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int y = __shfl_up_sync(kAll, sum, o);
      if (lane >= o) sum += y;
    }
    const uint32_t past = __ballot_sync(kAll, before + sum > u);
    if (past) {
      const int f = __ffs(past) - 1;
      if (lane == f) {
        const int pg = (first >> v.page_shift) + u - (before + sum - mine), at = pg << v.page_shift;
        const int page = v.table[(int64_t)b * v.max_pages + pg];
        r.s0 = max(first - at, 0);
        r.s1 = min(last + 1 - at, 1 << v.page_shift);
        r.pos = at + r.s0;
        r.tok = c0 + n - len + r.pos;
        if ((unsigned)page < (unsigned)v.n_pages)
          r.page = page;
        else
          set_err(v.err, kErrPage);
      }
      r.page = __shfl_sync(kAll, r.page, f);
      r.s0 = __shfl_sync(kAll, r.s0, f);
      r.s1 = __shfl_sync(kAll, r.s1, f);
      r.tok = __shfl_sync(kAll, r.tok, f);
      r.pos = __shfl_sync(kAll, r.pos, f);
      return r;
    }
    before += __shfl_sync(kAll, sum, 31);
  }
  return r;
}

template <bool BF16>
__device__ __forceinline__ float to_f(uint16_t x) {
  return unpack2<BF16>(x).x;
}

// 8 channels from `p` on, as pairs of the dtype
__device__ __forceinline__ uint4 load8(const uint8_t *p, bool wide) {
  if (wide) return *reinterpret_cast<const uint4 *>(p);
  const uint16_t *h = reinterpret_cast<const uint16_t *>(p);
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] = h[2 * i] | (uint32_t)h[2 * i + 1] << 16;
  return make_uint4(w[0], w[1], w[2], w[3]);
}

// magnitudes from here on are not finite
template <bool BF16>
constexpr uint32_t kInf = BF16 ? 0x7f80u : 0x7c00u;

template <int D, bool BF16>
__global__ void __launch_bounds__(kThreads, 4) append_codes_kernel(const __grid_constant__ CodeArgs a, int gt) {
  constexpr int C = D / 8;               // chunks of a row
  extern __shared__ float2 cs[];         // [new tokens][n_freq]
  __shared__ uint32_t s_top[kThreads / 32];
  const PagedView &pv = a.pv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int page_size = 1 << pv.page_shift;
  pdl_wait();
  const Unit u = find_unit(pv, blockIdx.x, lane);  // (every warp for itself: nobody waits)
  if (blockIdx.x == 0 && blockIdx.y == 0 && warp == 1) {
    for (int b = lane; b < pv.B; b += 32) {
      const int c0 = min(max(pv.cu[b], 0), pv.n_tokens), c1 = min(max(pv.cu[b + 1], c0), pv.n_tokens);
      if (c1 > c0 && pv.lens[b] > pv.max_pages << pv.page_shift) set_err(pv.err, kErrCapacity);
    }
  }
  if (u.page < 0) {
    pdl_trigger();
    return;
  }
  const int n = u.s1 - u.s0, nf = a.t.n_freq;
  const int grp = tid / gt, g = tid - grp * gt, pair = blockIdx.y * (kThreads / gt) + grp;
  const int h = pair >> 1, is_v = pair & 1;
  const bool on = pair < 2 * pv.Hkv;
  const int c = g % C, r0 = g / C, step = gt / C;
  const int rows = kChunks * step, turns = (n + rows - 1) / rows;
  const Rows &in = is_v ? a.v : a.k;
  uint4 x[kChunks];
  auto load = [&](int turn) {
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
      const int r = turn * rows + r0 + i * step;
      x[i] = make_uint4(0, 0, 0, 0);
      if (on && r < n) x[i] = load8(in.p + 2 * ((int64_t)(u.tok + r) * in.ts + h * in.hs + 8 * c), a.wide);
    }
  };
  load(0);
  const int64_t at_e = (int64_t)u.page * pv.Hkv + h;
  int8_t *exps = is_v ? pv.ve : pv.ke;
  const int old = on && u.s0 > 0 ? min(max((int)exps[at_e], pv.e_lo), pv.e_hi) : pv.e_lo;
  if (a.rotate) {
    for (int i = tid; i < n * nf; i += kThreads) {
      const int r = i / nf, f = i - r * nf;
      const int p = a.pos ? a.pos[(int64_t)a.t.axis[f] * pv.n_tokens + u.tok + r] : u.pos + r;
      const uint64_t angle = a.t.step[f] * (uint64_t)(int64_t)p;
      float sn, cn;
      sincospif((float)(int32_t)(uint32_t)(angle >> 32) * 0x1p-31f, &sn, &cn);
      cs[i] = make_float2(cn * a.t.factor, sn * a.t.factor);
    }
    __syncthreads();
  }
  // keys turned to their tokens' positions
  auto turned = [&](int turn) {
    if (!a.rotate || !on || is_v) return;
#pragma unroll 1
    for (int i = 0; i < kChunks; ++i) {
      const int r = turn * rows + r0 + i * step;
      if (r >= n) break;
      const uint8_t *row = in.p + 2 * ((int64_t)(u.tok + r) * in.ts + h * in.hs);
      uint32_t w[4] = {x[0].x, x[0].y, x[0].z, x[0].w};
#pragma unroll
      for (int y = 1; y < kChunks; ++y)
        if (y == i) w[0] = x[y].x, w[1] = x[y].y, w[2] = x[y].z, w[3] = x[y].w;
      uint16_t o[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int ch = 8 * c + e;
        o[e] = (uint16_t)(w[e >> 1] >> (16 * (e & 1)));
        if (ch >= 2 * nf) continue;
        const bool second = a.t.adjacent ? ch & 1 : ch >= nf;
        const int f = a.t.adjacent ? ch >> 1 : second ? ch - nf : ch;
        const int other = a.t.adjacent ? ch ^ 1 : second ? f : ch + nf;
        const float mine = to_f<BF16>(o[e]), theirs = to_f<BF16>(reinterpret_cast<const uint16_t *>(row)[other]);
        const float2 t = cs[r * nf + f];
        const float y = second ? mine * t.x + theirs * t.y : mine * t.x - theirs * t.y;
        o[e] = (uint16_t)pack2<BF16>(y, 0.f);
      }
#pragma unroll
      for (int y = 0; y < kChunks; ++y)
        if (y == i)
          x[y] = make_uint4(o[0] | (uint32_t)o[1] << 16, o[2] | (uint32_t)o[3] << 16, o[4] | (uint32_t)o[5] << 16,
                            o[6] | (uint32_t)o[7] << 16);
    }
  };
  // the largest magnitude, as the dtype's bits; of finite numbers if `all` has others
  auto largest = [&](bool &all_finite) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
      top = __vmaxu2(top, __vmaxu2(__vmaxu2(x[i].x & 0x7fff7fffu, x[i].y & 0x7fff7fffu),
                                   __vmaxu2(x[i].z & 0x7fff7fffu, x[i].w & 0x7fff7fffu)));
    top = max(top & 0xffffu, top >> 16);
    all_finite = top < kInf<BF16>;
    if (!all_finite) {
      top = 0;
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const uint32_t m0 = w[y] & 0x7fffu, m1 = w[y] >> 16 & 0x7fffu;
          top = max(top, max(m0 < kInf<BF16> ? m0 : 0u, m1 < kInf<BF16> ? m1 : 0u));
        }
      }
    }
    return top;
  };
  bool fine = true;
  turned(0);
  uint32_t top = largest(fine);
  for (int t = 1; t < turns; ++t) {
    load(t);
    turned(t);
    top = max(top, largest(fine));
  }
  top = __reduce_max_sync(kAll, top);
  if (gt > 32) {
    if (lane == 0) s_top[warp] = top;
    __syncthreads();
    const int w0 = grp * (gt / 32);
    for (int i = 0; i < gt / 32; ++i) top = max(top, s_top[w0 + i]);
  }
  if (on) {
    const int e = max(code_exponent(to_f<BF16>((uint16_t)top), pv.e_lo, pv.e_hi), old);
    uint8_t *dst = (is_v ? pv.v : pv.k) + at_e * page_size * D;
    if (u.s0 > 0 && e > old) {
      // the codes that are there
      const float down = pow2f(max(old - e, -126));
      for (int i = g; i < u.s0 * (D / 16); i += gt) {
        uint4 *p = reinterpret_cast<uint4 *>(dst) + i;
        const uint4 q = *p;
        *p = make_uint4(codes_times(q.x, down), codes_times(q.y, down), codes_times(q.z, down), codes_times(q.w, down));
      }
    }
    const float up = pow2f(-e);
    // the last turn's numbers are at hand
    for (int t = turns - 1; t >= 0; --t) {
      if (t < turns - 1) {
        load(t);
        turned(t);
        largest(fine);
      }
#pragma unroll
      for (int i = 0; i < kChunks; ++i) {
        const int r = t * rows + r0 + i * step;
        if (r >= n) continue;
        *reinterpret_cast<uint2 *>(dst + (int64_t)(u.s0 + r) * D + 8 * c) =
            fine ? make_uint2(code4<BF16>(x[i].x, x[i].y, up), code4<BF16>(x[i].z, x[i].w, up))
                 : make_uint2(code4_any<BF16>(x[i].x, x[i].y, up), code4_any<BF16>(x[i].z, x[i].w, up));
      }
    }
    // (the group's threads have read the old power)
    __syncwarp();
    if (g == 0) exps[at_e] = (int8_t)e;
  }
  pdl_trigger();
}

template <int D, bool BF16>
cudaError_t launch_t(const CodeArgs &a, cudaStream_t st) {
  const PagedView &v = a.pv;
  const int page = 1 << v.page_shift;
  // Threads that hold a page's new rows, 64 numbers each, a warp at least: those of a
  // whole page, or twice what a sequence has on average where that is less (64 single
  // tokens into pages of 128: 3.5 us, with groups for whole pages 10.8).
  const int64_t seqs = std::min(v.B, v.n_tokens), some = std::min<int64_t>(page, 2 * (v.n_tokens / seqs));
  int gt = 32;
  while (gt * 8 * kChunks < some * D) gt *= 2;
  const int64_t units = std::min<int64_t>(v.n_tokens, v.n_tokens / page + 2 * seqs);
  const int smem = a.rotate ? page * a.t.n_freq * (int)sizeof(float2) : 0;
  int dev = 0;
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) {
    e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = allow_smem<&append_codes_kernel<D, BF16>>(64 * 1024, dev);
    if (e != cudaSuccess) return e;
  }
  const int per = kThreads / gt;
  return launch_pdl(append_codes_kernel<D, BF16>, dim3((unsigned)units, (2 * v.Hkv + per - 1) / per), dim3(kThreads), smem, st, a,
                    gt);
}

}  // namespace

cudaError_t launch_append_codes(const CodeArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.B == 0 || a.pv.n_tokens == 0) return cudaSuccess;
  const bool bf = dtype == kSrvBf16;
  switch (a.pv.D) {
    case 128: return bf ? launch_t<128, true>(a, st) : launch_t<128, false>(a, st);
    case 64: return bf ? launch_t<64, true>(a, st) : launch_t<64, false>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
