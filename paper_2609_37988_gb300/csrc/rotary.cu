// rotary.cu -- rotary positions with several axes, and the append of new
// tokens to a paged cache (their keys rotated on the way).
//
// Frequency i (of R/2) turns with the position on its axis a(i): its pair of
// channels (x, y) becomes (x c - y s, y c + x s) with (c, s) = factor *
// (cos, sin)(pos[a(i)] f_i).  The angle is right to 2^-32 of a turn at any
// position: f_i / (2 pi) is kept as a 64-bit binary fraction of a turn (2^-64 off),
// its product with the position wraps modulo 2^64, which drops whole turns and
// nothing else, and cospi/sinpi of the leading 32 bits follow, rounded to binary32
// (2^-26 of a turn where the angle is near half of one, less in proportion below).
// (The angle in binary32 would be off by 0.06 at position 10^6.)
//
// Memory-bound: every channel is read once and written once.  A thread keeps one
// place in the rows of one token, 2 * VEC channels (two 16-byte pieces), with
// its cosines and sines in registers, and goes over a part of the token's heads,
// always with the next two rows' loads in flight; the first two leave before
// the angles are worked out.  (A thread that keeps a head and goes over tokens
// reads twice the bytes of its data in cosines and sines from shared memory:
// 16384 tokens of a 14B-shaped layer took 84-147 us so, 66 us this way: 6.1 TB/s.)
// Rounding: binary32 arithmetic, one rounding to the stored type.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kRotThreads = 256;
constexpr int kRotTokens = 16;  // of a CTA at most

constexpr int kErrCapacity = 2, kErrPage = 32;  // KVK_DEVERR_*

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_f<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f<__half>(__half x) { return __half2float(x); }
template <typename T>
__device__ __forceinline__ T from_f(float x);
template <>
__device__ __forceinline__ float from_f<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <>
__device__ __forceinline__ __half from_f<__half>(float x) { return __float2half_rn(x); }

template <typename T, int VEC>
struct alignas(sizeof(T) * VEC) Piece {
  T x[VEC];
};
template <typename T>
constexpr bool kIsBf16 = std::is_same<T, __nv_bfloat16>::value;

// Pairs (x, y) -> (x c - y s, y c + x s) of two pieces, (c, s) = w[i]: channel i
// of x0 with channel i of x1, or neighbours.
template <typename T, int VEC>
__device__ __forceinline__ void rotate(Piece<T, VEC> &x0, Piece<T, VEC> &x1, const float2 *w, bool adjacent) {
  if constexpr (sizeof(T) == 2 && VEC % 2 == 0) {
    constexpr int N = VEC / 2;  // words of a piece
    uint32_t(&u)[N] = reinterpret_cast<uint32_t(&)[N]>(x0), (&v)[N] = reinterpret_cast<uint32_t(&)[N]>(x1);
    constexpr bool B = kIsBf16<T>;
    if (!adjacent) {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 x = unpack2<B>(u[i]), y = unpack2<B>(v[i]), p = w[2 * i], q = w[2 * i + 1];
        u[i] = pack2<B>(x.x * p.x - y.x * p.y, x.y * q.x - y.y * q.y);
        v[i] = pack2<B>(y.x * p.x + x.x * p.y, y.y * q.x + x.y * q.y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        const float2 x = unpack2<B>(u[i]), y = unpack2<B>(v[i]), p = w[i], q = w[N + i];
        u[i] = pack2<B>(x.x * p.x - x.y * p.y, x.y * p.x + x.x * p.y);
        v[i] = pack2<B>(y.x * q.x - y.y * q.y, y.y * q.x + y.x * q.y);
      }
    }
  } else {
    auto turn = [&](T &a, T &b, float2 r) {
      const float x = to_f(a), y = to_f(b);
      a = from_f<T>(x * r.x - y * r.y);
      b = from_f<T>(y * r.x + x * r.y);
    };
    if (!adjacent || VEC == 1) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) turn(x0.x[i], x1.x[i], w[i]);
    } else {
#pragma unroll
      for (int i = 0; i + 1 < VEC; i += 2) {
        turn(x0.x[i], x0.x[i + 1], w[i / 2]);
        turn(x1.x[i], x1.x[i + 1], w[(VEC + i) / 2]);
      }
    }
  }
}

// Where token t goes: its sequence and position, or nothing.
struct Place {
  int seq, pos;   // seq < 0: in no sequence
  int64_t slot;   // page * (Hkv * page size) + slot in the page; < 0: not stored
};

// One warp: the sequence whose offsets hold token t is the number of
// sequences that end at or before it.
__device__ Place find_place(const PagedView &v, int t, int lane) {
  int n = 0;
  for (int i = lane; i < v.B; i += 32) n += v.cu[i + 1] <= t;
  n = __reduce_add_sync(0xffffffffu, n);
  Place p = {-1, 0, -1};
  if (n >= v.B) return p;
  const int c0 = v.cu[n], c1 = v.cu[n + 1];
  if (t < c0 || t >= c1) return p;
  p.seq = n;
  p.pos = max(v.lens[n], 0) - c1 + t;
  if (p.pos < 0) return p;
  const int pg = p.pos >> v.page_shift;
  if (pg >= v.max_pages) {
    if (lane == 0) set_err(v.err, kErrCapacity);
    return p;
  }
  const int page = v.table[(int64_t)n * v.max_pages + pg];
  if ((unsigned)page >= (unsigned)v.n_pages) {
    if (lane == 0) set_err(v.err, kErrPage);
    return p;
  }
  p.slot = (((int64_t)page * v.Hkv) << v.page_shift) + (p.pos & ((1 << v.page_shift) - 1));
  return p;
}

template <typename T, int VEC>
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotArgs a, int tok) {
  extern __shared__ float2 cs[];  // [tok][n_freq]
  __shared__ Place s_place[kRotTokens];
  using P = Piece<T, VEC>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t0 = blockIdx.x * tok, nt = min(tok, a.n_tokens - t0);
  const int half = a.t.n_freq;
  const bool paged = a.pv.k != nullptr;

  // this thread's place: piece c of the rows of token j, heads g, g + step, ...
  const int ipr = a.D / (2 * VEC), groups = kRotThreads / ipr, step = groups / tok;
  const int grp = tid / ipr, c = tid - grp * ipr, j = grp / step, g = grp - j * step;
  const bool on = j < nt;
  const bool turn = c < half / VEC;
  const int f = c * VEC;
  // channels: the turned ones, or those behind them (2 half of them)
  const int c0 = turn && !a.t.adjacent ? f : 2 * f, c1 = turn && !a.t.adjacent ? f + half : c0 + VEC;
  const int64_t t = t0 + j;

  // row r of the token: queries, then keys, then values
  const int rows = a.Hq + a.Hk + a.Hv;
  auto load = [&](int r, P &x0, P &x1) {
    if (!on || r >= rows) return;
    const bool q = r < a.Hq, v = r >= a.Hq + a.Hk;
    const Rows &in = q ? a.q : v ? a.v : a.k;
    const T *src = reinterpret_cast<const T *>(in.p) + t * in.ts + (r - (q ? 0 : v ? a.Hq + a.Hk : a.Hq)) * in.hs;
    x0 = *reinterpret_cast<const P *>(src + (v ? 2 * f : c0));
    x1 = *reinterpret_cast<const P *>(src + (v ? 2 * f + VEC : c1));
  };
  pdl_wait();
  P xa[2], xb[2];
  load(g, xa[0], xa[1]);
  load(g + step, xb[0], xb[1]);
  if (paged) {
    for (int i = warp; i < nt; i += kRotThreads / 32) {
      const Place p = find_place(a.pv, t0 + i, lane);
      if (lane == 0) s_place[i] = p;
    }
    if (!a.pos) __syncthreads();
  }
  for (int i = tid; i < nt * half; i += kRotThreads) {
    const int jj = i / half, fr = i - jj * half;
    const int p = a.pos ? a.pos[(int64_t)a.t.axis[fr] * a.n_tokens + t0 + jj] : s_place[jj].pos;
    // the angle's leading 32 bits, a signed fraction of a turn
    const uint64_t angle = a.t.step[fr] * (uint64_t)(int64_t)p;
    const float x = (float)(int32_t)(uint32_t)(angle >> 32) * 0x1p-31f;  // in half turns
    float sn, cn;
    sincospif(x, &sn, &cn);
    cs[i] = make_float2(cn * a.t.factor, sn * a.t.factor);
  }
  __syncthreads();
  if (on) {
    float2 w[VEC];
    if (turn) {
#pragma unroll
      for (int i = 0; i < VEC; ++i) w[i] = cs[j * half + f + i];
    }
    const Place pl = paged ? s_place[j] : Place{0, 0, 0};
    auto finish = [&](int r, P &x0, P &x1) {
      if (r >= rows) return;
      const bool q = r < a.Hq, v = r >= a.Hq + a.Hk;
      T *dst;
      if (q || !paged) {
        if (pl.seq < 0) return;
        const Rows &out = q ? a.qo : a.ko;
        dst = reinterpret_cast<T *>(out.p) + t * out.ts + (r - (q ? 0 : a.Hq)) * out.hs;
      } else {
        if (pl.slot < 0) return;
        dst = reinterpret_cast<T *>(v ? a.pv.v : a.pv.k) +
              (pl.slot + ((int64_t)(r - (v ? a.Hq + a.Hk : a.Hq)) << a.pv.page_shift)) * a.D;
      }
      if (!v && turn) rotate<T, VEC>(x0, x1, w, a.t.adjacent);
      *reinterpret_cast<P *>(dst + (v ? 2 * f : c0)) = x0;
      *reinterpret_cast<P *>(dst + (v ? 2 * f + VEC : c1)) = x1;
    };
    for (int r = g; r < rows; r += 2 * step) {
      finish(r, xa[0], xa[1]);
      load(r + 2 * step, xa[0], xa[1]);
      finish(r + step, xb[0], xb[1]);
      load(r + 3 * step, xb[0], xb[1]);
    }
  }
  pdl_trigger();
}

template <typename T, int VEC>
cudaError_t launch_t(const RotArgs &a, cudaStream_t st) {
  // Tokens of a CTA: as many as leave a thread six rows or so (16384 tokens of a
  // 14B-shaped layer: 104, 78, 66, 77 us with 1, 2, 4, 8), fewer where that would
  // leave SMs without work: one token per CTA is the quickest for few.
  const int ipr = a.D / (2 * VEC), groups = kRotThreads / ipr, rows = a.Hq + a.Hk + a.Hv;
  int tok = 1;
  while (2 * tok <= std::min(kRotTokens, groups) && 2 * tok * rows <= 7 * groups && a.n_tokens / (2 * tok) >= 600) tok *= 2;
  return launch_pdl(rotary_kernel<T, VEC>, dim3((a.n_tokens + tok - 1) / tok), dim3(kRotThreads),
                    (size_t)tok * a.t.n_freq * sizeof(float2), st, a, tok);
}

bool rows_aligned(const Rows &r, int elem) {
  return !r.p || ((reinterpret_cast<uintptr_t>(r.p) | (uint64_t)(r.ts * elem) | (uint64_t)(r.hs * elem)) & 15u) == 0;
}

template <typename T>
cudaError_t launch_vec(const RotArgs &a, cudaStream_t st) {
  constexpr int VEC = 16 / sizeof(T);
  // Pieces of 16 bytes where every row starts on 16 bytes and the rotated
  // part is whole pieces; single channels otherwise.
  const bool wide = a.D % (2 * VEC) == 0 && a.t.n_freq % VEC == 0 && rows_aligned(a.q, sizeof(T)) &&
                    rows_aligned(a.k, sizeof(T)) && rows_aligned(a.v, sizeof(T)) && rows_aligned(a.qo, sizeof(T)) &&
                    rows_aligned(a.ko, sizeof(T));
  return wide ? launch_t<T, VEC>(a, st) : launch_t<T, 1>(a, st);
}

}  // namespace

cudaError_t launch_rotary(const RotArgs &a, int dtype, cudaStream_t st) {
  if (a.n_tokens == 0 || a.Hq + a.Hk + a.Hv == 0) return cudaSuccess;
  switch (dtype) {
    case kSrvF32: return launch_vec<float>(a, st);
    case kSrvBf16: return launch_vec<__nv_bfloat16>(a, st);
    case kSrvF16: return launch_vec<__half>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
