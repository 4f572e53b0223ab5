// rotary.cu -- rotary positions with several axes, and the append of new
// tokens to a paged cache (their keys rotated on the way).
//
// Frequency i (of R/2) turns with the position on its axis a(i): its pair of
// channels (x, y) becomes (x c - y s, y c + x s) with (c, s) = factor *
// (cos, sin)(pos[a(i)] f_i).  Angles are exact to 2^-32 of a turn at any
// position: f_i / (2 pi) is kept as a 64-bit binary fraction of a turn, its
// product with the position wraps modulo 2^64, which drops whole turns and
// nothing else, and cospi/sinpi of the leading 32 bits follow.  (The angle in
// binary32 would be off by 0.06 at position 10^6.)
//
// Memory-bound: every channel is read once and written once.  A CTA takes
// `tok` tokens; 2 * VEC channels per thread and step (two 16-byte pieces), the
// first ones loaded before the angles, whose latency they hide.  Rounding:
// binary32 arithmetic, one rounding to the stored type.
#include <math.h>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kRotThreads = 256;
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
__global__ void __launch_bounds__(kRotThreads) rotary_kernel(const __grid_constant__ RotArgs a, int tok, uint32_t ipr_magic) {
  extern __shared__ float2 cs[];  // [tok][n_freq]
  __shared__ Place s_place[8];
  using P = Piece<T, VEC>;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int t0 = blockIdx.x * tok;
  const int nt = min(tok, a.n_tokens - t0);
  const int ipr = a.D / (2 * VEC);              // steps of a row
  const int rows = a.Hq + a.Hk + a.Hv;
  const int half = a.t.n_freq, rot = half / VEC;
  const int total = nt * rows * ipr;
  const bool paged = a.pv.k != nullptr;

  // step e: row r of the CTA's tokens, pieces at channels c0 and c1; the
  // first `turn` kinds are rotated with frequencies f..
  struct Step {
    const T *src;
    T *dst;       // null: not stored
    int c0, c1, f, j;
    bool turn;
  };
  auto decode = [&](int e, bool want_dst) {
    Step s;
    const int row = ipr == 1 ? e : (int)__umulhi((uint32_t)e, ipr_magic), c = e - row * ipr;
    s.j = row / rows;
    const int h = row - s.j * rows;
    const int64_t t = t0 + s.j;
    const Rows *in, *out;
    int hh = h;
    bool to_page = false;
    uint8_t *pages = nullptr;
    if (h < a.Hq) {
      in = &a.q;
      out = &a.qo;
    } else if (h < a.Hq + a.Hk) {
      hh = h - a.Hq;
      in = &a.k;
      out = &a.ko;
      to_page = paged;
      pages = a.pv.k;
    } else {
      hh = h - a.Hq - a.Hk;
      in = &a.v;
      out = &a.v;
      to_page = true;
      pages = a.pv.v;
    }
    s.src = reinterpret_cast<const T *>(in->p) + t * in->ts + hh * in->hs;
    s.turn = h < a.Hq + a.Hk && c < rot;
    s.f = c * VEC;
    if (s.turn) {
      s.c0 = a.t.adjacent ? 2 * VEC * c : VEC * c;
      s.c1 = a.t.adjacent ? s.c0 + VEC : s.c0 + half;
    } else {
      s.c0 = 2 * VEC * c;  // channels behind the rotated ones (2 * half of them), or a value row's
      s.c1 = s.c0 + VEC;
    }
    s.dst = nullptr;
    if (want_dst) {
      const Place &pl = s_place[s.j];
      if (to_page) {
        if (pl.slot >= 0)
          s.dst = reinterpret_cast<T *>(pages) + (pl.slot + ((int64_t)hh << a.pv.page_shift)) * a.D;
      } else if (!paged || pl.seq >= 0) {
        s.dst = reinterpret_cast<T *>(out->p) + t * out->ts + hh * out->hs;
      }
    }
    return s;
  };

  pdl_wait();
  // the first step's data, before the angles
  P x0, x1;
  if (tid < total) {
    const Step s = decode(tid, false);
    x0 = *reinterpret_cast<const P *>(s.src + s.c0);
    x1 = *reinterpret_cast<const P *>(s.src + s.c1);
  }
  if (paged) {
    for (int j = warp; j < nt; j += kRotThreads / 32) {
      const Place p = find_place(a.pv, t0 + j, lane);
      if (lane == 0) s_place[j] = p;
    }
    if (!a.pos) __syncthreads();
  }
  for (int i = tid; i < nt * half; i += kRotThreads) {
    const int j = i / half, f = i - j * half;
    const int p = a.pos ? a.pos[(int64_t)a.t.axis[f] * a.n_tokens + t0 + j] : s_place[j].pos;
    // the angle's leading 32 bits, a signed fraction of a turn
    const uint64_t turn = a.t.step[f] * (uint64_t)(int64_t)p;
    const float x = (float)(int32_t)(uint32_t)(turn >> 32) * 0x1p-31f;  // in half turns
    float sn, c;
    sincospif(x, &sn, &c);
    cs[i] = make_float2(c * a.t.factor, sn * a.t.factor);
  }
  __syncthreads();
  for (int e = tid; e < total; e += kRotThreads) {
    const Step s = decode(e, true);
    if (e != tid) {
      x0 = *reinterpret_cast<const P *>(s.src + s.c0);
      x1 = *reinterpret_cast<const P *>(s.src + s.c1);
    }
    if (!s.dst) continue;
    if (s.turn) {
      const float2 *w = cs + s.j * half + s.f;
      P y0, y1;
      if (!a.t.adjacent) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float u = to_f(x0.x[i]), v = to_f(x1.x[i]);
          y0.x[i] = from_f<T>(u * w[i].x - v * w[i].y);
          y1.x[i] = from_f<T>(v * w[i].x + u * w[i].y);
        }
      } else {
        T in[2 * VEC], out[2 * VEC];
#pragma unroll
        for (int i = 0; i < VEC; ++i) in[i] = x0.x[i], in[VEC + i] = x1.x[i];
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
          const float u = to_f(in[2 * i]), v = to_f(in[2 * i + 1]);
          out[2 * i] = from_f<T>(u * w[i].x - v * w[i].y);
          out[2 * i + 1] = from_f<T>(v * w[i].x + u * w[i].y);
        }
#pragma unroll
        for (int i = 0; i < VEC; ++i) y0.x[i] = out[i], y1.x[i] = out[VEC + i];
      }
      x0 = y0;
      x1 = y1;
    }
    *reinterpret_cast<P *>(s.dst + s.c0) = x0;
    *reinterpret_cast<P *>(s.dst + s.c1) = x1;
  }
  pdl_trigger();
}

template <typename T, int VEC>
cudaError_t launch_t(const RotArgs &a, cudaStream_t st) {
  const int ipr = a.D / (2 * VEC);
  // One token per CTA fills the machine soonest; with thousands of tokens
  // four per CTA leave fewer CTAs to start.
  const int tok = a.n_tokens >= 4096 ? 4 : 1;
  const dim3 grid((a.n_tokens + tok - 1) / tok);
  const uint32_t magic = (uint32_t)(((1ull << 32) + ipr - 1) / ipr);
  return launch_pdl(rotary_kernel<T, VEC>, grid, dim3(kRotThreads), (size_t)tok * a.t.n_freq * sizeof(float2), st, a, tok, magic);
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
