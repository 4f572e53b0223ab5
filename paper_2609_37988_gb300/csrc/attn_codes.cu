// attn_codes.cu -- attention of new tokens over a paged cache in 8 bits.
//
// A warp per (token, query head): its positions one by one, a key's dot product
// across the lanes, the softmax online in base 2, sums in binary32.
#include <math.h>

#include <algorithm>

#include "common.cuh"
#include "fp8.cuh"
#include "kernels.h"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kErrCount = 4, kErrPage = 32;  // KVK_DEVERR_*
constexpr uint32_t kAll = 0xffffffffu;

template <int D, bool BF16>
__global__ void __launch_bounds__(256) attn_codes_kernel(const __grid_constant__ AttnArgs a) {
  constexpr int N = D / 32;  // channels of a lane
  const PagedView &pv = a.pv;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  pdl_wait();
  pdl_trigger();
  const int t = (int)(w / a.Hq), h = (int)(w - (int64_t)t * a.Hq), kh = h / a.G;
  if (t >= pv.n_tokens) return;
  int seq = 0;
  for (int i = lane; i < pv.B; i += 32) seq += pv.cu[i + 1] <= t;
  seq = __reduce_add_sync(kAll, seq);
  if (seq >= pv.B || t < pv.cu[seq] || t >= pv.cu[seq + 1]) return;
  const int c0 = min(max(pv.cu[seq], 0), pv.n_tokens), n = min(max(pv.cu[seq + 1], c0), pv.n_tokens) - c0;
  int len = max(pv.lens[seq], 0);
  const int cap = pv.max_pages << pv.page_shift;
  if (len > cap || n > a.max_new) {
    if (lane == 0) set_err(pv.err, kErrCount);
    len = min(len, cap);
  }
  const int p = len - n + t - c0;
  float q[N], o[N] = {};
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint16_t x = *reinterpret_cast<const uint16_t *>(a.q.p + 2 * ((int64_t)t * a.q.ts + h * a.q.hs + N * lane + i));
    q[i] = unpack2<BF16>(x).x;
  }
  float m = -INFINITY, l = 0.f;
  for (int s = max(0, p - a.window + 1); s <= p; ++s) {
    const int page = pv.table[(int64_t)seq * pv.max_pages + (s >> pv.page_shift)];
    float k[N], v[N];
    if ((unsigned)page < (unsigned)pv.n_pages) {
      const int64_t at = (int64_t)page * pv.Hkv + kh, row = ((at << pv.page_shift) + (s & ((1 << pv.page_shift) - 1))) * D + N * lane;
      const float fk = pow2f(min(max((int)pv.ke[at], pv.e_lo), pv.e_hi)), fv = pow2f(min(max((int)pv.ve[at], pv.e_lo), pv.e_hi));
#pragma unroll
      for (int i = 0; i < N; i += 2) {
        const float2 x = unpack2<false>(code2_f16(*reinterpret_cast<const uint16_t *>(pv.k + row + i)));
        const float2 y = unpack2<false>(code2_f16(*reinterpret_cast<const uint16_t *>(pv.v + row + i)));
        k[i] = x.x * fk, k[i + 1] = x.y * fk, v[i] = y.x * fv, v[i + 1] = y.y * fv;
      }
    } else {
      if (lane == 0) set_err(pv.err, kErrPage);
#pragma unroll
      for (int i = 0; i < N; ++i) k[i] = v[i] = 0.f;
    }
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) x += q[i] * k[i];
#pragma unroll
    for (int y = 16; y; y >>= 1) x += __shfl_xor_sync(kAll, x, y);
    x *= a.sig_log2;
    const float mn = fmaxf(m, x), f = m == -INFINITY ? 0.f : fast_exp2(m - mn), pr = mn == -INFINITY ? 0.f : fast_exp2(x - mn);
    m = mn;
    l = l * f + pr;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = o[i] * f + pr * v[i];
  }
  const float inv = p >= 0 ? 1.f / l : 0.f;
  uint8_t *dst = static_cast<uint8_t *>(a.out) + 2 * (((int64_t)t * a.Hq + h) * D + N * lane);
#pragma unroll
  for (int i = 0; i < N; i += 2) reinterpret_cast<uint32_t *>(dst)[i / 2] = pack2<BF16>(o[i] * inv, o[i + 1] * inv);
}

template <int D>
cudaError_t launch_t(const AttnArgs &a, bool bf, cudaStream_t st) {
  const int64_t warps = (int64_t)a.pv.n_tokens * a.Hq;
  return launch_pdl(bf ? attn_codes_kernel<D, true> : attn_codes_kernel<D, false>, dim3((unsigned)((warps + 7) / 8)), dim3(256), 0,
                    st, a);
}

}  // namespace

cudaError_t launch_attn_codes(const AttnArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.B == 0 || a.pv.n_tokens == 0) return cudaSuccess;
  switch (a.pv.D) {
    case 128: return launch_t<128>(a, dtype == kSrvBf16, st);
    case 64: return launch_t<64>(a, dtype == kSrvBf16, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
