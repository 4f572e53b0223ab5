// attn_tc_codes.cu -- attention of chunks over pages in 8 bits (attn_tc.cuh).
#include "attn_tc.cuh"

namespace kvk {

cudaError_t launch_attn_tc_codes(const AttnArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.B == 0 || a.pv.n_tokens == 0) return cudaSuccess;
  const bool bf = dtype == kSrvBf16, few = a.max_new <= kTcT / a.G;
  if (few) {
    switch (a.pv.D) {
      case 128: return bf ? launch_t<128, true, kCodesFew>(a, st) : launch_t<128, false, kCodesFew>(a, st);
      case 64: return bf ? launch_t<64, true, kCodesFew>(a, st) : launch_t<64, false, kCodesFew>(a, st);
      default: return cudaErrorInvalidValue;
    }
  }
  switch (a.pv.D) {
    case 128: return bf ? launch_t<128, true, kCodes>(a, st) : launch_t<128, false, kCodes>(a, st);
    case 64: return bf ? launch_t<64, true, kCodes>(a, st) : launch_t<64, false, kCodes>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
