// attn_tc.cu -- attention of prompts and of chunks over pages in 16 bits
// (attn_tc.cuh).
#include "attn_tc.cuh"

namespace kvk {
namespace {

template <int D, bool BF16>
cudaError_t launch_src(const AttnArgs &a, cudaStream_t st) {
  return a.pv.k ? launch_t<D, BF16, kPaged>(a, st) : launch_t<D, BF16, kPacked>(a, st);
}

}  // namespace

// [pages, KV heads, slots, D] as boxes of up to 64 slots x 64 channels, or
// (`heads` > 0) x all channels, 64 at a time one behind another, x so many heads
cudaError_t make_pages_map(void *out, bool bf, void *pool, int D, int page, int Hkv, int n_pages, int heads) {
  const bool whole = heads > 0;
  const uint64_t row = (uint64_t)D * 2, P = (uint64_t)page, H = (uint64_t)Hkv, N = (uint64_t)n_pages;
  const uint64_t dims4[4] = {(uint64_t)D, P, H, N}, strides4[3] = {row, row * P, row * P * H};
  const uint64_t dims5[5] = {64, P, (uint64_t)D / 64, H, N}, strides5[4] = {row, 128, row * P, row * P * H};
  const uint32_t rows = (uint32_t)std::min(page, 64);
  const uint32_t box4[4] = {64, rows, 1, 1}, box5[5] = {64, rows, (uint32_t)D / 64, (uint32_t)heads, 1}, one[5] = {1, 1, 1, 1, 1};
  return encode_tensor_map_tiled(out, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, whole ? 5 : 4,
                                 pool, whole ? dims5 : dims4, whole ? strides5 : strides4, whole ? box5 : box4, one,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}

cudaError_t launch_attn_tc(const AttnArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.B == 0 || a.pv.n_tokens == 0) return cudaSuccess;
  const bool bf = dtype == kSrvBf16;
  switch (a.pv.D) {
    case 128: return bf ? launch_src<128, true>(a, st) : launch_src<128, false>(a, st);
    case 64: return bf ? launch_src<64, true>(a, st) : launch_src<64, false>(a, st);
    default: return cudaErrorInvalidValue;
  }
}

}  // namespace kvk
