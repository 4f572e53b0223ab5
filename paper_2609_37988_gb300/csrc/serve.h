// serve.h -- arguments of the serving kernels (rotary positions, paged cache,
// attention over packed prompts) and their launchers.
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace kvk {

// x / y, in 32 bits where they do (a 64-bit division takes 500 cycles)
__device__ __forceinline__ int64_t div_pos(int64_t x, int64_t y) {
  if (((x | y) >> 32) == 0) return (uint32_t)x / (uint32_t)y;
  return x / y;
}

constexpr int kSrvF32 = 0, kSrvBf16 = 1, kSrvF16 = 2;  // KVK_DTYPE_*
constexpr int kRotMaxFreq = 128;

// Rotation frequencies: step[i] = inv_freq[i] / (2 pi) of a turn as a 64-bit
// binary fraction, axis[i] the axis whose position it turns with.
struct RotTable {
  uint64_t step[kRotMaxFreq];
  uint8_t axis[kRotMaxFreq];
  float factor;
  int n_freq, n_axes, adjacent;
};

// [tokens, heads, head_dim] rows; strides in elements, channels contiguous
struct Rows {
  uint8_t *p;
  int64_t ts, hs;
};

// The pages of one layer and the batch that a call works on.
struct PagedView {
  uint8_t *k, *v;         // [n_pages, Hkv, page, D]
  const int32_t *cu;      // [B + 1] offsets of the new tokens
  const int32_t *lens;    // [B] positions held, the new tokens' included
  const int32_t *table;   // [B, max_pages]
  int B, max_pages, n_pages, page_shift, Hkv, D, n_tokens;
  int32_t *err;
};

struct RotArgs {
  RotTable t;
  Rows q, k, v, qo, ko;   // k and v go to the pages where pv.k is set
  int Hq, Hk, Hv, D, n_tokens;
  const int32_t *pos;     // [n_axes, n_tokens]; null: positions in the sequence
  PagedView pv;
};
cudaError_t launch_rotary(const RotArgs &a, int dtype, cudaStream_t st);

// Units of the few-token form whose tiles lie in several CTAs' runs.
constexpr int kRowsMaxCtas = 320;
struct RowsSplit {
  int32_t first, last;    // the CTAs where it starts and ends
  int32_t q0, p_base, head, rows;
};
struct RowsList {         // n and done are zero between calls
  int32_t n;
  uint32_t done;
  RowsSplit unit[kRowsMaxCtas];
};

// Jobs of the tensor-core form whose tiles lie in several CTAs' runs, likewise.
constexpr int kTcMaxCtas = 160;
struct TcSplit {
  int32_t first, last, q0, n, p0, tok0, h;
};
struct TcList {
  int32_t n;
  uint32_t done;
  TcSplit unit[kTcMaxCtas];
};

// Attention of packed queries over pages (pv.k set) or over packed keys and
// values (k, v), causal, each query seeing at most `window` positions.
struct AttnArgs {
  PagedView pv;
  Rows q, k, v;
  void *out;              // [n_tokens, Hq, D]
  int out_sector;         // on 32 bytes
  int Hq, G, window, max_new;
  int hc, rows, whole;    // few-token form: KV heads of a unit, its rows at most, units never cut
  int part_shift, pt_shift;  // positions of one copy, of a tile (log2)
  float sig_log2;
  // the pages' tensor maps (host memory, 128 bytes each): keys in boxes of 64
  // channels; keys and values in whole rows of rows_heads() KV heads, and of one
  const void *mk, *wk, *wv, *ok, *ov;
  float *part;            // partial results
  RowsList *list;
  TcList *tc_list;
  int runs;               // tensor-core form: equal runs of tiles
  int sms, device;
  int give_up;            // a CTA's copying warp gives up before its first tile
};
cudaError_t make_pages_map(void *out, bool bf, void *pool, int D, int page, int Hkv, int n_pages, int heads);
cudaError_t launch_attn_rows(const AttnArgs &a, int dtype, cudaStream_t st);
cudaError_t launch_attn_tc(const AttnArgs &a, int dtype, cudaStream_t st);
// CTAs that a split launch may use at most, and the partial slots of each
constexpr int kRowsPerUnit = 16, kRowsMaxHeads = 4;
// KV heads of a unit: as many as make a copy 64 rows of one page
constexpr int rows_heads(int page, int Hkv) {
  int hc = 1;
  while (hc < kRowsMaxHeads && 2 * hc * page <= 64 && Hkv % (2 * hc) == 0) hc *= 2;
  return hc;
}
// floats of one partial: rows of D sums, then maxima, then totals
__host__ __device__ constexpr int rows_part(int D) { return kRowsPerUnit * (D + 2); }

}  // namespace kvk
