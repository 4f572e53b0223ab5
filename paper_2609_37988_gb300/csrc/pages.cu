// pages.cu -- copying, forking and compacting the pages of a paged cache.
//
// A page's holders are counted on the device (refs); one that nobody holds is free.
// All choices go by the counts as they were before the call and by the order of
// pages and rows, so that they do not depend on how the GPU runs them.
//
// Bound: the pages that are copied (HBM, read and written once), for calls that
// copy few the launches.  Measured: 250 us for a copy of 805 MB and 145 us for
// compacting 470 MB, 0.95 of the bandwidth; a fork of 96 beams over 28 layers 14 us and
// one of 256 served rows, one layer, 10 us, most of it lookups that wait for one another.
// A fork's CTAs beside a row's own are launched whether it copies or not: 256 rows that
// copy nothing take 7 us with one layer of 8 KV heads of 128, with 48 layers in pages of
// 16 17 (8 bits) and 29 (16 bits), in pages of 128 103 and 202.
#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"

namespace kvk {
namespace {

constexpr int kThreads = 256;
constexpr int kPer = kPageChunk / kThreads;
constexpr int kErrCapacity = 2, kErrCount = 4, kErrPage = 32;  // KVK_DEVERR_*
constexpr uint32_t kAll = 0xffffffffu;

// Sum of x over the CTA's threads before this one; `total`: over all of them.
// Every thread calls it.
__device__ int scan_cta(int x, int &total) {
  __shared__ int s_sum[kThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int sum = x;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int y = __shfl_up_sync(kAll, sum, o);
    if (lane >= o) sum += y;
  }
  __syncthreads();  // the last call's readers are through
  if (lane == 31) s_sum[warp] = sum;
  __syncthreads();
  int before = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    before += w < warp ? s_sum[w] : 0;
    total += s_sum[w];
  }
  return before + sum - x;
}

__device__ __forceinline__ int pages_of(const PagesArgs &a, int len) {
  return (int)(((int64_t)len + (1 << a.page_shift) - 1) >> a.page_shift);
}
// Positions of a given row, within its table.
__device__ __forceinline__ int held(const PagesArgs &a, int b) {
  return (int)min((int64_t)max(a.lens[b], 0), (int64_t)a.max_pages << a.page_shift);
}

constexpr int kPiece = 8192;  // bytes that a CTA copies at a time, 32 a thread

// Pieces [first, end) of page s, of the pools of all layers one behind another, to
// page d; with piece 0 of a pool its powers.
template <bool CODED>
__device__ void copy_page(const CopyArgs &a, int s, int d, int first, int end) {
  const int tid = threadIdx.x, pieces = (int)((a.bytes + kPiece - 1) / kPiece);
  if (s == d) return;
  constexpr int U = 4;
  for (int w0 = first; w0 < end; w0 += U) {
    uint4 u[U], v[U];
    uint8_t *to[U];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int w = w0 + i, pool = w / pieces, piece = w - pool * pieces, l = pool >> 1;
      const int64_t off = (int64_t)piece * kPiece + 32 * tid;
      to[i] = nullptr;
      if (w >= end || off >= a.bytes) continue;
      uint8_t *x = pool & 1 ? a.v[l] : a.k[l];
      const uint4 *from = reinterpret_cast<const uint4 *>(x + s * a.bytes + off);
      u[i] = from[0], v[i] = from[1];
      to[i] = x + d * a.bytes + off;
    }
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (to[i]) st_sector(to[i], u[i], v[i]);
    if (CODED) {
#pragma unroll 1
      for (int w = w0; w < min(w0 + U, end); ++w) {
        const int pool = w / pieces;
        if (w != pool * pieces) continue;
        int8_t *e = pool & 1 ? a.ve[pool >> 1] : a.ke[pool >> 1];
        for (int h = tid; h < a.Hkv; h += kThreads) e[(int64_t)d * a.Hkv + h] = e[(int64_t)s * a.Hkv + h];
      }
    }
  }
}

// A CTA's part of a list of pages to copy: entry by entry, so many pieces at a time.
template <bool CODED>
__device__ void copy_list(const CopyArgs &a, int n, int share) {
  const int pieces = (int)((a.bytes + kPiece - 1) / kPiece) * 2 * a.layers, shares = (pieces + share - 1) / share;
  for (int64_t w = blockIdx.x; w < (int64_t)shares * n; w += gridDim.x) {
    const int i = (int)(w / shares), part = (int)(w - (int64_t)i * shares);
    const int s = a.src[i], d = a.dst[i];
    if (s == -1 || d == -1) continue;
    if ((unsigned)s >= (unsigned)a.n_pages || (unsigned)d >= (unsigned)a.n_pages) {
      if (threadIdx.x == 0) set_err(a.err, kErrPage);
      continue;
    }
    copy_page<CODED>(a, s, d, part * share, min((part + 1) * share, pieces));
  }
}

template <bool CODED>
__global__ void __launch_bounds__(kThreads) copy_pages_kernel(const __grid_constant__ CopyArgs a, int share) {
  pdl_wait();
  copy_list<CODED>(a, a.n_dev ? *a.n_dev : a.n, share);
  pdl_trigger();
}

// This thread's pages of chunk c and how many of them are used; the chunk's holders
// are kept as they are before the call (refs_out may be refs).
__device__ int count_chunk(const PagesArgs &a, int c, int32_t *keep) {
  int used = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = c * kPageChunk + i * kThreads + threadIdx.x;
    if (p >= a.n_pages) continue;
    const int r = a.refs[p];
    used += r > 0;
    a.before[p] = r;
    if (keep) keep[p] = r;
  }
  return used;
}

// Row i of a fork from its parent's: what it keeps of it, ends with.
__device__ void fork_row(const PagesArgs &a, int j, int &parent, int &old, int &want, bool &open) {
  parent = a.parents[j];
  if (parent < -1 || parent >= a.B) parent = -1;
  const int len = parent < 0 ? 0 : held(a, parent);
  const int64_t cap = (int64_t)a.width << a.page_shift;
  const int after = (int)min((int64_t)(a.after ? max(a.after[j], 0) : len), cap);
  const int kept = min(len, after);
  old = pages_of(a, kept);
  want = pages_of(a, after);
  open = (kept & ((1 << a.page_shift) - 1)) != 0;
}

// Pages counted, a CTA per chunk; then rows, a warp each.
__global__ void __launch_bounds__(kThreads) fork_count_kernel(const PagesArgs a, int chunks) {
  const int lane = threadIdx.x & 31;
  pdl_wait();
  if ((int)blockIdx.x < chunks) {
    int total;
    scan_cta(count_chunk(a, blockIdx.x, a.refs_out), total);
    if (threadIdx.x == 0)
      a.chunk[blockIdx.x] = min(kPageChunk, a.n_pages - (int)blockIdx.x * kPageChunk) - total;  // free
    pdl_trigger();
    return;
  }
  const int i = ((int)blockIdx.x - chunks) * (kThreads / 32) + (threadIdx.x >> 5);
  if (i < a.R) {
    ForkRow r;
    bool open;
    fork_row(a, i, r.parent, r.old, r.want, open);
    r.copy = -1;
    if (open) {
      // A page that is not full will be written to: it stays with the first row that
      // has it so if nobody else holds it and no row has it full.
      bool shared = false;
      const int page = a.table[(int64_t)r.parent * a.max_pages + r.old - 1];
#pragma unroll 4
      for (int j = lane; j < a.R; j += 32) {
        if (a.parents[j] != r.parent || j == i) continue;
        int p, o, w;
        bool op;
        fork_row(a, j, p, o, w, op);
        shared = shared || o > r.old || (o == r.old && (!op || j < i));
      }
      shared = __any_sync(kAll, shared);
      if ((unsigned)page < (unsigned)a.n_pages && (shared || a.refs[page] != 1)) r.copy = page;
    }
    if (lane == 0) {
      a.rows[i] = r;
      const int parent = a.parents[i];
      const int64_t cap = (int64_t)a.width << a.page_shift;
      const int64_t after = a.after ? a.after[i] : r.parent < 0 ? 0 : held(a, r.parent);
      if (parent < -1 || parent >= a.B || after < 0 || after > cap) set_err(a.err, kErrCount);
    }
  }
  pdl_trigger();
}

// Free pages number base .. base + need - 1 to `give(k, page)`; how many there were.
// Every thread of the CTA calls it.
template <typename F>
__device__ int take_free(const PagesArgs &a, int base, int need, F give) {
  __shared__ int s_chunk, s_before;
  const int tid = threadIdx.x;
  const int chunks = (a.n_pages + kPageChunk - 1) / kPageChunk;
  // the chunk with free page number `base`
  if (tid == 0) s_chunk = chunks, s_before = base;
  for (int c0 = 0, before = 0, total; c0 < chunks && before <= base; c0 += kThreads, before += total) {
    const int x = c0 + tid < chunks ? a.chunk[c0 + tid] : 0, at = before + scan_cta(x, total);
    if (at <= base && base < at + x) s_chunk = c0 + tid, s_before = at;
  }
  __syncthreads();
  // 16 pages a thread at a time: a row that takes hundreds goes over many chunks
  constexpr int kWide = 16;
  int before = s_before;
  for (int p0 = s_chunk * kPageChunk; p0 < a.n_pages && before < base + need; p0 += kWide * kThreads) {
    const int at = p0 + kWide * tid;
    int4 x[kWide / 4];
    if (at + kWide <= a.n_pages) {
#pragma unroll
      for (int i = 0; i < kWide / 4; ++i) x[i] = reinterpret_cast<const int4 *>(a.before + at)[i];
    } else {
#pragma unroll
      for (int i = 0; i < kWide / 4; ++i) {
        int y[4];
#pragma unroll
        for (int z = 0; z < 4; ++z) y[z] = at + 4 * i + z < a.n_pages ? a.before[at + 4 * i + z] : 1;
        x[i] = make_int4(y[0], y[1], y[2], y[3]);
      }
    }
    uint32_t free = 0;
#pragma unroll
    for (int i = 0; i < kWide / 4; ++i)
      free |= ((x[i].x <= 0) | (x[i].y <= 0) << 1 | (x[i].z <= 0) << 2 | (x[i].w <= 0) << 3) << (4 * i);
    int total, k = before + scan_cta(__popc(free), total) - base;
    for (; free; free &= free - 1, ++k)
      if (k >= 0 && k < need) give(k, at + __ffs(free) - 1);
    before += total;
  }
  return min(max(before - base, 0), need);
}

// A CTA per given row, which lets go of its pages, and one per new row, which takes its
// own.  Those beside a new row's (gridDim.y) copy a share of its copied page, as it does.
template <bool CODED>
__global__ void __launch_bounds__(kThreads) fork_rows_kernel(const PagesArgs a, const __grid_constant__ CopyArgs copy, int share) {
  __shared__ int s_to;
  const int tid = threadIdx.x, r = (int)blockIdx.x - a.B;
  const bool main = blockIdx.y == 0;
  pdl_wait();
  if (tid == 0) s_to = -1;
  if (main && r < 0) {
    const int r = blockIdx.x;
    const int n = pages_of(a, held(a, r));
    if (tid == 0 && (int64_t)a.lens[r] > (int64_t)a.max_pages << a.page_shift) set_err(a.err, kErrCount);
    for (int j = tid; j < n; j += kThreads) {
      const int page = a.table[(int64_t)r * a.max_pages + j];
      if ((unsigned)page >= (unsigned)a.n_pages) {
        set_err(a.err, kErrPage);
      } else if (a.before[page] <= 0) {
        set_err(a.err, kErrCount);
      } else {
        atomicSub(&a.refs_out[page], 1);
      }
    }
  }
  if (r >= 0) {
    const ForkRow row = a.rows[r];
    const int copied = row.copy >= 0, fresh_from = row.old - copied, need = main ? row.want - fresh_from : copied;
    int32_t *out = a.table_out + (int64_t)r * a.width;
    // free pages that the rows before take
    int mine = 0;
    if (need > 0) {  // (the same for the CTA)
#pragma unroll 4
      for (int j = tid; j < r; j += kThreads) {
        const ForkRow x = a.rows[j];
        mine += x.want - x.old + (x.copy >= 0);
      }
    }
    if (main) {
      for (int j = tid; j < a.width; j += kThreads) {
        if (j < fresh_from) {
          const int page = a.table[(int64_t)row.parent * a.max_pages + j];
          if ((unsigned)page < (unsigned)a.n_pages) atomicAdd(&a.refs_out[page], 1);
          out[j] = page;
        } else if (j >= row.want) {
          out[j] = -1;
        }
      }
    }
    if (need > 0) {
      int base;
      scan_cta(mine, base);
      const int got = take_free(a, base, need, [&](int k, int p) {
        if (main) {
          out[fresh_from + k] = p;
          a.refs_out[p] = 1;
        }
        if (copied && k == 0) s_to = p;
      });
      if (main) {  // those that no page is left for
        for (int j = fresh_from + got + tid; j < row.want; j += kThreads) out[j] = -1;
        if (got < need && tid == 0) set_err(a.err, kErrCapacity);
      }
      __syncthreads();
    }
    const int to = s_to;
    if (main && tid == 0) {  // for the layers of other launches
      a.src[r] = row.copy;
      a.dst[r] = to;
    }
    if (copied && to >= 0) {
      const int pieces = (int)((copy.bytes + kPiece - 1) / kPiece) * 2 * copy.layers;
      const int first = blockIdx.y * share;
      if (first < pieces) copy_page<CODED>(copy, row.copy, to, first, min(first + share, pieces));
    }
  }
  pdl_trigger();
}

__global__ void __launch_bounds__(kThreads) compact_count_kernel(const PagesArgs a) {
  int total;
  pdl_wait();
  scan_cta(count_chunk(a, blockIdx.x, nullptr), total);
  if (threadIdx.x == 0) a.chunk[blockIdx.x] = total;
  pdl_trigger();
}

// Which page goes where: used page number k at or behind the used count to free
// page number k before it.  COUNTED: by the chunks' counts; otherwise every CTA
// counts all pages, 4 a load, the holders being refs itself.
template <bool COUNTED>
__global__ void __launch_bounds__(kThreads) compact_moves_kernel(const PagesArgs a) {
  const int tid = threadIdx.x, c = blockIdx.x, chunks = gridDim.x;
  int mine = 0, all = 0, before, used, low_before, x;
  pdl_wait();
  if (COUNTED) {
    for (int i = tid; i < chunks; i += kThreads) {
      const int n = a.chunk[i];
      all += n;
      if (i < c) mine += n;
    }
  } else {
#pragma unroll 8
    for (int p = tid; p < a.n_pages; p += kThreads) {
      const int n = a.before[p] > 0;
      all += n;
      if (p < c * kPageChunk) mine += n;
    }
  }
  scan_cta(mine, before);
  scan_cta(all, used);
  // used pages before number `used`
  const int edge = COUNTED ? used / kPageChunk : 0;
  int low = 0;
  for (int i = tid; i < edge; i += kThreads) low += a.chunk[i];
#pragma unroll 8
  for (int p = edge * kPageChunk + tid; p < used; p += kThreads) low += a.before[p] > 0;
  scan_cta(low, low_before);
  bool in[kPer];
  int n = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = c * kPageChunk + kPer * tid + i;
    in[i] = p < a.n_pages && a.before[p] > 0;
    n += in[i];
  }
  int k = before + scan_cta(n, x);  // used pages before this one
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int p = c * kPageChunk + kPer * tid + i;
    if (p >= a.n_pages) break;
    if (p < used) {
      a.where[p] = in[i] ? p : -1;
      if (in[i])
        a.refs_out[p] = a.before[p];
      else
        a.dst[p - k] = p;
    } else {
      a.refs_out[p] = 0;
      if (in[i])
        a.src[k - low_before] = p;
      else
        a.where[p] = -1;
    }
    k += in[i];
  }
  if (c == 0 && tid == 0) {
    *a.n_moved = used - low_before;
    if (a.used) *a.used = used;
  }
  pdl_trigger();
}

// The moved pages' numbers and holders, the table, the pages.
template <bool CODED>
__global__ void __launch_bounds__(kThreads) compact_apply_kernel(const PagesArgs a, const __grid_constant__ CopyArgs copy, int share) {
  pdl_wait();
  const int n = *a.n_moved;
  const int64_t at = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = at; i < n; i += step) {
    const int s = a.src[i], d = a.dst[i];
    a.where[s] = d;
    a.refs_out[d] = a.before[s];
  }
  for (int64_t e = at; e < (int64_t)a.B * a.width; e += step) {
    const int b = (int)(e / a.width), j = (int)(e - (int64_t)b * a.width);
    int to = -1;
    if (j == 0 && (int64_t)a.lens[b] > (int64_t)a.max_pages << a.page_shift) set_err(a.err, kErrCount);
    if (j < pages_of(a, held(a, b))) {
      const int page = a.table[(int64_t)b * a.max_pages + j];
      if ((unsigned)page >= (unsigned)a.n_pages) {
        set_err(a.err, kErrPage);
      } else if (a.before[page] <= 0) {
        set_err(a.err, kErrCount);
      } else {
        // a page that moves stands in the list, which is in order
        int lo = 0, hi = n;
        while (lo < hi) {
          const int mid = (lo + hi) >> 1;
          if (a.src[mid] < page)
            lo = mid + 1;
          else
            hi = mid;
        }
        to = lo < n && a.src[lo] == page ? a.dst[lo] : page;
      }
    }
    a.table_out[e] = to;
  }
  copy_list<CODED>(copy, n, share);
  pdl_trigger();
}

}  // namespace

namespace {
int64_t pieces_of(const CopyArgs &c) { return (c.bytes + kPiece - 1) / kPiece * 2 * c.layers; }
// Pieces that a CTA takes of a page at once: 64 KB, fewer where that would leave SMs
// without work.
int share_of(const CopyArgs &c, int64_t pages, int sms) {
  int share = 8;
  while (share > 1 && pages * ((pieces_of(c) + share - 1) / share) < 4 * sms) share /= 2;
  return share;
}
}  // namespace

cudaError_t launch_copy_pages(const CopyArgs &a, bool coded, int sms, cudaStream_t st) {
  const int share = share_of(a, a.n, sms);
  const int64_t items = (pieces_of(a) + share - 1) / share * a.n;
  if (items == 0) return cudaSuccess;
  const dim3 grid((unsigned)std::min<int64_t>(items, (int64_t)8 * sms));
  return launch_pdl(coded ? copy_pages_kernel<true> : copy_pages_kernel<false>, grid, dim3(kThreads), 0, st, a, share);
}

cudaError_t launch_fork(const PagesArgs &a, const CopyArgs &copy, bool coded, int sms, cudaStream_t st) {
  const int chunks = (a.n_pages + kPageChunk - 1) / kPageChunk, rows = a.B + a.R;
  cudaError_t e = launch_pdl(fork_count_kernel, dim3(chunks + (a.R + kThreads / 32 - 1) / (kThreads / 32)), dim3(kThreads), 0, st, a,
                             chunks);
  if (e != cudaSuccess || rows == 0) return e;
  // CTAs beside a row's own: 64 KB of its copied page each
  const int share = share_of(copy, std::max(a.R, 1), sms);
  const int64_t beside = a.R ? std::min<int64_t>((pieces_of(copy) + share - 1) / share, 65535) : 1;
  const int each = (int)((pieces_of(copy) + beside - 1) / beside);
  return launch_pdl(coded ? fork_rows_kernel<true> : fork_rows_kernel<false>, dim3(rows, (unsigned)beside), dim3(kThreads), 0, st, a,
                    copy, each);
}

// Pools up to this size are counted by every CTA for itself, which saves a launch
// (77 pages 5.4 us for 8.0); not where the counts change in place meanwhile.
constexpr int kCountAll = 32768;

cudaError_t launch_compact(const PagesArgs &in, const CopyArgs &copy, bool coded, int sms, cudaStream_t st) {
  PagesArgs a = in;
  const int chunks = (a.n_pages + kPageChunk - 1) / kPageChunk;
  const bool apart = a.refs_out + a.n_pages <= a.refs || a.refs + a.n_pages <= a.refs_out;
  cudaError_t e = cudaSuccess;
  if (apart && a.n_pages <= kCountAll) {
    a.before = const_cast<int32_t *>(a.refs);  // (only read from here on)
    e = launch_pdl(compact_moves_kernel<false>, dim3(chunks), dim3(kThreads), 0, st, a);
  } else {
    e = launch_pdl(compact_count_kernel, dim3(chunks), dim3(kThreads), 0, st, a);
    if (e == cudaSuccess) e = launch_pdl(compact_moves_kernel<true>, dim3(chunks), dim3(kThreads), 0, st, a);
  }
  if (e != cudaSuccess) return e;
  const int share = share_of(copy, a.n_pages / 4, sms);
  const int64_t work = std::max(((int64_t)a.B * a.width + kThreads - 1) / kThreads,
                                (int64_t)(a.n_pages / 2) * ((pieces_of(copy) + share - 1) / share));
  return launch_pdl(coded ? compact_apply_kernel<true> : compact_apply_kernel<false>,
                    dim3((unsigned)std::max<int64_t>(1, std::min<int64_t>(work, (int64_t)8 * sms))), dim3(kThreads), 0, st, a, copy, share);
}

}  // namespace kvk
