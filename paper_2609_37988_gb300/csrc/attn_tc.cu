// attn_tc.cu -- causal attention of many packed queries on the 5th-generation
// tensor cores: whole prompts over their own keys and values, and chunks of new
// tokens over a paged cache.  Bound: the tensor pipe.
//
// Rows: token i of a sequence and head h of a KV head's group G are row
// i G + h; a query tile is the rows of P = 128 / G whole tokens (at most 128
// rows, TMEM lane = row), a job two such tiles of one (sequence, KV head).  Per
// 128 positions of keys and values, for either tile: S = Q K^T (fp32 in TMEM),
// then x = sigma log2(e) s; each row keeps a reference m that moves only when
// a score rises more than 8 above it (then O and the row's sum are rescaled in
// place; 6 for f16, whose weights are kept 2^8 larger so that small ones stay
// normal); P = 2^(x - m) in the stored type overwrites S, and O += P V with P
// the A operand from TMEM.  The two tiles take turns: while one's products run,
// the other's softmax does.
//
// One persistent CTA per SM, 12 warps: two softmax warpgroups (a thread: a
// row; they also write the tile's result), one that issues all products,
// one warp that schedules jobs and issues the TMA copies (query tiles; a ring
// of key and value tiles), two that look through the values of tiles which some
// row does not see in full: weight 0 times a value that is not finite would be
// NaN, so those enter as zeros, and a row that sees one gets NaN in that
// channel when it is written.
//
// Jobs in order of the positions that they see, the most first (with the order
// of their distance from their own sequence's end, prompts of 560 to 9000 tokens
// took 528 us, with this one 473), dealt to the CTAs back and forth.  (More than
// 128 sequences go one behind another: there are jobs enough to even out.)
// Chunks over pages that would fill a last round of jobs badly go in equal runs of
// tiles instead, one per CTA: jobs that a run cuts leave their pieces (result, reference and sum of each
// row) in the workspace, and a second kernel joins them.
//
// Measured: four prompts of 8192 tokens, 40 / 8 heads of 128, bf16: 1.82-1.92 ms,
// 1430-1520 TFLOP/s at the power limit (1.69 GHz), 1570 in a burst; a chunk of
// 2048 tokens over 4 x 32768 positions 3.4-3.7 ms.  The tensor pipe is active 70 %
// of the cycles: a pair of tiles takes about 2450 of them for 2048 of products.
#include <cuda.h>
#include <limits.h>
#include <math.h>
#include <string.h>

#include <cmath>
#include <type_traits>

#include <algorithm>

#include "common.cuh"
#include "kernels.h"
#include "serve.h"
#include "umma.cuh"

namespace kvk {
namespace {

constexpr int kTcT = 128;                 // positions per tile, rows per query tile
constexpr int kTcThreads = 384;
constexpr int kBox = 128 * 128;           // 64 channels x 128 rows
constexpr int kErrTimeout = 8, kErrCount = 4, kErrPage = 32;  // KVK_DEVERR_*
constexpr uint32_t kAll = 0xffffffffu;
constexpr uint32_t kWaits = 1u << 20;     // polls of up to 2 us each

struct TcArgs {
  CUtensorMap mq, mk, mv;
  AttnArgs a;
  int P;                                  // tokens of a query tile
};

struct Job {
  int b, h, q0, n;      // sequence, KV head, its first token in the batch, its tokens
  int p0, tok0;         // position of its token 0, the job's first token
  int lo, nt;           // position of tile 0, tiles
  int js[2], je[2];     // tiles that either query tile sees: [js, je)
  int first, low;       // tiles in [low, first] positions are seen by every row
  int two, bad;         // second query tile; values that are not finite
  int slot;             // where a piece of a job goes; -1: a whole job
};

// floats of a piece's query tile: D / 4 x 128 rows x 4 results, then references
// and sums
constexpr int tc_part(int D) { return kTcT * (D + 2); }
constexpr int kTcMinShare = 4;  // tiles of a run at least
constexpr int kTcOrdered = 128;  // sequences whose jobs are put in order

template <int D>
struct Smem {
  static constexpr int kTile = D / 64 * kBox;          // a query, key or value tile
  static constexpr int kStages = D == 128 ? 5 : 8;
  static constexpr int kQ = 0, kRing = 2 * kTile, kBar = kRing + kStages * kTile;
  static constexpr int kBars = 3 * kStages + 17;
  static constexpr int kJob = kBar + 8 * kBars;        // two jobs
  static constexpr int kWords = kJob + 2 * (int)sizeof(Job);
  static constexpr int kTotal = kWords + 16;
  static constexpr int kBytes = kTotal + 1024;         // + alignment of the base
};
static_assert(Smem<128>::kBytes <= 232448 && Smem<64>::kBytes <= 232448, "shared memory");
static_assert(Smem<64>::kBytes > 116 * 1024, "one CTA (holding all TMEM columns) per SM");

// 32 columns of this warp's lanes, not waited for
__device__ __forceinline__ void tmem_ld32_nw(uint32_t taddr, float *v) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int j = 0; j < 32; ++j) v[j] = __uint_as_float(r[j]);
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// Sets the top bit of a half where w's half is not finite: an exponent of all
// ones carries out of its field.
template <bool BF16>
__device__ __forceinline__ uint32_t carries(uint32_t w) {
  return BF16 ? (w & 0x7F807F80u) + 0x00800080u : (w & 0x7C007C00u) + 0x04000400u;
}
template <bool BF16>
__device__ __forceinline__ uint32_t pair_scrubbed(uint32_t w) {
  constexpr uint32_t m = BF16 ? 0x7F80u : 0x7C00u;
  if ((w & m) == m) w &= 0xFFFF0000u;
  if ((w >> 16 & m) == m) w &= 0xFFFFu;
  return w;
}

// Tokens of sequence b, its first one in the batch.
__device__ __forceinline__ int seq_tokens(const PagedView &v, int b, int &q0) {
  q0 = min(max(v.cu[b], 0), v.n_tokens);
  return min(max(v.cu[b + 1], q0), v.n_tokens) - q0;
}

template <int D, bool BF16, bool PAGED>
__global__ void __launch_bounds__(kTcThreads, 1) attn_tc_kernel(const __grid_constant__ TcArgs t) {
  using SM = Smem<D>;
  constexpr int NS = SM::kStages;
  extern __shared__ uint8_t tc_raw[];
  uint8_t *sm = tc_raw + ((1024u - (smem_u32(tc_raw) & 1023u)) & 1023u);
  uint64_t *bar = reinterpret_cast<uint64_t *>(sm + SM::kBar);
  // ring: full[NS] a tile landed, free[NS] its products done and the looking
  // warps past it, vclean[NS] a partly seen value tile looked through (the
  // looking warps pass every tile, so that no wait falls two phases behind, and
  // a stage is not used again before its vclean was awaited).  qfull / qfree
  // the job's query tiles; jfull[2] / jfree[2] the job's description (11
  // readers); per query tile: sfull scores done, pfull[2] either half of the
  // weights written (a warp each), odone value products done, ofree the result
  // read.
  uint64_t *full = bar, *free_ = bar + NS, *qfull = bar + 2 * NS, *qfree = qfull + 1, *jfull = qfree + 1, *jfree = jfull + 2,
           *sfull = jfree + 2, *pfull = sfull + 2, *odone = pfull + 4, *ofree = odone + 2, *vclean = ofree + 2,
           *drain = vclean + NS;
  Job *jobs = reinterpret_cast<Job *>(sm + SM::kJob);
  uint32_t *tbase = reinterpret_cast<uint32_t *>(sm + SM::kWords);
  volatile int *abort_flag = reinterpret_cast<volatile int *>(sm + SM::kWords + 4);
  const AttnArgs &a = t.a;
  const PagedView &pv = a.pv;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int P = t.P, G = a.G;

  if (tid == 0) {
    for (int i = 0; i < SM::kBars; ++i) {
      uint64_t *b = bar + i;
      const int n = b >= jfree && b < jfree + 2 ? 11
                    : (b >= pfull && b < pfull + 4) || (b >= ofree && b < ofree + 2) ? 4
                    : b >= vclean && b < vclean + NS ? 2
                    : b >= free_ && b < free_ + NS   ? 3
                                                     : 1;
      mbar_init(b, n);
    }
    *abort_flag = 0;
    fence_mbar_init();
  }
  if (warp == 9 && lane == 0) {
    prefetch_tensor_map(&t.mq);
    prefetch_tensor_map(&t.mk);
    prefetch_tensor_map(&t.mv);
  }
  if (warp == 8) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tbase)), "n"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tbase;
  const uint32_t tS = tmem, tO = tmem + 256;  // scores 2 x 128 columns, results 2 x D
  pdl_wait();

  auto wait = [&](uint64_t *b, uint32_t parity) {
    if (mbar_wait_or_abort(b, parity, kWaits, abort_flag)) return true;
    *abort_flag = 1;
    return false;
  };

  if (warp == 9) {
    // -- schedule and copies ---------------------------------------------------
    int s = 0;          // ring place and its round's parity
    uint32_t ph = 0;
    int loads = 0;      // query loads so far
    int k = 0;          // jobs handed out
    // lane 0 waits, the warp goes on together
    auto wait0 = [&](uint64_t *b, uint32_t parity) {
      int ok = 1;
      if (lane == 0) ok = wait(b, parity);
      return __shfl_sync(kAll, ok, 0) != 0;
    };
    constexpr int NB = D / 64;
    // describes block `blk` of sequence b (2 P tokens), KV head h
    auto describe = [&](int b, int h, int blk, int q0, int n) {
      Job j = {};
      j.b = b;
      j.h = h;
      j.q0 = q0;
      j.n = n;
      j.slot = -1;
      int len = n;
      if (PAGED) {
        len = max(pv.lens[b], 0);
        const int64_t cap = (int64_t)pv.max_pages << pv.page_shift;
        if (len > cap || n > a.max_new) {
          if (lane == 0) set_err(pv.err, kErrCount);
          len = (int)min((int64_t)len, cap);
        }
      }
      j.p0 = len - n;
      j.tok0 = blk * 2 * P;
      j.two = j.tok0 + P < n;
      j.lo = max(0, j.p0 + j.tok0 - a.window + 1) / kTcT * kTcT;
      int last = 0;
      for (int i = 0; i < 1 + j.two; ++i) {
        const int f = j.p0 + j.tok0 + i * P, l = j.p0 + min(n, j.tok0 + (i + 1) * P) - 1;
        if (l >= 0) {
          j.js[i] = (max(0, f - a.window + 1) - j.lo) / kTcT;
          j.je[i] = (l - j.lo) / kTcT + 1;
        }
        last = l;
      }
      j.nt = max(j.je[0], j.je[1]);
      j.first = j.p0 + j.tok0;
      j.low = last - a.window + 1;
      return j;
    };
    // hands a job out and copies its tiles
    auto emit = [&](const Job &j) {
      const int slot = k & 1;
      if (k >= 2 && !wait0(&jfree[slot], (k / 2 - 1) & 1)) return false;
      ++k;
      if (lane == 0) {
        jobs[slot] = j;
        mbar_arrive(&jfull[slot]);
      }
      __syncwarp();
      if (j.b < 0 || j.nt == 0) return true;
      if (loads > 0 && !wait0(qfree, (loads - 1) & 1)) return false;
      ++loads;
      if (lane == 0) mbar_expect_tx(qfull, (1 + j.two) * NB * G * P * 128);
      __syncwarp();
      if (lane < (1 + j.two) * NB) {
        const int i = lane / NB, half = lane % NB;
        tma_load_3d(sm + SM::kQ + i * SM::kTile + half * kBox, &t.mq, 64 * half, j.h * G, j.q0 + j.tok0 + i * P, qfull);
      }
      // (asked once a job: a limit from the arguments in every wait cost 4 %)
      if (a.give_up) {
        if (lane == 0) *abort_flag = 1;
        return false;
      }
      // page of this lane's part of a tile, one tile ahead
      const int shift = PAGED ? min(pv.page_shift, 6) : 7, parts = kTcT >> shift;
      const int part = lane / NB, half = lane % NB;
      auto page_of = [&](int jt) {
        const int pos = j.lo + jt * kTcT + (part << shift);
        // what no query sees reads as zeros, whatever its entry says
        if (part >= parts || pos >= j.p0 + j.n || pos + (1 << shift) <= j.first - a.window + 1) return pv.n_pages;
        const int page = pv.table[(int64_t)j.b * pv.max_pages + (pos >> pv.page_shift)];
        if ((unsigned)page < (unsigned)pv.n_pages) return page;
        set_err(pv.err, kErrPage);
        return pv.n_pages;
      };
      int page = PAGED ? page_of(0) : 0;
      for (int jt = 0; jt < j.nt; ++jt) {
        const int page_next = PAGED && jt + 1 < j.nt ? page_of(jt + 1) : 0;
#pragma unroll
        for (int kv = 0; kv < 2; ++kv) {
          if (!wait0(&free_[s], ph ^ 1)) return false;
          if (lane == 0) mbar_expect_tx(&full[s], SM::kTile);
          __syncwarp();
          uint8_t *dst = sm + SM::kRing + s * SM::kTile;
          const CUtensorMap *m = kv ? &t.mv : &t.mk;
          if (PAGED && kv) {
            // values of a page in one copy, its halves one behind the other
            const int pg = __shfl_sync(kAll, page, lane < parts ? lane * NB : 0);
            if (lane < parts)
              tma_load_5d(dst + (lane << shift) * (2 * D), m, 0, (lane << shift) & ((1 << pv.page_shift) - 1), 0, j.h, pg, &full[s]);
          } else if (lane < parts * NB) {
            // keys: their halves apart, 128 rows each, as the products' rows have to be
            if (PAGED)
              tma_load_4d(dst + half * kBox + (part << shift) * 128, m, 64 * half, (part << shift) & ((1 << pv.page_shift) - 1),
                          j.h, page, &full[s]);
            else
              tma_load_3d(dst + half * kBox, m, 64 * half, j.q0 + j.lo + jt * kTcT, j.h, &full[s]);
          }
          if (++s == NS) s = 0, ph ^= 1;
        }
        page = page_next;
      }
      return true;
    };
    auto read_blocks = [&](int b) {
      int q0;
      return b < pv.B ? (seq_tokens(pv, b, q0) + 2 * P - 1) / (2 * P) : 0;
    };
    Job end = {};
    end.b = -1;
    bool ok = true;
    if (PAGED && a.runs) {
      // tiles of one KV head of a sequence (describe()'s nt of every block), a
      // job of none counting as one
      auto head_tiles = [&](int b) {
        int q0, sum = 0;
        const int n = seq_tokens(pv, b, q0);
        if (n == 0) return 0;
        const int p0 = (int)min((int64_t)max(pv.lens[b], 0), (int64_t)pv.max_pages << pv.page_shift) - n;
        for (int tok = 0; tok < n; tok += 2 * P) {
          const int last = p0 + min(n, tok + 2 * P) - 1, lo = max(0, p0 + tok - a.window + 1) / kTcT;
          sum += last < 0 ? 1 : last / kTcT - lo + 1;
        }
        return sum;
      };
      const int tiles0 = lane < pv.B ? head_tiles(lane) : 0;
      int64_t total = (int64_t)pv.Hkv * tiles0;
      for (int b = lane + 32; b < pv.B; b += 32) total += (int64_t)pv.Hkv * head_tiles(b);
      for (int o = 16; o; o >>= 1) total += __shfl_xor_sync(kAll, total, o);
      const int64_t share = max(div_pos(total + gridDim.x - 1, gridDim.x), (int64_t)kTcMinShare);
      const int64_t w0 = share * blockIdx.x;
      int left = (int)max(min(share, total - w0), (int64_t)0);
      if (left > 0) {
        // the sequence, head, block and tile where the run starts
        int b = 0, h = 0, blk = 0, t = 0;
        int64_t off = 0;
        int per = 0;  // of the sequence found
        for (int b0 = 0; b0 < pv.B; b0 += 32) {
          const int tl = b0 == 0 ? tiles0 : b0 + lane < pv.B ? head_tiles(b0 + lane) : 0;
          const int64_t x = (int64_t)pv.Hkv * tl;
          int64_t sum = x;
          for (int o = 1; o < 32; o <<= 1) {
            const int64_t y = __shfl_up_sync(kAll, sum, o);
            if (lane >= o) sum += y;
          }
          const uint32_t past = __ballot_sync(kAll, off + sum > w0);
          if (past) {
            const int f = __ffs(past) - 1;
            b = b0 + f;
            per = __shfl_sync(kAll, tl, f);
            off = w0 - (off + __shfl_sync(kAll, sum - x, f));
            break;
          }
          off += __shfl_sync(kAll, sum, 31);
        }
        ok = per > 0;  // a sequence was found: the lengths are as they were
        int q0, n = seq_tokens(pv, b, q0);
        h = ok ? (int)div_pos(off, per) : 0;
        t = (int)(off - (int64_t)h * per);
        Job j = describe(b, h, 0, q0, n);
        while (ok && t >= max(1, j.nt) && (blk + 1) * 2 * P < n) {
          t -= max(1, j.nt);
          j = describe(b, h, ++blk, q0, n);
        }
        ok = ok && t < max(1, j.nt);
        while (ok) {
          const int nt = max(1, j.nt), t1 = min(nt, t + left);
          if (t > 0 || t1 < nt) {  // a piece: tiles [t, t1)
            j.slot = 2 * blockIdx.x + (t == 0);
            if (t == 0 && lane == 0) {
              const int at = atomicAdd(&a.tc_list->n, 1);  // a CTA adds one at most
              const int before = (int)(share - left);
              if ((unsigned)at < (unsigned)kTcMaxCtas)
                a.tc_list->unit[at] =
                    TcSplit{(int)blockIdx.x, min((int)blockIdx.x + (before + nt - 1) / (int)share, (int)gridDim.x - 1),
                            j.q0, j.n, j.p0, j.tok0, j.h};
            }
            j.lo += t * kTcT;
            for (int i = 0; i < 2; ++i) {
              j.js[i] = max(j.js[i] - t, 0);
              j.je[i] = min(j.je[i], t1) - t;
              if (j.js[i] >= j.je[i]) j.js[i] = j.je[i] = 0;
            }
            j.nt = t1 - t;
          }
          ok = emit(j);
          left -= t1 - t;
          if (left == 0) break;
          t = 0;
          if (++blk >= (n + 2 * P - 1) / (2 * P)) {
            blk = 0;
            if (++h >= pv.Hkv) {
              h = 0;
              do {
                n = ++b < pv.B ? seq_tokens(pv, b, q0) : -1;
              } while (n == 0);
              if (n < 0) break;
            }
          }
          j = describe(b, h, blk, q0, n);
        }
      }
    } else if (pv.B <= kTcOrdered) {
      // The batch's sequences, four a lane: a sequence's blocks are [from, to), in
      // blocks from its position 0 on, so that a block's number says how many
      // positions its rows see.
      int from[4], to[4], total = 0, top = 0, low = INT_MAX;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int b = lane + 32 * i, n = read_blocks(b);
        from[i] = 0;
        if (PAGED && n > 0) {
          int q0;
          const int held = (int)min((int64_t)max(pv.lens[b], 0), (int64_t)pv.max_pages << pv.page_shift);
          from[i] = max(held - seq_tokens(pv, b, q0), 0) / (2 * P);
        }
        to[i] = from[i] + n;
        total += n;
        if (n > 0) top = max(top, to[i]), low = min(low, from[i]);
      }
      total = (int)__reduce_add_sync(kAll, (unsigned)total);
      top = (int)__reduce_max_sync(kAll, (unsigned)top);
      low = (int)__reduce_min_sync(kAll, (unsigned)low);
      // jobs with one of the `d` largest numbers
      auto upto = [&](int d) {
        unsigned sum = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum += min(max(to[i] - (top - d), 0), to[i] - from[i]);
        return (int)__reduce_add_sync(kAll, sum);
      };
      const int n_jobs = total * pv.Hkv, step = gridDim.x;
      for (int i = 0; ok; ++i) {
        const int idx = i * step + (i & 1 ? step - 1 - (int)blockIdx.x : (int)blockIdx.x);
        if (idx >= n_jobs) break;
        const int r = idx / pv.Hkv;
        int d0 = 0, d1 = top - low, f0 = 0;  // upto(d0) <= r < upto(d1)
        while (d1 - d0 > 1) {
          const int mid = d0 + (d1 - d0) / 2, f = upto(mid);
          if (f <= r)
            d0 = mid, f0 = f;
          else
            d1 = mid;
        }
        const int number = top - 1 - d0;
        int rem = r - f0, b = 0, blk = 0;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          const uint32_t in = __ballot_sync(kAll, from[c] <= number && number < to[c]);
          const int m = __popc(in);
          if (rem >= 0 && rem < m) {
            const int f = (int)__fns(in, 0, rem + 1);
            b = 32 * c + f;
            blk = number - __shfl_sync(kAll, from[c], f);
          }
          rem -= m;
        }
        int q0;
        const int n = seq_tokens(pv, b, q0);
        ok = emit(describe(b, idx - r * pv.Hkv, blk, q0, n));
      }
    } else {
      // sequence by sequence, the search going on from where the last job was
      int b0 = 0, before = 0, x = 0, sum = 0;  // blocks of this lane's sequence; up to and with it
      auto chunk = [&]() {
        x = sum = read_blocks(b0 + lane);
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int y = __shfl_up_sync(kAll, sum, o);
          if (lane >= o) sum += y;
        }
      };
      chunk();
      for (int64_t idx = blockIdx.x; ok; idx += gridDim.x) {
        const int r = (int)(idx / pv.Hkv);
        while (b0 < pv.B && before + __shfl_sync(kAll, sum, 31) <= r) {
          before += __shfl_sync(kAll, sum, 31);
          b0 += 32;
          chunk();
        }
        if (b0 >= pv.B) break;
        const int f = __ffs(__ballot_sync(kAll, before + sum > r)) - 1;
        const int from_end = r - (before + __shfl_sync(kAll, sum - x, f));
        int q0;
        const int n = seq_tokens(pv, b0 + f, q0);
        ok = emit(describe(b0 + f, (int)(idx - (int64_t)r * pv.Hkv), (n + 2 * P - 1) / (2 * P) - 1 - from_end, q0, n));
      }
    }
    if (!__any_sync(kAll, *abort_flag)) emit(end);
    // the copies in flight land before the CTA ends, whoever waits for them: another
    // warp may give up after this one is through
    if (lane == 0) {
      if (loads > 0) mbar_wait(qfull, (loads - 1) & 1, kWaits);
      for (int i = 0; i < NS; ++i) {
        if (ph == 0 && i >= s) break;  // never used
        mbar_wait(&full[i], i < s ? ph : ph ^ 1, kWaits);
      }
    }
  } else if (warp == 8) {
    // -- products.  The whole warp runs the loop and one lane issues: operands
    // then stay in uniform registers, and a product is issued in fewer cycles
    // than it takes (a lone lane needed as many, so that every wait between
    // products left the pipe idle).
    constexpr uint32_t id_s = BF16 ? umma_idesc(128, kTcT, false, false) : umma_idesc_f16(128, kTcT, false, false);
    constexpr uint32_t id_v = BF16 ? umma_idesc(128, D, false, true) : umma_idesc_f16(128, D, false, true);
    constexpr uint32_t hi = umma_desc_hi_sw128(1024);
    const uint32_t ring = smem_u32(sm + SM::kRing), q_at = umma_desc_lo(smem_u32(sm + SM::kQ), 16);
    const bool leader = elect_one();
    // values: rows of a copy (log2), and where 16 of them start (in 16 bytes)
    const int v_shift = PAGED ? min(pv.page_shift, 6) : 7;
    auto v_step = [&](int x) {
      if (!PAGED) return 128 * x;
      return ((x >> (v_shift - 4)) << v_shift) * (2 * D / 16) + (x & ((1 << (v_shift - 4)) - 1)) * 128;
    };
    int s = 0;
    uint32_t ph = 0, loads = 0, cleans = 0;   // cleans: parity of either stage's vclean
    uint32_t tiles[2] = {0, 0}, done[2] = {0, 0};  // of either query tile: parity of its tiles, jobs with any
    auto scores = [&](auto I, int at) {
      constexpr int i = decltype(I)::value;
      const uint32_t q = q_at + i * (SM::kTile >> 4), kk = umma_desc_lo(ring + at * SM::kTile, 16);
#pragma unroll
      for (int b = 0; b < D / 64; ++b)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          umma_f16_ss_if(leader, tS + 128 * i, q + b * (kBox >> 4) + 2 * x, kk + b * (kBox >> 4) + 2 * x, hi, id_s, b + x > 0);
      umma_commit_if(leader, &sfull[i]);
    };
    auto values = [&](auto I, int at, bool acc) {
      constexpr int i = decltype(I)::value;
      const uint32_t vv = umma_desc_lo(ring + at * SM::kTile, 128 << v_shift);
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        if (!wait(&pfull[2 * i + hf], tiles[i])) return false;
        tc_fence_after();
#pragma unroll
        for (int x = 4 * hf; x < 4 * hf + 4; ++x)
          umma_f16_ts_if(leader, tO + D * i, tS + 128 * i + 8 * x, vv + v_step(x), hi, id_v, acc || x > 0);
      }
      umma_commit_if(leader, &odone[i]);
      tiles[i] ^= 1;
      return true;
    };
    constexpr std::integral_constant<int, 0> i0;
    constexpr std::integral_constant<int, 1> i1;
    bool ok = true;
    for (int k = 0; ok; ++k) {
      const int slot = k & 1;
      if (!wait(&jfull[slot], (k / 2) & 1)) break;
      const Job *j = &jobs[slot];
      const int jb = j->b, nt = j->nt, lo = j->lo, first = j->first, low = j->low;
      const int js0 = j->js[0], je0 = j->je[0], js1 = j->js[1], je1 = j->je[1];
      __syncwarp();
      if (lane == 0) mbar_arrive(&jfree[slot]);
      if (jb < 0) break;
      if (nt == 0) continue;
      if (!wait(qfull, loads)) break;
      loads ^= 1;
      // K of tile 0
      if (!wait(&full[s], ph)) break;
      tc_fence_after();
      if (js0 == 0 && je0 > 0) scores(i0, s);
      if (js1 == 0 && je1 > 0) scores(i1, s);
      umma_commit_if(leader, &free_[s]);
      if (nt == 1) umma_commit_if(leader, qfree);
      if (++s == NS) s = 0, ph ^= 1;
      // tiles [steady, steady_end): seen in full by every row, as a tile of both
      // query tiles that is neither one's first, the next one theirs too and not
      // the job's last: nothing to ask between the products
      const int steady = max(max(js0, js1) + 1, (low - lo + kTcT - 1) / kTcT);
      const int steady_end = min(min(min(je0, je1), nt - 1) - 1, first - lo >= kTcT - 1 ? (first - lo + 1) / kTcT : 0);
      for (int jt = 0; jt < nt; ++jt) {
        // V of this tile at s, K of the next at sk
        int sk = s + 1;
        uint32_t phk = ph;
        if (sk == NS) sk = 0, phk ^= 1;
        if (jt >= steady && jt < steady_end) {
          if (!(ok = wait(&full[s], ph))) break;
          if (!(ok = values(i0, s, true))) break;
          if (!(ok = wait(&full[sk], phk))) break;
          tc_fence_after();
          scores(i0, sk);
          if (!(ok = values(i1, s, true))) break;
          umma_commit_if(leader, &free_[s]);
          s = sk + 1, ph = phk;
          if (s == NS) s = 0, ph ^= 1;
          scores(i1, sk);
          umma_commit_if(leader, &free_[sk]);
          continue;
        }
        const bool more = jt + 1 < nt;
        const int t0 = lo + jt * kTcT;
        if (!(ok = wait(&full[s], ph))) break;
        if (t0 + kTcT - 1 > first || t0 < low) {
          if (!(ok = wait(&vclean[s], cleans >> s & 1))) break;
          cleans ^= 1u << s;
        }
        // either tile's values, then its next scores: a tile's softmax runs
        // beside the other's products
        auto half = [&](auto I, int js, int je) {
          constexpr int i = decltype(I)::value;
          if (jt >= js && jt < je) {
            if (jt == js) {  // the tile's last result has been read
              if (done[i] > 0 && !wait(&ofree[i], (done[i] - 1) & 1)) return false;
              ++done[i];
            }
            if (!values(I, s, jt > js)) return false;
          }
          if (more && i == 0) {
            if (!wait(&full[sk], phk)) return false;
            tc_fence_after();
          }
          if (jt + 1 >= js && jt + 1 < je) scores(I, sk);
          return true;
        };
        if (!(ok = half(i0, js0, je0))) break;
        if (!(ok = half(i1, js1, je1))) break;
        umma_commit_if(leader, &free_[s]);
        if (more) {
          umma_commit_if(leader, &free_[sk]);
          if (jt + 2 == nt) umma_commit_if(leader, qfree);
        }
        s = sk, ph = phk;
        if (more && ++s == NS) s = 0, ph ^= 1;
      }
    }
    // the products in flight end before TMEM is freed, likewise
    umma_commit_if(leader, drain);
    mbar_wait(drain, 0, kWaits);
    __syncwarp();
  } else if (warp >= 10) {
    // -- values of partly seen tiles ----------------------------------------------
    int s = 0;
    uint32_t ph = 0;
    for (int k = 0;; ++k) {
      const int slot = k & 1;
      if (!wait(&jfull[slot], (k / 2) & 1)) break;
      Job &js = jobs[slot];
      const int nt = js.b < 0 ? -1 : js.nt, lo = js.lo, first = js.first, low = js.low;
      bool ok = true;
      auto pass = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(&free_[s]);
        if (++s == NS) s = 0, ph ^= 1;
      };
      for (int jt = 0; jt < nt; ++jt) {
        if (!(ok = wait(&full[s], ph))) break;  // keys
        pass();
        if (!(ok = wait(&full[s], ph))) break;
        const int t0 = lo + jt * kTcT;
        if (t0 + kTcT - 1 > first || t0 < low) {
          uint4 *x = reinterpret_cast<uint4 *>(sm + SM::kRing + s * SM::kTile) + (warp - 10) * (SM::kTile / 32);
          bool fine = true;
#pragma unroll 1
          for (int e = lane; e < SM::kTile / 32; e += 32 * 8) {
            uint4 u[8];
            uint32_t any = 0;
#pragma unroll
            for (int y = 0; y < 8; ++y) u[y] = x[e + 32 * y];
#pragma unroll
            for (int y = 0; y < 8; ++y)
              any |= carries<BF16>(u[y].x) | carries<BF16>(u[y].y) | carries<BF16>(u[y].z) | carries<BF16>(u[y].w);
            if (any & 0x80008000u) {
              fine = false;
#pragma unroll 1
              for (int y = 0; y < 8; ++y) {
                const uint4 w = x[e + 32 * y];
                x[e + 32 * y] = make_uint4(pair_scrubbed<BF16>(w.x), pair_scrubbed<BF16>(w.y), pair_scrubbed<BF16>(w.z),
                                           pair_scrubbed<BF16>(w.w));
              }
            }
          }
          if (!fine) {
            js.bad = 1;
            fence_proxy_async();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&vclean[s]);
        }
        pass();
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&jfree[slot]);
      if (nt < 0 || !ok) break;
    }
  } else {
    // -- softmax and results: a thread per row of query tile i -----------------------
    const int i = warp >> 2;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tS + 128 * i + lane_off, to = tO + D * i + lane_off;
    const int row = (warp & 3) * 32 + lane, my_tok = row / G;
    const float sg = a.sig_log2;
    // f16 weights are 2^8 larger, and the reference moves sooner: at most 2^14
    constexpr float kShift = BF16 ? 0.f : 8.f, kLag = BF16 ? 8.f : 6.f;
    int tiles = 0;  // of this query tile so far
    auto arrive = [&](uint64_t *b) {
      __syncwarp();
      if (lane == 0) mbar_arrive(b);
    };
    for (int k = 0;; ++k) {
      const int slot = k & 1;
      if (!wait(&jfull[slot], (k / 2) & 1)) break;
      const Job &j = jobs[slot];
      const int jb = j.b;
      bool ok = true;
      if (jb >= 0 && (i == 0 || j.two)) {
        const int tok = j.tok0 + i * P + my_tok;
        const bool real = my_tok < P && tok < j.n;
        const int pos = j.p0 + tok;
        // rows that are nobody's are never masked: their own affair
        const int lim = real ? pos : 1 << 30, low = real ? pos - a.window + 1 : -(1 << 30);
        const int js = j.js[i], je = j.je[i], lo = j.lo;
        float m = -INFINITY, l = 0.f;
        for (int jt = js; jt < je; ++jt) {
          if (!(ok = wait(&sfull[i], tiles & 1))) break;
          tc_fence_after();
          float x[128];
#pragma unroll
          for (int c = 0; c < 4; ++c) tmem_ld32_nw(ts + 32 * c, x + 32 * c);
          tmem_wait_ld();
          const int t0 = lo + jt * kTcT;
          const int past = lim - t0, before = low - t0;  // columns [before, past] are seen
          if (__any_sync(kAll, past < kTcT - 1 || before > 0)) {
#pragma unroll
            for (int c = 0; c < 128; c += 32) {
              const int to = min(max(past + 1 - c, 0), 32), from = min(max(before - c, 0), 32);
              const uint32_t seen = (uint32_t)(((1ull << to) - 1) & ~((1ull << from) - 1));
#pragma unroll
              for (int y = 0; y < 32; ++y) x[c + y] = seen >> y & 1 ? x[c + y] : -INFINITY;
            }
          }
          float mx[4] = {x[0], x[1], x[2], x[3]};
#pragma unroll
          for (int c = 4; c < 128; c += 8)
#pragma unroll
            for (int y = 0; y < 4; ++y)
              mx[y] = c + 4 + y < 128 ? fmaxf(fmaxf(mx[y], x[c + y]), x[c + 4 + y]) : fmaxf(mx[y], x[c + y]);
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * sg;
          const bool move = real && top > m + kLag;
          if (__any_sync(kAll, move)) {
            const float mn = move ? top : m;
            const float f = m == -INFINITY ? 0.f : fast_exp2(m - mn);
            m = mn;
            l *= f;
            if (jt > js) {  // the products before this tile's have to be in
              if (!(ok = wait(&odone[i], (tiles - 1) & 1))) break;
              tc_fence_after();
#pragma unroll 1
              for (int c = 0; c < D; c += 16) {
                float o[16];
                tmem_ld16(to + c, o);
#pragma unroll
                for (int y = 0; y < 16; ++y) o[y] *= f;
                tmem_st16(to + c, o);
              }
            }
          }
          const float ref = (m == -INFINITY ? 0.f : m) - kShift;
          const uint64_t sg2 = pair_f32(sg, sg), ref2 = pair_f32(-ref, -ref);
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            uint32_t w[8];
#pragma unroll
            for (int y = 0; y < 8; ++y) {
              float u, v;
              unpair_f32(fma_f32x2(pair_f32(x[16 * c + 2 * y], x[16 * c + 2 * y + 1]), sg2, ref2), u, v);
              u = x[16 * c + 2 * y] = fast_exp2(u);
              v = x[16 * c + 2 * y + 1] = fast_exp2(v);
              w[y] = pack2<BF16>(u, v);
            }
            tmem_st8_nw(ts + 8 * c, w);
            if (c == 3 || c == 7) {
              tmem_wait_st();
              tc_fence_before();
              arrive(&pfull[2 * i + (c >> 2)]);
            }
          }
          // the row's sum, of the weights before their rounding: behind the hand-over,
          // which the products wait for
          uint64_t sum[2] = {0, 0};
#pragma unroll
          for (int c = 0; c < 128; c += 4) {
            sum[0] = add_f32x2(sum[0], pair_f32(x[c], x[c + 1]));
            sum[1] = add_f32x2(sum[1], pair_f32(x[c + 2], x[c + 3]));
          }
          float u, v;
          unpair_f32(add_f32x2(sum[0], sum[1]), u, v);
          l += u + v;
          ++tiles;
        }
        if (!ok) break;
        const float inv = real && pos >= 0 ? 1.f / l : 0.f;
        uint32_t nan[D / 32] = {};  // channels of which the row sees a value that is not finite
        if (je > js) {
          if (!wait(&odone[i], (tiles - 1) & 1)) break;
          tc_fence_after();
          if (j.bad && real) {
            const int first = j.first, lowest = j.low;
            for (int jt = js; jt < je; ++jt) {
              const int t0 = lo + jt * kTcT;
              if (t0 + kTcT - 1 <= first && t0 >= lowest) continue;
              for (int p = max(t0, low); p <= min(t0 + kTcT - 1, lim); ++p) {
                const uint8_t *src;
                if (PAGED) {
                  const int page = pv.table[(int64_t)jb * pv.max_pages + (p >> pv.page_shift)];
                  if ((unsigned)page >= (unsigned)pv.n_pages) continue;
                  src = pv.v + (((((int64_t)page * pv.Hkv + j.h) << pv.page_shift) + (p & ((1 << pv.page_shift) - 1))) * D) * 2;
                } else {
                  src = a.v.p + 2 * ((int64_t)(j.q0 + p) * a.v.ts + j.h * a.v.hs);
                }
#pragma unroll
                for (int c = 0; c < D / 8; ++c) {
                  const uint4 u = reinterpret_cast<const uint4 *>(src)[c];
                  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
                  for (int y = 0; y < 4; ++y) {
                    constexpr uint32_t mk = BF16 ? 0x7F80u : 0x7C00u;
                    const int ch = 8 * c + 2 * y;
                    nan[ch >> 5] |= ((w[y] & mk) == mk ? 1u : 0u) << (ch & 31);
                    nan[ch >> 5] |= ((w[y] >> 16 & mk) == mk ? 2u : 0u) << (ch & 31);
                  }
                }
              }
            }
          }
          __syncwarp();
        }
        const int slot_out = j.slot;
        float *part = a.part + ((int64_t)2 * slot_out + i) * tc_part(D) + 4 * row;
        if (slot_out >= 0) {  // the piece's reference and sum
          part[kTcT * D - 3 * row] = m == -INFINITY ? m : m - kShift;
          part[kTcT * (D + 1) - 3 * row] = l;
        }
        uint8_t *dst = static_cast<uint8_t *>(a.out) + 2 * ((int64_t)(j.q0 + tok) * a.Hq + j.h * G + (row - my_tok * G)) * D;
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
          float o[32];
          if (je > js) {
            tmem_ld32(to + 32 * c, o);
          } else {
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = 0.f;
          }
          if (nan[c]) {
#pragma unroll
            for (int y = 0; y < 32; ++y) o[y] = nan[c] >> y & 1 ? NAN : o[y];
          }
          if (slot_out >= 0 && real) {
#pragma unroll
            for (int y = 0; y < 8; ++y)
              __stcg(reinterpret_cast<float4 *>(part + (8 * c + y) * (4 * kTcT)),
                     make_float4(o[4 * y], o[4 * y + 1], o[4 * y + 2], o[4 * y + 3]));
          } else if (real) {
            // rows before position 0 have zeros here, and 0 as their factor
            uint32_t w[16];
#pragma unroll
            for (int y = 0; y < 16; ++y) w[y] = pack2<BF16>(o[2 * y] * inv, o[2 * y + 1] * inv);
#pragma unroll
            for (int y = 0; y < 4; y += 2) {
              const uint4 u = make_uint4(w[4 * y], w[4 * y + 1], w[4 * y + 2], w[4 * y + 3]);
              const uint4 v = make_uint4(w[4 * y + 4], w[4 * y + 5], w[4 * y + 6], w[4 * y + 7]);
              if (a.out_sector) {
                st_sector(dst + 64 * c + 16 * y, u, v);
              } else {
                reinterpret_cast<uint4 *>(dst)[4 * c + y] = u;
                reinterpret_cast<uint4 *>(dst)[4 * c + y + 1] = v;
              }
            }
          }
        }
        if (je > js) {
          tc_fence_before();
          arrive(&ofree[i]);
        }
      }
      arrive(&jfree[slot]);
      if (jb < 0) break;
    }
    __syncwarp();
  }

  if (*abort_flag && lane == 0) set_err(pv.err, kErrTimeout);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 8) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512) : "memory");
  pdl_trigger();
}

// Joins the pieces of the jobs that runs cut: a CTA takes CH channels of a query
// tile, a thread a row and every HALVES-th piece, U pieces' loads in flight; the
// halves meet in shared memory.  The last CTA clears the list for the next call.
// Two forms: 16 channels and 2 pieces at a time where many jobs were cut into a few
// pieces each; 8 channels, two halves and 8 at a time where a few were cut into
// dozens (one sequence of 65000 positions, 37 pieces a job: 55 -> 39 us; 512 new
// tokens of one over 8192, 88 jobs: 68 us, with the other form 80).
template <int D, bool BF16, int CH, int HALVES, int U>
__global__ void __launch_bounds__(HALVES *kTcT) attn_tc_join_kernel(const AttnArgs a, int P) {
  constexpr int C = D / CH;
  __shared__ float s_x[CH + 2][kTcT];
  const int row = threadIdx.x % kTcT, hf = threadIdx.x / kTcT, tok_row = row / a.G;
  pdl_wait();
  const int n = min(*reinterpret_cast<volatile int *>(&a.tc_list->n), kTcMaxCtas) * 2 * C;
  for (int item = blockIdx.x; item < n; item += gridDim.x) {
    const TcSplit u = a.tc_list->unit[item / (2 * C)];
    const int i = item / C & 1, c = item % C;
    const int tok = u.tok0 + i * P + tok_row;
    const bool real = tok_row < P && tok < u.n;
    float M = -INFINITY, L = 0.f, x[CH];
#pragma unroll
    for (int y = 0; y < CH; ++y) x[y] = 0.f;
    auto join = [&](float m, float l, const float *z) {
      if (m == -INFINITY && l == 0.f) return;  // saw nothing
      const float t = fmaxf(M, m), f = M == -INFINITY ? 0.f : fast_exp2(M - t), h = m == -INFINITY ? 0.f : fast_exp2(m - t);
      M = t;
      L = L * f + l * h;
#pragma unroll
      for (int y = 0; y < CH; ++y) x[y] = x[y] * f + z[y] * h;
    };
    for (int p0 = u.first + hf; real && p0 <= u.last; p0 += U * HALVES) {
      float pm[U], pl[U], z[U][CH];
#pragma unroll
      for (int k = 0; k < U; ++k) {
        const int p = p0 + k * HALVES;
        const bool in = p <= u.last;
        const float *part = a.part + (int64_t)(2 * (2 * p + (p == u.first)) + i) * tc_part(D);
        pm[k] = in ? __ldcg(part + kTcT * D + row) : -INFINITY;
        pl[k] = in ? __ldcg(part + kTcT * (D + 1) + row) : 0.f;
#pragma unroll
        for (int y = 0; y < CH / 4; ++y)
          *reinterpret_cast<float4 *>(&z[k][4 * y]) =
              in ? __ldcg(reinterpret_cast<const float4 *>(part + (CH / 4 * c + y) * (4 * kTcT) + 4 * row))
                 : make_float4(0.f, 0.f, 0.f, 0.f);
      }
#pragma unroll
      for (int k = 0; k < U; ++k) join(pm[k], pl[k], z[k]);
    }
    if constexpr (HALVES == 2) {
      if (hf == 1) {
#pragma unroll
        for (int y = 0; y < CH; ++y) s_x[y][row] = x[y];
        s_x[CH][row] = M;
        s_x[CH + 1][row] = L;
      }
      __syncthreads();
      if (hf == 0) {
        float z[CH];
#pragma unroll
        for (int y = 0; y < CH; ++y) z[y] = s_x[y][row];
        join(s_x[CH][row], s_x[CH + 1][row], z);
      }
      __syncthreads();
    }
    if (hf == 0 && real) {
      // a row before position 0 sees nothing and gives zeros
      const bool sees = u.p0 + tok >= 0;
      const float inv = sees ? 1.f / L : 0.f;
      uint32_t w[CH / 2];
#pragma unroll
      for (int y = 0; y < CH / 2; ++y) w[y] = sees ? pack2<BF16>(x[2 * y] * inv, x[2 * y + 1] * inv) : 0u;
      uint4 *dst = reinterpret_cast<uint4 *>(static_cast<uint8_t *>(a.out) +
                                             2 * (((int64_t)(u.q0 + tok) * a.Hq + u.h * a.G + (row - tok_row * a.G)) * D + CH * c));
#pragma unroll
      for (int y = 0; y < CH / 8; ++y) dst[y] = make_uint4(w[4 * y], w[4 * y + 1], w[4 * y + 2], w[4 * y + 3]);
    }
  }
  pdl_trigger();
  __syncthreads();
  if (threadIdx.x == 0) {
    __threadfence();
    if (atomicInc(&a.tc_list->done, gridDim.x - 1) == gridDim.x - 1) a.tc_list->n = 0;
  }
}

// [rows, heads, D] of 16-bit values as boxes of 64 channels: `inner` and
// `outer` dimensions with their strides in elements.
cudaError_t rows_map(CUtensorMap *m, bool bf, void *p, int D, int64_t n1, int64_t s1, int64_t n2, int64_t s2, int b1, int b2) {
  const uint64_t dims[3] = {(uint64_t)D, (uint64_t)n1, (uint64_t)n2};
  const uint64_t strides[2] = {(uint64_t)s1 * 2, (uint64_t)s2 * 2};
  const uint32_t box[3] = {64, (uint32_t)b1, (uint32_t)b2}, one[3] = {1, 1, 1};
  return encode_tensor_map_tiled(m, bf ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, p, dims,
                                 strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                                 CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
}
template <int D, bool BF16, bool PAGED>
cudaError_t launch_t(const AttnArgs &a, cudaStream_t st) {
  cudaError_t e = allow_smem<&attn_tc_kernel<D, BF16, PAGED>>(Smem<D>::kBytes, a.device);
  if (e != cudaSuccess) return e;
  TcArgs t;
  t.a = a;
  t.P = kTcT / a.G;
  t.a.out_sector = (reinterpret_cast<uintptr_t>(a.out) & 31u) == 0;
  const int N = a.pv.n_tokens;
  e = rows_map(&t.mq, BF16, a.q.p, D, a.Hq, a.q.hs, N, a.q.ts, a.G, t.P);
  if (PAGED) {
    memcpy(&t.mk, a.mk, sizeof t.mk);
    memcpy(&t.mv, a.ov, sizeof t.mv);
  } else {
    if (e == cudaSuccess) e = rows_map(&t.mk, BF16, a.k.p, D, N, a.k.ts, a.pv.Hkv, a.k.hs, kTcT, 1);
    if (e == cudaSuccess) e = rows_map(&t.mv, BF16, a.v.p, D, N, a.v.ts, a.pv.Hkv, a.v.hs, kTcT, 1);
  }
  if (e != cudaSuccess) return e;
  // at most so many jobs: every sequence's last one may be a partial one
  const int64_t jobs = (int64_t)a.pv.Hkv * (N / (2 * t.P) + std::min(a.pv.B, N));
  // Runs where whole jobs would leave SMs idle for longer than the pieces take on
  // their way through memory: the part of the last round of jobs that is not
  // filled, against 5 tiles for a second kernel and up to 18 for the pieces of as
  // many cut jobs (tiles by the table's width or the window, sequences taken to be
  // of equal shares).  Measured (us, whole / runs, 40 / 8 heads of 128; new tokens
  // over positions): 400 over 2000 27.7 / 32.2, over 4000 47 / 39; 1000 over 2000
  // 35 / 48, over 4000 73 / 66; 512 over 8192 86 / 70; 600 over 600 15 / 28; 4 x 33
  // over 2000 27 / 18; 32 x 4 over 1900 54 / 55, over 8192 182 / 174.  Up to four
  // rounds: of 2048 tokens over 32768, 1 (2.2 rounds) 971 / 916, 4 (8.6) 3473 / 3894.
  const int64_t seqs = std::min(a.pv.B, N), share = (N + seqs - 1) / seqs, blocks = (share + 2 * t.P - 1) / (2 * t.P);
  const int64_t seen = std::min((int64_t)a.pv.max_pages << a.pv.page_shift, (int64_t)a.window + 2 * t.P + kTcT);
  const double full = (double)a.pv.Hkv * seqs * blocks, waves = full / a.sms;
  const double idle = (std::ceil(waves) - waves) * (double)((seen + kTcT - 1) / kTcT);
  const double rows = (double)std::min<int64_t>(2 * t.P, share) * a.G / (2 * kTcT);
  t.a.runs = PAGED && waves < 4 && idle > 5 + 0.12 * std::min(full, (double)a.sms) * rows;
  if (!t.a.runs)
    return launch_pdl(attn_tc_kernel<D, BF16, PAGED>, dim3((int)std::min<int64_t>(a.sms, jobs)), dim3(kTcThreads),
                      Smem<D>::kBytes, st, t);
  const int grid = std::min(a.sms, kTcMaxCtas);
  e = launch_pdl(attn_tc_kernel<D, BF16, PAGED>, dim3(grid), dim3(kTcThreads), Smem<D>::kBytes, st, t);
  if (e != cudaSuccess) return e;
  // a CTA's run cuts off the start of one job at most
  const int64_t cut = std::min<int64_t>(jobs, grid);
  if (cut * 2 * (D / 8) <= 4 * a.sms)
    return launch_pdl(attn_tc_join_kernel<D, BF16, 8, 2, 8>, dim3((int)cut * 2 * (D / 8)), dim3(2 * kTcT), 0, st, t.a, t.P);
  return launch_pdl(attn_tc_join_kernel<D, BF16, 16, 1, 2>, dim3((int)std::min<int64_t>(cut * 2 * (D / 16), 8 * a.sms)), dim3(kTcT),
                    0, st, t.a, t.P);
}

template <int D, bool BF16>
cudaError_t launch_src(const AttnArgs &a, cudaStream_t st) {
  return a.pv.k ? launch_t<D, BF16, true>(a, st) : launch_t<D, BF16, false>(a, st);
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
