// serve_host.cu -- host side of the serving entry points of include/kvk.h:
// rotary positions, the paged cache and attention over packed prompts.
// Checks arguments, lays out the workspace and launches on the caller's
// stream; allocates no device memory.
#include <cuda_runtime.h>

#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>
#include <mutex>
#include <new>
#include <vector>

#include "../../include/kvk.h"
#include "kernels.h"
#include "serve.h"

// the thread's last error (kvk_host.cu)
kvk_status kvk_internal_fail(kvk_status s, const char *message);
kvk_status kvk_internal_cuda_error(cudaError_t e, const char *what);

using namespace kvk;

struct kvk_rotary {
  RotTable t;
  int head_dim;
};

constexpr int kMaps = 5;
struct PageMap {
  alignas(64) uint8_t bytes[128];
};

struct kvk_paged {
  kvk_paged_desc d;
  bool coded = false;             // a cache in 8 bits
  std::vector<uint8_t *> k, v;
  std::vector<int8_t *> ke, ve;   // its powers of two
  std::vector<PageMap> maps;  // kMaps tensor maps of a layer's pools, as AttnArgs has them
  uint8_t *ws;
  int device, sms, page_shift;
  std::atomic<int32_t> give_up{0};
  std::atomic<bool> cleared{false};  // the workspace, by kvk_paged_reset
  std::mutex calls;  // an attention's launches follow one another
};

namespace {

kvk_status fail(kvk_status s, const char *fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof buf, fmt, ap);
  va_end(ap);
  return kvk_internal_fail(s, buf);
}

bool aligned(const void *p, int bytes) { return !(reinterpret_cast<uintptr_t>(p) & (uintptr_t)(bytes - 1)); }

// A row view of the caller's as the kernels take it: elements of `elem` bytes,
// rows on `align` bytes.  The stride of a dimension of size one says nothing
// and is replaced.
kvk_status take_rows(const kvk_rows *r, const char *name, int n_tokens, int heads, int D, int elem, int align, Rows &out) {
  if (!r || !r->data) return fail(KVK_ERR_INVALID_ARG, "%s is null", name);
  out.p = static_cast<uint8_t *>(r->data);
  out.hs = heads == 1 ? D : r->head_stride;
  out.ts = n_tokens == 1 ? (int64_t)heads * out.hs : r->token_stride;
  if (out.hs < D || out.ts < D)
    return fail(KVK_ERR_INVALID_ARG, "%s: strides must be at least head_dim (no broadcast rows)", name);
  if (out.hs >= (1LL << 38) || out.ts >= (1LL << 38)) return fail(KVK_ERR_INVALID_ARG, "%s: stride too large", name);
  if (!aligned(out.p, align) || out.hs * elem % align || out.ts * elem % align)
    return fail(KVK_ERR_INVALID_ARG, "%s: rows must start on %d bytes", name, align);
  return KVK_OK;
}

// (a subnormal scale would be zero on the way, and zero times a masked score NaN)
bool scale_ok(float s) { return std::isfinite(s * 1.4426950408889634f) && std::isnormal(s) && s > 0.f; }

// heads and widths that the attention kernels take
kvk_status check_heads(int Hq, int Hkv, int D, int dtype) {
  if (Hkv <= 0 || Hq <= 0 || Hq % Hkv)
    return fail(KVK_ERR_INVALID_ARG, "n_q_heads must be a positive multiple of n_kv_heads");
  if (D <= 0) return fail(KVK_ERR_INVALID_ARG, "head_dim must be positive");
  if (D != 64 && D != 128) return fail(KVK_ERR_UNSUPPORTED, "head_dim %d (supported: 64 and 128)", D);
  if (Hq / Hkv > 64) return fail(KVK_ERR_UNSUPPORTED, "more than 64 query heads per KV head");
  if (Hkv > 65535) return fail(KVK_ERR_UNSUPPORTED, "more than 65535 KV heads");
  if (dtype != KVK_DTYPE_BF16 && dtype != KVK_DTYPE_F16)
    return fail(KVK_ERR_INVALID_ARG, "dtype must be BF16 or F16");
  return KVK_OK;
}

struct PagedWs {
  size_t err, list, tc_list, part, pages, total;
};
constexpr size_t kWsAlign = 256;
size_t up(size_t x) { return (x + kWsAlign - 1) / kWsAlign * kWsAlign; }
// what the operators on pages keep: holders, chunks' counts, rows, two lists
size_t chunks_of(int n_pages) { return ((size_t)n_pages + kPageChunk - 1) / kPageChunk; }
size_t list_of(int n_pages) { return (size_t)n_pages / 2 + 1 > (size_t)kForkRows ? (size_t)n_pages / 2 + 1 : (size_t)kForkRows; }
size_t pages_ws(int n_pages) {
  return up(4 * (size_t)n_pages) + up(4 * chunks_of(n_pages)) + up(sizeof(ForkRow) * kForkRows) + 2 * up(4 * list_of(n_pages)) + kWsAlign;
}
PagedWs paged_ws(int D, int n_pages) {
  PagedWs w;
  w.err = 0;
  w.list = 256;
  w.tc_list = w.list + ((sizeof(RowsList) + 255) & ~(size_t)255);
  w.part = w.tc_list + ((sizeof(TcList) + 255) & ~(size_t)255);
  // two pieces per CTA of either form
  const size_t rows = (size_t)2 * kRowsMaxCtas * kRowsMaxHeads * rows_part(D), tc = (size_t)2 * kTcMaxCtas * 2 * 128 * (D + 2);
  w.pages = up(w.part + (rows > tc ? rows : tc) * sizeof(float));
  w.total = w.pages + pages_ws(n_pages);
  return w;
}

kvk_status check_paged_desc(const kvk_paged_desc *d) {
  if (!d) return fail(KVK_ERR_INVALID_ARG, "null descriptor");
  if (d->n_layers <= 0 || d->n_pages <= 0) return fail(KVK_ERR_INVALID_ARG, "layers and pages must be positive");
  if (d->page_size != 16 && d->page_size != 32 && d->page_size != 64 && d->page_size != 128)
    return fail(KVK_ERR_UNSUPPORTED, "page_size %d (supported: 16, 32, 64 and 128)", d->page_size);
  return check_heads(d->n_q_heads, d->n_kv_heads, d->head_dim, d->dtype);
}

size_t pool_bytes(const kvk_paged_desc *d, bool coded) {
  return (size_t)d->n_pages * d->n_kv_heads * d->page_size * d->head_dim * (coded ? 1 : 2);
}
// powers of two that a cache in 8 bits uses: 2^e times any e4m3 code is a number of
// the dtype (f16: its subnormals' step is 2^-24; bf16: a margin to its ends)
int exp_lo(int dtype) { return dtype == KVK_DTYPE_BF16 ? -110 : -15; }
int exp_hi(int dtype) { return dtype == KVK_DTYPE_BF16 ? 119 : 7; }

kvk_status check_device(const kvk_paged *p) {
  int dev = -1;
  const cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "querying the current device");
  if (dev != p->device)
    return fail(KVK_ERR_INVALID_ARG, "current device %d is not the paged cache's device %d", dev, p->device);
  return KVK_OK;
}

kvk_status check_call(const kvk_paged *p, int layer, const kvk_paged_batch *b, bool &empty) {
  if (!p) return fail(KVK_ERR_INVALID_ARG, "null paged cache");
  if (layer < 0 || layer >= p->d.n_layers)
    return fail(KVK_ERR_INVALID_ARG, "layer %d out of range [0, %d)", layer, p->d.n_layers);
  const kvk_status dev = check_device(p);
  if (dev) return dev;
  if (!b) return fail(KVK_ERR_INVALID_ARG, "null batch");
  if (b->batch < 0 || b->n_tokens < 0 || b->max_pages < 0)
    return fail(KVK_ERR_INVALID_ARG, "batch, n_tokens and max_pages must not be negative");
  if ((int64_t)b->max_pages * p->d.page_size > (1 << 26))
    return fail(KVK_ERR_INVALID_ARG, "max_pages %d: more than 2^26 positions", b->max_pages);
  if ((int64_t)b->n_tokens * p->d.n_q_heads > (1 << 30)) return fail(KVK_ERR_INVALID_ARG, "n_tokens too large");
  empty = b->batch == 0 || b->n_tokens == 0;
  if (empty) return KVK_OK;
  if (!b->cu_new || !b->lengths || (!b->table && b->max_pages))
    return fail(KVK_ERR_INVALID_ARG, "null offsets, lengths or table");
  if (!aligned(b->cu_new, 4) || !aligned(b->lengths, 4) || !aligned(b->table, 4))
    return fail(KVK_ERR_INVALID_ARG, "misaligned offsets, lengths or table");
  return KVK_OK;
}

PagedView view_of(const kvk_paged *p, int layer, const kvk_paged_batch *b) {
  PagedView v;
  v.k = p->k[layer];
  v.v = p->v[layer];
  v.cu = b->cu_new;
  v.lens = b->lengths;
  v.table = b->table;
  v.B = b->batch;
  v.max_pages = b->max_pages;
  v.n_pages = p->d.n_pages;
  v.page_shift = p->page_shift;
  v.Hkv = p->d.n_kv_heads;
  v.D = p->d.head_dim;
  v.n_tokens = b->n_tokens;
  v.err = reinterpret_cast<int32_t *>(p->ws + paged_ws(v.D, p->d.n_pages).err);
  v.ke = p->coded ? p->ke[layer] : nullptr;
  v.ve = p->coded ? p->ve[layer] : nullptr;
  v.e_lo = exp_lo(p->d.dtype);
  v.e_hi = exp_hi(p->d.dtype);
  return v;
}

// The workspace of the operators on pages.
PagesArgs pages_args(const kvk_paged *p) {
  PagesArgs a = {};
  const int n = p->d.n_pages;
  uint8_t *at = p->ws + paged_ws(p->d.head_dim, n).pages;
  auto take = [&](size_t bytes) {
    uint8_t *x = at;
    at += up(bytes);
    return x;
  };
  a.before = reinterpret_cast<int32_t *>(take(4 * (size_t)n));
  a.chunk = reinterpret_cast<int32_t *>(take(4 * chunks_of(n)));
  a.rows = reinterpret_cast<ForkRow *>(take(sizeof(ForkRow) * kForkRows));
  a.src = reinterpret_cast<int32_t *>(take(4 * list_of(n)));
  a.dst = reinterpret_cast<int32_t *>(take(4 * list_of(n)));
  a.n_moved = reinterpret_cast<int32_t *>(take(4));
  a.n_pages = n;
  a.page_shift = p->page_shift;
  a.err = reinterpret_cast<int32_t *>(p->ws + paged_ws(p->d.head_dim, n).err);
  return a;
}

// Layers l0 on, as many as one launch takes.
CopyArgs copy_args(const kvk_paged *p, int l0, const int32_t *src, const int32_t *dst, int n, const int32_t *n_dev) {
  CopyArgs c = {};
  c.layers = p->d.n_layers - l0 < kCopyLayers ? p->d.n_layers - l0 : kCopyLayers;
  for (int l = 0; l < c.layers; ++l) {
    c.k[l] = p->k[l0 + l];
    c.v[l] = p->v[l0 + l];
    if (p->coded) c.ke[l] = p->ke[l0 + l], c.ve[l] = p->ve[l0 + l];
  }
  c.src = src;
  c.dst = dst;
  c.n = n;
  c.n_dev = n_dev;
  c.n_pages = p->d.n_pages;
  c.Hkv = p->d.n_kv_heads;
  c.bytes = (int64_t)p->d.n_kv_heads * p->d.page_size * p->d.head_dim * (p->coded ? 1 : 2);
  c.err = reinterpret_cast<int32_t *>(p->ws + paged_ws(p->d.head_dim, p->d.n_pages).err);
  return c;
}
// Pages of the layers from l0 on, `n` entries at most (n_dev: as many as it says).
cudaError_t copy_layers(const kvk_paged *p, int l0, const int32_t *src, const int32_t *dst, int n, const int32_t *n_dev, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  for (; l0 < p->d.n_layers && e == cudaSuccess; l0 += kCopyLayers)
    e = launch_copy_pages(copy_args(p, l0, src, dst, n, n_dev), p->coded, p->sms, st);
  return e;
}

// A call on pages: the rows that the table has.
kvk_status check_pages(const kvk_paged *p, const int32_t *refs, const int32_t *refs_out, const int32_t *table, const int32_t *lengths,
                       int batch, int max_pages) {
  if (!p) return fail(KVK_ERR_INVALID_ARG, "null paged cache");
  const kvk_status s = check_device(p);
  if (s) return s;
  if (batch < 0 || batch > (1 << 24) || max_pages < 0)
    return fail(KVK_ERR_INVALID_ARG, "batch must be in [0, 2^24], max_pages not negative");
  if ((int64_t)max_pages * p->d.page_size > (1 << 26))
    return fail(KVK_ERR_INVALID_ARG, "max_pages %d: more than 2^26 positions", max_pages);
  if (!refs || !refs_out || (batch && (!lengths || (!table && max_pages))))
    return fail(KVK_ERR_INVALID_ARG, "null holders, lengths or table");
  if (!aligned(refs, 4) || !aligned(refs_out, 4) || !aligned(table, 4) || !aligned(lengths, 4))
    return fail(KVK_ERR_INVALID_ARG, "misaligned holders, lengths or table");
  const int n = p->d.n_pages;
  if (refs_out != refs && refs_out < refs + n && refs < refs_out + n)
    return fail(KVK_ERR_INVALID_ARG, "refs_out may be refs, and may not overlap it otherwise");
  return KVK_OK;
}

// Rows of a KV head up to which the form for few tokens is the faster one (us,
// few / tensor cores, 14B-shaped layer, 16 bits: 4 x 8192 positions, 10 rows 39 / 40, 20
// rows 54 / 40; 1 x 1024, 10 rows 17 / 18).  In 8 bits, where that form ends at 16
// rows: 4 x 8192, 15 rows 34 / 42; 32 x 8192 116 / 167; 1 x 1024 17 / 26; 28 / 4 heads,
// 14 rows, 32 x 8192 69 / 92; 8 / 2 heads of 64, 16 rows, 32 x 8192 36 / 46.
constexpr int kFewRows = 16;
cudaError_t launch_attn(const AttnArgs &a, int dtype, cudaStream_t st) {
  if (a.pv.ke) return (int64_t)a.max_new * a.G <= kFewRows ? launch_attn_codes_rows(a, dtype, st) : launch_attn_tc_codes(a, dtype, st);
  if (a.pv.k && (int64_t)a.max_new * a.G <= kFewRows) return launch_attn_rows(a, dtype, st);
  return launch_attn_tc(a, dtype, st);
}

// The error word of prompts whose caller gives none, one a device.
__device__ int32_t g_prompt_err;
constexpr int kMaxDevices = 64;
std::mutex g_prompt_mu;
int32_t *g_prompt_word[kMaxDevices] = {};
std::atomic<int32_t> g_prompt_give_up{0};

// its address on the current device (looked up once)
cudaError_t prompt_word(int dev, int32_t **word) {
  if (dev < 0 || dev >= kMaxDevices) return cudaErrorInvalidDevice;
  std::lock_guard<std::mutex> lock(g_prompt_mu);
  if (!g_prompt_word[dev]) {
    void *p = nullptr;
    const cudaError_t e = cudaGetSymbolAddress(&p, g_prompt_err);
    if (e != cudaSuccess) return e;
    g_prompt_word[dev] = static_cast<int32_t *>(p);
  }
  *word = g_prompt_word[dev];
  return cudaSuccess;
}

// reads an error word and clears it
kvk_status take_error(int32_t *word, kvk_stream stream, int32_t *code) {
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int32_t h = 0;
  cudaError_t e = cudaMemcpyAsync(&h, word, 4, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess) e = cudaMemsetAsync(word, 0, 4, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "reading the device error word");
  *code = h;
  if (h) return fail(KVK_ERR_DEVICE, "device error word 0x%x", h);
  return KVK_OK;
}

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kNoWindow = 1 << 30;

}  // namespace

extern "C" {

kvk_status kvk_rotary_create(int32_t head_dim, int32_t rotary_dim, int32_t n_axes, const double *inv_freq,
                             const int32_t *axis, int32_t adjacent, float factor, kvk_rotary **out) {
  if (!out) return fail(KVK_ERR_INVALID_ARG, "null output handle");
  *out = nullptr;
  if (head_dim <= 0 || head_dim % 2 || head_dim > 2 * kRotMaxFreq)
    return fail(KVK_ERR_INVALID_ARG, "head_dim must be even and in [2, %d]", 2 * kRotMaxFreq);
  if (rotary_dim <= 0 || rotary_dim % 2 || rotary_dim > head_dim)
    return fail(KVK_ERR_INVALID_ARG, "rotary_dim must be even and in [2, head_dim]");
  if (n_axes < 1 || n_axes > 8) return fail(KVK_ERR_INVALID_ARG, "n_axes must be in [1, 8]");
  if (!inv_freq || !axis) return fail(KVK_ERR_INVALID_ARG, "null frequencies or axes");
  if (adjacent != 0 && adjacent != 1) return fail(KVK_ERR_INVALID_ARG, "adjacent must be 0 or 1");
  if (!std::isfinite(factor)) return fail(KVK_ERR_INVALID_ARG, "factor must be finite");
  const int n = rotary_dim / 2;
  for (int i = 0; i < n; ++i) {
    if (!std::isfinite(inv_freq[i])) return fail(KVK_ERR_INVALID_ARG, "frequency %d is not finite", i);
    if (axis[i] < 0 || axis[i] >= n_axes)
      return fail(KVK_ERR_INVALID_ARG, "axis %d of frequency %d out of range [0, %d)", axis[i], i, n_axes);
  }
  kvk_rotary *r = new (std::nothrow) kvk_rotary();
  if (!r) return fail(KVK_ERR_INVALID_ARG, "out of host memory");
  r->head_dim = head_dim;
  r->t = RotTable{};
  r->t.n_freq = n;
  r->t.n_axes = n_axes;
  r->t.adjacent = adjacent;
  r->t.factor = factor;
  // f / (2 pi) as a 64-bit fraction of a turn, 1 / (2 pi) in two doubles: of
  // |f| (whole turns of a number that is not negative drop out exactly), a signed
  // remainder added, the sign put back last; all modulo 2^64.
  constexpr double hi = 0.15915494309189535, lo = -9.839338337591243e-18;
  for (int i = 0; i < n; ++i) {
    const double f = std::fabs(inv_freq[i]), t = f * hi;
    const double frac = t - std::floor(t);  // exact, in [0, 1)
    double rest = std::fma(f, hi, -t) + f * lo;
    rest -= std::nearbyint(rest);  // exact, in [-1/2, 1/2]
    if (rest == 0.5) rest = -0.5;
    const uint64_t s = (uint64_t)std::nearbyint(std::ldexp(frac, 64)) + (uint64_t)(int64_t)std::nearbyint(std::ldexp(rest, 64));
    r->t.step[i] = inv_freq[i] < 0 ? 0 - s : s;
    r->t.axis[i] = (uint8_t)axis[i];
  }
  *out = r;
  return KVK_OK;
}

kvk_status kvk_rotary_destroy(kvk_rotary *r) {
  delete r;
  return KVK_OK;
}

kvk_status kvk_rotary_apply(const kvk_rotary *r, const kvk_rows *q, const kvk_rows *q_out, int32_t q_heads,
                            const kvk_rows *k, const kvk_rows *k_out, int32_t k_heads, int32_t dtype,
                            int32_t n_tokens, const int32_t *positions, kvk_stream stream) {
  if (!r) return fail(KVK_ERR_INVALID_ARG, "null rotary");
  if (dtype != KVK_DTYPE_F32 && dtype != KVK_DTYPE_BF16 && dtype != KVK_DTYPE_F16)
    return fail(KVK_ERR_INVALID_ARG, "dtype must be F32, BF16 or F16");
  if (n_tokens < 0 || q_heads < 0 || k_heads < 0 || q_heads > 65535 || k_heads > 65535)
    return fail(KVK_ERR_INVALID_ARG, "tokens or heads out of range");
  if (n_tokens == 0 || q_heads + k_heads == 0) return KVK_OK;
  if (!positions || !aligned(positions, 4)) return fail(KVK_ERR_INVALID_ARG, "null or misaligned positions");
  RotArgs a = {};
  a.t = r->t;
  a.D = r->head_dim;
  a.Hq = q_heads;
  a.Hk = k_heads;
  a.n_tokens = n_tokens;
  a.pos = positions;
  kvk_status s = KVK_OK;
  const int elem = dtype == KVK_DTYPE_F32 ? 4 : 2;
  if (q_heads) {
    s = take_rows(q, "q", n_tokens, q_heads, a.D, elem, elem, a.q);
    if (!s) s = take_rows(q_out, "q_out", n_tokens, q_heads, a.D, elem, elem, a.qo);
  }
  if (!s && k_heads) {
    s = take_rows(k, "k", n_tokens, k_heads, a.D, elem, elem, a.k);
    if (!s) s = take_rows(k_out, "k_out", n_tokens, k_heads, a.D, elem, elem, a.ko);
  }
  if (s) return s;
  const cudaError_t e = launch_rotary(a, dtype, reinterpret_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "rotary launch");
  return KVK_OK;
}

kvk_status kvk_paged_plan(const kvk_paged_desc *desc, size_t *pool, size_t *ws_bytes) {
  kvk_status s = check_paged_desc(desc);
  if (s) return s;
  if (!pool || !ws_bytes) return fail(KVK_ERR_INVALID_ARG, "null output");
  *pool = pool_bytes(desc, false);
  *ws_bytes = paged_ws(desc->head_dim, desc->n_pages).total;
  return KVK_OK;
}

static kvk_status paged_create(const kvk_paged_desc *desc, void *const *k_pages, void *const *v_pages, int8_t *const *k_exps,
                               int8_t *const *v_exps, bool coded, void *workspace, size_t ws_bytes, kvk_paged **out) {
  if (!out) return fail(KVK_ERR_INVALID_ARG, "null output handle");
  *out = nullptr;
  kvk_status s = check_paged_desc(desc);
  if (s) return s;
  if (!k_pages || !v_pages || (coded && (!k_exps || !v_exps))) return fail(KVK_ERR_INVALID_ARG, "null page pools");
  const int exp_align = desc->n_kv_heads % 4 == 0 ? 4 : desc->n_kv_heads % 2 == 0 ? 2 : 1;
  for (int l = 0; coded && l < desc->n_layers; ++l)
    for (const int8_t *p : {k_exps[l], v_exps[l]})
      if (!p || !aligned(p, exp_align))
        return fail(KVK_ERR_INVALID_ARG, "exponents of layer %d are null or not %d-byte aligned", l, exp_align);
  for (int l = 0; l < desc->n_layers; ++l)
    for (const void *p : {k_pages[l], v_pages[l]})
      if (!p || (reinterpret_cast<uintptr_t>(p) & 127u))
        return fail(KVK_ERR_INVALID_ARG, "pages of layer %d are null or not 128-byte aligned", l);
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255u))
    return fail(KVK_ERR_INVALID_ARG, "workspace null or not 256-byte aligned");
  if (ws_bytes < paged_ws(desc->head_dim, desc->n_pages).total)
    return fail(KVK_ERR_INVALID_ARG, "workspace too small: %zu < %zu", ws_bytes, paged_ws(desc->head_dim, desc->n_pages).total);
  kvk_paged *p = new (std::nothrow) kvk_paged();
  if (!p) return fail(KVK_ERR_INVALID_ARG, "out of host memory");
  p->d = *desc;
  p->coded = coded;
  try {
    for (int l = 0; l < desc->n_layers; ++l) {
      p->k.push_back(static_cast<uint8_t *>(k_pages[l]));
      p->v.push_back(static_cast<uint8_t *>(v_pages[l]));
      if (coded) {
        p->ke.push_back(k_exps[l]);
        p->ve.push_back(v_exps[l]);
      }
    }
    p->maps.resize((size_t)desc->n_layers * kMaps);
  } catch (const std::bad_alloc &) {
    delete p;
    return fail(KVK_ERR_INVALID_ARG, "out of host memory");
  }
  p->ws = static_cast<uint8_t *>(workspace);
  p->page_shift = desc->page_size == 16 ? 4 : desc->page_size == 32 ? 5 : desc->page_size == 64 ? 6 : 7;
  cudaError_t e = cudaGetDevice(&p->device);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&p->sms, cudaDevAttrMultiProcessorCount, p->device);
  if (e != cudaSuccess) {
    delete p;
    return kvk_internal_cuda_error(e, "querying the device");
  }
  const bool bf = desc->dtype == KVK_DTYPE_BF16;
  const int hc = rows_heads(desc->page_size, desc->n_kv_heads), heads[kMaps] = {0, hc, hc, 1, 1};
  const int code_hc = code_heads(desc->page_size, desc->n_kv_heads);
  for (int i = 0; i < desc->n_layers * kMaps && e == cudaSuccess; ++i) {
    const int l = i / kMaps, m = i % kMaps;
    const bool values = m == 2 || m == 4;
    if (coded) {
      if (m > 0)
        e = make_codes_map(p->maps[i].bytes, values ? p->v[l] : p->k[l], desc->head_dim, desc->page_size, desc->n_kv_heads,
                           desc->n_pages, m <= 2 ? code_hc : 1);
      continue;
    }
    e = make_pages_map(p->maps[i].bytes, bf, values ? p->v[l] : p->k[l], desc->head_dim, desc->page_size, desc->n_kv_heads,
                       desc->n_pages, heads[m]);
  }
  if (e != cudaSuccess) {
    delete p;
    return kvk_internal_cuda_error(e, "encoding the pages' tensor maps");
  }
  *out = p;
  return KVK_OK;
}

kvk_status kvk_paged_create(const kvk_paged_desc *desc, void *const *k_pages, void *const *v_pages, void *workspace,
                            size_t ws_bytes, kvk_paged **out) {
  return paged_create(desc, k_pages, v_pages, nullptr, nullptr, false, workspace, ws_bytes, out);
}

kvk_status kvk_paged_coded_plan(const kvk_paged_desc *desc, size_t *pool, size_t *exps, size_t *ws_bytes) {
  kvk_status s = check_paged_desc(desc);
  if (s) return s;
  if (!pool || !exps || !ws_bytes) return fail(KVK_ERR_INVALID_ARG, "null output");
  *pool = pool_bytes(desc, true);
  *exps = (size_t)desc->n_pages * desc->n_kv_heads;
  *ws_bytes = paged_ws(desc->head_dim, desc->n_pages).total;
  return KVK_OK;
}

kvk_status kvk_paged_coded_create(const kvk_paged_desc *desc, void *const *k_pages, void *const *v_pages, int8_t *const *k_exps,
                                  int8_t *const *v_exps, void *workspace, size_t ws_bytes, kvk_paged **out) {
  return paged_create(desc, k_pages, v_pages, k_exps, v_exps, true, workspace, ws_bytes, out);
}

kvk_status kvk_paged_destroy(kvk_paged *p) {
  delete p;
  return KVK_OK;
}

kvk_status kvk_paged_reset(kvk_paged *p, kvk_stream stream) {
  if (!p) return fail(KVK_ERR_INVALID_ARG, "null paged cache");
  const cudaError_t e =
      cudaMemsetAsync(p->ws, 0, paged_ws(p->d.head_dim, p->d.n_pages).part, reinterpret_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "resetting the workspace");
  p->cleared.store(true, std::memory_order_relaxed);
  return KVK_OK;
}

kvk_status kvk_paged_append(kvk_paged *p, int32_t layer, const kvk_paged_batch *batch, const kvk_rows *k,
                            const kvk_rows *v, const kvk_rotary *rotary, const int32_t *positions, const kvk_rows *q,
                            const kvk_rows *q_out, kvk_stream stream) {
  bool empty = false;
  kvk_status s = check_call(p, layer, batch, empty);
  if (s) return s;
  if (rotary && rotary->head_dim != p->d.head_dim)
    return fail(KVK_ERR_INVALID_ARG, "rotary of head_dim %d, cache of %d", rotary->head_dim, p->d.head_dim);
  if (rotary && !positions && rotary->t.n_axes != 1)
    return fail(KVK_ERR_INVALID_ARG, "a rotary of %d axes needs positions", rotary->t.n_axes);
  if (positions && !rotary) return fail(KVK_ERR_INVALID_ARG, "positions without a rotary");
  if (q && !rotary) return fail(KVK_ERR_INVALID_ARG, "queries are taken to be rotated: no rotary given");
  if (!aligned(positions, 4)) return fail(KVK_ERR_INVALID_ARG, "misaligned positions");
  if (empty) return KVK_OK;
  RotArgs a = {};
  const int N = batch->n_tokens, D = p->d.head_dim, Hkv = p->d.n_kv_heads;
  s = take_rows(k, "k", N, Hkv, D, 2, 2, a.k);
  if (!s) s = take_rows(v, "v", N, Hkv, D, 2, 2, a.v);
  if (!s && q) {
    s = take_rows(q, "q", N, p->d.n_q_heads, D, 2, 2, a.q);
    if (!s) s = take_rows(q_out, "q_out", N, p->d.n_q_heads, D, 2, 2, a.qo);
  }
  if (s) return s;
  if (rotary) a.t = rotary->t;
  a.D = D;
  a.Hq = q ? p->d.n_q_heads : 0;
  a.Hk = a.Hv = p->coded ? 0 : Hkv;
  a.n_tokens = N;
  a.pos = positions;
  a.pv = view_of(p, layer, batch);
  cudaError_t e = cudaSuccess;
  if (p->coded) {
    CodeArgs c = {};
    c.t = a.t;
    c.k = a.k;
    c.v = a.v;
    c.pos = positions;
    c.rotate = rotary != nullptr;
    c.wide = aligned(c.k.p, 16) && aligned(c.v.p, 16) && !((c.k.ts | c.k.hs | c.v.ts | c.v.hs) & 7);
    c.pv = a.pv;
    e = launch_append_codes(c, p->d.dtype, reinterpret_cast<cudaStream_t>(stream));
  }
  if (e == cudaSuccess) e = launch_rotary(a, p->d.dtype, reinterpret_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "paged append launch");
  return KVK_OK;
}

kvk_status kvk_paged_attention(kvk_paged *p, int32_t layer, const kvk_paged_batch *batch, const kvk_rows *q,
                               float softmax_scale, int32_t max_new, int32_t window, void *out, kvk_stream stream) {
  bool empty = false;
  kvk_status s = check_call(p, layer, batch, empty);
  if (s) return s;
  if (!scale_ok(softmax_scale)) return fail(KVK_ERR_INVALID_ARG, "softmax scale must be finite and positive");
  if (window < 0) return fail(KVK_ERR_INVALID_ARG, "window must not be negative");
  // (what an uncleared workspace holds would be taken for units to join)
  if (!p->cleared.load(std::memory_order_relaxed))
    return fail(KVK_ERR_INVALID_ARG, "kvk_paged_reset has to clear the workspace before the first attention");
  if (empty) return KVK_OK;
  if (max_new < 1) return fail(KVK_ERR_INVALID_ARG, "max_new must be positive");
  AttnArgs a = {};
  s = take_rows(q, "q", batch->n_tokens, p->d.n_q_heads, p->d.head_dim, 2, 16, a.q);
  if (s) return s;
  if (!out || (reinterpret_cast<uintptr_t>(out) & 15u)) return fail(KVK_ERR_INVALID_ARG, "null or misaligned out");
  a.pv = view_of(p, layer, batch);
  a.out = out;
  a.Hq = p->d.n_q_heads;
  a.G = a.Hq / p->d.n_kv_heads;
  a.window = window && window < kNoWindow ? window : kNoWindow;
  a.max_new = max_new < batch->n_tokens ? max_new : batch->n_tokens;
  a.sig_log2 = softmax_scale * kLog2e;
  const PagedWs w = paged_ws(p->d.head_dim, p->d.n_pages);
  a.list = reinterpret_cast<RowsList *>(p->ws + w.list);
  a.tc_list = reinterpret_cast<TcList *>(p->ws + w.tc_list);
  a.part = reinterpret_cast<float *>(p->ws + w.part);
  a.sms = p->sms;
  a.device = p->device;
  a.give_up = p->give_up.load(std::memory_order_relaxed);
  const PageMap *maps = &p->maps[(size_t)layer * kMaps];
  a.mk = maps[0].bytes;
  a.wk = maps[1].bytes;
  a.wv = maps[2].bytes;
  a.ok = maps[3].bytes;
  a.ov = maps[4].bytes;
  // Two launches around the workspace's list of cut units: another thread's must
  // not come between them, its units would be joined into this call's output.
  cudaError_t e;
  {
    std::lock_guard<std::mutex> one(p->calls);
    e = launch_attn(a, p->d.dtype, reinterpret_cast<cudaStream_t>(stream));
  }
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "paged attention launch");
  return KVK_OK;
}

kvk_status kvk_paged_copy(kvk_paged *p, const int32_t *src, const int32_t *dst, int32_t n, kvk_stream stream) {
  if (!p) return fail(KVK_ERR_INVALID_ARG, "null paged cache");
  const kvk_status s = check_device(p);
  if (s) return s;
  if (n < 0) return fail(KVK_ERR_INVALID_ARG, "n must not be negative");
  if (n == 0) return KVK_OK;
  if (!src || !dst || !aligned(src, 4) || !aligned(dst, 4)) return fail(KVK_ERR_INVALID_ARG, "null or misaligned pages");
  const cudaError_t e = copy_layers(p, 0, src, dst, n, nullptr, reinterpret_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "page copy launch");
  return KVK_OK;
}

kvk_status kvk_paged_fork(kvk_paged *p, const int32_t *refs, const int32_t *table, const int32_t *lengths, int32_t batch,
                          int32_t max_pages, const int32_t *parents, const int32_t *after, int32_t rows, int32_t *refs_out,
                          int32_t *table_out, int32_t max_pages_out, kvk_stream stream) {
  kvk_status s = check_pages(p, refs, refs_out, table, lengths, batch, max_pages);
  if (s) return s;
  if (rows < 0 || rows > kForkRows) return fail(KVK_ERR_INVALID_ARG, "rows must be in [0, %d]", kForkRows);
  if (max_pages_out < 0 || (int64_t)max_pages_out * p->d.page_size > (1 << 26))
    return fail(KVK_ERR_INVALID_ARG, "max_pages_out out of range");
  // (what all rows ask for is counted in 32 bits)
  if ((int64_t)rows * max_pages_out > (1 << 30))
    return fail(KVK_ERR_INVALID_ARG, "a table of %d x %d pages: more than 2^30 entries", rows, max_pages_out);
  if (rows && (!parents || (!table_out && max_pages_out))) return fail(KVK_ERR_INVALID_ARG, "null parents or table");
  if (!aligned(parents, 4) || !aligned(after, 4) || !aligned(table_out, 4))
    return fail(KVK_ERR_INVALID_ARG, "misaligned parents, lengths or table");
  const int64_t in = (int64_t)batch * max_pages, out = (int64_t)rows * max_pages_out;
  if (in && out && table_out < table + in && table < table_out + out)
    return fail(KVK_ERR_INVALID_ARG, "a fork's table may not overlap the one it is made from");
  PagesArgs a = pages_args(p);
  a.refs = refs;
  a.refs_out = refs_out;
  a.table = table;
  a.lens = lengths;
  a.parents = parents;
  a.after = after;
  a.table_out = table_out;
  a.B = batch;
  a.R = rows;
  a.max_pages = max_pages;
  a.width = max_pages_out;
  // launches that share the workspace follow one another
  cudaError_t e;
  {
    std::lock_guard<std::mutex> one(p->calls);
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    e = launch_fork(a, copy_args(p, 0, a.src, a.dst, rows, nullptr), p->coded, p->sms, st);
    if (e == cudaSuccess && rows) e = copy_layers(p, kCopyLayers, a.src, a.dst, rows, nullptr, st);
  }
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "page fork launch");
  return KVK_OK;
}

kvk_status kvk_paged_compact(kvk_paged *p, const int32_t *refs, const int32_t *table, const int32_t *lengths, int32_t batch,
                             int32_t max_pages, int32_t *refs_out, int32_t *table_out, int32_t *where, int32_t *used,
                             kvk_stream stream) {
  kvk_status s = check_pages(p, refs, refs_out, table, lengths, batch, max_pages);
  if (s) return s;
  if (!where || (batch && max_pages && !table_out)) return fail(KVK_ERR_INVALID_ARG, "null table or numbers");
  if (!aligned(where, 4) || !aligned(used, 4) || !aligned(table_out, 4))
    return fail(KVK_ERR_INVALID_ARG, "misaligned table or numbers");
  const int64_t in = (int64_t)batch * max_pages;
  if (in && table_out != table && table_out < table + in && table < table_out + in)
    return fail(KVK_ERR_INVALID_ARG, "table_out may be the table, and may not overlap it otherwise");
  const int n = p->d.n_pages;
  if ((where < refs + n && refs < where + n) || (where < refs_out + n && refs_out < where + n))
    return fail(KVK_ERR_INVALID_ARG, "where may not overlap the holders");
  PagesArgs a = pages_args(p);
  a.refs = refs;
  a.refs_out = refs_out;
  a.table = table;
  a.lens = lengths;
  a.table_out = table_out;
  a.where = where;
  a.used = used;
  a.B = batch;
  a.max_pages = a.width = max_pages;
  cudaError_t e;
  {
    std::lock_guard<std::mutex> one(p->calls);
    const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
    const int most = p->d.n_pages / 2;
    e = launch_compact(a, copy_args(p, 0, a.src, a.dst, most, a.n_moved), p->coded, p->sms, st);
    if (e == cudaSuccess) e = copy_layers(p, kCopyLayers, a.src, a.dst, most, a.n_moved, st);
  }
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "page compaction launch");
  return KVK_OK;
}

kvk_status kvk_paged_set_give_up(kvk_paged *p, int32_t give_up) {
  if (!p) return fail(KVK_ERR_INVALID_ARG, "null paged cache");
  if (give_up != 0 && give_up != 1) return fail(KVK_ERR_INVALID_ARG, "give_up must be 0 or 1");
  p->give_up.store(give_up, std::memory_order_relaxed);
  return KVK_OK;
}

kvk_status kvk_paged_get_device_error(kvk_paged *p, kvk_stream stream, int32_t *code) {
  if (!p || !code) return fail(KVK_ERR_INVALID_ARG, "null paged cache or output");
  return take_error(reinterpret_cast<int32_t *>(p->ws + paged_ws(p->d.head_dim, p->d.n_pages).err), stream, code);
}

kvk_status kvk_prompt_set_give_up(int32_t give_up) {
  if (give_up != 0 && give_up != 1) return fail(KVK_ERR_INVALID_ARG, "give_up must be 0 or 1");
  g_prompt_give_up.store(give_up, std::memory_order_relaxed);
  return KVK_OK;
}

kvk_status kvk_prompt_get_device_error(kvk_stream stream, int32_t *code) {
  if (!code) return fail(KVK_ERR_INVALID_ARG, "null output");
  int dev = 0;
  int32_t *word = nullptr;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = prompt_word(dev, &word);
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "looking up the prompts' error word");
  return take_error(word, stream, code);
}

kvk_status kvk_prompt_attention(const kvk_rows *q, const kvk_rows *k, const kvk_rows *v, int32_t n_tokens,
                                int32_t n_q_heads, int32_t n_kv_heads, int32_t head_dim, int32_t dtype,
                                const int32_t *cu_seqlens, int32_t batch, float softmax_scale, int32_t window, void *out,
                                int32_t *error, kvk_stream stream) {
  kvk_status s = check_heads(n_q_heads, n_kv_heads, head_dim, dtype);
  if (s) return s;
  if (!scale_ok(softmax_scale)) return fail(KVK_ERR_INVALID_ARG, "softmax scale must be finite and positive");
  if (window < 0) return fail(KVK_ERR_INVALID_ARG, "window must not be negative");
  if (batch < 0 || n_tokens < 0 || (int64_t)n_tokens * n_q_heads > (1 << 30))
    return fail(KVK_ERR_INVALID_ARG, "batch or n_tokens out of range");
  if (batch == 0 || n_tokens == 0) return KVK_OK;
  if (!cu_seqlens || !aligned(cu_seqlens, 4) || !aligned(error, 4))
    return fail(KVK_ERR_INVALID_ARG, "null or misaligned offsets or error word");
  if (!out || (reinterpret_cast<uintptr_t>(out) & 15u)) return fail(KVK_ERR_INVALID_ARG, "null or misaligned out");
  AttnArgs a = {};
  s = take_rows(q, "q", n_tokens, n_q_heads, head_dim, 2, 16, a.q);
  if (!s) s = take_rows(k, "k", n_tokens, n_kv_heads, head_dim, 2, 16, a.k);
  if (!s) s = take_rows(v, "v", n_tokens, n_kv_heads, head_dim, 2, 16, a.v);
  if (s) return s;
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = cudaDeviceGetAttribute(&a.sms, cudaDevAttrMultiProcessorCount, dev);
  if (e == cudaSuccess && !error) e = prompt_word(dev, &error);
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "querying the device");
  a.device = dev;
  a.give_up = g_prompt_give_up.load(std::memory_order_relaxed);
  a.pv.cu = cu_seqlens;
  a.pv.B = batch;
  a.pv.Hkv = n_kv_heads;
  a.pv.D = head_dim;
  a.pv.n_tokens = n_tokens;
  a.pv.err = error;
  a.out = out;
  a.Hq = n_q_heads;
  a.G = n_q_heads / n_kv_heads;
  a.window = window && window < kNoWindow ? window : kNoWindow;
  a.max_new = n_tokens;
  a.sig_log2 = softmax_scale * kLog2e;
  e = launch_attn(a, dtype, reinterpret_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return kvk_internal_cuda_error(e, "prompt attention launch");
  return KVK_OK;
}

}  // extern "C"
