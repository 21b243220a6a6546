// The C ABI of the paged cache operators (include/mbp.h): argument checks and launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "mbp.h"
#include "paged.h"

using namespace mbp;

namespace {

thread_local char g_error[256] = "";

int refuse(int code, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  std::vsnprintf(g_error, sizeof g_error, fmt, ap);
  va_end(ap);
  return code;
}

int launched(hipError_t e, const char* what) {
  if (e == hipSuccess) return MBP_OK;
  return refuse(MBP_EHIP, "HIP error in %s: %s", what, hipGetErrorString(e));
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

int64_t page_bytes_of(const mbp_paged_cache& c) {
  return c.dtype == MBP_MXFP4 ? (int64_t)c.page_size * (c.d_head / 2 + c.d_head / 32) : (int64_t)c.page_size * c.d_head * 2;
}

// The shape alone (the pools and the table may be missing).
int check_shape(const mbp_paged_cache* c) {
  if (c == nullptr) return refuse(MBP_EINVAL, "cache is null");
  if (c->dtype != MBP_BF16 && c->dtype != MBP_F16 && c->dtype != MBP_MXFP4)
    return refuse(MBP_EINVAL, "cache dtype must be MBP_BF16, MBP_F16 or MBP_MXFP4");
  if (c->d_head != 32 && c->d_head != 64 && c->d_head != 128) return refuse(MBP_EINVAL, "d_head must be 32, 64 or 128");
  if (c->n_kv_heads < 1 || c->n_kv_heads > 8192) return refuse(MBP_EINVAL, "n_kv_heads must be in [1, 8192]");
  if (c->page_size < 16 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return refuse(MBP_EINVAL, "page_size must be a power of two in [16, 1024]");
  if (c->n_pages < 1) return refuse(MBP_EINVAL, "n_pages must be >= 1");
  if (c->n_seqs < 0 || c->n_seqs > 65535) return refuse(MBP_EINVAL, "n_seqs must be in [0, 65535]");
  if (c->max_pages < 1 || (int64_t)c->max_pages * c->page_size > (1 << 30))
    return refuse(MBP_EINVAL, "max_pages must be >= 1 and max_pages x page_size at most 2^30");
  return MBP_OK;
}

int check_cache(const mbp_paged_cache* c, PagedCache* out) {
  const int rc = check_shape(c);
  if (rc) return rc;
  if (c->d_k == nullptr || c->d_v == nullptr || !aligned(c->d_k, 16) || !aligned(c->d_v, 16))
    return refuse(MBP_EINVAL, "d_k and d_v must be device pointers aligned to 16 bytes");
  if (c->n_seqs > 0 && (c->d_pages == nullptr || !aligned(c->d_pages, 4))) return refuse(MBP_EINVAL, "d_pages is null or misaligned");
  int shift = 4;
  while ((1 << shift) < c->page_size) ++shift;
  *out = PagedCache{reinterpret_cast<char*>(c->d_k), reinterpret_cast<char*>(c->d_v), c->d_pages, c->dtype, c->n_kv_heads,
                    c->d_head, shift, c->n_pages, c->n_seqs, c->max_pages, page_bytes_of(*c)};
  return MBP_OK;
}

// Bounds beyond the cache's are cut to it: a sequence has at most n_rows rows, a row sees
// at most the table's slots.
int check_rows(const mbp_paged_cache& c, const mbp_paged_rows* r, PagedRows* out) {
  if (r == nullptr) return refuse(MBP_EINVAL, "rows is null");
  if (r->n_rows < 0 || r->max_rows < 0 || r->max_slots < 0)
    return refuse(MBP_EINVAL, "n_rows, max_rows and max_slots must be >= 0");
  if (c.n_seqs > 0 && (r->d_row_start == nullptr || r->d_first_slot == nullptr || !aligned(r->d_row_start, 4) || !aligned(r->d_first_slot, 4)))
    return refuse(MBP_EINVAL, "d_row_start or d_first_slot is null or misaligned");
  *out = PagedRows{r->d_row_start, r->d_first_slot, r->n_rows, std::min(r->max_rows, r->n_rows),
                   (int32_t)std::min<int64_t>(r->max_slots, (int64_t)c.max_pages * c.page_size)};
  return MBP_OK;
}

int check_heads(const char* name, const mbp_paged_heads* h, int n_heads, int n_rows, int d_head, bool written, HeadRows* out) {
  if (h == nullptr || h->d == nullptr) return refuse(MBP_EINVAL, "%s is null", name);
  if (h->dtype != MBP_F32 && h->dtype != MBP_BF16 && h->dtype != MBP_F16)
    return refuse(MBP_EINVAL, "%s: dtype must be MBP_F32, MBP_BF16 or MBP_F16", name);
  const int es = h->dtype == MBP_F32 ? 4 : 2;
  if (!aligned(h->d, es)) return refuse(MBP_EINVAL, "%s is not aligned to its elements", name);
  const int64_t most = (int64_t)1 << 40;
  if (h->row_stride < 0 || h->head_stride < 0 || h->row_stride > most || h->head_stride > most)
    return refuse(MBP_EINVAL, "%s: strides must be in [0, 2^40]", name);
  if (written) {  // no two heads of any rows may overlap
    const int64_t rs = h->row_stride, hs = h->head_stride, d = d_head;
    const bool one_row = n_rows <= 1, one_head = n_heads == 1;
    const bool ok = (one_row && one_head) || (one_row && hs >= d) || (one_head && rs >= d) ||
                    (hs >= d && rs >= (n_heads - 1) * hs + d) || (rs >= d && hs >= (n_rows - 1) * rs + d);
    if (!ok) return refuse(MBP_EINVAL, "%s: rows or heads overlap", name);
  }
  const int vec = aligned(h->d, 16) && h->row_stride * es % 16 == 0 && h->head_stride * es % 16 == 0;
  *out = HeadRows{h->d, h->row_stride, h->head_stride, h->dtype, vec};
  return MBP_OK;
}

int check_count(int n_heads, const mbp_paged_cache& c) {
  if (n_heads < 1 || n_heads > 8192 || n_heads % c.n_kv_heads != 0)
    return refuse(MBP_EINVAL, "n_heads must be a multiple of n_kv_heads of at most 8192");
  return MBP_OK;
}

// Blocks of 256 threads must fit a one-dimensional grid.
int check_grid(int64_t blocks) {
  return blocks > 0x7fffffff ? refuse(MBP_ECAPACITY, "the call has too many rows for one launch") : MBP_OK;
}

#define CK(x)            \
  do {                   \
    const int rc_ = (x); \
    if (rc_) return rc_; \
  } while (0)

}  // namespace

extern "C" {

const char* mbp_paged_error(void) { return g_error; }

size_t mbp_paged_pool_bytes(const mbp_paged_cache* c) {
  if (check_shape(c)) return 0;
  return (size_t)c->n_pages * c->n_kv_heads * page_bytes_of(*c);
}

int mbp_rope_table(float* d_table, int32_t n_pos, int32_t d_head, float base, void* hip_stream) {
  if (d_table == nullptr || !aligned(d_table, 16)) return refuse(MBP_EINVAL, "d_table is null or not aligned to 16 bytes");
  if (n_pos < 1) return refuse(MBP_EINVAL, "n_pos must be >= 1");
  if (d_head != 32 && d_head != 64 && d_head != 128) return refuse(MBP_EINVAL, "d_head must be 32, 64 or 128");
  if (!(base > 0.f) || !std::isfinite(base)) return refuse(MBP_EINVAL, "base must be positive");
  return launched(launch_rope_table(reinterpret_cast<float2*>(d_table), n_pos, d_head, base, static_cast<hipStream_t>(hip_stream)),
                  "mbp_rope_table");
}

int mbp_paged_append(const mbp_paged_cache* cache, const mbp_paged_rows* rows, int32_t n_heads, const mbp_paged_heads* q,
                     const mbp_paged_heads* q_out, const mbp_paged_heads* k, const mbp_paged_heads* v, const int32_t* d_pos,
                     const float* d_rope, int32_t n_pos, void* hip_stream) {
  PagedAppend a{};
  CK(check_cache(cache, &a.c));
  CK(check_rows(*cache, rows, &a.r));
  if ((q == nullptr) != (q_out == nullptr)) return refuse(MBP_EINVAL, "q and q_out are given together or not at all");
  if (q != nullptr) {
    CK(check_count(n_heads, *cache));
    CK(check_heads("q", q, n_heads, a.r.n_rows, a.c.dh, false, &a.q));
    CK(check_heads("q_out", q_out, n_heads, a.r.n_rows, a.c.dh, true, &a.qo));
    if (q->dtype != q_out->dtype) return refuse(MBP_EINVAL, "q and q_out must have one dtype");
    if (q->d == q_out->d && (q->row_stride != q_out->row_stride || q->head_stride != q_out->head_stride))
      return refuse(MBP_EINVAL, "q_out in the place of q must have its strides");
    a.H = n_heads;
  }
  CK(check_heads("k", k, a.c.hk, a.r.n_rows, a.c.dh, false, &a.k));
  CK(check_heads("v", v, a.c.hk, a.r.n_rows, a.c.dh, false, &a.v));
  if (d_rope != nullptr && (!aligned(d_rope, 16) || n_pos < 1))
    return refuse(MBP_EINVAL, "d_rope must be aligned to 16 bytes and n_pos >= 1");
  if (d_pos != nullptr && (!aligned(d_pos, 4) || d_rope == nullptr))
    return refuse(MBP_EINVAL, "d_pos must be aligned to 4 bytes and needs d_rope");
  a.pos = d_pos;
  a.rope = reinterpret_cast<const float2*>(d_rope);
  a.n_pos = n_pos;
  if (a.r.n_rows == 0 || a.c.n_seqs == 0) return MBP_OK;
  CK(check_grid((int64_t)a.r.n_rows * (a.H + 2 * a.c.hk) * (a.c.dh / 8) / 256 + 1));
  return launched(launch_paged_append(a, static_cast<hipStream_t>(hip_stream)), "mbp_paged_append");
}

int mbp_paged_read(const mbp_paged_cache* cache, const mbp_paged_rows* rows, const mbp_paged_heads* k_out,
                   const mbp_paged_heads* v_out, void* hip_stream) {
  PagedCache c{};
  PagedRows r{};
  HeadRows k{}, v{};
  CK(check_cache(cache, &c));
  CK(check_rows(*cache, rows, &r));
  CK(check_heads("k_out", k_out, c.hk, r.n_rows, c.dh, true, &k));
  CK(check_heads("v_out", v_out, c.hk, r.n_rows, c.dh, true, &v));
  if (r.n_rows == 0) return MBP_OK;
  CK(check_grid((int64_t)r.n_rows * 2 * c.hk * (c.dh / 8) / 256 + 1));
  return launched(launch_paged_read(c, r, k, v, static_cast<hipStream_t>(hip_stream)), "mbp_paged_read");
}

size_t mbp_paged_workspace_bytes(const mbp_paged_cache* cache, const mbp_paged_rows* rows, int32_t n_heads) {
  if (check_shape(cache) || check_count(n_heads, *cache) || rows == nullptr || rows->n_rows < 0 || rows->max_rows < 0 || rows->max_slots < 0)
    return 0;
  PagedCache c{};
  c.hk = cache->n_kv_heads;
  c.dh = cache->d_head;
  c.type = cache->dtype;
  c.n_seqs = cache->n_seqs;
  const PagedRows r{nullptr, nullptr, rows->n_rows, std::min(rows->max_rows, rows->n_rows),
                    (int32_t)std::min<int64_t>(rows->max_slots, (int64_t)cache->max_pages * cache->page_size)};
  if (r.n_rows == 0 || c.n_seqs == 0 || r.max_rows == 0) return 0;
  return paged_work_bytes(c, r, n_heads);
}

int mbp_paged_attend(const mbp_paged_cache* cache, const mbp_paged_rows* rows, int32_t n_heads, const mbp_paged_heads* q,
                     const mbp_paged_heads* out, const int32_t* d_lo, const int32_t* d_hi, float scale, void* d_work,
                     size_t work_bytes, void* hip_stream) {
  PagedAttend a{};
  CK(check_cache(cache, &a.c));
  CK(check_rows(*cache, rows, &a.r));
  CK(check_count(n_heads, *cache));
  CK(check_heads("q", q, n_heads, a.r.n_rows, a.c.dh, false, &a.q));
  CK(check_heads("out", out, n_heads, a.r.n_rows, a.c.dh, true, &a.o));
  if (q->dtype != out->dtype) return refuse(MBP_EINVAL, "q and out must have one dtype");
  if (q->d == out->d && (q->row_stride != out->row_stride || q->head_stride != out->head_stride))
    return refuse(MBP_EINVAL, "out in the place of q must have its strides");
  if (q->dtype != MBP_F32 && cache->dtype != MBP_MXFP4 && q->dtype != cache->dtype)
    return refuse(MBP_EINVAL, "q must be MBP_F32 or of the cache's 16-bit dtype");
  if (!aligned(d_lo, 4) || !aligned(d_hi, 4)) return refuse(MBP_EINVAL, "d_lo and d_hi must be aligned to 4 bytes");
  if (!std::isfinite(scale * 1.44269504f)) return refuse(MBP_EINVAL, "scale must be finite and below 2.3e38");
  a.H = n_heads;
  a.lo = d_lo;
  a.hi = d_hi;
  a.scale = scale;
  if (a.r.n_rows == 0 || a.c.n_seqs == 0 || a.r.max_rows == 0) return MBP_OK;
  const int64_t packed = (int64_t)a.r.max_rows * (n_heads / a.c.hk);
  if (packed > (1 << 30)) return refuse(MBP_ECAPACITY, "max_rows is too large");
  // the most blocks that any split of a sequence's work takes: 64 parts of 16 rows
  CK(check_grid((packed + 15) / 16 * 64));
  CK(check_grid((int64_t)a.c.n_seqs * a.r.max_rows * n_heads / 4 + 1));
  const size_t need = paged_work_bytes(a.c, a.r, n_heads);
  if (need > 0 && (d_work == nullptr || !aligned(d_work, 16))) return refuse(MBP_EINVAL, "d_work is null or not aligned to 16 bytes");
  if (work_bytes < need) return refuse(MBP_ECAPACITY, "d_work holds %zu of %zu bytes", work_bytes, need);
  a.work = static_cast<float*>(d_work);
  return launched(launch_paged_attend(a, static_cast<hipStream_t>(hip_stream)), "mbp_paged_attend");
}

}  // extern "C"
