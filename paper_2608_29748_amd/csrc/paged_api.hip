// C entries of the paged-cache operators: argument checks (before any device work) and launches.
#include <hip/hip_runtime.h>
#include <float.h>
#include <math.h>

#include "host.h"
#include "paged.h"

namespace rt {

static int check_cache(const rt_paged_kv* kv) {
  if (!kv) return fail(RT_ERR_INVALID, "cache is null");
  if (kv->dtype != RT_F32 && kv->dtype != RT_BF16) return fail(RT_ERR_INVALID, "cache dtype must be RT_F32 or RT_BF16");
  if (kv->page_size != kPage) return fail(RT_ERR_INVALID, "page_size must be 16");
  if (kv->head_dim != 64 && kv->head_dim != 128) return fail(RT_ERR_INVALID, "head_dim must be 64 or 128");
  if (kv->n_kv_heads < 1 || kv->n_kv_heads > 1024) return fail(RT_ERR_INVALID, "n_kv_heads must be in [1, 1024]");
  if (kv->n_pages < 1) return fail(RT_ERR_INVALID, "the cache has no pages");
  if (kv->max_pages < 1 || kv->max_pages > (1 << 26)) return fail(RT_ERR_INVALID, "max_pages must be in [1, 2^26]");
  if (!kv->k || !kv->v || !kv->page_table) return fail(RT_ERR_INVALID, "null cache pointer");
  if ((uintptr_t)kv->k % 16 || (uintptr_t)kv->v % 16 || (uintptr_t)kv->page_table % 4)
    return fail(RT_ERR_INVALID, "cache pages must be 16-byte aligned, the page table 4-byte aligned");
  return RT_OK;
}
static int check_rows(const rt_paged_kv* kv, int n_seqs, int n_rows, int n_q_heads, const int32_t* row_start,
                      const int32_t* kv_len) {
  if (n_seqs < 0 || n_rows < 0) return fail(RT_ERR_INVALID, "negative count of sequences or rows");
  if (n_q_heads < kv->n_kv_heads || n_q_heads % kv->n_kv_heads)
    return fail(RT_ERR_INVALID, "n_q_heads must be a positive multiple of n_kv_heads");
  if ((long long)n_rows * n_q_heads > 0x3fffffff) return fail(RT_ERR_CAPACITY, "more than 2^30 - 1 (row, query head) pairs");
  if (n_rows == 0) return RT_OK;
  if (n_seqs < 1) return fail(RT_ERR_INVALID, "rows without a sequence");
  if (n_seqs > (1 << 20)) return fail(RT_ERR_CAPACITY, "more than 2^20 sequences");
  if (!row_start && n_rows % n_seqs) return fail(RT_ERR_INVALID, "without row_start every sequence has n_rows / n_seqs rows");
  if (!kv_len) return fail(RT_ERR_INVALID, "kv_len is null");
  if ((uintptr_t)kv_len % 4 || (uintptr_t)row_start % 4) return fail(RT_ERR_INVALID, "row_start and kv_len must be 4-byte aligned");
  return RT_OK;
}
// Rows of `cols` elements of `esz` bytes at p, ld elements apart, are read and written 16 bytes at a time.
static int check_tensor(const char* name, const void* p, int64_t ld, int64_t cols, int esz) {
  if (!p) return fail(RT_ERR_INVALID, "%s is null", name);
  if (ld < cols) return fail(RT_ERR_INVALID, "the row stride of %s is less than its row", name);
  if ((uintptr_t)p % 16 || ld * esz % 16) return fail(RT_ERR_INVALID, "rows of %s must be 16-byte aligned", name);
  return RT_OK;
}
static PagedRows rows_of(const rt_paged_kv* kv, int n_seqs, int n_rows, int n_q_heads, const int32_t* row_start,
                         const int32_t* kv_len) {
  PagedRows r{};
  r.k = kv->k; r.v = kv->v; r.page_table = kv->page_table; r.max_pages = kv->max_pages; r.n_pages = kv->n_pages;
  r.n_q_heads = n_q_heads; r.n_kv_heads = kv->n_kv_heads; r.head_dim = kv->head_dim;
  r.n_seqs = n_seqs; r.n_rows = n_rows; r.rows_each = n_seqs > 0 ? n_rows / n_seqs : 0;
  r.row_start = row_start; r.kv_len = kv_len; r.kv_stride = 1; r.kv_add = 0;
  return r;
}
static int launched(hipError_t e, const char* what) {
  if (e == hipErrorInvalidValue) return fail(RT_ERR_CAPACITY, "%s: too many workgroups for one launch", what);
  if (e != hipSuccess) return fail(RT_ERR_HIP, "%s: %s", what, hipGetErrorString(e));
  return RT_OK;
}

static int kv_append(const rt_paged_kv* kv, const rt_append_args* g, hipStream_t s) {
  int st = check_cache(kv);
  if (st) return st;
  if (!g) return fail(RT_ERR_INVALID, "arguments are null");
  if (g->src_dtype != RT_F32 && g->src_dtype != kv->dtype)
    return fail(RT_ERR_INVALID, "src_dtype must be RT_F32 or the cache's dtype");
  st = check_rows(kv, g->n_seqs, g->n_rows, g->q ? g->n_q_heads : kv->n_kv_heads, g->row_start, g->kv_len);
  if (st) return st;
  const int hd = kv->head_dim, esz = kv->dtype == RT_BF16 ? 2 : 4, ssz = g->src_dtype == RT_BF16 ? 2 : 4;
  if (g->rope) {
    if (g->rot_dim < 16 || g->rot_dim > hd || g->rot_dim % 16)
      return fail(RT_ERR_INVALID, "rot_dim must be a multiple of 16 in [16, head_dim]");
    if ((uintptr_t)g->rope % 16) return fail(RT_ERR_INVALID, "rope must be 16-byte aligned");
    if (g->rope_positions < (long long)kv->max_pages * kPage)
      return fail(RT_ERR_CAPACITY, "rope has %d positions, the page table %lld", g->rope_positions, (long long)kv->max_pages * kPage);
  }
  if ((uintptr_t)g->q_norm % 16 || (uintptr_t)g->k_norm % 16) return fail(RT_ERR_INVALID, "norm weights must be 16-byte aligned");
  if (!(g->eps >= 0.f) || !isfinite(g->eps)) return fail(RT_ERR_INVALID, "eps must be finite and not negative");
  if (g->n_rows == 0) return RT_OK;
  if ((st = check_tensor("k", g->k, g->ldk, (int64_t)kv->n_kv_heads * hd, ssz))) return st;
  if ((st = check_tensor("v", g->v, g->ldv, (int64_t)kv->n_kv_heads * hd, ssz))) return st;
  if (g->q) {
    if ((st = check_tensor("q", g->q, g->ldq, (int64_t)g->n_q_heads * hd, ssz))) return st;
    if ((st = check_tensor("q_out", g->q_out, g->ldqo, (int64_t)g->n_q_heads * hd, esz))) return st;
  }
  AppendArgs a{};
  a.r = rows_of(kv, g->n_seqs, g->n_rows, g->q ? g->n_q_heads : kv->n_kv_heads, g->row_start, g->kv_len);
  a.q = g->q; a.ks = g->k; a.vs = g->v; a.ldq = g->ldq; a.ldk = g->ldk; a.ldv = g->ldv;
  a.q_out = g->q_out; a.ldqo = g->ldqo;
  a.cos = g->rope; a.rot_dim = g->rot_dim;
  a.sin = g->rope ? g->rope + (size_t)g->rope_positions * (g->rot_dim / 2) : nullptr;
  a.q_norm = g->q_norm; a.k_norm = g->k_norm; a.eps = g->eps;
  return launched(kv->dtype == RT_F32      ? paged_append<float, float>(a, s)
                  : g->src_dtype == RT_F32 ? paged_append<bf16_t, float>(a, s)
                                           : paged_append<bf16_t, bf16_t>(a, s), "rt_kv_append");
}

// Checks an attention call and fills the launch arguments.  tensors: q and out are checked too.
static int attn_args(const rt_paged_kv* kv, const rt_attn_args* g, bool tensors, PagedAttnArgs* out) {
  int st = check_cache(kv);
  if (st) return st;
  if (!g) return fail(RT_ERR_INVALID, "arguments are null");
  st = check_rows(kv, g->n_seqs, g->n_rows, g->n_q_heads, g->row_start, g->kv_len);
  if (st) return st;
  const long long cap = (long long)kv->max_pages * kPage;
  if (g->max_rows < 0 || g->max_kv < 0) return fail(RT_ERR_INVALID, "negative max_rows or max_kv");
  if (g->window < 0 || g->sinks < 0) return fail(RT_ERR_INVALID, "negative window or sinks");
  if (g->prefix_len < 0 || g->prefix_len % kPage || g->prefix_len > cap)
    return fail(RT_ERR_INVALID, "prefix_len must be a multiple of 16 within the page table");
  if (!(g->scale >= 0.f) || !isfinite(g->scale)) return fail(RT_ERR_INVALID, "scale must be finite and not negative");
  if (g->scale > 0.f && g->scale < FLT_MIN) return fail(RT_ERR_INVALID, "scale is below the smallest normal number");
  const int esz = kv->dtype == RT_BF16 ? 2 : 4;
  const int64_t cols = (int64_t)g->n_q_heads * kv->head_dim;
  if (tensors && g->n_rows > 0) {
    if ((st = check_tensor("q", g->q, g->ldq, cols, esz))) return st;
    if ((st = check_tensor("out", g->out, g->ldo, cols, esz))) return st;
  }
  PagedAttnArgs a{};
  a.r = rows_of(kv, g->n_seqs, g->n_rows, g->n_q_heads, g->row_start, g->kv_len);
  a.q = g->q; a.ldq = g->ldq; a.out = g->out; a.ldo = g->ldo; a.packed = 0;
  a.scale = g->scale > 0.f ? g->scale : 1.0f / sqrtf((float)kv->head_dim);
  a.window = g->window; a.sinks = g->sinks; a.prefix = g->prefix_len;
  // (unknown: what a sequence has on the average over as many as can have any)
  const int n = g->n_seqs < g->n_rows ? g->n_seqs : g->n_rows;
  a.max_rows = !g->row_start    ? a.r.rows_each
               : g->max_rows == 0 ? (int)(n > 0 ? ((long)g->n_rows + n - 1) / n : 0)
                                  : g->max_rows < g->n_rows ? g->max_rows : g->n_rows;
  a.max_kv = (int)(g->max_kv > 0 && g->max_kv < cap ? g->max_kv : cap);
  *out = a;
  return RT_OK;
}
static size_t ws_bytes_of(const PagedAttnArgs& a, const PagedPlan& p, size_t* ml_off) {
  size_t ml;
  const size_t o = paged_part_floats(a, p, &ml);
  *ml_off = rup(o * 4, 256);
  return *ml_off + rup(ml * 4, 256);
}
static int attention(const rt_paged_kv* kv, const rt_attn_args* g, void* ws, size_t ws_bytes, hipStream_t s,
                     const char* what) {
  PagedAttnArgs a;
  const int st = attn_args(kv, g, true, &a);
  if (st) return st;
  if (g->n_rows == 0) return RT_OK;
  const int esz = kv->dtype == RT_BF16 ? 2 : 4;
  const PagedPlan p = paged_plan(a, esz);
  size_t ml_off;
  const size_t need = ws_bytes_of(a, p, &ml_off);
  if (need) {
    if (!ws) return fail(RT_ERR_WORKSPACE, "workspace is null, %zu bytes are needed", need);
    if ((uintptr_t)ws % 256) return fail(RT_ERR_WORKSPACE, "workspace must be 256-byte aligned");
    if (ws_bytes < need) return fail(RT_ERR_WORKSPACE, "workspace has %zu bytes, needs %zu", ws_bytes, need);
    a.part_o = (float*)ws;
    a.part_ml = (float*)((char*)ws + ml_off);
  }
  for (int i = 0; i < p.launches(); ++i) {
    const int e = launched(esz == 2 ? paged_launch<bf16_t>(a, p, i, s) : paged_launch<float>(a, p, i, s), what);
    if (e) return e;
  }
  return RT_OK;
}

}  // namespace rt

using namespace rt;

extern "C" {

int rt_kv_append(const rt_paged_kv* kv, const rt_append_args* args, void* hip_stream) {
  try {
    return kv_append(kv, args, (hipStream_t)hip_stream);
  } catch (...) {
    return fail(RT_ERR_INVALID, "unexpected exception in rt_kv_append");
  }
}

size_t rt_attn_workspace_bytes(const rt_paged_kv* kv, const rt_attn_args* args) {
  try {
    PagedAttnArgs a;
    if (attn_args(kv, args, false, &a) != RT_OK || a.r.n_rows == 0) return 0;
    size_t ml_off;
    return ws_bytes_of(a, paged_plan(a, kv->dtype == RT_BF16 ? 2 : 4), &ml_off);
  } catch (...) {
    (void)fail(RT_ERR_INVALID, "unexpected exception in rt_attn_workspace_bytes");
    return 0;
  }
}

int rt_debug_attn_choice(const rt_paged_kv* kv, const rt_attn_args* args, int32_t choice) {
  try {
    PagedAttnArgs a;
    const int st = attn_args(kv, args, false, &a);
    if (st) return st;
    if (a.r.n_rows == 0) return fail(RT_ERR_INVALID, "a call without rows launches nothing");
    const int esz = kv->dtype == RT_BF16 ? 2 : 4;
    const PagedPlan p = paged_plan(a, esz);
    const PagedChoice c = paged_choice(a, p, esz);
    switch (choice) {
      case RT_A_KERNEL: return c.kernel;
      case RT_A_STREAMED: return c.streamed;
      case RT_A_SPLITS: return p.splits;
      case RT_A_PREFIX_SPLITS: return p.shared;
      default: return fail(RT_ERR_INVALID, "unknown choice %d", choice);
    }
  } catch (...) {
    return fail(RT_ERR_INVALID, "unexpected exception in rt_debug_attn_choice");
  }
}

int rt_window_attention(const rt_paged_kv* kv, const rt_attn_args* args, void* d_workspace, size_t ws_bytes,
                        void* hip_stream) {
  try {
    if (args && args->window < 1) return fail(RT_ERR_INVALID, "window must be at least 1");
    if (args && args->prefix_len != 0) return fail(RT_ERR_INVALID, "window attention takes no shared prefix");
    return attention(kv, args, d_workspace, ws_bytes, (hipStream_t)hip_stream, "rt_window_attention");
  } catch (...) {
    return fail(RT_ERR_INVALID, "unexpected exception in rt_window_attention");
  }
}

int rt_prefix_attention(const rt_paged_kv* kv, const rt_attn_args* args, void* d_workspace, size_t ws_bytes,
                        void* hip_stream) {
  try {
    if (args && (args->window != 0 || args->sinks != 0)) return fail(RT_ERR_INVALID, "prefix attention takes no window");
    return attention(kv, args, d_workspace, ws_bytes, (hipStream_t)hip_stream, "rt_prefix_attention");
  } catch (...) {
    return fail(RT_ERR_INVALID, "unexpected exception in rt_prefix_attention");
  }
}

}  // extern "C"
