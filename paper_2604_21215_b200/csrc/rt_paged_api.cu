// C ABI of the operators around paged caches (see include/rt.h): argument checks and dispatch.
#include <math.h>
#include <string.h>

#include "rt_paged.h"

using namespace rt;

namespace {

bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }
bool aligned4(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 3) == 0; }
bool storage_type(int dtype) { return dtype == RT_F32 || dtype == RT_BF16; }
long long esize(int dtype) { return dtype == RT_F32 ? 4 : 2; }

// pointers and numbers that make sense; RT_ERR_UNSUPPORTED for those that this build has no kernel for
rt_status cache_ok(const rt_paged_cache* c) {
  if (!c || !c->k || !c->v || !c->page_table || c->n_pages <= 0 || c->page_size <= 0 || c->n_kv_heads <= 0 || c->head_dim <= 0 || c->n_seqs <= 0 ||
      c->max_pages <= 0)
    return RT_ERR_INVALID_ARG;
  if (!storage_type(c->dtype) && c->dtype != RT_E4M3) return RT_ERR_INVALID_ARG;
  if ((c->dtype == RT_E4M3) != (c->k_exp != nullptr) || (c->dtype == RT_E4M3) != (c->v_exp != nullptr)) return RT_ERR_INVALID_ARG;
  if (!aligned16(c->k) || !aligned16(c->v) || !aligned16(c->k_exp) || !aligned16(c->v_exp)) return RT_ERR_INVALID_ARG;
  if (!aligned4(c->page_table) || !aligned4(c->status)) return RT_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return RT_ERR_UNSUPPORTED;
  if (c->page_size < 16 || c->page_size > 256 || (c->page_size & (c->page_size - 1))) return RT_ERR_UNSUPPORTED;
  // (a page's bytes and the heads of all sequences are counted in 32 bits)
  if ((long long)c->n_kv_heads * c->page_size * c->head_dim > INT32_MAX / 4 || (long long)c->n_seqs * c->n_kv_heads > INT32_MAX) return RT_ERR_UNSUPPORTED;
  return RT_OK;
}

int log2_of(int n) { int r = 0; while ((1 << r) < n) ++r; return r; }

// rows of `row` elements at `stride` elements (a pointer without rows may be anything)
bool rows_ok(const void* p, int dtype, long long stride, long long row, long long rows) {
  if (rows == 0) return true;
  if (!p || !aligned16(p)) return false;
  return rows == 1 || (stride >= row && stride <= INT64_MAX / 16 / rows && stride * esize(dtype) % 16 == 0);
}

// Whether two arrays of such rows share bytes.  Rows of one stride may lie in turn in one array (queries, keys and values of a projection); rows of two strides are
// taken to overlap only where the arrays begin at the same place.
bool rows_overlap(const void* a, int dtype_a, long long stride_a, long long row_a, const void* b, int dtype_b, long long stride_b, long long row_b, long long rows) {
  if (rows == 0) return false;
  const long long ra = row_a * esize(dtype_a), rb = row_b * esize(dtype_b), sa = rows > 1 ? stride_a * esize(dtype_a) : ra, sb = rows > 1 ? stride_b * esize(dtype_b) : rb;
  const intptr_t pa = reinterpret_cast<intptr_t>(a), pb = reinterpret_cast<intptr_t>(b);
  if (pa >= pb + (rows - 1) * sb + rb || pb >= pa + (rows - 1) * sa + ra) return false;
  if (rows == 1 || (sa == ra && sb == rb)) return true;
  if (sa != sb) return pa == pb;
  const long long d = ((pb - pa) % sa + sa) % sa;                              // where b's rows begin between the beginnings of a's
  return d < ra || sa - d < rb;
}
// Whether the bytes of an array lie in a cache's pools, or the pools in one another.
bool ranges_overlap(const void* a, long long na, const void* b, long long nb) {
  const intptr_t pa = reinterpret_cast<intptr_t>(a), pb = reinterpret_cast<intptr_t>(b);
  return a && b && pa < pb + nb && pb < pa + na;
}
struct Pools {
  const void* at[4];
  long long bytes[4];
  explicit Pools(const rt_paged_cache* c) : at{c->k, c->v, c->k_exp, c->v_exp} {
    const long long heads_rows = (long long)c->n_pages * c->n_kv_heads * c->page_size;
    bytes[0] = bytes[1] = heads_rows * c->head_dim * (c->dtype == RT_E4M3 ? 1 : esize(c->dtype));
    bytes[2] = bytes[3] = heads_rows;
  }
  bool meet(const void* p, long long n, int first = 0) const {
    for (int i = first; i < 4; ++i) if (ranges_overlap(p, n, at[i], bytes[i])) return true;
    return false;
  }
  bool meet_each_other() const { return meet(at[0], bytes[0], 1) || meet(at[1], bytes[1], 2) || meet(at[2], bytes[2], 3); }
};
long long extent(int dtype, long long stride, long long row, long long rows) { return ((rows - 1) * (rows > 1 ? stride : 0) + row) * esize(dtype); }
bool same_rows(const void* a, long long stride_a, const void* b, long long stride_b, long long rows) { return a == b && (rows <= 1 || stride_a == stride_b); }

// The pointer is memory of the current device (a pointer of another one would be a fault on the GPU, not an error).
rt_status on_current_device(const void* p) {
  int dev = 0;
  cudaPointerAttributes a;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaPointerGetAttributes(&a, p) != cudaSuccess) { cudaGetLastError(); return RT_ERR_CUDA; }
  if (a.type == cudaMemoryTypeManaged) return RT_OK;
  return a.type == cudaMemoryTypeDevice && a.device == dev ? RT_OK : RT_ERR_INVALID_ARG;
}

rt_status cache_rows(const rt_paged_cache* c, int32_t dtype, const void* k, const void* v, int64_t k_stride, int64_t v_stride, const int32_t* seq,
                     const int32_t* pos, int32_t rows, CacheRowsParams* p) {
  const rt_status st = cache_ok(c);
  if (st != RT_OK) return st;
  if (!storage_type(dtype) || rows < 0) return RT_ERR_INVALID_ARG;
  const long long row = (long long)c->n_kv_heads * c->head_dim;
  if (!rows_ok(k, dtype, k_stride, row, rows) || !rows_ok(v, dtype, v_stride, row, rows)) return RT_ERR_INVALID_ARG;
  if (rows > 0 && (!seq || !pos || !aligned4(seq) || !aligned4(pos))) return RT_ERR_INVALID_ARG;
  memset(p, 0, sizeof(*p));
  p->c = *c;
  p->log_page = log2_of(c->page_size);
  p->k_stride = k_stride; p->v_stride = v_stride; p->seq = seq; p->pos = pos; p->rows = rows;
  return RT_OK;
}

rt_status rotate_ok(const rt_rotate_config* c, int32_t rows) {
  if (!c || !storage_type(c->dtype) || c->n_heads <= 0 || c->n_kv_heads < 0 || c->head_dim <= 0 || rows < 0) return RT_ERR_INVALID_ARG;
  if ((c->norm_flags & ~RT_NORM_QK) || !(c->rms_eps >= 0.f) || !isfinite(c->rms_eps)) return RT_ERR_INVALID_ARG;
  if (c->rot_dim < 0 || c->rot_dim > c->head_dim || (c->pairs != RT_PAIRS_HALVES && c->pairs != RT_PAIRS_NEIGHBOURS)) return RT_ERR_INVALID_ARG;
  if (c->rot_dim > 0 && !c->freq) return RT_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return RT_ERR_UNSUPPORTED;
  if (c->rot_dim % 16 || (long long)c->n_heads + c->n_kv_heads > 65535) return RT_ERR_UNSUPPORTED;
  for (int i = 0; i < c->rot_dim / 2; ++i) if (!isfinite(c->freq[i])) return RT_ERR_INVALID_ARG;
  return RT_OK;
}

void rotate_fill(const rt_rotate_config* c, RotateParams* p) {
  memset(p, 0, sizeof(*p));
  p->n_heads = c->n_heads; p->n_kv = c->n_kv_heads; p->hd = c->head_dim;
  p->norm = (c->norm_flags & RT_NORM_QK) != 0; p->rot = c->rot_dim; p->neighbours = c->pairs == RT_PAIRS_NEIGHBOURS;
  p->eps = c->rms_eps;
  for (int i = 0; i < c->rot_dim / 2; ++i) {
    double t = c->freq[i] / 6.283185307179586476925286766559;
    constexpr double kWhole = 6755399441055744.0;                             // 1.5 * 2^52: adding it rounds to a whole number (rint is a call, and there are up to 64)
    t -= fabs(t) < 1e15 ? (t + kWhole) - kWhole : rint(t);                     // (exact)
    const unsigned long long n = (unsigned long long)(fabs(t) * 18446744073709551616.0);      // 2^64 of them a turn; at most 2^63
    p->turns[i] = t < 0 ? 0 - n : n;
  }
}

}  // namespace

extern "C" {

rt_status rt_cache_write(const rt_paged_cache* cache, int32_t dtype, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                         const int32_t* seq, const int32_t* pos, int32_t rows, void* cuda_stream) {
  CacheRowsParams p;
  rt_status st = cache_rows(cache, dtype, k, v, k_stride, v_stride, seq, pos, rows, &p);
  if (st != RT_OK || rows == 0) return st;
  const long long row = (long long)cache->n_kv_heads * cache->head_dim;
  const Pools pools(cache);
  if (pools.meet_each_other() || pools.meet(k, extent(dtype, k_stride, row, rows)) || pools.meet(v, extent(dtype, v_stride, row, rows))) return RT_ERR_INVALID_ARG;
  if ((st = on_current_device(cache->k)) != RT_OK) return st;
  p.k_in = k; p.v_in = v;
  return cache_write_launch(dtype, p, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

rt_status rt_cache_read(const rt_paged_cache* cache, int32_t dtype, void* k, void* v, int64_t k_stride, int64_t v_stride, const int32_t* seq,
                        const int32_t* pos, int32_t rows, void* cuda_stream) {
  CacheRowsParams p;
  rt_status st = cache_rows(cache, dtype, k, v, k_stride, v_stride, seq, pos, rows, &p);
  if (st != RT_OK || rows == 0) return st;
  const long long row = (long long)cache->n_kv_heads * cache->head_dim;
  const Pools pools(cache);
  if (rows_overlap(k, dtype, k_stride, row, v, dtype, v_stride, row, rows) || pools.meet(k, extent(dtype, k_stride, row, rows)) ||
      pools.meet(v, extent(dtype, v_stride, row, rows)))
    return RT_ERR_INVALID_ARG;
  if ((st = on_current_device(cache->k)) != RT_OK) return st;
  p.k_out = k; p.v_out = v;
  return cache_read_launch(dtype, p, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

size_t rt_paged_attention_workspace_bytes(const rt_paged_cache* cache, int32_t n_heads) {
  if (cache_ok(cache) != RT_OK || n_heads <= 0 || n_heads % cache->n_kv_heads || !paged_attn_counts(cache, n_heads)) return 0;
  return paged_attn_workspace(cache, n_heads);
}

rt_status rt_paged_attention(const rt_paged_cache* cache, const rt_paged_query* q, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  rt_status st = cache_ok(cache);
  if (st != RT_OK) return st;
  if (!q || !storage_type(q->dtype) || q->n_heads <= 0 || q->n_heads % cache->n_kv_heads || !isfinite(q->softmax_scale)) return RT_ERR_INVALID_ARG;
  if (!q->lens || !workspace || !aligned16(workspace) || !aligned4(q->lens) || !aligned4(q->lse) || !aligned4(q->alibi_slopes))
    return RT_ERR_INVALID_ARG;
  const long long B = cache->n_seqs, row = (long long)q->n_heads * cache->head_dim, kv_row = (long long)cache->n_kv_heads * cache->head_dim;
  if (!rows_ok(q->q, q->dtype, q->q_stride, row, B) || !rows_ok(q->out, q->dtype, q->out_stride, row, B)) return RT_ERR_INVALID_ARG;
  if ((q->k_own != nullptr) != (q->v_own != nullptr)) return RT_ERR_INVALID_ARG;
  if (q->k_own && (!rows_ok(q->k_own, q->dtype, q->k_own_stride, kv_row, B) || !rows_ok(q->v_own, q->dtype, q->v_own_stride, kv_row, B)))
    return RT_ERR_INVALID_ARG;
  if (q->n_heads / cache->n_kv_heads > 1024 || !paged_attn_counts(cache, q->n_heads)) return RT_ERR_UNSUPPORTED;
  if (rows_overlap(q->out, q->dtype, q->out_stride, row, q->q, q->dtype, q->q_stride, row, B) ||
      (q->k_own && (rows_overlap(q->out, q->dtype, q->out_stride, row, q->k_own, q->dtype, q->k_own_stride, kv_row, B) ||
                    rows_overlap(q->out, q->dtype, q->out_stride, row, q->v_own, q->dtype, q->v_own_stride, kv_row, B))))
    return RT_ERR_INVALID_ARG;
  if (workspace_bytes < paged_attn_workspace(cache, q->n_heads)) return RT_ERR_WORKSPACE;
  const Pools pools(cache);
  if (pools.meet(q->out, extent(q->dtype, q->out_stride, row, B)) || pools.meet(q->lse, 4 * B * q->n_heads)) return RT_ERR_INVALID_ARG;
  if ((st = on_current_device(cache->k)) != RT_OK) return st;
  PagedAttnParams p;
  memset(&p, 0, sizeof(p));
  p.c = *cache; p.q = *q;
  p.log_page = log2_of(cache->page_size);
  p.group = q->n_heads / cache->n_kv_heads;
  p.scale_log2 = q->softmax_scale * kLog2e;
  return paged_attn_launch(p, workspace, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

rt_status rt_qk_rotate(const rt_rotate_config* cfg, const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* g_q, const void* g_k,
                       const int32_t* pos, int32_t rows, void* q_out, void* k_out, int64_t q_out_stride, int64_t k_out_stride, void* cuda_stream) {
  rt_status st = rotate_ok(cfg, rows);
  if (st != RT_OK) return st;
  const long long qrow = (long long)cfg->n_heads * cfg->head_dim, krow = (long long)cfg->n_kv_heads * cfg->head_dim;
  if (!rows_ok(q, cfg->dtype, q_stride, qrow, rows) || !rows_ok(q_out, cfg->dtype, q_out_stride, qrow, rows) || !aligned16(g_q) ||
      (rows > 0 && (!pos || !aligned4(pos))))
    return RT_ERR_INVALID_ARG;
  if (krow && (!rows_ok(k, cfg->dtype, k_stride, krow, rows) || !rows_ok(k_out, cfg->dtype, k_out_stride, krow, rows) || !aligned16(g_k)))
    return RT_ERR_INVALID_ARG;
  if (rows == 0) return RT_OK;
  const int t = cfg->dtype;
  if (!same_rows(q, q_stride, q_out, q_out_stride, rows) && rows_overlap(q, t, q_stride, qrow, q_out, t, q_out_stride, qrow, rows)) return RT_ERR_INVALID_ARG;
  if (krow && ((!same_rows(k, k_stride, k_out, k_out_stride, rows) && rows_overlap(k, t, k_stride, krow, k_out, t, k_out_stride, krow, rows)) ||
               rows_overlap(q_out, t, q_out_stride, qrow, k_out, t, k_out_stride, krow, rows) || rows_overlap(q_out, t, q_out_stride, qrow, k, t, k_stride, krow, rows) ||
               rows_overlap(k_out, t, k_out_stride, krow, q, t, q_stride, qrow, rows)))
    return RT_ERR_INVALID_ARG;
  if ((st = on_current_device(q)) != RT_OK) return st;
  RotateParams p;
  rotate_fill(cfg, &p);
  p.q = q; p.k = k; p.q_stride = q_stride; p.k_stride = k_stride; p.g_q = g_q; p.g_k = g_k; p.pos = pos; p.rows = rows;
  p.q_out = q_out; p.k_out = k_out; p.qo_stride = q_out_stride; p.ko_stride = k_out_stride;
  return rotate_launch(cfg->dtype, p, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

size_t rt_qk_rotate_backward_workspace_bytes(const rt_rotate_config* cfg, int32_t rows) {
  if (rotate_ok(cfg, rows) != RT_OK) return 0;
  return rotate_backward_workspace(cfg->n_heads + cfg->n_kv_heads, cfg->head_dim, rows);
}

rt_status rt_qk_rotate_backward(const rt_rotate_config* cfg, const void* q, const void* k, int64_t q_stride, int64_t k_stride, const void* g_q,
                                const void* g_k, const int32_t* pos, int32_t rows, const float* dq_out, const float* dk_out, float* dq, float* dk,
                                float* dg_q, float* dg_k, void* workspace, size_t workspace_bytes, void* cuda_stream) {
  rt_status st = rotate_ok(cfg, rows);
  if (st != RT_OK) return st;
  const long long qrow = (long long)cfg->n_heads * cfg->head_dim, krow = (long long)cfg->n_kv_heads * cfg->head_dim;
  if (!rows_ok(q, cfg->dtype, q_stride, qrow, rows) || !rows_ok(dq_out, RT_F32, qrow, qrow, rows) || !rows_ok(dq, RT_F32, qrow, qrow, rows) ||
      !aligned16(g_q) || !aligned16(dg_q) || (rows > 0 && (!pos || !aligned4(pos))) || !workspace || !aligned16(workspace))
    return RT_ERR_INVALID_ARG;
  if (krow && (!rows_ok(k, cfg->dtype, k_stride, krow, rows) || !rows_ok(dk_out, RT_F32, krow, krow, rows) || !rows_ok(dk, RT_F32, krow, krow, rows) ||
               !aligned16(g_k) || !aligned16(dg_k)))
    return RT_ERR_INVALID_ARG;
  auto clash = [&](const void* a, long long ra, const void* b, long long rb) { return rows_overlap(a, RT_F32, ra, ra, b, RT_F32, rb, rb, rows); };
  if ((dq != dq_out && clash(dq, qrow, dq_out, qrow)) || rows_overlap(dq, RT_F32, qrow, qrow, q, cfg->dtype, q_stride, qrow, rows)) return RT_ERR_INVALID_ARG;
  if (krow && ((dk != dk_out && clash(dk, krow, dk_out, krow)) || clash(dq, qrow, dk, krow) || clash(dq, qrow, dk_out, krow) || clash(dk, krow, dq_out, qrow) ||
               rows_overlap(dk, RT_F32, krow, krow, k, cfg->dtype, k_stride, krow, rows) || rows_overlap(dq, RT_F32, qrow, qrow, k, cfg->dtype, k_stride, krow, rows) ||
               rows_overlap(dk, RT_F32, krow, krow, q, cfg->dtype, q_stride, qrow, rows) || ranges_overlap(dg_q, 4 * qrow, dg_k, 4 * krow)))
    return RT_ERR_INVALID_ARG;
  if (workspace_bytes < rotate_backward_workspace(cfg->n_heads + cfg->n_kv_heads, cfg->head_dim, rows)) return RT_ERR_WORKSPACE;
  if ((st = on_current_device(workspace)) != RT_OK) return st;
  RotateParams p;
  rotate_fill(cfg, &p);
  p.q = q; p.k = k; p.q_stride = q_stride; p.k_stride = k_stride; p.g_q = g_q; p.g_k = g_k; p.pos = pos; p.rows = rows;
  p.dq_out = dq_out; p.dk_out = dk_out; p.dq = dq; p.dk = dk; p.dg_q = dg_q; p.dg_k = krow ? dg_k : nullptr;
  return rotate_backward_launch(cfg->dtype, p, workspace, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

}  // extern "C"
