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

// The bytes of an array: n rows, one every `stride` bytes (a whole array is one row).  Rows without a pointer are nowhere.
struct Bytes {
  intptr_t at = 0;
  long long row = 0, stride = 0, n = 0;
  Bytes() = default;
  Bytes(const void* p, long long bytes) : at(reinterpret_cast<intptr_t>(p)), row(bytes), stride(bytes), n(p && bytes > 0 ? 1 : 0) {}
  Bytes(const void* p, int dtype, long long stride_, long long row_, long long rows) : Bytes(p, row_ * esize(dtype)) {
    if (!n || rows <= 1 || stride_ == row_) { row *= rows; stride = row; n = p && row > 0 ? 1 : 0; }
    else { stride = stride_ * esize(dtype); n = rows; }
  }
  bool operator==(const Bytes& b) const { return at == b.at && row == b.row && stride == b.stride && n == b.n; }
  intptr_t end() const { return at + (n - 1) * stride + row; }
  bool meets(intptr_t from, intptr_t to) const {                               // whether a row shares bytes with [from, to)
    const long long i = from < at + row ? 0 : (from - at - row) / stride + 1;  // the first row that ends behind `from`
    return i < n && at + i * stride < to;
  }
};
// Whether two arrays share bytes.  Rows of one stride may lie in turn in one array (queries, keys and values of a projection).
bool overlap(const Bytes& a, const Bytes& b) {
  if (!a.n || !b.n || a.at >= b.end() || b.at >= a.end()) return false;
  if (a.n == 1) return b.meets(a.at, a.end());
  if (b.n == 1) return a.meets(b.at, b.end());
  if (a.stride == b.stride) {
    const long long d = ((b.at - a.at) % a.stride + a.stride) % a.stride;      // where b's rows begin between the beginnings of a's
    return d < a.row || a.stride - d < b.row;
  }
  // rows of two strides in one stretch of memory: most such calls end with the first
  for (long long i = b.at < a.at + a.row ? 0 : (b.at - a.at - a.row) / a.stride + 1; i < a.n && a.at + i * a.stride < b.end(); ++i)
    if (b.meets(a.at + i * a.stride, a.at + i * a.stride + a.row)) return true;
  return false;
}
// Whether one of the arrays that a call writes lies on another one, or on one that it reads.
template <size_t N, size_t M>
bool outputs_meet(const Bytes (&outs)[N], const Bytes (&ins)[M]) {
  for (size_t i = 0; i < N; ++i) {
    for (size_t j = 0; j < i; ++j) if (overlap(outs[i], outs[j])) return true;
    for (const Bytes& in : ins) if (overlap(outs[i], in)) return true;
  }
  return false;
}
// an input that an output may replace in its place
Bytes unless(const Bytes& in, const Bytes& out) { return in == out ? Bytes() : in; }

struct Pools {
  Bytes k, v, k_exp, v_exp, table, status;
  explicit Pools(const rt_paged_cache* c) : table(c->page_table, 4LL * c->n_seqs * c->max_pages), status(c->status, 4) {
    const long long head_rows = (long long)c->n_pages * c->n_kv_heads * c->page_size, bytes = head_rows * c->head_dim * (c->dtype == RT_E4M3 ? 1 : esize(c->dtype));
    k = Bytes(c->k, bytes); v = Bytes(c->v, bytes);
    k_exp = Bytes(c->k_exp, head_rows); v_exp = Bytes(c->v_exp, head_rows);
  }
};

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
  const Pools to(cache);
  const Bytes outs[] = {to.k, to.v, to.k_exp, to.v_exp};
  const Bytes ins[] = {Bytes(k, dtype, k_stride, row, rows), Bytes(v, dtype, v_stride, row, rows), Bytes(seq, 4LL * rows), Bytes(pos, 4LL * rows), to.table, to.status};
  if (outputs_meet(outs, ins)) return RT_ERR_INVALID_ARG;
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
  const Pools from(cache);
  const Bytes outs[] = {Bytes(k, dtype, k_stride, row, rows), Bytes(v, dtype, v_stride, row, rows)};
  const Bytes ins[] = {from.k, from.v, from.k_exp, from.v_exp, from.table, from.status, Bytes(seq, 4LL * rows), Bytes(pos, 4LL * rows)};
  if (outputs_meet(outs, ins)) return RT_ERR_INVALID_ARG;
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
  const Pools from(cache);
  const Bytes out(q->out, q->dtype, q->out_stride, row, B), lse(q->lse, 4 * B * q->n_heads);
  const Bytes ins[] = {Bytes(q->q, q->dtype, q->q_stride, row, B), Bytes(q->k_own, q->dtype, q->k_own_stride, kv_row, B), Bytes(q->v_own, q->dtype, q->v_own_stride, kv_row, B),
                       Bytes(q->lens, 4 * B), Bytes(q->alibi_slopes, 4LL * q->n_heads), from.k, from.v, from.k_exp, from.v_exp, from.table, from.status};
  for (int i = 0; i < 3; ++i) if (overlap(out, ins[i])) return RT_ERR_INVALID_ARG;
  const size_t need = paged_attn_workspace(cache, q->n_heads);
  if (workspace_bytes < need) return RT_ERR_WORKSPACE;
  const Bytes outs[] = {out, lse, Bytes(workspace, (long long)need)};
  if (outputs_meet(outs, ins)) return RT_ERR_INVALID_ARG;
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
  const Bytes qi(q, t, q_stride, qrow, rows), qo(q_out, t, q_out_stride, qrow, rows), ki = krow ? Bytes(k, t, k_stride, krow, rows) : Bytes(),
              ko = krow ? Bytes(k_out, t, k_out_stride, krow, rows) : Bytes();
  const Bytes outs[] = {qo, ko}, ins[] = {Bytes(g_q, qrow * esize(t)), krow ? Bytes(g_k, krow * esize(t)) : Bytes(), Bytes(pos, 4LL * rows)};
  if (outputs_meet(outs, ins) || overlap(qo, unless(qi, qo)) || overlap(ko, unless(ki, ko)) || overlap(qo, ki) || overlap(ko, qi)) return RT_ERR_INVALID_ARG;
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
  const int t = cfg->dtype;
  const Bytes dqo(dq_out, 4 * qrow * rows), dko = krow ? Bytes(dk_out, 4 * krow * rows) : Bytes(), dqi(dq, 4 * qrow * rows), dki = krow ? Bytes(dk, 4 * krow * rows) : Bytes();
  const Bytes outs[] = {dqi, dki, Bytes(dg_q, 4 * qrow), krow ? Bytes(dg_k, 4 * krow) : Bytes()};
  const Bytes ins[] = {Bytes(q, t, q_stride, qrow, rows), krow ? Bytes(k, t, k_stride, krow, rows) : Bytes(), Bytes(g_q, qrow * esize(t)),
                       krow ? Bytes(g_k, krow * esize(t)) : Bytes(), Bytes(pos, 4LL * rows)};
  if (outputs_meet(outs, ins) || overlap(dqi, unless(dqo, dqi)) || overlap(dki, unless(dko, dki)) || overlap(dqi, dko) || overlap(dki, dqo) || overlap(outs[2], dqo) ||
      overlap(outs[2], dko) || overlap(outs[3], dqo) || overlap(outs[3], dko))
    return RT_ERR_INVALID_ARG;
  const size_t need = rotate_backward_workspace(cfg->n_heads + cfg->n_kv_heads, cfg->head_dim, rows);
  if (workspace_bytes < need) return RT_ERR_WORKSPACE;
  if (dg_q || (krow && dg_k)) {                                                // (otherwise nothing is written there)
    const Bytes ws[] = {Bytes(workspace, (long long)need)}, all[] = {outs[0], outs[1], outs[2], outs[3], ins[0], ins[1], ins[2], ins[3], ins[4], dqo, dko};
    if (outputs_meet(ws, all)) return RT_ERR_INVALID_ARG;
  }
  if ((st = on_current_device(workspace)) != RT_OK) return st;
  RotateParams p;
  rotate_fill(cfg, &p);
  p.q = q; p.k = k; p.q_stride = q_stride; p.k_stride = k_stride; p.g_q = g_q; p.g_k = g_k; p.pos = pos; p.rows = rows;
  p.dq_out = dq_out; p.dk_out = dk_out; p.dq = dq; p.dk = dk; p.dg_q = dg_q; p.dg_k = krow ? dg_k : nullptr;
  return rotate_backward_launch(cfg->dtype, p, workspace, (cudaStream_t)cuda_stream) == cudaSuccess ? RT_OK : RT_ERR_CUDA;
}

}  // extern "C"
