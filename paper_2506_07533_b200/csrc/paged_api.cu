// C ABI of the paged caches (16-bit and 4-bit): argument validation and dispatch to the kernel launchers.
#include <math.h>

#include <new>
#include <vector>

#include "paged4.cuh"

namespace {

using moqae::AttnOptions;
using moqae::PagedView;
using moqae::RopeView;
using moqae::RowsView;

int cuda_rc(cudaError_t e) {
  if (e == cudaSuccess) return MOQAE_OK;
  moqae::record_cuda_error(e);
  return MOQAE_ERR_CUDA;
}

bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool known_dtype(int d) { return d == MOQAE_DTYPE_FP16 || d == MOQAE_DTYPE_BF16; }

// what caches of both kinds check: sizes, tables
template <typename C> int check_tables(const C* c, PagedView* v) {
  if (!known_dtype(c->dtype)) return MOQAE_ERR_UNSUPPORTED;
  if (c->n_pages < 0 || c->n_kv_heads < 1 || c->batch < 0 || c->max_pages < 0) return MOQAE_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 8 && (1 << shift) != c->page_size) ++shift;
  if ((1 << shift) != c->page_size) return MOQAE_ERR_UNSUPPORTED;
  // positions, and differences of them, are 32-bit
  if (static_cast<int64_t>(c->max_pages) * c->page_size > (1ll << 30)) return MOQAE_ERR_UNSUPPORTED;
  v->table = c->block_table;
  v->kv_len = c->kv_len;
  v->status = c->status;
  v->n_pages = c->n_pages;
  v->page_size = c->page_size;
  v->page_shift = shift;
  v->n_kv_heads = c->n_kv_heads;
  v->batch = c->batch;
  v->max_pages = c->max_pages;
  v->dtype = c->dtype;
  return MOQAE_OK;
}
template <typename C> int check_table_pointers(const C* c) {
  if (c->batch > 0 && (!c->kv_len || (c->max_pages > 0 && !c->block_table))) return MOQAE_ERR_INVALID_ARG;
  return !aligned(c->block_table, 4) || !aligned(c->kv_len, 4) || !aligned(c->status, 16) ? MOQAE_ERR_MISALIGNED : MOQAE_OK;
}

int check_pages(const moqae_paged_cache* c, PagedView* v) {
  if (!c) return MOQAE_ERR_INVALID_ARG;
  *v = PagedView{};
  const int rc = check_tables(c, v);
  if (rc != MOQAE_OK) return rc;
  for (int i = 0; i < 3; ++i) {
    if (c->k_stride[i] <= 0 || c->v_stride[i] <= 0) return MOQAE_ERR_INVALID_ARG;
    if (c->k_stride[i] % 8 != 0 || c->v_stride[i] % 8 != 0) return MOQAE_ERR_MISALIGNED;
  }
  if (c->n_pages > 0 && (!c->k_pages || !c->v_pages)) return MOQAE_ERR_INVALID_ARG;
  const int pointers = check_table_pointers(c);
  if (pointers == MOQAE_ERR_INVALID_ARG) return pointers;
  if (!aligned(c->k_pages, 16) || !aligned(c->v_pages, 16) || pointers != MOQAE_OK) return MOQAE_ERR_MISALIGNED;
  v->k = static_cast<uint16_t*>(c->k_pages);
  v->v = static_cast<uint16_t*>(c->v_pages);
  v->k_page = c->k_stride[0]; v->k_head = c->k_stride[1]; v->k_slot = c->k_stride[2];
  v->v_page = c->v_stride[0]; v->v_head = c->v_stride[1]; v->v_slot = c->v_stride[2];
  return MOQAE_OK;
}

int check_pages(const moqae_paged4_cache* c, PagedView* v) {
  if (!c) return MOQAE_ERR_INVALID_ARG;
  *v = PagedView{};
  const int rc = check_tables(c, v);
  if (rc != MOQAE_OK) return rc;
  if (c->page_stride <= 0 || c->head_stride <= 0) return MOQAE_ERR_INVALID_ARG;
  if (c->page_stride % 16 != 0 || c->head_stride % 16 != 0) return MOQAE_ERR_MISALIGNED;
  const int64_t bytes = static_cast<int64_t>(c->page_size) * moqae::kTokenBytes4;      // of a page and head: they lie apart
  if ((c->n_kv_heads > 1 && c->head_stride < bytes) || (c->n_pages > 1 && c->page_stride < bytes)) return MOQAE_ERR_INVALID_ARG;
  if (c->n_pages > 0 && !c->pages) return MOQAE_ERR_INVALID_ARG;
  const int pointers = check_table_pointers(c);
  if (pointers == MOQAE_ERR_INVALID_ARG) return pointers;
  if (!aligned(c->pages, 16) || pointers != MOQAE_OK) return MOQAE_ERR_MISALIGNED;
  v->k = static_cast<uint16_t*>(c->pages);
  v->k_page = c->page_stride;
  v->k_head = c->head_stride;
  return MOQAE_OK;
}

// NULL rows become rows without heads.  n_rows = 0 allows a NULL data pointer.
int check_rows(const moqae_rows* r, int64_t n_rows, RowsView* v) {
  *v = RowsView{};
  if (!r) return MOQAE_OK;
  if (r->n_heads < 1 || r->token_stride < 0 || r->head_stride < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_rows > 0 && !r->data) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(r->data, 16) || r->token_stride % 8 != 0 || r->head_stride % 8 != 0) return MOQAE_ERR_MISALIGNED;
  v->data = static_cast<uint16_t*>(r->data);
  v->token = r->token_stride;
  v->head = r->head_stride;
  v->n_heads = r->n_heads;
  return MOQAE_OK;
}
// an output's rows lie apart
int check_out_rows(const moqae_rows* r, int64_t n_rows, RowsView* v) {
  const int rc = check_rows(r, n_rows, v);
  if (rc != MOQAE_OK || !r) return rc;
  if ((r->n_heads > 1 && r->head_stride < moqae::kHeadDim) || (n_rows > 1 && r->token_stride < moqae::kHeadDim)) return MOQAE_ERR_INVALID_ARG;
  return MOQAE_OK;
}

int check_rope(const moqae_rope* r, RopeView* v) {
  *v = RopeView{};
  if (!r) return MOQAE_OK;
  if (r->rot_dim < 0 || r->rot_dim > moqae::kHeadDim || r->n_positions < 0) return MOQAE_ERR_INVALID_ARG;
  if (r->rot_dim % 16 != 0) return MOQAE_ERR_UNSUPPORTED;
  if (r->interleaved != 0 && r->interleaved != 1) return MOQAE_ERR_INVALID_ARG;
  if (r->rot_dim > 0 && r->n_positions > 0 && !r->cos_sin) return MOQAE_ERR_INVALID_ARG;
  if (!(r->eps >= 0.0f) || !isfinite(r->eps)) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(r->cos_sin, 16) || !aligned(r->q_weight, 16) || !aligned(r->k_weight, 16)) return MOQAE_ERR_MISALIGNED;
  v->cos_sin = r->cos_sin;
  v->q_weight = static_cast<const uint16_t*>(r->q_weight);
  v->k_weight = static_cast<const uint16_t*>(r->k_weight);
  v->n_positions = r->n_positions;
  v->rot_dim = r->rot_dim;
  v->interleaved = r->interleaved;
  v->eps = r->eps;
  return MOQAE_OK;
}

int check_options(const moqae_attn_options* o, AttnOptions* v) {
  *v = AttnOptions{};
  v->scale = 0.08838834764831845f;               // 1/sqrt(128)
  if (!o) return MOQAE_OK;
  if (!isfinite(o->scale) || !isfinite(o->cap) || o->cap < 0.0f || o->window < 0) return MOQAE_ERR_INVALID_ARG;
  if (o->cap > 0.0f && o->cap < 1e-4f) return MOQAE_ERR_UNSUPPORTED;
  if (!aligned(o->slopes, 4) || !aligned(o->prefix_len, 4)) return MOQAE_ERR_MISALIGNED;
  if (o->scale > 0.0f) v->scale = o->scale;
  v->slopes = o->slopes;
  v->prefix_len = o->prefix_len;
  v->cap = o->cap > 1e30f ? 0.0f : o->cap;       // a cap that no score can feel
  v->window = o->window;
  return MOQAE_OK;
}

int check_group(const PagedView& pv, int n_q_heads) {
  if (n_q_heads < 1 || n_q_heads % pv.n_kv_heads != 0) return MOQAE_ERR_INVALID_ARG;
  return n_q_heads / pv.n_kv_heads > moqae::kMaxQueryGroup ? MOQAE_ERR_UNSUPPORTED : MOQAE_OK;
}

// what both attention calls check
template <typename C>
int check_attention(const C* cache, const moqae_rows* q, const moqae_rows* out, int64_t n_rows,
                    const moqae_attn_options* options, PagedView* pv, RowsView* qv, RowsView* ov, AttnOptions* opt) {
  int rc = check_pages(cache, pv);
  if (rc == MOQAE_OK && (!q || !out)) rc = MOQAE_ERR_INVALID_ARG;
  if (rc == MOQAE_OK) rc = check_rows(q, n_rows, qv);
  if (rc == MOQAE_OK) rc = check_out_rows(out, n_rows, ov);
  if (rc == MOQAE_OK && qv->n_heads != ov->n_heads) rc = MOQAE_ERR_INVALID_ARG;
  if (rc == MOQAE_OK) rc = check_group(*pv, qv->n_heads);
  if (rc == MOQAE_OK) rc = check_options(options, opt);
  // a window as long as the longest sequence hides nothing
  if (rc == MOQAE_OK && opt->window >= static_cast<int64_t>(pv->max_pages) * pv->page_size) opt->window = 0;
  return rc;
}

template <typename C, typename F>
int append_rows(const C* cache, const moqae_rope* rope, const moqae_rows* k, const moqae_rows* v, const moqae_rows* q, const moqae_rows* q_out,
                const int32_t* positions, const int32_t* seq, int32_t n_tokens, void* stream, F launch) {
  PagedView pv;
  int rc = check_pages(cache, &pv);
  if (rc != MOQAE_OK) return rc;
  if (!k || !v || (q == nullptr) != (q_out == nullptr) || n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > 0 && !positions) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(positions, 4) || !aligned(seq, 4)) return MOQAE_ERR_MISALIGNED;
  RopeView rv;
  RowsView kr, vr, qv, qo;
  rc = check_rope(rope, &rv);
  if (rc == MOQAE_OK) rc = check_rows(k, n_tokens, &kr);
  if (rc == MOQAE_OK) rc = check_rows(v, n_tokens, &vr);
  if (rc == MOQAE_OK) rc = check_rows(q, n_tokens, &qv);
  if (rc == MOQAE_OK) rc = check_out_rows(q_out, n_tokens, &qo);
  if (rc != MOQAE_OK) return rc;
  if (kr.n_heads != pv.n_kv_heads || vr.n_heads != pv.n_kv_heads || qv.n_heads != qo.n_heads) return MOQAE_ERR_INVALID_ARG;
  return cuda_rc(launch(pv, rv, qv, qo, kr, vr, positions, seq, n_tokens, static_cast<cudaStream_t>(stream)));
}

template <typename C> int validate_pages(const C* cache, void* stream, int32_t* bad_seq, int32_t* bad_entry) {
  PagedView pv;
  const int rc = check_pages(cache, &pv);
  if (rc != MOQAE_OK) return rc;
  const size_t n = static_cast<size_t>(pv.batch) * pv.max_pages;
  std::vector<int32_t> table, len;
  try {
    table.resize(n);
    len.resize(pv.batch);
  } catch (const std::bad_alloc&) {
    return MOQAE_ERR_UNSUPPORTED;
  }
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  cudaError_t e = cudaSuccess;
  if (n) e = cudaMemcpyAsync(table.data(), pv.table, n * 4, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess && pv.batch) e = cudaMemcpyAsync(len.data(), pv.kv_len, len.size() * 4, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_rc(e);
  return moqae_paged_validate_host(table.data(), len.data(), pv.batch, pv.max_pages, pv.n_pages, pv.page_size, bad_seq, bad_entry);
}

template <typename C> int poll_status_of(const C* cache, void* stream, int32_t* out_status) {
  if (!cache || !out_status) return MOQAE_ERR_INVALID_ARG;
  *out_status = MOQAE_OK;
  if (!cache->status) return MOQAE_OK;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  int32_t h[4] = {0, 0, 0, 0};
  cudaError_t e = cudaMemcpyAsync(h, cache->status, sizeof(h), cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e != cudaSuccess) return cuda_rc(e);
  *out_status = h[0];
  return MOQAE_OK;
}

}  // namespace

#pragma GCC visibility push(default)
extern "C" {

int moqae_norm_rope(const moqae_rope* rope, int32_t dtype, const moqae_rows* q, const moqae_rows* k, const moqae_rows* q_out,
                    const moqae_rows* k_out, const int32_t* positions, int32_t n_tokens, int32_t* status, void* stream) {
  if (!rope || n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (!known_dtype(dtype)) return MOQAE_ERR_UNSUPPORTED;
  if ((q == nullptr) != (q_out == nullptr) || (k == nullptr) != (k_out == nullptr) || (!q && !k)) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > 0 && !positions) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(positions, 4) || !aligned(status, 16)) return MOQAE_ERR_MISALIGNED;
  RopeView rv;
  RowsView qv, kv, qo, ko;
  int rc = check_rope(rope, &rv);
  if (rc == MOQAE_OK) rc = check_rows(q, n_tokens, &qv);
  if (rc == MOQAE_OK) rc = check_rows(k, n_tokens, &kv);
  if (rc == MOQAE_OK) rc = check_out_rows(q_out, n_tokens, &qo);
  if (rc == MOQAE_OK) rc = check_out_rows(k_out, n_tokens, &ko);
  if (rc != MOQAE_OK) return rc;
  if (qv.n_heads != qo.n_heads || kv.n_heads != ko.n_heads) return MOQAE_ERR_INVALID_ARG;
  return cuda_rc(moqae::launch_norm_rope(rv, dtype, qv, kv, qo, ko, positions, n_tokens, status, static_cast<cudaStream_t>(stream)));
}

int moqae_paged_append(const moqae_paged_cache* cache, const moqae_rope* rope, const moqae_rows* k, const moqae_rows* v,
                       const moqae_rows* q, const moqae_rows* q_out, const int32_t* positions, const int32_t* seq,
                       int32_t n_tokens, void* stream) {
  return append_rows(cache, rope, k, v, q, q_out, positions, seq, n_tokens, stream, moqae::launch_paged_append);
}

int moqae_paged_decode_attn_workspace(const moqae_paged_cache* cache, int32_t n_q_heads, int64_t* out_bytes) {
  PagedView pv;
  int rc = check_pages(cache, &pv);
  if (rc == MOQAE_OK) rc = check_group(pv, n_q_heads);
  if (rc != MOQAE_OK) return rc;
  if (!out_bytes) return MOQAE_ERR_INVALID_ARG;
  if (!moqae::paged_decode_fits(pv)) return MOQAE_ERR_UNSUPPORTED;
  *out_bytes = moqae::paged_decode_workspace_bytes(n_q_heads / pv.n_kv_heads);
  return MOQAE_OK;
}

int moqae_paged_decode_attn(const moqae_paged_cache* cache, const moqae_rows* q, const moqae_rows* out,
                            const moqae_attn_options* options, void* workspace, int64_t workspace_bytes, void* stream) {
  PagedView pv;
  RowsView qv, ov;
  AttnOptions opt;
  const int rc = check_attention(cache, q, out, cache ? cache->batch : 0, options, &pv, &qv, &ov, &opt);
  if (rc != MOQAE_OK) return rc;
  if (!workspace) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return MOQAE_ERR_MISALIGNED;
  if (!moqae::paged_decode_fits(pv)) return MOQAE_ERR_UNSUPPORTED;
  if (workspace_bytes < moqae::paged_decode_workspace_bytes(qv.n_heads / pv.n_kv_heads)) return MOQAE_ERR_WORKSPACE_TOO_SMALL;
  return cuda_rc(moqae::launch_paged_decode(pv, qv, ov, opt, workspace, static_cast<cudaStream_t>(stream)));
}

int moqae_paged_prefill_attn_workspace(const moqae_paged_cache* cache, int32_t n_q_heads, int32_t n_tokens, int64_t* out_bytes) {
  PagedView pv;
  int rc = check_pages(cache, &pv);
  if (rc == MOQAE_OK) rc = check_group(pv, n_q_heads);
  if (rc != MOQAE_OK) return rc;
  if (!out_bytes || n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > moqae::kMaxQueryTokens || pv.batch > moqae::kMaxQueryTokens) return MOQAE_ERR_UNSUPPORTED;
  *out_bytes = moqae::paged_prefill_workspace_bytes(pv, n_q_heads / pv.n_kv_heads, n_tokens);
  return MOQAE_OK;
}

int moqae_paged_prefill_attn(const moqae_paged_cache* cache, const moqae_rows* q, const int32_t* cu_q, int32_t n_tokens,
                             const moqae_rows* out, const moqae_attn_options* options, void* workspace, int64_t workspace_bytes,
                             void* stream) {
  PagedView pv;
  RowsView qv, ov;
  AttnOptions opt;
  if (n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > moqae::kMaxQueryTokens || (cache && cache->batch > moqae::kMaxQueryTokens)) return MOQAE_ERR_UNSUPPORTED;
  const int rc = check_attention(cache, q, out, n_tokens, options, &pv, &qv, &ov, &opt);
  if (rc != MOQAE_OK) return rc;
  if (pv.batch > 0 && !cu_q) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(cu_q, 4) || !aligned(workspace, 16)) return MOQAE_ERR_MISALIGNED;
  if (workspace &&
      workspace_bytes < moqae::paged_prefill_workspace_bytes(pv, qv.n_heads / pv.n_kv_heads, n_tokens))
    return MOQAE_ERR_WORKSPACE_TOO_SMALL;
  const cudaError_t e = moqae::launch_paged_prefill(pv, qv, cu_q, n_tokens, ov, opt, workspace, static_cast<cudaStream_t>(stream));
  return e == cudaErrorNotSupported ? MOQAE_ERR_UNSUPPORTED : cuda_rc(e);
}

int moqae_paged_validate_host(const int32_t* block_table, const int32_t* kv_len, int32_t batch, int32_t max_pages, int32_t n_pages,
                              int32_t page_size, int32_t* bad_seq, int32_t* bad_entry) {
  if (batch < 0 || max_pages < 0 || n_pages < 0 || page_size < 1) return MOQAE_ERR_INVALID_ARG;
  if (batch > 0 && (!kv_len || (max_pages > 0 && !block_table))) return MOQAE_ERR_INVALID_ARG;
  auto fail = [&](int b, int e) {
    if (bad_seq) *bad_seq = b;
    if (bad_entry) *bad_entry = e;
    return MOQAE_ERR_CORRUPT_TABLE;
  };
  for (int b = 0; b < batch; ++b) {
    if (kv_len[b] < 0 || kv_len[b] > static_cast<int64_t>(max_pages) * page_size) return fail(b, -1);
    const int used = static_cast<int>((static_cast<int64_t>(kv_len[b]) + page_size - 1) / page_size);
    for (int i = 0; i < used; ++i) {
      const int32_t p = block_table[static_cast<int64_t>(b) * max_pages + i];
      if (p < 0 || p >= n_pages) return fail(b, i);
    }
  }
  return MOQAE_OK;
}

int moqae_paged_validate(const moqae_paged_cache* cache, void* stream, int32_t* bad_seq, int32_t* bad_entry) {
  return validate_pages(cache, stream, bad_seq, bad_entry);
}
int moqae_paged4_validate(const moqae_paged4_cache* cache, void* stream, int32_t* bad_seq, int32_t* bad_entry) {
  return validate_pages(cache, stream, bad_seq, bad_entry);
}

int moqae_paged_poll_status(const moqae_paged_cache* cache, void* stream, int32_t* out_status) { return poll_status_of(cache, stream, out_status); }
int moqae_paged4_poll_status(const moqae_paged4_cache* cache, void* stream, int32_t* out_status) { return poll_status_of(cache, stream, out_status); }

int moqae_paged_plan(const int32_t* past_len, const int32_t* n_new, int32_t batch, int32_t page_size, int32_t max_pages,
                     int32_t* block_table, int32_t* kv_len, const moqae_page_pool* pool, const int32_t* state, int32_t* cu_q,
                     int32_t* positions, int32_t* seq, int32_t n_rows, int32_t* status, void* stream) {
  if (!pool || batch < 0 || max_pages < 0 || n_rows < 0 || pool->n_pages < 0) return MOQAE_ERR_INVALID_ARG;
  int shift = 4;
  while (shift < 8 && (1 << shift) != page_size) ++shift;
  if ((1 << shift) != page_size || static_cast<int64_t>(max_pages) * page_size > (1ll << 30)) return MOQAE_ERR_UNSUPPORTED;
  if (n_rows > moqae::kMaxQueryTokens || batch > moqae::kMaxQueryTokens || pool->n_pages > moqae::kMaxQueryTokens) return MOQAE_ERR_UNSUPPORTED;
  if (!pool->state || (pool->n_pages > 0 && !pool->ring) || !cu_q || (n_rows > 0 && (!positions || !seq))) return MOQAE_ERR_INVALID_ARG;
  if (batch > 0 && (!past_len || !n_new || !kv_len || (max_pages > 0 && !block_table))) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(past_len, 4) || !aligned(n_new, 4) || !aligned(block_table, 4) || !aligned(kv_len, 4) || !aligned(pool->ring, 4) ||
      !aligned(pool->state, 16) || !aligned(state, 4) || !aligned(cu_q, 4) || !aligned(positions, 4) || !aligned(seq, 4) || !aligned(status, 16))
    return MOQAE_ERR_MISALIGNED;
  moqae::PlanJob job{past_len, n_new, block_table, kv_len, cu_q, positions, seq, status, batch, max_pages, shift, n_rows};
  const moqae::PoolView view{pool->ring, state ? state : pool->state, pool->state, pool->n_pages};
  return cuda_rc(moqae::launch_paged_plan(job, view, static_cast<cudaStream_t>(stream)));
}

int moqae_paged4_append(const moqae_paged4_cache* cache, const moqae_rope* rope, const moqae_rows* k, const moqae_rows* v,
                        const moqae_rows* q, const moqae_rows* q_out, const int32_t* positions, const int32_t* seq,
                        int32_t n_tokens, void* stream) {
  return append_rows(cache, rope, k, v, q, q_out, positions, seq, n_tokens, stream, moqae::launch_paged4_append);
}

int moqae_paged4_read(const moqae_paged4_cache* cache, const moqae_rows* k_out, const moqae_rows* v_out, const int32_t* positions,
                      const int32_t* seq, int32_t n_tokens, void* stream) {
  PagedView pv;
  RowsView ko, vo;
  int rc = check_pages(cache, &pv);
  if (rc != MOQAE_OK) return rc;
  if ((!k_out && !v_out) || n_tokens < 0 || (n_tokens > 0 && !positions)) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(positions, 4) || !aligned(seq, 4)) return MOQAE_ERR_MISALIGNED;
  rc = check_out_rows(k_out, n_tokens, &ko);
  if (rc == MOQAE_OK) rc = check_out_rows(v_out, n_tokens, &vo);
  if (rc != MOQAE_OK) return rc;
  if ((k_out && ko.n_heads != pv.n_kv_heads) || (v_out && vo.n_heads != pv.n_kv_heads)) return MOQAE_ERR_INVALID_ARG;
  return cuda_rc(moqae::launch_paged4_read(pv, ko, vo, positions, seq, n_tokens, static_cast<cudaStream_t>(stream)));
}

int moqae_paged4_decode_attn_workspace(const moqae_paged4_cache* cache, int32_t n_q_heads, int64_t* out_bytes) {
  PagedView pv;
  int rc = check_pages(cache, &pv);
  if (rc == MOQAE_OK) rc = check_group(pv, n_q_heads);
  if (rc != MOQAE_OK) return rc;
  if (!out_bytes) return MOQAE_ERR_INVALID_ARG;
  if (!moqae::paged4_decode_fits(pv)) return MOQAE_ERR_UNSUPPORTED;
  *out_bytes = moqae::paged4_decode_workspace_bytes(n_q_heads / pv.n_kv_heads);
  return MOQAE_OK;
}

int moqae_paged4_decode_attn(const moqae_paged4_cache* cache, const moqae_rows* q, const moqae_rows* out,
                             const moqae_attn_options* options, void* workspace, int64_t workspace_bytes, void* stream) {
  PagedView pv;
  RowsView qv, ov;
  AttnOptions opt;
  const int rc = check_attention(cache, q, out, cache ? cache->batch : 0, options, &pv, &qv, &ov, &opt);
  if (rc != MOQAE_OK) return rc;
  if (!workspace) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(workspace, 16)) return MOQAE_ERR_MISALIGNED;
  if (!moqae::paged4_decode_fits(pv)) return MOQAE_ERR_UNSUPPORTED;
  if (workspace_bytes < moqae::paged4_decode_workspace_bytes(qv.n_heads / pv.n_kv_heads)) return MOQAE_ERR_WORKSPACE_TOO_SMALL;
  return cuda_rc(moqae::launch_paged4_decode(pv, qv, ov, opt, workspace, static_cast<cudaStream_t>(stream)));
}

int moqae_paged4_prefill_attn_workspace(const moqae_paged4_cache* cache, int32_t n_q_heads, int32_t n_tokens, int64_t* out_bytes,
                                        int64_t* least_bytes) {
  PagedView pv;
  int rc = check_pages(cache, &pv);
  if (rc == MOQAE_OK) rc = check_group(pv, n_q_heads);
  if (rc != MOQAE_OK) return rc;
  if (!out_bytes || n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > moqae::kMaxQueryTokens || pv.batch > moqae::kMaxQueryTokens) return MOQAE_ERR_UNSUPPORTED;
  *out_bytes = moqae::paged4_prefill_workspace_bytes(pv, n_q_heads / pv.n_kv_heads, n_tokens);
  if (least_bytes) *least_bytes = moqae::paged4_prefill_least_bytes(pv, n_q_heads / pv.n_kv_heads, n_tokens);
  return MOQAE_OK;
}

int moqae_paged4_prefill_attn(const moqae_paged4_cache* cache, const moqae_rows* q, const int32_t* cu_q, int32_t n_tokens,
                              const moqae_rows* out, const moqae_attn_options* options, void* workspace,
                              int64_t workspace_bytes, void* stream) {
  PagedView pv;
  RowsView qv, ov;
  AttnOptions opt;
  if (n_tokens < 0) return MOQAE_ERR_INVALID_ARG;
  if (n_tokens > moqae::kMaxQueryTokens || (cache && cache->batch > moqae::kMaxQueryTokens)) return MOQAE_ERR_UNSUPPORTED;
  const int rc = check_attention(cache, q, out, n_tokens, options, &pv, &qv, &ov, &opt);
  if (rc != MOQAE_OK) return rc;
  if ((pv.batch > 0 && !cu_q) || !workspace) return MOQAE_ERR_INVALID_ARG;
  if (!aligned(cu_q, 4) || !aligned(workspace, 16)) return MOQAE_ERR_MISALIGNED;
  const int group = qv.n_heads / pv.n_kv_heads;
  if (workspace_bytes < moqae::paged4_prefill_least_bytes(pv, group, n_tokens)) return MOQAE_ERR_WORKSPACE_TOO_SMALL;
  const cudaError_t e = moqae::launch_paged4_prefill(pv, qv, cu_q, n_tokens, options ? options->max_new : 0, ov, opt, workspace, workspace_bytes,
                                                      static_cast<cudaStream_t>(stream));
  return e == cudaErrorNotSupported ? MOQAE_ERR_UNSUPPORTED : cuda_rc(e);
}

}  // extern "C"
#pragma GCC visibility pop
