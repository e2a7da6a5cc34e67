// moqae_paged_prefill_attn: launches of the large tiles (paged_prefill.cuh) over 16-bit pages, which arrive as tiled copies.
#include "paged_prefill.cuh"

namespace moqae {

long long paged_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens) {
  const long long few = paged_few_workspace_bytes();
  if (static_cast<long long>(n_tokens) * group <= kFewRows && paged_few_rows(pv, group, n_tokens)) return few;    // few rows however many sequences
  const long long cut = tiles_workspace_bytes(pv, group, n_tokens);
  return cut > few ? cut : few;
}

cudaError_t launch_paged_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                                 const AttnOptions& opt, void* workspace, cudaStream_t st) {
  const int group = q.n_heads / pv.n_kv_heads;
  if (workspace && paged_few_rows(pv, group, n_tokens)) return launch_paged_few(pv, q, cu_q, n_tokens, out, opt, workspace, st);
  if (pv.batch <= 0 || n_tokens <= 0) return cudaSuccess;
  PrefillJob job;
  long long grid;
  if (!make_job(job, grid, pv, q, cu_q, n_tokens, out, workspace, 0)) return cudaErrorInvalidConfiguration;
  job.box_rows = pv.page_size < 64 ? pv.page_size : 64;
  const long long ks[3] = {pv.k_slot, pv.k_head, pv.k_page}, vs[3] = {pv.v_slot, pv.v_head, pv.v_page};
  int order[3] = {0, 1, 2};                              // slot, head, page by the keys' strides
  for (int a = 0; a < 2; ++a)
    for (int b = 0; b < 2 - a; ++b)
      if (ks[order[b]] > ks[order[b + 1]]) {
        const int t = order[b];
        order[b] = order[b + 1];
        order[b + 1] = t;
      }
  for (int d = 0; d < 3; ++d) (order[d] == 0 ? job.dim_slot : (order[d] == 1 ? job.dim_head : job.dim_page)) = d + 1;
  CUtensorMap mk, mv, mq;
  const void* kb = pv.n_pages > 0 ? pv.k : q.data;     // without pages nothing inside the map is ever named
  const void* vb = pv.n_pages > 0 ? pv.v : q.data;
  if (!make_page_map(&mk, kb, pv, ks, order, job.box_rows) || !make_page_map(&mv, vb, pv, vs, order, job.box_rows)) return cudaErrorNotSupported;
  if (make_query_map(&mq, q, n_tokens, group)) job.q_box = kTileRows / group;
  else mq = mk;
  return launch_shaped<false>(pv, opt, job, mk, mv, mq, grid, st);
}

}  // namespace moqae
