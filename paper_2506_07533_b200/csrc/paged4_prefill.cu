// moqae_paged4_prefill_attn: launches over 4-bit pages.  Few rows per sequence go to the streaming kernel (paged4_decode.cu), the others to the
// large tiles (paged_prefill.cuh), behind a pass that brings the queries into fp16 and into the order of the channels there.
//   A query is read once and written once: 16300 tokens of 32 heads, 267 MB, about 45 us of the 1.8 ms that follow.
#include "paged_prefill.cuh"

namespace moqae {

namespace {

constexpr int kQueryThreads = 256;

// Unit i (8 channels) of row i / 16: channels 0, 4, 1, 5, 2, 6, 3, 7 of it, in fp16.
template <bool BF16> __global__ void __launch_bounds__(kQueryThreads) query4_kernel(RowsView q, uint16_t* to, long long units) {
  after_previous();
  for (long long i = static_cast<long long>(blockIdx.x) * kQueryThreads + threadIdx.x; i < units; i += static_cast<long long>(gridDim.x) * kQueryThreads) {
    const long long row = i >> 4, t = row / q.n_heads;
    const int u = static_cast<int>(i & 15), h = static_cast<int>(row - t * q.n_heads);
    const uint4 x = *reinterpret_cast<const uint4*>(q.data + t * q.token + h * q.head + 8 * u);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    uint32_t f[4];                                     // pairs (2 i, 2 i + 1)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 v = pair_to_float2<BF16>(w[k]);
      f[k] = BF16 ? float2_to_pair<false>(v.x, v.y) : w[k];
    }
    reinterpret_cast<uint4*>(to)[i] = make_uint4(__byte_perm(f[0], f[2], 0x5410), __byte_perm(f[0], f[2], 0x7632), __byte_perm(f[1], f[3], 0x5410),
                                                 __byte_perm(f[1], f[3], 0x7632));
  }
}

}  // namespace

// What the large tiles need, or the streaming kernel, and the queries.
long long paged4_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens) {
  const long long few = paged4_few_workspace_bytes(), cut = tiles_workspace_bytes(pv, group, n_tokens);
  return (cut > few ? cut : few) + static_cast<long long>(n_tokens) * group * pv.n_kv_heads * kHeadDim * 2;
}

cudaError_t launch_paged4_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                                  const AttnOptions& opt, void* workspace, cudaStream_t st) {
  if (pv.batch <= 0 || n_tokens <= 0) return cudaSuccess;
  const int group = q.n_heads / pv.n_kv_heads;
  if (paged4_few_rows(pv, group, n_tokens)) return launch_paged4_few(pv, q, cu_q, n_tokens, out, opt, workspace, st);
  RowsView q16{};
  q16.data = reinterpret_cast<uint16_t*>(static_cast<uint8_t*>(workspace) + tiles_workspace_bytes(pv, group, n_tokens));
  q16.token = static_cast<long long>(q.n_heads) * kHeadDim;
  q16.head = kHeadDim;
  q16.n_heads = q.n_heads;
  PrefillJob job;
  long long grid;
  if (!make_job(job, grid, pv, q16, cu_q, n_tokens, out, workspace)) return cudaErrorInvalidConfiguration;
  CUtensorMap mq;
  if (!make_query_map(&mq, q16, n_tokens, group)) return cudaErrorNotSupported;
  job.q_box = kTileRows / group;
  const long long units = static_cast<long long>(n_tokens) * q.n_heads * 16, ctas = (units + kQueryThreads - 1) / kQueryThreads, most = 16ll * sm_count_of_current_device();
  const unsigned q_grid = static_cast<unsigned>(ctas < most ? ctas : most);
  const cudaError_t e = launch_early(pv.dtype == MOQAE_DTYPE_BF16 ? query4_kernel<true> : query4_kernel<false>, q_grid, kQueryThreads, 0, st, q, q16.data, units);
  return e != cudaSuccess ? e : launch_shaped<true>(pv, opt, job, mq, mq, mq, grid, st);
}

}  // namespace moqae
