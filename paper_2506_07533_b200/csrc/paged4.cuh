// Shared declarations of the paged 4-bit cache: where a tile keeps what, kernel-side view, launchers.
#pragma once

#include "paged.cuh"

namespace moqae {

// A tile holds 16 tokens of one kv head in 2560 bytes.  In the order of the fragments that the attention kernels build:
//   keys    token t: 64 code bytes at 64 t; the byte of channels c, c + 1 (c even) of group g = c / 32 at 16 ((c % 32) / 8) + 4 g + (c % 8) / 2,
//           so that 16 bytes hold eight channels of each group; scales and zeros of the four groups, fp16, at 1024 + 16 t
//   values  token t: 64 code bytes in two pieces of 32, at 1280 + 512 p + 32 r(t), p = 0, 1; the byte of channels c, c + 1 at
//           8 (u % 4) + 2 g + (c % 4) / 2 of piece p = u / 4, u = (c % 32) / 4, so that 8 bytes hold four channels of each group; r(t) puts the tokens
//           of four lanes that load together side by side; scales and zeros of two neighbouring tokens, alternating, at 2304 + 32 (t / 2)
// The low four bits of a byte are the even channel's.
constexpr int kTileTokens4 = 16;
constexpr int kTileBytes4 = 2560, kTokenBytes4 = kTileBytes4 / kTileTokens4;
constexpr int kKeyMeta4 = 1024, kValueCodes4 = 1280, kValueMeta4 = 2304;
__host__ __device__ constexpr int value_row4(int t) { return (t & 8) | ((t & 1) << 2) | ((t >> 1) & 3); }

// The pages of a 4-bit cache: a PagedView whose k is the first byte and whose k_page and k_head count bytes; no other address or stride is used.
__device__ __forceinline__ uint8_t* tile4(const PagedView& pv, int page, int head, int slot) {
  return reinterpret_cast<uint8_t*>(pv.k) + page * pv.k_page + head * pv.k_head + static_cast<long long>(slot >> 4) * kTileBytes4;
}

// The page pool of a plan: a ring of page numbers.
struct PoolView {
  int32_t* ring;
  const int32_t* state;      // first free page, number of free pages
  int32_t* state_out;        // the same afterwards (may be the same words); the third word counts CTAs and is left at zero
  int n_pages;
};
struct PlanJob {
  const int32_t* past;
  const int32_t* n_new;
  int32_t* table;
  int32_t* kv_len;
  int32_t* cu_q;
  int32_t* positions;
  int32_t* seq;
  int32_t* status;
  int batch, max_pages, page_shift, n_rows;
};

cudaError_t launch_paged_plan(const PlanJob& job, const PoolView& pool, cudaStream_t st);
cudaError_t launch_paged4_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out, const RowsView& k,
                                 const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens, cudaStream_t st);
cudaError_t launch_paged4_read(const PagedView& pv, const RowsView& k_out, const RowsView& v_out, const int32_t* positions, const int32_t* seq,
                               int n_tokens, cudaStream_t st);
bool paged4_decode_fits(const PagedView& pv);
long long paged4_decode_workspace_bytes(int group);
cudaError_t launch_paged4_decode(const PagedView& pv, const RowsView& q, const RowsView& out, const AttnOptions& opt, void* workspace, cudaStream_t st);
bool paged4_few_fits(const PagedView& pv, int group, int n_tokens, int max_rows);
long long paged4_few_workspace_bytes();
// max_rows > 0: sequences of more rows (tokens times heads of a group) are left to another kernel
cudaError_t launch_paged4_few(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                              const AttnOptions& opt, void* workspace, int max_rows, cudaStream_t st);
long long paged4_prefill_least_bytes(const PagedView& pv, int group, int n_tokens);     // without room for expanded blocks
long long paged4_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens);
// max_new: the most new tokens of a sequence; <= 0: not known
cudaError_t launch_paged4_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, int max_new, const RowsView& out,
                                  const AttnOptions& opt, void* workspace, long long workspace_bytes, cudaStream_t st);

}  // namespace moqae
