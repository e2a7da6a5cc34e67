// moqae_paged4_prefill_attn: launches over 4-bit pages.  Sequences of few rows go to the streaming kernel (paged4_decode.cu), the others to the
// large tiles (paged_prefill.cuh), behind a pass that brings keys and values out of their codes and bf16 queries into fp16.
//   Expanding once costs 672 bytes per token and kv head (32612 tokens of 8 heads: 34 us for 175 MB) and one reading of 512; inside the large tiles every row tile would
//   expand the blocks that it sees again (see Four there).  The workspace holds kExpandBytes of expanded blocks at most, of tokens that some query sees; sequences
//   that find no room are expanded inside (512 tokens over 131000 under a window of 4096, 40 heads: 288 us inside, 125 this way).  Measured: 512 tokens over
//   32000 beside 255 single ones over 2000, 32 / 8 heads, bf16, 545 us (223 and 309 apart); beside 63, 40 / 40 heads, 771 (244 and 525).
#include "paged_prefill.cuh"

namespace moqae {

namespace {

constexpr int kExpandThreads = 256, kExpandWarps = kExpandThreads / 32;
constexpr long long kExpandBytes = 1ll << 30;
constexpr int kMaxExpanded = 1 << 20;              // blocks
// Rows (tokens times heads of a group) of a sequence up to which the streaming kernel is faster, although it streams the sequence once per
// 16 rows: it reads a third of the bytes, and expands nothing.  Streaming / large tiles, us: one sequence of 32000 tokens, 32 / 8 heads, with 32 rows 39 / 90,
// 64 62 / 90, 96 84 / 99, 128 106 / 100; 8 of 2000 with 64 40 / 55, 96 53 / 57, 128 66 / 60; 64 of 2000 with 96 293 / 295; 8 of 8000, 40 / 40 heads, with
// 64 450 / 804, 96 667 / 842, 128 884 / 838.
constexpr int kFewRows4 = 96;
// Calls of several sequences that the streaming kernel takes alone whoever has the rows: up to so many rows of all sequences together, and tiles of 16 tokens that one
// sequence with all of them could take at most (sets of 16 rows, kv heads, tiles of the longest sequence that the tables can hold).  Alone / both kernels, us,
// one of eight sequences having all rows: 8 kv heads, 132 rows behind 1000 tokens 23 / 35, 8000 46 / 56, 32000 122 / 109; 256 rows behind 1000 30 / 37, 4000 47 / 53,
// 8000 69 / 67, 32000 205 / 125; 32 and 40 kv heads, 132 behind 1000 36 / 45, 4000 79 / 70, 32000 534 / 355; 256 behind 500 37 / 33, 1000 50 / 44, 4000 126 / 77; 384 rows
// lose from 500 tokens on.  Even batches save the 12 us of the launches that find nothing: 15 sequences of four new tokens 11 / 17, 64 of 1000 50 / 62.
constexpr int kAloneRows4 = 256;
constexpr long long kAloneTiles4 = 1 << 15;
constexpr int kBlockTiles = kBlock / kTileTokens4;

struct ExpandJob {
  RowsView q;
  const int32_t* cu_q;
  uint16_t* q16;                                   // [n_tokens][heads][128], where the queries are bf16
  float* q_factor;                                 // [n_tokens][heads]: a query is its row of q16 times this
  uint16_t* k16;                                   // [blocks][kv heads][128 tokens][128]
  uint16_t* v16;
  int2* first;                                     // [batch]: a sequence's first block, -1: not expanded; blocks left out behind its prefix
  int n_tokens, blocks;                            // rows of q; room for blocks
  int group, few_rows;                             // sequences of at most few_rows rows are the streaming kernel's
};

// Room is dealt out in the order of the sequences that bring tokens: blocks of the prefix, then from the first that a window reaches on (what lies between
// takes none).  One that finds no room leaves it to those behind it.  A warp takes a tile of 16 tokens of one head.
template <bool BF16> __global__ void __launch_bounds__(kExpandThreads, 4) expand4_kernel(PagedView pv, AttnOptions opt, ExpandJob job) {
  __shared__ int block_to[kExpandThreads + 1], warp_sum[kExpandWarps];      // blocks in front of a sequence
  __shared__ int len_of[kExpandThreads], lo_of[kExpandThreads], pre_of[kExpandThreads];   // tokens, and which of them some row sees: [lo, len) and [0, pre)
  __shared__ int skip_of[kExpandThreads];          // blocks behind the prefix that no row sees
  __shared__ int without, left;                    // first sequence of a turn without room, and the room that there was
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int r8 = lane >> 2, u = lane & 3;          // four neighbouring lanes store 64 bytes of a row together
  after_previous();
  int before = 0;
  for (int base = 0; base < pv.batch; base += kExpandThreads) {
    const int b = base + tid;
    int need = 0, len = 0, lo = 0, pre = 0, skip = 0;
    if (b < pv.batch) {
      const int from = min(max(job.cu_q[b], 0), job.n_tokens), n = min(max(job.cu_q[b + 1], from), job.n_tokens) - from;
      len = paged_len(pv, b, false);
      lo = opt.window > 0 ? max(0, len - n - opt.window + 1) : 0;
      pre = opt.prefix_len ? min(max(opt.prefix_len[b], 0), len) : 0;
      if (pre < lo) skip = max(lo / kBlock - prefix_blocks(pre), 0);
      need = n * job.group > job.few_rows ? min((len + kBlock - 1) / kBlock - skip, kMaxExpanded + 1) : 0;
    }
    int to_here, in_front, all;                    // blocks up to this sequence, of the warps before, up to the turn's end
    for (;;) {
      to_here = need;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int x = __shfl_up_sync(0xffffffffu, to_here, o);
        if (lane >= o) to_here += x;
      }
      __syncthreads();                             // the turn before is done with the arrays
      if (lane == 31) warp_sum[warp] = to_here;
      __syncthreads();
      in_front = all = before;
#pragma unroll
      for (int w = 0; w < kExpandWarps; ++w) {
        const int x = warp_sum[w];
        if (w < warp) in_front += x;
        all += x;
      }
      if (all <= job.blocks) break;
      // the first for which it is not enough, and whoever behind it wants more than was left, go without
      const int at = in_front + to_here - need;
      if (at <= job.blocks && at + need > job.blocks) {
        without = tid;
        left = job.blocks - at;
      }
      __syncthreads();
      if (tid >= without && need > left) need = 0;
    }
    before = all;
    block_to[tid] = in_front + to_here - need;
    len_of[tid] = len;
    lo_of[tid] = lo;
    pre_of[tid] = pre;
    skip_of[tid] = skip;
    if (tid == kExpandThreads - 1) block_to[kExpandThreads] = all;
    if (blockIdx.x == 0 && b < pv.batch) job.first[b] = make_int2(need > 0 ? in_front + to_here - need : -1, skip);
    __syncthreads();
    const int from = block_to[0], tiles = (block_to[kExpandThreads] - from) * kBlockTiles, n_warps = static_cast<int>(gridDim.x) * kExpandWarps;
    const int step_t = n_warps / pv.n_kv_heads, step_h = n_warps - step_t * pv.n_kv_heads, id = static_cast<int>(blockIdx.x) * kExpandWarps + warp;
    int h = id % pv.n_kv_heads;
    for (int t = id / pv.n_kv_heads; t < tiles; t += step_t + (h + step_h >= pv.n_kv_heads), h = h + step_h >= pv.n_kv_heads ? h + step_h - pv.n_kv_heads : h + step_h) {
      const int block = from + t / kBlockTiles;
      int i = 0, hi = kExpandThreads;              // the sequence: block_to[i] <= block < block_to[i + 1]
      while (hi - i > 1) {
        const int mid = (i + hi) >> 1;
        if (block_to[mid] <= block) i = mid;
        else hi = mid;
      }
      const int kept = block - block_to[i], in_seq = kept < prefix_blocks(pre_of[i]) ? kept : kept + skip_of[i];
      const int j0 = (in_seq * kBlockTiles + t % kBlockTiles) * kTileTokens4;
      const uint8_t* tile = nullptr;
      // (a tile of the block that no row sees is zeros: its page may have been given back)
      if (j0 < len_of[i] && (j0 + kTileTokens4 > lo_of[i] || j0 < pre_of[i])) {
        const int page = pv.table[static_cast<long long>(base + i) * pv.max_pages + (j0 >> pv.page_shift)];
        if (page >= 0 && page < pv.n_pages) tile = tile4(pv, page, h, j0 & (pv.page_size - 1));
        else if (lane == 0) paged_status(pv.status, MOQAE_ERR_CORRUPT_TABLE, base + i, j0 >> pv.page_shift);
      }
      Raw4 raw[4];                                 // keys, values of tokens 0..7, of 8..15
#pragma unroll
      for (int k = 0; k < 4; ++k) raw[k].code = raw[k].s = raw[k].z = make_uint4(0, 0, 0, 0);
      if (tile) {
        load4<false>(raw[0], tile, r8, u);
        load4<false>(raw[1], tile, r8 + 8, u);
        load4<true>(raw[2], tile, r8, u);
        load4<true>(raw[3], tile, r8 + 8, u);
      }
      const long long row0 = (static_cast<long long>(block) * pv.n_kv_heads + h) * kBlock + (j0 & (kBlock - 1));
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int at = r8 + 8 * (k & 1), j = j0 + at;
        const bool used = j < len_of[i] && (j >= lo_of[i] || j < pre_of[i]);
        uint4* dst = reinterpret_cast<uint4*>((k < 2 ? job.k16 : job.v16) + (row0 + at) * kHeadDim) + u;
        auto put = [&](int g, const uint4& unit) { dst[4 * g] = unit; };
        if (k < 2) expand4<false>(raw[k], used, at, put);
        else expand4<true>(raw[k], used, at, put);
      }
    }
  }
  if (!BF16) return;
  // Queries: half a warp takes a row.  A row whose largest element is below 1, or 2^15 and more, is multiplied by a power of two that brings it to 8 .. 16, so
  // that bf16 elements are exact in fp16 down to 2^-17, and off by at most 2^-25 of the row's largest below.
  const int n_rows = static_cast<int>(gridDim.x) * (kExpandThreads / 16), id = static_cast<int>(blockIdx.x) * (kExpandThreads / 16) + (tid >> 4), c = tid & 15;
  const int step_t = n_rows / job.q.n_heads, step_h = n_rows - step_t * job.q.n_heads;
  const unsigned half_warp = 0xffffu << (lane & 16);
  int h = id % job.q.n_heads;
  for (int t = id / job.q.n_heads; t < job.n_tokens;) {
    const uint4 x = *reinterpret_cast<const uint4*>(job.q.data + t * job.q.token + h * job.q.head + 8 * c);
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
    float2 v[4];
    float big = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = pair_to_float2<BF16>(w[k]);
      big = fmaxf(big, fmaxf(fabsf(v[k].x), fabsf(v[k].y)));
    }
#pragma unroll
    for (int o = 1; o < 16; o <<= 1) big = fmaxf(big, __shfl_xor_sync(half_warp, big, o));
    const bool far = (big < 1.0f && big > 0.0f) || big >= 32768.0f;
    const uint32_t ex = max(__float_as_uint(big) >> 23, 4u);               // 2^(ex - 127) <= largest
    const float up = far ? __uint_as_float((257u - ex) << 23) : 1.0f;      // 2^(130 - ex)
    uint32_t f[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) f[k] = float2_to_pair<false>(v[k].x * up, v[k].y * up);
    const long long row = static_cast<long long>(t) * job.q.n_heads + h;
    *reinterpret_cast<uint4*>(job.q16 + row * kHeadDim + 8 * c) = make_uint4(f[0], f[1], f[2], f[3]);
    if (c == 0) job.q_factor[row] = far ? __uint_as_float((ex - 3u) << 23) : 1.0f;
    t += step_t;
    h += step_h;
    if (h >= job.q.n_heads) {
      h -= job.q.n_heads;
      ++t;
    }
  }
}

// The workspace behind what the large tiles need: queries, their factors, two numbers per sequence, blocks.
struct Layout {
  long long queries, factors, first, blocks;       // offsets
  long long block_bytes;                           // of keys and values
};
Layout layout_of(const PagedView& pv, int group, int n_tokens) {
  Layout l;
  l.queries = tiles_workspace_bytes(pv, group, n_tokens);
  const long long rows = pv.dtype == MOQAE_DTYPE_BF16 ? static_cast<long long>(n_tokens) * group * pv.n_kv_heads : 0;
  l.factors = l.queries + rows * kHeadDim * 2;
  l.first = l.factors + (4 * rows + 15) / 16 * 16;
  l.blocks = l.first + (8ll * pv.batch + 255) / 256 * 256;
  l.block_bytes = 2ll * pv.n_kv_heads * kBlock * kHeadDim * 2;
  return l;
}

}  // namespace

// What every call needs, and room for the blocks of the longest sequences that the tables allow, up to kExpandBytes.
long long paged4_prefill_least_bytes(const PagedView& pv, int group, int n_tokens) {
  const long long few = paged4_few_workspace_bytes(), tiles = layout_of(pv, group, n_tokens).blocks;
  return tiles > few ? tiles : few;
}
long long paged4_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens) {
  const Layout l = layout_of(pv, group, n_tokens);
  const long long a_sequence = (static_cast<long long>(pv.max_pages) * pv.page_size + kBlock - 1) / kBlock, room = kExpandBytes / l.block_bytes;
  const long long all = a_sequence * pv.batch;
  return paged4_prefill_least_bytes(pv, group, n_tokens) + (all < room ? all : room) * l.block_bytes;
}

cudaError_t launch_paged4_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, int max_new, const RowsView& out,
                                  const AttnOptions& opt, void* workspace, long long workspace_bytes, cudaStream_t st) {
  if (pv.batch <= 0 || n_tokens <= 0) return cudaSuccess;
  const int group = q.n_heads / pv.n_kv_heads;
  // Who takes which sequence is decided on the device, by its rows; the host knows their sum, all of which one sequence may have, and a bound where the
  // caller gave one.  Where no sequence can have many, the streaming kernel takes the call alone (the large tiles would cost two launches, 12 us, to
  // find nothing), as the large tiles do where there is one sequence.  Otherwise both run: a piece of a prompt beside single tokens expands and
  // tiles that one sequence only.
  const long long rows = static_cast<long long>(n_tokens) * group, most = max_new > 0 && max_new < n_tokens ? static_cast<long long>(max_new) * group : rows;
  auto tiles = [&]() { return (rows + 15) / 16 * pv.n_kv_heads * pv.max_pages * (pv.page_size / kTileTokens4); };
  if ((most <= kFewRows4 || (pv.batch > 1 && rows <= kAloneRows4 && tiles() <= kAloneTiles4)) && paged4_few_fits(pv, group, n_tokens, 0))
    return launch_paged4_few(pv, q, cu_q, n_tokens, out, opt, workspace, 0, st);
  const int few_rows = pv.batch > 1 && paged4_few_fits(pv, group, n_tokens, kFewRows4) ? kFewRows4 : 0;
  if (few_rows > 0) {
    const cudaError_t e = launch_paged4_few(pv, q, cu_q, n_tokens, out, opt, workspace, few_rows, st);
    if (e != cudaSuccess) return e;
  }
  const Layout l = layout_of(pv, group, n_tokens);
  uint8_t* space = static_cast<uint8_t*>(workspace);
  const long long room = (workspace_bytes - l.blocks) / l.block_bytes;
  ExpandJob ex{};
  ex.q = q;
  ex.cu_q = cu_q;
  ex.q16 = reinterpret_cast<uint16_t*>(space + l.queries);
  ex.q_factor = reinterpret_cast<float*>(space + l.factors);
  ex.first = reinterpret_cast<int2*>(space + l.first);
  ex.blocks = static_cast<int>(room < kMaxExpanded ? room : kMaxExpanded);
  ex.k16 = reinterpret_cast<uint16_t*>(space + l.blocks);
  ex.v16 = ex.k16 + static_cast<long long>(ex.blocks) * pv.n_kv_heads * kBlock * kHeadDim;
  ex.n_tokens = n_tokens;
  ex.group = group;
  ex.few_rows = few_rows;

  const bool bf16 = pv.dtype == MOQAE_DTYPE_BF16;
  RowsView q16 = q;
  if (bf16) {
    q16.data = ex.q16;
    q16.token = static_cast<long long>(q.n_heads) * kHeadDim;
    q16.head = kHeadDim;
  }
  PrefillJob job;
  long long grid;
  if (!make_job(job, grid, pv, q16, cu_q, n_tokens, out, workspace, few_rows)) return cudaErrorInvalidConfiguration;
  job.expanded = ex.first;
  job.q_factor = ex.q_factor;
  job.box_rows = 64;
  job.dim_slot = 1;
  job.dim_head = 2;
  job.dim_page = 3;
  PagedView blocks = pv;                           // the expanded blocks as pages of 128 tokens
  blocks.page_size = kBlock;
  blocks.n_pages = ex.blocks;
  const long long stride[3] = {kHeadDim, kBlock * kHeadDim, static_cast<long long>(pv.n_kv_heads) * kBlock * kHeadDim};
  const int order[3] = {0, 1, 2};
  CUtensorMap mk, mv, mq;
  const void* kb = ex.blocks > 0 ? ex.k16 : workspace;   // without room no block is ever named
  const void* vb = ex.blocks > 0 ? ex.v16 : workspace;
  if (!make_page_map(&mk, kb, blocks, stride, order, job.box_rows) || !make_page_map(&mv, vb, blocks, stride, order, job.box_rows)) return cudaErrorNotSupported;
  if (make_query_map(&mq, q16, n_tokens, group)) job.q_box = kTileRows / group;
  else mq = mk;
  const unsigned expand_grid = 4u * sm_count_of_current_device();
  const cudaError_t e = launch_early(bf16 ? expand4_kernel<true> : expand4_kernel<false>, expand_grid, kExpandThreads, 0, st, pv, opt, ex);
  return e != cudaSuccess ? e : launch_shaped<true>(pv, opt, job, mk, mv, mq, grid, st);
}

}  // namespace moqae
