// Attention of several new tokens per sequence over a paged 16-bit cache (moqae_paged_prefill_attn).
//
// For every query row  o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(f(q.k_j) - reference)  over the tokens it sees:
// two dense products with a softmax between them, on the 5th-generation tensor cores.
//
//   Rows.  The rows of a (sequence, kv head) are its tokens times the query heads of the group (row r = token
//   r / group, head r % group), so a group shares every key block and a few tokens fill a tile.  A CTA
//   owns 256 consecutive rows (two tiles of 128) and walks the blocks of 128 tokens that some row sees.
//   Pages.  The pages are a four-dimensional tensor map (channel, slot, head, page in the order of their
//   strides); a block is fetched with one tiled copy per page (or per 64 slots of a page) and half of the
//   channels, page numbers looked up one block ahead.  Rows of a block that no query may use (behind the
//   sequence, before every window) are not fetched where whole pages are concerned, and their values are
//   zeroed in shared memory before the product: a weight of zero does not silence a NaN.  Under a cap their keys are, too: the
//   form of the tanh goes by the largest score of 32 columns.  (Zeroing the scores instead: five capped fp16 prompts 471 us,
//   this way 455.)
//   Products, softmax and tensor memory as in the prefill attention over the quantised cache (prefill.cu):
//   S_i = Q_i K^T (M 128, N 128, K 16 steps), two threads per row, P_i written over S_i as 16-bit pairs, O_i += P_i V
//   with P_i as a tensor-memory operand, a reference that moves only when the weights of 32 columns
//   would add up to more than kSumLimit, so O_i is rarely rescaled.  Blocks are walked from the last to the
//   first: with a distance bias the largest scores come first (walking forwards moved the reference at every block).  P_i is rounded to the cache's dtype (the
//   product takes operands of one type), each weight by at most 2^-8 (bf16) or 2^-11 (small ones: see kLead), which averages out over the tokens:
//   with bf16 results, 0.0023 of their norm off instead of the 0.0017 of their own rounding.  Blocks that some row does not
//   see whole add up the rounded weights: a row of one token is then exact, rows of up to 128 are 0.0019 to 0.0020 off instead
//   of 0.0021 to 0.0023.  The other blocks add up the exact ones, as many tokens gain nothing from it (2 to 8 % of the time).
//   Pieces.  One CTA per SM stays for the whole launch and takes pieces of work, (row tile, kv head, run of blocks), from
//   a shared counter, rows late in their sequence first (they see the most).  A planning warp claims the next
//   piece and brings its queries while the last block of the current one is worked on, the fetching warps run ahead
//   into it, so between two pieces little but the softmax warps' way from the last product to memory shows.
//   Where the rows alone would leave SMs idle, the blocks of a row tile are cut into up to kMaxSegs pieces,
//   as many as an estimate of the turns favours; they leave float32 sums in the workspace and the last to arrive
//   joins them in the order of their tokens (results do not depend on timing).
//   What bounds it.  A block of 128 tokens takes a CTA about 3450 clocks (8192 tokens, 32 / 8 heads, bf16: 457 us, 1200
//   TFLOP/s), of which the products are 2048 (the tensor pipe is busy half of the time): a tile's own chain is as long as that.  Its
//   weights take its 8 warps 1790 clocks, from stored weights to the next scores it is 1710 (16 products of 64 clocks, 390 of
//   their latency, the wait for the other tile's), and with two tiles tensor memory is full.  It is not the exponential unit: with two
//   integer operations in the place of every exponential the same prompt takes 492 us.  Looked at and slower: scores of 64 columns, so that four
//   chains overlap (a product of N = 64 takes as long as one of 128: 1.45 x the time), an issuing thread per tile (products of the
//   two kinds interleaved: 1.45 x), no barrier between the two warps of a row (the same time).
// Every mbarrier wait is bounded; on expiry the CTA records MOQAE_ERR_TIMEOUT, every role stops and the
// tensor memory is still freed.
#include <cstring>
#include <type_traits>

#include "paged.cuh"
#include "umma.cuh"

namespace moqae {

namespace {

constexpr int kTileRows = 128, kItemRows = 2 * kTileRows;
constexpr int kBlock = 128;                          // tokens per block
constexpr int kTileBytes = kTileRows * 256;          // a query tile, a block of keys, a block of values
constexpr int kStages = 2;
constexpr int kSoftmaxWarps = 16, kIssueWarp = 16, kKeyWarp = 17, kValueWarp = 18, kPlanWarp = 19;
constexpr int kThreads = 20 * 32;
constexpr int kTmemCols = 512;
// The reference moves when the weights of 32 columns add up to more than kSumLimit; it then lies kLead below the largest score
// (base-2 units), and starts kLead below some score.  fp16 overflows at 65520, and its steps end at 2^-24: the lead keeps small weights,
// each is off by at most 2^-28 of the weight of a score that the row sees (without it 2^-24: what thousands of tokens beside one
// large score add up to was lost).  A longer lead moves the reference more often: five fp16 prompts with cap, bias and prefix take
// 466 us without one, 470 with 4, 475 with 5, 486 with 6.
template <bool BF16> constexpr float kSumLimit = BF16 ? 16384.0f : 61440.0f;
template <bool BF16> constexpr float kLead = BF16 ? 0.0f : 4.0f;
constexpr float kLog2e = 1.4426950408889634f;
constexpr long long kWaitLimit = 1ll << 31;          // about a second
constexpr long long kPieceWaitLimit = 1ll << 37;     // for what may take as long as a piece: about a minute
constexpr int kMaxSegs = 32;
constexpr int kMinSegBlocks = 2;                     // a piece of a cut row tile is at least this many blocks
constexpr int kMaxParts = 640;                       // partial sums that the workspace holds (of 130 KiB)
// More row tiles than this are never cut.  (Nor are most calls near it: 640 parts are one per row tile.  So a long context beside many
// short prompts is walked by one CTA per row tile: 64 tokens over 32000 take 86 us alone, 490 beside 55 prompts of 20 tokens, where
// the limit does not apply, and 496 beside 69, where it does.)
constexpr long long kSplitItems = 512;
constexpr int kPartFloats = kItemRows * (kHeadDim + 2);   // per piece: sums, then (reference, weight sum) per row
constexpr int kWarpStage = 2048;                     // shared memory of a softmax warp on the way to memory

// kfull / vfull: bytes of a block have landed (vfull of an edge block: and its rows are zeroed); vraw: the bytes of
// an edge block of values; kraw: the same of keys; kfree / vfree: the products that read the stage are done; sfull, pfull, ofull as in prefill.cu;
// qfull / qfree: the queries of a piece stand in shared memory / are not read any more; ifull / ifree: a piece's
// description is there / nobody reads it any more; parts, ticket: see the joining of pieces
enum { BAR_KFULL = 0, BAR_VFULL = kStages, BAR_KFREE = 2 * kStages, BAR_VFREE = 3 * kStages, BAR_SFULL = 4 * kStages,
       BAR_PFULL = BAR_SFULL + 2, BAR_OFULL = BAR_PFULL + 2, BAR_VRAW = BAR_OFULL + 2, BAR_KRAW, BAR_QFULL, BAR_QFREE, BAR_IFULL,
       BAR_IFREE = BAR_IFULL + 2, BAR_PARTS = BAR_IFREE + 2, BAR_TICKET, BAR_COUNT };
__host__ __device__ constexpr int arrivals_of(int bar) {
  return bar == BAR_PFULL || bar == BAR_PFULL + 1 ? 8
         : bar == BAR_IFREE || bar == BAR_IFREE + 1 ? kSoftmaxWarps + 3
         : bar == BAR_PARTS ? kSoftmaxWarps : 1;
}

// The same value, of which the compiler knows nothing: what is computed from it stays where it is written, instead of
// being kept in registers through the loop over the blocks, which has none to spare.
__device__ __forceinline__ int fresh(int x) {
  asm volatile("" : "+r"(x));
  return x;
}

struct PrefillJob {
  RowsView q, out;
  const int32_t* cu_q;
  int n_tokens, group;
  unsigned group_inv;                                // ceil(2^32 / group)
  float* part;                                       // [kMaxParts][kPartFloats], null: pieces are whole row tiles
  unsigned* counters;                                // next claim, CTAs that are through, arrivals [kSplitItems]; null: a fixed order
  int max_parts;
  int tile_rows;                                     // rows of a tile in use: whole tokens (128, or 125 to 127 for groups of 3, 5, 6, 7)
  int q_box;                                         // tokens per tile if the queries come by tiled copies, else 0
  int box_rows;                                      // slots per copy of a page
  int dim_slot, dim_head, dim_page;                  // tensor-map dimension (1..3) of each
};

// A piece of work: rows row0 .. row0 + rows - 1 of (sequence b, head h), blocks [idx0, idx1) of their walk.
struct Piece {
  int b, h, row0, q_first, rows;
  int kv_len, pos0;                                  // position of the sequence's first query token
  int prefix, win_lo, n_pre, first;                  // walk: blocks 0 .. n_pre - 1, then first, first + 1, ..
  int nb[2], total;                                  // blocks of the walk each tile needs; of the row tile
  int idx0, idx1;
  int seg, n_seg, item, part;                        // item: index of (row tile, head); part: of this piece's sums
};

// Everything in shared memory behind the operand tiles.
struct Control {
  uint64_t bar[BAR_COUNT];
  Piece piece[2];
  uint32_t tmem;
  int abort;
  unsigned ticket;
  int pair_flag[2][8][2];                            // [turn][warps of the same rows][half]
  float cap[14];                                     // products up to which the polynomial holds; its 6 coefficients; cap in base-2 units;
                                                     // scale / cap; products up to which 4 coefficients do; those
  PrefillJob job;                                    // the kernel's arguments, for the functions that are not inlined (a
  AttnOptions opt;                                   // reference to a parameter is read through global memory)
};

constexpr size_t kSmemBytes = 1024 + 2 * kTileBytes + 2 * kStages * kTileBytes + kSoftmaxWarps * kWarpStage + sizeof(Control);
static_assert(kSmemBytes <= 232448, "shared memory of a CTA");

// bounded wait that also gives up when another role has given up
__device__ __forceinline__ bool wait_bar(Control& ctl, int which, int completion, long long limit) {
  const uint32_t a = smem_u32(&ctl.bar[which]), parity = static_cast<uint32_t>(completion) & 1u;
  if (mbar_try_wait(a, parity)) return true;
  volatile int* abort_flag = &ctl.abort;
  const long long t0 = clock64();
  while (!*abort_flag) {
    if (mbar_try_wait(a, parity)) return true;
    if (clock64() - t0 > limit) *abort_flag = 1;
  }
  return false;
}

// The same without parking the thread between looks: for the one wait that is on the way of every product.
__device__ __forceinline__ bool spin_bar(Control& ctl, int which, uint32_t parity) {
  const uint32_t a = smem_u32(&ctl.bar[which]);
  const long long t0 = clock64();
  do {
    uint32_t done;
    asm volatile("{\n.reg .pred p;\nmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\nselp.u32 %0, 1, 0, p;\n}\n"
                 : "=r"(done) : "r"(a), "r"(parity & 1u) : "memory");
    if (done) return true;
  } while (clock64() - t0 < (1 << 14));
  return wait_bar(ctl, which, static_cast<int>(parity), kWaitLimit);
}

// row / group (exact for rows below 2^29: the product's error is row * group / 2^32 at most)
__device__ __forceinline__ int token_of(const PrefillJob& job, int row) {
  return job.group == 1 ? row : static_cast<int>(__umulhi(static_cast<unsigned>(row), job.group_inv));
}
// Row of a piece that the CTA's row r (tensor-memory lane r % 128 of tile r / 128) holds; -1: none.
__device__ __forceinline__ int row_at(const PrefillJob& job, const Piece& it, int r) {
  const int x = (r >> 7) * job.tile_rows + (r & 127);
  return (r & 127) < job.tile_rows && x < it.rows ? x : -1;
}
__device__ __forceinline__ int block_at(const Piece& it, int idx) { return idx < it.n_pre ? idx : it.first + idx - it.n_pre; }
__device__ __forceinline__ bool token_used(const Piece& it, int j) { return j < it.kv_len && (j >= it.win_lo || j < it.prefix); }

// Sequence b: its query rows, length and prefix.
struct Sequence {
  int first, n, kv_len, prefix;
};
__device__ __forceinline__ Sequence sequence(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, int b, bool report) {
  Sequence s;
  s.first = min(max(job.cu_q[b], 0), job.n_tokens);
  s.n = min(max(job.cu_q[b + 1], s.first), job.n_tokens) - s.first;
  s.kv_len = paged_len(pv, b, report);
  s.prefix = opt.prefix_len ? min(max(opt.prefix_len[b], 0), s.kv_len) : 0;
  return s;
}
__device__ __forceinline__ int row_tiles_of(const PrefillJob& job, const Sequence& s) { return (s.n * job.group + 2 * job.tile_rows - 1) / (2 * job.tile_rows); }

// The blocks that row tile rb of a sequence sees.
__device__ __forceinline__ void set_walk(const PrefillJob& job, const AttnOptions& opt, const Sequence& s, int rb, Piece& it) {
  it.row0 = rb * 2 * job.tile_rows;
  it.rows = min(2 * job.tile_rows, s.n * job.group - it.row0);
  it.q_first = s.first;
  it.kv_len = s.kv_len;
  it.pos0 = s.kv_len - s.n;
  it.prefix = s.prefix;
  const int p_lo = it.pos0 + token_of(job, it.row0);
  it.win_lo = opt.window > 0 ? max(0, p_lo - opt.window + 1) : 0;
  if (it.prefix >= it.win_lo) {
    it.win_lo = 0;
    it.n_pre = it.first = 0;
  } else {
    it.n_pre = (it.prefix + kBlock - 1) / kBlock;
    it.first = max(it.win_lo / kBlock, it.n_pre);
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int last = min(it.rows, job.tile_rows * (i + 1)) - 1;           // last row of the tile
    int end = 0;
    if (last >= job.tile_rows * i) {
      const int p = it.pos0 + token_of(job, it.row0 + last);
      end = p >= 0 ? p / kBlock + 1 : 0;
      if (it.win_lo == 0) end = max(end, (it.prefix + kBlock - 1) / kBlock);
      end = it.n_pre + max(0, end - it.first);
    }
    it.nb[i] = end;
  }
  it.total = max(it.nb[0], it.nb[1]);
}

// What all CTAs work out alike: row tiles of the call, and how they are cut.
struct Plan {
  int items, most;        // row tiles (of one head); of the longest sequence
  int segs, seg_blocks;   // pieces of a row tile at most; blocks per piece
  Sequence seq;           // sequence `lane`
  int mine;               // its row tiles
};

__device__ __forceinline__ int warp_sum(int x) { return __reduce_add_sync(0xffffffffu, x); }

__device__ __forceinline__ Plan make_plan(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, int lane, int grid) {
  Plan p;
  int items = 0, most = 0, long_blocks = 0;
  int mine_first = 0, mine_last = 0;                   // blocks of the first and the last row tile of sequence `lane`
  float blocks = 0.0f;
  p.mine = 0;
  p.seq = Sequence{0, 0, 0, 0};
  int tokens = 0;
  for (int b = lane; b < pv.batch && tokens <= job.n_tokens; b += 32) {
    const Sequence s = sequence(pv, opt, job, b, blockIdx.x == 0);
    const int n = row_tiles_of(job, s);
    tokens += s.n;
    if (b < 32) {
      p.seq = s;
      p.mine = n;
    }
    items += n;
    most = max(most, n);
    if (!job.part || n == 0) continue;
    Piece first, last;
    set_walk(job, opt, s, 0, first);
    set_walk(job, opt, s, n - 1, last);
    if (b < 32) {
      mine_first = first.total;
      mine_last = last.total;
    }
    long_blocks = max(long_blocks, max(first.total, last.total));
    blocks += 0.5f * static_cast<float>(n) * static_cast<float>(first.total + last.total);
  }
  tokens = warp_sum(tokens);
  if (tokens > job.n_tokens) {                         // sequences that share rows could have more row tiles than there are counters
    items = most = 0;
    if (blockIdx.x == 0 && lane == 0) paged_status(pv.status, MOQAE_ERR_INVALID_ARG, -1, tokens);
  }
  p.items = warp_sum(items);
  p.most = __reduce_max_sync(0xffffffffu, most);
  p.segs = 1;
  p.seg_blocks = 0x40000000;
  const int whole = p.items * pv.n_kv_heads;
  if (!job.part || whole == 0 || whole > kSplitItems) return p;
  const int longest = __reduce_max_sync(0xffffffffu, long_blocks);
  if (longest < 2 * kMinSegBlocks) return p;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) blocks += __shfl_xor_sync(0xffffffffu, blocks, o);
  // Lane s weighs s + 1 pieces for the longest row tile, in blocks (of 2 us): turns of one piece per CTA, each its blocks
  // and a fixed cost (3 us: queries, results; 7 us with the partial sums of a full row tile), what the longest piece is
  // above the mean, and the joining by one CTA (3.3 us per piece of a full row tile).
  const int segs = lane + 1, size = max((longest + segs - 1) / segs, kMinSegBlocks);
  const float heads = static_cast<float>(pv.n_kv_heads);
  float tiles = 0.0f;                                  // pieces of one head
  if (pv.batch <= 32) {
    for (int b = 0; b < pv.batch; ++b) {
      const int n = __shfl_sync(0xffffffffu, p.mine, b), f = __shfl_sync(0xffffffffu, mine_first, b), l = __shfl_sync(0xffffffffu, mine_last, b);
      tiles += 0.5f * static_cast<float>(n) * static_cast<float>(max(1, (f + size - 1) / size) + max(1, (l + size - 1) / size));
    }
  } else {
    tiles = blocks / static_cast<float>(size) + 0.5f * static_cast<float>(p.items);
  }
  if (segs == 1) tiles = static_cast<float>(p.items);
  const float mean = blocks / tiles;
  const float full = fminf(1.0f, static_cast<float>(job.n_tokens) * static_cast<float>(job.group) / (static_cast<float>(p.items) * static_cast<float>(2 * job.tile_rows)));
  float cost = ceilf(tiles * heads / static_cast<float>(grid) - 0.01f) * (mean + (segs == 1 ? 1.5f : 1.5f + 3.0f * full)) + static_cast<float>(size) - mean +
               (segs == 1 ? 0.0f : 2.5f + 1.6f * full * static_cast<float>(segs));
  if (segs > 1 && (whole * segs > job.max_parts || (longest + size - 1) / size < segs)) cost = 1e30f;
  int best = segs;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const float c = __shfl_xor_sync(0xffffffffu, cost, o);
    const int s = __shfl_xor_sync(0xffffffffu, best, o);
    if (c < cost || (c == cost && s < best)) {
      cost = c;
      best = s;
    }
  }
  if (best > 1) {
    p.segs = best;
    p.seg_blocks = max((longest + best - 1) / best, kMinSegBlocks);
  }
  return p;
}

// Claim -> piece; false: the row tile is cut into fewer pieces than this one's number.  Order of claims: piece number,
// then row tiles by their number in the sequence, the last first, then sequences, then heads (side by side in
// time, the CTAs of a head meet in its keys and values in the L2 cache).
__device__ __forceinline__ bool find_piece(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, const Plan& plan, unsigned claim,
                                           int lane, Piece& it) {
  const unsigned per_seg = static_cast<unsigned>(plan.items * pv.n_kv_heads);
  it.seg = plan.segs == 1 ? 0 : static_cast<int>(claim / per_seg);
  const int rest = static_cast<int>(claim - static_cast<unsigned>(it.seg) * per_seg);
  const int flat = rest / pv.n_kv_heads;
  it.h = rest - flat * pv.n_kv_heads;
  // row tiles with a number >= r: sum over the sequences of max(0, tiles - r); the tile's number is the largest r for
  // which this passes flat
  auto tiles_at = [&](int b) -> int { return b < pv.batch ? row_tiles_of(job, sequence(pv, opt, job, b, false)) : 0; };
  const int mine = plan.mine;
  auto at_least = [&](int r) -> int {
    int n = max(0, mine - r);
    for (int b = lane + 32; b < pv.batch; b += 32) n += max(0, tiles_at(b) - r);
    return warp_sum(n);
  };
  int lo = 0, hi = plan.most;                          // at_least(lo) > flat >= at_least(hi)
  int above = 0;                                       // at_least(lo + 1)
  if (pv.batch == 1) {
    lo = plan.most - 1 - flat;
    above = flat;
    hi = lo + 1;
  }
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1, n = at_least(mid);
    if (n > flat) lo = mid;
    else {
      hi = mid;
      above = n;
    }
  }
  int skip = flat - above;                             // among the sequences with more than lo tiles
  it.b = -1;
  for (int base = 0; base < pv.batch; base += 32) {
    const unsigned has = __ballot_sync(0xffffffffu, (base == 0 ? mine : tiles_at(base + lane)) > lo);
    const int n = __popc(has);
    if (skip >= n) {
      skip -= n;
      continue;
    }
    unsigned rest_bits = has;
    for (; skip > 0; --skip) rest_bits &= rest_bits - 1;
    it.b = base + __ffs(rest_bits) - 1;
    break;
  }
  if (it.b < 0) return false;
  Sequence seq;
  if (it.b < 32) {
    seq.first = __shfl_sync(0xffffffffu, plan.seq.first, it.b);
    seq.n = __shfl_sync(0xffffffffu, plan.seq.n, it.b);
    seq.kv_len = __shfl_sync(0xffffffffu, plan.seq.kv_len, it.b);
    seq.prefix = __shfl_sync(0xffffffffu, plan.seq.prefix, it.b);
  } else {
    seq = sequence(pv, opt, job, it.b, false);
  }
  set_walk(job, opt, seq, lo, it);
  // (a row tile between a sequence's first and last may see a block more than either)
  it.n_seg = plan.segs == 1 ? 1 : min(plan.segs, max(1, (it.total + plan.seg_blocks - 1) / plan.seg_blocks));
  if (it.seg >= it.n_seg) return false;
  it.idx0 = static_cast<int>(static_cast<long long>(it.total) * it.seg / it.n_seg);
  it.idx1 = static_cast<int>(static_cast<long long>(it.total) * (it.seg + 1) / it.n_seg);
  it.item = rest;
  it.part = rest * plan.segs + it.seg;
  return true;
}

// A softmax warp's 32 rows x 64 columns of O on their way out: results, or the float32 sums of a piece.  They leave through
// shared memory, 64 bytes of a row at a time, so that a store covers whole sectors of eight rows (a thread storing
// its own row took 32 half-sectors per instruction, 3 us for the 64 KiB of a CTA).
template <bool BF16>
__device__ __forceinline__ void store_rows(const PrefillJob& job, const Piece& it, uint32_t o_addr, bool has_sums, bool nothing, float inv,
                                        uint8_t* rows_at, int w_row, int half, int lane, float* piece) {
#pragma unroll 1
  for (int c4 = 0; c4 < 2; ++c4) {
    float v[32];
    if (has_sums) {
      tmem_ld32(v, o_addr + 32 * c4);
    } else {                                           // (never left undefined: that would keep 32 registers through the whole loop)
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = 0.0f;
    }
    if (nothing) {                                     // sees nothing here
#pragma unroll
      for (int e = 0; e < 32; ++e) v[e] = 0.0f;
    }
    const int parts = it.n_seg == 1 ? 1 : 2;           // results: 32 columns at once; sums: 16
#pragma unroll
    for (int part16 = 0; part16 < 2; ++part16) {
      if (part16 >= parts) break;
      if (parts == 1) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<uint4*>(rows_at + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
              make_uint4(float2_to_pair<BF16>(v[8 * e] * inv, v[8 * e + 1] * inv), float2_to_pair<BF16>(v[8 * e + 2] * inv, v[8 * e + 3] * inv),
                         float2_to_pair<BF16>(v[8 * e + 4] * inv, v[8 * e + 5] * inv), float2_to_pair<BF16>(v[8 * e + 6] * inv, v[8 * e + 7] * inv));
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          *reinterpret_cast<float4*>(rows_at + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
              make_float4(v[16 * part16 + 4 * e], v[16 * part16 + 4 * e + 1], v[16 * part16 + 4 * e + 2], v[16 * part16 + 4 * e + 3]);
      }
      __syncwarp();
#pragma unroll
      for (int k8 = 0; k8 < 4; ++k8) {
        const int r = 8 * k8 + (lane >> 2), u = lane & 3;
        const uint4 x = *reinterpret_cast<const uint4*>(rows_at + r * 64 + ((u ^ ((r >> 1) & 3)) << 4));
        const int mine = row_at(job, it, w_row + r);
        if (mine < 0) continue;
        if (parts == 1) {
          const int t = token_of(job, it.row0 + mine), g = it.row0 + mine - t * job.group;
          *reinterpret_cast<uint4*>(job.out.data + (it.q_first + t) * job.out.token + (it.h * job.group + g) * job.out.head + 64 * half + 32 * c4 + 8 * u) = x;
        } else {
          *reinterpret_cast<uint4*>(piece + mine * kHeadDim + 64 * half + 32 * c4 + 16 * part16 + 4 * u) = x;
        }
      }
      __syncwarp();
    }
  }
}

// The softmax threads add the pieces of a row tile: a thread takes four rows' units of 4 channels at a time, so that
// their loads are in flight together.
template <bool BF16> __device__ __forceinline__ void join_parts(const float* part, const Piece& it, const PrefillJob& job, int tid) {
  constexpr int kJoinThreads = kSoftmaxWarps * 32;
  const int units = it.rows * 32, n_seg = it.n_seg;
  for (int base = tid; base < units; base += 4 * kJoinThreads) {
    float m[4], lsum[4], acc[4][4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      m[k] = -INFINITY;
      lsum[k] = acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.0f;
    }
#pragma unroll 1
    for (int s = 0; s < n_seg; ++s) {
      const float* src = part + static_cast<long long>(s) * kPartFloats;
      float2 w[4];
      float4 v[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int x = min(base + k * kJoinThreads, units - 1);
        w[k] = __ldcg(reinterpret_cast<const float2*>(src + kItemRows * kHeadDim) + (x >> 5));
        v[k] = __ldcg(reinterpret_cast<const float4*>(src) + x);
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {                     // running reference: both sides are scaled to the larger
        const float top = fmaxf(m[k], w[k].x);
        const float f = w[k].x == -INFINITY ? 0.0f : ex2_approx(w[k].x - top), old = m[k] == -INFINITY ? 0.0f : ex2_approx(m[k] - top);
        m[k] = top;
        lsum[k] = fmaf(w[k].y, f, lsum[k] * old);
        acc[k][0] = fmaf(v[k].x, f, acc[k][0] * old);
        acc[k][1] = fmaf(v[k].y, f, acc[k][1] * old);
        acc[k][2] = fmaf(v[k].z, f, acc[k][2] * old);
        acc[k][3] = fmaf(v[k].w, f, acc[k][3] * old);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int x = base + k * kJoinThreads, row = x >> 5, c = (x & 31) * 4;
      if (x >= units) break;
      const float inv = lsum[k] == 0.0f ? 0.0f : 1.0f / lsum[k];
      const int t = token_of(job, it.row0 + row), g = it.row0 + row - t * job.group;
      *reinterpret_cast<uint2*>(job.out.data + (it.q_first + t) * job.out.token + (it.h * job.group + g) * job.out.head + c) =
          make_uint2(float2_to_pair<BF16>(acc[k][0] * inv, acc[k][1] * inv), float2_to_pair<BF16>(acc[k][2] * inv, acc[k][3] * inv));
    }
  }
}

// What a softmax thread brings out of the blocks of a piece.
struct SoftmaxState {
  float m_ref, l;        // reference and weight sum of its half row
  uint32_t phase;        // barrier parities (see the kernel)
  int ok;
};

// The softmax threads' loop over the blocks of a piece: two threads per row, 64 columns each, 32 at a time.
// A chunk's weights are stored over scores that this thread has read (half h of a tile: columns 64 h .. 64 h + 31 of S_i, so
// the products read P_i from two places), which keeps few registers live: the kernel has 96 per thread and next to no
// L1 cache beside its shared memory, a spill costs a trip to L2.
template <bool BF16, bool CAP, bool BIAS>
__device__ __forceinline__ SoftmaxState softmax_blocks(Control& ctl, int slot, uint32_t tmem, float* exch, uint32_t phase) {
    const AttnOptions& opt = ctl.opt;
    const PrefillJob& job = ctl.job;
    const Piece& it = ctl.piece[slot];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int half = warp >> 3, i = (warp & 7) >> 2, pair_id = warp & 7;
    const int row = 128 * i + 32 * (warp & 3) + lane;
    const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_addr + 128 * i + 64 * half, p_addr = s_addr;
    const uint32_t o_addr = lane_addr + 256 + 128 * i + 64 * half;
    const uint32_t bar0 = smem_u32(ctl.bar);
    auto bar = [&](int i) { return bar0 + 8u * i; };
    auto wait_all = [&](int which, int completion) -> bool { return __all_sync(0xffffffffu, wait_bar(ctl, which, completion, kWaitLimit)); };
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;\n" ::"r"(1 + pair_id) : "memory"); };
    // The two warps of the same rows meet and tell each other whether they are all right (flag 2: a wait ran
    // out, both leave) and whether a reference has to move (flag 1).  A warp whose wait ran out meets its
    // partner once more, wherever that is, so that nobody waits at the pair's barrier for good.
    auto meet = [&](int flag) -> int {
      volatile int* f = ctl.pair_flag[phase >> 3][pair_id];
      phase ^= 8;
      if (lane == 0) f[half] = flag;
      pair_sync();
      return f[0] | f[1];
    };
    const float scale_log2 = opt.scale * kLog2e;
    float slope = 0.0f;
    const bool live = row_at(job, it, row) >= 0;
    const volatile float* cap_of = ctl.cap;            // (the constants of the cap stay in shared memory between uses)
    // Scores of columns 32 c .. 32 c + 31 in base-2 units, plus `off`; `mul` and `add` are what is left to be done (nothing under
    // a cap, an addition with a bias, else both); column e is seen if lo < e <= hi or e < pre.
    auto scores = [&](auto masked, float (&v)[32], int c, float off, int hi, int lo, int pre, float& mul, float& add) {
      tmem_ld32(v, s_addr + 32 * c);
      mul = CAP || BIAS ? 1.0f : scale_log2;
      add = CAP ? 0.0f : off;
      // The bias of column e is slope * (e - dist), one step of arithmetic per pair with `off` in it; where tokens behind
      // the query may be seen it follows by itself.
      const float dist = static_cast<float>(hi - 32 * c);                 // of column 0
      const bool behind = BIAS && pre > 0;
      const float step = BIAS && !behind ? slope : 0.0f, base = BIAS ? fmaf(-step, dist, off) : off;
      // (column numbers are constants of the instruction here; as packed pairs they would have to be moved to registers)
      auto rest = [&](int e) -> uint64_t {
        return BIAS ? pack_f2(fmaf(step, static_cast<float>(e), base), fmaf(step, static_cast<float>(e + 1), base)) : pack_f2(base, base);
      };
      if (CAP) {
        // (the forms differ in their last bits: rows that hold nothing have no say, and tokens that nobody uses score 0)
        float big = 0.0f;
#pragma unroll
        for (int e = 0; e < 32; e += 2) asm("max.abs.f32 %0, %1, %2, %0;\n" : "+f"(big) : "f"(v[e]), "f"(v[e + 1]));
        const bool near = __all_sync(0xffffffffu, !live || big <= cap_of[9]);
        if (near) {                                                       // |x / cap| <= 1/2: 5 steps per pair instead of 7
          uint64_t t[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x = cap_of[10 + k];
            t[k] = pack_f2(x, x);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const uint64_t y = pack_f2(v[e], v[e + 1]), u = mul_f2(y, y);
            unpack_f2(fma_f2(y, fma_f2(fma_f2(fma_f2(t[3], u, t[2]), u, t[1]), u, t[0]), rest(e)), v[e], v[e + 1]);
          }
        } else if (__all_sync(0xffffffffu, !live || big <= cap_of[0])) {
          uint64_t t[6];
#pragma unroll
          for (int k = 0; k < 6; ++k) {
            const float x = cap_of[1 + k];
            t[k] = pack_f2(x, x);
          }
#pragma unroll
          for (int e = 0; e < 32; e += 2) {
            const uint64_t y = pack_f2(v[e], v[e + 1]), u = mul_f2(y, y);
            unpack_f2(fma_f2(y, fma_f2(fma_f2(fma_f2(fma_f2(fma_f2(t[5], u, t[4]), u, t[3]), u, t[2]), u, t[1]), u, t[0]), rest(e)), v[e], v[e + 1]);
          }
        } else {                                                          // some score passes the cap
          const float w = cap_of[8];
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(cap_of[7], tanh_of(v[e] * w), fmaf(step, static_cast<float>(e), base));
        }
      } else if (BIAS) {                                                  // (in `rest`, too, it would cost registers that are not there)
        const uint64_t scale2 = pack_f2(scale_log2, scale_log2);
#pragma unroll
        for (int e = 0; e < 32; e += 2) unpack_f2(mul_f2(pack_f2(v[e], v[e + 1]), scale2), v[e], v[e + 1]);
        if (pre > 0) {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(-slope, fabsf(dist - static_cast<float>(e)), v[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(slope, static_cast<float>(e), v[e]);
          add = off - slope * dist;
        }
      }
      if (CAP && behind) {
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] = fmaf(-slope, fabsf(dist - static_cast<float>(e)), v[e]);
      }
      if (masked) {
        if (pre <= 0 && opt.window == 0) {                                // the diagonal alone
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (32 * c + e > hi) v[e] = -INFINITY;
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e)
            if (!((32 * c + e <= hi && 32 * c + e > lo) || 32 * c + e < pre)) v[e] = -INFINITY;
        }
      }
    };
    // weights of a chunk against the reference, packed; their sum
    auto weights = [&](auto masked, int c, float ref, int hi, int lo, int pre, uint32_t (&pk)[16]) -> float {
      float v[32], mul, add;
      uint64_t part[2] = {0ull, 0ull};
      if (CAP && !decltype(masked)::value && !(BIAS && pre > 0)) {
        // The ordinary chunk under a cap in one go: arithmetic and exponentials of different columns overlap.
        tmem_ld32(v, s_addr + 32 * c);
        float big = 0.0f;
#pragma unroll
        for (int e = 0; e < 32; e += 2) asm("max.abs.f32 %0, %1, %2, %0;\n" : "+f"(big) : "f"(v[e]), "f"(v[e + 1]));
        if (__all_sync(0xffffffffu, !live || big <= cap_of[9])) {
          uint64_t t[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float x = cap_of[10 + k];
            t[k] = pack_f2(x, x);
          }
          const float base = BIAS ? fmaf(-slope, static_cast<float>(hi - 32 * c), -ref) : -ref;
#pragma unroll
          for (int e2 = 0; e2 < 16; ++e2) {
            const uint64_t rest = BIAS ? pack_f2(fmaf(slope, static_cast<float>(2 * e2), base), fmaf(slope, static_cast<float>(2 * e2 + 1), base))
                                       : pack_f2(base, base);
            const uint64_t y = pack_f2(v[2 * e2], v[2 * e2 + 1]), u = mul_f2(y, y);
            float x0, x1;
            unpack_f2(fma_f2(y, fma_f2(fma_f2(fma_f2(t[3], u, t[2]), u, t[1]), u, t[0]), rest), x0, x1);
            const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
            pk[e2] = float2_to_pair<BF16>(p0, p1);
            part[e2 & 1] = add_f2(part[e2 & 1], pack_f2(p0, p1));
          }
          float s0, s1;
          unpack_f2(add_f2(part[0], part[1]), s0, s1);
          return s0 + s1;
        }
      }
      scores(masked, v, c, -ref, hi, lo, pre, mul, add);
      const uint64_t scale2 = pack_f2(mul, mul), negm2 = pack_f2(add, add);
#pragma unroll
      for (int e2 = 0; e2 < 16; ++e2) {
        float x0, x1;
        const uint64_t vv = pack_f2(v[2 * e2], v[2 * e2 + 1]);
        unpack_f2(CAP ? vv : BIAS ? add_f2(vv, negm2) : fma_f2(vv, scale2, negm2), x0, x1);
        const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
        pk[e2] = float2_to_pair<BF16>(p0, p1);
        const float2 r = decltype(masked)::value ? pair_to_float2<BF16>(pk[e2]) : make_float2(p0, p1);
        part[e2 & 1] = add_f2(part[e2 & 1], pack_f2(r.x, r.y));
      }
      float s0, s1;
      unpack_f2(add_f2(part[0], part[1]), s0, s1);
      return s0 + s1;
    };
    // multiply the packed weights of chunk c by a power of two
    auto rescale_weights = [&](int c, float f) {
      uint32_t pw[16];
      tmem_ld16u(pw, p_addr + 16 * c);
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const float2 x = pair_to_float2<BF16>(pw[e]);
        pw[e] = float2_to_pair<BF16>(x.x * f, x.y * f);
      }
      tmem_st16u_nowait(p_addr + 16 * c, pw);
    };
    const int n_blocks = it.idx1 - it.idx0, first = min(max(it.idx1 - it.nb[i], 0), n_blocks);
    // rows behind the last one take its position: they cost no extra mask and are not stored
    auto position = [&](int r) {
      return it.pos0 + token_of(job, it.row0 + min((r >> 7) * job.tile_rows + min(r & 127, job.tile_rows - 1), it.rows - 1));
    };
    const int qpos = position(row);
    // tokens all_from .. all_to are seen by every row of the warp
    const int all_to = position(row & ~31), all_from = opt.window > 0 ? position(row | 31) - opt.window + 1 : -0x40000000;
    if (BIAS) {
      const int my_row = row_at(job, it, row);
      slope = my_row >= 0 ? opt.slopes[it.h * job.group + it.row0 + my_row - token_of(job, it.row0 + my_row) * job.group] * kLog2e : 0.0f;
    }
    float m_ref = -INFINITY, l = 0.0f;
    bool ok = true;
    for (int n = first; n < n_blocks && ok; ++n) {
      const int j0 = block_at(it, it.idx1 - 1 - n) * kBlock + 64 * half;  // token of this thread's first column
      const int hi = qpos - j0, lo = opt.window > 0 ? hi - opt.window : -0x40000000, pre = it.prefix - j0;
      const bool masked = !(j0 + 63 <= all_to && j0 >= all_from) && pre < 64;
      ok = wait_all(BAR_SFULL + i, phase);
      if (ok) tc_fence_after();
      if (ok && n == first) {
        // The first reference: any score that the row sees will do (its weight is then between a half and 1, times
        // 2^kLead, and larger scores may lead by the rest of kSumLimit).  All rows of the warp see token all_to, if this block
        // holds it; both threads of a row read its column, without a word between them.
        const int col = min(all_to - (j0 - 64 * half), kBlock - 1);
        if (col >= 0 && j0 - 64 * half + col >= all_from) {
          uint32_t raw;
          asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n" : "=r"(raw) : "r"(lane_addr + 128 * i + col));
          asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          float y = __uint_as_float(raw) * scale_log2;
          if (CAP) y = cap_of[7] * tanh_of(__uint_as_float(raw) * cap_of[8]);
          if (BIAS) y -= slope * static_cast<float>(qpos - (j0 - 64 * half + col));
          if (y > -1e30f && y < 1e30f) m_ref = ceilf(y) - kLead<BF16>;
        }
        // its partner overwrites a column of the other half only after both have read it
        if (meet(0) & 2) {
          ok = false;
          break;
        }
      }
      const float m_old = m_ref;
      float sum = 0.0f;
      bool moved = false;
      if (ok) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          uint32_t pk[16];
          float csum = masked ? weights(std::true_type{}, c, m_ref, hi, lo, pre, pk) : weights(std::false_type{}, c, m_ref, hi, lo, pre, pk);
          if (__any_sync(0xffffffffu, live && (!(csum < kSumLimit<BF16>) || m_ref == -INFINITY))) {
            // Rare: the weights add up to more than kSumLimit, or the row had seen nothing before.  The reference
            // moves to the chunk's largest score, the weights are formed again, what was stored follows.  A row that
            // still sees nothing keeps -inf and weighs its columns, all masked, against 0.
            float v[32], mul, add;
            scores(std::true_type{}, v, c, 0.0f, hi, lo, pre, mul, add);
            float top = v[0];
#pragma unroll
            for (int e = 1; e < 32; ++e) top = fmaxf(top, v[e]);
            const float m_new = fmaxf(m_ref, ceilf(fmaf(top, mul, add)) - kLead<BF16>);  // mul > 0
            const float corr = m_ref == -INFINITY ? 0.0f : ex2_approx(m_ref - m_new);
            if (c) {
              tmem_st_wait();
              rescale_weights(0, corr);
            }
            sum *= corr;
            m_ref = m_new;
            moved = true;
            csum = weights(std::true_type{}, c, m_ref == -INFINITY ? 0.0f : m_ref, hi, lo, pre, pk);
          }
          sum += csum;
          tmem_st16u_nowait(p_addr + 16 * c, pk);
        }
        tmem_st_wait();
      }
      const int flags = meet((moved ? 1 : 0) | (ok ? 0 : 2));
      if (flags & 2) {
        ok = false;
        break;
      }
      if (flags & 1) {
        // both threads of a row go on with the larger of their references
        exch[lane * 2 + half] = m_ref;
        pair_sync();
        const float m_new = fmaxf(exch[lane * 2], exch[lane * 2 + 1]);
        const float corr = m_ref == -INFINITY ? 0.0f : ex2_approx(m_ref - m_new);
        if (__any_sync(0xffffffffu, corr != 1.0f)) {
          rescale_weights(0, corr);
          rescale_weights(1, corr);
          tmem_st_wait();
          sum *= corr;
        }
        const float corr_old = m_old == -INFINITY ? 0.0f : ex2_approx(m_old - m_new);
        if (n > first) {
#pragma unroll 1
          for (int o4 = 0; o4 < 2; ++o4) {
            float o[32];
            tmem_ld32(o, o_addr + 32 * o4);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= corr_old;
            tmem_st32(o_addr + 32 * o4, o);
          }
        }
        l *= corr_old;
        m_ref = m_new;
      }
      l += sum;
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_PFULL + i));
      phase ^= 1;
    }
    return {m_ref, l, phase, ok ? 1 : 0};
}

template <bool BF16, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
paged_prefill_kernel(PagedView pv, AttnOptions opt, PrefillJob job, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v, const __grid_constant__ CUtensorMap map_q) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* sQ = smem;
  uint8_t* sK = sQ + 2 * kTileBytes;
  uint8_t* sV = sK + kStages * kTileBytes;
  uint8_t* sOut = sV + kStages * kTileBytes;           // [softmax warps][kWarpStage]
  Control& ctl = *reinterpret_cast<Control*>(sOut + kSoftmaxWarps * kWarpStage);
  const uint32_t bar0 = smem_u32(ctl.bar);
  auto bar = [&](int i) { return bar0 + 8u * i; };
  volatile int* abort_flag = &ctl.abort;

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  after_previous();
  // The planning warp has the first piece before the CTA's barriers stand.
  Plan plan;
  Piece it;                                            // (of the planning warp)
  unsigned claims = 0, claim = blockIdx.x;
  bool found = false;
  if (warp == kPlanWarp) {
    plan = make_plan(pv, opt, job, lane, static_cast<int>(gridDim.x));
    claims = static_cast<unsigned>(plan.items * pv.n_kv_heads) * static_cast<unsigned>(plan.segs);
    if (claim < claims) found = find_piece(pv, opt, job, plan, claim, lane, it);
  }
  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(&ctl.tmem)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (tid == kKeyWarp * 32) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_v) : "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_q) : "memory");
    for (int i = 0; i < BAR_COUNT; ++i) mbar_init(bar(i), arrivals_of(i));
    *abort_flag = 0;
    if (CAP) {
      // Up to the cap, cap tanh(x / cap) is a polynomial in the raw product: powers of w = scale / cap go into the
      // coefficients, where float32 holds them (otherwise every score takes the general way).
      const float w = opt.scale / opt.cap, cap2 = opt.cap * kLog2e;
      ctl.cap[0] = w > 1e-3f && w < 1e3f ? 1.0f / w : -1.0f;
      float power = w * cap2;
      for (int k = 0; k < 6; ++k, power *= w * w) ctl.cap[1 + k] = tanh_coef(k) * power;
      ctl.cap[9] = 0.5f * ctl.cap[0];
      power = w * cap2;
      for (int k = 0; k < 4; ++k, power *= w * w) ctl.cap[10 + k] = tanh_coef_near(k) * power;
      ctl.cap[7] = cap2;
      ctl.cap[8] = w;
    }
    ctl.job = job;
    ctl.opt = opt;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = ctl.tmem;

  auto wait = [&](int which, int completion, long long limit = kWaitLimit) -> bool { return wait_bar(ctl, which, completion, limit); };
  auto wait_all = [&](int which, int completion, long long limit = kWaitLimit) -> bool {
    return __all_sync(0xffffffffu, wait(which, completion, limit));
  };

  if (warp < kSoftmaxWarps) {
    // ================= softmax, two threads per row (see prefill.cu) =================
    const int half = warp >> 3, i = (warp & 7) >> 2, pair_id = warp & 7;
    const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    float* exch = reinterpret_cast<float*>(sOut + 2 * pair_id * kWarpStage);   // [32 rows][2 halves], while no rows are staged there
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;\n" ::"r"(1 + pair_id) : "memory"); };
    // The two warps of the same rows meet and tell each other whether they are all right (flag 2: a wait ran
    // out, both leave) and whether a reference has to move (flag 1).  A warp that leaves, because its wait ran out or because there
    // is no more work, meets its partner once more, wherever that is, so that nobody waits at the pair's barrier for good.
    uint32_t phase = 0;                                // parities: 1 sfull / pfull, 2 ofull, 4 parts / ticket, 8 turn of the flags
    auto meet = [&](int flag) -> int {
      volatile int* f = ctl.pair_flag[phase >> 3][pair_id];
      phase ^= 8;
      if (lane == 0) f[half] = flag;
      pair_sync();
      return f[0] | f[1];
    };
    for (int k = 0;; ++k) {
    const Piece& it = ctl.piece[k & 1];
    if (!wait_all(BAR_IFULL + (k & 1), k >> 1, kPieceWaitLimit)) {
      meet(2);
      break;
    }
    if (it.rows == 0) {                                // no more work
      meet(0);
      break;
    }
    const int n_blocks = it.idx1 - it.idx0, first = min(max(it.idx1 - it.nb[i], 0), n_blocks);
    const SoftmaxState state = softmax_blocks<BF16, CAP, BIAS>(ctl, k & 1, tmem, exch, phase);
    phase = state.phase;
    // A tile without blocks in this piece exchanges nothing (both sums are 0): its warps have not met since they sent out
    // the rows of the piece before, and the place of the sums may still hold rows of the partner's.
    const bool worked = first < n_blocks;
    bool ok = state.ok;
    if (ok && worked) {
      ok = wait_all(BAR_OFULL + i, phase >> 1);
      phase ^= 2;
      exch[lane * 2 + half] = state.l;
      ok = !(meet(ok ? 0 : 2) & 2);
    }
    if (!ok) break;
    tc_fence_after();
    const int ln = fresh(lane), wp = fresh(warp), out_half = wp >> 3;   // see fresh()
    uint8_t* rows_at = sOut + (2 * (wp & 7) + out_half) * kWarpStage;
    float lt = 0.0f;
    if (worked) {
      lt = exch[ln * 2] + exch[ln * 2 + 1];
      pair_sync();                                     // the sums have been read: their place takes rows
    }
    const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
    float* piece = job.part + static_cast<long long>(it.part) * kPartFloats;
    store_rows<BF16>(ctl.job, it, lane_addr + 256 + 128 * i + 64 * half, worked, lt == 0.0f, inv, rows_at, 32 * (wp & 7), out_half, ln, piece);
    if (it.n_seg > 1) {
      // ---- the last piece of a row tile to arrive joins all of them, in the order of their tokens ----
      const int mine = row_at(ctl.job, it, 32 * (wp & 7) + ln);
      if (out_half == 0 && mine >= 0) *reinterpret_cast<float2*>(piece + kItemRows * kHeadDim + 2 * mine) = make_float2(state.m_ref, lt);
      __threadfence();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_PARTS));
      ok = true;
      if (warp == 0) {
        ok = wait_all(BAR_PARTS, phase >> 2);
        if (ok && lane == 0) {
          __threadfence();
          ctl.ticket = atomicInc(job.counters + 2 + it.item, static_cast<unsigned>(it.n_seg - 1));
          mbar_arrive(bar(BAR_TICKET));
        }
      }
      if (ok) ok = wait_all(BAR_TICKET, phase >> 2);
      phase ^= 4;
      if (!ok) {
        meet(2);                                       // wherever the partner is, it leaves too
        break;
      }
      if (*const_cast<volatile unsigned*>(&ctl.ticket) == static_cast<unsigned>(it.n_seg - 1)) {
        __threadfence();
        const float* part = job.part + static_cast<long long>(it.part - it.seg) * kPartFloats;
        join_parts<BF16>(part, it, ctl.job, 32 * wp + ln);
      }
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(BAR_IFREE + (k & 1)));
    }
  } else if (warp == kPlanWarp) {
    // ================= plan: claim pieces, bring their queries =================
    auto next_claim = [&](unsigned claim) -> unsigned {
      if (!job.counters) return claim + gridDim.x < claim ? claims : claim + gridDim.x;
      unsigned next = 0;
      if (lane == 0) next = atomicAdd(job.counters, 1u);
      return gridDim.x + __shfl_sync(0xffffffffu, next, 0);
    };
    bool ok = true;
    for (int k = 0; ok; ++k) {
      while (!found && claim < claims) {
        found = find_piece(pv, opt, job, plan, claim, lane, it);
        if (!found) claim = next_claim(claim);
      }
      if (!found) it.rows = 0;
      if (k >= 2) ok = wait_all(BAR_IFREE + (k & 1), (k >> 1) - 1, kPieceWaitLimit);
      if (!ok) break;
      if (lane == 0) {
        ctl.piece[k & 1] = it;
        mbar_arrive(bar(BAR_IFULL + (k & 1)));
      }
      if (!found) break;
      if (job.q_box) {
        // whole tokens fill a tile: two tiled copies of 64 channels each; rows behind the sequence's last hold other
        // sequences' queries, whose results are dropped
        const int tiles = it.rows > job.tile_rows ? 2 : 1;
        if (lane == 0) mbar_expect_tx(bar(BAR_QFULL), tiles * job.tile_rows * 256);
        __syncwarp();
        if (lane < 2 * tiles) {
          const int tile = lane >> 1, part = lane & 1;
          tma_load_3d(smem_u32(sQ) + tile * kTileBytes + part * (kTileBytes / 2), &map_q, 64 * part, it.h * job.group,
                      it.q_first + token_of(job, it.row0) + tile * job.q_box, bar(BAR_QFULL));
        }
      } else {
        // strides that the copy engine cannot express: 16-byte units by plain loads, rows that hold nothing zero
        for (int x = lane; x < kItemRows * 16; x += 32) {
          const int r = x >> 4, u = x & 15, mine = row_at(job, it, r), t = token_of(job, it.row0 + max(mine, 0)), g = it.row0 + mine - t * job.group;
          uint4 v = make_uint4(0u, 0u, 0u, 0u);
          if (mine >= 0) v = *reinterpret_cast<const uint4*>(job.q.data + (it.q_first + t) * job.q.token + (it.h * job.group + g) * job.q.head + 8 * u);
          *reinterpret_cast<uint4*>(sQ + (r >> 7) * kTileBytes + (u >> 3) * (kTileBytes / 2) + (r & 127) * 128 + (((u ^ r) & 7) << 4)) = v;
        }
        fence_async_proxy();
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(BAR_QFULL));
      }
      // The next claim waits until the last product with these queries is done, a block before the piece's end: a
      // CTA that claimed earlier would take work that another is free for.
      ok = wait_all(BAR_QFREE, k, kPieceWaitLimit);
      if (!ok) break;
      claim = next_claim(claim);
      found = false;
    }
    // the last CTA to find no more work leaves the counters at zero
    if (job.counters && lane == 0 && atomicInc(job.counters + 1, gridDim.x - 1) == gridDim.x - 1) atomicExch(job.counters, 0u);
  } else if (warp > kIssueWarp) {
    // ================= fetch: key blocks (one warp) and value blocks (another) =================
    const bool is_v = warp == kValueWarp;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    const int boxes = kBlock / job.box_rows;
    int n_raw = 0, g = 0;                               // edge blocks, blocks of all pieces
    bool ok = true;
    for (int k = 0;; ++k) {
      if (!wait_all(BAR_IFULL + (k & 1), k >> 1, kPieceWaitLimit)) break;
      const Piece it = ctl.piece[k & 1];
      if (it.rows == 0) break;
      const int n_blocks = it.idx1 - it.idx0;
      auto box_token = [&](int n) { return block_at(it, it.idx1 - 1 - n) * kBlock + lane * job.box_rows; };
      auto look_up = [&](int n) -> int {                // page of this lane's box, -1: not needed
        if (n >= n_blocks || lane >= boxes) return -1;
        const int j = box_token(n);
        if (j >= it.kv_len || !(j + job.box_rows > it.win_lo || j < it.prefix)) return -1;
        const int page = pv.table[static_cast<long long>(it.b) * pv.max_pages + (j >> pv.page_shift)];
        if (page >= 0 && page < pv.n_pages) return page;
        paged_status(pv.status, MOQAE_ERR_CORRUPT_TABLE, it.b, j >> pv.page_shift);
        return max(pv.n_pages, 1);                      // outside the map: the copy fills zeros
      };
      int page = look_up(0);
      for (int n = 0; n < n_blocks; ++n, ++g) {
        const int st = g % kStages;
        const int next = look_up(n + 1);
        if (g >= kStages && !wait_all((is_v ? BAR_VFREE : BAR_KFREE) + st, g / kStages - 1)) {
          ok = false;
          break;
        }
        const int j0 = block_at(it, it.idx1 - 1 - n) * kBlock;
        const bool edge = (is_v || CAP) && (j0 + kBlock > it.kv_len || (j0 < it.win_lo && j0 + kBlock > it.prefix));
        const int raw = is_v ? BAR_VRAW : BAR_KRAW;
        const uint32_t full = bar((is_v ? BAR_VFULL : BAR_KFULL) + st), landed = edge ? bar(raw) : full;
        const unsigned need = __ballot_sync(0xffffffffu, page >= 0);
        if (lane == 0) mbar_expect_tx(landed, __popc(need) * job.box_rows * 256);
        __syncwarp();
        uint8_t* dst = (is_v ? sV : sK) + st * kTileBytes;
        if (page >= 0) {
          const int slot = box_token(n) & (pv.page_size - 1);
          const int y = job.dim_slot == 1 ? slot : (job.dim_head == 1 ? it.h : page);
          const int z = job.dim_slot == 2 ? slot : (job.dim_head == 2 ? it.h : page);
          const int w = job.dim_slot == 3 ? slot : (job.dim_head == 3 ? it.h : page);
          const uint32_t d = smem_u32(dst) + lane * job.box_rows * 128;
          tma_load_4d(d, map, 0, y, z, w, landed);                        // channels 0..63
          tma_load_4d(d + kTileBytes / 2, map, 64, y, z, w, landed);      // channels 64..127
        }
        if (edge) {
          if (!wait_all(raw, n_raw++)) {
            ok = false;
            break;
          }
          for (int r = lane; r < kBlock; r += 32)
            if (!token_used(it, j0 + r)) {
#pragma unroll
              for (int u = 0; u < 8; ++u) {
                *reinterpret_cast<uint4*>(dst + r * 128 + u * 16) = make_uint4(0, 0, 0, 0);
                *reinterpret_cast<uint4*>(dst + kTileBytes / 2 + r * 128 + u * 16) = make_uint4(0, 0, 0, 0);
              }
            }
          fence_async_proxy();
          __syncwarp();
          if (lane == 0) mbar_arrive(full);
        }
        page = next;
      }
      if (!ok) break;
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_IFREE + (k & 1)));
    }
    if (*abort_flag) {                                  // copies under way still land in this CTA's memory: let them
      const long long t0 = clock64();
      while (clock64() - t0 < (1 << 17)) {
      }
    }
  } else {
    // ================= MMA issue (one thread) =================
    constexpr uint32_t kFormat = BF16 ? (1u << 7) | (1u << 10) : 0u;      // operand type
    constexpr uint32_t kIdescS = (1u << 4) | kFormat | (16u << 17) | (8u << 24), kIdescPV = kIdescS | (1u << 16);
    const uint64_t qd = make_desc_sw128(smem_u32(sQ), 16, 1024);
    const uint64_t kd = make_desc_sw128(smem_u32(sK), 16, 1024), vd = make_desc_sw128(smem_u32(sV), kTileBytes / 2, 1024);
    const uint32_t qd_lo = static_cast<uint32_t>(qd), qd_hi = static_cast<uint32_t>(qd >> 32);
    const uint32_t kd_lo = static_cast<uint32_t>(kd), kd_hi = static_cast<uint32_t>(kd >> 32);
    const uint32_t vd_lo = static_cast<uint32_t>(vd), vd_hi = static_cast<uint32_t>(vd >> 32);
    static_assert(kStages == 2, "the stage of a block is its parity");
    uint32_t g = 0;                                     // blocks of all pieces so far
    uint32_t p_done = 0;                                // parities of pfull, one bit per tile
    bool ok = lane == 0;
    for (int k = 0; ok; ++k) {
      if (!wait(BAR_IFULL + (k & 1), k >> 1, kPieceWaitLimit)) break;
      const Piece& piece = ctl.piece[k & 1];
      if (piece.rows == 0) break;
      const int n_blocks = piece.idx1 - piece.idx0;
      // block idx1 - 1 - n is worked on at step n; tile i joins at step first0 / first1
      const int first0 = min(max(piece.idx1 - piece.nb[0], 0), n_blocks), first1 = min(max(piece.idx1 - piece.nb[1], 0), n_blocks);
      // the stage is free after the last tile that reads it: tile 1, or tile 0 where tile 1 has no such block
      auto issue_s = [&](int i, uint32_t st, bool frees, bool last) {
        const uint32_t a_lo = qd_lo + i * (kTileBytes >> 4), b_lo = kd_lo + st * (kTileBytes >> 4), d = tmem + 128 * i;
#pragma unroll
        for (int s = 0; s < 8; ++s)
          umma_f16_ss(d, a_lo + (s >> 2) * 1024 + (s & 3) * 2, qd_hi, b_lo + (s >> 2) * 1024 + (s & 3) * 2, kd_hi, kIdescS, s > 0);
        umma_commit(bar(BAR_SFULL + i));
        if (frees) {
          umma_commit(bar(BAR_KFREE + st));
          if (last) umma_commit(bar(BAR_QFREE));
        }
      };
      auto issue_pv = [&](int i, uint32_t st, bool frees, bool first, bool last) {
        const uint32_t lo = vd_lo + st * (kTileBytes >> 4), d = tmem + 256 + 128 * i, a = tmem + 128 * i;
        umma_f16_ta(d, a, lo, vd_hi, kIdescPV, !first);
#pragma unroll
        for (int s = 1; s < 8; ++s) umma_f16_ta(d, a + (s >> 2) * 32 + 8 * s, lo + 128 * s, vd_hi, kIdescPV, 1u);
        if (frees) umma_commit(bar(BAR_VFREE + st));
        if (last) umma_commit(bar(BAR_OFULL + i));
      };
      ok = wait(BAR_QFULL, k, kPieceWaitLimit);
      if (ok && n_blocks > 0) {
        ok = wait(BAR_KFULL + (g & 1), g >> 1);
        if (ok) {
          tc_fence_after();
          if (first0 == 0) issue_s(0, g & 1, 0 < first1, n_blocks == 1);
          if (first1 == 0) issue_s(1, g & 1, true, n_blocks == 1);
        }
      } else if (ok) {
        mbar_arrive(bar(BAR_QFREE));
      }
      for (int n = 0; n < n_blocks && ok; ++n, ++g) {
        const uint32_t st = g & 1, next = st ^ 1;
        const bool more = n + 1 < n_blocks, last_s = n + 2 == n_blocks;
        ok = wait(BAR_VFULL + st, g >> 1);
        if (ok && more) ok = wait(BAR_KFULL + next, (g + 1) >> 1);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int first = i ? first1 : first0;
          if (ok && n >= first) {
            ok = spin_bar(ctl, BAR_PFULL + i, p_done >> i);
            p_done ^= 1u << i;
          }
          if (!ok) break;
          tc_fence_after();
          if (n >= first) issue_pv(i, st, i == 1 || n < first1, n == first, !more);
          if (more && n + 1 >= first) issue_s(i, next, i == 1 || n + 1 < first1, last_s);
        }
      }
      mbar_arrive(bar(BAR_IFREE + (k & 1)));
    }
    __syncwarp();
  }
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && *abort_flag) paged_status(pv.status, MOQAE_ERR_TIMEOUT, static_cast<int>(blockIdx.x), -1);   // whoever gave up
  if (warp == kIssueWarp)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols) : "memory");
}

// (channel, slot, head, page) with the last three in the order of their strides; boxes of 64 channels x rows slots
bool make_page_map(CUtensorMap* m, const void* base, const PagedView& pv, const long long stride[3], const int order[3], int rows) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return false;
  const cuuint64_t size[3] = {static_cast<cuuint64_t>(pv.page_size), static_cast<cuuint64_t>(pv.n_kv_heads),
                              static_cast<cuuint64_t>(pv.n_pages > 0 ? pv.n_pages : 1)};
  cuuint64_t gdim[4] = {kHeadDim, 0, 0, 0}, gstride[3];
  cuuint32_t box[4] = {64, 1, 1, 1};
  const cuuint32_t estr[4] = {1, 1, 1, 1};
  for (int d = 0; d < 3; ++d) {
    gdim[d + 1] = size[order[d]];
    gstride[d] = static_cast<cuuint64_t>(stride[order[d]]) * 2;
    if (order[d] == 0) box[d + 1] = static_cast<cuuint32_t>(rows);
  }
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 4, const_cast<void*>(base), gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries (channel, head, token); boxes of 64 channels x the group's heads x the tokens of a tile.  False where the strides
// cannot be expressed.
bool make_query_map(CUtensorMap* m, const RowsView& q, int n_tokens, int group) {
  EncodeTiledFn enc = encode_tiled_fn();
  if (!enc) return false;
  const cuuint64_t gdim[3] = {kHeadDim, static_cast<cuuint64_t>(q.n_heads), static_cast<cuuint64_t>(n_tokens)};
  const cuuint64_t gstride[2] = {static_cast<cuuint64_t>(q.head) * 2, static_cast<cuuint64_t>(q.token) * 2};
  const cuuint32_t box[3] = {64, static_cast<cuuint32_t>(group), static_cast<cuuint32_t>(kTileRows / group)};
  const cuuint32_t estr[3] = {1, 1, 1};
  if ((q.n_heads > 1 && q.head == 0) || (n_tokens > 1 && q.token == 0)) return false;
  return enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT16, 3, q.data, gdim, gstride, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// row tiles of all sequences, at most: sum of ceil(rows / (two tiles' rows))
long long row_tiles(int batch, int group, int n_tokens) {
  const int rows = 2 * (kTileRows / group * group);
  return (static_cast<long long>(n_tokens) * group + static_cast<long long>(batch) * (rows - 1)) / rows;
}

template <bool BF16, bool CAP, bool BIAS>
cudaError_t launch(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, const CUtensorMap& mk, const CUtensorMap& mv,
                   const CUtensorMap& mq, long long grid, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_shared_memory(paged_prefill_kernel<BF16, CAP, BIAS>, kSmemBytes, done);
  if (e != cudaSuccess) return e;
  return launch_early(paged_prefill_kernel<BF16, CAP, BIAS>, static_cast<unsigned>(grid), kThreads, kSmemBytes, st, pv, opt, job, mk, mv, mq);
}

static_assert(2 + kSplitItems <= kWorkCounters, "counters of a call");

// partial sums that a call can use: row tiles are only cut where there are few
long long parts_of(long long items) { return items > kSplitItems ? 0 : (items * kMaxSegs < kMaxParts ? items * kMaxSegs : kMaxParts); }

}  // namespace

// Claim counter, CTAs that are through, arrivals per row tile; then the pieces' partial sums.  Enough for every call of up to
// n_tokens tokens and pv.batch sequences: a call of more row tiles than are ever cut still asks for the parts that a smaller one
// would use, so that a buffer sized for the largest call serves them all.
long long paged_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens) {
  const long long few = paged_few_workspace_bytes();
  if (static_cast<long long>(n_tokens) * group <= kFewRows && paged_few_rows(pv, group, n_tokens)) return few;    // few rows however many sequences
  const long long most = kSplitItems / pv.n_kv_heads, n_rb = row_tiles(pv.batch, group, n_tokens);
  const long long cut = kWorkCounterBytes + parts_of((n_rb < most ? n_rb : most) * pv.n_kv_heads) * kPartFloats * 4;
  return cut > few ? cut : few;
}

cudaError_t launch_paged_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                                 const AttnOptions& opt, void* workspace, cudaStream_t st) {
  const int group = q.n_heads / pv.n_kv_heads;
  if (workspace && paged_few_rows(pv, group, n_tokens)) return launch_paged_few(pv, q, cu_q, n_tokens, out, opt, workspace, st);
  const long long n_rb = row_tiles(pv.batch, group, n_tokens);
  if (pv.batch <= 0 || n_tokens <= 0 || n_rb == 0) return cudaSuccess;
  const long long items = n_rb * pv.n_kv_heads;
  if (items > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  PrefillJob job{};
  job.q = q;
  job.out = out;
  job.cu_q = cu_q;
  job.n_tokens = n_tokens;
  job.group = group;
  job.tile_rows = kTileRows / group * group;
  job.group_inv = group > 1 ? static_cast<unsigned>(((1ull << 32) + group - 1) / group) : 0u;
  long long grid = items;
  if (workspace) {
    job.counters = static_cast<unsigned*>(workspace);
    job.max_parts = static_cast<int>(parts_of(items));
    if (job.max_parts > 0) {
      job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWorkCounterBytes);
      grid = items * kMaxSegs;
    }
  }
  const int sms = sm_count_of_current_device();
  if (grid > sms) grid = sms;
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
  auto go = [&](auto bf16) {
    constexpr bool kBf16 = decltype(bf16)::value;
    if (opt.cap > 0.0f)
      return opt.slopes ? launch<kBf16, true, true>(pv, opt, job, mk, mv, mq, grid, st) : launch<kBf16, true, false>(pv, opt, job, mk, mv, mq, grid, st);
    return opt.slopes ? launch<kBf16, false, true>(pv, opt, job, mk, mv, mq, grid, st) : launch<kBf16, false, false>(pv, opt, job, mk, mv, mq, grid, st);
  };
  return pv.dtype == MOQAE_DTYPE_BF16 ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace moqae
