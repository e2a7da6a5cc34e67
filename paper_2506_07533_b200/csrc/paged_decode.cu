// Attention of one new token per sequence over a paged 16-bit cache (moqae_paged_decode_attn), and of a few
// (moqae_paged_prefill_attn where the sequences bring so few rows that the large tiles would be empty).
//
// Every cached row is used once per kv head, by the queries of its group, so the kernel is bound by the bytes of
// the pages; all else is arranged to keep copies in flight.
//
//   Rows.  The query rows of a (sequence, kv head) are its tokens times the query heads of the group (row r =
//   token r / group, head r % group); up to 8 of them (one token) or 16 (several) make a set.
//   Work.  The unit is a tile of 16 tokens of one (set, kv head), a "pair": 4 KiB of keys, 4 KiB of values,
//   always inside one page.  All tiles that some row sees, in the order (sequence, set, head, token), are cut into
//   equal contiguous pieces, one per CTA and, inside it, one per warp: lengths may be as uneven as they like, every
//   warp streams the same number of bytes, and only tiles at the ends of a piece belong to pairs that others
//   work on too.  Lengths are read on the device; every warp finds its own piece with a scan over the sequences.
//   Copies.  A warp owns a ring of tiles and fills it with 16-byte asynchronous copies, row by row (any strides);
//   rows that are not seen are filled with zeros instead of being read.
//   Products, on mma.sync m16n8k16: S^T = K q^T (16 tokens x 8 rows), whose accumulators, transposed by movmatrix,
//   are the B operand of O^T += V^T P^T.  A 128 x 8 output per 8 KiB leaves the tensor pipe idle either way; this
//   form needs no operand expansion and no accumulator outside registers.
//   Weights of a single token are kept as high + low 16-bit halves, so rounding them costs nothing visible: with a
//   query group of at most four the low halves ride in the unused columns 4..7, otherwise they take a second
//   product.  Those of several tokens are rounded to the cache's dtype, as in the large tiles: bf16 results 0.0022 of their norm
//   off instead of the 0.0017 of their own rounding.  (Their low halves as well: 2 to 5 % more time, 8 sequences of 1 to 8 tokens
//   24.1 instead of 23.6 us, 64 of 8000 with 4 365 instead of 353.)
//   Softmax against a reference that moves only when a weight would pass 2^kLag: one vote per
//   tile instead of a reduction over lanes.
//   Joining.  A warp that has a pair to itself writes the result.  Other pieces meet in shared memory after the
//   CTA's last tile; a pair that spans CTAs goes through the workspace, and the CTA that arrives last adds the
//   pieces in the order of their tokens (results do not depend on timing).
//   Measured.  61 sequences of 1 to 32000 tokens, 32 / 8 heads, bf16: 128 to 136 us for 798 MB (floor 122); 4 of 131000:
//   320 to 356 us (floor 328 at the rate of a copy, which writes as much as it reads).  Short calls pay about 10 us beside
//   their bytes: 2 us to find the work, 2 for the first tile, 1 to 3 to join inside a CTA, 1 for the fence and the
//   arrival, 2 to join what CTAs share (8 sequences of 1000: 16.2 us, floor 5; 128 of 300: 38, floor 24).
#include "paged.cuh"
#include "ptx.cuh"

namespace moqae {

namespace {

constexpr int kWarps = 8;
constexpr int kTile = 16;                        // tokens per tile
constexpr int kTileBytes = kTile * 256;          // of keys, and of values
constexpr int kStageBytes = 2 * kTileBytes;
constexpr int kMinTiles = 2;                     // a CTA is worth starting for this many tiles per warp
constexpr int kPairTiles = 48;                   // up to so many tiles per pair, a CTA takes whole pairs where it can
constexpr int kPairCost = 1;                     // what a pair costs beside its tiles, in tiles (its queries, its result)
// The reference lies kLead below the largest score so far and moves when a score exceeds it by kLag, in base-2 units: weights below
// 2^kLag.  In fp16, whose steps end at 2^-24, the lead keeps small weights: each is off by at most 2^-35 of the largest (without
// it 2^-25, which 131000 tokens behind one large score add up to 0.4 % of that score's weight).
template <bool BF16> constexpr float kLead = BF16 ? 0.0f : 10.0f;
template <bool BF16> constexpr float kLag = BF16 ? 8.0f : 15.0f;
constexpr float kLog2e = 1.4426950408889634f;

// How a launch forms its sets: one token of a group of at most 4 or 8 heads, or up to 16 rows of several tokens.
enum { kOne4, kOne8, kFew16 };
__host__ __device__ constexpr int set_rows(int form) { return form == kFew16 ? 16 : 8; }
// tiles in flight or in use per warp (the pieces of 16 rows take the room of the third)
__host__ __device__ constexpr int stages_of(int form) { return form == kFew16 ? 2 : 3; }

// A piece: the sums of a pair's tiles, float [rows][128], then (reference, weight sum) per row.
__host__ __device__ constexpr int piece_floats_of(int rows) { return (rows * (kHeadDim + 2) + 3) / 4 * 4; }

// total * i / n for i <= n < 256
__device__ __forceinline__ long long share(long long total, int i, int n) {
  if (total < (1ll << 23)) return static_cast<unsigned>(total) * static_cast<unsigned>(i) / static_cast<unsigned>(n);
  return total * i / n;
}

struct DecodeJob {
  RowsView q, out;
  const int32_t* cu_q;    // null: one token per sequence
  int n_tokens, group;
  float* part;            // [ctas][2] pieces
  int* arrived;           // [sets][n_kv_heads]
};

// A set of rows and the tiles that they see: tokens [lo, len) and [0, pre).
struct Seen {
  int len, lo, pre;       // pre <= lo
  int n_pre, first, n;    // tiles of the prefix, first tile behind them, number of tiles
  int sets;               // of the sequence
  int q_n;                // its query tokens
  int row0, rows;         // rows of the set
  int q_first, pos0;      // row of the queries, and position, of the sequence's first query token
  int prefix;             // what every row sees
  __device__ __forceinline__ int units() const { return n > 0 ? n + kPairCost : 0; }
};
template <int FORM>
__device__ __forceinline__ Seen seen_of(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, int b, int set, bool report) {
  Seen s;
  const int kv_len = paged_len(pv, b, report);
  s.prefix = opt.prefix_len ? min(max(opt.prefix_len[b], 0), kv_len) : 0;
  int p_first;
  if (FORM == kFew16) {
    s.q_first = min(max(job.cu_q[b], 0), job.n_tokens);
    s.q_n = min(max(job.cu_q[b + 1], s.q_first), job.n_tokens) - s.q_first;
    const int rows = s.q_n * job.group;
    s.sets = (rows + 15) / 16;
    s.row0 = set * 16;
    s.rows = min(16, rows - s.row0);
    s.pos0 = kv_len - s.q_n;
    p_first = s.pos0 + s.row0 / job.group;
    s.len = s.rows > 0 ? max(s.pos0 + (s.row0 + s.rows - 1) / job.group + 1, s.prefix) : 0;
    s.len = max(s.len, 0);
  } else {
    s.sets = s.q_n = 1;
    s.row0 = 0;
    s.rows = job.group;
    s.q_first = b;
    s.pos0 = p_first = kv_len - 1;
    s.len = kv_len;
  }
  s.lo = opt.window > 0 ? max(0, p_first + 1 - opt.window) : 0;
  s.pre = min(s.prefix, s.len);
  if (s.pre >= s.lo) s.lo = s.pre = 0;
  s.n_pre = (s.pre + kTile - 1) / kTile;
  s.first = max(s.lo / kTile, s.n_pre);
  s.n = s.n_pre + max(0, (s.len + kTile - 1) / kTile - s.first);
  return s;
}
__device__ __forceinline__ int tile_of(const Seen& s, int i) { return i < s.n_pre ? i : s.first + i - s.n_pre; }

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, bool fetch) {
  asm volatile("cp.async.cg.shared.global.L2::256B [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(fetch ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;\n" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_async_wait() { asm volatile("cp.async.wait_group %0;\n" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_trans(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];\n"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(x));
  return r;
}
template <bool BF16> __device__ __forceinline__ void mma16816(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}

// A position in the order of all tiles: tile i of set `set` of sequence b, head h.  Work is shared out in units: a pair
// is kPairCost units without a tile, then one unit per tile.
struct Cursor {
  int b, set, h, i;
  int flat;               // sets before this one, of all sequences
  Seen s;
};
// To the next tile; returns the units that this passes.
template <int FORM> __device__ __forceinline__ int advance(Cursor& c, const PagedView& pv, const AttnOptions& opt, const DecodeJob& job) {
  if (++c.i < c.s.n) return 1;
  c.i = 0;
  if (++c.h < pv.n_kv_heads) return 1 + kPairCost;
  c.h = 0;
  do {
    ++c.flat;
    if (++c.set >= c.s.sets) {
      c.set = 0;
      do {
        if (++c.b >= pv.batch) return 1 + kPairCost;
        c.s = seen_of<FORM>(pv, opt, job, c.b, 0, false);
      } while (c.s.sets == 0);
    } else {
      c.s = seen_of<FORM>(pv, opt, job, c.b, c.set, false);
    }
  } while (c.s.n == 0);
  return 1 + kPairCost;
}

// Which pair a piece in shared memory belongs to.
struct Piece {
  int pair, h;            // set * n_kv_heads + h, or -1; h
  int starts, ends;       // whether it holds the pair's first and last tile
  int set, n;             // set of the sequence, tiles of the pair
  int rows, q_first;      // rows of the set, first row of the sequence's queries
  long long unit;         // unit of the pair's first tile
};

// The end of a row's joining: the finished row (out != null), or the joined piece.
template <bool BF16>
__device__ __forceinline__ void put_row(const float (&acc)[8], float m, float l, int rows, int r, int sub, uint16_t* out, float* joined) {
  if (out) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint4*>(out + 8 * sub) =
        make_uint4(float2_to_pair<BF16>(acc[0] * inv, acc[1] * inv), float2_to_pair<BF16>(acc[2] * inv, acc[3] * inv),
                   float2_to_pair<BF16>(acc[4] * inv, acc[5] * inv), float2_to_pair<BF16>(acc[6] * inv, acc[7] * inv));
  } else {
    float4* dst = reinterpret_cast<float4*>(joined + r * kHeadDim) + 2 * sub;
    dst[0] = make_float4(acc[0], acc[1], acc[2], acc[3]);
    dst[1] = make_float4(acc[4], acc[5], acc[6], acc[7]);
    if (sub == 0) *reinterpret_cast<float2*>(joined + rows * kHeadDim + 2 * r) = make_float2(m, l);
  }
}

// Half a warp adds row r of n pieces of the workspace (piece(p): address of the p-th, in the order of their tokens), a
// lane eight channels, and writes the finished row.  r >= rows: it only keeps the other half company.  The first pieces'
// sums are on their way while the references are compared.
template <bool BF16, typename F>
__device__ __forceinline__ void join_far(F piece, int n, int rows, int r, int lane, uint16_t* out) {
  constexpr int kBatch = 4;
  const int sub = lane & 15;
  const bool act = r < rows;
  r = act ? r : rows - 1;
  const int at_ml = rows * kHeadDim + 2 * r;
  float m = -INFINITY, l = 0.0f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  float4 v[kBatch][2];
  auto load = [&](int p0) {
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const float4* src = reinterpret_cast<const float4*>(piece(min(p0 + k, n - 1)) + r * kHeadDim) + 2 * sub;
      v[k][0] = __ldcg(src);
      v[k][1] = __ldcg(src + 1);
    }
  };
  for (int base = 0; base < n; base += 16) {
    load(base);
    float2 w = make_float2(-INFINITY, 0.0f);
    if (base + sub < n) w = __ldcg(reinterpret_cast<const float2*>(piece(base + sub) + at_ml));
    float top = fmaxf(m, w.x);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float f = w.x == -INFINITY ? 0.0f : exp2_fast(w.x - top), old = m == -INFINITY ? 0.0f : exp2_fast(m - top);
    float fl = w.y * f;
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) fl += __shfl_xor_sync(0xffffffffu, fl, o);
    l = l * old + fl;
    m = top;
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[e] *= old;
    const int many = min(16, n - base);
    for (int p0 = 0; p0 < many; p0 += kBatch) {
      if (p0) load(base + p0);
#pragma unroll
      for (int k = 0; k < kBatch; ++k) {
        const float fp = __shfl_sync(0xffffffffu, f, p0 + k, 16);          // 0 behind the last piece
        const float* x = reinterpret_cast<const float*>(v[k]);
        if (p0 + k < many)
#pragma unroll
          for (int e = 0; e < 8; ++e) acc[e] = fmaf(x[e], fp, acc[e]);
      }
    }
  }
  if (act) put_row<BF16>(acc, m, l, rows, r, sub, out, nullptr);
}

// The same for pieces in shared memory (bit i of `run`: piece(i)), and where the run is not the whole pair (out == null) the
// sum goes on as a piece.  They are near enough to be read twice: a pass for the reference, one for the sums.  (The exchange between lanes above costs as much as a dozen pieces do here: jobs of two
// pieces took 2050 clocks instead of 1000.)
template <bool BF16, typename P>
__device__ __forceinline__ void join_near(P piece, unsigned run, int rows, int r, int lane, uint16_t* out, float* joined) {
  const int sub = lane & 15;
  const bool act = r < rows;
  r = act ? r : rows - 1;
  const int at_ml = rows * kHeadDim + 2 * r;
  float m = -INFINITY, l = 0.0f, acc[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  for (unsigned bits = run; bits; bits &= bits - 1) m = fmaxf(m, piece(__ffs(bits) - 1)[at_ml]);
#pragma unroll 2
  for (unsigned bits = run; bits; bits &= bits - 1) {
    const float* from = piece(__ffs(bits) - 1);
    const float2 w = *reinterpret_cast<const float2*>(from + at_ml);
    const float4* x = reinterpret_cast<const float4*>(from + r * kHeadDim) + 2 * sub;
    const float4 a = x[0], b = x[1];
    const float f = w.x == -INFINITY ? 0.0f : exp2_fast(w.x - m);
    l = fmaf(w.y, f, l);
    acc[0] = fmaf(a.x, f, acc[0]);
    acc[1] = fmaf(a.y, f, acc[1]);
    acc[2] = fmaf(a.z, f, acc[2]);
    acc[3] = fmaf(a.w, f, acc[3]);
    acc[4] = fmaf(b.x, f, acc[4]);
    acc[5] = fmaf(b.y, f, acc[5]);
    acc[6] = fmaf(b.z, f, acc[6]);
    acc[7] = fmaf(b.w, f, acc[7]);
  }
  if (act) put_row<BF16>(acc, m, l, rows, r, sub, out, joined);
}

template <bool BF16, int FORM>
__global__ void __launch_bounds__(kWarps * 32, 1) paged_decode_kernel(PagedView pv, AttnOptions opt, DecodeJob job) {
  constexpr int kRows = set_rows(FORM), kCols = kRows / 8, kStages = stages_of(FORM);
  extern __shared__ __align__(128) uint8_t smem[];
  // [warps][stages] tiles; then the piece each warp may leave behind at the start of its range (the piece
  // at its end goes into its ring, which is empty by then); then descriptors
  const int piece_rows = FORM == kFew16 ? kRows : job.group;
  const int piece_floats = piece_floats_of(piece_rows);
  float* head_piece = reinterpret_cast<float*>(smem + kWarps * kStages * kStageBytes);
  Piece* desc = reinterpret_cast<Piece*>(head_piece + kWarps * piece_floats);       // [2 * kWarps]
  int* turn = reinterpret_cast<int*>(desc + 2 * kWarps);                            // per pair that spans CTAs: arrivals before this one, first CTA, last CTA

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t4 = lane & 3;
  uint8_t* ring = smem + warp * kStages * kStageBytes;
  const uint32_t ring_u = smem_u32(ring);
  auto token_of = [&](int row) { return FORM == kFew16 ? row / job.group : 0; };

  if (threadIdx.x < 2 * kWarps) desc[threadIdx.x].pair = -1;
  after_previous();

  // ---- where the work is: units and sets of every sequence, then this warp's piece ----
  // sequence b, one head: its units; rows that see nothing are zeros (once per launch: `write`)
  int tokens = 0;                                 // query tokens that this lane has counted
  auto units_of = [&](int b, int& sets, bool write) -> int {
    int units = 0;
    sets = 1;
    for (int set = 0; set < sets; ++set) {
      const Seen s = seen_of<FORM>(pv, opt, job, b, set, write && set == 0 && blockIdx.x == 0);
      sets = s.sets;
      if (FORM == kFew16 && set == 0) tokens += s.q_n;
      units += s.units();
      if (s.n == 0 && write && b % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x))
        for (int h = 0; h < pv.n_kv_heads; ++h)
          for (int r = 0; r < s.rows; ++r) {
            const int t = token_of(s.row0 + r);
            uint16_t* row = job.out.data + (s.q_first + t) * job.out.token + (h * job.group + s.row0 + r - t * job.group) * job.out.head;
            for (int c = 0; c < kHeadDim; c += 8) *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
          }
    }
    return units;
  };
  int mine = 0, first_units = 0, first_sets = 0, all_sets = 0;
  for (int b = lane; b < pv.batch && (FORM != kFew16 || tokens <= job.n_tokens); b += 32) {
    int sets;
    const int u = units_of(b, sets, warp == 0);
    mine += u;
    all_sets += sets;
    if (b < 32) {
      first_units = u;
      first_sets = sets;
    }
  }
  if (FORM == kFew16) {                           // sequences that share rows could have more sets than there are counters
    tokens = __reduce_add_sync(0xffffffffu, tokens);
    if (tokens > job.n_tokens) {
      if (blockIdx.x == 0 && threadIdx.x == 0) paged_status(pv.status, MOQAE_ERR_INVALID_ARG, -1, tokens);
      return;
    }
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  all_sets = __reduce_add_sync(0xffffffffu, all_sets);
  const long long total = static_cast<long long>(mine) * pv.n_kv_heads;
  const long long pairs = static_cast<long long>(all_sets) * pv.n_kv_heads;
  // A CTA per pair while that is no more than kPairTiles tiles each: with equal lengths no pair then spans CTAs,
  // which saves the way through the workspace.  Otherwise every CTA gets at least kMinTiles tiles per warp.  Measured with a limit of
  // 8 / 24 / 48 / 96 tiles (us, timer steps of 2): 64 pairs of 19 tiles 16.4 / 14.3 / 14.3 / 14.3, 128 pairs of 19 18.4 / 16.4 / 16.4 / 16.4, of 44
  // 24.6 / 24.6 / 20.5 / 20.5, of 63 28.7 / 28.7 / 28.7 / 24.6; 2 or 8 pairs of 44 14.3 / 14.3 / 16.4 / 16.4, of 63 14.3 / 14.3 / 14.3 / 20.5.
  const int most = static_cast<int>(gridDim.x);
  int ctas = most;
  if (total <= static_cast<long long>(most) * kWarps * kMinTiles) ctas = static_cast<int>((total + kWarps * kMinTiles - 1) / (kWarps * kMinTiles));
  if (pairs <= most && total <= pairs * (kPairTiles + kPairCost) && total >= pairs) ctas = static_cast<int>(pairs);
  const int cta = static_cast<int>(blockIdx.x);
  if (cta >= ctas) return;
  const long long cta_lo = share(total, cta, ctas), cta_hi = share(total, cta + 1, ctas);
  const int in_cta = static_cast<int>(cta_hi - cta_lo);
  const long long lo = cta_lo + share(in_cta, warp, kWarps);
  int todo = static_cast<int>(cta_lo + share(in_cta, warp + 1, kWarps) - lo);

  __syncthreads();

  if (todo > 0) {
    // ---- the pair that holds unit `lo` ----
    Cursor put;                                   // next tile to copy
    long long at = lo;                            // unit of the tile that is worked on
    {
      int before = 0, sets_before = 0;            // of one head
      put.b = 0;
      for (int base = 0; base < pv.batch; base += 32) {
        const int b = base + lane;
        int n = first_units, sets = first_sets;
        if (base > 0) n = b < pv.batch ? units_of(b, sets, false) : (sets = 0);
        int inc = n, sinc = sets;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, inc, o), y = __shfl_up_sync(0xffffffffu, sinc, o);
          if (lane >= o) {
            inc += x;
            sinc += y;
          }
        }
        const unsigned hit = __ballot_sync(0xffffffffu, static_cast<long long>(before + inc) * pv.n_kv_heads > lo);
        if (hit) {
          const int l = __ffs(hit) - 1;
          put.b = base + l;
          before += __shfl_sync(0xffffffffu, inc - n, l);
          sets_before += __shfl_sync(0xffffffffu, sinc - sets, l);
          break;
        }
        before += __shfl_sync(0xffffffffu, inc, 31);
        sets_before += __shfl_sync(0xffffffffu, sinc, 31);
      }
      int off = static_cast<int>(lo - static_cast<long long>(before) * pv.n_kv_heads);
      put.set = 0;
      put.s = seen_of<FORM>(pv, opt, job, put.b, 0, false);
      while (off >= put.s.units() * pv.n_kv_heads) {
        off -= put.s.units() * pv.n_kv_heads;
        put.s = seen_of<FORM>(pv, opt, job, put.b, ++put.set, false);
      }
      put.flat = sets_before + put.set;
      put.h = off / put.s.units();
      put.i = off - put.h * put.s.units() - kPairCost;
      if (put.i < 0) {                            // the piece opens with units that hold no tile
        todo += put.i;
        at -= put.i;
        put.i = 0;
      }
    }
    Cursor get = put;                             // next tile to work on
    int to_put = todo;
    auto page_of = [&](const Cursor& c) -> int {
      if (c.b >= pv.batch) return -1;
      return pv.table[static_cast<long long>(c.b) * pv.max_pages + ((tile_of(c.s, c.i) * kTile) >> pv.page_shift)];
    };
    int page = page_of(put);
    // The queries of a pair are loaded while the pair before it is worked on (the next head, or the next sequence);
    // with several tokens the registers for that are not there.
    constexpr bool kAhead = FORM != kFew16;
    uint32_t qf[kCols][16], qn[kAhead ? 16 : 1];
    int qn_b = put.b, qn_h = put.h;
    auto load_ahead = [&]() {
      if constexpr (kAhead) {
        const int gq = FORM == kOne4 ? (g & 3) : g;
        const bool real = gq < job.group && qn_b < pv.batch;
        const uint16_t* src = job.q.data + (real ? qn_b * job.q.token + (qn_h * job.group + gq) * job.q.head : 0) + 2 * t4;
#pragma unroll
        for (int i = 0; i < 16; ++i) qn[i] = real ? *reinterpret_cast<const uint32_t*>(src + 8 * i) : 0u;
      }
    };
    load_ahead();
    auto load_rows = [&](const Cursor& c) {
      if constexpr (!kAhead) {
#pragma unroll
        for (int k = 0; k < kCols; ++k) {
          const int r = 8 * k + g, t = token_of(c.s.row0 + r);
          const bool real = r < c.s.rows;
          const uint16_t* src = job.q.data + 2 * t4;
          if (real) src += (c.s.q_first + t) * job.q.token + (c.h * job.group + c.s.row0 + r - t * job.group) * job.q.head;
#pragma unroll
          for (int i = 0; i < 16; ++i) qf[k][i] = real ? *reinterpret_cast<const uint32_t*>(src + 8 * i) : 0u;
        }
      }
    };
    load_rows(put);
    bool first_pair = true;
    const int unit = lane & 15, row0 = lane >> 4;
    // asynchronous copy of the next tile into stage st: rows of 16 units, unit u of row r at u ^ (r & 7)
    auto copy_tile = [&](int st) {
      const int t0 = tile_of(put.s, put.i) * kTile;
      const bool good = page >= 0 && page < pv.n_pages;
      if (!good && lane == 0) paged_status(pv.status, MOQAE_ERR_CORRUPT_TABLE, put.b, t0 >> pv.page_shift);
      const int slot = (t0 & (pv.page_size - 1)) + row0;
      const uint16_t* kp = pv.k + (good ? page : 0) * pv.k_page + put.h * pv.k_head + slot * pv.k_slot + unit * 8;
      const uint16_t* vp = pv.v + (good ? page : 0) * pv.v_page + put.h * pv.v_head + slot * pv.v_slot + unit * 8;
      const uint32_t dst = ring_u + st * kStageBytes + row0 * 256;
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        const int row = row0 + 2 * r, j = t0 + row;
        const bool see = good && j < put.s.len && (j >= put.s.lo || j < put.s.pre);
        const uint32_t d = dst + r * 512 + (((unit & 8) | ((unit ^ row) & 7)) << 4);
        cp_async16(d, kp + 2 * r * pv.k_slot, see);
        cp_async16(d + kTileBytes, vp + 2 * r * pv.v_slot, see);
      }
      to_put -= advance<FORM>(put, pv, opt, job);
      page = to_put > 0 ? page_of(put) : -1;
    };
#pragma unroll
    for (int st = 0; st < kStages - 1; ++st) {
      if (to_put > 0) copy_tile(st);
      cp_async_commit();
    }

    const float scale = opt.scale;
    const bool shaped = opt.cap > 0.0f;
    const float by_cap = shaped ? 1.0f / opt.cap : 0.0f;
    float slope[kCols][2], m[kCols][2], l[kCols][2], o[kCols][8][4];
    int pos[kCols][2];                            // positions of this lane's columns 8 c + 2 t4, + 1
    bool from_start = false;
    bool fresh = true;                            // the next tile opens a pair
    int stage = 0;
    while (todo > 0) {
      if (to_put > 0) copy_tile((stage + kStages - 1) % kStages);
      cp_async_commit();
      if (fresh) {
        fresh = false;
        from_start = get.i == 0;
        if constexpr (kAhead) {
          if (qn_b != get.b || qn_h != get.h) {   // sequences without tokens lie between
            qn_b = get.b;
            qn_h = get.h;
            load_ahead();
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) qf[0][i] = qn[i];
          if (++qn_h == pv.n_kv_heads) {
            qn_h = 0;
            ++qn_b;
          }
          if (todo > get.s.n - get.i + kPairCost) load_ahead();   // otherwise this is the warp's last pair
        } else if (!first_pair) {
          load_rows(get);
        }
        first_pair = false;
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            int r = 8 * c + 2 * t4 + e;           // row of the column
            if (FORM == kOne4) r &= 3;
            const int rr = min(r, get.s.rows - 1), t = token_of(get.s.row0 + rr);
            pos[c][e] = get.s.pos0 + t;
            slope[c][e] = opt.slopes && r < get.s.rows ? opt.slopes[get.h * job.group + get.s.row0 + rr - t * job.group] * kLog2e : 0.0f;
            m[c][e] = -INFINITY;
            l[c][e] = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) o[c][i][e] = o[c][i][2 + e] = 0.0f;
          }
      }
      cp_async_wait<kStages - 1>();
      __syncwarp();
      const uint32_t kt = ring_u + stage * kStageBytes, vt = kt + kTileBytes;

      // S^T = K q^T: lanes 0..15 give the rows of the first unit of a step, 16..31 those of the second
      float s[kCols][2][4];
#pragma unroll
      for (int c = 0; c < kCols; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[c][0][e] = s[c][1][e] = 0.0f;
      const int lr = lane & 15, lu = lane >> 4;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        uint32_t a[4];
        const int u = 2 * ks + lu;
        ldsm4(a, kt + lr * 256 + (((u & 8) | ((u ^ lr) & 7)) << 4));
#pragma unroll
        for (int c = 0; c < kCols; ++c) mma16816<BF16>(s[c][ks & 1], a, qf[c][2 * ks], qf[c][2 * ks + 1]);
      }
      const int t0 = tile_of(get.s, get.i) * kTile;
      float x[kCols][4];
      bool above = false;
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = t0 + g + 8 * (e >> 1);
          float y = (s[c][0][e] + s[c][1][e]) * scale;
          if (shaped) y = opt.cap * tanh_of(y * by_cap);
          const int p = pos[c][e & 1];
          y *= kLog2e;
          if (opt.slopes) y = fmaf(-slope[c][e & 1], fabsf(static_cast<float>(p - j)), y);
          const bool see = FORM == kFew16 ? (j <= p && (opt.window == 0 || j > p - opt.window)) || j < get.s.prefix
                                          : j < get.s.len && (j >= get.s.lo || j < get.s.pre);
          x[c][e] = see ? y : -INFINITY;
        }
        above = above || fmaxf(x[c][0], x[c][2]) > m[c][0] + kLag<BF16> || fmaxf(x[c][1], x[c][3]) > m[c][1] + kLag<BF16>;
      }
      if (__any_sync(0xffffffffu, above)) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float t = fmaxf(x[c][e], x[c][2 + e]);
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            t = fmaxf(t - kLead<BF16>, m[c][e]);
            const float f = t == -INFINITY ? 0.0f : exp2_fast(m[c][e] - t);
            m[c][e] = t;
            l[c][e] *= f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
              o[c][i][e] *= f;
              o[c][i][2 + e] *= f;
            }
          }
      }
      uint32_t b0[kCols], b1[kCols], c0 = 0, c1 = 0;
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
        float p[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) p[e] = x[c][e] == -INFINITY ? 0.0f : exp2_fast(x[c][e] - m[c][e & 1]);
        uint32_t h0 = float2_to_pair<BF16>(p[0], p[1]), h1 = float2_to_pair<BF16>(p[2], p[3]);
        const float2 f0 = pair_to_float2<BF16>(h0), f1 = pair_to_float2<BF16>(h1);
        // the sum of what is multiplied: without the low halves, the rounded weights
        l[c][0] += FORM == kFew16 ? f0.x + f1.x : p[0] + p[2];
        l[c][1] += FORM == kFew16 ? f0.y + f1.y : p[1] + p[3];
        if (FORM != kFew16) {
          const uint32_t r0 = float2_to_pair<BF16>(p[0] - f0.x, p[1] - f0.y), r1 = float2_to_pair<BF16>(p[2] - f1.x, p[3] - f1.y);
          if (FORM == kOne4 && t4 >= 2) {         // columns 4..7 carry the low halves of queries 0..3
            h0 = r0;
            h1 = r1;
          }
          if (FORM == kOne8) {
            c0 = transpose8(r0);
            c1 = transpose8(r1);
          }
        }
        b0[c] = transpose8(h0);
        b1[c] = transpose8(h1);
      }
      // O^T += V^T P^T: lanes 0..7 tokens 0..7 of a unit, 8..15 the next unit, 16..31 tokens 8..15
      const int vr = (lane & 7) + ((lane >> 4) << 3), vu = (lane >> 3) & 1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t a[4];
        const int u = 2 * i + vu;
        ldsm4_trans(a, vt + vr * 256 + (((u & 8) | ((u ^ vr) & 7)) << 4));
#pragma unroll
        for (int c = 0; c < kCols; ++c) mma16816<BF16>(o[c][i], a, b0[c], b1[c]);
        if (FORM == kOne8) mma16816<BF16>(o[0][i], a, c0, c1);
      }
      __syncwarp();                               // the stage may be filled again
      stage = stage + 1 == kStages ? 0 : stage + 1;

      const bool last_of_pair = get.i + 1 == get.s.n, last_of_all = todo <= (last_of_pair ? 1 + kPairCost : 1);
      if (last_of_pair || last_of_all) {
#pragma unroll
        for (int c = 0; c < kCols; ++c)
#pragma unroll
          for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) l[c][e] += __shfl_xor_sync(0xffffffffu, l[c][e], d);
        if (FORM == kOne4)
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[0][i][e] += __shfl_xor_sync(0xffffffffu, o[0][i][e], 2);
        if (from_start && last_of_pair) {
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            const float inv0 = l[c][0] == 0.0f ? 0.0f : 1.0f / l[c][0], inv1 = l[c][1] == 0.0f ? 0.0f : 1.0f / l[c][1];
            const int r = 8 * c + g, t = token_of(get.s.row0 + r);
            uint16_t* row = job.out.data + (get.s.q_first + t) * job.out.token + (get.h * job.group + get.s.row0 + r - t * job.group) * job.out.head;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                const uint32_t w = transpose8(float2_to_pair<BF16>(o[c][i][2 * e] * inv0, o[c][i][2 * e + 1] * inv1));
                if (r < get.s.rows)               // lane (g, t4): row 8 c + g, channels 16 i + 8 e + 2 t4
                  *reinterpret_cast<uint32_t*>(row + 16 * i + 8 * e + 2 * t4) = w;
              }
          }
        } else {
          const int which = from_start ? 1 : 0;
          float* dst = which ? reinterpret_cast<float*>(ring) : head_piece + warp * piece_floats;
          if (which) {                            // the ring holds no tile that is still needed: this was the warp's last
            cp_async_wait<0>();
            __syncwarp();
          }
#pragma unroll
          for (int c = 0; c < kCols; ++c)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const int r = 8 * c + 2 * t4 + e;
              if (r < piece_rows) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                  dst[r * kHeadDim + 16 * i + g] = o[c][i][e];
                  dst[r * kHeadDim + 16 * i + 8 + g] = o[c][i][2 + e];
                }
                if (g == 0) *reinterpret_cast<float2*>(dst + piece_rows * kHeadDim + 2 * r) = make_float2(m[c][e], l[c][e]);
              }
            }
          if (lane == 0) {
            Piece& d = desc[2 * warp + which];
            d.pair = get.flat * pv.n_kv_heads + get.h;
            d.h = get.h;
            d.starts = from_start;
            d.ends = last_of_pair;
            d.set = get.set;
            d.n = get.s.n;
            d.rows = get.s.rows;
            d.q_first = get.s.q_first;
            d.unit = at - get.i;
          }
        }
        fresh = true;
      }
      const int passed = advance<FORM>(get, pv, opt, job);
      todo -= passed;
      at += passed;
    }
    cp_async_wait<0>();
  }
  __syncthreads();

  // ---- join the pieces of this CTA; they stand in the order of their tokens ----
  auto piece_at = [&](int i) -> const float* {
    return (i & 1) ? reinterpret_cast<const float*>(smem + (i >> 1) * kStages * kStageBytes) : head_piece + (i >> 1) * piece_floats;
  };
  const int my_pair = lane < 2 * kWarps ? desc[lane].pair : -1;
  const unsigned valid = __ballot_sync(0xffffffffu, my_pair >= 0);
  if (valid == 0) return;
  // where row r of the pair of piece i goes
  auto row_of = [&](int i, int r) -> uint16_t* {
    const int h = desc[i].h, row = desc[i].set * kRows + r, t = token_of(row);
    return job.out.data + (desc[i].q_first + t) * job.out.token + static_cast<long long>(h * job.group + row - t * job.group) * job.out.head;
  };
  // Runs of pieces of one pair; a warp takes jobs of two rows of a run.  A run that is not the whole pair goes to the
  // workspace: slot 1 if it holds the pair's first tile (at most one run, the last), slot 0 otherwise (the first).
  // Lane i looks at piece i, so that a warp finds its jobs without walking over all runs.
  const unsigned run = __match_any_sync(0xffffffffu, my_pair);
  const bool opens = my_pair >= 0 && (run & ((1u << lane) - 1u)) == 0;          // the first piece of its run
  const bool starts = opens && desc[lane].starts, whole = starts && desc[31 - __clz(run)].ends;
  const int cross0 = __ffs(__ballot_sync(0xffffffffu, opens && !whole && !starts)) - 1;    // first pieces of the runs that span CTAs
  const int cross1 = __ffs(__ballot_sync(0xffffffffu, opens && !whole && starts)) - 1;
  const int jobs = opens ? (desc[lane].rows + 1) / 2 : 0;
  int jobs_to = jobs;                             // of pieces 0 .. lane
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, jobs_to, o);
    if (lane >= o) jobs_to += x;
  }
  const int n_jobs = __shfl_sync(0xffffffffu, jobs_to, 31);
  for (int j = warp; j < n_jobs; j += kWarps) {
    const int first = __ffs(__ballot_sync(0xffffffffu, jobs_to > j)) - 1;
    const int r = 2 * (j - __shfl_sync(0xffffffffu, jobs_to - jobs, first)) + (lane >> 4), rows = desc[first].rows;
    const bool to_out = __shfl_sync(0xffffffffu, whole ? 1 : 0, first) != 0;
    float* joined = job.part + (static_cast<long long>(cta) * 2 + (desc[first].starts ? 1 : 0)) * piece_floats;
    // (row `rows` of an odd count reads the last one and is not written)
    join_near<BF16>(piece_at, __shfl_sync(0xffffffffu, run, first), piece_rows, r < rows ? r : piece_rows, lane,
                    to_out && r < rows ? row_of(first, r) : nullptr, joined);
  }
  if (cross0 < 0 && cross1 < 0) return;

  // ---- pairs that span CTAs: the CTA that arrives last adds the pieces ----
  auto cta_of = [&](long long unit) -> int {      // largest c with share(total, c, ctas) <= unit
    int c = min(static_cast<int>(static_cast<float>(unit) * static_cast<float>(ctas) / static_cast<float>(total)), ctas - 1);
    while (c > 0 && share(total, c, ctas) > unit) --c;
    while (c + 1 < ctas && share(total, c + 1, ctas) <= unit) ++c;
    return c;
  };
  // (the last two warps speak for the two pairs: they have the fewest rows to join, if any)
  const int which = kWarps - 1 - warp, speaks_for = which == 0 ? cross0 : which == 1 ? cross1 : -1;
  int c0 = 0, c1 = 0;
  if (speaks_for >= 0) {                          // both ends at once, on two lanes
    c0 = cta_of(desc[speaks_for].unit + (lane == 1 ? desc[speaks_for].n - 1 : 0));
    c1 = __shfl_sync(0xffffffffu, c0, 1);
  }
  __threadfence();
  __syncthreads();
  if (speaks_for >= 0 && lane == 0) {
    turn[which] = static_cast<int>(atomicInc(reinterpret_cast<unsigned*>(job.arrived) + desc[speaks_for].pair, static_cast<unsigned>(c1 - c0)));
    turn[2 + which] = c0;
    turn[4 + which] = c1;
  }
  __syncthreads();
  int n_job = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int piece = k ? cross1 : cross0;
    if (piece < 0) continue;
    const int from = turn[2 + k], to = turn[4 + k];
    if (turn[k] != to - from) continue;
    __threadfence();
    const int rows = desc[piece].rows;
    for (int r0 = 0; r0 < rows; r0 += 2, ++n_job) {
      if (n_job % kWarps != warp) continue;
      const int r = r0 + (lane >> 4);
      join_far<BF16>([&](int p) -> const float* {
        return job.part + (static_cast<long long>(from + p) * 2 + (p == 0 ? 1 : 0)) * piece_floats;
      }, to - from + 1, piece_rows, r < rows ? r : piece_rows, lane, r < rows ? row_of(piece, r) : nullptr);
    }
  }
}

size_t decode_smem(int form, int rows) {
  return kWarps * stages_of(form) * kStageBytes + static_cast<size_t>(kWarps) * piece_floats_of(rows) * 4 + 2 * kWarps * sizeof(Piece) + 32;
}

template <bool BF16, int FORM> cudaError_t launch(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, cudaStream_t st) {
  const int rows = FORM == kFew16 ? 16 : job.group;
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_shared_memory(paged_decode_kernel<BF16, FORM>, decode_smem(FORM, FORM == kOne4 ? 4 : set_rows(FORM)), done);
  if (e != cudaSuccess) return e;
  return launch_early(paged_decode_kernel<BF16, FORM>, sm_count_of_current_device(), kWarps * 32, decode_smem(FORM, rows), st, pv, opt, job);
}

long long part_bytes(int rows) {
  const long long n = 2ll * sm_count_of_current_device() * piece_floats_of(rows) * 4;
  return (n + 15) / 16 * 16;
}

long long few_sets(int batch, int group, int n_tokens) { return (static_cast<long long>(n_tokens) * group + 15ll * batch) / 16; }

// Units of all heads are counted in 32 bits.
bool units_fit(const PagedView& pv, long long sets) {
  return sets * pv.n_kv_heads * (static_cast<long long>(pv.max_pages) * (pv.page_size / kTile) + kPairCost + 1) < (1ll << 31);
}

cudaError_t launch_form(PagedView pv, const AttnOptions& opt, const DecodeJob& job, cudaStream_t st) {
  if (pv.n_pages == 0) {                          // copies of no bytes still name an address
    pv.k = pv.v = job.q.data;
    pv.k_page = pv.k_head = pv.k_slot = pv.v_page = pv.v_head = pv.v_slot = 0;
  }
  const bool bf16 = pv.dtype == MOQAE_DTYPE_BF16;
  if (job.cu_q) return bf16 ? launch<true, kFew16>(pv, opt, job, st) : launch<false, kFew16>(pv, opt, job, st);
  if (job.group <= 4) return bf16 ? launch<true, kOne4>(pv, opt, job, st) : launch<false, kOne4>(pv, opt, job, st);
  return bf16 ? launch<true, kOne8>(pv, opt, job, st) : launch<false, kOne8>(pv, opt, job, st);
}

}  // namespace

bool paged_decode_fits(const PagedView& pv) {
  return static_cast<long long>(pv.batch) * pv.n_kv_heads <= kWorkCounters && units_fit(pv, pv.batch);
}

// one arrival counter per pair, then partial results of the CTAs' first and last pairs
long long paged_decode_workspace_bytes(int group) { return kWorkCounterBytes + part_bytes(group); }

cudaError_t launch_paged_decode(const PagedView& pv, const RowsView& q, const RowsView& out, const AttnOptions& opt, void* workspace,
                                cudaStream_t st) {
  if (pv.batch <= 0) return cudaSuccess;
  DecodeJob job{};
  job.q = q;
  job.out = out;
  job.group = q.n_heads / pv.n_kv_heads;
  job.arrived = static_cast<int*>(workspace);
  job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWorkCounterBytes);
  return launch_form(pv, opt, job, st);
}

// Several tokens per sequence by the same kernel: up to kFewRows rows per sequence and head on average, one set of rows.
// Measured against the large tiles (us, few / large; 32 / 8 heads, bf16, workspace).  Even batches: 8 sequences of 500 tokens with 4
// new ones each 20.5 / 22.6, of 8000 71.7 / 81.9; 64 of 500 with 1 to 4 45 to 49 / 57 to 59, of 8000 350 / 480; 40 / 40 heads, 16 of 2000
// with 16 139 / 174.  With 32 rows per sequence the large tiles win (8 of 8000: 93.3 / 74.4).
// Only the mean is known here (the lengths are on the device), and every set of a long sequence streams that sequence's tokens again.
// One sequence of 190 new tokens beside 63 single ones: all over 32000 tokens 2207 / 1890, over 8000 596 / 487, single ones of 300
// to 32000 and 8000 934 / 1028; the worst found is 190 over 32000 beside 63 of 300, 993 / 512.  A bound on how uneven a batch
// may be would send the even batches of the same size to the slower side, so there is none.
bool paged_few_rows(const PagedView& pv, int group, int n_tokens) {
  const long long sets = few_sets(pv.batch, group, n_tokens);
  return static_cast<long long>(n_tokens) * group <= static_cast<long long>(kFewRows) * pv.batch && sets * pv.n_kv_heads <= kWorkCounters &&
         units_fit(pv, sets);
}

long long paged_few_workspace_bytes() { return kWorkCounterBytes + part_bytes(16); }

cudaError_t launch_paged_few(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                             const AttnOptions& opt, void* workspace, cudaStream_t st) {
  if (pv.batch <= 0 || n_tokens <= 0) return cudaSuccess;
  DecodeJob job{};
  job.q = q;
  job.out = out;
  job.cu_q = cu_q;
  job.n_tokens = n_tokens;
  job.group = q.n_heads / pv.n_kv_heads;
  job.arrived = static_cast<int*>(workspace);
  job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWorkCounterBytes);
  return launch_form(pv, opt, job, st);
}

}  // namespace moqae
