// What the streaming attention kernels over paged caches share (16-bit pages: paged_decode.cu, 4-bit pages: paged4_decode.cu):
// sets of rows and the tiles that they see, the cutting of all tiles into equal pieces of work, and the joining of what
// the pieces leave.  What it is for stands at the kernels.
#pragma once

#include "paged.cuh"

namespace moqae {

namespace {

constexpr int kTile = 16;                        // tokens per tile
constexpr float kLog2e = 1.4426950408889634f;

// How a launch forms its sets: one token of a group of at most 4 or 8 heads, or up to 16 rows of several tokens; over 16-bit
// or 4-bit pages.
enum { kOne4, kOne8, kFew16, kOne4Q, kOne8Q, kFew16Q };
__host__ __device__ constexpr bool several(int form) { return form == kFew16 || form == kFew16Q; }
__host__ __device__ constexpr int set_rows(int form) { return several(form) ? 16 : 8; }
// What a pair costs beside its tiles, in tiles (its queries, its result).
__host__ __device__ constexpr int pair_cost(int form) { return form < kOne4Q ? 1 : 3; }

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
  int max_rows;           // 4-bit pages: sequences of more rows are another kernel's; 0: none is
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
  template <int FORM> __device__ __forceinline__ int units() const { return n > 0 ? n + pair_cost(FORM) : 0; }
};
template <int FORM>
__device__ __forceinline__ Seen seen_of(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, int b, int set, bool report) {
  Seen s;
  const int kv_len = paged_len(pv, b, report);
  s.prefix = opt.prefix_len ? min(max(opt.prefix_len[b], 0), kv_len) : 0;
  int p_first;
  if (several(FORM)) {
    s.q_first = min(max(job.cu_q[b], 0), job.n_tokens);
    s.q_n = min(max(job.cu_q[b + 1], s.q_first), job.n_tokens) - s.q_first;
    const int rows = s.q_n * job.group;
    s.sets = (rows + 15) / 16;
    s.row0 = set * 16;
    s.rows = min(16, rows - s.row0);
    if (FORM == kFew16Q && job.max_rows > 0 && rows > job.max_rows) s.sets = s.rows = 0;
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
// is pair_cost units without a tile, then one unit per tile.
struct Cursor {
  int b, set, h, i;
  int flat;               // sets before this one, of all sequences
  Seen s;
};
// To the first tile of the next pair; its b is the batch if there is none.
template <int FORM> __device__ __forceinline__ void next_pair(Cursor& c, const PagedView& pv, const AttnOptions& opt, const DecodeJob& job) {
  c.i = 0;
  if (++c.h < pv.n_kv_heads) return;
  c.h = 0;
  do {
    ++c.flat;
    if (++c.set >= c.s.sets) {
      c.set = 0;
      do {
        if (++c.b >= pv.batch) return;
        c.s = seen_of<FORM>(pv, opt, job, c.b, 0, false);
      } while (c.s.sets == 0);
    } else {
      c.s = seen_of<FORM>(pv, opt, job, c.b, c.set, false);
    }
  } while (c.s.n == 0);
}
// To the next tile; returns the units that this passes.
template <int FORM> __device__ __forceinline__ int advance(Cursor& c, const PagedView& pv, const AttnOptions& opt, const DecodeJob& job) {
  if (++c.i < c.s.n) return 1;
  next_pair<FORM>(c, pv, opt, job);
  return 1 + pair_cost(FORM);
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

// Row of the set's tokens that row `row` of a sequence belongs to.
template <int FORM> __device__ __forceinline__ int token_in_sequence(const DecodeJob& job, int row) { return several(FORM) ? row / job.group : 0; }

// Sequence b, one head: its units and sets; rows that see nothing are zeros (once per launch: `write`).  `tokens` counts query tokens.
template <int FORM>
__device__ __forceinline__ int units_of(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, int b, int& sets, int& tokens, bool write) {
  int units = 0;
  sets = 1;
  for (int set = 0; set < sets; ++set) {
    const Seen s = seen_of<FORM>(pv, opt, job, b, set, write && set == 0 && blockIdx.x == 0);
    sets = s.sets;
    if (several(FORM) && set == 0) tokens += s.q_n;
    units += s.units<FORM>();
    if (s.n == 0 && write && b % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x))
      for (int h = 0; h < pv.n_kv_heads; ++h)
        for (int r = 0; r < s.rows; ++r) {
          const int t = token_in_sequence<FORM>(job, s.row0 + r);
          uint16_t* row = job.out.data + (s.q_first + t) * job.out.token + (h * job.group + s.row0 + r - t * job.group) * job.out.head;
          for (int c = 0; c < kHeadDim; c += 8) *reinterpret_cast<uint4*>(row + c) = make_uint4(0, 0, 0, 0);
        }
  }
  return units;
}

// A CTA's and a warp's part of the work of a launch.
struct Part {
  long long total;               // units of all heads
  long long lo;                  // the warp's first unit
  int ctas, todo;                // CTAs with work; the warp's units
  int first_units, first_sets;   // of sequence `lane`
};

// What all CTAs work out alike: the units of the call, and how they are shared out: a CTA per pair while that is no more than
// PAIR_TILES tiles each (with equal lengths no pair then spans CTAs, which saves the way through the workspace), otherwise at
// least MIN_TILES tiles per warp.  False: nothing for this CTA.
template <int FORM, int WARPS, int MIN_TILES, int PAIR_TILES>
__device__ __forceinline__ bool share_work(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, int warp, int lane, Part& part) {
  int tokens = 0;                                 // query tokens that this lane has counted
  int mine = 0, all_sets = 0;
  part.first_units = part.first_sets = 0;
  for (int b = lane; b < pv.batch && (!several(FORM) || tokens <= job.n_tokens); b += 32) {
    int sets;
    const int u = units_of<FORM>(pv, opt, job, b, sets, tokens, warp == 0);
    mine += u;
    all_sets += sets;
    if (b < 32) {
      part.first_units = u;
      part.first_sets = sets;
    }
  }
  if (several(FORM)) {                           // sequences that share rows could have more sets than there are counters
    tokens = __reduce_add_sync(0xffffffffu, tokens);
    if (tokens > job.n_tokens) {
      if (blockIdx.x == 0 && threadIdx.x == 0) paged_status(pv.status, MOQAE_ERR_INVALID_ARG, -1, tokens);
      return false;
    }
  }
  mine = __reduce_add_sync(0xffffffffu, mine);
  all_sets = __reduce_add_sync(0xffffffffu, all_sets);
  part.total = static_cast<long long>(mine) * pv.n_kv_heads;
  const long long pairs = static_cast<long long>(all_sets) * pv.n_kv_heads;
  const int most = static_cast<int>(gridDim.x);
  part.ctas = most;
  if (part.total <= static_cast<long long>(most) * WARPS * MIN_TILES) part.ctas = static_cast<int>((part.total + WARPS * MIN_TILES - 1) / (WARPS * MIN_TILES));
  if (pairs <= most && part.total <= pairs * (PAIR_TILES + pair_cost(FORM)) && part.total >= pairs) part.ctas = static_cast<int>(pairs);
  const int cta = static_cast<int>(blockIdx.x);
  if (cta >= part.ctas) return false;
  const long long cta_lo = share(part.total, cta, part.ctas), cta_hi = share(part.total, cta + 1, part.ctas);
  const int in_cta = static_cast<int>(cta_hi - cta_lo);
  part.lo = cta_lo + share(in_cta, warp, WARPS);
  part.todo = static_cast<int>(cta_lo + share(in_cta, warp + 1, WARPS) - part.lo);
  return true;
}

// The tile that opens the warp's part (todo > 0), and the unit that it is.
template <int FORM>
__device__ __forceinline__ Cursor find_first(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, int lane, Part& part, long long& at) {
  const long long lo = part.lo;
  Cursor put;
  int tokens = 0;
  int before = 0, sets_before = 0;            // of one head
  put.b = 0;
  for (int base = 0; base < pv.batch; base += 32) {
    const int b = base + lane;
    int n = part.first_units, sets = part.first_sets;
    if (base > 0) n = b < pv.batch ? units_of<FORM>(pv, opt, job, b, sets, tokens, false) : (sets = 0);
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
  at = lo;
  int off = static_cast<int>(lo - static_cast<long long>(before) * pv.n_kv_heads);
  put.set = 0;
  put.s = seen_of<FORM>(pv, opt, job, put.b, 0, false);
  while (off >= put.s.units<FORM>() * pv.n_kv_heads) {
    off -= put.s.units<FORM>() * pv.n_kv_heads;
    put.s = seen_of<FORM>(pv, opt, job, put.b, ++put.set, false);
  }
  put.flat = sets_before + put.set;
  put.h = off / put.s.units<FORM>();
  put.i = off - put.h * put.s.units<FORM>() - pair_cost(FORM);
  if (put.i < 0) {                            // the piece opens with units that hold no tile
    part.todo += put.i;
    at -= put.i;
    put.i = 0;
  }
  return put;
}

// Join the pieces of this CTA, which stand in the order of their tokens (desc[2 * warp]: the piece at the start of a warp's
// part, desc[2 * warp + 1]: at its end; piece_at(i): its sums), and with the last CTA to arrive those of a pair that spans CTAs.
template <bool BF16, int FORM, int WARPS, typename P>
__device__ __forceinline__ void join_pieces(const DecodeJob& job, const Part& part, const Piece* desc, int* turn, int piece_rows, int piece_floats,
                                            int warp, int lane, P piece_at) {
  static_assert(WARPS <= 16, "a lane looks at a piece");
  constexpr int kRows = set_rows(FORM);
  const int cta = static_cast<int>(blockIdx.x), ctas = part.ctas;
  const long long total = part.total;
  const int my_pair = lane < 2 * WARPS ? desc[lane].pair : -1;
  const unsigned valid = __ballot_sync(0xffffffffu, my_pair >= 0);
  if (valid == 0) return;
  // where row r of the pair of piece i goes
  auto row_of = [&](int i, int r) -> uint16_t* {
    const int h = desc[i].h, row = desc[i].set * kRows + r, t = token_in_sequence<FORM>(job, row);
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
  for (int j = warp; j < n_jobs; j += WARPS) {
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
  const int which = WARPS - 1 - warp, speaks_for = which == 0 ? cross0 : which == 1 ? cross1 : -1;
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
      if (n_job % WARPS != warp) continue;
      const int r = r0 + (lane >> 4);
      join_far<BF16>([&](int p) -> const float* {
        return job.part + (static_cast<long long>(from + p) * 2 + (p == 0 ? 1 : 0)) * piece_floats;
      }, to - from + 1, piece_rows, r < rows ? r : piece_rows, lane, r < rows ? row_of(piece, r) : nullptr);
    }
  }
}

// bytes of the pieces that CTAs leave in the workspace, two each
inline long long part_bytes(int rows) {
  const long long n = 2ll * sm_count_of_current_device() * piece_floats_of(rows) * 4;
  return (n + 15) / 16 * 16;
}

inline long long few_sets(int batch, int group, int n_tokens) { return (static_cast<long long>(n_tokens) * group + 15ll * batch) / 16; }

// Units of all heads are counted in 32 bits.
inline bool units_fit(const PagedView& pv, long long sets, int form) {
  return sets * pv.n_kv_heads * (static_cast<long long>(pv.max_pages) * (pv.page_size / kTile) + pair_cost(form) + 1) < (1ll << 31);
}

}  // namespace

}  // namespace moqae
