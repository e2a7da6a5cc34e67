// Attention of one new token per sequence over a paged 16-bit cache (moqae_paged_decode_attn).
//
// Every cached row is used once per kv head, by the n_q_heads / n_kv_heads <= 8 queries of its group,
// so the kernel is bound by the bytes of the pages; all else is arranged to keep copies in flight.
//
//   Work.  The unit is a tile of 16 tokens of one (sequence, kv head): 4 KiB of keys, 4 KiB of
//   values, always inside one page.  All tiles that some query sees, in the order (sequence, head, token),
//   are cut into equal contiguous pieces, one per CTA and, inside it, one per warp: lengths may be as
//   uneven as they like, every warp streams the same number of bytes, and only tiles at the ends of a
//   piece belong to pairs that others work on too.  kv_len is read on the device; every warp finds its
//   own piece with a scan over the sequences.
//   Copies.  A warp owns a ring of kStages tiles and fills it with 16-byte asynchronous copies, row by
//   row (any strides); rows that are not seen are filled with zeros instead of being read.
//   Products, on mma.sync m16n8k16: S^T = K q^T (16 tokens x 8 queries), whose accumulators, transposed
//   by movmatrix, are the B operand of O^T += V^T P^T.  A 128 x 8 output per 8 KiB leaves the tensor
//   pipe idle either way; this form needs no operand expansion and no accumulator outside registers.
//   Weights are kept as high + low 16-bit halves, so rounding them costs nothing visible: with a query group
//   of at most four the low halves ride in the unused columns 4..7, otherwise they take a second product.
//   Softmax against a reference that moves only when a score exceeds it by 2^kLag (base-2 units): one
//   vote per tile instead of a reduction over lanes.
//   Joining.  A warp that has a pair to itself writes the result.  Other pieces meet in shared memory
//   after the CTA's last tile; a pair that spans CTAs goes through the workspace, and the CTA that
//   arrives last adds the pieces in the order of their tokens (results do not depend on timing).
#include "paged.cuh"
#include "ptx.cuh"

namespace moqae {

namespace {

constexpr int kWarps = 8;
constexpr int kStages = 3;                       // tiles in flight or in use per warp
constexpr int kTile = 16;                        // tokens per tile
constexpr int kTileBytes = kTile * 256;          // of keys, and of values
constexpr int kStageBytes = 2 * kTileBytes;
constexpr int kMinTiles = 2;                     // a CTA is worth starting for this many tiles per warp
constexpr int kPairTiles = 48;                   // up to so many tiles per pair, a CTA takes whole pairs where it can
constexpr int kPairCost = 1;                     // what a pair costs beside its tiles, in tiles (its queries, its result)
constexpr float kLag = 8.0f;
constexpr float kLog2e = 1.4426950408889634f;

// A piece: the sums of a pair's tiles, float [group][128], then (reference, weight sum) per query.
__host__ __device__ constexpr int piece_floats_of(int group) { return (group * (kHeadDim + 2) + 3) / 4 * 4; }

// total * i / n for i <= n < 256
__device__ __forceinline__ long long share(long long total, int i, int n) {
  if (total < (1ll << 23)) return static_cast<unsigned>(total) * static_cast<unsigned>(i) / static_cast<unsigned>(n);
  return total * i / n;
}

// Tiles of one sequence that its query sees: tokens [lo, len) and [0, pre).
struct Seen {
  int len, lo, pre;       // pre <= lo
  int n_pre, first, n;    // tiles of the prefix, first tile behind them, number of tiles
  __device__ __forceinline__ int units() const { return n > 0 ? n + kPairCost : 0; }
};
__device__ __forceinline__ Seen seen_of(const PagedView& pv, const AttnOptions& opt, int b, bool report) {
  Seen s;
  s.len = paged_len(pv, b, report);
  s.lo = opt.window > 0 ? max(0, s.len - opt.window) : 0;
  s.pre = opt.prefix_len ? min(max(opt.prefix_len[b], 0), s.len) : 0;
  if (s.pre >= s.lo) s.lo = s.pre = 0;
  s.n_pre = (s.pre + kTile - 1) / kTile;
  s.first = max(s.lo / kTile, s.n_pre);
  s.n = s.n_pre + (s.len + kTile - 1) / kTile - s.first;
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

// A position in the order of all tiles: tile `i` of sequence b, head h.  Work is shared out in units: a pair is
// kPairCost units without a tile, then one unit per tile.
struct Cursor {
  int b, h, i;
  Seen s;
};
// To the next tile; returns the units that this passes.
__device__ __forceinline__ int advance(Cursor& c, const PagedView& pv, const AttnOptions& opt) {
  if (++c.i < c.s.n) return 1;
  c.i = 0;
  if (++c.h < pv.n_kv_heads) return 1 + kPairCost;
  c.h = 0;
  do {
    if (++c.b >= pv.batch) break;
    c.s = seen_of(pv, opt, c.b, false);
  } while (c.s.n == 0);
  return 1 + kPairCost;
}

// Which pair a piece in shared memory belongs to.
struct Piece {
  int pair;               // b * n_kv_heads + h, or -1
  int starts, ends;       // whether it holds the pair's first and last tile
};

struct Workspace {
  float* part;            // [ctas][2] pieces
  int* arrived;           // [batch * n_kv_heads]
};

// One warp adds query g of n pieces (piece(p): address of the p-th, in the order of their tokens), a lane four
// channels, and writes the finished row (out != null) or the joined piece.
template <bool BF16, bool REMOTE, typename F>
__device__ __forceinline__ void join_query(F piece, int n, int group, int g, int lane, uint16_t* out, float* joined) {
  const int at_ml = group * kHeadDim + 2 * g;
  float m = -INFINITY, l = 0.0f, acc[4] = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = lane; p < n; p += 32) m = fmaxf(m, REMOTE ? __ldcg(piece(p) + at_ml) : piece(p)[at_ml]);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  for (int base = 0; base < n; base += 32) {
    float f = 0.0f, fl = 0.0f;                    // lane p: factor of piece base + p, and its share of the weight sum
    if (base + lane < n) {
      const float2* ml = reinterpret_cast<const float2*>(piece(base + lane) + at_ml);
      const float2 w = REMOTE ? __ldcg(ml) : *ml;
      f = w.x == -INFINITY ? 0.0f : exp2_fast(w.x - m);
      fl = w.y * f;
    }
    const int many = min(32, n - base);
#pragma unroll 8
    for (int p = 0; p < many; ++p) {
      const float4* src = reinterpret_cast<const float4*>(piece(base + p) + g * kHeadDim) + lane;
      const float4 v = REMOTE ? __ldcg(src) : *src;
      const float fp = __shfl_sync(0xffffffffu, f, p);
      l += __shfl_sync(0xffffffffu, fl, p);
      acc[0] = fmaf(v.x, fp, acc[0]);
      acc[1] = fmaf(v.y, fp, acc[1]);
      acc[2] = fmaf(v.z, fp, acc[2]);
      acc[3] = fmaf(v.w, fp, acc[3]);
    }
  }
  if (out) {
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    *reinterpret_cast<uint2*>(out + 4 * lane) =
        make_uint2(float2_to_pair<BF16>(acc[0] * inv, acc[1] * inv), float2_to_pair<BF16>(acc[2] * inv, acc[3] * inv));
  } else {
    *(reinterpret_cast<float4*>(joined + g * kHeadDim) + lane) = make_float4(acc[0], acc[1], acc[2], acc[3]);
    if (lane == 0) *reinterpret_cast<float2*>(joined + at_ml) = make_float2(m, l);
  }
}

template <bool BF16, bool SMALL>
__global__ void __launch_bounds__(kWarps * 32, 1)
paged_decode_kernel(PagedView pv, RowsView q, RowsView out, AttnOptions opt, int group, Workspace ws) {
  extern __shared__ __align__(128) uint8_t smem[];
  // [warps][stages] tiles; then the piece each warp may leave behind at the start of its range (the piece
  // at its end goes into its ring, which is empty by then); then descriptors
  const int piece_floats = piece_floats_of(group);
  float* head_piece = reinterpret_cast<float*>(smem + kWarps * kStages * kStageBytes);
  Piece* desc = reinterpret_cast<Piece*>(head_piece + kWarps * piece_floats);       // [2 * kWarps]
  int* turn = reinterpret_cast<int*>(desc + 2 * kWarps);                            // per pair that spans CTAs: arrivals before this one, first CTA, last CTA

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t4 = lane & 3;
  uint8_t* ring = smem + warp * kStages * kStageBytes;
  const uint32_t ring_u = smem_u32(ring);

  // ---- where the work is: total number of tiles, then this warp's piece ----
  int mine = 0, first_n = 0;                      // first_n: units of a head of sequence `lane`
  for (int b = lane; b < pv.batch; b += 32) {
    const Seen s = seen_of(pv, opt, b, blockIdx.x == 0 && warp == 0);
    mine += s.units();
    if (b < 32) first_n = s.units();
    // a sequence without tokens has no tile: its rows are zeros
    if (s.n == 0 && b % static_cast<int>(gridDim.x) == static_cast<int>(blockIdx.x) && warp == 0)
      for (int h = 0; h < q.n_heads; ++h)
        for (int c = 0; c < kHeadDim; c += 8)
          *reinterpret_cast<uint4*>(out.data + b * out.token + h * out.head + c) = make_uint4(0, 0, 0, 0);
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) mine += __shfl_xor_sync(0xffffffffu, mine, o);
  const long long total = static_cast<long long>(mine) * pv.n_kv_heads;
  const int pairs = pv.batch * pv.n_kv_heads;
  // A CTA per pair while that is no more than kPairTiles tiles each: with equal lengths no pair then spans CTAs,
  // which saves the way through the workspace (333 tokens x 8 heads: 8.1 instead of 10.5 us).  Otherwise every
  // CTA gets at least kMinTiles tiles per warp.
  const int most = static_cast<int>(gridDim.x);
  int ctas = most;
  if (total <= static_cast<long long>(most) * kWarps * kMinTiles) ctas = static_cast<int>((total + kWarps * kMinTiles - 1) / (kWarps * kMinTiles));
  if (pairs <= most && total <= static_cast<long long>(pairs) * (kPairTiles + kPairCost) && total >= pairs) ctas = pairs;
  const int cta = static_cast<int>(blockIdx.x);
  if (cta >= ctas) return;
  const long long cta_lo = share(total, cta, ctas), cta_hi = share(total, cta + 1, ctas);
  const int in_cta = static_cast<int>(cta_hi - cta_lo);
  const long long lo = cta_lo + share(in_cta, warp, kWarps);
  int todo = static_cast<int>(cta_lo + share(in_cta, warp + 1, kWarps) - lo);

  if (threadIdx.x < 2 * kWarps) desc[threadIdx.x].pair = -1;
  __syncthreads();

  if (todo > 0) {
    // ---- the sequence that holds unit `lo` ----
    Cursor put;                                   // next tile to copy
    {
      long long before = 0, seq_first = 0;
      for (int base = 0; base < pv.batch; base += 32) {
        const int b = base + lane;
        const int n = base == 0 ? first_n : (b < pv.batch ? seen_of(pv, opt, b, false).units() : 0);
        int inc = n;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int x = __shfl_up_sync(0xffffffffu, inc, o);
          if (lane >= o) inc += x;
        }
        const unsigned hit = __ballot_sync(0xffffffffu, (before + inc) * pv.n_kv_heads > lo);
        if (hit) {
          const int l = __ffs(hit) - 1;
          put.b = base + l;
          seq_first = (before + __shfl_sync(0xffffffffu, inc - n, l)) * pv.n_kv_heads;
          break;
        }
        before += __shfl_sync(0xffffffffu, inc, 31);
      }
      put.s = seen_of(pv, opt, put.b, false);
      const int off = static_cast<int>(lo - seq_first);
      put.h = off / put.s.units();
      put.i = off - put.h * put.s.units() - kPairCost;
      if (put.i < 0) {                            // the piece opens with units that hold no tile
        todo += put.i;
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
    // The queries of a pair are loaded while the pair before it is worked on (the next head, or the next sequence).
    uint32_t qn[16];
    int qn_b = put.b, qn_h = put.h;
    auto load_q = [&]() {
      const int gq = SMALL ? (g & 3) : g;
      const bool real = gq < group && qn_b < pv.batch;
      const uint16_t* src = q.data + (real ? qn_b * q.token + (qn_h * group + gq) * q.head : 0) + 2 * t4;
#pragma unroll
      for (int i = 0; i < 16; ++i) qn[i] = real ? *reinterpret_cast<const uint32_t*>(src + 8 * i) : 0u;
    };
    load_q();
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
      to_put -= advance(put, pv, opt);
      page = to_put > 0 ? page_of(put) : -1;
    };
#pragma unroll
    for (int st = 0; st < kStages - 1; ++st) {
      if (to_put > 0) copy_tile(st);
      cp_async_commit();
    }

    const float scale = opt.scale;
    const bool shaped = opt.cap > 0.0f;
    const int qi[2] = {SMALL ? (2 * t4) & 3 : 2 * t4, SMALL ? (2 * t4 + 1) & 3 : 2 * t4 + 1};   // this lane's queries
    uint32_t qf[16];
    float slope[2], m[2], l[2], o[8][4];
    bool from_start = false;
    bool fresh = true;                            // the next tile opens a pair
    int stage = 0;
    while (todo > 0) {
      if (to_put > 0) copy_tile((stage + kStages - 1) % kStages);
      cp_async_commit();
      if (fresh) {
        fresh = false;
        from_start = get.i == 0;
        if (qn_b != get.b || qn_h != get.h) {     // sequences without tokens lie between
          qn_b = get.b;
          qn_h = get.h;
          load_q();
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) qf[i] = qn[i];
        if (++qn_h == pv.n_kv_heads) {
          qn_h = 0;
          ++qn_b;
        }
        if (todo > get.s.n - get.i + kPairCost) load_q();   // otherwise this is the warp's last pair
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          slope[e] = opt.slopes && qi[e] < group ? opt.slopes[get.h * group + qi[e]] * kLog2e : 0.0f;
          m[e] = -INFINITY;
          l[e] = 0.0f;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
          for (int e = 0; e < 4; ++e) o[i][e] = 0.0f;
      }
      cp_async_wait<kStages - 1>();
      __syncwarp();
      const uint32_t kt = ring_u + stage * kStageBytes, vt = kt + kTileBytes;

      // S^T = K q^T: lanes 0..15 give the rows of the first unit of a step, 16..31 those of the second
      float s[2][4] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
      const int lr = lane & 15, lu = lane >> 4;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        uint32_t a[4];
        const int u = 2 * ks + lu;
        ldsm4(a, kt + lr * 256 + (((u & 8) | ((u ^ lr) & 7)) << 4));
        mma16816<BF16>(s[ks & 1], a, qf[2 * ks], qf[2 * ks + 1]);
      }
      const int t0 = tile_of(get.s, get.i) * kTile;
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = t0 + g + 8 * (e >> 1);
        float y = (s[0][e] + s[1][e]) * scale;
        if (shaped) {
          // tanh(z) = 1 - 2 / (exp(2 z) + 1): an error of a few 2^-24 of the cap, where tanh.approx has 2^-11
          const float z = exp2_fast(y * (2.0f * kLog2e / opt.cap));
          y = opt.cap - 2.0f * opt.cap * __frcp_rn(z + 1.0f);
        }
        y = fmaf(-slope[e & 1], static_cast<float>(get.s.len - 1 - j), y * kLog2e);
        const bool see = j < get.s.len && (j >= get.s.lo || j < get.s.pre);
        x[e] = see ? y : -INFINITY;
      }
      const float top[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
      if (__any_sync(0xffffffffu, top[0] > m[0] + kLag || top[1] > m[1] + kLag)) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float t = fmaxf(top[e], m[e]);
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
          const float f = t == -INFINITY ? 0.0f : exp2_fast(m[e] - t);
          m[e] = t;
          l[e] *= f;
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            o[i][e] *= f;
            o[i][2 + e] *= f;
          }
        }
      }
      float p[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = x[e] == -INFINITY ? 0.0f : exp2_fast(x[e] - m[e & 1]);
      l[0] += p[0] + p[2];
      l[1] += p[1] + p[3];
      uint32_t h0 = float2_to_pair<BF16>(p[0], p[1]), h1 = float2_to_pair<BF16>(p[2], p[3]);
      const float2 f0 = pair_to_float2<BF16>(h0), f1 = pair_to_float2<BF16>(h1);
      const uint32_t r0 = float2_to_pair<BF16>(p[0] - f0.x, p[1] - f0.y), r1 = float2_to_pair<BF16>(p[2] - f1.x, p[3] - f1.y);
      if (SMALL && t4 >= 2) {                     // columns 4..7 carry the low halves of queries 0..3
        h0 = r0;
        h1 = r1;
      }
      const uint32_t b0 = transpose8(h0), b1 = transpose8(h1);
      const uint32_t c0 = SMALL ? 0u : transpose8(r0), c1 = SMALL ? 0u : transpose8(r1);
      // O^T += V^T P^T: lanes 0..7 tokens 0..7 of a unit, 8..15 the next unit, 16..31 tokens 8..15
      const int vr = (lane & 7) + ((lane >> 4) << 3), vu = (lane >> 3) & 1;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        uint32_t a[4];
        const int u = 2 * i + vu;
        ldsm4_trans(a, vt + vr * 256 + (((u & 8) | ((u ^ vr) & 7)) << 4));
        mma16816<BF16>(o[i], a, b0, b1);
        if (!SMALL) mma16816<BF16>(o[i], a, c0, c1);
      }
      __syncwarp();                               // the stage may be filled again
      stage = stage + 1 == kStages ? 0 : stage + 1;

      const bool last_of_pair = get.i + 1 == get.s.n, last_of_all = todo <= (last_of_pair ? 1 + kPairCost : 1);
      if (last_of_pair || last_of_all) {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
          for (int d = 4; d < 32; d <<= 1) l[e] += __shfl_xor_sync(0xffffffffu, l[e], d);
        if (SMALL)
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][e] += __shfl_xor_sync(0xffffffffu, o[i][e], 2);
        if (from_start && last_of_pair) {
          const float inv0 = l[0] == 0.0f ? 0.0f : 1.0f / l[0], inv1 = l[1] == 0.0f ? 0.0f : 1.0f / l[1];
#pragma unroll
          for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const uint32_t w = transpose8(float2_to_pair<BF16>(o[i][2 * e] * inv0, o[i][2 * e + 1] * inv1));
              if (g < group)                      // lane (g, t4): query g, channels 16 i + 8 e + 2 t4
                *reinterpret_cast<uint32_t*>(out.data + get.b * out.token + (get.h * group + g) * out.head + 16 * i + 8 * e + 2 * t4) = w;
            }
        } else {
          const int which = from_start ? 1 : 0;
          float* dst = which ? reinterpret_cast<float*>(ring) : head_piece + warp * piece_floats;
          if (which) {                            // the ring holds no tile that is still needed: this was the warp's last
            cp_async_wait<0>();
            __syncwarp();
          }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int qq = 2 * t4 + e;
            if (qq < group) {
#pragma unroll
              for (int i = 0; i < 8; ++i) {
                dst[qq * kHeadDim + 16 * i + g] = o[i][e];
                dst[qq * kHeadDim + 16 * i + 8 + g] = o[i][2 + e];
              }
              if (g == 0) *reinterpret_cast<float2*>(dst + group * kHeadDim + 2 * qq) = make_float2(m[e], l[e]);
            }
          }
          if (lane == 0) {
            Piece& d = desc[2 * warp + which];
            d.pair = get.b * pv.n_kv_heads + get.h;
            d.starts = from_start;
            d.ends = last_of_pair;
          }
        }
        fresh = true;
      }
      todo -= advance(get, pv, opt);
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
  auto row_of = [&](int pair, int g) -> uint16_t* {
    const int b = pair / pv.n_kv_heads, h = pair - b * pv.n_kv_heads;
    return out.data + b * out.token + static_cast<long long>(h * group + g) * out.head;
  };
  // Runs of pieces of one pair; a warp takes (run, query) jobs.  A run that is not the whole pair goes to the
  // workspace: slot 1 if it holds the pair's first tile (at most one run, the last), slot 0 otherwise (the first).
  int job = 0, cross[2] = {-1, -1};
  for (unsigned rest = valid; rest;) {
    const int first = __ffs(rest) - 1, pair = __shfl_sync(0xffffffffu, my_pair, first);
    const unsigned run = __ballot_sync(0xffffffffu, my_pair == pair);
    rest &= ~run;
    const bool starts = desc[first].starts, whole = starts && desc[31 - __clz(run)].ends;
    if (!whole) cross[starts] = pair;
    float* joined = ws.part + (static_cast<long long>(cta) * 2 + (starts ? 1 : 0)) * piece_floats;
    for (int g2 = 0; g2 < group; ++g2, ++job)
      if (job % kWarps == warp)
        join_query<BF16, false>([&](int p) {
          unsigned r = run;                       // the p-th piece of the run
          for (; p > 0; --p) r &= r - 1;
          return piece_at(__ffs(r) - 1);
        }, __popc(run), group, g2, lane,
                                whole ? row_of(pair, g2) : nullptr, joined);
  }
  if (cross[0] < 0 && cross[1] < 0) return;

  // ---- pairs that span CTAs: the CTA that arrives last adds the pieces ----
  auto cta_of = [&](long long unit) -> int {      // largest c with share(total, c, ctas) <= unit
    int c = static_cast<int>(static_cast<double>(unit) * ctas / static_cast<double>(total));
    while (c > 0 && share(total, c, ctas) > unit) --c;
    while (c + 1 < ctas && share(total, c + 1, ctas) <= unit) ++c;
    return c;
  };
  int c0 = 0, c1 = 0;
  if (warp < 2 && cross[warp] >= 0) {
    const int pair = cross[warp], b = pair / pv.n_kv_heads, h = pair - b * pv.n_kv_heads;
    long long before = 0;
    for (int x = lane; x < b; x += 32) before += x < 32 ? first_n : seen_of(pv, opt, x, false).units();
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
    const int n = seen_of(pv, opt, b, false).units();
    const long long u0 = before * pv.n_kv_heads + static_cast<long long>(h) * n;
    c0 = cta_of(u0 + kPairCost);
    c1 = cta_of(u0 + n - 1);
  }
  __threadfence();
  __syncthreads();
  if (warp < 2 && cross[warp] >= 0 && lane == 0) {
    turn[warp] = static_cast<int>(atomicInc(reinterpret_cast<unsigned*>(ws.arrived) + cross[warp], static_cast<unsigned>(c1 - c0)));
    turn[2 + warp] = c0;
    turn[4 + warp] = c1;
  }
  __syncthreads();
  job = 0;
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    if (cross[k] < 0) continue;
    const int from = turn[2 + k], to = turn[4 + k];
    if (turn[k] != to - from) continue;
    __threadfence();
    for (int g2 = 0; g2 < group; ++g2, ++job)
      if (job % kWarps == warp)
        join_query<BF16, true>([&](int p) -> const float* {
          return ws.part + (static_cast<long long>(from + p) * 2 + (p == 0 ? 1 : 0)) * piece_floats;
        }, to - from + 1, group, g2, lane, row_of(cross[k], g2), nullptr);
  }
}

size_t decode_smem(int group) {
  return kWarps * kStages * kStageBytes + static_cast<size_t>(kWarps) * piece_floats_of(group) * 4 + 2 * kWarps * sizeof(Piece) + 32;
}

template <bool BF16, bool SMALL>
cudaError_t launch(const PagedView& pv, const RowsView& q, const RowsView& out, const AttnOptions& opt, int group, const Workspace& ws,
                   int grid, cudaStream_t st) {
  const size_t smem = decode_smem(group);
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_shared_memory(paged_decode_kernel<BF16, SMALL>, decode_smem(SMALL ? 4 : kMaxQueryGroup), done);
  if (e != cudaSuccess) return e;
  paged_decode_kernel<BF16, SMALL><<<grid, kWarps * 32, smem, st>>>(pv, q, out, opt, group, ws);
  return cudaGetLastError();
}

long long part_bytes(int group) {
  const long long n = 2ll * sm_count_of_current_device() * piece_floats_of(group) * 4;
  return (n + 15) / 16 * 16;
}

}  // namespace

// partial results of the CTAs' first and last pairs, then one arrival counter per (sequence, kv head)
long long paged_decode_workspace_bytes(int batch, int n_kv_heads, int group) {
  return (part_bytes(group) + static_cast<long long>(batch) * n_kv_heads * 4 + 15) / 16 * 16;
}

cudaError_t launch_paged_decode(const PagedView& cache, const RowsView& q, const RowsView& out, const AttnOptions& opt, void* workspace,
                                cudaStream_t st) {
  PagedView pv = cache;
  if (pv.batch <= 0) return cudaSuccess;
  if (pv.n_pages == 0) {                          // copies of no bytes still name an address
    pv.k = pv.v = q.data;
    pv.k_page = pv.k_head = pv.k_slot = pv.v_page = pv.v_head = pv.v_slot = 0;
  }
  const int group = q.n_heads / pv.n_kv_heads, grid = sm_count_of_current_device();
  Workspace ws;
  ws.part = static_cast<float*>(workspace);
  ws.arrived = reinterpret_cast<int*>(static_cast<uint8_t*>(workspace) + part_bytes(group));
  const bool bf16 = pv.dtype == MOQAE_DTYPE_BF16;
  if (group <= 4)
    return bf16 ? launch<true, true>(pv, q, out, opt, group, ws, grid, st) : launch<false, true>(pv, q, out, opt, group, ws, grid, st);
  return bf16 ? launch<true, false>(pv, q, out, opt, group, ws, grid, st) : launch<false, false>(pv, q, out, opt, group, ws, grid, st);
}

}  // namespace moqae
