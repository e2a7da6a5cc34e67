// Attention of one new token per sequence over a paged 4-bit cache (moqae_paged4_decode_attn), and of a few
// (moqae_paged4_prefill_attn where the sequences bring so few rows that the large tiles would be empty).
//
// Mathematics.  A cached key is k^ = z + s code per group of 32 channels, so for a query row q
//   q.k^_j = sum_g s_jg (q_g . code_jg) + z_jg (sum of q_g),     o_c = sum_j (p_j s_jg) code_jc + sum_j p_j z_jg:
// the codes go to the tensor cores as they are, as the small fp16 numbers code 2^-24 and (where they stand four bits higher)
// code 2^-20, one logic instruction per register of two; scales and zeros are a few values per token.
//
//   Work, tiles, pieces and their joining are those of the 16-bit pages (paged_split.cuh); a tile of 16 tokens of one kv
//   head is 2560 bytes in one place, fetched with one bulk copy by the warp that works on it, two at a time.
//   Products, on mma.sync m16n8k16.  S^T = codes q^T: per group two products whose sums meet the tokens' scales in registers, and one for the
//   zeros of all groups, with the sums of the queries' groups as high + low halves.  O^T += codes^T (p s)^T: weights become fp16, turn by movmatrix, and
//   meet a group's value scales as packed pairs; one more product sums what the zeros give and, in a row of ones, the weights.
//   Queries are scaled by a power of two to at most 16, so that bf16 rows and small ones keep their bits in fp16 (2^-24 of the largest).
//   Signs.  Codes are never negative, and a sum of many that the zeros then cancel loses what the mean over a long context leaves (the
//   tensor cores cut off the bits below 2^-23 of a running sum: 131000 tokens were off by 0.004 of their norm instead of the 0.0017 of
//   rounding to bf16, 32000 in one warp by 0.011).  So every second token has 15 - code with the weight -p, and the zeros become the
//   middles of the ranges, mid = z + 7.5 s: with sums over even and odd tokens
//     sum p (z + s code) = [sum_even p s code - sum_odd p s (15 - code)] + sum p mid - 7.5 (sum_even p s - sum_odd p s),
//   and none of the three grows with the number of tokens as they do not cancel one another.
//   Weights.  p and p s are rounded to fp16, mid too: fp16 results are 3.4e-4 to 5.6e-4 of their norm off instead of the 2.1e-4 of their own rounding, bf16
//   ones 1.72e-3 instead of 1.66e-3, beside the 0.1 of holding the cache in 4 bits.  (24 sequences under a window and a cap, fp16, 5.6e-4 and 137 us: the
//   last sum over the rounded products, four more small products per tile, 3.6e-4 and 143 us; p s rounded once, from halves of p, too, 3.1e-4 and 148 us.)  The largest weight is kept near 2^15 / (largest scale), so that small ones
//   do not vanish below fp16's steps; the sum of the weights is that of the rounded ones.
//   Measured.  4 sequences of 131000 tokens, 32 / 8 heads, bf16: 123 to 139 us for 671 MB (floor 102); 61 of 1 to 32000: 54 us for 233 MB (floor 36); 32 of 4000,
//   40 / 40 heads, fp16: 146 us for 820 MB (floor 125), under a cap 162, under a distance bias 157; 8 of 1000: 13 us; one of 60: 7 us.  Nothing is full:
//   with one sequence of 131071 tokens issue slots are 53 % busy, the ALU pipe (78 of a tile's 300 instructions bring codes out of their words, at half rate)
//   51 %, the tensor pipe 23 %, memory 44 % (60 % and 60 % of the first two with four sequences).  A scheduler has four warps, each a chain of
//   dependent steps, so instructions and their latency bound it together; about 17 us of a long call are its start, uneven ends and the joining.
//   (The 16-warp forms spill 8 bytes, 44 under a cap or bias.)
#include "paged4.cuh"
#include "paged_split.cuh"
#include "ptx.cuh"

namespace moqae {

namespace {

// Warps of a CTA (the most that registers and pieces leave room for: with 12 instead of 16 and a third stage, 4 sequences of 131000 tokens take 128 us
// instead of 123, 32 of 4000 with 40 heads 153 instead of 146) and stages of a warp's ring, of two tiles each.
__host__ __device__ constexpr int warps_of(int form) { return form == kFew16Q ? 8 : form == kOne8Q ? 12 : 16; }
__host__ __device__ constexpr int stages4_of(int form) { return form == kFew16Q ? 3 : 2; }
constexpr int kStageBytes4 = 2 * kTileBytes4;
// See share_work.  Measured with least tiles per warp / most per pair of 1 / 12, 1 / 24, 2 / 48, 2 / 96, 4 / 160 (us): 8 pairs of 21 tiles 12.2 / 10.2 / 10.2 / 10.2 / 10.2,
// of 63 12.8 / 13.0 / 13.3 / 13.5 / 13.4, of 157 13.4 / 13.6 / 13.8 / 13.7 / 18.7; 64 pairs of 63 13.2 / 13.2 / 13.4 / 13.5 / 13.6; 256 of 4 11.2 / 11.2 / 11.4 / 11.5 / 13.4.
constexpr int kMinTiles4 = 1, kPairTiles4 = 24;
// Weights of a row are 2^(score - reference), at most 2^top: the reference lies top - kLag below the largest score so far and moves when
// a score passes it by top.  top is 15, less where value scales above 1 would take p s out of fp16.
constexpr float kLag = 3.0f;
constexpr float kTop = 15.0f;
constexpr float kNothing = -1e30f;                // reference of a row that has seen nothing
constexpr uint32_t kLow = 0x000f000fu, kHigh = 0x00f000f0u;     // codes in bits 0..3 and 4..7 of both halves
constexpr uint32_t kOddSign = 0x80000000u;                      // the second token's sign

// d = a b + 0, d += a b: fp16 operands whatever the dtype of queries and results
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.0f));
}
__device__ __forceinline__ void mma_more(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];\n" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];\n" : "=r"(v.x), "=r"(v.y) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t v;
  asm volatile("ld.shared.u32 %0, [%1];\n" : "=r"(v) : "r"(a) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t mul2(uint32_t a, uint32_t b) {
  const __half2 r = __hmul2(*reinterpret_cast<const __half2*>(&a), *reinterpret_cast<const __half2*>(&b));
  return *reinterpret_cast<const uint32_t*>(&r);
}
// z + 7.5 s, the second token's negated
__device__ __forceinline__ uint32_t mid2(uint32_t s, uint32_t z) {
  const __half2 r = __hfma2(*reinterpret_cast<const __half2*>(&s), __float2half2_rn(7.5f), *reinterpret_cast<const __half2*>(&z));
  return *reinterpret_cast<const uint32_t*>(&r) ^ kOddSign;
}
__device__ __forceinline__ float low_half(uint32_t u) { return __low2float(*reinterpret_cast<const __half2*>(&u)); }
__device__ __forceinline__ float high_half(uint32_t u) { return __high2float(*reinterpret_cast<const __half2*>(&u)); }

// SHAPED: scores have a cap or a distance bias
template <bool BF16, int FORM, bool SHAPED>
__global__ void __launch_bounds__(warps_of(FORM) * 32, 1) paged4_decode_kernel(PagedView pv, AttnOptions opt, DecodeJob job) {
  constexpr int kRows = set_rows(FORM), kCols = kRows / 8, kStages = stages4_of(FORM), kWarps = warps_of(FORM);
  extern __shared__ __align__(128) uint8_t smem[];
  // [warps][stages] tiles; the piece each warp may leave behind at the start of its range (the one at its end goes into
  // its ring, which is empty by then); barriers of the stages; descriptors
  const int piece_rows = FORM == kFew16Q ? kRows : job.group;
  const int piece_floats = piece_floats_of(piece_rows);
  float* head_piece = reinterpret_cast<float*>(smem + kWarps * kStages * kStageBytes4);
  uint64_t* bars = reinterpret_cast<uint64_t*>(head_piece + kWarps * piece_floats);
  Piece* desc = reinterpret_cast<Piece*>(bars + kWarps * kStages);                  // [2 * kWarps]
  int* turn = reinterpret_cast<int*>(desc + 2 * kWarps);                            // see join_pieces
  volatile int* failed = turn + 6;
  Cursor* cursors = reinterpret_cast<Cursor*>(turn + 8);                            // [2 * kWarps]

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int g = lane >> 2, t4 = lane & 3;
  uint8_t* ring = smem + warp * kStages * kStageBytes4;
  const uint32_t ring_u = smem_u32(ring), bar_u = smem_u32(bars + warp * kStages);
  auto token_of = [&](int row) { return token_in_sequence<FORM>(job, row); };

  if (threadIdx.x < 2 * kWarps) desc[threadIdx.x].pair = -1;
  if (threadIdx.x == 0) *failed = 0;
  if (lane == 0) {
    for (int i = 0; i < kStages; ++i) mbar_init(bar_u + 8 * i, 1);
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  after_previous();

  Part part;
  if (!share_work<FORM, kWarps, kMinTiles4, kPairTiles4>(pv, opt, job, warp, lane, part)) return;
  __syncthreads();

  if (part.todo > 0) {
    long long at;                                 // unit of the pair's tile that is worked on first
    {
      const Cursor first = find_first<FORM>(pv, opt, job, lane, part, at);
      if (lane == 0) cursors[2 * warp] = cursors[2 * warp + 1] = first;
    }
    __syncwarp();
    // Two walks over the warp's tiles: `put` copies them, `get` works on them.  What a tile needs of its pair is in registers, the rest
    // in shared memory (lane 0 takes it to the next pair).
    Cursor &put = cursors[2 * warp], &get = cursors[2 * warp + 1];
    int todo = part.todo, to_put = part.todo;
    // Within a pair the tiles are walked backwards: under a distance bias the largest scores then come first (the reference would move with
    // nearly every tile the other way: 32 sequences of 4000, 40 heads, 194 us instead of 170 when that was changed).
    int put_i, put_left, put_pre, put_first;      // index of the next tile in the pair's walk, tiles left; the walk: see tile_of
    const int32_t* put_row;                       // the sequence's pages
    const uint8_t* put_head;                      // the head's part of page 0
    int at_token, page;                           // of lanes 0 and 1: first token of the next tile and of the one after it, and their pages
    auto look_up = [&]() {
      const int i = put_i - (lane & 1);
      at_token = (i < put_pre ? i : put_first + i - put_pre) * kTile;
      page = (lane & 1) < put_left ? put_row[at_token >> pv.page_shift] : 0;
    };
    auto open_put = [&]() {
      put_left = min(put.s.n - put.i, to_put);
      put_i = put.i + put_left - 1;
      put_pre = put.s.n_pre;
      put_first = put.s.first;
      put_row = pv.table + static_cast<long long>(put.b) * pv.max_pages;
      put_head = reinterpret_cast<const uint8_t*>(pv.k) + put.h * pv.k_head;
      to_put -= put_left + pair_cost(FORM);
      look_up();
    };
    open_put();
    __syncwarp();
    // copy of the next two tiles of the pair (or its last) into stage st; a tile without a page is all zeros
    auto copy_tiles = [&](int st) {
      if (put_left <= 0) return;
      const int count = min(put_left, 2);
      const uint32_t bar = bar_u + 8 * st;
      const bool mine = lane < count, good = static_cast<unsigned>(page) < static_cast<unsigned>(pv.n_pages);
      const unsigned bad = __ballot_sync(0xffffffffu, mine && !good);
      if (bad) {
        if (mine && !good) paged_status(pv.status, MOQAE_ERR_CORRUPT_TABLE, put.b, at_token >> pv.page_shift);
        for (int k = 0; k < 2; ++k)
          for (int i = lane; i < kTileBytes4 / 16 && (bad >> k & 1u); i += 32)
            *reinterpret_cast<uint4*>(ring + st * kStageBytes4 + k * kTileBytes4 + 16 * i) = make_uint4(0, 0, 0, 0);
        fence_async_smem();
        __syncwarp();
      }
      // (a copy may land before its bytes are announced: the phase ends with the arrival that announces them)
      if (lane == 0) mbar_expect_tx(bar, (count - __popc(bad)) * kTileBytes4);
      if (mine && good)
        bulk_load(ring_u + st * kStageBytes4 + lane * kTileBytes4, put_head + page * pv.k_page + (at_token & (pv.page_size - 1)) * kTokenBytes4,
                  kTileBytes4, bar);
      put_left -= count;
      put_i -= count;
      if (put_left > 0) {
        look_up();
      } else if (to_put > 0) {
        __syncwarp();
        if (lane == 0) next_pair<FORM>(put, pv, opt, job);
        __syncwarp();
        open_put();
      }
    };
#pragma unroll
    for (int st = 0; st < kStages - 1; ++st) copy_tiles(st);

    const bool capped = SHAPED && opt.cap > 0.0f;
    const float to_score = opt.scale * (capped ? 1.0f / opt.cap : kLog2e);
    int stage = 0;
    uint32_t parity = 0;
    while (todo > 0) {
      // ---- a pair: the tiles of it that are the warp's ----
      const int n_here = min(get.s.n - get.i, todo);
      const bool from_start = get.i == 0, last_of_pair = get.i + n_here == get.s.n;
      uint32_t qf[kCols][4][2][2], qz[kCols][2];  // fragments of the queries; sums of their groups
      float factor[kCols][2], slope[kCols][2], m[kCols][2], o[kCols][4][2][4], zo[kCols][4];
      float top = kTop;
      uint32_t most = 0x3c003c00u;                // largest scale that `top` allows, in both halves
      // Tiles that every row sees whole, by their index in the walk: whole_lo <= index < whole_lo + n_whole (of the prefix none is counted).
      int full_lo = get.s.lo, full_hi = get.s.len;
      if (FORM == kFew16Q) {
        full_hi = get.s.pos0 + token_of(get.s.row0) + 1;
        full_lo = opt.window > 0 ? get.s.pos0 + token_of(get.s.row0 + get.s.rows - 1) - opt.window + 1 : 0;
      }
      const int n_pre = get.s.n_pre, behind = get.s.first - n_pre;
      const int whole_lo = max(n_pre, (max(full_lo, 0) + kTile - 1) / kTile - behind), n_whole = max(full_hi / kTile - behind - whole_lo, 0);
#pragma unroll
      for (int c = 0; c < kCols; ++c) {
        // ---- queries: lane (g, t4) takes channels 8 t4 .. 8 t4 + 7 of every group of row 8 c + g ----
        const int r = 8 * c + g, t = token_of(get.s.row0 + r);
        const bool real = r < get.s.rows;
        const uint16_t* src = job.q.data + 8 * t4;
        if (real) src += (get.s.q_first + t) * job.q.token + (get.h * job.group + get.s.row0 + r - t * job.group) * job.q.head;
        uint4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = real ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0, 0, 0, 0);
        float big = 0.0f;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = pair_to_float2<BF16>(w[e]);
            big = fmaxf(big, fmaxf(fabsf(f.x), fabsf(f.y)));
          }
        }
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 1));
        big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, 2));
        const uint32_t ex = max(__float_as_uint(big) >> 23, 4u);        // 2^(ex - 127) <= largest
        const float up = __uint_as_float((257u - ex) << 23), down = __uint_as_float((ex - 3u) << 23);   // 2^(130 - ex) and its inverse
        float sums[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t w[4] = {raw[i].x, raw[i].y, raw[i].z, raw[i].w};
          float x[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = pair_to_float2<BF16>(w[e]);
            x[2 * e] = f.x * up;
            x[2 * e + 1] = f.y * up;
          }
          // channel e of a word of codes stands in its bits 4 e: pairs (e, e + 4), odd ones 16 times too large
          qf[c][i][0][0] = float2_to_pair<false>(x[0], x[4]);
          qf[c][i][0][1] = float2_to_pair<false>(x[1] * 0.0625f, x[5] * 0.0625f);
          qf[c][i][1][0] = float2_to_pair<false>(x[2], x[6]);
          qf[c][i][1][1] = float2_to_pair<false>(x[3] * 0.0625f, x[7] * 0.0625f);
          sums[i] = ((x[0] + x[1]) + (x[2] + x[3])) + ((x[4] + x[5]) + (x[6] + x[7]));
          sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 1);
          sums[i] += __shfl_xor_sync(0xffffffffu, sums[i], 2);
        }
        // zeros are columns 4..7 of a token's scales and zeros: lanes t4 = 2, 3
        const float s0 = t4 == 2 ? sums[0] : t4 == 3 ? sums[2] : 0.0f, s1 = t4 == 2 ? sums[1] : t4 == 3 ? sums[3] : 0.0f;
        qz[c][0] = float2_to_pair<false>(s0, s1);
        qz[c][1] = float2_to_pair<false>(s0 - low_half(qz[c][0]), s1 - high_half(qz[c][0]));
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          // (a row of zeros under a tiny scale would make it 0, which is no number beside the -inf of a masked score)
          factor[c][e] = fmaxf(__shfl_sync(0xffffffffu, down, 4 * (2 * t4 + e)) * 16777216.0f * to_score, 1.17549435e-38f);
          m[c][e] = kNothing;
          if (SHAPED) {
            const int rr = min(8 * c + 2 * t4 + e, get.s.rows - 1), head = get.s.row0 + rr - token_of(get.s.row0 + rr) * job.group;
            slope[c][e] = opt.slopes ? -kLog2e * opt.slopes[get.h * job.group + head] : 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          zo[c][i] = 0.0f;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[c][i][0][e] = o[c][i][1][e] = 0.0f;
        }
      }

      const int begin = get.i;
      int index = begin + n_here - 1;             // of the tile in the walk
      while (index >= begin) {
        copy_tiles(stage == 0 ? kStages - 1 : stage - 1);
        if (!mbar_try_wait(bar_u + 8 * stage, parity) && !*failed && !mbar_wait_bounded(bar_u + 8 * stage, parity)) *failed = 1;
        __syncwarp();
        const uint32_t stage_at = ring_u + stage * kStageBytes4;
#pragma unroll 1
        for (uint32_t tile = stage_at; tile < stage_at + kStageBytes4 && index >= begin; tile += kTileBytes4, --index) {
          const bool edge = static_cast<unsigned>(index - whole_lo) >= static_cast<unsigned>(n_whole);
          auto first_token = [&]() { return (index < n_pre ? index : index + behind) * kTile; };
          if (edge) {
            // what no row may use can hold anything: its scales and zeros become 0
            const int j = first_token() + lane;
            if (lane < kTile && !(j < get.s.len && (j >= get.s.lo || j < get.s.pre))) {
              uint8_t* tp = ring + (tile - ring_u);
              *reinterpret_cast<uint4*>(tp + kKeyMeta4 + 16 * lane) = make_uint4(0, 0, 0, 0);
#pragma unroll
              for (int i = 0; i < 8; ++i) reinterpret_cast<uint16_t*>(tp + kValueMeta4 + 32 * (lane >> 1))[2 * i + (lane & 1)] = 0;
            }
            fence_async_smem();
            __syncwarp();
          }

          // ---- scores ----
          float x[kCols][4];
          {
            const uint4 k0 = lds128(tile + 64 * g + 16 * t4), k1 = lds128(tile + 64 * (g + 8) + 16 * t4);
            const uint2 c0 = lds64(tile + kKeyMeta4 + 16 * g), c1 = lds64(tile + kKeyMeta4 + 16 * (g + 8));
            uint32_t zm[4];                           // scales and zeros of tokens 0..7, 8..15, and once more
            ldsm4(zm, tile + kKeyMeta4 + 16 * (lane & 15));
            const uint32_t w0[4] = {k0.x, k0.y, k0.z, k0.w}, w1[4] = {k1.x, k1.y, k1.z, k1.w};
            const float s0[4] = {low_half(c0.x), high_half(c0.x), low_half(c0.y), high_half(c0.y)};
            const float s1[4] = {low_half(c1.x), high_half(c1.x), low_half(c1.y), high_half(c1.y)};
#pragma unroll
            for (int c = 0; c < kCols; ++c) {
              float acc[4];
              mma_first(acc, zm[0], zm[1], zm[2], zm[3], qz[c][0], qz[c][1]);
#pragma unroll
              for (int e = 0; e < 4; ++e) x[c][e] = acc[e] * 5.9604645e-8f;     // 2^-24, as the codes have it
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t a = w0[i], b = w1[i], a8 = a >> 8, b8 = b >> 8;
#pragma unroll
              for (int c = 0; c < kCols; ++c) {
                float acc[4];
                mma_first(acc, a & kLow, b & kLow, a & kHigh, b & kHigh, qf[c][i][0][0], qf[c][i][0][1]);
                mma_more(acc, a8 & kLow, b8 & kLow, a8 & kHigh, b8 & kHigh, qf[c][i][1][0], qf[c][i][1][1]);
                x[c][0] = fmaf(acc[0], s0[i], x[c][0]);
                x[c][1] = fmaf(acc[1], s0[i], x[c][1]);
                x[c][2] = fmaf(acc[2], s1[i], x[c][2]);
                x[c][3] = fmaf(acc[3], s1[i], x[c][3]);
              }
            }
          }
          // value scales and zeros: pairs of tokens (2 t4, 2 t4 + 1), (2 t4 + 8, 2 t4 + 9)
          const uint32_t vm = tile + kValueMeta4 + 32 * t4;
          const uint32_t vs0 = lds32(vm + 4 * (g & 3)), vs1 = lds32(vm + 128 + 4 * (g & 3));     // scales of group g % 4
          const uint32_t vz0 = lds32(vm + 16 + 4 * (g & 3)), vz1 = lds32(vm + 144 + 4 * (g & 3));
          bool above;
          {
            const __half2 big = __hmax2(*reinterpret_cast<const __half2*>(&vs0), *reinterpret_cast<const __half2*>(&vs1));
            above = !__hble2(big, *reinterpret_cast<const __half2*>(&most));
          }
          if (SHAPED) {                               // otherwise x times factor is the score
            float far = 0.0f;
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                x[c][e] *= factor[c][e & 1];
                far = fmaxf(far, fabsf(x[c][e]));
              }
            // Both columns of a lane, or with groups of one head, where the second holds nothing, the first: f(c, e).
            auto columns = [&](auto f) {
#pragma unroll
              for (int c = 0; c < kCols; ++c) {
                f(c, 0);
                f(c, 2);
              }
              if (FORM == kFew16Q || job.group > 1)
#pragma unroll
                for (int c = 0; c < kCols; ++c) {
                  f(c, 1);
                  f(c, 3);
                }
            };
            if (capped) {
              const float cap2 = opt.cap * kLog2e;
              if (!__any_sync(0xffffffffu, far > 0.5f))          // no score passes half the cap
                columns([&](int c, int e) {
                  const float z = x[c][e], u = z * z;
                  x[c][e] = cap2 * z * fmaf(fmaf(fmaf(tanh_coef_near(3), u, tanh_coef_near(2)), u, tanh_coef_near(1)), u, tanh_coef_near(0));
                });
              else
                columns([&](int c, int e) { x[c][e] = cap2 * tanh_of(x[c][e]); });
            }
            if (opt.slopes) {
              const int t0 = first_token();
              columns([&](int c, int e) {
                const int p = FORM == kFew16Q ? get.s.pos0 + token_of(get.s.row0 + min(8 * c + 2 * t4 + (e & 1), get.s.rows - 1)) : get.s.pos0;
                x[c][e] = fmaf(slope[c][e & 1], fabsf(static_cast<float>(p - (t0 + g + 8 * (e >> 1)))), x[c][e]);
              });
            }
          }
          if (edge) {
            const int t0 = first_token();
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const int j = t0 + g + 8 * (e >> 1);
                bool see = j < get.s.len && (j >= get.s.lo || j < get.s.pre);
                if (FORM == kFew16Q) {
                  const int p = get.s.pos0 + token_of(get.s.row0 + min(8 * c + 2 * t4 + (e & 1), get.s.rows - 1));
                  see = (j <= p && (opt.window == 0 || j > p - opt.window)) || j < get.s.prefix;
                }
                if (!see) x[c][e] = -INFINITY;
              }
          }
          float r[kCols][4];                          // scores above the reference
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
#pragma unroll
            for (int e = 0; e < 4; ++e) r[c][e] = SHAPED ? x[c][e] - m[c][e & 1] : fmaf(x[c][e], factor[c][e & 1], -m[c][e & 1]);
            above = above || fmaxf(fmaxf(r[c][0], r[c][1]), fmaxf(r[c][2], r[c][3])) > top;
          }
          if (__any_sync(0xffffffffu, above)) {
            float sm = fmaxf(fmaxf(low_half(vs0), high_half(vs0)), fmaxf(low_half(vs1), high_half(vs1)));   // largest value scale of the tile
#pragma unroll
            for (int d = 1; d < 32; d <<= 1) sm = fmaxf(sm, __shfl_xor_sync(0xffffffffu, sm, d));
            float lower = 0.0f;
            const int up = static_cast<int>((__float_as_uint(sm) + 0x007fffffu) >> 23) - 127;     // sm <= 2^up
            if (static_cast<float>(up) > kTop - top) {
              lower = static_cast<float>(up) - (kTop - top);
              top -= lower;
              const uint32_t h = static_cast<uint32_t>(min(up, 15) + 15) << 10;
              most = h | (h << 16);
            }
#pragma unroll
            for (int c = 0; c < kCols; ++c)
#pragma unroll
              for (int e = 0; e < 2; ++e) {
                // (Scores are rounded before the reference is taken from them, and weights stay below 2^top whatever the difference of two roundings is: in one
                // step a score of 2^27 would be off from its own reference by more than fp16 can hold.)
                const float y0 = SHAPED ? x[c][e] : __fmul_rn(x[c][e], factor[c][e]), y1 = SHAPED ? x[c][2 + e] : __fmul_rn(x[c][2 + e], factor[c][e]);
                float t = fmaxf(y0, y1);
#pragma unroll
                for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
                t = fmaxf(t - (top - kLag), m[c][e] + lower);
                const float f = exp2_fast(m[c][e] - t);
                m[c][e] = t;
                r[c][e] = y0 - t > top ? top : y0 - t;         // (not a minimum: what is no number stays none)
                r[c][2 + e] = y1 - t > top ? top : y1 - t;
                zo[c][e] *= f;
                zo[c][2 + e] *= f;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                  o[c][i][0][e] *= f;
                  o[c][i][0][2 + e] *= f;
                  o[c][i][1][e] *= f;
                  o[c][i][1][2 + e] *= f;
                }
              }
          }
          uint32_t b0[kCols], b1[kCols];
          // rows 0..3: scales, 4..7: middles, 8: ones, with the signs of the weights
          const uint32_t a0 = g < 4 ? vs0 : mid2(vs0, vz0), a1 = g < 4 ? vs1 : mid2(vs1, vz1), ones = g == 0 ? 0xbc003c00u : 0u;
#pragma unroll
          for (int c = 0; c < kCols; ++c) {
            b0[c] = transpose8(float2_to_pair<false>(exp2_fast(r[c][0]), exp2_fast(r[c][1]))) ^ kOddSign;
            b1[c] = transpose8(float2_to_pair<false>(exp2_fast(r[c][2]), exp2_fast(r[c][3]))) ^ kOddSign;
            mma_more(zo[c], a0, ones, a1, ones, b0[c], b1[c]);
          }
          // ---- values ----
          {
            const uint4 v0 = lds128(vm), v1 = lds128(vm + 128);
            const uint32_t s0[4] = {v0.x, v0.y, v0.z, v0.w}, s1[4] = {v1.x, v1.y, v1.z, v1.w};
            const uint32_t vc = tile + kValueCodes4 + 512 * (g >> 2) + 32 * t4 + 8 * (g & 3);
            const uint2 a = lds64(vc), d = lds64(vc + 256);          // tokens 2 t4, + 8
            uint2 b = lds64(vc + 128), e = lds64(vc + 384);          // tokens 2 t4 + 1, + 9: 15 - code
            b = make_uint2(~b.x, ~b.y);
            e = make_uint2(~e.x, ~e.y);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const uint32_t p0 = __byte_perm(i < 2 ? a.x : a.y, i < 2 ? b.x : b.y, (i & 1) ? 0x7632 : 0x5410), q0 = p0 >> 8;
              const uint32_t p1 = __byte_perm(i < 2 ? d.x : d.y, i < 2 ? e.x : e.y, (i & 1) ? 0x7632 : 0x5410), q1 = p1 >> 8;
#pragma unroll
              for (int c = 0; c < kCols; ++c) {
                const uint32_t w0 = mul2(b0[c], s0[i]), w1 = mul2(b1[c], s1[i]);
                mma_more(o[c][i][0], p0 & kLow, p0 & kHigh, p1 & kLow, p1 & kHigh, w0, w1);
                mma_more(o[c][i][1], q0 & kLow, q0 & kHigh, q1 & kLow, q1 & kHigh, w0, w1);
              }
            }
          }
        }
        __syncwarp();                               // the stage may be filled again
        if (++stage == kStages) {
          stage = 0;
          parity ^= 1;
        }
      }
      {
        // lane (g, t4): rows 8 c + 2 t4 + e, channels 32 i + 4 g + 2 j + half; the middles' sums in lanes 4 + i, the scales' in i, the weights' in 0
        const bool whole = from_start && last_of_pair;
        const int which = from_start ? 1 : 0;
        float* dst = which ? reinterpret_cast<float*>(ring) : head_piece + warp * piece_floats;
#pragma unroll
        for (int c = 0; c < kCols; ++c) {
          float l[2], inv[2];
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            l[e] = __shfl_sync(0xffffffffu, zo[c][2 + e], t4);
            inv[e] = !whole ? 1.0f : l[e] == 0.0f ? 0.0f : 1.0f / l[e];
          }
          const int r = 8 * c + g, t = token_of(get.s.row0 + r);
          uint16_t* row = job.out.data + (get.s.q_first + t) * job.out.token + (get.h * job.group + get.s.row0 + r - t * job.group) * job.out.head;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            float v[2][4];                        // [row][channel 2 j + half]
#pragma unroll
            for (int e = 0; e < 2; ++e) {
              const float z = fmaf(-7.5f, __shfl_sync(0xffffffffu, zo[c][e], 4 * i + t4), __shfl_sync(0xffffffffu, zo[c][e], 4 * (4 + i) + t4));
              v[e][0] = fmaf(o[c][i][0][e], 16777216.0f, z) * inv[e];
              v[e][1] = fmaf(o[c][i][0][2 + e], 1048576.0f, z) * inv[e];
              v[e][2] = fmaf(o[c][i][1][e], 16777216.0f, z) * inv[e];
              v[e][3] = fmaf(o[c][i][1][2 + e], 1048576.0f, z) * inv[e];
            }
            if (whole) {
              uint32_t w[4];                      // lane (g, t4) then has row 8 c + g, channels 32 i + 8 t4 + k and + k + 4
#pragma unroll
              for (int k = 0; k < 4; ++k) w[k] = transpose8(float2_to_pair<BF16>(v[0][k], v[1][k]));
              if (r < get.s.rows)
                *reinterpret_cast<uint4*>(row + 32 * i + 8 * t4) = make_uint4(__byte_perm(w[0], w[1], 0x5410), __byte_perm(w[2], w[3], 0x5410),
                                                                            __byte_perm(w[0], w[1], 0x7632), __byte_perm(w[2], w[3], 0x7632));
            } else {
#pragma unroll
              for (int e = 0; e < 2; ++e)
                if (8 * c + 2 * t4 + e < piece_rows)
                  *reinterpret_cast<float4*>(dst + (8 * c + 2 * t4 + e) * kHeadDim + 32 * i + 4 * g) = make_float4(v[e][0], v[e][1], v[e][2], v[e][3]);
            }
          }
          if (!whole && g == 0)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              if (8 * c + 2 * t4 + e < piece_rows) *reinterpret_cast<float2*>(dst + piece_rows * kHeadDim + 2 * (8 * c + 2 * t4 + e)) = make_float2(m[c][e], l[e]);
        }
        if (!whole && lane == 0) {
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
      at += n_here + pair_cost(FORM);
      todo -= n_here + pair_cost(FORM);
      __syncwarp();
      if (todo > 0) {
        if (lane == 0) next_pair<FORM>(get, pv, opt, job);
        __syncwarp();
      }
    }
  }
  __syncthreads();
  if (*failed) {                                  // a copy did not come: what is still under way may land before the CTA leaves
    if (threadIdx.x == 0) paged_status(pv.status, MOQAE_ERR_TIMEOUT, static_cast<int>(blockIdx.x), -1);
    const long long since = clock64();
    while (clock64() - since < (1 << 20)) {
    }
    return;
  }

  auto piece_at = [&](int i) -> const float* {
    return (i & 1) ? reinterpret_cast<const float*>(smem + (i >> 1) * kStages * kStageBytes4) : head_piece + (i >> 1) * piece_floats;
  };
  join_pieces<BF16, FORM, kWarps>(job, part, desc, turn, piece_rows, piece_floats, warp, lane, piece_at);
}

size_t smem4(int form, int rows) {
  const int warps = warps_of(form), stages = stages4_of(form);
  return static_cast<size_t>(warps) * stages * (kStageBytes4 + 8) + static_cast<size_t>(warps) * piece_floats_of(rows) * 4 + 2 * warps * (sizeof(Piece) + sizeof(Cursor)) + 32;
}

template <bool BF16, int FORM, bool SHAPED> cudaError_t launch4(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, cudaStream_t st) {
  static_assert(stages4_of(FORM) * kStageBytes4 >= piece_floats_of(set_rows(FORM)) * 4, "a piece fits the ring");
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_shared_memory(paged4_decode_kernel<BF16, FORM, SHAPED>, smem4(FORM, FORM == kOne4Q ? 4 : set_rows(FORM)), done);
  if (e != cudaSuccess) return e;
  return launch_early(paged4_decode_kernel<BF16, FORM, SHAPED>, sm_count_of_current_device(), warps_of(FORM) * 32, smem4(FORM, FORM == kFew16Q ? 16 : job.group), st, pv, opt, job);
}

template <int FORM> cudaError_t launch_shaped4(const PagedView& pv, const AttnOptions& opt, const DecodeJob& job, cudaStream_t st) {
  const bool bf16 = pv.dtype == MOQAE_DTYPE_BF16;
  if (opt.cap > 0.0f || opt.slopes) return bf16 ? launch4<true, FORM, true>(pv, opt, job, st) : launch4<false, FORM, true>(pv, opt, job, st);
  return bf16 ? launch4<true, FORM, false>(pv, opt, job, st) : launch4<false, FORM, false>(pv, opt, job, st);
}

}  // namespace

bool paged4_decode_fits(const PagedView& pv) {
  return static_cast<long long>(pv.batch) * pv.n_kv_heads <= kWorkCounters && units_fit(pv, pv.batch, kOne8Q);
}

long long paged4_decode_workspace_bytes(int group) { return kWorkCounterBytes + part_bytes(group); }

cudaError_t launch_paged4_decode(const PagedView& pv, const RowsView& q, const RowsView& out, const AttnOptions& opt, void* workspace, cudaStream_t st) {
  if (pv.batch <= 0) return cudaSuccess;
  DecodeJob job{};
  job.q = q;
  job.out = out;
  job.group = q.n_heads / pv.n_kv_heads;
  job.arrived = static_cast<int*>(workspace);
  job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWorkCounterBytes);
  return job.group <= 4 ? launch_shaped4<kOne4Q>(pv, opt, job, st) : launch_shaped4<kOne8Q>(pv, opt, job, st);
}

// Several tokens per sequence by the same kernel, in sets of 16 rows.
bool paged4_few_fits(const PagedView& pv, int group, int n_tokens, int max_rows) {
  long long sets = few_sets(pv.batch, group, n_tokens);
  const long long most = static_cast<long long>(pv.batch) * ((max_rows + 15) / 16);
  if (max_rows > 0 && most < sets) sets = most;
  return sets * pv.n_kv_heads <= kWorkCounters && units_fit(pv, sets, kFew16Q);
}

long long paged4_few_workspace_bytes() { return kWorkCounterBytes + part_bytes(16); }

cudaError_t launch_paged4_few(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                              const AttnOptions& opt, void* workspace, int max_rows, cudaStream_t st) {
  if (pv.batch <= 0 || n_tokens <= 0) return cudaSuccess;
  DecodeJob job{};
  job.max_rows = max_rows;
  job.q = q;
  job.out = out;
  job.cu_q = cu_q;
  job.n_tokens = n_tokens;
  job.group = q.n_heads / pv.n_kv_heads;
  job.arrived = static_cast<int*>(workspace);
  job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kWorkCounterBytes);
  return launch_shaped4<kFew16Q>(pv, opt, job, st);
}

}  // namespace moqae
