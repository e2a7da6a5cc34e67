// Per-head RMS norm and position rotation of query and key rows (moqae_norm_rope), and the same pass
// with the keys and values going to their pages (moqae_paged_append), there in 4 bits (moqae_paged4_append); and
// rows of 4-bit pages as the values they stand for (moqae_paged4_read).
//
// Mathematics, per row x of 128 channels: y = x * (mean(x^2) + eps)^(-1/2) * w, then every pair (a, b)
// of the rotated channels becomes (a cos - b sin, a sin + b cos).  One pass: every row is read and
// written once, the rounding to 16 bits happens at the store, so the kernel is bound by memory.
// Eight lanes own a row, two 16-byte units each, chosen so that both partners of every pair sit in
// one lane: units j and j + rot_dim / 16 when a pair is (i, i + rot_dim / 2), any two when it is (2 i, 2 i + 1).
// The rotation then needs no exchange, the mean three shuffles.  A warp handles four rows of one token
// at a time; the cosines and sines of its token stay in registers over all the heads it works on.
// Measured: 32719 tokens, 32 + 32 heads, fp16: 178 us for 1.09 GB, 6.1 TB/s (a plain copy reaches 6.5); appending 32622
// tokens of 7 prompts, 40 + 2 x 40 heads, to their pages: 328 us for 2.01 GB, 6.1 TB/s.  One token of 32 + 8 heads: 2.5 to
// 3.1 us, a launch: where tokens are few a warp takes four rows of one, so that nobody has a second turn to wait for.
//
// In 4 bits a group of 32 channels becomes z = the largest fp16 value not above its smallest element, s = the smallest not below
// (largest - z) / 15, and codes rint((x - z) r), r = 1 / s in float32, the product taken exactly (the rule of the quantised chunks, and their
// code: quant_encode.cuh).  With the directed roundings no code leaves 0 .. 15.  Keys are quantised as they leave the rotation, in
// float32.  A key's lane holds two units of 8 channels of any two groups, so extremes and parameters pass through 1 KiB of shared memory
// per warp; a value's lane takes four channels of each group, whose extremes meet in shuffles of packed 16-bit pairs, and stores 8 bytes.
#include "paged4.cuh"
#include "quant_encode.cuh"

namespace moqae {

namespace {

constexpr int kRowLanes = 8;                    // lanes per row
constexpr int kRowsPerPass = 32 / kRowLanes;    // rows a warp handles at a time
constexpr int kAppendWarps = 4;

struct RowJob {
  RowsView q, k, v, q_out, k_out;               // k_out: only without pages
  const int32_t* positions;
  const int32_t* seq;
  int32_t* status;
  int n_tokens, parts_shift;                    // 2^parts_shift warps share a token
};

template <bool BF16> __device__ __forceinline__ void unpack8(float (&x)[8], const uint4& u) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 f = pair_to_float2<BF16>(w[i]);
    x[2 * i] = f.x;
    x[2 * i + 1] = f.y;
  }
}
template <bool BF16> __device__ __forceinline__ uint4 pack8(const float (&x)[8]) {
  return make_uint4(float2_to_pair<BF16>(x[0], x[1]), float2_to_pair<BF16>(x[2], x[3]), float2_to_pair<BF16>(x[4], x[5]),
                    float2_to_pair<BF16>(x[6], x[7]));
}

// (x - zero) * inv as codes behind the bits of kMagic, two at a time: one packed addition, one packed fused multiply-add.
__device__ __forceinline__ void encode_two(float x0, float x1, uint64_t negz2, uint64_t inv2, uint32_t& u0, uint32_t& u1) {
  uint64_t d2, r2;
  asm("add.rn.f32x2 %0, %1, %2;\n" : "=l"(d2) : "l"(pack_f2(x0, x1)), "l"(negz2));
  asm("fma.rn.f32x2 %0, %1, %2, %3;\n" : "=l"(r2) : "l"(d2), "l"(inv2), "l"(pack_f2(kMagic, kMagic)));
  asm("mov.b64 {%0, %1}, %2;\n" : "=r"(u0), "=r"(u1) : "l"(r2));
}
// Eight codes, the first in the lowest bits.  (What stands above a code's four bits is a multiple of 2^22: it leaves the low 16.)
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float zero, float inv) {
  const uint64_t negz2 = pack_f2(-zero, -zero), inv2 = pack_f2(inv, inv);
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; i += 2) encode_two(x[i], x[i + 1], negz2, inv2, u[i], u[i + 1]);
  return __byte_perm(pack4<4>(u[0], u[1], u[2], u[3]), pack4<4>(u[4], u[5], u[6], u[7]), 0x5410);
}

// A key row of a 4-bit page: units u0 and u1 (8 channels each, float32) of lane `sub` of the row's eight lanes (`mask`).  `at`: the
// row's 256 bytes of shared memory.
__device__ __forceinline__ void put_key4(uint8_t* tile, int t, const float (&x)[8], const float (&y)[8], int u0, int u1, int sub, unsigned mask, float2* at) {
  float lo0 = x[0], hi0 = x[0], lo1 = y[0], hi1 = y[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo0 = fminf(lo0, x[i]);
    hi0 = fmaxf(hi0, x[i]);
    lo1 = fminf(lo1, y[i]);
    hi1 = fmaxf(hi1, y[i]);
  }
  at[u0] = make_float2(lo0, hi0);
  at[u1] = make_float2(lo1, hi1);
  __syncwarp(mask);
  const int g = sub >> 1;                        // two lanes work out the parameters of a group
  const float4 a = *reinterpret_cast<const float4*>(at + 4 * g), b = *reinterpret_cast<const float4*>(at + 4 * g + 2);
  uint16_t s_bits, z_bits;
  float zero, inv;
  group_params(fminf(fminf(a.x, a.z), fminf(b.x, b.z)), fmaxf(fmaxf(a.y, a.w), fmaxf(b.y, b.w)), 15.0f, s_bits, z_bits, zero, inv);
  reinterpret_cast<uint16_t*>(tile + kKeyMeta4 + 16 * t)[g + 4 * (sub & 1)] = (sub & 1) ? z_bits : s_bits;
  if ((sub & 1) == 0) at[16 + g] = make_float2(zero, inv);
  __syncwarp(mask);
  const float2 p0 = at[16 + (u0 >> 2)], p1 = at[16 + (u1 >> 2)];
  *reinterpret_cast<uint32_t*>(tile + 64 * t + 16 * (u0 & 3) + 4 * (u0 >> 2)) = codes8(x, p0.x, p0.y);
  *reinterpret_cast<uint32_t*>(tile + 64 * t + 16 * (u1 & 3) + 4 * (u1 >> 2)) = codes8(y, p1.x, p1.y);
  __syncwarp(mask);                              // the place is free for the next row
}

// A value row: w[g] are the 16-bit channels 32 g + 4 sub .. + 3.
template <bool BF16> __device__ __forceinline__ void put_value4(uint8_t* tile, int t, const uint2 (&w)[4], int sub, unsigned mask) {
  uint32_t ext[4];                               // smallest element low, largest high
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const uint32_t lo = min2<BF16>(w[g].x, w[g].y), hi = max2<BF16>(w[g].x, w[g].y);
    const uint32_t l = min2<BF16>(lo, lo >> 16), h = max2<BF16>(hi, hi >> 16);    // (the upper halves do not count)
    ext[g] = __byte_perm(l, h, 0x5410);
  }
#pragma unroll
  for (int o = 1; o < kRowLanes; o <<= 1)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint32_t other = __shfl_xor_sync(mask, ext[g], o);
      ext[g] = __byte_perm(min2<BF16>(ext[g], other), max2<BF16>(ext[g], other), 0x7610);
    }
  const int mine = sub >> 1;
  const uint32_t e = mine == 0 ? ext[0] : mine == 1 ? ext[1] : mine == 2 ? ext[2] : ext[3];
  uint16_t s_bits, z_bits;
  float zero, inv;
  group_params(lo_f<BF16>(e), hi_f<BF16>(e), 15.0f, s_bits, z_bits, zero, inv);
  reinterpret_cast<uint16_t*>(tile + kValueMeta4 + 32 * (t >> 1))[2 * mine + (t & 1) + 8 * (sub & 1)] = (sub & 1) ? z_bits : s_bits;
  uint32_t half[4];                              // four codes of a group
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const float z = __shfl_sync(mask, zero, 2 * g, kRowLanes), r = __shfl_sync(mask, inv, 2 * g, kRowLanes);
    uint32_t u[4];
    encode2<BF16>(w[g].x, pack_f2(-z, -z), pack_f2(r, r), u[0], u[1]);
    encode2<BF16>(w[g].y, pack_f2(-z, -z), pack_f2(r, r), u[2], u[3]);
    half[g] = pack4<4>(u[0], u[1], u[2], u[3]);
  }
  *reinterpret_cast<uint2*>(tile + kValueCodes4 + 512 * (sub >> 2) + 32 * value_row4(t) + 8 * (sub & 3)) =
      make_uint2(__byte_perm(half[0], half[1], 0x5410), __byte_perm(half[2], half[3], 0x5410));
}

// Where the rows go: to rows, to 16-bit pages, to 4-bit pages.
enum { kToRows, kToPages, kToPages4 };

template <bool BF16, int DEST>
__global__ void __launch_bounds__(kAppendWarps * 32, DEST == kToPages4 ? 6 : 1) norm_rope_kernel(PagedView pv, RopeView rope, RowJob job) {
  constexpr bool PAGED = DEST != kToRows, FOUR = DEST == kToPages4;
  __shared__ __align__(16) float2 exchange[FOUR ? kAppendWarps * kRowsPerPass * 20 : 1];        // units' extremes, groups' parameters of a key row
  after_previous();
  const int lane = threadIdx.x & 31, sub = lane & (kRowLanes - 1), slot = lane / kRowLanes;
  const long long w = static_cast<long long>(blockIdx.x) * kAppendWarps + (threadIdx.x >> 5);
  const int t = static_cast<int>(w >> job.parts_shift), part = static_cast<int>(w) & ((1 << job.parts_shift) - 1);
  if (t >= job.n_tokens) return;
  const int step = kRowsPerPass << job.parts_shift;
  const int n_qk = job.q.n_heads + job.k.n_heads, n_rows = n_qk + job.v.n_heads;

  // the two 16-byte units of this lane, and which of them are rotated
  const int pairs = rope.rot_dim / 16;
  int u0 = sub, u1 = sub + 8;
  bool r0, r1;
  if (rope.interleaved) {
    r0 = u0 < 2 * pairs;
    r1 = u1 < 2 * pairs;
  } else {
    r0 = r1 = sub < pairs;
    u0 = r0 ? sub : 2 * sub;                    // 2 * pairs + 2 * (sub - pairs)
    u1 = r0 ? sub + pairs : 2 * sub + 1;
  }

  auto source = [&](int r) -> const uint16_t* {
    const RowsView& s = r < job.q.n_heads ? job.q : (r < n_qk ? job.k : job.v);
    const int h = r < job.q.n_heads ? r : (r < n_qk ? r - job.q.n_heads : r - n_qk);
    return s.data + t * s.token + h * s.head;
  };
  int r = part * kRowsPerPass + slot;
  uint4 a = make_uint4(0, 0, 0, 0), b = a;
  auto load = [&](int r) {
    const uint16_t* p = source(r);
    if (FOUR && r >= n_qk) {                    // values: four channels of each group
      const uint2 x = *reinterpret_cast<const uint2*>(p + 4 * sub), y = *reinterpret_cast<const uint2*>(p + 32 + 4 * sub);
      const uint2 z = *reinterpret_cast<const uint2*>(p + 64 + 4 * sub), w = *reinterpret_cast<const uint2*>(p + 96 + 4 * sub);
      a = make_uint4(x.x, x.y, y.x, y.y);
      b = make_uint4(z.x, z.y, w.x, w.y);
    } else {
      a = *reinterpret_cast<const uint4*>(p + 8 * u0);
      b = *reinterpret_cast<const uint4*>(p + 8 * u1);
    }
  };
  if (r < n_rows) load(r);                      // the first rows travel while the position is looked up

  const int pos = job.positions[t];
  if (pos < 0) return;
  if (rope.rot_dim > 0 && pos >= rope.n_positions) {
    if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_INVALID_ARG, t, pos);
    return;
  }
  uint16_t *k_dst = nullptr, *v_dst = nullptr;  // head 0 of the token's row in its page (of its tile)
  int slot_at = 0;
  if (PAGED) {
    const int s = job.seq ? job.seq[t] : t;
    const int entry = pos >> pv.page_shift;
    const bool known = s >= 0 && s < pv.batch && entry < pv.max_pages;
    const int page = known ? pv.table[static_cast<long long>(s) * pv.max_pages + entry] : -1;
    if (page < 0 || page >= pv.n_pages) {
      if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, t, pos);
      return;
    }
    const int at = slot_at = pos & (pv.page_size - 1);
    k_dst = FOUR ? reinterpret_cast<uint16_t*>(tile4(pv, page, 0, at)) : pv.k + page * pv.k_page + at * pv.k_slot;
    if (!FOUR) v_dst = pv.v + page * pv.v_page + at * pv.v_slot;
  }

  float c[8], s[8];
  const bool turn = r0 || r1;
  if (turn) {
    const float* row = rope.cos_sin + static_cast<long long>(pos) * rope.rot_dim;
    const int half = rope.rot_dim / 2;
    // halves: angles 8 sub .. 8 sub + 7; neighbours: 4 u0 .. 4 u0 + 3 and 4 u1 .. 4 u1 + 3
    const int f0 = rope.interleaved ? (r0 ? 4 * u0 : 0) : 8 * sub, f1 = rope.interleaved ? (r1 ? 4 * u1 : 0) : 8 * sub + 4;
    const float4 c0 = *reinterpret_cast<const float4*>(row + f0), c1 = *reinterpret_cast<const float4*>(row + f1);
    const float4 s0 = *reinterpret_cast<const float4*>(row + half + f0), s1 = *reinterpret_cast<const float4*>(row + half + f1);
    c[0] = c0.x; c[1] = c0.y; c[2] = c0.z; c[3] = c0.w; c[4] = c1.x; c[5] = c1.y; c[6] = c1.z; c[7] = c1.w;
    s[0] = s0.x; s[1] = s0.y; s[2] = s0.z; s[3] = s0.w; s[4] = s1.x; s[5] = s1.y; s[6] = s1.z; s[7] = s1.w;
  }

  // the loop count is the same for all lanes, so the shuffles are met by the whole warp
  for (int r_first = part * kRowsPerPass; r_first < n_rows; r_first += step, r += step) {
    const uint4 a0 = a, b0 = b;
    if (r + step < n_rows) load(r + step);
    const bool is_q = r < job.q.n_heads, is_v = r >= n_qk;
    const unsigned mask = 0xffu << (slot * kRowLanes);     // the eight lanes of a row always go the same way
    if (FOUR && is_v) {
      if (r < n_rows) {
        const uint2 w[4] = {make_uint2(a0.x, a0.y), make_uint2(a0.z, a0.w), make_uint2(b0.x, b0.y), make_uint2(b0.z, b0.w)};
        put_value4<BF16>(reinterpret_cast<uint8_t*>(k_dst) + (r - n_qk) * pv.k_head, slot_at & 15, w, sub, mask);
      }
      continue;
    }
    const bool to_codes = FOUR && !is_q;
    uint16_t* dst;
    if (is_q) dst = job.q_out.data + t * job.q_out.token + r * job.q_out.head;
    else if (!PAGED) dst = job.k_out.data + t * job.k_out.token + (r - job.q.n_heads) * job.k_out.head;
    else dst = is_v ? v_dst + (r - n_qk) * pv.v_head : k_dst + (r - job.q.n_heads) * pv.k_head;
    uint4 o0 = a0, o1 = b0;
    const uint16_t* weight = is_q ? rope.q_weight : rope.k_weight;
    if (!is_v && (weight || turn || to_codes)) {            // otherwise the bits go through as they are
      float x[8], y[8];
      unpack8<BF16>(x, a0);
      unpack8<BF16>(y, b0);
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], fmaf(y[i], y[i], sq));
      if (weight) {
#pragma unroll
        for (int o = 1; o < kRowLanes; o <<= 1) sq += __shfl_xor_sync(mask, sq, o);
        const float inv = 1.0f / sqrtf(sq * (1.0f / kHeadDim) + rope.eps);
        float wx[8], wy[8];
        unpack8<BF16>(wx, *reinterpret_cast<const uint4*>(weight + 8 * u0));
        unpack8<BF16>(wy, *reinterpret_cast<const uint4*>(weight + 8 * u1));
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          x[i] = x[i] * inv * wx[i];
          y[i] = y[i] * inv * wy[i];
        }
      }
      if (turn && !rope.interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float p0 = x[i], p1 = y[i];
          x[i] = fmaf(p0, c[i], -p1 * s[i]);
          y[i] = fmaf(p0, s[i], p1 * c[i]);
        }
      } else if (turn) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p0 = x[2 * i], p1 = x[2 * i + 1], e0 = y[2 * i], e1 = y[2 * i + 1];
          if (r0) {
            x[2 * i] = fmaf(p0, c[i], -p1 * s[i]);
            x[2 * i + 1] = fmaf(p0, s[i], p1 * c[i]);
          }
          if (r1) {
            y[2 * i] = fmaf(e0, c[4 + i], -e1 * s[4 + i]);
            y[2 * i + 1] = fmaf(e0, s[4 + i], e1 * c[4 + i]);
          }
        }
      }
      if (to_codes) {
        if (r < n_rows)
          put_key4(reinterpret_cast<uint8_t*>(k_dst) + (r - job.q.n_heads) * pv.k_head, slot_at & 15, x, y, u0, u1, sub, mask,
                   exchange + ((threadIdx.x >> 5) * kRowsPerPass + slot) * 20);
        continue;
      }
      o0 = pack8<BF16>(x);
      o1 = pack8<BF16>(y);
    }
    if (r < n_rows) {
      *reinterpret_cast<uint4*>(dst + 8 * u0) = o0;
      *reinterpret_cast<uint4*>(dst + 8 * u1) = o1;
    }
  }
}

// Rows of 4-bit pages as the 16-bit values nearest to what they stand for.  Eight lanes a row again: of a key a lane takes two units of 8
// channels, of a value four channels of each group.
template <bool BF16> __global__ void __launch_bounds__(kAppendWarps * 32) paged4_read_kernel(PagedView pv, RowJob job, RowsView v_out) {
  after_previous();
  const int lane = threadIdx.x & 31, sub = lane & (kRowLanes - 1), slot = lane / kRowLanes;
  const long long w = static_cast<long long>(blockIdx.x) * kAppendWarps + (threadIdx.x >> 5);
  const int t = static_cast<int>(w >> job.parts_shift), part = static_cast<int>(w) & ((1 << job.parts_shift) - 1);
  if (t >= job.n_tokens) return;
  const int pos = job.positions[t];
  if (pos < 0) return;
  const int s = job.seq ? job.seq[t] : t, entry = pos >> pv.page_shift;
  const bool known = s >= 0 && s < pv.batch && entry < pv.max_pages;
  const int page = known ? pv.table[static_cast<long long>(s) * pv.max_pages + entry] : -1;
  if (page < 0 || page >= pv.n_pages) {
    if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, t, pos);
    return;
  }
  const int at = pos & (pv.page_size - 1), tt = at & 15;
  const int n_k = job.k_out.n_heads, n_rows = n_k + v_out.n_heads;
  for (int r = part * kRowsPerPass + slot; r < n_rows; r += kRowsPerPass << job.parts_shift) {
    const bool is_v = r >= n_k;
    const int h = is_v ? r - n_k : r;
    const uint8_t* tile = tile4(pv, page, h, at);
    if (!is_v) {
      const uint4 meta = *reinterpret_cast<const uint4*>(tile + kKeyMeta4 + 16 * tt);
      uint16_t* dst = job.k_out.data + t * job.k_out.token + h * job.k_out.head;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = sub + 8 * i, g = u >> 2;
        const uint32_t code = *reinterpret_cast<const uint32_t*>(tile + 64 * tt + 16 * (u & 3) + 4 * g);
        const uint32_t s2 = i ? meta.y : meta.x, z2 = i ? meta.w : meta.z;
        const float sc = (g & 1) ? hi_f<false>(s2) : lo_f<false>(s2), z = (g & 1) ? hi_f<false>(z2) : lo_f<false>(z2);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(sc, static_cast<float>((code >> (4 * e)) & 15u), z);
        *reinterpret_cast<uint4*>(dst + 8 * u) = pack8<BF16>(x);
      }
    } else {
      const uint2 code = *reinterpret_cast<const uint2*>(tile + kValueCodes4 + 512 * (sub >> 2) + 32 * value_row4(tt) + 8 * (sub & 3));
      const uint4 s4 = *reinterpret_cast<const uint4*>(tile + kValueMeta4 + 32 * (tt >> 1)), z4 = *reinterpret_cast<const uint4*>(tile + kValueMeta4 + 32 * (tt >> 1) + 16);
      const uint32_t sw[4] = {s4.x, s4.y, s4.z, s4.w}, zw[4] = {z4.x, z4.y, z4.z, z4.w};
      uint16_t* dst = v_out.data + t * v_out.token + h * v_out.head;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const float sc = (tt & 1) ? hi_f<false>(sw[g]) : lo_f<false>(sw[g]), z = (tt & 1) ? hi_f<false>(zw[g]) : lo_f<false>(zw[g]);
        const uint32_t c = (g & 2 ? code.y : code.x) >> (16 * (g & 1));
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(sc, static_cast<float>((c >> (4 * e)) & 15u), z);
        *reinterpret_cast<uint2*>(dst + 32 * g + 4 * sub) = make_uint2(float2_to_pair<BF16>(x[0], x[1]), float2_to_pair<BF16>(x[2], x[3]));
      }
    }
  }
}

// Few tokens: several warps share one, until every SM has a few or every warp is down to one pass.
unsigned share_rows(RowJob& job, int n_rows) {
  const int wanted = sm_count_of_current_device() * 16;
  const int passes = (n_rows + kRowsPerPass - 1) / kRowsPerPass;
  job.parts_shift = 0;
  while ((1 << job.parts_shift) < passes && (static_cast<long long>(job.n_tokens) << job.parts_shift) < wanted) ++job.parts_shift;
  const long long warps = static_cast<long long>(job.n_tokens) << job.parts_shift;
  return static_cast<unsigned>((warps + kAppendWarps - 1) / kAppendWarps);
}

}  // namespace

template <int DEST>
static cudaError_t launch_rows(const PagedView& pv, const RopeView& rope, RowJob job, int dtype, cudaStream_t st) {
  const int n_rows = job.q.n_heads + job.k.n_heads + job.v.n_heads;
  if (job.n_tokens <= 0 || n_rows <= 0) return cudaSuccess;
  const unsigned grid = share_rows(job, n_rows);
  return launch_early(dtype == MOQAE_DTYPE_BF16 ? norm_rope_kernel<true, DEST> : norm_rope_kernel<false, DEST>, grid, kAppendWarps * 32, 0, st,
                      pv, rope, job);
}

cudaError_t launch_norm_rope(const RopeView& rope, int dtype, const RowsView& q, const RowsView& k, const RowsView& q_out,
                             const RowsView& k_out, const int32_t* positions, int n_tokens, int32_t* status, cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.q_out = q_out; job.k_out = k_out;
  job.positions = positions; job.status = status; job.n_tokens = n_tokens;
  return launch_rows<kToRows>(PagedView{}, rope, job, dtype, st);
}

cudaError_t launch_paged_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out,
                                const RowsView& k, const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens,
                                cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.v = v; job.q_out = q_out;
  job.positions = positions; job.seq = seq; job.status = pv.status; job.n_tokens = n_tokens;
  return launch_rows<kToPages>(pv, rope, job, pv.dtype, st);
}

cudaError_t launch_paged4_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out, const RowsView& k,
                                 const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens, cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.v = v; job.q_out = q_out;
  job.positions = positions; job.seq = seq; job.status = pv.status; job.n_tokens = n_tokens;
  return launch_rows<kToPages4>(pv, rope, job, pv.dtype, st);
}

cudaError_t launch_paged4_read(const PagedView& pv, const RowsView& k_out, const RowsView& v_out, const int32_t* positions, const int32_t* seq,
                               int n_tokens, cudaStream_t st) {
  RowJob job{};
  job.k_out = k_out;
  job.positions = positions; job.seq = seq; job.status = pv.status; job.n_tokens = n_tokens;
  const int n_rows = k_out.n_heads + v_out.n_heads;
  if (n_tokens <= 0 || n_rows <= 0) return cudaSuccess;
  const unsigned grid = share_rows(job, n_rows);
  return launch_early(pv.dtype == MOQAE_DTYPE_BF16 ? paged4_read_kernel<true> : paged4_read_kernel<false>, grid, kAppendWarps * 32, 0, st, pv, job, v_out);
}

}  // namespace moqae
