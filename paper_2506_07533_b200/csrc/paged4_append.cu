// Norm, rotation and quantisation of new tokens into 4-bit pages (moqae_paged4_append), and rows of 4-bit pages as the values they
// stand for (moqae_paged4_read).
//
// Mathematics.  A group of 32 channels becomes z = the largest fp16 value not above its smallest element, s = the smallest not below (largest - z) / 15,
// and codes rint((x - z) r), r = 1 / s in float32, the product taken exactly (the rule of the quantised chunks, and their code: quant_encode.cuh).
// With the directed roundings no code leaves 0 .. 15.  Keys are quantised as they leave the rotation, in float32.
//   A warp takes four heads of one token at a time, all queries, all keys or all values, eight lanes a row (paged_rows.cuh), so nothing in a pass
//   depends on the kind of its rows.  A key's lane holds two units of 8 channels of any two groups: extremes and parameters pass through shared memory.  A
//   value's lane takes 16 neighbouring channels, so that a group is two lanes; its codes change places in shared memory to leave 8 bytes at a
//   time.  A value is stored as two whole sectors, a key as two, each with 16 bytes of scales and zeros, which fill up with the neighbours' in L2.
//   Measured: 12233 tokens of 7 prompts, 40 + 2 x 40 heads, fp16: 116 us for 579 MB, 5.0 TB/s (88 us at the rate of a copy); issue slots are 63 % busy with 32
//   warps on an SM, which 64 registers a thread allow, with 20 to 36 bytes spilled (72: 123 us, 80: 139, 56: 141, with more).  Reading the same rows back: 66 us for 329 MB.
//   One token of 61 sequences: 3.1 and 1.9 us.
#include "paged4.cuh"
#include "paged_rows.cuh"
#include "quant_encode.cuh"

namespace moqae {

namespace {

// Eight codes, the first in the lowest bits: (x - zero) * inv behind the bits of kMagic.  (What stands above a code's four bits is a multiple of
// 2^22: it leaves the low 16.)
__device__ __forceinline__ uint32_t codes8(const float (&x)[8], float zero, float inv) {
  uint32_t u[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) u[i] = __float_as_uint(__fmaf_rn(__fsub_rn(x[i], zero), inv, kMagic));
  return __byte_perm(pack4<4>(u[0], u[1], u[2], u[3]), pack4<4>(u[4], u[5], u[6], u[7]), 0x5410);
}

// z, s and r = 1 / s of a group from its extremes.  s: the smallest fp16 value with 15 s >= max - z.  (That is the smallest not below the float32 quotient
// too: 15 s has 15 bits, so where the exact quotient passes an fp16 value it does so by a fifteenth of a float32 step of max - z, more than the half step
// that rounding could take away.)  A product a little below the quotient finds it, or the value before it.
__device__ __forceinline__ void params4(float mn, float mx, uint16_t& s_bits, uint16_t& z_bits, float& zero, float& inv) {
  z_bits = __half_as_ushort(__float2half_rd(mn));
  if (z_bits == 0x8000u) z_bits = 0;             // -0 is stored as +0
  zero = __half2float(__ushort_as_half(z_bits));
  const float span = __fsub_rn(mx, zero);
  s_bits = __half_as_ushort(__float2half_ru(__fmul_rn(span, 0.06666660f)));
  if (__fmul_rn(__half2float(__ushort_as_half(s_bits)), 15.0f) < span) ++s_bits;
  const float scale = __half2float(__ushort_as_half(s_bits));
  inv = scale == 0.0f ? 0.0f : __frcp_rn(scale);
}

// A key row: units w.u0 and w.u1 (float32).  at: 160 bytes of shared memory of the row; act: the row exists.
__device__ __forceinline__ void put_key4(uint8_t* tile, int t, const float (&x)[8], const float (&y)[8], const RowTurn& w, int sub, bool act, float2* at) {
  float lo0 = x[0], hi0 = x[0], lo1 = y[0], hi1 = y[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo0 = fminf(lo0, x[i]);
    hi0 = fmaxf(hi0, x[i]);
    lo1 = fminf(lo1, y[i]);
    hi1 = fmaxf(hi1, y[i]);
  }
  __syncwarp();                                  // the place is free
  at[w.u0] = make_float2(lo0, hi0);
  at[w.u1] = make_float2(lo1, hi1);
  __syncwarp();
  const int g = sub >> 1;                        // two lanes work out the parameters of a group
  const float4 a = *reinterpret_cast<const float4*>(at + 4 * g), b = *reinterpret_cast<const float4*>(at + 4 * g + 2);
  uint16_t s_bits, z_bits;
  float zero, inv;
  params4(fminf(fminf(a.x, a.z), fminf(b.x, b.z)), fmaxf(fmaxf(a.y, a.w), fmaxf(b.y, b.w)), s_bits, z_bits, zero, inv);
  if (act) reinterpret_cast<uint16_t*>(tile + kKeyMeta4 + 16 * t)[g + 4 * (sub & 1)] = (sub & 1) ? z_bits : s_bits;
  if ((sub & 1) == 0) at[16 + g] = make_float2(zero, inv);
  __syncwarp();
  const float2 p0 = at[16 + (w.u0 >> 2)], p1 = at[16 + (w.u1 >> 2)];
  const uint32_t c0 = codes8(x, p0.x, p0.y), c1 = codes8(y, p1.x, p1.y);
  if (act) {
    *reinterpret_cast<uint32_t*>(tile + 64 * t + 16 * (w.u0 & 3) + 4 * (w.u0 >> 2)) = c0;
    *reinterpret_cast<uint32_t*>(tile + 64 * t + 16 * (w.u1 & 3) + 4 * (w.u1 >> 2)) = c1;
  }
}

// A value row: a, b are the 16-bit channels 16 sub .. + 15.
template <bool BF16, typename F>
__device__ __forceinline__ void put_value4(uint8_t* tile, int t, const uint4& a, const uint4& b, int sub, bool act, uint16_t* at, F then_load) {
  const uint32_t v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  uint32_t lo = v[0], hi = v[0];
#pragma unroll
  for (int i = 1; i < 8; ++i) {
    lo = min2<BF16>(lo, v[i]);
    hi = max2<BF16>(hi, v[i]);
  }
  uint32_t ext = __byte_perm(min2<BF16>(lo, lo >> 16), max2<BF16>(hi, hi >> 16), 0x5410);   // smallest element low, largest high
  const uint32_t other = __shfl_xor_sync(0xffffffffu, ext, 1);
  ext = __byte_perm(min2<BF16>(ext, other), max2<BF16>(ext, other), 0x7610);
  const int g = sub >> 1, half = sub & 1;
  uint16_t s_bits, z_bits;
  float zero, inv;
  params4(lo_f<BF16>(ext), hi_f<BF16>(ext), s_bits, z_bits, zero, inv);
  if (act) reinterpret_cast<uint16_t*>(tile + kValueMeta4 + 32 * (t >> 1))[2 * g + (t & 1) + 8 * half] = half ? z_bits : s_bits;
  const uint64_t negz2 = pack_f2(-zero, -zero), inv2 = pack_f2(inv, inv);
  __syncwarp();                                  // the place is free
#pragma unroll
  for (int i = 0; i < 4; ++i) {                  // channels 4 i .. + 3 of the lane: unit 4 half + i, halfword g
    uint32_t u[4];
    encode2<BF16>(v[2 * i], negz2, inv2, u[0], u[1]);
    encode2<BF16>(v[2 * i + 1], negz2, inv2, u[2], u[3]);
    at[4 * (4 * half + i) + g] = static_cast<uint16_t>(pack4<4>(u[0], u[1], u[2], u[3]));
  }
  then_load();                                   // a and b have been read
  __syncwarp();
  if (act) *reinterpret_cast<uint2*>(tile + kValueCodes4 + 512 * (sub >> 2) + 32 * value_row4(t) + 8 * (sub & 3)) = *reinterpret_cast<const uint2*>(at + 4 * sub);
}

template <bool BF16> __global__ void __launch_bounds__(kAppendWarps * 32, 8) append4_kernel(PagedView pv, RopeView rope, RowJob job) {
  __shared__ __align__(16) float2 exchange[kAppendWarps * kRowsPerPass][20];      // units' extremes and groups' parameters of a key row; codes of a value row
  after_previous();
  const int lane = threadIdx.x & 31, sub = lane & (kRowLanes - 1), slot = lane / kRowLanes;
  const long long id = static_cast<long long>(blockIdx.x) * kAppendWarps + (threadIdx.x >> 5);
  const int t = static_cast<int>(id >> job.parts_shift), part = static_cast<int>(id) & ((1 << job.parts_shift) - 1);
  if (t >= job.n_tokens) return;
  RowTurn w;
  row_units(w, rope, sub);
  const int q_passes = (job.q.n_heads + kRowsPerPass - 1) / kRowsPerPass, kv_passes = (job.k.n_heads + kRowsPerPass - 1) / kRowsPerPass;
  const int k_end = q_passes + kv_passes, passes = k_end + kv_passes, step = 1 << job.parts_shift;
  const uint8_t* src = nullptr;                  // the lane's row of the pass that is loaded
  uint4 a = make_uint4(0, 0, 0, 0), b = a;
  const int c0 = 16 * w.u0, c1 = 16 * w.u1;      // its bytes of a query or key
  auto byte_step = [&](const RowsView& r) { return 2ll * kRowsPerPass * r.head << job.parts_shift; };
  // load of pass p, the first of its kind; of the next pass of a kind
  auto load_first = [&](int p) {
    const RowsView& r = p < q_passes ? job.q : p < k_end ? job.k : job.v;
    const int h = (p - (p < q_passes ? 0 : p < k_end ? q_passes : k_end)) * kRowsPerPass + slot;
    src = reinterpret_cast<const uint8_t*>(r.data + t * r.token + h * r.head);
    if (p < passes && h < r.n_heads) {
      a = *reinterpret_cast<const uint4*>(src + (p < k_end ? c0 : 32 * sub));
      b = *reinterpret_cast<const uint4*>(src + (p < k_end ? c1 : 32 * sub + 16));
    }
  };
  auto load_next = [&](long long by, bool act, int at0, int at1) {
    src += by;
    if (act) {
      a = *reinterpret_cast<const uint4*>(src + at0);
      b = *reinterpret_cast<const uint4*>(src + at1);
    }
  };
  load_first(part);                              // the first rows travel while the position is looked up

  const int pos = job.positions[t];
  if (pos < 0) return;
  if (rope.rot_dim > 0 && pos >= rope.n_positions) {
    if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_INVALID_ARG, t, pos);
    return;
  }
  const int s = job.seq ? job.seq[t] : t, entry = pos >> pv.page_shift;
  const bool known = s >= 0 && s < pv.batch && entry < pv.max_pages;
  const int page = known ? pv.table[static_cast<long long>(s) * pv.max_pages + entry] : -1;
  if (page < 0 || page >= pv.n_pages) {
    if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, t, pos);
    return;
  }
  uint8_t* tile = tile4(pv, page, 0, pos & (pv.page_size - 1));
  const int at = pos & (kTileTokens4 - 1);
  row_angles(w, rope, pos, sub);
  float2* place = exchange[(threadIdx.x >> 5) * kRowsPerPass + slot];
  const long long tile_step = (kRowsPerPass * pv.k_head) << job.parts_shift;
  const int h_step = kRowsPerPass << job.parts_shift;
  int p = part, h = p * kRowsPerPass + slot;
  if (p < q_passes) {
    const long long in_step = byte_step(job.q), out_step = byte_step(job.q_out);
    uint8_t* dst = reinterpret_cast<uint8_t*>(job.q_out.data + t * job.q_out.token + h * job.q_out.head);
    for (; p < q_passes; p += step, h += h_step, dst += out_step) {
      uint4 o0 = a, o1 = b;                      // without norm and rotation the bits go through as they are
      float x[8], y[8];
      unpack8<BF16>(x, a);
      unpack8<BF16>(y, b);
      if (p + step < q_passes) load_next(in_step, h + h_step < job.q.n_heads, c0, c1);
      else load_first(p + step);
      if (rope.q_weight || w.turn) {
        turn_row<BF16>(x, y, rope.q_weight, w, rope, 0xffffffffu);
        o0 = pack8<BF16>(x);
        o1 = pack8<BF16>(y);
      }
      if (h < job.q.n_heads) {
        *reinterpret_cast<uint4*>(dst + c0) = o0;
        *reinterpret_cast<uint4*>(dst + c1) = o1;
      }
    }
  }
  if (p < k_end) {
    const long long in_step = byte_step(job.k);
    h = (p - q_passes) * kRowsPerPass + slot;
    uint8_t* out = tile + h * pv.k_head;
    for (; p < k_end; p += step, h += h_step, out += tile_step) {
      float x[8], y[8];
      unpack8<BF16>(x, a);
      unpack8<BF16>(y, b);
      if (p + step < k_end) load_next(in_step, h + h_step < job.k.n_heads, c0, c1);
      else load_first(p + step);
      turn_row<BF16>(x, y, rope.k_weight, w, rope, 0xffffffffu);
      put_key4(out, at, x, y, w, sub, h < job.k.n_heads, place);
    }
  }
  const long long in_step = byte_step(job.v);
  h = (p - k_end) * kRowsPerPass + slot;
  uint8_t* out = tile + h * pv.k_head;
  for (; p < passes; p += step, h += h_step, out += tile_step) {
    put_value4<BF16>(out, at, a, b, sub, h < job.v.n_heads, reinterpret_cast<uint16_t*>(place), [&]() {
      if (p + step < passes) load_next(in_step, h + h_step < job.v.n_heads, 32 * sub, 32 * sub + 16);
    });
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
      const uint4 meta = __ldg(reinterpret_cast<const uint4*>(tile + kKeyMeta4 + 16 * tt));
      uint16_t* dst = job.k_out.data + t * job.k_out.token + h * job.k_out.head;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int u = sub + 8 * i, g = u >> 2;
        const uint32_t code = __ldg(reinterpret_cast<const uint32_t*>(tile + 64 * tt + 16 * (u & 3) + 4 * g));
        const uint32_t s2 = i ? meta.y : meta.x, z2 = i ? meta.w : meta.z;
        const float sc = (g & 1) ? hi_f<false>(s2) : lo_f<false>(s2), z = (g & 1) ? hi_f<false>(z2) : lo_f<false>(z2);
        float x[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = fmaf(sc, static_cast<float>((code >> (4 * e)) & 15u), z);
        *reinterpret_cast<uint4*>(dst + 8 * u) = pack8<BF16>(x);
      }
    } else {
      const uint2 code = __ldg(reinterpret_cast<const uint2*>(tile + kValueCodes4 + 512 * (sub >> 2) + 32 * value_row4(tt) + 8 * (sub & 3)));
      const uint4 s4 = __ldg(reinterpret_cast<const uint4*>(tile + kValueMeta4 + 32 * (tt >> 1))), z4 = __ldg(reinterpret_cast<const uint4*>(tile + kValueMeta4 + 32 * (tt >> 1) + 16));
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

}  // namespace

cudaError_t launch_paged4_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out, const RowsView& k,
                                 const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens, cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.v = v; job.q_out = q_out;
  job.positions = positions; job.seq = seq; job.status = pv.status; job.n_tokens = n_tokens;
  if (n_tokens <= 0) return cudaSuccess;
  auto whole = [](int heads) { return (heads + kRowsPerPass - 1) / kRowsPerPass * kRowsPerPass; };
  const unsigned grid = share_rows(job, whole(q.n_heads) + 2 * whole(k.n_heads));
  return launch_early(pv.dtype == MOQAE_DTYPE_BF16 ? append4_kernel<true> : append4_kernel<false>, grid, kAppendWarps * 32, 0, st, pv, rope, job);
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
