// Per-head RMS norm and position rotation of query and key rows (moqae_norm_rope), and the same pass
// with the keys and values going to their pages (moqae_paged_append).
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
#include "paged.cuh"

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

template <bool BF16, bool PAGED>
__global__ void __launch_bounds__(kAppendWarps * 32) norm_rope_kernel(PagedView pv, RopeView rope, RowJob job) {
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
  if (r < n_rows) {                             // the first rows travel while the position is looked up
    const uint16_t* p = source(r);
    a = *reinterpret_cast<const uint4*>(p + 8 * u0);
    b = *reinterpret_cast<const uint4*>(p + 8 * u1);
  }

  const int pos = job.positions[t];
  if (pos < 0) return;
  if (rope.rot_dim > 0 && pos >= rope.n_positions) {
    if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_INVALID_ARG, t, pos);
    return;
  }
  uint16_t *k_dst = nullptr, *v_dst = nullptr;  // head 0 of the token's row in its page
  if (PAGED) {
    const int s = job.seq ? job.seq[t] : t;
    const int entry = pos >> pv.page_shift;
    const bool known = s >= 0 && s < pv.batch && entry < pv.max_pages;
    const int page = known ? pv.table[static_cast<long long>(s) * pv.max_pages + entry] : -1;
    if (page < 0 || page >= pv.n_pages) {
      if (part == 0 && lane == 0) paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, t, pos);
      return;
    }
    const int at = pos & (pv.page_size - 1);
    k_dst = pv.k + page * pv.k_page + at * pv.k_slot;
    v_dst = pv.v + page * pv.v_page + at * pv.v_slot;
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
    if (r + step < n_rows) {
      const uint16_t* p = source(r + step);
      a = *reinterpret_cast<const uint4*>(p + 8 * u0);
      b = *reinterpret_cast<const uint4*>(p + 8 * u1);
    }
    const bool is_q = r < job.q.n_heads, is_v = r >= n_qk;
    uint16_t* dst;
    if (is_q) dst = job.q_out.data + t * job.q_out.token + r * job.q_out.head;
    else if (!PAGED) dst = job.k_out.data + t * job.k_out.token + (r - job.q.n_heads) * job.k_out.head;
    else dst = is_v ? v_dst + (r - n_qk) * pv.v_head : k_dst + (r - job.q.n_heads) * pv.k_head;
    uint4 o0 = a0, o1 = b0;
    const uint16_t* weight = is_q ? rope.q_weight : rope.k_weight;
    if (!is_v && (weight || turn)) {            // otherwise the bits go through as they are
      float x[8], y[8];
      unpack8<BF16>(x, a0);
      unpack8<BF16>(y, b0);
      float sq = 0.0f;
#pragma unroll
      for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], fmaf(y[i], y[i], sq));
      const unsigned mask = 0xffu << (slot * kRowLanes);   // the eight lanes of a row always go the same way
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
      o0 = pack8<BF16>(x);
      o1 = pack8<BF16>(y);
    }
    if (r < n_rows) {
      *reinterpret_cast<uint4*>(dst + 8 * u0) = o0;
      *reinterpret_cast<uint4*>(dst + 8 * u1) = o1;
    }
  }
}

}  // namespace

template <bool PAGED>
static cudaError_t launch_rows(const PagedView& pv, const RopeView& rope, RowJob job, int dtype, cudaStream_t st) {
  const int n_rows = job.q.n_heads + job.k.n_heads + job.v.n_heads;
  if (job.n_tokens <= 0 || n_rows <= 0) return cudaSuccess;
  // Few tokens: several warps share one, until every SM has a few or every warp is down to one pass.
  const int wanted = sm_count_of_current_device() * 16;
  const int passes = (n_rows + kRowsPerPass - 1) / kRowsPerPass;
  job.parts_shift = 0;
  while ((1 << job.parts_shift) < passes && (static_cast<long long>(job.n_tokens) << job.parts_shift) < wanted) ++job.parts_shift;
  const long long warps = static_cast<long long>(job.n_tokens) << job.parts_shift;
  const unsigned grid = static_cast<unsigned>((warps + kAppendWarps - 1) / kAppendWarps);
  return launch_early(dtype == MOQAE_DTYPE_BF16 ? norm_rope_kernel<true, PAGED> : norm_rope_kernel<false, PAGED>, grid, kAppendWarps * 32, 0, st,
                      pv, rope, job);
}

cudaError_t launch_norm_rope(const RopeView& rope, int dtype, const RowsView& q, const RowsView& k, const RowsView& q_out,
                             const RowsView& k_out, const int32_t* positions, int n_tokens, int32_t* status, cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.q_out = q_out; job.k_out = k_out;
  job.positions = positions; job.status = status; job.n_tokens = n_tokens;
  return launch_rows<false>(PagedView{}, rope, job, dtype, st);
}

cudaError_t launch_paged_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out,
                                const RowsView& k, const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens,
                                cudaStream_t st) {
  RowJob job{};
  job.q = q; job.k = k; job.v = v; job.q_out = q_out;
  job.positions = positions; job.seq = seq; job.status = pv.status; job.n_tokens = n_tokens;
  return launch_rows<true>(pv, rope, job, pv.dtype, st);
}

}  // namespace moqae
