// What the kernels that norm, rotate and store rows share (16-bit rows and pages: paged_append.cu, 4-bit pages: paged4_append.cu): eight lanes
// per row, two units of 8 channels each, so that both partners of every rotated pair sit in one lane (see paged_append.cu).
#pragma once

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

// The two units of lane `sub` of a row, which of them are rotated, and the cosines and sines of their angles at a position.
struct RowTurn {
  int u0, u1;
  bool r0, r1, turn;
  float c[8], s[8];
};
__device__ __forceinline__ void row_units(RowTurn& w, const RopeView& rope, int sub) {
  const int pairs = rope.rot_dim / 16;
  w.u0 = sub;
  w.u1 = sub + 8;
  if (rope.interleaved) {
    w.r0 = w.u0 < 2 * pairs;
    w.r1 = w.u1 < 2 * pairs;
  } else {
    w.r0 = w.r1 = sub < pairs;
    w.u0 = w.r0 ? sub : 2 * sub;                    // 2 * pairs + 2 * (sub - pairs)
    w.u1 = w.r0 ? sub + pairs : 2 * sub + 1;
  }
  w.turn = w.r0 || w.r1;
}
__device__ __forceinline__ void row_angles(RowTurn& w, const RopeView& rope, int pos, int sub) {
  if (!w.turn) return;
  const float* row = rope.cos_sin + static_cast<long long>(pos) * rope.rot_dim;
  const int half = rope.rot_dim / 2;
  // halves: angles 8 sub .. 8 sub + 7; neighbours: 4 u0 .. 4 u0 + 3 and 4 u1 .. 4 u1 + 3
  const int f0 = rope.interleaved ? (w.r0 ? 4 * w.u0 : 0) : 8 * sub, f1 = rope.interleaved ? (w.r1 ? 4 * w.u1 : 0) : 8 * sub + 4;
  const float4 c0 = *reinterpret_cast<const float4*>(row + f0), c1 = *reinterpret_cast<const float4*>(row + f1);
  const float4 s0 = *reinterpret_cast<const float4*>(row + half + f0), s1 = *reinterpret_cast<const float4*>(row + half + f1);
  w.c[0] = c0.x; w.c[1] = c0.y; w.c[2] = c0.z; w.c[3] = c0.w; w.c[4] = c1.x; w.c[5] = c1.y; w.c[6] = c1.z; w.c[7] = c1.w;
  w.s[0] = s0.x; w.s[1] = s0.y; w.s[2] = s0.z; w.s[3] = s0.w; w.s[4] = s1.x; w.s[5] = s1.y; w.s[6] = s1.z; w.s[7] = s1.w;
}

// Norm (where there is a weight) and rotation of a lane's 16 elements; mask: the lanes of the warp's rows that are here.
template <bool BF16>
__device__ __forceinline__ void turn_row(float (&x)[8], float (&y)[8], const uint16_t* weight, const RowTurn& w, const RopeView& rope, unsigned mask) {
  if (weight) {
    float sq = 0.0f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sq = fmaf(x[i], x[i], fmaf(y[i], y[i], sq));
#pragma unroll
    for (int o = 1; o < kRowLanes; o <<= 1) sq += __shfl_xor_sync(mask, sq, o);
    const float inv = 1.0f / sqrtf(sq * (1.0f / kHeadDim) + rope.eps);
    float wx[8], wy[8];
    unpack8<BF16>(wx, *reinterpret_cast<const uint4*>(weight + 8 * w.u0));
    unpack8<BF16>(wy, *reinterpret_cast<const uint4*>(weight + 8 * w.u1));
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      x[i] = x[i] * inv * wx[i];
      y[i] = y[i] * inv * wy[i];
    }
  }
  if (w.turn && !rope.interleaved) {
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float p0 = x[i], p1 = y[i];
      x[i] = fmaf(p0, w.c[i], -p1 * w.s[i]);
      y[i] = fmaf(p0, w.s[i], p1 * w.c[i]);
    }
  } else if (w.turn) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float p0 = x[2 * i], p1 = x[2 * i + 1], e0 = y[2 * i], e1 = y[2 * i + 1];
      if (w.r0) {
        x[2 * i] = fmaf(p0, w.c[i], -p1 * w.s[i]);
        x[2 * i + 1] = fmaf(p0, w.s[i], p1 * w.c[i]);
      }
      if (w.r1) {
        y[2 * i] = fmaf(e0, w.c[4 + i], -e1 * w.s[4 + i]);
        y[2 * i + 1] = fmaf(e0, w.s[4 + i], e1 * w.c[4 + i]);
      }
    }
  }
}

// Few tokens: several warps share one, until every SM has a few or every warp is down to one pass.
inline unsigned share_rows(RowJob& job, int n_rows) {
  const int wanted = sm_count_of_current_device() * 16;
  const int passes = (n_rows + kRowsPerPass - 1) / kRowsPerPass;
  job.parts_shift = 0;
  while ((1 << job.parts_shift) < passes && (static_cast<long long>(job.n_tokens) << job.parts_shift) < wanted) ++job.parts_shift;
  const long long warps = static_cast<long long>(job.n_tokens) << job.parts_shift;
  return static_cast<unsigned>((warps + kAppendWarps - 1) / kAppendWarps);
}

}  // namespace

}  // namespace moqae
