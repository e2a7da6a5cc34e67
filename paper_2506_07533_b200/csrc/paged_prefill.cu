// Attention of several new tokens per sequence over a paged 16-bit cache (moqae_paged_prefill_attn).
//
// For every query row  o = sum_j p_j v_j / sum_j p_j,  p_j = 2^(f(q.k_j) - reference)  over the tokens it sees:
// two dense products with a softmax between them, on the 5th-generation tensor cores.
//
//   Rows.  The rows of a (sequence, kv head) are its tokens times the query heads of the group (row r = token
//   r / group, head r % group), so a group shares every key block and a few tokens fill a tile.  A CTA
//   owns 256 consecutive rows (two tiles of 128) and walks the blocks of 128 tokens that some row sees.
//   Pages.  The pages are a four-dimensional tensor map (channel, slot, head, page in the order of their
//   strides); a block is fetched with one tiled copy per page (or per 128 slots of a page) and half of the
//   channels, page numbers looked up one block ahead.  Rows of a block that no query may use (behind the
//   sequence, before every window) are not fetched where whole pages are concerned, and their values are
//   zeroed in shared memory before the product: a weight of zero does not silence a NaN.
//   Products, softmax and tensor memory as in the prefill attention over the quantised cache (prefill.cu):
//   S_i = Q_i K^T (M 128, N 128, K 16 steps), two threads per row, P_i written over S_i as 16-bit pairs, O_i += P_i V
//   with P_i as a tensor-memory operand, a reference that moves only when the weights of 64 columns
//   would add up to more than 2^14, so O_i is rarely rescaled.  Blocks are walked from the last to the
//   first: with a distance bias the largest scores come first (walking forwards moved the reference at every block).  P_i is rounded to the cache's dtype (the
//   product takes operands of one type): 2^-9 or 2^-12 of each weight, which averages out over the tokens.
//   Few rows.  Where the rows alone would leave SMs idle, the blocks of a row tile are cut into up to
//   kMaxSegs pieces for as many CTAs, which leave float32 sums in the workspace; the last to arrive joins them.
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
constexpr int kSoftmaxWarps = 16, kIssueWarp = 16, kKeyWarp = 17, kValueWarp = 18;
constexpr int kThreads = 19 * 32;
constexpr int kTmemCols = 512;
constexpr float kSumLimit = 16384.0f;                // weights of 64 columns that sum to less cannot overflow fp16
constexpr float kLog2e = 1.4426950408889634f;
constexpr long long kWaitLimit = 1ll << 31;          // about a second
constexpr int kMaxSegs = 32;
constexpr int kMinSegBlocks = 4;                     // a piece is at least this many blocks
constexpr int kPartFloats = kItemRows * (kHeadDim + 2);   // per piece: sums, then (reference, weight sum) per row

// kfull / vfull: bytes of a block have landed (vfull of an edge block: and its rows are zeroed); vraw: the bytes of
// an edge block of values; qfull: the query rows stand in shared memory; kfree / vfree: the products that read the stage are done; sfull, pfull, ofull as in prefill.cu
enum { BAR_KFULL = 0, BAR_VFULL = kStages, BAR_KFREE = 2 * kStages, BAR_VFREE = 3 * kStages, BAR_SFULL = 4 * kStages,
       BAR_PFULL = BAR_SFULL + 2, BAR_OFULL = BAR_PFULL + 2, BAR_VRAW = BAR_OFULL + 2, BAR_QFULL = BAR_VRAW + 1, BAR_COUNT = BAR_QFULL + 1 };

constexpr int kExchangeBytes = kItemRows * 2 * 4 + 2 * 8 * 2 * 4;
constexpr size_t kSmemBytes = 1024 + 2 * kTileBytes + 2 * kStages * kTileBytes + BAR_COUNT * 8 + 24 + kExchangeBytes;

__device__ __forceinline__ float rcp_approx(float x) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(x));
  return r;
}

struct PrefillJob {
  RowsView q, out;
  const int32_t* cu_q;
  int n_tokens, group, n_rb, n_seg;                  // n_rb: upper bound of the row tiles of all sequences
  unsigned group_inv;                                // ceil(2^32 / group)
  float* part;                                       // [n_rb][heads][n_seg][kPartFloats]
  unsigned* arrived;                                 // [n_rb][heads]
  int box_rows;                                      // slots per copy
  int dim_slot, dim_head, dim_page;                  // tensor-map dimension (1..3) of each
};

// What a CTA works on: rows row0 .. row0 + rows - 1 of (sequence b, head h), blocks [idx0, idx0 + n) of its walk.
struct Item {
  int b, rb, q_first, q_len, rows;
  int kv_len, pos0;                                  // position of the sequence's first query token
  int prefix, win_lo, n_pre, first;                  // walk: blocks 0 .. n_pre - 1, then first, first + 1, ..
  int nb[2], total;                                  // blocks of the walk each tile needs; of the item
};

// row / group (exact for rows below 2^29: the product's error is row * group / 2^32 at most)
__device__ __forceinline__ int token_of(const PrefillJob& job, int row) {
  return job.group == 1 ? row : static_cast<int>(__umulhi(static_cast<unsigned>(row), job.group_inv));
}
__device__ __forceinline__ int block_at(const Item& it, int idx) { return idx < it.n_pre ? idx : it.first + idx - it.n_pre; }
__device__ __forceinline__ bool token_used(const Item& it, int j) { return j < it.kv_len && (j >= it.win_lo || j < it.prefix); }

// Find the flat row tile `flat` among the sequences; false: there are fewer.
__device__ __forceinline__ bool find_item(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, int flat, int lane, Item& it) {
  int before = 0;
  for (int base = 0; base < pv.batch; base += 32) {
    const int b = base + lane;
    int lo = 0, hi = 0, len = 0, pre = 0;
    if (b < pv.batch) {
      len = paged_len(pv, b, blockIdx.x == 0);
      pre = opt.prefix_len ? min(max(opt.prefix_len[b], 0), len) : 0;
      lo = min(max(job.cu_q[b], 0), job.n_tokens);
      hi = min(max(job.cu_q[b + 1], lo), job.n_tokens);
    }
    const int n = ((hi - lo) * job.group + kItemRows - 1) / kItemRows;
    int inc = n;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int x = __shfl_up_sync(0xffffffffu, inc, o);
      if (lane >= o) inc += x;
    }
    const unsigned hit = __ballot_sync(0xffffffffu, before + inc > flat);
    if (hit) {
      const int l = __ffs(hit) - 1;
      it.b = base + l;
      it.q_first = __shfl_sync(0xffffffffu, lo, l);
      it.q_len = __shfl_sync(0xffffffffu, hi, l) - it.q_first;
      const int n_l = __shfl_sync(0xffffffffu, n, l), start = before + __shfl_sync(0xffffffffu, inc, l) - n_l;
      it.rb = n_l - 1 - (flat - start);                                   // the longest rows first
      it.rows = min(kItemRows, it.q_len * job.group - it.rb * kItemRows);
      it.kv_len = __shfl_sync(0xffffffffu, len, l);
      it.pos0 = it.kv_len - it.q_len;
      it.prefix = __shfl_sync(0xffffffffu, pre, l);
      const int row0 = it.rb * kItemRows;
      const int p_lo = it.pos0 + token_of(job, row0);
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
        const int last = min(it.rows, kTileRows * (i + 1)) - 1;           // last row of the tile
        int end = 0;
        if (last >= kTileRows * i) {
          const int p = it.pos0 + token_of(job, row0 + last);
          end = p >= 0 ? p / kBlock + 1 : 0;
          if (it.win_lo == 0) end = max(end, (it.prefix + kBlock - 1) / kBlock);
          end = it.n_pre + max(0, end - it.first);
        }
        it.nb[i] = end;
      }
      it.total = max(it.nb[0], it.nb[1]);
      return true;
    }
    before += __shfl_sync(0xffffffffu, inc, 31);
  }
  return false;
}

template <bool BF16, bool CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
paged_prefill_kernel(PagedView pv, AttnOptions opt, PrefillJob job, const __grid_constant__ CUtensorMap map_k,
                     const __grid_constant__ CUtensorMap map_v) {
  extern __shared__ __align__(128) uint8_t smem_raw[];
  uint8_t* smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);
  uint8_t* sQ = smem;
  uint8_t* sK = sQ + 2 * kTileBytes;
  uint8_t* sV = sK + kStages * kTileBytes;
  uint64_t* bar_mem = reinterpret_cast<uint64_t*>(sV + kStages * kTileBytes);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bar_mem + BAR_COUNT);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  volatile unsigned* ticket = reinterpret_cast<volatile unsigned*>(tmem_slot + 2);
  float* exch = reinterpret_cast<float*>(bar_mem + BAR_COUNT + 3);        // [256 rows][2 halves]
  volatile int* pair_flag = reinterpret_cast<volatile int*>(exch + 2 * kItemRows);
  const uint32_t bar0 = smem_u32(bar_mem);
  auto bar = [&](int i) { return bar0 + 8u * i; };

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = pv.n_kv_heads;
  const int per_seg = job.n_rb * H;
  const int seg = static_cast<int>(blockIdx.x) / per_seg, rest = static_cast<int>(blockIdx.x) - seg * per_seg;
  const int flat = rest / H, h = rest - flat * H;        // heads side by side: the longest rows of all heads start first
  __shared__ Item it;                                  // in shared memory: its fields would cost the softmax threads registers
  __shared__ int found;
  if (warp == 0) {
    Item x;
    const bool ok = find_item(pv, opt, job, flat, lane, x);
    if (lane == 0) {
      found = ok;
      if (ok) it = x;
    }
  }
  if (warp == kIssueWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;\n" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  if (tid == kKeyWarp * 32) {
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_k) : "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(&map_v) : "memory");
    for (int i = 0; i < BAR_COUNT; ++i) mbar_init(bar(i), i == BAR_QFULL ? kSoftmaxWarps : (i >= BAR_PFULL && i < BAR_OFULL ? 8 : 1));
    *abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = *tmem_slot;
  auto free_tmem = [&]() {
    if (warp == kIssueWarp)
      asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;\n" ::"r"(tmem), "r"(kTmemCols) : "memory");
  };
  // this CTA's piece of the walk
  const int n_seg = found ? max(1, min(job.n_seg, it.total / kMinSegBlocks)) : 0;
  if (seg >= n_seg) {
    free_tmem();
    return;
  }
  const int idx0 = static_cast<int>(static_cast<long long>(it.total) * seg / n_seg);
  const int idx1 = static_cast<int>(static_cast<long long>(it.total) * (seg + 1) / n_seg);
  const int n_blocks = idx1 - idx0;
  // the piece is walked backwards, block idx1 - 1 - n at step n; tile i joins at step first0 / first1
  const int first0 = min(max(idx1 - it.nb[0], 0), n_blocks), first1 = min(max(idx1 - it.nb[1], 0), n_blocks);
  const int row0 = it.rb * kItemRows;

  // bounded wait that also gives up when another role has given up
  auto wait = [&](int which, int completion) -> bool {
    const uint32_t a = bar(which), parity = static_cast<uint32_t>(completion) & 1u;
    if (mbar_try_wait(a, parity)) return true;
    const long long t0 = clock64();
    while (!*abort_flag) {
      if (mbar_try_wait(a, parity)) return true;
      if (clock64() - t0 > kWaitLimit) *abort_flag = 1;
    }
    return false;
  };

  if (warp < kSoftmaxWarps) {
    // ================= softmax, two threads per row (see prefill.cu) =================
    const int half = warp >> 3, i = (warp & 7) >> 2, pair_id = warp & 7;
    const int first = i ? first1 : first0;
    const int row = 128 * i + 32 * (warp & 3) + lane;
    // rows behind the last one take its position: they cost no extra mask and are not stored
    auto position = [&](int r) { return it.pos0 + token_of(job, row0 + min(r, it.rows - 1)); };
    const int qpos = position(row);
    // tokens all_from .. all_to are seen by every row of the warp
    const int all_to = position(row - lane), all_from = opt.window > 0 ? position(row - lane + 31) - opt.window + 1 : -0x40000000;
    // the query rows as A operands, swizzled like the keys (rows behind the sequence's last are zero): 8 units of 16
    // bytes per thread
    {
      uint4 v[8];
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int r = 32 * u + (tid >> 4), t = token_of(job, row0 + r), g = row0 + r - t * job.group;
        v[u] = make_uint4(0u, 0u, 0u, 0u);
        if (r < it.rows)
          v[u] = *reinterpret_cast<const uint4*>(job.q.data + (it.q_first + t) * job.q.token + (h * job.group + g) * job.q.head + 8 * (tid & 15));
      }
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int r = 32 * u + (tid >> 4);
        *reinterpret_cast<uint4*>(sQ + (r >> 7) * kTileBytes + ((tid >> 3) & 1) * (kTileBytes / 2) + (r & 127) * 128 + (((tid ^ r) & 7) << 4)) = v[u];
      }
      fence_async_proxy();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_QFULL));
    }
    const uint32_t lane_addr = tmem + (static_cast<uint32_t>((warp & 3) * 32) << 16);
    const uint32_t s_addr = lane_addr + 128 * i + 64 * half, p_addr = lane_addr + 128 * i + 32 * half;
    const uint32_t o_addr = lane_addr + 256 + 128 * i + 64 * half;
    auto pair_sync = [&]() { asm volatile("bar.sync %0, 64;\n" ::"r"(1 + pair_id) : "memory"); };
    const float scale_log2 = opt.scale * kLog2e;
    const float slope = BIAS && row < it.rows ? opt.slopes[h * job.group + row0 + row - token_of(job, row0 + row) * job.group] * kLog2e : 0.0f;
    // tanh(z) / z for |z| <= 1 as a polynomial in z^2 (minimax, own fit, relative error 6e-7), for z = x / cap2
    // with x and cap2 in base-2 units: the coefficients take the powers of cap2
    const float cap2 = opt.cap * kLog2e, w2 = CAP ? 1.0f / (cap2 * cap2) : 0.0f;
    const float t1 = -0.33329042792f * w2, t2 = 0.13281433284f * w2 * w2, t3 = -0.05160567537f * w2 * w2 * w2;
    const float t4 = 0.01674311422f * (w2 * w2) * (w2 * w2), t5 = -0.00306706037f * (w2 * w2) * (w2 * w2) * w2;
    // Scores of columns 32 c .. 32 c + 31 in base-2 units, up to a factor and a term that `mul` and `add` give
    // (so that both join the subtraction of the reference); column e is seen if lo < e <= hi or e < pre.
    auto scores = [&](auto masked, float (&v)[32], int c, int hi, int lo, int pre, float& mul, float& add) {
      tmem_ld32(v, s_addr + 32 * c);
      mul = CAP || BIAS ? 1.0f : scale_log2;
      add = 0.0f;
      if (CAP || BIAS) {
#pragma unroll
        for (int e = 0; e < 32; ++e) v[e] *= scale_log2;
      }
      if (CAP) {
        float big = 0.0f;
#pragma unroll
        for (int e = 0; e < 32; ++e) big = fmaxf(big, fabsf(v[e]));
        if (__all_sync(0xffffffffu, big <= cap2)) {
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const float u = v[e] * v[e];
            v[e] *= fmaf(fmaf(fmaf(fmaf(fmaf(t5, u, t4), u, t3), u, t2), u, t1), u, 0.99999940395f);
          }
        } else {
          // some score passes the cap: tanh(z) = 1 - 2 / (exp(2 z) + 1), accurate to a few float32 roundings of the cap
          const float in = 2.0f * kLog2e / cap2;
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(-2.0f * cap2, rcp_approx(ex2_approx(v[e] * in) + 1.0f), cap2);
        }
      }
      if (BIAS) {
        const float dist = static_cast<float>(hi - 32 * c);               // of column 0
        if (pre > 0) {                                                    // tokens behind the query may be seen
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(-slope, fabsf(dist - static_cast<float>(e)), v[e]);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = fmaf(slope, static_cast<float>(e), v[e]);
          add = -slope * dist;
        }
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
    uint32_t pk[32];
    // weights of this thread's 64 columns against the reference, packed; their sum
    auto weights = [&](auto masked, float ref, int hi, int lo, int pre) -> float {
      float sum = 0.0f;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float v[32], mul, add;
        scores(masked, v, c, hi, lo, pre, mul, add);
        const uint64_t scale2 = pack_f2(mul, mul), negm2 = pack_f2(add - ref, add - ref);
        uint64_t part[2] = {0ull, 0ull};
#pragma unroll
        for (int e2 = 0; e2 < 16; ++e2) {
          float x0, x1;
          const uint64_t vv = pack_f2(v[2 * e2], v[2 * e2 + 1]);
          unpack_f2(CAP || BIAS ? add_f2(vv, negm2) : fma_f2(vv, scale2, negm2), x0, x1);
          const float p0 = ex2_approx(x0), p1 = ex2_approx(x1);
          part[e2 & 1] = add_f2(part[e2 & 1], pack_f2(p0, p1));
          pk[16 * c + e2] = float2_to_pair<BF16>(p0, p1);
        }
        float s0, s1;
        unpack_f2(add_f2(part[0], part[1]), s0, s1);
        sum += s0 + s1;
      }
      return sum;
    };
    float m_ref = -INFINITY, l = 0.0f;
    bool ok = true;
    for (int n = first; n < n_blocks && ok; ++n) {
      const int j0 = block_at(it, idx1 - 1 - n) * kBlock + 64 * half;     // token of this thread's first column
      const int hi = qpos - j0, lo = opt.window > 0 ? hi - opt.window : -0x40000000, pre = it.prefix - j0;
      const bool masked = !(j0 + 63 <= all_to && j0 >= all_from) && pre < 64;
      ok = __all_sync(0xffffffffu, wait(BAR_SFULL + i, n - first));
      if (ok) tc_fence_after();
      float csum = 0.0f;
      if (ok && n == first) {
        // The first reference: any score that the row sees will do (its weight is then at most 1 and at least
        // a half, and larger scores may lead by 2^14).  All rows of the warp see token all_to, if this block
        // holds it; both threads of a row read its column, without a word between them.
        const int col = min(all_to - (j0 - 64 * half), kBlock - 1);
        if (col >= 0 && j0 - 64 * half + col >= all_from) {
          uint32_t raw;
          asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n" : "=r"(raw) : "r"(lane_addr + 128 * i + col));
          asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
          float y = __uint_as_float(raw) * scale_log2;
          if (CAP) y = fmaf(-2.0f * cap2, rcp_approx(ex2_approx(y * (2.0f * kLog2e / cap2)) + 1.0f), cap2);
          if (BIAS) y -= slope * static_cast<float>(qpos - (j0 - 64 * half + col));
          if (y > -1e30f && y < 1e30f) m_ref = ceilf(y);
        }
      }
      bool over = m_ref == -INFINITY;                  // nothing seen yet
      over = __any_sync(0xffffffffu, over);
      if (ok && !over) {
        csum = masked ? weights(std::true_type{}, m_ref, hi, lo, pre) : weights(std::false_type{}, m_ref, hi, lo, pre);
        over = __any_sync(0xffffffffu, !(csum < kSumLimit));
      }
      if (lane == 0) pair_flag[((n & 1) * 8 + pair_id) * 2 + half] = (over ? 1 : 0) | (ok ? 0 : 2);
      pair_sync();
      const int flags = pair_flag[((n & 1) * 8 + pair_id) * 2] | pair_flag[((n & 1) * 8 + pair_id) * 2 + 1];
      if (flags & 2) {
        ok = false;
        break;
      }
      if (flags & 1) {
        // the reference moves to the row's largest score of this block (a row that has seen nothing yet keeps
        // -inf and weighs its columns, all masked, against 0)
        float mx = -INFINITY;
#pragma unroll 1
        for (int c = 0; c < 2; ++c) {
          float v[32], mul, add;
          scores(std::true_type{}, v, c, hi, lo, pre, mul, add);
          float top = v[0];
#pragma unroll
          for (int e = 1; e < 32; ++e) top = fmaxf(top, v[e]);
          mx = fmaxf(mx, fmaf(top, mul, add));         // mul > 0
        }
        exch[row * 2 + half] = mx;
        pair_sync();
        const float m_new = fmaxf(m_ref, ceilf(fmaxf(exch[row * 2], exch[row * 2 + 1])));
        const float corr = m_ref == -INFINITY ? 0.0f : ex2_approx(m_ref - m_new);
        if (n > first) {
#pragma unroll 1
          for (int o4 = 0; o4 < 2; ++o4) {
            float o[32];
            tmem_ld32(o, o_addr + 32 * o4);
#pragma unroll
            for (int e = 0; e < 32; ++e) o[e] *= corr;
            tmem_st32(o_addr + 32 * o4, o);
          }
        }
        l *= corr;
        m_ref = m_new;
        csum = weights(std::true_type{}, m_ref == -INFINITY ? 0.0f : m_ref, hi, lo, pre);
        pair_sync();
      }
      l += csum;
      tmem_st32u(p_addr, pk);
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(BAR_PFULL + i));
    }
    if (ok && first < n_blocks) ok = __all_sync(0xffffffffu, wait(BAR_OFULL + i, 0));
    exch[row * 2 + half] = l;
    pair_sync();
    if (ok) {
      tc_fence_after();
      const float lt = exch[row * 2] + exch[row * 2 + 1];
      const float inv = lt == 0.0f ? 0.0f : 1.0f / lt;
      float* piece = job.part + ((static_cast<long long>(flat) * H + h) * job.n_seg + seg) * kPartFloats;
      // Rows leave through shared memory (the place of this tile's queries, which no product reads any more; 4 KiB
      // per warp, 128 bytes per row, units swizzled), so that a store covers whole lines: a thread storing its
      // own row took 32 lines per instruction, 3 us for the 64 KiB of a CTA.
      uint8_t* stage = sQ + i * kTileBytes + ((warp & 3) * 2 + half) * 4096;
      const int w_row = 128 * i + 32 * (warp & 3);
#pragma unroll 1
      for (int c4 = 0; c4 < 2; ++c4) {
        float v[32];
        if (first < n_blocks) tmem_ld32(v, o_addr + 32 * c4);
        if (lt == 0.0f) {                              // sees nothing here (or its tile ran no block at all)
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0.0f;
        }
        if (n_seg == 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e)
            *reinterpret_cast<uint4*>(stage + lane * 128 + (((4 * c4 + e) ^ (lane & 7)) << 4)) =
                make_uint4(float2_to_pair<BF16>(v[8 * e] * inv, v[8 * e + 1] * inv), float2_to_pair<BF16>(v[8 * e + 2] * inv, v[8 * e + 3] * inv),
                           float2_to_pair<BF16>(v[8 * e + 4] * inv, v[8 * e + 5] * inv), float2_to_pair<BF16>(v[8 * e + 6] * inv, v[8 * e + 7] * inv));
          if (c4 == 0) continue;
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            *reinterpret_cast<float4*>(stage + lane * 128 + ((e ^ (lane & 7)) << 4)) = make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
        }
        __syncwarp();
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int r = 4 * k + (lane >> 3), u = lane & 7;
          const uint4 x = *reinterpret_cast<const uint4*>(stage + r * 128 + ((u ^ (r & 7)) << 4));
          if (w_row + r >= it.rows) continue;
          if (n_seg == 1) {
            const int t = token_of(job, row0 + w_row + r), g = row0 + w_row + r - t * job.group;
            *reinterpret_cast<uint4*>(job.out.data + (it.q_first + t) * job.out.token + (h * job.group + g) * job.out.head + 64 * half + 8 * u) = x;
          } else {
            *reinterpret_cast<uint4*>(piece + (w_row + r) * kHeadDim + 64 * half + 32 * c4 + 4 * u) = x;
          }
        }
        __syncwarp();
      }
      if (n_seg > 1 && half == 0 && row < it.rows)
        *reinterpret_cast<float2*>(piece + kItemRows * kHeadDim + 2 * row) = make_float2(m_ref, lt);
    } else if (lane == 0) {
      paged_status(pv.status, MOQAE_ERR_TIMEOUT, static_cast<int>(blockIdx.x), warp);
    }
    if (n_seg > 1) __threadfence();
  } else if (warp > kIssueWarp) {
    // ================= fetch: key blocks (one warp) and value blocks (another) =================
    const bool is_v = warp == kValueWarp;
    const CUtensorMap* map = is_v ? &map_v : &map_k;
    const int boxes = kBlock / job.box_rows;
    int n_raw = 0;
    auto box_token = [&](int n) { return block_at(it, idx1 - 1 - n) * kBlock + lane * job.box_rows; };
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
    for (int n = 0; n < n_blocks; ++n) {
      const int st = n % kStages;
      const int next = look_up(n + 1);
      if (n >= kStages && !__all_sync(0xffffffffu, wait((is_v ? BAR_VFREE : BAR_KFREE) + st, n / kStages - 1))) break;
      const int j0 = block_at(it, idx1 - 1 - n) * kBlock;
      const bool edge = is_v && (j0 + kBlock > it.kv_len || (j0 < it.win_lo && j0 + kBlock > it.prefix));
      const uint32_t full = bar((is_v ? BAR_VFULL : BAR_KFULL) + st), landed = edge ? bar(BAR_VRAW) : full;
      const unsigned need = __ballot_sync(0xffffffffu, page >= 0);
      if (lane == 0) mbar_expect_tx(landed, __popc(need) * job.box_rows * 256);
      __syncwarp();
      uint8_t* dst = (is_v ? sV : sK) + st * kTileBytes;
      if (page >= 0) {
        const int slot = box_token(n) & (pv.page_size - 1);
        const int y = job.dim_slot == 1 ? slot : (job.dim_head == 1 ? h : page);
        const int z = job.dim_slot == 2 ? slot : (job.dim_head == 2 ? h : page);
        const int w = job.dim_slot == 3 ? slot : (job.dim_head == 3 ? h : page);
        const uint32_t d = smem_u32(dst) + lane * job.box_rows * 128;
        tma_load_4d(d, map, 0, y, z, w, landed);                          // channels 0..63
        tma_load_4d(d + kTileBytes / 2, map, 64, y, z, w, landed);        // channels 64..127
      }
      if (edge) {
        if (!__all_sync(0xffffffffu, wait(BAR_VRAW, n_raw++))) break;
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
  } else {
    // ================= MMA issue (one thread) =================
    constexpr uint32_t kFormat = BF16 ? (1u << 7) | (1u << 10) : 0u;      // operand type
    constexpr uint32_t kIdescS = (1u << 4) | kFormat | (16u << 17) | (8u << 24), kIdescPV = kIdescS | (1u << 16);
    const uint64_t qd = make_desc_sw128(smem_u32(sQ), 16, 1024);
    const uint64_t kd = make_desc_sw128(smem_u32(sK), 16, 1024), vd = make_desc_sw128(smem_u32(sV), kTileBytes / 2, 1024);
    const uint32_t qd_lo = static_cast<uint32_t>(qd), qd_hi = static_cast<uint32_t>(qd >> 32);
    const uint32_t kd_lo = static_cast<uint32_t>(kd), kd_hi = static_cast<uint32_t>(kd >> 32);
    const uint32_t vd_lo = static_cast<uint32_t>(vd), vd_hi = static_cast<uint32_t>(vd >> 32);
    // the stage is free after the last tile that reads it: tile 1, or tile 0 where tile 1 has no such block
    auto issue_s = [&](int i, int n) {
      if (lane == 0) {
        const uint32_t a_lo = qd_lo + i * (kTileBytes >> 4), b_lo = kd_lo + (n % kStages) * (kTileBytes >> 4), d = tmem + 128 * i;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          umma_f16_ss(d, a_lo + (k >> 2) * 1024 + (k & 3) * 2, qd_hi, b_lo + (k >> 2) * 1024 + (k & 3) * 2, kd_hi, kIdescS, k > 0);
        umma_commit(bar(BAR_SFULL + i));
        if (i == 1 || n < first1) umma_commit(bar(BAR_KFREE + n % kStages));
      }
      __syncwarp();
    };
    auto issue_pv = [&](int i, int n) {
      if (lane == 0) {
        const uint32_t lo = vd_lo + (n % kStages) * (kTileBytes >> 4), d = tmem + 256 + 128 * i, a = tmem + 128 * i;
        umma_f16_ta(d, a, lo, vd_hi, kIdescPV, n > (i ? first1 : first0));
#pragma unroll
        for (int k = 1; k < 8; ++k) umma_f16_ta(d, a + 8 * k, lo + 128 * k, vd_hi, kIdescPV, 1u);
        if (i == 1 || n < first1) umma_commit(bar(BAR_VFREE + n % kStages));
        if (n + 1 == n_blocks) umma_commit(bar(BAR_OFULL + i));
      }
      __syncwarp();
    };
    bool ok = n_blocks > 0 && wait(BAR_QFULL, 0) && wait(BAR_KFULL, 0);
    if (ok) {
      tc_fence_after();
      if (first0 == 0) issue_s(0, 0);
      if (first1 == 0) issue_s(1, 0);
    }
    for (int n = 0; n < n_blocks && ok; ++n) {
      ok = wait(BAR_VFULL + n % kStages, n / kStages);
      if (ok && n + 1 < n_blocks) ok = wait(BAR_KFULL + (n + 1) % kStages, (n + 1) / kStages);
      for (int i = 0; i < 2 && ok; ++i) {
        const int first = i ? first1 : first0;
        if (n >= first) {
          ok = wait(BAR_PFULL + i, n - first);
          if (!ok) break;
        }
        tc_fence_after();
        if (n >= first) issue_pv(i, n);
        if (n + 1 < n_blocks && n + 1 >= first) issue_s(i, n + 1);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  free_tmem();

  if (n_seg > 1) {
    // ---- the last piece of the item to arrive joins all of them, in the order of their tokens ----
    const long long item = static_cast<long long>(flat) * H + h;
    if (tid == 0) {
      __threadfence();
      *ticket = atomicInc(job.arrived + item, static_cast<unsigned>(n_seg - 1));
    }
    __syncthreads();
    if (*ticket != static_cast<unsigned>(n_seg - 1)) return;
    __threadfence();
    const float* part = job.part + item * job.n_seg * kPartFloats;
    // a thread takes four rows' units of 4 channels at a time, so that their loads are in flight together
    const int units = it.rows * 32;
    for (int base = tid; base < units; base += 4 * kThreads) {
      float m[4], lsum[4], acc[4][4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        m[k] = -INFINITY;
        lsum[k] = acc[k][0] = acc[k][1] = acc[k][2] = acc[k][3] = 0.0f;
      }
      for (int s = 0; s < n_seg; ++s) {
        const float* src = part + static_cast<long long>(s) * kPartFloats;
        float2 w[4];
        float4 v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const int x = min(base + k * kThreads, units - 1);
          w[k] = __ldcg(reinterpret_cast<const float2*>(src + kItemRows * kHeadDim) + (x >> 5));
          v[k] = __ldcg(reinterpret_cast<const float4*>(src) + x);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {               // running reference: both sides are scaled to the larger
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
        const int x = base + k * kThreads, row = x >> 5, c = (x & 31) * 4;
        if (x >= units) break;
        const float inv = lsum[k] == 0.0f ? 0.0f : 1.0f / lsum[k];
        const int t = token_of(job, row0 + row), g = row0 + row - t * job.group;
        *reinterpret_cast<uint2*>(job.out.data + (it.q_first + t) * job.out.token + (h * job.group + g) * job.out.head + c) =
            make_uint2(float2_to_pair<BF16>(acc[k][0] * inv, acc[k][1] * inv), float2_to_pair<BF16>(acc[k][2] * inv, acc[k][3] * inv));
      }
    }
  }
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

// row tiles of all sequences, at most: sum of ceil(rows / 256)
long long row_tiles(int batch, int group, int n_tokens) {
  return (static_cast<long long>(n_tokens) * group + static_cast<long long>(batch) * (kItemRows - 1)) / kItemRows;
}

// Pieces per item.  With one CTA per SM, n pieces take ceil(items n / SMs) turns of blocks / n blocks plus a fixed
// cost per piece of about kPieceBlocks blocks (start, partial sums out and in).  `blocks` is what the block
// table can hold; an item with fewer blocks is cut into fewer pieces on the device.
int pieces(long long items, long long blocks, int sms) {
  constexpr double kPieceBlocks = 5.0;
  int best = 1;
  double best_cost = 1e300;
  for (int n = 1; n <= kMaxSegs && n * kMinSegBlocks <= blocks + kMinSegBlocks; ++n) {
    const double turns = static_cast<double>((items * n + sms - 1) / sms);
    const double cost = turns * (static_cast<double>(blocks) / n + kPieceBlocks) + (n > 1 ? n : 0);
    if (cost < best_cost * 0.98) {
      best_cost = cost;
      best = n;
    }
  }
  return best;
}

constexpr long long kSplitItems = 512;                // more row tiles than this are never cut

template <bool BF16, bool CAP, bool BIAS>
cudaError_t launch(const PagedView& pv, const AttnOptions& opt, const PrefillJob& job, const CUtensorMap& mk, const CUtensorMap& mv,
                   long long grid, cudaStream_t st) {
  static std::atomic<unsigned long long> done{0};
  cudaError_t e = allow_shared_memory(paged_prefill_kernel<BF16, CAP, BIAS>, kSmemBytes, done);
  if (e != cudaSuccess) return e;
  paged_prefill_kernel<BF16, CAP, BIAS><<<static_cast<unsigned>(grid), kThreads, kSmemBytes, st>>>(pv, opt, job, mk, mv);
  return cudaGetLastError();
}

long long counter_bytes(long long items) { return (items * 4 + 15) / 16 * 16; }

}  // namespace

// arrival counters, then the pieces' partial sums
long long paged_prefill_workspace_bytes(int batch, int n_kv_heads, int group, int n_tokens) {
  const long long items = row_tiles(batch, group, n_tokens) * n_kv_heads;
  if (items > kSplitItems || items == 0) return 16;
  return counter_bytes(kSplitItems) + items * kMaxSegs * kPartFloats * 4;
}

cudaError_t launch_paged_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                                 const AttnOptions& opt, void* workspace, cudaStream_t st) {
  const int group = q.n_heads / pv.n_kv_heads;
  const long long n_rb = row_tiles(pv.batch, group, n_tokens);
  if (pv.batch <= 0 || n_tokens <= 0 || n_rb == 0) return cudaSuccess;
  PrefillJob job{};
  job.q = q;
  job.out = out;
  job.cu_q = cu_q;
  job.n_tokens = n_tokens;
  job.group = group;
  job.group_inv = group > 1 ? static_cast<unsigned>(((1ull << 32) + group - 1) / group) : 0u;
  job.n_rb = static_cast<int>(n_rb);
  job.n_seg = 1;
  const long long items = n_rb * pv.n_kv_heads;
  if (workspace && items <= kSplitItems) {
    const long long blocks = (static_cast<long long>(pv.max_pages) * pv.page_size + kBlock - 1) / kBlock;
    job.n_seg = pieces(items, blocks, sm_count_of_current_device());
    job.arrived = static_cast<unsigned*>(workspace);
    job.part = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + counter_bytes(kSplitItems));
  }
  const long long grid = items * job.n_seg;
  if (grid > 0x7fffffffll) return cudaErrorInvalidConfiguration;
  job.box_rows = pv.page_size < 64 ? pv.page_size : 64;
  // one order of dimensions serves keys and values if both are laid out alike; otherwise it is the keys'
  const long long ks[3] = {pv.k_slot, pv.k_head, pv.k_page}, vs[3] = {pv.v_slot, pv.v_head, pv.v_page};
  int order[3] = {0, 1, 2};
  for (int a = 0; a < 2; ++a)
    for (int b = 0; b < 2 - a; ++b)
      if (ks[order[b]] > ks[order[b + 1]]) {
        const int t = order[b];
        order[b] = order[b + 1];
        order[b + 1] = t;
      }
  for (int d = 0; d < 3; ++d) (order[d] == 0 ? job.dim_slot : (order[d] == 1 ? job.dim_head : job.dim_page)) = d + 1;
  CUtensorMap mk, mv;
  const void* kb = pv.n_pages > 0 ? pv.k : q.data;     // without pages nothing inside the map is ever named
  const void* vb = pv.n_pages > 0 ? pv.v : q.data;
  if (!make_page_map(&mk, kb, pv, ks, order, job.box_rows) || !make_page_map(&mv, vb, pv, vs, order, job.box_rows)) return cudaErrorNotSupported;
  auto go = [&](auto bf16) {
    constexpr bool kBf16 = decltype(bf16)::value;
    if (opt.cap > 0.0f)
      return opt.slopes ? launch<kBf16, true, true>(pv, opt, job, mk, mv, grid, st) : launch<kBf16, true, false>(pv, opt, job, mk, mv, grid, st);
    return opt.slopes ? launch<kBf16, false, true>(pv, opt, job, mk, mv, grid, st) : launch<kBf16, false, false>(pv, opt, job, mk, mv, grid, st);
  };
  return pv.dtype == MOQAE_DTYPE_BF16 ? go(std::true_type{}) : go(std::false_type{});
}

}  // namespace moqae
