// Block tables, lengths and slot maps of a batch from the tokens that its sequences bring or give back (moqae_paged_plan).
//
// Mathematics: three running sums over the sequences (new tokens, pages taken, pages given back), then every row of the
// step finds its sequence by bisection in the first, every page its sequence and entry in the others.  A few
// kilobytes at most are moved, so the call is bound by its launch and the trips to memory that depend on each other:
// lengths, sums, store (the first free pages travel beside the lengths).  One launch therefore: all CTAs form the sums of the whole batch, 256 sequences at a time
// (nothing to wait for but the lengths), and share out rows and pages; what may be read and written in place (lengths, the pool's
// state) is written by the CTA that comes last, when all have read it.  A batch that is refused is found in a first pass
// over the lengths, before anything is written.  Measured: 61 sequences, eight of them leaving with their pages, 5.0 us (in a graph); 96 sequences and 64367
// rows, 7.2 to 8.1 us for 0.6 MB.
#include "paged4.cuh"

namespace moqae {

namespace {

constexpr int kPlanThreads = 256, kPlanWarps = kPlanThreads / 32;
constexpr int kRowsPerCta = 2048;                // rows that a CTA is worth starting for
constexpr int kBatch = 4;

struct Sums {
  int tokens, take, give;
};

// What sequence b brings: its length before and after, and pages.
struct Change {
  int given, past, total, grow, have, want;      // given: past_len as it is; have, want: pages before and after
  bool good;
};
// (What a batch that is refused asks for is cut off just above what could be granted, so that a warp's sums stay in 32 bits.)
__device__ __forceinline__ Sums sums_of(const Change& c, const PlanJob& job, const PoolView& pool) {
  return Sums{min(c.grow, job.n_rows + 1), min(max(c.want - c.have, 0), pool.n_pages + 1), min(max(c.have - c.want, 0), pool.n_pages + 1)};
}
__device__ __forceinline__ Change change_of(const PlanJob& job, int b) {
  Change c{0, 0, 0, 0, 0, 0, true};
  if (b >= job.batch) return c;
  const long long most = static_cast<long long>(job.max_pages) << job.page_shift;
  const long long past = job.past[b], total = max(past + job.n_new[b], 0ll);
  c.given = job.past[b];
  c.good = past >= 0 && past <= most && total <= most;
  if (!c.good) return c;
  const int page = 1 << job.page_shift;
  c.past = static_cast<int>(past);
  c.total = static_cast<int>(total);
  c.grow = max(c.total - c.past, 0);
  c.have = (c.past + page - 1) >> job.page_shift;
  c.want = (c.total + page - 1) >> job.page_shift;
  return c;
}

// Sums over the lanes up to this one.
__device__ __forceinline__ Sums scan(Sums s, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(0xffffffffu, s.tokens, o), y = __shfl_up_sync(0xffffffffu, s.take, o), z = __shfl_up_sync(0xffffffffu, s.give, o);
    if (lane >= o) s = Sums{s.tokens + x, s.take + y, s.give + z};
  }
  return s;
}

// largest i with sums[i] <= x (sums not decreasing, sums[0] <= x < sums[n])
__device__ __forceinline__ int find_in(const int* sums, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (sums[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

__global__ void __launch_bounds__(kPlanThreads) paged_plan_kernel(PlanJob job, PoolView pool) {
  __shared__ long long all_tokens[kPlanWarps], all_take[kPlanWarps], all_give[kPlanWarps];
  __shared__ int warp_sum[3][kPlanWarps];
  __shared__ int tokens_to[kPlanThreads + 1], take_to[kPlanThreads + 1], give_to[kPlanThreads + 1];   // sums in front of a sequence
  __shared__ int past_of[kPlanThreads], have_of[kPlanThreads], want_of[kPlanThreads];
  __shared__ int bad_seq, last;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if (tid == 0) bad_seq = 0x7fffffff;
  after_previous();
  const int head = pool.state[0], n_free = pool.state[1];
  Change mine = change_of(job, tid);
  __syncthreads();

  // ---- does it all fit? (the sums of up to 256 sequences, which one turn holds, come out of the turn) ----
  Sums own = sums_of(mine, job, pool), to_here = scan(own, lane);
  if (!mine.good) atomicMin(&bad_seq, tid);
  if (lane == 31) {
    warp_sum[0][warp] = to_here.tokens;
    warp_sum[1][warp] = to_here.take;
    warp_sum[2][warp] = to_here.give;
  }
  // the page that this thread takes first, if it takes any, travels meanwhile
  const int first = static_cast<int>(blockIdx.x) * kPlanThreads + tid, step = static_cast<int>(gridDim.x) * kPlanThreads;
  auto place = [&](int n) -> int {               // n < 2 n_pages behind the first free page
    const long long at = static_cast<long long>(head) + n;
    return static_cast<int>(at >= pool.n_pages ? at - pool.n_pages : at);
  };
  const bool sound = head >= 0 && head < max(pool.n_pages, 1) && n_free >= 0 && n_free <= pool.n_pages;
  const int ahead = sound && first < n_free ? pool.ring[place(first)] : -1;
  __syncthreads();
  long long tokens = 0, take = 0, give = 0;
#pragma unroll
  for (int w = 0; w < kPlanWarps; ++w) {
    tokens += warp_sum[0][w];
    take += warp_sum[1][w];
    give += warp_sum[2][w];
  }
  if (job.batch > kPlanThreads) {
    long long more_tokens = 0, more_take = 0, more_give = 0;
    for (int b = tid + kPlanThreads; b < job.batch; b += kPlanThreads) {
      const Change c = change_of(job, b);
      if (!c.good) atomicMin(&bad_seq, b);
      const Sums s = sums_of(c, job, pool);
      more_tokens += s.tokens;
      more_take += s.take;
      more_give += s.give;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      more_tokens += __shfl_xor_sync(0xffffffffu, more_tokens, o);
      more_take += __shfl_xor_sync(0xffffffffu, more_take, o);
      more_give += __shfl_xor_sync(0xffffffffu, more_give, o);
    }
    if (lane == 0) {
      all_tokens[warp] = more_tokens;
      all_take[warp] = more_take;
      all_give[warp] = more_give;
    }
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kPlanWarps; ++w) {
      tokens += all_tokens[w];
      take += all_take[w];
      give += all_give[w];
    }
  }
  int code = MOQAE_OK, d0 = -1, d1 = -1;
  if (!sound || give > pool.n_pages - n_free) {
    code = MOQAE_ERR_CORRUPT_TABLE;
  } else if (bad_seq != 0x7fffffff) {
    code = MOQAE_ERR_CORRUPT_TABLE;
    d0 = bad_seq;
  } else if (tokens > job.n_rows) {
    code = MOQAE_ERR_INVALID_ARG;
    d1 = static_cast<int>(min(tokens, 0x7fffffffll));
  } else if (take > n_free) {
    code = MOQAE_ERR_POOL_FULL;
    d0 = static_cast<int>(min(take, 0x7fffffffll));
    d1 = n_free;
  }
  const bool go = code == MOQAE_OK;
  if (blockIdx.x == 0 && tid == 0) {
    if (!go) paged_status(job.status, code, d0, d1);
    job.cu_q[0] = 0;
  }

  // ---- rows and pages, 256 sequences at a time ----
  Sums before{0, 0, 0};
  for (int base = 0; base < job.batch; base += kPlanThreads) {
    const int b = base + tid;
    Change c = mine;
    if (base > 0) {
      c = change_of(job, b);
      own = sums_of(c, job, pool);
      to_here = scan(own, lane);
      __syncthreads();                           // the turn before is done with the arrays
      if (lane == 31) {
        warp_sum[0][warp] = to_here.tokens;
        warp_sum[1][warp] = to_here.take;
        warp_sum[2][warp] = to_here.give;
      }
      __syncthreads();
    }
    Sums in_front = before;
#pragma unroll
    for (int w = 0; w < kPlanWarps; ++w) {
      const Sums v{warp_sum[0][w], warp_sum[1][w], warp_sum[2][w]};
      if (w < warp) in_front = Sums{in_front.tokens + v.tokens, in_front.take + v.take, in_front.give + v.give};
      before = Sums{before.tokens + v.tokens, before.take + v.take, before.give + v.give};
    }
    tokens_to[tid] = in_front.tokens + to_here.tokens - own.tokens;
    take_to[tid] = in_front.take + to_here.take - own.take;
    give_to[tid] = in_front.give + to_here.give - own.give;
    past_of[tid] = c.past;
    have_of[tid] = c.have;
    want_of[tid] = c.want;
    if (tid == kPlanThreads - 1) {
      tokens_to[kPlanThreads] = before.tokens;
      take_to[kPlanThreads] = before.take;
      give_to[kPlanThreads] = before.give;
    }
    if (blockIdx.x == 0 && b < job.batch) job.cu_q[b + 1] = go ? in_front.tokens + to_here.tokens : 0;
    __syncthreads();
    if (!go) continue;
    for (int r = tokens_to[0] + first; r < tokens_to[kPlanThreads]; r += step) {
      const int i = find_in(tokens_to, kPlanThreads, r);
      job.positions[r] = past_of[i] + r - tokens_to[i];
      job.seq[r] = base + i;
    }
    // pages: kBatch at a time, so that their trips overlap
    for (int k0 = take_to[0] + first; k0 < take_to[kPlanThreads]; k0 += kBatch * step) {
      int page[kBatch];
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const int k = k0 + e * step;
        page[e] = k == first ? ahead : k < take_to[kPlanThreads] ? pool.ring[place(k)] : 0;
      }
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const int k = k0 + e * step;
        if (k >= take_to[kPlanThreads]) break;
        const int i = find_in(take_to, kPlanThreads, k), entry = have_of[i] + k - take_to[i];
        if (page[e] < 0 || page[e] >= pool.n_pages) paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, base + i, entry);
        job.table[static_cast<long long>(base + i) * job.max_pages + entry] = page[e];
      }
    }
    for (int k0 = give_to[0] + first; k0 < give_to[kPlanThreads]; k0 += kBatch * step) {
      int page[kBatch];
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const int k = min(k0 + e * step, give_to[kPlanThreads] - 1), i = find_in(give_to, kPlanThreads, k);
        page[e] = job.table[static_cast<long long>(base + i) * job.max_pages + want_of[i] + k - give_to[i]];
      }
#pragma unroll
      for (int e = 0; e < kBatch; ++e) {
        const int k = k0 + e * step;
        if (k >= give_to[kPlanThreads]) break;
        if (page[e] < 0 || page[e] >= pool.n_pages) {
          const int i = find_in(give_to, kPlanThreads, k);
          paged_status(job.status, MOQAE_ERR_CORRUPT_TABLE, base + i, want_of[i] + k - give_to[i]);
        }
        pool.ring[place(n_free + k)] = page[e];  // behind the free ones: never one that this call takes
      }
    }
  }
  for (int r = (go ? static_cast<int>(tokens) : 0) + first; r < job.n_rows; r += step) job.positions[r] = job.seq[r] = -1;

  // ---- lengths and the pool's state, when every CTA has read them ----
  __syncthreads();
  if (gridDim.x > 1) {
    if (tid == 0) {
      __threadfence();
      last = atomicInc(reinterpret_cast<unsigned*>(pool.state_out) + 2, gridDim.x - 1) == gridDim.x - 1;
    }
    __syncthreads();
    if (!last) return;
  }
  if (tid < job.batch) job.kv_len[tid] = go ? mine.total : mine.given;
  for (int b = tid + kPlanThreads; b < job.batch; b += kPlanThreads) {
    const int past = job.past[b];
    job.kv_len[b] = go ? max(past + job.n_new[b], 0) : past;
  }
  if (tid == 0) {
    const long long at = static_cast<long long>(head) + take;
    pool.state_out[0] = go ? static_cast<int>(at >= pool.n_pages && pool.n_pages > 0 ? at - pool.n_pages : at) : head;
    pool.state_out[1] = go ? static_cast<int>(n_free - take + give) : n_free;
  }
}

}  // namespace

cudaError_t launch_paged_plan(const PlanJob& job, const PoolView& pool, cudaStream_t st) {
  const int sms = sm_count_of_current_device();
  const long long ctas = (static_cast<long long>(job.n_rows) + kRowsPerCta - 1) / kRowsPerCta;
  return launch_early(paged_plan_kernel, static_cast<unsigned>(ctas < 1 ? 1 : (ctas > sms ? sms : ctas)), kPlanThreads, 0, st, job, pool);
}

}  // namespace moqae
