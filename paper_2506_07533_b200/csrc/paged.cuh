// Shared declarations of the paged 16-bit cache: kernel-side views and launchers.
#pragma once

#include <atomic>

#include <cuda_bf16.h>

#include "common.cuh"

namespace moqae {

// A cache of 16-bit pages as the kernels see it (passed by value).
struct PagedView {
  uint16_t* k;
  uint16_t* v;
  long long k_page, k_head, k_slot, v_page, v_head, v_slot;   // element strides
  const int32_t* table;
  const int32_t* kv_len;
  int32_t* status;                                             // may be null
  int n_pages, page_size, page_shift, n_kv_heads, batch, max_pages, dtype;
};

// rows [n][heads][128]
struct RowsView {
  uint16_t* data;
  long long token, head;
  int n_heads;
};

struct RopeView {
  const float* cos_sin;
  const uint16_t* q_weight;
  const uint16_t* k_weight;
  int n_positions, rot_dim, interleaved;
  float eps;
};

constexpr int kMaxQueryTokens = 1 << 24;     // of one call, so that its rows and their tiles count in 32 bits

// A workspace of the attention calls starts with this many counters, which every completed call leaves at zero;
// what follows is plain scratch.  All calls lay it out alike, so calls of any sizes can share one buffer.
constexpr int kWorkCounters = 1 << 18;
constexpr long long kWorkCounterBytes = 4ll * kWorkCounters;

struct AttnOptions {
  const float* slopes;
  const int32_t* prefix_len;
  float scale, cap;
  int window;
};

__device__ __forceinline__ void paged_status(int32_t* status, int code, int d0, int d1) {
  if (status) set_status(status, code, d0, d1);
}

// kv_len[b]; a length that its row of the table cannot hold counts as 0.
__device__ __forceinline__ int paged_len(const PagedView& pv, int b, bool report) {
  const int n = pv.kv_len[b];
  if (n >= 0 && n <= static_cast<long long>(pv.max_pages) * pv.page_size) return n;
  if (report) paged_status(pv.status, MOQAE_ERR_CORRUPT_TABLE, b, -1);
  return 0;
}

// tanh(z) = z P(z^2) for |z| <= 1 (minimax fit of tanh(z) / z, own, relative error 6e-7); beyond, where the
// difference loses nothing, 1 - 2 / (exp(2 z) + 1).  tanh.approx has 2^-11, which a cap of 30 would carry into the weights.
__host__ __device__ constexpr float tanh_coef(int k) {
  return k == 0 ? 0.99999940395f : k == 1 ? -0.33329042792f : k == 2 ? 0.13281433284f : k == 3 ? -0.05160567537f : k == 4 ? 0.01674311422f : -0.00306706037f;
}
// The same up to 1/2 with four coefficients (5.5e-7).
__host__ __device__ constexpr float tanh_coef_near(int k) {
  return k == 0 ? 0.999999463558f : k == 1 ? -0.333263188601f : k == 2 ? 0.131902962923f : -0.0444022081792f;
}
__device__ __forceinline__ float tanh_far(float z) {
  float e, r;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(e) : "f"(z * 2.8853900818f));     // 2 log2(e)
  asm("rcp.approx.ftz.f32 %0, %1;\n" : "=f"(r) : "f"(e + 1.0f));
  return fmaf(-2.0f, r, 1.0f);
}
__device__ __forceinline__ float tanh_of(float z) {
  const float u = z * z;
  const float near = z * fmaf(fmaf(fmaf(fmaf(fmaf(tanh_coef(5), u, tanh_coef(4)), u, tanh_coef(3)), u, tanh_coef(2)), u, tanh_coef(1)), u, tanh_coef(0));
  return fabsf(z) <= 1.0f ? near : tanh_far(z);
}

// 16-bit element <-> float, in the dtype of the template
template <bool BF16> __device__ __forceinline__ float half_bits_to_float(uint16_t u) {
  return BF16 ? __uint_as_float(static_cast<uint32_t>(u) << 16) : __half2float(__ushort_as_half(u));
}
template <bool BF16> __device__ __forceinline__ float2 pair_to_float2(uint32_t u) {
  if (BF16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xffff0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
template <bool BF16> __device__ __forceinline__ uint32_t float2_to_pair(float a, float b) {
  if (BF16) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __half2 h = __floats2half2_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}

// Let `kernel` use `bytes` of dynamic shared memory on the current device; the driver is asked once per device
// (`done`: one bit per device, a variable of the kernel's own).
template <typename K> inline cudaError_t allow_shared_memory(K* kernel, size_t bytes, std::atomic<unsigned long long>& done) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const unsigned long long bit = dev >= 0 && dev < 64 ? 1ull << dev : 0ull;
  if (bit && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(bytes));
  if (e == cudaSuccess) done.fetch_or(bit, std::memory_order_release);
  return e;
}

// Launch so that the grid may be set up while the kernel before it on the stream is finishing.  The kernel starts with
// after_previous() in every thread, before it touches global memory, so the order of the stream holds.  In a loop of
// small calls this is 0.5 us (norm and rotation of one token, 3.8 -> 3.3) to 2.5 us (decode, 14.5 -> 11.9) of each.
template <typename... P, typename... A>
inline cudaError_t launch_early(void (*kernel)(P...), unsigned grid, unsigned block, size_t smem, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(block);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}
__device__ __forceinline__ void after_previous() { asm volatile("griddepcontrol.wait;\n" ::: "memory"); }

cudaError_t launch_norm_rope(const RopeView& rope, int dtype, const RowsView& q, const RowsView& k, const RowsView& q_out,
                             const RowsView& k_out, const int32_t* positions, int n_tokens, int32_t* status, cudaStream_t st);
cudaError_t launch_paged_append(const PagedView& pv, const RopeView& rope, const RowsView& q, const RowsView& q_out,
                                const RowsView& k, const RowsView& v, const int32_t* positions, const int32_t* seq, int n_tokens,
                                cudaStream_t st);
bool paged_decode_fits(const PagedView& pv);        // sizes that the kernel's counters and 32-bit sums hold
long long paged_decode_workspace_bytes(int group);
cudaError_t launch_paged_decode(const PagedView& pv, const RowsView& q, const RowsView& out, const AttnOptions& opt, void* workspace,
                                cudaStream_t st);
constexpr int kFewRows = 16;                 // see paged_few_rows
bool paged_few_rows(const PagedView& pv, int group, int n_tokens);
long long paged_few_workspace_bytes();
cudaError_t launch_paged_few(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                             const AttnOptions& opt, void* workspace, cudaStream_t st);
long long paged_prefill_workspace_bytes(const PagedView& pv, int group, int n_tokens);
cudaError_t launch_paged_prefill(const PagedView& pv, const RowsView& q, const int32_t* cu_q, int n_tokens, const RowsView& out,
                                 const AttnOptions& opt, void* workspace, cudaStream_t st);

}  // namespace moqae
