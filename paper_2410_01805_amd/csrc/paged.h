// Internal interface of the paged entry points (paged_api.hip) to their kernels.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace locret {

struct PagedDims {
  int h, h_kv, g, d;
  int bf16;
  int page_shift;       // log2 of the page size
  int n_pages;
  int max_pages;
  int window, n_sink;   // window 0: none
  float scale;
};

// One step's bookkeeping (locret_paged_plan).
struct PagedPlan {
  int n_req, max_tokens, page_shift, n_pages, max_pages;
  const int32_t* lens;
  const int32_t* n_new;
  int32_t* lens_out;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* n_free_out;
  int32_t* cu_new;
  int32_t* slots;
  int32_t* positions;
};
constexpr int PAGED_MAX_REQS = 4096;
void launch_paged_plan(const PagedPlan& p, hipStream_t st);

struct PagedRows {
  int T;
  const void* q;
  const void* k;
  const void* v;
  int64_t q_tok, q_head, k_tok, k_head, v_tok, v_head;      // strides in elements
  const int32_t* positions;
  const int32_t* slots;
  const double* freq;
  int rot, interleaved;
  float amplitude;
  const float* q_weight;
  const float* k_weight;
  float eps;
  void* q_out;
  void* K;
  void* V;
};
void launch_paged_append(const PagedDims& D, const PagedRows& a, hipStream_t st);

// Attention of T query tokens over pages.  cu NULL: token t is the last unit of request t (T = n_req).
struct PagedAttn {
  int n_req, T;
  const void* q;
  const void* K;
  const void* V;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
  void* out;
  float* lse;       // or NULL
  void* ws;
};
void launch_paged_decode(const PagedDims& D, const PagedAttn& a, hipStream_t st);
size_t paged_decode_workspace(const PagedDims& D, int max_reqs);
void launch_paged_prefill(const PagedDims& D, const PagedAttn& a, hipStream_t st);      // bf16
size_t paged_prefill_workspace(const PagedDims& D);
void launch_paged_prefill_f32(const PagedDims& D, const PagedAttn& a, hipStream_t st);
size_t paged_prefill_f32_workspace(const PagedDims& D);

// A length as the kernels take it.
__device__ __forceinline__ int paged_len(const int32_t* lens, int r, int max_pages, int page_shift) {
  return min(max(lens[r], 0), max_pages << page_shift);
}

__device__ __forceinline__ int64_t shfl_up64(int64_t x, int by) {
  const int lo = __shfl_up((int)(uint32_t)x, by, 64), hi = __shfl_up((int)(x >> 32), by, 64);
  return (int64_t)(((uint64_t)(uint32_t)hi << 32) | (uint32_t)lo);
}

// Exclusive sums of x over the workgroup's threads; `total` gets the sum of all.  part: one entry a wavefront, not in use by others
// until the next barrier but one.
__device__ __forceinline__ int64_t block_exclusive(int64_t x, int64_t* part, int64_t& total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, nw = blockDim.x >> 6;
  int64_t s = x;
#pragma unroll
  for (int by = 1; by < 64; by <<= 1) {
    const int64_t y = shfl_up64(s, by);
    if (lane >= by) s += y;
  }
  if (lane == 63) part[wave] = s;
  __syncthreads();
  int64_t before = 0;
  total = 0;
  for (int w = 0; w < nw; ++w) {
    const int64_t y = part[w];
    if (w < wave) before += y;
    total += y;
  }
  return before + s - x;
}

// An entry of cu_new as the kernels take it.
__device__ __forceinline__ int paged_cu(const int32_t* cu, int r, int T) { return min(max(cu[r], 0), T); }

}  // namespace locret
