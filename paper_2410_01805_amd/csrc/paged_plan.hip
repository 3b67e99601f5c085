// Block tables and slot maps of one serving step from the requests' lengths (locret_paged_plan).
//
// Whole numbers only.  With held = pages of a request's units, and over requests in their order
//   B_r = sum of held over the finished ones before r:   page p of finished request r goes to free_pages[n_free + B_r + p]
//   W_r = sum of the pages wanted before r:               page number held_r + i of request r is free_pages[F - 1 - W_r - i], F = all free
//   N_r = sum of new tokens before r:                     its token i is token N_r + i, at position len_r + i
// so everything follows from three prefix sums over at most 4096 requests, which one workgroup forms in registers and LDS
// (4 requests a thread).  Pages and tokens are then dealt out to threads one by one, each finding its request by bisection.  Bound by latency: a
// step of 48 requests moves a kilobyte.  Up to PLAN_ONE tokens the same workgroup writes tables and slots too; more of them (prompts)
// are written by a second launch over all CUs, whose workgroups form the sums of W and N again from what the first one left (lens_out and
// cu_new give the lengths before the step), so that no workspace is needed and the lengths may be updated in place.
#include "paged.h"

namespace locret {

constexpr int PLAN_MAX_THREADS = 1024, PLAN_IPT = PAGED_MAX_REQS / PLAN_MAX_THREADS;
constexpr int PLAN_ONE = 4096;
constexpr int FILL_THREADS = 256, FILL_TOKENS = 4 * FILL_THREADS;

struct PlanSmem {
  int len[PAGED_MAX_REQS];          // units before the step (0 where the request is finished)
  int cu[PAGED_MAX_REQS + 1];       // N_r
  int want[PAGED_MAX_REQS + 1];     // W_r
  uint32_t part[4 * PLAN_MAX_THREADS / 64];
};

__device__ __forceinline__ int pages_of(int units, int shift) { return (int)(((int64_t)units + (1 << shift) - 1) >> shift); }

// Table entries: pages [i0, n_pages) of the step in steps of i_step; slots of tokens t0 .. t1 - 1, four in a row a thread.
__device__ __forceinline__ void plan_fill(const PagedPlan& p, const PlanSmem& s, int n_all_free, int i0, int i_step, int t0, int t1) {
  const int n_new_pages = s.want[p.n_req], total = s.cu[p.n_req];
#pragma unroll 2
  for (int i = i0; i < n_new_pages; i += i_step) {
    const int r = last_at_or_before(s.want, p.n_req, i);
    p.table[(int64_t)r * p.max_pages + pages_of(s.len[r], p.page_shift) + (i - s.want[r])] = p.free_pages[n_all_free - 1 - i];
  }
  const int t_step = 4 * (int)blockDim.x;
  for (int t = t0; t < t1; t = t1 - t > t_step ? t + t_step : t1) {      // (max_tokens may be the largest number)
    int slot[4], pos[4], r = t < total ? last_at_or_before(s.cu, p.n_req, t) : 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      slot[e] = -1;
      pos[e] = 0;
      if (t + e < total) {
        while (s.cu[r + 1] <= t + e) ++r;
        pos[e] = s.len[r] + (t + e - s.cu[r]);
        const int page = pos[e] >> p.page_shift, i = page - pages_of(s.len[r], p.page_shift);
        const int id = i < 0 ? p.table[(int64_t)r * p.max_pages + page] : p.free_pages[n_all_free - 1 - s.want[r] - i];
        // (else the table or the list was not the pool's)
        if (id >= 0 && id < p.n_pages) slot[e] = (id << p.page_shift) | (pos[e] & ((1 << p.page_shift) - 1));
      }
    }
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (t + e < t1) {
        p.slots[t + e] = slot[e];
        p.positions[t + e] = pos[e];
      }
  }
}

__global__ __launch_bounds__(PLAN_MAX_THREADS) void plan_kernel(PagedPlan p, int ipt, int fill) {
  __shared__ PlanSmem s;
  const int tid = threadIdx.x, nt = blockDim.x;
  const int most = p.max_pages << p.page_shift;
  int len[PLAN_IPT], add[PLAN_IPT], held[PLAN_IPT];    // add: tokens asked for, -1 finished
  uint32_t mine[4] = {0, 0, 0, 0}, before[4], all[4];  // pages given back, pages wanted, tokens; requests that give back
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    const int r = tid * ipt + u;
    len[u] = add[u] = held[u] = 0;
    if (u < ipt && r < p.n_req) {
      len[u] = min(max(p.lens[r], 0), most);
      add[u] = p.n_new[r];
      held[u] = pages_of(len[u], p.page_shift);
      if (add[u] < 0) { add[u] = -1; mine[0] = add_sat(mine[0], held[u]); mine[3] += held[u] > 0; }
      else if (add[u] > most - len[u]) add[u] = 0;
      if (add[u] > 0) {
        mine[1] = add_sat(mine[1], pages_of(len[u] + add[u], p.page_shift) - held[u]);
        mine[2] = add_sat(mine[2], add[u]);
      }
    }
  }
  const int n_free = min(max(p.n_free[0], 0), p.n_pages);
  block_exclusive<4>(mine, before, all, s.part);
  const int n_all_free = (int)min(add_sat(n_free, all[0]), (uint32_t)p.n_pages);
  if (all[0] > 0) {
    // s.cu and s.want hold the requests that give pages back, and B_r, meanwhile.  A wavefront takes 256 pages: one bisection, four loads on their
    // way together (26 requests of 12.7 thousand pages 5.4 us; with a bisection over all requests for every page 10).
    uint32_t b = before[0], k = before[3];
#pragma unroll
    for (int u = 0; u < PLAN_IPT; ++u)
      if (add[u] < 0 && held[u] > 0) {
        s.cu[k] = tid * ipt + u;
        s.want[k++] = (int)min(b, (uint32_t)INT32_MAX);
        b = add_sat(b, held[u]);
      }
    __syncthreads();
    const int n = n_all_free - n_free, n_back = (int)all[3];
    for (int i0 = (tid >> 6) * 256; i0 < n; i0 += nt * 4) {
      int j = last_at_or_before(s.want, n_back, i0), id[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = min(i0 + e * 64 + (tid & 63), n - 1);
        while (j + 1 < n_back && s.want[j + 1] <= i) ++j;
        id[e] = p.table[(int64_t)s.cu[j] * p.max_pages + (i - s.want[j])];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (i0 + e * 64 + (tid & 63) < n) p.free_pages[n_free + i0 + e * 64 + (tid & 63)] = id[e];
    }
    __syncthreads();
  }
  // What fits is a prefix of the requests, since both sums only grow.
  uint32_t served[2] = {0, 0};                         // pages and tokens of this thread's served ones
  bool fits = true;
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    if (add[u] < 0) len[u] = held[u] = 0;
    if (add[u] > 0) {
      const uint32_t pages = pages_of(len[u] + add[u], p.page_shift) - held[u];
      fits = fits && add_sat(before[1], served[0] + pages) <= (uint32_t)n_all_free && add_sat(before[2], add_sat(served[1], add[u])) <= (uint32_t)p.max_tokens;
      if (!fits) add[u] = 0;
      else { served[0] += pages; served[1] += add[u]; }
    }
  }
  // A thread behind the first request that did not fit has served nothing.
  uint32_t at[2] = {before[1], before[2]}, sum[2] = {all[1], all[2]};
  if (all[1] > (uint32_t)n_all_free || all[2] > (uint32_t)p.max_tokens) {      // (the same in the whole workgroup)
    __syncthreads();                                   // s.part is free again
    block_exclusive<2>(served, at, sum, s.part);
  }
#pragma unroll
  for (int u = 0; u < PLAN_IPT; ++u) {
    const int r = tid * ipt + u;
    if (u < ipt && r < p.n_req) {
      s.len[r] = len[u];
      s.want[r] = (int)at[0];
      s.cu[r] = (int)at[1];
      p.cu_new[r] = (int)at[1];
      if (add[u] > 0) {
        at[0] += pages_of(len[u] + add[u], p.page_shift) - held[u];
        at[1] += add[u];
      }
      p.lens_out[r] = len[u] + max(add[u], 0);
    }
  }
  if (tid == 0) {
    s.want[p.n_req] = (int)sum[0];
    s.cu[p.n_req] = (int)sum[1];
    p.cu_new[p.n_req] = (int)sum[1];
    p.n_free_out[0] = n_all_free - (int)sum[0];
  }
  if (!fill) return;
  __syncthreads();
  plan_fill(p, s, n_all_free, tid, nt, 4 * tid, p.max_tokens);
}

// Tables and slots of a long step: every workgroup takes a share of the tokens and of the pages.
__global__ __launch_bounds__(FILL_THREADS) void plan_fill_kernel(PagedPlan p) {
  __shared__ PlanSmem s;
  const int tid = threadIdx.x;
  const int ipt = (p.n_req + FILL_THREADS - 1) / FILL_THREADS;
  uint32_t want = 0, all;
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < p.n_req) {
      const int c0 = p.cu_new[r], c1 = p.cu_new[r + 1], after = p.lens_out[r];
      s.len[r] = after - (c1 - c0);
      s.cu[r] = c0;
      const int pages = pages_of(after, p.page_shift) - pages_of(after - (c1 - c0), p.page_shift);
      s.want[r] = pages;
      want += pages;
      if (r == p.n_req - 1) s.cu[p.n_req] = c1;
    }
  }
  uint32_t before = block_exclusive(want, s.part, all);
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < p.n_req) { const int pages = s.want[r]; s.want[r] = (int)before; before += pages; }
  }
  if (tid == 0) s.want[p.n_req] = (int)all;
  __syncthreads();
  const int n_all_free = p.n_free_out[0] + (int)all;
  const int t0 = blockIdx.x * FILL_TOKENS, left = p.max_tokens - t0;
  plan_fill(p, s, n_all_free, blockIdx.x * FILL_THREADS + tid, gridDim.x * FILL_THREADS, t0 + 4 * tid, t0 + min(left, FILL_TOKENS));
}

void launch_paged_plan(const PagedPlan& p, hipStream_t st) {
  const bool one = p.max_tokens <= PLAN_ONE || p.n_req == 0;
  const int threads = p.n_req <= 256 ? 256 : PLAN_MAX_THREADS;
  const int ipt = p.n_req > 0 ? (p.n_req + threads - 1) / threads : 1;
  plan_kernel<<<1, threads, 0, st>>>(p, ipt, one ? 1 : 0);
  if (!one) plan_fill_kernel<<<(unsigned)(((int64_t)p.max_tokens + FILL_TOKENS - 1) / FILL_TOKENS), FILL_THREADS, 0, st>>>(p);
}

}  // namespace locret
