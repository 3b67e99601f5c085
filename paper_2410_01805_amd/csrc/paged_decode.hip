// Attention of one new token per request over its pages (locret_paged_decode): split over the keys, joined by a second launch.
//   s_j = scale q . k_j,  out = sum_j e^(s_j - M) v_j / L,  L = sum_j e^(s_j - M),  lse = M + ln L     over the visible keys j
// Every key and value is read once for all query heads of its group, so HBM is the bound; both products run on the matrix cores with
// the heads of a group (16 at a time) as one side of a 16 x 16 tile, so that the arithmetic stays far below that bound for any group.
//
// Work: an item is (request, KV head, 16 query heads), a unit four tiles of 32 keys of an item (one a wavefront).  Lengths are known on the device only, and
// differ, so the units of all items are laid end to end and every workgroup takes the same number of them, rounded up, as many workgroups
// as the chip holds at once (with a unit or two for each the last ones have none: 1032 units are two each for 516 of 768).  Each workgroup forms the sums of units over the requests by itself (at most 4096 numbers from L2, one scan) and
// finds its first unit by bisection.  An item that one workgroup holds whole is written by it; of one that is cut, every
// workgroup leaves maximum, sum and sum of values (two such pieces a workgroup at most), and the second launch, which has a workgroup
// per request and head, joins them in the order of the keys.  Results depend on no order of execution.
//
// Tiles go from memory to registers in the layout of the operands (paged_tile.h; float products are those of 32 bits):
// S^T = K Q^T has keys as rows, in an order in which a lane's accumulators are the eight keys whose probabilities it gives to
// O = P V.  The next keys are requested as soon as the logits are formed, the next values after their product, page numbers a unit
// earlier.  Probabilities of bf16 layers become two bf16 factors each; maximum, sum and accumulators are 32-bit.  The maximum moves only when a logit
// exceeds it by 8 binary orders.  What is not seen is taken out by selection: its logit before the maximum, its value before the product.
#include "paged.h"
#include "paged_tile.h"

namespace locret {

constexpr int PD_THREADS = 256, PD_NW = 4, PD_HEADS = 16;
constexpr float PD_RESCALE_LOG2 = 8.f;

// Workgroups a CU: what registers allow without spilling.
__host__ __device__ constexpr int paged_decode_occupancy(bool bf16, int d) { return bf16 ? (d >= 96 ? 3 : 4) : (d >= 96 ? 2 : 3); }
static int paged_decode_workgroups(const PagedDims& D) { return 256 * paged_decode_occupancy(D.bf16, D.d); }

// The visible keys of a request in tiles of 32: sinks, then from the first tile with a key in the window on; four tiles are a unit.
struct PagedSpan {
  int n, w0, ns, wb, st, total;      // units in the cache, first key of the window, sinks in front of it, its first tile, tiles of sinks; units
};
__device__ __forceinline__ PagedSpan paged_span(int n, int window, int n_sink) {
  PagedSpan s;
  s.n = n;
  s.w0 = window ? max(0, n - window) : 0;
  s.ns = min(n_sink, s.w0);
  s.wb = s.w0 & ~31;
  s.st = (int)(((uint32_t)s.ns + 31) / 32);
  s.total = (s.st + (int)(((uint32_t)(n - s.wb) + 31) / 32) + PD_NW - 1) / PD_NW;
  return s;
}

// Units a workgroup takes.  (Divisions of 64 bits are a hundred instructions in front of the first load; sums of units that need them are rare.)
__device__ __forceinline__ int64_t units_per_wg(int64_t all, int n_wg) {
  if (all < (int64_t)1 << 30) return ((uint32_t)all + n_wg - 1) / (uint32_t)n_wg;
  return (all + n_wg - 1) / n_wg;
}
// The item and tile of unit `in` of a request of t units a head.
__device__ __forceinline__ void unit_in_request(int64_t in, int t, int& item, int& tile) {
  int i, k;
  if (in < (int64_t)1 << 31) {
    i = (int)((uint32_t)in / (uint32_t)t);
    k = (int)((uint32_t)in - (uint32_t)i * (uint32_t)t);
  } else {
    i = (int)(in / t);
    k = (int)(in % t);
  }
  item = __builtin_amdgcn_readfirstlane(i);
  tile = __builtin_amdgcn_readfirstlane(k);
}
// The request, item and tile of unit u (below the number of units); the same in the whole wavefront.
__device__ __forceinline__ void find_unit(const int32_t* first, int n_req, int items, int64_t u, int& r, int& item, int& tile) {
  int lo = 0, hi = n_req - 1;
  while (lo < hi) {                                        // the last request that begins at or before u
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)first[mid] * items <= u) lo = mid; else hi = mid - 1;
  }
  r = __builtin_amdgcn_readfirstlane(lo);
  unit_in_request(u - (int64_t)first[lo] * items, first[lo + 1] - first[lo], item, tile);
}

// Where a piece lies in the workspace.
struct PagedPieces {
  int32_t* first;     // [n_req + 1] units of one head before each request (their sum fits by the configuration's limits)
  float2* ml;         // [2 workgroups][16] maximum (log2) and sum
  float* o;           // [2 workgroups][16][d]
};
__host__ __device__ inline PagedPieces paged_pieces(void* ws, int n_req, int n_wg) {
  PagedPieces p;
  p.first = (int32_t*)ws;
  p.ml = (float2*)((char*)ws + (((size_t)(n_req + 1) * 4 + 255) & ~(size_t)255));
  p.o = (float*)(p.ml + (size_t)2 * n_wg * PD_HEADS);
  return p;
}
size_t paged_decode_workspace(const PagedDims& D, int max_reqs) {
  const int n_wg = paged_decode_workgroups(D), rows = D.g < PD_HEADS ? D.g : PD_HEADS;
  return (size_t)((char*)paged_pieces(nullptr, max_reqs, n_wg).o - (char*)nullptr) + (size_t)2 * n_wg * rows * D.d * sizeof(float);
}

template <typename T, int D, bool SMALL>
__global__ __launch_bounds__(PD_THREADS, paged_decode_occupancy(sizeof(T) == 2, D)) void paged_decode_kernel(PagedAttn a, const int32_t* __restrict__ table, PagedDims Dm,
                                                                                           int passes, int ipt) {
  typedef typename PagedTileOf<T, D, SMALL>::type Tile;
  constexpr int NV = D / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float2 wml[PD_NW][PD_HEADS];
  __shared__ uint32_t scan[PD_NW];
  float* sets = (float*)smem;                              // [wavefront][rows][D]
  const int rows_max = min(Dm.g, PD_HEADS);
  int32_t* first = (int32_t*)(smem + (size_t)PD_NW * rows_max * D * sizeof(float));
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, kg = lane >> 4;
  const PagedPieces pc = paged_pieces(a.ws, a.n_req, gridDim.x);

  // Units of one head before every request.  Up to 64 requests: one a lane, in every wavefront by itself, without LDS and barriers (16K keys of one request
  // 21.4 -> 21.0 us, a few f32 requests 11.5 -> 10.9); more: in LDS.
  const bool few = a.n_req <= 64;
  const int items = Dm.h_kv * passes;
  uint32_t total;
  int my_len = 0, my_units = 0, my_first = 0;
  if (few) {
    if (lane < a.n_req) {
      my_len = paged_len(a.lens, lane, Dm.max_pages, Dm.page_shift);
      my_units = paged_span(my_len, Dm.window, Dm.n_sink).total;
    }
    const int upto = (int)wave_inclusive(my_units);
    total = __builtin_amdgcn_readlane(upto, 63);
    my_first = upto - my_units;
    if (blockIdx.x == 0 && wave == 0 && lane < a.n_req) {
      pc.first[lane + 1] = upto;
      if (lane == 0) pc.first[0] = 0;
    }
  } else {
    uint32_t mine = 0;
    for (int u = 0; u < ipt; ++u) {
      const int r = tid * ipt + u;
      if (r < a.n_req) {
        const int t = paged_span(paged_len(a.lens, r, Dm.max_pages, Dm.page_shift), Dm.window, Dm.n_sink).total;
        first[r + 1] = t;
        mine += t;
      }
    }
    uint32_t before = block_exclusive(mine, scan, total);
    for (int u = 0; u < ipt; ++u) {
      const int r = tid * ipt + u;
      if (r < a.n_req) {
        before += first[r + 1];
        first[r + 1] = (int)before;
        if (blockIdx.x == 0) pc.first[r + 1] = (int)before;
      }
    }
    if (tid == 0) {
      first[0] = 0;
      if (blockIdx.x == 0) pc.first[0] = 0;
    }
    __syncthreads();
  }
  const int64_t all = (int64_t)total * items, per = units_per_wg(all, gridDim.x);
  int64_t u = per * blockIdx.x;
  const int64_t u_end = min(all, u + per);
  if (u >= u_end) return;
  int r, item, tile;
  if (few) {
    r = __popcll(__ballot(lane < a.n_req && (int64_t)my_first * items <= u)) - 1;      // (requests without units begin where the next one does)
    unit_in_request(u - (int64_t)__builtin_amdgcn_readlane(my_first, r) * items, __builtin_amdgcn_readlane(my_units, r), item, tile);
  } else {
    find_unit(first, a.n_req, items, u, r, item, tile);
  }
  const float c = Dm.scale * 1.4426950408889634f;
  const int shift = Dm.page_shift, page = 1 << shift;
  bool begun = false;                                      // this workgroup has left a piece already: the next one goes to the second place

  while (u < u_end) {
    const PagedSpan sp = paged_span(few ? __builtin_amdgcn_readlane(my_len, r) : __builtin_amdgcn_readfirstlane(paged_len(a.lens, r, Dm.max_pages, shift)), Dm.window,
                                    Dm.n_sink);
    const int m = item / passes, hp = item % passes;
    const int j0 = m * Dm.g + hp * PD_HEADS, ng = min(PD_HEADS, Dm.g - hp * PD_HEADS);
    const int t_end = (int)min((int64_t)sp.total, tile + (u_end - u));
    const paged_const_i32 row = (paged_const_i32)(uint64_t)(table + (int64_t)r * Dm.max_pages);
    const T* Kp = (const T*)a.K + (int64_t)m * page * D;
    const T* Vp = (const T*)a.V + (int64_t)m * page * D;
    const int64_t page_stride = (int64_t)Dm.h_kv * page * D;

    // tile t of this wavefront: its keys kb .. kb + 31 of [lo, hi) and its two page numbers
    struct Place { int kb, lo, hi, id0, id1; };
    auto place = [&](int t) __attribute__((always_inline)) {
      Place p;
      const int i = t * PD_NW + wave;
      const bool sink = i < sp.st;
      p.kb = sink ? i * 32 : sp.wb + (i - sp.st) * 32;
      p.lo = sink ? 0 : sp.w0;
      p.hi = sink ? sp.ns : sp.n;
      p.id0 = p.id1 = -1;
      if (p.kb < p.hi) {
        p.id0 = row[p.kb >> shift];
        p.id1 = SMALL ? (p.kb + 16 < p.hi ? row[(p.kb >> 4) + 1] : -1) : p.id0;
      }
      return p;
    };
    auto address = [&](const T* base, const Place& p, const T*& lo, const T*& hi) __attribute__((always_inline)) {
      // (a number that is not the pool's: page 0, whose rows are masked then)
      const int i0 = (unsigned)p.id0 < (unsigned)Dm.n_pages ? p.id0 : 0, i1 = (unsigned)p.id1 < (unsigned)Dm.n_pages ? p.id1 : 0;
      lo = base + i0 * page_stride + (p.kb & (page - 1)) * D;
      hi = SMALL ? base + i1 * page_stride - 16 * D : lo;
    };

    typename Tile::q_t qb[Tile::NQ];
    Tile::load_q((const T*)a.q + ((int64_t)r * Dm.h + j0 + min(n, ng - 1)) * D, n < ng, qb);
    Tile tl;
    dec_f32x4 o[NV];
    float mrun, lrun;
    for (bool fine = Tile::HAS_FINE;;) {                   // (a second time where a value is not finite, see PagedTileBf16::add)
      Place p = place(tile);
      if (p.kb < p.hi) {
        const T *lo, *hi;
        address(Kp, p, lo, hi);
        tl.load_k(lo, hi);
        address(Vp, p, lo, hi);
        tl.load_v(lo, hi);
      }
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
      mrun = -INFINITY;
      lrun = 0.f;
      Place nx = place(min(tile + 1, t_end - 1));
      for (int t = tile; t < t_end; ++t) {
        const Place nn = place(min(t + 2, t_end - 1));
        const bool work = p.kb < p.hi && p.kb + 32 > p.lo, more = t + 1 < t_end && nx.kb < nx.hi;
        dec_f32x4 s[2];
        float pr[8];
        if (p.kb < p.hi) tl.logits(qb, s);
        const T *klo, *khi;
        if (more) {
          address(Kp, nx, klo, khi);
          tl.load_k(klo, khi);
        }
        if (work) {
          uint32_t seen = 0xffu;
          if (p.kb < p.lo || p.kb + 32 > p.hi || (unsigned)p.id0 >= (unsigned)Dm.n_pages || (unsigned)p.id1 >= (unsigned)Dm.n_pages) {
            seen = 0;
            const int id = kg >= 2 ? p.id1 : p.id0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
              const int key = p.kb + 8 * kg + j;
              seen |= (key >= p.lo && key < p.hi && (unsigned)id < (unsigned)Dm.n_pages) ? 1u << j : 0u;
            }
            tl.clear_v(seen);
#pragma unroll
            for (int j = 0; j < 8; ++j) s[j >> 2][j & 3] = (seen >> j) & 1 ? s[j >> 2][j & 3] : -INFINITY;
          }
          float mx = -INFINITY;
#pragma unroll
          for (int j = 0; j < 8; ++j) mx = fmaxf(mx, s[j >> 2][j & 3]);
          mx *= c;
          if (__any((mx - mrun) > PD_RESCALE_LOG2)) {        // also true from -inf to a number
            mx = max_across_quarters(mx);                    // the four lanes of a column move together
            const bool up = (mx - mrun) > PD_RESCALE_LOG2;
            const float alpha = up ? __builtin_amdgcn_exp2f(mrun - mx) : 1.f;
            if (up) mrun = mx;
            lrun *= alpha;
#pragma unroll
            for (int rr = 0; rr < 4; ++rr) {
              const float ar = __shfl(alpha, 4 * kg + rr, 64);      // accumulator row 4 kg + rr is that head
#pragma unroll
              for (int i = 0; i < NV; ++i) o[i][rr] *= ar;
            }
          }
          const float ref = mrun == -INFINITY ? 0.f : mrun;  // (nothing seen yet, or every logit so far is -inf)
#pragma unroll
          for (int j = 0; j < 8; ++j) {
            pr[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], c, -ref));
            lrun += pr[j];
          }
          tl.add(pr, o, fine);
        }
        if (more) {
          address(Vp, nx, klo, khi);
          tl.load_v(klo, khi);
        }
        p = nx;
        nx = nn;
      }
      if (!fine) break;
      float z[4] = {0.f, 0.f, 0.f, 0.f};                   // 0 times a number, or not a number
#pragma unroll
      for (int i = 0; i < NV; ++i)
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) z[rr] = fmaf(o[i][rr], 0.f, z[rr]);
      const bool bad = !((z[0] + z[1]) + (z[2] + z[3]) == 0.f);
      if (!__any(bad)) break;
      fine = false;
    }
    lrun = sum_across_quarters(lrun);
    // ---- the wavefronts' results together ------------------------------------------------------------------------------
    int tid_ = tid;
    asm volatile("" : "+v"(tid_));                         // (what follows from it is formed here, not kept in registers over the tiles)
    const int n_ = tid_ & 15, kg_ = (tid_ & 63) >> 4;
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) {
      const int head = 4 * kg_ + rr;
      if (head < ng)
#pragma unroll
        for (int i = 0; i < NV; ++i) sets[(wave * rows_max + head) * D + n_ * NV + i] = o[i][rr];
    }
    if ((tid_ & 63) < PD_HEADS) wml[wave][n_] = make_float2(mrun, lrun);
    __syncthreads();
    const bool whole = tile == 0 && t_end == sp.total;
    const int64_t slot = 2 * (int64_t)blockIdx.x + (begun ? 1 : 0);
    for (int idx = tid_; idx < ng * (D / 4); idx += PD_THREADS) {
      const int head = idx / (D / 4), e = idx % (D / 4) * 4;
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < PD_NW; ++w) M = fmaxf(M, wml[w][head].x);
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < PD_NW; ++w) {
        const float2 ml = wml[w][head];
        // a wavefront whose maximum is -inf has seen nothing, or only logits of -inf or NaN: its sum says which
        const float wt = ml.x == -INFINITY ? (ml.y == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(ml.x - M);
        const float4 y = *(const float4*)&sets[(w * rows_max + head) * D + e];
        L = fmaf(wt, ml.y, L);
        if (wt != 0.f) { x.x = fmaf(wt, y.x, x.x); x.y = fmaf(wt, y.y, x.y); x.z = fmaf(wt, y.z, x.z); x.w = fmaf(wt, y.w, x.w); }
      }
      if (whole) {
        const int64_t at = (int64_t)r * Dm.h + j0 + head;
        const bool none = M == -INFINITY && L == 0.f;
        const float inv = none ? 0.f : 1.f / L;
        T* dst = (T*)a.out + at * D + e;
        Elem<T>::st(dst, none ? 0.f : x.x * inv);
        Elem<T>::st(dst + 1, none ? 0.f : x.y * inv);
        Elem<T>::st(dst + 2, none ? 0.f : x.z * inv);
        Elem<T>::st(dst + 3, none ? 0.f : x.w * inv);
        if (a.lse && e == 0) a.lse[at] = none ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
      } else {
        *(float4*)&pc.o[(slot * rows_max + head) * D + e] = x;
        if (e == 0) pc.ml[slot * PD_HEADS + head] = make_float2(M, L);
      }
    }
    begun = begun || !whole;
    __syncthreads();
    u += t_end - tile;
    tile = 0;
    if (++item == items) {
      item = 0;
      do ++r; while (u < u_end && (few ? __builtin_amdgcn_readlane(my_units, r) == 0 : first[r + 1] == first[r]));
    }
  }
}

// Joins the pieces of the items that were cut, and answers for requests that see nothing.  One workgroup per (head, request); its threads
// are dims / 4 x groups of pieces, each of which goes over every NP-th piece with a running maximum.
template <typename T, int D>
__global__ __launch_bounds__(PD_THREADS) void paged_decode_join_kernel(PagedAttn a, PagedDims Dm, int passes, int n_wg) {
  constexpr int E = D / 4, NP = PD_THREADS / E;
  __shared__ float4 so[NP][E];
  __shared__ float2 sml[NP];
  const int j = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, e = tid % E, g = tid / E;
  const PagedPieces pc = paged_pieces(a.ws, a.n_req, n_wg);
  const int f0 = pc.first[r], t = pc.first[r + 1] - f0;
  const int64_t at = (int64_t)r * Dm.h + j;
  if (t == 0) {
    if (g == 0)
      for (int i = 0; i < 4; ++i) Elem<T>::st((T*)a.out + at * D + e * 4 + i, 0.f);
    if (a.lse && tid == 0) a.lse[at] = -INFINITY;
    return;
  }
  const int items = Dm.h_kv * passes, in = j % Dm.g, item = j / Dm.g * passes + in / PD_HEADS, head = in % PD_HEADS, rows_max = min(Dm.g, PD_HEADS);
  const int64_t per = units_per_wg((int64_t)pc.first[a.n_req] * items, n_wg), u0 = (int64_t)f0 * items + (int64_t)item * t, u1 = u0 + t;
  const bool fits = u1 < (int64_t)1 << 31;
  const int w0 = fits ? (int)((uint32_t)u0 / (uint32_t)per) : (int)(u0 / per), w1 = fits ? (int)((uint32_t)(u1 - 1) / (uint32_t)per) : (int)((u1 - 1) / per);
  if (w0 == w1) return;
  // The first workgroup's piece lies in its second place if it had left one before: if its first unit is not the first of an item.
  const int64_t b0 = per * w0;
  bool second = false;
  if (b0 < u0) {
    int br, bi, bt;
    find_unit(pc.first, r + 1, items, b0, br, bi, bt);
    second = bt != 0;
  }
  float M = -INFINITY, L = 0.f;
  float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
  if (g < NP) {
    constexpr int B = 8;                                   // pieces requested together: each is a trip to memory
    for (int wb = w0 + g; wb <= w1; wb += NP * B) {
      float2 ml[B];
      float4 y[B];
#pragma unroll
      for (int i = 0; i < B; ++i) {
        const int w = min(wb + i * NP, w1);
        const int64_t slot = 2 * (int64_t)w + (w == w0 && second ? 1 : 0);
        ml[i] = pc.ml[slot * PD_HEADS + head];
        y[i] = *(const float4*)&pc.o[(slot * rows_max + head) * D + e * 4];
      }
      float Mn = M;
#pragma unroll
      for (int i = 0; i < B; ++i) {
        if (wb + i * NP > w1) ml[i].y = 0.f;
        if (ml[i].y != 0.f) Mn = fmaxf(Mn, ml[i].x);       // (a piece whose sum is 0 saw nothing; one of NaN is not 0)
      }
      const float ref = Mn == -INFINITY ? 0.f : Mn;
      const float wa = M == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(M - ref);      // (nothing so far is 0, or not finite)
      L *= wa;
      x.x *= wa; x.y *= wa; x.z *= wa; x.w *= wa;
#pragma unroll
      for (int i = 0; i < B; ++i) {
        if (ml[i].y == 0.f) continue;
        const float wt = ml[i].x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml[i].x - ref);
        L = fmaf(wt, ml[i].y, L);
        x.x = fmaf(wt, y[i].x, x.x);
        x.y = fmaf(wt, y[i].y, x.y);
        x.z = fmaf(wt, y[i].z, x.z);
        x.w = fmaf(wt, y[i].w, x.w);
      }
      M = Mn;
    }
    so[g][e] = x;
    if (e == 0) sml[g] = make_float2(M, L);
  }
  __syncthreads();
  if (tid >= E) return;
  M = -INFINITY;
  L = 0.f;
#pragma unroll
  for (int p = 0; p < NP; ++p) M = fmaxf(M, sml[p].x);
  x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const float2 ml = sml[p];
    if (ml.y == 0.f) continue;
    const float wt = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
    const float4 y = so[p][e];
    L += wt * ml.y;
    x.x += wt * y.x; x.y += wt * y.y; x.z += wt * y.z; x.w += wt * y.w;
  }
  const bool none = M == -INFINITY && L == 0.f;
  const float inv = none ? 0.f : 1.f / L;
  T* dst = (T*)a.out + at * D + e * 4;
  Elem<T>::st(dst, none ? 0.f : x.x * inv);
  Elem<T>::st(dst + 1, none ? 0.f : x.y * inv);
  Elem<T>::st(dst + 2, none ? 0.f : x.z * inv);
  Elem<T>::st(dst + 3, none ? 0.f : x.w * inv);
  if (a.lse && tid == 0) a.lse[at] = none ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
}

template <typename T, int D>
static void decode_d(const PagedDims& Dm, const PagedAttn& a, hipStream_t st) {
  const int n_wg = paged_decode_workgroups(Dm), passes = (Dm.g + PD_HEADS - 1) / PD_HEADS;
  const int rows = Dm.g < PD_HEADS ? Dm.g : PD_HEADS, ipt = (a.n_req + PD_THREADS - 1) / PD_THREADS;
  const size_t lds = (size_t)PD_NW * rows * D * sizeof(float) + (size_t)(a.n_req + 1) * sizeof(int32_t);
  if (Dm.page_shift == 4) paged_decode_kernel<T, D, true><<<(unsigned)n_wg, PD_THREADS, lds, st>>>(a, a.table, Dm, passes, ipt);
  else paged_decode_kernel<T, D, false><<<(unsigned)n_wg, PD_THREADS, lds, st>>>(a, a.table, Dm, passes, ipt);
  paged_decode_join_kernel<T, D><<<dim3((unsigned)Dm.h, (unsigned)a.n_req), PD_THREADS, 0, st>>>(a, Dm, passes, n_wg);
}

void launch_paged_decode(const PagedDims& D, const PagedAttn& a, hipStream_t st) {
#define LOCRET_DECODE(T)                        \
  switch (D.d) {                                \
    case 32: decode_d<T, 32>(D, a, st); break;  \
    case 64: decode_d<T, 64>(D, a, st); break;  \
    case 96: decode_d<T, 96>(D, a, st); break;  \
    default: decode_d<T, 128>(D, a, st); break; \
  }
  if (D.bf16) { LOCRET_DECODE(bf16_t) } else { LOCRET_DECODE(float) }
#undef LOCRET_DECODE
}

}  // namespace locret
