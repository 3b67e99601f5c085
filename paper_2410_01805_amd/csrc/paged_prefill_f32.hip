// Causal attention of a ragged batch of chunks over pages (locret_paged_prefill), float.
//   s_tj = scale q_t . k_j over the visible keys j of query t,  out_t = sum_j e^(s_tj - M_t) v_j / L_t,  lse_t = M_t + ln L_t
// Both products with v_mfma_f32_16x16x4_f32 (157 TFLOP/s on the card), which bounds long chunks; short ones are bound by the chain of their
// launch.  A workgroup has 16 rows (token, query head of one KV head) and goes over the keys that any of them sees, 128 at a time, 32
// for each of its four wavefronts; their maxima, sums and accumulators are joined in LDS.  So few rows make many workgroups, and a chunk of 400
// tokens fills the chip.  Where there are at most half as many workgroups as CUs the keys of each are cut into parts, which a second launch joins.
// Keys and values go from the pages to registers in the layout of the operands (PagedTileF32); neighbouring workgroups read the same ones, from L2.
// Everything is 32-bit.  What a row does not see is taken out of its logits by selection; its value meets a factor 0, so a workgroup whose
// accumulators end up not finite forms its rows once more, key by key, from what each of them sees.
#include "paged.h"
#include "paged_tile.h"

namespace locret {

constexpr int PR_THREADS = 256, PR_NW = 4, PR_ROWS = 16;
// Parts of an item at most.  (8 heads, 2 KV heads of 64 dims: one token on 8192 units whole 100.8 us, in 8, 16, 32 parts 24.9, 22.5, 27.7; with more tokens parts are
// given by the CUs: 100 on 2000 units, 50 workgroups in 5 parts 18.1, in 10 21.6, whole 29.3)
constexpr int PR_CUS = 256, PR_MAX_PARTS = 16, PR_MAX_SLOTS = PR_CUS;
constexpr float PR_RESCALE_LOG2 = 8.f;

struct PrItem {
  int r, m, row0, n_rows, t0, pos0;      // request, KV head, first row and rows of it, first token (packed) and its position
};
// Item x: (16 rows, KV head).  first: LDS, n_req + 1 ints behind PR_NW words.
constexpr int PR_SCRATCH = PR_NW * 4;
__device__ __forceinline__ bool pr_item(const PagedAttn& a, const PagedDims& Dm, int x, unsigned char* scratch, PrItem& it) {
  uint32_t* scan = (uint32_t*)scratch;
  int32_t* first = (int32_t*)(scratch + PR_SCRATCH);
  const int tid = threadIdx.x, ipt = (a.n_req + PR_THREADS - 1) / PR_THREADS;
  uint32_t mine = 0, total;
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < a.n_req) {
      const int c0 = paged_cu(a.cu, r, a.T), n = max(paged_cu(a.cu, r + 1, a.T) - c0, 0);
      first[r + 1] = (int)(((int64_t)n * Dm.g + PR_ROWS - 1) / PR_ROWS);
      mine += first[r + 1];
    }
  }
  uint32_t before = block_exclusive(mine, scan, total);
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < a.n_req) {
      before += first[r + 1];
      first[r + 1] = (int)before;
    }
  }
  if (tid == 0) first[0] = 0;
  __syncthreads();
  const int tile = x / Dm.h_kv;
  if (tile >= (int)total) return false;
  const int lo = last_at_or_before(first, a.n_req, tile);
  const int c0 = paged_cu(a.cu, lo, a.T), n = paged_cu(a.cu, lo + 1, a.T) - c0;
  it.r = __builtin_amdgcn_readfirstlane(lo);
  it.m = __builtin_amdgcn_readfirstlane(x % Dm.h_kv);
  it.row0 = __builtin_amdgcn_readfirstlane((first[lo + 1] - 1 - tile) * PR_ROWS);       // the last rows first: they see the most keys
  it.n_rows = __builtin_amdgcn_readfirstlane((int)min((int64_t)PR_ROWS, (int64_t)n * Dm.g - it.row0));
  it.t0 = __builtin_amdgcn_readfirstlane(c0);
  it.pos0 = __builtin_amdgcn_readfirstlane(paged_len(a.lens, lo, Dm.max_pages, Dm.page_shift) - n);
  return true;
}

// The keys of an item in tiles of 32: sinks, then from the first tile with a key in a row's window on; four tiles are a unit.
struct PrSpan {
  int w0, ns, wb, end, st, total;
};
__device__ __forceinline__ PrSpan pr_span(const PrItem& it, const PagedDims& Dm) {
  PrSpan s;
  const int p0 = paged_pos(it.pos0 + it.row0 / Dm.g), p1 = paged_pos(it.pos0 + (it.row0 + it.n_rows - 1) / Dm.g);
  s.end = p1 + 1;
  s.w0 = Dm.window ? max(0, p0 - Dm.window + 1) : 0;
  s.ns = min(Dm.n_sink, s.w0);
  s.wb = s.w0 & ~31;
  s.st = (int)(((uint32_t)s.ns + 31) / 32);
  s.total = (s.st + (int)(((uint32_t)max(s.end - s.wb, 0) + 31) / 32) + PR_NW - 1) / PR_NW;
  return s;
}
__device__ __forceinline__ int pr_part_len(int total, int parts) { return (total + parts - 1) / parts; }

template <int D>
__global__ __launch_bounds__(PR_THREADS, D >= 96 ? 2 : 3) void paged_prefill_f32_kernel(PagedAttn a, const int32_t* __restrict__ table, PagedDims Dm,
                                                                                     int n_items, int parts, float* __restrict__ part) {
  typedef PagedTileF32<D, true> Tile;
  constexpr int NV = D / 16;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  float* sets = (float*)smem;                              // [wavefront][16][D]
  float2* wml = (float2*)(smem + PR_NW * PR_ROWS * D * sizeof(float));      // [wavefront][16]
  PrItem it;
  const int block = paged_block(), layer = block / n_items;
  if (layer >= parts || !pr_item(a, Dm, block - layer * n_items, smem, it)) return;
  __syncthreads();                                         // smem is `sets` from here on
  const PrSpan sp = pr_span(it, Dm);
  int u0 = 0, u1 = sp.total;
  bool cut = false;
  if (parts > 1) {
    const int len = pr_part_len(sp.total, parts);
    cut = sp.total > len;
    u0 = layer * len;
    u1 = min(u1, u0 + len);
    if (layer > 0 && u0 >= sp.total) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 15, kg = lane >> 4;
  const int shift = Dm.page_shift, page = 1 << shift;
  const int32_t* trow = table + (int64_t)it.r * Dm.max_pages;
  const int64_t page_stride = (int64_t)Dm.h_kv * page * D;
  const float* Kp = (const float*)a.K + (int64_t)it.m * page * D;
  const float* Vp = (const float*)a.V + (int64_t)it.m * page * D;
  // this lane's row (a column of S^T): spare ones repeat the last
  const int row = it.row0 + min(n, it.n_rows - 1), tok = row / Dm.g, pos = paged_pos(it.pos0 + tok);
  const int64_t at = (int64_t)(it.t0 + tok) * Dm.h + it.m * Dm.g + (row - tok * Dm.g);
  const int pmin = paged_pos(it.pos0 + it.row0 / Dm.g);
  const float c = Dm.scale * 1.4426950408889634f;
  // what the row sees of a tile: the keys [lo, hi), and behind the sinks' tiles the sinks [w0, s1) too
  struct Seen { int lo, hi, s1; };
  auto seen_of = [&](bool sink) __attribute__((always_inline)) {
    Seen v;
    v.lo = sink || Dm.window == 0 ? 0 : max(sp.w0, pos - Dm.window + 1);
    v.hi = sink ? min(sp.ns, pos + 1) : pos + 1;
    v.s1 = sink ? 0 : min(Dm.n_sink, pos + 1);
    return v;
  };
  auto sees = [&](const Seen& v, int key) __attribute__((always_inline)) {
    return ((key >= v.lo) & (key < v.hi)) | ((key >= sp.w0) & (key < v.s1));
  };
  struct Place { bool sink; int kb, end, id0, id1; };
  auto place = [&](int u) __attribute__((always_inline)) {
    Place p;
    const int i = u * PR_NW + wave;
    p.sink = i < sp.st;
    p.kb = p.sink ? i * 32 : sp.wb + (i - sp.st) * 32;
    p.end = p.sink ? sp.ns : sp.end;
    p.id0 = p.id1 = -1;
    if (p.kb < p.end) {
      p.id0 = trow[p.kb >> shift];
      p.id1 = shift == 4 ? (p.kb + 16 < p.end ? trow[(p.kb >> 4) + 1] : -1) : p.id0;
    }
    return p;
  };
  auto address = [&](const float* base, const Place& p, const float*& lo, const float*& hi) __attribute__((always_inline)) {
    const int i0 = (unsigned)p.id0 < (unsigned)Dm.n_pages ? p.id0 : 0, i1 = (unsigned)p.id1 < (unsigned)Dm.n_pages ? p.id1 : 0;
    lo = base + i0 * page_stride + (p.kb & (page - 1)) * D;
    hi = shift == 4 ? base + i1 * page_stride - 16 * D : lo;
  };

  typename Tile::q_t qb[Tile::NQ];
  Tile::load_q((const float*)a.q + at * D, true, qb);
  Tile tl;
  dec_f32x4 o[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) o[i] = dec_f32x4{0.f, 0.f, 0.f, 0.f};
  float mrun = -INFINITY, lrun = 0.f;
  Place p = {false, 0, 0, -1, -1}, nx = p;
  if (u0 < u1) {
    p = place(u0);
    if (p.kb < p.end) {
      const float *lo, *hi;
      address(Kp, p, lo, hi);
      tl.load_k(lo, hi);
      address(Vp, p, lo, hi);
      tl.load_v(lo, hi);
    }
    nx = place(min(u0 + 1, u1 - 1));
  }
  for (int u = u0; u < u1; ++u) {
    const Place nn = place(min(u + 2, u1 - 1));
    const bool sink = p.sink, work = p.kb < p.end, more = u + 1 < u1 && nx.kb < nx.end;
    dec_f32x4 s[2];
    float pr[8];
    if (work) tl.logits(qb, s);
    const float *lo, *hi;
    if (more) {
      address(Kp, nx, lo, hi);
      tl.load_k(lo, hi);
    }
    if (work) {
      // does every row see all 32 keys?
      const bool whole = (sink ? p.kb + 32 <= sp.ns : p.kb >= sp.w0 && p.kb + 31 <= pmin && (Dm.window == 0 || sp.end - 1 - p.kb < Dm.window)) &&
                         (unsigned)p.id0 < (unsigned)Dm.n_pages && (unsigned)p.id1 < (unsigned)Dm.n_pages;
      if (!whole) {
        // what no row may see goes out of the values: keys behind the last one or on no page, a bit each
        const int id = kg >= 2 ? p.id1 : p.id0, k0 = p.kb + 8 * kg;
        const uint32_t there = (unsigned)id < (unsigned)Dm.n_pages ? (1u << min(max(p.end - k0, 0), 8)) - 1u : 0u;
        tl.clear_v(there);
        const Seen v = seen_of(sink);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const bool see = ((there >> j) & 1) & (int)sees(v, k0 + j);
          s[j >> 2][j & 3] = see ? s[j >> 2][j & 3] : -INFINITY;
        }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int j = 0; j < 8; ++j) mx = fmaxf(mx, s[j >> 2][j & 3]);
      mx *= c;
      if (__any((mx - mrun) > PR_RESCALE_LOG2)) {          // also true from -inf to a number
        mx = max_across_quarters(mx);                      // the four lanes of a column move together
        const bool up = (mx - mrun) > PR_RESCALE_LOG2;
        const float alpha = up ? __builtin_amdgcn_exp2f(mrun - mx) : 1.f;
        if (up) mrun = mx;
        lrun *= alpha;
#pragma unroll
        for (int rr = 0; rr < 4; ++rr) {
          const float ar = __shfl(alpha, 4 * kg + rr, 64); // accumulator row 4 kg + rr is that row
#pragma unroll
          for (int i = 0; i < NV; ++i) o[i][rr] *= ar;
        }
      }
      const float ref = mrun == -INFINITY ? 0.f : mrun;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        pr[j] = __builtin_amdgcn_exp2f(fmaf(s[j >> 2][j & 3], c, -ref));
        lrun += pr[j];
      }
      tl.add(pr, o, true);
    }
    if (more) {
      address(Vp, nx, lo, hi);
      tl.load_v(lo, hi);
    }
    p = nx;
    nx = nn;
  }
  bool bad = false;                                        // an accumulator that is not finite
#pragma unroll
  for (int i = 0; i < NV; ++i)
#pragma unroll
    for (int rr = 0; rr < 4; ++rr) bad = bad || !(fabsf(o[i][rr]) < INFINITY);
  if (__any(bad)) {
    // the wavefront's keys again, one by one: lane (n, kg) has row n, dims kg D/4 ..
    float qv[D / 4], ov[D / 4];
#pragma unroll
    for (int e = 0; e < D / 4; ++e) {
      qv[e] = ((const float*)a.q)[at * D + kg * (D / 4) + e];
      ov[e] = 0.f;
    }
    mrun = -INFINITY;
    float l = 0.f;
#pragma unroll 1
    for (int u = u0; u < u1; ++u) {
      const Place w = place(u);
      const Seen v = seen_of(w.sink);
#pragma unroll 1
      for (int key = w.kb; key < min(w.end, w.kb + 32); ++key) {
        const int id = trow[key >> shift];
        if ((unsigned)id >= (unsigned)Dm.n_pages) continue;
        const int64_t off = id * page_stride + (key & (page - 1)) * D + kg * (D / 4);
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < D / 4; ++e) s = fmaf(qv[e], Kp[off + e], s);
        s = sum_across_quarters(s);
        const bool see = sees(v, key);
        const float x = see ? s * c : -INFINITY, m_new = fmaxf(mrun, x), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(mrun - ref), pk = __builtin_amdgcn_exp2f(x - ref);
        l = l * alpha + pk;
        mrun = m_new;
#pragma unroll
        for (int e = 0; e < D / 4; ++e) ov[e] = ov[e] * alpha + (see ? pk * Vp[off + e] : 0.f);
      }
    }
#pragma unroll
    for (int e = 0; e < D / 4; ++e) sets[(wave * PR_ROWS + n) * D + kg * (D / 4) + e] = ov[e];
    lrun = l;
  } else {
    lrun = sum_across_quarters(lrun);
#pragma unroll
    for (int rr = 0; rr < 4; ++rr)
#pragma unroll
      for (int i = 0; i < NV; ++i) sets[(wave * PR_ROWS + 4 * kg + rr) * D + n * NV + i] = o[i][rr];
  }
  if (lane < PR_ROWS) wml[wave * PR_ROWS + lane] = make_float2(mrun, lrun);
  __syncthreads();
  for (int idx = tid; idx < it.n_rows * (D / 4); idx += PR_THREADS) {
    const int rr = idx / (D / 4), e = idx % (D / 4) * 4;
    float M = -INFINITY, L = 0.f;
#pragma unroll
    for (int w = 0; w < PR_NW; ++w) M = fmaxf(M, wml[w * PR_ROWS + rr].x);
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int w = 0; w < PR_NW; ++w) {
      const float2 ml = wml[w * PR_ROWS + rr];
      if (ml.y == 0.f) continue;                           // saw nothing (a sum of NaN is not 0)
      const float wt = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
      const float4 y = *(const float4*)&sets[(w * PR_ROWS + rr) * D + e];
      L = fmaf(wt, ml.y, L);
      x.x = fmaf(wt, y.x, x.x);
      x.y = fmaf(wt, y.y, x.y);
      x.z = fmaf(wt, y.z, x.z);
      x.w = fmaf(wt, y.w, x.w);
    }
    if (cut) {
      *(float4*)&part[((int64_t)block * PR_ROWS + rr) * D + e] = x;
      if (e == 0) ((float2*)(part + (int64_t)PR_MAX_SLOTS * PR_ROWS * D))[(int64_t)block * PR_ROWS + rr] = make_float2(M, L);
      continue;
    }
    const int row_ = it.row0 + rr, tok_ = row_ / Dm.g;
    const int64_t to = (int64_t)(it.t0 + tok_) * Dm.h + it.m * Dm.g + (row_ - tok_ * Dm.g);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *(float4*)((float*)a.out + to * D + e) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (a.lse && e == 0) a.lse[to] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
  }
}

// Joins the parts of the items that were cut.  One workgroup per item, a thread per four dims of a row.
template <int D>
__global__ __launch_bounds__(PR_THREADS) void paged_prefill_f32_join_kernel(PagedAttn a, PagedDims Dm, int n_items, int parts, const float* __restrict__ part) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  PrItem it;
  if (!pr_item(a, Dm, blockIdx.x, smem, it)) return;
  const PrSpan sp = pr_span(it, Dm);
  const int len = pr_part_len(sp.total, parts);
  if (sp.total <= len) return;
  const int np = (sp.total + len - 1) / len;
  const float2* pml = (const float2*)(part + (int64_t)PR_MAX_SLOTS * PR_ROWS * D);
  for (int idx = threadIdx.x; idx < it.n_rows * (D / 4); idx += PR_THREADS) {
    const int rr = idx / (D / 4), e = idx % (D / 4) * 4;
    float M = -INFINITY, L = 0.f;
    for (int p = 0; p < np; ++p) {
      const float2 ml = pml[((int64_t)p * n_items + blockIdx.x) * PR_ROWS + rr];
      if (ml.y != 0.f) M = fmaxf(M, ml.x);
    }
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int p = 0; p < np; ++p) {
      const int64_t slot = ((int64_t)p * n_items + blockIdx.x) * PR_ROWS + rr;
      const float2 ml = pml[slot];
      const float4 y = *(const float4*)&part[slot * D + e];
      if (ml.y == 0.f) continue;
      const float wt = ml.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ml.x - M);
      L = fmaf(wt, ml.y, L);
      x.x = fmaf(wt, y.x, x.x);
      x.y = fmaf(wt, y.y, x.y);
      x.z = fmaf(wt, y.z, x.z);
      x.w = fmaf(wt, y.w, x.w);
    }
    const int row = it.row0 + rr, tok = row / Dm.g;
    const int64_t to = (int64_t)(it.t0 + tok) * Dm.h + it.m * Dm.g + (row - tok * Dm.g);
    const float inv = L == 0.f ? 0.f : 1.f / L;
    *(float4*)((float*)a.out + to * D + e) = make_float4(x.x * inv, x.y * inv, x.z * inv, x.w * inv);
    if (a.lse && e == 0) a.lse[to] = L == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(L)) * 0.6931471805599453f;
  }
}

size_t paged_prefill_f32_workspace(const PagedDims& D) { return (size_t)PR_MAX_SLOTS * PR_ROWS * (D.d + 2) * sizeof(float); }

template <int D>
static void prefill_f32_d(const PagedDims& Dm, const PagedAttn& a, hipStream_t st) {
  // 16-row tiles at most: every request's last one may be short
  int64_t tiles = ((int64_t)a.T * Dm.g + (int64_t)a.n_req * (PR_ROWS - 1)) / PR_ROWS;
  const int64_t most = (int64_t)a.T * ((Dm.g + PR_ROWS - 1) / PR_ROWS);
  if (tiles > most) tiles = most;
  const int n_items = (int)(tiles * Dm.h_kv);
  // (three ragged requests, 212 workgroups: whole 17.1 us, in two parts and joined 21.3)
  int parts = PR_CUS / n_items;
  parts = parts < 1 ? 1 : parts > PR_MAX_PARTS ? PR_MAX_PARTS : parts;
  const size_t scratch = PR_SCRATCH + (size_t)(a.n_req + 1) * sizeof(int32_t), body = (size_t)PR_NW * PR_ROWS * (D * sizeof(float) + sizeof(float2));
  paged_prefill_f32_kernel<D><<<paged_grid((int64_t)n_items * parts), PR_THREADS, scratch > body ? scratch : body, st>>>(a, a.table, Dm, n_items, parts,
                                                                                                                   (float*)a.ws);
  if (parts > 1) paged_prefill_f32_join_kernel<D><<<(unsigned)n_items, PR_THREADS, scratch, st>>>(a, Dm, n_items, parts, (const float*)a.ws);
}

void launch_paged_prefill_f32(const PagedDims& D, const PagedAttn& a, hipStream_t st) {
  switch (D.d) {
    case 32: prefill_f32_d<32>(D, a, st); break;
    case 64: prefill_f32_d<64>(D, a, st); break;
    case 96: prefill_f32_d<96>(D, a, st); break;
    default: prefill_f32_d<128>(D, a, st); break;
  }
}

}  // namespace locret
