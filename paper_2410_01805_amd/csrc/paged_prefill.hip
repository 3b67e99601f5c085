// Causal attention of a ragged batch of chunks over pages (locret_paged_prefill), bf16, on the matrix cores.
//   s_tj = scale q_t . k_j over the visible keys j of query t,  out_t = sum_j e^(s_tj - M_t) v_j / L_t,  lse_t = M_t + ln L_t
// Bound by the matrix cores: 4 d operations for each (query, key) pair against 4 d bytes for each key of 256 query rows.
//
// A workgroup takes 256 rows (token, query head of one KV head), 256 / g whole tokens of one request, so that short chunks
// fill it for any group size, and goes over the keys that any of them sees: first the sinks, then from the window of its first token to
// its last token.  Its 8 wavefronts have 32 rows each.  Products are transposed, v_mfma_f32_32x32x16_bf16: S^T = K Q^T (A = 32 keys from
// LDS, B = the rows' queries in registers), O^T += V^T P^T (A = V^T by the transposing LDS read, B = P^T as the S accumulators hold it: 16
// keys of one row a lane, so that sums are per lane).  Wavefronts 0..3 and 4..7, two of which share a SIMD, are held one S block apart by
// two barriers a tile, X and Y, so that the matrix pipe has S and PV of one half while the other is at its softmax:
//
//      X(t) | A: S(t)                     | Y(t) | A: softmax, PV, first K fragments of t+1
//           | B: loads of t+3, K fragments |      | B: S(t), softmax, PV
//
// Tiles (64 keys of 128 or 96 dims, 128 of 64 or 32) come from the pages to a ring of 4 stages in LDS without passing through registers: a
// load instruction of a wavefront covers 1 KB of LDS, which is 4 or 8 keys and lies inside 16 keys that start at a multiple of 16, so it
// lies inside one page of any size.  Its descriptor has those keys in the page as base and how many of them are there as length; where a page
// holds whole tiles, one serves the whole tile.  What is behind the last key, on no page, or padding of a row arrives as zeros.  LDS rows have 256 bytes (keys of 64 or 32 dims lie two
// in a row); position c' of row r holds the 16-byte chunk c' ^ f(r), with f chosen so that neither the fragment reads of K nor the
// transposing ones of V meet in a bank: f = r mod 16 for K; 4 (r mod 4), or 4 (r mod 2) with two keys in a row, for V.
// At X(t) tiles t and t+1 are in LDS, and every wavefront is done with t-1, whose stage the loads of t+3 overwrite.
//
// Softmax: logits stay unscaled in the accumulators and become exponents by one multiply-add (queries scaled before the product would have
// to be rounded again, which costs the outputs twice the error).  The running maximum of a row is that of the first tile in which it sees
// a key, and raised when the row's sum over a tile reaches 2^30.  Probabilities become one bf16 factor each, off by at most 2^-8 of themselves,
// which with the outputs' own rounding of the same size makes these 1.41 times as far off as that rounding alone; two factors, as in the decode
// kernel, would be half as many matrix instructions more (4096 tokens on 16384 units 841 -> 1170 us, 512 on 16384 136 -> 182, 12 ragged
// requests with a window 77 -> 101).  Sums, maxima and accumulators are 32-bit.
// Tiles that some row of a wavefront does not see whole are masked before the maximum.  A masked probability is 0, but 0 times a value that is
// not finite is not: where an accumulator is not finite in the end, the wavefront forms its rows once more behind the loop, key by key, from
// the keys that each row sees.  (There no tile's registers are alive; the same inside the loop took half of its speed in spills, and looking
// through the values of masked tiles a third of the time of 12 ragged requests with a window, 94 -> 59 us.)
//
// Few rows: where the items (token tile, KV head) are at most half as many as the CUs, each one's keys are cut into parts,
// workgroups of their own, which leave maximum, sum and accumulators; a second launch joins them.  (32 heads, 8 KV heads of 128 dims, us: 512 tokens
// on 4096 units, 64 items in 4 parts 48.5, whole 99, in 8 parts 65.5; 1024 on 8192, 128 items in 2 parts 135, whole 190, in 4 144;
// 1536 on 8192, 192 items whole 201, in 2 parts 212.)
#include "attn_common.h"
#include "paged.h"

namespace locret {

typedef __attribute__((address_space(3))) void* pf_lds_ptr;
typedef __attribute__((address_space(3))) unsigned char* pf_lds_u8;
typedef short pf_s16x4 __attribute__((ext_vector_type(4)));
typedef short pf_s16x8 __attribute__((ext_vector_type(8)));

constexpr int PF_NW = 8, PF_THREADS = PF_NW * 64, PF_ROWS = PF_NW * 32;
constexpr int PF_TILE_B = 64 * 256, PF_STAGE_B = 2 * PF_TILE_B;
constexpr int PF_KPRE = 4;                     // K fragments fetched ahead of the S block
// Parts of an item at most: the joining workgroups go over them one after the other.  (8 items: 16 tokens on 16384 units in 8, 16, 32 parts 51.4, 42.6,
// 56.6 us; on 131072 units 280, 170, 141)
constexpr int PF_CUS = 256, PF_MAX_PARTS = 16, PF_MAX_SLOTS = PF_CUS;
// Key tiles of a part at least: fewer do not pay for a part's prologue and joining, more leave CUs idle.  (64 tokens on 700 units with 1, 2, 4, 8 tiles 20.5,
// 18.6, 19.3, 24.2 us, on 1500 units 23.0, 22.8, 21.7, 25.0)
constexpr int PF_MIN_PART = 4;

// What a workgroup works on.
struct PfItem {
  int r, m, t0, n_tok;      // request, KV head, first token (in the packed order) and tokens
  int p0;                   // position of the first token
};

#define LOCRET_PF_TR(dst, addr, off) asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "i"(off) : "memory")
#define LOCRET_PF_WAIT(a, b, n) asm volatile("s_waitcnt lgkmcnt(%2)" : "+v"(a), "+v"(b) : "i"(n))

// Finds item x = (token tile, KV head): the token tiles of all requests in their order, a request's last tile first (it sees the most keys).
// scratch: LDS, PF_NW words and n_req + 1 ints, free again after the next barrier.  False: there is no such tile.  All results are the
// same in the whole workgroup.
constexpr int PF_SCRATCH = PF_NW * 4;
__device__ __forceinline__ bool pf_item(const PagedAttn& a, const PagedDims& Dm, int x, unsigned char* scratch, PfItem& it) {
  uint32_t* scan = (uint32_t*)scratch;
  int32_t* first = (int32_t*)(scratch + PF_SCRATCH);
  const int tid = threadIdx.x, tw = PF_ROWS / Dm.g, ipt = (a.n_req + PF_THREADS - 1) / PF_THREADS;
  uint32_t mine = 0, total;
  for (int u = 0; u < ipt; ++u) {
    const int r = tid * ipt + u;
    if (r < a.n_req) {
      const int c0 = paged_cu(a.cu, r, a.T), n = max(paged_cu(a.cu, r + 1, a.T) - c0, 0);
      first[r + 1] = (int)(((uint32_t)n + tw - 1) / tw);      // (n may be the largest number)
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
  // every eighth workgroup is on the same XCD: a KV head's items on one of them, where they find its pages in one L2
  int tile;
  if (Dm.h_kv % 8 == 0) {
    const int per = Dm.h_kv / 8;
    it.m = (x & 7) * per + (x >> 3) % per;
  } else {
    it.m = x % Dm.h_kv;
  }
  tile = x / Dm.h_kv;
  if (tile >= (int)total) return false;
  const int lo = last_at_or_before(first, a.n_req, tile);
  const int tt = first[lo + 1] - 1 - tile;
  const int c0 = paged_cu(a.cu, lo, a.T), n = paged_cu(a.cu, lo + 1, a.T) - c0;
  it.r = __builtin_amdgcn_readfirstlane(lo);
  it.t0 = __builtin_amdgcn_readfirstlane(c0 + tt * tw);
  it.n_tok = __builtin_amdgcn_readfirstlane(min(tw, n - tt * tw));
  it.p0 = __builtin_amdgcn_readfirstlane(paged_len(a.lens, lo, Dm.max_pages, Dm.page_shift) - n + tt * tw);
  it.m = __builtin_amdgcn_readfirstlane(it.m);
  return true;
}

// The keys of an item: sink tiles over [0, ns), then window tiles from wb, of which keys from w_lo on count (none of them a sink), up to n_keys.
// (Tiles start at multiples of 16, or of their own length where a page holds one.)
struct PfKeys {
  int n_keys, w_lo, ns, wb, ns_t, n_tiles;
};
__device__ __forceinline__ PfKeys pf_keys(const PfItem& it, const PagedDims& Dm, int KT) {
  PfKeys k;
  k.n_keys = max(it.p0 + it.n_tok, 0);                    // (positions below 0 see nothing)
  k.ns = Dm.window ? min(Dm.n_sink, k.n_keys) : 0;
  k.w_lo = Dm.window ? max(k.ns, paged_pos(it.p0) - Dm.window + 1) : 0;
  k.wb = k.w_lo & ~((1 << Dm.page_shift >= KT ? KT : 16) - 1);
  k.ns_t = (k.ns + KT - 1) / KT;
  k.n_tiles = k.ns_t + (max(k.n_keys - k.wb, 0) + KT - 1) / KT;
  return k;
}
// Parts of an item and the tiles of each.
__device__ __forceinline__ int pf_part_len(int n_tiles, int k) { return max((n_tiles + k - 1) / k, PF_MIN_PART); }

__host__ __device__ constexpr int pf_tile_keys(int d) { return d <= 64 ? 128 : 64; }

template <int D, bool ONE_PAGE>
__global__ __launch_bounds__(PF_THREADS, 2) void paged_prefill_kernel(PagedAttn a, const bf16_t* __restrict__ q, const bf16_t* __restrict__ K,
                                                                     const bf16_t* __restrict__ V, const int32_t* __restrict__ table, PagedDims Dm,
                                                                     int n_items, int parts, float* __restrict__ part) {
  constexpr int KH = D <= 64 ? 2 : 1;                      // keys of an LDS row
  constexpr int KT = 64 * KH, NKB = KT / 32;               // keys and 32-key blocks of a tile
  constexpr int NKS = D / 16, NDB = D / 32;                // contraction steps of S, 32-dim blocks of O^T
  constexpr int NKF = NKB * NKS, NVF = KT / 16 * NDB;      // K and V^T fragments of a tile
  constexpr int VPRE = KH == 2 ? 2 : 4;                    // V^T fragments in flight ahead of their MFMA
  constexpr int KC_B = 4096 / KH, KC_H = 2048 / KH;        // bytes of 16 keys and of 8 keys in LDS
  constexpr int YTAIL = D == 128 ? 4 : 1;                  // MFMAs of A's S block behind barrier Y
  // The only LDS variable: with a second one the compiler tells them apart by alias scopes, and then waits for all direct loads before every
  // read of `ring`, which it cannot tell from the stages in flight (4096 tokens on 16384 units: 948 us, 883 without
  // that and the queries' wait below).
  __shared__ __attribute__((aligned(1024))) unsigned char ring[4 * PF_STAGE_B];

  PfItem it;
  const int block = paged_block(), layer = block / n_items;
  if (layer >= parts || !pf_item(a, Dm, block - layer * n_items, ring, it)) return;
  const PfKeys ks_ = pf_keys(it, Dm, KT);
  int t_lo = 0, t_hi = ks_.n_tiles;
  bool cut = false;
  if (parts > 1) {
    const int len = pf_part_len(ks_.n_tiles, parts);
    cut = ks_.n_tiles > len;
    t_lo = layer * len;
    t_hi = min(t_hi, t_lo + len);
    if (layer > 0 && t_lo >= ks_.n_tiles) return;
  }
  const int tid = threadIdx.x, lane = tid & 63, n32 = lane & 31, hi = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int g = Dm.g, shift = Dm.page_shift, page = 1 << shift;
  const int rows = it.n_tok * g;
  const int32_t* trow = table + (int64_t)it.r * Dm.max_pages;

  auto tile_key = [&](int t) __attribute__((always_inline)) { return t < ks_.ns_t ? t * KT : ks_.wb + (t - ks_.ns_t) * KT; };
  auto tile_end = [&](int t) __attribute__((always_inline)) { return t >= t_hi ? 0 : t < ks_.ns_t ? ks_.ns : ks_.n_keys; };
  // this lane's row, and the first and last position of the wavefront's
  const int row = min(wave * 32 + n32, rows - 1), tok = row / g;
  const int64_t at = (int64_t)(it.t0 + tok) * Dm.h + it.m * g + (row - tok * g);
  const int pos = paged_pos(it.p0 + tok);
  const int pw0 = paged_pos(it.p0 + min(wave * 32, rows - 1) / g), pw1 = paged_pos(it.p0 + min(wave * 32 + 31, rows - 1) / g);
  // first keys of the tiles that all rows of the wavefront see whole (among the sinks: up to all_sink), and of those that some row sees a key of
  const int all_lo = Dm.window ? max(ks_.w_lo, pw1 - Dm.window + 1) : 0, all_hi = pw0 - KT + 1, all_sink = min(ks_.ns - KT, all_hi);
  const int any_lo = Dm.window ? pw0 - Dm.window - KT + 2 : 0, any_hi = wave * 32 < rows ? pw1 : -1;

  bf16x8 qf[NKS];
  {
    const bf16_t* qp = q + at * D + hi * 8;
#pragma unroll
    for (int s = 0; s < NKS; ++s) qf[s] = *(const bf16x8*)(qp + s * 16);
  }
  f32x16 oacc[NDB];
#pragma unroll
  for (int db = 0; db < NDB; ++db)
#pragma unroll
    for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  const float c = Dm.scale * 1.4426950408889634f;
  float m_run = 0.f, l_run = 0.f;              // of the lane's row, in log2 units; the sum over this lane's keys
  bool unset = true;                           // the row has seen no key yet

  // ---- tiles -----------------------------------------------------------------------------------------------------------
  const int w4 = wave & 3, l_row = lane >> 4, l_pos = lane & 15;
  constexpr int NCH = D / 8, SLOT = 16 / KH, KPI = 4 * KH;       // chunks of a key in memory and in LDS; keys of a load instruction
  constexpr int OUTSIDE = 0x7ffff000;                            // an offset no descriptor reaches: the load brings zeros
  auto offset = [&](int ch) { return ch % SLOT < NCH ? (l_row * KH + ch / SLOT) * (D * 2) + ch % SLOT * 16 : OUTSIDE; };
  const int k_vo = offset(l_pos ^ l_row ^ (w4 << 2)), v_vo = offset(l_pos ^ ((KH == 1 ? l_row : l_row & 1) << 2));
  const uint32_t page_b = (uint32_t)(Dm.h_kv * page) * (D * 2);          // (at most 1024 heads x 256 units x 256 bytes)
  const unsigned char* Kp = (const unsigned char*)K + (int64_t)it.m * page * (D * 2);
  const unsigned char* Vp = (const unsigned char*)V + (int64_t)it.m * page * (D * 2);
  auto scalar_ptr = [](const unsigned char* p) -> void* {
    const uint64_t x = (uint64_t)p;
    const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)x), up = __builtin_amdgcn_readfirstlane((uint32_t)(x >> 32));    // (the builtin is signed)
    return (void*)(((uint64_t)up << 32) | lo);
  };
  // Descriptors: one a tile where a page holds whole tiles (EPT = 1), else one for each of the wavefront's four load instructions.  Their parts are
  // formed by the lanes of the wavefront, a descriptor each, for 64 / EPT tiles at a time, and read from there; the page numbers of the next
  // lot are requested with each.  (A 4096-token chunk on 16384 units, pages of 64: formed tile by tile, 120 scalar instructions for four
  // descriptors 1000 us, one descriptor 911 us, its page number from LDS 909 us.)
  constexpr int EPT = ONE_PAGE ? 1 : 4, TPL = 64 / EPT;
  uint32_t e_off = 0, e_up = 0;                                  // this lane's descriptor: offset in the pool ...
  int e_len = 0, e_id = 0;                                       // ... and bytes there; page number of the next lot's
  auto entry_key = [&](int i, int& end) __attribute__((always_inline)) {      // first key of this lane's descriptor, lot from tile i of the part
    const int t = t_lo + i + lane / EPT;
    end = tile_end(t);
    return tile_key(t) + (EPT == 1 ? 0 : (w4 + lane % EPT * 4) * KPI);
  };
  auto request = [&](int i) __attribute__((always_inline)) {
    int end;
    const int key = entry_key(i, end);
    e_id = -1;
    if (key < end) e_id = trow[key >> shift];
  };
  auto form = [&](int i) __attribute__((always_inline)) {
    int end;
    const int key = entry_key(i, end);
    const bool ok = (uint32_t)e_id < (uint32_t)Dm.n_pages;
    const uint64_t off = (uint64_t)(ok ? (uint32_t)e_id : 0u) * page_b + (uint32_t)((key & (page - 1)) * (D * 2));
    e_off = (uint32_t)off;
    e_up = (uint32_t)(off >> 32);
    e_len = ok ? min(max(end - key, 0), EPT == 1 ? KT : KPI) * (D * 2) : 0;
  };
  auto issue = [&](int i) __attribute__((always_inline)) {       // tile i of the part, into stage i mod 4
    const int iu = __builtin_amdgcn_readfirstlane(i);
    if (iu % TPL == 0) {
      form(iu);
      request(iu + TPL);
    }
    unsigned char* sb = ring + (iu & 3) * PF_STAGE_B + w4 * 1024;
#pragma unroll
    for (int x = 0; x < EPT; ++x) {
      const int src = iu % TPL * EPT + x;
      const uint32_t lo = __builtin_amdgcn_readlane(e_off, src), up = __builtin_amdgcn_readlane(e_up, src);      // (the builtin is signed)
      const int len = __builtin_amdgcn_readlane(e_len, src);
      const uint64_t off = ((uint64_t)up << 32) | lo;
      __amdgpu_buffer_rsrc_t kr = __builtin_amdgcn_make_buffer_rsrc(scalar_ptr(Kp + off), 0, len, 0x00020000);
      __amdgpu_buffer_rsrc_t vr = __builtin_amdgcn_make_buffer_rsrc(scalar_ptr(Vp + off), 0, len, 0x00020000);
      constexpr int PER = 4 / EPT;                               // load instructions of a descriptor
      const int first = EPT == 1 ? w4 * (KPI * D * 2) : 0;
#pragma unroll
      for (int u = 0; u < PER; ++u) {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(kr, (pf_lds_ptr)(sb + (x + u) * 4096), 16, k_vo, first + u * (4 * KPI * D * 2), 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(vr, (pf_lds_ptr)(sb + PF_TILE_B + (x + u) * 4096), 16, v_vo, first + u * (4 * KPI * D * 2), 0, 0);
      }
    }
  };

  // The first page numbers and the queries are on their way; the pages are looked through meanwhile.
  if (wave >= PF_NW / 2) request(0);
  // does a page of the item's keys lie outside the pool?  All rows are then formed key by key.
  bool redo;                                   // the wavefront's rows have to be formed key by key
  {
    int odd = 0;
    const int s_end = (ks_.ns + page - 1) >> shift, e0 = ks_.wb >> shift, e1 = (ks_.n_keys + page - 1) >> shift;
    for (int i = tid; i < s_end; i += PF_THREADS) odd |= (unsigned)trow[i] >= (unsigned)Dm.n_pages;
    for (int i = e0 + tid; i < e1; i += PF_THREADS) odd |= (unsigned)trow[i] >= (unsigned)Dm.n_pages;
    // (said in the last stage, which is loaded behind further barriers; after this one `ring` no longer holds the sums of pf_item either)
    int32_t* said = (int32_t*)(ring + sizeof(ring)) - PF_NW;
    odd = __any(odd);
    if (lane == 0) said[wave] = odd;
    __syncthreads();
    odd = 0;
#pragma unroll
    for (int w = 0; w < PF_NW; ++w) odd |= said[w];
    redo = __builtin_amdgcn_readfirstlane(odd) != 0;
  }

  // waited for here: a wait in the loop, where they are used first, would be one for the tiles in flight too
#pragma unroll
  for (int s = 0; s < NKS; ++s) asm volatile("" : "+v"(qf[s]));

  // ---- fragment addresses (bytes inside a stage) -----------------------------------------------------------------------
  const int k_row = KH == 1 ? n32 : n32 >> 1, k_half = KH == 1 ? 0 : n32 & 1;
  const int k_base = k_row * 256 + (((k_half * 8 + hi) ^ (k_row & 15)) << 4);
  auto k_at = [&](int base, int f) __attribute__((always_inline)) {      // fragment f: step f / 2 of a pair of 32-key blocks, block f % 2 of it
    const int step = (f >> 1) % NKS, kb = (f >> 1) / NKS * 2 + (f & 1);
    return (base ^ (step << 5)) + kb * (32 / KH) * 256;
  };
  const int vs = lane & 15, vG = lane >> 4;
  const int v_row = KH == 1 ? (vG >> 1) * 4 + (vs >> 2) : (vG >> 1) * 2 + (vs >> 3), v_half = KH == 1 ? 0 : (vs >> 2) & 1;
  const int v_base = PF_TILE_B + v_row * 256 + (((v_half * 8 + (vG & 1) * 2 + ((vs & 3) >> 1)) ^ ((KH == 1 ? v_row & 3 : v_row & 1) << 2)) << 4) + ((vs & 1) << 3);
  const uint32_t ring_lds = (uint32_t)(uintptr_t)(pf_lds_u8)ring;

  bf16x8 kpre[PF_KPRE];
  auto prefetch_k = [&](int sb_off) __attribute__((always_inline)) {
    const int base = sb_off + k_base;
#pragma unroll
    for (int f = 0; f < PF_KPRE; ++f) kpre[f] = *(const bf16x8*)(ring + k_at(base, f));
  };
  // `mid` runs before the last TAIL MFMAs are issued (all fragment reads are out by then)
  auto s_block = [&](f32x16 (&sacc)[NKB], int sb_off, auto mid, auto tail_c) __attribute__((always_inline)) {
    constexpr int TAIL = decltype(tail_c)::value;
    const int base = sb_off + k_base;
    bf16x8 kf[NKF];
#pragma unroll
    for (int f = 0; f < NKF; ++f) kf[f] = f < PF_KPRE ? kpre[f] : *(const bf16x8*)(ring + k_at(base, f));
    auto mfma = [&](int f) __attribute__((always_inline)) {
      const int step = (f >> 1) % NKS, kb = (f >> 1) / NKS * 2 + (f & 1);
      f32x16 zero = {};
      sacc[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[f], qf[step], step == 0 ? zero : sacc[kb], 0, 0, 0);
    };
#pragma unroll
    for (int f = 0; f < NKF - TAIL; ++f) mfma(f);
#pragma unroll
    for (int i = 0; i < NKF - PF_KPRE; ++i) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
    }
    if (TAIL < PF_KPRE) __builtin_amdgcn_sched_group_barrier(0x008, PF_KPRE - TAIL, 0);
    if (TAIL > 0) {
      mid();
#pragma unroll
      for (int f = NKF - TAIL; f < NKF; ++f) mfma(f);
    }
  };

  // what the lane's row sees of tile t: the keys from lo on, n of them
  auto interval = [&](int t, int& lo, uint32_t& n) __attribute__((always_inline)) {
    const bool sink = t < ks_.ns_t;
    lo = sink || Dm.window == 0 ? 0 : max(ks_.w_lo, pos - Dm.window + 1);
    n = max((sink ? min(ks_.ns, pos + 1) : pos + 1) - lo, 0);
  };

  // softmax and PV of tile t, whose logits are in sacc
  auto softmax_pv = [&](f32x16 (&sacc)[NKB], int t, int sb_off) __attribute__((always_inline)) {
    const int kb0 = tile_key(t);
    // does every row of the wavefront see the whole tile?
    const bool whole = t < ks_.ns_t ? kb0 <= all_sink : kb0 >= all_lo && kb0 <= all_hi;
    if (!whole) {
      int lo;
      uint32_t n;
      interval(t, lo, n);
      const int x = lo - kb0 - hi * 4;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; ++r) sacc[kb][r] = (uint32_t)(kb * 32 + (r >> 2) * 8 + (r & 3) - x) < n ? sacc[kb][r] : -INFINITY;
    }
    uint32_t pw[NKB * 8];                      // probabilities, two keys a word
    float ps;
    auto exp_pack_sum = [&]() __attribute__((always_inline)) {
      float ps0 = 0.f, ps1 = 0.f;
      const float nm = -m_run;
#pragma unroll
      for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
        for (int r = 0; r < 16; r += 2) {
          const float e0 = __builtin_amdgcn_exp2f(fmaf(sacc[kb][r], c, nm)), e1 = __builtin_amdgcn_exp2f(fmaf(sacc[kb][r + 1], c, nm));
          pw[kb * 8 + (r >> 1)] = pack_bf16(e0, e1);
          ps0 += e0;
          ps1 += e1;
        }
      ps = ps0 + ps1;
    };
    auto softmax = [&]() __attribute__((always_inline)) {
      const bool none = __all(unset);                // no row has a maximum yet: nothing to try
      if (!none) exp_pack_sum();
      if (none || __any(unset || !(ps < RESCALE_SUM))) {     // rare: set or raise the running maximum
        float mx = -INFINITY;
#pragma unroll
        for (int kb = 0; kb < NKB; ++kb)
#pragma unroll
          for (int r = 0; r < 16; ++r) mx = fmaxf(mx, sacc[kb][r]);
        mx = max_across_halves(mx) * c;
        // (a row that still sees nothing keeps maximum 0; its accumulators are 0 until it sees a key)
        const float m_new = unset ? (mx == -INFINITY ? 0.f : mx) : fmaxf(m_run, mx);
        const float alpha = unset ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        unset = unset && mx == -INFINITY;
        m_run = m_new;
        l_run *= alpha;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) oacc[db][r] *= alpha;
        exp_pack_sum();
      }
      l_run += ps;
    };
    uint32_t va[NDB];
    pf_s16x4 vlo[NVF], vhi[NVF];
#pragma unroll
    for (int db = 0; db < NDB; ++db) va[db] = ring_lds + (uint32_t)((v_base ^ (db << 6)) + sb_off);
#pragma unroll
    for (int f = 0; f < VPRE; ++f) {
      LOCRET_PF_TR(vlo[f], va[f % NDB], (f / NDB) * KC_B);
      LOCRET_PF_TR(vhi[f], va[f % NDB], (f / NDB) * KC_B + KC_H);
    }
    softmax();
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int f = 0; f < NVF; ++f) {
      constexpr int LASTF = NVF - 1;
      const int newest = f + VPRE - 1 < LASTF ? f + VPRE - 1 : LASTF;        // newest fragment already requested: two reads each behind f's
      switch (2 * (newest - f)) {
        case 6: LOCRET_PF_WAIT(vlo[f], vhi[f], 6); break;
        case 4: LOCRET_PF_WAIT(vlo[f], vhi[f], 4); break;
        case 2: LOCRET_PF_WAIT(vlo[f], vhi[f], 2); break;
        default: LOCRET_PF_WAIT(vlo[f], vhi[f], 0); break;
      }
      const pf_s16x8 both = __builtin_shufflevector(vlo[f], vhi[f], 0, 1, 2, 3, 4, 5, 6, 7);
      const int kc = f / NDB;
      const uint4 pb = make_uint4(pw[kc * 4], pw[kc * 4 + 1], pw[kc * 4 + 2], pw[kc * 4 + 3]);
      oacc[f % NDB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, both), __builtin_bit_cast(bf16x8, pb), oacc[f % NDB], 0, 0, 0);
      if (f + VPRE < NVF) {
        const int fn = f + VPRE;
        LOCRET_PF_TR(vlo[fn], va[fn % NDB], (fn / NDB) * KC_B);
        LOCRET_PF_TR(vhi[fn], va[fn % NDB], (fn / NDB) * KC_B + KC_H);
      }
      __builtin_amdgcn_sched_barrier(0);
    }
  };

  auto wg_barrier = []() __attribute__((always_inline)) {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  // does some row of the wavefront see some key of tile t?
  auto active = [&](int t) __attribute__((always_inline)) {
    const int kb = tile_key(t);
    return kb <= any_hi && (t < ks_.ns_t || kb >= any_lo);
  };
  if (wave >= PF_NW / 2) {
    issue(0);
    issue(1);
    issue(2);
    asm volatile("s_waitcnt vmcnt(8)" ::: "memory");            // the first two tiles have landed
    wg_barrier();
    for (int t = t_lo; t < t_hi; ++t) {
      const int i = t - t_lo, sb_off = (i & 3) * PF_STAGE_B;
      wg_barrier();                                              // X
      issue(i + 3);
      const bool act = active(t);
      if (act) prefetch_k(sb_off);
      wg_barrier();                                              // Y
      if (act) {
        f32x16 sacc[NKB];
        s_block(sacc, sb_off, []() {}, IntC<0>());
        softmax_pv(sacc, t, sb_off);
      }
      asm volatile("s_waitcnt vmcnt(8)" ::: "memory");          // own loads of tile t + 2 have landed
    }
  } else {
    wg_barrier();
    prefetch_k(0);
    for (int t = t_lo; t < t_hi; ++t) {
      const int i = t - t_lo, sb_off = (i & 3) * PF_STAGE_B;
      wg_barrier();                                              // X
      if (active(t)) {
        f32x16 sacc[NKB];
        s_block(sacc, sb_off, wg_barrier, IntC<YTAIL>());        // Y inside
        softmax_pv(sacc, t, sb_off);
      } else {
        wg_barrier();                                            // Y
      }
      prefetch_k(((i + 1) & 3) * PF_STAGE_B);
    }
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");   // trailing empty loads

  // Has a value that is not finite met the matrix cores?  Then an accumulator is not finite either, and stays so.
  {
    uint32_t big = 0;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) big |= (__float_as_uint(oacc[db][r]) & 0x7f800000u) + 0x00800000u;      // an exponent of ones gives bit 31
    redo = redo || __any((big >> 31) != 0);
  }
  if (redo) {
    // The wavefront's rows again, key by key: a lane has the dims of its row that its accumulators hold.
    float qv[NDB][16];
    const bf16_t* qp = q + at * D + hi * 4;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        qv[db][r] = bf2f(qp[db * 32 + (r >> 2) * 8 + (r & 3)]);
        oacc[db][r] = 0.f;
      }
    m_run = -INFINITY;
    float l = 0.f;
#pragma unroll 1
    for (int t = t_lo; t < t_hi; ++t) {
      if (!active(t)) continue;
      int lo;
      uint32_t n;
      interval(t, lo, n);
      const int kb0 = tile_key(t), end = min(t < ks_.ns_t ? ks_.ns : ks_.n_keys, kb0 + KT);
#pragma unroll 1
      for (int key = kb0; key < end; ++key) {
        const int id = __builtin_amdgcn_readfirstlane(trow[key >> shift]);
        if ((unsigned)id >= (unsigned)Dm.n_pages) continue;
        const int64_t off = (int64_t)id * page_b + (key & (page - 1)) * (D * 2) + hi * 8;
        const bf16_t *kr = (const bf16_t*)(Kp + off), *vr = (const bf16_t*)(Vp + off);
        float s = 0.f;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r) s = fmaf(qv[db][r], bf2f(kr[db * 32 + (r >> 2) * 8 + (r & 3)]), s);
        s += __shfl_xor(s, 32, 64);
        const bool see = (uint32_t)(key - lo) < n;
        const float x = see ? s * c : -INFINITY, m_new = fmaxf(m_run, x), ref = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = __builtin_amdgcn_exp2f(m_run - ref), p = __builtin_amdgcn_exp2f(x - ref);
        l = l * alpha + p;
        m_run = m_new;
#pragma unroll
        for (int db = 0; db < NDB; ++db)
#pragma unroll
          for (int r = 0; r < 16; ++r)
            oacc[db][r] = oacc[db][r] * alpha + (see ? p * bf2f(vr[db * 32 + (r >> 2) * 8 + (r & 3)]) : 0.f);
      }
    }
    if (m_run == -INFINITY) m_run = 0.f;
    l_run = hi ? 0.f : l;
    if (l == 0.f)                              // only logits of -inf: 0, also where a value of weight 0 is not finite
#pragma unroll
      for (int db = 0; db < NDB; ++db)
#pragma unroll
        for (int r = 0; r < 16; ++r) oacc[db][r] = 0.f;
  }

  // ---- results ---------------------------------------------------------------------------------------------------------
  const float l = l_run + __shfl_xor(l_run, 32, 64);
  if (cut) {
    const int64_t slot = block;
    float4* op = (float4*)part + (slot * PF_NW + wave) * (NDB * 4 * 64) + lane;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq)
        op[(db * 4 + rq) * 64] = make_float4(oacc[db][rq * 4 + 0], oacc[db][rq * 4 + 1], oacc[db][rq * 4 + 2], oacc[db][rq * 4 + 3]);
    if (hi == 0) ((float2*)(part + (int64_t)PF_MAX_SLOTS * PF_ROWS * D))[slot * PF_ROWS + wave * 32 + n32] = make_float2(m_run, l);
  } else if (wave * 32 + n32 < rows) {
    const float inv = l == 0.f ? 0.f : 1.f / l;      // a row that sees nothing
    bf16_t* op = (bf16_t*)a.out + at * D;
#pragma unroll
    for (int db = 0; db < NDB; ++db)
#pragma unroll
      for (int rq = 0; rq < 4; ++rq) {
        uint2 w;
        w.x = pack_bf16(oacc[db][rq * 4 + 0] * inv, oacc[db][rq * 4 + 1] * inv);
        w.y = pack_bf16(oacc[db][rq * 4 + 2] * inv, oacc[db][rq * 4 + 3] * inv);
        *(uint2*)(op + db * 32 + rq * 8 + hi * 4) = w;
      }
    if (a.lse && hi == 0) a.lse[at] = l == 0.f ? -INFINITY : (m_run + __builtin_amdgcn_logf(l)) * 0.6931471805599453f;
  }
}

// out = sum_p w_p O_p / sum_p w_p l_p, w_p = 2^(m_p - max m), over the parts of an item that was cut.  One workgroup per (item, 32 dims), its
// threads as in the attention kernel.
template <int D>
__global__ __launch_bounds__(PF_THREADS) void paged_prefill_join_kernel(PagedAttn a, PagedDims Dm, int n_items, int parts, const float* __restrict__ part) {
  constexpr int NDB = D / 32;
  extern __shared__ __attribute__((aligned(16))) unsigned char scratch[];
  PfItem it;
  if (!pf_item(a, Dm, blockIdx.x, scratch, it)) return;
  const PfKeys k = pf_keys(it, Dm, pf_tile_keys(D));
  const int len = pf_part_len(k.n_tiles, parts), n = (k.n_tiles + len - 1) / len;
  if (n <= 1) return;
  const int db = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n32 = lane & 31, hi = lane >> 5;
  const int row = wave * 32 + n32;
  const float2* ml = (const float2*)(part + (int64_t)PF_MAX_SLOTS * PF_ROWS * D) + row;
  const float4* op = (const float4*)part + (int64_t)wave * (NDB * 4 * 64) + db * (4 * 64) + lane;
  float M = -INFINITY;
  for (int p = 0; p < n; ++p) {
    const float2 x = ml[((int64_t)p * n_items + blockIdx.x) * PF_ROWS];
    if (x.y != 0.f) M = fmaxf(M, x.x);
  }
  float acc[16], den = 0.f;
#pragma unroll
  for (int e = 0; e < 16; ++e) acc[e] = 0.f;
  for (int p = 0; p < n; ++p) {
    const int64_t slot = (int64_t)p * n_items + blockIdx.x;
    const float2 x = ml[slot * PF_ROWS];
    if (x.y == 0.f) continue;                        // saw nothing (a sum of NaN is not 0)
    const float w = __builtin_amdgcn_exp2f(x.x - M);
    den = fmaf(w, x.y, den);
#pragma unroll
    for (int rq = 0; rq < 4; ++rq) {
      const float4 o = op[slot * (PF_NW * NDB * 4 * 64) + rq * 64];
      acc[rq * 4 + 0] = fmaf(w, o.x, acc[rq * 4 + 0]);
      acc[rq * 4 + 1] = fmaf(w, o.y, acc[rq * 4 + 1]);
      acc[rq * 4 + 2] = fmaf(w, o.z, acc[rq * 4 + 2]);
      acc[rq * 4 + 3] = fmaf(w, o.w, acc[rq * 4 + 3]);
    }
  }
  if (row >= it.n_tok * Dm.g) return;
  const int64_t at = (int64_t)(it.t0 + row / Dm.g) * Dm.h + it.m * Dm.g + row % Dm.g;
  const float inv = den == 0.f ? 0.f : 1.f / den;
  bf16_t* dst = (bf16_t*)a.out + at * D + db * 32 + hi * 4;
#pragma unroll
  for (int rq = 0; rq < 4; ++rq) {
    uint2 w;
    w.x = pack_bf16(acc[rq * 4 + 0] * inv, acc[rq * 4 + 1] * inv);
    w.y = pack_bf16(acc[rq * 4 + 2] * inv, acc[rq * 4 + 3] * inv);
    *(uint2*)(dst + rq * 8) = w;
  }
  if (a.lse && hi == 0 && db == 0) a.lse[at] = den == 0.f ? -INFINITY : (M + __builtin_amdgcn_logf(den)) * 0.6931471805599453f;
}

size_t paged_prefill_workspace(const PagedDims& D) { return (size_t)PF_MAX_SLOTS * PF_ROWS * (D.d + 2) * sizeof(float); }

template <int D>
static void prefill_d(const PagedDims& Dm, const PagedAttn& a, hipStream_t st) {
  const int tw = PF_ROWS / Dm.g;
  // token tiles at most: every request's last one may be short
  int64_t tiles = ((int64_t)a.T + (int64_t)a.n_req * (tw - 1)) / tw;
  if (tiles > a.T) tiles = a.T;
  const int n_items = (int)(tiles * Dm.h_kv);
  int parts = PF_CUS / n_items;
  parts = parts < 1 ? 1 : parts > PF_MAX_PARTS ? PF_MAX_PARTS : parts;
  const dim3 n_wg = paged_grid((int64_t)n_items * parts);
  const bf16_t *q = (const bf16_t*)a.q, *K = (const bf16_t*)a.K, *V = (const bf16_t*)a.V;
  if (1 << Dm.page_shift >= pf_tile_keys(D)) paged_prefill_kernel<D, true><<<n_wg, PF_THREADS, 0, st>>>(a, q, K, V, a.table, Dm, n_items, parts, (float*)a.ws);
  else paged_prefill_kernel<D, false><<<n_wg, PF_THREADS, 0, st>>>(a, q, K, V, a.table, Dm, n_items, parts, (float*)a.ws);
  if (parts > 1)
    paged_prefill_join_kernel<D><<<dim3((unsigned)n_items, D / 32), PF_THREADS, PF_SCRATCH + (size_t)(a.n_req + 1) * sizeof(int32_t), st>>>(a, Dm, n_items, parts, (const float*)a.ws);
}

void launch_paged_prefill(const PagedDims& D, const PagedAttn& a, hipStream_t st) {
  switch (D.d) {
    case 32: prefill_d<32>(D, a, st); break;
    case 64: prefill_d<64>(D, a, st); break;
    case 96: prefill_d<96>(D, a, st); break;
    default: prefill_d<128>(D, a, st); break;
  }
}

}  // namespace locret
