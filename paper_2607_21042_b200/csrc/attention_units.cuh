// Attention of query tiles of up to 16 rows over units of 32 keys, on the warp-level tensor pipe: the batch that shares a long
// prefix, and cross attention with few queries a sequence (Section I: the decode engine's attention kernels).
//
// A tile is up to 16 query rows that read the same keys: the heads of a group for one row (its own pages), as many rows
// as fit for the shared pages, or neighbouring rows of a sequence.  For every tile, with scores s_j = scale q.k_j,
//     m = max s_j,   l = sum 2^(s_j - m),   o = sum 2^(s_j - m) v_j          (log2 units)
// over a range of its keys; the results of a tile's ranges, and of a row's two tiles, meet as
//     O = sum_p 2^(m_p - M) o_p / sum_p 2^(m_p - M) l_p,   M = max m_p,
// with M, the sums and o in fp32; zero where no key is left.
//
// Work split.  The units of all tiles are laid end to end and cut into ranges of equal size, one a warp, whatever the lengths
// are; a tile counts one unit more than its keys have, about what it costs besides them.  A tile inside one range, whose
// rows read no other keys, is finished by its warp.  The others' parts go to scratch and are added in the order of their keys, so
// that results do not depend on timing and no warp waits for another:
//   - by the CTA that comes last, at its end (cross attention, where only the tiles at a CTA's two ends reach another; few rows over
//     a shared prefix): a barrier, a fence and an atomic per tile, once a CTA;
//   - by a second kernel (many rows over a shared prefix, each of which reads two tiles).  The same tickets there took a warp with
//     twenty short rows 100 us: fence, atomic and reads at each of them.
//
// Instructions.  Queries are the 16-row operand of m16n8k16, keys the 8-wide one, so the scores come out in the layout in which
// P enters P V.  Queries in fp32 enter as two bf16 parts (16 bits), P is rounded to the cache's type (half a step of it: as
// much again as the rounding of the output).  A warp copies two units ahead (three of the 8-bit cache), as 16-key boxes of K and of V
// with the 128-byte swizzle; of the 8-bit cache as plain rows, whose codes become bf16 in registers (exact).
//
// Bound and measurements.  Where each row has keys of its own, the bytes: 128 rows behind 1024 shared tokens, 3 to 900 of their own,
// 20 heads, bf16, 302 MB: 64 us, 4.7 TB/s, of which the start and the second kernel take 8; 16 queries of one token by 100 to 1500
// keys, 20 heads, 65 MB: 20 us, half of them the start, the tickets and the merge.  Where many rows share keys, instructions: 300 rows of 20 heads
// by 4, 1536 shared tokens, 8 bits: 44.5 us, 59 TFLOP/s, 63 % of the issue slots and 54 % of the ALU pipe, which widens the codes anew for each tile
// of 16 rows; the tensor pipe is at 18 % (m16n8k16 alone gives 555 TFLOP/s here, a third of tcgen05).  16 by 32 queries by 90 to 1500
// keys: 30 us, latency: 29 % of the issue slots, 15 % of the tensor pipe, K and V read by two warps.  Five rows behind 448 tokens: 10.8 us,
// latency from end to end.
// Measured and not kept (us for 128 rows / 300 rows above): tiles of 32 rows 83 / 51; queries as the 8-wide operand 65 and 12.3 for five
// rows; tickets instead of the second kernel 79 / 56.
#pragma once
#include "attention_common.cuh"
#include "page_tables.cuh"
#include "tensor_map.cuh"

namespace ttsgpt {

constexpr int kUnWarps = 12;
constexpr int kUnKeys = 32;                 // keys of a unit: two to a page
constexpr int kUnBox = 16;                  // keys of one copy
constexpr int kUnTile = 16;                 // query rows of a tile
constexpr int kUnMaxSeq = 4096;             // rows (shared) or sequences (cross) of a call
constexpr int kUnMaxCtas = 160;
constexpr int kUnMaxWarps = kUnMaxCtas * kUnWarps;
constexpr int kUnMaxTiles = 64;             // tiles that a CTA can merge
constexpr int kUnTickets = 16384;
constexpr int kUnPitch = 68;                // floats of a partial row: o[64], m, l, and two to keep 16-byte rows
constexpr unsigned long long kUnWaitNs = 2000000000ull;

enum { KV_BF16 = 0, KV_F16 = 1, KV_E4M3 = 2 };   // what the keys and values are stored as

struct UnitArgs {
  const void *q;
  uint16_t *out;                // [rows][H * 64]
  long long q_stride;           // elements between query rows
  int q_rows, H, Hkv, G;        // G = H / Hkv query heads share a head of keys
  int rpt;                      // query rows of a tile: 16 / G, or two halves of 128 / G
  Div by_G, by_rpt, by_H, by_Hkv;
  // shared prefix: its tiles of a head of keys (0 without one), and the units of each of them
  int tiles_head, prefix_nu;
  Div by_tiles_head, by_prefix_nu;
  float scale;                  // of the scores, in log2 units
  // shared prefix: pages
  const int *page_table, *row_stream, *row_pos;
  const unsigned char *pool;
  int pps, n_shared, n_pages;
  // cross: sequences
  const int *q_start, *k_start;
  int n_seq, q_max, k_rows, few_rows;   // few_rows: a warp a row merges
  // scratch
  int *err;                     // [0]: set when a wait ran out; rows that are then not computed become NaN
  unsigned long long wait_ns;   // that a wait may take (in the tiles kernel always kUnWaitNs: as an argument it cost 1 % there)
  int starve;                   // test aid: the CTA whose copies never count as complete; -1: none
  unsigned *tickets;            // zero between calls; null: the second kernel merges
  int *plan;                    // ... which finds here {units of a range (a Div), running sums of units}
  float *part;
  int suffix_part0;             // partial row at which those of the rows' own tiles begin

  void set_heads(int n_head, int n_kv_head, int rows) {
    H = n_head; Hkv = n_kv_head; G = H / Hkv; rpt = rows;
    by_G.set(G); by_rpt.set(rpt); by_H.set(H); by_Hkv.set(Hkv);
    by_tiles_head.set(1); by_prefix_nu.set(1);
  }
  void set_shared(int pages) {
    n_shared = pages;
    tiles_head = pages > 0 ? (q_rows + rpt - 1) / rpt : 0;
    prefix_nu = 2 * pages + 1;
    by_tiles_head.set(tiles_head > 0 ? tiles_head : 1); by_prefix_nu.set(prefix_nu);
  }
};

template <int KV> struct UnitLayout {
  static constexpr int kStages = KV == KV_E4M3 ? 3 : 2;
  static constexpr int kHalf = KV == KV_E4M3 ? kUnKeys * kHeadDim : kUnKeys * kHeadDim * 2;   // K (or V) of a unit
  static constexpr int kStage = KV == KV_E4M3 ? 2 * kHalf + 2 * kUnKeys * 4 : 2 * kHalf;   // codes of K and V, scales of K and V
};
template <int KV> inline size_t units_smem_bytes(int n) {
  return (size_t)kUnWarps * UnitLayout<KV>::kStages * UnitLayout<KV>::kStage + 1024 + kUnWarps * UnitLayout<KV>::kStages * 8 + (size_t)(2 * n + 1) * 4 + 64;
}

template <bool F16>
__device__ __forceinline__ void un_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (F16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else mma_bf16_16816(c, a[0], a[1], a[2], a[3], b0, b1);
}
// First partial row of a part.  A tile's parts are numbered tile + range, which never repeats along the units; sequences, whose
// tiles only meet where a range ends, have two places a range: for the tile that goes on behind it, and the one that began before.
__device__ __forceinline__ size_t prefix_part(int tile, int range) { return (size_t)(tile + range) * kUnTile; }
__device__ __forceinline__ size_t own_part(const UnitArgs &a, int row, int kvh, int range) { return (size_t)a.suffix_part0 + (size_t)(row * a.Hkv + kvh + range) * a.G; }
__device__ __forceinline__ size_t seq_part(int range, bool begins) { return (size_t)(2 * range + (begins ? 1 : 0)) * kUnTile; }

// The parts of a query row, added in the order of their keys by 8 PG lanes: lane group pg takes every PG-th part, a lane eight
// dimensions.  part(p): the p-th of n partial rows.  sound: no wait has run out; otherwise the row is NaN.
template <int PG, bool F16, typename Part>
__device__ __forceinline__ void merge_parts(int n, Part part, uint16_t *out, bool store, bool sound) {
  const int sub = threadIdx.x & 7, pg = (threadIdx.x >> 3) & (PG - 1);
  float M = -INFINITY, l = 0.f, acc[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = 0.f;
  auto add = [&](float m, float pl, const float (&v)[8]) {
    if (pl == 0.f) return;                     // no key in it; a sum that is NaN goes in
    const float Mn = fmaxf(M, m), fo = M == Mn ? 1.f : pt_exp2(M - Mn), fn = pt_exp2(m - Mn);
    M = Mn;
    l = fmaf(l, fo, pl * fn);
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] = fmaf(acc[c], fo, v[c] * fn);
  };
#pragma unroll 2
  for (int p = pg; p < n; p += PG) {
    const float *x = part(p);
    const float2 ml = __ldcg(reinterpret_cast<const float2 *>(x + kHeadDim));
    const float4 a = __ldcg(reinterpret_cast<const float4 *>(x + 8 * sub)), b = __ldcg(reinterpret_cast<const float4 *>(x + 8 * sub + 4));
    const float v[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    add(ml.x, ml.y, v);
  }
#pragma unroll
  for (int o = 8; o < 8 * PG; o <<= 1) {       // the groups' sums, the lower group's first
    const float m2 = __shfl_down_sync(0xFFFFFFFFu, M, o), l2 = __shfl_down_sync(0xFFFFFFFFu, l, o);
    float v[8];
#pragma unroll
    for (int c = 0; c < 8; ++c) v[c] = __shfl_down_sync(0xFFFFFFFFu, acc[c], o);
    add(m2, l2, v);
  }
  if (store && pg == 0) {
    const float inv = !sound ? __int_as_float(0x7FFFFFFF) : l == 0.f ? 0.f : 1.0f / l;
    *reinterpret_cast<uint4 *>(out + 8 * sub) = make_uint4(un_pack<F16>(acc[0] * inv, acc[1] * inv), un_pack<F16>(acc[2] * inv, acc[3] * inv),
                                                           un_pack<F16>(acc[4] * inv, acc[5] * inv), un_pack<F16>(acc[6] * inv, acc[7] * inv));
  }
}

// Where the parts of a query row over a shared prefix are: those of its prefix tile, then those of its own keys.
struct RowParts {
  int p_n, o_n;
  size_t pp, op;
  __device__ __forceinline__ const float *at(const UnitArgs &a, int k) const {
    return a.part + (k < p_n ? pp + (size_t)k * kUnTile : op + (size_t)(k - p_n) * a.G) * kUnPitch;
  }
};
// size: units of a range; f0, f1: running sums of units of the row and of the next
__device__ __forceinline__ RowParts row_parts(const UnitArgs &a, int r, int kvh, int gi, const Div &size, int f0, int f1) {
  const int nu = f1 - f0;
  RowParts x = {0, 0, 0, 0};
  if (a.tiles_head > 0) {
    const int row_tile = a.by_rpt.of(r), tile = kvh * a.tiles_head + row_tile, u0 = tile * a.prefix_nu, w0 = size.of(u0);
    x.p_n = size.of(u0 + a.prefix_nu - 1) - w0 + 1;
    x.pp = prefix_part(tile, w0) + (r - row_tile * a.rpt) * a.G + gi;
  }
  if (nu > 0) {
    const int u0 = a.Hkv * (a.tiles_head * a.prefix_nu + f0) + kvh * nu, w0 = size.of(u0);
    x.o_n = size.of(u0 + nu - 1) - w0 + 1;
    x.op = own_part(a, r, kvh, w0) + gi;
  }
  return x;
}

template <int N> struct IntC { static constexpr int value = N; };

// what a unit is; one per lane, 32 units at a time
struct UnitDesc {
  int c1, c2;      // where its keys lie: token of the page and block of the pool, or head and token row
  int n;           // keys that exist (0: nothing is copied)
  int u0, nu;      // first unit and units of its tile
  int row0;        // first query row of the tile
  int hn;          // head of keys | query rows times heads of the tile << 16
  int own;         // shared prefix: 1: the keys are the row's own
};

// SHARED: pages, common ones first; otherwise sequences of their own.  KV: KV_*.  QF32: queries in fp32, else of the keys' type
// (bf16 for the 8-bit cache).
template <bool SHARED, int KV, bool QF32>
__global__ void __launch_bounds__(kUnWarps * 32, 1) attention_units_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                                                                           const UnitArgs a) {
  using L = UnitLayout<KV>;
  constexpr bool F16 = KV == KV_F16;
  extern __shared__ __align__(16) unsigned char un_smem_raw[];
  unsigned char *stages = un_smem_raw + ((1024u - (smem_u32(un_smem_raw) & 1023u)) & 1023u);
  uint64_t *bars = reinterpret_cast<uint64_t *>(stages + (size_t)kUnWarps * L::kStages * L::kStage);
  int *first = reinterpret_cast<int *>(bars + kUnWarps * L::kStages);   // running sums of units: of a head of each row, or of all tiles of each sequence
  int *stream_s = first + (SHARED ? a.q_rows : a.n_seq) + 1;             // shared: the rows' streams
  __shared__ int warp_tot[kUnWarps];
  __shared__ int4 tile_s[kUnMaxTiles];         // tiles whose parts this CTA may have to add: {first unit | own << 31, units, first row, heads and rows}
  __shared__ int n_tile_s, n_item_s;
  __shared__ Div size_s, aw_s;
  __shared__ unsigned long long lead_s;   // keys of the longest row, and that row: its list names the shared pages
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int n_items = SHARED ? a.q_rows : a.n_seq;

  const int failed = __ldcg(a.err);            // by an earlier call, unless the scratch has been zeroed since
  if (lane < L::kStages) mbar_init(&bars[warp * L::kStages + lane], (int)blockIdx.x == a.starve ? 2 : 1);
  if (tid == 0) {
    lead_s = 0; n_tile_s = 0; n_item_s = 0;
    if constexpr (KV != KV_E4M3) {
      asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
      if (!SHARED) asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
  }
  __syncthreads();
  // ---- running sums ----
  auto q_span = [&](int i, int &b, int &e) {   // query rows of a sequence
    b = min(max(a.q_start[i], 0), a.q_rows);
    e = min(min(max(a.q_start[i + 1], b), a.q_rows), b + a.q_max);
  };
  auto k_span = [&](int i, int &b, int &e) {
    b = min(max(a.k_start[i], 0), a.k_rows);
    e = min(max(a.k_start[i + 1], b), a.k_rows);
  };
  const int prefix_keys = SHARED ? a.n_shared * kPageTokens : 0;
  auto row_keys = [&](int r) { return min(max(a.row_pos[r], -1), a.pps * kPageTokens - 1) + 1; };   // of a row of no stream: none, whatever this says
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose units nothing bounds
  for (int base = 0; base < n_items; base += kUnWarps * 32) {
    const int i = base + tid;
    int u = 0;
    if (i < n_items) {
      if (SHARED) {
        const int s = a.row_stream[i], all = row_keys(i), keys = s < 0 ? 0 : all, n = keys - prefix_keys;   // n may be negative
        stream_s[i] = s;
        atomicMax(&lead_s, ((unsigned long long)(unsigned)keys << 32) | (unsigned)i);
        u = n > 0 ? 1 + (n + kUnKeys - 1) / kUnKeys : (a.n_shared == 0 ? 1 : 0);   // a row without any key still gets its zeros
      } else {
        int qb, qe, kb, ke;
        q_span(i, qb, qe);
        k_span(i, kb, ke);
        bad |= a.q_start[i + 1] < a.q_start[i] || a.k_start[i + 1] < a.k_start[i];
        u = a.Hkv * a.by_rpt.of(qe - qb + a.rpt - 1) * (1 + (ke - kb + kUnKeys - 1) / kUnKeys);
      }
    }
    int incl = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) warp_tot[warp] = incl;
    if constexpr (SHARED) __syncthreads();
    else bad = __syncthreads_or(bad);
    int before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < kUnWarps; ++w) { if (w < warp) before += warp_tot[w]; all += warp_tot[w]; }
    if (i < n_items) first[i] = before + incl - u;
    carry = all;
  }
  if (bad) carry = 0;
  if (tid == 0) first[n_items] = carry;
  __syncthreads();
  const int lead = (int)(lead_s & 0xFFFFFFFFu), lead_keys = (int)(lead_s >> 32);
  const int tiles_head = SHARED ? a.tiles_head : 0, prefix_nu = a.prefix_nu;
  const int U_prefix = SHARED ? a.Hkv * tiles_head * prefix_nu : 0;
  const int T = U_prefix + carry * (SHARED ? a.Hkv : 1);
  // ranges of `size` units, at least two; a CTA's are neighbours, `aw` of them, so that all CTAs have some
  if (tid == 0) {
    const int n = (int)gridDim.x * kUnWarps, units = max(2, (T + n - 1) / n), ranges = (T + units - 1) / units;
    size_s.set(units);
    aw_s.set(max(1, (ranges + (int)gridDim.x - 1) / (int)gridDim.x));
  }
  __syncthreads();
  const Div size = size_s;
  const int aw = aw_s.d, w_cta = blockIdx.x * aw, w = w_cta + warp;
  const int u_begin = w * (int)size.d, n_mine = warp < aw ? min(max(T - u_begin, 0), (int)size.d) : 0;
  auto warp_of = [&](int u) { return size.of(u); };
  if (SHARED && !a.tickets && blockIdx.x == 0) {
    for (int i = tid; i <= n_items; i += kUnWarps * 32) a.plan[sizeof(Div) / 4 + i] = first[i];
    if (tid == 0) *reinterpret_cast<Div *>(a.plan) = size;
  }
  pdl_launch_dependents();

  auto find = [&](int x) {   // last item that begins at or before x
    int lo = 0, hi = n_items - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (first[m] <= x) lo = m; else hi = m - 1; }
    return lo;
  };
  auto describe = [&](int u) {
    UnitDesc d = {0, 0, 0, u, 1, 0, 0, 0};
    if (u >= u_begin + n_mine) return d;
    if constexpr (SHARED) {
      int r, kvh, page, n, list, kk;            // unit 0 of a tile has no keys: it stands for what a tile costs besides them
      if (u < U_prefix) {
        const int tile = a.by_prefix_nu.of(u), k = u - tile * prefix_nu;
        kvh = a.by_tiles_head.of(tile);
        r = (tile - kvh * tiles_head) * a.rpt;
        d.u0 = u - k; d.nu = prefix_nu;
        d.hn = kvh | (min(a.rpt, a.q_rows - r) * a.G << 16);
        kk = k - 1;
        page = kk >> 1; list = lead;
        n = min(kUnKeys, lead_keys - kk * kUnKeys);   // a page of the shared ones holds 64 keys, unless no row is that long
      } else {
        const int v = u - U_prefix;
        r = find(a.by_Hkv.of(v));
        const int nu = first[r + 1] - first[r], x = v - first[r] * a.Hkv;
        kvh = (int)((unsigned)x / (unsigned)nu);
        const int k = x - kvh * nu;
        d.u0 = u - k; d.nu = nu; d.own = 1;
        d.hn = kvh | (a.G << 16);
        kk = k - 1;
        page = a.n_shared + (kk >> 1); list = r;
        n = kk < 0 ? 0 : min(kUnKeys, row_keys(r) - prefix_keys - kk * kUnKeys);
      }
      d.row0 = r;
      d.c1 = (kk & 1) * kUnKeys;
      if (kk >= 0 && stream_s[list] >= 0) {
        const int phys = a.page_table[(size_t)stream_s[list] * a.pps + page];
        if (n > 0 && phys >= 0 && phys < a.n_pages) { d.n = n; d.c2 = phys * 2 * a.Hkv + kvh; }   // a page that is none has no keys
      }
    } else {
      const int s = find(u), x = u - first[s];
      int qb, qe, kb, ke;
      q_span(s, qb, qe);
      k_span(s, kb, ke);
      const int nu = 1 + (ke - kb + kUnKeys - 1) / kUnKeys, tile = (int)((unsigned)x / (unsigned)nu), k = x - tile * nu;
      const int blocks = a.by_rpt.of(qe - qb + a.rpt - 1), kvh = (int)((unsigned)tile / (unsigned)blocks);
      d.row0 = qb + (tile - kvh * blocks) * a.rpt;
      d.u0 = u - k; d.nu = nu;
      d.hn = kvh | (min(a.rpt, qe - d.row0) * a.G << 16);
      d.c1 = kvh; d.c2 = kb + (k - 1) * kUnKeys;
      d.n = k == 0 ? 0 : min(kUnKeys, ke - d.c2);
    }
    return d;
  };

  unsigned char *stage0 = stages + (size_t)warp * L::kStages * L::kStage;
  uint64_t *bar = bars + warp * L::kStages;
  UnitDesc nxt = {}, cur = {};                          // descriptions of the units being copied, and of those being computed
  bool whole = true, dead = __any_sync(0xFFFFFFFFu, failed != 0);   // dead: nothing is copied or computed any more, rows become NaN
  auto issue = [&](int i) {                   // unit u_begin + i into stage i % kStages
    if ((i & 31) == 0) nxt = describe(u_begin + i + lane);
    const int c1 = __shfl_sync(0xFFFFFFFFu, nxt.c1, i & 31), c2 = __shfl_sync(0xFFFFFFFFu, nxt.c2, i & 31), n = __shfl_sync(0xFFFFFFFFu, nxt.n, i & 31);
    unsigned char *st = stage0 + (size_t)(i % L::kStages) * L::kStage;
    uint64_t *b = &bar[i % L::kStages];
    if (!dead && elect_one()) {
      if constexpr (KV == KV_E4M3) {
        const uint32_t codes = (uint32_t)n * kHeadDim, scales = (uint32_t)(n + 3) / 4 * 16;
        mbar_expect_tx(b, 2 * (codes + scales));
        if (n > 0) {
          const unsigned char *kp = a.pool + (size_t)c2 * kE4m3BlockBytes, *vp = kp + (size_t)a.Hkv * kE4m3BlockBytes;
          bulk_copy_g2s(st, kp + c1 * kHeadDim, codes, b);
          bulk_copy_g2s(st + 2 * L::kHalf, kp + kPageTokens * kHeadDim + 4 * c1, scales, b);
          bulk_copy_g2s(st + L::kHalf, vp + c1 * kHeadDim, codes, b);
          bulk_copy_g2s(st + 2 * L::kHalf + kUnKeys * 4, vp + kPageTokens * kHeadDim + 4 * c1, scales, b);
        }
      } else {
        const int boxes = (n + kUnBox - 1) / kUnBox;
        mbar_expect_tx(b, (uint32_t)boxes * 2 * kUnBox * 128);
#pragma unroll
        for (int x = 0; x < kUnKeys / kUnBox; ++x)
          if (x < boxes) {
            const int o = x * kUnBox;
            if constexpr (SHARED) {
              un_box(&k_map, c1 + o, c2, st + o * 128, b);
              un_box(&v_map, c1 + o, c2 + a.Hkv, st + L::kHalf + o * 128, b);
            } else {
              un_box(&k_map, c2 + o, c1, st + o * 128, b);
              un_box(&v_map, c2 + o, c1, st + L::kHalf + o * 128, b);
            }
          }
      }
    }
    __syncwarp();
  };

  // ---- state of the tile ----
  uint32_t qa[4][4], qlo[QF32 ? 4 : 1][4];    // query fragments by 16 dimensions; fp32: what the first part leaves
  float o[8][4], m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;   // rows g and g + 8
  int tile_u0 = -1, tile_nu = 0, row0 = 0, kvh = 0, n_i = 0, own = 0, vis0 = 0, vis1 = 0;

  auto q_ptr = [&](int i) { const int r = a.by_G.of(i); return (size_t)(row0 + r) * a.q_stride + (size_t)((kvh - r) * a.G + i) * kHeadDim; };
  auto load_q = [&]() {
    const bool h0 = g < n_i, h1 = g + 8 < n_i;
    const size_t p0 = h0 ? q_ptr(g) : 0, p1 = h1 ? q_ptr(g + 8) : 0;
#pragma unroll
    for (int ks = 0; ks < 4; ++ks)
#pragma unroll
      for (int f = 0; f < 4; ++f) {           // fragment f: row g + 8 (f & 1), upper half of the dimensions where f >= 2
        const int dim = KV == KV_E4M3 ? 16 * t + 4 * ks + 2 * (f >> 1) : 16 * ks + 2 * t + 8 * (f >> 1);
        const bool have = f & 1 ? h1 : h0;
        const size_t p = (f & 1 ? p1 : p0) + dim;
        if constexpr (QF32) {
          const float2 x = have ? *reinterpret_cast<const float2 *>(reinterpret_cast<const float *>(a.q) + p) : make_float2(0.f, 0.f);
          const float hx = __uint_as_float(__float_as_uint(x.x) & 0xFFFF0000u), hy = __uint_as_float(__float_as_uint(x.y) & 0xFFFF0000u);
          qa[ks][f] = pack_bf16x2(hx, hy);
          qlo[ks][f] = pack_bf16x2(x.x - hx, x.y - hy);
        } else {
          qa[ks][f] = have ? *reinterpret_cast<const uint32_t *>(reinterpret_cast<const uint16_t *>(a.q) + p) : 0u;
        }
      }
  };
  auto out_ptr = [&](int i) { const int r = a.by_G.of(i); return a.out + ((size_t)(row0 + r) * a.H + (kvh - r) * a.G + i) * kHeadDim; };

  auto finish = [&]() {                       // the warp leaves its tile
    l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 1); l0 += __shfl_xor_sync(0xFFFFFFFFu, l0, 2);
    l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 1); l1 += __shfl_xor_sync(0xFFFFFFFFu, l1, 2);
    const int last = tile_u0 + tile_nu - 1;
    const int w0 = warp_of(tile_u0), w1 = warp_of(last);
    // does nothing else feed this tile's rows?
    const bool alone = w0 == w1 && (!SHARED || (own && tiles_head == 0));
    if (alone || dead) {                       // (dead: NaN, whoever merges the tile's parts finds the error too)
      const float nan = __int_as_float(0x7FFFFFFF);
      const float i0 = dead ? nan : l0 > 0.f || l0 != l0 ? 1.0f / l0 : 0.f, i1 = dead ? nan : l1 > 0.f || l1 != l1 ? 1.0f / l1 : 0.f;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        if (g + 8 * e < n_i) {
          uint16_t *dst = out_ptr(g + 8 * e);
          const float inv = e ? i1 : i0;
          if constexpr (KV == KV_E4M3) {
#pragma unroll
            for (int hf = 0; hf < 2; ++hf)
              *reinterpret_cast<uint4 *>(dst + 16 * t + 8 * hf) =
                  make_uint4(un_pack<F16>(o[0][2 * e + hf] * inv, o[1][2 * e + hf] * inv), un_pack<F16>(o[2][2 * e + hf] * inv, o[3][2 * e + hf] * inv),
                             un_pack<F16>(o[4][2 * e + hf] * inv, o[5][2 * e + hf] * inv), un_pack<F16>(o[6][2 * e + hf] * inv, o[7][2 * e + hf] * inv));
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) *reinterpret_cast<uint32_t *>(dst + 8 * j + 2 * t) = un_pack<F16>(o[j][2 * e] * inv, o[j][2 * e + 1] * inv);
          }
        }
      }
      if (alone) return;
    }
    // this part into scratch
    float *dst = a.part + (SHARED ? (own ? own_part(a, row0, kvh, w) : prefix_part(a.by_prefix_nu.of(tile_u0), w)) : seq_part(w, w == w0)) * kUnPitch;
#pragma unroll
    for (int e = 0; e < 2; ++e)
      if (g + 8 * e < n_i) {
        float *p = dst + (g + 8 * e) * kUnPitch;
        if constexpr (KV == KV_E4M3) {
#pragma unroll
          for (int q = 0; q < 4; ++q)
            *reinterpret_cast<float4 *>(p + 16 * t + 4 * q) = make_float4(o[4 * (q & 1)][2 * e + (q >> 1)], o[4 * (q & 1) + 1][2 * e + (q >> 1)],
                                                                          o[4 * (q & 1) + 2][2 * e + (q >> 1)], o[4 * (q & 1) + 3][2 * e + (q >> 1)]);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) *reinterpret_cast<float2 *>(p + 8 * j + 2 * t) = make_float2(o[j][2 * e], o[j][2 * e + 1]);
        }
        if (t == 0) { p[64] = e ? m1 : m0; p[65] = e ? l1 : l0; }
      }
    // the tile's first range of this CTA enters it
    if (a.tickets && w == max(w0, w_cta) && lane == 0) {
      const int i = atomicAdd(&n_tile_s, 1);
      if (i < kUnMaxTiles) tile_s[i] = make_int4(tile_u0 | (own << 31), tile_nu, row0, kvh | (n_i << 16));
    }
  };

  // turn i copies unit i and computes unit i - kStages, whose stage it frees; one place for each in the code, which is fetched cold
#pragma unroll 1
  for (int turn = 0;; ++turn) {
    const int idx = turn - L::kStages;
    if (idx >= 0) {
      if ((idx & 31) == 0) cur = nxt;            // copies run a few units ahead: `nxt` still describes these
      const bool end = idx >= n_mine;
      const int u0 = end ? -2 : __shfl_sync(0xFFFFFFFFu, cur.u0, idx & 31), n = __shfl_sync(0xFFFFFFFFu, cur.n, idx & 31);
      if (u0 != tile_u0) {
        if (tile_u0 >= 0) finish();
        if (end) break;
        tile_u0 = u0;
        tile_nu = __shfl_sync(0xFFFFFFFFu, cur.nu, idx & 31);
        row0 = __shfl_sync(0xFFFFFFFFu, cur.row0, idx & 31);
        const int hn = __shfl_sync(0xFFFFFFFFu, cur.hn, idx & 31);
        own = __shfl_sync(0xFFFFFFFFu, cur.own, idx & 31);
        kvh = hn & 0xffff; n_i = hn >> 16;
        load_q();
        whole = true;
        if constexpr (SHARED) {
          if (!own) {                            // a row may end inside the shared pages
            const int r0 = row0 + a.by_G.of(min(g, n_i - 1)), r1 = row0 + a.by_G.of(min(g + 8, n_i - 1)), k0 = row_keys(r0), k1 = row_keys(r1);
            vis0 = stream_s[r0] < 0 ? 0 : k0;
            vis1 = stream_s[r1] < 0 ? 0 : k1;
            whole = __all_sync(0xFFFFFFFFu, vis0 >= prefix_keys && vis1 >= prefix_keys);
          }
        }
        m0 = m1 = -INFINITY; l0 = l1 = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
      }
      const int s = idx % L::kStages;
      unsigned char *st = stage0 + (size_t)s * L::kStage;
      if (!dead && !mbar_wait_bounded(&bar[s], (uint32_t)(idx / L::kStages) & 1u, a.wait_ns)) {
        atomicExch(a.err, 1);
        dead = true;
        const unsigned long long t0 = global_timer_ns();   // copies of the warp may still be in flight, and none may land in a CTA that has left
        while (global_timer_ns() - t0 <= 10000000ull) {}
      }
      dead = __any_sync(0xFFFFFFFFu, dead);
      if (n > 0 && !dead) {
        const uint32_t k_base = smem_u32(st), v_base = k_base + L::kHalf;
        float sc[4][4];
#pragma unroll
        for (int j = 0; j < 4; ++j) sc[j][0] = sc[j][1] = sc[j][2] = sc[j][3] = 0.f;
        if constexpr (KV == KV_E4M3) {
          const float *ks = reinterpret_cast<const float *>(st + 2 * L::kHalf);
#pragma unroll
          for (int j = 0; j < 4; ++j) {          // eight keys: lane (g, t) holds dimensions 16 t .. 16 t + 15 of key g
            const uint4 c = *reinterpret_cast<const uint4 *>(st + (8 * j + g) * kHeadDim + 16 * t);
            const uint32_t cw[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4) {
              const uint32_t b0 = e4m3x2_to_bf16x2(__byte_perm(cw[k4], 0u, 0x1404)), b1 = e4m3x2_to_bf16x2(__byte_perm(cw[k4], 0u, 0x3424));
              un_mma<false>(sc[j], qa[k4], b0, b1);
              if constexpr (QF32) un_mma<false>(sc[j], qlo[k4], b0, b1);
            }
            const float2 f = *reinterpret_cast<const float2 *>(ks + 8 * j + 2 * t);
            sc[j][0] *= f.x; sc[j][1] *= f.y; sc[j][2] *= f.x; sc[j][3] *= f.y;
          }
        } else {
          // V rows without a key may hold NaN, and 0 * NaN must not reach O
          if (n < kUnKeys) {
            const int zero_to = min(kUnKeys, (n + kUnBox - 1) / kUnBox * kUnBox);
            for (int i = n * 8 + lane; i < zero_to * 8; i += 32) *reinterpret_cast<uint4 *>(st + L::kHalf + i * 16) = make_uint4(0, 0, 0, 0);
            __syncwarp();
          }
#pragma unroll
          for (int np = 0; np < 2; ++np) {
            if (np * kUnBox >= n) break;
            const int key = 16 * np + 8 * (lane >> 4) + (lane & 7);
#pragma unroll
            for (int k4 = 0; k4 < 4; ++k4) {
              uint32_t f[4];
              ldmatrix_x4(f, k_base + key * 128 + (((2 * k4 + ((lane >> 3) & 1)) ^ (key & 7)) << 4));
              un_mma<F16>(sc[2 * np], qa[k4], f[0], f[1]);
              un_mma<F16>(sc[2 * np + 1], qa[k4], f[2], f[3]);
              if constexpr (QF32) {
                un_mma<F16>(sc[2 * np], qlo[k4], f[0], f[1]);
                un_mma<F16>(sc[2 * np + 1], qlo[k4], f[2], f[3]);
              }
            }
          }
        }
        if (n < kUnKeys || !whole) {
          const int k0 = (u_begin + idx - tile_u0 - 1) * kUnKeys;
          const int lim0 = whole ? n : min(n, vis0 - k0), lim1 = whole ? n : min(n, vis1 - k0);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int c = 8 * j + 2 * t;
            if (c >= lim0) sc[j][0] = -INFINITY;
            if (c + 1 >= lim0) sc[j][1] = -INFINITY;
            if (c >= lim1) sc[j][2] = -INFINITY;
            if (c + 1 >= lim1) sc[j][3] = -INFINITY;
          }
        }
        float x0 = -INFINITY, x1 = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) { x0 = fmaxf(x0, fmaxf(sc[j][0], sc[j][1])); x1 = fmaxf(x1, fmaxf(sc[j][2], sc[j][3])); }
        x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 1)); x0 = fmaxf(x0, __shfl_xor_sync(0xFFFFFFFFu, x0, 2));
        x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 1)); x1 = fmaxf(x1, __shfl_xor_sync(0xFFFFFFFFu, x1, 2));
        const float n0 = fmaxf(m0, x0 * a.scale), n1 = fmaxf(m1, x1 * a.scale);
        const float r0 = n0 == -INFINITY ? 0.f : n0, r1 = n1 == -INFINITY ? 0.f : n1;   // a row that has seen nothing keeps -inf
        const float f0 = pt_exp2(m0 - r0), f1 = pt_exp2(m1 - r1);
        m0 = n0; m1 = n1;
        float s0 = 0.f, s1 = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          sc[j][0] = pt_exp2(fmaf(sc[j][0], a.scale, -r0)); sc[j][1] = pt_exp2(fmaf(sc[j][1], a.scale, -r0));
          sc[j][2] = pt_exp2(fmaf(sc[j][2], a.scale, -r1)); sc[j][3] = pt_exp2(fmaf(sc[j][3], a.scale, -r1));
          s0 += sc[j][0] + sc[j][1];
          s1 += sc[j][2] + sc[j][3];
        }
        l0 = fmaf(l0, f0, s0); l1 = fmaf(l1, f1, s1);
        if (__any_sync(0xFFFFFFFFu, f0 != 1.0f || f1 != 1.0f)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) { o[j][0] *= f0; o[j][1] *= f0; o[j][2] *= f1; o[j][3] *= f1; }
        }
        if constexpr (KV == KV_E4M3) {
          const float *vs = reinterpret_cast<const float *>(st + 2 * L::kHalf + kUnKeys * 4);
#pragma unroll
          for (int j = 0; j < 4; ++j) {          // the values' scales belong to P; a key that is none may have any
            const float2 f = *reinterpret_cast<const float2 *>(vs + 8 * j + 2 * t);
            const float fx = 8 * j + 2 * t < n ? f.x : 0.f, fy = 8 * j + 2 * t + 1 < n ? f.y : 0.f;
            sc[j][0] *= fx; sc[j][1] *= fy; sc[j][2] *= fx; sc[j][3] *= fy;
          }
        }
#pragma unroll
        for (int np = 0; np < 2; ++np) {
          if (np * kUnBox >= n) break;
          const uint32_t pa[4] = {un_pack<F16>(sc[2 * np][0], sc[2 * np][1]), un_pack<F16>(sc[2 * np][2], sc[2 * np][3]),
                                  un_pack<F16>(sc[2 * np + 1][0], sc[2 * np + 1][1]), un_pack<F16>(sc[2 * np + 1][2], sc[2 * np + 1][3])};
          if constexpr (KV == KV_E4M3) {
            const unsigned char *vp = st + L::kHalf + (16 * np + 2 * t) * kHeadDim + 8 * g;   // dimensions 8 g .. 8 g + 7 of four keys
            const uint2 v0 = *reinterpret_cast<const uint2 *>(vp), v1 = *reinterpret_cast<const uint2 *>(vp + kHeadDim);
            const uint2 v8 = *reinterpret_cast<const uint2 *>(vp + 8 * kHeadDim), v9 = *reinterpret_cast<const uint2 *>(vp + 9 * kHeadDim);
#pragma unroll
            for (int j = 0; j < 8; ++j) {        // byte j of the first key below, of the second above
              constexpr uint32_t sel[4] = {0x4000, 0x5010, 0x6020, 0x7030};
              const uint32_t b0 = e4m3x2_to_bf16x2(__byte_perm(j < 4 ? v0.x : v0.y, j < 4 ? v1.x : v1.y, sel[j & 3]));
              const uint32_t b1 = e4m3x2_to_bf16x2(__byte_perm(j < 4 ? v8.x : v8.y, j < 4 ? v9.x : v9.y, sel[j & 3]));
              un_mma<false>(o[j], pa, b0, b1);
            }
          } else {
            const int key = 16 * np + 8 * ((lane >> 3) & 1) + (lane & 7);
#pragma unroll
            for (int dp = 0; dp < 4; ++dp) {
              uint32_t f[4];
              ldmatrix_x4_trans(f, v_base + key * 128 + (((2 * dp + (lane >> 4)) ^ (key & 7)) << 4));
              un_mma<F16>(o[2 * dp], pa, f[0], f[1]);
              un_mma<F16>(o[2 * dp + 1], pa, f[2], f[3]);
            }
          }
        }
      }
      // every lane has read the stage: refill it
      fence_proxy_async_smem();
      __syncwarp();
    }
    if (turn < n_mine) issue(turn);
  }
  if (a.tickets) {
    __threadfence();
    __syncthreads();
    const int n_tile = min(n_tile_s, kUnMaxTiles);
    int *item_s = reinterpret_cast<int *>(stages);   // query rows to be merged here: tile * 16 + row of the tile
    static_assert(kUnMaxTiles * kUnTile * 4 <= kUnWarps * L::kStages * L::kStage, "over the stages, which nothing is copied into any more");
    // ---- which rows are complete with this CTA's parts ----
    auto ctas = [&](int u0, int nu) { return aw_s.of(warp_of(u0 + nu - 1)) - aw_s.of(warp_of(u0)) + 1; };   // that have units of a tile
    for (int j = tid; j < n_tile * (SHARED ? kUnTile : 1); j += kUnWarps * 32) {
      const int4 d = tile_s[SHARED ? j / kUnTile : j];
      const int u0 = d.x & 0x7FFFFFFF, h = d.w & 0xffff, n = d.w >> 16;
      int want = ctas(u0, d.y), i0 = 0, cnt = n;
      unsigned *tk = a.tickets + warp_of(u0);   // a tile that reaches another CTA is the last one of its first range
      bool there = true;
      if constexpr (SHARED) {                   // a ticket for each row and group: its prefix tile's CTAs and its own
        const int li = j & (kUnTile - 1), r = d.z + li;
        there = li * a.G < n;
        if (there) {
          i0 = li * a.G; cnt = a.G;
          const int nu = first[r + 1] - first[r];
          if (d.x < 0) { if (tiles_head > 0) want += ctas((h * tiles_head + a.by_rpt.of(r)) * prefix_nu, prefix_nu); }
          else if (nu > 0) want += ctas(U_prefix + first[r] * a.Hkv + h * nu, nu);
          tk = a.tickets + (size_t)r * a.Hkv + h;
        }
      }
      if (there) {
        bool ready = want == 1;
        if (!ready && atomicAdd(tk, 1u) + 1u == (unsigned)want) { ready = true; *tk = 0u; }
        if (ready) {
          const int at = atomicAdd(&n_item_s, cnt);
          for (int i = 0; i < cnt; ++i) item_s[at + i] = (SHARED ? j / kUnTile : j) * kUnTile + i0 + i;
        }
      }
    }
    __threadfence();
    __syncthreads();
    // ---- and those are merged ----
    const int n_item = n_item_s;
    const bool sound = n_item == 0 || __ldcg(a.err) == 0;
    auto merge = [&](auto pg_c, int item) {
      constexpr int PG = decltype(pg_c)::value;
      const bool real = item < n_item;
      const int x = real ? item_s[item] : item_s[0], i = x & (kUnTile - 1);
      const int4 d = tile_s[x / kUnTile];
      const int h = d.w & 0xffff, li = a.by_G.of(i), r = d.z + li, gi = i - li * a.G;
      uint16_t *dst = a.out + ((size_t)r * a.H + h * a.G + gi) * kHeadDim;
      if constexpr (SHARED) {
        const RowParts p = row_parts(a, r, h, gi, size, first[r], first[r + 1]);
        merge_parts<PG, F16>(p.p_n + p.o_n, [&](int k) { return p.at(a, k); }, dst, real, sound);
      } else {
        const int f = warp_of(d.x);
        merge_parts<PG, F16>(warp_of(d.x + d.y - 1) - f + 1, [&](int k) { return a.part + (seq_part(f + k, k == 0) + i) * kUnPitch; }, dst, real, sound);
      }
    };
    // (a warp a row or a quarter of one: by the call, not by how many rows this CTA came last at, since the
    // two add the parts in other orders)
    if (SHARED || a.few_rows) for (int it = warp; it < n_item; it += kUnWarps) merge(IntC<4>(), it);
    else for (int it = warp * 4; it < n_item; it += kUnWarps * 4) merge(IntC<1>(), it + ((lane >> 3) & 3));
  }
}

constexpr int kMergeWarps = 8;
// a warp per query row and head
__global__ void __launch_bounds__(kMergeWarps * 32) merge_shared_kernel(const UnitArgs a) {
  pdl_wait();
  const int item = blockIdx.x * kMergeWarps + (threadIdx.x >> 5);
  if (item >= a.q_rows * a.H) return;          // whole warps
  const int r = a.by_H.of(item), h = item - r * a.H, kvh = a.by_G.of(h);
  const int4 size4 = __ldcg(reinterpret_cast<const int4 *>(a.plan));   // the Div, and the first sum
  const int f0 = __ldcg(a.plan + 3 + r), f1 = __ldcg(a.plan + 4 + r);
  const Div size = {(uint32_t)size4.x, (uint32_t)size4.y, (uint32_t)size4.z};
  const RowParts x = row_parts(a, r, kvh, h - kvh * a.G, size, f0, f1);
  if (x.p_n == 0 && x.o_n == 1) return;        // finished by its warp, as NaN where that gave up
  merge_parts<4, false>(x.p_n + x.o_n, [&](int p) { return x.at(a, p); }, a.out + ((size_t)r * a.H + h) * kHeadDim, true, __ldcg(a.err) == 0);
}

// partial rows of the shared form: prefix tiles (their number + ranges places of 16), then the rows' own (rows x heads + ranges
// places of G)
inline long long shared_prefix_part_rows(int R, int Hkv, int G) {
  const int rpt = kUnTile / G;
  return ((long long)Hkv * ((R + rpt - 1) / rpt) + kUnMaxWarps) * kUnTile;
}
inline long long shared_part_rows(int R, int Hkv, int G) { return shared_prefix_part_rows(R, Hkv, G) + ((long long)R * Hkv + kUnMaxWarps) * G; }
inline long long cross_part_rows() { return 2ll * kUnMaxWarps * kUnTile; }

template <bool SHARED, int KV, bool QF32>
inline cudaError_t launch_units_as(const CUtensorMap &k_map, const CUtensorMap &v_map, const UnitArgs &a, int n_sm, cudaStream_t st) {
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(attention_units_kernel<SHARED, KV, QF32>, units_smem_bytes<KV>(kUnMaxSeq))) return e;
  const int grid = std::min(n_sm, kUnMaxCtas);
  if (const cudaError_t e = launch_kernel(attention_units_kernel<SHARED, KV, QF32>, dim3(grid), dim3(kUnWarps * 32),
                                          units_smem_bytes<KV>(SHARED ? a.q_rows : a.n_seq), st, false, k_map, v_map, a)) return e;
  if (a.tickets) return cudaSuccess;
  return launch_kernel(merge_shared_kernel, dim3((a.q_rows * a.H + kMergeWarps - 1) / kMergeWarps), dim3(kMergeWarps * 32), 0, st, true, a);
}

// The maps of K and V: 16 keys of one head a copy, with the 128-byte swizzle.  A pool of 16-bit pages: [64, 64 tokens, blocks].
inline cudaError_t units_pool_map(CUtensorMap *map, const void *pool, size_t blocks) {
  const cuuint64_t dims[3] = {kHeadDim, kPageTokens, blocks}, strides[2] = {kHeadDim * 2, kPageElems * 2};
  const cuuint32_t box[3] = {kHeadDim, kUnBox, 1};
  return tensor_map_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, pool, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}
// Rows of 64 values [64, tokens, heads], tokens and heads `row` and `head` bytes apart; `box_rows` tokens of one head a copy.  The order
// of the two outer dimensions makes no difference in time.
inline cudaError_t units_rows_map(CUtensorMap *map, bool f16, const void *base, size_t heads, size_t rows, size_t head, size_t row, int box_rows) {
  const cuuint64_t dims[3] = {kHeadDim, rows, heads}, strides[2] = {row, head};
  const cuuint32_t box[3] = {kHeadDim, (cuuint32_t)box_rows, 1};
  return tensor_map_encode(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, base, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

}  // namespace ttsgpt
