// Attention of trees of drafted tokens over a paged cache, on the 5th-generation tensor cores (Section I: the decode engine's attention
// kernels, here for several tokens of a stream at once).
//
// Row r of tree i is a node.  It attends to all committed keys of its stream and to those of the stream's last T_i keys whose bits its
// mask has:  o = sum_j p_j v_j,  p_j = 2^(s_j - m) / sum 2^(s_j - m),  s_j = scale log2(e) q.k_j.  A row that sees no key is zero.
//
// Tile.  Rows of one tree times the G query heads of a head of keys, at most 128 / S of them, over blocks of 128 keys (two pages):
//     S = Q K^T     tcgen05.mma M=128 x N=128 x K=64, fp32 in tensor memory (fp32 queries as two bf16 parts, 16 bits)
//     softmax       a thread a lane of tensor memory: reference m and sum l in fp32, P rounded to bf16 back into tensor memory; the
//                   reference moves, and O with it, only where a score exceeds it by more than 8 (log2)
//     O += P V      M=128 x N=64 x K=128, V as stored
// Where a tile has at most 64 or 32 rows, they stand S = 2 or 4 times among the 128 lanes, and each copy's threads take only their half or
// quarter of a block's keys (their P is zero elsewhere): the exponentials, which would otherwise be one warp's, are spread over all four,
// and a row's S sums meet in shared memory at the end of the tile.
//
// K and V come page by page: bf16 by copies of 64 rows with the 128-byte swizzle, K a block ahead of V since it is needed a block earlier; of
// the 8-bit cache four more warps load codes, widen them to bf16 (exact) and store them as the tensor cores want them; K's scales multiply
// the scores and V's the weights.  Two CTAs an SM (one where 8-bit keys meet tiles of 128 rows), each with two blocks of K and of V.
//
// Work split.  Tiles are laid end to end by what they cost and cut into equal ranges, one a CTA, wherever the cut falls; parts of a tile that
// several CTAs share go to scratch with a ticket, and the CTA that comes last adds them in the order of their keys, so that results do not
// depend on timing.  Every wait is bounded.
#pragma once
#include "attention_common.cuh"
#include "draft_trees.cuh"
#include "tensor_map.cuh"

namespace ttsgpt {

constexpr int kTrKeys = 128;                // keys of a block
constexpr int kTrHalf = kTrKeys * 128;      // K or V of a block as bf16: 16 KB
constexpr int kTrQ = 2 * kTrHalf;           // Q of a tile, both parts; and where a row's copies meet
constexpr int kTrMaxSeq = 2048;
constexpr int kTrMaxCtas = 320;
constexpr int kTrPitch = 68;                // floats of a row's part
constexpr float kTrSlack = 8.0f;            // log2 by which a score may exceed the reference
constexpr int kTrCostBlock = 2, kTrCostTile = 2;   // what a range is measured in: a block, a tile besides its blocks
constexpr int kTrParts = 4;                 // that the copying warp is ahead at most
// What the copying warps write beside a block has four places, though K and V have two: block c + 4's is written when Q K^T of block c + 2 is
// done, which was issued after the softmax had read block c + 1's.
constexpr int kTrBeside = 4;
constexpr unsigned long long kTrWaitNs = 2000000000ull;

struct TreeAttnArgs {
  const void *q;
  uint16_t *out;                // [R][H * 64]
  long long q_stride;           // elements between rows
  int R, H, Hkv, G, rpt;        // G query heads a head of keys; tree rows of a tile
  Div by_G, by_rpt;
  float scale;                  // of the scores, in log2 units
  const int *row_start, *stream_ids, *kv_len, *page_table, *mask;
  int n_seq, t_max, words, max_streams, pps, n_pages;
  const unsigned char *pool;
  int *err;                     // [0]: set when a wait ran out; rows that are then not computed become NaN
  unsigned long long wait_ns;
  int starve;                   // test aid: the CTA whose copies never count as complete; -1: none
  unsigned *tickets;            // zero between calls
  float *part;
};

// The part of a tile that lies in a CTA's range.
struct TreePart {
  int row0, n_i, kvh, u0, nu;   // first row, rows times heads, head of keys; where the tile's cost begins, its cost
  int j0, j1, keys, committed, nodes, stream;   // its blocks here; keys of the stream, of them committed, nodes of the tree
};

struct TreeShared {
  TreePart part[kTrParts];
  uint64_t part_full[kTrParts], part_free[kTrParts];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t q_full, s_full, p_full, pv_done, meet;   // meet: the softmax warps among themselves, bounded like every wait
  uint32_t tmem;
  int failed;                   // 1: a wait of the CTA has run out; 2: one of an earlier call with the same scratch had
  int pages_ok[kTrBeside];      // of a block: bit p, its page p is there
  int found;                    // number (from 1 on) of the last block with a drafted key whose V is not finite
  unsigned bad[4];              // those keys
  float2 ml[4][32];
  TreePart meets;               // the tile that began before the CTA's range
  Div size;
  int warp_tot[16];
};

template <int S, bool E4M3> struct TreeShape {
  // warps 0-3: softmax, from 4 on: copies, behind them one for the products; the others of its group only give up their registers
  static constexpr int kCopyWarps = E4M3 ? 4 : 1, kThreads = E4M3 ? 384 : 256, kMmaWarp = 4 + kCopyWarps;
  static constexpr int kCtas = E4M3 && S == 1 ? 1 : 2;   // an SM
  // Registers of a thread, which the groups of four warps split anew: 128, 80 or 168 at launch times the groups is at least their sum.
  static constexpr int kRegsSoftmax = !E4M3 || S == 1 ? 216 : 128, kRegsCopy = !E4M3 ? 40 : S == 1 ? 128 : 88, kRegsMma = !E4M3 ? 40 : S == 1 ? 40 : 24;
  static constexpr int kScales = E4M3 ? kTrBeside * 2 * kTrKeys * 4 : 0;
};
template <int S, bool E4M3> inline size_t tree_smem_bytes(int n) {
  return 1024 + 4 * (size_t)kTrHalf + kTrQ + TreeShape<S, E4M3>::kScales + sizeof(TreeShared) + (size_t)(n + 1) * sizeof(int);
}

// 32 lanes x 16 columns of 32 bits into tensor memory, waited for later
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
               "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]) : "memory");
}

template <int S, bool E4M3, bool QF32>
__global__ void __launch_bounds__(TreeShape<S, E4M3>::kThreads, TreeShape<S, E4M3>::kCtas) attention_tree_kernel(const __grid_constant__ CUtensorMap kv_map,
                                                                                                                const TreeAttnArgs a) {
  using Shape = TreeShape<S, E4M3>;
  constexpr int kCols = kTrKeys / S, kDims = kHeadDim / S, kChunk = kDims < 32 ? kDims : 32;   // a thread's keys of a block, and its values of a finished row, some at a time
  extern __shared__ __align__(16) unsigned char tr_smem_raw[];
  unsigned char *base = tr_smem_raw + ((1024u - (smem_u32(tr_smem_raw) & 1023u)) & 1023u);
  unsigned char *Ks = base, *Vs = base + 2 * kTrHalf, *Qs = base + 4 * kTrHalf;   // [2] 128 keys x 64, 128 rows x 64 [2 parts]: 128-byte swizzle
  float *scales = reinterpret_cast<float *>(Qs + kTrQ);                           // 8-bit cache: [kTrBeside][K, V][128]
  TreeShared &sh = *reinterpret_cast<TreeShared *>(Qs + kTrQ + Shape::kScales);
  int *first = reinterpret_cast<int *>(&sh + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sh.failed;

  if (tid == 0) {
    const int full = (E4M3 ? Shape::kCopyWarps : 1) + ((int)blockIdx.x == a.starve ? 1 : 0);
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.k_full[i], full); mbar_init(&sh.v_full[i], full); mbar_init(&sh.k_empty[i], 1); mbar_init(&sh.v_empty[i], 1); }
    for (int i = 0; i < kTrParts; ++i) { mbar_init(&sh.part_full[i], 1); mbar_init(&sh.part_free[i], 4 + Shape::kCopyWarps); }
    mbar_init(&sh.q_full, 4); mbar_init(&sh.s_full, 1); mbar_init(&sh.p_full, 4); mbar_init(&sh.pv_done, 1); mbar_init(&sh.meet, 4);
    sh.found = 0;
    sh.failed = __ldcg(a.err) ? 2 : 0;
  }
  if (!E4M3 && warp == 4 && lane == 0) asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map) : "memory");
  if (warp == Shape::kMmaWarp) tmem_alloc(&sh.tmem, 256);   // S 128 columns, P 64, O 64
  // ---- running sums of cost over the trees ----
  struct Tree { int row0, rows, nodes, keys, committed, stream; };
  auto tree_of = [&](int i) {
    Tree x = {0, 0, 0, 0, 0, -1};
    if (!tree_rows(a.row_start, i, a.R, x.row0, x.nodes)) { x.rows = -1; return x; }
    x.rows = min(x.nodes, a.t_max);
    const int s = a.stream_ids ? a.stream_ids[i] : i;
    if (s >= 0 && s < a.max_streams) {         // a stream that is none has no keys
      const int len = a.kv_len[s];
      x.stream = s;
      x.keys = min(max(len, 0), a.pps * kPageTokens);
      x.committed = len - x.nodes;
    }
    return x;
  };
  auto tile_cost = [&](const Tree &x) { return kTrCostTile + kTrCostBlock * ((x.keys + kTrKeys - 1) / kTrKeys); };
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose rows nothing bounds
  for (int i0 = 0; i0 < a.n_seq; i0 += Shape::kThreads) {
    const int i = i0 + tid;
    int u = 0;
    if (i < a.n_seq) {
      const Tree x = tree_of(i);
      bad |= x.rows < 0;
      u = x.rows > 0 ? a.Hkv * a.by_rpt.of(x.rows + a.rpt - 1) * tile_cost(x) : 0;
    }
    int incl = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) sh.warp_tot[warp] = incl;
    bad = __syncthreads_or(bad);
    int before = carry, all = carry;
#pragma unroll
    for (int w = 0; w < Shape::kThreads / 32; ++w) { if (w < warp) before += sh.warp_tot[w]; all += sh.warp_tot[w]; }
    if (i < a.n_seq) first[i] = before + incl - u;
    carry = all;
  }
  const int T = bad ? 0 : carry;
  if (tid == 0) {
    first[a.n_seq] = T;
    sh.size.set(max(kTrCostBlock, (T + (int)gridDim.x - 1) / (int)gridDim.x));
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const Div size = sh.size;
  const int u_begin = blockIdx.x * (int)size.d, u_end = *failed ? u_begin : min(T, u_begin + (int)size.d);

  auto part_at = [&](int u) {                  // from unit u on
    TreePart p;
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (first[m] <= u) lo = m; else hi = m - 1; }
    const Tree x = tree_of(lo);
    const int tiles = a.by_rpt.of(x.rows + a.rpt - 1), blocks = (x.keys + kTrKeys - 1) / kTrKeys;
    p.nu = tile_cost(x);
    const int k = (int)((unsigned)(u - first[lo]) / (unsigned)p.nu);
    p.kvh = (int)((unsigned)k / (unsigned)tiles);
    p.u0 = first[lo] + k * p.nu;
    const int tile = k - p.kvh * tiles;
    p.row0 = x.row0 + tile * a.rpt;
    p.n_i = min(a.rpt, x.rows - tile * a.rpt) * a.G;
    p.keys = x.keys; p.committed = x.committed; p.nodes = x.nodes; p.stream = x.stream;
    auto blocks_before = [&](int y) { return min((max(y - p.u0 - kTrCostTile, 0) + kTrCostBlock - 1) / kTrCostBlock, blocks); };   // that begin before y
    p.j0 = blocks_before(u);
    p.j1 = blocks_before(u_end);
    return p;
  };
  auto wait = [&](uint64_t *bar, uint32_t parity) {   // the whole warp; false: some wait of the CTA has run out
    if (mbar_try_wait(bar, parity)) return true;
    unsigned long long t0 = 0;
#pragma unroll 1
    for (int polls = 1; !mbar_try_wait(bar, parity); ++polls) {
      if (polls & 15) continue;                // the timer is read only where the wait is long
      if (*failed) return false;
      const unsigned long long t1 = global_timer_ns();
      if (t0 == 0) t0 = t1;
      if (t1 - t0 > a.wait_ns) { *failed = 1; atomicExch(a.err, 1); return false; }
    }
    return true;
  };
  auto wait_warp = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)) != 0; };
  // part number n as the first copying warp has described it; who reads it gives its place back when the copy here is made
  auto take_part = [&](int n, TreePart &p) {
    const int k = n % kTrParts;
    if (!wait_warp(&sh.part_full[k], (uint32_t)(n / kTrParts) & 1u)) return false;
    p = sh.part[k];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_free[k]);
    return true;
  };
  auto give_part = [&](int n, const TreePart &p) {
    const int k = n % kTrParts;
    if (n >= kTrParts && !wait_warp(&sh.part_free[k], (uint32_t)(n / kTrParts - 1) & 1u)) return false;
    if (lane == 0) { sh.part[k] = p; mbar_arrive(&sh.part_full[k]); }
    __syncwarp();
    return true;
  };
  // page number pg of a stream's list, or -1: it has no keys, or is none
  auto page_of = [&](const TreePart &p, int pg) {
    if (pg * kPageTokens >= p.keys) return -1;
    const int phys = a.page_table[(size_t)p.stream * a.pps + pg];
    return phys >= 0 && phys < a.n_pages ? phys : -1;
  };

  auto products = [&]() {
    // ---- products.  Turn k comes when the softmax has block k's scores in registers and block k - 1's weights in tensor memory: P V of block
    //      k - 1 and Q K^T of block k + 1 are issued ----
    const uint32_t idesc_qk = tc_instr_desc(128, kTrKeys), idesc_pv = tc_instr_desc(128, kHeadDim) | (1u << 16);   // V is MN-major
    const uint64_t dq = tc_smem_desc(Qs), dks = tc_smem_desc(Ks), dvs = tc_smem_desc(Vs);
    int n_tile = 0, n_part = 0, n_block = 0, turns = 0;
    bool fine = true;
    for (int u = u_begin; u < u_end && fine;) {
      TreePart p;
      fine = take_part(n_part++, p);
      if (!fine) break;
      u = p.u0 + p.nu;
      const int nb = p.j1 - p.j0;
      if (nb <= 0) continue;
      fine = wait_warp(&sh.q_full, (uint32_t)n_tile++ & 1u);
#pragma unroll 1
      for (int k = -1; k <= nb && fine; ++k) {
        const int ck = n_block + k + 1, cv = n_block + k - 1;
        if (k + 1 < nb) fine = wait_warp(&sh.k_full[ck & 1], (uint32_t)(ck / 2) & 1u);
        if (fine && k >= 0) fine = wait_warp(&sh.p_full, (uint32_t)turns++ & 1u);
        if (fine && k >= 1) fine = wait_warp(&sh.v_full[cv & 1], (uint32_t)(cv / 2) & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        if (elect_one()) {
          if (k >= 1) {
            const uint64_t dv = dvs + (uint64_t)(cv & 1) * (kTrHalf >> 4);
#pragma unroll
            for (int q = 0; q < kTrKeys / 16; ++q)   // 16 keys an instruction: 8 columns of P, two groups of 8 rows of V
              tc_mma_ts(tmem + 192u, tmem + 128u + 8u * q, dv + 128 * q, idesc_pv, k == 1 && q == 0 ? 0u : 1u);
            tc_commit(&sh.v_empty[cv & 1]);
          }
          if (k + 1 < nb) {
            const uint64_t dk = dks + (uint64_t)(ck & 1) * (kTrHalf >> 4);
#pragma unroll
            for (int q = 0; q < 4; ++q) tc_mma(tmem, dq + 2 * q, dk + 2 * q, idesc_qk, q == 0 ? 0u : 1u);
            if constexpr (QF32) {
#pragma unroll
              for (int q = 0; q < 4; ++q) tc_mma(tmem, dq + (kTrHalf >> 4) + 2 * q, dk + 2 * q, idesc_qk, 1u);
            }
            tc_commit(&sh.k_empty[ck & 1]);
          }
          tc_commit(k < nb ? &sh.s_full : &sh.pv_done);
        }
        __syncwarp();
      }
      n_block += nb;
    }
  };

  if (E4M3 && warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsMma));
    if (warp == Shape::kMmaWarp) products();
  } else if (warp >= 4) {
    if constexpr (E4M3 && S > 1) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kRegsCopy));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsCopy));
    if (!E4M3 && warp == Shape::kMmaWarp) products();
    if constexpr (!E4M3) if (warp == 4) {
      // ---- copies: K of a block, then V of the one before ----
      int c = 0, n_part = 0, v0 = -1, v1 = -1, v_kvh = 0;   // blocks of this CTA, its parts; pages and head of the block whose V is due
      bool fine = true;
      auto copy = [&](unsigned char *dst, uint64_t *bar, int p0, int p1, int head) {   // head: of K, or n_kv_head further for V
        if (elect_one()) {
          mbar_expect_tx(bar, (uint32_t)((p0 >= 0) + (p1 >= 0)) * (kTrHalf / 2));
          if (p0 >= 0) un_box(&kv_map, 0, p0 * 2 * a.Hkv + head, dst, bar);
          if (p1 >= 0) un_box(&kv_map, 0, p1 * 2 * a.Hkv + head, dst + kTrHalf / 2, bar);
        }
        __syncwarp();
      };
      auto copy_v = [&](int b) {               // of block number b of this CTA
        if (b >= 2 && !wait_warp(&sh.v_empty[b & 1], (uint32_t)(b / 2 - 1) & 1u)) return false;
        copy(Vs + (b & 1) * kTrHalf, &sh.v_full[b & 1], v0, v1, v_kvh + a.Hkv);
        return true;
      };
      for (int u = u_begin; u < u_end && fine;) {
        const TreePart p = part_at(u);
        fine = give_part(n_part++, p);
        u = p.u0 + p.nu;
        int mine = -1;                         // a page of sixteen blocks each lane
#pragma unroll 1
        for (int j = p.j0; j < p.j1 && fine; ++j, ++c) {
          const int at = (j - p.j0) & 15;
          if (at == 0) mine = page_of(p, 2 * j + lane);
          const int p0 = __shfl_sync(0xFFFFFFFFu, mine, 2 * at), p1 = __shfl_sync(0xFFFFFFFFu, mine, 2 * at + 1);
          if (c >= 2) fine = wait_warp(&sh.k_empty[c & 1], (uint32_t)(c / 2 - 1) & 1u);
          if (!fine) break;
          if (lane == 0) sh.pages_ok[c % kTrBeside] = (p0 >= 0) + 2 * (p1 >= 0);
          __syncwarp();
          copy(Ks + (c & 1) * kTrHalf, &sh.k_full[c & 1], p0, p1, p.kvh);
          if (j > p.j0) fine = copy_v(c - 1);
          v0 = p0; v1 = p1; v_kvh = p.kvh;
        }
        // (the part's last V before the next part is described: that may wait until the softmax is done with this one)
        if (fine && p.j1 > p.j0) fine = copy_v(c - 1);
      }
    }
    if constexpr (E4M3) {
      // ---- codes out of memory, a block ahead of where they are widened: thread t takes 16 codes of rows t/4, t/4 + 32, .. of K and of V ----
      const int t = tid - 128, quad = t & 3, r0 = t >> 2;
      int n_part = 0, u = u_begin, j = 0;
      bool fine = true;
      TreePart p;
      p.j1 = 0;
      uint4 code[2][2][4];                     // [this block, the next][K, V][rows]
      float sc[2][2];                          // scales of key t: K, V
      int ok[2] = {0, 0};
      int mine = -1, j_mine = 0;               // pages of sixteen blocks, one a lane, and the first of those blocks
      // The next block's codes into registers.  A part behind the fourth is asked for only when this block has been handed over (`late`):
      // its place may be free no sooner than that.
      enum { kNone = 0, kLoaded = 1, kLater = 2 };
      auto load = [&](uint4 (&x)[2][4], float (&s)[2], int &pages, bool late) -> int {
        while (j >= p.j1) {                    // the next part that has blocks here
          if (u >= u_end) return kNone;
          if (n_part >= kTrParts && !late) return kLater;
          if (warp == 4) { p = part_at(u); fine = give_part(n_part++, p); }
          else fine = take_part(n_part++, p);
          if (!fine) return kNone;
          u = p.u0 + p.nu;
          j = p.j0;
          j_mine = j - 16;
        }
        if (j - j_mine >= 16) { j_mine = j; mine = page_of(p, 2 * j + lane); }
        const int n = p.keys - j * kTrKeys;    // keys from here on
        const int p0 = __shfl_sync(0xFFFFFFFFu, mine, 2 * (j - j_mine)), p1 = __shfl_sync(0xFFFFFFFFu, mine, 2 * (j - j_mine) + 1);
        pages = (p0 >= 0) + 2 * (p1 >= 0);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int r = r0 + 32 * i, pg = i < 2 ? p0 : p1;
            const unsigned char *blk = a.pool + ((size_t)pg * 2 * a.Hkv + p.kvh + w * a.Hkv) * kE4m3BlockBytes;
            x[w][i] = pg >= 0 && r < n ? ld_stream_u4(blk + (r & 63) * kHeadDim + 16 * quad) : make_uint4(0, 0, 0, 0);
          }
          const int pg = t < 64 ? p0 : p1;
          s[w] = pg >= 0 && t < n ? *reinterpret_cast<const float *>(a.pool + ((size_t)pg * 2 * a.Hkv + p.kvh + w * a.Hkv) * kE4m3BlockBytes + kPageTokens * kHeadDim + 4 * (t & 63)) : 0.f;
        }
        ++j;
        return kLoaded;
      };
      auto widen = [&](unsigned char *dst, const uint4 (&x)[4]) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int r = r0 + 32 * i;
          const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
          uint32_t y[8];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            y[2 * k] = e4m3x2_to_bf16x2(__byte_perm(w[k], 0u, 0x1404));
            y[2 * k + 1] = e4m3x2_to_bf16x2(__byte_perm(w[k], 0u, 0x3424));
          }
          *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad) ^ (r & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
          *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad + 1) ^ (r & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
        }
      };
      int c = 0;
      // hands this block over, the next one's codes on their way meanwhile; false: there is no next one
      auto step = [&](uint4 (&x)[2][4], float (&s)[2], int pages, uint4 (&nx)[2][4], float (&ns)[2], int &npages) -> bool {
        int got = load(nx, ns, npages, false);
        if (!fine) return false;
        const uint32_t parity = (uint32_t)(c / 2 - 1) & 1u;
        const int b = c & 1;
        if (c >= 2 && !wait_warp(&sh.k_empty[b], parity)) return false;
        if (t == 0) sh.pages_ok[c % kTrBeside] = pages;
        scales[(2 * (c % kTrBeside)) * kTrKeys + t] = s[0];
        scales[(2 * (c % kTrBeside) + 1) * kTrKeys + t] = s[1];
        widen(Ks + b * kTrHalf, x[0]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.k_full[b]);
        if (c >= 2 && !wait_warp(&sh.v_empty[b], parity)) return false;
        widen(Vs + b * kTrHalf, x[1]);
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.v_full[b]);
        ++c;
        if (got == kLater) got = load(nx, ns, npages, true);
        return got == kLoaded;
      };
      if (load(code[0], sc[0], ok[0], true) == kLoaded) {
#pragma unroll 1
        while (step(code[0], sc[0], ok[0], code[1], sc[1], ok[1]) && step(code[1], sc[1], ok[1], code[0], sc[0], ok[0])) {}
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kRegsSoftmax));
    // ---- softmax ----
    const int rg = warp % (4 / S), rep = warp / (4 / S);     // which 32 rows of the tile, and which copy of them
    const int i_row = 32 * rg + lane, col0 = rep * kCols;    // the thread's row, and its first key of a block
    const uint32_t t_lane = tmem + ((uint32_t)(32 * warp) << 16);
    int n_s = 0, n_o = 0, n_meet = 0, n_block = 0, n_part = 0;   // waits for s_full, pv_done and meet, blocks of the CTA, parts
    bool fine = true;
    int came_first = 0;                        // how many had a ticket of the tile that began before the CTA's range, this CTA among them
    if (S > 1) {                               // weights of the other copies' keys: zero throughout
      float z[32];
#pragma unroll
      for (int e = 0; e < 32; ++e) z[e] = 0.f;
      tmem_st32(t_lane + 128u, z);
      tmem_st32(t_lane + 160u, z);
    }
    auto meet = [&]() {                        // the four warps; shared memory that one has written the others see
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.meet);
      return wait_warp(&sh.meet, (uint32_t)n_meet++ & 1u);
    };
    // A tile that several CTAs share has a place in each: by warp, columns of four values of its 32 rows, then reference and sum.  A CTA has
    // two places: for the tile that began before its range, and the one that goes on behind it.
    auto place = [&](int c, int c0) { return a.part + (size_t)(2 * c + (c == c0)) * 128 * kTrPitch; };
    // chunk h of those of CTAs c .. c1, in the order of their keys, onto o, m, l; the sum of weights
    auto add_parts = [&](int c0, int c, int c1, int h, float (&o)[kChunk], float m, float l) {
#pragma unroll 1
      for (; c <= c1; ++c) {
        const float *x = place(c, c0);
        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(x + 128 * kHeadDim + 64 * warp + 2 * lane));
        float4 v[kChunk / 4];
#pragma unroll
        for (int e = 0; e < kChunk / 4; ++e) v[e] = __ldcg(reinterpret_cast<const float4 *>(x + warp * 32 * kDims + ((h * (kChunk / 4) + e) * 32 + lane) * 4));
        const bool has = ml.y != 0.f;          // a key in it
        const float mn = fmaxf(m, ml.x), fk = !has || m == mn ? 1.f : pt_exp2(m - mn), fn = has ? pt_exp2(ml.x - mn) : 0.f;
        if (has) m = mn;
        l = fmaf(l, fk, ml.y * fn);
#pragma unroll
        for (int e = 0; e < kChunk / 4; ++e) {
          o[4 * e] = fmaf(o[4 * e], fk, v[e].x * fn); o[4 * e + 1] = fmaf(o[4 * e + 1], fk, v[e].y * fn);
          o[4 * e + 2] = fmaf(o[4 * e + 2], fk, v[e].z * fn); o[4 * e + 3] = fmaf(o[4 * e + 3], fk, v[e].w * fn);
        }
      }
      return l;
    };
    auto leave = [&](const TreePart &p, int h, const float (&o)[kChunk], float l) {   // chunk h of the thread's values of its row
      if (i_row >= p.n_i) return;
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const int r = a.by_G.of(i_row);
      uint16_t *dst = a.out + ((size_t)(p.row0 + r) * a.H + (p.kvh - r) * a.G + i_row) * kHeadDim + rep * kDims + h * kChunk;
#pragma unroll
      for (int c = 0; c < kChunk; c += 8)
        *reinterpret_cast<uint4 *>(dst + c) = make_uint4(pack_bf16x2(o[c] * inv, o[c + 1] * inv), pack_bf16x2(o[c + 2] * inv, o[c + 3] * inv),
                                                         pack_bf16x2(o[c + 4] * inv, o[c + 5] * inv), pack_bf16x2(o[c + 6] * inv, o[c + 7] * inv));
    };
    for (int u = u_begin; u < u_end && fine;) {
      const int place_p = n_part % kTrParts;
      fine = wait_warp(&sh.part_full[place_p], (uint32_t)(n_part / kTrParts) & 1u);
      if (!fine) break;
      ++n_part;
      const TreePart &p = sh.part[place_p];    // stays there until the tile's rows have left: its registers would be spilled
      u = p.u0 + p.nu;
      const int nb = p.j1 - p.j0;
      const bool mine = i_row < p.n_i, live = 32 * rg < p.n_i;   // the thread's row exists, some row of the warp does
      float m = -INFINITY, l = 0.f;
      auto pass_turn = [&]() {                 // to the products
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full);
      };
      if (nb > 0) {
        // ---- the row's queries, as often as it stands among the lanes ----
        const int r = a.by_G.of(i_row);
        const size_t at = mine ? (size_t)(p.row0 + r) * a.q_stride + (size_t)((p.kvh - r) * a.G + i_row) * kHeadDim : 0;
#pragma unroll
        for (int c = 0; c < 8; ++c) {
          const int to = tid * 128 + ((c ^ (tid & 7)) << 4);
          if constexpr (QF32) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = 0.f;
            if (mine) load8(reinterpret_cast<const float *>(a.q) + at + 8 * c, x);
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float h0 = __uint_as_float(__float_as_uint(x[2 * e]) & 0xFFFF0000u), h1 = __uint_as_float(__float_as_uint(x[2 * e + 1]) & 0xFFFF0000u);
              hi[e] = pack_bf16x2(h0, h1);
              lo[e] = pack_bf16x2(x[2 * e] - h0, x[2 * e + 1] - h1);
            }
            *reinterpret_cast<uint4 *>(Qs + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            *reinterpret_cast<uint4 *>(Qs + kTrHalf + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
          } else {
            *reinterpret_cast<uint4 *>(Qs + to) = mine ? *reinterpret_cast<const uint4 *>(reinterpret_cast<const uint16_t *>(a.q) + at + 8 * c) : make_uint4(0, 0, 0, 0);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full);
        fine = wait_warp(&sh.s_full, (uint32_t)n_s++ & 1u);
        if (!fine) break;
        tc_fence_after_sync();
#pragma unroll 1
        for (int b = 0; b < nb; ++b) {
          const int c = n_block + b, key0 = (p.j0 + b) * kTrKeys, n = min(kTrKeys, p.keys - key0);
          float s[kCols], sc = 1.f;
          if (live) {
#pragma unroll
            for (int e = 0; e < kCols; e += 32) tmem_ld32_async(t_lane + (uint32_t)(col0 + e), s + e);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < kCols; e += 32) tmem_landed32(s + e);
          }
          const int pages = *reinterpret_cast<volatile int *>(&sh.pages_ok[c % kTrBeside]);
          pass_turn();
          const float *ks = scales + (2 * (c % kTrBeside)) * kTrKeys + col0, *vs = ks + kTrKeys;   // 8-bit cache: of K and V
          if (E4M3 && live) {
#pragma unroll
            for (int e = 0; e < kCols; e += 4) {
              const float4 f = *reinterpret_cast<const float4 *>(ks + e);
              s[e] *= f.x; s[e + 1] *= f.y; s[e + 2] *= f.z; s[e + 3] *= f.w;
            }
          }
          const bool drafted = key0 + kTrKeys > p.committed, special = drafted || n < kTrKeys || pages != 3;
          auto visible = [&](int x) {          // bits of the thread's keys 32 x .. 32 x + 31 that its row sees
            const int *row_mask = a.mask + (size_t)(p.row0 + a.by_G.of(min(i_row, p.n_i - 1))) * a.words;
            auto word = [&](int w) { return w < a.words && 32 * w < p.nodes ? (unsigned)row_mask[w] & (p.nodes - 32 * w < 32 ? (1u << (p.nodes - 32 * w)) - 1u : ~0u) : 0u; };
            const int k0 = col0 + 32 * x, d = key0 + k0 - p.committed;   // number of the first of these keys among the drafted
            unsigned v = ~0u;
            if (d >= 0) v = __funnelshift_r(word(d >> 5), d & 31 ? word((d >> 5) + 1) : 0u, d & 31);
            else if (d > -32) v = (word(0) << -d) | ((1u << -d) - 1u);
            const int there = pages >> (k0 >> 6) & 1 ? n - k0 : 0;
            return there <= 0 ? 0u : there < 32 ? v & ((1u << there) - 1u) : v;
          };
          if (special && live) {
#pragma unroll
            for (int x = 0; x < kCols / 32; ++x) {
              const unsigned v = visible(x);
#pragma unroll
              for (int e = 0; e < 32; ++e) s[32 * x + e] = v >> e & 1u ? s[32 * x + e] : -INFINITY;
            }
          }
          if (live) {
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < kCols; e += 8) {
#pragma unroll
              for (int q = 0; q < 4; ++q) mx[q] = max3(mx[q], s[e + 2 * q], s[e + 2 * q + 1]);
            }
            const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale;
            if (m == -INFINITY) { sc = 0.f; m = top; }   // nothing seen yet; O, where there is one, is zero
            else if (top > m + kTrSlack) { sc = pt_exp2(m - top); m = top; }
            if (!mine) { sc = 1.f; m = 0.f; }            // a row that does not exist holds anything
            const float ref = m == -INFINITY ? 0.f : m;
            const unsigned long long scale2 = pack_f32x2(a.scale, a.scale), ref2 = pack_f32x2(-ref, -ref);
            unsigned long long sum2[4] = {0ull, 0ull, 0ull, 0ull};
#pragma unroll
            for (int e = 0; e < kCols; e += 2) {
              float x, y;
              const unsigned long long d2 = fma_f32x2(pack_f32x2(s[e], s[e + 1]), scale2, ref2);
              if (S == 1 && (e >> 1) % 4 == 3) {         // a quarter of the exponentials on the FMA pipes where a thread has a whole block's
                unpack_f32x2(poly_exp2(d2), x, y);
              } else {
                unpack_f32x2(d2, x, y);
                x = pt_exp2(x); y = pt_exp2(y);
              }
              sum2[(e >> 1) & 3] = add_f32x2(sum2[(e >> 1) & 3], pack_f32x2(x, y));
              if constexpr (E4M3) {                      // a key that is not seen may have any scale
                const float2 f = *reinterpret_cast<const float2 *>(vs + e);
                x = x == 0.f ? 0.f : x * f.x;
                y = y == 0.f ? 0.f : y * f.y;
              }
              s[e >> 1] = __uint_as_float(pack_bf16x2(x, y));
            }
            float s0, s1;
            unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), s0, s1);
            l = fmaf(l, sc, s0 + s1);
          }
          // P V of the block before, to which P and O belong, and the scores of the next block, both under way since its turn began
          fine = wait_warp(&sh.s_full, (uint32_t)n_s++ & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          if (live) {
            if (b > 0 && __any_sync(0xFFFFFFFFu, sc != 1.f)) {
#pragma unroll
              for (int d = 0; d < kHeadDim; d += 32) {
                float x[32];
                tmem_ld32(t_lane + 192u + (uint32_t)d, x);
#pragma unroll
                for (int e = 0; e < 32; ++e) x[e] *= sc;
                tmem_st32(t_lane + 192u + (uint32_t)d, x);
              }
            }
            if constexpr (kCols >= 64) {
#pragma unroll
              for (int e = 0; e < kCols / 2; e += 32) tmem_st32_async(t_lane + 128u + (uint32_t)(col0 / 2 + e), s + e);
            } else {
              tmem_st16_async(t_lane + 128u + (uint32_t)(col0 / 2), s);
            }
            tmem_wait_st();
          }
          if constexpr (!E4M3) {
            if (special) {
              // V rows without a key hold anything, and so may those of drafted tokens that no row sees (a tree padded to a size): 0 * NaN
              // must not reach O.  They become zero, and rows that do see one that is not finite NaN.
              if (!wait_warp(&sh.v_full[c & 1], (uint32_t)(c / 2) & 1u)) { fine = false; break; }
              unsigned char *v = Vs + (c & 1) * kTrHalf;
              unsigned found = 0;
#pragma unroll
              for (int x = 0; x < 8; ++x) {
                const int k = (tid >> 3) + 16 * x;
                uint4 *piece = reinterpret_cast<uint4 *>(v + k * 128 + (tid & 7) * 16);
                if (k >= n || !(pages >> (k >> 6) & 1)) *piece = make_uint4(0, 0, 0, 0);
                else if (key0 + k >= p.committed) {
                  const uint4 w = *piece;
                  auto odd = [](uint32_t y) { return (y & 0x7F80u) == 0x7F80u || (y & 0x7F800000u) == 0x7F800000u; };
                  if (odd(w.x) || odd(w.y) || odd(w.z) || odd(w.w)) { *piece = make_uint4(0, 0, 0, 0); found |= 1u << x; }
                }
              }
              fence_proxy_async_smem();
              if (drafted) {
                if (found) sh.found = c + 1;   // (whoever writes writes the same)
                fine = meet();
                if (fine && *reinterpret_cast<volatile int *>(&sh.found) == c + 1) {   // rare: which keys, and who sees them
                  if (tid < 4) sh.bad[tid] = 0u;
                  fine = meet();
#pragma unroll
                  for (int x = 0; x < 8; ++x)
                    if (found >> x & 1) { const int k = (tid >> 3) + 16 * x; atomicOr(&sh.bad[k >> 5], 1u << (k & 31)); }
                  fine = meet() && fine;
                  if (live) {
#pragma unroll
                    for (int x = 0; x < kCols / 32; ++x)
                      if (visible(x) & *reinterpret_cast<volatile unsigned *>(&sh.bad[col0 / 32 + x])) l = __int_as_float(0x7FFFFFFF);
                  }
                  fine = meet() && fine;       // before the next block's are written
                }
                if (!fine) break;
              }
            }
          }
        }
        if (!fine) break;
        n_block += nb;
        pass_turn();
      }
      // ---- the tile's sums ----
      float met[S > 1 ? kChunk : 1];           // where a row stands once, its sums stay in tensor memory
#pragma unroll
      for (int c = 0; c < (S > 1 ? kChunk : 1); ++c) met[c] = 0.f;
      if (nb > 0) {
        fine = wait_warp(&sh.pv_done, (uint32_t)n_o++ & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        if constexpr (S > 1) {                 // a row's copies meet where its queries were, which no product reads any more
          float4 *stage = reinterpret_cast<float4 *>(Qs) + warp * 32 * (kHeadDim / 4);
          if (live) {
#pragma unroll
            for (int d = 0; d < kHeadDim; d += 32) {
              float x[32];
              tmem_ld32(t_lane + 192u + (uint32_t)d, x);
#pragma unroll
              for (int e = 0; e < 32; e += 4) stage[((d + e) / 4) * 32 + lane] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
            }
            sh.ml[warp][lane] = make_float2(m, l);
          }
          tc_fence_before_sync();
          fine = meet();
          if (!fine) break;
          if (live) {
            float2 ml[S];
            float M = -INFINITY;
#pragma unroll
            for (int x = 0; x < S; ++x) {
              ml[x] = sh.ml[rg + x * (4 / S)][lane];
              if (ml[x].y != 0.f) M = fmaxf(M, ml[x].x);
            }
            m = M; l = 0.f;
#pragma unroll
            for (int x = 0; x < S; ++x) {
              if (ml[x].y == 0.f) continue;    // no key in it
              const float f = pt_exp2(ml[x].x - M);
              l = fmaf(ml[x].y, f, l);
              const float4 *from = reinterpret_cast<const float4 *>(Qs) + (rg + x * (4 / S)) * 32 * (kHeadDim / 4) + rep * (kDims / 4) * 32;
#pragma unroll
              for (int e = 0; e < kDims / 4; ++e) {
                const float4 v = from[e * 32 + lane];
                met[4 * e] = fmaf(v.x, f, met[4 * e]); met[4 * e + 1] = fmaf(v.y, f, met[4 * e + 1]);
                met[4 * e + 2] = fmaf(v.z, f, met[4 * e + 2]); met[4 * e + 3] = fmaf(v.w, f, met[4 * e + 3]);
              }
            }
          }
          fine = meet();                       // the next tile's queries are written here
          if (!fine) break;
        }
      }
      // ---- the tile's rows leave, or this part of them goes to scratch ----
      const int c0 = size.of(p.u0), c1 = size.of(p.u0 + p.nu - 1);
      const bool begins = c0 == (int)blockIdx.x;
      bool whole = c0 == c1;
      auto sums = [&](int h, float (&o)[kChunk]) {
        if constexpr (S > 1) {
#pragma unroll
          for (int c = 0; c < kChunk; ++c) o[c] = met[c];
        } else if (nb > 0 && live) {
          tmem_ld32(t_lane + 192u + 32u * h, o);
        } else {
#pragma unroll
          for (int c = 0; c < kChunk; ++c) o[c] = 0.f;
        }
      };
      if (!whole) {                            // a ticket for the warp's 32 rows
        float *x = place(blockIdx.x, c0);
#pragma unroll
        for (int h = 0; h < kDims / kChunk; ++h) {
          float o[kChunk];
          sums(h, o);
          if (mine) {
#pragma unroll
            for (int e = 0; e < kChunk / 4; ++e)
              *reinterpret_cast<float4 *>(x + warp * 32 * kDims + ((h * (kChunk / 4) + e) * 32 + lane) * 4) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
          }
        }
        if (mine) *reinterpret_cast<float2 *>(x + 128 * kHeadDim + 64 * warp + 2 * lane) = make_float2(m, l);
        __threadfence();
        __syncwarp();
        int came = 0;
        if (lane == 0) came = (int)atomicAdd(a.tickets + 4 * c0 + warp, 1u) + 1;
        if (begins) {                          // the CTA's last tile; as a rule the others have long had theirs
          whole = __shfl_sync(0xFFFFFFFFu, came, 0) == c1 - c0 + 1;
          if (whole) {
            if (lane == 0) a.tickets[4 * c0 + warp] = 0u;
            __threadfence();
          }
        } else {                               // the CTA's first: the answer is looked at when its range is done
          came_first = came;
          if (lane == 0) sh.meets = p;         // (every warp writes the same)
        }
      }
      if (whole) {
#pragma unroll
        for (int h = 0; h < kDims / kChunk; ++h) {
          float o[kChunk];
          sums(h, o);
          const float total = mine && c0 != c1 ? add_parts(c0, c0 + 1, c1, h, o, m, l) : l;
          leave(p, h, o, total);
        }
      }
      if (S == 1) tc_fence_before_sync();      // O may be overwritten once this thread's next P is announced
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.part_free[place_p]);
    }
    // ---- the tile that began before this CTA's range, where this CTA came to it last ----
    __syncwarp();
    if (fine && (came_first = __shfl_sync(0xFFFFFFFFu, came_first, 0)) > 0) {
      const TreePart p = sh.meets;
      const int c0 = size.of(p.u0), c1 = size.of(p.u0 + p.nu - 1);
      if (came_first == c1 - c0 + 1) {
        if (lane == 0) a.tickets[4 * c0 + warp] = 0u;
        __threadfence();
#pragma unroll
        for (int h = 0; h < kDims / kChunk; ++h) {
          float o[kChunk];
#pragma unroll
          for (int c = 0; c < kChunk; ++c) o[c] = 0.f;
          const float l = i_row < p.n_i ? add_parts(c0, c0, c1, h, o, -INFINITY, 0.f) : 0.f;
          leave(p, h, o, l);
        }
      }
    }
    // ---- behind a wait that ran out: NaN into all rows of the call, among which are those that are not computed (a warp that has found the
    //      error covers them alone: others may have left before; one of an earlier call is found by all) ----
    if (*failed && first[a.n_seq] > 0) {
      const int x0 = *failed == 2 ? tid : lane, step = *failed == 2 ? 128 : 32;
#pragma unroll 1
      for (int i = 0; i < a.n_seq; ++i) {
        const Tree x = tree_of(i);
        uint4 *rows = reinterpret_cast<uint4 *>(a.out) + (size_t)x.row0 * a.H * (kHeadDim / 8);
        const size_t n = (size_t)max(x.rows, 0) * a.H * (kHeadDim / 8);
#pragma unroll 1
        for (size_t k = x0; k < n; k += step) rows[k] = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);
      }
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (*failed == 1) {   // copies and products may still be in flight
    const unsigned long long t0 = global_timer_ns();
    while (global_timer_ns() - t0 <= 10000000ull) {}
  }
  if (warp == Shape::kMmaWarp) tmem_dealloc(tmem, 256);
}

inline long long tree_part_floats() { return 2ll * kTrMaxCtas * 128 * kTrPitch; }

// pages of a bf16 pool [64, 64 tokens, blocks], one block a copy
inline cudaError_t tree_pool_map(CUtensorMap *map, const void *pool, size_t blocks) {
  const cuuint64_t dims[3] = {kHeadDim, kPageTokens, blocks}, strides[2] = {kHeadDim * 2, kPageElems * 2};
  const cuuint32_t box[3] = {kHeadDim, kPageTokens, 1};
  return tensor_map_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, pool, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <int S, bool E4M3, bool QF32>
inline cudaError_t launch_tree_as(const CUtensorMap &map, TreeAttnArgs a, int n_sm, cudaStream_t st) {
  using Shape = TreeShape<S, E4M3>;
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(attention_tree_kernel<S, E4M3, QF32>, tree_smem_bytes<S, E4M3>(kTrMaxSeq))) return e;
  a.rpt = 128 / S / a.G;
  a.by_rpt.set((uint32_t)a.rpt);
  return launch_kernel(attention_tree_kernel<S, E4M3, QF32>, dim3((unsigned)min(Shape::kCtas * n_sm, kTrMaxCtas)), dim3(Shape::kThreads), tree_smem_bytes<S, E4M3>(a.n_seq), st, false,
                       map, a);
}
template <bool E4M3, bool QF32>
inline cudaError_t launch_tree(const CUtensorMap &map, const TreeAttnArgs &a, int n_sm, cudaStream_t st) {
  const long long rows = (long long)a.t_max * a.G;
  return rows <= 32 ? launch_tree_as<4, E4M3, QF32>(map, a, n_sm, st) : rows <= 64 ? launch_tree_as<2, E4M3, QF32>(map, a, n_sm, st) : launch_tree_as<1, E4M3, QF32>(map, a, n_sm, st);
}

}  // namespace ttsgpt
