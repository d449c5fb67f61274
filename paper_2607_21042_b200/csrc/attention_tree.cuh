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
#include <cstddef>

namespace ttsgpt {

constexpr int kTrKeys = 128;                // keys of a block
constexpr int kTrHalf = kTrKeys * 128;      // K or V of a block as bf16: 16 KB
constexpr int kTrQ = 2 * kTrHalf;           // Q of two tiles (fp32: both parts of one); where a row's copies meet, too
constexpr int kTrMaxSeq = 2048;
constexpr int kTrNear = 256;                // trees up to which a CTA keeps what it has read of them
constexpr int kTrMaxCtas = 320;
constexpr int kTrPitch = 68;                // floats of a row's part
constexpr float kTrSlack = 8.0f;            // log2 by which a score may exceed the reference
constexpr int kTrCostBlock = 2, kTrCostTile = 5;   // what a range is measured in: a block, a tile besides its blocks
// Parts that the first copying warp may describe ahead.  Every part has a block, and no copy is more than five blocks ahead of the softmax, so
// that it never waits for a place while the softmax waits for it.
constexpr int kTrParts = 8;
// What the copying warps write beside a block has four places, though K and V have two: block c + 4's is written when Q K^T of block c + 2 is
// done, which was issued when the softmax was done with block c + 1.
constexpr int kTrBeside = 4;
constexpr unsigned long long kTrWaitNs = 2000000000ull;

struct TreeAttnArgs {
  const void *q;
  uint16_t *out;                // [R][H * 64]
  long long q_stride;           // elements between rows
  int R, H, Hkv, G, rpt;        // G query heads a head of keys; tree rows of a tile
  int lg;                       // log2 of how often a row stands among the 128 lanes
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
  int row0, n_i, kvh, next;     // first row, rows times heads, head of keys; where the next tile's cost begins
  int j0, j1, keys, committed, nodes, stream;   // its blocks here; keys of the stream, of them committed, nodes of the tree
  int c0, c1;                   // first and last CTA that have blocks of the tile
};
constexpr int kTrPartWords = sizeof(TreePart) / 4;

struct alignas(16) TreeShared {
  TreePart part[kTrParts];
  TreePart mine[4], shared[2][4];   // the softmax warps' own copies: the part at hand; of tiles of several CTAs the one that began before the range, and the last
  uint64_t part_full[kTrParts], part_free[kTrParts];
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], raw_full[2], raw_empty[2];
  uint64_t q_full[2], q_free[2];
  uint64_t s_full, p_full, o_full, meet;    // meet: the softmax warps among themselves, bounded like every wait
  uint32_t tmem;
  int failed;                   // 1: a wait of the CTA has run out; 2: one of an earlier call with the same scratch had
  int pages_ok[kTrBeside];      // of a block: bit p, its page p is there
  int found;                    // number (from 1 on) of the last block with a drafted key whose V is not finite
  unsigned bad[4];              // those keys
  float2 ml[4][32];
  Div size;
  int warp_tot[16];
};

template <bool E4M3> struct TreeShape {
  // warps 0-3: softmax, 4: copies, 5: products, 8-bit cache 6 and 7: codes to bf16
  static constexpr int kCopyWarp = 4, kMmaWarp = 5, kWidenWarp = 6, kWidenWarps = E4M3 ? 2 : 0, kThreads = 32 * (6 + kWidenWarps);
  static constexpr int kCtas = 2;            // an SM
  static constexpr int kRing = E4M3 ? 1 : 2; // blocks of K and of V as the tensor cores take them
  static constexpr int kRaw = E4M3 ? 2 : 0;  // blocks of K and V as they are in the cache: two pages' codes and scales of each
  static constexpr int kRawBlock = 4 * kE4m3BlockBytes;
  static constexpr int kScales = E4M3 ? kTrBeside * 2 * kTrKeys * 4 : 0;
  static constexpr int kBytes = 2 * kRing * kTrHalf + kTrQ + kRaw * kRawBlock + kScales;
};
template <bool E4M3> inline size_t tree_smem_bytes(int n) {
  return 1024 + TreeShape<E4M3>::kBytes + sizeof(TreeShared) + (n <= kTrNear ? (size_t)n * sizeof(int4) : 0) + (size_t)(n + 1) * sizeof(int);
}

// 32 lanes x 16 columns of 32 bits into tensor memory, waited for later
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
               "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]) : "memory");
}
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }

template <bool E4M3, bool QF32>
__global__ void __launch_bounds__(TreeShape<E4M3>::kThreads, TreeShape<E4M3>::kCtas) attention_tree_kernel(const __grid_constant__ CUtensorMap kv_map,
                                                                                                          const __grid_constant__ CUtensorMap q_map, const TreeAttnArgs a) {
  using Shape = TreeShape<E4M3>;
  extern __shared__ __align__(16) unsigned char tr_smem_raw[];
  unsigned char *base = tr_smem_raw + ((1024u - (smem_u32(tr_smem_raw) & 1023u)) & 1023u);
  constexpr int kRing = Shape::kRing;
  unsigned char *Qs = base, *Ks = base + kTrQ, *Vs = Ks + kRing * kTrHalf;   // 128 rows x 64 [2], 128 keys x 64 [kRing]: 128-byte swizzle
  unsigned char *raw = Vs + kRing * kTrHalf;                                 // 8-bit cache: [2][K, V][page]
  float *scales = reinterpret_cast<float *>(raw + Shape::kRaw * Shape::kRawBlock);   // and [kTrBeside][K, V][128]
  TreeShared &sh = *reinterpret_cast<TreeShared *>(base + Shape::kBytes);
  int4 *near_s = reinterpret_cast<int4 *>(&sh + 1);   // of each tree: first row, nodes, length and number of the stream
  int *first = reinterpret_cast<int *>(near_s + (a.n_seq <= kTrNear ? a.n_seq : 0));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sh.failed;

  if (warp == Shape::kMmaWarp) tmem_alloc(&sh.tmem, 256);   // S 128 columns, P 64, O 64
  if (tid == 0) {
    const int copied = (int)blockIdx.x == a.starve ? 2 : 1, full = E4M3 ? Shape::kWidenWarps : copied;
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.k_full[i], full); mbar_init(&sh.v_full[i], full); mbar_init(&sh.k_empty[i], 1); mbar_init(&sh.v_empty[i], 1);
      mbar_init(&sh.raw_full[i], copied); mbar_init(&sh.raw_empty[i], E4M3 ? Shape::kWidenWarps : 1);
      mbar_init(&sh.q_full[i], QF32 ? 4 : 1); mbar_init(&sh.q_free[i], 4);
    }
    for (int i = 0; i < kTrParts; ++i) { mbar_init(&sh.part_full[i], 1); mbar_init(&sh.part_free[i], 5 + Shape::kWidenWarps); }
    mbar_init(&sh.s_full, 1); mbar_init(&sh.p_full, 4); mbar_init(&sh.o_full, 1); mbar_init(&sh.meet, 4);
    sh.found = 0;
    sh.failed = __ldcg(a.err) ? 2 : 0;
  }
  if (warp == Shape::kCopyWarp && lane == 0) {
    if (!E4M3) asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map) : "memory");
    if (!QF32) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
  }
  // ---- running sums of cost over the trees ----
  struct Tree { int row0, rows, nodes, keys, committed, stream; };
  auto read_tree = [&](int i) {
    int4 x;
    if (!tree_rows(a.row_start, i, a.R, x.x, x.y)) x.y = -1;
    x.w = a.stream_ids ? a.stream_ids[i] : i;
    if (x.w < 0 || x.w >= a.max_streams) x.w = -1;   // a stream that is none has no keys
    x.z = x.w >= 0 ? a.kv_len[x.w] : 0;
    return x;
  };
  auto tree_from = [&](const int4 &x) {
    return Tree{x.x, x.y < 0 ? -1 : min(x.y, a.t_max), x.y, min(max(x.z, 0), a.pps * kPageTokens), x.z - x.y, x.w};
  };
  auto tree_of = [&](int i) { return tree_from(a.n_seq <= kTrNear ? near_s[i] : read_tree(i)); };
  auto tile_cost = [&](int keys) { return kTrCostTile + kTrCostBlock * ((keys + kTrKeys - 1) / kTrKeys); };
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose rows nothing bounds
#pragma unroll 1
  for (int i0 = 0; i0 < a.n_seq; i0 += Shape::kThreads) {
    const int i = i0 + tid;
    int u = 0;
    if (i < a.n_seq) {
      const int4 read = read_tree(i);
      if (a.n_seq <= kTrNear) near_s[i] = read;
      if (read.w >= 0) prefetch_l2(a.page_table + (size_t)read.w * a.pps);
      const Tree x = tree_from(read);
      bad |= x.rows < 0;
      u = x.rows > 0 ? a.Hkv * a.by_rpt.of(x.rows + a.rpt - 1) * tile_cost(x.keys) : 0;
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
    int before = carry;
#pragma unroll 1
    for (int w = 0; w < Shape::kThreads / 32; ++w) { const int x = sh.warp_tot[w]; if (w < warp) before += x; carry += x; }
    if (i < a.n_seq) first[i] = before + incl - u;
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

  // The part at unit u or behind it that this CTA has blocks of; false: there is none.  Tiles without keys get their zeros here.
  auto part_at = [&](int u, TreePart &p) {
    while (u < u_end) {
      int lo = 0, hi = a.n_seq - 1;
      while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (first[m] <= u) lo = m; else hi = m - 1; }
      const Tree x = tree_of(lo);
      const int tiles = a.by_rpt.of(x.rows + a.rpt - 1), blocks = (x.keys + kTrKeys - 1) / kTrKeys, nu = tile_cost(x.keys);
      const int k = (int)((unsigned)(u - first[lo]) / (unsigned)nu), u0 = first[lo] + k * nu;
      p.kvh = (int)((unsigned)k / (unsigned)tiles);
      const int tile = k - p.kvh * tiles;
      p.row0 = x.row0 + tile * a.rpt;
      p.n_i = min(a.rpt, x.rows - tile * a.rpt) * a.G;
      p.keys = x.keys; p.committed = x.committed; p.nodes = x.nodes; p.stream = x.stream;
      p.next = u0 + nu;
      // Blocks before the border of CTAs c - 1 and c.  A border one or two blocks (an eighth of a range at most) from an end of the tile is moved there: what
      // they cost is less than another part.
      const int near_end = min(2, (int)size.d / (8 * kTrCostBlock));
      auto border = [&](int c) {
        const int b = min((max(c * (int)size.d - u0 - kTrCostTile, 0) + kTrCostBlock - 1) / kTrCostBlock, blocks);
        return b <= near_end && 2 * b <= blocks ? 0 : blocks - b <= near_end ? blocks : b;
      };
      const int ca = size.of(u0), cb = size.of(u0 + nu - 1), me = blockIdx.x;
      p.j0 = me == ca ? 0 : border(me);
      p.j1 = me == cb ? blocks : border(me + 1);
      if (p.j1 > p.j0) {
        for (p.c0 = ca; p.c0 < cb && border(p.c0 + 1) == 0;) ++p.c0;
        for (p.c1 = cb; p.c1 > ca && border(p.c1) == blocks;) --p.c1;
        return true;
      }
      if (blocks == 0 && me == ca) {
        uint4 *rows = reinterpret_cast<uint4 *>(a.out);
        for (int i = lane; i < p.n_i * (kHeadDim / 8); i += 32) {
          const int r = a.by_G.of(i >> 3);
          rows[((size_t)(p.row0 + r) * a.H + (p.kvh - r) * a.G + (i >> 3)) * (kHeadDim / 8) + (i & 7)] = make_uint4(0, 0, 0, 0);
        }
      }
      u = p.next;
    }
    return false;
  };
  auto wait = [&](uint64_t *bar, uint32_t parity) {   // the whole warp; false: some wait of the CTA has run out
    unsigned long long t0 = 0;
#pragma unroll 1
    for (int polls = 0; !mbar_try_wait(bar, parity); ++polls) {
      if ((polls & 15) != 15) continue;        // the timer is read only where the wait is long
      if (*failed) return false;
      const unsigned long long t1 = global_timer_ns();
      if (t0 == 0) t0 = t1;
      if (t1 - t0 > a.wait_ns) { *failed = 1; atomicExch(a.err, 1); return false; }
    }
    return true;
  };
  auto wait_warp = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)) != 0; };
  // Part number n as the first copying warp has described it: a lane a word, into the warp's own copy or to be handed out.  The last one says so.
  auto take_part = [&](int n, int &word) {
    const int k = n % kTrParts;
    if (!wait_warp(&sh.part_full[k], (uint32_t)(n / kTrParts) & 1u)) return false;
    word = lane < kTrPartWords ? reinterpret_cast<const int *>(&sh.part[k])[lane] : 0;
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_free[k]);
    return __shfl_sync(0xFFFFFFFFu, word, offsetof(TreePart, n_i) / 4) > 0;
  };
  auto give_part = [&](int n, const TreePart &p) {
    const int k = n % kTrParts;
    if (n >= kTrParts && !wait_warp(&sh.part_free[k], (uint32_t)(n / kTrParts - 1) & 1u)) return false;
    if (lane == 0) { sh.part[k] = p; mbar_arrive(&sh.part_full[k]); }
    __syncwarp();
    return true;
  };
#define TR_FIELD(word, name) __shfl_sync(0xFFFFFFFFu, word, offsetof(TreePart, name) / 4)
  // page number pg of a stream's list, or -1: it has no keys, or is none
  auto page_of = [&](int stream, int keys, int pg) {
    if (pg * kPageTokens >= keys) return -1;
    const int phys = a.page_table[(size_t)stream * a.pps + pg];
    return phys >= 0 && phys < a.n_pages ? phys : -1;
  };

  if (warp == Shape::kCopyWarp) {
    // ---- copies: 16-bit queries of a tile as often as its rows stand among the lanes, two tiles ahead at most, then its keys and values ----
    int c = 0;                                 // blocks of this CTA
    bool fine = true;
    TreePart p;
    int u = u_begin;
#pragma unroll 1
    for (int n_part = 0; fine; ++n_part) {
      const bool there = part_at(u, p);
      if (!there) p.n_i = 0;                   // the part behind the last has no rows
      fine = give_part(n_part, p) && there;
      if (!fine) break;
      u = p.next;
      if constexpr (!QF32) {
        const int qb = n_part & 1;
        if (n_part >= 2) fine = wait_warp(&sh.q_free[qb], (uint32_t)(n_part / 2 - 1) & 1u);
        if (!fine) break;
        if (elect_one()) {
          mbar_expect_tx(&sh.q_full[qb], (uint32_t)((a.rpt * a.G * 128) << a.lg));
          for (int x = 0; x < 1 << a.lg; ++x) un_box(&q_map, p.kvh * a.G, p.row0, Qs + qb * kTrHalf + x * (kTrHalf >> a.lg), &sh.q_full[qb]);
        }
        __syncwarp();
      }
      int mine = -1;                           // a page of sixteen blocks each lane
#pragma unroll 1
      for (int j = p.j0; j < p.j1 && fine; ++j, ++c) {
        const int at = (j - p.j0) & 15, s = c & 1;
        if (at == 0) mine = page_of(p.stream, p.keys, 2 * j + lane);
        const int p0 = __shfl_sync(0xFFFFFFFFu, mine, 2 * at), p1 = __shfl_sync(0xFFFFFFFFu, mine, 2 * at + 1);
#pragma unroll 1
        for (int w = 0; w < 2; ++w) {          // K, V
          if (c >= 2 && (w == 0 || !E4M3)) fine = wait_warp(E4M3 ? &sh.raw_empty[s] : w ? &sh.v_empty[s] : &sh.k_empty[s], (uint32_t)(c / 2 - 1) & 1u);
          if (!fine) break;
          if (w == 0 && lane == 0) sh.pages_ok[c % kTrBeside] = (p0 >= 0) + 2 * (p1 >= 0);
          __syncwarp();
          if (elect_one()) {
            uint64_t *full = E4M3 ? &sh.raw_full[s] : w ? &sh.v_full[s] : &sh.k_full[s];
            const uint32_t pages = (uint32_t)((p0 >= 0) + (p1 >= 0));
            if constexpr (E4M3) {
              if (w == 0) mbar_expect_tx(full, 2 * pages * kE4m3BlockBytes);
              unsigned char *dst = raw + s * Shape::kRawBlock + 2 * w * kE4m3BlockBytes;
              const size_t head = (size_t)w * a.Hkv + p.kvh;
              if (p0 >= 0) bulk_copy_g2s(dst, a.pool + ((size_t)p0 * 2 * a.Hkv + head) * kE4m3BlockBytes, kE4m3BlockBytes, full);
              if (p1 >= 0) bulk_copy_g2s(dst + kE4m3BlockBytes, a.pool + ((size_t)p1 * 2 * a.Hkv + head) * kE4m3BlockBytes, kE4m3BlockBytes, full);
            } else {
              mbar_expect_tx(full, pages * (kTrHalf / 2));
              unsigned char *dst = (w ? Vs : Ks) + s * kTrHalf;
              if (p0 >= 0) un_box(&kv_map, 0, (p0 * 2 + w) * a.Hkv + p.kvh, dst, full);
              if (p1 >= 0) un_box(&kv_map, 0, (p1 * 2 + w) * a.Hkv + p.kvh, dst + kTrHalf / 2, full);
            }
          }
          __syncwarp();
        }
      }
    }
  } else if (E4M3 && warp >= Shape::kWidenWarp) {
    // ---- codes to bf16, 16 of a row at a time, as soon as the products are done with the block before; and the scales ----
    const int t = tid - 32 * Shape::kWidenWarp, quad = t & 3;
    int word, c = 0;
    bool fine = true;
#pragma unroll 1
    for (int n_part = 0; fine && take_part(n_part, word); ++n_part) {
      const int nb = TR_FIELD(word, j1) - TR_FIELD(word, j0);
#pragma unroll 1
      for (int b = 0; b < nb && fine; ++b, ++c) {
        const unsigned char *from = raw + (c & 1) * Shape::kRawBlock;
        fine = wait_warp(&sh.raw_full[c & 1], (uint32_t)(c / 2) & 1u);
#pragma unroll 1
        for (int w = 0; w < 2 && fine; ++w) {
          if (c > 0) fine = wait_warp(w ? &sh.v_empty[0] : &sh.k_empty[0], (uint32_t)(c - 1) & 1u);
          if (!fine) break;
          if (w == 0) {                        // (both with K: the weights want V's before V is waited for)
#pragma unroll
            for (int e = 0; e < 4; ++e)        // [K, V][page]: 64 scales behind the codes
              scales[(c % kTrBeside) * 2 * kTrKeys + 64 * e + t] = *reinterpret_cast<const float *>(from + e * kE4m3BlockBytes + kPageElems + 4 * t);
          }
          unsigned char *dst = w ? Vs : Ks;
#pragma unroll 2
          for (int r = t >> 2; r < kTrKeys; r += 16) {
            const uint4 code = *reinterpret_cast<const uint4 *>(from + (2 * w + (r >> 6)) * kE4m3BlockBytes + (r & 63) * kHeadDim + 16 * quad);
            const uint32_t x[4] = {code.x, code.y, code.z, code.w};
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[2 * e] = e4m3x2_to_bf16x2(__byte_perm(x[e], 0u, 0x1404));
              y[2 * e + 1] = e4m3x2_to_bf16x2(__byte_perm(x[e], 0u, 0x3424));
            }
            *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad) ^ (r & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad + 1) ^ (r & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(w ? &sh.v_full[0] : &sh.k_full[0]);
            if (w) mbar_arrive(&sh.raw_empty[c & 1]);
          }
        }
      }
    }
  } else if (warp == Shape::kMmaWarp) {
    // ---- products: Q K^T of a tile's first block, then, each time the softmax has block c's weights in tensor memory (and is done with its scores), Q K^T of
    //      block c + 1 and P V of block c, whichever's copy is there first ----
    const uint32_t idesc_qk = tc_instr_desc(128, kTrKeys), idesc_pv = tc_instr_desc(128, kHeadDim) | (1u << 16);   // V is MN-major
    const uint64_t dqs = tc_smem_desc(Qs), dks = tc_smem_desc(Ks), dvs = tc_smem_desc(Vs);
    int n_tile = 0, c = 0, word;               // tiles, and blocks whose weights were waited for
    bool fine = true;
    auto scores = [&](int ck) {                // of block ck
      fine = wait_warp(&sh.k_full[ck % kRing], (uint32_t)(ck / kRing) & 1u);
      if (!fine) return;
      tc_fence_after_sync();
      if (elect_one()) {
        const uint64_t dk = dks + (uint64_t)(ck % kRing) * (kTrHalf >> 4), dq = dqs + (uint64_t)(QF32 ? 0 : n_tile & 1) * (kTrHalf >> 4);
#pragma unroll
        for (int q = 0; q < (QF32 ? 8 : 4); ++q) tc_mma(tmem, dq + (uint64_t)(q >> 2) * (kTrHalf >> 4) + 2 * (q & 3), dk + 2 * (q & 3), idesc_qk, q == 0 ? 0u : 1u);
        tc_commit(&sh.k_empty[ck % kRing]);
        tc_commit(&sh.s_full);
      }
      __syncwarp();
    };
#pragma unroll 1
    for (int n_part = 0; fine && take_part(n_part, word); ++n_part, ++n_tile) {
      const int nb = TR_FIELD(word, j1) - TR_FIELD(word, j0);
      fine = wait_warp(&sh.q_full[QF32 ? 0 : n_tile & 1], (uint32_t)(QF32 ? n_tile : n_tile / 2) & 1u);
#pragma unroll 1
      for (int k = -1; k < nb && fine; ++k) {
        // (the scores first where their keys are there, else the values)
        bool asked = k + 1 == nb;
        if (k >= 0) {
          fine = wait_warp(&sh.p_full, (uint32_t)c & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          const bool now = !asked && __all_sync(0xFFFFFFFFu, mbar_try_wait(&sh.k_full[(c + 1) % kRing], (uint32_t)((c + 1) / kRing) & 1u));
          if (now) { scores(c + 1); asked = true; }
          if (fine) fine = wait_warp(&sh.v_full[c % kRing], (uint32_t)(c / kRing) & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          if (elect_one()) {
            const uint64_t dv = dvs + (uint64_t)(c % kRing) * (kTrHalf >> 4);
#pragma unroll
            for (int q = 0; q < kTrKeys / 16; ++q)   // 16 keys an instruction: 8 columns of P, two groups of 8 rows of V
              tc_mma_ts(tmem + 192u, tmem + 128u + 8u * q, dv + 128 * q, idesc_pv, k == 0 && q == 0 ? 0u : 1u);
            tc_commit(&sh.v_empty[c % kRing]);
            tc_commit(&sh.o_full);
          }
          __syncwarp();
          ++c;
        }
        if (!asked) scores(c);
      }
    }
  } else {
    // ---- softmax ----
    const int copies = 1 << a.lg, rgs = 4 >> a.lg, rg = warp & (rgs - 1), rep = warp >> (2 - a.lg);   // which 32 rows of the tile, and which copy of them
    const int i_row = 32 * rg + lane, chunks = rgs, col0 = rep * 32 * chunks;                         // the thread's row, and its first key of a block
    const uint32_t t_lane = tmem + ((uint32_t)(32 * warp) << 16);
    int n_meet = 0, c = 0, n_tile = 0, word;                 // waits for meet, blocks, tiles
    bool fine = true;
    // Of the tile that began before the CTA's range, and of its last one, where other CTAs share them: how many had a ticket when this CTA took its own (0: it has
    // no part, or none yet), and which of the two tickets is still to be taken.
    int came[2] = {0, 0}, due = -1;
    TreePart &p = sh.mine[warp];
    if (copies > 1) {                          // weights of the other copies' keys: zero throughout
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
    // A tile that several CTAs share has a place in each: by warp, its values' columns of four for 32 rows, then reference and sum.  A CTA has
    // two places: for the tile that began before its range, and the one that goes on behind it.
    auto place = [&](int cta, int c0) { return a.part + (size_t)(2 * cta + (cta == c0)) * 128 * kTrPitch; };
    auto at_values = [&](int x) { return (warp * chunks + x) * 4 * 128 + lane * 4; };   // of 16 values x of the thread's row
    // those of CTAs c .. c1, in the order of their keys, onto o, m, l; the sum of weights
    auto add_parts = [&](int c0, int cta, int c1, int x, float (&o)[16], float m, float l) {
#pragma unroll 1
      for (; cta <= c1; ++cta) {
        const float *from = place(cta, c0);
        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(from + 128 * kHeadDim + 64 * warp + 2 * lane));
        float4 v[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __ldcg(reinterpret_cast<const float4 *>(from + at_values(x) + 128 * e));
        const bool has = ml.y != 0.f;          // a key in it
        const float mn = fmaxf(m, ml.x), fk = !has || m == mn ? 1.f : pt_exp2(m - mn), fn = has ? pt_exp2(ml.x - mn) : 0.f;
        if (has) m = mn;
        l = fmaf(l, fk, ml.y * fn);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          o[4 * e] = fmaf(o[4 * e], fk, v[e].x * fn); o[4 * e + 1] = fmaf(o[4 * e + 1], fk, v[e].y * fn);
          o[4 * e + 2] = fmaf(o[4 * e + 2], fk, v[e].z * fn); o[4 * e + 3] = fmaf(o[4 * e + 3], fk, v[e].w * fn);
        }
      }
      return l;
    };
    auto leave = [&](const TreePart &p, int x, const float (&o)[16], float l) {   // 16 values x of the thread's row
      if (i_row >= p.n_i) return;
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      const int r = a.by_G.of(i_row);
      uint4 *dst = reinterpret_cast<uint4 *>(a.out + ((size_t)(p.row0 + r) * a.H + (p.kvh - r) * a.G + i_row) * kHeadDim + 16 * (rep * chunks + x));
#pragma unroll
      for (int e = 0; e < 2; ++e)
        dst[e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                            pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
    };
    auto take_ticket = [&]() {                 // for the part written some time ago
      fence_gpu();
      __syncwarp();
      int n = 0;
      if (lane == 0) n = (int)atomicAdd(a.tickets + 4 * sh.shared[due][warp].c0 + warp, 1u) + 1;
      if (due == 0) came[0] = n; else came[1] = n;
      due = -1;
    };
#pragma unroll 1
    for (int n_part = 0; fine && take_part(n_part, word); ++n_part, ++n_tile) {
      if (lane < kTrPartWords) reinterpret_cast<int *>(&p)[lane] = word;
      __syncwarp();
      const int j0 = p.j0, nb = p.j1 - j0;
      const bool mine = i_row < p.n_i, live = 32 * rg < p.n_i;   // the thread's row exists, some row of the warp does
      float m = -INFINITY, l = 0.f;
      if constexpr (QF32) {                    // the row's queries, as often as it stands among the lanes
        const int r = a.by_G.of(i_row);
        const size_t at = mine ? (size_t)(p.row0 + r) * a.q_stride + (size_t)((p.kvh - r) * a.G + i_row) * kHeadDim : 0;
#pragma unroll 4
        for (int e8 = 0; e8 < 8; ++e8) {
          const int to = tid * 128 + ((e8 ^ (tid & 7)) << 4);
          float x[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) x[e] = 0.f;
          if (mine) load8(reinterpret_cast<const float *>(a.q) + at + 8 * e8, x);
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float f0 = __uint_as_float(__float_as_uint(x[2 * e]) & 0xFFFF0000u), f1 = __uint_as_float(__float_as_uint(x[2 * e + 1]) & 0xFFFF0000u);
            hi[e] = pack_bf16x2(f0, f1);
            lo[e] = pack_bf16x2(x[2 * e] - f0, x[2 * e + 1] - f1);
          }
          *reinterpret_cast<uint4 *>(Qs + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
          *reinterpret_cast<uint4 *>(Qs + kTrHalf + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[0]);
      }
      const int *row_mask = a.mask + (size_t)(p.row0 + a.by_G.of(min(i_row, p.n_i - 1))) * a.words;
      const unsigned mask0 = (unsigned)row_mask[0], mask1 = a.words > 1 ? (unsigned)row_mask[1] : 0u;   // asked for here, wanted where drafted keys begin
#pragma unroll 1
      for (int b = 0; b < nb; ++b, ++c) {
        const int key0 = (j0 + b) * kTrKeys, n = min(kTrKeys, p.keys - key0), committed = p.committed;
        fine = wait_warp(&sh.s_full, (uint32_t)c & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        const int pages = *reinterpret_cast<volatile int *>(&sh.pages_ok[c % kTrBeside]);
        const bool drafted = key0 + kTrKeys > committed, special = drafted || n < kTrKeys || pages != 3;
        const float *ks = scales + (2 * (c % kTrBeside)) * kTrKeys + col0, *vs = ks + kTrKeys;   // 8-bit cache: of K and V
        auto visible = [&](int x) {            // bits of the thread's keys 32 x .. 32 x + 31 that its row sees
          const int nodes = p.nodes;
          auto bits = [&](int w) {
            if (w >= a.words || 32 * w >= nodes) return 0u;
            const unsigned v = w == 0 ? mask0 : w == 1 ? mask1 : (unsigned)row_mask[w];
            return nodes - 32 * w < 32 ? v & ((1u << (nodes - 32 * w)) - 1u) : v;
          };
          const int k0 = col0 + 32 * x, d = key0 + k0 - committed;   // number of the first of these keys among the drafted
          unsigned v = ~0u;
          if (d >= 0) v = __funnelshift_r(bits(d >> 5), d & 31 ? bits((d >> 5) + 1) : 0u, d & 31);
          else if (d > -32) v = (bits(0) << -d) | ((1u << -d) - 1u);
          const int there = pages >> (k0 >> 6) & 1 ? n - k0 : 0;
          return there <= 0 ? 0u : there < 32 ? v & ((1u << there) - 1u) : v;
        };
        if (live) {
          float s[32];
          unsigned seen = ~0u;
          auto scores = [&](int x) {           // of the thread's keys 32 x .. 32 x + 31
            tmem_ld32_async(t_lane + (uint32_t)(col0 + 32 * x), s);
            if (special) seen = visible(x);
            tmem_wait_ld();
            tmem_landed32(s);
            if constexpr (E4M3) {
#pragma unroll
              for (int e = 0; e < 32; e += 4) {
                const ulonglong2 f = *reinterpret_cast<const ulonglong2 *>(ks + 32 * x + e);
                unpack_f32x2(mul_f32x2(pack_f32x2(s[e], s[e + 1]), f.x), s[e], s[e + 1]);
                unpack_f32x2(mul_f32x2(pack_f32x2(s[e + 2], s[e + 3]), f.y), s[e + 2], s[e + 3]);
              }
            }
            if (special) {
#pragma unroll
              for (int e = 0; e < 32; ++e) s[e] = seen >> e & 1u ? s[e] : -INFINITY;
            }
          };
          float top = -INFINITY, sc = 1.f;
#pragma unroll 1
          for (int x = 0; x < chunks; ++x) {
            scores(x);
            float mx[4] = {top, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 32; e += 8) {
#pragma unroll
              for (int q = 0; q < 4; ++q) mx[q] = max3(mx[q], s[e + 2 * q], s[e + 2 * q + 1]);
            }
            top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
          }
          top *= a.scale;
          if (m == -INFINITY) { sc = 0.f; m = top; }   // nothing seen yet; O, where there is one, is zero
          else if (top > m + kTrSlack) { sc = pt_exp2(m - top); m = top; }
          if (!mine) { sc = 1.f; m = 0.f; }            // a row that does not exist holds anything
          // P V of the block before, to which P and O belong
          if (b > 0) {
            fine = wait_warp(&sh.o_full, (uint32_t)(c - 1) & 1u);
            if (!fine) break;
            tc_fence_after_sync();
            if (__any_sync(0xFFFFFFFFu, sc != 1.f)) {
              float keep[32];                          // (the scores stay where there is one chunk of them)
#pragma unroll 1
              for (int d = 0; d < kHeadDim; d += 32) {
                tmem_ld32(t_lane + 192u + (uint32_t)d, keep);
#pragma unroll
                for (int e = 0; e < 32; ++e) keep[e] *= sc;
                tmem_st32(t_lane + 192u + (uint32_t)d, keep);
              }
            }
          }
          const float ref = m == -INFINITY ? 0.f : m;
          const unsigned long long scale2 = pack_f32x2(a.scale, a.scale), ref2 = pack_f32x2(-ref, -ref);
          unsigned long long sum2[2] = {0ull, 0ull};
#pragma unroll 1
          for (int x = 0; x < chunks; ++x) {
            if (chunks > 1) scores(x);
#pragma unroll
            for (int e = 0; e < 32; e += 2) {
              float y, z;
              const unsigned long long d2 = fma_f32x2(pack_f32x2(s[e], s[e + 1]), scale2, ref2);
              if ((e >> 1) % 4 == 3) {                 // a quarter of the exponentials on the FMA pipes
                unpack_f32x2(poly_exp2(d2), y, z);
              } else {
                unpack_f32x2(d2, y, z);
                y = pt_exp2(y); z = pt_exp2(z);
              }
              sum2[(e >> 1) & 1] = add_f32x2(sum2[(e >> 1) & 1], pack_f32x2(y, z));
              if constexpr (E4M3) {
                float fy, fz;
                unpack_f32x2(*reinterpret_cast<const unsigned long long *>(vs + 32 * x + e), fy, fz);
                if (special) {                         // a key that is not seen may have any scale
                  fy = seen >> e & 1u ? fy : 0.f;
                  fz = seen >> (e + 1) & 1u ? fz : 0.f;
                }
                y *= fy; z *= fz;
              }
              s[e >> 1] = __uint_as_float(pack_bf16x2(y, z));
            }
            tmem_st16_async(t_lane + 128u + (uint32_t)(col0 / 2 + 16 * x), s);
          }
          float s0, s1;
          unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
          l = fmaf(l, sc, s0 + s1);
          tmem_wait_st();
        } else if (b > 0) {
          fine = wait_warp(&sh.o_full, (uint32_t)(c - 1) & 1u);
          if (!fine) break;
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
              else if (key0 + k >= committed) {
                const uint4 y = *piece;
                auto odd = [](uint32_t z) { return (z & 0x7F80u) == 0x7F80u || (z & 0x7F800000u) == 0x7F800000u; };
                if (odd(y.x) || odd(y.y) || odd(y.z) || odd(y.w)) { *piece = make_uint4(0, 0, 0, 0); found |= 1u << x; }
              }
            }
            fence_proxy_async_smem();
            if (drafted) {
              if (found) sh.found = c + 1;     // (whoever writes writes the same)
              fine = meet();
              if (fine && *reinterpret_cast<volatile int *>(&sh.found) == c + 1) {   // rare: which keys, and who sees them
                if (tid < 4) sh.bad[tid] = 0u;
                fine = meet();
#pragma unroll 1
                for (int x = 0; x < 8; ++x)
                  if (found >> x & 1) { const int k = (tid >> 3) + 16 * x; atomicOr(&sh.bad[k >> 5], 1u << (k & 31)); }
                fine = meet() && fine;
                if (live) {
#pragma unroll 1
                  for (int x = 0; x < chunks; ++x)
                    if (visible(x) & *reinterpret_cast<volatile unsigned *>(&sh.bad[col0 / 32 + x])) l = __int_as_float(0x7FFFFFFF);
                }
                fine = meet() && fine;         // before the next block's are written
              }
              if (!fine) break;
            }
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full);
        if (due >= 0) take_ticket();
      }
      if (!fine) break;
      // ---- the tile's sums ----
      fine = wait_warp(&sh.o_full, (uint32_t)(c - 1) & 1u);
      if (!fine) break;
      tc_fence_after_sync();
      float met[16];                           // where a row stands several times: its sums, or a half or a quarter of them at a time
      float4 *stage = reinterpret_cast<float4 *>(Qs + (QF32 ? 0 : (n_tile & 1) * kTrHalf));   // where the queries were, which no product reads any more
      if (copies > 1 && live) sh.ml[warp][lane] = make_float2(m, l);
      float mine_f[4];                         // what each copy's sums are multiplied by
      const int c0 = p.c0, c1 = p.c1;
      const bool begins = c0 == (int)blockIdx.x;
      bool whole = c0 == c1, others = false;   // others: their parts are there
      unsigned *ticket = a.tickets + 4 * c0 + warp;   // for the warp's 32 rows
      if (begins && !whole) {                  // the CTA's last tile; as a rule the others have long had their tickets
        unsigned came = 0;
        if (lane == 0) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(came) : "l"(ticket) : "memory");
        others = __shfl_sync(0xFFFFFFFFu, came, 0) == (unsigned)(c1 - c0);
        whole = others;
        if (others) fence_gpu();
      }
      float *to = place(blockIdx.x, c0);
      auto pass_on = [&](int x, float (&o)[16]) {   // 16 values x of the thread's row leave, or go to scratch
        if (whole) {
          const float total = others && mine ? add_parts(c0, c0 + 1, c1, x, o, m, l) : l;
          leave(p, x, o, total);
        } else if (mine) {
#pragma unroll
          for (int e = 0; e < 4; ++e) *reinterpret_cast<float4 *>(to + at_values(x) + 128 * e) = make_float4(o[4 * e], o[4 * e + 1], o[4 * e + 2], o[4 * e + 3]);
        }
      };
      if (copies == 1) {
#pragma unroll 1
        for (int x = 0; x < 4; ++x) {
          if (live) tmem_ld16(t_lane + 192u + 16u * x, met);
          pass_on(x, met);
        }
      } else {
        // half of the values at a time: that is what one tile's queries took
#pragma unroll 1
        for (int h = 0; h < 2 && fine; ++h) {
          if (live) {
            float x[32];
            tmem_ld32(t_lane + 192u + 32u * h, x);
#pragma unroll
            for (int e = 0; e < 32; e += 4) stage[(warp * 8 + e / 4) * 32 + lane] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
          }
          fine = meet();
          if (!fine) break;
          if (h == 0) {
            float M = -INFINITY, ly[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const float2 ml = x < copies && live ? sh.ml[rg + x * rgs][lane] : make_float2(-INFINITY, 0.f);
              mine_f[x] = ml.x; ly[x] = ml.y;
              if (ml.y != 0.f) M = fmaxf(M, ml.x);
            }
            m = M; l = 0.f;
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              mine_f[x] = ly[x] == 0.f ? 0.f : pt_exp2(mine_f[x] - M);   // no key in it
              l = fmaf(ly[x], mine_f[x], l);
            }
          }
#pragma unroll 1
          for (int x = 0; x < chunks; ++x) {
            const int d16 = rep * chunks + x;  // which 16 values of the 64
            if (d16 >> 1 != h) continue;
#pragma unroll
            for (int e = 0; e < 16; ++e) met[e] = 0.f;
            if (live) {
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                if (y >= copies) continue;
                const float f = mine_f[y];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  const float4 v = stage[((rg + y * rgs) * 8 + (d16 & 1) * 4 + e) * 32 + lane];
                  met[4 * e] = fmaf(v.x, f, met[4 * e]); met[4 * e + 1] = fmaf(v.y, f, met[4 * e + 1]);
                  met[4 * e + 2] = fmaf(v.z, f, met[4 * e + 2]); met[4 * e + 3] = fmaf(v.w, f, met[4 * e + 3]);
                }
              }
            }
            pass_on(x, met);
          }
          fine = meet();                       // before the other half, or the next queries, are written there
        }
        if (!fine) break;
      }
      tc_fence_before_sync();                  // O may be overwritten once this thread's next P is announced
      if constexpr (!QF32) {                   // the queries of the tile after next are copied over these
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_free[n_tile & 1]);
      }
      if (whole) {
        if (others && lane == 0) *ticket = 0u;
        continue;
      }
      if (mine) *reinterpret_cast<float2 *>(to + 128 * kHeadDim + 64 * warp + 2 * lane) = make_float2(m, l);
      due = begins;
      if (lane < kTrPartWords) reinterpret_cast<int *>(&sh.shared[due][warp])[lane] = word;
      __syncwarp();
    }
    // ---- the tiles that other CTAs share, where this CTA came last: the one that began before its range, and its last ----
    if (fine && due >= 0) take_ticket();
#pragma unroll 1
    for (int which = 0; fine && which < 2; ++which) {
      const int n = __shfl_sync(0xFFFFFFFFu, which ? came[1] : came[0], 0);
      if (n == 0) continue;
      const TreePart &q = sh.shared[which][warp];
      if (n != q.c1 - q.c0 + 1) continue;
      if (lane == 0) a.tickets[4 * q.c0 + warp] = 0u;
      fence_gpu();
#pragma unroll 1
      for (int x = 0; x < chunks; ++x) {
        float o[16];
#pragma unroll
        for (int e = 0; e < 16; ++e) o[e] = 0.f;
        const float l = i_row < q.n_i ? add_parts(q.c0, q.c0, q.c1, x, o, -INFINITY, 0.f) : 0.f;
        leave(q, x, o, l);
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
#undef TR_FIELD
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

// rows of bf16 queries [64, heads, rows], a group's heads of a tile's rows a copy
inline cudaError_t tree_q_map(CUtensorMap *map, const TreeAttnArgs &a) {
  const cuuint64_t dims[3] = {kHeadDim, (cuuint64_t)a.H, (cuuint64_t)a.R}, strides[2] = {kHeadDim * 2, (cuuint64_t)a.q_stride * 2};
  const cuuint32_t box[3] = {kHeadDim, (cuuint32_t)a.G, (cuuint32_t)a.rpt};
  return tensor_map_encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, a.q, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

template <bool E4M3, bool QF32>
inline cudaError_t launch_tree(const CUtensorMap &map, TreeAttnArgs a, int n_sm, cudaStream_t st) {
  using Shape = TreeShape<E4M3>;
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(attention_tree_kernel<E4M3, QF32>, tree_smem_bytes<E4M3>(kTrMaxSeq))) return e;
  const long long rows = (long long)a.t_max * a.G;
  a.lg = rows <= 32 ? 2 : rows <= 64 ? 1 : 0;
  a.rpt = (128 >> a.lg) / a.G;
  a.by_rpt.set((uint32_t)a.rpt);
  CUtensorMap q_map = {};
  if (!QF32)
    if (const cudaError_t e = tree_q_map(&q_map, a)) return e;
  return launch_kernel(attention_tree_kernel<E4M3, QF32>, dim3((unsigned)min(Shape::kCtas * n_sm, kTrMaxCtas)), dim3(Shape::kThreads), tree_smem_bytes<E4M3>(a.n_seq), st, false,
                       map, q_map, a);
}

}  // namespace ttsgpt
