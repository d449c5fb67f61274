// Attention of trees of drafted tokens over a paged cache, on the 5th-generation tensor cores (Section I: the decode engine's attention
// kernels, here for several tokens of a stream at once).
//
// Row r of tree i is a node.  It attends to all committed keys of its stream and to those of the stream's last T_i keys whose bits its
// mask has:  o = sum_j p_j v_j,  p_j = 2^(s_j - m) / sum 2^(s_j - m),  s_j = scale log2(e) q.k_j.  A row that sees no key is zero.
//
// Tile.  Rows of one tree times the G query heads of a head of keys, at most 128 / S of them, a step a page of 64 keys:
//     S = Q K^T     tcgen05.mma M=128 x N=64 x K=64, fp32 in tensor memory (fp32 queries as two bf16 parts, 16 bits)
//     softmax       a thread a lane of tensor memory: reference m and sum l in fp32, P rounded to bf16 back into tensor memory; the
//                   reference moves, and O with it, only where a score exceeds it by more than 8 (log2): weights stay below 2^8, sums below 2^8 per key
//     O += P V      M=128 x N=64 x K=64, V as stored
// Scores and weights have two places each, by turns, so that the products of a step run beside the softmax of the next: S 2 x 64, P 2 x 32, O 64 columns, 256 in
// all, two CTAs an SM.  Where a tile has at most 64 or 32 rows, they stand S = 2 or 4 times among the 128 lanes, and each copy's threads take only their half or quarter of a
// step's keys (their P is zero elsewhere): the exponentials, which would otherwise be one or two warps', are spread over all four, and a row's S sums meet
// in shared memory at the end of the tile.  (S = 4, 2, 1: 16 trees of up to 32 nodes, 20 heads 25.7, 27.7, 33.8 us; 128 trees of up to 6, 5 heads to each of 4 32.2,
// 33.7, 38.0; S = 2, 1: 64 nodes 29.8, 35.7.)
//
// Warps.  Four of softmax; one that finds the CTA's tiles, describes them to the others and copies queries and pages by TMA, four pages ahead; one that issues
// the products, over the borders of tiles too; one that takes tickets (below).  Blocks of the 8-bit cache come as they are by bulk copies, four ahead, and two or four more warps widen the
// codes to bf16 (exact) where the tensor cores take them, two ahead; K's scales multiply the scores and V's the weights, in fp32, before those are rounded.
//
// Work split.  Tiles are laid end to end by what they cost and cut into equal ranges, one a CTA, wherever the cut falls; parts of a tile that
// several CTAs share go to scratch with a ticket, and the CTA that comes last adds them in the order of their keys, so that results do not
// depend on timing.  Every wait is bounded.
//
// Bound.  One tree of 8 nodes, 20 heads, 341 keys: 9.6 us, of which 4 pass before the first scores (tensor memory, the trees, the first copy); then come steps of
// 0.7 us, the end of a tile and the parts' joining, 3 us.  16 trees of up to 64 nodes, 20 heads, 88 MB of keys and values: 29.4 us against 14.2 of reading; steps of 0.6 to 0.75 us each,
// of which scores to weights take most (tensor memory there and back, 2^x, the two products' latency), not bytes.  128 trees of 25 nodes by 5 heads to each of 4 heads of the
// 8-bit cache: 58 us, the softmax warps' instructions (512 tiles of up to 125 rows); tensor cores and memory wait.
#pragma once
#include "attention_common.cuh"
#include "draft_trees.cuh"
#include "tensor_map.cuh"
#include <atomic>
#include <cstddef>

namespace ttsgpt {

constexpr int kTrKeys = kPageTokens;        // keys of a step: a page
constexpr int kTrPage = kTrKeys * 128;      // K or V of a page as bf16: 8 KB
constexpr int kTrRows = 128 * 128;          // queries of a tile, as often as they stand among the 128 lanes: 16 KB
constexpr int kTrQ = 2 * kTrRows;           // of two tiles (fp32: both parts of one)
constexpr int kTrMaxSeq = 2048;
constexpr int kTrNear = 256;                // trees up to which a CTA keeps what it has read of them
constexpr int kTrMaxCtas = 320;
constexpr int kTrPitch = 68;                // floats of a row's part
constexpr float kTrSlack = 8.0f;            // log2 by which a score may exceed the reference
constexpr int kTrCostTile = 3;              // what a tile costs besides its steps, in steps (us of 16 trees of 64 nodes by 20 heads / 128 of 25 by 5 heads to each of 4, bf16: 1, 2, 3, 4, 5: 29.1 / 47.9, 29.4 / 44.6, 29.4 / 43.2, 29.7 / 44.5, 29.9 / 44.5)
// Parts that the copying warp may describe ahead.  Every part has a step, and no copy is more than six steps ahead of the softmax, so that it
// never waits for a place while the softmax waits for it.
constexpr int kTrParts = 8;
// Places of what is written beside a page: whether it is there (by the copying warp, four pages ahead of the products, which are two ahead of the softmax)
// and the scales of the 8-bit cache (by the widening warps, two ahead of the products).
constexpr int kTrThere = 8, kTrScales = 4;
constexpr int kTrNodes = 1024;              // of a tree that masks can name
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
  int row0, n_i, kvh, next;     // first row, rows times heads, head of keys; where the next tile's cost begins
  int j0, j1, keys, committed, nodes, stream;   // its pages here; keys of the stream, of them committed, nodes of the tree
  int c0, c1;                   // first and last CTA that have pages of the tile
};
constexpr int kTrPartWords = sizeof(TreePart) / 4;

struct alignas(16) TreeShared {
  TreePart part[kTrParts];
  TreePart mine[4], shared[2][4];   // the softmax warps' own copies: the part at hand; of tiles of several CTAs the one that began before the range, and the last
  uint64_t part_full[kTrParts], part_free[kTrParts];
  uint64_t k_full[4], v_full[4], raw_full[4], raw_empty[4];
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[4], p_full[2], o_full[4];   // by step: scores there (and K read), weights there, their product done (and V read)
  uint64_t written, came_full;  // the first tile's part is in scratch; its tickets are taken
  uint64_t meet;                // the softmax warps among themselves, bounded like every wait
  uint32_t tmem;
  int failed;                   // 1: a wait of the CTA has run out; 2: one of an earlier call with the same scratch had
  int there[kTrThere];          // of a step: is its page one?
  int found;                    // number (from 1 on) of the last tile that has a drafted key whose V is not finite
  int came[4];                  // how many CTAs had a ticket then, of each warp's rows
  unsigned bad[kTrNodes / 32];  // those keys; zero between tiles
  float2 ml[4][32];
  Div size;
  int warp_tot[16], top_cost;   // ... and the most that a tile costs
};

// The tile whose sums may still stand in the place of V that page `i` (from 0 on) of part n_part takes, where there are four places; -1: none.  A tile's sums meet in the
// places of its last page and of the one before, which are those of the next part's fourth and third page: the third waits for both.  Older tiles have left: the part's
// queries are copied behind the end of the tile two before.  To wait for one of those could go wrong, because its barrier serves every second tile: when the next
// of these has left too, the phase that is asked for looks as if it had not ended.
__host__ __device__ constexpr int tree_tile_in_place(int n_part, int i) { return i == 2 ? n_part - 1 : -1; }

template <int S, bool E4M3> struct TreeShape {
  // warps 0-3: softmax, 4: copies, 5: products; 8-bit cache: codes to bf16, two warps (6, 7) where the softmax takes longer than they do, or four (8-11; 6
  // and 7 only give up their registers)
  static constexpr int kCopyWarp = 4, kMmaWarp = 5, kWidenWarp = S == 1 ? 6 : 8, kWidenWarps = !E4M3 ? 0 : S == 1 ? 2 : 4;
  static constexpr bool kTicketWarp = S > 1;  // warp 6 takes the first tile's tickets; else the copying warp does
  static constexpr int kThreads = !E4M3 ? (S == 1 ? 192 : 224) : S == 1 ? 256 : 384;
  // 8-bit cache: registers of a thread, which the groups of four warps split anew; at launch each has 128 or 80 (tiles of 128 rows: softmax 168, 176, 184, 192, 200: 62.4, 61.1, 58.5,
  // 59.6, 59.6 us; of 64: 120, 136: 45.6, 45.0)
  static constexpr int kRegsLaunch = S == 1 ? 128 : 80, kRegsSoftmax = S == 1 ? 184 : 136, kRegsCopy = S == 1 ? 72 : 56, kRegsWiden = S == 1 ? 0 : 48;
  static_assert(kRegsSoftmax + kRegsCopy + kRegsWiden <= kRegsLaunch * (S == 1 ? 2 : 3), "a split of more registers than the launch has would wait forever");
  static constexpr int kCtas = 2;            // an SM
  static constexpr int kRing = E4M3 ? 2 : 4; // pages of K and of V as the tensor cores take them
  static_assert(E4M3 || kRing == 4, "tree_tile_in_place counts on four places");
  static constexpr int kRaw = E4M3 ? 4 : 0;  // pages of K and V as they are in the cache, codes and scales
  static constexpr int kRawPage = 2 * kE4m3BlockBytes;
  static constexpr int kScales = E4M3 ? kTrScales * 2 * kTrKeys * 4 : 0;
  static constexpr int kBytes = kTrQ + 2 * kRing * kTrPage + kRaw * kRawPage + kScales;
};
template <int S, bool E4M3> inline size_t tree_smem_bytes(int n) {
  return 1024 + TreeShape<S, E4M3>::kBytes + sizeof(TreeShared) + (n <= kTrNear ? (size_t)n * sizeof(int4) : 0) + (size_t)(n + 1) * sizeof(int);
}

__device__ __forceinline__ void tmem_st8_async(uint32_t taddr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
               ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]) : "memory");
}
// 32 lanes x 16 columns of 32 bits into tensor memory, waited for later
__device__ __forceinline__ void tmem_st16_async(uint32_t taddr, const float *v) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
               ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]),
               "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15]) : "memory");
}
// Has the phase ended?  (Does not suspend the thread, as mbar_try_wait may.)  The whole warp asks and has one answer: lanes that look at a barrier while
// others arrive may see different things, and what follows has votes of all lanes in it.
__device__ __forceinline__ bool mbar_test_warp(uint64_t *bar, uint32_t parity) {
  uint32_t done;
  asm volatile("{\n\t.reg .pred p;\n\tmbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(done) : "r"(smem_u32(bar)), "r"(parity) : "memory");
  return __any_sync(0xFFFFFFFFu, done != 0);
}
__device__ __forceinline__ void fence_gpu() { asm volatile("fence.acq_rel.gpu;" ::: "memory"); }

template <int S, bool E4M3, bool QF32>
__global__ void __launch_bounds__(TreeShape<S, E4M3>::kThreads, TreeShape<S, E4M3>::kCtas) attention_tree_kernel(const __grid_constant__ CUtensorMap kv_map,
                                                                                                          const __grid_constant__ CUtensorMap q_map, const TreeAttnArgs a) {
  using Shape = TreeShape<S, E4M3>;
  extern __shared__ __align__(16) unsigned char tr_smem_raw[];
  unsigned char *base = tr_smem_raw + ((1024u - (smem_u32(tr_smem_raw) & 1023u)) & 1023u);
  constexpr int kRing = Shape::kRing, kCols = kTrKeys / S, kRgs = 4 / S;   // a thread's keys of a step; groups of 32 rows of a tile
  unsigned char *Qs = base, *Ks = base + kTrQ, *Vs = Ks + kRing * kTrPage;   // 128 rows x 64 [2], 64 keys x 64 [kRing]: 128-byte swizzle
  unsigned char *raw = Vs + kRing * kTrPage;                                 // 8-bit cache: [kRaw][K, V]
  float *scales = reinterpret_cast<float *>(raw + Shape::kRaw * Shape::kRawPage);   // and [kTrScales][K, V][64]
  TreeShared &sh = *reinterpret_cast<TreeShared *>(base + Shape::kBytes);
  int4 *near_s = reinterpret_cast<int4 *>(&sh + 1);   // of each tree: first row, nodes, length and number of the stream
  int *first = reinterpret_cast<int *>(near_s + (a.n_seq <= kTrNear ? a.n_seq : 0));
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sh.failed;

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
  auto tile_cost = [&](int keys) { return kTrCostTile + (keys + kTrKeys - 1) / kTrKeys; };
  pdl_wait();                                  // nothing of memory is touched before
  const int4 own = tid < a.n_seq ? read_tree(tid) : make_int4(0, 0, 0, -1);   // asked for before anything else
  if (warp == Shape::kMmaWarp) tmem_alloc(&sh.tmem, 256);   // S 2 x 64 columns, P 2 x 32, O 64
  const int failed_before = tid == 0 ? __ldcg(a.err) : 0;
  if (tid == 32) {
    const int copied = (int)blockIdx.x == a.starve ? 2 : 1, full = E4M3 ? Shape::kWidenWarps / 2 : copied;
    for (int i = 0; i < 4; ++i) {
      mbar_init(&sh.k_full[i], full); mbar_init(&sh.v_full[i], full); mbar_init(&sh.s_full[i], 1); mbar_init(&sh.o_full[i], 1);
      mbar_init(&sh.raw_full[i], copied); mbar_init(&sh.raw_empty[i], E4M3 ? Shape::kWidenWarps : 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_full[i], QF32 ? 4 : 1); mbar_init(&sh.q_free[i], 4); mbar_init(&sh.p_full[i], 4);
    }
    for (int i = 0; i < kTrParts; ++i) { mbar_init(&sh.part_full[i], 1); mbar_init(&sh.part_free[i], 5 + Shape::kWidenWarps + Shape::kTicketWarp); }
    mbar_init(&sh.meet, 4); mbar_init(&sh.written, 4); mbar_init(&sh.came_full, 1);
    sh.found = 0;
    for (int i = 0; i < kTrNodes / 32; ++i) sh.bad[i] = 0u;
    sh.top_cost = 0;
  }
  if (warp == Shape::kCopyWarp && lane == 0) {
    if (!E4M3) asm volatile("prefetch.tensormap [%0];" ::"l"(&kv_map) : "memory");
    if (!QF32) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
  }
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose rows nothing bounds
#pragma unroll 1
  for (int i0 = 0; i0 < a.n_seq; i0 += Shape::kThreads) {
    const int i = i0 + tid;
    int u = 0, cost = 0;
    if (i < a.n_seq) {
      const int4 read = i0 == 0 ? own : read_tree(i);
      if (a.n_seq <= kTrNear) near_s[i] = read;
      if (read.w >= 0) prefetch_l2(a.page_table + (size_t)read.w * a.pps);
      const Tree x = tree_from(read);
      bad |= x.rows < 0;
      cost = x.rows > 0 ? tile_cost(x.keys) : 0;
      u = x.rows > 0 ? a.Hkv * a.by_rpt.of(x.rows + a.rpt - 1) * cost : 0;
    }
    const int dearest = (int)__reduce_max_sync(0xFFFFFFFFu, (unsigned)cost);
    int incl = u;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 31) { sh.warp_tot[warp] = incl; atomicMax(&sh.top_cost, dearest); }
    bad = __syncthreads_or(bad);
    int before = carry;
#pragma unroll 1
    for (int w = 0; w < Shape::kThreads / 32; ++w) { const int x = sh.warp_tot[w]; if (w < warp) before += x; carry += x; }
    if (i < a.n_seq) first[i] = before + incl - u;
  }
  const int T = bad ? 0 : carry;
  if (tid == 0) {
    first[a.n_seq] = T;
    // Few tiles are cut into ranges of three pages at least, and not at all where they have no more than eight: parts cost more than they take off another CTA (20
    // heads, ranges of 1, 2, 3, 4, 8 pages: a tree of 256 nodes, 856 keys 21.9, 21.2, 21.8, 21.3, 28.3 us, of 8 nodes, 1908 keys 13.5, 13.5, 13.4, 13.6, 14.7; of 8
    // nodes, 341 keys, uncut 9.5, cut 10.0 to 11.9).
    const int least = sh.top_cost <= kTrCostTile + 8 ? sh.top_cost : kTrCostTile + 3;
    sh.size.set(max(least, max(1, (T + (int)gridDim.x - 1) / (int)gridDim.x)));
    sh.failed = failed_before ? 2 : 0;
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  pdl_launch_dependents();                     // the CTA has its tensor memory: the next kernel can take none from under it
  const Div size = sh.size;
  const int u_begin = blockIdx.x * (int)size.d, u_end = __any_sync(0xFFFFFFFFu, *failed) ? u_begin : min(T, u_begin + (int)size.d);   // one for the warp: part_at votes

  // The part at unit u or behind it that this CTA has pages of; false: there is none.  Tiles without keys get their zeros here.
  auto part_at = [&](int u, TreePart &p) {
    while (u < u_end) {
      int lo = 0;                              // last tree that begins at or before u: a 32nd at a time
      for (int span = a.n_seq <= 32 ? 32 : a.n_seq <= 1024 ? 1024 : 32768; span > 1; span >>= 5) {
        const int at = lo + lane * (span >> 5);
        lo += (__popc(__ballot_sync(0xFFFFFFFFu, at < a.n_seq && first[at] <= u)) - 1) * (span >> 5);
      }
      const Tree x = tree_of(lo);
      const int tiles = a.by_rpt.of(x.rows + a.rpt - 1), pages = (x.keys + kTrKeys - 1) / kTrKeys, nu = tile_cost(x.keys);
      const int k = (int)((unsigned)(u - first[lo]) / (unsigned)nu), u0 = first[lo] + k * nu;
      p.kvh = (int)((unsigned)k / (unsigned)tiles);
      const int tile = k - p.kvh * tiles;
      p.row0 = x.row0 + tile * a.rpt;
      p.n_i = min(a.rpt, x.rows - tile * a.rpt) * a.G;
      p.keys = x.keys; p.committed = x.committed; p.nodes = x.nodes; p.stream = x.stream;
      p.next = u0 + nu;
      // pages before the border of CTAs c - 1 and c (a border near an end of the tile is not moved there: a page 66.0 us, none 64.6, in 128 trees of 25 nodes)
      auto border = [&](int c) { return min(max(c * (int)size.d - u0 - kTrCostTile, 0), pages); };
      const int ca = size.of(u0), cb = size.of(u0 + nu - 1), me = blockIdx.x;
      p.j0 = me == ca ? 0 : border(me);
      p.j1 = me == cb ? pages : border(me + 1);
      if (p.j1 > p.j0) {
        for (p.c0 = ca; p.c0 < cb && border(p.c0 + 1) == 0;) ++p.c0;
        for (p.c1 = cb; p.c1 > ca && border(p.c1) == pages;) --p.c1;
        return true;
      }
      if (pages == 0 && me == ca) {
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

  auto widen = [&]() {
    // ---- codes to bf16, 16 of a row at a time, by one half of these warps those of K (and the scales), by the other those of V, as soon as the products
    //      are done with the page two before ----
    constexpr int kWarps = E4M3 ? Shape::kWidenWarps / 2 : 1, kThreads = 32 * kWarps, kIter = 4 * kTrKeys / kThreads;   // 16 codes a thread and turn
    const int w = (warp - Shape::kWidenWarp) / kWarps, t = (tid - 32 * Shape::kWidenWarp) % kThreads, quad = t & 3;
    int word, c = 0;
    bool fine = true;
#pragma unroll 1
    for (int n_part = 0; fine && take_part(n_part, word); ++n_part) {
      const int steps = TR_FIELD(word, j1) - TR_FIELD(word, j0);
#pragma unroll 1
      for (int b = 0; b < steps; ++b, ++c) {
        const int s = c & 1;
        const unsigned char *from = raw + (c & 3) * Shape::kRawPage + w * kE4m3BlockBytes;
        fine = wait_warp(&sh.raw_full[c & 3], (uint32_t)(c / 4) & 1u);
        if (c >= 2 && fine) fine = wait_warp(w ? &sh.o_full[(c - 2) & 3] : &sh.s_full[(c - 2) & 3], (uint32_t)((c - 2) / 4) & 1u);
        // sums of the tile before met in both places of V
        if (S > 1 && !QF32 && w == 1 && b < 2 && n_part > 0 && fine) fine = wait_warp(&sh.q_free[(n_part - 1) & 1], (uint32_t)((n_part - 1) / 2) & 1u);
        if (!fine) break;
        if (w == 0) {                          // K's and V's; a V scale that is not finite is put into the score, since 0 * NaN must not reach rows that do not see its key
#pragma unroll
          for (int x = t; x < kTrKeys; x += kThreads) {
            const float ks = *reinterpret_cast<const float *>(from + kPageElems + 4 * x), vs = *reinterpret_cast<const float *>(from + kE4m3BlockBytes + kPageElems + 4 * x);
            const bool sound = fabsf(vs) < INFINITY;
            scales[(c % kTrScales) * 2 * kTrKeys + x] = sound ? ks : __int_as_float(0x7FFFFFFF);
            scales[(c % kTrScales) * 2 * kTrKeys + kTrKeys + x] = sound ? vs : 0.f;
          }
        }
        unsigned char *dst = (w ? Vs : Ks) + s * kTrPage;
#pragma unroll 1
        for (int k0 = 0; k0 < kIter; k0 += 4) {
          uint4 code[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) code[k] = *reinterpret_cast<const uint4 *>(from + ((t >> 2) + kThreads / 4 * (k0 + k)) * kHeadDim + 16 * quad);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = (t >> 2) + kThreads / 4 * (k0 + k);
            const uint32_t x[4] = {code[k].x, code[k].y, code[k].z, code[k].w};
            uint32_t y[8];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              y[2 * e] = e4m3x2_to_bf16x2(__byte_perm(x[e], 0u, 0x1404));
              y[2 * e + 1] = e4m3x2_to_bf16x2(__byte_perm(x[e], 0u, 0x3424));
            }
            *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad) ^ (r & 7)) << 4)) = make_uint4(y[0], y[1], y[2], y[3]);
            *reinterpret_cast<uint4 *>(dst + r * 128 + (((2 * quad + 1) ^ (r & 7)) << 4)) = make_uint4(y[4], y[5], y[6], y[7]);
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          mbar_arrive(w ? &sh.v_full[s] : &sh.k_full[s]);
          mbar_arrive(&sh.raw_empty[c & 3]);
        }
      }
    }
  };

  if (warp >= 4 && (!E4M3 || warp < 8)) {
    if constexpr (E4M3) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsCopy));
    if constexpr (E4M3 && S == 1)
      if (warp >= Shape::kWidenWarp) widen();
    // The tickets of the first tile, c0 its first CTA, where it began before the CTA's range.  Not the softmax warps' work: the fence takes microseconds
    // while copies are under way (16 trees of up to 32 nodes 28.0 us with it on them, 26.6 so).
    auto tickets = [&](int c0) {
      if (!wait_warp(&sh.written, 0)) return false;
      fence_gpu();
      if (lane < 4) sh.came[lane] = (int)atomicAdd(a.tickets + 4 * c0 + lane, 1u) + 1;
      fence_gpu();
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.came_full);
      return true;
    };
    if (Shape::kTicketWarp && warp == 6) {
      int word;
#pragma unroll 1
      for (int n_part = 0; take_part(n_part, word); ++n_part) {
        const int c0 = TR_FIELD(word, c0);
        if (n_part == 0 && c0 != (int)blockIdx.x && !tickets(c0)) break;
      }
    }
    if (warp == Shape::kCopyWarp) {
    // ---- copies: 16-bit queries of a tile as often as its rows stand among the lanes, two tiles ahead at most, then its keys and values ----
    int c = 0;                                 // pages of this CTA
    bool fine = true;
    TreePart p;
    int u = u_begin;
    int due = -1;                              // first CTA of the first tile, where its tickets are to be taken here
#pragma unroll 1
    for (int n_part = 0; fine; ++n_part) {
      const bool there = part_at(u, p);
      if (!there) p.n_i = 0;                   // the part behind the last has no rows
      fine = give_part(n_part, p) && there;
      if (!fine) break;
      u = p.next;
      if (!Shape::kTicketWarp && n_part == 0 && p.c0 != (int)blockIdx.x) due = p.c0;
      int mine = page_of(p.stream, p.keys, p.j0 + lane);   // a page each lane
      if constexpr (!QF32) {
        const int qb = n_part & 1;
        if (n_part >= 2) fine = wait_warp(&sh.q_free[qb], (uint32_t)(n_part / 2 - 1) & 1u);
        if (!fine) break;
        if (elect_one()) {
          mbar_expect_tx(&sh.q_full[qb], (uint32_t)(S * a.rpt * a.G * 128));
#pragma unroll
          for (int x = 0; x < S; ++x) un_box(&q_map, p.kvh * a.G, p.row0, Qs + qb * kTrRows + x * (kTrRows / S), &sh.q_full[qb]);
        }
        __syncwarp();
      }
#pragma unroll 1
      for (int j = p.j0; j < p.j1 && fine; ++j, ++c) {
        const int at = (j - p.j0) & 31, s = c & 3;
        if (at == 0 && j > p.j0) mine = page_of(p.stream, p.keys, j + lane);
        const int page = __shfl_sync(0xFFFFFFFFu, mine, at);
        if (c >= 4) fine = wait_warp(E4M3 ? &sh.raw_empty[s] : &sh.s_full[s], (uint32_t)(c / 4 - 1) & 1u);
        if (!fine) break;
        if (lane == 0) sh.there[c % kTrThere] = page >= 0;
        __syncwarp();
        if constexpr (E4M3) {
          if (elect_one()) {
            mbar_expect_tx(&sh.raw_full[s], page >= 0 ? 2 * kE4m3BlockBytes : 0);
            if (page >= 0) {
              const unsigned char *from = a.pool + ((size_t)page * 2 * a.Hkv + p.kvh) * kE4m3BlockBytes;
              bulk_copy_g2s(raw + s * Shape::kRawPage, from, kE4m3BlockBytes, &sh.raw_full[s]);
              bulk_copy_g2s(raw + s * Shape::kRawPage + kE4m3BlockBytes, from + (size_t)a.Hkv * kE4m3BlockBytes, kE4m3BlockBytes, &sh.raw_full[s]);
            }
          }
        } else {
          if (elect_one()) {
            mbar_expect_tx(&sh.k_full[s], page >= 0 ? kTrPage : 0);
            if (page >= 0) un_box(&kv_map, 0, page * 2 * a.Hkv + p.kvh, Ks + s * kTrPage, &sh.k_full[s]);
          }
          __syncwarp();
          if (c >= 4) fine = wait_warp(&sh.o_full[s], (uint32_t)(c / 4 - 1) & 1u);
          if (S > 1 && !QF32) {
            const int tile = tree_tile_in_place(n_part, j - p.j0);
            if (tile >= 0 && fine) fine = wait_warp(&sh.q_free[tile & 1], (uint32_t)(tile / 2) & 1u);
          }
          if (!fine) break;
          if (elect_one()) {
            mbar_expect_tx(&sh.v_full[s], page >= 0 ? kTrPage : 0);
            if (page >= 0) un_box(&kv_map, 0, (page * 2 + 1) * a.Hkv + p.kvh, Vs + s * kTrPage, &sh.v_full[s]);
          }
        }
        __syncwarp();
        if (due >= 0 && mbar_test_warp(&sh.written, 0)) { fine = tickets(due) && fine; due = -1; }
      }
    }
    if (due >= 0) tickets(due);
    } else if (warp == Shape::kMmaWarp) {
    // ---- products: each time the softmax has step c's weights in tensor memory (and its scores in registers), P V of step c and Q K^T of step c + 2,
    //      over the borders of tiles too.  Scores and weights have two places, by turns ----
    const uint32_t idesc_qk = tc_instr_desc(128, kTrKeys), idesc_pv = tc_instr_desc(128, kHeadDim) | (1u << 16);   // V is MN-major
    const uint64_t dqs = tc_smem_desc(Qs), dks = tc_smem_desc(Ks), dvs = tc_smem_desc(Vs);
    int n_part = 0, left = 0, c_qk = 0, word;  // parts, steps of the last of them that are still to be asked for, steps that were
    bool fine = true, more = true;
    unsigned first_bits = 0;                   // bit c % 32: step c is the first of its tile
    auto scores = [&]() {                      // of the next step, if there is one
      if (more && left == 0) {
        more = take_part(n_part, word);
        if (more) {
          left = TR_FIELD(word, j1) - TR_FIELD(word, j0);
          fine = wait_warp(&sh.q_full[QF32 ? 0 : n_part & 1], (uint32_t)(QF32 ? n_part : n_part / 2) & 1u);
          first_bits |= 1u << (c_qk & 31);
          ++n_part;
        }
      }
      if (!more || !fine) return;
      fine = wait_warp(&sh.k_full[c_qk % kRing], (uint32_t)(c_qk / kRing) & 1u);
      if (!fine) return;
      tc_fence_after_sync();
      if (elect_one()) {
        const uint64_t dk = dks + (uint64_t)(c_qk % kRing) * (kTrPage >> 4), dq = dqs + (uint64_t)(QF32 ? 0 : (n_part - 1) & 1) * (kTrRows >> 4);
#pragma unroll
        for (int q = 0; q < (QF32 ? 8 : 4); ++q)
          tc_mma(tmem + 64u * (c_qk & 1), dq + (uint64_t)(q >> 2) * (kTrRows >> 4) + 2 * (q & 3), dk + 2 * (q & 3), idesc_qk, q == 0 ? 0u : 1u);
        tc_commit(&sh.s_full[c_qk & 3]);
      }
      __syncwarp();
      ++c_qk; --left;
    };
    // (fp32 queries have one place: a tile's are written when the one before has left, so that nothing is asked for across that border before)
#pragma unroll 1
    for (int k = 0; k < 2; ++k)
      if (fine && (!QF32 || k == 0 || left > 0)) scores();
#pragma unroll 1
    for (int c = 0; fine && c < c_qk; ++c) {
      fine = wait_warp(&sh.p_full[c & 1], (uint32_t)(c / 2) & 1u) && wait_warp(&sh.v_full[c % kRing], (uint32_t)(c / kRing) & 1u);
      if (!fine) break;
      tc_fence_after_sync();
      if (elect_one()) {
        const uint64_t dv = dvs + (uint64_t)(c % kRing) * (kTrPage >> 4);
        const bool opens = first_bits >> (c & 31) & 1u;
#pragma unroll
        for (int q = 0; q < kTrKeys / 16; ++q)   // 16 keys an instruction: 8 columns of P, two groups of 8 rows of V
          tc_mma_ts(tmem + 192u, tmem + 128u + 32u * (c & 1) + 8u * q, dv + 128 * q, idesc_pv, opens && q == 0 ? 0u : 1u);
        tc_commit(&sh.o_full[c & 3]);
      }
      __syncwarp();
      first_bits &= ~(1u << (c & 31));
      if (!QF32 || left > 0) scores();
      else if (c + 1 == c_qk) { scores(); if (fine && left > 0) scores(); }
    }
    }
  } else if (E4M3 && S > 1 && warp >= Shape::kWidenWarp) {
    if constexpr (E4M3 && S > 1) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Shape::kRegsWiden));
    widen();
  } else {
    if constexpr (E4M3) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Shape::kRegsSoftmax));
    // ---- softmax ----
    constexpr int kChunks = kRgs;              // 16 values each, that a thread finishes of its row
    const int rg = warp % kRgs, rep = warp / kRgs, i_row = 32 * rg + lane, col0 = rep * kCols;   // which 32 rows of the tile and which copy of them; the row, its first key of a step
    const uint32_t t_lane = tmem + ((uint32_t)(32 * warp) << 16);
    int n_meet = 0, c = 0, n_tile = 0, word;                 // waits for meet, steps, tiles
    bool fine = true;
    // Of the tile that began before the CTA's range, and of the last one where it goes on behind it: is there a part in scratch, and how many CTAs had a ticket
    // when this one took its own?
    bool due0 = false, due1 = false;
    int came0 = 0, came1 = 0;
    TreePart &p = sh.mine[warp];
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
    // A tile that several CTAs share has a place in each: by warp, its values' columns of four for 32 rows, then reference and sum.  A CTA has
    // two places: for the tile that began before its range, and the one that goes on behind it.
    auto place = [&](int cta, int c0) { return a.part + (size_t)(2 * cta + (cta == c0)) * 128 * kTrPitch; };
    auto at_values = [&](int x) { return (warp * kChunks + x) * 4 * 128 + lane * 4; };   // of 16 values x of the thread's row
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
      uint4 *dst = reinterpret_cast<uint4 *>(a.out + ((size_t)(p.row0 + r) * a.H + (p.kvh - r) * a.G + i_row) * kHeadDim + 16 * (rep * kChunks + x));
#pragma unroll
      for (int e = 0; e < 2; ++e)
        dst[e] = make_uint4(pack_bf16x2(o[8 * e] * inv, o[8 * e + 1] * inv), pack_bf16x2(o[8 * e + 2] * inv, o[8 * e + 3] * inv),
                            pack_bf16x2(o[8 * e + 4] * inv, o[8 * e + 5] * inv), pack_bf16x2(o[8 * e + 6] * inv, o[8 * e + 7] * inv));
    };
#pragma unroll 1
    for (int n_part = 0; fine && take_part(n_part, word); ++n_part, ++n_tile) {
      if (lane < kTrPartWords) reinterpret_cast<int *>(&p)[lane] = word;
      __syncwarp();
      const int j0 = p.j0, steps = p.j1 - j0;
      const bool mine = i_row < p.n_i, live = 32 * rg < p.n_i;   // the thread's row exists, some row of the warp does
      float m = -INFINITY, l = 0.f;
      if constexpr (QF32) {                    // the tile's queries, 16 rows a turn and 8 values a thread, as often as they stand among the lanes
        constexpr int kTileRows = 128 / S, kTurns = kTileRows / 16;
        // Turns whose loads are under way together, as many as registers allow (us, tiles of 128, 64 rows, bf16: 8 59.7, -; 4 55.1, 35.5; 2 59.3, 38.2; 8-bit: 8 69.6, -; 4
        // 74.4, 60.2; 2 74.1, 54.6).
        constexpr int kAhead = !E4M3 ? (kTurns < 4 ? kTurns : 4) : S == 1 ? kTurns : 2;
        const int e8 = tid & 7;
#pragma unroll 1
        for (int y0 = 0; y0 < kTurns; y0 += kAhead) {
          float x[kAhead][8];
#pragma unroll
          for (int y = 0; y < kAhead; ++y) {
            const int i = (tid >> 3) + 16 * (y0 + y), r = a.by_G.of(i);
#pragma unroll
            for (int e = 0; e < 8; ++e) x[y][e] = 0.f;
            if (i < p.n_i) load8(reinterpret_cast<const float *>(a.q) + (size_t)(p.row0 + r) * a.q_stride + (size_t)((p.kvh - r) * a.G + i) * kHeadDim + 8 * e8, x[y]);
          }
#pragma unroll
          for (int y = 0; y < kAhead; ++y) {
            const int i = (tid >> 3) + 16 * (y0 + y);
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const float f0 = __uint_as_float(__float_as_uint(x[y][2 * e]) & 0xFFFF0000u), f1 = __uint_as_float(__float_as_uint(x[y][2 * e + 1]) & 0xFFFF0000u);
              hi[e] = pack_bf16x2(f0, f1);
              lo[e] = pack_bf16x2(x[y][2 * e] - f0, x[y][2 * e + 1] - f1);
            }
#pragma unroll
            for (int z = 0; z < S; ++z) {
              const int to = (i + z * kTileRows) * 128 + ((e8 ^ (i & 7)) << 4);
              *reinterpret_cast<uint4 *>(Qs + to) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
              *reinterpret_cast<uint4 *>(Qs + kTrRows + to) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
          }
        }
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_full[0]);
      }
      const int *row_mask = a.mask + (size_t)(p.row0 + a.by_G.of(min(i_row, p.n_i - 1))) * a.words;
      const unsigned mask0 = (unsigned)row_mask[0], mask1 = a.words > 1 ? (unsigned)row_mask[1] : 0u;   // asked for here, wanted where drafted keys begin
#pragma unroll 1
      for (int b = 0; b < steps; ++b, ++c) {
        const int key0 = (j0 + b) * kTrKeys, n = min(kTrKeys, p.keys - key0), committed = p.committed, turn = c & 1;
        fine = wait_warp(&sh.s_full[c & 3], (uint32_t)(c / 4) & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        float s[kCols];
        if (live) {
          const uint32_t from = t_lane + 64u * turn + col0;
          if constexpr (kCols == 16) tmem_ld16(from, s);
          else {
#pragma unroll
            for (int e = 0; e < kCols; e += 32) tmem_ld32_async(from + (uint32_t)e, s + e);
            tmem_wait_ld();
#pragma unroll
            for (int e = 0; e < kCols; e += 32) tmem_landed32(s + e);
          }
        }
        const bool there = *reinterpret_cast<volatile int *>(&sh.there[c % kTrThere]) != 0, drafted = key0 + kTrKeys > committed;
        const bool special = drafted || n < kTrKeys || !there;
        const float *ks = scales + (c % kTrScales) * 2 * kTrKeys + col0, *vs = ks + kTrKeys;   // 8-bit cache: of K and V
        auto visible = [&](int k0) {           // bits of keys k0 .. k0 + 31 of the step that the row sees
          const int nodes = p.nodes;
          auto bits = [&](int w) {
            if (w >= a.words || 32 * w >= nodes) return 0u;
            const unsigned v = w == 0 ? mask0 : w == 1 ? mask1 : (unsigned)row_mask[w];
            return nodes - 32 * w < 32 ? v & ((1u << (nodes - 32 * w)) - 1u) : v;
          };
          const int d = key0 + k0 - committed; // number of the first of these keys among the drafted
          unsigned v = ~0u;
          if (d >= 0) v = __funnelshift_r(bits(d >> 5), d & 31 ? bits((d >> 5) + 1) : 0u, d & 31);
          else if (d > -32) v = (bits(0) << -d) | ((1u << -d) - 1u);
          const int left = there ? n - k0 : 0;
          return left <= 0 ? 0u : left < 32 ? v & ((1u << left) - 1u) : v;
        };
        if (live) {
          if constexpr (E4M3) {
#pragma unroll
            for (int e = 0; e < kCols; e += 4) {
              const ulonglong2 f = *reinterpret_cast<const ulonglong2 *>(ks + e);
              unpack_f32x2(mul_f32x2(pack_f32x2(s[e], s[e + 1]), f.x), s[e], s[e + 1]);
              unpack_f32x2(mul_f32x2(pack_f32x2(s[e + 2], s[e + 3]), f.y), s[e + 2], s[e + 3]);
            }
          }
          if (special) {
#pragma unroll
            for (int x = 0; x < (kCols > 32 ? 2 : 1); ++x) {
              const unsigned seen = visible(col0 + 32 * x);
#pragma unroll
              for (int e = 0; e < (kCols < 32 ? kCols : 32); ++e) s[32 * x + e] = seen >> e & 1u ? s[32 * x + e] : -INFINITY;
            }
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY}, sc = 1.f;
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
          unsigned long long sum2[2] = {0ull, 0ull};
          float w[kCols / 2];                          // weights, two to a column
#pragma unroll
          for (int e = 0; e < kCols; e += 2) {
            float y, z;
            unpack_f32x2(fma_f32x2(pack_f32x2(s[e], s[e + 1]), scale2, ref2), y, z);
            y = pt_exp2(y); z = pt_exp2(z);
            sum2[(e >> 1) & 1] = add_f32x2(sum2[(e >> 1) & 1], pack_f32x2(y, z));
            if constexpr (E4M3) {
              const ulonglong2 f = *reinterpret_cast<const ulonglong2 *>(vs + (e & ~3));
              unpack_f32x2(mul_f32x2(pack_f32x2(y, z), e & 2 ? f.y : f.x), y, z);
            }
            w[e >> 1] = __uint_as_float(pack_bf16x2(y, z));
          }
          float s0, s1;
          unpack_f32x2(add_f32x2(sum2[0], sum2[1]), s0, s1);
          l = fmaf(l, sc, s0 + s1);
          // This place of P is free: the product of the step before last was issued ahead of this step's scores, by the same thread, whose commit counts all before it (a
          // wait for it costs 3 %).  O holds still when the last step's product is done.
          if (b > 0 && __any_sync(0xFFFFFFFFu, sc != 1.f)) {
            fine = wait_warp(&sh.o_full[(c - 1) & 3], (uint32_t)((c - 1) / 4) & 1u);
            if (!fine) break;
            tc_fence_after_sync();
#pragma unroll 1
            for (int d = 0; d < kHeadDim; d += 16) {
              float keep[16];
              tmem_ld16(t_lane + 192u + (uint32_t)d, keep);
#pragma unroll
              for (int e = 0; e < 16; ++e) keep[e] *= sc;
              tmem_st16_async(t_lane + 192u + (uint32_t)d, keep);
            }
          }
          const uint32_t to = t_lane + 128u + 32u * turn + col0 / 2;
          if constexpr (kCols == 64) tmem_st32_async(to, w);
          else if constexpr (kCols == 32) tmem_st16_async(to, w);
          else tmem_st8_async(to, w);
          tmem_wait_st();
        }
        if constexpr (!E4M3) {
          if (special) {
            // V rows without a key hold anything, and so may those of drafted tokens that no row sees (a tree padded to a size): 0 * NaN
            // must not reach O.  They become zero, and rows that do see one that is not finite NaN.
            if (!wait_warp(&sh.v_full[c % kRing], (uint32_t)(c / kRing) & 1u)) { fine = false; break; }
            unsigned char *v = Vs + (c % kRing) * kTrPage + (tid >> 3) * 128 + (tid & 7) * 16;   // every 16th row, from the thread's on
            uint4 y[4];
#pragma unroll
            for (int x = 0; x < 4; ++x) y[x] = *reinterpret_cast<const uint4 *>(v + x * 2048);
#pragma unroll
            for (int x = 0; x < 4; ++x) {
              const int k = (tid >> 3) + 16 * x, d = key0 + k - committed;
              auto odd = [](uint32_t z) { return (z & 0x7F807F80u) + 0x00800080u; };   // bits 15 and 31: an exponent of ones
              const bool none = k >= n || !there, bad = ((odd(y[x].x) | odd(y[x].y) | odd(y[x].z) | odd(y[x].w)) & 0x80008000u) != 0 && d >= 0;
              if (none || bad) *reinterpret_cast<uint4 *>(v + x * 2048) = make_uint4(0, 0, 0, 0);
              if (bad && !none && d < kTrNodes) { atomicOr(&sh.bad[d >> 5], 1u << (d & 31)); *reinterpret_cast<volatile int *>(&sh.found) = n_tile + 1; }
            }
            fence_proxy_async_smem();
          }
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[turn]);
      }
      if (!fine) break;
      // ---- the tile's sums ----
      fine = wait_warp(&sh.o_full[(c - 1) & 3], (uint32_t)((c - 1) / 4) & 1u);
      if (!fine) break;
      tc_fence_after_sync();
      if (!E4M3 && *reinterpret_cast<volatile int *>(&sh.found) == n_tile + 1) {   // rare: rows that see a V that is not finite
        for (int w = 0; w < a.words && 32 * w < p.nodes; ++w)
          if ((unsigned)row_mask[w] & (p.nodes - 32 * w < 32 ? (1u << (p.nodes - 32 * w)) - 1u : ~0u) & *reinterpret_cast<volatile unsigned *>(&sh.bad[w])) l = __int_as_float(0x7FFFFFFF);
        fine = meet();
        if (tid < kTrNodes / 32) sh.bad[tid] = 0u;
        fine = meet() && fine;                 // before those of the next tile
        if (!fine) break;
      }
      float met[16];                           // where a row stands several times: its sums, or a half or a quarter of them at a time
      // Copies of a row meet where the tile's queries and (16-bit ones) the values of the last two steps were, which no product reads any more: half of a
      // row's values each.
      auto stage = [&](int h, int w) -> float4 * {   // of warp w's rows, half h
        if (h == 0) return reinterpret_cast<float4 *>(Qs + (QF32 ? 0 : (n_tile & 1) * kTrRows)) + w * 256;
        if (QF32) return reinterpret_cast<float4 *>(Qs + kTrRows) + w * 256;
        return reinterpret_cast<float4 *>(Vs + ((c - 1 - (w >> 1)) & (kRing - 1)) * kTrPage) + (w & 1) * 256;
      };
      if (S > 1 && live) sh.ml[warp][lane] = make_float2(m, l);
      float mine_f[S];                         // what each copy's sums are multiplied by
      const int c0 = p.c0, c1 = p.c1;
      const bool begins = c0 == (int)blockIdx.x;
      bool whole = c0 == c1, others = false;   // others: their parts are there
      unsigned *ticket = a.tickets + 4 * c0 + warp;   // for the warp's 32 rows
      if (begins && !whole) {                  // the CTA's last tile; as a rule the others have long had their tickets
        unsigned came = 0;
        if (lane == 0) asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(came) : "l"(ticket) : "memory");
        others = __shfl_sync(0xFFFFFFFFu, came, 0) == (unsigned)(c1 - c0);
        whole = others;
        __syncwarp();                          // what lane 0 has acquired the others see
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
      if constexpr (S == 1) {
#pragma unroll 1
        for (int x = 0; x < 4; ++x) {
          if (live) tmem_ld16(t_lane + 192u + 16u * x, met);
          pass_on(x, met);
        }
      } else {
        if (live) {
#pragma unroll 1
          for (int h = 0; h < 2; ++h) {
            float x[32];
            tmem_ld32(t_lane + 192u + 32u * h, x);
            float4 *to4 = stage(h, warp);
#pragma unroll
            for (int e = 0; e < 32; e += 4) to4[e / 4 * 32 + lane] = make_float4(x[e], x[e + 1], x[e + 2], x[e + 3]);
          }
        }
        fine = meet();
        if (!fine) break;
        if (live) {
          float M = -INFINITY, ly[S];
#pragma unroll
          for (int x = 0; x < S; ++x) {
            const float2 ml = sh.ml[rg + x * kRgs][lane];
            mine_f[x] = ml.x; ly[x] = ml.y;
            if (ml.y != 0.f) M = fmaxf(M, ml.x);
          }
          m = M; l = 0.f;
#pragma unroll
          for (int x = 0; x < S; ++x) {
            mine_f[x] = ly[x] == 0.f ? 0.f : pt_exp2(mine_f[x] - M);   // no key in it
            l = fmaf(ly[x], mine_f[x], l);
          }
#pragma unroll 1
          for (int x = 0; x < kChunks; ++x) {
            const int d16 = rep * kChunks + x; // which 16 values of the 64
#pragma unroll
            for (int e = 0; e < 16; ++e) met[e] = 0.f;
#pragma unroll
            for (int y = 0; y < S; ++y) {
              const float f = mine_f[y];
              const float4 *from4 = stage(d16 >> 1, rg + y * kRgs) + (d16 & 1) * 128 + lane;
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                const float4 v = from4[e * 32];
                met[4 * e] = fmaf(v.x, f, met[4 * e]); met[4 * e + 1] = fmaf(v.y, f, met[4 * e + 1]);
                met[4 * e + 2] = fmaf(v.z, f, met[4 * e + 2]); met[4 * e + 3] = fmaf(v.w, f, met[4 * e + 3]);
              }
            }
            pass_on(x, met);
          }
        }
        if constexpr (QF32) {                  // the next tile's queries are written there
          fine = meet();
          if (!fine) break;
        }
      }
      tc_fence_before_sync();                  // O may be overwritten once this thread's next P is announced
      if constexpr (!QF32) {                   // queries of the tile after next, and values of the next one, are written there
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_free[n_tile & 1]);
      }
      if (whole) {
        if (others && lane == 0) *ticket = 0u;
        continue;
      }
      if (mine) *reinterpret_cast<float2 *>(to + 128 * kHeadDim + 64 * warp + 2 * lane) = make_float2(m, l);
      (begins ? due1 : due0) = true;
      if (lane < kTrPartWords) reinterpret_cast<int *>(&sh.shared[begins][warp])[lane] = word;
      __syncwarp();
      if (!begins && lane == 0) mbar_arrive(&sh.written);
    }
    // ---- the tiles that other CTAs share, where this CTA came last: the one that began before its range, and its last ----
    if (fine && due1) {
      fence_gpu();
      __syncwarp();
      if (lane == 0) came1 = (int)atomicAdd(a.tickets + 4 * sh.shared[1][warp].c0 + warp, 1u) + 1;
    }
    if (fine && due0) {
      fine = wait_warp(&sh.came_full, 0);
      came0 = *reinterpret_cast<volatile int *>(&sh.came[warp]);
    }
#pragma unroll 1
    for (int which = 0; fine && which < 2; ++which) {
      const int n = __shfl_sync(0xFFFFFFFFu, which ? came1 : came0, 0);
      if (n == 0) continue;
      const TreePart &q = sh.shared[which][warp];
      if (n != q.c1 - q.c0 + 1) continue;
      if (lane == 0) a.tickets[4 * q.c0 + warp] = 0u;
      fence_gpu();
#pragma unroll 1
      for (int x = 0; x < kChunks; ++x) {
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

template <int S, bool E4M3, bool QF32>
inline cudaError_t launch_tree_as(const CUtensorMap &map, TreeAttnArgs a, int n_sm, cudaStream_t st) {
  using Shape = TreeShape<S, E4M3>;
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(attention_tree_kernel<S, E4M3, QF32>, tree_smem_bytes<S, E4M3>(kTrMaxSeq))) return e;
  if constexpr (E4M3) {               // the kernel splits the launch's registers anew: has a thread as many as the split counts on?
    static std::atomic<bool> enough{false};
    if (!enough.load(std::memory_order_acquire)) {
      cudaFuncAttributes at;
      if (const cudaError_t e = cudaFuncGetAttributes(&at, attention_tree_kernel<S, E4M3, QF32>)) return e;
      if ((at.numRegs + 7) / 8 * 8 < Shape::kRegsLaunch) return cudaErrorInvalidKernelImage;
      enough.store(true, std::memory_order_release);
    }
  }
  a.rpt = 128 / S / a.G;
  a.by_rpt.set((uint32_t)a.rpt);
  CUtensorMap q_map = {};
  if (!QF32)
    if (const cudaError_t e = tree_q_map(&q_map, a)) return e;
  return launch_kernel(attention_tree_kernel<S, E4M3, QF32>, dim3((unsigned)min(Shape::kCtas * n_sm, kTrMaxCtas)), dim3(Shape::kThreads), tree_smem_bytes<S, E4M3>(a.n_seq), st, true,
                       map, q_map, a);
}
template <bool E4M3, bool QF32>
inline cudaError_t launch_tree(const CUtensorMap &map, const TreeAttnArgs &a, int n_sm, cudaStream_t st) {
  const long long rows = (long long)a.t_max * a.G;
  return rows <= 32 ? launch_tree_as<4, E4M3, QF32>(map, a, n_sm, st) : rows <= 64 ? launch_tree_as<2, E4M3, QF32>(map, a, n_sm, st) : launch_tree_as<1, E4M3, QF32>(map, a, n_sm, st);
}

}  // namespace ttsgpt
