// Attention of query tiles of 256 rows over blocks of 128 keys on the 5th-generation tensor cores: cross attention where a
// sequence has more queries than a tile of the warp-level kernel (Section I: the decode engine's attention kernels).
//
// A tile is two halves of 128 (row, head of the group) pairs of one sequence and one head of keys; thread t of a half's four softmax
// warps owns its row t = accumulator lane t.  For each block of 128 keys, which both halves read from one copy in shared memory,
//     S = Q K^T     tcgen05.mma M=128 x N=128 x K=64, S (fp32) in tensor memory
//     softmax       S out of tensor memory, running reference m and sum l in fp32, P = 2^(S scale - m) rounded to the inputs' type
//                   back into tensor memory.  The reference moves, and O with it, only where a scaled score (log2 units) exceeds it by
//                   more than 8: weights stay at or below 2^8 and the rounding of a weight is relative, so nothing is lost
//     O += P V      M=128 x N=64 x K=128, P as the operand in tensor memory, V as stored
// S takes 128 columns, P 64 and O 64 of each half: all of an SM's tensor memory.  S of block j + 1 is computed while the softmax works on
// S of block j, which by then is in registers; one half's softmax runs beside the other's.
//
// Bound and measurements.  A block of 256 rows by 128 keys is 1024 tensor cycles, and 2048 cycles of exponentials at 16 a cycle and
// SM; a quarter of them goes through a polynomial on the FMA pipes (every 8th, 4th, 3rd, 2nd pair: 99, 94, 95, 107 us for 8 sequences
// of 517 to 1500 queries by 700 to 1500 keys, 20 heads, fp16; none: 99).  With the loads and stores of tensor memory and the maximum a
// block takes some 2500 cycles, a change of tile 4500.  Those sequences take 94.7 us, 0.52 PFLOP/s, the tensor pipe at 27 %, that of the
// exponentials at 38 %, 43 % of the issue slots; 1536 by 1536 take 145 us, 0.67 PFLOP/s.
// What came before: S only once P of the block before was there 102 us (3000 cycles a block, though no pipe had more than 2048 to do);
// 128 rows a CTA, two or four CTAs an SM, K and V out of L2 twice as often 131 us; two threads a row 134 us.
//
// Work split.  Tiles are laid end to end by what they cost (blocks of one half or two, a tile besides its blocks) and cut into equal
// ranges, one a CTA.  A part of a tile that several CTAs share goes to scratch with a ticket; the CTA that comes last adds the
// parts in the order of their keys, so that results do not depend on timing.  As a rule that is the CTA in which the tile begins, at
// the end of its range, with its own part, the first, still in registers.  Every wait on a copy or a product is bounded: two seconds.
#pragma once
#include "attention_units.cuh"

namespace ttsgpt {

constexpr int kTlRows = 128, kTlKeys = 128;   // rows of a half tile, keys of a block
constexpr int kTlTile = 2 * kTlRows;
constexpr int kTlThreads = 384;             // warps 0-3 and 4-7: softmax of a half, 8: copies, 9: products; 10 and 11 only give up their registers
// Registers of a thread: 168 at launch, of which the last four warps hand 96 each to the first eight, whose rows' 128 scores then
// stay in registers: 256 x 216 + 128 x 72 = 384 x 168.
constexpr int kTlRegsSoftmax = 216, kTlRegsOthers = 72;
constexpr int kTlHalf = kTlKeys * 128;      // K or V of a block: 16 KB
constexpr int kTlBlock = 2 * kTlHalf;       // both
constexpr int kTlRing = 4;                  // places for blocks
constexpr int kTlQ = kTlTile * 128;         // Q of a tile: 32 KB
constexpr int kTlMaxSeq = 2048;
constexpr int kTlMaxCtas = kUnMaxCtas;
constexpr float kTlSlack = 8.0f;            // log2 by which a score may exceed the reference
// What a range is measured in, about 620 cycles each: a block of both halves, of one half alone, and a tile besides its blocks (for a tile
// 8 instead of 6: 30 sequences of 100 to 700 queries by 100 to 900 keys 93 instead of 95 us).
constexpr int kTlCost2 = 4, kTlCost1 = 3, kTlCostTile = 8;

// The part of a tile that lies in a CTA's range.
struct TilePart {
  int row0, n_i, kvh, u0, nu;     // first query row, rows times heads, head of keys; where the tile's cost begins, its cost
  int j0, j1, key0, keys;         // its blocks here; first key row and number of keys of the sequence
};
constexpr int kTlParts = 4;       // that the copying warp is ahead at most

struct TileShared {
  TilePart part[kTlParts];
  uint64_t part_full[kTlParts], part_free[kTlParts];
  uint64_t full[kTlRing], empty[kTlRing];   // blocks
  uint64_t q_full[2], q_free[2];
  uint64_t s_full[2], p_full[2], pv_done[2];   // by half
  uint32_t tmem;
  int failed;                     // 1: a wait of the CTA has run out; 2: one of an earlier call with the same scratch had
  TilePart meets;                 // the tile that began before the CTA's range
  Div size;
  int warp_tot[kTlThreads / 32];
};
inline size_t tiles_smem_bytes(int n) { return 1024 + (size_t)kTlRing * kTlBlock + 2 * kTlQ + sizeof(TileShared) + (size_t)(n + 1) * sizeof(int); }

// 32 lanes x 32 columns of 32 bits out of and into tensor memory, several of which are waited for at once
__device__ __forceinline__ void tmem_ld32_async(uint32_t taddr, float *v) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]), "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]),
        "=f"(v[13]), "=f"(v[14]), "=f"(v[15]), "=f"(v[16]), "=f"(v[17]), "=f"(v[18]), "=f"(v[19]), "=f"(v[20]), "=f"(v[21]), "=f"(v[22]), "=f"(v[23]), "=f"(v[24]),
        "=f"(v[25]), "=f"(v[26]), "=f"(v[27]), "=f"(v[28]), "=f"(v[29]), "=f"(v[30]), "=f"(v[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// no use of the registers moves ahead of this, which stands behind the wait
__device__ __forceinline__ void tmem_landed32(float *v) {
  asm volatile("" : "+f"(v[0]), "+f"(v[1]), "+f"(v[2]), "+f"(v[3]), "+f"(v[4]), "+f"(v[5]), "+f"(v[6]), "+f"(v[7]), "+f"(v[8]), "+f"(v[9]), "+f"(v[10]), "+f"(v[11]),
               "+f"(v[12]), "+f"(v[13]), "+f"(v[14]), "+f"(v[15]), "+f"(v[16]), "+f"(v[17]), "+f"(v[18]), "+f"(v[19]), "+f"(v[20]), "+f"(v[21]), "+f"(v[22]), "+f"(v[23]),
               "+f"(v[24]), "+f"(v[25]), "+f"(v[26]), "+f"(v[27]), "+f"(v[28]), "+f"(v[29]));
  asm volatile("" : "+f"(v[30]), "+f"(v[31]));
}
__device__ __forceinline__ void tmem_st32_async(uint32_t taddr, const float *v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};"
      ::"r"(taddr), "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]), "f"(v[10]), "f"(v[11]), "f"(v[12]),
        "f"(v[13]), "f"(v[14]), "f"(v[15]), "f"(v[16]), "f"(v[17]), "f"(v[18]), "f"(v[19]), "f"(v[20]), "f"(v[21]), "f"(v[22]), "f"(v[23]), "f"(v[24]), "f"(v[25]),
        "f"(v[26]), "f"(v[27]), "f"(v[28]), "f"(v[29]), "f"(v[30]), "f"(v[31]) : "memory");
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// 2^x of two values by additions and products: x = n + f with n the nearest integer and |f| <= 1/2, 2^f by the polynomial of degree 5 with
// the least relative error there (found by iterated least squares; 2.1e-07 with all roundings), times 2^n put together from its bits.  Zero below 2^-126;
// x <= 127; NaN stays NaN.
__device__ __forceinline__ unsigned long long poly_exp2(unsigned long long x2) {
  constexpr float kMagic = 12582912.0f;        // 1.5 * 2^23: the sum's last bits are n
  auto both = [](float v) { return pack_f32x2(v, v); };
  float x, y;
  unpack_f32x2(x2, x, y);
  x2 = pack_f32x2(max_nan(x, -127.0f), max_nan(y, -127.0f));
  const unsigned long long z2 = add_f32x2(x2, both(kMagic)), f2 = add_f32x2(x2, fma_f32x2(z2, both(-1.0f), both(kMagic)));
  unsigned long long p2 = fma_f32x2(f2, both(0.00132764608f), both(0.00967554096f));
  p2 = fma_f32x2(p2, f2, both(0.0555071346f));
  p2 = fma_f32x2(p2, f2, both(0.240221202f));
  p2 = fma_f32x2(p2, f2, both(0.693146944f));
  p2 = fma_f32x2(p2, f2, both(1.00000012f));
  unpack_f32x2(z2, x, y);
  return mul_f32x2(p2, pack_f32x2(__int_as_float((__float_as_int(x) << 23) + 0x3F800000), __int_as_float((__float_as_int(y) << 23) + 0x3F800000)));
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
// A in tensor memory (row = lane, two 16-bit values of consecutive k a column), B in shared memory
__device__ __forceinline__ void tc_mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, {%5, %5, %5, %5}, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(0u) : "memory");
}

template <bool F16>
__global__ void __launch_bounds__(kTlThreads, 1) attention_tiles_kernel(const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                                                                        const __grid_constant__ CUtensorMap v_map, const UnitArgs a) {
  extern __shared__ __align__(16) unsigned char tl_smem_raw[];
  unsigned char *base = tl_smem_raw + ((1024u - (smem_u32(tl_smem_raw) & 1023u)) & 1023u);
  unsigned char *ring = base, *Qs = base + kTlRing * kTlBlock;      // [2] 256 rows x 64 values, K-major, 128-byte swizzle
  TileShared &sh = *reinterpret_cast<TileShared *>(Qs + 2 * kTlQ);
  int *first = reinterpret_cast<int *>(&sh + 1);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  volatile int *failed = &sh.failed;

  if (tid == 0) {
    for (int i = 0; i < kTlRing; ++i) { mbar_init(&sh.full[i], (int)blockIdx.x == a.starve ? 2 : 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_free[i], kTlTile / 32); }
    for (int i = 0; i < kTlParts; ++i) { mbar_init(&sh.part_full[i], 1); mbar_init(&sh.part_free[i], 1 + kTlTile / 32); }
    for (int h = 0; h < 2; ++h) { mbar_init(&sh.s_full[h], 1); mbar_init(&sh.p_full[h], kTlRows / 32); mbar_init(&sh.pv_done[h], 1); }
    sh.failed = __ldcg(a.err) ? 2 : 0;
  }
  if (warp == 8) {
    if (lane < 3) asm volatile("prefetch.tensormap [%0];" ::"l"(lane == 0 ? &q_map : lane == 1 ? &k_map : &v_map) : "memory");
    __syncwarp();
  }
  if (warp == 9) tmem_alloc(&sh.tmem, 512);   // half h, from column 256 h on: S 128 columns, P 64, O 64
  // ---- running sums of blocks over the sequences ----
  auto q_span = [&](int i, int &b, int &e) {
    b = min(max(a.q_start[i], 0), a.q_rows);
    e = min(min(max(a.q_start[i + 1], b), a.q_rows), b + a.q_max);
  };
  auto k_span = [&](int i, int &b, int &e) {
    b = min(max(a.k_start[i], 0), a.k_rows);
    e = min(max(a.k_start[i + 1], b), a.k_rows);
  };
  // a head of a sequence: tiles, of which the last may have one half; cost of a tile, a block of the last one, and all of them
  struct SeqCost { int tiles, blocks, full, last_block, head; };
  auto seq_cost = [&](int q, int k) {
    SeqCost c;
    c.tiles = a.by_rpt.of(q + a.rpt - 1);
    c.blocks = (k + kTlKeys - 1) / kTlKeys;
    c.full = kTlCostTile + kTlCost2 * c.blocks;
    c.last_block = q - (c.tiles - 1) * a.rpt > (a.rpt >> 1) ? kTlCost2 : kTlCost1;
    c.head = c.tiles > 0 ? (c.tiles - 1) * c.full + kTlCostTile + c.last_block * c.blocks : 0;
    return c;
  };
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose blocks nothing bounds
  for (int i0 = 0; i0 < a.n_seq; i0 += kTlThreads) {
    const int i = i0 + tid;
    int u = 0;
    if (i < a.n_seq) {
      int qb, qe, kb, ke;
      q_span(i, qb, qe);
      k_span(i, kb, ke);
      bad |= a.q_start[i + 1] < a.q_start[i] || a.k_start[i + 1] < a.k_start[i];
      const SeqCost c = seq_cost(qe - qb, ke - kb);
      u = a.Hkv * c.head;
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
    for (int w = 0; w < kTlThreads / 32; ++w) { if (w < warp) before += sh.warp_tot[w]; all += sh.warp_tot[w]; }
    if (i < a.n_seq) first[i] = before + incl - u;
    carry = all;
  }
  const int T = bad ? 0 : carry;
  if (tid == 0) {
    first[a.n_seq] = T;
    sh.size.set(max(2 * kTlCost2, (T + (int)gridDim.x - 1) / (int)gridDim.x));
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const Div size = sh.size;
  const int u_begin = blockIdx.x * (int)size.d, u_end = *failed ? u_begin : min(T, u_begin + (int)size.d);

  // from unit u on
  auto part_at = [&](int u) {
    TilePart p;
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (first[m] <= u) lo = m; else hi = m - 1; }
    int qb, qe, kb, ke;
    q_span(lo, qb, qe);
    k_span(lo, kb, ke);
    const SeqCost c = seq_cost(qe - qb, ke - kb);
    p.key0 = kb; p.keys = ke - kb;
    p.kvh = (int)((unsigned)(u - first[lo]) / (unsigned)c.head);
    p.u0 = first[lo] + p.kvh * c.head;
    const int tile = min((int)((unsigned)(u - p.u0) / (unsigned)c.full), c.tiles - 1), block = tile + 1 < c.tiles ? kTlCost2 : c.last_block;
    p.u0 += tile * c.full;
    p.nu = kTlCostTile + block * c.blocks;
    p.row0 = qb + tile * a.rpt;
    p.n_i = min(a.rpt, qe - p.row0) * a.G;
    auto blocks_before = [&](int x) { return min((int)((unsigned)(max(x - p.u0 - kTlCostTile, 0) + block - 1) / (unsigned)block), c.blocks); };   // that begin before x
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
      if (t1 - t0 > kUnWaitNs) { *failed = 1; atomicExch(a.err, 1); return false; }
    }
    return true;
  };
  auto wait_warp = [&](uint64_t *bar, uint32_t parity) { return __all_sync(0xFFFFFFFFu, wait(bar, parity)) != 0; };
  // part number n as the copying warp has described it; the reader's warp has it in registers when it gives the place back
  auto take_part = [&](int n, TilePart &p) {
    const int k = n % kTlParts;
    if (!wait_warp(&sh.part_full[k], (uint32_t)(n / kTlParts) & 1u)) return false;
    p = sh.part[k];
    __syncwarp();
    if (lane == 0) mbar_arrive(&sh.part_free[k]);
    return true;
  };

  if (warp >= 8) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kTlRegsOthers));
    if (warp == 8) {
      // ---- copies: K and V blocks into the ring in turn, Q ahead of its first block ----
      int slot = 0, n_tile = 0, n_part = 0;      // blocks, tiles with blocks, and parts of this CTA
      for (int u = u_begin; u < u_end;) {
        const TilePart p = part_at(u);
        const int k = n_part % kTlParts;
        if (n_part >= kTlParts && !wait_warp(&sh.part_free[k], (uint32_t)(n_part / kTlParts - 1) & 1u)) break;
        if (lane == 0) { sh.part[k] = p; mbar_arrive(&sh.part_full[k]); }
        __syncwarp();
        ++n_part;
        u = p.u0 + p.nu;
        if (p.j1 <= p.j0) continue;
        const int qb = n_tile & 1;
        if (n_tile >= 2 && !wait_warp(&sh.q_free[qb], (uint32_t)(n_tile / 2 - 1) & 1u)) break;
        if (elect_one()) {
          const int rows = a.rpt >> 1;         // of a half
          mbar_expect_tx(&sh.q_full[qb], (uint32_t)(rows * a.G) * (p.n_i > rows * a.G ? 256 : 128));
          un_box(&q_map, p.kvh * a.G, p.row0, Qs + qb * kTlQ, &sh.q_full[qb]);
          if (p.n_i > rows * a.G) un_box(&q_map, p.kvh * a.G, p.row0 + rows, Qs + qb * kTlQ + kTlHalf, &sh.q_full[qb]);
        }
        __syncwarp();
        ++n_tile;
        bool fine = true;
        for (int j = p.j0; j < p.j1 && fine; ++j, ++slot) {
          const int s = slot % kTlRing;
          fine = slot < kTlRing || wait_warp(&sh.empty[s], (uint32_t)(slot / kTlRing - 1) & 1u);
          if (!fine) break;
          if (elect_one()) {
            mbar_expect_tx(&sh.full[s], kTlBlock);
            un_box(&k_map, p.key0 + j * kTlKeys, p.kvh, ring + s * kTlBlock, &sh.full[s]);
            un_box(&v_map, p.key0 + j * kTlKeys, p.kvh, ring + s * kTlBlock + kTlHalf, &sh.full[s]);
          }
          __syncwarp();
        }
        if (!fine) break;
      }
    } else if (warp == 9) {
      // ---- products: of either half in turn.  A half's turn k comes when its softmax has taken S of block k into registers and
      //      left P of block k - 1: then P V of block k - 1 and Q K^T of block k + 1 are issued, one wait and one commit for both (a wait
      //      and a commit for each product made seven waits of this warp a block: 106 us where 102 were) ----
      const uint32_t kind = F16 ? ~((1u << 7) | (1u << 10)) : ~0u;
      const uint32_t idesc_qk = tc_instr_desc(kTlRows, kTlKeys) & kind, idesc_pv = (tc_instr_desc(kTlRows, kHeadDim) & kind) | (1u << 16);   // V is MN-major
      int n_tile = 0, n_part = 0;                // tiles with blocks, and parts of this CTA
      bool fine = true;
      const uint64_t dring = tc_smem_desc(ring);
      uint32_t odd = 0, n_block = 0;             // bit h: half h has had an odd number of turns; blocks of the CTA
      for (int u = u_begin; u < u_end && fine;) {
        TilePart p;
        fine = take_part(n_part++, p);
        if (!fine) break;
        u = p.u0 + p.nu;
        if (p.j1 <= p.j0) continue;
        const int qb = n_tile & 1, halves = p.n_i > (a.rpt >> 1) * a.G ? 2 : 1;
        fine = wait_warp(&sh.q_full[qb], (uint32_t)(n_tile / 2) & 1u);
        ++n_tile;
        const uint64_t dq = tc_smem_desc(Qs + qb * kTlQ);
        const int nb = p.j1 - p.j0;
#pragma unroll 1
        for (int k = -1; k <= nb && fine; ++k) {   // turn k: P V of block k - 1 and Q K^T of block k + 1
          const uint32_t s_qk = (n_block + k + 1) % kTlRing, s_pv = (n_block + k - 1) % kTlRing;
          if (k + 1 < nb) fine = wait_warp(&sh.full[s_qk], (n_block + k + 1) / kTlRing & 1u);
          const uint64_t dk = dring + (uint64_t)((s_qk * kTlBlock) >> 4), dv = dring + (uint64_t)((s_pv * kTlBlock + kTlHalf) >> 4);
#pragma unroll 1
          for (int h = 0; h < halves && fine; ++h) {
            if (k >= 0) {
              fine = wait_warp(&sh.p_full[h], odd >> h & 1u);
              odd ^= 1u << h;
              if (!fine) break;
              tc_fence_after_sync();
            }
            const uint32_t t = tmem + 256u * h;
            if (elect_one()) {
              if (k >= 1) {
#pragma unroll
                for (int q = 0; q < kTlKeys / 16; ++q)   // 16 keys an instruction: 8 columns of P, two groups of 8 rows of V
                  tc_mma_ts(t + 192u, t + 128u + 8u * q, dv + 128 * q, idesc_pv, k == 1 && q == 0 ? 0u : 1u);
                if (h + 1 == halves) tc_commit(&sh.empty[s_pv]);   // no other half reads that block any more
              }
              if (k + 1 < nb) {
#pragma unroll
                for (int q = 0; q < 4; ++q) tc_mma(t, dq + (uint64_t)(h * (kTlHalf >> 4) + 2 * q), dk + 2 * q, idesc_qk, q == 0 ? 0u : 1u);
              }
              tc_commit(k < nb ? &sh.s_full[h] : &sh.pv_done[h]);
            }
            __syncwarp();
          }
        }
        n_block += nb;
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTlRegsSoftmax));
    // ---- softmax ----
    const int half = warp >> 2, quarter = warp & 3, t = tid & (kTlRows - 1);   // the thread's row of the half
    const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16) + 256u * half;
    int i = 0, n_o = 0, n_block = 0, n_tile = 0, n_part = 0;   // waits of this half for s_full and for pv_done, blocks of the CTA, tiles with blocks, parts
    bool fine = true;
    int came_first = 0;                        // how many had a ticket of the tile that began before the CTA's range, this CTA among them
    // A tile that several CTAs share has a place in each: 256 rows, 16 columns of four dimensions, then reference and sum.  A CTA has two
    // places: for the tile that began before its range, and the one that goes on behind it.
    auto part_at_place = [&](int c, int c0) { return a.part + (size_t)(2 * c + (c == c0)) * kTlTile * kUnPitch; };
    auto add_parts = [&](int c0, int c, int c1, float (&o)[kHeadDim], float &m, float &l) {   // those of CTAs c .. c1, in the order of their keys
#pragma unroll 1
      for (; c <= c1; ++c) {
        const float *x = part_at_place(c, c0);
        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(x + kTlTile * kHeadDim + 2 * tid));
        float4 v[kHeadDim / 4];
#pragma unroll
        for (int e = 0; e < kHeadDim / 4; ++e) v[e] = __ldcg(reinterpret_cast<const float4 *>(x + (e * kTlTile + tid) * 4));
        const bool has = ml.y != 0.f;          // a key in it
        const float mn = fmaxf(m, ml.x), fk = !has || m == mn ? 1.f : pt_exp2(m - mn), fn = has ? pt_exp2(ml.x - mn) : 0.f;
        if (has) m = mn;
        l = fmaf(l, fk, ml.y * fn);
#pragma unroll
        for (int e = 0; e < kHeadDim / 4; ++e) {
          o[4 * e] = fmaf(o[4 * e], fk, v[e].x * fn); o[4 * e + 1] = fmaf(o[4 * e + 1], fk, v[e].y * fn);
          o[4 * e + 2] = fmaf(o[4 * e + 2], fk, v[e].z * fn); o[4 * e + 3] = fmaf(o[4 * e + 3], fk, v[e].w * fn);
        }
      }
    };
    auto row_ptr = [&](const TilePart &p, int i2) {
      const int r = a.by_G.of(i2);
      return a.out + ((size_t)(p.row0 + half * (a.rpt >> 1) + r) * a.H + (p.kvh - r) * a.G + i2) * kHeadDim;
    };
    // the warp's rows, by way of shared memory: whole 128-byte rows
    auto leave = [&](const TilePart &p, int n_i, const float (&o)[kHeadDim], float l, unsigned char *stage) {
      const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
      for (int c = 0; c < kHeadDim; c += 8)
        *reinterpret_cast<uint4 *>(stage + t * 128 + (((c >> 3) ^ (t & 7)) << 4)) =
            make_uint4(un_pack<F16>(o[c] * inv, o[c + 1] * inv), un_pack<F16>(o[c + 2] * inv, o[c + 3] * inv),
                       un_pack<F16>(o[c + 4] * inv, o[c + 5] * inv), un_pack<F16>(o[c + 6] * inv, o[c + 7] * inv));
      __syncwarp();
#pragma unroll
      for (int it = 0; it < 8; ++it) {
        const int r = 32 * quarter + 4 * it + (lane >> 3), c8 = lane & 7;
        if (r < n_i) *reinterpret_cast<uint4 *>(row_ptr(p, r) + 8 * c8) = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((c8 ^ (r & 7)) << 4));
      }
    };
    for (int u = u_begin; u < u_end && fine;) {
      const int place_p = n_part % kTlParts;
      fine = wait_warp(&sh.part_full[place_p], (uint32_t)(n_part / kTlParts) & 1u);
      if (!fine) break;
      ++n_part;
      const TilePart &p = sh.part[place_p];    // stays there until the tile's rows have left: its registers would be spilled
      u = p.u0 + p.nu;
      const int n_half = (a.rpt >> 1) * a.G, n_i = min(p.n_i - half * n_half, n_half);   // rows of this half, none where not positive
      const bool live = 32 * quarter < n_i, mine = t < n_i;   // some row of the warp exists, the thread's own does
      const int j0 = p.j0, j1 = p.j1, keys = p.keys, blocks = n_i > 0 ? j1 : j0;
      if (n_i <= 0 && j1 > j0) {           // no such half here: no block holds it back, but it gives Q back below, once for each Q
        fine = wait_warp(&sh.q_full[n_tile & 1], (uint32_t)(n_tile / 2) & 1u);
        if (!fine) break;
      }
      float m = -INFINITY, l = 0.f;
      auto pass_turn = [&]() {                       // to the products
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[half]);
      };
      if (blocks > j0) {
        fine = wait_warp(&sh.s_full[half], (uint32_t)i++ & 1u);
        if (!fine) break;
        tc_fence_after_sync();
      }
      auto clear_v = [&](int j, int n) {       // the sequence's last block: V rows behind its keys may hold NaN, and 0 * NaN must not reach O
        // (both halves write the same zeros, each ahead of its own P V; S of the block is there, so its K and V are)
        unsigned char *v = ring + (n_block + j - j0) % kTlRing * kTlBlock + kTlHalf;
        for (int x = n * 8 + t; x < kTlKeys * 8; x += kTlRows) *reinterpret_cast<uint4 *>(v + x * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
      };
      if (!live) {                             // no row of this warp exists: it takes its turns
#pragma unroll 1
        for (int j = j0; j < blocks; ++j) {
          pass_turn();
          fine = wait_warp(&sh.s_full[half], (uint32_t)i++ & 1u);
          if (!fine) break;
          if (keys - j * kTlKeys < kTlKeys) clear_v(j, keys - j * kTlKeys);
        }
      } else {
#pragma unroll 1
        for (int j = j0; j < blocks; ++j) {
          const int n = min(kTlKeys, keys - j * kTlKeys);
          // all scores of the row into registers; the next block's may then come in their place
          float s[kTlKeys], sc = 1.f;
#pragma unroll
          for (int c = 0; c < kTlKeys; c += 32) tmem_ld32_async(t_lane + (uint32_t)c, s + c);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < kTlKeys; c += 32) tmem_landed32(s + c);
          pass_turn();
          if (n < kTlKeys) {                   // scores of keys that do not exist
#pragma unroll
            for (int e = 0; e < kTlKeys; ++e) s[e] = e < n ? s[e] : -INFINITY;
          }
          float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
          for (int e = 0; e < kTlKeys; e += 8) {
#pragma unroll
            for (int q = 0; q < 4; ++q) mx[q] = max3(mx[q], s[e + 2 * q], s[e + 2 * q + 1]);
          }
          const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * a.scale;
          if (m == -INFINITY) { sc = 0.f; m = top; }   // nothing seen yet; O, where there is one, is zero
          else if (top > m + kTlSlack) { sc = pt_exp2(m - top); m = top; }
          if (!mine) { sc = 1.f; m = 0.f; }            // a row that does not exist holds anything
          const float ref = m == -INFINITY ? 0.f : m;
          const unsigned long long scale2 = pack_f32x2(a.scale, a.scale), ref2 = pack_f32x2(-ref, -ref);
          unsigned long long sum2[4] = {0ull, 0ull, 0ull, 0ull};
          auto weights = [&](int e0, int e1) {
#pragma unroll
            for (int e = e0; e < e1; e += 2) {
              float x, y;
              const unsigned long long d2 = fma_f32x2(pack_f32x2(s[e], s[e + 1]), scale2, ref2);
              if ((e >> 1) % 4 == 3) {
                unpack_f32x2(poly_exp2(d2), x, y);
              } else {
                unpack_f32x2(d2, x, y);
                x = pt_exp2(x); y = pt_exp2(y);
              }
              sum2[(e >> 1) & 3] = add_f32x2(sum2[(e >> 1) & 3], pack_f32x2(x, y));
              s[e >> 1] = __uint_as_float(un_pack<F16>(x, y));
            }
          };
          weights(0, kTlKeys);
          float s0, s1;
          unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), s0, s1);
          l = fmaf(l, sc, s0 + s1);
          // P V of the block before, to which P and O belong, and the scores of the next block, both under way since its turn began
          fine = wait_warp(&sh.s_full[half], (uint32_t)i++ & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          if (j > j0 && __any_sync(0xFFFFFFFFu, sc != 1.f)) {
#pragma unroll
            for (int c = 0; c < kHeadDim; c += 32) {
              float o[32];
              tmem_ld32(t_lane + 192u + (uint32_t)c, o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= sc;
              tmem_st32(t_lane + 192u + (uint32_t)c, o);
            }
          }
          tmem_st32_async(t_lane + 128u, s);
          tmem_st32_async(t_lane + 160u, s + 32);
          tmem_wait_st();
          if (n < kTlKeys) clear_v(j, n);
        }
      }
      if (!fine) break;
      // ---- the tile's rows leave ----
      float o[kHeadDim];
#pragma unroll
      for (int c = 0; c < kHeadDim; ++c) o[c] = 0.f;
      n_block += j1 - j0;
      if (blocks > j0) {
        pass_turn();
        fine = wait_warp(&sh.pv_done[half], (uint32_t)n_o++ & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        if (live) {
#pragma unroll
          for (int c = 0; c < kHeadDim; c += 32) tmem_ld32(t_lane + 192u + (uint32_t)c, *reinterpret_cast<float (*)[32]>(o + c));
        }
        tc_fence_before_sync();                // O may be overwritten once this thread's next P is announced
      }
      const int c0 = size.of(p.u0), c1 = size.of(p.u0 + p.nu - 1);
      bool whole = c0 == c1;
      if (!whole) {                            // this part into scratch, and a ticket for the warp's 32 rows
        const bool begins = c0 == (int)blockIdx.x;
        if (mine) {
          float *x = part_at_place(blockIdx.x, c0);
#pragma unroll
          for (int c = 0; c < kHeadDim / 4; ++c) *reinterpret_cast<float4 *>(x + (c * kTlTile + tid) * 4) = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
          *reinterpret_cast<float2 *>(x + kTlTile * kHeadDim + 2 * tid) = make_float2(m, l);
        }
        __threadfence();
        __syncwarp();
        int came = 0;
        if (lane == 0) came = (int)atomicAdd(a.tickets + (kTlTile / 32) * c0 + warp, 1u) + 1;
        if (begins) {                          // the CTA's last tile; as a rule the others have long had theirs
          whole = __shfl_sync(0xFFFFFFFFu, came, 0) == c1 - c0 + 1;
          if (whole) {
            if (lane == 0) a.tickets[(kTlTile / 32) * c0 + warp] = 0u;
            __threadfence();
            if (mine) add_parts(c0, c0 + 1, c1, o, m, l);
          }
        } else {                               // the CTA's first: the answer is looked at when its range is done
          came_first = came;
          if (lane == 0) sh.meets = p;         // (every warp writes the same)
        }
      }
      if (j1 > j0) {                           // through the tile's Q, which no product reads any more
        const int qb = n_tile++ & 1;
        if (whole && live) leave(p, n_i, o, l, Qs + qb * kTlQ + half * kTlHalf);
        fence_proxy_async_smem();              // Q of the tile after next is copied over it
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_free[qb]);
      } else if (whole && mine) {   // no block here, and no Q: zeros, or the sum of other CTAs' parts
        const float inv = l == 0.f ? 0.f : 1.0f / l;
#pragma unroll
        for (int c = 0; c < kHeadDim; c += 8)
          *reinterpret_cast<uint4 *>(row_ptr(p, t) + c) = make_uint4(un_pack<F16>(o[c] * inv, o[c + 1] * inv), un_pack<F16>(o[c + 2] * inv, o[c + 3] * inv),
                                                                     un_pack<F16>(o[c + 4] * inv, o[c + 5] * inv), un_pack<F16>(o[c + 6] * inv, o[c + 7] * inv));
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(&sh.part_free[place_p]);
    }
    // ---- the tile that began before this CTA's range, where this CTA came to it last ----
    if (fine && (came_first = __shfl_sync(0xFFFFFFFFu, came_first, 0)) > 0) {
      const TilePart &p = sh.meets;
      const int c0 = size.of(p.u0), c1 = size.of(p.u0 + p.nu - 1), n_half = (a.rpt >> 1) * a.G, n_i = min(p.n_i - half * n_half, n_half);
      if (came_first == c1 - c0 + 1) {
        if (lane == 0) a.tickets[(kTlTile / 32) * c0 + warp] = 0u;
        __threadfence();
        float m = -INFINITY, l = 0.f, o[kHeadDim];
#pragma unroll
        for (int c = 0; c < kHeadDim; ++c) o[c] = 0.f;
        if (t < n_i) add_parts(c0, c0, c1, o, m, l);
        // (through the first Q: the products of this half are done, and its other warps keep to their own rows)
        if (32 * quarter < n_i) leave(p, n_i, o, l, Qs + half * kTlHalf);
      }
    }
    // ---- behind a wait that ran out: NaN into all rows of the call, among which are those that are not computed (a warp that has found the
    //      error covers them alone: others may have left before; one of an earlier call is found by all) ----
    if (*failed && first[a.n_seq] > 0) {
      const int x0 = *failed == 2 ? t : lane, step = *failed == 2 ? kTlRows : 32;
#pragma unroll 1
      for (int i = 0; i < a.n_seq; ++i) {
        int qb, qe;
        q_span(i, qb, qe);
        uint4 *rows = reinterpret_cast<uint4 *>(a.out) + (size_t)qb * a.H * (kHeadDim / 8);
        const size_t n = (size_t)(qe - qb) * a.H * (kHeadDim / 8);
#pragma unroll 1
        for (size_t x = x0; x < n; x += step) rows[x] = make_uint4(0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu, 0x7FFF7FFFu);
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
  if (warp == 9) tmem_dealloc(tmem, 512);
}

inline long long tiles_part_rows() { return 2ll * kTlMaxCtas * kTlTile; }

template <bool F16>
inline cudaError_t launch_tiles_as(const CUtensorMap &q_map, const CUtensorMap &k_map, const CUtensorMap &v_map, const UnitArgs &a, int n_sm, cudaStream_t st) {
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(attention_tiles_kernel<F16>, tiles_smem_bytes(kTlMaxSeq))) return e;
  return launch_kernel(attention_tiles_kernel<F16>, dim3(std::min(n_sm, kTlMaxCtas)), dim3(kTlThreads), tiles_smem_bytes(a.n_seq), st, false, q_map, k_map, v_map, a);
}

// Query rows: G heads of one group and `rows` rows a copy.
inline cudaError_t tiles_q_map(CUtensorMap *map, bool f16, const void *q, size_t heads, size_t rows, size_t row, int G, int n) {
  const cuuint64_t dims[3] = {kHeadDim, heads, rows}, strides[2] = {kHeadDim * 2, rows == 1 ? heads * kHeadDim * 2 : row};
  const cuuint32_t box[3] = {kHeadDim, (cuuint32_t)G, (cuuint32_t)n};
  return tensor_map_encode(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, q, 3, dims, strides, box, CU_TENSOR_MAP_SWIZZLE_128B);
}

}  // namespace ttsgpt
