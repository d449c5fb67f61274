// Attention of query tiles of 256 rows over blocks of 128 keys on the 5th-generation tensor cores: cross attention where a
// sequence has more queries than a tile of the warp-level kernel (Section I: the decode engine's attention kernels).
//
// A tile is two halves of 128 (row, head of the group) pairs of one sequence and one head of keys; thread t of a half's four softmax
// warps owns its row t = accumulator lane t.  For each block of 128 keys, which both halves read from one copy in shared memory,
//     S = Q K^T     tcgen05.mma M=128 x N=128 x K=64, S (fp32) in tensor memory
//     softmax       S out of tensor memory, running reference m and sum l in fp32, P = 2^(S scale - m) rounded to the inputs' type
//                   back into tensor memory.  The reference moves, and O with it, only where a score exceeds it by 2^8: weights
//                   stay below 256 and the rounding of a weight is relative, so nothing is lost
//     O += P V      M=128 x N=64 x K=128, P as the operand in tensor memory, V as stored
// S takes 128 columns, P 64 and O 64 of each half: all of an SM's tensor memory.  One half's softmax runs while the other's products
// do.  With 128 rows a CTA, two or four CTAs an SM, a block's copies alone took 1460 cycles of an SM (K and V came out of L2 for
// every 128 rows, 6.2 TB/s); for 256 rows they are half of that, and the exponentials, 16 a cycle and SM, bound the kernel.
//
// Work split.  The blocks of all tiles are laid end to end and cut into one range a CTA, equal to within a block; a tile counts
// one block more than its keys have.  The parts of a tile that several CTAs share meet as in the warp-level kernel: in scratch,
// added in the order of their keys by the CTA that arrives last at the tile's ticket.  Every wait on a copy or a product is bounded.
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

// The part of a tile that lies in a CTA's range.
struct TilePart {
  int row0, n_i, kvh, u0, nu;     // first query row, rows times heads, head of keys; the tile's units
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
  int failed;
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
    for (int i = 0; i < kTlRing; ++i) { mbar_init(&sh.full[i], 1); mbar_init(&sh.empty[i], 1); }
    for (int i = 0; i < 2; ++i) { mbar_init(&sh.q_full[i], 1); mbar_init(&sh.q_free[i], kTlTile / 32); }
    for (int i = 0; i < kTlParts; ++i) { mbar_init(&sh.part_full[i], 1); mbar_init(&sh.part_free[i], 1 + kTlTile / 32); }
    for (int h = 0; h < 2; ++h) { mbar_init(&sh.s_full[h], 1); mbar_init(&sh.p_full[h], kTlRows / 32); mbar_init(&sh.pv_done[h], 1); }
    sh.failed = 0;
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
  int carry = 0, bad = 0;                      // bad: starts that do not ascend, whose blocks nothing bounds
  for (int i0 = 0; i0 < a.n_seq; i0 += kTlThreads) {
    const int i = i0 + tid;
    int u = 0;
    if (i < a.n_seq) {
      int qb, qe, kb, ke;
      q_span(i, qb, qe);
      k_span(i, kb, ke);
      bad |= a.q_start[i + 1] < a.q_start[i] || a.k_start[i + 1] < a.k_start[i];
      u = a.Hkv * a.by_rpt.of(qe - qb + a.rpt - 1) * (1 + (ke - kb + kTlKeys - 1) / kTlKeys);
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
    sh.size.set(max(2, (T + (int)gridDim.x - 1) / (int)gridDim.x));
  }
  tc_fence_before_sync();
  __syncthreads();
  tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const Div size = sh.size;
  const int u_begin = blockIdx.x * (int)size.d, u_end = min(T, u_begin + (int)size.d);

  // from unit u on
  auto part_at = [&](int u) {
    TilePart p;
    int lo = 0, hi = a.n_seq - 1;
    while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (first[m] <= u) lo = m; else hi = m - 1; }
    int qb, qe, kb, ke;
    q_span(lo, qb, qe);
    k_span(lo, kb, ke);
    p.key0 = kb; p.keys = ke - kb;
    p.nu = 1 + (p.keys + kTlKeys - 1) / kTlKeys;
    const int x = u - first[lo], tile = (int)((unsigned)x / (unsigned)p.nu), blocks = a.by_rpt.of(qe - qb + a.rpt - 1);
    p.u0 = first[lo] + tile * p.nu;
    p.kvh = (int)((unsigned)tile / (unsigned)blocks);
    p.row0 = qb + (tile - p.kvh * blocks) * a.rpt;
    p.n_i = min(a.rpt, qe - p.row0) * a.G;
    p.j0 = max(u - p.u0 - 1, 0);
    p.j1 = min(u_end - p.u0, p.nu) - 1;
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
        u = p.u0 + p.j1 + 1;
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
      // ---- products: of either half in turn, when P of block j - 1 is there (and S has been read), Q K^T of block j, which its softmax
      //      waits for, and P V of block j - 1 behind it.  (Q K^T ahead of P, with a barrier of its own, made seven waits of this warp a
      //      block where there are three: 106 -> 165 us.) ----
      const uint32_t kind = F16 ? ~((1u << 7) | (1u << 10)) : ~0u;
      const uint32_t idesc_qk = tc_instr_desc(kTlRows, kTlKeys) & kind, idesc_pv = (tc_instr_desc(kTlRows, kHeadDim) & kind) | (1u << 16);   // V is MN-major
      int n_tile = 0, n_part = 0;                // tiles with blocks, and parts of this CTA
      bool fine = true;
      const uint64_t dring = tc_smem_desc(ring);
      int done[2] = {0, 0}, n_block = 0;       // blocks of either half that have had their P V, blocks of the CTA
      // P V of the block that half h has come to, block b of the CTA; last: no other half reads that block any more
      auto pv = [&](int h, int b, bool begins, bool last) {
        const int s = b % kTlRing;
        const uint64_t dv = dring + (uint64_t)((s * kTlBlock + kTlHalf) >> 4);
        const uint32_t t = tmem + 256u * h;
        if (elect_one()) {
#pragma unroll
          for (int q = 0; q < kTlKeys / 16; ++q)   // 16 keys an instruction: 8 columns of P, two groups of 8 rows of V
            tc_mma_ts(t + 192u, t + 128u + 8u * q, dv + 128 * q, idesc_pv, begins && q == 0 ? 0u : 1u);
          tc_commit(&sh.pv_done[h]);
          if (last) tc_commit(&sh.empty[s]);
        }
        __syncwarp();
        ++done[h];
      };
      for (int u = u_begin; u < u_end && fine;) {
        TilePart p;
        fine = take_part(n_part++, p);
        if (!fine) break;
        u = p.u0 + p.j1 + 1;
        if (p.j1 <= p.j0) continue;
        const int qb = n_tile & 1, halves = p.n_i > (a.rpt >> 1) * a.G ? 2 : 1;
        fine = wait_warp(&sh.q_full[qb], (uint32_t)(n_tile / 2) & 1u);
        ++n_tile;
        const uint64_t dq = tc_smem_desc(Qs + qb * kTlQ);
        for (int j = p.j0; j < p.j1 && fine; ++j, ++n_block) {
          fine = wait_warp(&sh.full[n_block % kTlRing], (uint32_t)(n_block / kTlRing) & 1u);
          const uint64_t dk = dring + (uint64_t)((n_block % kTlRing * kTlBlock) >> 4);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (h == halves || !fine) break;
            if (j > p.j0) fine = wait_warp(&sh.p_full[h], (uint32_t)done[h] & 1u);
            if (!fine) break;
            tc_fence_after_sync();
            if (elect_one()) {
#pragma unroll
              for (int q = 0; q < 4; ++q) tc_mma(tmem + 256u * h, dq + (uint64_t)(h * (kTlHalf >> 4) + 2 * q), dk + 2 * q, idesc_qk, q == 0 ? 0u : 1u);
              tc_commit(&sh.s_full[h]);
            }
            __syncwarp();
            if (j > p.j0) pv(h, n_block - 1, j - 1 == p.j0, h + 1 == halves);
          }
        }
        for (int h = 0; h < halves && fine; ++h) {   // the tile's last
          fine = wait_warp(&sh.p_full[h], (uint32_t)done[h] & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          pv(h, n_block - 1, p.j1 - 1 == p.j0, h + 1 == halves);
        }
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kTlRegsSoftmax));
    // ---- softmax ----
    const int half = warp >> 2, quarter = warp & 3, t = tid & (kTlRows - 1);   // the thread's row of the half
    const uint32_t t_lane = tmem + ((uint32_t)(32 * quarter) << 16) + 256u * half;
    int i = 0, n_block = 0, n_tile = 0, n_part = 0;   // blocks of this half and of the CTA, tiles with blocks, parts
    bool fine = true;
    for (int u = u_begin; u < u_end && fine;) {
      TilePart p;
      fine = take_part(n_part++, p);
      if (!fine) break;
      u = p.u0 + p.j1 + 1;
      const int n_half = (a.rpt >> 1) * a.G, n_i = min(p.n_i - half * n_half, n_half);   // rows of this half, none where not positive
      const bool live = 32 * quarter < n_i, mine = t < n_i;   // some row of the warp exists, the thread's own does
      const int blocks = n_i > 0 ? p.j1 : p.j0;
      if (n_i <= 0 && p.j1 > p.j0) {           // no such half here: no block holds it back, but it gives Q back below, once for each Q
        fine = wait_warp(&sh.q_full[n_tile & 1], (uint32_t)(n_tile / 2) & 1u);
        if (!fine) break;
      }
      float m = -INFINITY, l = 0.f;
      for (int j = p.j0; j < blocks; ++j, ++i) {
        fine = wait_warp(&sh.s_full[half], (uint32_t)i & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        const int n = min(kTlKeys, p.keys - j * kTlKeys);
        // all scores of the row into registers
        float s[kTlKeys], sc = 1.f;
        if (live) {
#pragma unroll
          for (int c = 0; c < kTlKeys; c += 32) tmem_ld32_async(t_lane + (uint32_t)c, s + c);
          tmem_wait_ld();
#pragma unroll
          for (int c = 0; c < kTlKeys; c += 32) tmem_landed32(s + c);
        }
        if (live) {
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
#pragma unroll
          for (int e = 0; e < kTlKeys; e += 2) {
            float x, y;
            unpack_f32x2(fma_f32x2(pack_f32x2(s[e], s[e + 1]), scale2, ref2), x, y);
            x = pt_exp2(x); y = pt_exp2(y);
            sum2[(e >> 1) & 3] = add_f32x2(sum2[(e >> 1) & 3], pack_f32x2(x, y));
            s[e >> 1] = __uint_as_float(un_pack<F16>(x, y));
          }
          float s0, s1;
          unpack_f32x2(add_f32x2(add_f32x2(sum2[0], sum2[1]), add_f32x2(sum2[2], sum2[3])), s0, s1);
          l = fmaf(l, sc, s0 + s1);
        }
        // P and O belong to the tensor core until P V of the block before has completed
        if (j > p.j0) {
          fine = wait_warp(&sh.pv_done[half], (uint32_t)(i - 1) & 1u);
          if (!fine) break;
          tc_fence_after_sync();
          if (__any_sync(0xFFFFFFFFu, sc != 1.f)) {
#pragma unroll
            for (int c = 0; c < kHeadDim; c += 32) {
              float o[32];
              tmem_ld32(t_lane + 192u + (uint32_t)c, o);
#pragma unroll
              for (int e = 0; e < 32; ++e) o[e] *= sc;
              tmem_st32(t_lane + 192u + (uint32_t)c, o);
            }
          }
        }
        if (live) {
#pragma unroll
          for (int c = 0; c < kTlKeys / 2; c += 32) tmem_st32_async(t_lane + 128u + (uint32_t)c, s + c);
          tmem_wait_st();
        }
        if (n < kTlKeys) {                     // the sequence's last block: V rows behind its keys may hold NaN, and 0 * NaN must not reach O
          // (both halves write the same zeros, each ahead of its own P V; S of the block is there, so its K and V are)
          unsigned char *v = ring + (n_block + j - p.j0) % kTlRing * kTlBlock + kTlHalf;
          for (int x = n * 8 + t; x < kTlKeys * 8; x += kTlRows) *reinterpret_cast<uint4 *>(v + x * 16) = make_uint4(0, 0, 0, 0);
          fence_proxy_async_smem();
        }
        tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.p_full[half]);
      }
      if (!fine) break;
      // ---- the tile's rows leave ----
      float o[kHeadDim];
#pragma unroll
      for (int c = 0; c < kHeadDim; ++c) o[c] = 0.f;
      n_block += p.j1 - p.j0;
      if (blocks > p.j0) {
        fine = wait_warp(&sh.pv_done[half], (uint32_t)(i - 1) & 1u);
        if (!fine) break;
        tc_fence_after_sync();
        if (live) {
#pragma unroll
          for (int c = 0; c < kHeadDim; c += 32) tmem_ld32(t_lane + 192u + (uint32_t)c, *reinterpret_cast<float (*)[32]>(o + c));
        }
        tc_fence_before_sync();                // O may be overwritten once this thread's next P is announced
      }
      const int c0 = size.of(p.u0), c1 = size.of(p.u0 + p.nu - 1);
      bool write = c0 == c1;
      if (!write) {
        // a place of 256 rows: 16 columns of four dimensions, then reference and sum; for the tile that goes on behind a CTA's range, and
        // the one that began before
        auto place = [&](int c) { return a.part + (size_t)(2 * c + (c == c0)) * kTlTile * kUnPitch; };
        if (mine) {
          float *x = place(blockIdx.x);
#pragma unroll
          for (int c = 0; c < kHeadDim / 4; ++c) *reinterpret_cast<float4 *>(x + (c * kTlTile + tid) * 4) = make_float4(o[4 * c], o[4 * c + 1], o[4 * c + 2], o[4 * c + 3]);
          *reinterpret_cast<float2 *>(x + kTlTile * kHeadDim + 2 * tid) = make_float2(m, l);
        }
        // a ticket for each warp's 32 rows
        __threadfence();
        __syncwarp();
        int last = 0;
        if (lane == 0) {
          unsigned *tk = a.tickets + (kTlTile / 32) * c0 + warp;
          last = atomicAdd(tk, 1u) + 1u == (unsigned)(c1 - c0 + 1);
          if (last) *tk = 0u;
        }
        write = __shfl_sync(0xFFFFFFFFu, last, 0) != 0;
        if (write && mine) {                   // all parts, this CTA's own among them, in the order of their keys
          __threadfence();
          m = -INFINITY; l = 0.f;
#pragma unroll
          for (int c = 0; c < kHeadDim; ++c) o[c] = 0.f;
#pragma unroll 1
          for (int c = c0; c <= c1; ++c) {
            const float *x = place(c);
            const float2 ml = __ldcg(reinterpret_cast<const float2 *>(x + kTlTile * kHeadDim + 2 * tid));
            const float mn = fmaxf(m, ml.x), fo = m == mn ? 1.f : pt_exp2(m - mn), fn = ml.y == 0.f ? 0.f : pt_exp2(ml.x - mn);   // 0: no key in it
            if (ml.y != 0.f) m = mn;
            const float fk = ml.y != 0.f ? fo : 1.f;
            l = fmaf(l, fk, ml.y * fn);
#pragma unroll
            for (int e = 0; e < kHeadDim / 4; ++e) {
              const float4 v = __ldcg(reinterpret_cast<const float4 *>(x + (e * kTlTile + tid) * 4));
              o[4 * e] = fmaf(o[4 * e], fk, v.x * fn); o[4 * e + 1] = fmaf(o[4 * e + 1], fk, v.y * fn);
              o[4 * e + 2] = fmaf(o[4 * e + 2], fk, v.z * fn); o[4 * e + 3] = fmaf(o[4 * e + 3], fk, v.w * fn);
            }
          }
        }
      }
      write = write && !*failed && __ldcg(a.err) == 0;
      const float inv = l == 0.f ? 0.f : 1.0f / l;
      auto row_ptr = [&](int i2) { const int r = a.by_G.of(i2); return a.out + ((size_t)(p.row0 + half * (a.rpt >> 1) + r) * a.H + (p.kvh - r) * a.G + i2) * kHeadDim; };
      if (p.j1 > p.j0) {                       // through the tile's Q, which no product reads any more: whole 128-byte rows leave
        const int qb = n_tile++ & 1;
        unsigned char *stage = Qs + qb * kTlQ + half * kTlHalf;
        if (write && live) {
#pragma unroll
          for (int c = 0; c < kHeadDim; c += 8)
            *reinterpret_cast<uint4 *>(stage + t * 128 + (((c >> 3) ^ (t & 7)) << 4)) =
                make_uint4(un_pack<F16>(o[c] * inv, o[c + 1] * inv), un_pack<F16>(o[c + 2] * inv, o[c + 3] * inv),
                           un_pack<F16>(o[c + 4] * inv, o[c + 5] * inv), un_pack<F16>(o[c + 6] * inv, o[c + 7] * inv));
          __syncwarp();
#pragma unroll
          for (int it = 0; it < 8; ++it) {
            const int r = 32 * quarter + 4 * it + (lane >> 3), c8 = lane & 7;
            if (r < n_i) *reinterpret_cast<uint4 *>(row_ptr(r) + 8 * c8) = *reinterpret_cast<const uint4 *>(stage + r * 128 + ((c8 ^ (r & 7)) << 4));
          }
        }
        fence_proxy_async_smem();              // Q of the tile after next is copied over it
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_free[qb]);
      } else if (write && mine) {              // no block here, and no Q: zeros, or the sum of other CTAs' parts
#pragma unroll
        for (int c = 0; c < kHeadDim; c += 8)
          *reinterpret_cast<uint4 *>(row_ptr(t) + c) = make_uint4(un_pack<F16>(o[c] * inv, o[c + 1] * inv), un_pack<F16>(o[c + 2] * inv, o[c + 3] * inv),
                                                                    un_pack<F16>(o[c + 4] * inv, o[c + 5] * inv), un_pack<F16>(o[c + 6] * inv, o[c + 7] * inv));
      }
    }
  }
  __syncwarp();
  tc_fence_before_sync();
  __syncthreads();
  if (*failed) {   // copies and products may still be in flight
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
