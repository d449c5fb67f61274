// Trees of drafted tokens: ancestors and positions from the parents, the path that the model agrees with, and its keys and values
// to where they belong in the cache (Section I: KV-cache management of the decode engine, here for several tokens a step).
//
// Tree i is rows row_start[i] .. row_start[i + 1] - 1, nodes 0, 1, ..; parent[r] < r's own number is a node, or -1.  Its nodes are the last
// T_i of the kv_len[stream] tokens that the stream holds; those before them are committed.
#pragma once
#include <algorithm>
#include "../../include/tts_gpt.h"
#include "common.cuh"
#include "page_tables.cuh"

namespace ttsgpt {

constexpr int kTreeNodes = 256, kTreeWords = kTreeNodes / 32;   // nodes of a tree at most, and words of a node's mask
constexpr int kTreeMaxSeq = 4096;

// rows of tree i of arrays with R rows; false: starts that do not ascend, or lie outside
__device__ __forceinline__ bool tree_rows(const int *row_start, int i, int R, int &first, int &n) {
  first = row_start[i];
  const int end = row_start[i + 1];
  n = end - first;
  return first >= 0 && end >= first && end <= R;
}

// ---------------------------------------------------------------------------------------------
// Ancestors and positions.  With A_j the set {j} and up_j the parent of j, a round takes  A_j |= A_(up_j), up_j = up_(up_j):  after k rounds
// A_j has 2^k ancestors and up_j is the one behind them, so that the sets are complete when every up_j is -1.  A CTA a tree, a thread a
// node, sets in shared memory.  Depth: |A_j| - 1.  Bound: launch, two dependent reads, log2(depth) rounds of two barriers.
// Measured: 16 trees of up to 40 nodes 1.6 us (a launch), 128 of up to 200 2.9 us.
// ---------------------------------------------------------------------------------------------
struct TreeTableArgs {
  int n, R, max_streams, words;
  const int *row_start, *stream_ids, *kv_len, *parent;
  int *mask, *row_pos, *info;
};

template <int WORDS>
__global__ void __launch_bounds__(32 * WORDS) tree_tables_kernel(const TreeTableArgs a) {
  __shared__ unsigned set_s[WORDS][32 * WORDS];
  __shared__ int up_s[32 * WORDS];
  pdl_launch_dependents();
  pdl_wait();                                  // nothing of memory is touched before (in all of these kernels)
  const int i = blockIdx.x, j = threadIdx.x;
  int first, n;
  const bool sound = tree_rows(a.row_start, i, a.R, first, n);
  const int stream = a.stream_ids ? a.stream_ids[i] : i;
  const int code = !sound ? TTS_GPT_E_ARG : n > 32 * WORDS || n > 32 * a.words ? TTS_GPT_E_WORKSPACE : stream < 0 || stream >= a.max_streams ? TTS_GPT_E_STREAM : TTS_GPT_OK;
  if (code != TTS_GPT_OK) {                    // the same for the whole CTA
    if (j == 0) atomicMin(a.info, code);
    return;
  }
  const int up0 = j < n ? a.parent[first + j] : -1, len = a.kv_len[stream];
  if (__syncthreads_or(j < n && (up0 < -1 || up0 >= j)) || len < n) {
    if (j == 0) atomicMin(a.info, (int)TTS_GPT_E_ARG);
    return;
  }
  unsigned set[WORDS];
  int up = up0;
#pragma unroll
  for (int w = 0; w < WORDS; ++w) set[w] = w == j >> 5 ? 1u << (j & 31) : 0u;
  while (__syncthreads_or(up >= 0)) {
#pragma unroll
    for (int w = 0; w < WORDS; ++w) set_s[w][j] = set[w];
    up_s[j] = up;
    __syncthreads();
    if (up >= 0) {
#pragma unroll
      for (int w = 0; w < WORDS; ++w) set[w] |= set_s[w][up];
      up = up_s[up];
    }
  }
  if (j >= n) return;
  int depth = -1;
#pragma unroll
  for (int w = 0; w < WORDS; ++w) depth += __popc(set[w]);
  int *row = a.mask + (size_t)(first + j) * a.words;
#pragma unroll
  for (int w = 0; w < WORDS; ++w)
    if (w < a.words) row[w] = (int)set[w];
  a.row_pos[first + j] = len - n + depth;
}

inline cudaError_t launch_tree_tables(const TreeTableArgs &a, cudaStream_t st) {
  const dim3 grid((unsigned)a.n);
  if (a.words <= 1) return launch_kernel(tree_tables_kernel<1>, grid, dim3(32), 0, st, true, a);
  if (a.words <= 2) return launch_kernel(tree_tables_kernel<2>, grid, dim3(64), 0, st, true, a);
  if (a.words <= 4) return launch_kernel(tree_tables_kernel<4>, grid, dim3(128), 0, st, true, a);
  return launch_kernel(tree_tables_kernel<8>, grid, dim3(256), 0, st, true, a);
}

// ---------------------------------------------------------------------------------------------
// Acceptance.  From node 0 on, the first child whose drafted token is what the model says after its parent, as long as there is one: every node's first such
// child is found at once (a minimum in shared memory), then a path is a walk along them.  A warp a tree.  One CTA then takes the streams' lengths back to the
// accepted nodes and returns the pages behind them: request by request in the order of the call, the last page of a list first; or, where something is wrong, takes all
// paths back.  It is the only one up to 32
// trees, the first of a cluster up to 256, which finds the others' counts in their shared memory, and else the one that comes last.
// Bound: launch, two dependent reads, two sums over the requests and a read of the pages.  Measured: 16 trees of up to 40 nodes 4.9 us, 128 of up to 200 7.0 us
// (8.0 and 12.5 with a search of the children at every step of the path, 256 threads and tickets; 7.1 and 11.6 with parents and tokens in registers).
// ---------------------------------------------------------------------------------------------
struct TreeAcceptArgs {
  int n, R, max_streams, pps, n_pages;
  const int *row_start, *stream_ids, *draft, *target, *parent, *kv_len, *page_table, *free_top;
  int *free_pages, *kv_len_out, *free_top_out, *path, *n_accepted, *next_token;
  int *info;   // {status, accepted, pages returned, stack height, 0, 0, what was found wrong, CTAs that have left}
};

constexpr int kAcceptThreads = 1024, kAcceptWarps = kAcceptThreads / 32, kAcceptCluster = 8;
enum { kTreeBadArg = 1, kTreeBadStream = 2, kTreeOverflow = 4, kTreeNodesOver = 8 };
inline size_t tree_accept_smem_bytes(int max_streams) { return (size_t)(kAcceptWarps * 2 * kTreeNodes + (max_streams + 31) / 32) * 4; }

__device__ __forceinline__ int ld_shared_of_rank(const int *p, uint32_t rank) {   // the word at p's place in the shared memory of a CTA of the cluster
  int v;
  asm volatile("{\n\t.reg .b32 a;\n\tmapa.shared::cluster.u32 a, %1, %2;\n\tld.shared::cluster.s32 %0, [a];\n\t}" : "=r"(v) : "r"(smem_u32(p)), "r"(rank) : "memory");
  return v;
}

// CLUSTER: all CTAs of the launch are one cluster
template <bool CLUSTER>
__global__ void __launch_bounds__(kAcceptThreads, 1) tree_accept_kernel(const TreeAcceptArgs a) {
  extern __shared__ int accept_smem[];
  int *child_s = accept_smem, *target_s = child_s + kAcceptWarps * kTreeNodes;   // of each warp's tree, by node: its first child on the path, what the model says
  unsigned *seen_s = reinterpret_cast<unsigned *>(target_s + kAcceptWarps * kTreeNodes);   // a bit a stream
  __shared__ int bad_s, last_s, warp_s[kAcceptWarps], acc_s[kAcceptWarps], count_s[kAcceptWarps];
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool alone = gridDim.x == 1;
  // ---- paths ----
  const int i = blockIdx.x * kAcceptWarps + warp;
  int first = 0, n = 0, bad = 0;
  if (i < a.n) {
    if (!tree_rows(a.row_start, i, a.R, first, n)) { bad = kTreeBadArg; first = n = 0; }
    if (n > kTreeNodes) { bad = kTreeNodesOver; n = 0; }
  }
  int up[kTreeWords], token[kTreeWords];
  int *child = child_s + warp * kTreeNodes, *target = target_s + warp * kTreeNodes;
#pragma unroll
  for (int w = 0; w < kTreeWords; ++w) {
    const int j = 32 * w + lane;
    up[w] = -1; token[w] = 0;
    if (j < n) { up[w] = a.parent[first + j]; token[w] = a.draft[first + j]; target[j] = a.target[first + j]; child[j] = kTreeNodes; }
  }
  // of tree x: stream, nodes, length; asked for before they are wanted.  wrong: what keeps the call from being carried out
  struct Seq { int stream, nodes, len, wrong; };
  auto read = [&](int x) {
    Seq s = {0, 0, 0, 0};
    int x0;
    s.stream = a.stream_ids ? a.stream_ids[x] : x;
    if (!tree_rows(a.row_start, x, a.R, x0, s.nodes)) s.wrong = kTreeBadArg;
    if (s.stream < 0 || s.stream >= a.max_streams) { s.wrong |= kTreeBadStream; s.stream = 0; return s; }
    s.len = a.kv_len[s.stream];
    if (s.wrong == 0 && s.len < s.nodes) s.wrong = kTreeBadArg;
    if (s.wrong == 0 && (int)((unsigned)(s.len + kPageTokens - 1) / kPageTokens) > a.pps) s.wrong = kTreeOverflow;
    return s;
  };
  const bool candidate = !CLUSTER || blockIdx.x == 0;   // may this CTA be the one that carries the rest out?
  const Seq mine = candidate && tid < a.n ? read(tid) : Seq{0, 0, 0, 0};
  const int top = *a.free_top;
  if (tid == 0) bad_s = 0;
  if (candidate)
    for (int w = tid; w < (a.max_streams + 31) / 32; w += kAcceptThreads) seen_s[w] = 0u;
  __syncthreads();
  if (i < a.n) {
    bool wrong = false;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) {
      const int j = 32 * w + lane;
      wrong |= j < n && (up[w] < -1 || up[w] >= j);
      if (j < n && up[w] >= 0 && up[w] < j && token[w] == target[up[w]]) atomicMin(&child[up[w]], j);
    }
    if (__any_sync(0xFFFFFFFFu, wrong)) bad = kTreeBadArg;
    __syncwarp();
    int count = 0, last = -1, at = n > 0 && !bad ? 0 : kTreeNodes, held = -1;   // held: of the path's rows, the lane's, until 32 are together
    while (at < kTreeNodes) {                  // a child has a higher number: at most n turns
      if ((count & 31) == lane) held = first + at;
      last = at;
      ++count;
      at = child[at];
      if ((count & 31) == 0) a.path[first + count - 32 + lane] = held;
    }
    const int done = count & ~31;
    if (done + lane < count) a.path[first + done + lane] = held;
    for (int k = count + lane; k < n; k += 32) a.path[first + k] = -1;
    if (lane == 0) {
      a.n_accepted[i] = count;
      a.next_token[i] = last >= 0 ? target[last] : -1;
      count_s[warp] = count;
      if (bad) atomicOr(&bad_s, bad);
    }
  }
  __syncthreads();
  // ---- lengths and pages, by one CTA ----
  if constexpr (CLUSTER) {
    cluster_arrive_release();
    cluster_wait();
    if (blockIdx.x > 0) {                      // its shared memory is still read
      cluster_arrive_relaxed();
      cluster_wait();
      return;
    }
    if (tid > 0 && tid < (int)gridDim.x) { const int x = ld_shared_of_rank(&bad_s, tid); if (x) atomicOr(&bad_s, x); }
  } else if (!alone) {
    if (tid == 0) {
      if (bad_s) atomicOr(a.info + 6, bad_s);
      __threadfence();
      last_s = atomicAdd(a.info + 7, 1) == (int)gridDim.x - 1;
      __threadfence();
      if (last_s) bad_s = __ldcg(a.info + 6);
    }
    __syncthreads();
    if (!last_s) return;
  }
  if (tid == 0 && (top < 0 || top > a.n_pages)) atomicOr(&bad_s, (int)kTreeBadArg);
  auto held = [](int len) { return (int)((unsigned)(len + kPageTokens - 1) / kPageTokens); };
  // pass 0: is every request sound, and how many pages come back?  pass 1: they do.  (Up to a CTA's threads the first pass leaves all that the second needs.)
  int freed_all = 0, accepted = 0, count = 0, before = 0;
  const bool once = a.n <= kAcceptThreads;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    int carry = 0, wrong = 0, acc = 0;
#pragma unroll 1
    for (int x0 = 0; x0 < a.n; x0 += kAcceptThreads) {
      const int x = x0 + tid;
      const Seq s = x >= a.n ? Seq{0, 0, 0, 0} : x0 == 0 ? mine : read(x);
      const bool there = x < a.n && s.wrong == 0;
      if (pass == 0 || !once) {
        if constexpr (CLUSTER) {
          count = x < a.n ? ld_shared_of_rank(&count_s[x & (kAcceptWarps - 1)], x / kAcceptWarps) : 0;
        } else {
          count = x >= a.n ? 0 : alone ? count_s[x] : __ldcg(a.n_accepted + x);
        }
        acc += count;
      }
      const int after = s.len - s.nodes + count, freed = there ? held(s.len) - held(after) : 0;
      if (pass == 0 && x < a.n) {
        wrong |= s.wrong;
        if (!(s.wrong & kTreeBadStream) && (atomicOr(&seen_s[s.stream >> 5], 1u << (s.stream & 31)) >> (s.stream & 31) & 1u)) wrong |= kTreeBadStream;
      }
      if (pass == 0 || !once) {
        int incl = freed;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
          const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
          if (lane >= o) incl += v;
        }
        __syncthreads();
        if (lane == 31) warp_s[warp] = incl;
        __syncthreads();
        // each warp adds the warps' sums up for itself
        const int all = warp_s[lane];
        const int total = __reduce_add_sync(0xFFFFFFFFu, all), below = __reduce_add_sync(0xFFFFFFFFu, lane < warp ? all : 0);
        before = carry + below + incl - freed;
        carry += total;
      }
      if (pass == 1 && there) {
        const int *list = a.page_table + (size_t)s.stream * a.pps + held(s.len) - 1;
        int *to = a.free_pages + top + before;
        for (int k = 0; k < freed; ++k) to[k] = list[-k];
        a.kv_len_out[s.stream] = after;
      }
    }
    if (pass == 0) {
      acc = __reduce_add_sync(0xFFFFFFFFu, acc);
      if (lane == 0) acc_s[warp] = acc;
      if (wrong) atomicOr(&bad_s, wrong);
      __syncthreads();
      if (tid == 0 && bad_s == 0 && (carry > a.n_pages || top > a.n_pages - carry)) bad_s = kTreeBadArg;   // more pages than there are
      __syncthreads();
      freed_all = carry;
      accepted = __reduce_add_sync(0xFFFFFFFFu, acc_s[lane]);
      if (bad_s) break;
    }
  }
  if (bad_s) {   // nothing is accepted: no path is left, not this call's nor what stood there, so that moves behind it move nothing
#pragma unroll 1
    for (int x = warp; x < a.n; x += kAcceptWarps) {
      const int r0 = max(a.row_start[x], 0), r1 = min(max(a.row_start[x + 1], 0), a.R);   // starts may be anything
#pragma unroll 1
      for (unsigned k = lane; k < (unsigned)max(r1 - r0, 0); k += 32) a.path[r0 + k] = -1;
    }
  }
  if (tid == 0) {
    const int what = bad_s;
    a.info[0] = what & kTreeBadArg ? TTS_GPT_E_ARG : what & kTreeBadStream ? TTS_GPT_E_STREAM : what & kTreeOverflow ? TTS_GPT_E_CTX_OVERFLOW : what ? TTS_GPT_E_WORKSPACE : TTS_GPT_OK;
    a.info[1] = what ? 0 : accepted;
    a.info[2] = what ? 0 : freed_all;
    a.info[3] = what ? top : top + freed_all;
    if (!what) *a.free_top_out = top + freed_all;
    a.info[6] = 0;
    a.info[7] = 0;
  }
  if constexpr (CLUSTER) {
    cluster_arrive_relaxed();
    cluster_wait();
  }
}

inline cudaError_t launch_tree_accept(const TreeAcceptArgs &a, cudaStream_t st) {
  const int ctas = (a.n + kAcceptWarps - 1) / kAcceptWarps;
  const size_t smem = tree_accept_smem_bytes(a.max_streams);
  if (ctas > 1 && ctas <= kAcceptCluster) {
    static SmemOptIn opt_in;
    if (const cudaError_t e = opt_in(tree_accept_kernel<true>, tree_accept_smem_bytes(kTabMaxStreams))) return e;
    return launch_kernel_cluster_dims(tree_accept_kernel<true>, dim3((unsigned)ctas), dim3(kAcceptThreads), smem, dim3((unsigned)ctas), st, true, a);
  }
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(tree_accept_kernel<false>, tree_accept_smem_bytes(kTabMaxStreams))) return e;
  return launch_kernel(tree_accept_kernel<false>, dim3((unsigned)ctas), dim3(kAcceptThreads), smem, st, true, a);
}

// ---------------------------------------------------------------------------------------------
// K and V rows of a path to the places behind the committed tokens: the k-th of path[first ..] to the slot of row first + k.  A CTA takes a
// tree and a layer; its threads own 16 bytes of a (K|V, head) row each and move it for all rows of the path, eight read before they are
// written.  Row k comes from a row behind it (path[k] > k where it moves at all, and path ascends), which is behind every place that
// rows before it go to: nothing is written before it has been read.
// Bound: three dependent reads of indices, then bytes.  Measured: a layer of 16 trees' paths 2.7 us; 24 layers of 32 9.2 us, 4.1 TB/s (12.4 with the pieces of all rows
// spread over the threads and a barrier between reads and writes).
// ---------------------------------------------------------------------------------------------
struct KvMoveArgs {
  int n, R, K, n_slots, layers;
  long long layer_bytes;
  const int *row_start, *path, *row_slot;
  unsigned char *pool;
};

constexpr int kMoveMaxThreads = 512, kMoveBatch = 8;

template <bool E4M3>
__global__ void __launch_bounds__(kMoveMaxThreads) kv_move_kernel(const KvMoveArgs a) {
  __shared__ int2 move_s[kMoveMaxThreads];     // {from, to}, slots
  __shared__ int2 warp_s[kMoveMaxThreads / 32];   // {rows that move, does the path end}
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, threads = blockDim.x;
  int first, n;
  if (!tree_rows(a.row_start, blockIdx.x, a.R, first, n)) return;
  unsigned char *pool = a.pool + (size_t)blockIdx.y * a.layer_bytes;
  bool more = true;                            // the path has not ended
#pragma unroll 1
  for (int k0 = 0; k0 < n && more; k0 += threads) {
    const int k = k0 + tid, r = k < n ? a.path[first + k] : -1;
    const unsigned ends = __ballot_sync(0xFFFFFFFFu, r < 0);
    const bool on = r > first + k && r < first + n && (ends & ((1u << lane) - 1)) == 0;   // a row that is where it belongs stays; nothing behind an end moves
    const int from = on ? a.row_slot[r] : -1, to = on ? a.row_slot[first + k] : -1;
    bool moves = from >= 0 && from < a.n_slots && to >= 0 && to < a.n_slots;
    const unsigned votes = __ballot_sync(0xFFFFFFFFu, moves);
    if (lane == 0) warp_s[warp] = make_int2(__popc(votes), ends != 0);
    __syncthreads();
    int at = __popc(votes & ((1u << lane) - 1)), count = 0;
#pragma unroll 1
    for (int w = 0; w < threads / 32 && more; ++w) {
      const int2 x = warp_s[w];
      if (w < warp) { at += x.x; moves = moves && !x.y; }
      count += x.x;
      more = !x.y;
    }
    if (moves) move_s[at] = make_int2(from, to);
    __syncthreads();
    constexpr int kLanes = E4M3 ? 4 : 8;       // 16-byte pieces of a row
    constexpr size_t kBlock = E4M3 ? kE4m3BlockBytes : kPageElems * 2;
    for (int piece = tid; piece < 2 * a.K * kLanes; piece += threads) {
      const int l16 = piece % kLanes, kv = piece / kLanes;   // K|V and head, as the pool has them
      unsigned char *mine = pool + (size_t)kv * kBlock + 16 * l16;
      const size_t page = (size_t)2 * a.K * kBlock;
      auto row = [&](int slot) { return reinterpret_cast<uint4 *>(mine + (size_t)(slot / kPageTokens) * page + slot % kPageTokens * (kLanes * 16)); };
      auto scale = [&](int slot) { return reinterpret_cast<float *>(mine + (size_t)(slot / kPageTokens) * page + kPageElems + 4 * (slot % kPageTokens)); };   // of lane 0
#pragma unroll 1
      for (int m = 0; m < count; m += kMoveBatch) {
        uint4 x[kMoveBatch];
        float s[kMoveBatch];
#pragma unroll
        for (int b = 0; b < kMoveBatch; ++b)
          if (m + b < count) {
            x[b] = *row(move_s[m + b].x);
            if (E4M3 && l16 == 0) s[b] = *scale(move_s[m + b].x);
          }
#pragma unroll
        for (int b = 0; b < kMoveBatch; ++b)
          if (m + b < count) {
            *row(move_s[m + b].y) = x[b];
            if (E4M3 && l16 == 0) *scale(move_s[m + b].y) = s[b];
          }
      }
    }
    __syncthreads();                           // the list is written anew
  }
}

inline cudaError_t launch_kv_move(const KvMoveArgs &a, bool e4m3, cudaStream_t st) {
  const int pieces = 2 * a.K * (e4m3 ? 4 : 8);   // a thread each, where there are not too many
  return launch_kernel(e4m3 ? kv_move_kernel<true> : kv_move_kernel<false>, dim3((unsigned)a.n, (unsigned)a.layers),
                       dim3((unsigned)std::min(kMoveMaxThreads, std::max(64, (pieces + 31) / 32 * 32))), 0, st, true, a);
}

}  // namespace ttsgpt
