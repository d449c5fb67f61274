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
  if (a.words <= 1) return launch_kernel(tree_tables_kernel<1>, grid, dim3(32), 0, st, false, a);
  if (a.words <= 2) return launch_kernel(tree_tables_kernel<2>, grid, dim3(64), 0, st, false, a);
  if (a.words <= 4) return launch_kernel(tree_tables_kernel<4>, grid, dim3(128), 0, st, false, a);
  return launch_kernel(tree_tables_kernel<8>, grid, dim3(256), 0, st, false, a);
}

// ---------------------------------------------------------------------------------------------
// Acceptance.  From node 0 on, the first child whose drafted token is what the model says after its parent, as long as there is one.  A warp a
// tree, whose nodes stay in its registers.  The CTA that comes last then takes the streams' lengths back to the accepted nodes and
// returns the pages behind them: request by request in the order of the call, the last page of a list first.
// Bound: launch, two dependent reads, a vote a node of the path; then, from several CTAs, a ticket and two sums over the requests.
// ---------------------------------------------------------------------------------------------
struct TreeAcceptArgs {
  int n, R, max_streams, pps, n_pages;
  const int *row_start, *stream_ids, *draft, *target, *parent, *kv_len, *page_table, *free_top;
  int *free_pages, *kv_len_out, *free_top_out, *path, *n_accepted, *next_token;
  int *info;   // {status, accepted, pages returned, stack height, 0, 0, what was found wrong, CTAs that have left}
};

constexpr int kAcceptThreads = 512;
enum { kTreeBadArg = 1, kTreeBadStream = 2, kTreeOverflow = 4, kTreeNodesOver = 8 };

__global__ void __launch_bounds__(kAcceptThreads) static tree_accept_kernel(const TreeAcceptArgs a) {
  extern __shared__ unsigned seen_s[];         // a bit a stream
  __shared__ int bad_s, last_s, warp_s[kAcceptThreads / 32], acc_s[kAcceptThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (tid == 0) bad_s = 0;
  __syncthreads();
  // ---- paths ----
  const int i = blockIdx.x * (kAcceptThreads / 32) + warp;
  if (i < a.n) {
    int first, n, bad = 0;
    if (!tree_rows(a.row_start, i, a.R, first, n)) { bad = kTreeBadArg; first = n = 0; }
    if (n > kTreeNodes) { bad = kTreeNodesOver; n = 0; }
    int up[kTreeWords], says[kTreeWords], token[kTreeWords];
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) {
      const int j = 32 * w + lane;
      up[w] = -2; says[w] = token[w] = 0;
      if (j < n) { up[w] = a.parent[first + j]; token[w] = a.draft[first + j]; says[w] = a.target[first + j]; }
    }
    bool wrong = false;
#pragma unroll
    for (int w = 0; w < kTreeWords; ++w) wrong |= 32 * w + lane < n && (up[w] < -1 || up[w] >= 32 * w + lane);
    if (__any_sync(0xFFFFFFFFu, wrong)) bad = kTreeBadArg;
    int count = 0, next = -1, at = n > 0 && !bad ? 0 : -1;
    while (at >= 0) {                          // a child has a higher number: at most n turns
      int said = 0;
#pragma unroll
      for (int w = 0; w < kTreeWords; ++w)
        if (w == at >> 5) said = says[w];
      next = __shfl_sync(0xFFFFFFFFu, said, at & 31);
      if (lane == 0) a.path[first + count] = first + at;
      ++count;
      int to = -1;
#pragma unroll
      for (int w = kTreeWords - 1; w >= 0; --w)
        if (32 * w < n) {                      // the same for the whole warp
          const unsigned hit = __ballot_sync(0xFFFFFFFFu, up[w] == at && token[w] == next);
          if (hit) to = 32 * w + __ffs((int)hit) - 1;
        }
      at = to;
    }
    for (int k = count + lane; k < n; k += 32) a.path[first + k] = -1;
    if (lane == 0) { a.n_accepted[i] = count; a.next_token[i] = next; if (bad) atomicOr(&bad_s, bad); }
  }
  __syncthreads();
  // ---- lengths and pages, by the CTA that comes last ----
  if (gridDim.x > 1) {
    if (tid == 0) {
      if (bad_s) atomicOr(a.info + 6, bad_s);
      __threadfence();
      last_s = atomicAdd(a.info + 7, 1) == (int)gridDim.x - 1;
      __threadfence();
    }
    __syncthreads();
    if (!last_s) return;
  }
  for (int w = tid; w < (a.max_streams + 31) / 32; w += kAcceptThreads) seen_s[w] = 0u;
  if (tid == 0 && gridDim.x > 1) bad_s = __ldcg(a.info + 6);
  __syncthreads();
  const int top = *a.free_top;
  if (top < 0 || top > a.n_pages) { if (tid == 0) atomicOr(&bad_s, (int)kTreeBadArg); }
  struct Seq { int stream, len, after, held, freed, count; };
  // of tree x; wrong: what keeps the call from being carried out
  auto read = [&](int x, int &wrong) {
    Seq s = {0, 0, 0, 0, 0, 0};
    int first, n;
    s.stream = a.stream_ids ? a.stream_ids[x] : x;
    if (s.stream < 0 || s.stream >= a.max_streams) { wrong |= kTreeBadStream; return s; }
    if (!tree_rows(a.row_start, x, a.R, first, n)) { wrong |= kTreeBadArg; return s; }
    s.len = a.kv_len[s.stream];
    s.count = __ldcg(a.n_accepted + x);
    if (s.len < n) { wrong |= kTreeBadArg; return s; }
    s.after = s.len - n + s.count;
    s.held = (int)((unsigned)(s.len + kPageTokens - 1) / kPageTokens);
    if (s.held > a.pps) { wrong |= kTreeOverflow; return s; }
    s.freed = s.held - (int)((unsigned)(s.after + kPageTokens - 1) / kPageTokens);
    return s;
  };
  // pass 0: is every request sound, and how many pages come back?  pass 1: they do
  int freed = 0, accepted = 0;
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    int carry = 0, wrong = 0, acc = 0;
#pragma unroll 1
    for (int x0 = 0; x0 < a.n; x0 += kAcceptThreads) {
      const int x = x0 + tid;
      Seq s = {0, 0, 0, 0, 0, 0};
      if (x < a.n) {
        s = read(x, wrong);
        if (pass == 0 && !(wrong & kTreeBadStream) && (atomicOr(&seen_s[s.stream >> 5], 1u << (s.stream & 31)) >> (s.stream & 31) & 1u)) wrong |= kTreeBadStream;
      }
      acc += s.count;
      int incl = s.freed;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int v = __shfl_up_sync(0xFFFFFFFFu, incl, o);
        if (lane >= o) incl += v;
      }
      __syncthreads();
      if (lane == 31) warp_s[warp] = incl;
      __syncthreads();
      int before = carry;
#pragma unroll
      for (int w = 0; w < kAcceptThreads / 32; ++w) { if (w < warp) before += warp_s[w]; carry += warp_s[w]; }
      if (pass == 1 && x < a.n) {
        const int *list = a.page_table + (size_t)s.stream * a.pps + s.held - 1;
        int *to = a.free_pages + top + before + incl - s.freed;
        for (int k = 0; k < s.freed; ++k) to[k] = list[-k];
        a.kv_len_out[s.stream] = s.after;
      }
    }
    if (pass == 0) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xFFFFFFFFu, acc, o);
      if (lane == 0) acc_s[warp] = acc;
      if (wrong) atomicOr(&bad_s, wrong);
      __syncthreads();
      if (tid == 0 && bad_s == 0 && (carry > a.n_pages || top > a.n_pages - carry)) bad_s = kTreeBadArg;   // more pages than there are
      __syncthreads();
      freed = carry;
      for (int w = 0; w < kAcceptThreads / 32; ++w) accepted += acc_s[w];
      if (bad_s) break;
    }
  }
  if (tid == 0) {
    const int bad = bad_s;
    a.info[0] = bad & kTreeBadArg ? TTS_GPT_E_ARG : bad & kTreeBadStream ? TTS_GPT_E_STREAM : bad & kTreeOverflow ? TTS_GPT_E_CTX_OVERFLOW : bad ? TTS_GPT_E_WORKSPACE : TTS_GPT_OK;
    a.info[1] = bad ? 0 : accepted;
    a.info[2] = bad ? 0 : freed;
    a.info[3] = bad ? top : top + freed;
    if (!bad) *a.free_top_out = top + freed;
    a.info[6] = 0;
    a.info[7] = 0;
  }
}

inline cudaError_t launch_tree_accept(const TreeAcceptArgs &a, cudaStream_t st) {
  const int per = kAcceptThreads / 32;
  return launch_kernel(tree_accept_kernel, dim3((unsigned)((a.n + per - 1) / per)), dim3(kAcceptThreads), (size_t)(a.max_streams + 31) / 32 * 4, st, false, a);
}

// ---------------------------------------------------------------------------------------------
// K and V rows of a path to the places behind the committed tokens: the k-th of path[first ..] to the slot of row first + k.  A CTA takes a
// tree and a layer; its threads own 16 bytes of a (K|V, head) row each and move it for all rows of the path, several read before they are
// written.  Row k comes from a row behind it (path[k] > k where it moves at all, and path ascends), which is behind every place that
// rows before it go to: nothing is written before it has been read.
// Bound: three dependent reads of indices, then bytes.
// ---------------------------------------------------------------------------------------------
struct KvMoveArgs {
  int n, R, K, n_slots, layers;
  long long layer_bytes;
  const int *row_start, *path, *row_slot;
  unsigned char *pool;
};

constexpr int kMoveThreads = 256, kMoveBatch = 4;

template <bool E4M3>
__global__ void __launch_bounds__(kMoveThreads) kv_move_kernel(const KvMoveArgs a) {
  __shared__ int2 move_s[kMoveThreads];        // {from, to}, slots
  __shared__ int warp_s[kMoveThreads / 32];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int first, n;
  if (!tree_rows(a.row_start, blockIdx.x, a.R, first, n)) return;
  unsigned char *pool = a.pool + (size_t)blockIdx.y * a.layer_bytes;
  bool more = true;
#pragma unroll 1
  for (int k0 = 0; k0 < n && more; k0 += kMoveThreads) {
    const int k = k0 + tid, r = k < n ? a.path[first + k] : -1;
    const bool on = k < n && r > first + k && r < first + n;     // a row that is where it belongs stays
    const int from = on ? a.row_slot[r] : -1, to = on ? a.row_slot[first + k] : -1;
    const bool moves = from >= 0 && from < a.n_slots && to >= 0 && to < a.n_slots;
    const unsigned votes = __ballot_sync(0xFFFFFFFFu, moves);
    if (lane == 0) warp_s[warp] = __popc(votes);
    more = __syncthreads_or(k < n && r >= 0);  // nothing behind a path's end
    int at = __popc(votes & ((1u << lane) - 1)), count = 0;
#pragma unroll
    for (int w = 0; w < kMoveThreads / 32; ++w) { if (w < warp) at += warp_s[w]; count += warp_s[w]; }
    if (moves) move_s[at] = make_int2(from, to);
    __syncthreads();
    constexpr int kLanes = E4M3 ? 4 : 8;       // 16-byte pieces of a row
    constexpr size_t kBlock = E4M3 ? kE4m3BlockBytes : kPageElems * 2;
    for (int piece = tid; piece < 2 * a.K * kLanes; piece += kMoveThreads) {
      const int lane16 = piece % kLanes, kv = piece / kLanes;   // K|V and head, as the pool has them
      auto row = [&](int slot) { return pool + ((size_t)(slot / kPageTokens) * 2 * a.K + kv) * kBlock + slot % kPageTokens * (kLanes * 16); };
      auto scale = [&](int slot) { return reinterpret_cast<float *>(pool + ((size_t)(slot / kPageTokens) * 2 * a.K + kv) * kBlock + kPageElems + 4 * (slot % kPageTokens)); };
#pragma unroll 1
      for (int m = 0; m < count; m += kMoveBatch) {
        uint4 x[kMoveBatch];
        float s[kMoveBatch];
#pragma unroll
        for (int b = 0; b < kMoveBatch; ++b)
          if (m + b < count) {
            x[b] = reinterpret_cast<const uint4 *>(row(move_s[m + b].x))[lane16];
            if (E4M3 && lane16 == 0) s[b] = *scale(move_s[m + b].x);
          }
#pragma unroll
        for (int b = 0; b < kMoveBatch; ++b)
          if (m + b < count) {
            reinterpret_cast<uint4 *>(row(move_s[m + b].y))[lane16] = x[b];
            if (E4M3 && lane16 == 0) *scale(move_s[m + b].y) = s[b];
          }
      }
    }
    __syncthreads();                           // the list is written anew
  }
}

inline cudaError_t launch_kv_move(const KvMoveArgs &a, bool e4m3, cudaStream_t st) {
  return launch_kernel(e4m3 ? kv_move_kernel<true> : kv_move_kernel<false>, dim3((unsigned)a.n, (unsigned)a.layers), dim3(kMoveThreads), 0, st, false, a);
}

}  // namespace ttsgpt
