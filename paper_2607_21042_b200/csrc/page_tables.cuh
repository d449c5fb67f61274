// Page lists and slot maps of a pass, built on the GPU from the requests' lengths, and the pass's K and V rows into those
// slots (Section I: KV-cache management of the decode engine).
//
// Tables.  Request i adds n_i = new_len[i] tokens to stream s_i, which holds c_i.  With b_i = c_i, or 64 n_shared where a
// stream opens behind shared pages, the request's rows are positions b_i .. b_i + n_i - 1 and it takes
//     p_i = ceil((b_i + n_i) / 64) - ceil(b_i / 64)
// pages from the top of the stack: page number j of the request is free_pages[top - 1 - (p_0 + .. + p_(i-1)) - j].  Row
// r = n_0 + .. + n_(i-1) + k has slot page(pos / 64) * 64 + pos % 64.
//
// Every CTA computes both running sums over all requests for itself (at most 4096 of them, out of L2) and then writes its share
// of the rows and of the list entries, which it finds by bisection: one launch, no CTA waits for another.  What a caller may
// update in place (contexts, stack height) is then written by the CTA that leaves last, when every CTA has read it.
// Bound: two dependent reads (ids, contexts), one of the page stack, the launch; 12 bytes a row where there are many.  16 requests of a
// token 3.5 us, 128 requests with 3315 rows 5.2 us, 1000 requests with half a million rows 6.8 us; updated in place 0.1 us more from one CTA, 0.3 to
// 1 us from several, whose last one's turn it then is.
#pragma once
#include <cuda_fp8.h>
#include <algorithm>
#include "../../include/tts_gpt.h"
#include "common.cuh"

namespace ttsgpt {

constexpr int kTabMaxRequests = 4096;
constexpr int kTabMaxStreams = 32768;     // a bit each in shared memory, where an id that comes twice is found
constexpr int kTabMaxListPages = 32768;   // pages of a list: keeps a pass's rows below 2^36 and its pages below 2^28, as packed in one sum
constexpr int kTabPageBits = 28;

struct TableArgs {
  int n, max_streams, pps, n_pages, n_shared, max_rows;
  const int *stream_ids, *new_len, *ctx_len, *free_pages, *free_top, *shared_pages;
  int *ctx_len_out, *free_top_out, *page_table, *row_start, *row_stream, *row_pos, *row_slot;
  int in_place;   // ctx_len_out or free_top_out overlaps what every CTA reads
  int *info;   // {status, rows, pages taken, stack height, 0, 0, 0, CTAs that have left}
};

enum { kTabBadArg = 1, kTabBadStream = 2, kTabOverflow = 4, kTabRows = 8, kTabNoPages = 16 };

inline size_t page_tables_smem_bytes(int n, int max_streams) { return (size_t)(5 * n + 2 + (max_streams + 31) / 32) * sizeof(int); }

// THREADS * ITEMS requests at most
template <int THREADS, int ITEMS>
__global__ void __launch_bounds__(THREADS, 1) page_tables_kernel(const TableArgs a) {
  extern __shared__ int tab_smem[];
  int *row_s = tab_smem, *page_s = row_s + a.n + 1;              // running sums, one more than requests
  int *base_s = page_s + a.n + 1, *held_s = base_s + a.n, *id_s = held_s + a.n;
  unsigned *seen = reinterpret_cast<unsigned *>(id_s + a.n);
  __shared__ unsigned long long warp_sum_s[THREADS / 32];
  __shared__ int bad_s, last_s;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  int id[ITEMS], add[ITEMS], ctx[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = tid * ITEMS + k;
    id[k] = i < a.n ? (a.stream_ids ? a.stream_ids[i] : i) : -1;
    add[k] = i < a.n ? a.new_len[i] : 0;
  }
  const int top = *a.free_top;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) ctx[k] = id[k] >= 0 && id[k] < a.max_streams ? a.ctx_len[id[k]] : 0;
  for (int w = tid; w < (a.max_streams + 31) / 32; w += THREADS) seen[w] = 0u;
  if (tid == 0) bad_s = top < 0 || top > a.n_pages ? kTabBadArg : 0;
  __syncthreads();
  int bad = 0;
  unsigned long long mine[ITEMS], sum = 0;   // rows and pages of each request, and of the thread's
  int base[ITEMS], held[ITEMS];
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    mine[k] = 0; base[k] = 0; held[k] = 0;
    if (tid * ITEMS + k < a.n) {
      if (id[k] < 0 || id[k] >= a.max_streams || (atomicOr(&seen[id[k] >> 5], 1u << (id[k] & 31)) >> (id[k] & 31) & 1u)) bad |= kTabBadStream;
      else if (add[k] < 0 || ctx[k] < 0) bad |= kTabBadArg;
      else {
        base[k] = ctx[k] == 0 && add[k] > 0 ? a.n_shared * kPageTokens : ctx[k];
        if ((long long)base[k] + add[k] > (long long)a.pps * kPageTokens) bad |= kTabOverflow;
        else {
          held[k] = (int)((unsigned)(base[k] + kPageTokens - 1) / kPageTokens);
          const int taken = (int)((unsigned)(base[k] + add[k] + kPageTokens - 1) / kPageTokens) - held[k];
          mine[k] = ((unsigned long long)add[k] << kTabPageBits) + (unsigned long long)taken;
        }
      }
    }
    sum += mine[k];
  }
  // running sums: inside the warp, then of the warps
  auto scan = [&](unsigned long long v) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const unsigned long long u = __shfl_up_sync(0xFFFFFFFFu, v, o);
      if (lane >= o) v += u;
    }
    return v;
  };
  const unsigned long long incl = scan(sum);
  if (lane == 31) warp_sum_s[warp] = incl;
  __syncthreads();
  if (warp == 0) {
    const unsigned long long v = lane < THREADS / 32 ? warp_sum_s[lane] : 0ull, w = scan(v);
    __syncwarp();
    if (lane < THREADS / 32) warp_sum_s[lane] = w;   // inclusive
  }
  __syncthreads();
  const unsigned long long carry = warp_sum_s[THREADS / 32 - 1];
  unsigned long long e = (warp > 0 ? warp_sum_s[warp - 1] : 0ull) + incl - sum;
#pragma unroll
  for (int k = 0; k < ITEMS; ++k) {
    const int i = tid * ITEMS + k;
    if (i < a.n) {
      row_s[i] = (int)(e >> kTabPageBits);   // beyond 2^31 rows the pass is refused below
      page_s[i] = (int)(e & ((1u << kTabPageBits) - 1));
      base_s[i] = base[k]; held_s[i] = held[k]; id_s[i] = id[k];
    }
    e += mine[k];
  }
  const long long rows = (long long)(carry >> kTabPageBits);
  const int pages = (int)(carry & ((1u << kTabPageBits) - 1));
  if (tid == 0) { row_s[a.n] = (int)rows; page_s[a.n] = pages; }
  if (rows > a.max_rows) bad |= kTabRows;
  if (pages > top) bad |= kTabNoPages;
  if (bad) atomicOr(&bad_s, bad);
  __syncthreads();
  bad = bad_s;
  if (bad == 0) {
    auto request_of = [&](const int *start, int x, int lo, int hi) {   // last request of lo .. hi that starts at or before x
      while (lo < hi) { const int m = (lo + hi + 1) >> 1; if (start[m] <= x) lo = m; else hi = m - 1; }
      return lo;
    };
    const int me = blockIdx.x * THREADS + tid, all = gridDim.x * THREADS;
    // 128 rows a warp: the requests of the first and the last, then each row's between them (where prompts are long, one or two)
#pragma unroll 1
    for (unsigned r0 = (me >> 5) * 128; r0 < (unsigned)rows; r0 += (all >> 5) * 128) {   // unsigned: the last turn may step past 2^31
      const int i0 = request_of(row_s, (int)r0, 0, a.n - 1), i1 = request_of(row_s, (int)min(r0 + 127, (unsigned)rows - 1), i0, a.n - 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const unsigned r = r0 + 32 * e + lane;
        if (r < (unsigned)rows) {
          const int i = request_of(row_s, (int)r, i0, i1), pos = base_s[i] + (int)r - row_s[i], pg = (unsigned)pos / kPageTokens;
          // on a page that the stream holds, or the next of the stack
          const int *page = pg < held_s[i] ? a.page_table + (size_t)id_s[i] * a.pps + pg : a.free_pages + top - 1 - (page_s[i] + pg - held_s[i]);
          a.row_stream[r] = id_s[i];
          a.row_pos[r] = pos;
          a.row_slot[r] = *page * kPageTokens + (unsigned)pos % kPageTokens;
        }
      }
    }
#pragma unroll 1
    for (int k = me; k < pages; k += all) {                  // new entries of the page lists
      const int i = request_of(page_s, k, 0, a.n - 1);
      a.page_table[(size_t)id_s[i] * a.pps + held_s[i] + k - page_s[i]] = a.free_pages[top - 1 - k];
    }
    if (a.n_shared > 0) {                                    // the shared pages of the streams that open: a request a warp
#pragma unroll 1
      for (int i = blockIdx.x * (THREADS / 32) + warp; i < a.n; i += gridDim.x * (THREADS / 32))
        if (row_s[i + 1] > row_s[i] && base_s[i] == a.n_shared * kPageTokens && a.ctx_len[id_s[i]] == 0)
          for (int j = lane; j < a.n_shared; j += 32) a.page_table[(size_t)id_s[i] * a.pps + j] = a.shared_pages[j];
    }
    if (blockIdx.x == 0)
      for (int i = tid; i <= a.n; i += THREADS) a.row_start[i] = row_s[i];
  }
  if (a.in_place) {   // by the CTA that leaves last, when every CTA has read what is updated
    __syncthreads();
    if (tid == 0) {
      last_s = 1;
      if (gridDim.x > 1) { __threadfence(); last_s = atomicAdd(a.info + 7, 1) == (int)gridDim.x - 1; }
    }
    __syncthreads();
    if (!last_s) return;
  } else if (blockIdx.x > 0) {
    return;
  }
  if (bad == 0)
    for (int i = tid; i < a.n; i += THREADS) {
      const int len = row_s[i + 1] - row_s[i];
      a.ctx_len_out[id_s[i]] = base_s[i] + len;
    }
  if (tid == 0) {
    const int code = bad & kTabBadArg ? TTS_GPT_E_ARG : bad & kTabBadStream ? TTS_GPT_E_STREAM : bad & kTabOverflow ? TTS_GPT_E_CTX_OVERFLOW
                     : bad & kTabRows ? TTS_GPT_E_WORKSPACE : bad ? TTS_GPT_E_NO_PAGES : TTS_GPT_OK;
    a.info[0] = code;
    a.info[1] = bad ? 0 : (int)rows;
    a.info[2] = bad ? 0 : pages;
    a.info[3] = bad ? top : top - pages;
    if (!bad) *a.free_top_out = top - pages;
    if (a.in_place) a.info[7] = 0;
  }
}

// A thread writes up to four rows; more CTAs than that only repeat the sums.
inline int page_tables_grid(int n, int max_rows, int n_sm) {
  return n <= 256 ? std::min(2 * n_sm, (max_rows - 1) / 1024 + 1) : std::min(n_sm, (max_rows - 1) / 2048 + 1);   // max_rows is 1 at least
}

inline cudaError_t launch_page_tables(const TableArgs &a, int n_sm, cudaStream_t st) {
  const size_t smem = page_tables_smem_bytes(a.n, a.max_streams);
  const int grid = page_tables_grid(a.n, a.max_rows, n_sm);
  if (a.n <= 256) {
    static SmemOptIn opt_in;
    if (const cudaError_t e = opt_in(page_tables_kernel<256, 1>, page_tables_smem_bytes(256, kTabMaxStreams))) return e;
    return launch_kernel(page_tables_kernel<256, 1>, dim3(grid), dim3(256), smem, st, false, a);
  }
  static SmemOptIn opt_in;
  if (const cudaError_t e = opt_in(page_tables_kernel<1024, 4>, page_tables_smem_bytes(kTabMaxRequests, kTabMaxStreams))) return e;
  return launch_kernel(page_tables_kernel<1024, 4>, dim3(grid), dim3(1024), smem, st, false, a);
}

// ---------------------------------------------------------------------------------------------
// K and V rows into their slots
// ---------------------------------------------------------------------------------------------
constexpr int kE4m3BlockBytes = kPageTokens * kHeadDim + kPageTokens * 4;   // codes, then the tokens' fp32 scales

struct AppendArgs {
  const void *k, *v;
  long long k_stride, v_stride;   // elements between rows
  const int *row_slot;
  unsigned char *pool;
  int R, H, n_slots;              // slots of the pool: 64 n_pages
};

__device__ __forceinline__ void load8(const float *p, float (&x)[8]) {
  const float4 lo = *reinterpret_cast<const float4 *>(p), hi = *reinterpret_cast<const float4 *>(p + 4);
  x[0] = lo.x; x[1] = lo.y; x[2] = lo.z; x[3] = lo.w; x[4] = hi.x; x[5] = hi.y; x[6] = hi.z; x[7] = hi.w;
}
__device__ __forceinline__ void load8(const uint16_t *p, float (&x)[8]) {
  const uint4 w = *reinterpret_cast<const uint4 *>(p);
  const uint32_t ww[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) { x[2 * i] = bf16_lo(ww[i]); x[2 * i + 1] = bf16_hi(ww[i]); }
}

// Eight lanes take the 64 values of one (row, K|V, head), eight values each.  16-bit cache: each value rounded once.  8-bit cache:
// s = max|x| / 448 over the 64 (1 where that is zero in fp32), codes e4m3(x / s).  Bound: bytes in and out; a thread has PER such pieces under
// way, of rows far apart (3584 fp32 rows of 20 heads, 55 MB: four 10.4 us, 5.3 TB/s; one 11.8 us; 16 rows 1.8 us).
constexpr int kAppendThreads = 256;
template <typename Src, bool E4M3, int PER>
__global__ void __launch_bounds__(kAppendThreads) kv_append_kernel(const AppendArgs a) {
  const int e = threadIdx.x & 7;
  const int items = a.R * 2 * a.H, step = (items + PER - 1) / PER;   // host: below 2^31
  const int item0 = (int)(((long long)blockIdx.x * kAppendThreads + threadIdx.x) >> 3);
  float x[PER][8];
  int slot[PER], which[PER], h[PER];
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const int item = item0 + p * step;
    const bool live = item0 < step && item < items;    // the same for the eight lanes of an item
    const int r = live ? (int)((unsigned)item / (unsigned)(2 * a.H)) : 0, rem = live ? item - r * 2 * a.H : 0;
    which[p] = rem >= a.H ? 1 : 0;
    h[p] = rem - which[p] * a.H;
    slot[p] = live ? a.row_slot[r] : -1;
    load8(reinterpret_cast<const Src *>(which[p] ? a.v : a.k) + (size_t)r * (which[p] ? a.v_stride : a.k_stride) + h[p] * kHeadDim + 8 * e, x[p]);
  }
#pragma unroll
  for (int p = 0; p < PER; ++p) {
    const bool there = slot[p] >= 0 && slot[p] < a.n_slots;
    const int page = there ? slot[p] / kPageTokens : 0, off = there ? slot[p] % kPageTokens : 0;
    const size_t block = ((size_t)page * 2 + which[p]) * a.H + h[p];
    const float (&v)[8] = x[p];
    if constexpr (E4M3) {
      float m = fabsf(v[0]);
#pragma unroll
      for (int i = 1; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
      const float quotient = m / 448.0f, s = quotient > 0.f ? quotient : 1.0f;   // below 448 2^-150 it is zero though m is not
      uint32_t w[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * i], s), __fdiv_rn(v[4 * i + 1], s)), __NV_SATFINITE, __NV_E4M3);
        const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * i + 2], s), __fdiv_rn(v[4 * i + 3], s)), __NV_SATFINITE, __NV_E4M3);
        w[i] = lo | (hi << 16);
      }
      if (there) {
        unsigned char *blk = a.pool + block * kE4m3BlockBytes;
        *reinterpret_cast<uint2 *>(blk + off * kHeadDim + 8 * e) = make_uint2(w[0], w[1]);
        if (e == 0) *reinterpret_cast<float *>(blk + kPageTokens * kHeadDim + 4 * off) = s;
      }
    } else if (there) {
      *reinterpret_cast<uint4 *>(a.pool + block * (kPageElems * 2) + off * (kHeadDim * 2) + 16 * e) =
          make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
    }
  }
}

template <typename Src, bool E4M3>
inline cudaError_t launch_kv_append_as(const AppendArgs &a, int n_sm, cudaStream_t st) {
  const long long items = (long long)a.R * 2 * a.H;
  auto go = [&](auto kernel, int per) {
    const long long threads = (items + per - 1) / per * 8;
    return launch_kernel(kernel, dim3((unsigned)((threads + kAppendThreads - 1) / kAppendThreads)), dim3(kAppendThreads), 0, st, false, a);
  };
  // from eight CTAs an SM on there are rows enough to give a thread four pieces
  if (items * 8 >= 8ll * n_sm * kAppendThreads) return go(kv_append_kernel<Src, E4M3, 4>, 4);
  return go(kv_append_kernel<Src, E4M3, 1>, 1);
}
inline cudaError_t launch_kv_append(const AppendArgs &a, bool src_f32, bool e4m3, int n_sm, cudaStream_t st) {
  if (src_f32) return e4m3 ? launch_kv_append_as<float, true>(a, n_sm, st) : launch_kv_append_as<float, false>(a, n_sm, st);
  return e4m3 ? launch_kv_append_as<uint16_t, true>(a, n_sm, st) : launch_kv_append_as<uint16_t, false>(a, n_sm, st);
}

}  // namespace ttsgpt
