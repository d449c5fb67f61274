// A pass's queries and keys rotated by their positions, keys and values into their slots of the paged cache (Section I: KV-cache
// management of the decode engine, here for models with rotary positions).
//
// Pair i of a head, values a and b, at position p turns by theta = p w_i:
//     a' = m (a cos theta - b sin theta),   b' = m (b cos theta + a sin theta)
// where the pair is (i, i + r/2) or (2i, 2i + 1) of the first r values; the others stay.  V stays.
//
// Angles.  The table holds w_i / 2 pi as a fraction of 2^64, so that p times it, in 64-bit integers that wrap, is the phase in turns
// modulo one, to 2^-64 of a turn a position, however far p is (in fp32 the angle of position 10^5 is off by 2^-8 radians).  The nearest quarter turn is taken
// off in integers; what is left, at most an eighth of a turn either way, is rounded to fp32 (2^-27 half turns) and goes to sincospif.
//
// Split.  Eight lanes take the 64 values of a (row, head), eight values each; a CTA takes whole rows, whose sines and cosines it computes
// once for all heads while their values are on the way.  Bound: bytes in and out.
#pragma once
#include "attention_common.cuh"
#include "page_tables.cuh"

namespace ttsgpt {

constexpr int kRopeThreads = 256, kRopeSlots = kRopeThreads / 8;
constexpr int kRopePer = 2;                    // (row, head) pieces of a thread under way at once
constexpr int kRopeRows = 16;                  // rows of a CTA at most

struct RopeArgs {
  const void *q, *k, *v;
  long long q_stride, k_stride, v_stride, out_stride;   // elements between rows
  const int *row_pos, *row_slot;
  const unsigned long long *turns;             // of a pair: turns a position, in 2^-64
  void *q_out;
  unsigned char *pool;
  int R, H, K, pairs, n_slots;                 // heads of q and of the pool; slots: 64 n_pages
  int rows;                                    // of a CTA
  int out_f32;
  float magnitude;
  Div by_heads;                                // H + 2 K
};

// cosine and sine of a phase, in 2^-64 turns
__device__ __forceinline__ float2 cos_sin_of_phase(unsigned long long phase) {
  const unsigned quarter = (unsigned)((phase + (1ull << 61)) >> 62);
  const long long rest = (long long)(phase - ((unsigned long long)quarter << 62));
  float s, c;
  sincospif((float)rest * 0x1p-63f, &s, &c);
  const float x = quarter & 1 ? s : c, y = quarter & 1 ? c : s;
  return make_float2((quarter + 1) & 2 ? -x : x, quarter & 2 ? -y : y);
}

enum { ROPE_HALF8 = 0, ROPE_HALF = 1, ROPE_NEIGHBOURS = 2 };   // pairs (i, i + r/2) with r/2 a multiple of 8, with any r/2; pairs (2i, 2i + 1)

template <typename Src, bool E4M3, int ORDER>
__global__ void __launch_bounds__(kRopeThreads) rope_kv_append_kernel(const RopeArgs a) {
  __shared__ __align__(16) float cos_s[kRopeRows][kHeadDim], sin_s[kRopeRows][kHeadDim];   // by value of the head; the sine with its sign
  const int tid = threadIdx.x, e = tid & 7, heads = a.H + 2 * a.K, rot = 2 * a.pairs;
  const int row0 = blockIdx.x * a.rows, n_rows = min(a.rows, a.R - row0), n = n_rows * heads;
#pragma unroll 1
  for (int base = 0; base < n; base += kRopePer * kRopeSlots) {
    float x[kRopePer][8], y[kRopePer][8];
    int slot[kRopePer], rl[kRopePer], head[kRopePer];
#pragma unroll
    for (int p = 0; p < kRopePer; ++p) {
      const int item = base + p * kRopeSlots + (tid >> 3);
      const bool live = item < n;
      rl[p] = live ? a.by_heads.of(item) : 0;
      head[p] = live ? item - rl[p] * heads : 0;
      const int r = row0 + rl[p], h = head[p];
      slot[p] = live ? a.row_slot[r] : -1;
      const Src *src = h < a.H ? reinterpret_cast<const Src *>(a.q) + (size_t)r * a.q_stride + h * kHeadDim
                       : h < a.H + a.K ? reinterpret_cast<const Src *>(a.k) + (size_t)r * a.k_stride + (h - a.H) * kHeadDim
                                       : reinterpret_cast<const Src *>(a.v) + (size_t)r * a.v_stride + (h - a.H - a.K) * kHeadDim;
      load8(src + 8 * e, x[p]);
      if constexpr (ORDER == ROPE_HALF) {      // the partners one by one
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int d = 8 * e + i, o = d < a.pairs ? d + a.pairs : d < rot ? d - a.pairs : d;
          if constexpr (sizeof(Src) == 4) y[p][i] = src[o];
          else y[p][i] = bf16_bits_to_float(src[o]);
        }
      }
    }
    if (base == 0) {
      for (int i = tid; i < n_rows * a.pairs; i += kRopeThreads) {
        const int r = i / a.pairs, j = i - r * a.pairs;
        const float2 cs = cos_sin_of_phase((unsigned long long)(long long)a.row_pos[row0 + r] * a.turns[j]);
        const int d0 = ORDER == ROPE_NEIGHBOURS ? 2 * j : j, d1 = ORDER == ROPE_NEIGHBOURS ? 2 * j + 1 : j + a.pairs;
        const float c = cs.x * a.magnitude, s = cs.y * a.magnitude;
        cos_s[r][d0] = c; cos_s[r][d1] = c;
        sin_s[r][d0] = -s; sin_s[r][d1] = s;
      }
      __syncthreads();
    }
    // (the output may lie over the queries: all lanes of a head have read it)
    __syncwarp();
#pragma unroll
    for (int p = 0; p < kRopePer; ++p) {
      const bool turn = head[p] < a.H + a.K, there = slot[p] >= 0 && slot[p] < a.n_slots;
      if constexpr (ORDER == ROPE_HALF8) {     // the partners are another lane's; lanes that turn nothing have themselves
        const int half = a.pairs >> 3, at = e < half ? e + half : e < 2 * half ? e - half : e, from = (tid & 24) | at;
#pragma unroll
        for (int i = 0; i < 8; ++i) y[p][i] = __shfl_sync(0xFFFFFFFFu, x[p][i], from);
      }
      if constexpr (ORDER == ROPE_NEIGHBOURS) {
#pragma unroll
        for (int i = 0; i < 8; ++i) y[p][i] = x[p][i ^ 1];
      }
      float c[8], s[8];
#pragma unroll
      for (int i = 0; i < 8; i += 4) {
        const float4 c4 = *reinterpret_cast<const float4 *>(&cos_s[rl[p]][8 * e + i]), s4 = *reinterpret_cast<const float4 *>(&sin_s[rl[p]][8 * e + i]);
        c[i] = c4.x; c[i + 1] = c4.y; c[i + 2] = c4.z; c[i + 3] = c4.w;
        s[i] = s4.x; s[i + 1] = s4.y; s[i + 2] = s4.z; s[i + 3] = s4.w;
      }
      float v[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = turn && 8 * e + i < rot ? fmaf(x[p][i], c[i], y[p][i] * s[i]) : x[p][i];
      const int r = row0 + rl[p], h = head[p];
      float scale = 1.f;
      if constexpr (E4M3) {                    // of the rotated values; all lanes of the warp take part
        float m = fabsf(v[0]);
#pragma unroll
        for (int i = 1; i < 8; ++i) m = fmaxf(m, fabsf(v[i]));
#pragma unroll
        for (int o = 1; o < 8; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const float quotient = m / 448.0f;
        scale = quotient > 0.f ? quotient : 1.0f;   // below 448 2^-150 it is zero though m is not
      }
      if (!there) continue;
      if (h < a.H) {
        if (a.out_f32) {
          float4 *dst = reinterpret_cast<float4 *>(reinterpret_cast<float *>(a.q_out) + (size_t)r * a.out_stride + h * kHeadDim + 8 * e);
          dst[0] = make_float4(v[0], v[1], v[2], v[3]);
          dst[1] = make_float4(v[4], v[5], v[6], v[7]);
        } else {
          *reinterpret_cast<uint4 *>(reinterpret_cast<uint16_t *>(a.q_out) + (size_t)r * a.out_stride + h * kHeadDim + 8 * e) =
              make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
        }
        continue;
      }
      const int kv = h - a.H, which = kv >= a.K, page = slot[p] / kPageTokens, off = slot[p] % kPageTokens;
      const size_t block = ((size_t)page * 2 + which) * a.K + (kv - which * a.K);
      if constexpr (E4M3) {
        uint32_t w[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * i], scale), __fdiv_rn(v[4 * i + 1], scale)), __NV_SATFINITE, __NV_E4M3);
          const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[4 * i + 2], scale), __fdiv_rn(v[4 * i + 3], scale)), __NV_SATFINITE, __NV_E4M3);
          w[i] = lo | (hi << 16);
        }
        unsigned char *blk = a.pool + block * kE4m3BlockBytes;
        *reinterpret_cast<uint2 *>(blk + off * kHeadDim + 8 * e) = make_uint2(w[0], w[1]);
        if (e == 0) *reinterpret_cast<float *>(blk + kPageTokens * kHeadDim + 4 * off) = scale;
      } else {
        *reinterpret_cast<uint4 *>(a.pool + block * (kPageElems * 2) + off * (kHeadDim * 2) + 16 * e) =
            make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
      }
    }
  }
}

template <typename Src, bool E4M3>
inline cudaError_t launch_rope_as(const RopeArgs &a, bool neighbours, cudaStream_t st) {
  const dim3 grid((unsigned)((a.R + a.rows - 1) / a.rows)), block(kRopeThreads);
  if (neighbours) return launch_kernel(rope_kv_append_kernel<Src, E4M3, ROPE_NEIGHBOURS>, grid, block, 0, st, false, a);
  if (a.pairs % 8 == 0) return launch_kernel(rope_kv_append_kernel<Src, E4M3, ROPE_HALF8>, grid, block, 0, st, false, a);
  return launch_kernel(rope_kv_append_kernel<Src, E4M3, ROPE_HALF>, grid, block, 0, st, false, a);
}
inline cudaError_t launch_rope(RopeArgs a, bool src_f32, bool e4m3, bool neighbours, cudaStream_t st) {
  const int heads = a.H + 2 * a.K;
  a.by_heads.set((uint32_t)heads);
  a.rows = max(1, min(kRopeRows, kRopePer * kRopeSlots / heads));   // pieces for all threads where a row has few
  if (src_f32) return e4m3 ? launch_rope_as<float, true>(a, neighbours, st) : launch_rope_as<float, false>(a, neighbours, st);
  return e4m3 ? launch_rope_as<uint16_t, true>(a, neighbours, st) : launch_rope_as<uint16_t, false>(a, neighbours, st);
}

}  // namespace ttsgpt
