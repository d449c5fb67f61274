// A pass's queries and keys rotated by their positions, keys and values into their slots of the paged cache (Section I: KV-cache
// management of the decode engine, here for models with rotary positions).
//
// Pair i of a head, values a and b, at position p turns by theta = p w_i:
//     a' = m (a cos theta - b sin theta),   b' = m (b cos theta + a sin theta)
// where the pair is (i, i + r/2) or (2i, 2i + 1) of the first r values; the others stay.  V stays.
//
// Angles.  The table holds w_i / 2 pi as a fraction of 2^64, so that p times it, in 64-bit integers that wrap, is the phase in turns
// modulo one, to two units of that a position, however far p is (in fp32 the angle of position 10^5 is off by 2^-8 radians).  The nearest quarter turn is taken
// off in integers; what is left, at most an eighth of a turn either way, is rounded to fp32 (2^-27 half turns) and goes to sincospif.
//
// Split.  A thread takes two times 16 bytes of a (row, head): eight lanes of fp32 or four of bf16 have its 64 values, and where pairs lie half the rotated
// values apart, a thread's are those of four or eight pairs, so that no lane asks another.  A CTA takes as many (row, head) pieces at once as it has such groups
// of lanes, in rows as wide as a power of two that holds the heads, and computes its rows' sines and cosines once for all heads while the values are under way.
// Bound: bytes in and out.  Measured: 16 fp32 rows of 20 heads 2.0 us (a launch), 3584 of them 15.2 us (5.4 TB/s; 21.4 with eight lanes a head that exchange halves by
// shuffles), 777 bf16 rows of 20 + 4 + 4 heads into the 8-bit cache 2.8 us, 3584 bf16 rows of 60 heads 13.3 us (in CTAs of 256 threads 16.0, with 8 bytes a time 17.4; CTAs that stay
// for more rows and load the next ahead: no faster, and 18.7 instead of 15.7 from fp32).  CTAs an SM by registers: one more or less costs 3 to 7 %.
#pragma once
#include "attention_common.cuh"
#include "page_tables.cuh"

namespace ttsgpt {

template <typename Src, int THREADS> struct RopeShape {
  static constexpr int kVals = 16 / sizeof(Src), kLanes = kHeadDim / (2 * kVals), kSlots = THREADS / kLanes;   // (row, head) pieces of a CTA
  static constexpr int kPer = sizeof(Src) == 4 ? 2 : 1;   // of a thread under way at once, where a row has more heads
  static constexpr int kRows = kSlots / 2;     // of a CTA at most
};

struct RopeArgs {
  const void *q, *k, *v;
  long long q_stride, k_stride, v_stride, out_stride;   // elements between rows
  const int *row_pos, *row_slot;
  const unsigned long long *turns;             // of a pair: turns a position, in 2^-64
  void *q_out;
  unsigned char *pool;
  int R, H, K, pairs, n_slots;                 // heads of q and of the pool; slots: 64 n_pages
  int lg;                                      // log2 of the slots of a row: as many as it has heads, as far as there are slots
  int out_f32;
  float magnitude;
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

enum { ROPE_HALVES = 0, ROPE_HALF = 1, ROPE_NEIGHBOURS = 2 };   // pairs (i, i + r/2) with r/2 a multiple of 16 bytes' values, with any r/2; pairs (2i, 2i + 1)

// 16 bytes as values
__device__ __forceinline__ void values_of(const uint4 &w, float (&x)[4]) { x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w); }
__device__ __forceinline__ void values_of(const uint4 &w, float (&x)[8]) {
  x[0] = bf16_lo(w.x); x[1] = bf16_hi(w.x); x[2] = bf16_lo(w.y); x[3] = bf16_hi(w.y);
  x[4] = bf16_lo(w.z); x[5] = bf16_hi(w.z); x[6] = bf16_lo(w.w); x[7] = bf16_hi(w.w);
}
// N values as bf16, as fp32, as e4m3 codes of scale s
template <int N> __device__ __forceinline__ void store_bf16(uint16_t *p, const float (&v)[N]) {
  if constexpr (N == 4) *reinterpret_cast<uint2 *>(p) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
  else *reinterpret_cast<uint4 *>(p) = make_uint4(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]), pack_bf16x2(v[4], v[5]), pack_bf16x2(v[6], v[7]));
}
template <int N> __device__ __forceinline__ void store_f32(float *p, const float (&v)[N]) {
#pragma unroll
  for (int i = 0; i < N; i += 4) *reinterpret_cast<float4 *>(p + i) = make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]);
}
template <int N> __device__ __forceinline__ void store_e4m3(unsigned char *p, const float (&v)[N], float s) {
  uint32_t w[N / 4];
#pragma unroll
  for (int i = 0; i < N; i += 4) {
    const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[i], s), __fdiv_rn(v[i + 1], s)), __NV_SATFINITE, __NV_E4M3);
    const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(__fdiv_rn(v[i + 2], s), __fdiv_rn(v[i + 3], s)), __NV_SATFINITE, __NV_E4M3);
    w[i / 4] = lo | (hi << 16);
  }
  if constexpr (N == 4) *reinterpret_cast<uint32_t *>(p) = w[0];
  else *reinterpret_cast<uint2 *>(p) = make_uint2(w[0], w[1]);
}

// CTAs an SM by registers
template <typename Src, bool E4M3, int ORDER, int THREADS> __host__ __device__ constexpr int rope_ctas() {
  return 256 / THREADS * (ORDER == ROPE_HALF ? (sizeof(Src) == 2 ? 2 : 3) : sizeof(Src) == 2 ? 3 : E4M3 ? 4 : 5);
}

template <typename Src, bool E4M3, int ORDER, int THREADS>
__global__ void __launch_bounds__(THREADS, rope_ctas<Src, E4M3, ORDER, THREADS>()) rope_kv_append_kernel(const RopeArgs a) {
  using Shape = RopeShape<Src, THREADS>;
  constexpr int kVals = Shape::kVals, kLanes = Shape::kLanes, kSlots = Shape::kSlots, kPer = Shape::kPer;
  __shared__ __align__(16) float cos_s[Shape::kRows][kHeadDim / 2], sin_s[Shape::kRows][kHeadDim / 2];   // by pair
  pdl_launch_dependents();
  pdl_wait();                                  // nothing of memory is touched before
  const int tid = threadIdx.x, e = tid % kLanes, heads = a.H + 2 * a.K, rot = 2 * a.pairs;
  const int rows = kSlots >> a.lg, rl = (tid / kLanes) >> a.lg, h0 = (tid / kLanes) & ((1 << a.lg) - 1);
  // the thread's values, kVals from d0 and from d1 on: of as many pairs, or of what is not rotated
  const int groups = a.pairs / kVals;
  const bool turns_half = ORDER == ROPE_HALVES && e < groups;
  const int d0 = ORDER != ROPE_HALVES || turns_half ? kVals * e : 2 * kVals * e, d1 = ORDER != ROPE_HALVES ? kVals * e + 32 : turns_half ? kVals * e + a.pairs : 2 * kVals * e + kVals;
  auto source = [&](int r, int h) {
    return h < a.H ? reinterpret_cast<const Src *>(a.q) + (size_t)r * a.q_stride + h * kHeadDim
           : h < a.H + a.K ? reinterpret_cast<const Src *>(a.k) + (size_t)r * a.k_stride + (h - a.H) * kHeadDim
                           : reinterpret_cast<const Src *>(a.v) + (size_t)r * a.v_stride + (h - a.H - a.K) * kHeadDim;
  };
  const int row0 = blockIdx.x * rows, r = row0 + rl;
  uint4 now[kPer][2];
  auto load = [&](int base) {
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      const int h = base + p * kSlots + h0;
      now[p][0] = now[p][1] = make_uint4(0, 0, 0, 0);
      if (r < a.R && h < heads) {
        const Src *src = source(r, h);
        now[p][0] = *reinterpret_cast<const uint4 *>(src + d0);
        now[p][1] = *reinterpret_cast<const uint4 *>(src + d1);
      }
    }
  };
  load(0);
  const int slot = r < a.R ? a.row_slot[r] : -1;
  for (int i = tid; i < rows * a.pairs; i += THREADS) {   // beside the loads
    const int k = i / a.pairs, j = i - k * a.pairs;
    if (row0 + k >= a.R) break;
    const float2 cs = cos_sin_of_phase((unsigned long long)(long long)a.row_pos[row0 + k] * a.turns[j]);
    cos_s[k][j] = cs.x * a.magnitude; sin_s[k][j] = cs.y * a.magnitude;
  }
  __syncthreads();
  const bool there = slot >= 0 && slot < a.n_slots;
  const int page = there ? slot / kPageTokens : 0, off = there ? slot % kPageTokens : 0;
  constexpr int kTurns = ORDER == ROPE_HALF ? 2 * kVals : kVals;
  float c[kTurns], s[kTurns];                // of the pairs of the thread's values; with any r/2 of each value, the second of a pair with its sign
  const float *cs = cos_s[rl], *sn = sin_s[rl];
  if constexpr (ORDER == ROPE_HALVES) {
    if (turns_half) {
#pragma unroll
      for (int i = 0; i < kVals; i += 4) {
        const float4 c4 = *reinterpret_cast<const float4 *>(cs + d0 + i), s4 = *reinterpret_cast<const float4 *>(sn + d0 + i);
        c[i] = c4.x; c[i + 1] = c4.y; c[i + 2] = c4.z; c[i + 3] = c4.w;
        s[i] = s4.x; s[i + 1] = s4.y; s[i + 2] = s4.z; s[i + 3] = s4.w;
      }
    }
  } else if constexpr (ORDER == ROPE_NEIGHBOURS) {
#pragma unroll
    for (int i = 0; i < kVals; ++i) {        // (of what is not rotated: not used)
      const int j = ((i < kVals / 2 ? d0 : d1) >> 1) + i % (kVals / 2);
      c[i] = cs[j]; s[i] = sn[j];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 2 * kVals; ++i) {
      const int d = i < kVals ? d0 + i : d1 + i - kVals, j = d < a.pairs ? d : d < rot ? d - a.pairs : 0;
      c[i] = cs[j];
      s[i] = d < a.pairs ? -sn[j] : sn[j];
    }
  }
#pragma unroll 1
  for (int base = 0; base < heads; base += kPer * kSlots) {   // the same for all threads
    if (base > 0) load(base);
    float y[ORDER == ROPE_HALF ? kPer : 1][2 * kVals];
    if constexpr (ORDER == ROPE_HALF) {      // the partners one by one
#pragma unroll
      for (int p = 0; p < kPer; ++p) {
        const int h = base + p * kSlots + h0;
#pragma unroll
        for (int i = 0; i < 2 * kVals; ++i) {
          const int d = i < kVals ? d0 + i : d1 + i - kVals, o = d < a.pairs ? d + a.pairs : d < rot ? d - a.pairs : d;
          if constexpr (sizeof(Src) == 4) y[p][i] = r < a.R && h < heads ? source(r, h)[o] : 0.f;
          else y[p][i] = r < a.R && h < heads ? bf16_bits_to_float(source(r, h)[o]) : 0.f;
        }
      }
    }
    __syncwarp();                            // (the output may lie over the queries: all lanes of a head have read it)
#pragma unroll
    for (int p = 0; p < kPer; ++p) {
      if (base + p * kSlots >= heads) break;         // the same for all threads
      const int h = base + p * kSlots + h0;
      float x[2][kVals], v[2][kVals];
      values_of(now[p][0], x[0]);
      values_of(now[p][1], x[1]);
#pragma unroll
      for (int i = 0; i < kVals; ++i) { v[0][i] = x[0][i]; v[1][i] = x[1][i]; }
      if (h < a.H + a.K) {
        if constexpr (ORDER == ROPE_HALVES) {
          if (turns_half) {
#pragma unroll
            for (int i = 0; i < kVals; ++i) {
              v[0][i] = fmaf(x[0][i], c[i], -(x[1][i] * s[i]));
              v[1][i] = fmaf(x[1][i], c[i], x[0][i] * s[i]);
            }
          }
        } else if constexpr (ORDER == ROPE_NEIGHBOURS) {
#pragma unroll
          for (int i = 0; i < kVals; ++i) {
            const int k = i / (kVals / 2), o = 2 * (i % (kVals / 2));
            if ((k ? d1 : d0) + o < rot) {
              v[k][o] = fmaf(x[k][o], c[i], -(x[k][o + 1] * s[i]));
              v[k][o + 1] = fmaf(x[k][o + 1], c[i], x[k][o] * s[i]);
            }
          }
        } else {
#pragma unroll
          for (int i = 0; i < 2 * kVals; ++i)
            if ((i < kVals ? d0 + i : d1 + i - kVals) < rot) v[i / kVals][i % kVals] = fmaf(x[i / kVals][i % kVals], c[i], y[p][i] * s[i]);
        }
      }
      float scale = 1.f;
      if constexpr (E4M3) {                  // of the rotated values; all lanes of the warp take part
        float m = 0.f;
#pragma unroll
        for (int i = 0; i < kVals; ++i) m = max_nan(m, max_nan(fabsf(v[0][i]), fabsf(v[1][i])));
#pragma unroll
        for (int o = 1; o < kLanes; o <<= 1) m = max_nan(m, __shfl_xor_sync(0xFFFFFFFFu, m, o));
        const float quotient = m / 448.0f;
        scale = quotient == 0.f ? 1.0f : quotient;   // below 448 2^-150 it is zero though m is not; NaN (and so the whole row) where a value is: codes have none that attention knows
      }
      if (!there || h >= heads) continue;
      if (h < a.H) {
        if (a.out_f32) {
          float *dst = reinterpret_cast<float *>(a.q_out) + (size_t)r * a.out_stride + h * kHeadDim;
          store_f32(dst + d0, v[0]);
          store_f32(dst + d1, v[1]);
        } else {
          uint16_t *dst = reinterpret_cast<uint16_t *>(a.q_out) + (size_t)r * a.out_stride + h * kHeadDim;
          store_bf16(dst + d0, v[0]);
          store_bf16(dst + d1, v[1]);
        }
        continue;
      }
      const size_t block = (size_t)page * 2 * a.K + (h - a.H);   // K's heads, then V's
      if constexpr (E4M3) {
        unsigned char *blk = a.pool + block * kE4m3BlockBytes;
        store_e4m3(blk + off * kHeadDim + d0, v[0], scale);
        store_e4m3(blk + off * kHeadDim + d1, v[1], scale);
        if (e == 0) *reinterpret_cast<float *>(blk + kPageTokens * kHeadDim + 4 * off) = scale;
      } else {
        uint16_t *dst = reinterpret_cast<uint16_t *>(a.pool + block * (kPageElems * 2)) + off * kHeadDim;
        store_bf16(dst + d0, v[0]);
        store_bf16(dst + d1, v[1]);
      }
    }
  }
}

template <typename Src, bool E4M3, int ORDER, int THREADS>
inline cudaError_t launch_rope_with(RopeArgs a, cudaStream_t st) {
  constexpr int kSlots = RopeShape<Src, THREADS>::kSlots;
  for (a.lg = 1; (1 << a.lg) < kSlots && (1 << a.lg) < a.H + 2 * a.K;) ++a.lg;
  return launch_kernel(rope_kv_append_kernel<Src, E4M3, ORDER, THREADS>, dim3((unsigned)((a.R - 1) / (kSlots >> a.lg) + 1)), dim3(THREADS), 0, st, true, a);
}
// CTAs of 256 threads have the shortest way through a row, CTAs of 128 wait less for one another where there are more than fit at once (3584 rows: of 60 bf16 heads 16.0 against 13.2 us,
// of 60 fp32 heads into the 8-bit cache 20.1, 18.5, 30 values rotated 27.8, 23.5; 16 fp32 rows 2.0, 2.6), but not where fp32 goes to 16 bits (60 heads 15.2, 15.0; 12 heads 5.0, 5.5).
template <typename Src, bool E4M3, int ORDER>
inline cudaError_t launch_rope_in(const RopeArgs &a, int n_sm, cudaStream_t st) {
  if constexpr (sizeof(Src) == 2 || E4M3 || ORDER == ROPE_HALF) {
    const long long pieces = (long long)a.R * (a.H + 2 * a.K);
    if (pieces > (long long)rope_ctas<Src, E4M3, ORDER, 256>() * n_sm * RopeShape<Src, 256>::kSlots) return launch_rope_with<Src, E4M3, ORDER, 128>(a, st);
  }
  return launch_rope_with<Src, E4M3, ORDER, 256>(a, st);
}
template <typename Src, bool E4M3>
inline cudaError_t launch_rope_as(const RopeArgs &a, bool neighbours, int n_sm, cudaStream_t st) {
  if (neighbours) return launch_rope_in<Src, E4M3, ROPE_NEIGHBOURS>(a, n_sm, st);
  if (a.pairs % (16 / sizeof(Src)) == 0) return launch_rope_in<Src, E4M3, ROPE_HALVES>(a, n_sm, st);
  return launch_rope_in<Src, E4M3, ROPE_HALF>(a, n_sm, st);
}
inline cudaError_t launch_rope(const RopeArgs &a, bool src_f32, bool e4m3, bool neighbours, int n_sm, cudaStream_t st) {
  if (src_f32) return e4m3 ? launch_rope_as<float, true>(a, neighbours, n_sm, st) : launch_rope_as<float, false>(a, neighbours, n_sm, st);
  return e4m3 ? launch_rope_as<uint16_t, true>(a, neighbours, n_sm, st) : launch_rope_as<uint16_t, false>(a, neighbours, n_sm, st);
}

}  // namespace ttsgpt
