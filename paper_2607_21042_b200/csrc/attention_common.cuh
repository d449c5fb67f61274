// What the attention operators share: division by a launch's constants, copies of boxes, 16-bit packing, moves between registers and
// tensor memory, 2^x on the FMA pipes.
#pragma once
#include <cuda.h>
#include <cuda_fp16.h>
#include "common.cuh"
#include "tcgen05.cuh"

namespace ttsgpt {

// Division by a number that is the same throughout a launch, in three instructions and not in the thirty of a general one: code is
// fetched cold in every launch, and these kernels divide in many places.  For 0 <= n < 2^31: with l = ceil(log2 d) and
// m = ceil(2^(31 + l) / d), n / d = floor(n m / 2^(31 + l)) (m d exceeds 2^(31 + l) by less than d <= 2^l).
struct Div {
  uint32_t d, m, s;
  __host__ __device__ void set(uint32_t by) {
    d = by; m = 0; s = 0;
    if (by > 1) {
      uint32_t q = 0x80000000u / by, r = 0x80000000u - q * by, l = 0;   // 2^31 = q d + r, doubled l times
      while ((1u << l) < by) {
        ++l;
        q <<= 1; r <<= 1;
        if (r >= by) { r -= by; ++q; }
      }
      m = q + (r != 0);
      s = l - 1;
    }
  }
  __device__ __forceinline__ int of(int n) const {
#ifdef __CUDA_ARCH__
    return d == 1 ? n : (int)(__umulhi((uint32_t)n, m) >> s);
#else
    return n / (int)d;
#endif
  }
};

__device__ __forceinline__ void un_box(const CUtensorMap *map, int c1, int c2, unsigned char *dst, uint64_t *bar) {
  asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
               ::"r"(smem_u32(dst)), "l"(map), "r"(0), "r"(c1), "r"(c2), "r"(smem_u32(bar)) : "memory");
}
template <bool F16>
__device__ __forceinline__ uint32_t un_pack(float lo, float hi) {
  if constexpr (F16) { const __half2 v = __floats2half2_rn(lo, hi); return *reinterpret_cast<const uint32_t *>(&v); }
  else return pack_bf16x2(lo, hi);
}
// Two e4m3 codes, in the upper bytes of the halves of x (the lower bytes are ignored), as bf16: the bits moved into place are the
// value times 2^-120, exactly (denormals too).  The NaN code reads as 480.
__device__ __forceinline__ uint32_t e4m3x2_to_bf16x2(uint32_t x) {
  const uint32_t y = (x & 0x80008000u) | ((x >> 4) & 0x07F007F0u);
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(y), "r"(0x7B807B80u));   // 2^120
  return r;
}

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

}  // namespace ttsgpt
