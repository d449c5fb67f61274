// What the entry points of the single-kernel operators check their arguments with.
#pragma once
#include "common.cuh"
#include "host.cuh"
#include "page_tables.cuh"

namespace ttsgpt {

#define OP_TRY(expr)                                                                                   \
  do {                                                                                                 \
    cudaError_t e_ = (expr);                                                                           \
    if (e_ != cudaSuccess) return fail_op(TTS_GPT_E_CUDA, "%s: %s", #expr, cudaGetErrorString(e_));   \
  } while (0)

inline bool aligned(const void *p, size_t n) { return (uintptr_t)p % n == 0; }

// test aid: the CTA of this thread's attention calls whose copies never count as complete, and how long it waits for them
struct Expire { int cta; unsigned long long wait_ns; };
Expire &op_expire();

struct Bytes { const void *p; size_t n; };
inline bool overlap(const Bytes &a, const Bytes &b) {
  return a.p && b.p && a.n && b.n && (uintptr_t)a.p < (uintptr_t)b.p + b.n && (uintptr_t)b.p < (uintptr_t)a.p + a.n;
}
// rows of `width` elements, `stride` apart
inline Bytes rows_of(const void *p, long long rows, long long stride, long long width, size_t size) {
  return {p, rows > 0 ? (size_t)((rows - 1) * stride + width) * size : 0};
}

inline Bytes pool_of(const void *kv_layer, int32_t kv_fmt, int32_t n_pages, int32_t heads) {
  return {kv_layer, (size_t)n_pages * 2 * heads * (kv_fmt == TTS_GPT_KV_BF16 ? (size_t)kPageElems * 2 : (size_t)kE4m3BlockBytes)};
}

}  // namespace ttsgpt
