// Single-kernel entry points of a program that assembles its own step over a paged cache: page lists and slot maps, K/V rows
// into their slots, attention of a batch that shares a prefix, attention to an encoder's states.  A translation unit of its
// own: the engine's kernels keep their places in its module, which decide how their code is fetched.
#include <algorithm>
#include <cmath>

#include "op_checks.cuh"
#include "attention_tiles.cuh"

using namespace ttsgpt;

Expire &ttsgpt::op_expire() {
  static thread_local Expire e = {-1, kUnWaitNs};
  return e;
}

namespace {

// Scratch of the two attentions: [error word][tickets][plan][partial rows], the first three of the same size in every call, so
// that calls of other sizes, of either kind, find the tickets at zero where the call before left them.
constexpr size_t kOpTicketBytes = kUnTickets * sizeof(unsigned), kOpPlanBytes = align256((kUnMaxSeq + 4) * sizeof(int));
constexpr size_t kOpHeaderBytes = 256 + kOpTicketBytes + kOpPlanBytes;
static_assert(kUnTickets >= kUnMaxWarps && kUnTickets >= kTlTile / 32 * kTlMaxCtas && kUnTickets >= kUnMaxTiles * kUnMaxCtas, "a ticket per range, or per row and group of a call that merges itself");
size_t scratch_bytes(long long part_rows) { return kOpHeaderBytes + (size_t)part_rows * kUnPitch * sizeof(float); }

int check_heads(const char *op, int32_t n_head, int32_t n_kv_head) {
  if (n_head < 1 || n_kv_head < 1 || n_head % n_kv_head) return fail_op(TTS_GPT_E_ARG, "%s: n_head must be a multiple of n_kv_head", op);
  if (n_head / n_kv_head > kUnTile || n_head > 1024)
    return fail_op(TTS_GPT_E_UNSUPPORTED, "%s: at most %d query heads to a head of keys, and 1024 in all", op, kUnTile);
  return TTS_GPT_OK;
}

}  // namespace

extern "C" {

int32_t tts_gpt_debug_expire_op(int32_t cta, uint32_t limit_us) {
  if (cta < -1 || (cta >= 0 && (limit_us < 1 || limit_us > 100000))) return fail_op(TTS_GPT_E_ARG, "expire_op: cta must be -1 or more, limit_us in 1..100000");
  op_expire() = cta >= 0 ? Expire{cta, (unsigned long long)limit_us * 1000ull} : Expire{-1, kUnWaitNs};
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_page_tables(int32_t n, const int32_t *stream_ids, const int32_t *new_len, int32_t max_streams, const int32_t *ctx_len,
                               int32_t *ctx_len_out, int32_t n_pages, const int32_t *free_pages, const int32_t *free_top, int32_t *free_top_out,
                               int32_t n_shared, const int32_t *shared_pages, int32_t pages_per_stream, int32_t *page_table, int32_t max_rows,
                               int32_t *row_start, int32_t *row_stream, int32_t *row_pos, int32_t *row_slot, int32_t *info, void *cuda_stream) {
  if (!new_len || !ctx_len || !ctx_len_out || !free_pages || !free_top || !free_top_out || !page_table || !row_start || !row_stream || !row_pos ||
      !row_slot || !info || (n_shared > 0 && !shared_pages))
    return fail_op(TTS_GPT_E_ARG, "op_page_tables: null argument");
  const void *all[] = {stream_ids, new_len, ctx_len, ctx_len_out, free_pages, free_top, free_top_out, shared_pages, page_table, row_start, row_stream, row_pos,
                       row_slot, info};
  for (const void *p : all)
    if (!aligned(p, 4)) return fail_op(TTS_GPT_E_ARG, "op_page_tables: index arrays must be 4-byte aligned");
  if (n < 1 || max_streams < 1 || (!stream_ids && n > max_streams) || n_pages < 1 || n_pages > INT32_MAX / kPageTokens || max_rows < 1 || n_shared < 0 ||
      pages_per_stream < 1 || n_shared > pages_per_stream)
    return fail_op(TTS_GPT_E_ARG, "op_page_tables: bad argument");
  if (n > kTabMaxRequests || max_streams > kTabMaxStreams || pages_per_stream > kTabMaxListPages)
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_page_tables: at most %d requests, %d streams, %d pages to a stream", kTabMaxRequests, kTabMaxStreams, kTabMaxListPages);
  // CTAs read the inputs while others already write: only ctx_len and free_top may be updated in place
  const size_t streams = (size_t)max_streams * 4, rows = (size_t)max_rows * 4;
  const Bytes in[] = {{ctx_len, streams}, {free_top, 4}, {stream_ids, (size_t)n * 4}, {new_len, (size_t)n * 4}, {free_pages, (size_t)n_pages * 4},
                      {shared_pages, (size_t)n_shared * 4}};
  const Bytes out[] = {{ctx_len_out, streams}, {free_top_out, 4}, {page_table, streams * pages_per_stream}, {row_start, (size_t)(n + 1) * 4}, {row_stream, rows},
                       {row_pos, rows}, {row_slot, rows}, {info, 32}};
  for (int o = 0; o < 8; ++o) {
    for (int i = 0; i < 6; ++i)
      if (overlap(out[o], in[i]) && !(o < 2 && o == i && out[o].p == in[i].p)) return fail_op(TTS_GPT_E_ARG, "op_page_tables: an output overlaps an input");
    for (int i = 0; i < o; ++i)
      if (overlap(out[o], out[i])) return fail_op(TTS_GPT_E_ARG, "op_page_tables: two outputs overlap");
  }
  TableArgs a;
  a.n = n; a.max_streams = max_streams; a.pps = pages_per_stream; a.n_pages = n_pages; a.n_shared = n_shared; a.max_rows = max_rows;
  a.stream_ids = stream_ids; a.new_len = new_len; a.ctx_len = ctx_len; a.free_pages = free_pages; a.free_top = free_top; a.shared_pages = shared_pages;
  a.ctx_len_out = ctx_len_out; a.free_top_out = free_top_out; a.page_table = page_table; a.row_start = row_start; a.row_stream = row_stream;
  a.row_pos = row_pos; a.row_slot = row_slot; a.info = info;
  a.in_place = ctx_len_out == ctx_len || free_top_out == free_top;
  OP_TRY(launch_page_tables(a, device_sms(), (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_kv_append(int32_t R, int32_t n_head, int32_t type, const void *k, int64_t k_stride, const void *v, int64_t v_stride,
                             const int32_t *row_slot, int32_t kv_fmt, int32_t n_pages, void *kv_layer, void *cuda_stream) {
  if (R == 1) k_stride = v_stride = (int64_t)n_head * kHeadDim;   // the stride of a single row addresses nothing
  if (R < 1 || n_head < 1 || !k || !v || !row_slot || !kv_layer || n_pages < 1 || n_pages > INT32_MAX / kPageTokens || (type != TTS_GPT_T_F32 && type != TTS_GPT_T_BF16) ||
      (kv_fmt != TTS_GPT_KV_BF16 && kv_fmt != TTS_GPT_KV_FP8_E4M3) || k_stride < (int64_t)n_head * kHeadDim || v_stride < (int64_t)n_head * kHeadDim)
    return fail_op(TTS_GPT_E_ARG, "op_kv_append: bad argument");
  const int per16 = type == TTS_GPT_T_F32 ? 4 : 8;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride % per16 || v_stride % per16 || !aligned(kv_layer, 16) || !aligned(row_slot, 4))
    return fail_op(TTS_GPT_E_ARG, "op_kv_append: K and V rows and the pool must be 16-byte aligned, slots 4-byte");
  if ((long long)R * n_head >= (1ll << 29)) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_kv_append: R * n_head must be below 2^29");
  const size_t size = type == TTS_GPT_T_F32 ? 4 : 2;
  const Bytes pool = pool_of(kv_layer, kv_fmt, n_pages, n_head);
  if (overlap(pool, rows_of(k, R, k_stride, (long long)n_head * kHeadDim, size)) || overlap(pool, rows_of(v, R, v_stride, (long long)n_head * kHeadDim, size)) ||
      overlap(pool, {row_slot, (size_t)R * 4}))
    return fail_op(TTS_GPT_E_ARG, "op_kv_append: K, V or the slots overlap the pool");
  AppendArgs a;
  a.k = k; a.v = v; a.k_stride = k_stride; a.v_stride = v_stride; a.row_slot = row_slot; a.pool = (unsigned char *)kv_layer;
  a.R = R; a.H = n_head; a.n_slots = n_pages * kPageTokens;
  OP_TRY(launch_kv_append(a, type == TTS_GPT_T_F32, kv_fmt == TTS_GPT_KV_FP8_E4M3, device_sms(), (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

static int check_shared(int32_t R, int32_t n_head, int32_t n_kv_head) {
  if (const int rc = check_heads("op_attention_shared", n_head, n_kv_head)) return rc;
  if (R < 1) return fail_op(TTS_GPT_E_ARG, "op_attention_shared: R must be positive");
  if (R > kUnMaxSeq) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_shared: at most %d rows", kUnMaxSeq);
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_shared_scratch_bytes(int32_t R, int32_t n_head, int32_t n_kv_head, size_t *bytes) {
  if (!bytes) return fail_op(TTS_GPT_E_ARG, "op_attention_shared: null argument");
  if (const int rc = check_shared(R, n_head, n_kv_head)) return rc;
  *bytes = scratch_bytes(shared_part_rows(R, n_kv_head, n_head / n_kv_head));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_shared(int32_t R, int32_t n_head, int32_t n_kv_head, int32_t type, const void *q, int64_t q_stride, int32_t kv_fmt,
                                    int32_t n_pages, const void *kv_layer, int32_t n_shared, const int32_t *page_table, int32_t pages_per_stream,
                                    const int32_t *row_stream, const int32_t *row_pos, void *out, void *scratch, size_t scratch_size, void *cuda_stream) {
  if (const int rc = check_shared(R, n_head, n_kv_head)) return rc;
  if (R == 1) q_stride = (int64_t)n_head * kHeadDim;
  if (!q || !kv_layer || !page_table || !row_stream || !row_pos || !out || !scratch || (type != TTS_GPT_T_F32 && type != TTS_GPT_T_BF16) ||
      (kv_fmt != TTS_GPT_KV_BF16 && kv_fmt != TTS_GPT_KV_FP8_E4M3) || n_pages < 1 || pages_per_stream < 1 || n_shared < 0 || n_shared > pages_per_stream ||
      q_stride < (int64_t)n_head * kHeadDim)
    return fail_op(TTS_GPT_E_ARG, "op_attention_shared: bad argument");
  if (!aligned(q, 16) || q_stride % (type == TTS_GPT_T_F32 ? 4 : 8) || !aligned(kv_layer, 16) || !aligned(out, 16) || !aligned(scratch, 256) ||
      !aligned(page_table, 4) || !aligned(row_stream, 4) || !aligned(row_pos, 4))
    return fail_op(TTS_GPT_E_ARG, "op_attention_shared: q rows, out and the KV pool must be 16-byte aligned, scratch 256-byte, index arrays 4-byte");
  // units of 32 keys are numbered in 31 bits, one of them for what a division rounds up; blocks of the pool too
  const int G = n_head / n_kv_head;
  const long long tiles = (long long)n_kv_head * ((R + kUnTile / G - 1) / (kUnTile / G));
  const long long units = tiles * (2ll * n_shared + 1) + (long long)R * n_kv_head * (2ll * (pages_per_stream - n_shared) + 1);
  if (pages_per_stream > (1 << 24) || units >= (1ll << 30) ||
      2ll * n_pages * n_kv_head >= (1ll << 31))
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_shared: too many pages");
  if (scratch_size < scratch_bytes(shared_part_rows(R, n_kv_head, G)))
    return fail_op(TTS_GPT_E_WORKSPACE, "op_attention_shared: scratch of %zu bytes, %zu needed", scratch_size, scratch_bytes(shared_part_rows(R, n_kv_head, G)));
  const Bytes to = {out, (size_t)R * n_head * kHeadDim * 2}, own = {scratch, scratch_bytes(shared_part_rows(R, n_kv_head, G))};
  // (of the page lists, whose number the call does not know, the first)
  const Bytes read[] = {rows_of(q, R, q_stride, (long long)n_head * kHeadDim, type == TTS_GPT_T_F32 ? 4 : 2), pool_of(kv_layer, kv_fmt, n_pages, n_kv_head),
                        {page_table, (size_t)pages_per_stream * 4}, {row_stream, (size_t)R * 4}, {row_pos, (size_t)R * 4}};
  for (const Bytes &x : read)
    if (overlap(to, x) || overlap(own, x))
      return fail_op(TTS_GPT_E_ARG, "op_attention_shared: out or scratch overlaps q, the pool, the page lists or the rows' streams and positions");
  if (overlap(to, own)) return fail_op(TTS_GPT_E_ARG, "op_attention_shared: out and scratch overlap");
  UnitArgs a = {};
  a.q = q; a.out = (uint16_t *)out; a.q_stride = q_stride; a.q_rows = R;
  a.set_heads(n_head, n_kv_head, kUnTile / G);
  a.set_shared(n_shared);
  a.scale = 0.125f * 1.4426950408889634f;
  a.page_table = page_table; a.row_stream = row_stream; a.row_pos = row_pos; a.pool = (const unsigned char *)kv_layer; a.pps = pages_per_stream;
  a.n_pages = n_pages;
  a.err = (int *)scratch;
  a.wait_ns = op_expire().wait_ns; a.starve = op_expire().cta;
  a.plan = (int *)((char *)scratch + 256 + kOpTicketBytes);
  a.part = (float *)((char *)scratch + kOpHeaderBytes);
  a.suffix_part0 = (int)shared_prefix_part_rows(R, n_kv_head, G);
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int n_sm = device_sms();
  // One kernel where no CTA can have more tiles than it has room to merge (at most a unit a range more than its share).
  a.tickets = units <= (long long)(kUnMaxTiles - kUnWarps) * std::min(n_sm, kUnMaxCtas) ? (unsigned *)((char *)scratch + 256) : nullptr;
  CUtensorMap map = {};
  if (kv_fmt == TTS_GPT_KV_BF16) {
    OP_TRY(units_pool_map(&map, kv_layer, (size_t)n_pages * 2 * n_kv_head));
    OP_TRY((type == TTS_GPT_T_F32 ? launch_units_as<true, KV_BF16, true> : launch_units_as<true, KV_BF16, false>)(map, map, a, n_sm, st));
  } else {
    OP_TRY((type == TTS_GPT_T_F32 ? launch_units_as<true, KV_E4M3, true> : launch_units_as<true, KV_E4M3, false>)(map, map, a, n_sm, st));
  }
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_cross_scratch_bytes(size_t *bytes) {
  if (!bytes) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: null argument");
  *bytes = scratch_bytes(std::max(cross_part_rows(), tiles_part_rows()));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_cross(int32_t n, int32_t n_head, int32_t n_kv_head, int32_t type, int32_t q_rows, const void *q, int64_t q_stride,
                                   int32_t k_rows, const void *k, int64_t k_stride, int64_t k_head_stride, const void *v, int64_t v_stride,
                                   int64_t v_head_stride, const int32_t *q_start, const int32_t *k_start, int32_t q_max, float scale, void *out,
                                   void *scratch, size_t scratch_size, void *cuda_stream) {
  if (const int rc = check_heads("op_attention_cross", n_head, n_kv_head)) return rc;
  if (q_rows == 1) q_stride = (int64_t)n_head * kHeadDim;
  if (k_rows <= 1) k_stride = v_stride = kHeadDim;
  if (n_kv_head == 1) k_head_stride = v_head_stride = kHeadDim;
  if (n < 1 || q_rows < 1 || k_rows < 0 || q_max < 1 || !q || (k_rows > 0 && (!k || !v)) || !q_start || !k_start || !out || !scratch ||
      (type != TTS_GPT_T_BF16 && type != TTS_GPT_T_F16) || q_stride < (int64_t)n_head * kHeadDim || !std::isfinite(scale))
    return fail_op(TTS_GPT_E_ARG, "op_attention_cross: bad argument");
  if (!(scale > 0.f)) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: scale must be positive");
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(out, 16) || !aligned(scratch, 256) || !aligned(q_start, 4) || !aligned(k_start, 4) || q_stride % 8 ||
      k_stride % 8 || v_stride % 8 || k_head_stride % 8 || v_head_stride % 8)
    return fail_op(TTS_GPT_E_ARG, "op_attention_cross: rows of q, K, V and out must be 16-byte aligned, scratch 256-byte, index arrays 4-byte");
  if (k_stride < kHeadDim || v_stride < kHeadDim) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: rows of K or V overlap");
  if (k_rows > 0 && (k_head_stride < kHeadDim || v_head_stride < kHeadDim)) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: heads of K or V overlap");
  if (n > kUnMaxSeq) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_cross: at most %d sequences", kUnMaxSeq);
  if (q_rows >= (1 << 30) || k_rows >= (1 << 30)) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_cross: rows must be below 2^30");
  if (q_max > q_rows) q_max = q_rows;
  const int G = n_head / n_kv_head;
  // Up to two tiles of 16 read K and V at most twice; more rows take a tile of 256, which reads them once (us, 16 sequences of 90 to 1500 keys
  // by 20 heads, warp-level / tcgen05: 20 queries 27 / 32, 32 queries 30 / 33, 48 queries 35 / 33, 128 queries 63 / 35; four heads of
  // keys, 7 queries of 5 heads each 18 / 16), where there are keys to read: a block has 128 (30 sequences by 20 heads: 100 to 400 queries
  // by 100 to 120 keys 50 / 40, by 60 to 70 keys 39 / 39; 40 to 100 queries by 60 to 70 keys 23 / 27, by 10 to 20 keys 10 / 27).
  // The choice is the call's, not a sequence's: 127 sequences of one query by 100 to 1360 keys and one of 700 by 700 take 181 us on tiles
  // together, 106 (warp-level) and 22 (tiles) in two calls.
  const bool tiles = (long long)q_max * G > 2 * kUnTile && k_rows > 64ll * n && n <= kTlMaxSeq;
  // units of keys are numbered in 31 bits, one of them for what a division rounds up; blocks by their cost
  const int rpt = tiles ? 2 * (kTlRows / G) : kUnTile / G, keys = tiles ? kTlKeys : kUnKeys;
  const long long limit = (1ll << 30) / (tiles ? kTlCost2 : 1);
  const long long blocks = std::min((long long)n * ((q_max + rpt - 1) / rpt), (long long)q_rows / rpt + n);
  if ((long long)n_kv_head * blocks * ((long long)k_rows / keys + 2) >= limit &&
      (long long)n_kv_head * ((q_max + rpt - 1) / rpt) * ((long long)k_rows / keys + 2 * n) >= limit)
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_cross: too many queries times keys");
  if (scratch_size < scratch_bytes(std::max(cross_part_rows(), tiles_part_rows())))
    return fail_op(TTS_GPT_E_WORKSPACE, "op_attention_cross: scratch of %zu bytes, %zu needed", scratch_size, scratch_bytes(std::max(cross_part_rows(), tiles_part_rows())));
  const Bytes to = {out, (size_t)q_rows * n_head * kHeadDim * 2}, own = {scratch, scratch_bytes(std::max(cross_part_rows(), tiles_part_rows()))};
  const Bytes read[] = {rows_of(q, q_rows, q_stride, (long long)n_head * kHeadDim, 2), rows_of(k, k_rows, k_stride, (n_kv_head - 1) * k_head_stride + kHeadDim, 2),
                        rows_of(v, k_rows, v_stride, (n_kv_head - 1) * v_head_stride + kHeadDim, 2), {q_start, (size_t)(n + 1) * 4}, {k_start, (size_t)(n + 1) * 4}};
  for (const Bytes &x : read)
    if (overlap(to, x) || overlap(own, x)) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: out or scratch overlaps q, K, V or the starts");
  if (overlap(to, own)) return fail_op(TTS_GPT_E_ARG, "op_attention_cross: out and scratch overlap");
  UnitArgs a = {};
  a.q = q; a.out = (uint16_t *)out; a.q_stride = q_stride; a.q_rows = q_rows;
  a.set_heads(n_head, n_kv_head, rpt);
  a.scale = scale * 1.4426950408889634f;
  a.q_start = q_start; a.k_start = k_start; a.n_seq = n; a.q_max = q_max; a.k_rows = k_rows;
  // a warp a row merges where tiles have few rows, or many parts since there are few tiles (us: 20 tiles of 47 units 15, a quarter of a
  // warp a row 19; 64 tiles 17.6 and 18.7; 160 tiles 24.6 and 23.3)
  const int n_sm = device_sms();
  a.few_rows = (long long)q_max * G <= 4 || n_kv_head * blocks * 16 <= (long long)std::min(n_sm, kUnMaxCtas) * kUnWarps;
  a.err = (int *)scratch;
  a.wait_ns = op_expire().wait_ns; a.starve = op_expire().cta;
  a.tickets = (unsigned *)((char *)scratch + 256);
  a.part = (float *)((char *)scratch + kOpHeaderBytes);
  CUtensorMap k_map = {}, v_map = {};
  const bool f16 = type == TTS_GPT_T_F16;
  if (k_rows > 0) {
    OP_TRY(units_rows_map(&k_map, f16, k, n_kv_head, k_rows, k_head_stride * 2, k_stride * 2, tiles ? kTlKeys : kUnBox));
    OP_TRY(units_rows_map(&v_map, f16, v, n_kv_head, k_rows, v_head_stride * 2, v_stride * 2, tiles ? kTlKeys : kUnBox));
  }
  if (tiles) {
    CUtensorMap q_map;
    OP_TRY(tiles_q_map(&q_map, f16, q, n_head, q_rows, q_stride * 2, G, rpt / 2));
    OP_TRY((f16 ? launch_tiles_as<true> : launch_tiles_as<false>)(q_map, k_map, v_map, a, n_sm, (cudaStream_t)cuda_stream));
    return TTS_GPT_OK;
  }
  OP_TRY((f16 ? launch_units_as<false, KV_F16, false> : launch_units_as<false, KV_BF16, false>)(k_map, v_map, a, n_sm, (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

}  // extern "C"
