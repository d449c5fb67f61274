// Single-kernel entry points of a program that decodes several drafted tokens a step over a paged cache: rotary positions on the way
// into the cache, trees of drafted tokens, attention over them, acceptance, and keys and values to where they belong.
#include <algorithm>
#include <cmath>

#include "op_checks.cuh"
#include "rope.cuh"
#include "draft_trees.cuh"
#include "attention_tree.cuh"

using namespace ttsgpt;

namespace {

constexpr long double kTwoPi = 6.28318530717958647692528676655900576839L;

// Do rows of `wa` bytes, `sa` apart, share a byte with others?  Rows of the same distance may lie side by side, as parts of one array.
bool rows_overlap(const void *pa, long long na, long long wa, long long sa, const void *pb, long long nb, long long wb, long long sb) {
  if (na <= 0 || nb <= 0) return false;
  const uintptr_t a = (uintptr_t)pa, b = (uintptr_t)pb;
  if (a >= b + (uintptr_t)((nb - 1) * sb + wb) || b >= a + (uintptr_t)((na - 1) * sa + wa)) return false;
  if (sa != sb || sa <= 0 || wa > sa || wb > sa) return true;
  const uintptr_t d = b >= a ? (b - a) % (uintptr_t)sa : ((uintptr_t)sa - (a - b) % (uintptr_t)sa) % (uintptr_t)sa;   // of b's rows inside a's
  return d < (uintptr_t)wa || d + (uintptr_t)wb > (uintptr_t)sa;
}

// header as in the other attentions' scratch: [error word][tickets]..[parts], so that scratch of either kind serves
constexpr size_t kTreeHeaderBytes = 256 + 16384 * sizeof(unsigned) + align256(4100 * sizeof(int));
size_t tree_scratch_bytes() { return kTreeHeaderBytes + (size_t)tree_part_floats() * sizeof(float); }

struct Named { const char *name; Bytes at; };
// the first of the outputs that shares a byte with an input or another output
template <size_t NO, size_t NI>
const char *shared_bytes(const Named (&out)[NO], const Named (&in)[NI]) {
  for (size_t o = 0; o < NO; ++o) {
    for (size_t i = 0; i < NI; ++i)
      if (overlap(out[o].at, in[i].at)) return out[o].name;
    for (size_t i = 0; i < o; ++i)
      if (overlap(out[o].at, out[i].at)) return out[o].name;
  }
  return nullptr;
}

}  // namespace

extern "C" {

int32_t tts_gpt_op_rope_frequencies(int32_t n_rot, int32_t scaling, double base, double factor, double original, double low, double high, const double *inv_freq,
                                    uint64_t *turns, float *magnitude) {
  if (!turns || !magnitude || n_rot < 2 || n_rot > kHeadDim || n_rot % 2 || scaling < TTS_GPT_ROPE_NONE || scaling > TTS_GPT_ROPE_GIVEN)
    return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: n_rot must be even, 2..%d, and the scaling known", kHeadDim);
  if (scaling == TTS_GPT_ROPE_GIVEN ? !inv_freq : !(std::isfinite(base) && base > 1.0)) return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: base must exceed 1, frequencies be given");
  if (scaling != TTS_GPT_ROPE_NONE && scaling != TTS_GPT_ROPE_GIVEN && !(std::isfinite(factor) && factor >= 1.0))
    return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: factor must be 1 at least");
  if ((scaling == TTS_GPT_ROPE_YARN || scaling == TTS_GPT_ROPE_BANDS) &&
      !(std::isfinite(original) && original > 0.0 && std::isfinite(low) && std::isfinite(high) && low > 0.0 && high > low))
    return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: original must be positive, and 0 < low < high");
  if (scaling == TTS_GPT_ROPE_NTK && n_rot < 4) return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: a base can be raised for 4 values or more");
  // In long double, whose last place is 2^-64 of a value: in double a frequency is off by 2^-53 of itself, some 200 units of the table.
  const int n = n_rot / 2;
  const long double stretch = factor;
  long double from = base;
  if (scaling == TTS_GPT_ROPE_NTK) from *= std::pow(stretch, (long double)n_rot / (n_rot - 2));
  double first = 0.0, last = 0.0;              // of the pairs between which yarn blends: whole numbers
  if (scaling == TTS_GPT_ROPE_YARN) {
    auto pair_of = [&](double rotations) { return n_rot * std::log(original / (rotations * (double)kTwoPi)) / (2.0 * std::log(base)); };   // that turns so often
    first = std::max(std::floor(pair_of(high)), 0.0);
    last = std::min(std::ceil(pair_of(low)), (double)n_rot - 1.0);
    if (last - first < 0.001) last = first + 0.001;
  }
  for (int i = 0; i < n; ++i) {
    long double w = scaling == TTS_GPT_ROPE_GIVEN ? (long double)inv_freq[i] : std::pow(from, -2.0L * i / n_rot);
    if (scaling == TTS_GPT_ROPE_LINEAR) w /= stretch;
    if (scaling == TTS_GPT_ROPE_YARN) {
      const long double slow = std::min(std::max(((long double)i - first) / ((long double)last - first), 0.0L), 1.0L);
      w = w / stretch * slow + w * (1.0L - slow);
    }
    if (scaling == TTS_GPT_ROPE_BANDS) {
      const long double rotations = original * w / kTwoPi;
      const long double fast = std::min(std::max((rotations - low) / ((long double)high - low), 0.0L), 1.0L);   // 0: slow, divided; 1: fast, as it is
      w = w / stretch * (1.0L - fast) + w * fast;
    }
    if (!std::isfinite(w)) return fail_op(TTS_GPT_E_ARG, "op_rope_frequencies: frequency %d is not finite", i);
    const long double t = w / kTwoPi, part = t - std::floor(t);   // turns a position, modulo one
    turns[i] = part >= 1.0L - 0x1p-64L ? 0u : (uint64_t)std::ldexp(part, 64);
  }
  *magnitude = scaling == TTS_GPT_ROPE_YARN ? (float)(0.1 * std::log(factor) + 1.0) : 1.0f;
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_rope_kv_append(int32_t R, int32_t n_head, int32_t n_kv_head, int32_t type, const void *q, int64_t q_stride, const void *k, int64_t k_stride,
                                  const void *v, int64_t v_stride, const int32_t *row_pos, const int32_t *row_slot, int32_t n_rot, const uint64_t *turns,
                                  int32_t interleaved, float magnitude, int32_t out_type, void *q_out, int64_t out_stride, int32_t kv_fmt, int32_t n_pages, void *kv_layer,
                                  void *cuda_stream) {
  const long long qw = (long long)n_head * kHeadDim, kw = (long long)n_kv_head * kHeadDim;
  if (R == 1) { q_stride = out_stride = qw; k_stride = v_stride = kw; }   // the stride of a single row addresses nothing
  if (R < 1 || n_head < 0 || n_kv_head < 1 || (n_head > 0 && (!q || !q_out)) || !k || !v || !row_pos || !row_slot || !turns || !kv_layer || n_pages < 1 ||
      n_pages > INT32_MAX / kPageTokens || (type != TTS_GPT_T_F32 && type != TTS_GPT_T_BF16) || (out_type != TTS_GPT_T_F32 && out_type != TTS_GPT_T_BF16) ||
      (kv_fmt != TTS_GPT_KV_BF16 && kv_fmt != TTS_GPT_KV_FP8_E4M3) || k_stride < kw || v_stride < kw || (n_head > 0 && (q_stride < qw || out_stride < qw)))
    return fail_op(TTS_GPT_E_ARG, "op_rope_kv_append: bad argument");
  if (n_rot < 2 || n_rot > kHeadDim || n_rot % 2) return fail_op(TTS_GPT_E_ARG, "op_rope_kv_append: n_rot must be even, 2..%d", kHeadDim);
  if (!std::isfinite(magnitude)) return fail_op(TTS_GPT_E_ARG, "op_rope_kv_append: magnitude must be finite");
  const int size = type == TTS_GPT_T_F32 ? 4 : 2, out_size = out_type == TTS_GPT_T_F32 ? 4 : 2;
  if (!aligned(k, 16) || !aligned(v, 16) || k_stride * size % 16 || v_stride * size % 16 || !aligned(kv_layer, 16) || !aligned(row_pos, 4) || !aligned(row_slot, 4) ||
      !aligned(turns, 8) || (n_head > 0 && (!aligned(q, 16) || !aligned(q_out, 16) || q_stride * size % 16 || out_stride * out_size % 16)))
    return fail_op(TTS_GPT_E_ARG, "op_rope_kv_append: rows of q, K, V and q_out and the pool must be 16-byte aligned, index arrays 4-byte, turns 8-byte");
  if (n_head > 4096 || n_kv_head > 4096) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_rope_kv_append: at most 4096 heads of either kind");
  const Bytes pool = pool_of(kv_layer, kv_fmt, n_pages, n_kv_head);
  const Bytes index[] = {{row_pos, (size_t)R * 4}, {row_slot, (size_t)R * 4}, {turns, (size_t)n_rot * 4}};
  const Bytes out = n_head > 0 ? rows_of(q_out, R, out_stride, qw, out_size) : Bytes{nullptr, 0};
  bool over = overlap(pool, rows_of(k, R, k_stride, kw, size)) || overlap(pool, rows_of(v, R, v_stride, kw, size)) || overlap(pool, out) ||
              (n_head > 0 && overlap(pool, rows_of(q, R, q_stride, qw, size)));
  for (const Bytes &x : index) over = over || overlap(pool, x) || overlap(out, x);
  if (n_head > 0) {
    over = over || rows_overlap(q_out, R, qw * out_size, out_stride * out_size, k, R, kw * size, k_stride * size) ||
           rows_overlap(q_out, R, qw * out_size, out_stride * out_size, v, R, kw * size, v_stride * size);
    // q_out may be q itself
    if (!(q_out == q && out_type == type && out_stride == q_stride))
      over = over || rows_overlap(q_out, R, qw * out_size, out_stride * out_size, q, R, qw * size, q_stride * size);
  }
  if (over) return fail_op(TTS_GPT_E_ARG, "op_rope_kv_append: the pool or q_out overlaps something else that the call is given");
  RopeArgs a = {};
  a.q = q; a.k = k; a.v = v; a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.out_stride = out_stride;
  a.row_pos = row_pos; a.row_slot = row_slot; a.turns = (const unsigned long long *)turns; a.q_out = q_out; a.pool = (unsigned char *)kv_layer;
  a.R = R; a.H = n_head; a.K = n_kv_head; a.pairs = n_rot / 2; a.n_slots = n_pages * kPageTokens;
  a.out_f32 = out_type == TTS_GPT_T_F32; a.magnitude = magnitude;
  OP_TRY(launch_rope(a, type == TTS_GPT_T_F32, kv_fmt == TTS_GPT_KV_FP8_E4M3, interleaved != 0, device_sms(), (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_tree_tables(int32_t n, int32_t R, const int32_t *row_start, const int32_t *stream_ids, int32_t max_streams, const int32_t *kv_len, const int32_t *parent,
                               int32_t mask_words, int32_t *tree_mask, int32_t *row_pos, int32_t *info, void *cuda_stream) {
  if (n < 1 || R < 1 || !row_start || !kv_len || !parent || !tree_mask || !row_pos || !info || max_streams < 1 || (!stream_ids && n > max_streams) || mask_words < 1)
    return fail_op(TTS_GPT_E_ARG, "op_tree_tables: bad argument");
  const void *all[] = {row_start, stream_ids, kv_len, parent, tree_mask, row_pos, info};
  for (const void *p : all)
    if (!aligned(p, 4)) return fail_op(TTS_GPT_E_ARG, "op_tree_tables: index arrays must be 4-byte aligned");
  if (n > kTreeMaxSeq || mask_words > kTreeWords || max_streams > kTabMaxStreams)
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_tree_tables: at most %d trees of %d nodes, %d streams", kTreeMaxSeq, kTreeNodes, kTabMaxStreams);
  const Named in[] = {{"row_start", {row_start, (size_t)(n + 1) * 4}}, {"stream_ids", {stream_ids, (size_t)n * 4}}, {"kv_len", {kv_len, (size_t)max_streams * 4}}, {"parent", {parent, (size_t)R * 4}}};
  const Named out[] = {{"tree_mask", {tree_mask, (size_t)R * mask_words * 4}}, {"row_pos", {row_pos, (size_t)R * 4}}, {"info", {info, 4}}};
  if (const char *name = shared_bytes(out, in)) return fail_op(TTS_GPT_E_ARG, "op_tree_tables: %s overlaps something else that the call is given", name);
  TreeTableArgs a;
  a.n = n; a.R = R; a.max_streams = max_streams; a.words = mask_words; a.row_start = row_start; a.stream_ids = stream_ids; a.kv_len = kv_len; a.parent = parent;
  a.mask = tree_mask; a.row_pos = row_pos; a.info = info;
  OP_TRY(launch_tree_tables(a, (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_tree_scratch_bytes(size_t *bytes) {
  if (!bytes) return fail_op(TTS_GPT_E_ARG, "op_attention_tree: null argument");
  *bytes = tree_scratch_bytes();
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_attention_tree(int32_t n, int32_t R, int32_t n_head, int32_t n_kv_head, int32_t type, const void *q, int64_t q_stride, int32_t kv_fmt, int32_t n_pages,
                                  const void *kv_layer, int32_t max_streams, const int32_t *page_table, int32_t pages_per_stream, const int32_t *row_start,
                                  const int32_t *stream_ids, const int32_t *kv_len, int32_t mask_words, const int32_t *tree_mask, int32_t t_max, float scale, void *out,
                                  void *scratch, size_t scratch_size, void *cuda_stream) {
  if (n_head < 1 || n_kv_head < 1 || n_head % n_kv_head) return fail_op(TTS_GPT_E_ARG, "op_attention_tree: n_head must be a multiple of n_kv_head");
  if (n_head / n_kv_head > 16 || n_head > 1024) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_tree: at most 16 query heads to a head of keys, and 1024 in all");
  const long long width = (long long)n_head * kHeadDim;
  if (R == 1) q_stride = width;
  if (n < 1 || R < 1 || !q || !kv_layer || !page_table || !row_start || !kv_len || !tree_mask || !out || !scratch || (type != TTS_GPT_T_F32 && type != TTS_GPT_T_BF16) ||
      (kv_fmt != TTS_GPT_KV_BF16 && kv_fmt != TTS_GPT_KV_FP8_E4M3) || n_pages < 1 || max_streams < 1 || (!stream_ids && n > max_streams) || pages_per_stream < 1 ||
      mask_words < 1 || t_max < 1 || q_stride < width || !std::isfinite(scale))
    return fail_op(TTS_GPT_E_ARG, "op_attention_tree: bad argument");
  if (!(scale > 0.f)) return fail_op(TTS_GPT_E_ARG, "op_attention_tree: scale must be positive");
  if (!aligned(q, 16) || q_stride % (type == TTS_GPT_T_F32 ? 4 : 8) || !aligned(kv_layer, 16) || !aligned(out, 16) || !aligned(scratch, 256) || !aligned(page_table, 4) ||
      !aligned(row_start, 4) || !aligned(stream_ids, 4) || !aligned(kv_len, 4) || !aligned(tree_mask, 4))
    return fail_op(TTS_GPT_E_ARG, "op_attention_tree: q rows, out and the KV pool must be 16-byte aligned, scratch 256-byte, index arrays 4-byte");
  t_max = std::min(t_max, R);
  // what ranges are measured in is counted in 31 bits; so are blocks of the pool
  const int G = n_head / n_kv_head;
  const long long tiles = (long long)n_kv_head * (R / (32 / G) + (long long)n), cost = kTrCostTile + pages_per_stream + 1ll;
  if (n > kTrMaxSeq || R >= (1 << 28) || mask_words > kTreeWords * 4 || pages_per_stream > (1 << 24) || tiles * cost >= (1ll << 30) || 2ll * n_pages * n_kv_head >= (1ll << 31))
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_attention_tree: too many trees (%d at most), rows, nodes or pages", kTrMaxSeq);
  if (scratch_size < tree_scratch_bytes()) return fail_op(TTS_GPT_E_WORKSPACE, "op_attention_tree: scratch of %zu bytes, %zu needed", scratch_size, tree_scratch_bytes());
  const Named in[] = {{"q", rows_of(q, R, q_stride, width, type == TTS_GPT_T_F32 ? 4 : 2)}, {"kv_layer", pool_of(kv_layer, kv_fmt, n_pages, n_kv_head)},
                      {"page_table", {page_table, (size_t)max_streams * pages_per_stream * 4}}, {"row_start", {row_start, (size_t)(n + 1) * 4}},
                      {"stream_ids", {stream_ids, (size_t)n * 4}}, {"kv_len", {kv_len, (size_t)max_streams * 4}}, {"tree_mask", {tree_mask, (size_t)R * mask_words * 4}}};
  const Named to[] = {{"out", {out, (size_t)R * width * 2}}, {"scratch", {scratch, tree_scratch_bytes()}}};
  if (const char *name = shared_bytes(to, in)) return fail_op(TTS_GPT_E_ARG, "op_attention_tree: %s overlaps something else that the call is given", name);
  TreeAttnArgs a = {};
  a.q = q; a.out = (uint16_t *)out; a.q_stride = q_stride; a.R = R; a.H = n_head; a.Hkv = n_kv_head; a.G = G;
  a.by_G.set((uint32_t)G);
  a.scale = scale * 1.4426950408889634f;
  a.row_start = row_start; a.stream_ids = stream_ids; a.kv_len = kv_len; a.page_table = page_table; a.mask = tree_mask;
  a.n_seq = n; a.t_max = t_max; a.words = mask_words; a.max_streams = max_streams; a.pps = pages_per_stream; a.n_pages = n_pages;
  a.pool = (const unsigned char *)kv_layer;
  a.err = (int *)scratch;
  a.wait_ns = op_expire().wait_ns; a.starve = op_expire().cta;
  a.tickets = (unsigned *)((char *)scratch + 256);
  a.part = (float *)((char *)scratch + kTreeHeaderBytes);
  const int n_sm = device_sms();
  cudaStream_t st = (cudaStream_t)cuda_stream;
  CUtensorMap map = {};
  const bool f32 = type == TTS_GPT_T_F32;
  if (kv_fmt == TTS_GPT_KV_BF16) {
    OP_TRY(tree_pool_map(&map, kv_layer, (size_t)n_pages * 2 * n_kv_head));
    OP_TRY((f32 ? launch_tree<false, true> : launch_tree<false, false>)(map, a, n_sm, st));
  } else {
    OP_TRY((f32 ? launch_tree<true, true> : launch_tree<true, false>)(map, a, n_sm, st));
  }
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_tree_accept(int32_t n, int32_t R, const int32_t *row_start, const int32_t *stream_ids, const int32_t *draft, const int32_t *target, const int32_t *parent,
                               int32_t max_streams, const int32_t *kv_len, int32_t *kv_len_out, const int32_t *page_table, int32_t pages_per_stream, int32_t n_pages,
                               int32_t *free_pages, const int32_t *free_top, int32_t *free_top_out, int32_t *path, int32_t *n_accepted, int32_t *next_token, int32_t *info,
                               void *cuda_stream) {
  if (n < 1 || R < 1 || !row_start || !draft || !target || !parent || max_streams < 1 || (!stream_ids && n > max_streams) || !kv_len || !kv_len_out || !page_table ||
      pages_per_stream < 1 || n_pages < 1 || n_pages > INT32_MAX / kPageTokens || !free_pages || !free_top || !free_top_out || !path || !n_accepted || !next_token || !info)
    return fail_op(TTS_GPT_E_ARG, "op_tree_accept: bad argument");
  const void *all[] = {row_start, stream_ids, draft, target, parent, kv_len, kv_len_out, page_table, free_pages, free_top, free_top_out, path, n_accepted, next_token, info};
  for (const void *p : all)
    if (!aligned(p, 4)) return fail_op(TTS_GPT_E_ARG, "op_tree_accept: index arrays must be 4-byte aligned");
  if (n > kTreeMaxSeq || max_streams > kTabMaxStreams || pages_per_stream > kTabMaxListPages)
    return fail_op(TTS_GPT_E_UNSUPPORTED, "op_tree_accept: at most %d trees, %d streams, %d pages to a stream", kTreeMaxSeq, kTabMaxStreams, kTabMaxListPages);
  const size_t streams = (size_t)max_streams * 4, rows = (size_t)R * 4, trees = (size_t)n * 4;
  const Bytes in[] = {{kv_len, streams}, {free_top, 4}, {row_start, trees + 4}, {stream_ids, trees}, {draft, rows}, {target, rows}, {parent, rows}, {page_table, streams * pages_per_stream}};
  const Bytes out[] = {{kv_len_out, streams}, {free_top_out, 4}, {free_pages, (size_t)n_pages * 4}, {path, rows}, {n_accepted, trees}, {next_token, trees}, {info, 32}};
  for (int o = 0; o < 7; ++o) {
    for (int i = 0; i < 8; ++i)                // lengths and height may be updated in place
      if (overlap(out[o], in[i]) && !(o < 2 && o == i && out[o].p == in[i].p)) return fail_op(TTS_GPT_E_ARG, "op_tree_accept: an output overlaps an input");
    for (int i = 0; i < o; ++i)
      if (overlap(out[o], out[i])) return fail_op(TTS_GPT_E_ARG, "op_tree_accept: two outputs overlap");
  }
  TreeAcceptArgs a;
  a.n = n; a.R = R; a.max_streams = max_streams; a.pps = pages_per_stream; a.n_pages = n_pages; a.row_start = row_start; a.stream_ids = stream_ids; a.draft = draft;
  a.target = target; a.parent = parent; a.kv_len = kv_len; a.page_table = page_table; a.free_top = free_top; a.free_pages = free_pages; a.kv_len_out = kv_len_out;
  a.free_top_out = free_top_out; a.path = path; a.n_accepted = n_accepted; a.next_token = next_token; a.info = info;
  OP_TRY(launch_tree_accept(a, (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

int32_t tts_gpt_op_kv_move(int32_t n, int32_t R, const int32_t *row_start, const int32_t *path, const int32_t *row_slot, int32_t n_kv_head, int32_t kv_fmt, int32_t n_pages,
                           int32_t n_layers, int64_t layer_bytes, void *kv_layers, void *cuda_stream) {
  if (n < 1 || R < 1 || !row_start || !path || !row_slot || n_kv_head < 1 || (kv_fmt != TTS_GPT_KV_BF16 && kv_fmt != TTS_GPT_KV_FP8_E4M3) || n_pages < 1 ||
      n_pages > INT32_MAX / kPageTokens || n_layers < 1 || !kv_layers)
    return fail_op(TTS_GPT_E_ARG, "op_kv_move: bad argument");
  const Bytes pool = pool_of(kv_layers, kv_fmt, n_pages, n_kv_head);
  if (n_layers == 1) layer_bytes = (int64_t)pool.n;
  if (!aligned(kv_layers, 16) || layer_bytes % 16 || !aligned(row_start, 4) || !aligned(path, 4) || !aligned(row_slot, 4))
    return fail_op(TTS_GPT_E_ARG, "op_kv_move: layers must be 16-byte aligned, index arrays 4-byte");
  if (layer_bytes < (int64_t)pool.n) return fail_op(TTS_GPT_E_ARG, "op_kv_move: layers overlap");
  if (n > (1 << 20) || n_layers > 65535 || n_kv_head > 4096) return fail_op(TTS_GPT_E_UNSUPPORTED, "op_kv_move: at most 2^20 trees, 65535 layers, 4096 heads");
  const Bytes layers = {kv_layers, (size_t)layer_bytes * (n_layers - 1) + pool.n};
  if (overlap(layers, {row_start, (size_t)(n + 1) * 4}) || overlap(layers, {path, (size_t)R * 4}) || overlap(layers, {row_slot, (size_t)R * 4}))
    return fail_op(TTS_GPT_E_ARG, "op_kv_move: the layers overlap the path, the slots or the starts");
  KvMoveArgs a;
  a.n = n; a.R = R; a.K = n_kv_head; a.n_slots = n_pages * kPageTokens; a.layers = n_layers; a.layer_bytes = layer_bytes;
  a.row_start = row_start; a.path = path; a.row_slot = row_slot; a.pool = (unsigned char *)kv_layers;
  OP_TRY(launch_kv_move(a, kv_fmt == TTS_GPT_KV_FP8_E4M3, (cudaStream_t)cuda_stream));
  return TTS_GPT_OK;
}

}  // extern "C"
