// plan_answers.cpp -- argument checks and work plans of the operators for several answers
// of one prompt.  Pure host arithmetic, no HIP call: every error path runs on a
// machine without a GPU.
#include <limits.h>

#include <algorithm>

#include "answers.h"

namespace md {

namespace {

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

typedef __int128 wide;  // byte spans of any sizes

// Whether [a, a + n) and [b, b + m) share a byte.
bool overlap(const void* a, wide n, const void* b, wide m) {
  const wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && n && m && x < y + m && y < x + n;
}

struct Span {
  const void* p;
  wide bytes;
};
// Whether an output shares memory with an input or with another output.
template <int O, int I>
bool outputs_overlap(const Span (&out)[O], const Span (&in)[I]) {
  for (int i = 0; i < O; ++i) {
    for (const Span& x : in)
      if (overlap(out[i].p, out[i].bytes, x.p, x.bytes)) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return true;
  }
  return false;
}

// The geometry of K and V that a call reads up to max_len tokens of.
struct KvGeom {
  int64_t s_blk, s_tok, s_head;
  int32_t page_size, max_pages;
  int64_t num_pages;
  int32_t max_len;
};

int check_kv_geom(const KvGeom& g) {
  if (g.page_size < 0 || g.s_blk < 0 || g.s_tok < 0 || g.s_head < 0) return MD_ERR_INVALID_ARG;
  if (g.page_size) {
    if ((g.page_size & (g.page_size - 1)) || g.max_pages < 1 || g.num_pages < 1 ||
        g.num_pages > INT32_MAX || ceil_div(g.max_len, g.page_size) > g.max_pages)
      return MD_ERR_INVALID_ARG;
  }
  return MD_OK;
}

// Rows on 16-byte boundaries that do not run into the next head's.
bool rows_ok(const KvGeom& g, int32_t heads, int32_t d, int32_t dtype) {
  const int64_t per16 = dtype == MD_BF16 ? 8 : 4;
  return !(g.s_blk % per16 || g.s_tok % per16 || g.s_head % per16) &&
         (heads == 1 || g.s_head >= d);
}

KvGeom geom(const md_attn_args* a) {
  return {a->kv_stride_blk, a->kv_stride_tok,     a->kv_stride_head, a->page_size,
          a->max_pages_per_seq, a->num_pages, a->max_kv_len};
}
KvGeom geom(const md_prefix* p) {
  return {p->kv_stride_blk, p->kv_stride_tok,        p->kv_stride_head, p->page_size,
          p->max_pages_per_prefix, p->num_pages, p->max_len};
}
KvGeom geom(const md_kv_mass_args* a) {
  return {a->kv_stride_blk, a->kv_stride_tok,     a->kv_stride_head, a->page_size,
          a->max_pages_per_seq, a->num_pages, a->max_kv_len};
}

bool valid_dtype(int32_t t) { return t == MD_F32 || t == MD_BF16; }

}  // namespace

// ---- attention over a shared prefix ----

int check_prefix_sizes(const md_attn_args* a, const md_prefix* p) {
  if (!a || !p) return MD_ERR_INVALID_ARG;
  if (p->num_prefixes < 1 || a->num_seqs % p->num_prefixes || p->max_len < 0 ||
      !valid_dtype(a->dtype))
    return MD_ERR_INVALID_ARG;
  const int st = check_attn_sizes(a);
  if (st == MD_ERR_INVALID_ARG) return st;
  const int own = check_kv_geom(geom(a)), pre = check_kv_geom(geom(p));
  if (own != MD_OK || pre != MD_OK) return MD_ERR_INVALID_ARG;
  if (st != MD_OK) return st;
  if (p->kv_stride_tok > kMaxTokStride || p->max_len > kMaxPosition) return MD_ERR_UNSUPPORTED;
  // Workgroups, and rows of a group, in 32 bits at any split.
  const int64_t rows = static_cast<int64_t>(a->num_seqs) * a->q_len * a->num_q_heads;
  const int64_t units = static_cast<int64_t>(a->num_seqs) * a->num_kv_heads;
  if (rows > INT32_MAX || units > kMaxWgs256 / 64) return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

PrefixPlan make_prefix_plan(const md_attn_args* a, const md_prefix* p, int num_cus) {
  PrefixPlan pl;
  const int64_t cus = num_cus > 0 ? num_cus : 256;
  const int64_t G = a->num_q_heads / a->num_kv_heads;
  pl.n_rows = static_cast<int64_t>(a->num_seqs) * a->q_len * a->num_q_heads;
  pl.group_rows = static_cast<int32_t>(a->num_seqs / p->num_prefixes * a->q_len * G);
  // The wide kernel where its workgroups, one a compute unit, have tiles enough to start and end for.  (8 heads
  // over 32768 tokens, a call: 160 rows 65 us streamed and 68 wide, 192 rows 72 and 70, 256 rows 87 and 73.
  // Over 4096: 256 rows 32 and 39, 512 rows 43 and 49.)
  const int64_t heads = static_cast<int64_t>(p->num_prefixes) * a->num_kv_heads;
  pl.wide = a->dtype == MD_BF16 && pl.group_rows > kPrefixFewRows &&
            heads * ceil_div(pl.group_rows, kPrefixWideRows) * p->max_len >= kPrefixWideTokens * cus &&
            (p->page_size == 0 || p->page_size >= kPrefixWidePage(a->head_dim));
  // (Workgroups of 128 rows, two waves with a half of each tile's keys, where the last one of 256 is half empty: 320
  // rows a call over 16384 and 32768 tokens 66 and 99 us for 65 and 98, 576 rows 95 and 148 for 92 and 144, 832 rows
  // 129 and 209 for 113 and 179; 64 channels at best 2% less.)
  pl.row_blocks = static_cast<int32_t>(ceil_div(pl.group_rows, pl.wide ? kPrefixWideRows : kPrefixStreamRows));
  pl.own_blocks = static_cast<int32_t>(ceil_div(G * a->q_len, kPrefixStreamRows));
  const int64_t units = heads * pl.row_blocks;
  const int64_t own = static_cast<int64_t>(a->num_seqs) * a->num_kv_heads * pl.own_blocks;
  // Parts of a range: as many workgroups as the device has places (two a compute unit; one of the wide kernel
  // and, by its registers, of fp32 with 128 channels: 4 sequences over 32768 tokens 79 us so, 95 with
  // two), of 256 tokens, two tiles a wave, at least; 128 up to one a compute unit.
  // (8 sequences of 8 heads over a prefix of 8192: 15.5 us in 16 or 32 parts, 20 in 8, 21 in 64; 2 heads
  // over one of 512, fp32: 8.6 us in 4 parts, 10.9 in 2.  Own caches, 64 x 4 heads of 1024 tokens: 26 us in
  // 1 part, 28 in 2, 35 in 4; 64 x 8: 38, 37, 44.)
  const bool big = a->dtype == MD_F32 && a->head_dim == 128;
  auto parts = [cus, big](int64_t len, int64_t n, bool wide) {
    const int64_t once = std::max<int64_t>(cus / std::max<int64_t>(n, 1), 1);
    const int64_t twice = std::max<int64_t>((wide || big ? 1 : 2) * cus / std::max<int64_t>(n, 1), 1);
    return static_cast<int32_t>(std::max<int64_t>(
        1, std::max(std::min(once, ceil_div(len, 128)), std::min(twice, ceil_div(len, 256)))));
  };
  pl.c_pre = parts(p->max_len, units, pl.wide);
  pl.c_own = parts(a->max_kv_len, own, false);
  pl.n_pre = static_cast<int32_t>(ceil_div(heads * pl.c_pre, 8) * 8 * pl.row_blocks);
  if (p->max_len == 0) pl.c_pre = pl.n_pre = 0;
  pl.pre_parts = pl.c_pre * PrefixPlan::split;
  pl.n_own = ceil_div(static_cast<int64_t>(a->num_seqs) * pl.c_own, 8) * 8 * a->num_kv_heads * pl.own_blocks;
  const size_t n = static_cast<size_t>(pl.pre_parts + pl.c_own) * static_cast<size_t>(pl.n_rows);
  pl.part_o_bytes = align_up(n * a->head_dim * 4, 256);
  pl.part_lse_bytes = align_up(n * 4, 256);
  pl.workspace_bytes = pl.part_o_bytes + pl.part_lse_bytes;
  return pl;
}

size_t prefix_workspace_need(const md_attn_args* a, const md_prefix* p, int num_cus) {
  return make_prefix_plan(a, p, num_cus).workspace_bytes;
}

int validate_prefix(const md_attn_args* a, const md_prefix* p, PrefixPlan* plan) {
  const int st = check_prefix_sizes(a, p);
  if (st != MD_OK || a->num_seqs == 0) return st;
  if (!a->q || !a->k || !a->v || !a->o || !a->kv_lens || !p->lens) return MD_ERR_INVALID_ARG;
  if (p->max_len > 0 && (!p->k || !p->v)) return MD_ERR_INVALID_ARG;
  if ((a->page_size != 0) != (a->page_table != nullptr) ||
      (p->page_size != 0) != (p->page_table != nullptr))
    return MD_ERR_INVALID_ARG;
  for (const void* x : {a->q, a->k, a->v, static_cast<const void*>(a->o), p->k, p->v})
    if (!aligned(x, 16)) return MD_ERR_INVALID_ARG;
  if (!aligned(a->kv_lens, 4) || !aligned(a->lse, 4) || !aligned(a->page_table, 4) ||
      !aligned(a->err_word, 4) || !aligned(p->lens, 4) || !aligned(p->page_table, 4))
    return MD_ERR_INVALID_ARG;
  if (!rows_ok(geom(a), a->num_kv_heads, a->head_dim, a->dtype) ||
      !rows_ok(geom(p), a->num_kv_heads, a->head_dim, a->dtype))
    return MD_ERR_INVALID_ARG;
  *plan = make_prefix_plan(a, p, device_cu_count());
  if (plan->n_pre + plan->n_own > kMaxWgs256) return MD_ERR_UNSUPPORTED;
  if (!a->workspace || a->workspace_bytes < plan->workspace_bytes || !aligned(a->workspace, 256))
    return MD_ERR_WORKSPACE;
  return MD_OK;
}

// ---- accumulated weights ----

int check_mass_sizes(const md_kv_mass_args* a) {
  if (!a || a->num_seqs < 0 || a->q_len < 1 || a->num_q_heads < 1 || a->num_kv_heads < 1 ||
      a->num_q_heads % a->num_kv_heads || a->head_dim < 1 || !valid_dtype(a->dtype) ||
      a->max_kv_len < a->q_len || a->slot_stride < a->max_kv_len)
    return MD_ERR_INVALID_ARG;
  if (check_kv_geom(geom(a)) != MD_OK) return MD_ERR_INVALID_ARG;
  if (a->head_dim != 64 && a->head_dim != 128) return MD_ERR_UNSUPPORTED;
  // (Key blocks of 256 may end past the last token.)
  if (a->kv_stride_tok > kMaxTokStride || a->max_kv_len > INT32_MAX - kMassPromptKeys)
    return MD_ERR_UNSUPPORTED;
  const int64_t G = a->num_q_heads / a->num_kv_heads;
  if (G * a->q_len > (1 << 30)) return MD_ERR_UNSUPPORTED;
  const int64_t units = static_cast<int64_t>(a->num_seqs) * a->num_kv_heads;
  if (units > kMaxWgs256 || units * ceil_div(a->max_kv_len, 128) > kMaxWgs256)
    return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

MassPlan make_mass_plan(const md_kv_mass_args* a, int num_cus) {
  MassPlan pl;
  const int64_t cus = num_cus > 0 ? num_cus : 256;
  const int64_t units = static_cast<int64_t>(a->num_seqs) * a->num_kv_heads;
  const int64_t rows = static_cast<int64_t>(a->num_q_heads / a->num_kv_heads) * a->q_len;
  pl.prompt = rows > kMassStepRows;
  if (!pl.prompt) {
    // Enough workgroups for the device's places, two a compute unit; a tile of 32 keys a wave at least.
    // (64 x 8 heads of 2054 tokens: 52 us whole, 59 in two parts, 61 in four.)
    pl.key_parts = static_cast<int32_t>(std::max<int64_t>(
        1, std::min(2 * cus / std::max<int64_t>(units, 1), ceil_div(a->max_kv_len, 128))));
    // Whole rounds of the XCDs, which take all heads of a part (see kv_mass.hip).
    pl.n_wgs = ceil_div(static_cast<int64_t>(a->num_seqs) * pl.key_parts, 8) * 8 * a->num_kv_heads;
    return pl;
  }
  // A unit's key blocks go in pairs, the i-th with the i-th from the end: in a prompt, where later keys
  // have fewer rows, all pairs have as many (kv_mass.hip).  Their rows are cut into parts that fill the
  // device's places (two workgroups a compute unit) once, or, where that would leave an eighth of them
  // empty, about four times; 256 rows of a pair at least.
  const int64_t pairs = units * ceil_div(ceil_div(a->max_kv_len, kMassPromptKeys), 2);
  const int64_t places = 2 * cus, once = places / pairs;
  const int64_t parts = pairs * once * 8 >= places * 7 ? once : ceil_div(4 * places, pairs);
  pl.row_parts = static_cast<int32_t>(std::max<int64_t>(1, std::min(parts, ceil_div(rows, 256))));
  pl.n_wgs = pairs * pl.row_parts;
  pl.reduce_wgs = units * ceil_div(a->max_kv_len, 256);
  if (pl.row_parts > 1)
    pl.workspace_bytes = align_up(static_cast<size_t>(pl.row_parts) * units * a->max_kv_len * 4, 256);
  return pl;
}

int validate_mass(const md_kv_mass_args* a, MassPlan* plan) {
  const int st = check_mass_sizes(a);
  if (st != MD_OK || a->num_seqs == 0) return st;
  if (!a->q || !a->k || !a->kv_lens || !a->lse || !a->pos0 || !a->mass || !a->slot_pos)
    return MD_ERR_INVALID_ARG;
  if ((a->page_size != 0) != (a->page_table != nullptr)) return MD_ERR_INVALID_ARG;
  if (!aligned(a->q, 16) || !aligned(a->k, 16)) return MD_ERR_INVALID_ARG;
  for (const void* x : {static_cast<const void*>(a->kv_lens), static_cast<const void*>(a->lse),
                        static_cast<const void*>(a->accepted), static_cast<const void*>(a->pos0),
                        static_cast<const void*>(a->mass), static_cast<const void*>(a->slot_pos),
                        static_cast<const void*>(a->page_table)})
    if (!aligned(x, 4)) return MD_ERR_INVALID_ARG;
  if (!rows_ok(geom(a), a->num_kv_heads, a->head_dim, a->dtype)) return MD_ERR_INVALID_ARG;
  *plan = make_mass_plan(a, device_cu_count());
  // (The launches as they are padded, which the count of units above does not bound.)
  if (plan->n_wgs > kMaxWgs256 || plan->reduce_wgs > kMaxWgs256) return MD_ERR_UNSUPPORTED;
  if (plan->workspace_bytes && (!a->workspace || a->workspace_bytes < plan->workspace_bytes ||
                                !aligned(a->workspace, 256)))
    return MD_ERR_WORKSPACE;
  const wide B = a->num_seqs, es = a->dtype == MD_BF16 ? 2 : 4;
  const wide rows = B * a->q_len * a->num_q_heads, slots = B * a->num_kv_heads * a->slot_stride * 4;
  const wide blocks = a->page_size ? static_cast<wide>(a->num_pages) : B;
  const wide toks = a->page_size ? a->page_size : a->max_kv_len;
  const Span out[] = {{a->mass, slots}, {a->slot_pos, slots},
                      {a->workspace, static_cast<wide>(plan->workspace_bytes)}};
  const Span in[] = {{a->q, rows * a->head_dim * es}, {a->lse, rows * 4}, {a->kv_lens, B * 4},
                     {a->accepted, B * 4}, {a->pos0, B * 4},
                     {a->page_table, B * a->max_pages_per_seq * 4},
                     {a->k, ((blocks - 1) * a->kv_stride_blk + (toks - 1) * a->kv_stride_tok +
                             (a->num_kv_heads - 1) * static_cast<wide>(a->kv_stride_head) +
                             a->head_dim) * es}};
  return outputs_overlap(out, in) ? MD_ERR_INVALID_ARG : MD_OK;
}

// ---- eviction ----

int check_evict_sizes(const md_kv_cache* c, int64_t slot_stride, int32_t budget) {
  const int st = validate_kv_cache(c, 0);
  if (st != MD_OK) return st;
  if (slot_stride < 1 || budget < 1 || c->num_pages > INT32_MAX) return MD_ERR_INVALID_ARG;
  const int64_t heads = c->num_kv_heads;
  if (heads > 1 && c->kv_stride_head < c->head_dim) return MD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return MD_ERR_UNSUPPORTED;
  // (A thread's slots go on by up to 1024.)
  if (slot_stride > INT32_MAX - 2048 || static_cast<int64_t>(c->num_seqs) * heads > kMaxWgs1024)
    return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

EvictPlan make_evict_plan(const md_kv_cache* c, int64_t slot_stride, int32_t budget) {
  EvictPlan pl;
  const int64_t held = c->page_size ? static_cast<int64_t>(c->max_pages_per_seq) * c->page_size
                                    : c->capacity;
  pl.slots = std::min(held, slot_stride);
  pl.max_moves = static_cast<int32_t>(std::max<int64_t>(
      0, std::min<int64_t>(budget, pl.slots - budget)));
  if (pl.max_moves > kEvictFused) {
    const size_t units = static_cast<size_t>(c->num_seqs) * c->num_kv_heads;
    pl.workspace_bytes = align_up(units * 4, 256) +
                         align_up(units * static_cast<size_t>(pl.max_moves) * 8, 256);
  }
  return pl;
}

int validate_evict(const md_kv_cache* c, const void* mass, const void* slot_pos,
                   int64_t slot_stride, const void* lens, const void* seq_lens, int32_t budget,
                   int32_t n_sink, int32_t recent, const void* lens_out, const void* workspace,
                   size_t workspace_bytes, EvictPlan* plan) {
  const int st = check_evict_sizes(c, slot_stride, budget);
  if (st == MD_ERR_INVALID_ARG) return st;
  if (n_sink < 0 || recent < 0 || static_cast<int64_t>(n_sink) + recent > budget)
    return MD_ERR_INVALID_ARG;
  if (st != MD_OK || c->num_seqs == 0) return st;
  if (!c->k || !c->v || !mass || !slot_pos || !lens || !seq_lens) return MD_ERR_INVALID_ARG;
  if (!aligned(c->k, 16) || !aligned(c->v, 16)) return MD_ERR_INVALID_ARG;
  for (const void* x : {mass, slot_pos, lens, seq_lens, lens_out,
                        static_cast<const void*>(c->page_table)})
    if (!aligned(x, 4)) return MD_ERR_INVALID_ARG;
  *plan = make_evict_plan(c, slot_stride, budget);
  if (plan->workspace_bytes && (!workspace || workspace_bytes < plan->workspace_bytes ||
                                !aligned(workspace, 256)))
    return MD_ERR_WORKSPACE;
  const wide B = c->num_seqs, es = c->dtype == MD_BF16 ? 2 : 4;
  const wide units = B * c->num_kv_heads;
  const wide blocks = c->page_size ? static_cast<wide>(c->num_pages) : B;
  const wide toks = c->page_size ? c->page_size : c->capacity;
  const wide kv = ((blocks - 1) * c->kv_stride_blk + (toks - 1) * c->kv_stride_tok +
                   (c->num_kv_heads - 1) * static_cast<wide>(c->kv_stride_head) + c->head_dim) * es;
  const Span out[] = {{mass, units * slot_stride * 4}, {slot_pos, units * slot_stride * 4},
                      {lens_out, B * 4}, {workspace, static_cast<wide>(plan->workspace_bytes)}};
  // The cache itself is written: K and V may interleave, but nothing else may be among them.
  const Span in[] = {{lens, B * 4}, {seq_lens, B * 4}, {c->k, kv}, {c->v, kv},
                     {c->page_table, B * c->max_pages_per_seq * 4}};
  if (outputs_overlap(out, in)) return MD_ERR_INVALID_ARG;
  for (const Span& x : {in[0], in[1], in[4]})
    if (overlap(x.p, x.bytes, c->k, kv) || overlap(x.p, x.bytes, c->v, kv)) return MD_ERR_INVALID_ARG;
  return MD_OK;
}

// ---- token log probabilities ----

int check_logp_sizes(int64_t rows, int32_t vocab, int64_t row_stride, int32_t dtype, int32_t top_k) {
  if (rows < 0 || vocab < 1 || vocab > (1 << 30) || (rows > 1 && row_stride < vocab) ||
      row_stride < 0 || top_k < 0 || top_k > kLogpMaxTop || !valid_dtype(dtype))
    return MD_ERR_INVALID_ARG;
  if (rows > kMaxWgs1024) return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

LogpPlan make_logp_plan(int64_t rows, int32_t vocab, int32_t top_k, int num_cus) {
  LogpPlan pl;
  const int64_t cus = num_cus > 0 ? num_cus : 256;
  // Segments of 16384 logits, 32 a lane twice; of 4096 where that leaves compute units without work.
  const bool many = rows * ceil_div(vocab, 64 * 256) >= cus;
  pl.per_lane = many ? 32 : 16;
  const int64_t at_once = many ? 64 * 256 : 16 * 256;
  // Up to 256 segments a row, fewer where the grid's 32 bits would end.
  const int64_t most = std::max<int64_t>(1, std::min<int64_t>(256, kMaxWgs256 / std::max<int64_t>(rows, 1)));
  pl.seg_len = static_cast<int32_t>(at_once * ceil_div(ceil_div(vocab, at_once), most));
  pl.n_segs = static_cast<int32_t>(ceil_div(vocab, pl.seg_len));
  if (pl.n_segs > 1) {
    const size_t n = static_cast<size_t>(rows) * pl.n_segs;
    pl.stats_bytes = align_up(n * 12, 256);
    pl.cand_bytes = align_up(n * static_cast<size_t>(top_k) * 8, 256);
    pl.workspace_bytes = pl.stats_bytes + pl.cand_bytes;
  }
  return pl;
}

int validate_logp(int64_t rows, int32_t vocab, int64_t row_stride, int32_t dtype,
                  const void* logits, const void* tokens, int32_t top_k, const void* logprobs,
                  const void* entropy, const void* top, const void* top_logprobs,
                  const void* workspace, size_t workspace_bytes, LogpPlan* plan) {
  const int st = check_logp_sizes(rows, vocab, row_stride, dtype, top_k);
  if (st == MD_ERR_INVALID_ARG || rows == 0 || st != MD_OK) return st;
  const wide es = dtype == MD_BF16 ? 2 : 4;
  if (!logits || !aligned(logits, static_cast<uintptr_t>(es))) return MD_ERR_INVALID_ARG;
  if ((tokens == nullptr) != (logprobs == nullptr)) return MD_ERR_INVALID_ARG;
  if (top_k > 0 ? (!top || !top_logprobs) : (top || top_logprobs)) return MD_ERR_INVALID_ARG;
  for (const void* x : {tokens, logprobs, entropy, top, top_logprobs})
    if (!aligned(x, 4)) return MD_ERR_INVALID_ARG;
  *plan = make_logp_plan(rows, vocab, top_k, device_cu_count());
  if (plan->workspace_bytes && (!workspace || workspace_bytes < plan->workspace_bytes ||
                                !aligned(workspace, 256)))
    return MD_ERR_WORKSPACE;
  const wide n = rows;
  const Span out[] = {{logprobs, n * 4}, {entropy, n * 4}, {top, n * top_k * 4},
                      {top_logprobs, n * top_k * 4},
                      {workspace, static_cast<wide>(plan->workspace_bytes)}};
  const Span in[] = {{logits, ((n - 1) * row_stride + vocab) * es}, {tokens, n * 4}};
  return outputs_overlap(out, in) ? MD_ERR_INVALID_ARG : MD_OK;
}

}  // namespace md
