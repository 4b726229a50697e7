// plan_ops.cpp -- argument checks and work plans of the 4-bit KV cache, sampled
// acceptance and the query/key norm with rotation.  Pure host arithmetic, no HIP
// call: every error path runs on a machine without a GPU.
#include <limits.h>

#include <algorithm>

#include "ops.h"

namespace md {

namespace {

bool aligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }
int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

typedef __int128 wide;  // byte spans of any strides

// Whether [a, a + n) and [b, b + m) share a byte.
bool overlap(const void* a, wide n, const void* b, wide m) {
  const wide x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return a && b && n && m && x < y + m && y < x + n;
}

}  // namespace

int validate_kv4_cache(const md_kv4_cache* c) {
  if (!c || c->num_seqs < 0 || c->num_kv_heads < 1 || c->head_dim < 1) return MD_ERR_INVALID_ARG;
  if (c->page_size != 0) {
    if (c->page_size < 0 || (c->page_size & (c->page_size - 1)) || c->max_pages_per_seq < 1 ||
        c->num_pages < 1 || c->num_pages > INT32_MAX)
      return MD_ERR_INVALID_ARG;
  } else if (c->page_table || c->capacity < 1) {
    return MD_ERR_INVALID_ARG;
  }
  if (c->stride_blk < 0 || c->stride_tok < 0 || c->stride_head < 0) return MD_ERR_INVALID_ARG;
  if (c->head_dim != 64 && c->head_dim != 128) return MD_ERR_UNSUPPORTED;
  const int64_t row = c->head_dim / 2;
  if (c->stride_blk % row || c->stride_tok % row || c->stride_head % row)
    return MD_ERR_INVALID_ARG;
  // Rows of neighbouring heads and tokens must not share bytes.
  const int64_t toks = c->page_size ? c->page_size : c->capacity;
  if ((c->num_kv_heads > 1 && c->stride_head < row) || (toks > 1 && c->stride_tok < row))
    return MD_ERR_INVALID_ARG;
  if (c->stride_tok > kKv4MaxTokStride) return MD_ERR_UNSUPPORTED;
  if (static_cast<int64_t>(c->num_seqs) * c->num_kv_heads > INT32_MAX) return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

int validate_kv4_buffers(const md_kv4_cache* c) {
  if (!c->k || !c->v || !c->k_scale || !c->v_scale) return MD_ERR_INVALID_ARG;
  const uintptr_t sc = static_cast<uintptr_t>(c->head_dim) / 32;
  if (!aligned(c->k, 16) || !aligned(c->v, 16) || !aligned(c->k_scale, sc) ||
      !aligned(c->v_scale, sc))
    return MD_ERR_INVALID_ARG;
  if (c->page_size && (!c->page_table || !aligned(c->page_table, 4))) return MD_ERR_INVALID_ARG;
  return MD_OK;
}

int check_kv4_attn_sizes(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                         int window) {
  if (!a || (mode != MD_MODE_VERIFY && mode != MD_MODE_DRAFT)) return MD_ERR_INVALID_ARG;
  if (mode == MD_MODE_DRAFT && (n_sink < 0 || window < 1)) return MD_ERR_INVALID_ARG;
  if (a->q_len < 1 || a->q_len > 16 || a->num_q_heads < 1 || a->max_kv_len < a->q_len)
    return MD_ERR_INVALID_ARG;
  if (a->dtype != MD_F32 && a->dtype != MD_BF16) return MD_ERR_INVALID_ARG;
  const int st = validate_kv4_cache(c);
  if (st == MD_ERR_INVALID_ARG) return st;
  if (a->num_q_heads % c->num_kv_heads) return MD_ERR_INVALID_ARG;
  if (c->page_size ? ceil_div(a->max_kv_len, c->page_size) > c->max_pages_per_seq
                   : c->capacity < a->max_kv_len)
    return MD_ERR_INVALID_ARG;
  if (st != MD_OK) return st;
  if (static_cast<int64_t>(a->num_q_heads / c->num_kv_heads) * a->q_len > kMaxRows)
    return MD_ERR_UNSUPPORTED;
  // Up to two passes, a workgroup each, a (sequence, head).
  if (static_cast<int64_t>(c->num_seqs) * c->num_kv_heads > kMaxWgs256 / 4)
    return MD_ERR_UNSUPPORTED;
  if (a->max_kv_len > kMaxPosition) return MD_ERR_UNSUPPORTED;
  if (mode == MD_MODE_DRAFT && (window > kMaxPosition || n_sink > kMaxPosition))
    return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

// Whether a workgroup for each unit is put at less than equal ranges of all units' tiles.
// Ranges cost some 8 us more (the scan of the lengths, the pieces' partial results, the second
// launch: 64 x 8 units of 1024 tokens 28.0 us against 19.9); whole units leave compute units
// short of workgroups.  A compute unit with one of the three workgroups it can hold streams at
// 0.62 of its rate, with two at 0.93: 32 x 8 units of 2048 tokens 26.5 us whole, 25.4 in
// ranges; 64 x 8 of 2048 31.6 and 39.7, of 4096 56.9 and 61.0; 128 x 8 of 2048 62.7 and 66.1, of
// 4096 114.6 and 108.1.  Lengths are not known here: from 4096 tokens on, unequal ones would
// cost whole units more than that.  All of this was measured with bf16 queries of one row tile at
// d = 128, three workgroups a compute unit; the other instances take the same rates.
static bool whole_units(int64_t tiles, int64_t units, int64_t cus, int64_t resident, int d) {
  if (tiles <= kKv4WholeTiles) return true;
  if (tiles > kKv4RangeTiles) return false;
  const double round_us =  // of a workgroup in every place
      static_cast<double>(cus * resident * tiles * kKv4Tile * (d + d / 16)) / 6.2e6;
  const double share = static_cast<double>(units) / static_cast<double>(cus * resident);
  const int64_t left = units % (cus * resident), per_cu = ceil_div(left, cus);
  const double rate = per_cu >= resident ? 1.0 : (per_cu > 1 ? 0.93 : 0.62);
  const double rounds = static_cast<double>(units / (cus * resident)) +
                        static_cast<double>(per_cu) / static_cast<double>(resident) / rate;
  return round_us * (rounds - share) < 8.0;
}

namespace {

// What the plans of all lengths share, and the most tiles any unit has: those of the whole
// context, or of the sinks and of the union of the windows, each cut at tile boundaries.
struct Kv4Sizes {
  Kv4Plan p;
  int64_t units, tiles, cus, resident;
};

Kv4Sizes kv4_sizes(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                   int window, int num_cus) {
  Kv4Sizes s;
  s.p.G = a->num_q_heads / c->num_kv_heads;
  s.p.R = s.p.G * a->q_len;
  const int max_rows = 16 * kKv4MaxNT(a->dtype == MD_BF16);
  s.p.passes = (s.p.R + max_rows - 1) / max_rows;
  s.p.NT = (std::min(s.p.R, max_rows) + 15) / 16;
  s.units = static_cast<int64_t>(c->num_seqs) * c->num_kv_heads * s.p.passes;
  // How many neighbouring units share memory lines: the passes of a head, and the heads whose
  // scales of a token (16-token page) are within a line of 128 bytes.
  const int64_t apart = c->stride_head / 16;  // bytes between two heads' scales
  const int64_t heads = apart <= 32 ? 4 : (apart < 128 ? 2 : 1);
  for (int64_t n : {int64_t{2}, int64_t{4}})
    if (n <= heads * s.p.passes && c->num_kv_heads * s.p.passes % n == 0)
      s.p.share = static_cast<int32_t>(n);
  s.tiles = ceil_div(a->max_kv_len, kKv4Tile);
  if (mode == MD_MODE_DRAFT)
    s.tiles = std::min(s.tiles, ceil_div(n_sink, kKv4Tile) +
                                    ceil_div(int64_t{window} + a->q_len - 1, kKv4Tile) + 1);
  s.cus = num_cus > 0 ? num_cus : 256;
  s.resident = kKv4Resident(a->dtype == MD_BF16, s.p.NT, c->head_dim);
  return s;
}

// Workgroups for n of them in groups, each group's on one XCD of eight.
int32_t whole_groups(int64_t n, int32_t share) {
  return static_cast<int32_t>(share == 1 ? n : ceil_div(n, 8 * share) * 8 * share);
}

bool kv4_whole(const Kv4Sizes& s, int64_t tiles, const md_kv4_cache* c) {
  return c->num_seqs > kKv4BalMaxSeqs || tiles * s.units >= (int64_t{1} << 30) ||
         whole_units(tiles, s.units, s.cus, s.resident, c->head_dim);
}

void kv4_balance(const Kv4Sizes& s, int64_t tiles, int head_dim, Kv4Plan* p) {
  const size_t rows = 16 * static_cast<size_t>(p->NT);
  p->balanced = true;
  p->n_blocks = whole_groups(std::min(s.cus * s.resident, ceil_div(tiles * s.units, kWaves)),
                             p->share);
  p->part_o_bytes =
      align_up(static_cast<size_t>(2 * p->n_blocks) * rows * head_dim * sizeof(float), 256);
  p->part_ml_bytes = align_up(static_cast<size_t>(2 * p->n_blocks) * rows * 2 * sizeof(float), 256);
  p->workspace_bytes =
      p->part_o_bytes + p->part_ml_bytes + align_up(static_cast<size_t>(p->n_blocks) * 16, 256);
}

}  // namespace

Kv4Plan make_kv4_plan(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                      int window, int num_cus) {
  const Kv4Sizes s = kv4_sizes(c, a, mode, n_sink, window, num_cus);
  Kv4Plan p = s.p;
  if (kv4_whole(s, s.tiles, c))
    p.n_blocks = whole_groups(s.units, p.share);
  else
    kv4_balance(s, s.tiles, c->head_dim, &p);
  return p;
}

// A range's need grows with its length, but a longer one may run whole: the need is that of
// the longest one that does not.
size_t kv4_workspace_need(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                          int window, int num_cus) {
  const Kv4Sizes s = kv4_sizes(c, a, mode, n_sink, window, num_cus);
  if (c->num_seqs > kKv4BalMaxSeqs) return 0;
  int64_t tiles = std::min(s.tiles, ((int64_t{1} << 30) - 1) / s.units);
  while (tiles > kKv4WholeTiles && kv4_whole(s, tiles, c)) --tiles;
  Kv4Plan p = s.p;
  if (tiles > kKv4WholeTiles) kv4_balance(s, tiles, c->head_dim, &p);
  return p.workspace_bytes;
}

int validate_kv4_attn(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                      int window, Kv4Plan* plan) {
  const int st = check_kv4_attn_sizes(c, a, mode, n_sink, window);
  if (st != MD_OK) return st;
  if (c->num_seqs == 0) return MD_OK;
  const int bufs = validate_kv4_buffers(c);
  if (bufs != MD_OK) return bufs;
  if (!a->q || !a->o || !a->kv_lens || !aligned(a->q, 16) || !aligned(a->o, 16) ||
      !aligned(a->kv_lens, 4) || !aligned(a->lse, 4))
    return MD_ERR_INVALID_ARG;
  *plan = make_kv4_plan(c, a, mode, n_sink, window, device_cu_count());
  if (plan->workspace_bytes && (!a->workspace || a->workspace_bytes < plan->workspace_bytes ||
                                !aligned(a->workspace, 256)))
    return MD_ERR_WORKSPACE;
  return MD_OK;
}

int validate_spec_accept(int32_t num_seqs, int32_t n_draft, int32_t vocab, int32_t dtype) {
  if (num_seqs < 0 || n_draft < 0 || n_draft > 1023 || vocab < 1 || vocab > (1 << 30))
    return MD_ERR_INVALID_ARG;
  if (dtype != MD_F32 && dtype != MD_BF16) return MD_ERR_INVALID_ARG;
  if (num_seqs > kMaxWgs1024) return MD_ERR_UNSUPPORTED;
  return MD_OK;
}

SpecPlan make_spec_plan(int32_t num_seqs, int32_t vocab, int num_cus) {
  SpecPlan pl;
  const int64_t cus = num_cus > 0 ? num_cus : 256;
  // Segments of 1024 tokens (four 16-byte loads a lane and row in fp32), more in long rows.
  const int64_t len = std::max<int64_t>(1024, ceil_div(ceil_div(vocab, kSpecMaxSegs), 512) * 512);
  pl.seg_len = static_cast<int32_t>(len);
  pl.n_segs = static_cast<int32_t>(ceil_div(vocab, len));
  const int64_t wgs = std::min(ceil_div(4 * cus, std::max(num_seqs, 1)), ceil_div(pl.n_segs, 4));
  // One workgroup's sixteen waves do 32 segments in a go: one or two goes beat a second launch
  // (64 rows of 40000 fp32 tokens 11.5 us against 15.1).
  if (num_seqs > 0 && wgs > 1 && pl.n_segs > 64) {
    pl.wgs = static_cast<int32_t>(wgs);
    pl.workspace_bytes = static_cast<size_t>(num_seqs) * pl.n_segs * sizeof(double);
  }
  return pl;
}

bool spec_accept_overlaps(int32_t num_seqs, int32_t n_draft, int32_t vocab, int32_t dtype,
                          const void* p, const void* q, const void* draft, const void* u,
                          const void* accepted, const void* tokens, const void* ws,
                          size_t ws_bytes) {
  const wide B = num_seqs, n = n_draft, row = static_cast<wide>(vocab) * (dtype == MD_BF16 ? 2 : 4);
  const struct {
    const void* p;
    wide bytes;
  } out[3] = {{accepted, B * 4}, {tokens, B * (n + 1) * 4}, {ws, static_cast<wide>(ws_bytes)}},
    in[4] = {{p, B * (n + 1) * row}, {q, B * n * row}, {draft, B * n * 4}, {u, B * (n + 1) * 4}};
  for (int i = 0; i < 3; ++i) {
    for (const auto& x : in)
      if (overlap(out[i].p, out[i].bytes, x.p, x.bytes)) return true;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return true;
  }
  return false;
}

int validate_qk_norm_rope(const md_qk_norm_rope_args* a, const md_kv_cache* c) {
  if (!a) return MD_ERR_INVALID_ARG;
  if (a->num_seqs < 0 || a->n_new < 0 || a->num_q_heads < 1 || a->num_kv_heads < 1 ||
      a->head_dim < 1)
    return MD_ERR_INVALID_ARG;
  if (a->dtype != MD_F32 && a->dtype != MD_BF16) return MD_ERR_INVALID_ARG;
  if (!(a->eps >= 0.f)) return MD_ERR_INVALID_ARG;
  if (!a->norm && (a->q_weight || a->k_weight)) return MD_ERR_INVALID_ARG;
  if (a->rot_dim < 0 || a->rot_dim > a->head_dim || a->rot_dim % 16) return MD_ERR_INVALID_ARG;
  const int64_t es = a->dtype == MD_BF16 ? 2 : 4;
  for (int64_t s : {a->q_stride_seq, a->q_stride_tok, a->k_stride_seq, a->k_stride_tok,
                    a->v_stride_seq, a->v_stride_tok})
    if (s < 0 || s % (16 / es)) return MD_ERR_INVALID_ARG;
  if (c) {
    const int st = validate_kv_cache(c, a->n_new);
    if (st != MD_OK) return st;
    if (c->num_seqs != a->num_seqs || c->num_kv_heads != a->num_kv_heads ||
        c->head_dim != a->head_dim || c->dtype != a->dtype)
      return MD_ERR_INVALID_ARG;
  }
  if (a->head_dim != 64 && a->head_dim != 128) return MD_ERR_UNSUPPORTED;
  const int64_t tokens = static_cast<int64_t>(a->num_seqs) * a->n_new;
  if (tokens > INT32_MAX || a->num_q_heads > 65536 || a->num_kv_heads > 65536)
    return MD_ERR_UNSUPPORTED;
  if (tokens == 0) {  // lens_out alone
    const wide n4 = static_cast<wide>(a->num_seqs) * 4;
    return a->num_seqs && a->lens_out &&
                   (!a->pos0 || !aligned(a->pos0, 4) || !aligned(a->lens_out, 4) ||
                    overlap(a->lens_out, n4, a->pos0, n4))
               ? MD_ERR_INVALID_ARG
               : MD_OK;
  }
  if (!a->q || !a->k_new || !a->pos0 || !a->q_out || (!c && !a->k_out) || (c != nullptr) != (a->v_new != nullptr))
    return MD_ERR_INVALID_ARG;
  if (a->rot_dim && !a->inv_freq) return MD_ERR_INVALID_ARG;
  for (const void* x : {a->q, a->k_new, a->v_new, a->q_weight, a->k_weight,
                        static_cast<const void*>(a->q_out), static_cast<const void*>(a->k_out)})
    if (!aligned(x, 16)) return MD_ERR_INVALID_ARG;
  if (!aligned(a->inv_freq, 4) || !aligned(a->pos0, 4) || !aligned(a->lens_out, 4))
    return MD_ERR_INVALID_ARG;
  if (c && (!c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16) ||
            !aligned(c->page_table, 4)))
    return MD_ERR_INVALID_ARG;
  const wide nb = static_cast<wide>(a->num_seqs) * 4;
  if (overlap(a->lens_out, nb, a->pos0, nb)) return MD_ERR_INVALID_ARG;
  // In place only row for row: any other overlap would read rows already written.
  const int64_t d = a->head_dim, B = a->num_seqs, n = a->n_new;
  struct Rows {
    const void* p;
    int64_t seq, tok, heads;
    bool dense(wide n_tok, wide hd) const { return tok == heads * hd && seq == n_tok * tok; }
    wide bytes(wide b, wide n_tok, wide hd, wide e) const {
      return ((b - 1) * seq + (n_tok - 1) * tok + heads * hd) * e;
    }
  };
  const Rows in[3] = {{a->q, a->q_stride_seq, a->q_stride_tok, a->num_q_heads},
                      {a->k_new, a->k_stride_seq, a->k_stride_tok, a->num_kv_heads},
                      {a->v_new, a->v_stride_seq, a->v_stride_tok, a->num_kv_heads}};
  const Rows out[2] = {{a->q_out, n * a->num_q_heads * d, a->num_q_heads * d, a->num_q_heads},
                       {a->k_out, n * a->num_kv_heads * d, a->num_kv_heads * d, a->num_kv_heads}};
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 3; ++i)
      if (overlap(out[o].p, out[o].bytes(B, n, d, es), in[i].p, in[i].bytes(B, n, d, es)) &&
          !(o == i && out[o].p == in[i].p && in[i].dense(n, d)))
        return MD_ERR_INVALID_ARG;
  if (overlap(out[0].p, out[0].bytes(B, n, d, es), out[1].p, out[1].bytes(B, n, d, es)))
    return MD_ERR_INVALID_ARG;
  return MD_OK;
}

}  // namespace md
