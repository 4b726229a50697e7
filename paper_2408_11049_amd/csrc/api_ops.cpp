// api_ops.cpp -- the C entry points of the 4-bit KV cache, sampled acceptance and
// the query/key norm with rotation: checks, plans and launches on the caller's
// stream.  No allocation, no host synchronisation.
#include <hip/hip_runtime.h>
#include <math.h>

#include "kv4.h"

namespace md {

namespace {

int page_shift(int32_t page_size) {
  int s = 0;
  while ((int64_t{1} << s) < page_size) ++s;
  return s;
}

Kv4View kv4_view(const md_kv4_cache* c) {
  Kv4View v{};
  v.k = static_cast<unsigned char*>(c->k);
  v.v = static_cast<unsigned char*>(c->v);
  v.ks = static_cast<unsigned char*>(c->k_scale);
  v.vs = static_cast<unsigned char*>(c->v_scale);
  v.s_blk = c->stride_blk;
  v.s_tok = c->stride_tok;
  v.s_head = c->stride_head;
  v.page_table = c->page_table;
  v.page_shift = page_shift(c->page_size);
  v.max_pages = c->max_pages_per_seq;
  v.num_pages = c->num_pages;
  v.capacity = c->capacity;
  return v;
}

int status(hipError_t e) { return e == hipSuccess ? MD_OK : hip_fail(e); }

bool misaligned(const void* p, uintptr_t n) { return reinterpret_cast<uintptr_t>(p) % n != 0; }

// The shared part of append and read: rows [B, n, Hkv, d] at positions pos0[b] + i.
int kv4_rows(const md_kv4_cache* c, int32_t n, int32_t dtype, const void* k_rows,
             const void* v_rows, const int32_t* pos0, Kv4RowsParams* p) {
  const int st = validate_kv4_cache(c);
  if (st == MD_ERR_INVALID_ARG) return st;
  if (n < 0 || (dtype != MD_F32 && dtype != MD_BF16)) return MD_ERR_INVALID_ARG;
  if (st != MD_OK) return st;
  const int64_t units = static_cast<int64_t>(c->num_seqs) * c->num_kv_heads;
  if (n > 0 && units > INT32_MAX / n) return MD_ERR_UNSUPPORTED;
  if (c->num_seqs == 0 || n == 0) return MD_OK;
  const int bufs = validate_kv4_buffers(c);
  if (bufs != MD_OK) return bufs;
  if (!k_rows || !v_rows || !pos0 || misaligned(k_rows, 16) || misaligned(v_rows, 16) ||
      misaligned(pos0, 4))
    return MD_ERR_INVALID_ARG;
  p->c = kv4_view(c);
  p->k_rows = const_cast<void*>(k_rows);
  p->v_rows = const_cast<void*>(v_rows);
  p->pos0 = pos0;
  p->B = c->num_seqs;
  p->n = n;
  p->Hkv = c->num_kv_heads;
  p->rows = static_cast<int32_t>(units * n);
  return MD_OK;
}

int run_kv4_attn(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                 int window, void* stream) {
  Kv4Plan pl;
  const int st = validate_kv4_attn(c, a, mode, n_sink, window, &pl);
  if (st != MD_OK || c->num_seqs == 0) return st;
  Kv4AttnParams p{};
  p.c = kv4_view(c);
  p.q = a->q;
  p.kv_lens = a->kv_lens;
  p.max_kv_len = a->max_kv_len;
  p.B = c->num_seqs;
  p.L = a->q_len;
  p.Hq = a->num_q_heads;
  p.G = pl.G;
  p.R = pl.R;
  p.passes = pl.passes;
  p.units = c->num_kv_heads * pl.passes;
  p.share = pl.share;
  p.groups = p.units / pl.share;
  const float scale =
      a->sm_scale > 0.f ? a->sm_scale : 1.0f / sqrtf(static_cast<float>(c->head_dim));
  p.scale_log2 = scale * 1.44269504088896340736f;
  p.mode = mode;
  p.n_sink = mode == MD_MODE_DRAFT ? n_sink : 0;
  p.window = mode == MD_MODE_DRAFT ? window : 1;
  p.balanced = pl.balanced;
  p.o = a->o;
  p.lse = a->lse;
  if (pl.balanced) {
    unsigned char* ws = static_cast<unsigned char*>(a->workspace);
    p.part_o = reinterpret_cast<float*>(ws);
    p.part_ml = reinterpret_cast<float*>(ws + pl.part_o_bytes);
    p.joins = reinterpret_cast<Join*>(ws + pl.part_o_bytes + pl.part_ml_bytes);
  }
  return status(launch_kv4_attn(p, pl, c->head_dim, a->dtype == MD_BF16,
                                static_cast<hipStream_t>(stream)));
}

}  // namespace

}  // namespace md

extern "C" {

int md_kv4_append(const md_kv4_cache* c, int32_t n_new, int32_t dtype, const void* k_new,
                  const void* v_new, const int32_t* pos0, int32_t* lens_out, void* stream) {
  md::Kv4RowsParams p{};
  const int st = md::kv4_rows(c, n_new, dtype, k_new, v_new, pos0, &p);
  if (st != MD_OK || c->num_seqs == 0) return st;
  if (lens_out) {  // one thread writes lens_out[b] while others still read pos0[b]
    if (!pos0 || md::misaligned(pos0, 4)) return MD_ERR_INVALID_ARG;
    const uintptr_t lo = reinterpret_cast<uintptr_t>(lens_out);
    const uintptr_t po = reinterpret_cast<uintptr_t>(pos0);
    const uintptr_t nb = static_cast<uintptr_t>(c->num_seqs) * 4;
    if (lo % 4 || (lo < po + nb && po < lo + nb)) return MD_ERR_INVALID_ARG;
  }
  if (p.rows == 0)  // no token: the lengths alone
    return lens_out ? md::status(md::launch_copy_lens(c->num_seqs, pos0, lens_out,
                                                      static_cast<hipStream_t>(stream)))
                    : MD_OK;
  p.lens_out = lens_out;
  return md::status(md::launch_kv4_append(p, c->head_dim, dtype == MD_BF16, c->page_size != 0,
                                          static_cast<hipStream_t>(stream)));
}

int md_kv4_read(const md_kv4_cache* c, int32_t n, int32_t dtype, const int32_t* pos0, void* k_out,
                void* v_out, void* stream) {
  md::Kv4RowsParams p{};
  const int st = md::kv4_rows(c, n, dtype, k_out, v_out, pos0, &p);
  if (st != MD_OK || p.rows == 0) return st;
  return md::status(md::launch_kv4_read(p, c->head_dim, dtype == MD_BF16, c->page_size != 0,
                                        static_cast<hipStream_t>(stream)));
}

int md_kv4_verify_attn(const md_kv4_cache* c, const md_kv4_attn_args* a, void* stream) {
  return md::run_kv4_attn(c, a, MD_MODE_VERIFY, 0, 1, stream);
}

int md_kv4_draft_attn(const md_kv4_cache* c, const md_kv4_attn_args* a, int32_t n_sink,
                      int32_t window, void* stream) {
  return md::run_kv4_attn(c, a, MD_MODE_DRAFT, n_sink, window, stream);
}

size_t md_kv4_workspace_bytes(const md_kv4_cache* c, const md_kv4_attn_args* a, int32_t mode,
                              int32_t n_sink, int32_t window) {
  if (!c || md::check_kv4_attn_sizes(c, a, mode, n_sink, window) != MD_OK || c->num_seqs == 0)
    return 0;
  return md::kv4_workspace_need(c, a, mode, n_sink, window, md::device_cu_count());
}

size_t md_spec_accept_workspace_bytes(int32_t num_seqs, int32_t n_draft, int32_t vocab) {
  if (md::validate_spec_accept(num_seqs, n_draft, vocab, MD_F32) != MD_OK) return 0;
  return md::make_spec_plan(num_seqs, vocab, md::device_cu_count()).workspace_bytes;
}

int md_spec_accept(int32_t num_seqs, int32_t n_draft, int32_t vocab, int32_t dtype,
                   const void* target_probs, const void* draft_probs, const int32_t* draft,
                   const float* u, int32_t* accepted, int32_t* tokens, void* workspace,
                   size_t workspace_bytes, void* stream) {
  const int st = md::validate_spec_accept(num_seqs, n_draft, vocab, dtype);
  if (st != MD_OK || num_seqs == 0) return st;
  const uintptr_t es = dtype == MD_BF16 ? 2 : 4;
  if (!target_probs || (n_draft > 0 && !draft) || !u || !accepted || !tokens ||
      md::misaligned(target_probs, es) || md::misaligned(draft_probs, es) ||
      md::misaligned(draft, 4) || md::misaligned(u, 4) || md::misaligned(accepted, 4) ||
      md::misaligned(tokens, 4))
    return MD_ERR_INVALID_ARG;
  const md::SpecPlan pl = md::make_spec_plan(num_seqs, vocab, md::device_cu_count());
  if (pl.workspace_bytes && (!workspace || workspace_bytes < pl.workspace_bytes ||
                             md::misaligned(workspace, 256)))
    return MD_ERR_WORKSPACE;
  if (md::spec_accept_overlaps(num_seqs, n_draft, vocab, dtype, target_probs, draft_probs, draft, u,
                               accepted, tokens, workspace, pl.workspace_bytes))
    return MD_ERR_INVALID_ARG;
  md::SpecAcceptParams p{};
  p.p = target_probs;
  p.q = draft_probs;
  p.draft = draft;
  p.u = u;
  p.B = num_seqs;
  p.n_draft = n_draft;
  p.vocab = vocab;
  p.n_segs = pl.n_segs;
  p.seg_len = pl.seg_len;
  p.wgs = pl.wgs;
  p.seg_sum = static_cast<double*>(workspace);
  p.accepted = accepted;
  p.tokens = tokens;
  return md::status(
      md::launch_spec_accept(p, dtype == MD_BF16, static_cast<hipStream_t>(stream)));
}

int md_qk_norm_rope(const md_qk_norm_rope_args* a, const md_kv_cache* c, void* stream) {
  const int st = md::validate_qk_norm_rope(a, c);
  if (st != MD_OK || a->num_seqs == 0) return st;
  if (a->n_new == 0)  // no token: the lengths alone
    return a->lens_out ? md::status(md::launch_copy_lens(a->num_seqs, a->pos0, a->lens_out,
                                                         static_cast<hipStream_t>(stream)))
                       : MD_OK;
  md::NormRopeParams p{};
  p.q = a->q;
  p.k = a->k_new;
  p.v = a->v_new;
  p.q_seq = a->q_stride_seq;
  p.q_tok = a->q_stride_tok;
  p.k_seq = a->k_stride_seq;
  p.k_tok = a->k_stride_tok;
  p.v_seq = a->v_stride_seq;
  p.v_tok = a->v_stride_tok;
  p.q_weight = a->q_weight;
  p.k_weight = a->k_weight;
  p.inv_freq = a->inv_freq;
  p.pos0 = a->pos0;
  p.q_out = a->q_out;
  p.k_out = a->k_out;
  p.lens_out = a->lens_out;
  p.B = a->num_seqs;
  p.n = a->n_new;
  p.Hq = a->num_q_heads;
  p.Hkv = a->num_kv_heads;
  p.rot = a->rot_dim;
  p.norm = a->norm != 0;
  p.interleaved = a->interleaved != 0;
  p.eps = a->eps;
  if (c) {
    p.has_cache = 1;
    p.paged = c->page_size != 0;
    p.c.k = static_cast<unsigned char*>(c->k);
    p.c.v = static_cast<unsigned char*>(c->v);
    p.c.s_blk = c->kv_stride_blk;
    p.c.s_tok = c->kv_stride_tok;
    p.c.s_head = c->kv_stride_head;
    p.c.page_table = c->page_table;
    p.c.page_shift = md::page_shift(c->page_size);
    p.c.max_pages = c->max_pages_per_seq;
    p.c.num_pages = c->num_pages;
    p.c.capacity = c->capacity;
  }
  return md::status(md::launch_qk_norm_rope(p, a->head_dim, a->dtype == MD_BF16,
                                            static_cast<hipStream_t>(stream)));
}

}  // extern "C"
