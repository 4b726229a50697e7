// api_answers.cpp -- the C entry points of the operators for several answers of one
// prompt: checks, plans and launches on the caller's stream.  No allocation, no
// host synchronisation.
#include <hip/hip_runtime.h>
#include <math.h>

#include "answers_kernels.h"

namespace md {

namespace {

int page_shift(int32_t page_size) {
  int s = 0;
  while ((int64_t{1} << s) < page_size) ++s;
  return s;
}

int status(hipError_t e) { return e == hipSuccess ? MD_OK : hip_fail(e); }

float scale_log2(float sm_scale, int32_t d) {
  const float scale = sm_scale > 0.f ? sm_scale : 1.0f / sqrtf(static_cast<float>(d));
  return scale * 1.44269504088896340736f;
}

KvView view(const void* k, const void* v, int64_t s_blk, int64_t s_tok, int64_t s_head,
            const int32_t* table, int32_t page_size, int32_t max_pages, int64_t num_pages,
            const int32_t* lens, int32_t max_len) {
  return {static_cast<const unsigned char*>(k), static_cast<const unsigned char*>(v), s_blk, s_tok,
          s_head, table, page_shift(page_size), max_pages, num_pages, lens, max_len};
}

}  // namespace

}  // namespace md

extern "C" {

size_t md_prefix_workspace_bytes(const md_attn_args* a, const md_prefix* prefix) {
  if (md::check_prefix_sizes(a, prefix) != MD_OK || a->num_seqs == 0) return 0;
  return md::prefix_workspace_need(a, prefix, md::device_cu_count());
}

int md_prefix_attn(const md_attn_args* a, const md_prefix* prefix, void* stream) {
  md::PrefixPlan pl;
  const int st = md::validate_prefix(a, prefix, &pl);
  if (st != MD_OK || a->num_seqs == 0) return st;
  md::PrefixParams p{};
  p.pre = md::view(prefix->k, prefix->v, prefix->kv_stride_blk, prefix->kv_stride_tok,
                   prefix->kv_stride_head, prefix->page_table, prefix->page_size,
                   prefix->max_pages_per_prefix, prefix->num_pages, prefix->lens, prefix->max_len);
  p.own = md::view(a->k, a->v, a->kv_stride_blk, a->kv_stride_tok, a->kv_stride_head, a->page_table,
                   a->page_size, a->max_pages_per_seq, a->num_pages, a->kv_lens, a->max_kv_len);
  p.q = a->q;
  p.P = prefix->num_prefixes;
  p.n = a->num_seqs / prefix->num_prefixes;
  p.L = a->q_len;
  p.Hq = a->num_q_heads;
  p.Hkv = a->num_kv_heads;
  p.G = a->num_q_heads / a->num_kv_heads;
  p.group_rows = pl.group_rows;
  p.row_blocks = pl.row_blocks;
  p.own_blocks = pl.own_blocks;
  p.c_pre = pl.c_pre;
  p.c_own = pl.c_own;
  p.n_pre = pl.n_pre;
  p.scale_log2 = md::scale_log2(a->sm_scale, a->head_dim);
  p.part_o = static_cast<float*>(a->workspace);
  p.part_lse = reinterpret_cast<float*>(static_cast<unsigned char*>(a->workspace) + pl.part_o_bytes);
  p.n_rows = pl.n_rows;
  p.err = a->err_word;
  const hipStream_t s = static_cast<hipStream_t>(stream);
  const bool bf16 = a->dtype == MD_BF16;
  const int rc = md::status(md::launch_prefix_attn(p, pl, a->head_dim, bf16, s));
  if (rc != MD_OK) return rc;
  return md::status(md::launch_merge_lse(pl.pre_parts + pl.c_own, pl.n_rows, a->head_dim, bf16, p.part_o,
                                         p.part_lse, a->o, a->lse, s, true));
}

size_t md_kv_mass_workspace_bytes(const md_kv_mass_args* a) {
  if (md::check_mass_sizes(a) != MD_OK || a->num_seqs == 0) return 0;
  return md::make_mass_plan(a, md::device_cu_count()).workspace_bytes;
}

int md_kv_mass(const md_kv_mass_args* a, void* stream) {
  md::MassPlan pl;
  const int st = md::validate_mass(a, &pl);
  if (st != MD_OK || a->num_seqs == 0) return st;
  md::MassParams p{};
  p.c = md::view(a->k, nullptr, a->kv_stride_blk, a->kv_stride_tok, a->kv_stride_head, a->page_table,
                 a->page_size, a->max_pages_per_seq, a->num_pages, a->kv_lens, a->max_kv_len);
  p.q = a->q;
  p.lse = a->lse;
  p.accepted = a->accepted;
  p.pos0 = a->pos0;
  p.mass = a->mass;
  p.slot_pos = a->slot_pos;
  p.slot_stride = a->slot_stride;
  p.B = a->num_seqs;
  p.L = a->q_len;
  p.Hq = a->num_q_heads;
  p.Hkv = a->num_kv_heads;
  p.G = a->num_q_heads / a->num_kv_heads;
  p.key_parts = pl.key_parts;
  p.row_parts = pl.row_parts;
  p.parts = static_cast<float*>(a->workspace);
  p.scale_log2 = md::scale_log2(a->sm_scale, a->head_dim);
  return md::status(md::launch_kv_mass(p, pl, a->head_dim, a->dtype == MD_BF16,
                                       static_cast<hipStream_t>(stream)));
}

size_t md_kv_evict_workspace_bytes(const md_kv_cache* c, int64_t slot_stride, int32_t budget) {
  if (md::check_evict_sizes(c, slot_stride, budget) != MD_OK || c->num_seqs == 0) return 0;
  return md::make_evict_plan(c, slot_stride, budget).workspace_bytes;
}

int md_kv_evict(const md_kv_cache* c, float* mass, int32_t* slot_pos, int64_t slot_stride,
                const int32_t* lens, const int32_t* seq_lens, int32_t budget, int32_t n_sink,
                int32_t recent, int32_t* lens_out, void* workspace, size_t workspace_bytes,
                void* stream) {
  md::EvictPlan pl;
  const int st = md::validate_evict(c, mass, slot_pos, slot_stride, lens, seq_lens, budget, n_sink,
                                    recent, lens_out, workspace, workspace_bytes, &pl);
  if (st != MD_OK || c->num_seqs == 0) return st;
  md::EvictParams p{};
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
  p.paged = c->page_size != 0;
  p.esize = c->dtype == MD_BF16 ? 2 : 4;
  p.row_vecs = c->head_dim * p.esize / 16;
  p.mass = mass;
  p.slot_pos = slot_pos;
  p.slot_stride = slot_stride;
  p.lens = lens;
  p.seq_lens = seq_lens;
  p.lens_out = lens_out;
  p.B = c->num_seqs;
  p.Hkv = c->num_kv_heads;
  p.budget = budget;
  p.n_sink = n_sink;
  p.recent = recent;
  p.slots = static_cast<int32_t>(pl.slots);
  p.max_moves = pl.max_moves;
  if (pl.workspace_bytes) {
    p.counts = static_cast<int32_t*>(workspace);
    const size_t units = static_cast<size_t>(c->num_seqs) * c->num_kv_heads;
    p.moves = reinterpret_cast<int2*>(static_cast<unsigned char*>(workspace) +
                                      md::align_up(units * 4, 256));
  }
  return md::status(md::launch_kv_evict(p, static_cast<hipStream_t>(stream)));
}

size_t md_token_logprobs_workspace_bytes(int64_t rows, int32_t vocab, int32_t top_k) {
  if (md::check_logp_sizes(rows, vocab, vocab, MD_F32, top_k) != MD_OK || rows == 0) return 0;
  return md::make_logp_plan(rows, vocab, top_k, md::device_cu_count()).workspace_bytes;
}

int md_token_logprobs(int64_t rows, int32_t vocab, int64_t row_stride, int32_t dtype,
                      const void* logits, const int32_t* tokens, int32_t top_k, float* logprobs,
                      float* entropy, int32_t* top, float* top_logprobs, void* workspace,
                      size_t workspace_bytes, void* stream) {
  md::LogpPlan pl;
  const int st = md::validate_logp(rows, vocab, row_stride, dtype, logits, tokens, top_k, logprobs,
                                   entropy, top, top_logprobs, workspace, workspace_bytes, &pl);
  if (st != MD_OK || rows == 0) return st;
  md::LogpParams p{};
  p.logits = logits;
  p.row_stride = row_stride;
  p.rows = static_cast<int32_t>(rows);
  p.vocab = vocab;
  p.seg_len = pl.seg_len;
  p.n_segs = pl.n_segs;
  p.top_k = top_k;
  p.tokens = tokens;
  p.logprobs = logprobs;
  p.entropy = entropy;
  p.top = top;
  p.top_logprobs = top_logprobs;
  if (pl.workspace_bytes) {
    p.stats = static_cast<float*>(workspace);
    p.cand = reinterpret_cast<uint2*>(static_cast<unsigned char*>(workspace) + pl.stats_bytes);
  }
  return md::status(md::launch_token_logprobs(p, pl, dtype == MD_BF16,
                                              static_cast<hipStream_t>(stream)));
}

}  // extern "C"
