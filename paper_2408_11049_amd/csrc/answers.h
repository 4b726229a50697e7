// answers.h -- host-side checks and plans of the operators for several answers of one
// prompt: attention over a shared prefix, eviction by accumulated weight, token log
// probabilities.  No HIP types, so they compile and run without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "internal.h"
#include "magicdec.h"
#include "ops.h"

namespace md {

// Shared-prefix attention: query rows of a workgroup and keys of a tile where the call is bound by
// reading K and V, and where bf16 groups of more than kPrefixFewRows rows a KV head, with kPrefixWideTokens
// tokens of the prefix a workgroup at least, are by the products.
constexpr int kPrefixStreamRows = 32, kPrefixStreamTile = 32;
constexpr int kPrefixWideRows = 256, kPrefixWideTile = 64, kPrefixFewRows = 160, kPrefixWideTokens = 512;
// Tokens that a page has to hold for the latter: a load instruction's rows.
constexpr int kPrefixWidePage(int d) { return d == 128 ? 4 : 8; }
struct PrefixPlan {
  bool wide = false;
  int32_t group_rows = 0;   // rows of a (prefix, KV head): B / P * L * G
  int32_t row_blocks = 0, own_blocks = 0;  // of the workgroups' rows: a group's, a sequence's
  int32_t c_pre = 0, c_own = 0;  // parts of the prefix's and of the own keys
  static constexpr int32_t split = 1;  // results of a part of the prefix a row
  int32_t pre_parts = 0;    // and of the whole prefix
  int32_t n_pre = 0;        // workgroups of the prefix, padded to whole rounds of the XCDs
  int64_t n_own = 0;        // and of the own caches
  int64_t n_rows = 0;       // B * L * Hq
  size_t part_o_bytes = 0, part_lse_bytes = 0, workspace_bytes = 0;
};
// Sizes alone: MD_OK, MD_ERR_INVALID_ARG or MD_ERR_UNSUPPORTED.
int check_prefix_sizes(const md_attn_args* a, const md_prefix* p);
PrefixPlan make_prefix_plan(const md_attn_args* a, const md_prefix* p, int num_cus);
size_t prefix_workspace_need(const md_attn_args* a, const md_prefix* p, int num_cus);
int validate_prefix(const md_attn_args* a, const md_prefix* p, PrefixPlan* plan);

// Accumulated weights: more rows than kMassStepRows a KV head are a prompt's, whose workgroups take
// kMassPromptKeys keys each.
constexpr int kMassPromptKeys = 256, kMassStepRows = 128;
struct MassPlan {
  bool prompt = false;
  int32_t key_parts = 1;    // of a sequence, a step's
  int32_t row_parts = 1;    // of a pair of key blocks; the workspace holds each part's weights
  int64_t n_wgs = 0, reduce_wgs = 0;
  size_t workspace_bytes = 0;
};
int check_mass_sizes(const md_kv_mass_args* a);
MassPlan make_mass_plan(const md_kv_mass_args* a, int num_cus);
int validate_mass(const md_kv_mass_args* a, MassPlan* plan);

// Eviction: the most rows that any (sequence, KV head) moves; up to kEvictFused of them the
// workgroup that selects moves them, more are a launch of their own, listed in the workspace.
constexpr int kEvictFused = 512;
struct EvictPlan {
  int64_t slots = 0;        // tokens a sequence can hold
  int32_t max_moves = 0;
  size_t workspace_bytes = 0;  // [units] counts, then [units][max_moves] (to, from)
};
EvictPlan make_evict_plan(const md_kv_cache* c, int64_t slot_stride, int32_t budget);
int check_evict_sizes(const md_kv_cache* c, int64_t slot_stride, int32_t budget);
int validate_evict(const md_kv_cache* c, const void* mass, const void* slot_pos,
                   int64_t slot_stride, const void* lens, const void* seq_lens, int32_t budget,
                   int32_t n_sink, int32_t recent, const void* lens_out, const void* workspace,
                   size_t workspace_bytes, EvictPlan* plan);

// Log probabilities: rows in segments, a workgroup each.
constexpr int kLogpMaxTop = 32;
struct LogpPlan {
  int32_t per_lane = 0;     // logits a lane holds at once
  int32_t seg_len = 0, n_segs = 0;
  size_t stats_bytes = 0, cand_bytes = 0, workspace_bytes = 0;
};
int check_logp_sizes(int64_t rows, int32_t vocab, int64_t row_stride, int32_t dtype, int32_t top_k);
LogpPlan make_logp_plan(int64_t rows, int32_t vocab, int32_t top_k, int num_cus);
int validate_logp(int64_t rows, int32_t vocab, int64_t row_stride, int32_t dtype,
                  const void* logits, const void* tokens, int32_t top_k, const void* logprobs,
                  const void* entropy, const void* top, const void* top_logprobs,
                  const void* workspace, size_t workspace_bytes, LogpPlan* plan);

}  // namespace md
