// answers_kernels.h -- parameter blocks and launchers of the kernels for several answers
// of one prompt.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "answers.h"
#include "kernels.h"

namespace md {

// A K/V cache as the kernels read it; strides in elements.
struct KvView {
  const unsigned char* k;
  const unsigned char* v;
  int64_t s_blk, s_tok, s_head;
  const int32_t* page_table;  // [blocks, max_pages], or nullptr: contiguous
  int32_t page_shift, max_pages;
  int64_t num_pages;
  const int32_t* lens;
  int32_t max_len;
};

struct PrefixParams {
  KvView pre, own;
  const void* q;
  int32_t P, n;               // prefixes, sequences of each
  int32_t L, Hq, Hkv, G;
  int32_t group_rows, row_blocks, own_blocks, c_pre, c_own, n_pre;
  float scale_log2;           // softmax scale * log2(e)
  float* part_o;              // [c_pre + c_own][n_rows][d]
  float* part_lse;            // [c_pre + c_own][n_rows]
  int64_t n_rows;
  int32_t* err;               // md_attn_args.err_word, or nullptr
};

struct MassParams {
  KvView c;                   // v unused
  const void* q;
  const float* lse;
  const int32_t* accepted;
  const int32_t* pos0;
  float* mass;
  int32_t* slot_pos;
  int64_t slot_stride;
  int32_t B, L, Hq, Hkv, G;
  int32_t key_parts, row_parts;
  float* parts;               // [row_parts][B, Hkv][max_len] (row_parts > 1)
  float scale_log2;
};

struct EvictParams {
  CacheView c;
  int32_t paged, esize, row_vecs;  // 16-byte vectors of a row
  float* mass;
  int32_t* slot_pos;
  int64_t slot_stride;
  const int32_t* lens;
  const int32_t* seq_lens;
  int32_t* lens_out;
  int32_t B, Hkv, budget, n_sink, recent;
  int32_t slots, max_moves;
  int32_t* counts;            // [B * Hkv], or nullptr: the selecting workgroup moves
  int2* moves;                // [B * Hkv][max_moves] (to, from)
};

struct LogpParams {
  const void* logits;
  int64_t row_stride;
  int32_t rows, vocab, seg_len, n_segs, top_k;
  const int32_t* tokens;
  float* logprobs;
  float* entropy;
  int32_t* top;
  float* top_logprobs;
  float* stats;               // [rows][n_segs][3]: max, sum, weighted sum
  uint2* cand;                // [rows][n_segs][top_k]: value, index
};

hipError_t launch_prefix_attn(const PrefixParams& p, const PrefixPlan& pl, int head_dim, bool bf16,
                              hipStream_t s);
hipError_t launch_kv_mass(const MassParams& p, const MassPlan& pl, int head_dim, bool bf16,
                          hipStream_t s);
hipError_t launch_kv_evict(const EvictParams& p, hipStream_t s);
hipError_t launch_token_logprobs(const LogpParams& p, const LogpPlan& pl, bool bf16, hipStream_t s);

}  // namespace md
