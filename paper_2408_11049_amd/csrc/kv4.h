// kv4.h -- the 4-bit KV cache: its format on the device, the parameter blocks
// of its kernels and of the other step operators (sampled acceptance, query/key
// norm with rotation), and their launchers.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "internal.h"
#include "kernels.h"
#include "magicdec.h"
#include "ops.h"

namespace md {

// A cache of 4-bit rows as the kernels address it.  Strides are bytes of codes;
// a row's scale bytes sit at its code offset / 16 in the scale arrays (32
// channels are 16 code bytes and one scale byte).
struct Kv4View {
  unsigned char* k;
  unsigned char* v;
  unsigned char* ks;
  unsigned char* vs;
  int64_t s_blk, s_tok, s_head;
  const int32_t* page_table;  // [B, max_pages] (paged)
  int32_t page_shift;
  int32_t max_pages;
  int64_t num_pages;
  int64_t capacity;           // tokens per sequence (contiguous)
};

struct Kv4RowsParams {
  Kv4View c;
  void* k_rows;               // [B, n, Hkv, d]: read by append, written by read
  void* v_rows;
  const int32_t* pos0;
  int32_t* lens_out;          // append: [B] or nullptr
  int32_t B, n, Hkv;
  int32_t rows;               // B * n * Hkv
};

hipError_t launch_kv4_append(const Kv4RowsParams& p, int head_dim, bool bf16, bool paged,
                             hipStream_t s);
// lens_out = pos0: a call with no new token.
hipError_t launch_copy_lens(int B, const int32_t* pos0, int32_t* lens_out, hipStream_t s);
hipError_t launch_kv4_read(const Kv4RowsParams& p, int head_dim, bool bf16, bool paged,
                           hipStream_t s);

// The unit (a member of group j of sequence b) that the boundary where range w begins cuts as
// its first: its pieces are those of ranges w - 1 (partial slot `first`) .. `last`.  b < 0: none.
struct Join {
  int32_t b, j, last, first;
};

struct Kv4AttnParams {
  Kv4View c;
  const void* q;
  const int32_t* kv_lens;
  int32_t max_kv_len;
  int32_t B, L, Hq, G, R;
  int32_t passes, units;      // passes over a head's K and V; units of a sequence: Hkv * passes
  int32_t share, groups;      // units of a group (see kv4_attn.hip); groups of a sequence
  float scale_log2;           // softmax scale * log2(e)
  int32_t mode, n_sink, window;
  int32_t balanced;           // 1: workgroups share all units' tiles equally
  void* o;
  float* lse;
  float* part_o;              // balanced: [2 * workgroups][16 NT][d], unnormalised
  float* part_ml;             // balanced: [2 * workgroups][16 NT][2]: running max (log2), sum
  Join* joins;                // balanced: [workgroups]
};

hipError_t launch_kv4_attn(const Kv4AttnParams& p, const Kv4Plan& pl, int head_dim, bool bf16,
                           hipStream_t s);

struct SpecAcceptParams {
  const void* p;              // [B, n_draft + 1, vocab]
  const void* q;              // [B, n_draft, vocab], or nullptr: drafts without probabilities
  const int32_t* draft;       // [B, n_draft]
  const float* u;             // [B, n_draft + 1]
  int32_t B, n_draft, vocab, n_segs, seg_len;
  int32_t wgs;                // workgroups a sequence, or 0: one does all (spec_fused)
  double* seg_sum;            // [B, n_segs] (wgs > 0)
  int32_t* accepted;
  int32_t* tokens;            // [B, n_draft + 1]
};
hipError_t launch_spec_accept(const SpecAcceptParams& p, bool bf16, hipStream_t s);

struct NormRopeParams {
  const void* q;
  const void* k;
  const void* v;              // read with a cache only
  int64_t q_seq, q_tok, k_seq, k_tok, v_seq, v_tok;  // element strides; heads are dense
  const void* q_weight;       // [d] or nullptr (ones)
  const void* k_weight;
  const float* inv_freq;      // [rot / 2]
  const int32_t* pos0;
  void* q_out;                // [B, n, Hq, d]
  void* k_out;                // [B, n, Hkv, d] or nullptr
  int32_t* lens_out;
  int32_t B, n, Hq, Hkv, rot;
  int32_t norm, interleaved, has_cache, paged;
  float eps;
  CacheView c;
};
hipError_t launch_qk_norm_rope(const NormRopeParams& p, int head_dim, bool bf16, hipStream_t s);

}  // namespace md
