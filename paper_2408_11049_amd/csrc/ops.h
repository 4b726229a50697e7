// ops.h -- host-side checks and plans of the 4-bit KV cache, sampled acceptance
// and the query/key norm with rotation.  No HIP types, so they compile and run
// without a GPU.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "internal.h"
#include "magicdec.h"

namespace md {

// Tokens of one step of a wave of the 4-bit attention.
constexpr int kKv4Tile = 32;
// Byte stride of a token row: a tile's rows are addressed with 32-bit offsets.
constexpr int64_t kKv4MaxTokStride = int64_t{1} << 25;
// Row tiles of 16 a pass over K and V takes: an fp32 query is three registers' worth of bf16.
constexpr int kKv4MaxNT(bool bf16) { return bf16 ? 4 : 2; }
// Workgroups a compute unit holds, a wave per SIMD each: as many as the registers of their
// instances allow.  32 x 8 units of 16384 .. 32768 tokens against one less (fp32: against two):
// bf16 d = 64, one row tile 99 us and 103, three 152 and 155; fp32 d = 64, one 113 and 133, two
// 179 and 183, d = 128, one 181 and 190.  (bf16, two row tiles of d = 64: 124 with three or four.)
constexpr int kKv4Resident(bool bf16, int NT, int d) {
  if (d == 64) return bf16 ? (NT == 1 ? 4 : NT <= 3 ? 3 : 2) : (NT == 1 ? 4 : 3);
  return bf16 ? (NT <= 2 ? 3 : 2) : (NT == 1 ? 3 : 2);
}
// Workgroups of 256 and of 1024 threads a launch may have: its threads are counted in 32 bits.
constexpr int64_t kMaxWgs256 = (int64_t{1} << 24) - 1, kMaxWgs1024 = (int64_t{1} << 22) - 1;
// The balanced plan ranks every sequence's tiles in each workgroup.
constexpr int kKv4BalMaxSeqs = 1024;
// A unit of at most so many tiles is never cut, one of more than the second always may be.
constexpr int64_t kKv4WholeTiles = 32, kKv4RangeTiles = 128;

int validate_kv4_cache(const md_kv4_cache* c);
// The buffers of a call that touches the cache (B > 0).
int validate_kv4_buffers(const md_kv4_cache* c);

struct Kv4Plan {
  int32_t G = 0, R = 0;           // query heads and rows a KV head
  int32_t NT = 0, passes = 1;     // 16-row tiles of a pass over K and V, and passes
  int32_t share = 1;              // units whose workgroups run side by side (kv4_attn.hip)
  bool balanced = false;
  int32_t n_blocks = 0;           // workgroups
  size_t part_o_bytes = 0, part_ml_bytes = 0, workspace_bytes = 0;  // then 16 bytes a workgroup
};
int check_kv4_attn_sizes(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                         int window);
Kv4Plan make_kv4_plan(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                      int window, int num_cus);
// What md_kv4_workspace_bytes answers: enough for this max_kv_len and every smaller one.
size_t kv4_workspace_need(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                          int window, int num_cus);
int validate_kv4_attn(const md_kv4_cache* c, const md_kv4_attn_args* a, int mode, int n_sink,
                      int window, Kv4Plan* plan);

// Sampled acceptance: a row in segments, a wave each at a time.
constexpr int kSpecMaxSegs = 1024;
struct SpecPlan {
  int32_t n_segs = 0, seg_len = 0;
  int32_t wgs = 0;                // workgroups of four waves a sequence; 0: one of sixteen does all
  size_t workspace_bytes = 0;
};
int validate_spec_accept(int32_t num_seqs, int32_t n_draft, int32_t vocab, int32_t dtype);
SpecPlan make_spec_plan(int32_t num_seqs, int32_t vocab, int num_cus);
// Whether an output or the workspace (its first ws_bytes) shares memory with an input or with
// each other: they are written while other workgroups read.
bool spec_accept_overlaps(int32_t num_seqs, int32_t n_draft, int32_t vocab, int32_t dtype,
                          const void* p, const void* q, const void* draft, const void* u,
                          const void* accepted, const void* tokens, const void* ws,
                          size_t ws_bytes);

// Sizes, strides, pointers and overlaps; c may be NULL (no cache).
int validate_qk_norm_rope(const md_qk_norm_rope_args* a, const md_kv_cache* c);

}  // namespace md
