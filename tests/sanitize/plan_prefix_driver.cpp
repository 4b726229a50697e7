// Prints the plan of md_prefix_attn at 256 compute units: wide, parts of the prefix
// (tests/test_prefix_wide_plans.py).  Arguments: B P L Hq Hkv d, the own and the prefix's page size, the bound on the prefix.
#include <stdio.h>
#include <stdlib.h>

#include "answers.h"

namespace md {
int device_cu_count() { return 256; }
}  // namespace md

int main(int argc, char** argv) {
  if (argc != 10) return 2;
  int x[10];
  for (int i = 1; i < 10; ++i) x[i] = atoi(argv[i]);
  md_attn_args a{};
  a.num_seqs = x[1];
  a.q_len = x[3];
  a.num_q_heads = x[4];
  a.num_kv_heads = x[5];
  a.head_dim = x[6];
  a.dtype = MD_BF16;
  a.page_size = x[7];
  a.max_kv_len = x[3] + 8;
  a.kv_stride_tok = int64_t{x[5]} * x[6];
  a.kv_stride_head = x[6];
  a.max_pages_per_seq = a.max_kv_len;
  a.num_pages = 1;
  md_prefix p{};
  p.num_prefixes = x[2];
  p.page_size = x[8];
  p.max_len = x[9];
  p.kv_stride_tok = a.kv_stride_tok;
  p.kv_stride_head = a.kv_stride_head;
  p.max_pages_per_prefix = p.max_len;
  p.num_pages = 1;
  if (md::check_prefix_sizes(&a, &p) != MD_OK) return 1;
  const md::PrefixPlan pl = md::make_prefix_plan(&a, &p, 256);
  printf("%d %d\n", pl.wide, pl.c_pre);
  return 0;
}
