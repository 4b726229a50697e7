// Host-side checks and plans of csrc/plan_ops.cpp under AddressSanitizer and
// UndefinedBehaviorSanitizer (tests/test_ops_abi.py): extreme arguments through every
// validator, a sweep of shapes through every plan, and the plans' invariants.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>
#include <stdlib.h>

#include <initializer_list>

#include "ops.h"

namespace md {
int device_cu_count() { return 256; }
}  // namespace md

namespace {

int g_fail = 0;
void check(bool ok, const char* what, long long a = 0, long long b = 0) {
  if (!ok) {
    fprintf(stderr, "FAILED: %s (%lld, %lld)\n", what, a, b);
    ++g_fail;
  }
}

unsigned char* const kFake = reinterpret_cast<unsigned char*>(uintptr_t{1} << 40);

md_kv4_cache cache(int B, int Hkv, int d, int64_t S, int page) {
  md_kv4_cache c{};
  c.num_seqs = B;
  c.num_kv_heads = Hkv;
  c.head_dim = d;
  c.k = c.v = c.k_scale = c.v_scale = kFake;
  c.stride_tok = d / 2;
  c.stride_head = (page ? page : S) * c.stride_tok;
  c.stride_blk = Hkv * c.stride_head;
  if (page) {
    c.page_size = page;
    c.max_pages_per_seq = static_cast<int32_t>((S + page - 1) / page);
    c.num_pages = 1000;
    c.page_table = reinterpret_cast<const int32_t*>(kFake);
  } else {
    c.capacity = static_cast<int32_t>(S);
  }
  return c;
}

md_kv4_attn_args args(int L, int Hq, int dtype, int64_t S) {
  md_kv4_attn_args a{};
  a.q_len = L;
  a.num_q_heads = Hq;
  a.dtype = dtype;
  a.q = kFake;
  a.o = kFake;
  a.kv_lens = reinterpret_cast<const int32_t*>(kFake);
  a.max_kv_len = static_cast<int32_t>(S);
  a.workspace = kFake;
  a.workspace_bytes = SIZE_MAX;
  return a;
}

}  // namespace

int main() {
  const int64_t lens[] = {1, 16, 31, 512, 1024, 1025, 1537, 2048, 2600, 3500, 4001, 4096, 4097, 32768, 131072, 1 << 24, INT_MAX - 64};
  long plans = 0, balanced = 0;
  for (int B : {1, 2, 7, 64, 300, 1024, 1025, 1 << 18})
    for (int Hkv : {1, 3, 8})
      for (int G : {1, 4, 7})
        for (int L : {1, 5, 9, 16})
          for (int d : {64, 128})
            for (int dtype : {0, 1})
              for (int page : {0, 1, 16}) {
                size_t last = 0;
                for (int64_t S : lens) {
                  if (S < L) continue;
                  const md_kv4_cache c = cache(B, Hkv, d, S, page);
                  const md_kv4_attn_args a = args(L, Hkv * G, dtype, S);
                  for (int mode : {MD_MODE_VERIFY, MD_MODE_DRAFT}) {
                    md::Kv4Plan p;
                    const int st = md::validate_kv4_attn(&c, &a, mode, 7, 300, &p);
                    if (G * L > 64) {
                      check(st == MD_ERR_UNSUPPORTED, "too many rows", G, L);
                      continue;
                    }
                    check(st == MD_OK, "a valid call", st, S);
                    ++plans;
                    balanced += p.balanced;
                    const int64_t units = int64_t{B} * Hkv * p.passes;
                    check(p.R == G * L && p.NT >= 1 && p.NT <= md::kKv4MaxNT(dtype == MD_BF16), "rows", p.R, p.NT);
                    check(Hkv * p.passes % p.share == 0 && (p.share == 1 || p.n_blocks % (8 * p.share) == 0),
                          "whole groups", p.share, p.n_blocks);
                    check(p.NT * 16 * p.passes >= p.R && p.NT * 16 * (p.passes - 1) < p.R, "passes", p.passes, p.R);
                    check(p.n_blocks >= 1 && (p.balanced || (p.n_blocks >= units && p.n_blocks < units + 8 * p.share)), "workgroups", p.n_blocks, units);
                    if (p.balanced) {
                      check(B <= md::kKv4BalMaxSeqs && p.n_blocks <= 256 * 4, "ranges", B, p.n_blocks);
                      check(p.part_o_bytes >= size_t(2) * p.n_blocks * p.NT * 16 * d * 4, "partials");
                      check(p.workspace_bytes >= p.part_o_bytes + p.part_ml_bytes + size_t(16) * p.n_blocks,
                            "workspace");
                    } else {
                      check(p.workspace_bytes == 0, "no workspace");
                    }
                    const size_t need = md::kv4_workspace_need(&c, &a, mode, 7, 300, 256);
                    check(need >= p.workspace_bytes, "the query covers the call", S, B);
                    if (mode == MD_MODE_VERIFY) {
                      check(need >= last, "a longer one needs no less", S, B);
                      last = need;
                    }
                  }
                }
              }
  check(balanced > 1000 && plans > 10000, "the sweep reached both plans", balanced, plans);

  for (int B : {0, 1, 3, 64, 511, 512, (1 << 22) - 1})
    for (int V : {1, 2, 1000, 32768, 32769, 50001, 128256, 1 << 20, 1 << 30}) {
      const md::SpecPlan p = md::make_spec_plan(B, V, 256);
      check(p.n_segs >= 1 && p.n_segs <= md::kSpecMaxSegs, "segments", p.n_segs, V);
      check(int64_t{p.seg_len} * p.n_segs >= V && int64_t{p.seg_len} * (p.n_segs - 1) < V, "cover", p.seg_len, V);
      check(p.seg_len % 8 == 0 && int64_t{B} * p.wgs <= INT_MAX, "whole vectors; grid", p.seg_len, p.wgs);
      check(p.wgs == 0 ? p.workspace_bytes == 0 : p.workspace_bytes == size_t(B) * p.n_segs * 8, "sums");
    }
  for (int x : {INT_MIN, -1, 0, 1, INT_MAX})
    for (int y : {INT_MIN, 0, 1, INT_MAX})
      for (int z : {INT_MIN, 0, 1, INT_MAX}) {
        (void)md::validate_spec_accept(x, y, z, 0);
        md_kv4_cache c = cache(1, 1, 128, 64, 0);
        c.num_seqs = x;
        c.num_kv_heads = y;
        c.head_dim = z;
        (void)md::validate_kv4_cache(&c);
        c = cache(1, 1, 128, 64, 0);
        c.page_size = x;
        c.max_pages_per_seq = y;
        c.capacity = z;
        (void)md::validate_kv4_cache(&c);
        md_kv4_attn_args a = args(1, 4, 1, 64);
        md::Kv4Plan p;
        a.max_kv_len = x;
        (void)md::validate_kv4_attn(&c, &a, MD_MODE_DRAFT, y, z, &p);
        a.q_len = y;
        a.num_q_heads = z;
        (void)md::validate_kv4_attn(&c, &a, MD_MODE_VERIFY, 0, 1, &p);
        md_qk_norm_rope_args n{};
        n.num_seqs = x;
        n.n_new = y;
        n.num_q_heads = n.num_kv_heads = 4;
        n.head_dim = 64;
        n.rot_dim = z;
        n.q = n.k_new = n.q_out = n.k_out = kFake;
        n.pos0 = reinterpret_cast<const int32_t*>(kFake);
        n.inv_freq = reinterpret_cast<const float*>(kFake);
        n.q_stride_seq = n.k_stride_tok = INT64_MAX - 7;
        n.q_stride_tok = n.v_stride_seq = INT64_MAX - 15;
        (void)md::validate_qk_norm_rope(&n, nullptr);
      }
  if (g_fail) return 1;
  printf("plan ops driver: ok (%ld plans, %ld balanced)\n", plans, balanced);
  return 0;
}
