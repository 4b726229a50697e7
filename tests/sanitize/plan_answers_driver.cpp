// Host-side checks and plans of csrc/plan_answers.cpp under AddressSanitizer and
// UndefinedBehaviorSanitizer (tests/test_answers_abi.py): extreme arguments through every
// validator, a sweep of shapes through every plan, and the plans' invariants.
#include <limits.h>
#include <stdint.h>
#include <stdio.h>

#include <initializer_list>

#include "answers.h"

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
const int32_t* const kInts = reinterpret_cast<const int32_t*>(kFake);
void* at(int i) { return kFake + (int64_t{i} << 40); }

md_attn_args attn(int B, int L, int Hq, int Hkv, int d, int dtype, int64_t S, int page) {
  md_attn_args a{};
  a.num_seqs = B;
  a.q_len = L;
  a.num_q_heads = Hq;
  a.num_kv_heads = Hkv;
  a.head_dim = d;
  a.dtype = dtype;
  a.q = a.k = a.v = kFake;
  a.o = kFake;
  a.kv_lens = kInts;
  a.kv_stride_head = d;
  a.kv_stride_tok = int64_t{Hkv} * d;
  a.kv_stride_blk = (page ? page : S) * a.kv_stride_tok;
  a.max_kv_len = static_cast<int32_t>(S);
  if (page) {
    a.page_size = page;
    a.max_pages_per_seq = static_cast<int32_t>((S + page - 1) / page);
    a.num_pages = 1000;
    a.page_table = kInts;
  }
  a.workspace = kFake;
  a.workspace_bytes = SIZE_MAX;
  return a;
}

md_prefix prefix(int P, int64_t T, int d, int Hkv, int page) {
  md_prefix p{};
  p.num_prefixes = P;
  p.k = p.v = kFake;
  p.lens = kInts;
  p.kv_stride_head = d;
  p.kv_stride_tok = int64_t{Hkv} * d;
  p.kv_stride_blk = (page ? page : T) * p.kv_stride_tok;
  p.max_len = static_cast<int32_t>(T);
  if (page) {
    p.page_size = page;
    p.max_pages_per_prefix = static_cast<int32_t>(T ? (T + page - 1) / page : 1);
    p.num_pages = 1000;
    p.page_table = kInts;
  }
  return p;
}

md_kv_mass_args mass(int B, int L, int Hq, int Hkv, int d, int dtype, int64_t S, int64_t stride) {
  md_kv_mass_args a{};
  a.num_seqs = B;
  a.q_len = L;
  a.num_q_heads = Hq;
  a.num_kv_heads = Hkv;
  a.head_dim = d;
  a.dtype = dtype;
  a.q = at(1);
  a.k = at(2);
  a.lse = static_cast<float*>(at(3));
  a.mass = static_cast<float*>(at(4));
  a.slot_pos = static_cast<int32_t*>(at(5));
  a.kv_lens = static_cast<int32_t*>(at(6));
  a.pos0 = static_cast<int32_t*>(at(7));
  a.kv_stride_head = d;
  a.kv_stride_tok = int64_t{Hkv} * d;
  a.kv_stride_blk = S * a.kv_stride_tok;
  a.max_kv_len = static_cast<int32_t>(S);
  a.slot_stride = stride;
  a.workspace = at(8);
  a.workspace_bytes = SIZE_MAX;
  return a;
}

// Parts that fill the list without gaps: the kernels' own arithmetic.
void check_parts(int64_t n_tiles, int parts) {
  int64_t at = 0;
  for (int c = 0; c < parts; ++c) {
    const int64_t lo = n_tiles * c / parts, hi = n_tiles * (c + 1) / parts;
    check(lo == at && hi >= lo, "parts leave a gap", n_tiles, parts);
    at = hi;
  }
  check(at == n_tiles, "parts end early", n_tiles, parts);
}

}  // namespace

int main() {
  using namespace md;
  const int64_t lens[] = {1, 31, 32, 33, 127, 128, 129, 255, 257, 2054, 8192, 32768, 70001, 1 << 24, INT32_MAX - 64};
  const int batches[] = {1, 2, 8, 63, 64, 129, 1000, 40000};

  for (int B : batches)
    for (int P : {1, 2, B})
      for (int L : {1, 5, 16})
        for (int G : {1, 3, 4, 64 / L})
          for (int Hkv : {1, 8})
            for (int64_t T : lens)
              for (int64_t S : {int64_t{16}, int64_t{300}, int64_t{9000}})
                for (int page : {0, 1, 4, 16})
                  for (int dtype : {MD_F32, MD_BF16}) {
                    if (B % P || G * L > 64) continue;
                    md_attn_args a = attn(B, L, G * Hkv, Hkv, 128, dtype, S, page);
                    md_prefix p = prefix(P, T, 128, Hkv, page);
                    PrefixPlan pl;
                    const int st = validate_prefix(&a, &p, &pl);
                    if (st == MD_ERR_UNSUPPORTED) continue;
                    check(st == MD_OK, "prefix plan", B, T);
                    check(pl.c_pre >= 1 && pl.c_own >= 1 && pl.n_pre + pl.n_own <= kMaxWgs256, "prefix parts", B, T);
                    check(int64_t{pl.row_blocks} * (pl.wide ? kPrefixWideRows / pl.split : kPrefixStreamRows) >= pl.group_rows,
                          "prefix rows", B, L);
                    check(int64_t{pl.own_blocks} * kPrefixStreamRows >= G * L, "own rows", B, L);
                    check(int64_t{pl.n_pre} >= int64_t{P} * Hkv * pl.c_pre * pl.row_blocks && pl.n_pre % 8 == 0,
                          "prefix workgroups", B, T);
                    check(pl.n_own >= int64_t{B} * Hkv * pl.c_own * pl.own_blocks && pl.n_own % 8 == 0, "own workgroups", B, S);
                    check(pl.pre_parts == pl.c_pre * pl.split && (pl.wide || pl.split == 1), "prefix split", B, T);
                    check(!pl.wide || (dtype == MD_BF16 && (page == 0 || page >= 4)), "wide", page, dtype);
                    const size_t parts = static_cast<size_t>(pl.pre_parts + pl.c_own) * static_cast<size_t>(pl.n_rows);
                    check(pl.part_o_bytes >= parts * 512 && pl.part_lse_bytes >= parts * 4 &&
                              pl.workspace_bytes == pl.part_o_bytes + pl.part_lse_bytes,
                          "prefix workspace", B, T);
                    check_parts((T + 31) / 32, pl.c_pre);
                  }

  for (int B : batches)
    for (int64_t S : lens)
      for (int64_t L : {int64_t{1}, int64_t{5}, int64_t{200}, S})
        for (int G : {1, 4, 9})
          for (int Hkv : {1, 8}) {
            if (L > S) continue;
            md_kv_mass_args a = mass(B, static_cast<int>(L), G * Hkv, Hkv, 64, MD_BF16, S, S + 3);
            MassPlan pl;
            const int st = validate_mass(&a, &pl);
            if (st == MD_ERR_UNSUPPORTED || st == MD_ERR_INVALID_ARG) continue;  // (INVALID: spans meet)
            check(st == MD_OK, "mass plan", B, S);
            const int64_t units = int64_t{B} * Hkv;
            check(pl.prompt == (L * G > kMassStepRows), "a prompt", L, G);
            check(pl.n_wgs >= 1 && pl.n_wgs <= INT32_MAX, "mass workgroups", B, S);
            if (!pl.prompt) {
              check(pl.n_wgs % 8 == 0 && pl.n_wgs >= units * pl.key_parts && pl.workspace_bytes == 0, "step workgroups", B, S);
              check_parts((S + 31) / 32, pl.key_parts);
            } else {
              const int64_t blocks = (S + kMassPromptKeys - 1) / kMassPromptKeys;
              check(pl.row_parts >= 1 && pl.n_wgs == units * ((blocks + 1) / 2) * pl.row_parts, "prompt workgroups", B, S);
              check(pl.workspace_bytes >= (pl.row_parts > 1 ? static_cast<size_t>(pl.row_parts) * units * S * 4 : 0),
                    "prompt workspace", B, S);
              // A row's number, and that of the second tile ahead of it, stays in 32 bits.
              check(L * G + 3 * int64_t{64} * pl.row_parts <= INT32_MAX, "prompt rows", L, pl.row_parts);
            }
          }

  for (int B : batches)
    for (int64_t S : lens)
      for (int budget : {1, 64, 511, 512, 513, 2048, INT32_MAX}) {
        md_kv_cache c{};
        c.num_seqs = B;
        c.num_kv_heads = 8;
        c.head_dim = 128;
        c.dtype = MD_BF16;
        c.k = at(1);
        c.v = at(20);
        c.kv_stride_head = 128;
        c.kv_stride_tok = 1024;
        c.kv_stride_blk = 0;
        c.capacity = static_cast<int32_t>(S);
        EvictPlan pl;
        const int st = validate_evict(&c, at(40), at(60), S, at(80), at(81), budget, 0, 1, at(82), at(90), SIZE_MAX, &pl);
        if (st != MD_OK) continue;
        check(pl.slots == S && pl.max_moves >= 0 && pl.max_moves <= budget && pl.max_moves <= S, "evict plan", S, budget);
        check(pl.max_moves > kEvictFused
                  ? pl.workspace_bytes >= size_t(B) * 8 * (4 + 8 * static_cast<size_t>(pl.max_moves))
                  : pl.workspace_bytes == 0,
              "evict workspace", S, budget);
      }

  for (int64_t rows : {int64_t{1}, int64_t{5}, int64_t{320}, int64_t{70000}, int64_t{1} << 21, (int64_t{1} << 22) - 1})
    for (int32_t vocab : {1, 255, 4096, 4097, 16385, 128256, 1 << 24, 1 << 30})
      for (int k : {0, 1, 32})
        for (int cus : {0, 1, 64, 256, 1024}) {
          check(check_logp_sizes(rows, vocab, vocab, MD_F32, k) == MD_OK, "logp sizes", rows, vocab);
          const LogpPlan pl = make_logp_plan(rows, vocab, k, cus);
          check(pl.n_segs >= 1 && pl.n_segs <= 256 && int64_t{pl.seg_len} * pl.n_segs >= vocab &&
                    int64_t{pl.seg_len} * (pl.n_segs - 1) < vocab,
                "segments", rows, vocab);
          check(rows * pl.n_segs <= kMaxWgs256, "logp workgroups", rows, vocab);
          check(pl.workspace_bytes >= (pl.n_segs > 1 ? static_cast<size_t>(rows) * pl.n_segs * (12 + 8 * size_t(k)) : 0),
                "logp workspace", rows, vocab);
        }

  // Extremes through the validators: no overflow, and no status but an error.
  md_attn_args a = attn(INT32_MAX, 16, INT32_MAX, 1, 128, MD_BF16, INT32_MAX, 0);
  md_prefix p = prefix(1, INT32_MAX, 128, 1, 0);
  PrefixPlan pp;
  check(validate_prefix(&a, &p, &pp) == MD_ERR_UNSUPPORTED, "extreme prefix");
  a = attn(4, 1, 8, 2, 128, MD_BF16, 64, 0);
  p = prefix(INT32_MIN, INT32_MIN, 128, 2, 0);
  check(validate_prefix(&a, &p, &pp) == MD_ERR_INVALID_ARG, "negative prefix");
  p = prefix(1, 64, 128, 2, 0);
  p.kv_stride_blk = p.kv_stride_tok = INT64_MAX - 7;
  check(validate_prefix(&a, &p, &pp) == MD_ERR_UNSUPPORTED, "strides of the prefix");
  md_kv_mass_args m = mass(INT32_MAX, INT32_MAX - 64, INT32_MAX, 1, 128, MD_F32, INT32_MAX - 64, INT64_MAX);
  MassPlan mp;
  check(validate_mass(&m, &mp) != MD_OK, "extreme mass");
  m = mass(2, 1, 8, 2, 128, MD_BF16, 64, INT64_MAX);
  m.kv_stride_blk = INT64_MAX - 7;
  m.kv_stride_head = INT64_MAX - 7;
  check(validate_mass(&m, &mp) == MD_ERR_INVALID_ARG, "spans past 64 bits meet");

  if (g_fail) return 1;
  printf("plan answers driver: ok\n");
  return 0;
}
