// The launches of csrc/plan_answers.cpp against what a grid can hold (tests/test_answers_grids.py): sizes at which
// the rounding up to whole rounds of the XCDs passes 32 bits of threads.  Whatever is not refused fits.
#include <stdint.h>
#include <stdio.h>

#include <initializer_list>

#include "answers.h"

namespace md {
int device_cu_count() { return 256; }
}  // namespace md

int main() {
  using namespace md;
  int fail = 0, taken = 0, refused = 0;
  auto at = [](int i) { return reinterpret_cast<unsigned char*>(uintptr_t{1} << 40) + (int64_t{i} << 56); };
  for (int log_heads = 0; log_heads <= 24; ++log_heads)
    for (int more : {-1, 0, 1})
      for (int B : {1, 2, 7, 8, 9, 15, 16, 17, 31, 100})
        for (int L : {1, 5, 200})
          for (int S : {200, 256, 300, 2054}) {
            const int64_t heads = (int64_t{1} << log_heads) + more;
            if (heads < 1) continue;
            md_kv_mass_args a{};
            a.num_seqs = B;
            a.q_len = L;
            a.num_q_heads = a.num_kv_heads = static_cast<int32_t>(heads);
            a.head_dim = 64;
            a.dtype = MD_BF16;
            a.q = at(1);
            a.k = at(2);
            a.lse = reinterpret_cast<float*>(at(3));
            a.mass = reinterpret_cast<float*>(at(4));
            a.slot_pos = reinterpret_cast<int32_t*>(at(5));
            a.kv_lens = reinterpret_cast<int32_t*>(at(6));
            a.pos0 = reinterpret_cast<int32_t*>(at(7));
            a.kv_stride_head = 64;
            a.kv_stride_tok = heads * 64;
            a.kv_stride_blk = S * a.kv_stride_tok;
            a.max_kv_len = S;
            a.slot_stride = S;
            a.workspace = at(8);
            a.workspace_bytes = SIZE_MAX;
            MassPlan pl;
            const int st = validate_mass(&a, &pl);
            if (st == MD_ERR_UNSUPPORTED) {
              ++refused;
              continue;
            }
            if (st == MD_OK) ++taken;
            if (st != MD_OK || pl.n_wgs < 1 || pl.n_wgs > kMaxWgs256 || pl.reduce_wgs > kMaxWgs256) {
              fprintf(stderr, "FAILED: B %d, heads %lld, L %d, S %d: status %d, %lld and %lld workgroups\n", B,
                      static_cast<long long>(heads), L, S, st, static_cast<long long>(pl.n_wgs),
                      static_cast<long long>(pl.reduce_wgs));
              ++fail;
            }
          }
  if (fail || !taken || !refused) return 1;
  printf("grids driver: ok, %d taken, %d refused\n", taken, refused);
  return 0;
}
