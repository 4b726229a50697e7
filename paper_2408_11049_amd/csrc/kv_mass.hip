// kv_mass.hip -- the attention weights that a call's queries give each cached token, summed
// over rows and the query heads of a KV head, added to what the token had:
//   w(j) = sum_r exp(scale q_r . k_j - lse_r)
//
// A workgroup takes 128 keys of one KV head, 32 a wave, which stay in registers as the second
// operand while the rows of Q go past in LDS tiles of 32: S = Q K^T leaves a lane one key and 16
// rows, so the sum over rows is in the lane but for one exchange at the end.  Every sum has a
// fixed order: a tile's 32 rows first, then the tiles.
#include "answers_kernels.h"

namespace md {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr int kRows = 32;  // of a tile

template <int D, bool BF16>
__global__ void __launch_bounds__(256)
kv_mass_kernel(const MassParams p) {
  constexpr int ES = BF16 ? 2 : 4, ROW = D * ES, CH = ROW / 16, ST = CH / 2;
  constexpr int NP = kRows * CH / 256;  // chunks of a Q tile a thread moves
  constexpr float kLog2e = 1.44269504088896340736f;
  // Q rows unpadded, chunk c of row r in place c ^ turn(r): see the shared-prefix attention.
  __shared__ __attribute__((aligned(16))) unsigned char qt[2][kRows * ROW];
  __shared__ __attribute__((aligned(16))) float nl[2][kRows];  // -lse in log2, -inf: weighs nothing
  auto at = [](int r, int c) {
    const int turn = ROW == 128 ? (r >> 1) & 7 : r & 15;
    return r * ROW + ((c ^ turn) << 4);
  };

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5, wave = tid >> 6;
  const int units = p.B * p.Hkv;
  const int unit = static_cast<int>(blockIdx.x) % units;
  const int kb = static_cast<int>(blockIdx.x) / units;
  const int hk = unit % p.Hkv, b = unit / p.Hkv;
  const int S = min(max(p.c.lens[b], 0), p.c.max_len);
  const int key_first = kb * p.keys;
  if (key_first >= S) return;
  const int key = key_first + wave * 32 + l32;
  const bool live = key < S;
  const int base = S - p.L;  // the key that row 0 sits at (below 0: a length shorter than L)

  // This lane's key as an operand: chunks 2 st + half of its row.
  u32x4 k[ST];
  {
    int64_t off = 0;
    bool ok = live;
    if (p.c.page_table != nullptr) {
      const int pid = ok ? p.c.page_table[static_cast<int64_t>(b) * p.c.max_pages + (key >> p.c.page_shift)] : -1;
      ok = pid >= 0 && pid < p.c.num_pages;
      off = static_cast<int64_t>(pid) * p.c.s_blk +
            static_cast<int64_t>(key & ((1 << p.c.page_shift) - 1)) * p.c.s_tok;
    } else {
      off = static_cast<int64_t>(b) * p.c.s_blk + static_cast<int64_t>(key) * p.c.s_tok;
    }
    off = ok ? (off + static_cast<int64_t>(hk) * p.c.s_head) * ES : 0;
#pragma unroll
    for (int st = 0; st < ST; ++st)
      k[st] = *reinterpret_cast<const u32x4*>(p.c.k + off + (2 * st + half) * 16);
  }

  // Rows i * G + g that count and see a key of this workgroup.
  int n_count = p.L;
  if (p.accepted) n_count = min(max(p.accepted[b], 0), p.L - 1) + 1;
  const int r_begin = max(0, key_first - base) * p.G;  // base may be < 0: then rows start later
  const int r_end = n_count * p.G;
  // The first row that sees this lane's key.
  const int r_sees = max(0, key - base) * p.G;

  u32x4 stage_q[NP];
  float stage_l = -INFINITY;
  auto load_tile = [&](int r0) {
    if (r0 >= r_end) return;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int x = n * 256 + tid, r = r0 + x / CH;
      const bool ok = r < r_end;
      const int i = r / p.G;
      const int64_t row = (static_cast<int64_t>(b) * p.L + i) * p.Hq + hk * p.G + (r - i * p.G);
      stage_q[n] = ok ? *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(p.q) +
                                                        row * ROW + (x % CH) * 16)
                      : u32x4{0, 0, 0, 0};
    }
    if (tid < kRows) {
      const int r = r0 + tid;
      stage_l = -INFINITY;
      if (r < r_end) {
        const int i = r / p.G;
        const float l = p.lse[(static_cast<int64_t>(b) * p.L + i) * p.Hq + hk * p.G + (r - i * p.G)];
        if (l != -INFINITY) stage_l = -l * kLog2e;
      }
    }
  };
  auto store_tile = [&](int buf, int r0) {
    if (r0 >= r_end) return;
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int x = n * 256 + tid;
      *reinterpret_cast<u32x4*>(qt[buf] + at(x / CH, x % CH)) = stage_q[n];
    }
    if (tid < kRows) nl[buf][tid] = stage_l;
  };

  float w = 0.f;
  load_tile(r_begin);
  store_tile(0, r_begin);
  load_tile(r_begin + kRows);
  __syncthreads();
  int buf = 0;
  for (int r0 = r_begin; r0 < r_end; r0 += kRows, buf ^= 1) {
    store_tile(buf ^ 1, r0 + kRows);
    load_tile(r0 + 2 * kRows);
    f32x16 s = {};
#pragma unroll
    for (int st = 0; st < ST; ++st) {
      const u32x4 q = *reinterpret_cast<const u32x4*>(qt[buf] + at(l32, 2 * st + half));
      if constexpr (BF16) {
        s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q),
                                                    __builtin_bit_cast(bf16x8, k[st]), s, 0, 0, 0);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(q[j]), __uint_as_float(k[st][j]), s,
                                                   0, 0, 0);
      }
    }
    // Rows r0 + 8 (e / 4) + 4 half + e % 4.
    const bool masked = __any(r0 < r_sees);
    float part[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 l4 = *reinterpret_cast<const f32x4*>(&nl[buf][8 * j + 4 * half]);
      part[j] = 0.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * j + e], p.scale_log2, l4[e]));
        if (l4[e] == -INFINITY || (masked && r0 + 8 * j + 4 * half + e < r_sees)) x = 0.f;
        part[j] += x;
      }
    }
    w += (part[0] + part[1]) + (part[2] + part[3]);
    __syncthreads();
  }
  w += __shfl_xor(w, 32);
  if (half || !live) return;
  const int64_t slot = static_cast<int64_t>(unit) * p.slot_stride + key;
  if (key >= base) {  // a newest token
    p.mass[slot] = w;
    p.slot_pos[slot] = p.pos0[b] + (key - base);
  } else {
    p.mass[slot] += w;
  }
}

}  // namespace

hipError_t launch_kv_mass(const MassParams& p, int64_t n_wgs, int head_dim, bool bf16, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(n_wgs)), block(256);
#define MD_MASS(D, BF) hipLaunchKernelGGL((kv_mass_kernel<D, BF>), grid, block, 0, s, p)
  if (head_dim == 128) {
    if (bf16) MD_MASS(128, true); else MD_MASS(128, false);
  } else {
    if (bf16) MD_MASS(64, true); else MD_MASS(64, false);
  }
#undef MD_MASS
  return hipGetLastError();
}

}  // namespace md
