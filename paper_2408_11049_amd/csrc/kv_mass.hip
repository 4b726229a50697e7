// kv_mass.hip -- the attention weights that a call's queries give each cached token, summed
// over rows and the query heads of a KV head, added to what the token had:
//   w(j) = sum_r exp(scale q_r . k_j - lse_r)
//
// A wave holds 32 or 64 keys of one KV head in registers as the second operand while the rows of
// Q go past in LDS: S = Q K^T leaves a lane one key and 16 rows, so the sum over rows is in the
// lane but for one exchange at the end.  Every sum has a fixed order: a tile's 32 rows first,
// then the tiles, then the parts.
//
//   mass_step    few rows (a step's): bound by reading K, which goes through LDS in whole rows
//                (the operand's own pattern, 32 bytes of each row an instruction, streams at two
//                thirds of that): 64 x 5 rows over 2054 tokens 52 us, 5.4 TB/s;
//   mass_prompt  many rows (a prompt's): bound by the matrix and vector units alike.  The rows are
//                cut into parts, whose sums mass_reduce adds, so that early keys, which
//                most rows see, are no longer work than late ones: a prompt of 4096 tokens, 32
//                heads on 8, 92 + 5 us.
#include <type_traits>

#include "kv_stream.h"

namespace md {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

namespace {

constexpr float kLog2e = 1.44269504088896340736f;

// Byte offset of a key's row, or -1: no token of the pool.
__device__ __forceinline__ int64_t key_offset(const MassParams& p, int b, int hk, int key, int es) {
  int64_t off;
  if (p.c.page_table != nullptr) {
    const int pid = p.c.page_table[static_cast<int64_t>(b) * p.c.max_pages + (key >> p.c.page_shift)];
    if (pid < 0 || pid >= p.c.num_pages) return -1;
    off = static_cast<int64_t>(pid) * p.c.s_blk +
          static_cast<int64_t>(key & ((1 << p.c.page_shift) - 1)) * p.c.s_tok;
  } else {
    off = static_cast<int64_t>(b) * p.c.s_blk + static_cast<int64_t>(key) * p.c.s_tok;
  }
  return (off + static_cast<int64_t>(hk) * p.c.s_head) * es;
}

// Row r = i * G + g of KV head hk: its place among the [B, L, Hq] rows.
__device__ __forceinline__ int64_t query_row(const MassParams& p, int b, int hk, int r) {
  const int i = r / p.G;
  return (static_cast<int64_t>(b) * p.L + i) * p.Hq + hk * p.G + (r - i * p.G);
}

// What a row's score gets under the exponential: -lse in log2; -inf: the row weighs nothing.
__device__ __forceinline__ float neg_lse(float lse) {
  return lse == -INFINITY ? -INFINITY : -lse * kLog2e;
}

template <int D, bool BF16>
__device__ __forceinline__ f32x16 scores(const u32x4 (&q)[D * (BF16 ? 2 : 4) / 32],
                                         const u32x4 (&k)[D * (BF16 ? 2 : 4) / 32]) {
  f32x16 s = {};
#pragma unroll
  for (int st = 0; st < Tile<D, BF16>::CH / 2; ++st) {
    if constexpr (BF16) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, q[st]),
                                                  __builtin_bit_cast(bf16x8, k[st]), s, 0, 0, 0);
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(q[st][j]), __uint_as_float(k[st][j]), s,
                                                 0, 0, 0);
    }
  }
  return s;
}

// The weights of a tile's 16 rows in this lane (8 (e / 4) + 4 half + e % 4), summed.  nl: the tile's
// neg_lse.  masked: rows before `first` do not see the lane's key, and rows of -inf count nothing
// whatever their score (else -inf alone does that, where the score is finite).
__device__ __forceinline__ float weigh(const f32x16& s, const float* nl, float scale_log2, int half,
                                       bool masked, int first) {
  float part[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const f32x4 l4 = *reinterpret_cast<const f32x4*>(nl + 8 * j + 4 * half);
    part[j] = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      float x = __builtin_amdgcn_exp2f(__builtin_fmaf(s[4 * j + e], scale_log2, l4[e]));
      if (masked && (l4[e] == -INFINITY || 8 * j + 4 * half + e < first)) x = 0.f;
      part[j] += x;
    }
  }
  return (part[0] + part[1]) + (part[2] + part[3]);
}

// w onto the token's weight so far; a newest token has none.
__device__ __forceinline__ void store(const MassParams& p, int unit, int b, int key, int base, float w,
                                      float old) {
  const int64_t slot = static_cast<int64_t>(unit) * p.slot_stride + key;
  p.mass[slot] = key >= base ? w : old + w;
  if (key >= base) p.slot_pos[slot] = p.pos0[b] + (key - base);
}

// Up to RT tiles of 32 rows, in LDS for the whole call; each wave streams its own tiles of 32 keys of a
// part of the sequence, the next one on its way while one is weighed.
template <int D, bool BF16, int RT>
__global__ void __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(D == 128 && !BF16 ? 1 : 2)))
mass_step(const MassParams p) {
  using T = Tile<D, BF16>;
  constexpr int ST = T::CH / 2;
  __shared__ __attribute__((aligned(16))) unsigned char kt[4][32 * T::ROW];
  __shared__ __attribute__((aligned(16))) unsigned char qt[RT * 32 * T::ROW];
  __shared__ __attribute__((aligned(16))) float nl[RT * 32];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);
  // The heads of a sequence's part on one XCD, one after another: they share its token rows.
  const int x8 = static_cast<int>(blockIdx.x) >> 3;
  const int x = x8 / p.Hkv * 8 + (static_cast<int>(blockIdx.x) & 7);
  if (x >= p.B * p.key_parts) return;
  const int hk = x8 % p.Hkv, part = x % p.key_parts, b = x / p.key_parts, unit = b * p.Hkv + hk;
  const int S = uniform(min(max(p.c.lens[b], 0), p.c.max_len));
  const int n_tiles = (S + 31) / 32;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * part / p.key_parts);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (part + 1) / p.key_parts);
  if (t0 >= t1) return;
  const int base = S - p.L;  // the key that row 0 sits at (below 0: a length shorter than L)
  int n_count = p.L;
  if (p.accepted) n_count = min(max(uniform(p.accepted[b]), 0), p.L - 1) + 1;
  const int r_end = n_count * p.G;

  Stream<D, BF16, false, false> rows(p.c, b, hk, min(S, t1 * 32), lane);  // (the next part is not read ahead)
  const int first = t0 + wave;
  const int block = rows.load_block(first);
  int block_next = rows.load_block(first + 4);
  // A token's weight so far comes ahead of its tile: loads return in order, and behind the next tile's
  // it would hold up this one.
  const float* const weights = p.mass + static_cast<int64_t>(unit) * p.slot_stride;
  float old = weights[min(first * 32 + l32, S - 1)];
  rows.load(first, block);
#pragma unroll
  for (int n = 0; n < RT * 32 * T::CH / 256; ++n) {
    const int c = n * 256 + tid, r = c / T::CH;
    u32x4 q = {0, 0, 0, 0};
    if (r < r_end)
      q = *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(p.q) +
                                          query_row(p, b, hk, r) * T::ROW + (c % T::CH) * 16);
    *reinterpret_cast<u32x4*>(qt + T::at(r, c % T::CH)) = q;
  }
  if (tid < RT * 32) nl[tid] = tid < r_end ? neg_lse(p.lse[query_row(p, b, hk, tid)]) : -INFINITY;
  __syncthreads();

  for (int t = first; t < t1; t += 4) {
    rows.store(kt[wave], nullptr);
    const int ahead = rows.load_block(t + 8);
    const float old_next = weights[min(t * 32 + 128 + l32, S - 1)];
    rows.load(t + 4, block_next);
    block_next = ahead;
    wave_sync();
    u32x4 k[ST];
#pragma unroll
    for (int st = 0; st < ST; ++st)
      k[st] = *reinterpret_cast<const u32x4*>(kt[wave] + T::at(l32, 2 * st + half));
    wave_sync();  // the next tile overwrites this one
    const int key = t * 32 + l32;
    const int sees = max(0, key - base) * p.G;  // the first row that sees this lane's key
    float w = 0.f;
    for (int r0 = 0; r0 < r_end; r0 += 32) {
      u32x4 q[ST];
#pragma unroll
      for (int st = 0; st < ST; ++st)
        q[st] = *reinterpret_cast<const u32x4*>(qt + T::at(r0 + l32, 2 * st + half));
      w += weigh(scores<D, BF16>(q, k), nl + r0, p.scale_log2, half, true, sees - r0);
    }
    w += __shfl_xor(w, 32);
    if (!half && key < S) store(p, unit, b, key, base, w, old);
    old = old_next;
  }
}

// The rows that a prompt's key blocks of 256 keys see, in tiles of 64.  Blocks go in pairs, i with the i-th
// from the end, as one list of tiles, i's first: later keys have fewer rows, and every pair has as many.
// Part c takes every n_parts-th tile from the c-th on, and so as many masked ones as the others (in
// contiguous parts those with the diagonal took half as long again).
struct PairRows {
  int kb[2], r0[2], tiles[2], n_parts;
  __device__ __forceinline__ PairRows(int pair, int S, int base, int G, int r_end, int parts) : n_parts(parts) {
    const int n = (S + kMassPromptKeys - 1) / kMassPromptKeys;
    kb[0] = pair;
    kb[1] = n - 1 - pair;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      r0[x] = max(0, kb[x] * kMassPromptKeys - base) * G;
      tiles[x] = max(0, (r_end - r0[x] + 63) >> 6);
    }
    if (kb[1] <= kb[0]) tiles[1] = 0;  // a block in the middle is a pair by itself
  }
  // The part's first tile of the first or second block (from tiles[seg] on: none).
  __device__ __forceinline__ int first(int seg, int part) const {
    if (!seg) return part;
    const int x = part - tiles[0] % n_parts;
    return x < 0 ? x + n_parts : x;
  }
};

// A part of a pair's rows, 64 of them in LDS at a time (two such tiles in turn); 256 keys a
// workgroup, 64 a wave.
template <int D, bool BF16>
__global__ void __launch_bounds__(256)
__attribute__((amdgpu_waves_per_eu(D == 128 && !BF16 ? 1 : 2)))
mass_prompt(const MassParams p) {
  using T = Tile<D, BF16>;
  constexpr int ST = T::CH / 2;
  constexpr int NR = 64, QP = NR * T::CH / 256;
  __shared__ __attribute__((aligned(16))) unsigned char qt[2][NR * T::ROW];
  __shared__ __attribute__((aligned(16))) float nl[2][NR];
  __shared__ int odd[2];  // the tile has rows that count nothing

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int units = p.B * p.Hkv;
  const int unit = static_cast<int>(blockIdx.x) % units;
  const int part = (static_cast<int>(blockIdx.x) / units) % p.row_parts;
  const int pair = static_cast<int>(blockIdx.x) / units / p.row_parts;
  const int hk = unit % p.Hkv, b = unit / p.Hkv;
  const int S = uniform(min(max(p.c.lens[b], 0), p.c.max_len));
  const int base = S - p.L;
  int n_count = p.L;
  if (p.accepted) n_count = min(max(uniform(p.accepted[b]), 0), p.L - 1) + 1;
  const PairRows list(pair, S, base, p.G, n_count * p.G, p.row_parts);
  if (list.kb[1] < list.kb[0]) return;

  for (int seg = 0; seg <= (list.kb[1] > list.kb[0]); ++seg) {
    // Rows of this part that count and see a key of the block.
    const int kb = seg ? list.kb[1] : list.kb[0], r0_block = seg ? list.r0[1] : list.r0[0];
    const int tiles = seg ? list.tiles[1] : list.tiles[0], first = list.first(seg, part);
    if (first >= tiles && p.row_parts > 1) continue;  // mass_reduce does not ask for it
    const int r_begin = r0_block + first * NR, r_end = min(n_count * p.G, r0_block + tiles * NR);
    const int next = NR * p.row_parts;  // rows to the next tile

    int key[2], sees[2];
    u32x4 k[2][ST];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      key[x] = kb * kMassPromptKeys + wave * 64 + x * 32 + l32;
      sees[x] = max(0, min(key[x], S - 1) - base) * p.G;
      const int64_t off = key[x] < S ? key_offset(p, b, hk, key[x], T::ES) : -1;
#pragma unroll
      for (int st = 0; st < ST; ++st)
        k[x][st] = *reinterpret_cast<const u32x4*>(p.c.k + (off < 0 ? 0 : off) + (2 * st + half) * 16);
    }

    // Four threads a row.  Their row's place moves by a step of whole tokens and a rest among the G
    // of a token, without a division (which made 117 us of 108).
    const int64_t token = static_cast<int64_t>(p.Hq) * T::ROW;
    const int step_g = next % p.G;
    const int64_t step = next / p.G * token + step_g * T::ROW, carry = token - static_cast<int64_t>(p.G) * T::ROW;
    const unsigned char* at = static_cast<const unsigned char*>(p.q) +
                              query_row(p, b, hk, r_begin + tid / 4) * T::ROW + (tid & 3) * 16;
    int at_g = (r_begin + tid / 4) % p.G;
    u32x4 sq[QP];
    float sl = -INFINITY;
    auto load_tile = [&](int r0) {
      if (r0 >= r_end) return;
      const bool there = r0 + tid / 4 < r_end;
#pragma unroll
      for (int n = 0; n < QP; ++n)
        sq[n] = there ? *reinterpret_cast<const u32x4*>(at + n * 64) : u32x4{0, 0, 0, 0};
      at_g += step_g;
      const bool over = at_g >= p.G;
      at += step + (over ? carry : 0);
      at_g -= over ? p.G : 0;
      // As it is: arithmetic here would wait for the tile's rows, which were asked for before it.
      if (tid < NR) sl = r0 + tid < r_end ? p.lse[query_row(p, b, hk, r0 + tid)] : -INFINITY;
    };
    auto store_tile = [&](int buf, int r0) {
      if (r0 >= r_end) return;
#pragma unroll
      for (int n = 0; n < QP; ++n) *reinterpret_cast<u32x4*>(qt[buf] + T::at(tid / 4, n * 4 + (tid & 3))) = sq[n];
      if (tid < NR) {
        const float x = neg_lse(sl);
        nl[buf][tid] = x;
        const bool none = __any(x == -INFINITY);
        if (tid == 0) odd[buf] = none;
      }
    };

    float w[2] = {};
    load_tile(r_begin);
    store_tile(0, r_begin);
    // The keys arrive here: a wait for them inside the loop would be one for the rows on their way too.
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int st = 0; st < ST; ++st) asm volatile("" : "+v"(k[x][st]));
    load_tile(r_begin + next);
    __syncthreads();
    int buf = 0;
    for (int r0 = r_begin; r0 < r_end; r0 += next, buf ^= 1) {
      store_tile(buf ^ 1, r0 + next);
      load_tile(r0 + 2 * next);
      // One block of 32 rows and 32 keys is weighed beside the next one's products.  (The compiler's order
      // stands: one matrix instruction to four vector ones, forced, took the same 97 us.)
      auto weigh_tile = [&](auto masked) {
        u32x4 q[ST];
        f32x16 s[2];
        auto read_q = [&](int y) {
#pragma unroll
          for (int st = 0; st < ST; ++st)
            q[st] = *reinterpret_cast<const u32x4*>(qt[buf] + T::at(y * 32 + l32, 2 * st + half));
        };
        read_q(0);
        s[0] = scores<D, BF16>(q, k[0]);
#pragma unroll
        for (int n = 0; n < NR / 16; ++n) {
          const int y = n / 2, x = n & 1;
          if (n + 1 < NR / 16) {
            if (x) read_q(y + 1);
            s[x ^ 1] = scores<D, BF16>(q, k[x ^ 1]);
          }
          w[x] += weigh(s[x], nl[buf] + y * 32, p.scale_log2, half, masked, sees[x] - (r0 + y * 32));
        }
      };
      // Two instances: the mask costs as much as the rest of the vector work.
      if (odd[buf] || __any(r0 < sees[1])) {
        if (__any(r0 + NR > sees[0])) weigh_tile(std::true_type{});  // else no row sees the wave's keys
      } else {
        weigh_tile(std::false_type{});
      }
      __syncthreads();
    }
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const float sum = w[x] + __shfl_xor(w[x], 32);
      if (half || key[x] >= S) continue;
      if (p.row_parts == 1)
        store(p, unit, b, key[x], base, sum, p.mass[static_cast<int64_t>(unit) * p.slot_stride + key[x]]);
      else
        p.parts[(static_cast<int64_t>(part) * units + unit) * p.c.max_len + key[x]] = sum;
    }
  }
}

// The parts' sums, in order; a thread a key.
__global__ void __launch_bounds__(256)
mass_reduce(const MassParams p) {
  const int units = p.B * p.Hkv;
  const int unit = static_cast<int>(blockIdx.x) % units;
  const int key = static_cast<int>(blockIdx.x) / units * 256 + static_cast<int>(threadIdx.x);
  const int b = unit / p.Hkv;
  const int S = uniform(min(max(p.c.lens[b], 0), p.c.max_len));
  if (key >= S) return;
  const int base = S - p.L;
  int n_count = p.L;
  if (p.accepted) n_count = min(max(uniform(p.accepted[b]), 0), p.L - 1) + 1;
  const int kb = uniform(key / kMassPromptKeys), n_kb = (S + kMassPromptKeys - 1) / kMassPromptKeys;
  const int seg = kb > n_kb - 1 - kb;
  const PairRows list(seg ? n_kb - 1 - kb : kb, S, base, p.G, n_count * p.G, p.row_parts);
  const int tiles = seg ? list.tiles[1] : list.tiles[0];
  float w = 0.f;
#pragma unroll 4
  for (int c = 0; c < p.row_parts; ++c)
    if (list.first(seg, c) < tiles) w += p.parts[(static_cast<int64_t>(c) * units + unit) * p.c.max_len + key];
  store(p, unit, b, key, base, w, p.mass[static_cast<int64_t>(unit) * p.slot_stride + key]);
}

}  // namespace

hipError_t launch_kv_mass(const MassParams& p, const MassPlan& pl, int head_dim, bool bf16,
                          hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(pl.n_wgs)), block(256);
#define MD_MASS(D, BF)                                                          \
  do {                                                                          \
    if (pl.prompt)                                                              \
      hipLaunchKernelGGL((mass_prompt<D, BF>), grid, block, 0, s, p);           \
    else if (p.L * p.G <= 32)                                                   \
      hipLaunchKernelGGL((mass_step<D, BF, 1>), grid, block, 0, s, p);          \
    else                                                                        \
      hipLaunchKernelGGL((mass_step<D, BF, 4>), grid, block, 0, s, p);          \
  } while (0)
  if (head_dim == 128) {
    if (bf16) MD_MASS(128, true); else MD_MASS(128, false);
  } else {
    if (bf16) MD_MASS(64, true); else MD_MASS(64, false);
  }
#undef MD_MASS
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.row_parts == 1) return e;
  hipLaunchKernelGGL(mass_reduce, dim3(static_cast<uint32_t>(pl.reduce_wgs)), block, 0, s, p);
  return hipGetLastError();
}

}  // namespace md
