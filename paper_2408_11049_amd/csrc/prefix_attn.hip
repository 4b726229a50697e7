// prefix_attn.hip -- attention of a batch whose sequences share a long prefix: the prefix's
// K and V are read once for all query rows of its group, each sequence's own cache for
// its own rows, and the parts meet by log-sum-exp (md_merge_lse's kernels).
//
//   prefix_stream  32 query rows of a KV head against a part of a range of keys (of the prefix, or of
//                  one sequence's own tokens), each wave its own tiles of 32 keys: bound by reading K
//                  and V.  Own caches always, prefixes of few rows.
//   prefix_wide    256 rows against a part of the prefix, in tiles that the waves share: bound by the
//                  matrix and vector units.
//
// 32 query heads on 8 of 128 channels, bf16, 16-token pages: 64 x 5 rows over 32768 shared tokens 190 us
// (wide, 0.9 PFLOP/s), over 256 .. 2048 own ones 70 us (stream, 4.3 TB/s); 64 x 1 rows 57 us and, of up to
// 1024, 40 us; 8 x 1 rows over 8001 and up to 301 in one launch of the stream 16 us.
//
// Both compute S^T = K Q^T, which leaves a lane one query row: the softmax needs no shuffles but one
// exchange between the halves of the wave when the running maximum moves, and P^T is in place as the
// second product's operand, O^T += V^T P^T, V read transposed from LDS.
#include "kv_stream.h"

namespace md {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

namespace {

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}

constexpr float kLazy = 8.f;  // log2 headroom before a running maximum must move

// Reports page ids outside the pool among the pages of tokens [from, to) of a block: a look of its
// own ahead of the stream, for callers that ask.
__device__ void check_pages(const KvView& c, int blk, int from, int to, int32_t* err) {
  const int64_t size = int64_t{1} << c.page_shift;
  for (int64_t page = from / size + threadIdx.x; page <= (to - 1) / size; page += 256) {
    const int id = c.page_table[static_cast<int64_t>(blk) * c.max_pages + page];
    if (id < 0 || id >= c.num_pages)
      atomicOr(reinterpret_cast<unsigned int*>(err), static_cast<unsigned int>(MD_ERRW_BAD_PAGE));
  }
}
__device__ __forceinline__ void check_length(int raw, int least, int most, int32_t* err) {
  const int bits = (raw > most ? MD_ERRW_LONG_LEN : 0) | (raw < least ? MD_ERRW_SHORT_LEN : 0);
  if (bits) atomicOr(reinterpret_cast<unsigned int*>(err), static_cast<unsigned int>(bits));
}

// The lse of a part from its maximum (in log2) and sum.  An empty part's is -inf; a NaN stays NaN, for
// -inf would tell the merge that the part is empty.
__device__ __forceinline__ float part_lse(float m, float sum) {
  return sum > 0.f ? (m + __builtin_amdgcn_logf(sum)) * 0.69314718055994530942f
                   : (sum == sum ? -INFINITY : sum);
}

// A row's part: its normalised O (32 channels a block, 8 j + 4 half + .. of each in this lane) and
// lse, from the maximum m (in log2) and the sum of the weights in both halves.
template <int D>
__device__ __forceinline__ void store_part(const PrefixParams& p, int part, int64_t row, int half,
                                           const f32x16 (&acc)[D / 32], float m, float sum) {
  const float inv = sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
  const int64_t prow = static_cast<int64_t>(part) * p.n_rows + row;
  float* const out = p.part_o + prow * D + 4 * half;
#pragma unroll
  for (int cb = 0; cb < D / 32; ++cb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 x = {acc[cb][4 * j], acc[cb][4 * j + 1], acc[cb][4 * j + 2], acc[cb][4 * j + 3]};
      *reinterpret_cast<f32x4*>(out + cb * 32 + 8 * j) = x * inv;
    }
  if (half == 0) p.part_lse[prow] = part_lse(m, sum);
}

// Places of a block of 32 keys in an LDS tile as matrix operands; rows 32 (V: 16) further on are a
// constant away, for they are turned alike.
//   K  lane: key l32, channels of chunk 2 st + half
//   V  transposed reads: lane k of 16 supplies row k / 4 and four channels of it, and gets one channel
//      of the four rows; lo and hi are the slots' keys 4 half + {0..3} and {8..11} of 16
template <int D, bool BF16>
struct Places {
  using T = Tile<D, BF16>;
  int k[T::CH / 2], v[2][D / 32];
  __device__ __forceinline__ explicit Places(int lane) {
    const int half = lane >> 5;
#pragma unroll
    for (int st = 0; st < T::CH / 2; ++st) k[st] = T::at(lane & 31, 2 * st + half);
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int cb = 0; cb < D / 32; ++cb)
        v[h][cb] = T::at(8 * h + 4 * half + ((lane & 15) >> 2),
                         cb * 4 + ((lane >> 4) & 1) * 2 + ((lane & 3) >> 1)) + (lane & 1) * 8;
  }
  // V of 16 keys from `tile` on, channels 32 cb ...
  __device__ __forceinline__ bf16x8 read_v(const unsigned char* tile, int cb) const {
    const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + v[0][cb])));
    const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(tile + v[1][cb])));
    return __builtin_bit_cast(bf16x8, u32x4{lo.x, lo.y, hi.x, hi.y});
  }
};

template <int D, bool BF16, bool CACHED>
__global__ void __launch_bounds__(256)
// Two workgroups a compute unit; 128 fp32 channels need more than 256 registers.
__attribute__((amdgpu_waves_per_eu(D == 128 && !BF16 ? 1 : 2)))
prefix_stream_kernel(const PrefixParams p) {
  using T = Tile<D, BF16>;
  constexpr int KEYS = kPrefixStreamTile;
  static_assert(KEYS == Stream<D, BF16, true, CACHED>::KEYS, "tiles of the plan");
  constexpr int ST = T::CH / 2;       // 16-byte operand chunks a lane holds of its row
  constexpr int CB = D / 32;          // blocks of 32 channels
  constexpr int BYTES = KEYS * T::ROW;
  // A wave's K tile and V tile; after the loop its O (as its lanes hold it) for the others.
  __shared__ __attribute__((aligned(16))) unsigned char lds[4][2 * BYTES];
  __shared__ float l_m[4][32], l_l[4][32];
  static_assert(2 * BYTES >= CB * 16 * 64 * 4, "O fits in a wave's tiles");

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);

  // What this workgroup does.  The row blocks that read one part of a range are neighbours on one XCD and
  // find its K and V in that L2; so are the heads of a sequence's part, which share token rows.
  const bool pre = static_cast<int>(blockIdx.x) < p.n_pre;
  const int x8 = (static_cast<int>(blockIdx.x) - (pre ? 0 : p.n_pre)) >> 3, xcd = static_cast<int>(blockIdx.x) & 7;
  int blk, hk, chunk, C, row_base, tok0, n_rows;
  if (pre) {
    const int u = x8 / p.row_blocks * 8 + xcd;
    C = p.c_pre;
    if (u >= p.P * p.Hkv * C) return;
    chunk = u % C;
    hk = (u / C) % p.Hkv;
    blk = u / (C * p.Hkv);
    row_base = x8 % p.row_blocks * 32;
    tok0 = blk * p.n * p.L;
    n_rows = p.group_rows;
  } else {
    const int per = p.Hkv * p.own_blocks, v = x8 / per * 8 + xcd;
    C = p.c_own;
    if (v >= p.P * p.n * C) return;
    row_base = x8 % p.own_blocks * 32;
    hk = x8 / p.own_blocks % p.Hkv;
    chunk = v % C;
    blk = v / C;
    tok0 = blk * p.L;
    n_rows = p.L * p.G;
  }
  const KvView c = pre ? p.pre : p.own;
  const int raw_len = uniform(c.lens[blk]);
  const int len = min(max(raw_len, 0), c.max_len);
  const int n_tiles = (len + KEYS - 1) / KEYS;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * chunk / C);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (chunk + 1) / C);
  const int end = min(len, t1 * KEYS);
  const bool paged = c.page_table != nullptr;
  if (p.err && row_base == 0 && hk == 0) {
    if (chunk == 0 && tid == 0) {
      check_length(raw_len, pre ? 0 : p.L, c.max_len, p.err);
      // Prefixes of no tokens have no workgroup: the first of their sequences looks at the length.
      if (p.c_pre == 0 && blk % p.n == 0) check_length(p.pre.lens[blk / p.n], 0, 0, p.err);
    }
    if (paged && t0 < t1) check_pages(c, blk, t0 * KEYS, end, p.err);
  }

  // This lane's query row, and the keys it sees: those below lim.
  const int r = row_base + l32, tq = r / p.G;
  const bool valid = r < n_rows;
  const int64_t row_g = static_cast<int64_t>(tok0 + tq) * p.Hq + hk * p.G + (r - tq * p.G);
  const int lim = min(end, valid && !pre ? len - p.L + tq + 1 : end);

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};

  if (t0 + wave < t1) {
    const Places<D, BF16> at(lane);
    unsigned char* const kt = lds[wave];
    unsigned char* const vt = lds[wave] + BYTES;
    Stream<D, BF16, true, CACHED> rows(c, blk, hk, end, lane);
    const int block = rows.load_block(t0 + wave);
    int block_next = rows.load_block(t0 + wave + 4);
    rows.load(t0 + wave, block);
    // Q as the second operand: chunk 2 st + half of the row, that is channels 8 (bf16) or 4 a
    // chunk; K's chunks are taken in the same order.
    u32x4 q[ST];
#pragma unroll
    for (int x = 0; x < ST; ++x)
      q[x] = valid ? *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(p.q) +
                                                     row_g * T::ROW + (2 * x + half) * 16)
                   : u32x4{0, 0, 0, 0};

    for (int t = t0 + wave; t < t1; t += 4) {
      // The tile to LDS; its registers take the wave's next one while this is computed.
      rows.store(kt, vt);
      const int ahead = rows.load_block(t + 8);
      rows.load(t + 4, block_next);
      block_next = ahead;
      wave_sync();

      // S^T: a lane gets keys 8 (e / 4) + 4 half + e % 4 of its row.
      f32x16 s = {};
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        const u32x4 kk = *reinterpret_cast<const u32x4*>(kt + at.k[st]);
        if constexpr (BF16) {
          s = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kk),
                                                      __builtin_bit_cast(bf16x8, q[st]), s, 0, 0, 0);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            s = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kk[j]), __uint_as_float(q[st][j]), s, 0, 0, 0);
        }
      }
      const int key0 = t * KEYS;
      if (__any(lim < key0 + KEYS)) {
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[e] = key0 + 8 * (e >> 2) + 4 * half + (e & 3) < lim ? s[e] : -INFINITY;
      }
      float mx = s[0];
#pragma unroll
      for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[e]);
      mx *= p.scale_log2;
      // The running maximum moves only when some row's exceeds it by 2^kLazy: weights stay below
      // that, and most tiles skip the rescale.
      if (__any(mx > m_run + kLazy)) {
        const float m_new = fmaxf(m_run, fmaxf(mx, __shfl_xor(mx, 32)));
        const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
        m_run = m_new;
        l_run *= f;
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) acc[cb] *= f;
      }
      const float m_use = m_run == -INFINITY ? 0.f : m_run;
      float sum[4] = {};
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[e], p.scale_log2, -m_use));
        sum[e & 3] += s[e];
      }
      l_run += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      // O^T += V^T P^T.
      if constexpr (BF16) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          // Weights to bf16, half a step each: the matrix units take bf16, and O is rounded to
          // it in the end.
          const u32x4 pb = {pack2(s[8 * x], s[8 * x + 1]), pack2(s[8 * x + 2], s[8 * x + 3]),
                            pack2(s[8 * x + 4], s[8 * x + 5]), pack2(s[8 * x + 6], s[8 * x + 7])};
#pragma unroll
          for (int cb = 0; cb < CB; ++cb)
            acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(at.read_v(vt + 16 * x * T::ROW, cb),
                                                              __builtin_bit_cast(bf16x8, pb), acc[cb], 0, 0, 0);
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const int channel = cb * 32 + l32;
            const float va = *reinterpret_cast<const float*>(vt + T::at(key, channel >> 2) + (channel & 3) * 4);
            acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(va, s[e], acc[cb], 0, 0, 0);
          }
        }
      }
      wave_sync();  // the next tile overwrites this one
    }
  }

  // ---- the waves' parts of the rows, each lane's like the other waves' same lane's
  l_run += __shfl_xor(l_run, 32);
  if (half == 0) {
    l_m[wave][l32] = m_run;
    l_l[wave][l32] = l_run;
  }
  wave_sync();
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int j = 0; j < 4; ++j)
      *reinterpret_cast<f32x4*>(lds[wave] + ((cb * 4 + j) * 64 + lane) * 16) =
          f32x4{acc[cb][4 * j], acc[cb][4 * j + 1], acc[cb][4 * j + 2], acc[cb][4 * j + 3]};
  __syncthreads();
  if (!valid) return;
  float m = -INFINITY, sum = 0.f, f[4];
#pragma unroll
  for (int w = 0; w < 4; ++w) m = fmaxf(m, l_m[w][l32]);
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    f[w] = l_m[w][l32] == -INFINITY ? (l_l[w][l32] == 0.f ? 0.f : 1.f) : __builtin_amdgcn_exp2f(l_m[w][l32] - m);
    sum += l_l[w][l32] * f[w];
  }
  const float inv = sum > 0.f ? 1.f / sum : (sum == sum ? 0.f : sum);
  const int64_t prow = static_cast<int64_t>(pre ? chunk : p.c_pre + chunk) * p.n_rows + row_g;
#pragma unroll
  for (int y = 0; y < (CB + 3) / 4; ++y) {
    const int cb = y * 4 + wave;
    if (cb >= CB) break;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      f32x4 o = {};
#pragma unroll
      for (int w = 0; w < 4; ++w)
        o += *reinterpret_cast<const f32x4*>(lds[w] + ((cb * 4 + j) * 64 + lane) * 16) * f[w];
      *reinterpret_cast<f32x4*>(p.part_o + prow * D + cb * 32 + 8 * j + 4 * half) = o * inv;
    }
  }
  if (tid < 32) p.part_lse[prow] = part_lse(m, sum);
}

// The prefix's part for groups of many rows, bf16: 256 rows a workgroup, two tiles of 32 a wave, A and B, so that
// what a wave reads of K and V from LDS serves twice the products (with 32 rows the reads alone take longer
// than the matrix instructions).  One wave a SIMD then holds Q, O and S in
// registers, and hides its vector work behind its own matrix instructions: per 32 keys
//   S_B = K Q_B^T        beside the softmax of S_A,
//   O_A += V^T P_A^T     beside the softmax of S_B,
//   O_B += V^T P_B^T,    then S_A of the next 32 keys.
// The softmax goes ahead with the old maximum and is redone in the rare block that exceeds it by
// 2^kLazy, so that no branch stands between the products and the vector work beside them.
//
// Tiles of 64 tokens are whole but for the last one of the prefix, which comes after the loop.  In a whole
// tile a wave's load instruction covers RPW rows of one page (pages hold at least RPW tokens here) at
// one scalar address and a fixed offset a lane: no address arithmetic in the vector unit.
template <int D, bool PAGED>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(1, 1)))
prefix_wide_kernel(const PrefixParams p) {
  using T = Tile<D, true>;
  constexpr int KEYS = kPrefixWideTile, ST = T::CH / 2, CB = D / 32, RPW = kPrefixWidePage(D);
  constexpr int NP = KEYS * T::CH / 256;  // chunks of K a thread moves
  static_assert(RPW == 64 / T::CH, "rows of a load instruction");
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][KEYS * T::ROW];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);
  const int t8 = static_cast<int>(blockIdx.x) >> 3;
  const int u = (t8 / p.row_blocks) * 8 + (static_cast<int>(blockIdx.x) & 7);
  if (u >= p.P * p.Hkv * p.c_pre) return;
  const int chunk = u % p.c_pre, hk = (u / p.c_pre) % p.Hkv, blk = u / (p.c_pre * p.Hkv);
  const int row_base = (t8 % p.row_blocks) * kPrefixWideRows, tok0 = blk * p.n * p.L;
  const KvView& c = p.pre;
  const int raw_len = uniform(c.lens[blk]);
  const int len = min(max(raw_len, 0), c.max_len);
  const int n_tiles = (len + KEYS - 1) / KEYS;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * chunk / p.c_pre);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (chunk + 1) / p.c_pre);
  const int tw = min(t1, len / KEYS);  // whole tiles: [t0, tw)
  if (p.err && row_base == 0 && hk == 0) {
    if (chunk == 0 && tid == 0) check_length(raw_len, 0, c.max_len, p.err);
    if (PAGED && t0 < t1) check_pages(c, blk, t0 * KEYS, min(len, t1 * KEYS), p.err);
  }

  const int r0 = row_base + wave * 64;
  int64_t row_g[2];
  bool valid[2];
  u32x4 q[2][ST];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const int r = r0 + x * 32 + l32, tq = r / p.G;
    valid[x] = r < p.group_rows;
    row_g[x] = static_cast<int64_t>(tok0 + tq) * p.Hq + hk * p.G + (r - tq * p.G);
#pragma unroll
    for (int st = 0; st < ST; ++st)
      q[x][st] = valid[x] ? *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(p.q) +
                                                            row_g[x] * T::ROW + (2 * st + half) * 16)
                          : u32x4{0, 0, 0, 0};
  }

  const Places<D, true> at(lane);
  float m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
  f32x16 acc[2][CB], s[2];
#pragma unroll
  for (int x = 0; x < 2; ++x)
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) acc[x][cb] = f32x16{};
  bf16x8 kf[ST], vf[2][CB];
  u32x4 pb[2][2];

  auto read_k = [&](const unsigned char* kt) {
#pragma unroll
    for (int st = 0; st < ST; ++st)
      kf[st] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4*>(kt + at.k[st]));
  };
  auto read_v = [&](const unsigned char* vt) {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) vf[x][cb] = at.read_v(vt + 16 * x * T::ROW, cb);
  };
  auto scores = [&](int x) {
    s[x] = f32x16{};
#pragma unroll
    for (int st = 0; st < ST; ++st)
      s[x] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[st], __builtin_bit_cast(bf16x8, q[x][st]), s[x], 0, 0, 0);
  };
  auto values = [&](int x) {
#pragma unroll
    for (int y = 0; y < 2; ++y)
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
        acc[x][cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[y][cb], __builtin_bit_cast(bf16x8, pb[x][y]),
                                                             acc[x][cb], 0, 0, 0);
  };
  // Weights of s[x] under the running maximum: their sum and bf16 operands (half a step each: the
  // matrix units take bf16, and O is rounded to it in the end), and the block's own maximum.
  auto weights = [&](int x, float& sum, float& mx) {
    const float m_use = m[x] == -INFINITY ? 0.f : m[x];
    float w[16];
#pragma unroll
    for (int e = 0; e < 16; ++e)
      w[e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[x][e], p.scale_log2, -m_use));
    mx = s[x][0];
#pragma unroll
    for (int e = 1; e < 16; ++e) mx = fmaxf(mx, s[x][e]);
    float a[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) a[e] = (w[e] + w[4 + e]) + (w[8 + e] + w[12 + e]);
    sum = (a[0] + a[1]) + (a[2] + a[3]);
#pragma unroll
    for (int y = 0; y < 2; ++y)
      pb[x][y] = u32x4{pack2(w[8 * y], w[8 * y + 1]), pack2(w[8 * y + 2], w[8 * y + 3]),
                       pack2(w[8 * y + 4], w[8 * y + 5]), pack2(w[8 * y + 6], w[8 * y + 7])};
  };
  // The running maximum moved, where the block's is too far above it, and its weights redone.
  auto settle = [&](int x, float& sum, float mx) {
    // The weights are made here, not behind the branch, where nothing would run beside them.
#pragma unroll
    for (int y = 0; y < 2; ++y)
      asm volatile("" : "+v"(pb[x][y][0]), "+v"(pb[x][y][1]), "+v"(pb[x][y][2]), "+v"(pb[x][y][3]), "+v"(sum));
    mx *= p.scale_log2;
    if (__any(mx > m[x] + kLazy)) {
      const float m_new = fmaxf(m[x], fmaxf(mx, __shfl_xor(mx, 32)));
      const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[x] - m_new);
      m[x] = m_new;
      l[x] *= f;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) acc[x][cb] *= f;
      float again;
      weights(x, sum, again);
    }
    l[x] += sum;
  };

  if (t0 < tw) {
    // Tiles of even and of odd number: two are on their way in registers while one is computed.
    // Those past the last whole tile are that one again, so that every load is issued.
    u32x4 ks[2][NP], vs[2][NP];
    int pid[2];
    const uint32_t lane_off = static_cast<uint32_t>((lane / T::CH) * c.s_tok * T::ES + (lane % T::CH) * 16);
    auto load_pages = [&](int x, int t) {
      if constexpr (PAGED) {
        const int tok = min(t, tw - 1) * KEYS + (wave * NP + (lane & (NP - 1))) * RPW;
        pid[x] = c.page_table[static_cast<int64_t>(blk) * c.max_pages + (tok >> c.page_shift)];
      }
    };
    auto load = [&](int x, int t) {
      const int first = min(t, tw - 1) * KEYS + wave * NP * RPW;
      // A page outside the pool: its rows' results are unspecified, the pool's first is read.
      const int page = PAGED && pid[x] >= 0 && pid[x] < c.num_pages ? pid[x] : 0;
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        const int tok = first + n * RPW;
        const int64_t row =
            PAGED ? static_cast<int64_t>(__builtin_amdgcn_readlane(page, n)) * c.s_blk +
                        static_cast<int64_t>(tok & ((1 << c.page_shift) - 1)) * c.s_tok
                  : static_cast<int64_t>(blk) * c.s_blk + static_cast<int64_t>(tok) * c.s_tok;
        const int64_t byte = (row + static_cast<int64_t>(hk) * c.s_head) * T::ES;
        ks[x][n] = *reinterpret_cast<const u32x4*>(c.k + byte + lane_off);
        vs[x][n] = *reinterpret_cast<const u32x4*>(c.v + byte + lane_off);
      }
    };
    int place[NP];
#pragma unroll
    for (int n = 0; n < NP; ++n) place[n] = T::at((wave * NP + n) * RPW + lane / T::CH, lane % T::CH);
    auto store = [&](int x, int buf) {
#pragma unroll
      for (int n = 0; n < NP; ++n) {
        *reinterpret_cast<u32x4*>(lds[buf][0] + place[n]) = ks[x][n];
        *reinterpret_cast<u32x4*>(lds[buf][1] + place[n]) = vs[x][n];
      }
    };
    // One tile from buffer `buf`; set buf ^ 1 holds tile t + 1, which goes to the other buffer, and
    // takes t + 3.
    auto turn = [&](int t, int buf) {
      store(buf ^ 1, buf ^ 1);
      load(buf ^ 1, t + 3);
      load_pages(buf ^ 1, t + 5);
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        float sum, mx;
        read_v(lds[buf][1] + j * 32 * T::ROW);
        scores(1);
        weights(0, sum, mx);
#pragma unroll
        for (int i = 0; i < ST; ++i) {  // vector work between the matrix instructions
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          if (i < ST / 2) __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 48 / ST, 0);
          __builtin_amdgcn_sched_group_barrier(0x400, 16 / ST, 0);
        }
        settle(0, sum, mx);
        values(0);
        weights(1, sum, mx);
#pragma unroll
        for (int i = 0; i < 2 * CB; ++i) {
          __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x002, 48 / (2 * CB), 0);
          __builtin_amdgcn_sched_group_barrier(0x400, 16 / (2 * CB), 0);
        }
        settle(1, sum, mx);
        if (j == 1) __syncthreads();  // tile t + 1 is there; this buffer's last reads are done
        read_k(j == 1 ? lds[buf ^ 1][0] : lds[buf][0] + 32 * T::ROW);
        values(1);
        scores(0);
      }
    };
    load_pages(0, t0);
    load_pages(1, t0 + 1);
    load(0, t0);
    load_pages(0, t0 + 2);
    load(1, t0 + 1);
    load_pages(1, t0 + 3);
    store(0, 0);
    load(0, t0 + 2);
    load_pages(0, t0 + 4);
    __syncthreads();
    read_k(lds[0][0]);
    scores(0);
    for (int t = t0;; t += 2) {
      turn(t, 0);
      if (t + 1 >= tw) break;
      turn(t + 1, 1);
      if (t + 2 >= tw) break;
    }
    __syncthreads();  // the last look at the next tile is done
  }
  if (tw < t1) {  // the prefix's last tile, in part
#pragma unroll
    for (int n = 0; n < NP; ++n) {
      const int row = n * (256 / T::CH) + tid / T::CH, tok = tw * KEYS + row;
      u32x4 kv = {0, 0, 0, 0}, vv = kv;
      int64_t block = blk;
      if (PAGED && tok < len) {
        block = c.page_table[static_cast<int64_t>(blk) * c.max_pages + (tok >> c.page_shift)];
        if (block < 0 || block >= c.num_pages) block = 0;
      }
      if (tok < len) {
        const int64_t byte = (block * c.s_blk +
                              static_cast<int64_t>(PAGED ? tok & ((1 << c.page_shift) - 1) : tok) * c.s_tok +
                              static_cast<int64_t>(hk) * c.s_head) * T::ES + (tid % T::CH) * 16;
        kv = *reinterpret_cast<const u32x4*>(c.k + byte);
        vv = *reinterpret_cast<const u32x4*>(c.v + byte);
      }
      *reinterpret_cast<u32x4*>(lds[0][0] + T::at(row, tid % T::CH)) = kv;
      *reinterpret_cast<u32x4*>(lds[0][1] + T::at(row, tid % T::CH)) = vv;
    }
    __syncthreads();
#pragma unroll 1
    for (int j = 0; j < 2; ++j) {
      read_k(lds[0][0] + j * 32 * T::ROW);
      read_v(lds[0][1] + j * 32 * T::ROW);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        scores(x);
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[x][e] = tw * KEYS + j * 32 + 8 * (e >> 2) + 4 * half + (e & 3) < len ? s[x][e] : -INFINITY;
        float sum, mx;
        weights(x, sum, mx);
        settle(x, sum, mx);
        values(x);
      }
    }
  }
#pragma unroll
  for (int x = 0; x < 2; ++x)
    if (valid[x]) store_part<D>(p, chunk, row_g[x], half, acc[x], m[x], l[x] + __shfl_xor(l[x], 32));
}

template <int D, bool BF16>
hipError_t launch(const PrefixParams& p, const PrefixPlan& pl, hipStream_t s) {
  PrefixParams a = p;
  if constexpr (BF16) {
    if (pl.wide) {
      const dim3 grid(static_cast<uint32_t>(p.n_pre)), block(256);
      if (p.pre.page_table)
        hipLaunchKernelGGL((prefix_wide_kernel<D, true>), grid, block, 0, s, p);
      else
        hipLaunchKernelGGL((prefix_wide_kernel<D, false>), grid, block, 0, s, p);
      const hipError_t e = hipGetLastError();
      if (e != hipSuccess) return e;
      a.n_pre = 0;  // the own caches are left
    }
  }
  // Whether workgroups share rows of K and V: the prefix's, where it is in this launch, or the own ones.
  const dim3 grid(static_cast<uint32_t>(a.n_pre + pl.n_own)), block(256);
  if ((a.n_pre > 0 && pl.row_blocks > 1) || pl.own_blocks > 1)
    hipLaunchKernelGGL((prefix_stream_kernel<D, BF16, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((prefix_stream_kernel<D, BF16, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attn(const PrefixParams& p, const PrefixPlan& pl, int head_dim, bool bf16,
                              hipStream_t s) {
  if (head_dim == 128) return bf16 ? launch<128, true>(p, pl, s) : launch<128, false>(p, pl, s);
  return bf16 ? launch<64, true>(p, pl, s) : launch<64, false>(p, pl, s);
}

}  // namespace md
