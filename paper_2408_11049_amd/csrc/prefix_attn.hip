// prefix_attn.hip -- attention of a batch whose sequences share a long prefix: the prefix's
// K and V are read once for all query rows of its group, each sequence's own cache for
// its own rows, and the parts meet by log-sum-exp (md_merge_lse's kernels).
//
// A workgroup takes 128 query rows of one KV head (32 a wave) and a part of a range of keys:
// of the prefix, for rows of every sequence of the group, or of one sequence's own tokens, for
// its L * G rows.  K and V tiles of 64 keys (fp32: 32) go through LDS, two in turn, shared by
// the waves; S^T = K Q^T leaves a lane one query row, so the softmax needs no shuffles but one
// exchange between the halves of the wave when the running maximum moves, and P^T is in place
// as the second product's operand: O^T += V^T P^T, V read transposed from LDS.
#include "answers_kernels.h"

namespace md {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;

namespace {

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

template <int D, bool BF16>
struct Tile {
  static constexpr int ES = BF16 ? 2 : 4;
  static constexpr int ROW = D * ES;          // bytes of a row
  static constexpr int CH = ROW / 16;         // 16-byte chunks of a row
  static constexpr int KEYS = kPrefixTile(BF16);
  static constexpr int RPP = 256 / CH;        // rows that the workgroup loads at once
  static constexpr int NP = KEYS / RPP;
  static constexpr int BYTES = KEYS * ROW;
  // Rows sit unpadded, chunk c of row r in place c ^ turn(r): 16 rows at one c, as the waves
  // read K, then cover all banks.
  static __device__ __forceinline__ int at(int r, int c) {
    const int turn = ROW == 128 ? (r >> 1) & 7 : r & 15;
    return r * ROW + ((c ^ turn) << 4);
  }
};

template <int D, bool BF16>
__global__ void __launch_bounds__(256)
// Two workgroups a compute unit; 128 fp32 channels need more than 256 registers.
__attribute__((amdgpu_waves_per_eu(D == 128 && !BF16 ? 1 : 2)))
prefix_attn_kernel(const PrefixParams p) {
  using T = Tile<D, BF16>;
  constexpr int KB = T::KEYS / 32;    // blocks of 32 keys
  constexpr int ST = T::CH / 2;       // 16-byte operand chunks a lane holds of its row
  constexpr int CB = D / 32;          // blocks of 32 channels
  constexpr float kLazy = 8.f;        // log2 headroom before the running maximum must move
  __shared__ __attribute__((aligned(16))) unsigned char lds[2][2][T::BYTES];

  const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, half = lane >> 5;
  const int wave = uniform(tid >> 6);

  // What this workgroup does.  The row blocks that read one part of the prefix are numbered 8
  // apart, so they run on one XCD and find its K and V in that L2.
  const bool pre = static_cast<int>(blockIdx.x) < p.n_pre;
  int blk, hk, chunk, C, row_base, tok0, rows;
  if (pre) {
    const int t = static_cast<int>(blockIdx.x) >> 3;
    const int u = (t / p.row_blocks) * 8 + (static_cast<int>(blockIdx.x) & 7);
    C = p.c_pre;
    if (u >= p.P * p.Hkv * C) return;
    hk = u % p.Hkv;
    blk = (u / p.Hkv) % p.P;
    chunk = u / (p.Hkv * p.P);
    row_base = (t % p.row_blocks) * kPrefixRows;
    tok0 = blk * p.n * p.L;
    rows = p.group_rows;
  } else {
    const int y = static_cast<int>(blockIdx.x) - p.n_pre, B = p.P * p.n;
    C = p.c_own;
    hk = y % p.Hkv;
    blk = (y / p.Hkv) % B;
    chunk = y / (p.Hkv * B);
    row_base = 0;
    tok0 = blk * p.L;
    rows = p.L * p.G;
  }
  const KvView c = pre ? p.pre : p.own;
  const int raw_len = uniform(c.lens[blk]);
  const int len = min(max(raw_len, 0), c.max_len);
  const int n_tiles = (len + T::KEYS - 1) / T::KEYS;
  const int t0 = static_cast<int>(static_cast<int64_t>(n_tiles) * chunk / C);
  const int t1 = static_cast<int>(static_cast<int64_t>(n_tiles) * (chunk + 1) / C);
  if (p.err && chunk == 0 && row_base == 0 && hk == 0 && tid == 0) {
    const int bits = (raw_len > c.max_len ? MD_ERRW_LONG_LEN : 0) |
                     (raw_len < (pre ? 0 : p.L) ? MD_ERRW_SHORT_LEN : 0);
    if (bits) atomicOr(reinterpret_cast<unsigned int*>(p.err), static_cast<unsigned int>(bits));
  }

  // This lane's query row, and how many keys it sees.
  const int r0 = row_base + wave * 32, r = r0 + l32;
  const bool active = r0 < rows, valid = r < rows;
  const int tq = r / p.G;
  const int64_t row_g = static_cast<int64_t>(tok0 + tq) * p.Hq + hk * p.G + (r - tq * p.G);
  // A row past the end keeps the mask off: its results are not stored.
  const int lim = !valid ? INT32_MAX : (pre ? len : len - p.L + tq + 1);

  // Q as the second operand: chunk 2 st + half of the row, that is channels 8 (bf16) or 4 a
  // chunk; K's chunks are taken in the same order.
  u32x4 q[ST];
#pragma unroll
  for (int st = 0; st < ST; ++st)
    q[st] = valid ? *reinterpret_cast<const u32x4*>(static_cast<const unsigned char*>(p.q) +
                                                    row_g * T::ROW + (2 * st + half) * 16)
                  : u32x4{0, 0, 0, 0};

  // Staging: thread tid moves chunk tid % CH of rows tid / CH + n * RPP.
  const int st_row = tid / T::CH, st_chunk = tid % T::CH;
  const int pmask = (1 << c.page_shift) - 1;
  const bool paged = c.page_table != nullptr;
  const int32_t* table = paged ? c.page_table + static_cast<int64_t>(blk) * c.max_pages : nullptr;
  const int64_t head_off = static_cast<int64_t>(hk) * c.s_head;
  int pid[T::NP];
  u32x4 kr[T::NP], vr[T::NP];
  uint32_t ok = 0;  // bit n: row n of this thread is a token

  auto load_pids = [&](int t) {
    if (!paged) return;
#pragma unroll
    for (int n = 0; n < T::NP; ++n) {
      const int tok = t * T::KEYS + n * T::RPP + st_row;
      pid[n] = t < t1 && tok < len ? table[tok >> c.page_shift] : 0;
    }
  };
  // A token that must not be read (past the end, on a page outside the pool) is redirected to
  // the first row, and its K and V are staged as zeros.
  auto load_tile = [&](int t) {
    if (t >= t1) return;
    ok = 0;
#pragma unroll
    for (int n = 0; n < T::NP; ++n) {
      const int tok = t * T::KEYS + n * T::RPP + st_row;
      bool good = tok < len;
      int64_t off;
      if (paged) {
        const bool in_pool = pid[n] >= 0 && pid[n] < c.num_pages;
        if (p.err && good && !in_pool)
          atomicOr(reinterpret_cast<unsigned int*>(p.err), static_cast<unsigned int>(MD_ERRW_BAD_PAGE));
        good = good && in_pool;
        off = static_cast<int64_t>(pid[n]) * c.s_blk + static_cast<int64_t>(tok & pmask) * c.s_tok;
      } else {
        off = static_cast<int64_t>(blk) * c.s_blk + static_cast<int64_t>(tok) * c.s_tok;
      }
      off = good ? (off + head_off) * T::ES + st_chunk * 16 : 0;
      kr[n] = *reinterpret_cast<const u32x4*>(c.k + off);
      vr[n] = *reinterpret_cast<const u32x4*>(c.v + off);
      ok |= static_cast<uint32_t>(good) << n;
    }
  };
  auto stage = [&](int t) {
    if (t >= t1) return;
    unsigned char* const kt = lds[t & 1][0];
    unsigned char* const vt = lds[t & 1][1];
#pragma unroll
    for (int n = 0; n < T::NP; ++n) {
      const bool good = (ok >> n) & 1u;
      const int a = T::at(n * T::RPP + st_row, st_chunk);
      *reinterpret_cast<u32x4*>(kt + a) = good ? kr[n] : u32x4{0, 0, 0, 0};
      *reinterpret_cast<u32x4*>(vt + a) = good ? vr[n] : u32x4{0, 0, 0, 0};
    }
  };

  float m_run = -INFINITY, l_run = 0.f;
  f32x16 acc[CB];
#pragma unroll
  for (int cb = 0; cb < CB; ++cb) acc[cb] = f32x16{};

  auto compute = [&](int t) {
    const unsigned char* const kt = lds[t & 1][0];
    const unsigned char* const vt = lds[t & 1][1];
    // S^T: a lane gets keys 32 kb + 8 (e / 4) + 4 half + e % 4 of its row.
    f32x16 s[KB];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      s[kb] = f32x16{};
#pragma unroll
      for (int st = 0; st < ST; ++st) {
        const u32x4 kk = *reinterpret_cast<const u32x4*>(kt + T::at(kb * 32 + l32, 2 * st + half));
        if constexpr (BF16) {
          s[kb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kk),
                                                          __builtin_bit_cast(bf16x8, q[st]), s[kb], 0, 0, 0);
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            s[kb] = __builtin_amdgcn_mfma_f32_32x32x2f32(__uint_as_float(kk[j]),
                                                         __uint_as_float(q[st][j]), s[kb], 0, 0, 0);
        }
      }
    }
    const int key0 = t * T::KEYS;
    if (__any(lim < key0 + T::KEYS)) {
#pragma unroll
      for (int kb = 0; kb < KB; ++kb)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          s[kb][e] = key0 + kb * 32 + 8 * (e >> 2) + 4 * half + (e & 3) < lim ? s[kb][e] : -INFINITY;
    }
    float mx = s[0][0];
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) mx = fmaxf(mx, s[kb][e]);
    mx *= p.scale_log2;
    // The running maximum moves only when some row's exceeds it by 2^kLazy: weights stay below
    // that, and most tiles skip the rescale.
    if (__any(mx > m_run + kLazy)) {
      mx = fmaxf(mx, __shfl_xor(mx, 32));
      const float m_new = fmaxf(m_run, mx);
      const float f = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_run *= f;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) acc[cb] *= f;
    }
    const float m_use = m_run == -INFINITY ? 0.f : m_run;
    float sum = 0.f;
#pragma unroll
    for (int kb = 0; kb < KB; ++kb)
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        s[kb][e] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[kb][e], p.scale_log2, -m_use));
        sum += s[kb][e];
      }
    l_run += sum;
    // O^T: operands of 16 keys; slots of this half are keys 16 x + 4 half + {0..3, 8..11}.
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
      if constexpr (BF16) {
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          // Weights to bf16, half a step each: the matrix units take bf16, and O is rounded to
          // it in the end.
          const u32x4 pb = {pack2(s[kb][8 * x], s[kb][8 * x + 1]), pack2(s[kb][8 * x + 2], s[kb][8 * x + 3]),
                            pack2(s[kb][8 * x + 4], s[kb][8 * x + 5]), pack2(s[kb][8 * x + 6], s[kb][8 * x + 7])};
          // Transposed reads: lane k of 16 supplies row k / 4 and four channels of it, and gets one
          // channel of the four rows.
          const int l16 = lane & 15, key = kb * 32 + 16 * x + 4 * half + (l16 >> 2);
          const int ch = ((lane >> 4) & 1) * 2 + ((l16 & 3) >> 1), sub = (l16 & 1) * 8;
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_i16x4*)(vt + T::at(key, cb * 4 + ch) + sub));
            const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                (lds_i16x4*)(vt + T::at(key + 8, cb * 4 + ch) + sub));
            const bf16x8 va = __builtin_bit_cast(
                bf16x8, u32x4{__builtin_bit_cast(u32x2, lo).x, __builtin_bit_cast(u32x2, lo).y,
                              __builtin_bit_cast(u32x2, hi).x, __builtin_bit_cast(u32x2, hi).y});
            acc[cb] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va, __builtin_bit_cast(bf16x8, pb),
                                                              acc[cb], 0, 0, 0);
          }
        }
      } else {
#pragma unroll
        for (int e = 0; e < 16; ++e) {
          const int key = kb * 32 + 8 * (e >> 2) + 4 * half + (e & 3);
#pragma unroll
          for (int cb = 0; cb < CB; ++cb) {
            const int channel = cb * 32 + l32;
            const float va = *reinterpret_cast<const float*>(vt + T::at(key, channel >> 2) + (channel & 3) * 4);
            acc[cb] = __builtin_amdgcn_mfma_f32_32x32x2f32(va, s[kb][e], acc[cb], 0, 0, 0);
          }
        }
      }
    }
  };

  // Tile t is computed from one buffer while t + 1 is written to the other and t + 2 is on its
  // way in registers.  The barrier at the end of a turn makes t + 1 visible and t's buffer free.
  load_pids(t0);
  load_tile(t0);
  load_pids(t0 + 1);
  stage(t0);
  load_tile(t0 + 1);
  load_pids(t0 + 2);
  __syncthreads();
  for (int t = t0; t < t1; ++t) {
    stage(t + 1);
    load_tile(t + 2);
    load_pids(t + 3);
    if (active) compute(t);
    __syncthreads();
  }

  if (!valid) return;
  // ---- this part's normalised O and lse
  const float l = l_run + __shfl_xor(l_run, 32);
  const float inv = l > 0.f ? 1.f / l : (l == l ? 0.f : l);
  const int64_t prow = static_cast<int64_t>(pre ? chunk : p.c_pre + chunk) * p.n_rows + row_g;
  float* const out = p.part_o + prow * D + 4 * half;
#pragma unroll
  for (int cb = 0; cb < CB; ++cb)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const f32x4 x = {acc[cb][4 * j], acc[cb][4 * j + 1], acc[cb][4 * j + 2], acc[cb][4 * j + 3]};
      *reinterpret_cast<f32x4*>(out + cb * 32 + 8 * j) = x * inv;
    }
  // A NaN stays NaN: -inf would tell the merge that the part is empty.
  if (half == 0)
    p.part_lse[prow] = l > 0.f ? (m_run + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f
                               : (l == l ? -INFINITY : l);
}

template <int D, bool BF16>
hipError_t launch(const PrefixParams& p, int64_t n_wgs, hipStream_t s) {
  hipLaunchKernelGGL((prefix_attn_kernel<D, BF16>), dim3(static_cast<uint32_t>(n_wgs)), dim3(256), 0,
                     s, p);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attn(const PrefixParams& p, int64_t n_wgs, int head_dim, bool bf16,
                              hipStream_t s) {
  if (head_dim == 128) return bf16 ? launch<128, true>(p, n_wgs, s) : launch<128, false>(p, n_wgs, s);
  return bf16 ? launch<64, true>(p, n_wgs, s) : launch<64, false>(p, n_wgs, s);
}

}  // namespace md
