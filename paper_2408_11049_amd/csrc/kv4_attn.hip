// kv4_attn.hip -- decode attention over a 4-bit KV cache (MXFP4; format in kv4.h).
//
//   s = scale q.K_j,  o = sum_j exp(s_j - lse) V_j
//
// A unit is a (sequence, KV head): its G * L query rows share one pass over its K and
// V (fp32 queries: 32 of them do, more take a second pass, for want of registers).  136
// bytes a token and head (d = 128) instead of bf16's 512 leave a compute unit some 380 cycles
// per 32 tokens at the HBM rate, so the work per element decides the layout:
//   K   never passes through LDS.  A lane loads 32 consecutive channels of a token --
//       one 16-byte load, one scale -- and v_cvt_scalef32_pk_bf16_fp4 turns them
//       into four MFMA A operands; the contraction's order is free, so Q is held in
//       the same channel order.  The scale costs nothing: the conversion applies it,
//       exactly.
//   V   is converted the same way, then staged in LDS as bf16 rows and read back
//       transposed (ds_read_b64_tr_b16), since O^T += V^T P^T contracts over tokens.
//   Q   waits in LDS: its registers are worth more as a third workgroup a compute unit.
//   S^T, the softmax state and O^T keep each lane on one query row, as in
//   attn_kernel.h: no lane moves between the two products.
// fp32 queries: K and V are exact in bf16, so Q and P split into three bf16 parts
// (24 bits) give fp32 products on the bf16 matrix instructions.
//
// Work split: the 32-token tiles of all units form one stream cut into equal ranges,
// one a workgroup, so neither ragged lengths nor few sequences leave units idle; a
// unit that a cut crosses is computed in pieces, which a second launch joins.  Where a
// workgroup for each unit is put at less than that, the plan takes that (plan_ops.cpp).
//
// Measured (bf16, d = 128, 32 query heads on 8): a call over 64 sequences of 16384 .. 32768
// tokens, 5 query tokens, 16-token pages 323 to 361 us by the card, 8 of them the joins: 1.78 GB at
// 4.9 to 5.5 TB/s (its loads alone: 280 to 306 us).  That is in a loop, once the clock has settled:
// calls 5 to 20 after an idle second take up to 426.  32 of 8192, one query token 48 us and 4.6 for
// the joins: 6.0 TB/s.
#include "kv4.h"

namespace md {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
typedef const __attribute__((address_space(1))) unsigned char global_bytes;

namespace {

constexpr int T = kKv4Tile;
constexpr int W = kWaves;

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{lo, hi}, bf16x2));
}
__device__ __forceinline__ float lo_f32(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float hi_f32(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

// 8 codes -> 8 bf16 values.
__device__ __forceinline__ u32x4 values8(uint32_t codes, float scale) {
  return u32x4{
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3))};
}
template <int N>
__device__ __forceinline__ void load_words(global_bytes* at, uint32_t (&w)[N]) {
  typedef uint32_t vec __attribute__((ext_vector_type(N)));
  const vec x =
      __builtin_nontemporal_load((const __attribute__((address_space(1))) vec*)(at));
#pragma unroll
  for (int i = 0; i < N; ++i) w[i] = x[i];
}
// base + off, the same for the whole wave (but for small pages): kept in scalar registers, so
// that a lane's own offset needs no 64-bit addition.  The empty asm hides the sum from the
// compiler, which would otherwise add the lane's offset to the base outside the loop.
template <int PG>
__device__ __forceinline__ global_bytes* block_ptr(const unsigned char* base, int64_t off) {
  uintptr_t at = reinterpret_cast<uintptr_t>(base) + static_cast<uintptr_t>(off);
  if constexpr (PG != 2) asm("" : "+s"(at));
  return reinterpret_cast<global_bytes*>(at);
}
// The scale's power of two; byte 255 becomes infinity's pattern with a mantissa bit: NaN.
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float((byte << 23) | (byte == 255u ? 0x400000u : 0u));
}

// The bits below bit n: none for n <= 0, all from 32 on.
__device__ __forceinline__ uint32_t below(int n) {
  return n <= 0 ? 0u : (n >= 32 ? 0xffffffffu : (1u << n) - 1u);
}

// ---- the tiles of a sequence ----
// Tiles are cut at multiples of T of the token position, so a tile's blocks of 16
// lie in one page of 16 tokens or more.  Tile v of a unit is real tile v below
// `head` (sinks), v - head + tail0 from there on (the windows).
struct Tiles {
  int S;      // clamped length
  int n;      // tiles that hold a visible token
  int head, tail0;
};
__device__ __forceinline__ int length(const Kv4AttnParams& p, int b) {
  return max(min(p.kv_lens[b], p.max_kv_len), 0);
}
__device__ __forceinline__ Tiles tiles_of(const Kv4AttnParams& p, int S) {
  Tiles t;
  t.S = S;
  const int end = (t.S + T - 1) / T;
  t.head = end;
  t.tail0 = end;
  t.n = end;
  if (p.mode == MD_MODE_DRAFT) {
    const int lo = t.S - p.L - p.window + 1;  // first position of any window
    const int sinks = p.n_sink / T + (p.n_sink % T != 0);
    if (lo > 0 && lo / T > sinks) {
      t.head = sinks;
      t.tail0 = lo / T;
      t.n = sinks + end - t.tail0;
    }
  }
  return t;
}

// Neighbouring units share memory lines: two passes the whole of K and V, heads of a 16-token
// page the lines of its scales (64 bytes a head, d = 128), heads of a token-major cache those of
// its codes too.  So `share` consecutive units form a group, and its units' workgroups run side
// by side on one XCD, whose L2 then reads each line once.  Workgroups go to the eight XCDs in
// turn: workgroup w has member w / 8 % share of range (or group) place(w).  32 x 8 units of 16384
// tokens, alone and in groups: token-major 203 us and 177, fp32 206 and 168; 16-token pages of the
// head-major layout 103 and 101; two fp32 passes 366 and 354.  (Groups of eight: 180 and 175.)
__device__ __forceinline__ int member(const Kv4AttnParams& p, int w) { return w / 8 % p.share; }
__device__ __forceinline__ int place(const Kv4AttnParams& p, int w) {
  return w / (8 * p.share) * 8 + w % 8;
}

// Balanced plan: groups in order (sequence, group), max(1, tiles) stream tiles each; range w
// of NW is [w TT / NW, (w + 1) TT / NW).
struct Cursor {
  int t, hi;       // next stream tile, end of the range
  int b, j;        // the current group: group j of sequence b
  int g0, gt;      // its first stream tile and its number of tiles
  int TT, NW;
};

// Inclusive tile counts of the sequences in sl[0..B), their lengths in sl[kKv4BalMaxSeqs ..);
// the total.  256 threads.
__device__ int scan_tiles(const Kv4AttnParams& p, int* sl) {
  constexpr int kPer = kKv4BalMaxSeqs / 256;
  __shared__ int wave_sum[W];
  const int tid = threadIdx.x, lane = tid & 63;
  int v[kPer], mine = 0;
  for (int e = 0; e < kPer; ++e) {
    const int b = tid * kPer + e;
    v[e] = 0;
    if (b < p.B) {
      const int S = length(p, b);
      sl[kKv4BalMaxSeqs + b] = S;
      v[e] = max(tiles_of(p, S).n, 1) * p.groups;
    }
    mine += v[e];
  }
  int incl = mine;
  for (int o = 1; o < 64; o <<= 1) {
    const int x = __shfl_up(incl, o);
    if (lane >= o) incl += x;
  }
  if (lane == 63) wave_sum[tid >> 6] = incl;
  __syncthreads();
  int run = incl - mine;
  for (int w = 0; w < (tid >> 6); ++w) run += wave_sum[w];
  for (int e = 0; e < kPer; ++e) {
    run += v[e];
    if (tid * kPer + e < p.B) sl[tid * kPer + e] = run;
  }
  __syncthreads();
  return uniform(sl[p.B - 1]);
}

// The group that holds stream tile t.  sl as scan_tiles leaves it.
__device__ void group_at(const Kv4AttnParams& p, const int* sl, int t, Cursor& c) {
  int lo = 0, hi = p.B - 1;  // the first sequence whose inclusive count passes t
  while (lo < hi) {
    const int mid = (lo + hi) / 2;
    if (sl[mid] > t) hi = mid;
    else lo = mid + 1;
  }
  c.b = uniform(lo);
  const int ex = c.b ? uniform(sl[c.b - 1]) : 0;
  c.gt = (uniform(sl[c.b]) - ex) / p.groups;
  c.j = (t - ex) / c.gt;
  c.g0 = ex + c.j * c.gt;
}

// Ranges of a stream of TT tiles: at least a tile for each wave where there are as many.
__device__ __forceinline__ int ranges(int grid, int TT) { return min(grid, max(1, TT / W)); }
__device__ __forceinline__ int range_start(const Cursor& c, int w) {
  return static_cast<int>(static_cast<int64_t>(w) * c.TT / c.NW);
}
__device__ __forceinline__ int range_of(const Cursor& c, int t) {
  return static_cast<int>((static_cast<int64_t>(t + 1) * c.NW - 1) / c.TT);
}

// Row r of a unit: query token i = r / G, query head hk * G + r % G.
__device__ __forceinline__ int64_t out_row(const Kv4AttnParams& p, int b, int hk, int r) {
  return (static_cast<int64_t>(b) * p.L + r / p.G) * p.Hq + hk * p.G + r % p.G;
}

template <bool BF16>
__device__ __forceinline__ void store4(const Kv4AttnParams& p, int64_t e, f32x4 x) {
  if constexpr (BF16)
    *reinterpret_cast<u32x2*>(static_cast<uint16_t*>(p.o) + e) =
        u32x2{pack2(x[0], x[1]), pack2(x[2], x[3])};
  else
    *reinterpret_cast<f32x4*>(static_cast<float*>(p.o) + e) = x;
}

// O and lse of a row from its unnormalised O, running max (log2) and sum.  A sum of 0: no
// visible key.  A NaN sum (a NaN score) makes the row NaN.
__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }
__device__ __forceinline__ float lse_of(float m, float l) {
  return l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f;
}

// PG: 0 contiguous, 1 pages of at least 16 tokens, 2 smaller pages.
template <int D, bool BF16, int NT, int PG>
__global__ void __launch_bounds__(W * 64) __attribute__((amdgpu_waves_per_eu(kKv4Resident(BF16, NT, D))))
kv4_attn_kernel(const Kv4AttnParams p) {
  constexpr int LB = D / 8;         // code bytes a lane loads of a token: D / 4 channels
  constexpr int LW = LB / 4;        // their dwords: MFMA steps over the channels
  constexpr int CB = D / 16;        // 16-channel blocks of O
  constexpr int PARTS = BF16 ? 1 : 3;
  constexpr int ROWS = NT * 16;
  constexpr int kAhead = 4;         // channel blocks of V read ahead of their use
  constexpr int VROW = D * 2 + 16;  // bytes of a staged V row
  constexpr int QROW = D * 2 + 16;  // bytes of a staged row of Q (of one part)
  constexpr int MROW = D + 4;       // floats of a row in the waves' merge
  // LDS: the scan of the lengths; then Q, the waves' V tiles, and over those their O of one
  // row tile at a time.
  constexpr int kQ = PARTS * ROWS * QROW;
  constexpr int kV = W * T * VROW;
  constexpr int kMergeO = W * 16 * MROW * 4;
  constexpr int kMl = 2 * W * ROWS * 4;
  constexpr int kWork = kV > kMergeO ? kV : kMergeO;
  constexpr int kScan = 2 * kKv4BalMaxSeqs * 4;
  constexpr int kLds = kQ + kMl + kWork > kScan ? kQ + kMl + kWork : kScan;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kLds];

  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
  const int wave = uniform(tid >> 6);

  const int range = place(p, static_cast<int>(blockIdx.x));
  const int mem = member(p, static_cast<int>(blockIdx.x));
  Cursor c{};
  int S_next;  // length of the next piece's sequence
  if (p.balanced) {
    int* sl = reinterpret_cast<int*>(lds);
    c.TT = scan_tiles(p, sl);
    c.NW = ranges(static_cast<int>(gridDim.x) / p.share, c.TT);
    Join join{-1, 0, 0, 0};
    if (range < c.NW) {
      c.t = range_start(c, range);
      c.hi = range_start(c, range + 1);
      group_at(p, sl, c.t, c);
      // The boundary where this range begins cuts a unit, as its first?  Then join it later.
      if (c.t != c.g0 && range_start(c, range - 1) <= c.g0)
        join = Join{c.b, c.j, range_of(c, c.g0 + c.gt - 1),
                    2 * ((range - 1) * p.share + mem) + (range_start(c, range - 1) != c.g0)};
    }
    if (tid == 0) p.joins[blockIdx.x] = join;
    if (range >= c.NW) return;  // the whole workgroup
    S_next = sl[kKv4BalMaxSeqs + c.b];
    __syncthreads();        // the LDS is reused
  } else {
    if (range >= p.B * p.groups) return;  // the whole workgroup
    c.b = range / p.groups;
    c.j = range % p.groups;
    S_next = length(p, c.b);
  }

  for (;;) {  // one pass a piece
    const int b = c.b, unit = c.j * p.share + mem, hk = unit / p.passes;
    const int r0 = unit % p.passes * ROWS;  // its rows of the head's R: r0 .. r0 + rows - 1
    const int rows = min(p.R - r0, ROWS);
    const Tiles u = tiles_of(p, uniform(S_next));
    if (!p.balanced) c = Cursor{0, max(u.n, 1), b, c.j, 0, max(u.n, 1), max(u.n, 1), 1};
    const int S = u.S;
    const int lt0 = c.t - c.g0;
    const int lt1 = min(c.hi, c.g0 + c.gt) - c.g0;
    const bool whole = lt0 == 0 && lt1 == c.gt;
    const int n_tiles = min(lt1, u.n) - lt0;  // <= 0: nothing visible

    int row_pos[NT];  // position of this lane's query rows; padding rows see nothing
#pragma unroll
    for (int rt = 0; rt < NT; ++rt) {
      const int r = rt * 16 + l16;
      row_pos[rt] = r < rows ? S - p.L + (r0 + r) / p.G : -1;
    }
    // ---- loads ----
    struct TileRegs {
      uint32_t k[2][LW], v[2][LW];
      uint32_t ks[2], vs[2];
    };
    const int pmask = (1 << p.c.page_shift) - 1;
    const int32_t* ptab = PG ? p.c.page_table + static_cast<int64_t>(b) * p.c.max_pages : nullptr;
    // Byte offset of the head's rows (contiguous: of the sequence's), added to every block's.
    const int64_t unit_off = static_cast<int64_t>(hk) * p.c.s_head +
                             (PG ? 0 : static_cast<int64_t>(b) * p.c.s_blk);
    const uint32_t s_tok = static_cast<uint32_t>(p.c.s_tok);
    // This lane's scale byte in its row.  d = 128: the row's four are one dword, loaded whole, and
    // the byte is taken out of it where it is used.  (A loaded byte is widened to a register behind
    // the softmax already, which waits for the loads in flight; d = 64 does.)
    constexpr bool kWholeRow = D == 128;
    const uint32_t sidx = grp * (D / 4) / 32;
    const uint32_t sfirst = kWholeRow ? 0 : sidx;
    auto scale_byte = [&](uint32_t loaded) {
      return kWholeRow ? (loaded >> (8 * sidx)) & 255u : loaded;
    };
    auto load_scale = [](global_bytes* at) -> uint32_t {
      if constexpr (kWholeRow) return *(const __attribute__((address_space(1))) uint32_t*)(at);
      return *at;
    };
    auto real_tile = [&](int v) { return v < u.head ? v : v - u.head + u.tail0; };
    // First token of block tb of piece tile v, in a block that holds a real token.
    auto block_at = [&](int v, int tb) {
      return min(real_tile(lt0 + min(v, n_tiles - 1)) * T + tb * 16, (S - 1) & ~15);
    };
    // An id outside the pool reads the pool's first page: in bounds, results unspecified.
    auto page_ok = [&](int id) { return id >= 0 && id < p.c.num_pages ? id : 0; };

    // Page ids (pages of 16 tokens or more): lane j holds that of block j % 2 of this wave's
    // tile batch + j / 2, so one load serves 32 tiles; the next batch's is in flight.
    int ids = 0, ids_next = 0;
    auto load_ids = [&](int batch) {
      if constexpr (PG == 1) {
        const int bt = block_at(wave + (batch + lane / 2) * W, lane % 2);
        return page_ok(ptab[bt >> p.c.page_shift]);
      }
      return 0;
    };

    // Tile k of this wave (piece tile wave + k W).  A block's 16 rows are read whole, those past
    // the sequence too where they are in the cache (masked below): the lanes' offsets are then
    // the same for every block.  Tiles past the piece are its last one, never used.
    const uint32_t code_off = static_cast<uint32_t>(l16) * s_tok + grp * LB;
    const uint32_t scale_off = static_cast<uint32_t>(l16) * (s_tok >> 4) + sfirst;
    auto load_tile = [&](TileRegs& r, int k) {
      const int v = wave + k * W;
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        const int bt = block_at(v, tb);
        int64_t base;
        uint32_t code = code_off, scale = scale_off;
        if constexpr (PG == 0) {
          base = unit_off + static_cast<int64_t>(static_cast<uint64_t>(bt) * s_tok);
          if (bt + 16 > p.c.capacity) {  // the cache ends inside the block
            const uint32_t dt = static_cast<uint32_t>(min(l16, S - 1 - bt));
            code = dt * s_tok + grp * LB;
            scale = dt * (s_tok >> 4) + sfirst;
          }
        } else if constexpr (PG == 1) {
          const int id = __builtin_amdgcn_readlane(ids, (k & 31) * 2 + tb);
          base = unit_off + static_cast<int64_t>(id) * p.c.s_blk +
                 static_cast<int64_t>(static_cast<uint64_t>(bt & pmask) * s_tok);
        } else {
          const int t = min(bt + l16, S - 1);
          base = unit_off + static_cast<int64_t>(page_ok(ptab[t >> p.c.page_shift])) * p.c.s_blk +
                 static_cast<int64_t>(static_cast<uint64_t>(t & pmask) * s_tok);
          code = grp * LB;
          scale = sfirst;
        }
        asm("" : "+v"(code), "+v"(scale));  // 32 bits up to the load: see block_ptr
        load_words(block_ptr<PG>(p.c.k, base) + code, r.k[tb]);
        load_words(block_ptr<PG>(p.c.v, base) + code, r.v[tb]);
        r.ks[tb] = load_scale(block_ptr<PG>(p.c.ks, base >> 4) + scale);
        r.vs[tb] = load_scale(block_ptr<PG>(p.c.vs, base >> 4) + scale);
      }
    };

    // The first tiles' loads, before anything waits.
    const int mine = n_tiles > wave ? (n_tiles - wave + W - 1) / W : 0;  // tiles of this wave
    TileRegs tile;
    if (mine > 0) {
      ids = load_ids(0);
      ids_next = load_ids(32);
      load_tile(tile, 0);
    }
    __builtin_amdgcn_sched_barrier(0);

    // Q into LDS (its registers are worth more: a third wave per SIMD), fp32 as three bf16 parts:
    // the leading 8 bits, then those of what is left.
    unsigned char* q_lds = lds;
    for (int item = tid; item < ROWS * (D / 8); item += W * 64) {
      const int r = item / (D / 8), c0 = item % (D / 8) * 8;
      const int64_t e = r < rows ? out_row(p, b, hk, r0 + r) * D + c0 : 0;
      if constexpr (BF16) {
        u32x4 x = {0, 0, 0, 0};
        if (r < rows) x = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(p.q) + e);
        *reinterpret_cast<u32x4*>(q_lds + r * QROW + c0 * 2) = x;
      } else {
        f32x4 x[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        if (r < rows) {
          const f32x4* src = reinterpret_cast<const f32x4*>(static_cast<const float*>(p.q) + e);
          x[0] = src[0];
          x[1] = src[1];
        }
#pragma unroll
        for (int k = 0; k < PARTS; ++k) {
          u32x4 w;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            w[2 * h] = pack2(x[h][0], x[h][1]);
            w[2 * h + 1] = pack2(x[h][2], x[h][3]);
            x[h] = f32x4{x[h][0] - lo_f32(w[2 * h]), x[h][1] - hi_f32(w[2 * h]),
                         x[h][2] - lo_f32(w[2 * h + 1]), x[h][3] - hi_f32(w[2 * h + 1])};
          }
          *reinterpret_cast<u32x4*>(q_lds + (k * ROWS + r) * QROW + c0 * 2) = w;
        }
      }
    }
    __syncthreads();

    float m_run[NT], l_run[NT];  // log2; 0 and a threshold of -inf: no key seen yet
    float lazy[NT];
    f32x4 acc[NT][CB];
    uint32_t nan_v[NT];  // bit i: the row sees a token whose V is NaN in channels 32 i ..
#pragma unroll
    for (int rt = 0; rt < NT; ++rt) {
      m_run[rt] = 0.f;
      lazy[rt] = -INFINITY;
      l_run[rt] = 0.f;
      nan_v[rt] = 0;
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) acc[rt][cb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    unsigned char* vt = lds + kQ + kMl + wave * (T * VROW);
    const unsigned char* q_lane = q_lds + l16 * QROW + grp * (D / 2);
    constexpr float kLazy = 8.f;

    auto visible = [&](int t, int pos) {
      return t <= pos && (p.mode != MD_MODE_DRAFT || t < p.n_sink || t > pos - p.window);
    };

    // One tile.  masked (uniform): some query row does not see all of it.  `refill` issues
    // the loads that reuse the tile's registers, once they are free.
    auto process = [&](bool masked, TileRegs& r, int t0, auto refill) {
      // V into LDS as bf16 rows.  In a masked tile a row past the sequence, or one that is NaN
      // in this lane's block, is staged as zeros: 0 * NaN must not reach a query that does
      // not see it; those that see it are noted and get their NaN at the end.
      const uint32_t vbyte[2] = {scale_byte(r.vs[0]), scale_byte(r.vs[1])};
      float vscale[2] = {scale_of(vbyte[0]), scale_of(vbyte[1])};
      if (masked) {
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) {
          const bool past = t0 + tb * 16 + l16 >= S;
          const bool bad = vbyte[tb] == 255u;
          for (unsigned long long left = __ballot(bad && !past); left; left &= left - 1) {
            const int at = __ffsll(static_cast<long long>(left)) - 1;
#pragma unroll
            for (int rt = 0; rt < NT; ++rt)
              if (visible(t0 + tb * 16 + (at & 15), row_pos[rt]))
                nan_v[rt] |= 1u << ((at >> 4) * (D / 4) / 32);
          }
          if (past || bad) {
            vscale[tb] = 1.f;
#pragma unroll
            for (int w = 0; w < LW; ++w) r.v[tb][w] = 0u;
          }
        }
      }
#pragma unroll
      for (int tb = 0; tb < 2; ++tb) {
        unsigned char* dst = vt + (tb * 16 + l16) * VROW + grp * (D / 2);
#pragma unroll
        for (int w = 0; w < LW; ++w)
          *reinterpret_cast<u32x4*>(dst + w * 16) = values8(r.v[tb][w], vscale[tb]);
      }

      __builtin_amdgcn_sched_barrier(0);
      // S^T = K Q^T.
      f32x4 s[NT][2];
#pragma unroll
      for (int rt = 0; rt < NT; ++rt)
#pragma unroll
        for (int tb = 0; tb < 2; ++tb) s[rt][tb] = f32x4{0.f, 0.f, 0.f, 0.f};
      const float ks[2] = {scale_of(scale_byte(r.ks[0])), scale_of(scale_byte(r.ks[1]))};
#pragma unroll
      for (int w = 0; w < LW; ++w) {
        bf16x8 kk[2];
#pragma unroll
        for (int tb = 0; tb < 2; ++tb)
          kk[tb] = __builtin_bit_cast(bf16x8, values8(r.k[tb][w], ks[tb]));
#pragma unroll
        for (int k = PARTS - 1; k >= 0; --k)
#pragma unroll
          for (int rt = 0; rt < NT; ++rt) {
            const bf16x8 qq = *reinterpret_cast<const bf16x8*>(
                q_lane + (k * ROWS + rt * 16) * QROW + w * 16);
#pragma unroll
            for (int tb = 0; tb < 2; ++tb)
              s[rt][tb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[tb], qq, s[rt][tb], 0, 0, 0);
          }
      }

      __builtin_amdgcn_sched_barrier(0);
      refill();
      // V^T for the first channel blocks, under way during the softmax.  Transposed reads:
      // lane k of a 16-lane group supplies row 4 grp + k / 4 and channels cb*16 + 4 (k % 4)
      // .. + 3, and lane i gets channel cb*16 + i of those rows.
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
      auto read_v = [&](int cb) {
        const unsigned char* src =
            vt + (4 * grp + (l16 >> 2)) * VROW + (cb * 16 + 4 * (l16 & 3)) * 2;
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_i16x4*)(src + 16 * VROW));
        const u32x2 a = __builtin_bit_cast(u32x2, lo), d = __builtin_bit_cast(u32x2, hi);
        return __builtin_bit_cast(bf16x8, u32x4{a[0], a[1], d[0], d[1]});
      };
      bf16x8 va[kAhead];
#pragma unroll
      for (int cb = 0; cb < kAhead; ++cb) va[cb] = read_v(cb);
      __builtin_amdgcn_sched_barrier(0);

      // bf16 queries: a weight is rounded to bf16 before it multiplies V, its sum is not.  O is then
      // 2.1e-3 to 2.3e-3 off (root mean square, of which its own rounding to bf16 is 1.66e-3) and
      // lse 4e-8 of itself.  Weights in two bf16 parts give 1.66e-3, but take 409 us where this takes 357 to
      // 361 (64 x 16384 .. 32768 tokens, two row tiles, one card; one row tile 57.4 and 55.7); a sum
      // of the rounded weights gives O 2.11e-3 for 2.25e-3, but lse 2.7e-5.
      // Softmax weights 2^y, y = c s - m, c = scale * log2 e: lane's row l16, tokens tb*16 + 4
      // grp + e.  A row's m moves only when some y passes kLazy (at first: whenever a key is
      // visible), so most tiles need no exchange between the four lanes of a row; until
      // then a weight is at most 2^kLazy.
      if (masked) {
        const int first = t0 + 4 * grp;
#pragma unroll
        for (int rt = 0; rt < NT; ++rt) {
          // visible() of this lane's tokens as bits, relative to its first.
          // (Padding rows see none: their `last` is below 0.)
          const int last = row_pos[rt] - first;
          uint32_t seen = below(last + 1);
          if (p.mode == MD_MODE_DRAFT)
            seen &= ~below(static_cast<int>(static_cast<uint32_t>(last) - p.window + 1u)) |
                    below(p.n_sink - first);
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (!((seen >> (j / 4 * 16 + j % 4)) & 1u)) s[rt][j / 4][j % 4] = -INFINITY;
        }
      }
      u32x4 pb[NT][PARTS];
#pragma unroll
      for (int rt = 0; rt < NT; ++rt) {
        float x[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = fmaf(s[rt][j / 4][j % 4], p.scale_log2, -m_run[rt]);
        float mx = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                         fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
        if (__any(mx > lazy[rt])) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          if (mx > lazy[rt]) {  // the same for the four lanes of a row
            const float alpha = lazy[rt] == kLazy ? exp2_fast(-mx) : 1.f;
            m_run[rt] += mx;
            lazy[rt] = kLazy;
            l_run[rt] *= alpha;
#pragma unroll
            for (int cb = 0; cb < CB; ++cb) acc[rt][cb] *= alpha;
          }
#pragma unroll
          for (int j = 0; j < 8; ++j) x[j] = fmaf(s[rt][j / 4][j % 4], p.scale_log2, -m_run[rt]);
        }
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          x[j] = exp2_fast(x[j]);
          sum += x[j];
        }
        l_run[rt] += sum;  // of the unrounded weights: lse keeps fp32
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t h = pack2(x[2 * j], x[2 * j + 1]);
            pb[rt][k][j] = h;
            if constexpr (!BF16) {
              x[2 * j] -= lo_f32(h);
              x[2 * j + 1] -= hi_f32(h);
            }
          }
      }

      // O^T += V^T P^T.
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const bf16x8 v_now = va[cb % kAhead];
        if (cb + kAhead < CB) va[cb % kAhead] = read_v(cb + kAhead);
#pragma unroll
        for (int rt = 0; rt < NT; ++rt)
#pragma unroll
          for (int k = PARTS - 1; k >= 0; --k)
            acc[rt][cb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                v_now, __builtin_bit_cast(bf16x8, pb[rt][k]), acc[rt][cb], 0, 0, 0);
      }
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
    };

    for (int k = 0; k < mine; ++k) {
      const int t0 = real_tile(lt0 + wave + k * W) * T;
      bool masked = t0 + T - 1 > S - p.L;
      if (p.mode == MD_MODE_DRAFT)
        masked = masked || !(t0 + T <= p.n_sink || t0 > S - 1 - p.window);
      // The next tile is loaded in any case (behind the last: the last again).  Registers filled
      // on some paths only would be copied at the loop's end, and the copy would wait for them.
      process(masked, tile, t0, [&]() {
        if (PG == 1 && ((k + 1) & 31) == 0) {
          ids = ids_next;
          ids_next = load_ids(k + 33);
        }
        load_tile(tile, k + 1);
      });
    }
#pragma unroll
    for (int rt = 0; rt < NT; ++rt)
      if (__any(nan_v[rt] != 0)) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
          if ((nan_v[rt] >> (cb / 2)) & 1u) acc[rt][cb] += __uint_as_float(0x7fc00000u);
      }

    // ---- join the waves: each row's max, then sums weighted by 2^(m_w - M), in wave order
#pragma unroll
    for (int rt = 0; rt < NT; ++rt) {
      l_run[rt] += __shfl_xor(l_run[rt], 16);
      l_run[rt] += __shfl_xor(l_run[rt], 32);
    }
    float* sm = reinterpret_cast<float*>(lds + kQ);
    float* sl = sm + W * ROWS;
    float* mo = sl + W * ROWS;
    if (grp == 0) {
#pragma unroll
      for (int rt = 0; rt < NT; ++rt) {
        sm[wave * ROWS + rt * 16 + l16] = lazy[rt] == -INFINITY ? -INFINITY : m_run[rt];
        sl[wave * ROWS + rt * 16 + l16] = l_run[rt];
      }
    }
    // A cut unit's piece: two slots for each range of each member, its first piece's and its last's.
    const int64_t slot = 2 * (static_cast<int64_t>(range) * p.share + mem) +
                         (p.balanced && c.t != range_start(c, range));
#pragma unroll
    for (int rt = 0; rt < NT; ++rt) {
      __syncthreads();  // the V tiles, or the last row tile's O, are done with
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
        *reinterpret_cast<f32x4*>(mo + (wave * 16 + l16) * MROW + cb * 16 + grp * 4) = acc[rt][cb];
      __syncthreads();
      constexpr int kQuads = D / 4;
      for (int item = tid; item < 16 * kQuads; item += W * 64) {
        const int rr = item / kQuads, r = rt * 16 + rr, c0 = item % kQuads * 4;
        if (r >= rows) break;
        float M = -INFINITY;
        for (int w = 0; w < W; ++w) M = fmaxf(M, sm[w * ROWS + r]);
        const float m_use = M == -INFINITY ? 0.f : M;
        float L = 0.f;
        f32x4 o = {0.f, 0.f, 0.f, 0.f};
        for (int w = 0; w < W; ++w) {
          const float f = exp2_fast(sm[w * ROWS + r] - m_use);
          L += f * sl[w * ROWS + r];
          const f32x4 x = *reinterpret_cast<const f32x4*>(mo + (w * 16 + rr) * MROW + c0);
          for (int j = 0; j < 4; ++j) o[j] += f * x[j];
        }
        if (whole) {
          const int64_t row = out_row(p, b, hk, r0 + r);
          const float inv = inverse(L);
          for (int j = 0; j < 4; ++j) o[j] *= inv;
          store4<BF16>(p, row * D + c0, o);
          if (c0 == 0 && p.lse) p.lse[row] = lse_of(M, L);
        } else {
          *reinterpret_cast<f32x4*>(p.part_o + (slot * ROWS + r) * D + c0) = o;
          if (c0 == 0)
            *reinterpret_cast<f32x2*>(p.part_ml + (slot * ROWS + r) * 2) = f32x2{M, L};
        }
      }
    }

    // ---- the next piece of the range
    c.t = min(c.hi, c.g0 + c.gt);
    if (c.t >= c.hi) return;
    c.g0 += c.gt;
    if (++c.j == p.groups) {
      c.j = 0;
      ++c.b;
      S_next = length(p, c.b);
      c.gt = max(uniform(tiles_of(p, S_next).n), 1);
    }
    __syncthreads();  // the LDS is reused
  }
}

// Joins the pieces of the units that range boundaries cut: workgroup (x, y) takes rows
// 4 y .. of the unit whose first cut is where the range of workgroup x begins, if it is one.  The waves take the
// pieces in turn (fixed order), then their sums are joined through LDS.
template <int D, bool BF16, int NT>
__global__ void __launch_bounds__(W * 64) kv4_join_kernel(const Kv4AttnParams p, int rows_per_wg) {
  constexpr int kQuads = D / 4, ROWS = NT * 16, kRows = 64 / kQuads;  // rows a wave takes at once
  __shared__ __attribute__((aligned(16))) float so[W][64][4];
  __shared__ float sm[W][64], sl[W][64];
  const Join join = p.joins[blockIdx.x];
  if (join.b < 0) return;  // the whole workgroup
  const int w = place(p, static_cast<int>(blockIdx.x)), mem = member(p, static_cast<int>(blockIdx.x));
  const int unit = join.j * p.share + mem, hk = unit / p.passes, r0 = unit % p.passes * ROWS;
  const int rows = min(p.R - r0, ROWS);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c0 = lane % kQuads * 4;
  const int n = join.last - w + 2;  // pieces: ranges w - 1 .. last
  // With few pieces each wave takes rows of its own instead.
  const bool split = n > W;
  const int first = static_cast<int>(blockIdx.y) * rows_per_wg;
  const int end = min(rows, first + rows_per_wg);
  for (int rb = first + (split ? 0 : wave * kRows); rb < end; rb += split ? kRows : W * kRows) {
    const int r = rb + lane / kQuads;
    const bool live = r < end;
    float M = -INFINITY, L = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = split ? wave : 0; k < n; k += split ? W : 1) {
      const int64_t row =
          static_cast<int64_t>(k == 0 ? join.first : 2 * ((w - 1 + k) * p.share + mem)) * ROWS +
          (live ? r : first);
      const f32x2 ml = *reinterpret_cast<const f32x2*>(p.part_ml + row * 2);
      const f32x4 x = *reinterpret_cast<const f32x4*>(p.part_o + row * D + c0);
      const float m_new = fmaxf(M, ml[0]);
      const float m_use = m_new == -INFINITY ? 0.f : m_new;
      const float f = exp2_fast(M - m_use), g = exp2_fast(ml[0] - m_use);
      L = L * f + ml[1] * g;
      for (int j = 0; j < 4; ++j) o[j] = o[j] * f + x[j] * g;
      M = m_new;
    }
    if (split) {
      __syncthreads();  // the last rows' sums are read
      *reinterpret_cast<f32x4*>(so[wave][lane]) = o;
      sm[wave][lane] = M;
      sl[wave][lane] = L;
      __syncthreads();
      if (wave != 0) continue;
      for (int k = 1; k < W; ++k) M = fmaxf(M, sm[k][lane]);
      const float m_use = M == -INFINITY ? 0.f : M;
      L = 0.f;
      o = f32x4{0.f, 0.f, 0.f, 0.f};
      for (int k = 0; k < W; ++k) {
        const float f = exp2_fast(sm[k][lane] - m_use);
        L += f * sl[k][lane];
        for (int j = 0; j < 4; ++j) o[j] += f * so[k][lane][j];
      }
    }
    if (!live) continue;
    const int64_t row = out_row(p, join.b, hk, r0 + r);
    const float inv = inverse(L);
    for (int j = 0; j < 4; ++j) o[j] *= inv;
    store4<BF16>(p, row * D + c0, o);
    if (c0 == 0 && p.lse) p.lse[row] = lse_of(M, L);
  }
}

template <int D, bool BF16, int NT>
hipError_t launch_nt(const Kv4AttnParams& p, const Kv4Plan& pl, hipStream_t s) {
  const dim3 g(static_cast<uint32_t>(pl.n_blocks)), blk(W * 64);
  if (!p.c.page_table)
    hipLaunchKernelGGL((kv4_attn_kernel<D, BF16, NT, 0>), g, blk, 0, s, p);
  else if (p.c.page_shift >= 4)
    hipLaunchKernelGGL((kv4_attn_kernel<D, BF16, NT, 1>), g, blk, 0, s, p);
  else
    hipLaunchKernelGGL((kv4_attn_kernel<D, BF16, NT, 2>), g, blk, 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !pl.balanced) return e;
  // Units cut in many pieces are few: their rows go to several workgroups, four each.
  const int rows = NT * 16 < p.R ? NT * 16 : p.R;
  const bool many = pl.n_blocks > 4 * static_cast<int64_t>(p.B) * p.units;
  const int per_wg = many && rows > 4 ? 4 : rows;
  const dim3 gj(g.x, static_cast<uint32_t>((rows + per_wg - 1) / per_wg));
  hipLaunchKernelGGL((kv4_join_kernel<D, BF16, NT>), gj, blk, 0, s, p, per_wg);
  return hipGetLastError();
}

template <int D, bool BF16>
hipError_t launch_d(const Kv4AttnParams& p, const Kv4Plan& pl, hipStream_t s) {
  static_assert(kKv4MaxNT(true) == 4 && kKv4MaxNT(false) == 2, "one instance for each");
  switch (pl.NT) {
    case 1: return launch_nt<D, BF16, 1>(p, pl, s);
    case 2: return launch_nt<D, BF16, 2>(p, pl, s);
  }
  if constexpr (BF16) {
    switch (pl.NT) {
      case 3: return launch_nt<D, BF16, 3>(p, pl, s);
      case 4: return launch_nt<D, BF16, 4>(p, pl, s);
    }
  }
  return hipErrorInvalidValue;
}

}  // namespace

hipError_t launch_kv4_attn(const Kv4AttnParams& p, const Kv4Plan& pl, int head_dim, bool bf16,
                           hipStream_t s) {
  if (head_dim == 128)
    return bf16 ? launch_d<128, true>(p, pl, s) : launch_d<128, false>(p, pl, s);
  return bf16 ? launch_d<64, true>(p, pl, s) : launch_d<64, false>(p, pl, s);
}

}  // namespace md
