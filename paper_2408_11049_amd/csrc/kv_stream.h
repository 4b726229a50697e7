// kv_stream.h -- how a wave reads rows of a KV cache, tile by tile, for the matrix units: shared by
// the shared-prefix attention and the accumulated weights.
#pragma once

#include "answers_kernels.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
// LDS that only this wave touches: writes before, reads after.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// Rows of D channels in LDS.
template <int D, bool BF16>
struct Tile {
  static constexpr int ES = BF16 ? 2 : 4;
  static constexpr int ROW = D * ES;          // bytes of a row
  static constexpr int CH = ROW / 16;         // 16-byte chunks of a row
  // Rows sit unpadded, chunk c of row r in place c ^ turn(r).  The banks hold 256 bytes, and both ways
  // of reading cover them all: 16 rows at one c (an operand), and four rows of a multiple of four at
  // four chunks from a multiple of four on (a transposed operand; turned by r alone, those were half of
  // the LDS's cycles in conflicts).
  static __device__ __forceinline__ int at(int r, int c) {
    const int turn = ROW == 512 ? r & 15
                   : ROW == 256 ? (r & 3) << 2 | ((r >> 2) & 3)
                                : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
    return r * ROW + ((c ^ turn) << 4);
  }
};

// The rows of K (and V) of tokens [.., end) of one (block, KV head), 32 a tile, one tile in a wave's registers
// on its way.  Every load is issued whatever the tile, so that no branch stands between the loads and their
// use and those on their way can be counted: a row past the end, or on a page outside the pool, is
// redirected to one that may be read and staged as zeros.  CACHED: other workgroups read the same rows
// soon, else the loads are nontemporal (own caches of 64 x 256 .. 2048 tokens, 5 query tokens: 88 us nontemporal
// and 98 not with one workgroup a KV head's rows, 131 and 119 with two).
template <int D, bool BF16, bool VALUES, bool CACHED>
struct Stream {
  using T = Tile<D, BF16>;
  static constexpr int KEYS = 32, NV = KEYS * T::CH / 64, RPW = 64 / T::CH;  // RPW: rows a load instruction
  const unsigned char *k, *v;
  int64_t s_blk, s_tok, head, num_pages;
  // A contiguous cache loads a length of no use in a page id's place, so that as many loads are on their way.
  const int32_t* table;
  int blk, end, lane, page_shift;
  bool paged, groups;
  uint32_t lane_off;
  u32x4 kr[NV], vr[VALUES ? NV : 1];
  uint32_t ok;         // bit n: row n of this lane is a token

  __device__ __forceinline__ Stream(const KvView& c, int blk_, int hk, int end_, int lane_)
      : k(c.k), v(c.v), s_blk(c.s_blk), s_tok(c.s_tok), head(static_cast<int64_t>(hk) * c.s_head),
        num_pages(c.num_pages), blk(blk_), end(end_), lane(lane_), page_shift(c.page_shift),
        paged(c.page_table != nullptr) {
    table = paged ? c.page_table + static_cast<int64_t>(blk) * c.max_pages : c.lens;
    groups = !paged || (1 << page_shift) >= RPW;
    lane_off = static_cast<uint32_t>((lane / T::CH) * s_tok * T::ES + (lane % T::CH) * 16);
  }
  // This lane's token of tile t, past the end the last one.  Tiles ahead of the last one's end may lie past
  // 31 bits.
  __device__ __forceinline__ int token(int t) const {
    return min(min(t, (end - 1) / KEYS) * KEYS + (lane & 31), end - 1);
  }
  // The block (sequence or page) of this lane's token of tile t, lane & 31; past the end the last one's.
  __device__ __forceinline__ int load_block(int t) const {
    const int tok = token(t);
    const int id = table[paged ? tok >> page_shift : 0];
    return paged ? id : blk;
  }
  // Tile t, whole rows: RPW of them an instruction, at one scalar address and a fixed offset a lane
  // where they are all tokens of one page, else each lane at its row's.
  __device__ __forceinline__ void load(int t, int block) {
    const bool in_pool = !paged || (block >= 0 && block < num_pages);
    const unsigned long long pool = __ballot(in_pool);
    const int tok = token(t);
    const int64_t row = (static_cast<int64_t>(in_pool ? block : 0) * s_blk +
                         static_cast<int64_t>(paged ? tok & ((1 << page_shift) - 1) : tok) * s_tok + head) * T::ES;
    const int lo = static_cast<int>(row), hi = static_cast<int>(row >> 32);
    auto join = [](int a, int b) {
      return static_cast<int64_t>((static_cast<uint64_t>(static_cast<uint32_t>(b)) << 32) | static_cast<uint32_t>(a));
    };
    auto get = [&](int n, int64_t byte) {
      auto one = [](const unsigned char* x) {
        const u32x4* const p = reinterpret_cast<const u32x4*>(x);
        return CACHED ? *p : __builtin_nontemporal_load(p);
      };
      kr[n] = one(k + byte);
      if constexpr (VALUES) vr[n] = one(v + byte);
    };
    ok = 0;
    if (groups && t < end / KEYS) {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        get(n, join(__builtin_amdgcn_readlane(lo, n * RPW), __builtin_amdgcn_readlane(hi, n * RPW)) + lane_off);
        ok |= static_cast<uint32_t>((pool >> (n * RPW)) & 1ull) << n;
      }
    } else {
#pragma unroll
      for (int n = 0; n < NV; ++n) {
        const int of = n * RPW + lane / T::CH;
        get(n, join(__shfl(lo, of), __shfl(hi, of)) + (lane % T::CH) * 16);
        ok |= static_cast<uint32_t>(t <= (end - 1 - of) / KEYS && of < end && ((pool >> of) & 1ull)) << n;
      }
    }
  }
  // The loaded tile to the wave's LDS.
  __device__ __forceinline__ void store(unsigned char* kt, unsigned char* vt) {
    if (__any(ok != (1u << NV) - 1u)) {
#pragma unroll
      for (int n = 0; n < NV; ++n)
        if (!((ok >> n) & 1u)) {
          kr[n] = u32x4{0, 0, 0, 0};
          if constexpr (VALUES) vr[n] = u32x4{0, 0, 0, 0};
        }
    }
#pragma unroll
    for (int n = 0; n < NV; ++n) {
      const int a = T::at(n * RPW + lane / T::CH, lane % T::CH);
      *reinterpret_cast<u32x4*>(kt + a) = kr[n];
      if constexpr (VALUES) *reinterpret_cast<u32x4*>(vt + a) = vr[n];
    }
  }
};

}  // namespace

}  // namespace md
