// kv_evict.hip -- a cache cut down to its budget by accumulated weight: per (sequence, KV
// head) the n - budget tokens of least weight go, and the tokens kept behind the budget move
// into the slots that this frees.
//
// One workgroup a (sequence, KV head) finds the key of rank n - budget by a radix select (three
// rounds over keys in LDS), counts in slot order and lists (freed slot, kept slot) pairs; pairs are
// moved by the same workgroup or, where a call may have more than kEvictFused of them a head, by a
// second launch over the whole device.  8 x 8 heads of 16384 .. 32768 tokens cut to 2049: 41 us for the select,
// bound by its dependent rounds, and 18 for the moves (6.5 TB/s); 64 x 8 of 2054: 10 us in all (more in caches
// that can hold more: see the launch).
#include <type_traits>

#include "answers_kernels.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr uint32_t kHeld = 0xffffffffu;  // sinks and recent tokens: above every weight
constexpr int kFew = 8;                  // tokens that go one after another rather than by a select

struct EvictUnit {
  const float* mass;
  const int32_t* pos;
  int32_t n_sink;
  int64_t recent_from;
};

// The order of a slot's token: its weight's, NaN least, held tokens last.
__device__ __forceinline__ uint32_t order_key(const EvictUnit& u, int pos, float mass) {
  const uint32_t x = __float_as_uint(mass + 0.f);  // -0 and 0 are equal
  const uint32_t key = mass != mass ? 0u : ((x >> 31) ? ~x : x | 0x80000000u);
  return pos < u.n_sink || pos >= u.recent_from ? kHeld : key;
}

// Byte offset of a token's row of head hk, or -1: on no page of the pool.
__device__ __forceinline__ int64_t row_offset(const EvictParams& p, int b, int hk, int j) {
  int64_t off;
  if (p.paged) {
    const int pid = p.c.page_table[static_cast<int64_t>(b) * p.c.max_pages + (j >> p.c.page_shift)];
    if (pid < 0 || pid >= p.c.num_pages) return -1;
    off = static_cast<int64_t>(pid) * p.c.s_blk +
          static_cast<int64_t>(j & ((1 << p.c.page_shift) - 1)) * p.c.s_tok;
  } else {
    off = static_cast<int64_t>(b) * p.c.s_blk + static_cast<int64_t>(j) * p.c.s_tok;
  }
  return (off + static_cast<int64_t>(hk) * p.c.s_head) * p.esize;
}

// The least pair over the wave, by DPP moves; all lanes get it.
__device__ __forceinline__ unsigned long long wave_least(unsigned long long x) {
#define MD_STEP(ctrl, rows)                                                                          \
  do {                                                                                               \
    const uint32_t lo = __builtin_amdgcn_update_dpp(-1, static_cast<int>(x), ctrl, rows, 0xf, false);  \
    const uint32_t hi = __builtin_amdgcn_update_dpp(-1, static_cast<int>(x >> 32), ctrl, rows, 0xf, false); \
    const unsigned long long y = (static_cast<unsigned long long>(hi) << 32) | lo;                   \
    x = y < x ? y : x;                                                                               \
  } while (0)
  MD_STEP(0x111, 0xf);  // within rows of 16: row_shr 1, 2, 4, 8
  MD_STEP(0x112, 0xf);
  MD_STEP(0x114, 0xf);
  MD_STEP(0x118, 0xf);
  MD_STEP(0x142, 0xa);  // the last lane of rows 0 and 2 to rows 1 and 3,
  MD_STEP(0x143, 0xc);  // of row 1 to rows 2 and 3
#undef MD_STEP
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(x), 63);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(x >> 32), 63);
  return (static_cast<unsigned long long>(hi) << 32) | lo;
}

// One 16-byte vector of a pair's K or V row (item: pair, then K or V, then the vector); the first of
// a pair moves its mass and position.
__device__ __forceinline__ void move_vector(const EvictParams& p, int unit, int2 pair, int vec) {
  const int b = unit / p.Hkv, hk = unit % p.Hkv;
  const int64_t to = row_offset(p, b, hk, pair.x), from = row_offset(p, b, hk, pair.y);
  if (to >= 0 && from >= 0) {
    unsigned char* const base = vec < p.row_vecs ? p.c.k : p.c.v;
    const int at = (vec < p.row_vecs ? vec : vec - p.row_vecs) * 16;
    *reinterpret_cast<u32x4*>(base + to + at) = *reinterpret_cast<const u32x4*>(base + from + at);
  }
  if (vec == 0) {
    const int64_t s = static_cast<int64_t>(unit) * p.slot_stride;
    p.mass[s + pair.x] = p.mass[s + pair.y];
    p.slot_pos[s + pair.x] = p.slot_pos[s + pair.y];
  }
}

// NT threads; the order of the first KEYS slots is kept in LDS (of more, it is made from memory every
// time).
template <int NT, int KEYS>
__global__ void __launch_bounds__(NT)
evict_select(const EvictParams p) {
  constexpr int NW = NT / 64, BINS = 2048;
  __shared__ uint32_t hist[BINS];
  __shared__ int counts[3][NW];
  __shared__ uint32_t pick[2];
  __shared__ uint32_t keys[KEYS];
  int2* const listed = reinterpret_cast<int2*>(hist);  // after the select
  static_assert(sizeof(hist) >= sizeof(int2) * kEvictFused, "the pairs take the histogram's place");
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int unit = blockIdx.x, b = unit / p.Hkv;
  const int n = min(max(p.lens[b], 0), p.slots);
  if (p.lens_out && unit % p.Hkv == 0 && tid == 0) p.lens_out[b] = min(n, p.budget);
  if (n <= p.budget) {
    if (p.counts && tid == 0) p.counts[unit] = 0;
    return;
  }
  const int64_t s0 = static_cast<int64_t>(unit) * p.slot_stride;
  const EvictUnit u = {p.mass + s0, p.slot_pos + s0, p.n_sink,
                       static_cast<int64_t>(p.seq_lens[b]) - p.recent};
  for (int j0 = 0; j0 < min(n, KEYS); j0 += 8 * NT) {
    int pos[8];
    float w[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = min(j0 + i * NT + tid, n - 1);
      pos[i] = u.pos[j];
      w[i] = u.mass[j];
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int j = j0 + i * NT + tid;
      if (j < min(n, KEYS)) keys[j] = order_key(u, pos[i], w[i]);
    }
  }
  const int vecs = 2 * p.row_vecs;
  if (n - p.budget <= kFew && n <= KEYS) {
    // A step's few tokens: the least (key, slot) pair above the last one found, one after another
    // (up to six of 2055 tokens in 512 heads: 10.0 us a call so, 17.8 by the select and its scans).
    __shared__ unsigned long long least[2][NW];
    const int m = n - p.budget;
    unsigned long long last = 0;  // below every pair, as slots are counted from 1 in them
    int gone[kFew];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kFew; ++i) {
      gone[i] = INT32_MAX;
      if (i >= m) continue;
      unsigned long long mine = ~0ull;
      for (int j = tid; j < n; j += NT) {
        const unsigned long long x = (static_cast<unsigned long long>(keys[j]) << 32) | static_cast<uint32_t>(j + 1);
        if (x > last && x < mine) mine = x;
      }
      mine = wave_least(mine);
      if (lane == 0) least[i & 1][wave] = mine;
      __syncthreads();
      last = least[i & 1][0];
      for (int x = 1; x < NW; ++x) last = least[i & 1][x] < last ? least[i & 1][x] : last;
      gone[i] = static_cast<int>(static_cast<uint32_t>(last)) - 1;
    }
    // The kept slots behind the budget, in order, take the freed ones below it, in order.
    if (tid == 0) {
      int total = 0, at = -1;
      for (int j = p.budget; j < n; ++j) {
        bool out = false;
        int next = INT32_MAX;  // the least freed slot above the last one taken
#pragma unroll
        for (int i = 0; i < kFew; ++i) {
          out |= gone[i] == j;
          if (gone[i] > at && gone[i] < next) next = gone[i];
        }
        if (out) continue;
        listed[total++] = make_int2(next, j);
        at = next;
      }
      counts[0][0] = total;
    }
    __syncthreads();
    const int total = counts[0][0];
    if (p.counts && tid == 0) p.counts[unit] = 0;  // moved here
    for (int x = tid; x < total * vecs; x += NT) move_vector(p, unit, listed[x / vecs], x % vecs);
    return;
  }

  // (With the choice of LDS or memory inside its loops the select waits for every key in turn.)
  auto select = [&](auto in_lds) {
    auto key_of = [&](int j) {
      if constexpr (in_lds) return keys[j];
      return j < KEYS ? keys[j] : order_key(u, u.pos[j], u.mass[j]);
    };

    // The key of rank n - budget (from 1), 11, 11 and 10 bits a round (weights spread over few exponents, and
    // atomics on one bin take turns: with the upper 8 bits alone they took longer than the rest): of the
    // keys that agree with `prefix` in the bits above, `want` is the rank looked for.
    uint32_t prefix = 0;
    int want = n - p.budget;
#pragma unroll
    for (int round = 0; round < 3; ++round) {
      const int shift = round == 0 ? 21 : (round == 1 ? 10 : 0), bits = round == 2 ? 10 : 11;
      for (int i = tid; i < BINS; i += NT) hist[i] = 0;
      __syncthreads();
#pragma unroll 4
      for (int j = tid; j < n; j += NT) {
        const uint32_t key = key_of(j);
        if (round == 0 || (key >> (shift + bits)) == (prefix >> (shift + bits)))
          atomicAdd(&hist[(key >> shift) & ((1u << bits) - 1u)], 1u);
      }
      __syncthreads();
      // The bin in which the running count reaches `want`: 256 threads of eight bins each.
      uint32_t h[8], mine = 0, incl = 0;
      if (tid < 256) {
#pragma unroll
        for (int i = 0; i < 8; ++i) mine += h[i] = hist[tid * 8 + i];
        incl = mine;
        for (int o = 1; o < 64; o <<= 1) {
          const uint32_t x = __shfl_up(incl, o);
          if (lane >= o) incl += x;
        }
        if (lane == 63) counts[0][wave] = static_cast<int>(incl);
      }
      __syncthreads();
      if (tid < 256) {
        uint32_t run = incl - mine;
        for (int x = 0; x < wave; ++x) run += static_cast<uint32_t>(counts[0][x]);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (run < static_cast<uint32_t>(want) && static_cast<uint32_t>(want) <= run + h[i]) {
            pick[0] = tid * 8 + i;
            pick[1] = want - run;
          }
          run += h[i];
        }
      }
      __syncthreads();
      prefix |= pick[0] << shift;
      want = static_cast<int>(pick[1]);
    }
    // Evicted: keys below `prefix`, and the first `want` slots whose key is `prefix`.

    // Each wave takes a run of slots and counts, below and from the budget on, those that go by their key,
    // those that stay, and those with the key `prefix`.
    const int per = (n + NW * 64 - 1) / (NW * 64) * 64, lo = min(n, wave * per), hi = min(n, lo + per);
    int holes = 0, extras = 0, ties_low = 0, ties_high = 0;
    for (int j0 = lo; j0 < hi; j0 += 4 * 64) {
      uint32_t key[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) key[i] = key_of(min(j0 + i * 64 + lane, n - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = j0 + i * 64 + lane;
        const bool in = j < hi, low = j < p.budget;
        holes += __popcll(__ballot(in && low && key[i] < prefix));
        extras += __popcll(__ballot(in && !low && key[i] > prefix));
        ties_low += __popcll(__ballot(in && low && key[i] == prefix));
        ties_high += __popcll(__ballot(in && !low && key[i] == prefix));
      }
    }
    __syncthreads();
    if (lane == 0) counts[0][wave] = ties_low + ties_high;
    __syncthreads();
    int tie0 = 0;
    for (int x = 0; x < wave; ++x) tie0 += counts[0][x];
    // Of this wave's ties the first `go` go.
    const int go = min(max(want - tie0, 0), ties_low + ties_high);
    holes += min(go, ties_low);
    extras += ties_high - max(go - ties_low, 0);
    if (lane == 0) {
      counts[1][wave] = holes;
      counts[2][wave] = extras;
    }
    __syncthreads();
    int hole = 0, extra = 0, total = 0, tie = tie0;
    for (int x = 0; x < NW; ++x) {
      if (x < wave) {
        hole += counts[1][x];
        extra += counts[2][x];
      }
      total += counts[1][x];
    }
    // As many slots are freed below the budget as tokens are kept behind it: the x-th takes the x-th.
    int2* const pairs = p.counts ? p.moves + static_cast<int64_t>(unit) * p.max_moves : listed;
    auto before = [](unsigned long long m) {  // lanes of m before this one
      return static_cast<int>(__builtin_amdgcn_mbcnt_hi(static_cast<uint32_t>(m >> 32),
                                                        __builtin_amdgcn_mbcnt_lo(static_cast<uint32_t>(m), 0u)));
    };
    for (int j0 = lo; j0 < hi; j0 += 4 * 64) {
      uint32_t keys4[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) keys4[i] = key_of(min(j0 + i * 64 + lane, n - 1));
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = j0 + i * 64 + lane;
        const bool in = j < hi;
        const uint32_t key = keys4[i];
        const unsigned long long eq = __ballot(in && key == prefix);
        const bool out = key < prefix || (key == prefix && tie + before(eq) < want);
        tie += __popcll(eq);
        const bool is_hole = in && out && j < p.budget, is_extra = in && !out && j >= p.budget;
        const unsigned long long hm = __ballot(is_hole), em = __ballot(is_extra);
        if (is_hole) pairs[hole + before(hm)].x = j;
        if (is_extra) pairs[extra + before(em)].y = j;
        hole += __popcll(hm);
        extra += __popcll(em);
      }
    }
    if (p.counts) {
      if (tid == 0) p.counts[unit] = total;
      return;
    }
    __syncthreads();
    for (int x = tid; x < total * vecs; x += NT) move_vector(p, unit, listed[x / vecs], x % vecs);
  };
  if (n <= KEYS)
    select(std::true_type{});
  else
    select(std::false_type{});
}

// Workgroups (unit, y): each takes every gridDim.y-th run of 256 vectors of the unit's pairs.
__global__ void __launch_bounds__(256)
evict_move(const EvictParams p) {
  const int unit = blockIdx.x, vecs = 2 * p.row_vecs;
  const int64_t total = static_cast<int64_t>(p.counts[unit]) * vecs;
  const int2* const pairs = p.moves + static_cast<int64_t>(unit) * p.max_moves;
  const int64_t step = static_cast<int64_t>(gridDim.y) * 256;
  for (int64_t x = static_cast<int64_t>(blockIdx.y) * 256 + threadIdx.x; x < total; x += step)
    move_vector(p, unit, pairs[x / vecs], static_cast<int>(x % vecs));
}

}  // namespace

hipError_t launch_kv_evict(const EvictParams& p, hipStream_t s) {
  const uint32_t units = static_cast<uint32_t>(p.B) * static_cast<uint32_t>(p.Hkv);
  // By what the cache can hold, for its lengths are on the device: a step's eviction of 64 x 8 heads of up to 2055
  // tokens is 10.7 us a call in a cache of 2054, 12.9 in one of 4096, and 17.5 in one of 4097 to 32768, whose
  // workgroups are one a compute unit and whose launch of moves finds none.
  if (p.slots <= 4096)
    hipLaunchKernelGGL((evict_select<256, 4096>), dim3(units), dim3(256), 0, s, p);
  else
    hipLaunchKernelGGL((evict_select<1024, 32768>), dim3(units), dim3(1024), 0, s, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || !p.counts) return e;
  const uint32_t y = units >= 2048 ? 1 : (2048 + units - 1) / units;
  hipLaunchKernelGGL(evict_move, dim3(units, y), dim3(256), 0, s, p);
  return hipGetLastError();
}

}  // namespace md
