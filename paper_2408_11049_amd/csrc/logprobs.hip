// logprobs.hip -- per row of logits: the log probability of a given token, the entropy and
// the top_k most likely tokens, from one pass over the row (see the top tokens for what is read again).
//
// A workgroup takes a segment of a row, 256 lanes holding 16 or 32 logits each in
// registers at a time.  Sums: each lane keeps a maximum m, z = sum exp(x - m) and
// t = sum exp(x - m) (x - m); a log probability is (x - m) - ln z, the entropy ln z - t / z.  Differences to the
// maximum are taken before the scaling to log2, and m + ln z, which would be rounded by half a step of m, is never
// formed, so that large logits lose nothing.
// Top tokens: with each wave's (top_k / 4)-th largest lane maximum, the least of the four is below
// top_k logits at least, so only logits from there on are candidates, some twice top_k of them; they go
// to a list in LDS, which is cut to its best top_k where it would overflow (rows of equal
// or clustered values; those logits are read again).  Where no bound stands, the masked ones are looked for, from
// memory too.  Candidates are ranked by counting the better ones.
// Rows of several segments are joined by a second launch.  320 rows of 128256 fp32, top 20: 36 us (4.6 TB/s,
// vector issue 54%) and 6 for the join, 41 a call, of bf16 38; one row of 50001 bf16, top 5: 6.5 and 4.
#include <float.h>

#include "answers_kernels.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kList = 256;  // candidates a wave lists

// A candidate as one number: the larger value first, then the lower index.
typedef unsigned long long Key;
__device__ __forceinline__ uint32_t order(float v) {  // v is no NaN
  const uint32_t x = __float_as_uint(v + 0.f);  // -0 and 0 are equal
  return (x >> 31) ? ~x : x | 0x80000000u;
}
__device__ __forceinline__ Key make_key(float v, int i) {
  return (static_cast<Key>(order(v)) << 32) | ~static_cast<uint32_t>(i);
}
__device__ __forceinline__ float key_value(Key k) {
  const uint32_t x = static_cast<uint32_t>(k >> 32);
  return __uint_as_float((x >> 31) ? x & 0x7fffffffu : ~x);
}
__device__ __forceinline__ int key_index(Key k) { return static_cast<int>(~static_cast<uint32_t>(k)); }

struct Stats {
  float m, z, t;
};
// Of two disjoint sets of logits.  An empty set is (-inf, 0, 0).
__device__ __forceinline__ Stats join(const Stats& a, const Stats& b) {
  const float m = fmaxf(a.m, b.m);
  if (m == -INFINITY) return Stats{m, a.z + b.z, a.t + b.t};  // nothing, or NaN
  // A set far below the other has weight 0; its distance must stay finite times z.
  const float da = a.m == -INFINITY ? 0.f : fmaxf(a.m - m, -1e20f);
  const float db = b.m == -INFINITY ? 0.f : fmaxf(b.m - m, -1e20f);
  const float fa = a.m == -INFINITY && a.z == 0.f ? 0.f : __builtin_amdgcn_exp2f(da * kLog2e);
  const float fb = b.m == -INFINITY && b.z == 0.f ? 0.f : __builtin_amdgcn_exp2f(db * kLog2e);
  // exp(x - m) (x - m) = f exp(x - a.m) ((x - a.m) + da)
  return Stats{m, a.z * fa + b.z * fb, fa * (a.t + a.z * da) + fb * (b.t + b.z * db)};
}
// A reduction over the wave by DPP moves: within rows of 16, then over the rows; all lanes get it.
template <typename F>
__device__ __forceinline__ float wave_reduce(float x, float none, F f) {
  const int id = __float_as_int(none);
#define MD_STEP(ctrl, rows) \
  x = f(x, __int_as_float(__builtin_amdgcn_update_dpp(id, __float_as_int(x), ctrl, rows, 0xf, false)))
  MD_STEP(0x111, 0xf);  // row_shr 1, 2, 4, 8
  MD_STEP(0x112, 0xf);
  MD_STEP(0x114, 0xf);
  MD_STEP(0x118, 0xf);
  MD_STEP(0x142, 0xa);  // the last lane of rows 0 and 2 to rows 1 and 3,
  MD_STEP(0x143, 0xc);  // of row 1 to rows 2 and 3
#undef MD_STEP
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
}
__device__ __forceinline__ Stats wave_join(const Stats& s) {
  const float m = wave_reduce(s.m, -INFINITY, [](float a, float b) { return fmaxf(a, b); });
  const Stats at = join(s, Stats{m, 0.f, 0.f});  // each lane's sums under the common maximum
  auto add = [](float a, float b) { return a + b; };
  return Stats{m, wave_reduce(at.z, 0.f, add), wave_reduce(at.t, 0.f, add)};
}

struct Finals {
  float m, lz, entropy;  // lse = m + lz, apart
};
// A row of nothing but -inf has m -inf and entropy 0; a NaN or +inf makes lz and the entropy NaN.
__device__ __forceinline__ Finals finals(const Stats& s) {
  if (s.z != s.z) return Finals{s.m, s.z, s.z};
  if (s.m == -INFINITY) return Finals{-INFINITY, 0.f, 0.f};
  const float lz = __builtin_amdgcn_logf(s.z) * kLn2;
  return Finals{s.m, lz, lz - s.t / s.z};
}
// x - lse of a logit: -inf for a masked one, whatever the row.
__device__ __forceinline__ float log_prob(float x, const Finals& f) {
  if (f.lz != f.lz) return f.lz;
  return x == -INFINITY ? -INFINITY : (x - f.m) - f.lz;
}

template <bool BF16>
__device__ __forceinline__ float logit(const void* base, int64_t e) {
  if constexpr (BF16)
    return __uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(base)[e]) << 16);
  return static_cast<const float*>(base)[e];
}

// How many of list[0 .. n) are above k; the entries from n to the next multiple of 8 are 0.
__device__ __forceinline__ int count_above(const Key* list, int n, Key k) {
  int above = 0;
  for (int e = 0; e < n; e += 8) {
    Key x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = list[e + j];
#pragma unroll
    for (int j = 0; j < 8; ++j) above += x[j] > k;
  }
  return above;
}
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// A wave's list of candidates and what a logit has to beat to enter it.
struct List {
  Key* key;        // kList, and 8 behind them
  int n;           // the same in all lanes
  float floor;     // no logit below it enters
  Key floor_key;   // nor any candidate that is not above this
};
__device__ __forceinline__ void pad(const List& l, int lane) {
  wave_sync();
  if (lane < 8) l.key[l.n + lane] = 0;
  wave_sync();
}
// The list cut to its best top_k, best first.  All lanes of the wave take part.
__device__ __forceinline__ void cut(List& l, int top_k, int lane) {
  pad(l, lane);
  Key k[kList / 64];
  int rank[kList / 64];
#pragma unroll
  for (int x = 0; x < kList / 64; ++x) {
    const int e = x * 64 + lane;
    k[x] = e < l.n ? l.key[e] : 0;
    rank[x] = e < l.n ? count_above(l.key, l.n, k[x]) : kList;
  }
  wave_sync();
#pragma unroll
  for (int x = 0; x < kList / 64; ++x)
    if (rank[x] < top_k) l.key[rank[x]] = k[x];
  wave_sync();
  l.n = min(l.n, top_k);
}
// Adds the keys of the lanes in m.
__device__ __forceinline__ void append(List& l, unsigned long long m, Key k, int lane) {
  if ((m >> lane) & 1ull) l.key[l.n + __popcll(m & ((1ull << lane) - 1))] = k;
  l.n += __popcll(m);
}
// The same where `in`, cutting a list that is full.
__device__ __forceinline__ void push(List& l, bool in, Key k, int top_k, int lane) {
  unsigned long long m = __ballot(in);
  if (l.n + __popcll(m) > kList) {
    cut(l, top_k, lane);
    l.floor_key = l.key[top_k - 1];  // kList > 2 * kLogpMaxTop: the list held more than top_k
    l.floor = key_value(l.floor_key);
    m = __ballot(in && k > l.floor_key);
  }
  append(l, m, k, lane);
}

// The best top_k of four waves' lists, by the whole workgroup: a thread takes a candidate in
// turn and counts those above it.  f(rank, value, index) for each of the best.
template <typename F>
__device__ __forceinline__ void best_of(const Key (&key)[4][kList + 8], const int (&n)[4], int top_k, F f) {
  const int total = n[0] + n[1] + n[2] + n[3];
  for (int e0 = threadIdx.x; e0 < total; e0 += 256) {
    int w = 0, e = e0;
    while (e >= n[w]) e -= n[w++];
    const Key k = key[w][e];
    int rank = 0;
#pragma unroll
    for (int x = 0; x < 4; ++x) rank += count_above(key[x], n[x], k);
    if (rank < top_k) f(rank, key_value(k), key_index(k));
  }
}

// PL logits a lane at a time.
template <bool BF16, int PL>
__global__ void __launch_bounds__(256)
logprobs_kernel(const LogpParams p) {
  constexpr int VN = BF16 ? 8 : 4, NV = PL / VN;  // logits of a 16-byte vector, vectors a lane
  __shared__ __attribute__((aligned(16))) Key l_key[4][kList + 8];
  __shared__ int l_n[4];
  __shared__ int l_bound[4];  // apart from l_n, which a wave without logits writes while others still read these
  __shared__ Stats l_stats[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = static_cast<int>(blockIdx.x) / p.n_segs, seg = static_cast<int>(blockIdx.x) % p.n_segs;
  const int64_t row0 = row * p.row_stride;
  const int seg0 = seg * p.seg_len, seg1 = static_cast<int>(min(static_cast<int64_t>(p.vocab),
                                                                 static_cast<int64_t>(seg0) + p.seg_len));
  const int K = p.top_k;
  float x_tok = 0.f;
  int tok = -1;
  if (p.n_segs == 1 && p.tokens && tid == 0) {
    tok = p.tokens[row];
    if (tok >= 0 && tok < p.vocab) x_tok = logit<BF16>(p.logits, row0 + tok);
  }

  Stats st = {-INFINITY, 0.f, 0.f};
  List list = {l_key[wave], 0, -INFINITY, 0};
  // Element j of vector v of this lane.
  auto at = [&](int wave0, int v, int j) { return wave0 + v * 64 * VN + lane * VN + j; };
  for (int c0 = seg0; c0 < seg1; c0 += 256 * PL) {
    float x[PL];
    const int wave0 = c0 + wave * PL * 64;
    if (wave0 + PL * 64 <= seg1) {
      u32x4 raw[NV];
      // Rows begin where the vocabulary puts them: any element's address will do for a load.
      typedef u32x4 at2 __attribute__((aligned(2)));
      typedef u32x4 at4 __attribute__((aligned(4)));
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int64_t e = row0 + at(wave0, v, 0);
        if constexpr (BF16)
          raw[v] = __builtin_nontemporal_load(
              reinterpret_cast<const at2*>(static_cast<const uint16_t*>(p.logits) + e));
        else
          raw[v] = __builtin_nontemporal_load(
              reinterpret_cast<const at4*>(static_cast<const float*>(p.logits) + e));
      }
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if constexpr (BF16) {
            x[v * 8 + 2 * j] = __uint_as_float(raw[v][j] << 16);
            x[v * 8 + 2 * j + 1] = __uint_as_float(raw[v][j] & 0xffff0000u);
          } else {
            x[v * 4 + j] = __uint_as_float(raw[v][j]);
          }
        }
    } else {
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int j = 0; j < VN; ++j) {
          const int i = at(wave0, v, j);
          x[v * VN + j] = i < seg1 ? logit<BF16>(p.logits, row0 + i) : -INFINITY;
        }
    }

    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < PL; ++e) mx = fmaxf(mx, x[e]);
    {
      const float m_use = mx == -INFINITY ? 0.f : mx;
      float z[4] = {}, t[4] = {};
#pragma unroll
      for (int e = 0; e < PL; ++e) {
        const float d = x[e] - m_use;
        const float w = __builtin_amdgcn_exp2f(d * kLog2e);
        z[e & 3] += w;
        t[e & 3] = __builtin_fmaf(w, fmaxf(d, -1e30f), t[e & 3]);  // 0 * -inf is no term
      }
      st = join(st, Stats{mx, (z[0] + z[1]) + (z[2] + z[3]), (t[0] + t[1]) + (t[2] + t[3])});
    }

    if (K > 0) {
      if (c0 == seg0) {
        // A bound below no more than K of the logits: of a whole segment the least, over the waves, of each
        // wave's (K / 4)-th largest lane maximum, else the largest of each one's K-th.  In the upper 16
        // bits of its order (rounded down, as a lower bound may be), bit by bit: whether enough lanes still
        // reach it.
        const bool whole = c0 + 256 * PL <= seg1;
        const int count = whole ? (K + 3) / 4 : K;
        const uint32_t key = order(mx);
        uint32_t kth = 0;
#pragma unroll
        for (int bit = 31; bit >= 16; --bit) {
          const uint32_t trial = kth | (1u << bit);
          if (__popcll(__ballot(key >= trial)) >= count) kth = trial;
        }
        if (lane == 0) l_bound[wave] = static_cast<int>(kth >> 1);  // in 31 bits, for signed comparisons
        __syncthreads();
        const int lo = min(min(l_bound[0], l_bound[1]), min(l_bound[2], l_bound[3]));
        const int hi = max(max(l_bound[0], l_bound[1]), max(l_bound[2], l_bound[3]));
        kth = static_cast<uint32_t>(whole ? lo : hi) << 1;
        if (kth > 0x007fffffu)  // above the order of -inf
          list.floor = __uint_as_float((kth >> 31) ? kth & 0x7fffffffu : ~kth);
        if (list.floor != list.floor) list.floor = -INFINITY;
      }
      // Without a bound, everything above -inf.
      const float least = fmaxf(list.floor, -FLT_MAX);
      const int n0 = list.n;
      bool room = true;
#pragma unroll
      for (int e = 0; e < PL; ++e) {
        const unsigned long long hit = __ballot(x[e] >= least);
        if (hit && room) {
          const Key k = make_key(x[e], at(wave0, e / VN, e % VN));
          const unsigned long long m = __ballot(x[e] >= least && k > list.floor_key);
          room = list.n + __popcll(m) <= kList;
          if (room) append(list, m, k, lane);
        }
      }
      if (!room) {  // clustered values: once more from memory, with the list cut where it is full
        list.n = n0;
        for (int e = 0; e < PL; ++e) {
          const int i = at(wave0, e / VN, e % VN);
          const float v = i < seg1 ? logit<BF16>(p.logits, row0 + i) : -INFINITY;
          const Key k = make_key(v, i);
          push(list, v >= least && k > list.floor_key, k, K, lane);
        }
      }
      // No bound, and fewer than K above -inf so far: tokens of -inf and NaN count too, by index.
      for (int v = 0; list.floor == -INFINITY && v < NV && list.n < K && at(wave0, v, 0) - lane * VN < seg1; ++v)
        for (int j = 0; j < VN; ++j) {
          const int i = at(wave0, v, j);
          const bool none = i < seg1 && !(logit<BF16>(p.logits, row0 + i) > -INFINITY);
          const Key k = make_key(-INFINITY, i);
          push(list, none && k > list.floor_key, k, K, lane);
        }
    }
  }

  st = wave_join(st);
  pad(list, lane);
  if (lane == 0) {
    l_stats[wave] = st;
    l_n[wave] = list.n;
  }
  __syncthreads();
  st = join(join(l_stats[0], l_stats[1]), join(l_stats[2], l_stats[3]));
  const int total = l_n[0] + l_n[1] + l_n[2] + l_n[3];
  if (p.n_segs > 1) {
    const int64_t s = static_cast<int64_t>(row) * p.n_segs + seg;
    if (tid == 0) {
      p.stats[3 * s] = st.m;
      p.stats[3 * s + 1] = st.z;
      p.stats[3 * s + 2] = st.t;
    }
    uint2* const out = p.cand + s * K;
    if (K > 0) {
      best_of(l_key, l_n, K, [&](int r, float v, int i) {
        out[r] = make_uint2(__float_as_uint(v), static_cast<uint32_t>(i));
      });
      if (tid < K && tid >= total) out[tid] = make_uint2(__float_as_uint(-INFINITY), 0xffffffffu);
    }
    return;
  }
  const Finals f = finals(st);
  if (tid == 0) {
    if (p.tokens)
      p.logprobs[row] = tok < 0 ? 0.f : (tok < p.vocab ? log_prob(x_tok, f) : NAN);
    if (p.entropy) p.entropy[row] = f.entropy;
  }
  if (K > 0) {
    const int64_t o = static_cast<int64_t>(row) * K;
    best_of(l_key, l_n, K, [&](int r, float v, int i) {
      p.top[o + r] = i;
      p.top_logprobs[o + r] = log_prob(v, f);
    });
    if (tid < K && tid >= total) {
      p.top[o + tid] = -1;
      p.top_logprobs[o + tid] = -INFINITY;
    }
  }
}

// Joins a row's segments.
template <bool BF16>
__global__ void __launch_bounds__(256)
logprobs_join_kernel(const LogpParams p) {
  __shared__ __attribute__((aligned(16))) Key l_key[4][kList + 8];
  __shared__ int l_n[4];
  __shared__ Stats l_stats[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int row = blockIdx.x, K = p.top_k;
  float x_tok = 0.f;
  int tok = -1;
  if (p.tokens && tid == 0) {
    tok = p.tokens[row];
    if (tok >= 0 && tok < p.vocab) x_tok = logit<BF16>(p.logits, row * p.row_stride + tok);
  }
  Stats st = {-INFINITY, 0.f, 0.f};
  for (int s = tid; s < p.n_segs; s += 256) {
    const float* const x = p.stats + 3 * (static_cast<int64_t>(row) * p.n_segs + s);
    st = join(st, Stats{x[0], x[1], x[2]});
  }
  st = wave_join(st);
  List list = {l_key[wave], 0, -INFINITY, 0};
  const uint2* const cand = p.cand + static_cast<int64_t>(row) * p.n_segs * K;
  for (int c0 = wave * 64; c0 < p.n_segs * K; c0 += 256) {
    const int c = c0 + lane;
    const uint2 e = c < p.n_segs * K ? cand[c] : make_uint2(0u, 0xffffffffu);
    const float v = __uint_as_float(e.x);
    const int i = static_cast<int>(e.y);
    const Key k = make_key(v, i);
    push(list, i >= 0 && k > list.floor_key, k, K, lane);
  }
  pad(list, lane);
  if (lane == 0) {
    l_stats[wave] = st;
    l_n[wave] = list.n;
  }
  __syncthreads();
  const Finals f = finals(join(join(l_stats[0], l_stats[1]), join(l_stats[2], l_stats[3])));
  if (tid == 0) {
    if (p.tokens)
      p.logprobs[row] = tok < 0 ? 0.f : (tok < p.vocab ? log_prob(x_tok, f) : NAN);
    if (p.entropy) p.entropy[row] = f.entropy;
  }
  if (K > 0) {
    const int64_t o = static_cast<int64_t>(row) * K;
    best_of(l_key, l_n, K, [&](int r, float v, int i) {
      p.top[o + r] = i;
      p.top_logprobs[o + r] = log_prob(v, f);
    });
    const int total = l_n[0] + l_n[1] + l_n[2] + l_n[3];
    if (tid < K && tid >= total) {
      p.top[o + tid] = -1;
      p.top_logprobs[o + tid] = -INFINITY;
    }
  }
}

}  // namespace

hipError_t launch_token_logprobs(const LogpParams& p, const LogpPlan& pl, bool bf16, hipStream_t s) {
  const dim3 grid(static_cast<uint32_t>(static_cast<int64_t>(p.rows) * p.n_segs)), block(256);
#define MD_LOGP(BF, PL) hipLaunchKernelGGL((logprobs_kernel<BF, PL>), grid, block, 0, s, p)
  if (pl.per_lane == 32) {
    if (bf16) MD_LOGP(true, 32); else MD_LOGP(false, 32);
  } else {
    if (bf16) MD_LOGP(true, 16); else MD_LOGP(false, 16);
  }
#undef MD_LOGP
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.n_segs == 1) return e;
  if (bf16)
    hipLaunchKernelGGL((logprobs_join_kernel<true>), dim3(static_cast<uint32_t>(p.rows)), block, 0, s, p);
  else
    hipLaunchKernelGGL((logprobs_join_kernel<false>), dim3(static_cast<uint32_t>(p.rows)), block, 0, s, p);
  return hipGetLastError();
}

}  // namespace md
