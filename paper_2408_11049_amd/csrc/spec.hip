// spec.hip -- sampled acceptance: drafted tokens kept or refused by the target's
// probabilities, and the token drawn after the kept ones.
//
// The row is cut into segments, a wave each.  A wave finds the sequence's accepted count
// a (a comparison per draft) and sums r = max(p_a - q_a, 0) over its segments; then one
// wave finds the segment, the span of it and the token in which the running sum of r
// passes u * sum r.
//
//   spec_fused  one workgroup per sequence does both, the segment sums in LDS;
//   spec_sum, spec_pick  the same in two launches, the segments over many workgroups.
//
// Bound by HBM where many rows are long: p_a and q_a are read once (the search reads one
// segment of them again, from the caches); otherwise by the chain of loads, each of which needs
// the one before: the drafts, their probabilities, the row, the segment.  64 sequences of
// 128256 tokens in fp32: 13.3 us for 66 MB (4.9 TB/s; the first two loads of the chain are some
// 3 us of it) and 4.0 us for the search.  One sequence of 32000 in one launch: 8.5 us.
// Where nothing of p_a is above q_a, which equal rows alone give, the one wave that searches reads
// the whole row: 132 us for those 64 sequences, 30 for 32000 tokens.
// Loads are of 16 bytes wherever a row starts: element by element 64 rows of 50257 took 21.9 us
// a call, so 14.5.
// Lanes exchange by DPP moves; with LDS shuffles the search took 4.6 us.
// Sums are 64-bit: r is exact there, and a sum's error, some 1e-15 of it, is far below the
// share of a token that 32-bit sums of 10^5 terms would misplace.  Every sum has a fixed order.
#include "kv4.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// A probability as the formulas take it: 0 where negative, NaN or infinite.
__device__ __forceinline__ float prob(float x) { return x > 0.f && x < INFINITY ? x : 0.f; }

template <bool BF16>
__device__ __forceinline__ float load_prob(const void* base, int64_t e) {
  if constexpr (BF16)
    return prob(__uint_as_float(static_cast<uint32_t>(static_cast<const uint16_t*>(base)[e]) << 16));
  return prob(static_cast<const float*>(base)[e]);
}

template <bool BF16>
struct Vec {  // 16 bytes of probabilities
  static constexpr int N = BF16 ? 8 : 4;
  // Rows begin where the vocabulary puts them: any element's address will do for a load.
  static __device__ __forceinline__ u32x4 load(const void* base, int64_t e) {
    typedef u32x4 at2 __attribute__((aligned(2)));
    typedef u32x4 at4 __attribute__((aligned(4)));
    if constexpr (BF16) return *reinterpret_cast<const at2*>(static_cast<const uint16_t*>(base) + e);
    return *reinterpret_cast<const at4*>(static_cast<const float*>(base) + e);
  }
  static __device__ __forceinline__ void get(const u32x4& w, float (&x)[N]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if constexpr (BF16) {
        x[2 * j] = prob(__uint_as_float(w[j] << 16));
        x[2 * j + 1] = prob(__uint_as_float(w[j] & 0xffff0000u));
      } else {
        x[j] = prob(__uint_as_float(w[j]));
      }
    }
  }
};

// The accepted count of sequence b, found by the whole wave (64 drafts at a time).
template <bool BF16>
__device__ __forceinline__ int accepted_count(const SpecAcceptParams& p, int b, int lane) {
  const int n = p.n_draft;
  for (int i0 = 0; i0 < n; i0 += 64) {
    const int i = i0 + lane;
    bool ok = true;
    if (i < n) {
      const int d = p.draft[static_cast<int64_t>(b) * n + i];
      const float u = p.u[static_cast<int64_t>(b) * (n + 1) + i];
      ok = d >= 0 && d < p.vocab;
      if (ok) {
        const double pt = load_prob<BF16>(p.p, (static_cast<int64_t>(b) * (n + 1) + i) * p.vocab + d);
        const double qd =
            p.q ? load_prob<BF16>(p.q, (static_cast<int64_t>(b) * n + i) * p.vocab + d) : 1.f;
        ok = static_cast<double>(u) * qd < pt;  // exact: two 24-bit factors
      }
    }
    const unsigned long long miss = __ballot(!ok);
    if (miss) return i0 + __ffsll(static_cast<long long>(miss)) - 1;
  }
  return n;
}

// r of one sequence: p_a, less q_a (or 1 at the refused draft).
struct Residual {
  int64_t prow, qrow;  // element offsets; qrow < 0: no draft row
  int one_at;          // token with q = 1, or -1
};
__device__ __forceinline__ Residual residual(const SpecAcceptParams& p, int b, int a) {
  Residual r;
  r.prow = (static_cast<int64_t>(b) * (p.n_draft + 1) + a) * p.vocab;
  r.qrow = a < p.n_draft && p.q ? (static_cast<int64_t>(b) * p.n_draft + a) * p.vocab : -1;
  r.one_at = a < p.n_draft && !p.q ? p.draft[static_cast<int64_t>(b) * p.n_draft + a] : -1;
  return r;
}
template <bool BF16>
__device__ __forceinline__ double weight(const SpecAcceptParams& p, const Residual& r, int t) {
  double w = load_prob<BF16>(p.p, r.prow + t);
  if (r.qrow >= 0) w -= load_prob<BF16>(p.q, r.qrow + t);
  if (t == r.one_at) w -= 1.0;
  return w > 0.0 ? w : 0.0;
}

// The sum of r over one vector of each row (zeros for no draft row), tokens t ..
template <bool BF16>
__device__ __forceinline__ double vec_sum(const u32x4& x, const u32x4& y, int t, int one_at) {
  constexpr int N = Vec<BF16>::N;
  float fp[N], fq[N];
  Vec<BF16>::get(x, fp);
  Vec<BF16>::get(y, fq);
  double sum = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    double w = static_cast<double>(fp[j]) - static_cast<double>(fq[j]);
    if (t + j == one_at) w -= 1.0;
    sum += w > 0.0 ? w : 0.0;
  }
  return sum;
}

// One step of the wave's scans and broadcasts: no LDS exchange, no latency to wait for.
template <int CTRL, int ROWS>
__device__ __forceinline__ double dpp(double x) {  // zeros where there is no such lane
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, static_cast<int>(b), CTRL, ROWS, 0xf, false);
  const uint32_t hi = __builtin_amdgcn_update_dpp(0, static_cast<int>(b >> 32), CTRL, ROWS, 0xf, false);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ double lane_value(double x, int lane) {  // lane: uniform
  const uint64_t b = __builtin_bit_cast(uint64_t, x);
  const uint32_t lo = __builtin_amdgcn_readlane(static_cast<int>(b), lane);
  const uint32_t hi = __builtin_amdgcn_readlane(static_cast<int>(b >> 32), lane);
  return __builtin_bit_cast(double, static_cast<uint64_t>(hi) << 32 | lo);
}
// Inclusive sums over the lanes: within rows of 16, then over the rows.
__device__ __forceinline__ double wave_scan(double x) {
  x += dpp<0x111, 0xf>(x);  // from 1, 2, 4, 8 lanes below in the row
  x += dpp<0x112, 0xf>(x);
  x += dpp<0x114, 0xf>(x);
  x += dpp<0x118, 0xf>(x);
  x += dpp<0x142, 0xa>(x);  // rows 1 and 3: the last lane of the row before
  x += dpp<0x143, 0xc>(x);  // rows 2 and 3: lane 31
  return x;
}
__device__ __forceinline__ double wave_sum(double x) { return lane_value(wave_scan(x), 63); }

// Segment `seg` by one wave: its loads, then (every lane gets it) the sum of r.
template <bool BF16>
struct SegVecs {
  static constexpr int U = BF16 ? 2 : 4;  // a segment of 1024 tokens
  u32x4 x[U], y[U];
};
template <bool BF16>
__device__ __forceinline__ void load_vecs(const SpecAcceptParams& p, const Residual& r, int t, int t1,
                                          SegVecs<BF16>& v) {
  constexpr int N = Vec<BF16>::N;
#pragma unroll
  for (int u = 0; u < v.U; ++u) {
    const int at = t + u * 64 * N;
    v.x[u] = v.y[u] = u32x4{0u, 0u, 0u, 0u};
    if (at + N <= t1) {
      v.x[u] = Vec<BF16>::load(p.p, r.prow + at);
      if (r.qrow >= 0) v.y[u] = Vec<BF16>::load(p.q, r.qrow + at);
    }
  }
}
template <bool BF16>
__device__ __forceinline__ double sum_vecs(const Residual& r, int t, const SegVecs<BF16>& v) {
  double sum = 0.0;
#pragma unroll
  for (int u = 0; u < v.U; ++u)  // what is behind the end is 0
    sum += vec_sum<BF16>(v.x[u], v.y[u], t + u * 64 * Vec<BF16>::N, r.one_at);
  return sum;
}
// Segments seg and seg + next (that one: where there is one): both are loaded before either is
// summed.
template <bool BF16>
__device__ __forceinline__ void segment_sums(const SpecAcceptParams& p, const Residual& r, int seg,
                                             int next, int lane, double* out) {
  constexpr int N = Vec<BF16>::N, kStep = 64 * N * SegVecs<BF16>::U;
  const bool two = seg + next < p.n_segs;
  double sum[2] = {0.0, 0.0};
  for (int c = 0; c < p.seg_len; c += kStep) {
    SegVecs<BF16> v[2];
    int t[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int s0 = (k && two ? seg + next : seg) * p.seg_len;
      t[k] = s0 + c + lane * N;
      if (k == 0 || two) load_vecs<BF16>(p, r, t[k], min(p.vocab, s0 + p.seg_len), v[k]);
    }
    sum[0] += sum_vecs<BF16>(r, t[0], v[0]);
    if (two) sum[1] += sum_vecs<BF16>(r, t[1], v[1]);
  }
  // What is behind the row's last whole vector, in its last segment.
  const int rest = p.vocab - p.vocab % N + lane;
  if (rest < p.vocab) {
    const double w = weight<BF16>(p, r, rest);
    if (seg == p.n_segs - 1) sum[0] += w;
    if (seg + next == p.n_segs - 1) sum[1] += w;
  }
  const double a = wave_sum(sum[0]), b = wave_sum(sum[1]);
  if (lane == 0) {
    out[seg] = a;
    if (two) out[seg + next] = b;
  }
}

// Where a running sum that starts at `before` passes `want`: the first lane, in order, whose
// own weight w > 0 brings it past, else the last lane with any weight (-1: none has).
// before becomes the sum ahead of that lane; `all`: only a lane that passes counts, and without
// one before becomes the whole sum.
__device__ __forceinline__ int find_lane(double w, double want, bool all, double& before) {
  const double incl = before + wave_scan(w);
  const unsigned long long some = __ballot(w > 0.0), pass = __ballot(w > 0.0 && incl > want);
  if (!pass && (all || !some)) {
    before = lane_value(incl, 63);
    return -1;
  }
  const int at = pass ? __ffsll(static_cast<long long>(pass)) - 1
                      : 63 - __clzll(static_cast<long long>(some));
  if (at) before = lane_value(incl, at - 1);
  return at;
}

// The drawn token, by one wave; sums: the segments' (LDS or global).
template <bool BF16>
__device__ int draw_token(const SpecAcceptParams& p, int b, Residual r, const double* sums, int lane) {
  const double u = p.u[static_cast<int64_t>(b) * (p.n_draft + 1) + p.n_draft];
  // A lane takes `per` consecutive segments.
  const int per = (p.n_segs + 63) / 64;
  const int s0 = min(p.n_segs, lane * per), s1 = min(p.n_segs, s0 + per);
  double mine = 0.0;
  for (int k = s0; k < s1; ++k) mine += sums[k];
  const double total = wave_sum(mine);
  int c0 = 0, c1 = p.vocab;  // the tokens in which it is
  double before = 0.0, want = u * total;
  if (total > 0.0) {
    const int at = find_lane(mine, want, false, before);
    int seg = -1, last = 0;
    double run = before;
    for (int k = min(p.n_segs, at * per); k < min(p.n_segs, (at + 1) * per); ++k) {
      const double w = sums[k];
      if (w > 0.0) {
        last = k;
        before = run;
        if (run + w > want) {
          seg = k;
          break;
        }
      }
      run += w;
    }
    if (seg < 0) seg = last;
    c0 = seg * p.seg_len;
    c1 = min(p.vocab, c0 + p.seg_len);
  } else {  // nothing of p_a is above q_a: the target's own row, whole
    r.qrow = -1;
    r.one_at = -1;
  }
  // The span of them, consecutive tokens of a lane.
  constexpr int kSpan = 16;  // tokens a lane can hold
  const int span = ((c1 - c0 + 63) / 64 + 7) / 8 * 8;
  const int t0 = min(c1, c0 + lane * span), t1 = min(c1, t0 + span);
  if (total > 0.0 && span <= kSpan) {  // every segment of rows up to 2^20 tokens
    float fp[kSpan], fq[kSpan];
    if (t0 + kSpan <= t1) {
      constexpr int N = Vec<BF16>::N;
#pragma unroll
      for (int j = 0; j < kSpan; j += N) {
        const u32x4 x = Vec<BF16>::load(p.p, r.prow + t0 + j);
        u32x4 y = {0u, 0u, 0u, 0u};
        if (r.qrow >= 0) y = Vec<BF16>::load(p.q, r.qrow + t0 + j);
        float a[N], c[N];
        Vec<BF16>::get(x, a);
        Vec<BF16>::get(y, c);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          fp[j + k] = a[k];
          fq[j + k] = c[k];
        }
      }
    } else {
#pragma unroll
      for (int j = 0; j < kSpan; ++j) {
        const bool in = t0 + j < t1;
        fp[j] = in ? load_prob<BF16>(p.p, r.prow + t0 + j) : 0.f;
        fq[j] = in && r.qrow >= 0 ? load_prob<BF16>(p.q, r.qrow + t0 + j) : 0.f;
      }
    }
    auto held = [&](int j) {
      double w = static_cast<double>(fp[j]) - static_cast<double>(fq[j]);
      if (t0 + j == r.one_at) w -= 1.0;
      return w > 0.0 ? w : 0.0;
    };
    double w = 0.0;
#pragma unroll
    for (int j = 0; j < kSpan; ++j) w += held(j);
    const int at = find_lane(w, want, false, before);
    // Each lane looks among its own as if it were that one.
    int past = -1, last = 0;
    double run = before;
#pragma unroll
    for (int j = 0; j < kSpan; ++j) {
      const double x = held(j);
      run += x;
      if (x > 0.0) {
        last = j;
        if (past < 0 && run > want) past = j;
      }
    }
    return __builtin_amdgcn_readlane(t0 + (past >= 0 ? past : last), at);
  }
  double w = 0.0;
  {
    constexpr int N = Vec<BF16>::N;
    int t = t0;
#pragma unroll 4
    for (; t + N <= t1; t += N) {
      const u32x4 x = Vec<BF16>::load(p.p, r.prow + t);
      u32x4 y = {0u, 0u, 0u, 0u};
      if (r.qrow >= 0) y = Vec<BF16>::load(p.q, r.qrow + t);
      w += vec_sum<BF16>(x, y, t, r.one_at);
    }
    for (; t < t1; ++t) w += weight<BF16>(p, r, t);
  }
  if (!(total > 0.0)) want = u * wave_sum(w);
  const int at = find_lane(w, want, false, before);
  if (at < 0) return 0;  // p_a is all 0
  // The token, 64 at a time.
  const int e0 = c0 + at * span, e1 = min(c1, e0 + span);
  int tok = 0;
  for (int t = e0; t < e1; t += 64) {
    const double wt = t + lane < e1 ? weight<BF16>(p, r, t + lane) : 0.0;
    const unsigned long long some = __ballot(wt > 0.0);
    if (some) tok = t + 63 - __clzll(static_cast<long long>(some));
    const int found = find_lane(wt, want, true, before);
    if (found >= 0) return t + found;
  }
  return tok;
}

__device__ __forceinline__ void store_tokens(const SpecAcceptParams& p, int b, int a, int tok, int lane) {
  const int n = p.n_draft;
  for (int i = lane; i <= n; i += 64)
    p.tokens[static_cast<int64_t>(b) * (n + 1) + i] =
        i < a ? p.draft[static_cast<int64_t>(b) * n + i] : (i == a ? tok : -1);
}

template <bool BF16>
__global__ void __launch_bounds__(256) spec_sum_kernel(const SpecAcceptParams p) {
  const int b = static_cast<int>(blockIdx.x) / p.wgs;
  const int lane = threadIdx.x & 63;
  const int first = static_cast<int>(blockIdx.x) % p.wgs * 4 + (static_cast<int>(threadIdx.x) >> 6);
  const int a = accepted_count<BF16>(p, b, lane);
  if (first == 0 && lane == 0) p.accepted[b] = a;
  const Residual r = residual(p, b, a);
  for (int seg = first; seg < p.n_segs; seg += 8 * p.wgs)
    segment_sums<BF16>(p, r, seg, 4 * p.wgs, lane,
                            p.seg_sum + static_cast<int64_t>(b) * p.n_segs);
}

template <bool BF16>
__global__ void __launch_bounds__(64) spec_pick_kernel(const SpecAcceptParams p) {
  const int b = blockIdx.x, lane = threadIdx.x;
  const int a = p.accepted[b];
  const int tok = draw_token<BF16>(p, b, residual(p, b, a),
                                        p.seg_sum + static_cast<int64_t>(b) * p.n_segs, lane);
  store_tokens(p, b, a, tok, lane);
}

template <bool BF16>
__global__ void __launch_bounds__(1024) spec_fused_kernel(const SpecAcceptParams p) {
  __shared__ double sums[kSpecMaxSegs];
  const int b = blockIdx.x, lane = threadIdx.x & 63;
  const int wave = static_cast<int>(threadIdx.x) >> 6;
  const int a = accepted_count<BF16>(p, b, lane);
  const Residual r = residual(p, b, a);
  for (int seg = wave; seg < p.n_segs; seg += 32)
    segment_sums<BF16>(p, r, seg, 16, lane, sums);
  __syncthreads();
  if (wave != 0) return;
  if (lane == 0) p.accepted[b] = a;
  store_tokens(p, b, a, draw_token<BF16>(p, b, r, sums, lane), lane);
}

template <bool BF16>
static void launch_spec(const SpecAcceptParams& p, hipStream_t s) {
  if (p.wgs == 0) {
    hipLaunchKernelGGL((spec_fused_kernel<BF16>), dim3(p.B), dim3(1024), 0, s, p);
    return;
  }
  const dim3 g(static_cast<uint32_t>(p.B) * static_cast<uint32_t>(p.wgs));
  hipLaunchKernelGGL((spec_sum_kernel<BF16>), g, dim3(256), 0, s, p);
  hipLaunchKernelGGL((spec_pick_kernel<BF16>), dim3(p.B), dim3(64), 0, s, p);
}

hipError_t launch_spec_accept(const SpecAcceptParams& p, bool bf16, hipStream_t s) {
  if (bf16) launch_spec<true>(p, s);
  else launch_spec<false>(p, s);
  return hipGetLastError();
}

}  // namespace md
