// spec.hip -- sampled acceptance: drafted tokens kept or refused by the target's
// probabilities, and the token drawn after the kept ones.
//
//   spec_sum   one workgroup per (sequence, chunk of the vocabulary): finds the
//              sequence's accepted count a (a comparison per draft) and sums r =
//              max(p_a - q_a, 0) over its chunk;
//   spec_pick  one workgroup per sequence: finds the chunk, the span of it and the
//              token in which the running sum of r passes u * sum r.
//
// Bound by HBM: the rows p_a and q_a are read once (spec_pick reads one chunk of
// them again, from the caches).  Sums are 64-bit: r is exact there, and a sum's
// error, some 1e-15 of it, is far below the share of a token that 32-bit sums of
// 10^5 terms would misplace.  Every sum has a fixed order.
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

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(256) spec_sum_kernel(const SpecAcceptParams p) {
  constexpr int N = Vec<BF16>::N, U = 4;
  const int b = static_cast<int>(blockIdx.x) / p.n_chunks;
  const int chunk = static_cast<int>(blockIdx.x) % p.n_chunks;
  const int tid = threadIdx.x, lane = tid & 63;
  const int a = accepted_count<BF16>(p, b, lane);
  if (chunk == 0 && tid == 0) p.accepted[b] = a;
  const Residual r = residual(p, b, a);
  const int c0 = chunk * p.chunk_len, c1 = min(p.vocab, c0 + p.chunk_len);
  double sum = 0.0;
  if constexpr (VEC) {
    constexpr int ES = BF16 ? 2 : 4;
    const u32x4* pv = reinterpret_cast<const u32x4*>(static_cast<const char*>(p.p) + r.prow * ES);
    const u32x4* qv =
        reinterpret_cast<const u32x4*>(static_cast<const char*>(p.q) + (r.qrow < 0 ? 0 : r.qrow) * ES);
    const int v0 = c0 / N, v1 = c1 / N;
    for (int v = v0 + tid; v < v1; v += 256 * U) {
      u32x4 x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int vv = v + u * 256 < v1 ? v + u * 256 : v0;  // in bounds, not counted below
        x[u] = pv[vv];
        y[u] = r.qrow >= 0 ? qv[vv] : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        if (v + u * 256 >= v1) continue;
        float fp[N], fq[N];
        Vec<BF16>::get(x[u], fp);
        Vec<BF16>::get(y[u], fq);
#pragma unroll
        for (int j = 0; j < N; ++j) {
          double w = static_cast<double>(fp[j]) - static_cast<double>(fq[j]);
          if ((v + u * 256) * N + j == r.one_at) w -= 1.0;
          sum += w > 0.0 ? w : 0.0;
        }
      }
    }
  } else {
    for (int t = c0 + tid; t < c1; t += 256) sum += weight<BF16>(p, r, t);
  }
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  __shared__ double s[4];
  if (lane == 0) s[tid >> 6] = sum;
  __syncthreads();
  if (tid == 0)
    p.part_sum[static_cast<int64_t>(b) * p.n_chunks + chunk] = (s[0] + s[1]) + (s[2] + s[3]);
}

// Inclusive sum over the workgroup's threads in thread order; `total` its last.
__device__ __forceinline__ double block_scan(double x, double* s, double& total) {
  const int tid = threadIdx.x, lane = tid & 63;
  for (int o = 1; o < 64; o <<= 1) {
    const double y = __shfl_up(x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();
  if (lane == 63) s[tid >> 6] = x;
  __syncthreads();
  double base = 0.0;
  for (int w = 0; w < (tid >> 6); ++w) base += s[w];
  total = ((s[0] + s[1]) + s[2]) + s[3];
  return base + x;
}

// The sum of r over tokens [t0, t1), in order.
template <bool BF16, bool VEC>
__device__ __forceinline__ double span_sum(const SpecAcceptParams& p, const Residual& r, int t0,
                                           int t1) {
  double sum = 0.0;
  if constexpr (VEC) {  // t0 and t1 are multiples of the vector's width
    constexpr int N = Vec<BF16>::N, ES = BF16 ? 2 : 4;
    for (int t = t0; t < t1; t += N) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.p) + (r.prow + t) * ES);
      u32x4 y = {0u, 0u, 0u, 0u};
      if (r.qrow >= 0)
        y = *reinterpret_cast<const u32x4*>(static_cast<const char*>(p.q) + (r.qrow + t) * ES);
      float fp[N], fq[N];
      Vec<BF16>::get(x, fp);
      Vec<BF16>::get(y, fq);
#pragma unroll
      for (int j = 0; j < N; ++j) {
        double w = static_cast<double>(fp[j]) - static_cast<double>(fq[j]);
        if (t + j == r.one_at) w -= 1.0;
        sum += w > 0.0 ? w : 0.0;
      }
    }
  } else {
    for (int t = t0; t < t1; ++t) sum += weight<BF16>(p, r, t);
  }
  return sum;
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(256) spec_pick_kernel(const SpecAcceptParams p) {
  __shared__ double s[4];
  __shared__ double span_before;
  __shared__ int first_span, last_span;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int n = p.n_draft;
  const int a = p.accepted[b];
  Residual r = residual(p, b, a);
  const double* part = p.part_sum + static_cast<int64_t>(b) * p.n_chunks;
  const double u = p.u[static_cast<int64_t>(b) * (n + 1) + n];
  double total = 0.0;
  for (int k = 0; k < p.n_chunks; ++k) total += part[k];
  int c0 = 0, c1 = p.vocab;
  double before = 0.0, want = u * total;
  if (total > 0.0) {
    // The chunk in which the sum passes; the last one with any weight if none.
    int at = -1;
    double run = 0.0;
    for (int k = 0; k < p.n_chunks; ++k) {
      const double w = part[k];
      if (w > 0.0) {
        at = k;
        before = run;
        if (run + w > want) break;
      }
      run += w;
    }
    c0 = at * p.chunk_len;
    c1 = min(p.vocab, c0 + p.chunk_len);
  } else {  // nothing of p_a is above q_a: the target's own row, whole
    r.qrow = -1;
    r.one_at = -1;
  }
  if (tid == 0) {
    first_span = 256;
    last_span = 0;
  }
  // The span of the chunk (consecutive tokens of one thread) in which it passes.
  const int span = ((c1 - c0 + 255) / 256 + 7) / 8 * 8;
  const int t0 = min(c1, c0 + tid * span), t1 = min(c1, t0 + span);
  const double w = span_sum<BF16, VEC>(p, r, t0, t1);
  double sum;
  const double run = before + block_scan(w, s, sum);
  if (!(total > 0.0)) want = u * sum;
  if (w > 0.0) {
    if (run > want) atomicMin(&first_span, tid);
    atomicMax(&last_span, tid);
  }
  __syncthreads();
  const int at = first_span < 256 ? first_span : last_span;
  if (tid == at) span_before = run - w;
  __syncthreads();
  if (tid >= 64) return;
  // Its token, 64 at a time.
  const int s0 = min(c1, c0 + at * span), s1 = min(c1, s0 + span);
  double acc = span_before;
  int tok = -1, last = 0;
  for (int t = s0; t < s1 && tok < 0; t += 64) {
    const double wt = t + lane < s1 ? weight<BF16>(p, r, t + lane) : 0.0;
    double x = wt;
    for (int o = 1; o < 64; o <<= 1) {
      const double y = __shfl_up(x, o);
      if (lane >= o) x += y;
    }
    const unsigned long long pass = __ballot(wt > 0.0 && acc + x > want);
    const unsigned long long some = __ballot(wt > 0.0);
    if (pass) tok = t + __ffsll(static_cast<long long>(pass)) - 1;
    if (some) last = t + 63 - __clzll(static_cast<long long>(some));
    acc += __shfl(x, 63);
  }
  if (tok < 0) tok = last;
  for (int i = tid; i <= n; i += 64)
    p.tokens[static_cast<int64_t>(b) * (n + 1) + i] =
        i < a ? p.draft[static_cast<int64_t>(b) * n + i] : (i == a ? tok : -1);
}

template <bool BF16>
static void launch_spec(const SpecAcceptParams& p, hipStream_t s) {
  const dim3 g(static_cast<uint32_t>(p.B) * static_cast<uint32_t>(p.n_chunks)), blk(256);
  // Whole 16-byte vectors where every row starts on one.
  const bool vec = p.vocab % Vec<BF16>::N == 0 && (reinterpret_cast<uintptr_t>(p.p) & 15u) == 0 &&
                   (reinterpret_cast<uintptr_t>(p.q) & 15u) == 0;
  if (vec) {
    hipLaunchKernelGGL((spec_sum_kernel<BF16, true>), g, blk, 0, s, p);
    hipLaunchKernelGGL((spec_pick_kernel<BF16, true>), dim3(p.B), blk, 0, s, p);
  } else {
    hipLaunchKernelGGL((spec_sum_kernel<BF16, false>), g, blk, 0, s, p);
    hipLaunchKernelGGL((spec_pick_kernel<BF16, false>), dim3(p.B), blk, 0, s, p);
  }
}

hipError_t launch_spec_accept(const SpecAcceptParams& p, bool bf16, hipStream_t s) {
  if (bf16)
    launch_spec<true>(p, s);
  else
    launch_spec<false>(p, s);
  return hipGetLastError();
}

}  // namespace md
