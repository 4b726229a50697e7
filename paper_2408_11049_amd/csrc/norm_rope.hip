// norm_rope.hip -- RMS norm of query and key heads and the rotation by position, with
// the new K and V rows written into the cache in the same pass.
//
//   y = x / sqrt(mean x^2 + eps) * w;  (y1, y2) -> (y1 cos t - y2 sin t, y2 cos t + y1 sin t)
//
// Bound by HBM for prompts, by latency for a step: every row is read once and written
// once.  A row of d channels is d / 8 threads of 8 channels (16 bytes of bf16), so its
// sum of squares is reduced over 8 or 16 neighbouring lanes and a pair's other half is
// one lane exchange away.  A workgroup takes one token: the rot / 2 angles are turned
// into cosines and sines once (64-bit product and reduction, so far positions keep
// their fraction of a turn) and serve all the token's heads from LDS.
//
// What keeps the memory busy is many small workgroups, each with two passes' rows loaded and
// the next two under way: 4 x 4096 tokens of 32 + 8 heads of 128 in bf16 78 us, 5.2 TB/s read
// and written (a large copy: 4.9).  Against that, on one card: one pass at a time 97 to 93, three
// 98, four tokens a workgroup 104, no rows ahead 100.  A step of 64 x 5 tokens takes 6.1 us, of
// which the bytes would need 1.6.
#include "kv4.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

namespace {

template <bool BF16>
struct Raw {  // 8 channels as stored
  u32x4 w[BF16 ? 1 : 2];
};

template <bool BF16>
__device__ __forceinline__ Raw<BF16> load_raw(const void* base, int64_t e) {
  Raw<BF16> r;
  const u32x4* p = reinterpret_cast<const u32x4*>(static_cast<const char*>(base) + e * (BF16 ? 2 : 4));
  r.w[0] = p[0];
  if constexpr (!BF16) r.w[1] = p[1];
  return r;
}

template <bool BF16>
__device__ __forceinline__ void store_raw(void* base, int64_t e, const Raw<BF16>& r) {
  u32x4* p = reinterpret_cast<u32x4*>(static_cast<char*>(base) + e * (BF16 ? 2 : 4));
  __builtin_nontemporal_store(r.w[0], p);
  if constexpr (!BF16) __builtin_nontemporal_store(r.w[1], p + 1);
}

template <bool BF16>
__device__ __forceinline__ void widen(const Raw<BF16>& r, float (&x)[8]) {
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) {
      x[2 * j] = __uint_as_float(r.w[0][j] << 16);
      x[2 * j + 1] = __uint_as_float(r.w[0][j] & 0xffff0000u);
    } else {
      x[j] = __uint_as_float(r.w[0][j]);
      x[4 + j] = __uint_as_float(r.w[1][j]);
    }
  }
}

template <bool BF16>
__device__ __forceinline__ Raw<BF16> narrow(const float (&x)[8]) {
  Raw<BF16> r;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    if constexpr (BF16) {
      r.w[0][j] = __builtin_bit_cast(
          uint32_t, __builtin_convertvector(f32x2{x[2 * j], x[2 * j + 1]}, bf16x2));
    } else {
      r.w[0][j] = __float_as_uint(x[j]);
      r.w[1][j] = __float_as_uint(x[4 + j]);
    }
  }
  return r;
}

constexpr int64_t kTokensX = kMaxWgs256 / 2;

// Where a token is: its sequence, its place in it, its position.
struct At {
  int token, b, i;
  int64_t pos;
};
__device__ __forceinline__ At at_token(const NormRopeParams& p, int token) {
  At t;
  t.token = token;
  t.b = token / p.n;
  t.i = token - t.b * p.n;
  t.pos = static_cast<int64_t>(p.pos0[t.b]) + t.i;
  return t;
}
// Element offset of the token's rows in the cache, -1: not in it.
__device__ __forceinline__ int64_t cache_offset(const NormRopeParams& p, const At& t) {
  if (!p.has_cache || t.pos < 0) return -1;
  if (!p.paged) return t.pos < p.c.capacity ? t.b * p.c.s_blk + t.pos * p.c.s_tok : -1;
  const int64_t pg = t.pos >> p.c.page_shift;
  if (pg >= p.c.max_pages) return -1;
  const int64_t id = p.c.page_table[static_cast<int64_t>(t.b) * p.c.max_pages + pg];
  if (id < 0 || id >= p.c.num_pages) return -1;
  return id * p.c.s_blk + (t.pos & ((int64_t{1} << p.c.page_shift) - 1)) * p.c.s_tok;
}

// Row `row` of a token: Hq query heads, Hkv key heads, then (with a cache) Hkv value heads.
// A workgroup takes one token (blockIdx.x, blockIdx.z) and its share of the passes over its rows.
template <int D, bool BF16>
__global__ void __launch_bounds__(256) qk_norm_rope_kernel(const NormRopeParams p) {
  constexpr int LPR = D / 8;       // threads a row
  constexpr int RPP = 256 / LPR;   // rows a pass
  constexpr int U = 2;             // passes whose loads are in flight together
  __shared__ float cs[D / 2], sn[D / 2];
  const int tid = threadIdx.x;
  const int c = tid % LPR, rr = tid / LPR;
  const uint32_t token = blockIdx.x + blockIdx.z * gridDim.x;
  if (token >= static_cast<uint32_t>(p.B * p.n)) return;  // the whole workgroup
  const int rows = p.Hq + p.Hkv * (p.has_cache ? 2 : 1);
  const At here = at_token(p, static_cast<int>(token));
  const int first = static_cast<int>(blockIdx.y) * RPP;
  const int step = static_cast<int>(gridDim.y) * RPP;

  // Whatever does not depend on another load comes first.
  auto load = [&](Raw<BF16> (&raw)[U], int r0) {
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = r0 + u * step + rr;
      if (row >= rows) continue;
      const int64_t b = here.b, i = here.i;
      const bool is_q = row < p.Hq, is_k = !is_q && row < p.Hq + p.Hkv;
      const void* src = is_q ? p.q : (is_k ? p.k : p.v);
      const int64_t at = is_q ? b * p.q_seq + i * p.q_tok + static_cast<int64_t>(row) * D
                         : is_k ? b * p.k_seq + i * p.k_tok + static_cast<int64_t>(row - p.Hq) * D
                                : b * p.v_seq + i * p.v_tok +
                                      static_cast<int64_t>(row - p.Hq - p.Hkv) * D;
      raw[u] = load_raw<BF16>(src, at + c * 8);
    }
  };
  Raw<BF16> raw[U];
  load(raw, first);
  Raw<BF16> wq, wk;
  if (p.q_weight) wq = load_raw<BF16>(p.q_weight, c * 8);
  if (p.k_weight) wk = load_raw<BF16>(p.k_weight, c * 8);
  const float freq = tid < p.rot / 2 ? p.inv_freq[tid] : 0.f;
  const int64_t cache_at = cache_offset(p, here);

  if (tid < p.rot / 2) {  // an angle a thread
    constexpr double kInv2Pi = 0.15915494309189533577;
    constexpr double k2PiHi = 6.283185307179586232, k2PiLo = 2.4492935982947064e-16;
    const double t = static_cast<double>(here.pos) * static_cast<double>(freq);
    const double n = rint(t * kInv2Pi);
    const float f = static_cast<float>(fma(-n, k2PiLo, fma(-n, k2PiHi, t)));
    sincosf(f, &sn[tid], &cs[tid]);
  }
  if (here.i == 0 && tid == 0 && blockIdx.y == 0 && p.lens_out)
    p.lens_out[here.b] = static_cast<int32_t>(here.pos + p.n);
  __syncthreads();

  for (int r0 = first; r0 < rows; r0 += U * step) {
    Raw<BF16> raw_next[U];
    load(raw_next, r0 + U * step);  // none behind the last row
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int row = r0 + u * step + rr;
      if (r0 + u * step >= rows) break;  // uniform: the lanes of a row exchange values below
      const bool live = row < rows;
      const bool is_q = row < p.Hq, is_k = !is_q && row < p.Hq + p.Hkv;
      const int head = is_q ? row : (is_k ? row - p.Hq : row - p.Hq - p.Hkv);
      float x[8];
      if (live) {
        widen<BF16>(raw[u], x);
      } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = 0.f;
      }
      if (p.norm) {
        float ss = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss += x[j] * x[j];
        for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
        const float rs = 1.0f / sqrtf(ss * (1.0f / D) + p.eps);
        float wt[8];
        if (is_q ? p.q_weight != nullptr : p.k_weight != nullptr) {
          widen<BF16>(is_q ? wq : wk, wt);
        } else {
#pragma unroll
          for (int j = 0; j < 8; ++j) wt[j] = 1.f;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = x[j] * rs * wt[j];
      }
      if (p.interleaved) {
        if (c * 8 < p.rot) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const float co = cs[c * 4 + j], si = sn[c * 4 + j];
            const float y1 = x[2 * j], y2 = x[2 * j + 1];
            x[2 * j] = y1 * co - y2 * si;
            x[2 * j + 1] = y2 * co + y1 * si;
          }
        }
      } else {
        const int half = p.rot / 16;  // threads a half of the turned channels takes
        const int lane = tid & 63;
        const bool lo = c < half, hi = !lo && c < 2 * half;
        const int other = lo ? lane + half : (hi ? lane - half : lane);
        const int j0 = (lo ? c : c - half) * 8;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float y = __shfl(x[j], other);
          if (lo || hi) {
            const float co = cs[j0 + j], si = sn[j0 + j];
            x[j] = lo ? x[j] * co - y * si : x[j] * co + y * si;
          }
        }
      }
      if (!live) continue;
      if (is_q) {
        store_raw<BF16>(p.q_out, (static_cast<int64_t>(here.token) * p.Hq + head) * D + c * 8,
                        narrow<BF16>(x));
        continue;
      }
      // A value row moves as it is.
      const Raw<BF16> out = is_k ? narrow<BF16>(x) : raw[u];
      if (is_k && p.k_out)
        store_raw<BF16>(p.k_out, (static_cast<int64_t>(here.token) * p.Hkv + head) * D + c * 8, out);
      if (cache_at >= 0)
        store_raw<BF16>(is_k ? p.c.k : p.c.v, cache_at + head * p.c.s_head + c * 8, out);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) raw[u] = raw_next[u];
  }
}

template <int D, bool BF16>
void launch_norm(const NormRopeParams& p, hipStream_t s) {
  const int64_t tokens = static_cast<int64_t>(p.B) * p.n;
  const int rows = p.Hq + p.Hkv * (p.has_cache ? 2 : 1);
  const int rpp = 256 / (D / 8), passes = (rows + rpp - 1) / rpp;
  // Few tokens: a workgroup for each pass of a token's rows instead of one for all.
  const int split = static_cast<int>(tokens <= 4 * device_cu_count() ? passes : 1);
  // Tokens over x and, past the threads that one dimension counts, z.
  const int64_t layers = (tokens + kTokensX - 1) / kTokensX;
  const dim3 g(static_cast<uint32_t>((tokens + layers - 1) / layers),
               static_cast<uint32_t>(split), static_cast<uint32_t>(layers));
  hipLaunchKernelGGL((qk_norm_rope_kernel<D, BF16>), g, dim3(256), 0, s, p);
}

}  // namespace

hipError_t launch_qk_norm_rope(const NormRopeParams& p, int head_dim, bool bf16, hipStream_t s) {
  if (head_dim == 128) {
    if (bf16) launch_norm<128, true>(p, s);
    else launch_norm<128, false>(p, s);
  } else {
    if (bf16) launch_norm<64, true>(p, s);
    else launch_norm<64, false>(p, s);
  }
  return hipGetLastError();
}

}  // namespace md
