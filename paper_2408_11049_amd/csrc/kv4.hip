// kv4.hip -- rows into and out of the 4-bit KV cache.
//
//   kv4_append  per 32 channels: a = max |x|, scale 2^e, codes round(x / 2^e);
//   kv4_read    code * 2^e.
//
// Both are bound by HBM (append reads 256 B a bf16 row of 128 channels and writes
// 68).  A thread takes 8 channels of the K row and of the V row -- one 16-byte bf16
// vector each, so a wave reads whole rows, and one dword of codes each -- and
// four neighbouring threads find their block's maximum in two lane swaps.  Rows go
// (sequence, head, token): neighbouring rows of a [block][head][token] cache are
// then written side by side, whole lines by one workgroup.  8 x 4096 tokens of 8 heads of 128,
// bf16: append 32 us, read 28 us, 170 MB each (a large copy would take 35).  A step of 64 x 5
// tokens takes 3.4 and 5.7 us, a launch and one or two dependent loads.
#include "kv4.h"

namespace md {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

// 8 channels from 8 * c on, widened to fp32 (exact).
template <bool BF16>
__device__ __forceinline__ void load8(const void* base, int64_t e, float (&x)[8]) {
  if constexpr (BF16) {
    const u32x4 w = __builtin_nontemporal_load(
        reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(base) + e));
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[2 * j] = __uint_as_float(w[j] << 16);
      x[2 * j + 1] = __uint_as_float(w[j] & 0xffff0000u);
    }
  } else {
    const f32x4* p = reinterpret_cast<const f32x4*>(static_cast<const float*>(base) + e);
    const f32x4 a = __builtin_nontemporal_load(p), b = __builtin_nontemporal_load(p + 1);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      x[j] = a[j];
      x[4 + j] = b[j];
    }
  }
}

// The codes of 8 channels and their block's scale byte.  v_cvt_scalef32_pk_fp4_f32
// divides by the scale, rounds to nearest even and saturates at 6, exactly the
// format's rounding (its quotients are exact: powers of two).
__device__ __forceinline__ uint32_t quantise8(const float (&x)[8], int& scale_byte) {
  uint32_t m = 0;  // |x| as integers: the order of non-negative floats, NaN above infinity
#pragma unroll
  for (int j = 0; j < 8; ++j) m = max(m, __float_as_uint(x[j]) & 0x7fffffffu);
  m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 1)));
  m = max(m, static_cast<uint32_t>(__shfl_xor(static_cast<int>(m), 2)));
  // floor(log2(8 a / 7)): one more than a's exponent from a mantissa of 1.75 on.
  const int e = min(max(static_cast<int>((m + 0x00200000u) >> 23) - 127 - 2, -125), 125);
  const bool bad = m >= 0x7f800000u;
  scale_byte = bad ? 255 : e + 127;
  const float s = __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
  uint32_t r = 0;
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[0], x[1], s, 0);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[2], x[3], s, 1);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[4], x[5], s, 2);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(r, x[6], x[7], s, 3);
  return bad ? 0u : r;
}

// Byte offset of position j of sequence b and head hk in the code arrays, or false
// where the cache has no such row.
template <bool PAGED>
__device__ __forceinline__ bool kv4_row(const Kv4View& c, int b, int hk, int64_t j, int64_t& off) {
  if (j < 0) return false;
  int64_t blk, tok;
  if (PAGED) {
    const int64_t pg = j >> c.page_shift;
    if (pg >= c.max_pages) return false;
    blk = c.page_table[static_cast<int64_t>(b) * c.max_pages + pg];
    if (blk < 0 || blk >= c.num_pages) return false;
    tok = j & ((int64_t{1} << c.page_shift) - 1);
  } else {
    if (j >= c.capacity) return false;
    blk = b;
    tok = j;
  }
  off = blk * c.s_blk + tok * c.s_tok + hk * c.s_head;
  return true;
}

struct RowAt {
  int b, hk, i;
};
__device__ __forceinline__ RowAt row_at(const Kv4RowsParams& p, uint32_t r) {
  const uint32_t n = static_cast<uint32_t>(p.n), h = static_cast<uint32_t>(p.Hkv);
  const uint32_t u = r / n, b = u / h;
  return RowAt{static_cast<int>(b), static_cast<int>(u - b * h), static_cast<int>(r - u * n)};
}

template <int D, bool BF16, bool PAGED>
__global__ void __launch_bounds__(256) kv4_append_kernel(const Kv4RowsParams p) {
  constexpr int LPR = D / 8;  // threads a row
  const int c = threadIdx.x % LPR;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (256 / LPR);
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * (256 / LPR) + threadIdx.x / LPR; r < p.rows;
       r += step) {
    const RowAt a = row_at(p, static_cast<uint32_t>(r));
    const int64_t src =
        ((static_cast<int64_t>(a.b) * p.n + a.i) * p.Hkv + a.hk) * D + c * 8;
    float xk[8], xv[8];
    load8<BF16>(p.k_rows, src, xk);
    load8<BF16>(p.v_rows, src, xv);
    const int32_t base = p.pos0[a.b];
    if (a.hk == 0 && a.i == 0 && c == 0 && p.lens_out) p.lens_out[a.b] = base + p.n;
    int64_t off = 0;
    const bool in = kv4_row<PAGED>(p.c, a.b, a.hk, static_cast<int64_t>(base) + a.i, off);
    int sk, sv;  // all four threads of a block take part in its maximum
    const uint32_t ck = quantise8(xk, sk), cv = quantise8(xv, sv);
    if (!in) continue;
    *reinterpret_cast<uint32_t*>(p.c.k + off + c * 4) = ck;
    *reinterpret_cast<uint32_t*>(p.c.v + off + c * 4) = cv;
    if ((c & 3) == 0) {
      p.c.ks[off / 16 + c / 4] = static_cast<unsigned char>(sk);
      p.c.vs[off / 16 + c / 4] = static_cast<unsigned char>(sv);
    }
  }
}

__global__ void __launch_bounds__(256) copy_lens_kernel(int B, const int32_t* pos0, int32_t* lens_out) {
  const int64_t step = static_cast<int64_t>(gridDim.x) * 256;
  for (int64_t b = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; b < B; b += step)
    lens_out[b] = pos0[b];
}

hipError_t launch_copy_lens(int B, const int32_t* pos0, int32_t* lens_out, hipStream_t s) {
  const int wgs = B / 256 + 1;
  hipLaunchKernelGGL(copy_lens_kernel, dim3(wgs < 1024 ? wgs : 1024), dim3(256), 0, s, B, pos0,
                     lens_out);
  return hipGetLastError();
}

// 8 values of a row: codes * scale.  v_cvt_scalef32_pk_{bf16,f32}_fp4 multiply by
// the scale's power of two (exactly, subnormals too) and give NaN for a NaN scale.
template <bool BF16>
__device__ __forceinline__ void store8(void* base, int64_t e, uint32_t codes, int scale_byte) {
  const float s = scale_byte == 255 ? __uint_as_float(0x7fc00000u)
                                    : __uint_as_float(static_cast<uint32_t>(scale_byte) << 23);
  const uint32_t w[4] = {
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 0)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 1)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 2)),
      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, s, 3))};
  if constexpr (BF16) {
    __builtin_nontemporal_store(
        u32x4{w[0], w[1], w[2], w[3]},
        reinterpret_cast<u32x4*>(static_cast<uint16_t*>(base) + e));
  } else {
    u32x4* o = reinterpret_cast<u32x4*>(static_cast<float*>(base) + e);
    __builtin_nontemporal_store(
        u32x4{w[0] << 16, w[0] & 0xffff0000u, w[1] << 16, w[1] & 0xffff0000u}, o);
    __builtin_nontemporal_store(
        u32x4{w[2] << 16, w[2] & 0xffff0000u, w[3] << 16, w[3] & 0xffff0000u}, o + 1);
  }
}

template <int D, bool BF16, bool PAGED>
__global__ void __launch_bounds__(256) kv4_read_kernel(const Kv4RowsParams p) {
  constexpr int LPR = D / 8;
  const int c = threadIdx.x % LPR;
  const int64_t step = static_cast<int64_t>(gridDim.x) * (256 / LPR);
  for (int64_t r = static_cast<int64_t>(blockIdx.x) * (256 / LPR) + threadIdx.x / LPR; r < p.rows;
       r += step) {
    const RowAt a = row_at(p, static_cast<uint32_t>(r));
    const int64_t dst =
        ((static_cast<int64_t>(a.b) * p.n + a.i) * p.Hkv + a.hk) * D + c * 8;
    int64_t off = 0;
    uint32_t ck = 0, cv = 0;
    int sk = 0, sv = 0;
    if (kv4_row<PAGED>(p.c, a.b, a.hk, static_cast<int64_t>(p.pos0[a.b]) + a.i, off)) {
      ck = *reinterpret_cast<const uint32_t*>(p.c.k + off + c * 4);
      cv = *reinterpret_cast<const uint32_t*>(p.c.v + off + c * 4);
      sk = p.c.ks[off / 16 + c / 4];
      sv = p.c.vs[off / 16 + c / 4];
    }
    store8<BF16>(p.k_rows, dst, ck, sk);
    store8<BF16>(p.v_rows, dst, cv, sv);
  }
}

static dim3 rows_grid(const Kv4RowsParams& p, int D) {
  const int64_t want = (static_cast<int64_t>(p.rows) * (D / 8) + 255) / 256;
  return dim3(static_cast<uint32_t>(want < (1 << 20) ? want : (1 << 20)));
}

template <int D>
static void launch_append(const Kv4RowsParams& p, bool bf16, bool paged, hipStream_t s) {
  const dim3 g = rows_grid(p, D), b(256);
  if (bf16) {
    if (paged) hipLaunchKernelGGL((kv4_append_kernel<D, true, true>), g, b, 0, s, p);
    else hipLaunchKernelGGL((kv4_append_kernel<D, true, false>), g, b, 0, s, p);
  } else {
    if (paged) hipLaunchKernelGGL((kv4_append_kernel<D, false, true>), g, b, 0, s, p);
    else hipLaunchKernelGGL((kv4_append_kernel<D, false, false>), g, b, 0, s, p);
  }
}

hipError_t launch_kv4_append(const Kv4RowsParams& p, int head_dim, bool bf16, bool paged,
                             hipStream_t s) {
  if (head_dim == 128) launch_append<128>(p, bf16, paged, s);
  else launch_append<64>(p, bf16, paged, s);
  return hipGetLastError();
}

template <int D>
static void launch_read(const Kv4RowsParams& p, bool bf16, bool paged, hipStream_t s) {
  const dim3 g = rows_grid(p, D), b(256);
  if (bf16) {
    if (paged) hipLaunchKernelGGL((kv4_read_kernel<D, true, true>), g, b, 0, s, p);
    else hipLaunchKernelGGL((kv4_read_kernel<D, true, false>), g, b, 0, s, p);
  } else {
    if (paged) hipLaunchKernelGGL((kv4_read_kernel<D, false, true>), g, b, 0, s, p);
    else hipLaunchKernelGGL((kv4_read_kernel<D, false, false>), g, b, 0, s, p);
  }
}

hipError_t launch_kv4_read(const Kv4RowsParams& p, int head_dim, bool bf16, bool paged,
                           hipStream_t s) {
  if (head_dim == 128) launch_read<128>(p, bf16, paged, s);
  else launch_read<64>(p, bf16, paged, s);
  return hipGetLastError();
}

}  // namespace md
