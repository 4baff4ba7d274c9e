// Microscaled 4-bit floating point (MXFP4): quantisation, read-back and product.
//
// A block of 32 consecutive elements of a row shares the scale 2^e, e = floor(log2(largest magnitude)) - 2 clamped
// to [-127, 127], so that the largest element lands in [4, 8); each element is x / 2^e rounded to nearest even on
// {0, .5, 1, 1.5, 2, 3, 4, 6}, magnitudes above 6 becoming 6.  A block of zeros has e = -127; a block that holds an
// infinity or NaN has the NaN scale (0xFF) and reads back, and multiplies, as NaN.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_fp4.h>
#include <atomic>

#include "../../include/gcada.h"
#include "common.cuh"
#include "mx.h"
#include "tc.cuh"

namespace gcada {
namespace {

// ----------------------------------------------------------------- elements
__device__ __forceinline__ uint32_t scale_code(float top) {  // biased exponent of the block's scale
  const uint32_t e = __float_as_uint(top) >> 23;             // top >= 0 or NaN; subnormal: 0
  return (e & 255u) == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}
__device__ __forceinline__ float inverse_scale(uint32_t code) {  // 2^(127 - code); codes up to 252 or 255
  return __uint_as_float((code == 255u ? 127u : 254u - code) << 23);
}
__device__ __forceinline__ float scale_value(uint32_t code) {
  return code == 255u ? __uint_as_float(0x7fffffffu) : (code ? __uint_as_float(code << 23) : __uint_as_float(0x400000u));
}
// Eight elements (already divided by the scale) as eight codes, the first in the lowest half byte.
__device__ __forceinline__ uint32_t codes8(const float (&f)[8]) {
  uint32_t w = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    w |= (uint32_t)__nv_cvt_float2_to_fp4x2(make_float2(f[2 * j], f[2 * j + 1]), __NV_E2M1, cudaRoundNearest) << (8 * j);
  return w;
}
__device__ __forceinline__ float2 values2(uint32_t byte) {
  const __half2_raw h = __nv_cvt_fp4x2_to_halfraw2((__nv_fp4x2_storage_t)byte, __NV_E2M1);
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
// fmaxf drops NaN: the largest magnitude of a block keeps it instead (as bits: NaN is above infinity)
__device__ __forceinline__ uint32_t abs_bits(float x) { return __float_as_uint(x) & 0x7fffffffu; }

template <typename T>
__device__ __forceinline__ void load8(const T* p, long long n, float (&f)[8]) {
  if (n >= 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    if (sizeof(T) == 4) {
      const float4 x = *reinterpret_cast<const float4*>(p), y = *(reinterpret_cast<const float4*>(p) + 1);
      f[0] = x.x; f[1] = x.y; f[2] = x.z; f[3] = x.w; f[4] = y.x; f[5] = y.y; f[6] = y.z; f[7] = y.w;
    } else {
      const uint4 x = *reinterpret_cast<const uint4*>(p);
      const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(j & 1 ? w[j >> 1] & 0xffff0000u : w[j >> 1] << 16);
    }
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = j < n ? (float)p[j] : 0.f;
  }
}

__device__ __forceinline__ long long scale_word(const MxView& q, int r, int ct, int half) {  // byte of a row's four scales
  return ((long long)(r >> 7) * q.col_tiles + ct) * 1024 + half * 512 + (r & 31) * 16 + ((r & 127) >> 5) * 4;
}

// A warp takes one column tile (256 columns, eight a lane, four lanes to a block of 32) of every `pass`-th row; warps
// next to each other take neighbouring tiles of a row.  ROWS_AT_ONCE rows' loads are on their way together.
constexpr int ROWS_AT_ONCE = 4;
struct WarpPlace {
  int ct, row;
};
__device__ __forceinline__ WarpPlace warp_place(const MxView& q, int pass) {
  const unsigned int g = blockIdx.x * 8u + (threadIdx.x >> 5), tiles = (unsigned int)q.col_tiles, row = g / tiles;
  return WarpPlace{(int)(g - row * tiles), (int)row < pass ? (int)row : 1 << 30};
}

// Rows run to the end of the last row tile (their scales are zeroed).
template <typename T>
__global__ void __launch_bounds__(256) mx_quantize_kernel(const T* __restrict__ x, long long ld, const MxView q, int pass) {
  __shared__ __align__(16) float row_sm[8][256];
  float* row = row_sm[threadIdx.x >> 5];
  const bool aligned = ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(ld * sizeof(T))) & 15) == 0;  // every row is
  const int lane = threadIdx.x & 31, rows = (int)q.rows, row_end = (rows + 127) / 128 * 128;
  const WarpPlace at = warp_place(q, pass);
  pdl_launch_dependents();
  pdl_wait();
  const int ct = at.ct;
  const long long c = (long long)ct * 256 + lane * 8;
  for (int r0 = at.row; r0 < row_end; r0 += ROWS_AT_ONCE * pass) {
    float f[ROWS_AT_ONCE][8];
    if (aligned) {
#pragma unroll
      for (int u = 0; u < ROWS_AT_ONCE; ++u) {
        const int r = r0 + u * pass;
#pragma unroll
        for (int j = 0; j < 8; ++j) f[u][j] = 0.f;
        if (r < rows && c < q.cols) load8(x + r * ld + c, q.cols - c, f[u]);
      }
    } else {  // neighbouring lanes take neighbouring elements, eight for each lane come back through shared memory
#pragma unroll
      for (int u = 0; u < ROWS_AT_ONCE; ++u) {
        const int r = r0 + u * pass;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const long long at = (long long)ct * 256 + j * 32 + lane;
          f[u][j] = r < rows && at < q.cols ? (float)x[r * ld + at] : 0.f;
        }
      }
#pragma unroll
      for (int u = 0; u < ROWS_AT_ONCE; ++u) {
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) row[j * 32 + lane] = f[u][j];
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; j += 4) {
          const float4 v = *reinterpret_cast<const float4*>(row + lane * 8 + j);
          f[u][j] = v.x; f[u][j + 1] = v.y; f[u][j + 2] = v.z; f[u][j + 3] = v.w;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < ROWS_AT_ONCE; ++u) {
      const int r = r0 + u * pass;
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) top = max(top, abs_bits(f[u][j]));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const uint32_t sc = scale_code(__uint_as_float(top));
      const float inv = inverse_scale(sc);
#pragma unroll
      for (int j = 0; j < 8; ++j) f[u][j] *= inv;
      if (r < rows && c < q.pitch * 2) *reinterpret_cast<uint32_t*>(q.codes + r * q.pitch + c / 2) = codes8(f[u]);
      // four blocks' scales are one word of a tile
      uint32_t word = sc << (8 * ((lane >> 2) & 3));
      word |= __shfl_xor_sync(0xffffffffu, word, 4);
      word |= __shfl_xor_sync(0xffffffffu, word, 8);
      if ((lane & 15) == 0 && r < row_end) *reinterpret_cast<uint32_t*>(q.scales + scale_word(q, r, ct, lane >> 4)) = word;
    }
  }
}

// The same for bf16 rows that start on 16 bytes: a lane takes a whole block (four loads of 16 bytes, each line's
// quarters by neighbouring instructions), so that nothing is exchanged between lanes: 85 MB in 16 us instead of 28.
// `i` counts the blocks of all rows, tiles' padding included.
__global__ void __launch_bounds__(256) mx_quantize_blocks_kernel(const __nv_bfloat16* __restrict__ x, long long ld, const MxView q) {
  pdl_launch_dependents();
  pdl_wait();
  const unsigned int per_row = (unsigned int)q.col_tiles * 8u;
  const long long total = (q.rows + 127) / 128 * 128 * per_row;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const long long r = total < (1LL << 31) ? (long long)((unsigned int)i / per_row) : i / per_row;
    const int blk = (int)(i - r * per_row);
    const long long c = (long long)blk * 32;
    uint32_t sc = 0;
    if (r < q.rows && c < q.cols) {
      const __nv_bfloat16* p = x + r * ld + c;
      uint32_t v[16];
      if (c + 32 <= q.cols) {
#pragma unroll
        for (int g = 0; g < 4; ++g) *reinterpret_cast<uint4*>(v + 4 * g) = *reinterpret_cast<const uint4*>(p + 8 * g);
      } else {
#pragma unroll
        for (int j = 0; j < 16; ++j) {
          const uint32_t a = c + 2 * j < q.cols ? __bfloat16_as_ushort(p[2 * j]) : 0u, b = c + 2 * j + 1 < q.cols ? __bfloat16_as_ushort(p[2 * j + 1]) : 0u;
          v[j] = a | (b << 16);
        }
      }
      uint32_t top = 0;
#pragma unroll
      for (int j = 0; j < 16; ++j) top = max(top, max((v[j] << 16) & 0x7fffffffu, v[j] & 0x7fff0000u));
      sc = scale_code(__uint_as_float(top));
      const float inv = inverse_scale(sc);
      uint32_t o[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        float f[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) f[j] = __uint_as_float(j & 1 ? v[4 * g + (j >> 1)] & 0xffff0000u : v[4 * g + (j >> 1)] << 16) * inv;
        o[g] = codes8(f);
      }
      *reinterpret_cast<uint4*>(q.codes + r * q.pitch + c / 2) = make_uint4(o[0], o[1], o[2], o[3]);
    }
    q.scales[scale_word(q, (int)r, blk >> 3, (blk >> 2) & 1) + (blk & 3)] = (unsigned char)sc;
  }
}

// Two neighbouring elements, as loaded.
template <typename T>
struct Pair2;
template <>
struct Pair2<float> {
  using raw = float2;
  static __device__ __forceinline__ float lo(float2 v) { return v.x; }
  static __device__ __forceinline__ float hi(float2 v) { return v.y; }
  static __device__ __forceinline__ float2 make(float a, float b) { return make_float2(a, b); }
};
template <>
struct Pair2<__nv_bfloat16> {
  using raw = uint32_t;
  static __device__ __forceinline__ float lo(uint32_t v) { return __uint_as_float(v << 16); }
  static __device__ __forceinline__ float hi(uint32_t v) { return __uint_as_float(v & 0xffff0000u); }
  static __device__ __forceinline__ uint32_t make(__nv_bfloat16 a, __nv_bfloat16 b) {
    return (uint32_t)__bfloat16_as_ushort(a) | ((uint32_t)__bfloat16_as_ushort(b) << 16);
  }
};

// Transposed source: x is [q.cols][q.rows], blocks run down its columns.  A CTA takes 64 columns (rows of the
// result) x 256 rows; warp w the block of 32 rows w, two columns per lane, all 32 loads on their way together
// (guarded one by one they were not: 321 us for 32768 x 4096 bf16); codes and scales leave through shared memory so
// that a result row's 128 bytes are written together.  CTAs that run together take neighbouring columns.
template <typename T>
__global__ void __launch_bounds__(256) mx_quantize_t_kernel(const T* __restrict__ x, long long ld, const MxView q) {
  using P = Pair2<T>;
  __shared__ __align__(16) uint4 codes_sm[64][9];  // [row][block], padded
  __shared__ uint32_t scale_sm[64][2];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const long long strips = (q.rows + 127) / 128 * 2, ct = blockIdx.x / strips, r0 = (blockIdx.x - ct * strips) * 64;
  const long long k0 = ct * 256 + w * 32, r = r0 + 2 * lane;
  typename P::raw v[32];
  const T* p = x + k0 * ld + r;
  const bool aligned = (reinterpret_cast<uintptr_t>(x) & (2 * sizeof(T) - 1)) == 0 && (ld & 1) == 0;
  pdl_launch_dependents();
  pdl_wait();
  if (aligned && r0 + 64 <= q.rows && k0 + 32 <= q.cols) {  // the same for the whole warp
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = *reinterpret_cast<const typename P::raw*>(p + j * ld);
  } else if (r0 + 64 <= q.rows && k0 + 32 <= q.cols) {
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = P::make(p[j * ld], p[j * ld + 1]);
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) {
      const bool in = k0 + j < q.cols;
      v[j] = P::make(in && r < q.rows ? p[j * ld] : (T)0.f, in && r + 1 < q.rows ? p[j * ld + 1] : (T)0.f);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) top = max(top, abs_bits(h ? P::hi(v[j]) : P::lo(v[j])));
    const uint32_t sc = scale_code(__uint_as_float(top));
    const float inv = inverse_scale(sc);
    uint32_t c[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = (h ? P::hi(v[8 * g + j]) : P::lo(v[8 * g + j])) * inv;
      c[g] = codes8(f);
    }
    codes_sm[2 * lane + h][w] = make_uint4(c[0], c[1], c[2], c[3]);
    reinterpret_cast<unsigned char*>(scale_sm[2 * lane + h])[w] = (unsigned char)sc;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * 8; i += 256) {
    const int rr = i >> 3, b = i & 7;
    const long long at = ct * 128 + b * 16;
    if (r0 + rr < q.rows && at < q.pitch) *reinterpret_cast<uint4*>(q.codes + (r0 + rr) * q.pitch + at) = codes_sm[rr][b];
  }
  if (threadIdx.x < 128) {  // rows behind the end have zero elements, hence zero scales
    const int rr = threadIdx.x >> 1, half = threadIdx.x & 1;
    *reinterpret_cast<uint32_t*>(q.scales + scale_word(q, (int)r0 + rr, (int)ct, half)) = scale_sm[rr][half];
  }
}

// Eight codes as four pairs of bfloat16 numbers: the magnitudes' two bytes looked up four codes at a time, the signs
// put in their place, one product with the scale (exact: a power of two).
__device__ __forceinline__ void values8(uint32_t w, uint32_t sc, uint32_t (&o)[4]) {
  const uint32_t s16 = sc == 255u ? 0x7fffu : (sc ? sc << 7 : 0x40u), scale = s16 | (s16 << 16);
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const uint32_t v = w >> (16 * h), sel = v & 0x7777u;
    const uint32_t top = __byte_perm(0x3f3f3f00u, 0x40404040u, sel), low = __byte_perm(0xc0800000u, 0xc0804000u, sel);
    uint32_t a = __byte_perm(low, top, 0x5140), b = __byte_perm(low, top, 0x7362);
    a |= ((v << 12) & 0x8000u) | ((v << 24) & 0x80000000u);
    b |= ((v << 4) & 0x8000u) | ((v << 16) & 0x80000000u);
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[2 * h]) : "r"(a), "r"(scale));
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[2 * h + 1]) : "r"(b), "r"(scale));
  }
}

template <typename T>
__global__ void __launch_bounds__(256) mx_dequantize_kernel(const MxView q, T* __restrict__ out, long long ld, int pass) {
  __shared__ __align__(16) T row_sm[8][256];
  T* row = row_sm[threadIdx.x >> 5];
  const bool aligned = ((reinterpret_cast<uintptr_t>(out) | (uintptr_t)(ld * sizeof(T))) & 15) == 0;  // every row is
  const int lane = threadIdx.x & 31, rows = (int)q.rows;
  const WarpPlace at = warp_place(q, pass);
  pdl_launch_dependents();
  pdl_wait();
  const int ct = at.ct;
  const long long c = (long long)ct * 256 + lane * 8;
  const bool in = c < q.cols, direct = sizeof(T) == 2 && aligned && c + 8 <= q.cols;
  for (int r0 = at.row; r0 < rows; r0 += ROWS_AT_ONCE * pass) {
    uint32_t w[ROWS_AT_ONCE], sc[ROWS_AT_ONCE];
#pragma unroll
    for (int u = 0; u < ROWS_AT_ONCE; ++u) {
      const int r = r0 + u * pass < rows ? r0 + u * pass : r0;
      w[u] = in ? *reinterpret_cast<const uint32_t*>(q.codes + r * q.pitch + c / 2) : 0u;
      sc[u] = q.scales[scale_word(q, r, ct, lane >> 4) + ((lane >> 2) & 3)];
    }
#pragma unroll
    for (int u = 0; u < ROWS_AT_ONCE; ++u) {
      const int r = r0 + u * pass;
      if (r >= rows) break;  // (the same for the whole warp)
      T* to = direct ? out + r * ld + c : row + lane * 8;
      if (sizeof(T) == 2) {
        uint32_t v[4];
        values8(w[u], sc[u], v);
        *reinterpret_cast<uint4*>(to) = make_uint4(v[0], v[1], v[2], v[3]);
      } else {
        const float s = scale_value(sc[u]);
        float f[8];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float2 t = values2((w[u] >> (8 * j)) & 255u);
          f[2 * j] = t.x * s;
          f[2 * j + 1] = t.y * s;
        }
        reinterpret_cast<float4*>(to)[0] = make_float4(f[0], f[1], f[2], f[3]);
        reinterpret_cast<float4*>(to)[1] = make_float4(f[4], f[5], f[6], f[7]);
      }
      if (sizeof(T) == 4 || !__all_sync(0xffffffffu, direct)) {  // by way of shared memory: neighbouring lanes write neighbouring elements (32 bytes a lane, as floats are, half fill their sectors)
        __syncwarp();
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int i = j * 32 + lane;
          const long long col = (long long)ct * 256 + i;
          if (col < q.cols && !(sizeof(T) == 2 && aligned && (col | 7) < q.cols)) out[r * ld + col] = row[i];
        }
        __syncwarp();
      }
    }
  }
}

// Uploads: a CTA takes 64 columns x 128 rows of one selected group's factor (warp w: the block of 32 rows w, two
// columns a lane), as mx_quantize_t_kernel does; a result row's 64 bytes and four scales are written together.
__global__ void __launch_bounds__(128) mx_quantize_uploads_kernel(const Params P, const __nv_bfloat16* __restrict__ x, int ld,
                                                                  int Bp, const MxView q) {
  using T = Pair2<__nv_bfloat16>;
  __shared__ __align__(16) uint4 codes_sm[64][5];
  __shared__ uint32_t scale_sm[64];
  if ((int)blockIdx.z >= P.sel_count[0]) return;
  const int g = P.sel_list[blockIdx.z], lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  if (!GCADA_INDEX_OK(P.st, g, P.G, CHK_FACTOR)) return;
  const int r0 = blockIdx.x * 64, r = r0 + 2 * lane, b0 = blockIdx.y * 128;
  const long long k0 = (long long)g * Bp + b0;  // first column of the result
  const __nv_bfloat16* p = x + (((long long)P.cur[g] * P.G + g) * Bp + b0 + w * 32) * ld + r;
  uint32_t v[32];
  if (r0 + 64 <= q.rows) {  // (rows are whole 128-byte lines: pairs are aligned)
#pragma unroll
    for (int j = 0; j < 32; ++j) v[j] = *reinterpret_cast<const uint32_t*>(p + (long long)j * ld);
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      v[j] = T::make(r < q.rows ? p[(long long)j * ld] : (__nv_bfloat16)0.f, r + 1 < q.rows ? p[(long long)j * ld + 1] : (__nv_bfloat16)0.f);
  }
  // behind the minibatch's end the factor holds what the network makes of a row of zeros (activations relu(b)): no part of
  // the upload, and it must not decide the scale of a block that it shares with samples
  const int samples = P.B - b0 - w * 32;
  if (samples < 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (j >= samples) v[j] = 0;
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 32; ++j) top = max(top, abs_bits(h ? T::hi(v[j]) : T::lo(v[j])));
    const uint32_t sc = scale_code(__uint_as_float(top));
    const float inv = inverse_scale(sc);
    uint32_t c[4];
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      float f[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) f[j] = (h ? T::hi(v[8 * t + j]) : T::lo(v[8 * t + j])) * inv;
      c[t] = codes8(f);
    }
    codes_sm[2 * lane + h][w] = make_uint4(c[0], c[1], c[2], c[3]);
    reinterpret_cast<unsigned char*>(&scale_sm[2 * lane + h])[w] = (unsigned char)sc;
  }
  __syncthreads();
  for (int i = threadIdx.x; i < 64 * 4; i += 128) {
    const int rr = i >> 2;
    if (r0 + rr < q.rows) *reinterpret_cast<uint4*>(q.codes + (r0 + rr) * q.pitch + k0 / 2 + (i & 3) * 16) = codes_sm[rr][i & 3];
  }
  if (threadIdx.x < 64)
    *reinterpret_cast<uint32_t*>(q.scales + scale_word(q, r0 + threadIdx.x, (int)(k0 / 256), (int)(k0 / 128 % 2))) = scale_sm[threadIdx.x];
}

// One group's share of a product, for getters: a value a thread.
__global__ void __launch_bounds__(256) mx_upload_product_kernel(const MxView a, const MxView b, long long k0, int K, float* out) {
  const int n = blockIdx.x * 32 + (threadIdx.x & 31), m = blockIdx.y * 8 + (threadIdx.x >> 5);
  if (m >= a.rows || n >= b.rows) return;
  float sum = 0.f;
  for (int k = 0; k < K; k += 32) {
    const long long c = k0 + k;
    const uint4 x = *reinterpret_cast<const uint4*>(a.codes + m * a.pitch + c / 2), y = *reinterpret_cast<const uint4*>(b.codes + n * b.pitch + c / 2);
    const int ct = (int)(c / 256), half = (int)(c / 128 % 2), q = (int)(c / 32 % 4);
    const float s = scale_value(a.scales[scale_word(a, m, ct, half) + q]) * scale_value(b.scales[scale_word(b, n, ct, half) + q]);
    const uint32_t xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
    float t = 0.f;
    for (int i = 0; i < 16; ++i) {
      const float2 u = values2((xs[i >> 2] >> (8 * (i & 3))) & 255u), v = values2((ys[i >> 2] >> (8 * (i & 3))) & 255u);
      t += u.x * v.x + u.y * v.y;
    }
    sum += s * t;
  }
  out[(long long)m * b.rows + n] = sum;
}

// ----------------------------------------------------------------- product
// Warp 0 copies the operands' codes (128-byte rows of 256 elements, 128-byte swizzle) and scales into a ring of
// stages, warp 1 copies a stage's scales into tensor memory and issues the block-scaled products (64 K values each),
// sixteen warps write the result.  As in the fp16 products of muon.cu there are two kinds of shapes:
//   PAIR: two CTAs on a 256 x BN tile (cta_group::2), persistent.  A CTA holds 128 rows of A and of the result, half of
//         the columns of B, and the scales of its rows and of all columns.  BN = 256 needs the fewest bytes; its accumulator
//         takes 256 of the 512 columns of tensor memory and the stages' scales most of the rest, so there is only one, and
//         the epilogue first moves it to registers (64 a thread), which frees it for the next tile.  BN = 192 leaves room
//         for two, so that the epilogue of a tile runs beside the products of the next: faster where K is short.
//   else: a CTA on a 128 x BN tile; with fewer tiles than SMs the CTAs of a cluster share the K range and add up
//         their partial tiles through distributed shared memory in rank order.
constexpr int BM = 128, KB = 256;
constexpr int EPI_WARPS = 16;
constexpr int THREADS = 64 + 32 * EPI_WARPS;

template <bool PAIR, int BN>
struct MxTile {
  static constexpr int TM = PAIR ? 256 : 128, TN = BN;  // the tile
  static constexpr int ROWS_B = PAIR ? BN / 2 : BN;     // rows of B that this CTA copies
  static constexpr int NB = (TN + 127) / 128;           // row tiles of B's scales that the tile touches
  static constexpr int ACC = TN == 256 ? 1 : 2;         // accumulators in tensor memory
  static constexpr int CODE_BYTES = (BM + ROWS_B) * (KB / 2);
  static constexpr int STAGE_BYTES = CODE_BYTES + (1 + NB) * 1024;
  static constexpr int STAGES = BN == 64 ? 7 : 5;
  static constexpr int PIECE_BYTES = 32 * 64;  // a warp's 32 rows of 64 bytes of a result on their way out
  static constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + EPI_WARPS * PIECE_BYTES + 1024;
  static constexpr int SF_COL = ACC * TN;                 // first tensor-memory column of the scales
  static constexpr int SF_COLS = 8 + 8 * NB;              // per stage: A 2 x 4, B 2 x 4 NB
  static constexpr int TMEM_COLS = SF_COL + STAGES * SF_COLS <= 256 ? 256 : 512;
  static_assert(SF_COL + STAGES * SF_COLS <= 512, "tensor memory");
  static_assert(STAGE_BYTES % 1024 == 0, "swizzle atoms");
  static_assert(PAIR || BM * TN * 4 <= STAGES * STAGE_BYTES, "a partial tile lies in the stages");
  static_assert(SMEM_BYTES <= 232448 - 1024, "shared memory");
};

// 512 bytes of scales (32 rows x 16 bytes, no swizzle; groups of 8 rows 128 bytes apart) into four columns of
// tensor memory, the same for every quadrant of lanes; with PAIR in both CTAs.
template <bool PAIR>
__device__ __forceinline__ void tc_copy_scales(uint32_t taddr, uint32_t smem_addr) {
  const uint64_t desc = (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | ((uint64_t)(128 >> 4) << 32) | (1ull << 46);
  if (PAIR)
    asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
  else
    asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(taddr), "l"(desc) : "memory");
}
template <bool PAIR>
__device__ __forceinline__ void tc_mma_mxf4(uint32_t tmem_c, uint64_t da, uint64_t db, uint32_t idesc, uint32_t sfa,
                                            uint32_t sfb, uint32_t accum) {
  if (PAIR)
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(tmem_c),
        "l"(da), "l"(db), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accum)
        : "memory");
  else
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %6, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}" ::"r"(tmem_c),
        "l"(da), "l"(db), "r"(idesc), "r"(sfa), "r"(sfb), "r"(accum)
        : "memory");
}

// Sixteen sums of row m from column n on (n < N), scaled and written.
__device__ __forceinline__ void mx_finish16(const MxGemm& p, int m, int n, float (&f)[16]) {
  const int N = (int)p.b.rows;
#pragma unroll
  for (int j = 0; j < 16; ++j) f[j] *= p.alpha;
  if (p.bias) {
#pragma unroll
    for (int j = 0; j < 16; ++j)
      if (n + j < N) f[j] += p.bias[n + j];
  }
  if (!p.d_bf16) {
    float* o = static_cast<float*>(p.d) + (long long)m * p.ld + n;
    if (n + 16 <= N && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
      float4* o4 = reinterpret_cast<float4*>(o);
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        float4 v = make_float4(f[4 * t], f[4 * t + 1], f[4 * t + 2], f[4 * t + 3]);
        if (p.beta != 0.f) {
          const float4 d = o4[t];
          v = make_float4(v.x + p.beta * d.x, v.y + p.beta * d.y, v.z + p.beta * d.z, v.w + p.beta * d.w);
        }
        o4[t] = v;
      }
    } else {
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (n + t < N) o[t] = p.beta != 0.f ? f[t] + p.beta * o[t] : f[t];
    }
  } else {
    __nv_bfloat16* o = static_cast<__nv_bfloat16*>(p.d) + (long long)m * p.ld + n;
    if (p.beta != 0.f) {
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (n + t < N) f[t] += p.beta * __bfloat162float(o[t]);
    }
    if (n + 16 <= N && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
      uint32_t w[8];
#pragma unroll
      for (int t = 0; t < 8; ++t) {
        const __nv_bfloat162 b2 = __floats2bfloat162_rn(f[2 * t], f[2 * t + 1]);
        w[t] = *reinterpret_cast<const uint32_t*>(&b2);
      }
      reinterpret_cast<uint4*>(o)[0] = make_uint4(w[0], w[1], w[2], w[3]);
      reinterpret_cast<uint4*>(o)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    } else {
#pragma unroll
      for (int t = 0; t < 16; ++t)
        if (n + t < N) o[t] = __float2bfloat16_rn(f[t]);
    }
  }
}

// A warp's 32 rows x W columns from (m0, n) on, a lane a row: through shared memory in pieces of 64 bytes a row, so that four
// lanes write a row's and an instruction meets 8 lines instead of 32 (8192 x 4096 x 1024, fp32: 60 -> 33 us).
template <int W>
__device__ __forceinline__ void mx_finish_rows(const MxGemm& p, unsigned char* buf, int lane, int m0, int n, const uint32_t (&v)[W / 16][16]) {
  const int M = (int)p.a.rows, N = (int)p.b.rows;
  const bool even = ((reinterpret_cast<uintptr_t>(p.d) | (uintptr_t)(p.ld * (p.d_bf16 ? 2 : 4))) & 15) == 0;
#pragma unroll
  for (int j = 0; j < W / 16; ++j) {
    const int nj = n + 16 * j;
    if (nj >= N) continue;
    // a piece: 16 columns in fp32, in bf16 32, taken together with the even sixteen
    const bool whole = even && (p.d_bf16 ? p.beta == 0.f && (j | 1) < W / 16 && n + 16 * (j | 1) + 16 <= N : nj + 16 <= N);
    if (whole && p.d_bf16 && (j & 1)) continue;
    float f[16];
#pragma unroll
    for (int t = 0; t < 16; ++t) f[t] = __uint_as_float(v[j][t]);
    if (!whole) {
      if (m0 + lane < M) mx_finish16(p, m0 + lane, nj, f);
      continue;
    }
    uint4 x[4];
#pragma unroll
    for (int t = 0; t < 16; ++t) f[t] = p.alpha * f[t] + (p.bias ? p.bias[nj + t] : 0.f);
    if (!p.d_bf16) {
#pragma unroll
      for (int c = 0; c < 4; ++c)
        x[c] = make_uint4(__float_as_uint(f[4 * c]), __float_as_uint(f[4 * c + 1]), __float_as_uint(f[4 * c + 2]), __float_as_uint(f[4 * c + 3]));
    } else {
      constexpr int LAST = W / 16 - 1;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (c == 2) {
#pragma unroll
          for (int t = 0; t < 16; ++t)
            f[t] = p.alpha * __uint_as_float(v[j < LAST ? j + 1 : j][t]) + (p.bias ? p.bias[nj + 16 + t] : 0.f);
        }
        uint32_t w[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const __nv_bfloat162 b2 = __floats2bfloat162_rn(f[8 * (c & 1) + 2 * t], f[8 * (c & 1) + 2 * t + 1]);
          w[t] = *reinterpret_cast<const uint32_t*>(&b2);
        }
        x[c] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    const int ch = lane & 3;
#pragma unroll
    for (int c = 0; c < 4; ++c) *reinterpret_cast<uint4*>(buf + lane * 64 + ((c ^ ((lane >> 1) & 3)) << 4)) = x[c];
    __syncwarp();
#pragma unroll
    for (int r0 = 0; r0 < 32; r0 += 8) {
      const int r = r0 + (lane >> 2), m = m0 + r;
      uint4 y = *reinterpret_cast<const uint4*>(buf + r * 64 + ((ch ^ ((r >> 1) & 3)) << 4));
      if (m < M) {
        uint4* o = reinterpret_cast<uint4*>(static_cast<char*>(p.d) + ((long long)m * p.ld + nj) * (p.d_bf16 ? 2 : 4)) + ch;
        if (p.beta != 0.f) {  // (fp32)
          const float4 d = *reinterpret_cast<const float4*>(o);
          y = make_uint4(__float_as_uint(__uint_as_float(y.x) + p.beta * d.x), __float_as_uint(__uint_as_float(y.y) + p.beta * d.y),
                         __float_as_uint(__uint_as_float(y.z) + p.beta * d.z), __float_as_uint(__uint_as_float(y.w) + p.beta * d.w));
        }
        *o = y;
      }
    }
    __syncwarp();
  }
}

template <bool PAIR, int BN>
__global__ void __launch_bounds__(THREADS, 1) mx_gemm_kernel(const __grid_constant__ CUtensorMap tmA,
                                                             const __grid_constant__ CUtensorMap tmB,
                                                             const __grid_constant__ CUtensorMap tmSA,
                                                             const __grid_constant__ CUtensorMap tmSB, const MxGemm p,
                                                             const int split) {
  using T = MxTile<PAIR, BN>;
  constexpr int STAGES = T::STAGES, WCOLS = T::TN / 4;  // columns of an epilogue warp
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t full_bar[STAGES], empty_bar[STAGES], tfull_bar[2], tempty_bar[2];
  __shared__ uint32_t tmem_base_sm;
  unsigned char* tiles = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int csize = PAIR ? 2 : split;
  const int rank = csize > 1 ? (int)cluster_rank() : 0;
  const int first = (int)blockIdx.x / csize, stride = (int)gridDim.x / csize;
  const int M = (int)p.a.rows, N = (int)p.b.rows;
  const int tiles_m = (M + T::TM - 1) / T::TM, tiles_n = (N + T::TN - 1) / T::TN, total = tiles_m * tiles_n;
  const int n_local = first < total ? (total - first + stride - 1) / stride : 0;
  const int kb_all = (int)p.a.col_tiles;
  const int kb0 = PAIR ? 0 : (int)((long long)kb_all * rank / csize);
  const int kb1 = PAIR ? kb_all : (int)((long long)kb_all * (rank + 1) / csize);

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&tfull_bar[s], 1);
      mbar_init(&tempty_bar[s], PAIR ? 2 * EPI_WARPS : EPI_WARPS);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) tmem_alloc<PAIR>(&tmem_base_sm, (uint32_t)T::TMEM_COLS);
  if (threadIdx.x == 64) {
    prefetch_map(&tmA);
    prefetch_map(&tmB);
    prefetch_map(&tmSA);
    prefetch_map(&tmSB);
  }
  tc_fence_before();
  __syncthreads();
  if (PAIR) cluster_sync();  // the peer's barriers exist
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sm;
  pdl_launch_dependents();
  const bool leader = elect_one();

  if (warp == 0) {
    // the warp runs the loop as a whole and elects a thread for the copies: what they take is uniform to the compiler then
    bool ok = true;
    int it = 0;
    for (int i = 0; i < n_local && ok; ++i) {
      const int u = first + i * stride, mt = u / tiles_n, nt = u - mt * tiles_n;
      const int rank_b = PAIR ? rank * T::ROWS_B : 0;
      const int rA = mt * T::TM + (PAIR ? rank * 128 : 0), rB = nt * T::TN + rank_b;
      for (int kb = kb0; kb < kb1; ++kb, ++it) {
        const int s = it % STAGES;
        ok = __all_sync(0xffffffffu, mbar_spin_bounded(&empty_bar[s], (uint32_t)(((it / STAGES) & 1) ^ 1)));
        if (!ok) break;
        if (it == 0) pdl_wait();  // here and not earlier: the first run of what lies before costs as much as a copy
        if (elect_one()) {
          unsigned char* sa = tiles + (size_t)s * T::STAGE_BYTES;
          if (!PAIR || rank == 0) mbar_expect_tx(&full_bar[s], (PAIR ? 2 : 1) * T::STAGE_BYTES);
          const uint32_t bar = PAIR ? cluster_map(smem_u32(&full_bar[s]), 0) : smem_u32(&full_bar[s]);
          tma_load_2d_to<PAIR>(sa, &tmA, kb * (KB / 2), rA, bar);
          tma_load_2d_to<PAIR>(sa + BM * (KB / 2), &tmB, kb * (KB / 2), rB, bar);
          // scale tiles are rows of their maps; one behind the end (its columns are not kept) arrives as zeros
          tma_load_2d_to<PAIR>(sa + T::CODE_BYTES, &tmSA, 0, (rA >> 7) * (int)p.a.col_tiles + kb, bar);
#pragma unroll
          for (int j = 0; j < T::NB; ++j)
            tma_load_2d_to<PAIR>(sa + T::CODE_BYTES + (1 + j) * 1024, &tmSB, 0, ((nt * T::TN >> 7) + j) * (int)p.b.col_tiles + kb, bar);
        }
      }
    }
    if (!ok && leader) raise_error(p.err);
  } else if (warp == 1) {
    if (leader && (!PAIR || rank == 0)) {
      // its bounded waits count from here: a predecessor that let this kernel start early may run for any time
      pdl_wait();
      // E2M1 operands (1 at bits 7 and 10), E8M0 scales (bit 23); bits 29 / 4: which pair of a column's four scale
      // bytes an instruction's two blocks take
      constexpr uint32_t IDESC =
          (1u << 7) | (1u << 10) | ((uint32_t)(T::TN >> 3) << 17) | (1u << 23) | ((uint32_t)(T::TM >> 4) << 24);
      bool ok = true;
      int it = 0;
      for (int i = 0; i < n_local && ok; ++i) {
        const int slot = i % T::ACC;
        const int u = first + i * stride, nt = u % tiles_n;
        ok = mbar_spin_bounded(&tempty_bar[slot], (uint32_t)(((i / T::ACC) & 1) ^ 1));
        if (!ok) break;
        tc_fence_after();
        for (int kb = kb0; kb < kb1 && ok; ++kb, ++it) {
          const int s = it % STAGES;
          ok = mbar_spin_bounded(&full_bar[s], (uint32_t)((it / STAGES) & 1));
          if (!ok) break;
          tc_fence_after();
          const uint32_t sa = smem_u32(tiles + (size_t)s * T::STAGE_BYTES);
          const uint32_t sf = tmem_base + (uint32_t)(T::SF_COL + s * T::SF_COLS);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            tc_copy_scales<PAIR>(sf + h * 4, sa + T::CODE_BYTES + h * 512);
#pragma unroll
            for (int j = 0; j < T::NB; ++j)
              tc_copy_scales<PAIR>(sf + 8 + h * 4 * T::NB + j * 4, sa + T::CODE_BYTES + (1 + j) * 1024 + h * 512);
          }
          const uint64_t da = make_desc(sa), db = make_desc(sa + BM * (KB / 2));
          // a tile may start in the middle of a scale tile, at one of its groups of 32 rows = one of the four columns
          const uint32_t sub = T::TN % 128 ? (uint32_t)((nt * T::TN & 127) >> 5) : 0u;
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            const uint32_t id = (uint32_t)(kk & 1) * 2u;
            tc_mma_mxf4<PAIR>(tmem_base + (uint32_t)(slot * T::TN), da + (uint64_t)(kk * 2), db + (uint64_t)(kk * 2),
                              IDESC | (id << 29) | (id << 4), sf + (kk >> 1) * 4, sf + 8 + (kk >> 1) * 4 * T::NB + sub,
                              (kb != kb0 || kk != 0) ? 1u : 0u);
          }
          tc_commit_to<PAIR>(&empty_bar[s]);
        }
        if (ok) tc_commit_to<PAIR>(&tfull_bar[slot]);
      }
      if (!ok) raise_error(p.err);
    }
  } else {
    const int quad = warp & 3, sub = (warp - 2) >> 2;
    unsigned char* buf = tiles + (size_t)STAGES * T::STAGE_BYTES + (size_t)(warp - 2) * T::PIECE_BYTES;
    bool ok = true;
    pdl_wait();
    for (int i = 0; i < n_local; ++i) {
      const int slot = i % T::ACC;
      const int u = first + i * stride, mt = u / tiles_n, nt = u - mt * tiles_n;
      const int m0 = mt * T::TM + (PAIR ? rank * 128 : 0) + quad * 32, c0 = sub * WCOLS, n0 = nt * T::TN + c0;
      if (ok) {
        ok = mbar_wait_bounded(&tfull_bar[slot], (uint32_t)((i / T::ACC) & 1));
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok) continue;
      tc_fence_after();
      const uint32_t tbase = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(slot * T::TN + c0);
      uint32_t v[WCOLS / 16][16];
#pragma unroll
      for (int q = 0; q < WCOLS / 16; ++q) tc_ld16_issue(tbase + (uint32_t)(q * 16), v[q]);
      tc_ld_wait();
      tc_fence_before();
      __syncwarp();
      if (leader) {
        if (PAIR)
          mbar_arrive_cluster(cluster_map(smem_u32(&tempty_bar[slot]), 0));
        else
          mbar_arrive(&tempty_bar[slot]);
      }
      if (!PAIR && csize > 1) {
        float* part = reinterpret_cast<float*>(tiles) + (size_t)c0 * BM + quad * 32 + lane;
#pragma unroll
        for (int j = 0; j < WCOLS; ++j) part[j * BM] = __uint_as_float(v[j >> 4][j & 15]);
      } else {
        mx_finish_rows<WCOLS>(p, buf, lane, m0, n0, v);
      }
    }
    if (!ok && leader) raise_error(p.err);
  }
  if (!PAIR && csize > 1) {
    // one tile per cluster; every stage had been consumed before the partial tiles were written over them
    __syncwarp();
    cluster_sync();
    // columns are dealt out 16 at a time, to the CTAs, then to the four warps of a quadrant: one group a thread at most
    const int quad = warp & 3, c = 16 * (rank + ((warp - 2) >> 2) * csize), mt = first / tiles_n, nt = first - mt * tiles_n;
    const int m = mt * T::TM + quad * 32 + lane, n = nt * T::TN + c;
    if (warp >= 2 && c < T::TN && m < M && n < N) {
      float f[16];
#pragma unroll
      for (int j = 0; j < 16; ++j) f[j] = 0.f;
      const uint32_t place = smem_u32(tiles) + (uint32_t)((c * BM + quad * 32 + lane) * 4);
      for (int p0 = 0; p0 < csize; p0 += 4) {
        float x[4][16];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (p0 + r < csize) {
            const uint32_t from = cluster_map(place, (uint32_t)(p0 + r));
#pragma unroll
            for (int j = 0; j < 16; ++j) x[r][j] = cluster_load(from + (uint32_t)(j * BM * 4));
          }
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          if (p0 + r < csize) {
#pragma unroll
            for (int j = 0; j < 16; ++j) f[j] += x[r][j];
          }
        }
      }
      mx_finish16(p, m, n, f);
    }
  }
  tc_fence_before();
  __syncthreads();
  if (csize > 1) cluster_sync();  // nobody reads this CTA's shared or tensor memory any more
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc<PAIR>(tmem_base, (uint32_t)T::TMEM_COLS);
  }
}

// ----------------------------------------------------------------- host
// codes as bytes [rows][pitch]; boxes of 128 bytes (256 elements) x box_rows, 128-byte swizzle, zero fill outside.
bool make_map_codes(CUtensorMap* tm, const MxView& v, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {(cuuint64_t)mx_pitch(v.cols), (cuuint64_t)v.rows};
  cuuint64_t strides[1] = {(cuuint64_t)v.pitch};
  cuuint32_t box[2] = {128, (cuuint32_t)box_rows};
  cuuint32_t es[2] = {1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, v.codes, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// scale tiles as rows of 256 words, one a box
bool make_map_scales(CUtensorMap* tm, const MxView& v) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[2] = {256, (cuuint64_t)((v.rows + 127) / 128 * v.col_tiles)};
  cuuint64_t strides[1] = {1024};
  cuuint32_t box[2] = {256, 1};
  cuuint32_t es[2] = {1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_UINT32, 2, v.scales, dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t set_attributes() {
  const cudaFuncAttribute at = cudaFuncAttributeMaxDynamicSharedMemorySize;
  cudaError_t e = cudaFuncSetAttribute(mx_gemm_kernel<true, 256>, at, MxTile<true, 256>::SMEM_BYTES);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_gemm_kernel<true, 192>, at, MxTile<true, 192>::SMEM_BYTES);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_gemm_kernel<false, 128>, at, MxTile<false, 128>::SMEM_BYTES);
  if (e == cudaSuccess) e = cudaFuncSetAttribute(mx_gemm_kernel<false, 64>, at, MxTile<false, 64>::SMEM_BYTES);
  return e;
}

template <bool PAIR, int BN>
cudaError_t launch_shape(const MxGemm& p, int split, long long ctas, cudaStream_t st, const char** why) {
  using T = MxTile<PAIR, BN>;
  CUtensorMap ta, tb, sa, sb;
  if (!make_map_codes(&ta, p.a, BM) || !make_map_codes(&tb, p.b, T::ROWS_B) || !make_map_scales(&sa, p.a) || !make_map_scales(&sb, p.b))
    return *why = "tensor map creation failed for this shape", cudaErrorInvalidValue;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)ctas);
  cfg.blockDim = dim3(THREADS);
  cfg.dynamicSmemBytes = T::SMEM_BYTES;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = PAIR ? 2 : (unsigned)split;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = PAIR || split > 1 ? 2 : 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, mx_gemm_kernel<PAIR, BN>, ta, tb, sa, sb, p, split);
  if (e != cudaSuccess) *why = "kernel launch";
  return e;
}

}  // namespace

// Rows that the row-wise kernels take in one pass: as many as fill the machine with warps.
static int rows_per_pass(long long rows, long long col_tiles) {
  const long long fill = 148 * 8 * 8 / col_tiles;
  return (int)(fill < 1 ? 1 : fill < rows ? fill : rows);
}

cudaError_t mx_quantize(const void* x, int bf16, long long ld, int transpose, const MxView& q, cudaStream_t st) {
  const float* f = static_cast<const float*>(x);
  const __nv_bfloat16* h = static_cast<const __nv_bfloat16*>(x);
  if (transpose) {
    const dim3 grid((unsigned)((q.rows + 127) / 128 * 2 * q.col_tiles));
    return bf16 ? launch_k(mx_quantize_t_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, true, h, ld, q)
                : launch_k(mx_quantize_t_kernel<float>, grid, dim3(256), 0, st, true, f, ld, q);
  }
  if (bf16 && ((reinterpret_cast<uintptr_t>(x) | (uintptr_t)(ld * 2)) & 15) == 0) {
    const long long want = ((q.rows + 127) / 128 * 128 * q.col_tiles * 8 + 255) / 256;
    return launch_k(mx_quantize_blocks_kernel, dim3((unsigned)(want < 148 * 16 ? want : 148 * 16)), dim3(256), 0, st, true, h, ld, q);
  }
  const int pass = rows_per_pass((q.rows + 127) / 128 * 128, q.col_tiles);
  const dim3 grid((unsigned)((pass * q.col_tiles + 7) / 8));
  return bf16 ? launch_k(mx_quantize_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, true, h, ld, q, pass)
              : launch_k(mx_quantize_kernel<float>, grid, dim3(256), 0, st, true, f, ld, q, pass);
}

cudaError_t mx_dequantize(const MxView& q, void* out, int bf16, long long ld, cudaStream_t st) {
  const int pass = rows_per_pass(q.rows, q.col_tiles);
  const dim3 grid((unsigned)((pass * q.col_tiles + 7) / 8));
  return bf16 ? launch_k(mx_dequantize_kernel<__nv_bfloat16>, grid, dim3(256), 0, st, true, q, static_cast<__nv_bfloat16*>(out), ld, pass)
              : launch_k(mx_dequantize_kernel<float>, grid, dim3(256), 0, st, true, q, static_cast<float*>(out), ld, pass);
}

cudaError_t mx_gemm(const MxGemm& p, cudaStream_t st, const char** why) {
  *why = "";
  static std::atomic<int> known[MAX_DEVICES];
  int sms = 0;
  cudaError_t e = device_ready(known, set_attributes, &sms, why);
  if (e != cudaSuccess) return e;
  // The shape with the least work in sequence, in units of 0.34 us = 32 KiB on their way to an SM: a K block costs 35 and 31
  // KiB in the pairs' shapes, 34 and 26 in the single ones; what a round of tiles, the filling and draining and a cluster's
  // sum cost beside that is measured.  (fp32 results, us, with 256 / 192 / 128 / 64 columns: 4096 x 4096 x 32768 210 / 232 /
  // 284 / 400, 4096 x 4096 x 4096 38 / 34 / 40 / 56, 3000 x 3000 x 2048 17 / 17 / 15 / 20, 8192 x 4096 x 1024 41 / 44 / 36 /
  // 40, 1024 x 1024 x 4096 13 / 10 / 10 / 8.)
  const int kb = (int)p.a.col_tiles;
  auto tiles = [&](int tm, int tn) { return ((p.a.rows + tm - 1) / tm) * ((p.b.rows + tn - 1) / tn); };
  const long long pairs = tiles(256, 256), p192 = tiles(256, 192), t128 = tiles(128, 128), t64 = tiles(128, 64);
  int bn = 256, split = 1;
  auto rounds = [](long long n, int places) { return (double)((n + places - 1) / places); };
  double cost = rounds(pairs, sms / 2) * (kb * 1.1 + 8) + 17;
  const double c192 = rounds(p192, sms / 2) * (kb * 1.02 + 2 > 12.5 ? kb * 1.02 + 2 : 12.5) + 9;
  if (c192 < cost) {
    cost = c192;
    bn = 192;
  }
  for (int w = 128; w >= 64; w -= 64) {
    const long long t = w == 128 ? t128 : t64;
    const double unit = w == 128 ? 1.06 : 0.8, ramp = w == 128 ? 6 : 4;
    for (int k = 1; k <= 8 && k <= kb; ++k) {
      if (k > 1 && (t * k > sms || k * t > (long long)max_clusters(k, sms) * k)) break;
      const double c = (k == 1 ? rounds(t, sms) : 1.0) * (((kb + k - 1) / k) * unit + 1) + (k > 1 ? 2 : 1) * ramp;
      if (c < cost) {
        cost = c;
        bn = w;
        split = k;
      }
    }
  }
  if (bn == 192) return launch_shape<true, 192>(p, 1, 2 * (p192 < sms / 2 ? p192 : sms / 2), st, why);
  if (bn == 256) return launch_shape<true, 256>(p, 1, 2 * (pairs < sms / 2 ? pairs : sms / 2), st, why);
  const long long t = bn == 128 ? t128 : t64, want = t * split, ctas = want < sms ? want : sms;
  if (bn == 128) return launch_shape<false, 128>(p, split, ctas, st, why);
  return launch_shape<false, 64>(p, split, ctas, st, why);
}

cudaError_t mx_quantize_uploads(const Params& P, const void* x_bf16, int ld, int Bp, const MxView& q, cudaStream_t st) {
  const dim3 grid((unsigned)((q.rows + 127) / 128 * 2), (unsigned)(Bp / 128), (unsigned)P.G);
  mx_quantize_uploads_kernel<<<grid, 128, 0, st>>>(P, static_cast<const __nv_bfloat16*>(x_bf16), ld, Bp, q);
  return cudaGetLastError();
}

cudaError_t mx_upload_product(const MxView& a, const MxView& b, long long k0, int K, float* out, cudaStream_t st) {
  const dim3 grid((unsigned)((b.rows + 31) / 32), (unsigned)((a.rows + 7) / 8));
  mx_upload_product_kernel<<<grid, 256, 0, st>>>(a, b, k0, K, out);
  return cudaGetLastError();
}

}  // namespace gcada
