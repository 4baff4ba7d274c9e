// Orthogonalised updates: Newton-Schulz steps on a matrix (or a batch of equal ones), and the momentum update that
// uses them for a weight matrix.
//
//     X_0 = G / (||G||_F + eps),   X_{j+1} = a X_j + (b A + c A^2) X_j,   A = X_j X_j^T   (X_j^T X_j for tall G)
//
// The products run on the tensor cores with fp16 operands and fp32 accumulation.  Every matrix is stored times 2^10
// as a pair of fp16 numbers hi + lo (22 significant bits; the factor keeps lo clear of the subnormal range), so:
//   - precision HALF: the products take the hi parts only (one rounding of 2^-11 per operand element), while the
//     linear term a X_j takes hi + lo.  That term is the one that matters: a step multiplies small singular values,
//     and whatever was rounded into their directions, by a = 3.44, so a rounding of X itself would grow up to
//     3.44^4 = 140-fold; the products' own roundings only reach directions whose singular values are already of
//     order one.  (Simulated error after 5 steps, spectra i^-2 / rank 10 / Gaussian: 2e-4 / 4e-4 / 1.7e-3 of the
//     result's norm; with X kept in 11 bits 2e-2 / 4e-2 / 1.4e-3; in bf16 2e-1 / 3e-1 / 1.3e-2.)
//   - precision FULL: each product is lo*hi' + hi*lo' + hi*hi' (the smallest terms first), which is fp32 accuracy
//     (simulated 4e-7 .. 8e-6 of the result's norm on the same spectra, fp32 arithmetic itself 6e-6 .. 3e-5).
// A and b A + c A^2 are symmetric: only tiles that touch the upper triangle are computed, each element is written
// to both places, and the polynomial can be read as either operand.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <math.h>

#include <atomic>

#include "../../include/gcada.h"
#include "common.cuh"
#include "muon.h"
#include "tc.cuh"

namespace gcada {
namespace {

constexpr int BM = 128, BN = 256, BK = 64;
constexpr int BLK_BYTES = 64 * BK * 2;                 // one copy box: 64 x 64 fp16
constexpr int STAGE_BYTES = (BM + BN) * BK * 2;        // 48 KiB
constexpr int STAGES = 4;
constexpr int EPI_WARPS = 8;
constexpr int THREADS = 64 + 32 * EPI_WARPS;
constexpr int SMEM_BYTES = STAGES * STAGE_BYTES + 1024;
constexpr float SCALE = 1024.f;                        // stored value = SCALE * matrix element
constexpr float INV_SCALE = 1.f / 1024.f;
constexpr uint32_t IDESC = (1u << 4) | ((uint32_t)(BN >> 3) << 17) | ((uint32_t)(BM >> 4) << 24);  // fp16 operands, fp32 sum
constexpr int NORM_BLOCKS = 296;                       // partial sums of a matrix's squared norm

enum { OUT_SPLIT = 0, OUT_F32 = 1, OUT_BF16 = 2, OUT_UPDATE_F32 = 3, OUT_UPDATE_BF16 = 4 };

// A matrix whose norm is far below eps starts from an X_0 far below one, which fp16 pairs could not hold.  The stored
// iterate is then SCALE * X_j / rho_j with powers of two rho_0 ~ ||X_0||, rho_{j+1} = min(1, rho_j g), g >= |a|: an
// iterate that small grows by |a| a step.  For every other matrix all rho are 1.
constexpr int MAX_STEPS = 100;
enum { RHO_NONE = 0, RHO_POLY = 1, RHO_APPLY = 2, RHO_LAST = 3 };

struct NsGemm {
  int M, N, K, batch;
  int a_mn, b_mn;        // the operand's M / N index is the contiguous one of its array
  int sym;               // the result is symmetric (M == N)
  int terms;             // 1: hi*hi, 3: lo*hi + hi*lo + hi*hi
  float c_src, c_acc;    // value = c_src * src + c_acc * accumulator, times factors of the iterate's own scale rho:
  int rho_mode;          // RHO_*
  const float* rho;      // [batch][MAX_STEPS + 1]; entry `step_no` is that of the iterate the step starts from
  int step_no;
  const __half* src;     // [batch][2][.][ld_src] hi / lo planes, or null
  long long ld_src, src_plane;
  __half* dst;           // OUT_SPLIT: the same layout
  long long ld_dst, dst_plane;
  int write_lo;
  int out;               // OUT_*
  void* user;            // OUT_F32 ... : user's matrix
  long long ld_user, user_stride;
  float decay, step;     // OUT_UPDATE_*: w <- decay * w - step * value
  int* err;
};

// Tiles of 128 x 256; of a symmetric result only those with an element on or above the diagonal: row mt starts at
// column tile mt / 2.
__device__ __forceinline__ void tile_of(int u, int tiles_m, int tiles_n, int sym, int& mt, int& nt) {
  if (!sym) {
    mt = u / tiles_n;
    nt = u - mt * tiles_n;
    return;
  }
  for (mt = 0; mt < tiles_m; ++mt) {
    const int w = tiles_n - mt / 2;
    if (u < w) break;
    u -= w;
  }
  nt = mt / 2 + u;
}
__host__ __device__ inline int tile_count(int tiles_m, int tiles_n, int sym) {
  if (!sym) return tiles_m * tiles_n;
  int n = 0;
  for (int mt = 0; mt < tiles_m; ++mt) n += tiles_n - mt / 2;
  return n;
}

__device__ __forceinline__ void tc_mma_f16(uint32_t tmem_c, uint64_t da, uint64_t db, uint32_t idesc, uint32_t accum) {
  tc_mma_bf16(tmem_c, da, db, idesc, accum);  // kind::f16 covers both 16-bit types; the descriptor says which
}

// v[0..7] += or -> helpers on eight consecutive columns
__device__ __forceinline__ void load_split8(const __half* hi, const __half* lo, float (&f)[8]) {
  const uint4 h = *reinterpret_cast<const uint4*>(hi), l = *reinterpret_cast<const uint4*>(lo);
  const uint32_t hw[4] = {h.x, h.y, h.z, h.w}, lw[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&hw[i]));
    const float2 b = __half22float2(*reinterpret_cast<const __half2*>(&lw[i]));
    f[2 * i] = a.x + b.x;
    f[2 * i + 1] = a.y + b.y;
  }
}
__device__ __forceinline__ void split8(const float (&f)[8], uint4& h, uint4& l) {
  uint32_t hw[4], lw[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const __half2 a = __floats2half2_rn(f[2 * i], f[2 * i + 1]);
    const float2 b = __half22float2(a);
    const __half2 c = __floats2half2_rn(f[2 * i] - b.x, f[2 * i + 1] - b.y);
    hw[i] = *reinterpret_cast<const uint32_t*>(&a);
    lw[i] = *reinterpret_cast<const uint32_t*>(&c);
  }
  h = make_uint4(hw[0], hw[1], hw[2], hw[3]);
  l = make_uint4(lw[0], lw[1], lw[2], lw[3]);
}

__global__ void __launch_bounds__(THREADS, 1) ns_gemm_kernel(const __grid_constant__ CUtensorMap tmA,
                                                             const __grid_constant__ CUtensorMap tmB, const NsGemm a) {
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  __shared__ uint64_t full_bar[STAGES], empty_bar[STAGES], tfull_bar[2], tempty_bar[2];
  __shared__ uint32_t tmem_base_sm;
  unsigned char* tiles = reinterpret_cast<unsigned char*>(((uintptr_t)smem_raw + 1023) & ~(uintptr_t)1023);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int tiles_m = (a.M + BM - 1) / BM, tiles_n = (a.N + BN - 1) / BN;
  const int per = tile_count(tiles_m, tiles_n, a.sym), total = per * a.batch;
  const int nkb = (a.K + BK - 1) / BK, steps = nkb * a.terms;
  const int n_local = (int)blockIdx.x < total ? (total - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x : 0;

  if (threadIdx.x == 0) {
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(&full_bar[s], 1);
      mbar_init(&empty_bar[s], 1);
    }
    for (int s = 0; s < 2; ++s) {
      mbar_init(&tfull_bar[s], 1);
      mbar_init(&tempty_bar[s], EPI_WARPS);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base_sm)),
                 "r"(512u)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = tmem_base_sm;

  if (warp == 0) {
    if (lane == 0) {
      bool ok = true;
      int it = 0;
      for (int i = 0; i < n_local && ok; ++i) {
        const int u = (int)blockIdx.x + i * (int)gridDim.x, b = u / per;
        int mt, nt;
        tile_of(u - b * per, tiles_m, tiles_n, a.sym, mt, nt);
        for (int s0 = 0; s0 < steps; ++s0, ++it) {
          const int t = a.terms == 1 ? 2 : s0 / nkb, kc = (a.terms == 1 ? s0 : s0 - t * nkb) * BK;
          const int zA = 2 * b + (t == 0 ? 1 : 0), zB = 2 * b + (t == 1 ? 1 : 0);  // plane 0 = hi, 1 = lo
          const int s = it % STAGES;
          ok = mbar_spin_bounded(&empty_bar[s], (uint32_t)(((it / STAGES) & 1) ^ 1));
          if (!ok) break;
          unsigned char* sa = tiles + (size_t)s * STAGE_BYTES;
          mbar_expect_tx(&full_bar[s], STAGE_BYTES);
#pragma unroll
          for (int j = 0; j < BM / 64; ++j) {
            const int r = mt * BM + j * 64;
            tma_load_3d(sa + j * BLK_BYTES, &tmA, a.a_mn ? r : kc, a.a_mn ? kc : r, zA, &full_bar[s]);
          }
#pragma unroll
          for (int j = 0; j < BN / 64; ++j) {
            const int r = nt * BN + j * 64;
            tma_load_3d(sa + BM * BK * 2 + j * BLK_BYTES, &tmB, a.b_mn ? r : kc, a.b_mn ? kc : r, zB, &full_bar[s]);
          }
        }
      }
      if (!ok) raise_error(a.err);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = IDESC | (a.a_mn ? 1u << 15 : 0u) | (a.b_mn ? 1u << 16 : 0u);
      const uint64_t ka = a.a_mn ? 128u : 2u, kb = a.b_mn ? 128u : 2u;  // descriptor step of 16 K values
      bool ok = true;
      int it = 0;
      for (int i = 0; i < n_local && ok; ++i) {
        const int slot = i & 1;
        ok = mbar_spin_bounded(&tempty_bar[slot], (uint32_t)(((i >> 1) & 1) ^ 1));
        if (!ok) break;
        tc_fence_after();
        for (int s0 = 0; s0 < steps && ok; ++s0, ++it) {
          const int s = it % STAGES;
          ok = mbar_spin_bounded(&full_bar[s], (uint32_t)((it / STAGES) & 1));
          if (!ok) break;
          tc_fence_after();
          const uint32_t sa = smem_u32(tiles + (size_t)s * STAGE_BYTES);
          const uint64_t da = a.a_mn ? make_desc_mn(sa) : make_desc(sa);
          const uint64_t db = a.b_mn ? make_desc_mn(sa + BM * BK * 2) : make_desc(sa + BM * BK * 2);
#pragma unroll
          for (int kk = 0; kk < BK / 16; ++kk)
            tc_mma_f16(tmem_base + (uint32_t)(slot * BN), da + kk * ka, db + kk * kb, idesc, (s0 | kk) != 0 ? 1u : 0u);
          tc_commit(&empty_bar[s]);
        }
        if (ok) tc_commit(&tfull_bar[slot]);
      }
      if (!ok) raise_error(a.err);
    }
  } else {
    // epilogue: warp w may touch TMEM lanes 32*(w%4) .. +31; the two warps of a quadrant split the columns
    const int quad = warp & 3, half = (warp - 2) >> 2;
    bool ok = true;
    for (int i = 0; i < n_local; ++i) {
      const int slot = i & 1;
      const int u = (int)blockIdx.x + i * (int)gridDim.x, b = u / per;
      int mt, nt;
      tile_of(u - b * per, tiles_m, tiles_n, a.sym, mt, nt);
      const int m = mt * BM + quad * 32 + lane;
      if (ok) {
        ok = mbar_wait_bounded(&tfull_bar[slot], (uint32_t)((i >> 1) & 1));
        ok = __all_sync(0xffffffffu, ok);
      }
      if (!ok) continue;
      tc_fence_after();
      const uint32_t tbase = tmem_base + ((uint32_t)(quad * 32) << 16) + (uint32_t)(slot * BN);
      const __half* src = a.src ? a.src + (long long)b * 2 * a.src_plane + (long long)m * a.ld_src : nullptr;
      __half* dst = a.dst + (long long)b * 2 * a.dst_plane;
      float c_src = a.c_src, c_acc = a.c_acc;
      if (a.rho_mode != RHO_NONE) {
        const float* r = a.rho + (long long)b * (MAX_STEPS + 1) + a.step_no;
        const float r0 = r[0], k = a.rho_mode == RHO_APPLY ? r0 / r[1] : (a.rho_mode == RHO_LAST ? r0 : r0 * r0);
        c_src *= k;
        c_acc *= a.rho_mode == RHO_POLY ? k * k : k;
      }
      auto chunk = [&](const uint32_t (&v)[32], int c) {
        const int n0 = nt * BN + c;
        if (m >= a.M || n0 >= a.N) return;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int n = n0 + 8 * g;
          if (n >= a.N) break;
          float f[8];
          if (src) {
            load_split8(src + n, src + a.src_plane + n, f);
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = c_src * f[j] + c_acc * __uint_as_float(v[8 * g + j]);
          } else {
#pragma unroll
            for (int j = 0; j < 8; ++j) f[j] = c_acc * __uint_as_float(v[8 * g + j]);
          }
          if (a.out == OUT_SPLIT) {
            uint4 h, l;
            split8(f, h, l);
            if (!a.sym) {
              *reinterpret_cast<uint4*>(dst + (long long)m * a.ld_dst + n) = h;
              if (a.write_lo) *reinterpret_cast<uint4*>(dst + a.dst_plane + (long long)m * a.ld_dst + n) = l;
            } else {
              const __half* h8 = reinterpret_cast<const __half*>(&h);
              const __half* l8 = reinterpret_cast<const __half*>(&l);
              if (n >= m) {
                *reinterpret_cast<uint4*>(dst + (long long)m * a.ld_dst + n) = h;
                if (a.write_lo) *reinterpret_cast<uint4*>(dst + a.dst_plane + (long long)m * a.ld_dst + n) = l;
              }
#pragma unroll
              for (int j = 0; j < 8; ++j) {
                if (n + j >= a.N || n + j < m) continue;  // below the diagonal: the mirrored element is written
                if (n < m) {
                  dst[(long long)m * a.ld_dst + n + j] = h8[j];
                  if (a.write_lo) dst[a.dst_plane + (long long)m * a.ld_dst + n + j] = l8[j];
                }
                if (n + j > m) {
                  dst[(long long)(n + j) * a.ld_dst + m] = h8[j];
                  if (a.write_lo) dst[a.dst_plane + (long long)(n + j) * a.ld_dst + m] = l8[j];
                }
              }
            }
          } else if (a.out == OUT_F32 || a.out == OUT_UPDATE_F32) {
            float* o = static_cast<float*>(a.user) + (long long)b * a.user_stride + (long long)m * a.ld_user + n;
            const bool upd = a.out == OUT_UPDATE_F32;
            if (n + 8 <= a.N && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
#pragma unroll
              for (int j = 0; j < 8; j += 4) {
                float4 w = make_float4(f[j], f[j + 1], f[j + 2], f[j + 3]);
                if (upd) {
                  const float4 p = *reinterpret_cast<const float4*>(o + j);
                  w = make_float4(a.decay * p.x - a.step * w.x, a.decay * p.y - a.step * w.y,
                                  a.decay * p.z - a.step * w.z, a.decay * p.w - a.step * w.w);
                }
                *reinterpret_cast<float4*>(o + j) = w;
              }
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (n + j < a.N) o[j] = upd ? a.decay * o[j] - a.step * f[j] : f[j];
            }
          } else {
            __nv_bfloat16* o =
                static_cast<__nv_bfloat16*>(a.user) + (long long)b * a.user_stride + (long long)m * a.ld_user + n;
            const bool upd = a.out == OUT_UPDATE_BF16;
            if (n + 8 <= a.N && (reinterpret_cast<uintptr_t>(o) & 15) == 0) {
              if (upd) {
                const uint4 p = *reinterpret_cast<const uint4*>(o);
                const uint32_t pw[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
                for (int j = 0; j < 8; ++j)
                  f[j] = a.decay * __uint_as_float(j & 1 ? pw[j >> 1] & 0xffff0000u : pw[j >> 1] << 16) - a.step * f[j];
              }
              uint32_t w[4];
#pragma unroll
              for (int j = 0; j < 4; ++j) {
                const __nv_bfloat162 t = __floats2bfloat162_rn(f[2 * j], f[2 * j + 1]);
                w[j] = *reinterpret_cast<const uint32_t*>(&t);
              }
              *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j)
                if (n + j < a.N)
                  o[j] = __float2bfloat16_rn(upd ? a.decay * __bfloat162float(o[j]) - a.step * f[j] : f[j]);
            }
          }
        }
      };
      for (int c = half * (BN / 2); c < (half + 1) * (BN / 2); c += 32) {
        uint32_t v[32];
        tc_ld32_issue(tbase + (uint32_t)c, v);
        tc_ld_wait();
        chunk(v, c);
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&tempty_bar[slot]);
    }
    if (!ok && lane == 0) raise_error(a.err);
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem_base), "r"(512u) : "memory");
  }
}

// ----------------------------------------------------------------- source: a matrix, or the momentum's look-ahead
struct NsSource {
  const void* g;  // float or bf16, row stride ld, matrix stride
  long long ld, stride;
  int bf16;
  float* m;       // momentum (row stride ld_m), or null: the matrix itself
  long long ld_m, m_stride;
  float beta, omb;
  int nesterov;
  int rows, cols;
};

template <typename T>
__device__ __forceinline__ void load8(const T* p, int n, float (&f)[8]) {
  if (n == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
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
__device__ __forceinline__ void store8(float* p, int n, const float (&f)[8]) {
  if (n == 8 && (reinterpret_cast<uintptr_t>(p) & 15) == 0) {
    *reinterpret_cast<float4*>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *(reinterpret_cast<float4*>(p) + 1) = make_float4(f[4], f[5], f[6], f[7]);
  } else {
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (j < n) p[j] = f[j];
  }
}

// Eight elements of the matrix that is orthogonalised, from column c of row r.  FIRST: the momentum is moved first.
template <bool FIRST>
__device__ __forceinline__ void source8(const NsSource& s, int b, int r, int c, float (&f)[8]) {
  const int n = s.cols - c < 8 ? s.cols - c : 8;
  const long long o = (long long)b * s.stride + (long long)r * s.ld + c;
  if (s.bf16)
    load8(static_cast<const __nv_bfloat16*>(s.g) + o, n, f);
  else
    load8(static_cast<const float*>(s.g) + o, n, f);
  if (s.m) {
    float m[8];
    float* pm = s.m + (long long)b * s.m_stride + (long long)r * s.ld_m + c;
    load8(pm, n, m);
    if (FIRST) {
#pragma unroll
      for (int j = 0; j < 8; ++j) m[j] = s.beta * m[j] + s.omb * f[j];
      store8(pm, n, m);
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = s.nesterov ? s.omb * f[j] + s.beta * m[j] : m[j];
  }
}

// Squared Frobenius norm in doubles, NORM_BLOCKS partial sums per matrix (fixed order: bitwise reproducible).
__global__ void __launch_bounds__(256) ns_norm_kernel(const NsSource s, double* part) {
  __shared__ double scratch[40];
  const int b = blockIdx.y, cpr = (s.cols + 7) / 8;
  const long long total = (long long)cpr * s.rows;
  double acc = 0.0;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int r = (int)(i / cpr), c = (int)(i - (long long)r * cpr) * 8;
    float f[8];
    source8<true>(s, b, r, c, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) acc += (double)f[j] * (double)f[j];
  }
  acc = block_sum(acc, scratch);
  if (threadIdx.x == 0) part[(long long)b * gridDim.x + blockIdx.x] = acc;
}

// X_0 = source / (norm + eps), stored as SCALE * X_0 / rho_0 = hi + lo; and the rho_j.
__global__ void __launch_bounds__(256) ns_scale_kernel(const NsSource s, const double* part, int n_part, double eps,
                                                       float growth, int steps, float* rho, __half* x, long long ld,
                                                       long long plane) {
  __shared__ double scratch[40];
  const int b = blockIdx.y, cpr = (s.cols + 7) / 8;
  const long long total = (long long)cpr * s.rows;
  double ss = 0.0;
  for (int i = threadIdx.x; i < n_part; i += 256) ss += part[(long long)b * n_part + i];
  ss = block_sum(ss, scratch);
  const double norm = sqrt(ss), size = norm / (norm + eps);  // size = ||X_0||
  const double rho0 = size > 0.0 && size < 0.0625 ? exp2(floor(log2(size))) : 1.0;
  const double k = (double)SCALE / rho0 / (norm + eps);
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    double r = rho0;
    for (int j = 0; j <= steps; ++j, r = r * growth < 1.0 ? r * growth : 1.0)
      rho[(long long)b * (MAX_STEPS + 1) + j] = (float)r;
  }
  __half* hi = x + (long long)b * 2 * plane;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int r = (int)(i / cpr), c = (int)(i - (long long)r * cpr) * 8;
    float f[8];
    source8<false>(s, b, r, c, f);
#pragma unroll
    for (int j = 0; j < 8; ++j) f[j] = (float)((double)f[j] * k);
    uint4 h, l;
    split8(f, h, l);
    *reinterpret_cast<uint4*>(hi + (long long)r * ld + c) = h;
    *reinterpret_cast<uint4*>(hi + plane + (long long)r * ld + c) = l;
  }
}

// No steps at all: the normalised matrix itself.
__global__ void __launch_bounds__(256) ns_copy_kernel(const NsGemm a) {
  const int b = blockIdx.y;
  const long long total = (long long)a.M * a.N;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < total; i += (long long)gridDim.x * 256) {
    const int r = (int)(i / a.N), c = (int)(i - (long long)r * a.N);
    const __half* p = a.src + (long long)b * 2 * a.src_plane + (long long)r * a.ld_src + c;
    const float v = a.c_src * a.rho[(long long)b * (MAX_STEPS + 1)] * (__half2float(p[0]) + __half2float(p[a.src_plane]));
    const long long o = (long long)b * a.user_stride + (long long)r * a.ld_user + c;
    if (a.out == OUT_F32 || a.out == OUT_UPDATE_F32) {
      float* w = static_cast<float*>(a.user) + o;
      *w = a.out == OUT_F32 ? v : a.decay * *w - a.step * v;
    } else {
      __nv_bfloat16* w = static_cast<__nv_bfloat16*>(a.user) + o;
      *w = __float2bfloat16_rn(a.out == OUT_BF16 ? v : a.decay * __bfloat162float(*w) - a.step * v);
    }
  }
}

// ----------------------------------------------------------------- host
// fp16 array [planes][rows][cols], row stride ld elements; boxes of 64 x 64, 128-byte swizzle, zero fill outside.
bool make_map_f16(CUtensorMap* tm, const void* base, long long cols, long long rows, long long planes, long long ld,
                  long long plane) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)plane * 2};
  cuuint32_t box[3] = {64, 64, 1};
  cuuint32_t es[3] = {1, 1, 1};
  return fn(tm, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, es,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct NsLayout {
  int r, c;                // short and long side
  long long ld_x, plane_x;  // X: [batch][2][rows][ld_x]
  long long ld_s, plane_s;  // A, polynomial: [batch][2][r][ld_s]
  size_t x0, x1, s0, s1, part, rho, bytes;
};

NsLayout layout(int batch, int rows, int cols) {
  NsLayout L{};
  L.r = rows < cols ? rows : cols;
  L.c = rows < cols ? cols : rows;
  L.ld_x = (cols + 7) / 8 * 8;
  L.plane_x = L.ld_x * rows;
  L.ld_s = (L.r + 7) / 8 * 8;
  L.plane_s = L.ld_s * L.r;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t o = at;
    at += (bytes + 255) / 256 * 256;
    return o;
  };
  L.part = take(sizeof(double) * NORM_BLOCKS * (size_t)batch);
  L.rho = take(sizeof(float) * (MAX_STEPS + 1) * (size_t)batch);
  L.x0 = take((size_t)batch * 2 * L.plane_x * 2);
  L.x1 = take((size_t)batch * 2 * L.plane_x * 2);
  L.s0 = take((size_t)batch * 2 * L.plane_s * 2);
  L.s1 = take((size_t)batch * 2 * L.plane_s * 2);
  L.bytes = at;
  return L;
}

cudaError_t set_attributes() {
  return cudaFuncSetAttribute(ns_gemm_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SMEM_BYTES);
}

cudaError_t launch_ns_gemm(const CUtensorMap& ta, const CUtensorMap& tb, const NsGemm& a, int sms, cudaStream_t st) {
  const long long units =
      (long long)tile_count((a.M + BM - 1) / BM, (a.N + BN - 1) / BN, a.sym) * a.batch;
  const int ctas = (int)(units < sms ? units : sms);
  ns_gemm_kernel<<<ctas, THREADS, SMEM_BYTES, st>>>(ta, tb, a);
  return cudaGetLastError();
}

}  // namespace

size_t ns_work_bytes(int batch, int rows, int cols) { return layout(batch, rows, cols).bytes; }

// Everything an orthogonalisation enqueues.  `why` names the step that failed.
cudaError_t ns_run(const NsProblem& p, void* work, cudaStream_t st, const char** why, int* launches) {
  *why = "";
  static std::atomic<int> known[MAX_DEVICES];
  int sms = 0;
  cudaError_t e = device_ready(known, set_attributes, &sms, why);
  if (e != cudaSuccess) return e;
  const NsLayout L = layout(p.batch, p.rows, p.cols);
  char* base = static_cast<char*>(work);
  double* part = reinterpret_cast<double*>(base + L.part);
  float* rho = reinterpret_cast<float*>(base + L.rho);
  __half* X[2] = {reinterpret_cast<__half*>(base + L.x0), reinterpret_cast<__half*>(base + L.x1)};
  __half* A = reinterpret_cast<__half*>(base + L.s0);
  __half* Q = reinterpret_cast<__half*>(base + L.s1);
  CUtensorMap tx[2], ta, tq;
  bool ok = make_map_f16(&ta, A, L.r, L.r, 2LL * p.batch, L.ld_s, L.plane_s) &&
            make_map_f16(&tq, Q, L.r, L.r, 2LL * p.batch, L.ld_s, L.plane_s);
  for (int i = 0; i < 2 && ok; ++i) ok = make_map_f16(&tx[i], X[i], p.cols, p.rows, 2LL * p.batch, L.ld_x, L.plane_x);
  if (!ok) return *why = "tensor map creation failed for this shape", cudaErrorInvalidValue;

  NsSource s{};
  s.g = p.g;
  s.ld = p.ld_g;
  s.stride = p.stride_g;
  s.bf16 = p.g_bf16;
  s.m = p.m;
  s.ld_m = p.ld_m;
  s.beta = (float)p.beta;
  s.omb = (float)(1.0 - p.beta);
  s.nesterov = p.nesterov;
  s.rows = p.rows;
  s.cols = p.cols;
  const long long chunks = (long long)((p.cols + 7) / 8) * p.rows;
  const long long want = (chunks + 255) / 256;
  const int nb = (int)(want < NORM_BLOCKS ? want : NORM_BLOCKS);
  float growth = 1.f;  // power of two >= max(1, |a|)
  while (growth < fabs(p.coef[0])) growth *= 2.f;
  ns_norm_kernel<<<dim3(nb, p.batch), 256, 0, st>>>(s, part);
  ns_scale_kernel<<<dim3(nb, p.batch), 256, 0, st>>>(s, part, nb, p.eps, growth, p.steps, rho, X[0], L.ld_x,
                                                         L.plane_x);
  if ((e = cudaGetLastError()) != cudaSuccess) return *why = "kernel launch", e;
  int n = 2;

  const bool tall = p.rows > p.cols;
  NsGemm f{};  // the last product's (or the copy's) way to the user's matrix
  f.batch = p.batch;
  f.M = p.rows;
  f.N = p.cols;
  f.out = p.w_update ? (p.o_bf16 ? OUT_UPDATE_BF16 : OUT_UPDATE_F32) : (p.o_bf16 ? OUT_BF16 : OUT_F32);
  f.user = p.o;
  f.ld_user = p.ld_o;
  f.user_stride = p.stride_o;
  f.decay = (float)p.decay;
  f.step = (float)p.step;
  f.ld_src = L.ld_x;
  f.src_plane = L.plane_x;
  f.err = p.err;
  f.rho = rho;
  for (int j = 0; j < p.steps; ++j) {
    const int cur = j & 1;
    NsGemm g{};
    g.batch = p.batch;
    g.terms = p.full ? 3 : 1;
    g.err = p.err;
    g.rho = rho;
    g.step_no = j;
    // A
    g.M = g.N = L.r;
    g.K = L.c;
    g.a_mn = g.b_mn = tall;
    g.sym = 1;
    g.c_acc = INV_SCALE;
    g.dst = A;
    g.ld_dst = L.ld_s;
    g.dst_plane = L.plane_s;
    g.write_lo = 1;
    if ((e = launch_ns_gemm(tx[cur], tx[cur], g, sms, st)) != cudaSuccess) return *why = "kernel launch", e;
    // b A + c A^2
    g.K = L.r;
    g.a_mn = g.b_mn = 0;
    g.src = A;
    g.ld_src = L.ld_s;
    g.src_plane = L.plane_s;
    g.c_src = (float)p.coef[1];
    g.c_acc = (float)p.coef[2] * INV_SCALE;
    g.rho_mode = RHO_POLY;
    g.dst = Q;
    g.write_lo = p.full;
    if ((e = launch_ns_gemm(ta, ta, g, sms, st)) != cudaSuccess) return *why = "kernel launch", e;
    // a X + (.) X, or a X + X (.) for a tall matrix
    const bool last = j == p.steps - 1;
    NsGemm h = last ? f : g;
    h.terms = g.terms;
    h.step_no = j;
    h.rho_mode = last ? RHO_LAST : RHO_APPLY;
    h.M = p.rows;
    h.N = p.cols;
    h.K = L.r;
    h.a_mn = 0;
    h.b_mn = tall ? 0 : 1;
    h.sym = 0;
    h.src = X[cur];
    h.ld_src = L.ld_x;
    h.src_plane = L.plane_x;
    const float k = last ? INV_SCALE : 1.f;
    h.c_src = (float)p.coef[0] * k;
    h.c_acc = INV_SCALE * k;
    if (!last) {
      h.dst = X[cur ^ 1];
      h.ld_dst = L.ld_x;
      h.dst_plane = L.plane_x;
      h.write_lo = 1;
    }
    if ((e = launch_ns_gemm(tall ? tx[cur] : tq, tall ? tq : tx[cur], h, sms, st)) != cudaSuccess)
      return *why = "kernel launch", e;
    n += 3;
  }
  if (p.steps == 0) {
    f.src = X[0];
    f.c_src = INV_SCALE;
    ns_copy_kernel<<<dim3(nb, p.batch), 256, 0, st>>>(f);
    if ((e = cudaGetLastError()) != cudaSuccess) return *why = "kernel launch", e;
    n += 1;
  }
  if (launches) *launches = n;
  return cudaSuccess;
}

}  // namespace gcada
