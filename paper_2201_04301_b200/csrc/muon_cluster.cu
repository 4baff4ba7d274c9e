// Newton-Schulz steps of a narrow matrix (short side up to 64) in one launch: the long side is dealt out to the CTAs
// of a thread-block cluster, which keep their slices of X in shared memory for all steps, in fp32 throughout.
//
// A step: every CTA forms its slice's share of A = X X^T, one cluster barrier, every CTA adds up all shares (read
// through distributed shared memory, in rank order: bitwise reproducible), forms b A + c A^2 for itself and applies
// it to its slice.  Shares are double-buffered, so one barrier a step is enough.  Bound: latency - each phase is
// some hundred cycles of FMAs between barriers.  As separate tensor-core launches the same steps cost 4 to 5 us per
// product however small it is (10 x 200: 76 us, 64 x 512: 98 us).
#include <cuda_bf16.h>

#include "common.cuh"
#include "muon.h"
#include "tc.cuh"

namespace gcada {
namespace {

constexpr int NC_THREADS = 512;
constexpr int NC_MAX_R = 64;
constexpr int NC_MAX_SMEM = 220 * 1024;

struct NcArgs {
  int r, c, cs;   // short and long side; columns of the long side per CTA
  int rp, csp;    // padded row length (4 x odd: rows start in different banks) and slice length (multiple of 4)
  int tall, csize, steps;
  float a, b, cc;
  double eps;
};

__device__ __forceinline__ float cluster_load_f32(uint32_t base, uint32_t rank, int index) {
  return cluster_load(cluster_map(base, rank) + 4u * (uint32_t)index);
}

// out[i][j] (symmetric, n x n in rows of rp) = sum over k < K of M[k][i] M[k][j] (M in rows of rp) times s_acc, plus
// s_src * add[i][j].  4 x 4 values a thread; `kp` neighbouring lanes share the sum over k.
__device__ void symmetric_product(const float* M, int K, int rp, float* out, const float* add, float s_src, float s_acc) {
  const int nt = rp >> 2, tiles = nt * (nt + 1) / 2;
  int kp = 1;
  while (kp < 32 && tiles * kp * 2 <= NC_THREADS && kp * 4 <= K) kp *= 2;
  for (int base = 0; base < tiles * kp; base += NC_THREADS) {
    const int id = base + (int)threadIdx.x, tile = id / kp, part = id % kp;
    const bool on = tile < tiles;
    int ti = 0, tj = 0;
    if (on) {
      int u = tile;
      while (u >= nt - ti) u -= nt - ti, ++ti;
      tj = ti + u;
    }
    float acc[4][4] = {};
    if (on) {
#pragma unroll 4
      for (int k = part; k < K; k += kp) {
        const float4 x = *reinterpret_cast<const float4*>(M + k * rp + 4 * ti), y = *reinterpret_cast<const float4*>(M + k * rp + 4 * tj);
        const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) acc[i][j] += xs[i] * ys[j];
      }
    }
    for (int o = 1; o < kp; o *= 2) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += __shfl_xor_sync(0xffffffffu, acc[i][j], o);
    }
    if (on && part == 0) {
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int p = (4 * ti + i) * rp + 4 * tj + j;
          const float v = s_acc * acc[i][j] + (add ? s_src * add[p] : 0.f);
          out[p] = v;
          out[(4 * tj + j) * rp + 4 * ti + i] = v;
        }
    }
  }
}

__global__ void __launch_bounds__(NC_THREADS, 1) ns_cluster_kernel(const NsSource s, const NsSink o, const NcArgs n) {
  extern __shared__ __align__(16) float sm[];
  __shared__ double scratch[40];
  __shared__ double share[1];
  const int rp = n.rp, sq = rp * rp;
  float* X = sm;                       // [csp][rp]: X transposed, element (i, k) at k * rp + i
  float* Y = X + (size_t)n.csp * rp;   // the next iterate
  float* part[2] = {Y + (size_t)n.csp * rp, Y + (size_t)n.csp * rp + sq};  // this CTA's share of A
  float* A = part[1] + sq;
  float* Q = A + sq;
  const int b = blockIdx.x / n.csize, rank = n.csize > 1 ? (int)cluster_rank() : 0;
  const int k0 = rank * n.cs, kn = max(0, min(n.cs, n.c - k0));
  const int tid = threadIdx.x;

  // the slice, momentum moved on the way; squares in doubles
  for (int e = tid; e < n.csp * rp; e += NC_THREADS) X[e] = 0.f;
  __syncthreads();
  const int count = kn * n.r;
  double ss = 0.0;
  for (int e = tid; e < count; e += NC_THREADS) {
    const int major = n.tall ? n.r : kn, q = e / major, w = e - q * major;
    const int i = n.tall ? w : q, k = n.tall ? q : w;
    const long long row = n.tall ? k0 + k : i, col = n.tall ? i : k0 + k;
    const long long at = (long long)b * s.stride + row * s.ld + col;
    float v = s.bf16 ? __bfloat162float(static_cast<const __nv_bfloat16*>(s.g)[at]) : static_cast<const float*>(s.g)[at];
    if (s.m) {
      float* pm = s.m + (long long)b * s.m_stride + row * s.ld_m + col;
      const float m = s.beta * *pm + s.omb * v;
      *pm = m;
      v = s.nesterov ? s.omb * v + s.beta * m : m;
    }
    X[k * rp + i] = v;
    ss += (double)v * (double)v;
  }
  ss = block_sum(ss, scratch);
  if (n.csize > 1) {
    if (tid == 0) share[0] = ss;
    cluster_sync();
    if (tid == 0) {
      ss = 0.0;
      for (int p = 0; p < n.csize; ++p) {
        double v;
        asm volatile("ld.shared::cluster.f64 %0, [%1];" : "=d"(v) : "r"(cluster_map(smem_u32(share), (uint32_t)p)) : "memory");
        ss += v;
      }
      scratch[0] = ss;
    }
    __syncthreads();
    ss = scratch[0];
  }
  const double norm = sqrt(ss) + n.eps;
  for (int e = tid; e < n.csp * rp; e += NC_THREADS) X[e] = (float)((double)X[e] / norm);
  __syncthreads();

  const int nt = rp >> 2, kgroups = (kn + 3) >> 2, items = kgroups * nt;
  int kp = 1;  // lanes that share an item's sum over j
  while (kp < 16 && items * kp * 2 <= NC_THREADS && kp * 2 <= nt) kp *= 2;
  for (int step = 0; step < n.steps; ++step) {
    float* mine = n.csize > 1 ? part[step & 1] : A;
    symmetric_product(X, kn, rp, mine, nullptr, 0.f, 1.f);
    if (n.csize > 1) {
      cluster_sync();
      const uint32_t from = smem_u32(mine);
      for (int e = tid; e < sq; e += NC_THREADS) {
        float v = 0.f;
        for (int p = 0; p < n.csize; ++p) v += cluster_load_f32(from, (uint32_t)p, e);
        A[e] = v;
      }
    }
    __syncthreads();
    symmetric_product(A, n.r, rp, Q, A, n.b, n.cc);
    __syncthreads();
    // Y = a X + X Q: 4 columns of the slice x 4 rows a thread
    for (int base = 0; base < items * kp; base += NC_THREADS) {
      const int id = base + tid, item = id / kp, p = id % kp;
      const bool on = item < items;
      const int kg = on ? item / nt : 0, ti = on ? item - kg * nt : 0;
      const float* x = X + (size_t)kg * 4 * rp;
      float acc[4][4] = {};
      if (on) {
        for (int j = 4 * p; j < rp; j += 4 * kp) {
          float4 xv[4], qv[4];
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            xv[t] = *reinterpret_cast<const float4*>(x + t * rp + j);
            qv[t] = *reinterpret_cast<const float4*>(Q + (j + t) * rp + 4 * ti);
          }
#pragma unroll
          for (int t = 0; t < 4; ++t) {
            const float xs[4] = {xv[t].x, xv[t].y, xv[t].z, xv[t].w};
#pragma unroll
            for (int u = 0; u < 4; ++u) {
              acc[t][0] += xs[u] * qv[u].x;
              acc[t][1] += xs[u] * qv[u].y;
              acc[t][2] += xs[u] * qv[u].z;
              acc[t][3] += xs[u] * qv[u].w;
            }
          }
        }
      }
      for (int w = 1; w < kp; w *= 2) {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int u = 0; u < 4; ++u) acc[t][u] += __shfl_xor_sync(0xffffffffu, acc[t][u], w);
      }
      if (on && p == 0) {
#pragma unroll
        for (int t = 0; t < 4; ++t) {
          const float4 v = *reinterpret_cast<const float4*>(x + t * rp + 4 * ti);
          *reinterpret_cast<float4*>(Y + (size_t)(kg * 4 + t) * rp + 4 * ti) =
              make_float4(n.a * v.x + acc[t][0], n.a * v.y + acc[t][1], n.a * v.z + acc[t][2], n.a * v.w + acc[t][3]);
        }
      }
    }
    __syncthreads();
    float* t = X;
    X = Y;
    Y = t;
  }

  for (int e = tid; e < count; e += NC_THREADS) {
    const int major = n.tall ? n.r : kn, q = e / major, w = e - q * major;
    const int i = n.tall ? w : q, k = n.tall ? q : w;
    const long long row = n.tall ? k0 + k : i, col = n.tall ? i : k0 + k;
    const long long at = (long long)b * o.stride + row * o.ld + col;
    const float v = X[k * rp + i];
    if (o.bf16) {
      __nv_bfloat16* w16 = static_cast<__nv_bfloat16*>(o.o) + at;
      *w16 = __float2bfloat16_rn(o.update ? o.decay * __bfloat162float(*w16) - o.step * v : v);
    } else {
      float* w32 = static_cast<float*>(o.o) + at;
      *w32 = o.update ? o.decay * *w32 - o.step * v : v;
    }
  }
  if (n.csize > 1) cluster_sync();  // the others have read this CTA's last share
}

// CTAs for a matrix: enough for its slices to fit, and more while a CTA's products outweigh a wider barrier.
NcArgs plan(int rows, int cols, size_t* bytes) {
  NcArgs n{};
  n.tall = rows > cols;
  n.r = n.tall ? cols : rows;
  n.c = n.tall ? rows : cols;
  if (n.r > NC_MAX_R) return n;
  const int q = (n.r + 3) / 4;
  n.rp = 4 * (q | 1);
  for (int cs = 1; cs <= 8; cs *= 2) {
    n.cs = (n.c + cs - 1) / cs;
    n.csp = (n.cs + 3) / 4 * 4;
    *bytes = sizeof(float) * ((size_t)2 * n.csp * n.rp + (size_t)4 * n.rp * n.rp);
    n.csize = 0;
    if (*bytes > NC_MAX_SMEM) continue;
    n.csize = cs;
    if ((long long)n.rp * n.rp * n.cs <= 64 * 1024) break;
  }
  return n;
}

}  // namespace

int ns_cluster_size(int rows, int cols, size_t* smem_bytes) {
  size_t bytes = 0;
  const NcArgs n = plan(rows, cols, &bytes);
  if (smem_bytes) *smem_bytes = bytes;
  return n.csize;
}

cudaError_t ns_cluster_set_attributes() {
  return cudaFuncSetAttribute(ns_cluster_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, NC_MAX_SMEM);
}

cudaError_t launch_ns_cluster(const NsSource& s, const NsSink& o, int batch, const float coef[3], int steps, double eps,
                              cudaStream_t st) {
  size_t bytes = 0;
  NcArgs n = plan(s.rows, s.cols, &bytes);
  n.steps = steps;
  n.a = coef[0];
  n.b = coef[1];
  n.cc = coef[2];
  n.eps = eps;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(batch * n.csize));
  cfg.blockDim = dim3(NC_THREADS);
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = (unsigned)n.csize;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = n.csize > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, ns_cluster_kernel, s, o, n);
}

}  // namespace gcada
