// Newton-Schulz steps of a narrow matrix (short side up to 64) in one launch: the long side is dealt out to the CTAs
// of a thread-block cluster, which keep their slices of X in shared memory for all steps, in fp32 throughout.
//
// A step: every CTA forms its slice's share of A = X X^T; cluster barrier; A is added up from all shares through
// distributed shared memory, in rank order (bitwise reproducible); every CTA forms b A + c A^2 for itself and applies
// it to its slice.  Bound: latency - each phase is about a thousand cycles of dependent loads, FMAs and a barrier for
// narrow matrices, some thousands for 64 rows.  As separate tensor-core launches the same steps cost 3 us and more
// per product however small it is.
#include <cuda_bf16.h>

#include "common.cuh"
#include "muon.h"
#include "tc.cuh"

namespace gcada {
namespace {

constexpr int NC_THREADS = 512;
constexpr int NC_MAX_R = NS_NARROW;
static_assert(NC_MAX_R <= 64, "the tiles of A fit the smallest block that they are given");
constexpr int NC_MAX_SMEM = 220 * 1024;
// Multiply-adds of a product, for an eighth of them a CTA, beyond which the tensor cores win in spite of their launches
// (here / there, us: 64 x 512 60 / 77, 64 x 800 76 / 72, 48 x 1400 77 / 75, 32 x 3000 73 / 77, 32 x 1024 38 / 67; batches,
// with fewer CTAs for a matrix: 40 of 64 x 512 149 / 98, 100 of 32 x 200 42 / 90).
constexpr long long NC_MAX_WORK = 3000000;

struct NcArgs {
  int r, c, cs;   // short and long side; columns of the long side per CTA
  int rp, csp;    // padded row length (4 x odd: rows start in different banks) and slice length (multiple of 4)
  int tall, csize, steps;
  int growth;     // see ns_growth
  int direct;     // every CTA reads all shares of A
  float a, b, cc;
  double eps;
};

// A thread's place in a symmetric product: a 4 x 4 tile on or above the diagonal, whose sum 2^lk neighbouring lanes
// share (all of a warp's lanes take part in every exchange).
struct SymPlace {
  int ti, tj, part, lk;
  bool on;
};
__device__ SymPlace sym_place(int nt, int K) {
  const int tiles = nt * (nt + 1) / 2;
  SymPlace p;
  p.lk = 0;
  while (p.lk < 5 && (tiles << (p.lk + 1)) <= (int)blockDim.x && (4 << p.lk) <= K) ++p.lk;
  const int tile = (int)threadIdx.x >> p.lk;
  p.part = (int)threadIdx.x & ((1 << p.lk) - 1);
  p.on = tile < tiles;
  p.ti = 0;
  int u = p.on ? tile : 0;
  while (u >= nt - p.ti) u -= nt - p.ti++;
  p.tj = p.ti + u;
  return p;
}

// out[i][j] (symmetric, in rows of rp) = s_acc * sum over k < K of M[k][i] M[k][j] + s_src * add[i][j].
__device__ __forceinline__ void symmetric_product(const SymPlace& p, const float* M, int K, int rp, float* out, const float* add,
                                                  float s_src, float s_acc) {
  float acc[4][4] = {};
  if (p.on) {
    const float* mi = M + 4 * p.ti;
    const float* mj = M + 4 * p.tj;
#pragma unroll 4
    for (int k = p.part; k < K; k += 1 << p.lk) {
      const float4 x = *reinterpret_cast<const float4*>(mi + k * rp), y = *reinterpret_cast<const float4*>(mj + k * rp);
      const float xs[4] = {x.x, x.y, x.z, x.w}, ys[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] += xs[i] * ys[j];
    }
  }
  for (int o = 1; o < 1 << p.lk; o *= 2) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[i][j] += __shfl_xor_sync(0xffffffffu, acc[i][j], o);
  }
  if (p.on && p.part == 0) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int at = (4 * p.ti + i) * rp + 4 * p.tj;
      float4 v = make_float4(s_acc * acc[i][0], s_acc * acc[i][1], s_acc * acc[i][2], s_acc * acc[i][3]);
      if (add) {
        const float4 w = *reinterpret_cast<const float4*>(add + at);
        v = make_float4(v.x + s_src * w.x, v.y + s_src * w.y, v.z + s_src * w.z, v.w + s_src * w.w);
      }
      *reinterpret_cast<float4*>(out + at) = v;
      acc[i][0] = v.x; acc[i][1] = v.y; acc[i][2] = v.z; acc[i][3] = v.w;
    }
    if (p.ti != p.tj) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        *reinterpret_cast<float4*>(out + (4 * p.tj + j) * rp + 4 * p.ti) = make_float4(acc[0][j], acc[1][j], acc[2][j], acc[3][j]);
    }
  }
}

// TINY: X_0 may be beyond fp32's normal range.  Its non-zero elements are at least 2^-149 / eps where the norm is far below
// eps, which for eps <= 1e-7 (the default) is 2^-125.7: nothing is lost then.  (10 x 200 takes 15.0 us without TINY, 15.7 with.)
template <bool TINY>
__global__ void __launch_bounds__(NC_THREADS, 1) ns_cluster_kernel(const NsSource s, const NsSink o, const NcArgs n) {
  extern __shared__ __align__(16) float sm[];
  __shared__ double share[NC_THREADS / 32];
  const int rp = n.rp, sq = rp * rp;
  float* X = sm;                       // [csp][rp]: X transposed, element (i, k) at k * rp + i
  float* Y = X + (size_t)n.csp * rp;   // the next iterate
  float* A = Y + (size_t)n.csp * rp;
  float* Q = A + sq;
  float* part = Q + sq;                // clusters: this CTA's share of A (two of them if read directly)
  const int b = blockIdx.x / n.csize, rank = n.csize > 1 ? (int)cluster_rank() : 0;
  const int k0 = rank * n.cs, kn = max(0, min(n.cs, n.c - k0));
  const int tid = threadIdx.x, threads = blockDim.x;

  // the slice, momentum moved on the way; squares in doubles
  for (int e = tid; e < n.csp * rp; e += threads) X[e] = 0.f;
  pdl_launch_dependents();
  pdl_wait();
  __syncthreads();
  const int count = kn * n.r;
  double ss = 0.0;
  for (int e = tid; e < count; e += threads) {
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
  // every warp adds up all warps' sums of all CTAs itself, in one order
  ss = warp_sum(ss);
  const int warps = threads >> 5, lane = tid & 31;
  if (lane == 0) share[tid >> 5] = ss;
  if (n.csize > 1)
    cluster_sync();
  else
    __syncthreads();
  ss = 0.0;
  for (int i = lane; i < warps * n.csize; i += 32) {
    const int p = i / warps, w = i - p * warps;
    ss += n.csize > 1 ? cluster_load_f64(cluster_map(smem_u32(share + w), (uint32_t)p)) : share[w];
  }
  ss = warp_sum(ss);
  const double norm = sqrt(ss);
  double inv = 1.0 / (norm + n.eps);
  int rho = 0;  // TINY: the iterate is kept times 2^-rho, rho as in muon.cu
  if (TINY && norm > 0.0 && norm * inv < 0x1p-60) {
    rho = ilogb(norm * inv);
    inv = ldexp(inv, -rho);
  }
  for (int e = tid; e < kn * rp; e += threads) X[e] = (float)((double)X[e] * inv);
  __syncthreads();

  const int nt = rp >> 2, kgroups = (kn + 3) >> 2, items = kgroups * nt;
  int lk = 0;  // 2^lk lanes share an item's sum over j
  while (lk < 4 && (items << (lk + 1)) <= threads && (2 << lk) <= nt) ++lk;
  const SymPlace gram = sym_place(nt, kn), poly = sym_place(nt, n.r);
  const int e0 = n.direct ? 0 : (sq >> 2) * rank / n.csize, e1 = n.direct ? sq >> 2 : (sq >> 2) * (rank + 1) / n.csize;
  for (int step = 0; step < n.steps; ++step) {
    float* mine = n.csize > 1 ? part + (n.direct && (step & 1) ? sq : 0) : A;
    symmetric_product(gram, X, kn, rp, mine, nullptr, 0.f, 1.f);
    if (n.csize > 1) {
      // A is the sum of all shares: of a small matrix every CTA reads them all (from alternating buffers, so that the
      // next step's may be written meanwhile), of a larger one each adds up a part and hands it to all
      cluster_sync();
      for (int e = e0 + tid; e < e1; e += threads) {
        float4 v[8];
#pragma unroll
        for (int p = 0; p < 8; ++p)
          if (p < n.csize) v[p] = cluster_load4(cluster_map(smem_u32(mine + 4 * e), (uint32_t)p));
        float4 t = v[0];
#pragma unroll
        for (int p = 1; p < 8; ++p)
          if (p < n.csize) t = make_float4(t.x + v[p].x, t.y + v[p].y, t.z + v[p].z, t.w + v[p].w);
        if (n.direct) {
          *reinterpret_cast<float4*>(A + 4 * e) = t;
        } else {
#pragma unroll
          for (int p = 0; p < 8; ++p)
            if (p < n.csize) cluster_store4(cluster_map(smem_u32(A + 4 * e), (uint32_t)p), t);
        }
      }
      if (n.direct)
        __syncthreads();
      else
        cluster_sync();
    } else {
      __syncthreads();
    }
    float ca = n.a, cb = n.b, cc = n.cc;
    if (TINY && rho) {
      const int next = min(rho + n.growth, 0);
      ca = ldexpf(ca, rho - next);
      cb = ldexpf(cb, 3 * rho - next);
      cc = ldexpf(cc, 5 * rho - next);
      rho = next;
    }
    symmetric_product(poly, A, n.r, rp, Q, A, cb, cc);
    __syncthreads();
    // Y = a X + X Q: 4 columns of the slice x 4 rows a thread
    for (int base = 0; base < items << lk; base += threads) {
      const int id = base + tid, item = id >> lk, p = id & ((1 << lk) - 1);
      const bool on = item < items;
      const int kg = on ? item / nt : 0, ti = on ? item - kg * nt : 0;
      const float* x = X + (size_t)kg * 4 * rp;
      float acc[4][4] = {};
      if (on) {
        for (int j = 4 * p; j < rp; j += 4 << lk) {
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
      for (int w = 1; w < 1 << lk; w *= 2) {
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
              make_float4(ca * v.x + acc[t][0], ca * v.y + acc[t][1], ca * v.z + acc[t][2], ca * v.w + acc[t][3]);
        }
      }
    }
    __syncthreads();
    float* t = X;
    X = Y;
    Y = t;
  }

  const NsTarget to = o.at ? *o.at : o.to;
  for (int e = tid; e < count; e += threads) {
    const int major = n.tall ? n.r : kn, q = e / major, w = e - q * major;
    const int i = n.tall ? w : q, k = n.tall ? q : w;
    const long long row = n.tall ? k0 + k : i, col = n.tall ? i : k0 + k;
    const long long at = (long long)b * o.stride + row * o.ld + col;
    const float v = TINY && rho ? ldexpf(X[k * rp + i], rho) : X[k * rp + i];
    if (o.bf16)
      static_cast<__nv_bfloat16*>(to.o)[at] = __float2bfloat16_rn(
          o.update ? to.decay * __bfloat162float(static_cast<const __nv_bfloat16*>(to.prev)[at]) - to.step * v : v);
    else
      static_cast<float*>(to.o)[at] = o.update ? to.decay * static_cast<const float*>(to.prev)[at] - to.step * v : v;
  }
  // nobody reads this CTA's shared memory any more: with steps in between, since the last barrier or, read directly, once
  // all have passed this one
  if (n.csize > 1 && (n.direct || n.steps == 0)) cluster_sync();
}

// CTAs for a matrix.  One is fastest only while a barrier costs more than the work (16 x 16: 12 us with one, 15 with
// eight; 16 x 64: 15 and 16); from there on eight (10 x 200: 17 and 15 us, 64 x 200: 111 and 40), but no more than let
// all matrices of a batch run at once, and enough for the slices to fit.
NcArgs plan(int batch, int rows, int cols, size_t* bytes) {
  NcArgs n{};
  n.tall = rows > cols;
  n.r = n.tall ? cols : rows;
  n.c = n.tall ? rows : cols;
  if (n.r > NC_MAX_R) return n;
  const int q = (n.r + 3) / 4;
  n.rp = 4 * (q | 1);
  n.direct = n.rp <= 20;  // at most 100 pieces of 16 bytes from each of eight CTAs
  int want = (long long)n.rp * n.c <= 1300 ? 1 : 8;
  while (want > 1 && batch * want > 128) want /= 2;
  for (int cs = want; cs <= 8; cs *= 2) {
    n.cs = (n.c + cs - 1) / cs;
    n.csp = (n.cs + 3) / 4 * 4;
    const double size = sizeof(float) * ((double)2 * n.csp * n.rp + (double)(cs > 1 ? (n.direct ? 4 : 3) : 2) * n.rp * n.rp);
    if (size > NC_MAX_SMEM) continue;
    if ((long long)n.r * n.r * n.c * (8 / cs) > NC_MAX_WORK) break;
    *bytes = (size_t)size;
    n.csize = cs;
    break;
  }
  return n;
}

}  // namespace

bool ns_fits_cluster(int batch, int rows, int cols) {
  size_t bytes = 0;
  return plan(batch, rows, cols, &bytes).csize != 0;
}

cudaError_t ns_cluster_set_attributes() {
  const cudaError_t e = cudaFuncSetAttribute(ns_cluster_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, NC_MAX_SMEM);
  return e == cudaSuccess ? cudaFuncSetAttribute(ns_cluster_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, NC_MAX_SMEM) : e;
}

cudaError_t launch_ns_cluster(const NsSource& s, const NsSink& o, int batch, const float coef[3], int steps, double eps,
                              cudaStream_t st) {
  size_t bytes = 0;
  NcArgs n = plan(batch, s.rows, s.cols, &bytes);
  n.steps = steps;
  n.a = coef[0];
  n.b = coef[1];
  n.cc = coef[2];
  n.growth = ns_growth(coef[0]);
  n.eps = eps;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3((unsigned)(batch * n.csize));
  // a thread at least for every 4 x 4 tile of A (153 at most: a symmetric product is one pass), and as many as the
  // slice's own tiles keep busy
  const int nt = n.rp >> 2, tiles = nt * (nt + 1) / 2, items = (n.csp >> 2) * nt, want = tiles > items ? tiles : items;
  cfg.blockDim = dim3((unsigned)(want <= 64 ? 128 : want <= 192 ? 256 : NC_THREADS));
  cfg.dynamicSmemBytes = bytes;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = (unsigned)n.csize;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = n.csize > 1 ? 2 : 1;
  return eps > 1e-7 ? cudaLaunchKernelEx(&cfg, ns_cluster_kernel<true>, s, o, n)
                    : cudaLaunchKernelEx(&cfg, ns_cluster_kernel<false>, s, o, n);
}

}  // namespace gcada
