// Server update rule Muon: for every weight matrix W of an MLP
//     H <- beta1 H + (1 - beta1) agg                                   (Eq. 8a)
//     W <- (1 - alpha^k wd) W - alpha^k s ortho(U),   U = beta1 H + (1 - beta1) agg, or H without look-ahead,
//     s = scale * sqrt(max(1, rows / cols)),
// ortho() being the Newton-Schulz steps of muon.cu; the biases keep Eq. (8a)-(8c).  The iterate goes from its ring slot
// to the next one as with Eq. (8), and ||theta^{k+1} - theta^k||^2 is summed over all parameters.
#include "server.h"

#include <math.h>

namespace gcada {
namespace {

struct Layers {
  int n = 0;
  long long w_off[MLP_MAX_LAYERS + 1], b_off[MLP_MAX_LAYERS + 1];
  int n_out[MLP_MAX_LAYERS + 1], n_in[MLP_MAX_LAYERS + 1];
  float scale[MLP_MAX_LAYERS + 1];
};

// First kernel: this iteration's targets of the weight matrices, and (fold) the aggregate of Eq. (3): the selected
// groups' fresh gradients in, the ones they replace out, groups ascending, kept as an unevaluated sum hi + lo.
__global__ void __launch_bounds__(256) muon_prepare_kernel(const Params P, const Layers L, float weight_decay, int fold,
                                                           NsTarget* targets) {
  pdl_wait();
  if (blockIdx.x == 0 && (int)threadIdx.x >= 1 && (int)threadIdx.x <= L.n) {
    const int l = threadIdx.x, ring = P.D + 1;
    const long long k = P.st->k;
    const float alpha = step_size(P, k);
    NsTarget t;
    t.prev = P.theta_ring + (k % ring) * P.p_pad + L.w_off[l];
    t.o = P.theta_ring + ((k + 1) % ring) * P.p_pad + L.w_off[l];
    t.decay = 1.f - alpha * weight_decay;
    t.step = alpha * L.scale[l];
    targets[l] = t;
  }
  if (!fold) return;
  const int n_sel = P.sel_count[0];
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < P.p; i += (long long)gridDim.x * 256) {
    float hi = P.agg_hi[i], lo = P.agg_lo[i];
    for (int j = 0; j < n_sel; ++j) {
      const int g = P.sel_list[j];
      const float d[2] = {last_row(P, g)[i], -other_row(P, g)[i]};
#pragma unroll
      for (int t = 0; t < 2; ++t) {  // exact sum of hi and d, the remainder to lo
        const float s = hi + d[t], v = s - hi;
        lo += (hi - (s - v)) + (d[t] - v);
        hi = s;
      }
    }
    const float s = hi + lo;
    P.agg_lo[i] = lo - (s - hi);
    P.agg_hi[i] = s;
  }
}

// Last kernel: the biases by Eq. (8a)-(8c), the squared step norm over all parameters, the iteration counter.
__global__ void __launch_bounds__(256) muon_finish_kernel(const Params P, const Layers L) {
  __shared__ double scratch[40];
  __shared__ bool is_last;
  pdl_launch_dependents();
  pdl_wait();
  const int tid = threadIdx.x, ring = P.D + 1;
  const long long k = P.st->k;
  const float alpha = step_size(P, k);
  const float* th = P.theta_ring + (k % ring) * P.p_pad;
  float* tn = P.theta_ring + ((k + 1) % ring) * P.p_pad;
  double local = 0.0;
  for (int l = 1; l <= L.n; ++l) {
    const long long n = (long long)L.n_out[l] * L.n_in[l];
    const float *a = th + L.w_off[l], *b = tn + L.w_off[l];
#pragma unroll 4
    for (long long i = (long long)blockIdx.x * 256 + tid; i < n; i += (long long)gridDim.x * 256) {
      const float d = b[i] - a[i];
      local += (double)d * (double)d;
    }
    for (long long i = L.b_off[l] + (long long)blockIdx.x * 256 + tid; i < L.b_off[l] + L.n_out[l]; i += (long long)gridDim.x * 256) {
      const float g = P.agg_hi[i], h = P.beta1 * P.h[i] + P.omb1 * g;
      const float vh = fmaxf(P.vhat[i], P.beta2 * P.vhat[i] + P.omb2 * (g * g));
      const float up = alpha * h / sqrtf(P.eps + vh);
      P.h[i] = h;
      P.vhat[i] = vh;
      tn[i] = th[i] - up;
      local += (double)up * (double)up;
    }
  }
  const double tot = block_sum(local, scratch);
  if (tid == 0) {
    P.upd_part[blockIdx.x] = tot;
    __threadfence();
    is_last = atomicAdd(&P.st->ticket_update, 1u) == gridDim.x - 1u;
  }
  __syncthreads();
  if (!is_last) return;
  __threadfence();
  const volatile double* parts = P.upd_part;
  double s = 0.0;
  for (unsigned int b = tid; b < gridDim.x; b += 256) s += parts[b];
  s = block_sum(s, scratch);
  if (tid == 0) {
    P.s_ring[k % P.D] = s;
    P.st->k = k + 1;
    if (P.chain_last) P.st->k_chain = k + 1;
    P.st->ticket_update = 0u;
  }
}

}  // namespace

size_t muon_work_bytes(const MlpPlan& pl) {
  size_t most = 0;
  for (int l = 1; l <= pl.n_layers; ++l) {
    const size_t b = ns_work_bytes(1, pl.dims[l], pl.dims[l - 1]);
    if (b > most) most = b;
  }
  return most;
}

int muon_kernels(const MlpPlan& pl, const MuonPlan& m) {
  int n = 2;
  for (int l = 1; l <= pl.n_layers; ++l) n += ns_launches(pl.dims[l], pl.dims[l - 1], m.steps);
  return n;
}

cudaError_t launch_muon_update(const Params& P, const MlpPlan& pl, const MuonPlan& m, cudaStream_t st, int* launches) {
  Layers L{};
  L.n = pl.n_layers;
  for (int l = 1; l <= pl.n_layers; ++l) {
    L.w_off[l] = pl.w_off[l];
    L.b_off[l] = pl.b_off[l];
    L.n_out[l] = pl.dims[l];
    L.n_in[l] = pl.dims[l - 1];
    L.scale[l] = (float)(m.scale * sqrt(fmax(1.0, (double)pl.dims[l] / pl.dims[l - 1])));
  }
  const long long cols4 = P.p_pad / 4, want = (cols4 + 255) / 256;
  // (update_part holds at least a slot for every 32 columns of 16 bytes: see plan_tail)
  const int blocks = (int)(want < 4LL * pl.sm_count ? want : 4LL * pl.sm_count);
  const int fold = P.agg_direct ? 0 : 1;
  cudaError_t e = launch_k(muon_prepare_kernel, dim3(fold ? (unsigned)(4 * pl.sm_count) : 1u), dim3(256), 0, st, false, P, L,
                           (float)m.weight_decay, fold, m.targets);
  if (e != cudaSuccess) return e;
  *launches = 2;
  for (int l = 1; l <= pl.n_layers; ++l) {
    NsProblem p{};
    p.batch = 1;
    p.rows = pl.dims[l];
    p.cols = pl.dims[l - 1];
    p.g = P.agg_hi + pl.w_off[l];
    p.ld_g = p.cols;
    p.m = P.h + pl.w_off[l];
    p.ld_m = p.cols;
    p.beta = m.beta;
    p.nesterov = m.nesterov;
    p.ld_o = p.cols;
    p.w_update = 1;
    p.at = m.targets + l;
    p.steps = m.steps;
    p.coef[0] = 3.4445;
    p.coef[1] = -4.7750;
    p.coef[2] = 2.0315;
    p.eps = 1e-7;
    p.full = m.full;
    p.err = &P.st->err;
    const char* why = "";
    int n = 0;
    if ((e = ns_run(p, m.work, st, &why, &n)) != cudaSuccess) return e;
    *launches += n;
  }
  return launch_k(muon_finish_kernel, dim3((unsigned)blocks), dim3(256), 0, st, false, P, L);
}

}  // namespace gcada
