// The server's update rules other than Eq. (8): Muon on the weight matrices of an MLP (see server.cu).
#pragma once
#include <cuda_runtime.h>

#include "common.cuh"
#include "mlp.h"
#include "muon.h"

namespace gcada {

struct MuonPlan {
  double beta = 0, weight_decay = 0, scale = 1;
  int nesterov = 1, steps = 5;
  int full = 1;                 // 0: products of 11-bit operands
  NsTarget* targets = nullptr;  // [n_layers + 1] device: where layer l's weights come from and go to this iteration
  void* work = nullptr;
};
size_t muon_work_bytes(const MlpPlan& pl);
int muon_kernels(const MlpPlan& pl, const MuonPlan& m);
// Enqueues the whole update of an iteration: the aggregate (where it is not formed yet), the weights, the biases,
// the squared step norm and the iteration counter.
cudaError_t launch_muon_update(const Params& P, const MlpPlan& pl, const MuonPlan& m, cudaStream_t st, int* launches);

}  // namespace gcada
