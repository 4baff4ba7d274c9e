// Newton-Schulz orthogonalisation and the optimiser step built on it (see muon.cu).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>

namespace gcada {

// The matrix that is orthogonalised: g itself, or with m the momentum or its look-ahead.
struct NsSource {
  const void* g;  // float or bf16, row stride ld, matrix stride
  long long ld, stride;
  int bf16;
  float* m;       // momentum (row stride ld_m), or null
  long long ld_m, m_stride;
  float beta, omb;
  int nesterov;
  int rows, cols;
};
// Where the result goes: o <- x, or o <- decay * prev - step * x.
struct NsTarget {
  void* o;           // float or bf16, row stride ld, matrix stride
  const void* prev;
  float decay, step;
};
struct NsSink {
  NsTarget to;
  long long ld, stride;
  int bf16, update;
  const NsTarget* at;  // not null: the target is read from here when the result is there (a context's iterates lie in
                       // a ring, so that their places and the step size follow from the iteration number)
};

struct NsProblem {
  int batch, rows, cols;
  const void* g;        // float or bf16, row stride ld_g, matrix stride stride_g
  long long ld_g, stride_g;
  int g_bf16;
  float* m = nullptr;   // momentum (one matrix), moved first; the matrix orthogonalised is then the momentum or,
  long long ld_m = 0;   // with nesterov, its look-ahead (1 - beta) g + beta m
  double beta = 0;
  int nesterov = 0;
  void* o;              // result, float or bf16
  long long ld_o, stride_o;
  int o_bf16;
  int w_update = 0;     // 1: o <- decay * prev - step * result
  const void* prev = nullptr;
  double decay = 1, step = 0;
  const NsTarget* at = nullptr;  // see NsSink
  int steps;
  double coef[3];
  double eps;
  int full;             // 1: products of hi / lo pairs (fp32 accuracy), 0: of the hi parts
  int* err = nullptr;   // device error word, or null
};
// Exponent of the smallest power of two that is at least max(1, |a|): what a step multiplies a tiny iterate by.
inline int ns_growth(double a) {
  int g = 0;
  while ((double)(1 << g) < (a < 0 ? -a : a)) ++g;
  return g;
}
// Narrow matrices, all steps on chip (muon_cluster.cu).
constexpr int NS_NARROW = 64;  // short side
bool ns_fits_cluster(int batch, int rows, int cols);
cudaError_t ns_cluster_set_attributes();
cudaError_t launch_ns_cluster(const NsSource& s, const NsSink& o, int batch, const float coef[3], int steps, double eps,
                              cudaStream_t st);

int ns_launches(int rows, int cols, int steps);  // kernels that ns_run enqueues
size_t ns_work_bytes(int batch, int rows, int cols);
cudaError_t ns_run(const NsProblem& p, void* work, cudaStream_t st, const char** why, int* launches);

}  // namespace gcada
