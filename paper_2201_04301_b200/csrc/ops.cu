// Entry points of the matrix operators (include/gcada.h): checks of arguments, then the launchers.
#include <cuda_runtime.h>
#include <math.h>
#include <stdarg.h>
#include <stdint.h>
#include <stdio.h>

#include "../../include/gcada.h"
#include "muon.h"
#include "mx.h"

namespace {

gcada_status op_fail(char* errbuf, size_t len, gcada_status st, const char* fmt, ...) {
  if (errbuf && len) {
    va_list ap;
    va_start(ap, fmt);
    vsnprintf(errbuf, len, fmt, ap);
    va_end(ap);
  }
  return st;
}

gcada_status op_cuda(char* errbuf, size_t len, cudaError_t e, const char* why) {
  if (e == cudaSuccess) return GCADA_OK;
  return op_fail(errbuf, len, e == cudaErrorMemoryAllocation ? GCADA_ENOMEM : GCADA_ECUDA, "%s: %s", why, cudaGetErrorString(e));
}

bool known_type(int t) { return t == GCADA_COMPUTE_FP32 || t == GCADA_COMPUTE_BF16; }
size_t type_bytes(int t) { return t == GCADA_COMPUTE_BF16 ? 2 : 4; }
bool aligned_to(const void* p, size_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

#define REFUSE(cond, ...) \
  do {                    \
    if (cond) return op_fail(errbuf, errbuf_len, GCADA_EINVAL, __VA_ARGS__); \
  } while (0)

constexpr long long MAX_SIDE = 1 << 20;  // rows or columns of a matrix

__device__ int own_status_word;  // gcada_operator_status: zero when the library is loaded, one on every device

const double DEFAULT_COEF[3] = {3.4445, -4.7750, 2.0315};

gcada_status check_steps(int precision, int steps, const double* coef, double eps, char* errbuf, size_t errbuf_len) {
  REFUSE(precision != GCADA_PRECISION_FULL && precision != GCADA_PRECISION_HALF, "unknown precision %d", precision);
  REFUSE(steps < 0 || steps > 100, "steps must be in [0, 100]");
  for (int i = 0; coef && i < 3; ++i) REFUSE(!(fabs(coef[i]) <= 16.0), "coefficients must be in [-16, 16]");
  REFUSE(!(eps >= 1e-30 && eps <= 1e30), "eps must be in [1e-30, 1e30]");
  return GCADA_OK;
}

}  // namespace

extern "C" {

gcada_status gcada_operator_status(int** word_dev) {
  if (!word_dev) return GCADA_EINVAL;
  void* p = nullptr;
  if (cudaGetSymbolAddress(&p, own_status_word) != cudaSuccess) return *word_dev = nullptr, GCADA_ECUDA;
  *word_dev = static_cast<int*>(p);
  return GCADA_OK;
}

gcada_status gcada_orthogonalize_work(int batch, int rows, int cols, size_t* bytes) {
  if (!bytes || batch < 0 || rows < 0 || cols < 0 || rows > MAX_SIDE || cols > MAX_SIDE) return GCADA_EINVAL;
  *bytes = batch && rows && cols ? gcada::ns_work_bytes(batch, rows, cols) : 0;
  return GCADA_OK;
}

gcada_status gcada_orthogonalize(const void* g_dev, void* o_dev, int type, int batch, int rows, int cols, long long ld_g,
                                 long long stride_g, long long ld_o, long long stride_o, int precision, int steps,
                                 const double* coef, double eps, void* work_dev, size_t work_bytes, int* status_dev,
                                 void* cuda_stream, char* errbuf, size_t errbuf_len) {
  if (errbuf && errbuf_len) errbuf[0] = 0;
  REFUSE(!known_type(type), "unknown type %d", type);
  REFUSE(batch < 0 || rows < 0 || cols < 0, "batch, rows and cols must not be negative");
  REFUSE(rows > MAX_SIDE || cols > MAX_SIDE || batch > 65535, "at most 65535 matrices of at most 2^20 rows and columns");
  gcada_status st = check_steps(precision, steps, coef, eps, errbuf, errbuf_len);
  if (st != GCADA_OK) return st;
  if (!batch || !rows || !cols) return GCADA_OK;
  REFUSE(!g_dev || !o_dev, "a matrix pointer is NULL");
  REFUSE(!aligned_to(g_dev, type_bytes(type)) || !aligned_to(o_dev, type_bytes(type)), "a matrix pointer is not aligned to its type");
  REFUSE(ld_g < cols || ld_o < cols, "a row stride is smaller than cols");
  REFUSE(batch > 1 && (stride_g < 0 || stride_o < ld_o * (rows - 1) + cols), "matrix strides: need stride_g >= 0 and results that do not overlap");
  // a matrix of the batch may be written before another has been read
  REFUSE(batch > 1 && o_dev == g_dev && (stride_o != stride_g || (rows > 1 && ld_o != ld_g)), "a batch takes its results in place in the same layout only");
  const size_t need = gcada::ns_work_bytes(batch, rows, cols);
  REFUSE(!work_dev || !aligned_to(work_dev, 256) || work_bytes < need, "need a 256-byte aligned work area of %zu bytes", need);
  gcada::NsProblem p{};
  p.batch = batch;
  p.rows = rows;
  p.cols = cols;
  p.g = g_dev;
  p.ld_g = ld_g;
  p.stride_g = stride_g;
  p.g_bf16 = type == GCADA_COMPUTE_BF16;
  p.o = o_dev;
  p.ld_o = ld_o;
  p.stride_o = stride_o;
  p.o_bf16 = p.g_bf16;
  p.steps = steps;
  for (int i = 0; i < 3; ++i) p.coef[i] = (coef ? coef : DEFAULT_COEF)[i];
  p.eps = eps;
  p.full = precision == GCADA_PRECISION_FULL;
  p.err = status_dev;
  const char* why = "";
  return op_cuda(errbuf, errbuf_len, gcada::ns_run(p, work_dev, static_cast<cudaStream_t>(cuda_stream), &why, nullptr), why);
}

gcada_status gcada_muon_update(void* w_dev, int w_type, float* m_dev, const void* g_dev, int g_type, int rows, int cols,
                               long long ld_w, long long ld_m, long long ld_g, double lr, double beta, int nesterov,
                               double weight_decay, double scale, int precision, int steps, const double* coef, double eps,
                               void* work_dev, size_t work_bytes, int* status_dev, void* cuda_stream, char* errbuf,
                               size_t errbuf_len) {
  if (errbuf && errbuf_len) errbuf[0] = 0;
  REFUSE(!known_type(w_type) || !known_type(g_type), "unknown type %d", known_type(w_type) ? g_type : w_type);
  REFUSE(rows < 0 || cols < 0 || rows > MAX_SIDE || cols > MAX_SIDE, "rows and cols must be in [0, 2^20]");
  REFUSE(!(fabs(lr) <= 1e30) || !(fabs(weight_decay) <= 1e30) || !(fabs(scale) <= 1e30), "lr, weight_decay and scale must be finite");
  REFUSE(!(beta >= 0 && beta < 1), "beta must be in [0, 1)");
  gcada_status st = check_steps(precision, steps, coef, eps, errbuf, errbuf_len);
  if (st != GCADA_OK) return st;
  if (!rows || !cols) return GCADA_OK;
  REFUSE(!w_dev || !m_dev || !g_dev, "a matrix pointer is NULL");
  REFUSE(!aligned_to(w_dev, type_bytes(w_type)) || !aligned_to(m_dev, 4) || !aligned_to(g_dev, type_bytes(g_type)),
         "a matrix pointer is not aligned to its type");
  REFUSE(ld_w < cols || ld_m < cols || ld_g < cols, "a row stride is smaller than cols");
  REFUSE(w_dev == m_dev || w_dev == g_dev || m_dev == g_dev, "w, m and g must be different matrices");
  const size_t need = gcada::ns_work_bytes(1, rows, cols);
  REFUSE(!work_dev || !aligned_to(work_dev, 256) || work_bytes < need, "need a 256-byte aligned work area of %zu bytes", need);
  gcada::NsProblem p{};
  p.batch = 1;
  p.rows = rows;
  p.cols = cols;
  p.g = g_dev;
  p.ld_g = ld_g;
  p.g_bf16 = g_type == GCADA_COMPUTE_BF16;
  p.m = m_dev;
  p.ld_m = ld_m;
  p.beta = beta;
  p.nesterov = nesterov != 0;
  p.o = w_dev;
  p.prev = w_dev;
  p.ld_o = ld_w;
  p.o_bf16 = w_type == GCADA_COMPUTE_BF16;
  p.w_update = 1;
  p.decay = 1.0 - lr * weight_decay;
  p.step = lr * scale;
  p.steps = steps;
  for (int i = 0; i < 3; ++i) p.coef[i] = (coef ? coef : DEFAULT_COEF)[i];
  p.eps = eps;
  p.full = precision == GCADA_PRECISION_FULL;
  p.err = status_dev;
  const char* why = "";
  return op_cuda(errbuf, errbuf_len, gcada::ns_run(p, work_dev, static_cast<cudaStream_t>(cuda_stream), &why, nullptr), why);
}

gcada_status gcada_mx_size(long long rows, long long cols, size_t* code_bytes, size_t* scale_bytes) {
  if (rows < 0 || cols < 0 || rows > (1LL << 31) || cols > (1LL << 31) || !code_bytes || !scale_bytes) return GCADA_EINVAL;
  *code_bytes = (size_t)(rows * gcada::mx_pitch(cols));
  *scale_bytes = (size_t)gcada::mx_scale_bytes(rows, cols);
  return GCADA_OK;
}

static gcada_status mx_view(const void* codes, const void* scales, long long rows, long long cols, gcada::MxView* v,
                            char* errbuf, size_t errbuf_len) {
  REFUSE(rows < 0 || cols < 0 || rows > 4 * MAX_SIDE || cols > 32 * MAX_SIDE,
         "at most 2^22 rows and 2^25 columns of a 4-bit matrix");
  v->codes = static_cast<unsigned char*>(const_cast<void*>(codes));
  v->scales = static_cast<unsigned char*>(const_cast<void*>(scales));
  v->rows = rows;
  v->cols = cols;
  v->pitch = gcada::mx_pitch(cols);
  v->col_tiles = gcada::mx_col_tiles(cols);
  if (!rows || !cols) return GCADA_OK;
  REFUSE(!codes || !scales, "a pointer is NULL");
  REFUSE(!aligned_to(codes, 16) || !aligned_to(scales, 16), "codes and scales must be 16-byte aligned");
  return GCADA_OK;
}

gcada_status gcada_mx_quantize(const void* x_dev, int type, long long rows, long long cols, long long ld, int transpose,
                               void* codes_dev, void* scales_dev, void* cuda_stream, char* errbuf, size_t errbuf_len) {
  if (errbuf && errbuf_len) errbuf[0] = 0;
  REFUSE(!known_type(type), "unknown type %d", type);
  gcada::MxView q;
  gcada_status st = mx_view(codes_dev, scales_dev, transpose ? cols : rows, transpose ? rows : cols, &q, errbuf, errbuf_len);
  if (st != GCADA_OK) return st;
  if (!rows || !cols) return GCADA_OK;
  REFUSE(!x_dev || !aligned_to(x_dev, type_bytes(type)), "x is NULL or not aligned to its type");
  REFUSE(ld < cols, "the row stride is smaller than cols");
  return op_cuda(errbuf, errbuf_len,
                 gcada::mx_quantize(x_dev, type == GCADA_COMPUTE_BF16, ld, transpose, q, static_cast<cudaStream_t>(cuda_stream)),
                 "kernel launch");
}

gcada_status gcada_mx_dequantize(const void* codes_dev, const void* scales_dev, long long rows, long long cols, void* x_dev,
                                 int type, long long ld, void* cuda_stream, char* errbuf, size_t errbuf_len) {
  if (errbuf && errbuf_len) errbuf[0] = 0;
  REFUSE(!known_type(type), "unknown type %d", type);
  gcada::MxView q;
  gcada_status st = mx_view(codes_dev, scales_dev, rows, cols, &q, errbuf, errbuf_len);
  if (st != GCADA_OK) return st;
  if (!rows || !cols) return GCADA_OK;
  REFUSE(!x_dev || !aligned_to(x_dev, type_bytes(type)), "x is NULL or not aligned to its type");
  REFUSE(ld < cols, "the row stride is smaller than cols");
  return op_cuda(errbuf, errbuf_len,
                 gcada::mx_dequantize(q, x_dev, type == GCADA_COMPUTE_BF16, ld, static_cast<cudaStream_t>(cuda_stream)),
                 "kernel launch");
}

gcada_status gcada_mx_gemm(const void* a_codes, const void* a_scales, long long m, const void* b_codes, const void* b_scales,
                           long long n, long long k, void* d_dev, int type, long long ld, double alpha, double beta,
                           const float* bias_dev, int* status_dev, void* cuda_stream, char* errbuf, size_t errbuf_len) {
  if (errbuf && errbuf_len) errbuf[0] = 0;
  REFUSE(!known_type(type), "unknown type %d", type);
  gcada::MxGemm p{};
  gcada_status st = mx_view(a_codes, a_scales, m, k, &p.a, errbuf, errbuf_len);
  if (st == GCADA_OK) st = mx_view(b_codes, b_scales, n, k, &p.b, errbuf, errbuf_len);
  if (st != GCADA_OK) return st;
  REFUSE(!(fabs(alpha) <= 1e30) || !(fabs(beta) <= 1e30), "alpha and beta must be finite");
  if (!m || !n) return GCADA_OK;
  REFUSE(!k, "a product over no columns at all");
  REFUSE(!d_dev || !aligned_to(d_dev, type_bytes(type)) || !aligned_to(bias_dev, 4), "d is NULL, or d or bias is not aligned to its type");
  REFUSE(ld < n, "the row stride of d is smaller than n");
  p.d = d_dev;
  p.d_bf16 = type == GCADA_COMPUTE_BF16;
  p.ld = ld;
  p.alpha = (float)alpha;
  p.beta = (float)beta;
  p.bias = bias_dev;
  p.err = status_dev;
  const char* why = "";
  return op_cuda(errbuf, errbuf_len, gcada::mx_gemm(p, static_cast<cudaStream_t>(cuda_stream), &why), why);
}

}  // extern "C"
