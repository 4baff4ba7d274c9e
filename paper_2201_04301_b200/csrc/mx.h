// Microscaled 4-bit matrices: quantisation, read-back and product (see mx.cu).
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"

namespace gcada {

// A matrix in 4-bit form.  Codes: E2M1, two to a byte (the even column in the low half), rows of pitch bytes.
// Scales: E8M0, one per 32 columns of a row, in tiles of 128 rows x 256 columns of 1024 bytes each, tile
// (row / 128) * col_tiles + column / 256; inside a tile byte
//     (column % 256 / 128) * 512 + (row % 32) * 16 + (row % 128 / 32) * 4 + column % 128 / 32,
// which is the order in which the tensor cores take them.  Bytes of rows and blocks behind the end are zero.
struct MxView {
  unsigned char* codes;
  unsigned char* scales;
  long long rows, cols;
  long long pitch;      // bytes per row of codes, a multiple of 16
  long long col_tiles;  // column tiles per row tile
};
inline long long mx_pitch(long long cols) { return (cols + 31) / 32 * 16; }
inline long long mx_col_tiles(long long cols) { return (cols + 255) / 256; }
inline long long mx_scale_bytes(long long rows, long long cols) { return (rows + 127) / 128 * mx_col_tiles(cols) * 1024; }

// q.rows x q.cols from a row-major source of that shape, or with `transpose` of the transposed shape.
cudaError_t mx_quantize(const void* x, int bf16, long long ld, int transpose, const MxView& q, cudaStream_t st);
cudaError_t mx_dequantize(const MxView& q, void* out, int bf16, long long ld, cudaStream_t st);

struct MxGemm {
  MxView a, b;          // a.cols == b.cols
  void* d;              // a.rows x b.rows, row stride ld
  int d_bf16;
  long long ld;
  float alpha, beta;    // d = alpha * a b^T + beta * d (+ bias); beta == 0: d is not read
  const float* bias;    // b.rows values added to every row, or null
  int* err;             // device error word, or null
};
cudaError_t mx_gemm(const MxGemm& p, cudaStream_t st, const char** why);

// Uploads of the bf16 MLP: of every group selected this iteration the [Bp][ld] factor in entry cur[g] * G + g of `x`,
// transposed, into columns g * Bp .. of q (Bp a multiple of 128).
cudaError_t mx_quantize_uploads(const Params& P, const void* x_bf16, int ld, int Bp, const MxView& q, cudaStream_t st);
// out[m][n] = sum over columns k0 .. k0 + K - 1 of a[m][k] b[n][k], out with rows of b.rows floats (getters; K a
// multiple of 32).
cudaError_t mx_upload_product(const MxView& a, const MxView& b, long long k0, int K, float* out, cudaStream_t st);

}  // namespace gcada
