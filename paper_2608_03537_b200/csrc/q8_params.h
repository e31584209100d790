// Parameter blocks and launchers of the 8-bit integer layers (plain data).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "host_common.h"

namespace comfuse {

struct QuantizeRowsParams {
  int rows, N;
  int split;  // CTAs (a cluster) that share a row
  const void *x, *residual, *gamma;
  void* h;
  int8_t* q;
  float* scale;
  uint16_t* values;
  long long ldx, ldr, ldh, ldq, ldv;
  float eps;
  unsigned int* status;
};
cudaError_t launch_quantize_rows(int dtype, bool norm, QuantizeRowsParams p, const DeviceInfo& dev, cudaStream_t stream);

struct GemmQ8Params {
  int batch, M, N, K;
  int activation;  // comfuse_op_t, 0 = none
  const float *scale_a, *scale_b;
  const void *bias, *residual;
  void* Y;
  long long ldr, ldy, batch_stride_r, batch_stride_y;
  int mtiles, ntiles;   // tiles of one batch; few rows: groups of rows, 128-channel tiles
  int split;            // few rows: CTAs (a cluster) that share a tile's contraction; a handful: warps that do
  long long tiles;      // tiles of all batches
  unsigned int* status;
  unsigned long long timeout_ns;
};

// A handful of rows: the operands themselves (the other forms read them through tensor maps).
constexpr int kGemmQ8Tokens = 16;
struct GemmQ8TokensParams {
  const int8_t *A, *B;
  long long lda, ldb, batch_stride_a, batch_stride_b;
};
bool gemm_q8_tokens_fits(int batch, int M, int N, int K, const DeviceInfo& dev);
cudaError_t launch_gemm_q8_tokens(int dtype, const GemmQ8TokensParams& t, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream);

// Few rows: rows per group (the UMMA's N: 16, 32, 64 or 128) and CTAs that share a contraction; rows = 0: the call does not take this form.
struct GemmQ8FewPlan {
  int rows = 0, split = 1;
};
// long_epilogue: a residual, or an activation that is more than a comparison.
GemmQ8FewPlan gemm_q8_few_plan(int batch, int M, int N, int K, bool long_epilogue, const DeviceInfo& dev);
// tmW: the weights in boxes of 128 bytes x 128 rows, tmX: the rows in boxes of 128 bytes x plan.rows rows.
cudaError_t launch_gemm_q8_few(int dtype, const GemmQ8FewPlan& plan, const CUtensorMap& tmW, const CUtensorMap& tmX, GemmQ8Params p, cudaStream_t stream);
// Columns of Y that leave by TMA: up to the last whole 16-byte unit of a row.
__host__ __device__ inline int gemm_q8_stored_columns(int dtype, int N) { return dtype == COMFUSE_DTYPE_F32 ? N & ~3 : N & ~7; }

// Many rows.  `columns` of a tile (128 or 256): B's boxes have half as many rows.
int gemm_q8_pair_columns(int batch, int M, int N, const DeviceInfo& dev);
struct GemmQ8PairMaps {
  CUtensorMap A, B, R, Y;  // boxes of 128 bytes x 128 rows (A), x columns / 2 rows (B), x 32 rows (R; Y up to its last whole 16 bytes); R unused without a residual
};
cudaError_t launch_gemm_q8_pair(int dtype, int columns, const GemmQ8PairMaps& maps, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream);

}  // namespace comfuse
