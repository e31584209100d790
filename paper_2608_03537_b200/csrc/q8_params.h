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
};
cudaError_t launch_quantize_rows(int dtype, bool norm, QuantizeRowsParams p, const DeviceInfo& dev, cudaStream_t stream);

struct GemmQ8Params {
  int batch, M, N, K;
  int activation;  // comfuse_op_t, 0 = none
  const float *scale_a, *scale_b;
  const void *bias, *residual;
  void* Y;
  long long ldr, ldy, batch_stride_r, batch_stride_y;
  int wide;             // rows of Y and of the residual start on 32-byte boundaries
  int mtiles, ntiles;   // tiles of one batch; few rows: groups of rows, 128-channel tiles
  int split;            // few rows: CTAs (a cluster) that share a tile's contraction
  long long tiles;      // tiles of all batches
  unsigned int* status;
  unsigned long long timeout_ns;
};

// Few rows: rows per group (the UMMA's N: 16, 32, 64, 128 or 256) and CTAs that share a contraction; rows = 0: the call does not take this form.
struct GemmQ8FewPlan {
  int rows = 0, split = 1;
};
GemmQ8FewPlan gemm_q8_few_plan(int batch, int M, int N, int K, const DeviceInfo& dev);
// tmW: the weights in boxes of 128 bytes x 128 rows, tmX: the rows in boxes of 128 bytes x plan.rows rows.
cudaError_t launch_gemm_q8_few(int dtype, const GemmQ8FewPlan& plan, const CUtensorMap& tmW, const CUtensorMap& tmX, GemmQ8Params p, cudaStream_t stream);
// tmA, tmB: boxes of 128 bytes x 128 rows.
cudaError_t launch_gemm_q8_pair(int dtype, const CUtensorMap& tmA, const CUtensorMap& tmB, GemmQ8Params p, const DeviceInfo& dev, cudaStream_t stream);

}  // namespace comfuse
