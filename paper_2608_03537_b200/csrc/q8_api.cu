// C entry points of the 8-bit integer layers: argument checks, tensor maps, choice of the form.
#include <cmath>

#include "../../include/comfuse.h"
#include "q8_params.h"

namespace comfuse {
namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
int dtype_bytes(int dtype) { return dtype == COMFUSE_DTYPE_F32 ? 4 : 2; }
bool known_dtype(int dtype) { return dtype == COMFUSE_DTYPE_BF16 || dtype == COMFUSE_DTYPE_F16 || dtype == COMFUSE_DTYPE_F32; }
// rows that start on 16-byte boundaries
bool rows_aligned(long long ld, int bytes) { return ((ld * bytes) & 15) == 0; }

comfuse_status_t check_quantize(const comfuse_quantize_desc_t* d, const void* x, const void* residual, const void* gamma, const void* h, const int8_t* q,
                                const float* scale, const void* values) {
  if (!d) return COMFUSE_ERR_INVALID_ARG;
  if (d->rows < 1 || d->N < 1 || !known_dtype(d->dtype) || d->reserved != 0) return COMFUSE_ERR_INVALID_ARG;
  if (d->kind != COMFUSE_QUANTIZE_PLAIN && d->kind != COMFUSE_QUANTIZE_RMSNORM) return COMFUSE_ERR_INVALID_ARG;
  if (d->kind == COMFUSE_QUANTIZE_RMSNORM ? !(d->eps > 0.f && std::isfinite(d->eps)) : d->eps != 0.f) return COMFUSE_ERR_INVALID_ARG;
  if (!x || !q || !scale) return COMFUSE_ERR_INVALID_ARG;
  if (d->kind == COMFUSE_QUANTIZE_PLAIN && (residual || gamma || h)) return COMFUSE_ERR_INVALID_ARG;
  if (d->ldx < d->N || d->ldq < d->N || (residual && d->ldr < d->N) || (h && d->ldh < d->N) || (values && d->ldv < d->N)) return COMFUSE_ERR_INVALID_ARG;
  if ((h && h == x && d->ldh != d->ldx) || (h && h == residual && d->ldh != d->ldr)) return COMFUSE_ERR_INVALID_ARG;
  const int e = dtype_bytes(d->dtype);
  if (!rows_aligned(d->ldx, e) || !rows_aligned(d->ldq, 1) || (residual && !rows_aligned(d->ldr, e)) || (h && !rows_aligned(d->ldh, e)) ||
      (values && !rows_aligned(d->ldv, 2)))
    return COMFUSE_ERR_ALIGNMENT;
  if (!aligned(x, 16) || !aligned(residual, 16) || !aligned(gamma, 16) || !aligned(h, 16) || !aligned(q, 16) || !aligned(values, 16) || !aligned(scale, 4))
    return COMFUSE_ERR_ALIGNMENT;
  if (d->N > 65536) return COMFUSE_ERR_UNSUPPORTED;
  return COMFUSE_OK;
}

comfuse_status_t check_gemm(const comfuse_gemm_q8_desc_t* d, const void* A, const float* scale_a, const void* B, const float* scale_b, const void* bias,
                            const void* residual, const void* Y) {
  if (!d) return COMFUSE_ERR_INVALID_ARG;
  if (d->batch < 1 || d->M < 1 || d->N < 1 || d->K < 1 || !known_dtype(d->dtype) || d->flags != 0 || d->reserved != 0) return COMFUSE_ERR_INVALID_ARG;
  switch (d->activation) {
    case 0: case COMFUSE_OP_RELU: case COMFUSE_OP_GELU_TANH: case COMFUSE_OP_TANH: case COMFUSE_OP_SIGMOID: break;
    default: return COMFUSE_ERR_INVALID_ARG;
  }
  if (!A || !scale_a || !B || !scale_b || !Y) return COMFUSE_ERR_INVALID_ARG;
  if (d->lda < d->K || d->ldb < d->K || d->ldy < d->N || (residual && d->ldr < d->N)) return COMFUSE_ERR_INVALID_ARG;
  auto spans = [&](long long stride, long long rows, long long ld, long long n) { return d->batch == 1 || stride >= (rows - 1) * ld + n; };
  if (!spans(d->batch_stride_a, d->M, d->lda, d->K) || !spans(d->batch_stride_b, d->N, d->ldb, d->K) || !spans(d->batch_stride_y, d->M, d->ldy, d->N) ||
      (residual && !spans(d->batch_stride_r, d->M, d->ldr, d->N)))
    return COMFUSE_ERR_INVALID_ARG;
  if (residual == Y && (d->ldr != d->ldy || (d->batch > 1 && d->batch_stride_r != d->batch_stride_y))) return COMFUSE_ERR_INVALID_ARG;
  const int e = dtype_bytes(d->dtype);
  if (!rows_aligned(d->lda, 1) || !rows_aligned(d->ldb, 1) || !rows_aligned(d->ldy, e) || (residual && !rows_aligned(d->ldr, e))) return COMFUSE_ERR_ALIGNMENT;
  if (d->batch > 1 && (!rows_aligned(d->batch_stride_a, 1) || !rows_aligned(d->batch_stride_b, 1) || !rows_aligned(d->batch_stride_y, e) ||
                       (residual && !rows_aligned(d->batch_stride_r, e))))
    return COMFUSE_ERR_ALIGNMENT;
  if (!aligned(A, 16) || !aligned(B, 16) || !aligned(bias, 16) || !aligned(residual, 16) || !aligned(Y, 16) || !aligned(scale_a, 4) || !aligned(scale_b, 4))
    return COMFUSE_ERR_ALIGNMENT;
  // 131072 * 128 * 128 leaves int32, and so would the rows of the last tile
  if (d->N > 65536 || d->K > 131071 || d->M >= 0x7FFFFF00) return COMFUSE_ERR_UNSUPPORTED;
  return COMFUSE_OK;
}

}  // namespace
}  // namespace comfuse

using namespace comfuse;

extern "C" {

comfuse_status_t comfuse_quantize_rows(const comfuse_quantize_desc_t* desc, const void* x, const void* residual, const void* gamma, void* h, int8_t* q,
                                       float* scale, void* values, void* cuda_stream) {
  comfuse_status_t s = check_quantize(desc, x, residual, gamma, h, q, scale, values);
  if (s != COMFUSE_OK) return s;
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  QuantizeRowsParams p = {};
  p.rows = desc->rows; p.N = desc->N;
  p.x = x; p.residual = residual; p.gamma = gamma; p.h = h;
  p.q = q; p.scale = scale; p.values = static_cast<uint16_t*>(values);
  p.ldx = desc->ldx; p.ldr = desc->ldr; p.ldh = desc->ldh; p.ldq = desc->ldq; p.ldv = desc->ldv;
  p.eps = desc->eps;
  p.status = dev->status_word;
  const cudaError_t e = launch_quantize_rows(desc->dtype, desc->kind == COMFUSE_QUANTIZE_RMSNORM, p, *dev, static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? COMFUSE_OK : COMFUSE_ERR_CUDA;
}

comfuse_status_t comfuse_gemm_q8(const comfuse_gemm_q8_desc_t* desc, const int8_t* A, const float* scale_a, const int8_t* B, const float* scale_b,
                                 const void* bias, const void* residual, void* Y, void* cuda_stream) {
  comfuse_status_t s = check_gemm(desc, A, scale_a, B, scale_b, bias, residual, Y);
  if (s != COMFUSE_OK) return s;
  const DeviceInfo* dev = nullptr;
  s = check_device(&dev);
  if (s != COMFUSE_OK) return s;
  const comfuse_gemm_q8_desc_t& d = *desc;
  auto stride = [&](long long given, long long rows, long long ld) { return static_cast<uint64_t>(d.batch > 1 ? given : rows * ld); };
  GemmQ8Params p = {};
  p.batch = d.batch; p.M = d.M; p.N = d.N; p.K = d.K;
  p.activation = d.activation;
  p.scale_a = scale_a; p.scale_b = scale_b; p.bias = bias; p.residual = residual; p.Y = Y;
  p.ldr = d.ldr; p.ldy = d.ldy;
  p.batch_stride_r = d.batch > 1 ? d.batch_stride_r : 0;
  p.batch_stride_y = d.batch > 1 ? d.batch_stride_y : 0;
  p.status = dev->status_word;
  p.timeout_ns = timeout_ns();
  const cudaStream_t st = static_cast<cudaStream_t>(cuda_stream);
  if (few_rows_enabled() && gemm_q8_tokens_fits(d.batch, d.M, d.N, d.K, *dev)) {
    const GemmQ8TokensParams t = {A, B, d.lda, d.ldb, d.batch > 1 ? d.batch_stride_a : 0, d.batch > 1 ? d.batch_stride_b : 0};
    return launch_gemm_q8_tokens(d.dtype, t, p, *dev, st) == cudaSuccess ? COMFUSE_OK : COMFUSE_ERR_CUDA;
  }
  GemmQ8FewPlan few;
  const bool long_epilogue = residual || (d.activation != 0 && d.activation != COMFUSE_OP_RELU);
  if (few_rows_enabled()) few = gemm_q8_few_plan(d.batch, d.M, d.N, d.K, long_epilogue, *dev);
  constexpr CUtensorMapDataType kCodes = CU_TENSOR_MAP_DATA_TYPE_UINT8;
  const uint64_t bsa = stride(d.batch_stride_a, d.M, d.lda), bsb = stride(d.batch_stride_b, d.N, d.ldb);
  if (few.rows) {
    CUtensorMap tmW, tmX;
    if (!encode_tmap_128b_3d(&tmX, kCodes, 1, A, d.K, d.M, d.batch, d.lda, bsa, few.rows) ||
        !encode_tmap_128b_3d(&tmW, kCodes, 1, B, d.K, d.N, d.batch, d.ldb, bsb, 128))
      return COMFUSE_ERR_CUDA;
    return launch_gemm_q8_few(d.dtype, few, tmW, tmX, p, st) == cudaSuccess ? COMFUSE_OK : COMFUSE_ERR_CUDA;
  }
  const CUtensorMapDataType type = d.dtype == COMFUSE_DTYPE_BF16  ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16
                                   : d.dtype == COMFUSE_DTYPE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                                                  : CU_TENSOR_MAP_DATA_TYPE_FLOAT32;
  if (static_cast<long long>(d.batch) * ((d.M + 255ll) / 256) * ((d.N + 127) / 128) > 0x7FFFFFFF) return COMFUSE_ERR_UNSUPPORTED;  // (tiles are counted in 32 bits)
  const int columns = gemm_q8_pair_columns(d.batch, d.M, d.N, *dev), e = dtype_bytes(d.dtype);
  const int stored = gemm_q8_stored_columns(d.dtype, d.N);  // (0: no store goes through the map)
  GemmQ8PairMaps maps;
  if (!encode_tmap_128b_3d(&maps.A, kCodes, 1, A, d.K, d.M, d.batch, d.lda, bsa, 128) ||
      !encode_tmap_128b_3d(&maps.B, kCodes, 1, B, d.K, d.N, d.batch, d.ldb, bsb, columns / 2) ||
      !encode_tmap_128b_3d(&maps.Y, type, e, Y, stored ? stored : d.N, d.M, d.batch, d.ldy, stride(d.batch_stride_y, d.M, d.ldy), 32))
    return COMFUSE_ERR_CUDA;
  maps.R = maps.Y;
  if (residual && !encode_tmap_128b_3d(&maps.R, type, e, residual, d.N, d.M, d.batch, d.ldr, stride(d.batch_stride_r, d.M, d.ldr), 32))
    return COMFUSE_ERR_CUDA;
  return launch_gemm_q8_pair(d.dtype, columns, maps, p, *dev, st) == cudaSuccess ? COMFUSE_OK : COMFUSE_ERR_CUDA;
}

}  // extern "C"
