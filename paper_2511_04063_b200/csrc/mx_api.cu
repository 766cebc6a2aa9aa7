// C entry points of the microscaled operators: checks of arguments, then the launches of mx_quant.cu and mx_matmul.cu.
#include "mx_common.cuh"

using namespace dq;

namespace {
constexpr int64_t MAX_K = (int64_t)1 << 24, MAX_ROWS = ((int64_t)1 << 31) - 256;
inline bool is_float(int t) { return t == DQ_FP32 || t == DQ_BF16 || t == DQ_FP16; }
inline bool is_format(int f) { return f == DQ_MXFP4 || f == DQ_MXFP8; }
inline dq_status sizes(int64_t rows, int64_t k) {
  if (rows < 0 || k <= 0) return DQ_ERR_INVALID_ARG;
  return rows > MAX_ROWS || k > MAX_K ? DQ_ERR_UNSUPPORTED : DQ_OK;
}
inline bool aligned(const void* p, uintptr_t to) { return ((uintptr_t)p & (to - 1)) == 0; }
// codes and scales as the kernels read and write them
inline dq_status quantised(const void* codes, const void* scales) {
  if (!codes || !scales) return DQ_ERR_INVALID_ARG;
  return aligned(codes, 32) && aligned(scales, 16) ? DQ_OK : DQ_ERR_UNSUPPORTED;
}
inline bool typed(const void* p, int dtype) { return aligned(p, dtype == DQ_FP32 ? 4 : 2); }
inline dq_status product_args(int a_fmt, const void* a_codes, const void* a_scales, int64_t m, const void* w_codes, const void* w_scales,
                              int64_t n, int64_t k, const void* Y, int y_dtype, int64_t ldy) {
  DQ_CHECK(sizes(m, k));
  DQ_CHECK(sizes(n, k));
  if (n == 0 || !is_format(a_fmt) || !is_float(y_dtype) || ldy < n) return DQ_ERR_INVALID_ARG;
  if (m == 0) return DQ_OK;
  if (!Y || !typed(Y, y_dtype)) return DQ_ERR_INVALID_ARG;
  DQ_CHECK(quantised(a_codes, a_scales));
  return quantised(w_codes, w_scales);
}
}  // namespace

extern "C" {

int64_t dq_mx_row_bytes(int32_t fmt, int64_t k) { return is_format(fmt) && sizes(0, k) == DQ_OK ? mx::row_bytes(fmt, k) : -1; }

int64_t dq_mx_scale_bytes(int64_t rows, int64_t k) { return sizes(rows, k) == DQ_OK ? mx::scale_bytes(rows, k) : -1; }

int64_t dq_mx_linear_workspace(int32_t a_fmt, int64_t m, int64_t k) {
  if (!is_format(a_fmt) || sizes(m, k) != DQ_OK) return -1;
  return m * mx::row_bytes(a_fmt, k) + mx::scale_bytes(m, k);
}

dq_status dq_mx_quantize(const void* d_X, int32_t x_dtype, int64_t rows, int64_t k, int64_t ldx, int32_t fmt, void* d_codes,
                         void* d_scales, void* d_values, int64_t ldv, void* cuda_stream) {
  DQ_CHECK(sizes(rows, k));
  if (!is_float(x_dtype) || !is_format(fmt) || ldx < k || (d_values && ldv < k)) return DQ_ERR_INVALID_ARG;
  if (rows == 0) return DQ_OK;
  if (!d_X) return DQ_ERR_INVALID_ARG;
  DQ_CHECK(quantised(d_codes, d_scales));
  if (!typed(d_X, x_dtype) || !typed(d_values, x_dtype)) return DQ_ERR_INVALID_ARG;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  return mx::quantize((cudaStream_t)cuda_stream, d_X, x_dtype, rows, k, ldx, fmt, (uint8_t*)d_codes, (uint8_t*)d_scales,
                      d_values, ldv);
}

dq_status dq_mx_dequantize(int32_t fmt, const void* d_codes, const void* d_scales, int64_t rows, int64_t k, void* d_Y,
                           int32_t y_dtype, int64_t ldy, void* cuda_stream) {
  DQ_CHECK(sizes(rows, k));
  if (!is_float(y_dtype) || !is_format(fmt) || ldy < k) return DQ_ERR_INVALID_ARG;
  if (rows == 0) return DQ_OK;
  if (!d_Y || !typed(d_Y, y_dtype)) return DQ_ERR_INVALID_ARG;
  DQ_CHECK(quantised(d_codes, d_scales));
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  return mx::dequantize((cudaStream_t)cuda_stream, fmt, (const uint8_t*)d_codes, (const uint8_t*)d_scales, rows, k, d_Y,
                        y_dtype, ldy);
}

dq_status dq_rmsnorm_quantize(const void* d_X, const void* d_residual, int32_t dtype, int64_t rows, int64_t k, int64_t ldx,
                              int64_t ldr, const void* d_gamma, int32_t gamma_dtype, float eps, int32_t fmt, void* d_codes,
                              void* d_scales, void* d_sum, int64_t lds, void* d_values, int64_t ldv, void* cuda_stream) {
  DQ_CHECK(sizes(rows, k));
  if (!is_float(dtype) || !is_format(fmt) || ldx < k || (d_residual && ldr < k) || (d_sum && lds < k) ||
      (d_values && ldv < k) || !(eps >= 0.f))
    return DQ_ERR_INVALID_ARG;
  if (d_gamma && gamma_dtype != DQ_FP32 && gamma_dtype != dtype) return DQ_ERR_INVALID_ARG;
  if (rows == 0) return DQ_OK;
  if (!d_X) return DQ_ERR_INVALID_ARG;
  DQ_CHECK(quantised(d_codes, d_scales));
  if (!typed(d_X, dtype) || !typed(d_residual, dtype) || !typed(d_sum, dtype) || !typed(d_values, dtype) ||
      !typed(d_gamma, gamma_dtype))
    return DQ_ERR_INVALID_ARG;
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  return mx::rmsnorm_quantize((cudaStream_t)cuda_stream, d_X, dtype, rows, k, ldx, d_residual, ldr, d_gamma, gamma_dtype, eps,
                              fmt, (uint8_t*)d_codes, (uint8_t*)d_scales, d_sum, lds, d_values, ldv);
}

dq_status dq_mx_matmul(int32_t a_fmt, const void* d_a_codes, const void* d_a_scales, int64_t m, const void* d_w_codes,
                       const void* d_w_scales, int64_t n, int64_t k, void* d_Y, int32_t y_dtype, int64_t ldy,
                       void* cuda_stream) {
  DQ_CHECK(product_args(a_fmt, d_a_codes, d_a_scales, m, d_w_codes, d_w_scales, n, k, d_Y, y_dtype, ldy));
  if (m == 0) return DQ_OK;
  return mx::matmul((cudaStream_t)cuda_stream, a_fmt, (const uint8_t*)d_a_codes, (const uint8_t*)d_a_scales, m,
                    (const uint8_t*)d_w_codes, (const uint8_t*)d_w_scales, n, k, d_Y, y_dtype, ldy);
}

dq_status dq_mx_selftest_bounded_wait(int32_t a_fmt, const void* d_a_codes, const void* d_a_scales, int64_t m, const void* d_w_codes,
                                      const void* d_w_scales, int64_t n, int64_t k, void* d_Y, int32_t y_dtype, int64_t ldy,
                                      int64_t step, uint64_t limit_ns, void* cuda_stream) {
  if (step < 0 || limit_ns == 0 || limit_ns > 100000000ull) return DQ_ERR_INVALID_ARG;   // at most 0.1 s
  DQ_CHECK(product_args(a_fmt, d_a_codes, d_a_scales, m, d_w_codes, d_w_scales, n, k, d_Y, y_dtype, ldy));
  if (m == 0) return DQ_OK;
  return mx::matmul_giving_up((cudaStream_t)cuda_stream, a_fmt, (const uint8_t*)d_a_codes, (const uint8_t*)d_a_scales, m,
                              (const uint8_t*)d_w_codes, (const uint8_t*)d_w_scales, n, k, d_Y, y_dtype, ldy, step, limit_ns);
}

dq_status dq_mx_linear(const void* d_X, int32_t x_dtype, int64_t m, int64_t k, int64_t ldx, int32_t a_fmt,
                       const void* d_w_codes, const void* d_w_scales, int64_t n, void* d_Y, int32_t y_dtype, int64_t ldy,
                       void* d_workspace, void* cuda_stream) {
  DQ_CHECK(sizes(m, k));
  DQ_CHECK(sizes(n, k));
  if (n == 0 || !is_float(x_dtype) || !is_format(a_fmt) || !is_float(y_dtype) || ldx < k || ldy < n) return DQ_ERR_INVALID_ARG;
  if (m == 0) return DQ_OK;
  if (!d_X || !d_Y || !d_workspace || !typed(d_X, x_dtype) || !typed(d_Y, y_dtype)) return DQ_ERR_INVALID_ARG;
  if (!aligned(d_workspace, 32)) return DQ_ERR_UNSUPPORTED;
  DQ_CHECK(quantised(d_w_codes, d_w_scales));
  return mx::linear((cudaStream_t)cuda_stream, d_X, x_dtype, m, k, ldx, a_fmt, (const uint8_t*)d_w_codes,
                    (const uint8_t*)d_w_scales, n, d_Y, y_dtype, ldy, (uint8_t*)d_workspace);
}

dq_status dq_mx_status(void* cuda_stream) {
  mx::Device dev;
  DQ_CHECK(mx::current_device(dev));
  int code = 0, zero = 0;
  cudaStream_t s = (cudaStream_t)cuda_stream;
  DQ_CHECK_CUDA(cudaMemcpyAsync(&code, dev.d_status, sizeof(int), cudaMemcpyDeviceToHost, s));
  DQ_CHECK_CUDA(cudaStreamSynchronize(s));
  if (code != 0) {
    DQ_CHECK_CUDA(cudaMemcpyAsync(dev.d_status, &zero, sizeof(int), cudaMemcpyHostToDevice, s));
    DQ_CHECK_CUDA(cudaStreamSynchronize(s));
  }
  return (dq_status)code;
}

}  // extern "C"
