// C entries of the operators on rows and weights in 8 bits.
#pragma once

#include "linear_launch.h"

extern "C" {

int hsd_quant_rows(void *stream, int32_t n_rows, int32_t dim, int32_t dtype, const void *x, int64_t x_stride, const hsd_rows_quant *out) {
  const int rc = check_rows_quant(out, n_rows, dim);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype)) return HSD_EINVAL;
  if (n_rows == 0) return HSD_OK;
  if (x == nullptr || x_stride < dim) return HSD_EINVAL;
  const NormRows a{n_rows, dim, 0, nullptr, 0., x_stride, 0, 0, rows_quant(out)};
  return run_norm(static_cast<hipStream_t>(stream), a, dtype, x, dtype, nullptr, nullptr);
}

int hsd_quant_norm_rows(void *stream, int32_t n_rows, int32_t dim, int32_t dtype, const void *x, int64_t x_stride, int32_t res_dtype,
                        const void *residual, int64_t res_stride, void *sum, int64_t sum_stride, const float *gain, float eps,
                        const hsd_rows_quant *out) {
  const int rc = check_rows_quant(out, n_rows, dim);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype) || !is_type(res_dtype) || !(eps >= 0.f) || !std::isfinite(eps)) return HSD_EINVAL;
  if (n_rows == 0) return HSD_OK;
  if (x == nullptr || x_stride < dim || (residual != nullptr && res_stride < dim) || (sum != nullptr && sum_stride < dim)) return HSD_EINVAL;
  if (residual == nullptr && sum != nullptr) return HSD_EINVAL;
  const NormRows a{n_rows, dim, 1, gain, eps, x_stride, res_stride, sum_stride, rows_quant(out)};
  return run_norm(static_cast<hipStream_t>(stream), a, dtype, x, res_dtype, residual, sum);
}

int hsd_quant_read_rows(void *stream, int32_t n_rows, int32_t dim, const hsd_rows_quant *rows, int32_t dtype, void *out, int64_t out_stride) {
  const int rc = check_rows_quant(rows, n_rows, dim);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype)) return HSD_EINVAL;
  if (n_rows == 0) return HSD_OK;
  if (out == nullptr || out_stride < dim) return HSD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  int lanes = 16;   // of a row
  while (lanes < 256 && 8 * lanes < dim) lanes *= 2;
  const dim3 grid((static_cast<unsigned>(n_rows) + 256 / lanes - 1) / (256 / lanes));
  if (dtype == HSD_BF16)
    hipLaunchKernelGGL((k_quant_read_rows<bf16>), grid, dim3(256), 0, st, rows_quant(rows), n_rows, dim, lanes, static_cast<bf16 *>(out), out_stride);
  else
    hipLaunchKernelGGL((k_quant_read_rows<float>), grid, dim3(256), 0, st, rows_quant(rows), n_rows, dim, lanes, static_cast<float *>(out), out_stride);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int hsd_quant_weights(void *stream, int32_t n_out, int32_t dim, int32_t dtype, const void *w, int64_t w_stride, const hsd_weight_quant *out) {
  const int rc = check_weight_quant(out, n_out, dim);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype) || w == nullptr || w_stride < dim) return HSD_EINVAL;
  const dim3 grid(quant_blocks(dim), quant_blocks(n_out));
  if (grid.y > 65535) return HSD_ERANGE;
  uint8_t *codes = static_cast<uint8_t *>(const_cast<void *>(out->codes)), *byte = nullptr;
  float *scale = nullptr;
  if (out->scale_type == HSD_SCALE_POW2) byte = static_cast<uint8_t *>(const_cast<void *>(out->scale));
  else scale = static_cast<float *>(const_cast<void *>(out->scale));
  hipStream_t st = static_cast<hipStream_t>(stream);
  if (dtype == HSD_BF16)
    hipLaunchKernelGGL((k_quant_weights<bf16>), grid, dim3(256), 0, st, n_out, dim, static_cast<const bf16 *>(w), w_stride, codes, out->code_stride,
                       byte, scale, out->scale_stride);
  else
    hipLaunchKernelGGL((k_quant_weights<float>), grid, dim3(256), 0, st, n_out, dim, static_cast<const float *>(w), w_stride, codes, out->code_stride,
                       byte, scale, out->scale_stride);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int hsd_quant_linear(void *stream, int32_t n_rows, int32_t n_out, int32_t dim, const hsd_rows_quant *rows, const hsd_weight_quant *w, int32_t dtype,
                     void *out, int64_t out_stride) {
  int rc = check_rows_quant(rows, n_rows, dim);
  if (rc == HSD_OK) rc = check_weight_quant(w, n_out, dim);
  if (rc != HSD_OK) return rc;
  if (!is_type(dtype)) return HSD_EINVAL;
  if (n_rows == 0) return HSD_OK;
  if (out == nullptr || out_stride < n_out) return HSD_EINVAL;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const RowsQuant a = rows_quant(rows);
  const WeightQuant b = weight_quant(w);
  const int nk = quant_blocks(dim);
  const bool floats = w->scale_type == HSD_SCALE_FP32;
  if (dtype == HSD_BF16) {
    bf16 *y = static_cast<bf16 *>(out);
    return floats ? run_linear<true, false>(st, a, b, n_rows, n_out, nk, y, out_stride) : run_linear<false, false>(st, a, b, n_rows, n_out, nk, y, out_stride);
  }
  float *y = static_cast<float *>(out);
  return floats ? run_linear<true, true>(st, a, b, n_rows, n_out, nk, y, out_stride) : run_linear<false, true>(st, a, b, n_rows, n_out, nk, y, out_stride);
}

int hsd_quant_gated(void *stream, int32_t n_rows, int32_t d_ffn, int32_t dim, const hsd_rows_quant *rows, const hsd_weight_quant *w,
                    const hsd_rows_quant *out) {
  int rc = check_rows_quant(rows, n_rows, dim);
  if (rc != HSD_OK) return rc;
  if (d_ffn < 1 || d_ffn % kQuantBlock != 0) return HSD_EINVAL;
  if (d_ffn > kMostQuantDim) return HSD_ERANGE;
  rc = check_weight_quant(w, 2 * d_ffn, dim);
  if (rc == HSD_OK) rc = check_rows_quant(out, n_rows, d_ffn);
  if (rc != HSD_OK) return rc;
  if (n_rows == 0) return HSD_OK;
  hipStream_t st = static_cast<hipStream_t>(stream);
  const int nk = quant_blocks(dim);
  if (w->scale_type == HSD_SCALE_FP32) return run_gated<true>(st, rows_quant(rows), weight_quant(w), n_rows, d_ffn, nk, rows_quant(out));
  return run_gated<false>(st, rows_quant(rows), weight_quant(w), n_rows, d_ffn, nk, rows_quant(out));
}

}  // extern "C"
