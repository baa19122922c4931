// What the operators on rows and weights in 8 bits check, and their launches.
#pragma once

namespace {

constexpr int kMostQuantRows = (1 << 24) - 1, kMostQuantDim = 1 << 20;   // a launch has fewer than 2^32 threads, 256 of them a row

int quant_blocks(int32_t dim) { return (dim + kQuantBlock - 1) / kQuantBlock; }

int check_rows_quant(const hsd_rows_quant *q, int32_t n_rows, int32_t dim) {
  if (n_rows < 0 || dim < 1) return HSD_EINVAL;
  if (n_rows > kMostQuantRows || dim > kMostQuantDim) return HSD_ERANGE;
  if (n_rows == 0) return HSD_OK;
  if (q == nullptr || q->codes == nullptr || q->scale == nullptr) return HSD_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q->codes) & 15) != 0 || (reinterpret_cast<uintptr_t>(q->scale) & 3) != 0) return HSD_EINVAL;
  if ((q->code_stride & 15) != 0 || (q->scale_stride & 3) != 0) return HSD_EINVAL;
  const int64_t blocks = quant_blocks(dim);
  return q->code_stride < blocks * kQuantBlock || q->scale_stride < (blocks + 3) / 4 * 4 ? HSD_EINVAL : HSD_OK;
}

int check_weight_quant(const hsd_weight_quant *w, int32_t n_out, int32_t dim) {
  if (w == nullptr || n_out < 1 || dim < 1) return HSD_EINVAL;
  if (n_out > kMostQuantRows || dim > kMostQuantDim) return HSD_ERANGE;
  if (w->codes == nullptr || w->scale == nullptr || (w->scale_type != HSD_SCALE_FP32 && w->scale_type != HSD_SCALE_POW2)) return HSD_EINVAL;
  if ((reinterpret_cast<uintptr_t>(w->codes) & 15) != 0 || (w->code_stride & 15) != 0) return HSD_EINVAL;
  if (w->scale_type == HSD_SCALE_FP32 && (reinterpret_cast<uintptr_t>(w->scale) & 3) != 0) return HSD_EINVAL;
  const int64_t blocks = quant_blocks(dim);
  return w->code_stride < blocks * kQuantBlock || w->scale_stride < blocks ? HSD_EINVAL : HSD_OK;
}

RowsQuant rows_quant(const hsd_rows_quant *q) { return RowsQuant{static_cast<uint8_t *>(q->codes), q->scale, q->code_stride, q->scale_stride}; }
WeightQuant weight_quant(const hsd_weight_quant *w) {
  return WeightQuant{static_cast<const uint8_t *>(w->codes), w->scale, w->code_stride, w->scale_stride, w->scale_type == HSD_SCALE_POW2};
}

template <typename TX, typename TR>
int launch_norm(hipStream_t st, const NormRows &a, const void *x, const void *res, void *sum) {
  hipLaunchKernelGGL((k_quant_rows<TX, TR>), dim3(static_cast<unsigned>(a.n_rows)), dim3(256), 0, st, a, static_cast<const TX *>(x),
                     static_cast<const TR *>(res), static_cast<TR *>(sum));
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int run_norm(hipStream_t st, const NormRows &a, int32_t x_dtype, const void *x, int32_t res_dtype, const void *res, void *sum) {
  if (x_dtype == HSD_BF16) return res_dtype == HSD_BF16 ? launch_norm<bf16, bf16>(st, a, x, res, sum) : launch_norm<bf16, float>(st, a, x, res, sum);
  return res_dtype == HSD_BF16 ? launch_norm<float, bf16>(st, a, x, res, sum) : launch_norm<float, float>(st, a, x, res, sum);
}

}  // namespace
