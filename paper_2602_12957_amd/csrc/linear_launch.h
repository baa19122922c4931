// What the operators on rows and weights in 8 bits check, and their launches.
#pragma once

namespace {

constexpr int kMostQuantRows = (1 << 24) - 1, kMostQuantDim = 1 << 20;   // a launch has fewer than 2^32 threads, 256 of them a row
constexpr int64_t kMostCodeStride = 1 << 23;                             // offsets within a tile of 256 rows take 31 bits

int quant_blocks(int32_t dim) { return (dim + kQuantBlock - 1) / kQuantBlock; }

int check_rows_quant(const hsd_rows_quant *q, int32_t n_rows, int32_t dim) {
  if (n_rows < 0 || dim < 1) return HSD_EINVAL;
  if (n_rows > kMostQuantRows || dim > kMostQuantDim) return HSD_ERANGE;
  if (n_rows == 0) return HSD_OK;
  if (q == nullptr || q->codes == nullptr || q->scale == nullptr) return HSD_EINVAL;
  if ((reinterpret_cast<uintptr_t>(q->codes) & 15) != 0 || (reinterpret_cast<uintptr_t>(q->scale) & 3) != 0) return HSD_EINVAL;
  if ((q->code_stride & 15) != 0 || (q->scale_stride & 3) != 0) return HSD_EINVAL;
  if (q->code_stride > kMostCodeStride) return HSD_ERANGE;
  const int64_t blocks = quant_blocks(dim);
  return q->code_stride < blocks * kQuantBlock || q->scale_stride < (blocks + 3) / 4 * 4 ? HSD_EINVAL : HSD_OK;
}

int check_weight_quant(const hsd_weight_quant *w, int32_t n_out, int32_t dim) {
  if (w == nullptr || n_out < 1 || dim < 1) return HSD_EINVAL;
  if (n_out > kMostQuantRows || dim > kMostQuantDim) return HSD_ERANGE;
  if (w->codes == nullptr || w->scale == nullptr || (w->scale_type != HSD_SCALE_FP32 && w->scale_type != HSD_SCALE_POW2)) return HSD_EINVAL;
  if ((reinterpret_cast<uintptr_t>(w->codes) & 15) != 0 || (w->code_stride & 15) != 0) return HSD_EINVAL;
  if (w->code_stride > kMostCodeStride) return HSD_ERANGE;
  if (w->scale_type == HSD_SCALE_FP32 && (reinterpret_cast<uintptr_t>(w->scale) & 3) != 0) return HSD_EINVAL;
  const int64_t blocks = quant_blocks(dim);
  return w->code_stride < blocks * kQuantBlock || w->scale_stride < blocks ? HSD_EINVAL : HSD_OK;
}

RowsQuant rows_quant(const hsd_rows_quant *q) { return RowsQuant{static_cast<uint8_t *>(q->codes), q->scale, q->code_stride, q->scale_stride}; }
WeightQuant weight_quant(const hsd_weight_quant *w) {
  return WeightQuant{static_cast<const uint8_t *>(w->codes), w->scale, w->code_stride, w->scale_stride};
}

template <typename TX, typename TR>
int launch_norm(hipStream_t st, const NormRows &a, const void *x, const void *res, void *sum) {
  const TX *px = static_cast<const TX *>(x);
  const TR *pr = static_cast<const TR *>(res);
  TR *ps = static_cast<TR *>(sum);
  auto launch = [&](auto kern, int wpr) {
    const int rows = std::max(4 / wpr, 1);   // of a workgroup; one where it takes several waves
    const int per = wpr == 1 ? rows : 1;
    hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((a.n_rows + per - 1) / per)), dim3(64 * wpr * per), 0, st, a, wpr, px, pr, ps);
  };
  // few rows: a lane's eight columns at a time, so that a row is short; many: up to 32, so that a row is a wave's own
  const int waves1 = (a.dim + 511) / 512, waves2 = (a.dim + 1023) / 1024, waves4 = (a.dim + 2047) / 2048;
  if (waves1 == 1 || (waves1 <= 16 && a.n_rows * waves1 <= 1024)) launch(k_quant_rows<TX, TR, 1>, waves1);
  else if (waves2 == 1) launch(k_quant_rows<TX, TR, 2>, 1);
  else if (waves4 <= 16) launch(k_quant_rows<TX, TR, 4>, waves4);
  else launch(k_quant_rows<TX, TR, 0>, 16);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int run_norm(hipStream_t st, const NormRows &a, int32_t x_dtype, const void *x, int32_t res_dtype, const void *res, void *sum) {
  if (x_dtype == HSD_BF16) return res_dtype == HSD_BF16 ? launch_norm<bf16, bf16>(st, a, x, res, sum) : launch_norm<bf16, float>(st, a, x, res, sum);
  return res_dtype == HSD_BF16 ? launch_norm<float, bf16>(st, a, x, res, sum) : launch_norm<float, float>(st, a, x, res, sum);
}

// Products of many rows
template <typename Cfg, bool GATED, bool FLOATS, bool EXACT, typename T>
int launch_product(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride, const RowsQuant &q) {
  auto kern = k_gemm_quant<Cfg, GATED, FLOATS, EXACT, T>;
  static const hipError_t attr_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, Cfg::kLds);
  if (attr_rc != hipSuccess) return HSD_EHIP;
  constexpr int COLS = GATED ? Cfg::BN / 2 : Cfg::BN;
  const int64_t tiles = static_cast<int64_t>((M + Cfg::BM - 1) / Cfg::BM) * ((N + COLS - 1) / COLS);
  if (tiles > INT32_MAX / Cfg::kThreads) return HSD_ERANGE;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(tiles)), dim3(Cfg::kThreads), Cfg::kLds, st, a, w, M, N, nk, out, out_stride, q);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

// Products of up to 64 rows
template <bool GATED, bool FLOATS, bool EXACT, int MT, typename T>
int launch_few(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride, const RowsQuant &q) {
  using Few = FewRows<MT>;
  auto kern = k_gemm_quant_few<GATED, FLOATS, EXACT, MT, T>;
  constexpr int per_wave = Few::kSlots * Few::kBlock;
  static_assert(!GATED || Few::kMostWaves == 16, "a wave for each 16 of the gate's and the up projection's 128 rows");
  static const hipError_t attr_rc = hipFuncSetAttribute(reinterpret_cast<const void *>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, Few::kMostWaves * per_wave);
  if (attr_rc != hipSuccess) return HSD_EHIP;
  const int waves = GATED ? 16 : std::min(nk, Few::kMostWaves), cols = GATED ? kQuantBlock : 16;
  hipLaunchKernelGGL(kern, dim3((N + cols - 1) / cols), dim3(64 * waves), waves * per_wave, st, a, w, M, N, nk, out, out_stride, q);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}
template <bool FLOATS, bool EXACT, typename T>
int launch_few_rows(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride) {
  const RowsQuant none{};
  if (M <= 16) return launch_few<false, FLOATS, EXACT, 1, T>(st, a, w, M, N, nk, out, out_stride, none);
  if (M <= 32) return launch_few<false, FLOATS, EXACT, 2, T>(st, a, w, M, N, nk, out, out_stride, none);
  return launch_few<false, FLOATS, EXACT, 4, T>(st, a, w, M, N, nk, out, out_stride, none);
}

int64_t quant_tiles(int M, int N, int bm, int bn) { return static_cast<int64_t>((M + bm - 1) / bm) * ((N + bn - 1) / bn); }

template <bool FLOATS, bool EXACT, typename T>
int run_linear(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride) {
  const RowsQuant none{};
#ifdef HSD_QUANT_TRY
  const char *e = getenv("HSD_QCFG");
  const int cfg = e ? atoi(e) : -1;
#define TRY(ok, id, ...) if constexpr (ok) { if (cfg == id) return launch_product<ProductTile<__VA_ARGS__>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none); }
  TRY(!FLOATS && !EXACT, 6, 256, 256, 2, 2, 2)
  TRY(!EXACT, 1, 256, 128, 4, 2, 3)
  TRY(true, 8, 128, 128, 2, 2, 2)
  if (cfg == 20) return launch_few_rows<FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride);
  TRY(true, 50, 64, 128, 2, 2, 5, 2, true)
  TRY(true, 51, 64, 128, 2, 2, 3, 2, true)
  TRY(true, 58, 64, 128, 2, 2, 3, 1, true)
  TRY(true, 52, 64, 64, 2, 2, 4, 2, true)
  TRY(!(FLOATS && EXACT), 56, 128, 128, 2, 2, 4, 1, true)
  TRY(!FLOATS && !EXACT, 54, 128, 128, 2, 2, 4, 2, true)
#endif
  if (M <= 16 || (M <= 64 && quant_tiles(M, N, 64, 64) < 128)) return launch_few_rows<FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride);
  if constexpr (!FLOATS && !EXACT) {
    if (quant_tiles(M, N, 256, 256) >= 192) return launch_product<ProductTile<256, 256, 2, 2, 2>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  }
  if (quant_tiles(M, N, 128, 128) >= 256) return launch_product<ProductTile<128, 128, 2, 2, 2>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  if (quant_tiles(M, N, 64, 128) >= 192) return launch_product<ProductTile<64, 128, 2, 2, 3, 2, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  return launch_product<ProductTile<64, 64, 2, 2, 4, 2, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
}

template <bool FLOATS>
int run_gated(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, const RowsQuant &q) {
  bf16 *none = nullptr;
#ifdef HSD_QUANT_TRY
  const char *e = getenv("HSD_QCFG");
  const int cfg = e ? atoi(e) : -1;
#define TRYG(ok, id, ...) if constexpr (ok) { if (cfg == id) return launch_product<ProductTile<__VA_ARGS__>, true, FLOATS, false, bf16>(st, a, w, M, N, nk, none, 0, q); }
  if (cfg == 20) return launch_few<true, FLOATS, false, 1, bf16>(st, a, w, M, N, nk, none, 0, q);
  TRYG(!FLOATS, 6, 256, 256, 2, 2, 2)
  TRYG(true, 4, 128, 256, 2, 4, 3)
  TRYG(!FLOATS, 60, 128, 256, 2, 2, 3, 1, true)
  TRYG(true, 61, 64, 256, 1, 4, 3, 1, true)
  TRYG(!FLOATS, 62, 64, 256, 1, 4, 3, 2, true)
  TRYG(true, 3, 64, 256, 1, 4, 3)
#endif
  if (M <= 16) return launch_few<true, FLOATS, false, 1, bf16>(st, a, w, M, N, nk, none, 0, q);
  if constexpr (!FLOATS) {
    if (quant_tiles(M, N, 256, 128) >= 192) return launch_product<ProductTile<256, 256, 2, 2, 2>, true, FLOATS, false, bf16>(st, a, w, M, N, nk, none, 0, q);
  }
  if (quant_tiles(M, N, 128, 128) >= 192) return launch_product<ProductTile<128, 256, 2, 4, 3>, true, FLOATS, false, bf16>(st, a, w, M, N, nk, none, 0, q);
  return launch_product<ProductTile<64, 256, 1, 4, 3, 1, true>, true, FLOATS, false, bf16>(st, a, w, M, N, nk, none, 0, q);
}

}  // namespace
