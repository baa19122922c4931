// What the operators on rows and weights in 8 bits check, and their launches.
#pragma once

#include <atomic>

namespace {

constexpr int kMostQuantRows = (1 << 24) - 1, kMostQuantDim = 1 << 20;   // a launch has fewer than 2^32 threads, up to 256 of them a row (the norm's: below)
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

RowsQuant rows_from(const RowsQuant &r, int64_t m) { return RowsQuant{r.codes + m * r.code_stride, r.scale + m * r.scale_stride, r.code_stride, r.scale_stride}; }

template <typename TX, typename TR>
int launch_norm(hipStream_t st, const NormRows &a, const void *x, const void *res, void *sum) {
  // (up to 1024 threads a row: launches of 2^31 threads at most)
  auto launch = [&](auto kern, int wpr) {
    const int held = wpr == 1 ? 4 : 1, most = (1 << 25) / wpr;   // rows of a workgroup and of a launch
    NormRows b = a;
    for (int64_t first = 0; first < a.n_rows; first += most) {
      const TX *px = static_cast<const TX *>(x) + first * a.x_stride;
      const TR *pr = res ? static_cast<const TR *>(res) + first * a.res_stride : nullptr;
      TR *ps = sum ? static_cast<TR *>(sum) + first * a.sum_stride : nullptr;
      b.n_rows = std::min<int64_t>(most, a.n_rows - first);
      b.out.codes = a.out.codes + first * a.out.code_stride, b.out.scale = a.out.scale + first * a.out.scale_stride;
      hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>((b.n_rows + held - 1) / held)), dim3(64 * wpr * held), 0, st, b, wpr, px, pr, ps);
    }
  };
  // few rows: a lane's eight columns at a time, so that a row is short; many: up to 32, so that a row is a wave's own
  const int waves1 = (a.dim + 511) / 512, waves2 = (a.dim + 1023) / 1024, waves4 = (a.dim + 2047) / 2048;
  if (waves1 == 1 || (waves1 <= 16 && a.n_rows * waves1 <= 1024)) launch(k_quant_rows<TX, TR, 1>, waves1);
  else if (waves2 == 1) launch(k_quant_rows<TX, TR, 2>, 1);
  else if (waves4 <= 8) launch(k_quant_rows<TX, TR, 4>, waves4);
  else launch(k_quant_rows<TX, TR, 0>, 16);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int run_norm(hipStream_t st, const NormRows &a, int32_t x_dtype, const void *x, int32_t res_dtype, const void *res, void *sum) {
  if (x_dtype == HSD_BF16) return res_dtype == HSD_BF16 ? launch_norm<bf16, bf16>(st, a, x, res, sum) : launch_norm<bf16, float>(st, a, x, res, sum);
  return res_dtype == HSD_BF16 ? launch_norm<float, bf16>(st, a, x, res, sum) : launch_norm<float, float>(st, a, x, res, sum);
}

constexpr int kUnits = 256;   // compute units

// Lets a kernel have `bytes` of LDS on the current device (asked for once a device; `done`: a bit a device, of the kernel's own)
hipError_t allow_lds(const void *kern, int bytes, std::atomic<uint64_t> &done) {
  int dev = 0;
  if (const hipError_t rc = hipGetDevice(&dev); rc != hipSuccess) return rc;
  const uint64_t bit = uint64_t{1} << (dev & 63);
  if (dev < 64 && (done.load(std::memory_order_relaxed) & bit) != 0) return hipSuccess;
  const hipError_t rc = hipFuncSetAttribute(kern, hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (rc == hipSuccess) done.fetch_or(bit, std::memory_order_relaxed);
  return rc;
}

template <typename Cfg, bool GATED, bool FLOATS, bool EXACT, typename T>
int launch_product(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride, const RowsQuant &q) {
  auto kern = k_gemm_quant<Cfg, GATED, FLOATS, EXACT, T>;
  static std::atomic<uint64_t> done{0};
  if (allow_lds(reinterpret_cast<const void *>(kern), Cfg::kLds, done) != hipSuccess) return HSD_EHIP;
  constexpr int COLS = GATED ? Cfg::BN / 2 : Cfg::BN;
  // (launches of 2^31 threads at most, by whole tiles of rows: 2^24 rows to 8192 gated take two)
  const int tiles_n = (N + COLS - 1) / COLS, most = INT32_MAX / Cfg::kThreads / tiles_n * Cfg::BM;
  for (int64_t first = 0; first < M; first += most) {
    const int rows = static_cast<int>(std::min<int64_t>(most, M - first));
    const unsigned tiles = static_cast<unsigned>((rows + Cfg::BM - 1) / Cfg::BM) * tiles_n;
    hipLaunchKernelGGL(kern, dim3(tiles), dim3(Cfg::kThreads), Cfg::kLds, st, rows_from(a, first), w, rows, N, nk, GATED ? out : out + first * out_stride, out_stride,
                       GATED ? rows_from(q, first) : q);
  }
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

template <bool FLOATS, bool EXACT, int MT, typename T>
int launch_few(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride) {
  using Few = FewRows<MT>;
  auto kern = k_gemm_quant_few<FLOATS, EXACT, MT, T>;
  constexpr int per_wave = Few::kSlots * Few::kBlock;
  static std::atomic<uint64_t> done{0};
  if (allow_lds(reinterpret_cast<const void *>(kern), Few::kMostWaves * per_wave, done) != hipSuccess) return HSD_EHIP;
  const int waves = std::min(nk, Few::kMostWaves);
  hipLaunchKernelGGL(kern, dim3((N + 15) / 16), dim3(64 * waves), waves * per_wave, st, a, w, M, N, nk, out, out_stride);
  HSD_LAUNCH_CHECK();
  return HSD_OK;
}

int64_t quant_tiles(int M, int N, int bm, int bn) { return static_cast<int64_t>((M + bm - 1) / bm) * ((N + bn - 1) / bn); }
int64_t rounds(int64_t tiles) { return (tiles + kUnits - 1) / kUnits; }
// Rows at the end of a call that would cost tiles of 256 rows a round of their own over the chip, and that go by themselves instead (32772 rows
// of 4096 to 1024, four of them in 516 - 512 tiles: 164 us in one launch, 134 in two); 0: none
int last_rows(int M, int N, int bn) {
  const int rest = M % 256;
  return rest > 0 && rest <= 64 && M > 256 && rounds(quant_tiles(M, N, 256, bn)) > rounds(quant_tiles(M - rest, N, 256, bn)) ? rest : 0;
}

// The form of a product goes by how many tiles it has: the smallest tiles that leave no second round over the chip (a compute unit works as fast on
// one large tile as on a small one, until it has all that the matrix unit can do); us a call, by tiles of 64x64 / 64x128 / 128x128 / 128x128 two a
// unit / 256x256, 1024 columns to 4096 and 16384 rows of weights:
//   200 rows to 4096  4.7 /  5.5 /  6.9 /  8.4 / 15.5     512 to 4096   7.1 /  6.0 /  7.4 /  8.8 / 15.9     1024 to 4096   12.3 /  9.4 /  8.7 /  9.8 / 16.5
//   2048 to 4096     20.6 / 15.9 / 15.4 / 13.8 / 17.8     4096 to 4096 38.1 / 29.5 / 28.1 / 24.0 / 21.8     4096 to 16384 176.5 / 130.4 / 139.5 / 109.6 / 82.8
// Few rows: a split of K over waves (k_gemm_quant_few), where that makes enough workgroups but not too many, each of which reads all rows: 64 rows of 4096 to
// 1024 6.7 where tiles take 8.6, to 4096 8.2 / 8.7; 16 of 8192 to 8192 17.1 / 20.0, of 4096 to 16384 20.8 / 16.8.
// The count of tiles does not see that few rows leave most of a large one empty: beyond 32768 columns 64x128 would be the better ones for them (1 row of 1024 to
// 131072 in 256x256 37.4, in 64x128 26.3; 64 rows 41.1 / 30.7).
template <bool FLOATS, bool EXACT, typename T>
int run_linear(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, T *out, int64_t out_stride) {
  const RowsQuant none{};
  if ((M <= 64 && N <= 4096) || (M <= 16 && N <= 8192)) {
    if (M <= 16) return launch_few<FLOATS, EXACT, 1, T>(st, a, w, M, N, nk, out, out_stride);
    if (M <= 32) return launch_few<FLOATS, EXACT, 2, T>(st, a, w, M, N, nk, out, out_stride);
    return launch_few<FLOATS, EXACT, 4, T>(st, a, w, M, N, nk, out, out_stride);
  }
  if (quant_tiles(M, N, 64, 64) <= kUnits) return launch_product<ProductTile<64, 64, 2, 2, 4, 2, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  if (quant_tiles(M, N, 64, 128) <= kUnits) return launch_product<ProductTile<64, 128, 2, 2, 3, 2, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  if constexpr (EXACT) {
    // (a block's sums beside the sums take the registers of larger tiles with float scales: 4096 rows of 4096 to 4096 143 us in tiles of 64x128, 159 of
    // 128x128, of 1024 47.0 / 46.6; with scales in bytes 136 / 121)
    if constexpr (FLOATS) return launch_product<ProductTile<64, 128, 2, 2, 3, 1, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
    else return launch_product<ProductTile<128, 128, 2, 2, 2>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
  } else {
    const int64_t tiles = quant_tiles(M, N, 128, 128);
    if (tiles <= kUnits) return launch_product<ProductTile<128, 128, 2, 2, 4, 2, true>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
    if (tiles <= 2 * kUnits) return launch_product<ProductTile<128, 128, 2, 2, 2>, false, FLOATS, EXACT, T>(st, a, w, M, N, nk, out, out_stride, none);
    // (eight waves: two a SIMD, one's first reads and results beside the other's products, and sums that the vector unit can multiply where they are, for
    // float scales.  Four, whose operands come from LDS two thirds as often: 32768 rows of 4096 to 1024 128.8 us, here 124.5; 8192^3 437, here 443)
    using Cfg = ProductTile<256, 256, 4, 2, 2>;
    const int rest = last_rows(M, N, Cfg::BN);
    const int rc = launch_product<Cfg, false, FLOATS, EXACT, T>(st, a, w, M - rest, N, nk, out, out_stride, none);
    if (rc != HSD_OK || rest == 0) return rc;
    return run_linear<FLOATS, EXACT, T>(st, rows_from(a, M - rest), w, rest, N, nk, out + (M - rest) * out_stride, out_stride);
  }
}

// Gate and up: bf16 products of the codes, so that rows in 8 bits differ from the definition's by fp32's roundings alone (8-bit products took 293 us where these take 458, and move
// values across the borders between codes: errors of a feed-forward block 1.1 to 1.9 times those of the definition's roundings).  Tiles of 32, 64, 128 or 256 rows by
// 128 columns of both, the smallest that leave no second round, 256 beyond; us a call, 1024 columns to 4096: 16 rows of 32 / 64 8.2 / 10.2, 512 16.9 / 12.5,
// 1024 of 64 / 128 / 256 21.9 / 19.0 / 25.9, 1856 40.2 / 33.3 / 30.9, 32768 636 / 537 / 458 (with float scales 520 to 541)
template <bool FLOATS>
int run_gated(hipStream_t st, const RowsQuant &a, const WeightQuant &w, int M, int N, int nk, const RowsQuant &q) {
  bf16 *none = nullptr;
  if (quant_tiles(M, N, 32, 128) <= kUnits) return launch_product<ProductTile<32, 256, 1, 4, 4, 2, true>, true, FLOATS, true, bf16>(st, a, w, M, N, nk, none, 0, q);
  if (quant_tiles(M, N, 64, 128) <= kUnits) return launch_product<ProductTile<64, 256, 1, 4, 3, 1, true>, true, FLOATS, true, bf16>(st, a, w, M, N, nk, none, 0, q);
  if (quant_tiles(M, N, 128, 128) <= kUnits) return launch_product<ProductTile<128, 256, 2, 4, 3>, true, FLOATS, true, bf16>(st, a, w, M, N, nk, none, 0, q);
  const int rest = last_rows(M, N, 128);
  const int rc = launch_product<ProductTile<256, 256, 4, 2, 2>, true, FLOATS, true, bf16>(st, a, w, M - rest, N, nk, none, 0, q);
  if (rc != HSD_OK || rest == 0) return rc;
  return run_gated<FLOATS>(st, rows_from(a, M - rest), w, rest, N, nk, rows_from(q, M - rest));
}

}  // namespace
