// Attention of drafted trees over a cache of 4 bits on the matrix pipe: instances and launches of decoder_stream.h and decoder_tiles.h.
#include <limits.h>

#include <atomic>

#include "decoder_launch.h"
#include "decoder_stream.h"
#include "decoder_tiles.h"
#include "nf_host.h"
#include "nf_launch.h"

namespace nf {
namespace {

template <typename T, int D, int RT, int KS, bool EXACT, bool FOLD>
nf_status go_rows(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  constexpr int kRows = 4 / KS * RT * 16, kBytes = stream_lds_bytes(RT, KS, D / 16);
  const long long R = (long long)a.N * (a.heads / a.kv), row_blocks = (R + kRows - 1) / kRows;
  const long long total = prod({a.M, a.B, a.kv, row_blocks, splits});
  if (!grid_fits(total, 256)) return NF_EUNSUPPORTED;
  const auto kernel = decoder_stream_kernel<T, D, RT, KS, true, true, EXACT, FOLD>;
  static std::atomic<bool> opted_in{false};                // more than 64 KB of LDS: one opt-in per process (idempotent)
  if (kBytes > 64 * 1024 && !opted_in.load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess) return NF_ELAUNCH;
    opted_in.store(true, std::memory_order_release);
  }
  nf_launch(kernel, dim3((unsigned)total), dim3(256), kBytes, s, a, (int)row_blocks, splits, chunk);
  return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH;
}

template <typename T, int D, int RT, int KS, bool FOLD = false>
nf_status go(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  return a.d == D ? go_rows<T, D, RT, KS, true, FOLD>(a, splits, chunk, s) : go_rows<T, D, RT, KS, false, FOLD>(a, splits, chunk, s);
}

template <typename T, int D>
nf_status tree(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  const int R = a.N * (a.heads / a.kv);
  // 32 rows per wavefront would open keys and values once for both halves, but hold few other registers (8 tokens of groups of 4 over 32 caches of 4096, 8 key heads of 128: 58 us,
  // 32 rows 61; float32 84 and 314).
  // Up to 4 rows share their scores among four lanes (one token of groups of 4 over the two long caches 49 us, shared 46; of 8 rows among two the gain was 2 % at most).
  constexpr int kMost = sizeof(T) == 4 ? INT_MAX : tree_fp4_streamed(D);                // rows that come here
  if constexpr (D <= 128) if (R <= 4) return go<T, D, 1, 4, true>(a, splits, chunk, s);
  if constexpr (kMost > 32) if (R > 32) return go<T, D, 1, 1>(a, splits, chunk, s);
  if constexpr (kMost > 16) if (R > 16) return go<T, D, 1, 2>(a, splits, chunk, s);
  return go<T, D, 1, 4>(a, splits, chunk, s);
}

template <int D, int KS, int FORM>
nf_status go_tiles(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  constexpr int kRows = 4 / KS * 32, kBytes = DecLds<D, 64 * KS>::kBytes;
  const long long R = (long long)a.N * (a.heads / a.kv), row_blocks = (R + kRows - 1) / kRows;
  const long long total = prod({a.M, a.B, a.kv, row_blocks, splits});
  if (!grid_fits(total, 256)) return NF_EUNSUPPORTED;
  const auto kernel = decoder_tiles_kernel<D, KS, true, FORM, true>;
  static std::atomic<bool> opted_in{false};
  if (kBytes > 64 * 1024 && !opted_in.load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess) return NF_ELAUNCH;
    opted_in.store(true, std::memory_order_release);
  }
  nf_launch(kernel, dim3((unsigned)total), dim3(256), kBytes, s, a, (int)row_blocks, splits, chunk);
  return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH;
}

template <int D, int KS>
nf_status tiles(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  const bool raw = a.cap == 0.f && a.scale >= 1e-12f && a.scale <= 1e12f;          // a scale that the bias can be divided by
  if (a.slope) return raw ? go_tiles<D, KS, kRawBiased>(a, splits, chunk, s) : go_tiles<D, KS, kAnyBiased>(a, splits, chunk, s);
  return raw ? go_tiles<D, KS, kRawScore>(a, splits, chunk, s) : go_tiles<D, KS, kAnyScore>(a, splits, chunk, s);
}

}  // namespace

nf_status launch_tree_fp4_tiles(const DecArgs& a, int chunk, int splits, hipStream_t s) {
  const int R = a.N * (a.heads / a.kv);
  if (a.d <= 64) return R <= 64 ? tiles<64, 2>(a, splits, chunk, s) : tiles<64, 1>(a, splits, chunk, s);
  return a.d <= 128 ? tiles<128, 1>(a, splits, chunk, s) : tiles<256, 1>(a, splits, chunk, s);
}

nf_status launch_tree_fp4_stream(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s) {
  if (dt == NF_F32) return a.d <= 64 ? tree<float, 64>(a, splits, chunk, s) : a.d <= 128 ? tree<float, 128>(a, splits, chunk, s) : tree<float, 256>(a, splits, chunk, s);
  return a.d <= 64 ? tree<bf16_t, 64>(a, splits, chunk, s) : a.d <= 128 ? tree<bf16_t, 128>(a, splits, chunk, s) : tree<bf16_t, 256>(a, splits, chunk, s);
}

}  // namespace nf
