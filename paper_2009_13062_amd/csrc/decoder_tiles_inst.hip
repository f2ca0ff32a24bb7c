// bfloat16 attention of prompts and trees: instances and launches of decoder_tiles.h.
#include <atomic>

#include "decoder_launch.h"
#include "decoder_tiles.h"
#include "nf_host.h"
#include "nf_launch.h"

namespace nf {
namespace {

template <int D, int KS, bool TREE, int FORM>
nf_status go_form(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  constexpr int kRows = 4 / KS * 32, kBytes = DecLds<D, 64 * KS>::kBytes;
  const long long R = (long long)a.N * (a.heads / a.kv), row_blocks = (R + kRows - 1) / kRows;
  const long long total = prod({a.M, a.B, a.kv, row_blocks, splits});
  if (!grid_fits(total, 256)) return NF_EUNSUPPORTED;
  const auto kernel = decoder_tiles_kernel<D, KS, TREE, FORM>;
  static std::atomic<bool> opted_in{false};                // more than 64 KB of LDS: one opt-in per process (idempotent)
  if (kBytes > 64 * 1024 && !opted_in.load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess) return NF_ELAUNCH;
    opted_in.store(true, std::memory_order_release);
  }
  nf_launch(kernel, dim3((unsigned)total), dim3(256), kBytes, s, a, (int)row_blocks, splits, chunk);
  return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH;
}

template <int D, int KS, bool TREE>
nf_status go(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  const bool raw = a.cap == 0.f && a.scale >= 1e-12f && a.scale <= 1e12f;          // a scale that the bias can be divided by
  if (a.slope) return raw ? go_form<D, KS, TREE, kRawBiased>(a, splits, chunk, s) : go_form<D, KS, TREE, kAnyBiased>(a, splits, chunk, s);
  return raw ? go_form<D, KS, TREE, kRawScore>(a, splits, chunk, s) : go_form<D, KS, TREE, kAnyScore>(a, splits, chunk, s);
}

}  // namespace

nf_status launch_prompt_tiles(const DecArgs& a, hipStream_t s) {
  return a.d <= 64 ? go<64, 1, false>(a, 1, 0, s) : a.d <= 128 ? go<128, 1, false>(a, 1, 0, s) : go<256, 1, false>(a, 1, 0, s);
}

nf_status launch_tree_tiles(const DecArgs& a, int chunk, int splits, hipStream_t s) {
  const int R = a.N * (a.heads / a.kv);
  // Up to 64 rows of small heads two wavefronts share the keys of 32 rows (16 caches of 4096 entries, 8 key heads, us, each its rows / shared: 20 rows 42.2 / 37.5, 36 38.7 /
  // 31.7, 64 40.0 / 33.2); larger heads would hold a whole LDS for it.
  if (a.d <= 64) return R <= 64 ? go<64, 2, true>(a, splits, chunk, s) : go<64, 1, true>(a, splits, chunk, s);
  return a.d <= 128 ? go<128, 1, true>(a, splits, chunk, s) : go<256, 1, true>(a, splits, chunk, s);
}

}  // namespace nf
