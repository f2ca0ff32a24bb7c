// Attention of prompts and trees without LDS stages, weights of cached keys: instances and launches of decoder_stream.h and weigh_kernels.h.
#include <algorithm>
#include <atomic>

#include "decoder_launch.h"
#include "decoder_stream.h"
#include "nf_host.h"
#include "nf_launch.h"
#include "weigh_kernels.h"

namespace nf {
namespace {

inline nf_status launched() { return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH; }

template <typename T, int D, int RT, int KS, bool TREE>
nf_status go(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  constexpr int kRows = 4 / KS * RT * 16, kBytes = stream_lds_bytes(RT, KS, D / 16);
  const long long R = (long long)a.N * (a.heads / a.kv), row_blocks = (R + kRows - 1) / kRows;
  const long long total = prod({a.M, a.B, a.kv, row_blocks, splits});
  if (!grid_fits(total, 256)) return NF_EUNSUPPORTED;
  const auto kernel = decoder_stream_kernel<T, D, RT, KS, TREE>;
  static std::atomic<bool> opted_in{false};                // more than 64 KB of LDS: one opt-in per process (idempotent)
  if (kBytes > 64 * 1024 && !opted_in.load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess) return NF_ELAUNCH;
    opted_in.store(true, std::memory_order_release);
  }
  nf_launch(kernel, dim3((unsigned)total), dim3(256), kBytes, s, a, (int)row_blocks, splits, chunk);
  return launched();
}

template <typename T, int D>
nf_status tree(const DecArgs& a, int splits, int chunk, hipStream_t s) {
  const int R = a.N * (a.heads / a.kv);
  constexpr bool kBf = sizeof(T) == 2;                     // of more than 32 rows (16 up to 64 features): decoder_tiles.h
  if (R <= 16) return go<T, D, 1, 4, true>(a, splits, chunk, s);
  if constexpr (D == 128) {
    // 32 rows per wavefront: its keys and values serve twice the rows, and their loads are what bounds it (4 models of 4 caches of 4096 entries, 8 key heads of 128,
    // groups of 4, us, 16 rows / 32: bfloat16 5 tokens 73.6 / 55.6; float32 5 140 / 112, 12 187 / 176, 26 353 / 375; 8 heads of 64 31.3 / 33.7, of 256 spill)
    if (R <= 32) return go<T, D, 2, 4, true>(a, splits, chunk, s);
    if constexpr (!kBf) if (R <= 64) return go<T, D, 2, 2, true>(a, splits, chunk, s);
  } else if constexpr (D == 256 || !kBf) {
    if (R <= 32) return go<T, D, 1, 2, true>(a, splits, chunk, s);
  }
  if constexpr (kBf) return NF_EUNSUPPORTED;
  else return go<T, D, 1, 1, true>(a, splits, chunk, s);
}

// From 12 steps of keys on the four wavefronts of a workgroup share the keys of 16 rows, below that they take 16 rows each: by the length alone, so that a
// model's bits do not depend on what is merged with it (float32, 12 heads of 64, us, rows each / keys shared: 8 models of 128 tokens 12.4 / 11.3, 32 of 128 24.7 /
// 33.1, 12 of 300 38.5 / 42.2, 8 of 512 72.7 / 61.7, 2 of 1024 95.7 / 52.6, 8 of 1024 207 / 181; 16 heads of 128, 4 of 256 51.3 / 35.8, 4 of 1024 338 / 251).
template <typename T, int D>
nf_status prompt(const DecArgs& a, hipStream_t s) {
  return a.N >= 12 * 16 * StreamShape<T, D>::NK ? go<T, D, 1, 4, false>(a, 1, 0, s) : go<T, D, 1, 1, false>(a, 1, 0, s);
}

template <typename T, int D>
nf_status weigh(const WeighArgs& a, hipStream_t s) {
  constexpr int kKeys = 4 * weigh_keys<T, D>();            // of a workgroup and turn
  const long long heads = prod({a.M, a.B, a.kv}), pieces = ((long long)a.C + kKeys - 1) / kKeys;
  // as many turns as leave 16 workgroups per compute unit (one token over 32 caches of 8192 entries, 8 heads of 128: 4 turns 78 us, 8 81; before four wavefronts fit a SIMD
  // 1 turn 118, 2 102, 4 96, 8 95, 32 in a quarter of the workgroups 119)
  const int turns = (int)std::max<long long>(1, std::min<long long>(8, prod({heads, pieces}) / 4096));
  const int per_head = (int)((pieces + turns - 1) / turns);
  const long long blocks = prod({heads, per_head});
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  if ((long long)a.n * (a.heads / a.kv) > 16) nf_launch((weigh_tiles_kernel<T, D, true>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head, turns);
  else nf_launch((weigh_tiles_kernel<T, D, false>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head, turns);
  return launched();
}

}  // namespace

nf_status launch_prompt_stream(const DecArgs& a, hipStream_t s) {
  return a.d <= 64 ? prompt<float, 64>(a, s) : a.d <= 128 ? prompt<float, 128>(a, s) : prompt<float, 256>(a, s);
}

nf_status launch_tree_stream(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s) {
  if (dt == NF_F32) return a.d <= 64 ? tree<float, 64>(a, splits, chunk, s) : a.d <= 128 ? tree<float, 128>(a, splits, chunk, s) : tree<float, 256>(a, splits, chunk, s);
  return a.d <= 64 ? tree<bf16_t, 64>(a, splits, chunk, s) : a.d <= 128 ? tree<bf16_t, 128>(a, splits, chunk, s) : tree<bf16_t, 256>(a, splits, chunk, s);
}

// Up to 8 chunks a row's are loads of one group of lanes at a time; above that the groups of a workgroup share them (two caches of 196 chunks, whole call 142 us, by one group 162).
long long tree_join_blocks(const DecArgs& a, int splits) {
  const long long rows = prod({a.M, a.B, a.heads, a.N});
  return splits > 8 ? rows : (prod({rows, tree_features(a.d) / 4}) + 255) / 256;
}

nf_status launch_tree_join(const DecArgs& a, int chunk, int splits, nf_dtype dt, hipStream_t s) {
  const int features = tree_features(a.d);
  const bool shared = splits > 8;
  const long long blocks = tree_join_blocks(a, splits);
#define NF_JOIN(T, D, LOG2)                                                                                                              \
  if (shared) nf_launch((decoder_join_kernel<T, D, LOG2, 1024 / D>), dim3((unsigned)blocks), dim3(256), 0, s, a, splits, chunk);         \
  else nf_launch((decoder_join_kernel<T, D, LOG2, 1>), dim3((unsigned)blocks), dim3(256), 0, s, a, splits, chunk)
  if (dt == NF_F32) {
    if (features == 64) { NF_JOIN(float, 64, false); } else if (features == 128) { NF_JOIN(float, 128, false); } else { NF_JOIN(float, 256, false); }
  } else {
    if (features == 64) { NF_JOIN(bf16_t, 64, true); } else if (features == 128) { NF_JOIN(bf16_t, 128, true); } else { NF_JOIN(bf16_t, 256, true); }
  }
#undef NF_JOIN
  return launched();
}

nf_status launch_weigh_tiles(const WeighArgs& a, nf_dtype dt, hipStream_t s) {
  if (dt == NF_F32) return a.d <= 64 ? weigh<float, 64>(a, s) : a.d <= 128 ? weigh<float, 128>(a, s) : weigh<float, 256>(a, s);
  return a.d <= 64 ? weigh<bf16_t, 64>(a, s) : a.d <= 128 ? weigh<bf16_t, 128>(a, s) : weigh<bf16_t, 256>(a, s);
}

}  // namespace nf
