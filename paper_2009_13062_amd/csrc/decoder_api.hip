// C ABI of the decoders' operators (attention of prompts and of drafted trees, the cache): argument validation on the host before any
// HIP call, kernel selection by sizes, type and alignment, launch with the models folded into the grid.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "cache_kernels.h"
#include "decoder.h"
#include "decoder_generic.h"
#include "decoder_launch.h"
#include "nf_host.h"
#include "nf_launch.h"

using namespace nf;

namespace {

inline nf_status launched() { return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH; }

bool score_ok(float scale, float cap) {
  return std::isfinite(scale) && (cap == 0.f || (cap >= 1e-30f && cap <= 1e30f));
}

// Rows of M models, `rows` of `width` elements each: a row's heads side by side, models one behind the other.
bool rows_ok(int M, long long rows, long long width, long stride_m, long stride_row) {
  if (width > INT_MAX || stride_row < width || stride_m < 0) return false;
  if (prod({rows, stride_row}) >= kMaxElems || prod({M, stride_m}) >= kMaxElems) return false;
  return M == 1 || stride_m >= (rows - 1) * stride_row + width;
}

constexpr int kMostEntries = 1 << 30;                      // slot numbers and what is added to them stay in an int

bool heads_ok(int heads, int kv_heads, int d) { return heads > 0 && kv_heads > 0 && d > 0 && heads % kv_heads == 0; }

// What the kernels on the matrix pipe take: rows in 16-byte pieces, row numbers in an int.
bool pieces_sizes(int N, int heads, int kv_heads, int d, nf_dtype dt) {
  return d % (dt == NF_F32 ? 4 : 8) == 0 && d <= 256 && (long long)N * (heads / kv_heads) <= INT_MAX / 2;
}
bool pieces_strides(long stride_m, long stride_row, nf_dtype dt) {
  const int n = dt == NF_F32 ? 4 : 8;
  return stride_m % n == 0 && stride_row % n == 0;
}
// The bfloat16 kernels on the matrix pipe take scale / cap in one factor, which has to be a normal number.  (Two factors there cost 4 % of the weights of a capped token;
// the general kernels have them.)
bool ratio_ok(float scale, float cap, nf_dtype dt) {
  const double r = cap != 0.f ? fabs((double)scale) / cap : 0.0;
  return dt == NF_F32 || r == 0.0 || (r > 1e-37 && r < 1e38);
}
bool pieces_ok(const DecArgs& a, nf_dtype dt) {
  // 64 rows of keys within 31 bits of bytes: a tile's offsets
  return ratio_ok(a.scale, a.cap, dt) && a.kv_stride_row < (1L << 31) / 64 / (dt == NF_F32 ? 4 : 2) && pieces_sizes(a.N, a.heads, a.kv, a.d, dt) && pieces_strides(a.q_stride_m, a.q_stride_row, dt) && pieces_strides(a.kv_stride_m, a.kv_stride_row, dt) &&
         aligned(a.Q, 16) && aligned(a.K, 16) && aligned(a.V, 16) && aligned(a.Kc, 16) && aligned(a.Vc, 16) && aligned(a.O, 16);
}

template <bool TREE>
nf_status launch_rows(const DecArgs& a, nf_dtype dt, hipStream_t s) {
  const long long blocks = (prod({a.M, a.B, a.heads, a.N}) + 3) / 4;
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
#define NF_ROWS(T, DPL) nf_launch((decoder_rows_kernel<T, DPL, TREE>), dim3((unsigned)blocks), dim3(256), 0, s, a)
  if (dt == NF_F32) {
    if (a.d <= 64) NF_ROWS(float, 1); else if (a.d <= 128) NF_ROWS(float, 2); else NF_ROWS(float, 4);
  } else {
    if (a.d <= 64) NF_ROWS(bf16_t, 1); else if (a.d <= 128) NF_ROWS(bf16_t, 2); else NF_ROWS(bf16_t, 4);
  }
#undef NF_ROWS
  return launched();
}

template <int NT, int E, bool MOVE = false, typename U = uint32_t>
nf_status select_held(const EvictArgs& a, long long heads, hipStream_t s) {
  constexpr int kBytes = EvictLds<NT, E>::kBytes;
  const auto kernel = evict_select_held_kernel<NT, E, MOVE, U>;
  static std::atomic<bool> opted_in{false};                // more than 64 KB of LDS: one opt-in per process (idempotent)
  if (kBytes > 64 * 1024 && !opted_in.load(std::memory_order_acquire)) {
    if (hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, kBytes) != hipSuccess) return NF_ELAUNCH;
    opted_in.store(true, std::memory_order_release);
  }
  nf_launch(kernel, dim3((unsigned)heads), dim3(NT), kBytes, s, a);
  return launched();
}

}  // namespace

extern "C" {

nf_status netfuse_attention_prompt(const void* Q, const void* K, const void* V, const float* slope, const int* len,
                                   const int* prefix, const int* doc, void* O, int M, int B, int S, int heads, int kv_heads,
                                   int d, long q_stride_m, long q_stride_row, long kv_stride_m, long kv_stride_row, int causal,
                                   float scale, float cap, nf_dtype dt, void* stream) {
  if (!Q || !K || !V || !O) return NF_EINVAL;
  if (M <= 0 || B <= 0 || S <= 0 || !heads_ok(heads, kv_heads, d)) return NF_EINVAL;
  if (!is_dtype(dt) || !score_ok(scale, cap) || (prefix && !causal)) return NF_EINVAL;
  if (prod({B, S}) > INT_MAX / 2 || prod({M, B, S, heads, d}) >= kMaxElems) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * S, (long long)heads * d, q_stride_m, q_stride_row) ||
      !rows_ok(M, (long long)B * S, (long long)kv_heads * d, kv_stride_m, kv_stride_row))
    return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Q, esz) || !aligned(K, esz) || !aligned(V, esz) || !aligned(O, esz) || !aligned(slope, 4) || !aligned(len, 4) ||
      !aligned(prefix, 4) || !aligned(doc, 4))
    return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  DecArgs a = {};
  a.Q = Q; a.K = K; a.V = V; a.slope = slope; a.len = len; a.prefix = prefix; a.doc = doc; a.O = O;
  a.M = M; a.B = B; a.N = S; a.heads = heads; a.kv = kv_heads; a.d = d; a.causal = causal != 0;
  a.q_stride_m = q_stride_m; a.q_stride_row = q_stride_row; a.kv_stride_m = kv_stride_m; a.kv_stride_row = kv_stride_row;
  a.scale = scale; a.cap = cap; a.inv_cap = cap != 0.f ? 1.f / cap : 0.f;
  if (pieces_ok(a, dt)) return dt == NF_BF16 ? launch_prompt_tiles(a, (hipStream_t)stream) : launch_prompt_stream(a, (hipStream_t)stream);
  return launch_rows<false>(a, dt, (hipStream_t)stream);
}

long long netfuse_attention_tree_workspace(int M, int B, int T, int C, int heads, int kv_heads, int d, nf_dtype dt) {
  if (M <= 0 || B <= 0 || T <= 0 || T > 64 || C <= 0 || C > kMostEntries || !heads_ok(heads, kv_heads, d) || d > 256 || !is_dtype(dt)) return -1;
  if (!pieces_sizes(T, heads, kv_heads, d, dt)) return 0;
  const int chunk = tree_chunk(T * (heads / kv_heads), dt), splits = (int)(((long long)C + chunk - 1) / chunk);
  if (splits == 1) return 0;                               // no cache is shared out
  const long long bytes = prod({M, B, heads, T, splits, 4LL * (tree_features(d) + 2)});      // a row's sums, its maximum and its total per chunk
  return bytes >= kMaxElems ? -1 : bytes;
}

nf_status netfuse_attention_tree(const void* Q, const void* K, const void* V, const void* Kc, const void* Vc, const int* pos,
                                 const int* len, const int* start, const int* parent, const int* nodes, const float* slope,
                                 void* O, float* lse, void* workspace, long long workspace_bytes, int M, int B, int T, int C,
                                 int heads, int kv_heads, int d, long q_stride_m, long q_stride_row, long kv_stride_m,
                                 long kv_stride_row, float scale, float cap, nf_dtype dt, void* stream) {
  if (!Q || !K || !V || !Kc || !Vc || !len || !O) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || C <= 0 || C > kMostEntries || !heads_ok(heads, kv_heads, d)) return NF_EINVAL;
  if (!is_dtype(dt) || !score_ok(scale, cap)) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({M, B, T, heads, d}) >= kMaxElems || prod({M, B, kv_heads, C, d}) >= kMaxElems) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, (long long)heads * d, q_stride_m, q_stride_row) ||
      !rows_ok(M, (long long)B * T, (long long)kv_heads * d, kv_stride_m, kv_stride_row))
    return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Q, esz) || !aligned(K, esz) || !aligned(V, esz) || !aligned(Kc, esz) || !aligned(Vc, esz) || !aligned(O, esz) ||
      !aligned(pos, 4) || !aligned(len, 4) || !aligned(start, 4) || !aligned(parent, 4) || !aligned(nodes, 4) || !aligned(slope, 4) ||
      !aligned(lse, 4) || !aligned(workspace, 16))
    return NF_EINVAL;
  if (T > 64 || d > 256) return NF_EUNSUPPORTED;
  const long long need = netfuse_attention_tree_workspace(M, B, T, C, heads, kv_heads, d, dt);
  if (need < 0) return NF_EUNSUPPORTED;
  if (need > 0 && (!workspace || workspace_bytes < need)) return NF_EINVAL;
  DecArgs a = {};
  a.Q = Q; a.K = K; a.V = V; a.Kc = Kc; a.Vc = Vc; a.slope = slope; a.len = len; a.start = start; a.parent = parent; a.nodes = nodes;
  a.pos = pos; a.O = O; a.lse = lse; a.ws = (float*)workspace;
  a.M = M; a.B = B; a.N = T; a.C = C; a.heads = heads; a.kv = kv_heads; a.d = d;
  a.q_stride_m = q_stride_m; a.q_stride_row = q_stride_row; a.kv_stride_m = kv_stride_m; a.kv_stride_row = kv_stride_row;
  a.scale = scale; a.cap = cap; a.inv_cap = cap != 0.f ? 1.f / cap : 0.f;
  if (pieces_ok(a, dt)) {
    const int rows = T * (heads / kv_heads), chunk = tree_chunk(rows, dt), splits = (int)(((long long)C + chunk - 1) / chunk);
    if (splits > 1 && !grid_fits(tree_join_blocks(a, splits), 256)) return NF_EUNSUPPORTED;      // before the first of the two is enqueued
    // Many rows of bfloat16 take their keys through LDS, few ones straight into registers (16 caches of 4096 entries, groups of 4, us, registers / LDS: 8 key heads of 128 features, 20 rows
    // 53 / 66, 36 66 / 56, 64 67 / 58; 8 of 64, 20 rows 41 / 37; 4 of 256, 20 rows 68 / 85, 36 76 / 78; 32 caches of 700, 8 key heads of 128, 18 rows 25 / 29, 64 features 20.6 / 18.3).
    const bool tiles = dt == NF_BF16 && rows > (d <= 64 ? 16 : 32);
    const nf_status st = tiles ? launch_tree_tiles(a, chunk, splits, (hipStream_t)stream) : launch_tree_stream(a, chunk, splits, dt, (hipStream_t)stream);
    return st != NF_OK || splits == 1 ? st : launch_tree_join(a, chunk, splits, dt, (hipStream_t)stream);
  }
  return launch_rows<true>(a, dt, (hipStream_t)stream);
}

nf_status netfuse_cache_append(const void* K, const void* V, const int* index, const int* count, const int* len, const int* start,
                               void* Kc, void* Vc, int* pos, float* weight, int M, int B, int T, int n, int C, int kv_heads, int d,
                               long kv_stride_m, long kv_stride_row, nf_dtype dt, void* stream) {
  if (!K || !V || !Kc || !Vc || !len) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || n <= 0 || C <= 0 || C > kMostEntries || kv_heads <= 0 || d <= 0 || !is_dtype(dt)) return NF_EINVAL;
  if (!index && n != T) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({B, n}) > INT_MAX / 2 || prod({M, B, kv_heads, C, d}) >= kMaxElems) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, (long long)kv_heads * d, kv_stride_m, kv_stride_row)) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(K, esz) || !aligned(V, esz) || !aligned(Kc, esz) || !aligned(Vc, esz) || !aligned(index, 4) || !aligned(count, 4) ||
      !aligned(len, 4) || !aligned(start, 4) || !aligned(pos, 4) || !aligned(weight, 4))
    return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  const bool wide = d * esz % 16 == 0 && kv_stride_m * esz % 16 == 0 && kv_stride_row * esz % 16 == 0 && aligned(K, 16) && aligned(V, 16) &&
                    aligned(Kc, 16) && aligned(Vc, 16);
  const size_t unit = wide ? 16 : esz;
  AppendArgs a = {K, V, index, count, len, start, Kc, Vc, pos, weight, M, B, T, n, C, kv_heads, (int)(d * esz / unit),
                  (long)(kv_stride_m * esz / unit), (long)(kv_stride_row * esz / unit)};
  const long long per_row = (long long)kv_heads * a.units;
  if (per_row > INT_MAX / 2) return NF_EUNSUPPORTED;
  const int rows = (int)std::max<long long>(1, std::min<long long>(n, 1024 / per_row));       // about 4 pieces per thread and tensor
  const int per_seq = (n + rows - 1) / rows;
  const long long blocks = prod({M, B, per_seq});
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
#define NF_APPEND(U) nf_launch((cache_append_kernel<U>), dim3((unsigned)blocks), dim3(256), 0, s, a, rows, per_seq)
  if (wide) NF_APPEND(uint4); else if (esz == 4) NF_APPEND(uint32_t); else NF_APPEND(uint16_t);
#undef NF_APPEND
  return launched();
}

nf_status netfuse_cache_weigh(const void* Q, const float* lse, const int* index, const int* count, const void* Kc, const int* pos,
                              const int* len, const int* start, const float* slope, const float* weight, float* weight_out, int M,
                              int B, int T, int n, int C, int heads, int kv_heads, int d, long q_stride_m, long q_stride_row,
                              float scale, float cap, nf_dtype dt, void* stream) {
  if (!Q || !lse || !Kc || !len || !weight || !weight_out) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || n <= 0 || C <= 0 || C > kMostEntries || !heads_ok(heads, kv_heads, d) || !is_dtype(dt) || !score_ok(scale, cap)) return NF_EINVAL;
  if (!index && n != T) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({B, n}) > INT_MAX / 2 || prod({M, B, T, heads}) >= kMaxElems || prod({M, B, kv_heads, C, d}) >= kMaxElems)
    return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, (long long)heads * d, q_stride_m, q_stride_row)) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Q, esz) || !aligned(Kc, esz) || !aligned(lse, 4) || !aligned(index, 4) || !aligned(count, 4) || !aligned(pos, 4) ||
      !aligned(len, 4) || !aligned(start, 4) || !aligned(slope, 4) || !aligned(weight, 4) || !aligned(weight_out, 4))
    return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  WeighArgs a = {Q, lse, index, count, Kc, pos, len, start, slope, weight, weight_out, M, B, T, n, C, heads, kv_heads, d,
                 q_stride_m, q_stride_row, scale, cap, cap != 0.f ? 1.f / cap : 0.f};
  if (ratio_ok(scale, cap, dt) && pieces_sizes(n, heads, kv_heads, d, dt) && pieces_strides(q_stride_m, q_stride_row, dt) && aligned(Q, 16) && aligned(Kc, 16))
    return launch_weigh_tiles(a, dt, (hipStream_t)stream);
  const int per_head = (int)((C + 255LL) / 256);
  const long long blocks = prod({M, B, kv_heads, per_head});
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  if (dt == NF_F32) nf_launch((weigh_rows_kernel<float>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head);
  else nf_launch((weigh_rows_kernel<bf16_t>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head);
  return launched();
}

long long netfuse_cache_evict_workspace(int M, int B, int C, int kv_heads, int budget) {
  if (M <= 0 || B <= 0 || C <= 0 || C > kMostEntries || kv_heads <= 0 || budget <= 0 || budget > C) return -1;
  const long long bytes = prod({M, B, kv_heads, 4, 1 + 2LL * std::min(budget, C - budget)});
  return bytes >= kMaxElems ? -1 : bytes;
}

nf_status netfuse_cache_evict(void* Kc, void* Vc, const int* pos, const float* weight, const int* len, const int* start, int* pos_out,
                              float* weight_out, void* workspace, long long workspace_bytes, int M, int B, int C, int kv_heads,
                              int d, int budget, int recent, nf_dtype dt, void* stream) {
  if (!Kc || !Vc || !weight || !len || !weight_out || !workspace) return NF_EINVAL;
  if (M <= 0 || B <= 0 || C <= 0 || C > kMostEntries || kv_heads <= 0 || d <= 0 || budget <= 0 || budget > C || recent < 0 || !is_dtype(dt)) return NF_EINVAL;
  if ((pos == nullptr) != (pos_out == nullptr) || (recent > 0 && !pos)) return NF_EINVAL;
  if (prod({M, B, kv_heads, C, d}) >= kMaxElems) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Kc, esz) || !aligned(Vc, esz) || !aligned(pos, 4) || !aligned(weight, 4) || !aligned(len, 4) || !aligned(start, 4) ||
      !aligned(pos_out, 4) || !aligned(weight_out, 4) || !aligned(workspace, 16))
    return NF_EINVAL;
  const long long need = netfuse_cache_evict_workspace(M, B, C, kv_heads, budget);
  if (need < 0 || workspace_bytes < need) return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  const bool wide = d * esz % 16 == 0 && aligned(Kc, 16) && aligned(Vc, 16);
  EvictArgs a = {Kc, Vc, pos, weight, len, start, pos_out, weight_out, (int*)workspace, M, B, C, kv_heads,
                 (int)(d * esz / (wide ? 16 : esz)), budget, recent, std::min(budget, C - budget)};
  const long long heads = prod({M, B, kv_heads});
  const int rows = std::max(1, 256 / a.units);                             // a piece of each tensor per thread
  const int per_head = std::max(1, (a.most + rows - 1) / rows);
  const long long blocks = prod({heads, per_head});
  const bool moves = C <= 1024 && wide && (long long)a.most * a.units <= 4096;
  if (!grid_fits(heads, C <= 4096 ? 256 : 1024) || (!moves && !grid_fits(blocks, 256))) return NF_EUNSUPPORTED;
  hipStream_t s = (hipStream_t)stream;
  // Small heads: the workgroup that picks the entries moves them too, as long as a head's rows are a few loads per thread (192 heads of 1024 entries cut to 896: 13.6 us by two
  // kernels, 12.8 by one).  Up to 32768 entries a head's weights stay in registers, of as few threads and as few to a thread as hold them (us, whole evictions: 128 heads of
  // 32768 147, by the kernel that reads them again for each digit 192; 128 / 768 heads of 6000, 8 or 32 to a thread 59 / 103 and 70 / 145; of 4096, 256 or 1024 threads
  // 53 / 73 and 48 / 76, of 2048 33 / 41 and 30 / 45).
  if (moves) return select_held<256, 4, true, uint4>(a, heads, s);
  nf_status st;
  if (C <= 1024) st = select_held<256, 4>(a, heads, s);
  else if (C <= 4096) st = select_held<256, 16>(a, heads, s);
  else if (C <= 8192) st = select_held<1024, 8>(a, heads, s);
  else if (C <= 32768) st = select_held<1024, 32>(a, heads, s);
  else {
    nf_launch(evict_select_kernel, dim3((unsigned)heads), dim3(1024), 0, s, a);
    st = launched();
  }
  if (st != NF_OK) return st;                              // without its lists nothing moves
  if (a.most > 0) {
#define NF_MOVE(U) nf_launch((evict_move_kernel<U>), dim3((unsigned)blocks), dim3(256), 0, s, a, rows, per_head)
    if (wide) NF_MOVE(uint4); else if (esz == 4) NF_MOVE(uint32_t); else NF_MOVE(uint16_t);
#undef NF_MOVE
  }
  return launched();
}

}  // extern "C"
