// C ABI of what surrounds the decoders' attention: heads normed and rotated, the cache of 4 bits and the attention over it, log probabilities of tokens.  Argument validation
// on the host before any HIP call, kernel selection by sizes, type and alignment.
#include <hip/hip_runtime.h>
#include <math.h>

#include <algorithm>

#include "cache_fp4_kernels.h"
#include "decoder.h"
#include "decoder_fp4_generic.h"
#include "decoder_host.h"
#include "decoder_launch.h"
#include "logprob_kernels.h"
#include "nf_host.h"
#include "nf_launch.h"
#include "rotate_kernels.h"

using namespace nf;

namespace {

inline nf_status launched() { return hipGetLastError() == hipSuccess ? NF_OK : NF_ELAUNCH; }
constexpr long long kSecondCaches = 32LL << 20, kLastCache = 256LL << 20;                // bytes that the second ones hold together, and the last one
inline bool whole_pieces(long stride_m, long stride_row, size_t esz) { return stride_m * (long)esz % 16 == 0 && stride_row * (long)esz % 16 == 0; }

template <typename T>
nf_status launch_rotate_rows(const RotateArgs& a, hipStream_t s) {
  const long long blocks = (prod({a.M, a.B, a.S, a.heads + (long long)a.kv}) + 3) / 4;
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  nf_launch((rotate_rows_kernel<T>), dim3((unsigned)blocks), dim3(256), 0, s, a);
  return launched();
}

template <typename T>
nf_status launch_rotate(const RotateArgs& a, hipStream_t s) {
  constexpr int P = kPieceFeatures;
  const int units = (a.d + 2 * P - 1) / (2 * P);
  int lph = 1;
  while (lph < units) lph *= 2;
  const int at_once = kWave / lph, steps = (a.heads + at_once - 1) / at_once + (a.kv + at_once - 1) / at_once;
  // a token's steps are shared out where there are few tokens (32 heads over 8 of 128: 8 tokens 5.4 us, by one wavefront each 7.3)
  const long long tokens = prod({a.M, a.B, a.S});
  const int most = (int)std::max<long long>(1, std::min<long long>(steps, 2048 / tokens)), per_wave = (steps + most - 1) / most, parts = (steps + per_wave - 1) / per_wave;
  const long long blocks = (prod({tokens, parts}) + 3) / 4;
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  const bool past = prod({tokens, a.heads + (long long)a.kv, a.d, (long long)sizeof(T)}) > kLastCache;
#define NF_ROTATE(LPH)                                                                                                        \
  if (past) nf_launch((rotate_pieces_kernel<T, LPH, true>), dim3((unsigned)blocks), dim3(256), 0, s, a, parts, per_wave);     \
  else nf_launch((rotate_pieces_kernel<T, LPH, false>), dim3((unsigned)blocks), dim3(256), 0, s, a, parts, per_wave)
  switch (lph) {
    case 1: NF_ROTATE(1); break;
    case 2: NF_ROTATE(2); break;
    case 4: NF_ROTATE(4); break;
    case 8: NF_ROTATE(8); break;
    case 16: NF_ROTATE(16); break;
    default: NF_ROTATE(32); break;
  }
#undef NF_ROTATE
  return launched();
}

nf_status launch_fp4_rows(const DecArgs& a, nf_dtype dt, hipStream_t s) {
  const long long blocks = (prod({a.M, a.B, a.heads, a.N}) + 3) / 4;
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
#define NF_ROWS(T, DPL) nf_launch((decoder_fp4_rows_kernel<T, DPL>), dim3((unsigned)blocks), dim3(256), 0, s, a)
  if (dt == NF_F32) {
    if (a.d <= 64) NF_ROWS(float, 1); else if (a.d <= 128) NF_ROWS(float, 2); else NF_ROWS(float, 4);
  } else {
    if (a.d <= 64) NF_ROWS(bf16_t, 1); else if (a.d <= 128) NF_ROWS(bf16_t, 2); else NF_ROWS(bf16_t, 4);
  }
#undef NF_ROWS
  return launched();
}

// Codes come in rows of 16 bytes, scales in rows of 2, 4 or (over 128 features) single bytes.
bool cache_fp4_aligned(const void* Kc, const void* Ks, const void* Vc, const void* Vs, int d) {
  const size_t n = d <= 64 ? 2 : d <= 128 ? 4 : 1;
  return aligned(Kc, 16) && aligned(Vc, 16) && aligned(Ks, n) && aligned(Vs, n);
}

int logprob_chunks(int V, int chunk) { return (int)(((long long)V + chunk - 1) / chunk); }

}  // namespace

extern "C" {

nf_status netfuse_rotate_heads(const void* Q, const void* K, const float* gamma_q, const float* gamma_k, const float* freq, const int* pos,
                               const int* start, const int* len, const int* sections, void* Qo, void* Ko, int M, int B, int S, int heads,
                               int kv_heads, int d, int rot, int axes, long q_stride_m, long q_stride_row, long k_stride_m,
                               long k_stride_row, long qo_stride_m, long qo_stride_row, long ko_stride_m, long ko_stride_row, float eps,
                               int interleaved, nf_dtype dt, void* stream) {
  if (!Q || !Qo || (K == nullptr) != (Ko == nullptr) || (K == nullptr) != (kv_heads == 0)) return NF_EINVAL;
  if (M <= 0 || B <= 0 || S <= 0 || heads <= 0 || kv_heads < 0 || d <= 0 || !is_dtype(dt)) return NF_EINVAL;
  if (rot < 0 || rot > d || rot % 2 || (rot > 0 && !freq) || axes < 1 || axes > 4 || (axes > 1 && (!sections || !pos))) return NF_EINVAL;
  if (!std::isfinite(eps) || eps < 0.f) return NF_EINVAL;
  if (prod({B, S}) > INT_MAX / 2 || prod({M, B, S, heads, d}) >= kMaxElems || (long long)heads + kv_heads > INT_MAX) return NF_EINVAL;
  const long long N = (long long)B * S;
  if (!rows_ok(M, N, (long long)heads * d, q_stride_m, q_stride_row) || !rows_ok(M, N, (long long)heads * d, qo_stride_m, qo_stride_row)) return NF_EINVAL;
  if (K && (!rows_ok(M, N, (long long)kv_heads * d, k_stride_m, k_stride_row) || !rows_ok(M, N, (long long)kv_heads * d, ko_stride_m, ko_stride_row))) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Q, esz) || !aligned(K, esz) || !aligned(Qo, esz) || !aligned(Ko, esz) || !aligned(gamma_q, 4) || !aligned(gamma_k, 4) || !aligned(freq, 4) ||
      !aligned(pos, 4) || !aligned(start, 4) || !aligned(len, 4))
    return NF_EINVAL;
  if ((Q == Qo && (q_stride_m != qo_stride_m || q_stride_row != qo_stride_row)) || (K && K == Ko && (k_stride_m != ko_stride_m || k_stride_row != ko_stride_row))) return NF_EINVAL;
  RotateArgs a = {};
  a.Q = Q; a.K = K; a.gamma_q = gamma_q; a.gamma_k = gamma_k; a.freq = freq; a.pos = pos; a.start = start; a.len = len; a.Qo = Qo; a.Ko = Ko;
  a.M = M; a.B = B; a.S = S; a.heads = heads; a.kv = kv_heads; a.d = d; a.rot = rot; a.axes = axes; a.interleaved = interleaved != 0;
  long long pairs = 0;
  for (int x = 0; x < 3; ++x) a.axis_end[x] = INT_MAX;
  for (int x = 0; x < axes && sections; ++x) {
    if (sections[x] < 0) return NF_EINVAL;
    pairs += sections[x];
    if (x + 1 < axes) a.axis_end[x] = (int)std::min<long long>(pairs, INT_MAX);
  }
  if (sections && pairs != rot / 2) return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  a.q_stride_m = q_stride_m; a.q_stride_row = q_stride_row; a.k_stride_m = k_stride_m; a.k_stride_row = k_stride_row;
  a.qo_stride_m = qo_stride_m; a.qo_stride_row = qo_stride_row; a.ko_stride_m = ko_stride_m; a.ko_stride_row = ko_stride_row;
  a.eps = eps;
  // rows, strides and pointers of whole pieces
  const int P = kPieceFeatures;
  auto whole = [&](const void* p, long stride_m, long stride_row) { return !p || (stride_m % P == 0 && stride_row % P == 0 && aligned(p, P * esz)); };
  const bool pieces = d % P == 0 && rot % (2 * P) == 0 && whole(Q, q_stride_m, q_stride_row) && whole(K, k_stride_m, k_stride_row) && whole(Qo, qo_stride_m, qo_stride_row) &&
                      whole(Ko, ko_stride_m, ko_stride_row);
  hipStream_t s = (hipStream_t)stream;
  if (dt == NF_F32) return pieces ? launch_rotate<float>(a, s) : launch_rotate_rows<float>(a, s);
  return pieces ? launch_rotate<bf16_t>(a, s) : launch_rotate_rows<bf16_t>(a, s);
}

nf_status netfuse_cache_append_fp4(const void* K, const void* V, const int* index, const int* count, const int* len, const int* start, void* Kc,
                                   void* Ks, void* Vc, void* Vs, int* pos, float* weight, int M, int B, int T, int n, int C, int kv_heads,
                                   int d, long kv_stride_m, long kv_stride_row, nf_dtype dt, void* stream) {
  if (!K || !V || !Kc || !Ks || !Vc || !Vs || !len) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || n <= 0 || C <= 0 || C > kMostEntries || kv_heads <= 0 || d <= 0 || !is_dtype(dt)) return NF_EINVAL;
  if (!index && n != T) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({B, n}) > INT_MAX / 2 || prod({M, B, kv_heads, C, d}) >= kMaxElems) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, (long long)kv_heads * d, kv_stride_m, kv_stride_row)) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(K, esz) || !aligned(V, esz) || !cache_fp4_aligned(Kc, Ks, Vc, Vs, d) || !aligned(index, 4) || !aligned(count, 4) ||
      !aligned(len, 4) || !aligned(start, 4) || !aligned(pos, 4) || !aligned(weight, 4))
    return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  const AppendFp4Args a = {K, V, index, count, len, start, (uint8_t*)Kc, (uint8_t*)Ks, (uint8_t*)Vc, (uint8_t*)Vs, pos, weight, M, B, T, n, C, kv_heads, d, kv_stride_m, kv_stride_row};
  const int groups = fp4_groups(d), rows = 256 / (4 * groups), per_head = (int)((n + (long long)rows - 1) / rows);
  const long long blocks = prod({M, B, kv_heads, per_head});
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  const bool wide = d * esz % 16 == 0 && whole_pieces(kv_stride_m, kv_stride_row, esz) && aligned(K, 16) && aligned(V, 16);
  hipStream_t s = (hipStream_t)stream;
#define NF_APPEND_G(T, WIDE, G) nf_launch((cache_append_fp4_kernel<T, WIDE, G>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head)
#define NF_APPEND(T, WIDE) if (groups == 4) NF_APPEND_G(T, WIDE, 4); else if (groups == 2) NF_APPEND_G(T, WIDE, 2); else NF_APPEND_G(T, WIDE, 0)
  if (dt == NF_F32) { if (wide) { NF_APPEND(float, true); } else { NF_APPEND(float, false); } }
  else { if (wide) { NF_APPEND(bf16_t, true); } else { NF_APPEND(bf16_t, false); } }
#undef NF_APPEND
#undef NF_APPEND_G
  return launched();
}

nf_status netfuse_cache_read_fp4(const void* Kc, const void* Ks, const void* Vc, const void* Vs, const int* first, const int* count, void* K, void* V,
                                 int M, int B, int n, int C, int kv_heads, int d, nf_dtype dt, void* stream) {
  if (!Kc || !Ks || !K || (Vc == nullptr) != (V == nullptr) || (Vs == nullptr) != (V == nullptr)) return NF_EINVAL;
  if (M <= 0 || B <= 0 || n <= 0 || C <= 0 || C > kMostEntries || n > kMostEntries || kv_heads <= 0 || d <= 0 || !is_dtype(dt)) return NF_EINVAL;
  if (prod({M, B, kv_heads, C, d}) >= kMaxElems || prod({M, B, kv_heads, n, d}) >= kMaxElems) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!cache_fp4_aligned(Kc, Ks, Vc, Vs, d) || !aligned(K, esz) || !aligned(V, esz) || !aligned(first, 4) || !aligned(count, 4)) return NF_EINVAL;
  if (d > 256) return NF_EUNSUPPORTED;
  const ReadFp4Args a = {(const uint8_t*)Kc, (const uint8_t*)Ks, (const uint8_t*)Vc, (const uint8_t*)Vs, first, count, K, V, M, B, n, C, kv_heads, d};
  const int features = 16 / (int)esz, rows = 256 / ((d + features - 1) / features), per_head = (int)((n + (long long)rows - 1) / rows);
  const long long blocks = prod({M, B, kv_heads, per_head});
  if (!grid_fits(blocks, 256)) return NF_EUNSUPPORTED;
  const bool wide = d % features == 0 && aligned(K, 16) && aligned(V, 16);
  hipStream_t s = (hipStream_t)stream;
  const bool past = prod({M, B, kv_heads, n, d, (long long)esz, V ? 2 : 1}) > kSecondCaches;
#define NF_READ(T, WIDE, PAST) nf_launch((cache_read_fp4_kernel<T, WIDE, PAST>), dim3((unsigned)blocks), dim3(256), 0, s, a, per_head)
  if (dt == NF_F32) { if (!wide) NF_READ(float, false, false); else if (past) NF_READ(float, true, true); else NF_READ(float, true, false); }
  else { if (!wide) NF_READ(bf16_t, false, false); else if (past) NF_READ(bf16_t, true, true); else NF_READ(bf16_t, true, false); }
#undef NF_READ
  return launched();
}

long long netfuse_attention_tree_fp4_workspace(int M, int B, int T, int C, int heads, int kv_heads, int d, nf_dtype dt) {
  if (M <= 0 || B <= 0 || T <= 0 || T > 64 || C <= 0 || C > kMostEntries || !heads_ok(heads, kv_heads, d) || d > 256 || !is_dtype(dt)) return -1;
  if (!pieces_sizes(T, heads, kv_heads, d, dt)) return 0;
  const int splits = (int)(((long long)C + kTreeFp4Chunk - 1) / kTreeFp4Chunk);
  if (splits == 1) return 0;                               // no cache is shared out
  const long long bytes = prod({M, B, heads, T, splits, 4LL * (tree_features(d) + 2)});
  return bytes >= kMaxElems ? -1 : bytes;
}

nf_status netfuse_attention_tree_fp4(const void* Q, const void* K, const void* V, const void* Kc, const void* Ks, const void* Vc, const void* Vs,
                                     const int* pos, const int* len, const int* start, const int* parent, const int* nodes, const float* slope,
                                     void* O, float* lse, void* workspace, long long workspace_bytes, int M, int B, int T, int C, int heads,
                                     int kv_heads, int d, long q_stride_m, long q_stride_row, long kv_stride_m, long kv_stride_row,
                                     float scale, float cap, nf_dtype dt, void* stream) {
  if (!Q || !K || !V || !Kc || !Ks || !Vc || !Vs || !len || !O) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || C <= 0 || C > kMostEntries || !heads_ok(heads, kv_heads, d)) return NF_EINVAL;
  if (!is_dtype(dt) || !score_ok(scale, cap)) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({M, B, T, heads, d}) >= kMaxElems || prod({M, B, kv_heads, C, d}) >= kMaxElems) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, (long long)heads * d, q_stride_m, q_stride_row) ||
      !rows_ok(M, (long long)B * T, (long long)kv_heads * d, kv_stride_m, kv_stride_row))
    return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(Q, esz) || !aligned(K, esz) || !aligned(V, esz) || !cache_fp4_aligned(Kc, Ks, Vc, Vs, d) || !aligned(O, esz) ||
      !aligned(pos, 4) || !aligned(len, 4) || !aligned(start, 4) || !aligned(parent, 4) || !aligned(nodes, 4) || !aligned(slope, 4) || !aligned(lse, 4) || !aligned(workspace, 16))
    return NF_EINVAL;
  if (T > 64 || d > 256) return NF_EUNSUPPORTED;
  const long long need = netfuse_attention_tree_fp4_workspace(M, B, T, C, heads, kv_heads, d, dt);
  if (need < 0) return NF_EUNSUPPORTED;
  if (need > 0 && (!workspace || workspace_bytes < need)) return NF_EINVAL;
  DecArgs a = {};
  a.Q = Q; a.K = K; a.V = V; a.Kc = Kc; a.Vc = Vc; a.Ks = (const uint8_t*)Ks; a.Vs = (const uint8_t*)Vs; a.slope = slope; a.len = len; a.start = start; a.parent = parent;
  a.nodes = nodes; a.pos = pos; a.O = O; a.lse = lse; a.ws = (float*)workspace;
  a.M = M; a.B = B; a.N = T; a.C = C; a.heads = heads; a.kv = kv_heads; a.d = d;
  a.q_stride_m = q_stride_m; a.q_stride_row = q_stride_row; a.kv_stride_m = kv_stride_m; a.kv_stride_row = kv_stride_row;
  a.scale = scale; a.cap = cap; a.inv_cap = cap != 0.f ? 1.f / cap : 0.f;
  if (pieces_ok(a, dt)) {
    const int chunk = kTreeFp4Chunk, splits = (int)(((long long)C + chunk - 1) / chunk), rows = T * (heads / kv_heads);
    if (splits > 1 && !grid_fits(tree_join_blocks(a, splits), 256)) return NF_EUNSUPPORTED;      // before the first of the two is enqueued
    const bool tiles = dt == NF_BF16 && rows > tree_fp4_streamed(d);
    const nf_status st = tiles ? launch_tree_fp4_tiles(a, chunk, splits, (hipStream_t)stream) : launch_tree_fp4_stream(a, chunk, splits, dt, (hipStream_t)stream);
    return st != NF_OK || splits == 1 ? st : launch_tree_join(a, chunk, splits, dt, (hipStream_t)stream);
  }
  return launch_fp4_rows(a, dt, (hipStream_t)stream);
}

long long netfuse_token_logprobs_workspace(int M, int B, int T, int V, int k) {
  if (M <= 0 || B <= 0 || T <= 0 || V <= 0 || V > kMostEntries || k < 0 || k > kMostAlternatives) return -1;
  const long long bytes = prod({M, B, T, logprob_chunks(V, logprob_chunk(4, V)), 4LL * kChunkWords + 8LL * k});        // a wavefront per chunk, of either type's
  return bytes >= kMaxElems ? -1 : bytes;
}

nf_status netfuse_token_logprobs(const void* logits, const int* token, const int* vocab, const int* nodes, float* logp, float* entropy, int* top,
                                 float* top_logp, void* workspace, long long workspace_bytes, int M, int B, int T, int V, int n, int k,
                                 long stride_m, long stride_row, float scale, float cap, nf_dtype dt, void* stream) {
  if (!logits || !entropy || !workspace) return NF_EINVAL;
  if (M <= 0 || B <= 0 || T <= 0 || V <= 0 || V > kMostEntries || n < 0 || k < 0 || !is_dtype(dt)) return NF_EINVAL;
  if ((n > 0 && (!token || !logp)) || (k > 0 && (!top || !top_logp))) return NF_EINVAL;
  if (!score_ok(scale, cap) || scale < 1e-30f || scale > 1e30f) return NF_EINVAL;
  if (prod({B, T}) > INT_MAX / 2 || prod({M, B, T, V}) >= kMaxElems || prod({M, B, T, n}) >= kMaxElems || prod({M, B, T}) > INT_MAX) return NF_EINVAL;
  if (!rows_ok(M, (long long)B * T, V, stride_m, stride_row)) return NF_EINVAL;
  const size_t esz = dt == NF_F32 ? 4 : 2;
  if (!aligned(logits, esz) || !aligned(token, 4) || !aligned(vocab, 4) || !aligned(nodes, 4) || !aligned(logp, 4) || !aligned(entropy, 4) || !aligned(top, 4) ||
      !aligned(top_logp, 4) || !aligned(workspace, 16))
    return NF_EINVAL;
  if (k > kMostAlternatives) return NF_EUNSUPPORTED;
  const long long need = netfuse_token_logprobs_workspace(M, B, T, V, k);
  if (need < 0 || workspace_bytes < need) return NF_EINVAL;
  const long long rows = prod({M, B, T});
  const int chunk = logprob_chunk(esz, V), chunks = logprob_chunks(V, chunk);
  // As many chunks to a wavefront as leave two wavefronts for each that the device holds: its alternatives then are few and soon have a high border (4084 rows of 50001 in float32, 20 alternatives,
  // chunks and join, us: a wavefront per chunk 174 + 13, 8 chunks 164 + 8, 16 168 + 8, 32 188 + 8).
  const int per_wave = (int)std::max<long long>(1, std::min<long long>(16, prod({rows, chunks}) / 8192)), groups = (chunks + per_wave - 1) / per_wave;
  const LogprobArgs a = {logits, token, vocab, nodes, logp, entropy, top, top_logp, (float*)workspace, M, B, T, V, n, k, chunks, groups,
                         stride_m, stride_row, scale, cap, cap != 0.f ? 1.f / cap : 0.f};
  const long long blocks = (prod({rows, groups}) + 3) / 4;
  if (!grid_fits(blocks, 256) || !grid_fits(rows, 64)) return NF_EUNSUPPORTED;          // before the first of the two is enqueued
  hipStream_t s = (hipStream_t)stream;
#define NF_CHUNKS(T, CHUNK)                                                                                                 \
  if (cap != 0.f) nf_launch((logprob_chunks_kernel<T, true, CHUNK>), dim3((unsigned)blocks), dim3(256), 0, s, a);           \
  else nf_launch((logprob_chunks_kernel<T, false, CHUNK>), dim3((unsigned)blocks), dim3(256), 0, s, a)
  if (dt == NF_F32) { NF_CHUNKS(float, 2048); } else if (chunk == 2048) { NF_CHUNKS(bf16_t, 2048); } else { NF_CHUNKS(bf16_t, 4096); }
#undef NF_CHUNKS
  const nf_status st = launched();
  if (st != NF_OK) return st;
  if (dt == NF_F32) nf_launch((logprob_join_kernel<float>), dim3((unsigned)rows), dim3(64), 0, s, a);
  else nf_launch((logprob_join_kernel<bf16_t>), dim3((unsigned)rows), dim3(64), 0, s, a);
  return launched();
}

}  // extern "C"
