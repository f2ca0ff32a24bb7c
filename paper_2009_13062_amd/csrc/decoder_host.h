// Host-side checks that the decoders' entry points share.
#pragma once
#include <math.h>

#include <cmath>

#include "decoder.h"
#include "nf_host.h"

namespace nf {

inline bool score_ok(float scale, float cap) {
  return std::isfinite(scale) && (cap == 0.f || (cap >= 1e-30f && cap <= 1e30f));
}

// Rows of M models, `rows` of `width` elements each: a row's heads side by side, models one behind the other.
inline bool rows_ok(int M, long long rows, long long width, long stride_m, long stride_row) {
  if (width > INT_MAX || stride_row < width || stride_m < 0) return false;
  if (prod({rows, stride_row}) >= kMaxElems || prod({M, stride_m}) >= kMaxElems) return false;
  return M == 1 || stride_m >= (rows - 1) * stride_row + width;
}

constexpr int kMostEntries = 1 << 30;                      // slot numbers and what is added to them stay in an int

inline bool heads_ok(int heads, int kv_heads, int d) { return heads > 0 && kv_heads > 0 && d > 0 && heads % kv_heads == 0; }

// What the kernels on the matrix pipe take: rows in 16-byte pieces, row numbers in an int.
inline bool pieces_sizes(int N, int heads, int kv_heads, int d, nf_dtype dt) {
  return d % (dt == NF_F32 ? 4 : 8) == 0 && d <= 256 && (long long)N * (heads / kv_heads) <= INT_MAX / 2;
}
inline bool pieces_strides(long stride_m, long stride_row, nf_dtype dt) {
  const int n = dt == NF_F32 ? 4 : 8;
  return stride_m % n == 0 && stride_row % n == 0;
}
// The bfloat16 kernels on the matrix pipe take scale / cap in one factor, which has to be a normal number.  (Two factors there cost 4 % of the weights of a capped token;
// the general kernels have them.)
inline bool ratio_ok(float scale, float cap, nf_dtype dt) {
  const double r = cap != 0.f ? fabs((double)scale) / cap : 0.0;
  return dt == NF_F32 || r == 0.0 || (r > 1e-37 && r < 1e38);
}
inline bool pieces_ok(const DecArgs& a, nf_dtype dt) {
  // 64 rows of keys within 31 bits of bytes: a tile's offsets
  return ratio_ok(a.scale, a.cap, dt) && a.kv_stride_row < (1L << 31) / 64 / (dt == NF_F32 ? 4 : 2) && pieces_sizes(a.N, a.heads, a.kv, a.d, dt) && pieces_strides(a.q_stride_m, a.q_stride_row, dt) && pieces_strides(a.kv_stride_m, a.kv_stride_row, dt) &&
         aligned(a.Q, 16) && aligned(a.K, 16) && aligned(a.V, 16) && aligned(a.Kc, 16) && aligned(a.Vc, 16) && aligned(a.O, 16);
}

}  // namespace nf
