// What the kernels of merged decoders share: their operands, scores and masks.
//
// Score of query i and key j:  f(scale q_i . k_j) - slope |position_i - position_j|,  f(x) = cap tanh(x / cap) or x.  A key that a row does not
// see is left out by a select on its weight (and on its values where these could be infinite or NaN), never by adding to its score.
#pragma once
#include <type_traits>

#include "nf_common.h"

namespace nf {

constexpr float kLowestScore = -3.402823466e38f;          // running maxima start here: finite, so that a difference of two is no NaN

struct DecArgs {
  const void* Q; const void* K; const void* V;          // new rows: [M][B * N] of heads * d and kv * d, strides below
  const void* Kc; const void* Vc;                       // cache [M][B][kv][C][d]; null for prompts
  const float* slope;                                   // [M][heads] or null
  const int* len; const int* prefix; const int* doc;    // [M][B], [M][B], [M][B][N], each or null
  const int* start; const int* parent; const int* nodes; const int* pos;
  void* O; float* lse; float* ws;
  int M, B, N, C, heads, kv, d, causal;
  long q_stride_m, q_stride_row, kv_stride_m, kv_stride_row;
  float scale, cap, inv_cap;                            // inv_cap = 1 / cap, 0 without a cap
};

struct WeighArgs {
  const void* Q; const float* lse; const int* index; const int* count; const void* Kc; const int* pos; const int* len; const int* start;
  const float* slope; const float* weight; float* out;
  int M, B, T, n, C, heads, kv, d;
  long q_stride_m, q_stride_row;
  float scale, cap, inv_cap;
};

// Loads of whole tiles go through a buffer resource over the rows from the tile's first key on: a key or feature that is not there gets an
// offset outside it and comes back as 0.  (A load under a condition is a branch, and the compiler then waits for one load at a time.)  Offsets are 32 bits
// of bytes: the host takes other kernels where 64 rows do not fit.
typedef uint32_t dec_u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t dec_u32x2_t __attribute__((ext_vector_type(2)));
constexpr unsigned kDecOob = 0x80000000u;
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const void* first) { return __builtin_amdgcn_make_buffer_rsrc((void*)first, 0, (int)kDecOob, 0x00020000); }
template <int AUX = 0> __device__ __forceinline__ uint4 rows_load16(__amdgpu_buffer_rsrc_t r, unsigned off) {
  const dec_u32x4_t v = __builtin_amdgcn_raw_buffer_load_b128(r, (int)off, 0, AUX);
  return make_uint4(v.x, v.y, v.z, v.w);
}

__device__ __forceinline__ int clamp_len(int v, int top) { return min(max(v, 0), top); }

// f of the score, the exact way: tanhf in natural units.
__device__ __forceinline__ float capped(float x, const DecArgs& a) { return a.cap != 0.f ? a.cap * tanhf(x * a.inv_cap) : x; }

// The nodes that node t of a tree sees, itself among them, a bit each.  Ancestors have lower numbers, so the walk ends after at most t steps
// whatever `parent` holds, and the distance from t to node u of its path is the number of path nodes above u: popcount(path >> u) - 1.
__device__ __forceinline__ uint64_t tree_path(const int* parent, int t) {
  if (!parent) return (2ull << t) - 1;
  uint64_t path = 1ull << t;
  for (int u = t;;) {
    const int p = parent[u];
    if (p < 0 || p >= u) return path;
    path |= 1ull << p;
    u = p;
  }
}

}  // namespace nf
