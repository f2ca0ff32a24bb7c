// Merged decoders: log probabilities of given tokens, the entropy of each row and its most likely tokens, in one pass over the logits.
//
//   x_j = f(scale * logit_j), j < V_m;   log p_t = x_t - top - log S,  S = sum exp(x_j - top);   entropy = log S - sum (x_j - top) exp(x_j - top) / S
//
// Both terms of the entropy are positive, and top + log S is never formed, so nothing is lost to large logits.  f grows with its argument and scale is positive, so the order of
// the logits is that of the probabilities, and it is taken from the logits as they are stored: no two that differ become equal.
//
// A wavefront takes a chunk of a row, each lane 16 bytes at a time of it, and keeps all of them in registers.  The chunks of a row and the join of their results follow from V
// alone, so a row's bits do not depend on what is merged with it.  Bound by the logits' bytes.
#pragma once
#include "decoder.h"
#include "decoder_tiles.h"

namespace nf {

constexpr int kMostAlternatives = 32;

struct LogprobArgs {
  const void* logits; const int* token; const int* vocab; const int* nodes;
  float* logp; float* entropy; int* top; float* top_logp; float* ws;
  int M, B, T, V, n, k, chunks;
  long stride_m, stride_row;
  float scale, cap, inv_cap;
};

// A logit in the order of its value, lower ones first, -0 as 0; 0 for what is no alternative: -infinity and NaN.
__device__ __forceinline__ uint32_t logit_order(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return v > -INFINITY ? (u & 0x80000000u ? ~u : u | 0x80000000u) : 0u;
}
__device__ __forceinline__ float logit_of(uint32_t order) { return order == 0u ? -INFINITY : __uint_as_float(order & 0x80000000u ? order & 0x7fffffffu : ~order); }

__device__ __forceinline__ float logit_value(float v, const LogprobArgs& a) {
  v *= a.scale;
  return a.cap != 0.f ? a.cap * tanhf(v * a.inv_cap) : v;
}

struct LogprobShape { static constexpr int kChunk = 4096, kPer = kChunk / kWave; };    // logits of a wavefront, of a lane

// What a chunk leaves in the workspace: its largest logit, the two sums at it (of 1 and of x - top), then k pairs (order, token), the most likely first.
constexpr int logprob_words(int k) { return 4 + 2 * k; }

// The better of two alternatives over the wavefront: the larger order, then the lower token.
__device__ __forceinline__ uint64_t wave_best(uint64_t v) {
#pragma unroll
  for (int o = 1; o < kWave; o *= 2) {
    const uint32_t x = __shfl_xor((uint32_t)v, o, kWave), y = __shfl_xor((uint32_t)(v >> 32), o, kWave);
    const uint64_t w = (uint64_t)y << 32 | x;
    v = w > v ? w : v;
  }
  return v;
}
__device__ __forceinline__ uint64_t alternative(uint32_t order, int token) { return (uint64_t)order << 32 | (uint32_t)~token; }

template <typename T>
__global__ __launch_bounds__(256) void logprob_chunks_kernel(LogprobArgs a) {
  constexpr int E = LogprobShape::kPer, P = 16 / (int)sizeof(T), N = E / P;      // logits per lane, per 16 bytes, loads
  const int lane = threadIdx.x % kWave;
  const long wid = (long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const long row = wid / a.chunks;
  if (row >= (long)a.M * a.B * a.T) return;                // uniform per wavefront, as the next ones
  const int chunk = (int)(wid % a.chunks), t = (int)(row % a.T);
  const long mb = row / a.T, m = mb / a.B;
  const int V = a.vocab ? clamp_len(a.vocab[m], a.V) : a.V;
  const int base = chunk * LogprobShape::kChunk, left = V - base;
  if (left <= 0 || (a.nodes && t >= a.nodes[mb])) return;
  const T* p = (const T*)a.logits + m * a.stride_m + (row - m * a.B * a.T) * a.stride_row + base;
  float v[E];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int j = (i * kWave + lane) * P;
#pragma unroll
    for (int e = 0; e < P; ++e) v[i * P + e] = j + e < left ? load_f32(p + j + e) : -INFINITY;
  }
  float top = -INFINITY;
#pragma unroll
  for (int e = 0; e < E; ++e) top = fmaxf(top, v[e]);
  top = wave_max(top);
  const float most = logit_value(top, a);
  float sum = 0.f, first = 0.f;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    const int j = (e / P * kWave + lane) * P + e % P;
    const float x = logit_value(v[e], a) - most, w = j < left && v[e] != -INFINITY ? expf(x) : 0.f;
    sum += w;
    first += w != 0.f ? x * w : 0.f;
  }
  sum = wave_sum(sum);
  first = wave_sum(first);
  float* out = a.ws + (row * a.chunks + chunk) * logprob_words(a.k);
  if (lane == 0) *reinterpret_cast<float2*>(out) = make_float2(top, sum), out[2] = first;
  uint64_t last = ~0ull;
  for (int r = 0; r < a.k; ++r) {
    uint64_t best = 0;
#pragma unroll
    for (int e = 0; e < E; ++e) {
      const int j = base + (e / P * kWave + lane) * P + e % P;
      const uint64_t x = alternative(logit_order(v[e]), j);
      best = x < last && x > best ? x : best;
    }
    last = wave_best(best);
    if (lane == 0) *reinterpret_cast<uint2*>(out + 4 + 2 * r) = make_uint2((uint32_t)(last >> 32), ~(uint32_t)last);
  }
}

// A row's chunks: one wavefront.
template <typename T>
__global__ __launch_bounds__(64) void logprob_join_kernel(LogprobArgs a) {
  const int lane = threadIdx.x;
  const long row = blockIdx.x;
  const int t = (int)(row % a.T);
  const long mb = row / a.T, m = mb / a.B;
  const int V = a.nodes && t >= a.nodes[mb] ? 0 : a.vocab ? clamp_len(a.vocab[m], a.V) : a.V;
  const int chunks = (V + LogprobShape::kChunk - 1) / LogprobShape::kChunk, words = logprob_words(a.k);
  const float* ws = a.ws + row * a.chunks * words;
  float top = -INFINITY;
  for (int c = lane; c < chunks; c += kWave) top = fmaxf(top, ws[(long)c * words]);
  top = wave_max(top);
  const float most = logit_value(top, a);
  float sum = 0.f, first = 0.f;
  for (int c = lane; c < chunks; c += kWave) {
    const float* w = ws + (long)c * words;
    const float x = logit_value(w[0], a) - most, f = w[0] != -INFINITY ? expf(x) : 0.f;
    if (w[1] != 0.f) {                                     // a chunk of -infinity alone adds nothing
      sum = fmaf(w[1], f, sum);
      first += f != 0.f ? f * fmaf(x, w[1], w[2]) : 0.f;
    }
  }
  sum = wave_sum(sum);
  first = wave_sum(first);
  const bool none = sum == 0.f;
  const float log_sum = none ? 0.f : logf(sum);
  if (lane == 0) a.entropy[row] = none ? 0.f : log_sum - first / sum;
  const T* p = (const T*)a.logits + m * a.stride_m + (row - m * a.B * a.T) * a.stride_row;
  for (int i = lane; i < a.n; i += kWave) {
    const int j = a.token[row * a.n + i];
    float x = -INFINITY;
    if (!none && j >= 0 && j < V) {
      const float v = load_f32(p + j);
      x = v == -INFINITY ? v : logit_value(v, a) - most - log_sum;
    }
    a.logp[row * a.n + i] = x;
  }
  if (a.k == 0) return;
  // the best of the chunks' first ones, k times: lane c % 64 keeps how far chunk c is used up (at most 32 of 2^31 / 4096 chunks: read again each time)
  uint64_t last = ~0ull;
  for (int r = 0; r < a.k; ++r) {
    uint64_t best = 0;
    for (int c = lane; c < chunks; c += kWave)
      for (int i = 0; i < a.k; ++i) {
        const uint2 w = *reinterpret_cast<const uint2*>(ws + (long)c * words + 4 + 2 * i);
        const uint64_t x = (uint64_t)w.x << 32 | ~w.y;
        if (x < last) {
          best = x > best ? x : best;
          break;
        }
      }
    last = wave_best(best);
    const uint32_t order = (uint32_t)(last >> 32);
    if (lane == 0) {
      a.top[row * a.k + r] = order ? (int)~(uint32_t)last : -1;
      a.top_logp[row * a.k + r] = order && !none ? logit_value(logit_of(order), a) - most - log_sum : -INFINITY;
    }
  }
}

}  // namespace nf
