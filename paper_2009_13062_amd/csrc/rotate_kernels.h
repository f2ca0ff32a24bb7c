// Merged decoders: queries and keys normed head by head and rotated by position, in one pass over their rows.
//
//   y = x / sqrt(mean x^2 + eps) * gamma;   pair i of the first `rot` features: (y_a, y_b) -> (y_a cos t - y_b sin t, y_a sin t + y_b cos t),  t = position * freq[i]
//
// pairs (i, i + rot / 2) or (2 i, 2 i + 1).  The angle is a product in 64 bits, taken in whole turns before it becomes a float32: an angle is
// off by 2^-51 of itself, a far position's bits are not lost to a float32.  Bound by the rows' bytes (16 prompts of up to 2039 tokens, 32 heads over 8 of 128, normed, three axes: 97 us, 5.1 TB/s where a copy
// reaches 4.94), a few tokens by latency (8 of them, 32 heads over 8 of 128, 5.4 us; 12 heads of 64 4.0).
#pragma once
#include "decoder.h"

namespace nf {

struct RotateArgs {
  const void* Q; const void* K; const float* gamma_q; const float* gamma_k; const float* freq; const int* pos; const int* start; const int* len;
  void* Qo; void* Ko;
  int M, B, S, heads, kv, d, rot, axes, interleaved;
  int axis_end[3];                                         // pairs of axes 0, 0 and 1, 0 to 2
  long q_stride_m, q_stride_row, k_stride_m, k_stride_row, qo_stride_m, qo_stride_row, ko_stride_m, ko_stride_row;
  float eps;
};

// Cosine and sine of 2 pi t, t in turns.  The nearest quarter is taken off in 64 bits; what is left, at most pi / 4, goes into the two Taylor series, whose first terms left
// out are below 2^-28 and 2^-25; both results are within 2^-22 of the exact ones.
__device__ __forceinline__ float2 cos_sin_turns(double t) {
  const double quarter = rint(4.0 * t);
  const float x = (float)(fma(quarter, -0.25, t) * 6.283185307179586);
  const float w = x * x;
  float s = fmaf(w, 2.7557319223985893e-06f, -1.9841269841269841e-04f);
  s = fmaf(s, w, 8.3333333333333332e-03f);
  s = fmaf(s, w, -1.6666666666666666e-01f);
  s = fmaf(s * w, x, x);
  float c = fmaf(w, 2.4801587301587302e-05f, -1.3888888888888889e-03f);
  c = fmaf(c, w, 4.1666666666666664e-02f);
  c = fmaf(c, w, -0.5f);
  c = fmaf(c, w, 1.0f);
  const int q = (int)((long long)quarter & 3);
  const float a = q & 1 ? s : c, b = q & 1 ? c : s;        // quarter turns: (c, s), (-s, c), (-c, -s), (s, -c)
  return make_float2(q == 1 || q == 2 ? -a : a, q >= 2 ? -b : b);
}

__device__ __forceinline__ float2 rotate_angle(const RotateArgs& a, long mb, int s, int pair) {
  const int axis = (pair >= a.axis_end[0]) + (pair >= a.axis_end[1]) + (pair >= a.axis_end[2]);
  const double p = a.pos ? (double)a.pos[(mb * a.S + s) * a.axes + axis] : (double)(a.start ? a.start[mb] : 0) + s;
  return cos_sin_turns(p * (double)a.freq[pair] * 0.15915494309189535);
}

// Sum over LPH neighbouring lanes, in all of them
template <int LPH> __device__ __forceinline__ float lanes_sum(float v) {
  constexpr int kHalfMirror = 0x141, kMirror = 0x140;      // lanes 7 - i of 8, 15 - i of 16: by then equal within the halves that they exchange
  if constexpr (LPH > 1) v += dpp<kQuadXor1>(v);
  if constexpr (LPH > 2) v += dpp<kQuadXor2>(v);
  if constexpr (LPH > 4) v += dpp<kHalfMirror>(v);
  if constexpr (LPH > 8) v += dpp<kMirror>(v);
  if constexpr (LPH > 16) v = across_rows(v, AddOp{});
  return v;
}

// Four neighbouring features of a row in one load: 16 bytes of float32, 8 of bfloat16.  (Eight of bfloat16 hold twice the registers: 16 prompts of up to 2039 tokens, 32 heads over 8 of 128, 106 us
// and 103; 32 of 512, 12 heads of 64, 26.5 and 22.6, both with results in the caches.  And 80 features of which 40 turn are no whole pieces of 16: one by one 525 us, so 81.)
template <typename T> struct Piece;
template <> struct Piece<float> {
  typedef uint4 words_t;
  typedef nf_u32x4_t store_t;
  __device__ static __forceinline__ void open(const uint4& w, float* x) { x[0] = __uint_as_float(w.x); x[1] = __uint_as_float(w.y); x[2] = __uint_as_float(w.z); x[3] = __uint_as_float(w.w); }
  __device__ static __forceinline__ uint4 close(const float* x) { return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])); }
};
template <> struct Piece<bf16_t> {
  typedef uint2 words_t;
  typedef uint32_t store_t __attribute__((ext_vector_type(2)));
  __device__ static __forceinline__ void open(const uint2& w, float* x) {
    x[0] = __uint_as_float(w.x << 16); x[1] = __uint_as_float(w.x & 0xffff0000u); x[2] = __uint_as_float(w.y << 16); x[3] = __uint_as_float(w.y & 0xffff0000u);
  }
  __device__ static __forceinline__ uint2 close(const float* x) { return make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3])); }
};
constexpr int kPieceFeatures = 4;

// A wavefront takes one token, or `per_wave` steps of it.  Its lanes work out the token's angles once, a pair each; then LPH lanes take a head, each two pieces, whose features turn with
// each other or within each (or, past `rot`, not at all), so 64 / LPH heads are read and written at a time and a lane keeps its angles and weights over all of them.
// PAST: results that the last cache does not hold go past them all (rows of the 16 prompts above 105 us, so 98).  Smaller ones would leave this call earlier too, but the attention that reads them next
// pays for more than that (rotation alone, then with the attention, us, through the caches / past them: 16 prompts of 1024, 32 heads over 8 of 128, 168 MB, 72 / 53, 269 / 275; 8 of them 30 / 30,
// 134 / 138; 64 of 512, 12 heads of 64, 101 MB, 40 / 38, 127 / 131; and above, 32 of 1024, 336 MB, 135 / 129, 530 / 532).
template <typename T, int LPH, bool PAST>
__global__ __launch_bounds__(256) void rotate_pieces_kernel(RotateArgs a, int parts, int per_wave) {
  using Pc = Piece<T>;
  typedef typename Pc::words_t words_t;
  constexpr int P = kPieceFeatures, kHeads = kWave / LPH, kAhead = 4;
  __shared__ float2 angle[4][128];
  const int lane = threadIdx.x % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const unsigned wid = blockIdx.x * 4 + wave, token = wid / parts;
  if (token >= (unsigned)(a.M * a.B) * (unsigned)a.S) return;                    // uniform per wavefront, as the next one
  const unsigned umb = token / a.S;
  const int s = (int)(token - umb * a.S), b = (int)(umb % a.B);
  const long mb = umb, m = umb / a.B;
  if (a.len && s >= a.len[mb]) return;
  const int q_steps = (a.heads + kHeads - 1) / kHeads, steps = q_steps + (a.kv + kHeads - 1) / kHeads;
  const int step0 = (int)(wid - token * parts) * per_wave, step1 = min(steps, step0 + per_wave);
  const int u = lane % LPH, sub = lane / LPH, pairs = a.rot / 2, turning = a.rot / (2 * P);
  const bool turns = u < turning;
  // pieces of the two halves, of what turns and of the rest: neighbouring lanes have neighbouring pieces, so each load and store covers whole lines (pairs of neighbours, their two pieces side by
  // side, 123 us of the rows above, so 98)
  const int rest = (a.d - a.rot) / P, half = (rest + 1) / 2, v = u - turning;
  const int f0 = turns ? P * u : v < half ? a.rot + P * v : a.d, f1 = f0 + (turns ? pairs : P * half);
  const long row = (long)b * a.S + s;
  const T* const q = (const T*)a.Q + m * a.q_stride_m + row * a.q_stride_row;
  const T* const k = (const T*)a.K + m * a.k_stride_m + row * a.k_stride_row;
  T* const qo = (T*)a.Qo + m * a.qo_stride_m + row * a.qo_stride_row;
  T* const ko = (T*)a.Ko + m * a.ko_stride_m + row * a.ko_stride_row;

  // Every lane loads, from some row that is there where it has none of its own: a load under a condition is waited for before the next one.
  words_t x0[kAhead], x1[kAhead];
  const int at0 = f0 < a.d ? f0 : 0, at1 = f1 < a.d ? f1 : 0;
  auto load = [&](int step) {
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      if (step + t >= step1) break;                        // uniform
      const int st = step + t;
      const bool key = st >= q_steps;                      // uniform
      const int h = min((st - (key ? q_steps : 0)) * kHeads + sub, (key ? a.kv : a.heads) - 1);
      const T* p = (key ? k : q) + (long)h * a.d;
      x0[t] = *reinterpret_cast<const words_t*>(p + at0);
      x1[t] = *reinterpret_cast<const words_t*>(p + at1);
    }
  };
  load(step0);
  for (int i = lane; i < pairs; i += kWave) angle[wave][i] = rotate_angle(a, mb, s, i);
  __builtin_amdgcn_wave_barrier();
  float c[P], sn[P];
#pragma unroll
  for (int e = 0; e < P; ++e) {
    // pairs of neighbours: two of each piece
    const int pair = !a.interleaved ? P * u + e : e < P / 2 ? P / 2 * u + e : pairs / 2 + P / 2 * (u - 1) + e;
    const float2 t = turns ? angle[wave][pair] : make_float2(1.f, 0.f);
    c[e] = t.x;
    sn[e] = t.y;
  }
  float g[2 * P];
  int gamma_of = -1;
  for (int step = step0; step < step1; step += kAhead) {
#pragma unroll
    for (int t = 0; t < kAhead; ++t) {
      if (step + t >= step1) break;                        // uniform
      const int key = step + t >= q_steps;
      const int h = (step + t - (key ? q_steps : 0)) * kHeads + sub;
      const float* const gamma = key ? a.gamma_k : a.gamma_q;
      float x[2 * P];
      Pc::open(x0[t], x);
      Pc::open(x1[t], x + P);
      if (gamma) {
        if (gamma_of != key) {
          gamma_of = key;
#pragma unroll
          for (int e = 0; e < P; ++e) {
            g[e] = f0 + e < a.d ? gamma[m * a.d + f0 + e] : 0.f;
            g[P + e] = f1 + e < a.d ? gamma[m * a.d + f1 + e] : 0.f;
          }
        }
        float sum = 0.f, more = 0.f;
#pragma unroll
        for (int e = 0; e < P; ++e) sum = fmaf(x[e], x[e], sum), more = fmaf(x[P + e], x[P + e], more);
        sum = (f0 < a.d ? sum : 0.f) + (f1 < a.d ? more : 0.f);
        const float r = rsqrtf(lanes_sum<LPH>(sum) / (float)a.d + a.eps);
#pragma unroll
        for (int e = 0; e < 2 * P; ++e) x[e] = x[e] * r * g[e];
      }
      if (turns) {
        if (a.interleaved) {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float y = x[2 * e], z = x[2 * e + 1];
            x[2 * e] = y * c[e] - z * sn[e];
            x[2 * e + 1] = y * sn[e] + z * c[e];
          }
        } else {
#pragma unroll
          for (int e = 0; e < P; ++e) {
            const float y = x[e], z = x[P + e];
            x[e] = y * c[e] - z * sn[e];
            x[P + e] = y * sn[e] + z * c[e];
          }
        }
      }
      if (h < (key ? a.kv : a.heads)) {
        T* o = (key ? ko : qo) + (long)h * a.d;
        auto put = [&](T* p, const float* v) __attribute__((always_inline)) {
          if constexpr (PAST) __builtin_nontemporal_store(__builtin_bit_cast(typename Pc::store_t, Pc::close(v)), (typename Pc::store_t*)p);
          else *reinterpret_cast<words_t*>(p) = Pc::close(v);
        };
        if (f0 < a.d) put(o + f0, x);
        if (f1 < a.d) put(o + f1, x + P);
      }
    }
    if (step + kAhead < step1) load(step + kAhead);
  }
}

// A wavefront per token and head, feature lane + 64 e and the one that it turns with per lane: any head up to 256, stride and alignment.  What a lane writes another one
// may still have to read where rows are turned in place, so everything is read before anything is written.
template <typename T>
__global__ __launch_bounds__(256) void rotate_rows_kernel(RotateArgs a) {
  const int lane = threadIdx.x % kWave;
  const long wid = (long)blockIdx.x * 4 + threadIdx.x / kWave, all = a.heads + a.kv, token = wid / all;
  if (token >= (long)a.M * a.B * a.S) return;
  const long mb = token / a.S, m = mb / a.B, row = mb % a.B * a.S + token % a.S;
  const int s = (int)(token % a.S), h0 = (int)(wid % all);
  if (a.len && s >= a.len[mb]) return;
  const bool key = h0 >= a.heads;
  const int h = key ? h0 - a.heads : h0, pairs = a.rot / 2;
  const T* x = key ? (const T*)a.K + m * a.k_stride_m + row * a.k_stride_row : (const T*)a.Q + m * a.q_stride_m + row * a.q_stride_row;
  T* o = key ? (T*)a.Ko + m * a.ko_stride_m + row * a.ko_stride_row : (T*)a.Qo + m * a.qo_stride_m + row * a.qo_stride_row;
  x += (long)h * a.d;
  o += (long)h * a.d;
  const float* gamma = key ? a.gamma_k : a.gamma_q;
  float v[4], w[4];                                        // the lane's features and those that they turn with
  int other[4];
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int f = lane + kWave * e;
    other[e] = f >= a.rot ? f : a.interleaved ? f ^ 1 : f < pairs ? f + pairs : f - pairs;
    v[e] = f < a.d ? load_f32(x + f) : 0.f;
    w[e] = f < a.d ? load_f32(x + other[e]) : 0.f;
    sum = fmaf(v[e], v[e], sum);
  }
  const float r = gamma ? rsqrtf(wave_sum(sum) / (float)a.d + a.eps) : 1.f;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int f = lane + kWave * e;
    if (f >= a.d) continue;
    if (gamma) {
      v[e] = v[e] * r * gamma[m * a.d + f];
      w[e] = w[e] * r * gamma[m * a.d + other[e]];
    }
    if (f < a.rot) {
      const bool upper = a.interleaved ? f & 1 : f >= pairs;
      const float2 t = rotate_angle(a, mb, s, a.interleaved ? f / 2 : upper ? f - pairs : f);
      v[e] = upper ? w[e] * t.y + v[e] * t.x : v[e] * t.x - w[e] * t.y;
    }
  }
  __builtin_amdgcn_s_waitcnt(0);                           // every load of the wavefront has arrived
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (lane + kWave * e < a.d) store_f32(o + lane + kWave * e, v[e]);
}

}  // namespace nf
