// Merged decoders, the kernels that take any head size up to 256, any stride and any alignment.
#pragma once
#include "decoder.h"

namespace nf {

// One wavefront per query row; keys 64 at a time, one per lane, with a running maximum and sum; feature t = lane + 64 e of the output
// per lane.  Bound by latency: a key's dot product is a chain of dependent loads over its row.
template <typename T, int DPL, bool TREE>
__global__ __launch_bounds__(256) void decoder_rows_kernel(DecArgs a) {
  __shared__ float qs[4][64 * DPL];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const long wid = (long)blockIdx.x * 4 + wave;
  if (wid >= (long)a.M * a.B * a.heads * a.N) return;      // uniform per wavefront
  const int i = (int)(wid % a.N);
  long t = wid / a.N;
  const int h = (int)(t % a.heads);  t /= a.heads;
  const long mb = t;
  const int b = (int)(t % a.B), m = (int)(t / a.B);
  const int g = h / (a.heads / a.kv);
  const long row0 = (long)b * a.N;
  const T* Qp = (const T*)a.Q + m * a.q_stride_m + (row0 + i) * a.q_stride_row + (long)h * a.d;
  const T* Kp = (const T*)a.K + m * a.kv_stride_m + row0 * a.kv_stride_row + (long)g * a.d;
  const T* Vp = (const T*)a.V + m * a.kv_stride_m + row0 * a.kv_stride_row + (long)g * a.d;
  const float slope = a.slope ? a.slope[(long)m * a.heads + h] : 0.f;
#pragma unroll
  for (int e = 0; e < DPL; ++e) {
    const int tt = lane + 64 * e;
    qs[wave][tt] = tt < a.d ? load_f32(Qp + tt) : 0.f;
  }
  __builtin_amdgcn_wave_barrier();
  float mrun = kLowestScore, lrun = 0.f, acc[DPL];
#pragma unroll
  for (int e = 0; e < DPL; ++e) acc[e] = 0.f;

  // one key per lane: its row, whether this query sees it and how far away it is; the 64 value rows begin at v0
  auto visit = [&](const T* kr, bool seen, float dist, const T* v0, long vstride, int nj) {
    float s = -INFINITY;
    if (seen) {
      float dot = 0.f;
      for (int tt = 0; tt < a.d; ++tt) dot = fmaf(qs[wave][tt], load_f32(kr + tt), dot);
      s = fmaf(-slope, dist, capped(dot * a.scale, a));
    }
    const float mnew = fmaxf(mrun, wave_max(s));
    const float p = seen ? expf(s - mnew) : 0.f, corr = expf(mrun - mnew);
    lrun = lrun * corr + wave_sum(p);
    mrun = mnew;
#pragma unroll
    for (int e = 0; e < DPL; ++e) acc[e] *= corr;
    for (int jj = 0; jj < nj; ++jj) {
      const float pj = __shfl(p, jj, kWave);
      if (pj == 0.f) continue;                             // uniform; a key without weight adds nothing, whatever its values
      const T* vr = v0 + (long)jj * vstride;
#pragma unroll
      for (int e = 0; e < DPL; ++e) {
        const int tt = lane + 64 * e;
        if (tt < a.d) acc[e] = fmaf(pj, load_f32(vr + tt), acc[e]);
      }
    }
  };

  if constexpr (TREE) {
    const int there = a.nodes ? clamp_len(a.nodes[mb], a.N) : a.N;
    if (i < there) {
      const int L = clamp_len(a.len[mb], a.C);
      const uint64_t path = tree_path(a.parent ? a.parent + mb * a.N : nullptr, i);
      const int mine = (a.start ? a.start[mb] : L) + __popcll(path) - 1;
      const long head = (mb * a.kv + g) * a.C;
      const T* Kh = (const T*)a.Kc + head * a.d;
      const T* Vh = (const T*)a.Vc + head * a.d;
      for (int j0 = 0; j0 < L; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < L;
        const float dist = a.slope && seen ? fabsf((float)(mine - (a.pos ? a.pos[head + j] : j))) : 0.f;
        visit(Kh + (long)j * a.d, seen, dist, Vh + (long)j0 * a.d, a.d, min(64, L - j0));
      }
      const float dist = (float)(__popcll(path >> lane) - 1);
      visit(Kp + (long)lane * a.kv_stride_row, (path >> lane) & 1, dist, Vp, a.kv_stride_row, i + 1);
    }
  } else {
    const int L = a.len ? clamp_len(a.len[mb], a.N) : a.N;
    const int* doc = a.doc ? a.doc + mb * a.N : nullptr;
    if (i < L && (!doc || doc[i] >= 0)) {
      const int first = a.prefix ? clamp_len(a.prefix[mb], L) : 0;           // keys below it are seen by every row
      const int end = a.causal ? max(i + 1, first) : L;
      for (int j0 = 0; j0 < end; j0 += 64) {
        const int j = j0 + lane;
        const bool seen = j < end && (!doc || doc[j] == doc[i]);
        visit(Kp + (long)j * a.kv_stride_row, seen, (float)abs(i - j), Vp + (long)j0 * a.kv_stride_row, a.kv_stride_row, min(64, end - j0));
      }
    }
  }

  T* Op = (T*)a.O + (mb * a.N + i) * ((long)a.heads * a.d) + (long)h * a.d;
  const float inv = lrun == 0.f ? 0.f : 1.f / lrun;        // a row that sees nothing: acc is 0
#pragma unroll
  for (int e = 0; e < DPL; ++e) {
    const int tt = lane + 64 * e;
    if (tt < a.d) store_f32(Op + tt, lrun == 0.f ? 0.f : acc[e] * inv);
  }
  if (TREE && a.lse && lane == 0) a.lse[(mb * a.N + i) * a.heads + h] = lrun == 0.f ? -INFINITY : mrun + logf(lrun);
}

// One thread per slot; its key row is read again for every token and head.
template <typename T>
__global__ __launch_bounds__(256) void weigh_rows_kernel(WeighArgs a, int blocks_per_head) {
  const long head = blockIdx.x / blocks_per_head;          // (m, b, g)
  const int j = (int)(blockIdx.x % blocks_per_head) * 256 + threadIdx.x;
  if (j >= a.C) return;
  const long mb = head / a.kv;
  const int g = (int)(head % a.kv), b = (int)(mb % a.B), m = (int)(mb / a.B), group = a.heads / a.kv;
  const int L = clamp_len(a.len[mb], a.C), cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n;
  const int begin = a.start ? a.start[mb] : L;
  const T* kr = (const T*)a.Kc + (head * a.C + j) * a.d;
  float sum = 0.f;
  for (int i = max(0, j - L); i < cnt; ++i) {              // token i sees slots up to L + i
    const int row = a.index ? a.index[mb * a.n + i] : i;
    if (row < 0 || row >= a.T) continue;
    const float dist = a.slope ? fabsf((float)(begin + i - (a.pos ? a.pos[head * a.C + j] : j))) : 0.f;
    for (int x = 0; x < group; ++x) {
      const int h = g * group + x;
      const float lse = a.lse[((long)mb * a.T + row) * a.heads + h];
      if (lse == -INFINITY) continue;
      const T* q = (const T*)a.Q + m * a.q_stride_m + ((long)b * a.T + row) * a.q_stride_row + (long)h * a.d;
      float dot = 0.f;
      for (int t = 0; t < a.d; ++t) dot = fmaf(load_f32(q + t), load_f32(kr + t), dot);
      float s = dot * a.scale;
      if (a.cap != 0.f) s = a.cap * tanhf(s * a.inv_cap);
      if (a.slope) s = fmaf(-a.slope[(long)m * a.heads + h], dist, s);
      sum += expf(s - lse);
    }
  }
  const long o = head * a.C + j;
  if (a.out != a.weight || sum != 0.f) a.out[o] = a.weight[o] + sum;
}

}  // namespace nf
