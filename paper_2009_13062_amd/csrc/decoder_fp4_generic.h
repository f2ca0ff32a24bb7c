// Merged decoders, attention of drafted trees over a cache of 4 bits: the kernel that takes any head size up to 256, any stride and any alignment.
#pragma once
#include "decoder.h"
#include "fp4.h"

namespace nf {

// As decoder_rows_kernel: one wavefront per query row; keys 64 at a time, one per lane, with a running maximum and sum; feature t = lane + 64 e of the output per lane.
template <typename T, int DPL>
__global__ __launch_bounds__(256) void decoder_fp4_rows_kernel(DecArgs a) {
  __shared__ float qs[4][64 * DPL];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const long wid = (long)blockIdx.x * 4 + wave;
  if (wid >= (long)a.M * a.B * a.heads * a.N) return;      // uniform per wavefront
  const int i = (int)(wid % a.N);
  const long mb = wid / a.N / a.heads;
  const int h = (int)(wid / a.N % a.heads), b = (int)(mb % a.B), m = (int)(mb / a.B), g = h / (a.heads / a.kv);
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

  // one key per lane, its feature t key(t), whether this query sees it and how far away it is; feature t of the value of key jj value(jj, t)
  auto visit = [&](auto key, bool seen, float dist, auto value, int nj) {
    float s = -INFINITY;
    if (seen) {
      float dot = 0.f;
      for (int tt = 0; tt < a.d; ++tt) dot = fmaf(qs[wave][tt], key(tt), dot);
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
#pragma unroll
      for (int e = 0; e < DPL; ++e) {
        const int tt = lane + 64 * e;
        if (tt < a.d) acc[e] = fmaf(pj, value(jj, tt), acc[e]);
      }
    }
  };

  const int there = a.nodes ? clamp_len(a.nodes[mb], a.N) : a.N;
  if (i < there) {
    const int L = clamp_len(a.len[mb], a.C), CB = fp4_code_bytes(a.d), SB = fp4_scale_bytes(a.d);
    const uint64_t path = tree_path(a.parent ? a.parent + mb * a.N : nullptr, i);
    const int mine = (a.start ? a.start[mb] : L) + __popcll(path) - 1;
    const long head = (mb * a.kv + g) * a.C;
    const uint8_t *Kh = (const uint8_t*)a.Kc + head * CB, *Vh = (const uint8_t*)a.Vc + head * CB, *Kz = a.Ks + head * SB, *Vz = a.Vs + head * SB;
    for (int j0 = 0; j0 < L; j0 += 64) {
      const int j = j0 + lane;
      const bool seen = j < L;
      const float dist = a.slope && seen ? fabsf((float)(mine - (a.pos ? a.pos[head + j] : j))) : 0.f;
      visit([&](int tt) { return fp4_value(Kh + (long)j * CB, Kz + (long)j * SB, tt); }, seen, dist,
            [&](int jj, int tt) { return fp4_value(Vh + (long)(j0 + jj) * CB, Vz + (long)(j0 + jj) * SB, tt); }, min(64, L - j0));
    }
    const float dist = (float)(__popcll(path >> lane) - 1);
    visit([&](int tt) { return load_f32(Kp + (long)lane * a.kv_stride_row + tt); }, (path >> lane) & 1, dist,
          [&](int jj, int tt) { return load_f32(Vp + (long)jj * a.kv_stride_row + tt); }, i + 1);
  }

  T* Op = (T*)a.O + (mb * a.N + i) * ((long)a.heads * a.d) + (long)h * a.d;
  const float inv = lrun == 0.f ? 0.f : 1.f / lrun;        // a row that sees nothing: acc is 0
#pragma unroll
  for (int e = 0; e < DPL; ++e) {
    const int tt = lane + 64 * e;
    if (tt < a.d) store_f32(Op + tt, lrun == 0.f ? 0.f : acc[e] * inv);
  }
  if (a.lse && lane == 0) a.lse[(mb * a.N + i) * a.heads + h] = lrun == 0.f ? -INFINITY : mrun + logf(lrun);
}

}  // namespace nf
