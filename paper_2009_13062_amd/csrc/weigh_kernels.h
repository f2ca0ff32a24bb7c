// Merged decoders: the attention weight that new tokens gave to the entries of a cache, on the matrix pipe.
//
// weight_j + sum over the rows i (accepted tokens times query heads of the key head) of exp(s_ij - lse_i).  A wavefront loads 16 NK keys straight into
// operands (64-byte slices of a row, as in decoder_stream.h) and keeps them while the rows pass 16 at a time: S = Q K^T, so a lane has rows 4 g + r of ONE
// key and the sum over rows needs no exchange until the end.  What a row adds besides its queries (lse, slope, position, last slot that it sees)
// lies in a table of the wavefront in LDS, read 4 rows at a time.  Keys are read once and each slot belongs to one lane: no atomics, one order of
// the sum.  Bound by the keys' bytes.
#pragma once
#include "decoder_stream.h"

namespace nf {

template <typename T, int D> constexpr int weigh_keys() { return 16 * StreamShape<T, D>::NK * (D == 256 ? 1 : 2); }   // per wavefront: 64 registers

template <typename T, int D>
__global__ __launch_bounds__(256) void weigh_tiles_kernel(WeighArgs a, int blocks_per_head) {
  using Sh = StreamShape<T, D>;
  constexpr bool kBf = Sh::kBf;
  constexpr int kKeys = weigh_keys<T, D>(), NK = kKeys / 16, SL = Sh::kSlices;
  __shared__ __align__(16) float table[4][4][16];          // per wavefront: lse, slope, position, end of 16 rows
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int g4 = lane / 16, l16 = lane % 16;
  const long head = blockIdx.x / blocks_per_head;          // (m, b, g)
  const int j0 = ((int)(blockIdx.x % blocks_per_head) * 4 + wave) * kKeys;
  if (j0 >= a.C) return;                                   // uniform per wavefront; no barrier below
  const long mb = head / a.kv;
  const int g = (int)(head % a.kv), b = (int)(mb % a.B), group = a.heads / a.kv;
  const long m = mb / a.B;
  const int L = clamp_len(a.len[mb], a.C), cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n;
  const int begin = a.start ? a.start[mb] : L, held = min(L + cnt, a.C);
  const float unit = kBf ? kLog2e : 1.f;
  float sum[NK];
#pragma unroll
  for (int k = 0; k < NK; ++k) sum[k] = 0.f;
  if (j0 < held) {
    const auto rk = rows_from((const T*)a.Kc + (head * a.C + j0) * a.d);
    uint4 kf[NK][SL];
    int at[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      const int key = j0 + 16 * k + l16;
#pragma unroll
      for (int sl = 0; sl < SL; ++sl) {
        const int f = sl * Sh::kSliceF + g4 * Sh::kPiece;
        kf[k][sl] = rows_load16(rk, (key < held) & (f < a.d) ? ((16 * k + l16) * a.d + f) * (unsigned)sizeof(T) : kDecOob);
      }
      at[k] = key;
      if (a.slope && a.pos) at[k] = a.pos[head * a.C + min(key, held - 1)];
    }
    const int rows = cnt * group;
    lds_f32_t* const tab = (lds_f32_t*)&table[wave][0][0];
    for (int r0 = 0; r0 < rows; r0 += 16) {
      const int r = r0 + l16, i = min(r, rows - 1) / group, h = g * group + (min(r, rows - 1) - i * group);
      const int row = a.index ? a.index[mb * a.n + i] : i;
      const bool there = r < rows && row >= 0 && row < a.T;
      const float lse = there ? a.lse[(mb * a.T + row) * a.heads + h] : -INFINITY;
      const bool counts = lse != -INFINITY;
      const T* q = (const T*)a.Q + m * a.q_stride_m + ((long)b * a.T + (there ? row : 0)) * a.q_stride_row + (long)h * a.d;
      uint4 qf[SL];
#pragma unroll
      for (int sl = 0; sl < SL; ++sl) {
        const int f = sl * Sh::kSliceF + g4 * Sh::kPiece;
        qf[sl] = make_uint4(0, 0, 0, 0);
        if (counts && f < a.d) qf[sl] = *reinterpret_cast<const uint4*>(q + f);
      }
      __builtin_amdgcn_wave_barrier();
      if (g4 == 0) {
        tab[l16] = counts ? lse * unit : 0.f;
        tab[16 + l16] = a.slope ? a.slope[m * a.heads + h] * unit : 0.f;
        tab[32 + l16] = __int_as_float(begin + i);
        tab[48 + l16] = __int_as_float(counts ? min(L + i + 1, a.C) : 0);
      }
      __builtin_amdgcn_wave_barrier();
      f32x4_t s[NK];
#pragma unroll
      for (int k = 0; k < NK; ++k) s[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int sl = 0; sl < SL; ++sl)
#pragma unroll
        for (int k = 0; k < NK; ++k) s[k] = slice_product<T>(qf[sl], kf[k][sl], s[k]);
      // element e of s[k]: row r0 + 4 g4 + e against key j0 + 16 k + l16
      if (r0 + 4 * g4 < rows) {
        const f32x4v_t z = *(const lds_f32x4_t*)(tab + 4 * g4), w = *(const lds_f32x4_t*)(tab + 16 + 4 * g4), mine = *(const lds_f32x4_t*)(tab + 32 + 4 * g4), end = *(const lds_f32x4_t*)(tab + 48 + 4 * g4);
#pragma unroll
        for (int k = 0; k < NK; ++k) {
          const int key = j0 + 16 * k + l16;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            float x = s[k][e];
            if (a.cap != 0.f) {
              if constexpr (kBf) {
                x = tanh_either(x * (a.scale * a.inv_cap)) * (a.cap * kLog2e);
              } else {
                x = a.cap * tanhf(x * a.scale * a.inv_cap);
              }
            } else {
              x *= a.scale * unit;
            }
            if (a.slope) x = fmaf(-w[e], fabsf((float)(__float_as_int(mine[e]) - at[k])), x);
            x -= z[e];
            const float p = kBf ? __builtin_amdgcn_exp2f(x) : expf(x);
            sum[k] += key < __float_as_int(end[e]) ? p : 0.f;
          }
        }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < NK; ++k) {
    const float total = across_halves(across_rows(sum[k], AddOp{}), AddOp{});
    const int key = j0 + 16 * k + l16;
    if (k % 4 == g4 && key < a.C && (a.out != a.weight || key < held)) {
      const long o = head * a.C + key;
      a.out[o] = a.weight[o] + total;
    }
  }
}

}  // namespace nf
