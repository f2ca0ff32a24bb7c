// Merged decoders: the attention weight that new tokens gave to the entries of a cache, on the matrix pipe.
//
// weight_j + sum over the rows i (accepted tokens times query heads of the key head) of exp(s_ij - lse_i).  A wavefront loads 16 NK keys straight into
// operands (64-byte slices of a row, as in decoder_stream.h) and keeps them while the rows pass 16 at a time: S = Q K^T, so a lane has rows 4 g + r of ONE
// key and the sum over rows needs no exchange until the end.  What a row adds besides its queries (lse, slope, position, last slot that it sees)
// lies in a table of the wavefront in LDS, read 4 rows at a time.  Keys are read once and each slot belongs to one lane: no atomics, one order of
// the sum.  Bound by the keys' bytes up to 16 rows (5.4 TB/s of 7.1; above, by looking the rows up: float32, 8 tokens of groups of 4 over 32 caches of 8192, 419 us): a wavefront takes `turns` blocks of keys one after the other, the next one's on their way meanwhile, and up to 16 rows
// are looked up once for all of them.
#pragma once
#include "decoder_stream.h"

namespace nf {

// Two loads of 8 rows by 128 bytes (lanes 0-7 of each 16 the first 64, lanes 8-15 the second) into two of 16 rows by 64: lanes 8-15 of the first against
// lanes 0-7 of the second.
__device__ __forceinline__ void trade_halves(uint4& a, uint4& b) {
  auto one = [](uint32_t& x, uint32_t& y) {
    const uint32_t p = (uint32_t)__builtin_amdgcn_update_dpp((int)x, (int)y, kRowRor8, 0xf, 0xc, false);
    y = (uint32_t)__builtin_amdgcn_update_dpp((int)y, (int)x, kRowRor8, 0xf, 0x3, false);
    x = p;
  };
  one(a.x, b.x);
  one(a.y, b.y);
  one(a.z, b.z);
  one(a.w, b.w);
}

template <typename T, int D> constexpr int weigh_keys() { return 16 * StreamShape<T, D>::NK; }   // per wavefront and turn

// MANY: more than 16 rows.  (A kernel of its own for fewer: they are looked up once, and without the loop four wavefronts fit a SIMD where three did; one token over 32 caches of
// 8192 entries, 8 heads of 128: 94.5 -> 78 us.  The next rows on their way while one block of them is worked on: 26 tokens of groups of 4 46 -> 42 and 17.4 -> 15 us, 6
// tokens 20.0 -> 21.0, not kept.)
template <typename T, int D, bool MANY>
__global__ __launch_bounds__(256) void weigh_tiles_kernel(WeighArgs a, int blocks_per_head, int turns) {
  using Sh = StreamShape<T, D>;
  constexpr bool kBf = Sh::kBf;
  constexpr int kKeys = weigh_keys<T, D>(), NK = kKeys / 16, SL = Sh::kSlices;
  __shared__ __align__(16) float table[4][4][16];          // per wavefront: lse, slope, position, end of 16 rows
  const int tid = threadIdx.x, lane = tid % kWave;
  const int wave = __builtin_amdgcn_readfirstlane(tid / kWave);
  const int g4 = lane / 16, l16 = lane % 16;
  const unsigned uhead = blockIdx.x / blocks_per_head, umb = uhead / a.kv;      // (m, b, g)
  const int first = ((int)(blockIdx.x % blocks_per_head) * 4 * turns + wave) * kKeys;
  if (first >= a.C) return;                                // uniform per wavefront; no barrier below
  const long head = uhead, mb = umb, m = umb / a.B;
  const int g = (int)(uhead % a.kv), b = (int)(umb % a.B), group = a.heads / a.kv;
  const int L = clamp_len(a.len[mb], a.C), cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n;
  const int held = min(L + cnt, a.C), rows = cnt * group;
  const float unit = kBf ? kLog2e : 1.f;
  const T* const Kh = (const T*)a.Kc + head * a.C * a.d;
  const bool inplace = a.out == a.weight;

  uint4 kf[NK][SL], knext[NK][SL];
  float w[NK], wnext[NK];
  // Each 128-byte line in one load and past the caches (one token over 32 caches of 8192 entries, 8 heads of 128: 104 -> 95 us; as 64-byte slices past
  // the caches 119, full lines through them 101).
  auto fetch = [&](int j0) {
    const auto rk = rows_from(Kh + (long)j0 * a.d);
#pragma unroll
    for (int k = 0; k < NK; ++k) {
#pragma unroll
      for (int sl = 0; sl < SL; ++sl) {
        const int f = (sl / 2 * 2 + l16 / 8) * Sh::kSliceF + g4 * Sh::kPiece, key = 16 * k + l16 % 8 + sl % 2 * 8;
        knext[k][sl] = rows_load16<2>(rk, (j0 + key < held) & (f < a.d) ? (key * a.d + f) * (unsigned)sizeof(T) : kDecOob);
      }
      wnext[k] = a.weight[head * a.C + min(j0 + 16 * k + l16, a.C - 1)];
    }
  };
  fetch(first);

  uint4 qf[SL];
  lds_f32_t* const tab = (lds_f32_t*)&table[wave][0][0];
  auto look_up = [&](int r0) {                             // rows r0 .. + 15
    const int r = min(r0 + l16, rows - 1), i = r / group, h = g * group + (r - i * group);
    const int row = a.index ? a.index[mb * a.n + i] : i;
    const bool there = r0 + l16 < rows && row >= 0 && row < a.T;
    const int safe = there ? row : 0;
    const float lse = there ? a.lse[(mb * a.T + safe) * a.heads + h] : -INFINITY;
    const bool counts = lse != -INFINITY;
    const T* q = (const T*)a.Q + m * a.q_stride_m + ((long)b * a.T + safe) * a.q_stride_row + (long)h * a.d;
#pragma unroll
    for (int sl = 0; sl < SL; ++sl) {
      const int f = sl * Sh::kSliceF + g4 * Sh::kPiece;
      qf[sl] = make_uint4(0, 0, 0, 0);
      if (there && f < a.d) qf[sl] = *reinterpret_cast<const uint4*>(q + f);
    }
    __builtin_amdgcn_wave_barrier();
    if (g4 == 0) {
      tab[l16] = counts ? lse * unit : 0.f;
      tab[16 + l16] = a.slope ? a.slope[m * a.heads + h] * unit : 0.f;
      tab[32 + l16] = __int_as_float((a.start ? a.start[mb] : L) + i);
      tab[48 + l16] = __int_as_float(counts ? min(L + i + 1, a.C) : 0);
    }
    __builtin_amdgcn_wave_barrier();
  };
  if (!MANY && rows > 0) look_up(0);

  for (int turn = 0; turn < turns; ++turn) {
    const int j0 = first + turn * 4 * kKeys;
    if (j0 >= a.C) return;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
#pragma unroll
      for (int sl = 0; sl < SL; sl += 2) {
        kf[k][sl] = knext[k][sl];
        kf[k][sl + 1] = knext[k][sl + 1];
        trade_halves(kf[k][sl], kf[k][sl + 1]);
      }
      w[k] = wnext[k];
    }
    if (turn + 1 < turns && j0 + 4 * kKeys < a.C) fetch(j0 + 4 * kKeys);
    float sum[NK];
    int at[NK];
#pragma unroll
    for (int k = 0; k < NK; ++k) {
      sum[k] = 0.f;
      at[k] = j0 + 16 * k + l16;
    }
    if (j0 < held && rows > 0) {
      if (a.slope && a.pos) {
#pragma unroll
        for (int k = 0; k < NK; ++k) at[k] = a.pos[head * a.C + min(at[k], held - 1)];
      }
      for (int r0 = 0; r0 < (MANY ? rows : 1); r0 += 16) {
        if (MANY) look_up(r0);
        f32x4_t s[NK];
#pragma unroll
        for (int k = 0; k < NK; ++k) s[k] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int sl = 0; sl < SL; ++sl)
#pragma unroll
          for (int k = 0; k < NK; ++k) s[k] = slice_product<T>(qf[sl], kf[k][sl], s[k]);
        // element e of s[k]: row r0 + 4 g4 + e against key j0 + 16 k + l16
        if (r0 + 4 * g4 < rows) {
          const f32x4v_t z = *(const lds_f32x4_t*)(tab + 4 * g4), slope = *(const lds_f32x4_t*)(tab + 16 + 4 * g4), mine = *(const lds_f32x4_t*)(tab + 32 + 4 * g4),
                         end = *(const lds_f32x4_t*)(tab + 48 + 4 * g4);
#pragma unroll
          for (int k = 0; k < NK; ++k) {
            const int key = j0 + 16 * k + l16;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              float x = s[k][e];
              if (a.cap != 0.f) {
                if constexpr (kBf) x = tanh_either(x * (a.scale * a.inv_cap)) * (a.cap * kLog2e);
                else x = a.cap * tanhf(x * a.scale * a.inv_cap);
              } else {
                x *= a.scale * unit;
              }
              if (a.slope) x = fmaf(-slope[e], fabsf((float)(__float_as_int(mine[e]) - at[k])), x);
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
      if (k % 4 == g4 && key < a.C && (!inplace || key < held)) a.out[head * a.C + key] = w[k] + total;
    }
  }
}

}  // namespace nf
