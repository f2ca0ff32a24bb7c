// A cache held in 4 bits: rows quantised as they are appended, entries read back.
//
// Bound by bytes in large calls (32 prompts of up to 2039 rows, 8 heads of 128, bfloat16: 261 MB read and written, then read back, 465 MB in 96 us together; 16 caches of up to
// 16384 read back: 0.2 GB read and 1.07 written, the 0 past the counts too, in 206 us, 6.2 TB/s), by the launch in small ones (3 us each).
#pragma once
#include "decoder.h"
#include "fp4.h"

namespace nf {

struct AppendFp4Args {
  const void* K; const void* V; const int* index; const int* count; const int* len; const int* start;
  uint8_t* Kc; uint8_t* Ks; uint8_t* Vc; uint8_t* Vs; int* pos; float* weight;
  int M, B, T, n, C, kv, d;
  long stride_m, stride_row;
};

// The largest magnitude over the four lanes of a group: each has eight of its features.
__device__ __forceinline__ uint32_t group_top(uint32_t top) {
  top = max(top, (uint32_t)dpp<kQuadXor1>((int)top));
  return max(top, (uint32_t)dpp<kQuadXor2>((int)top));
}

// Eight features of a row from feature f on, those past d as 0, and their codes; the scale of the lane's group comes along (every lane of a quad has to come there).  WIDE: d, strides and
// pointers in 16-byte pieces.  A piece of bfloat16 is read once, past the caches (append and read back of the prompts above 102 us, so 96); of float32 two lie in a line (97 us of the same
// rows of 64 features, past the caches 107).
template <typename T, bool WIDE> struct Eight {
  float x[8];
  __device__ __forceinline__ void load(const T* row, int f, int d) {
    if constexpr (WIDE) {
#pragma unroll
      for (int h = 0; h < 8; h += 4) {
        const float4 v = *reinterpret_cast<const float4*>(row + (f + h < d ? f + h : 0));
        const bool in = f + h < d;
        x[h] = in ? v.x : 0.f; x[h + 1] = in ? v.y : 0.f; x[h + 2] = in ? v.z : 0.f; x[h + 3] = in ? v.w : 0.f;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = load_f32(row + (f + e < d ? f + e : 0));
        x[e] = f + e < d ? v : 0.f;
      }
    }
  }
  __device__ __forceinline__ uint32_t codes(uint32_t& scale) const {
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    scale = fp4_scale(group_top(top));
    return fp4_codes(x, scale);
  }
};
template <> struct Eight<bf16_t, true> {
  uint4 w;
  __device__ __forceinline__ void load(const bf16_t* row, int f, int d) {
    w = ldnt16(row + (f < d ? f : 0));
    if (f >= d) w = make_uint4(0, 0, 0, 0);
  }
  __device__ __forceinline__ uint32_t codes(uint32_t& scale) const {
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(ws[e] << 16 & 0x7fffffffu, ws[e] & 0x7fff0000u));
    scale = fp4_scale(group_top(top));
    return fp4_codes(w, scale);
  }
};

// The scales of a head's groups, a byte each in lanes 0, 4, .. of the head's, to one number in the first of them (2 or 4 groups: the lanes of a head lie in a row of 16).
template <int G> __device__ __forceinline__ uint32_t gather_scales(uint32_t s) {
  constexpr int kRowShl = 0x100;
  uint32_t all = s | (uint32_t)dpp<kRowShl + 4>((int)s) << 8;
  if constexpr (G == 4) all |= (uint32_t)dpp<kRowShl + 8>((int)s) << 16 | (uint32_t)dpp<kRowShl + 12>((int)s) << 24;
  return all;
}

// A workgroup takes rows of one head of one sequence, so what it writes is one run of codes, of scales, of positions and of weights; a lane takes eight features of a key and its value, four
// lanes a group.  G: the groups of a head where these are 2 or 4, 0 for others.  (A lane that takes four rows, all their loads on their way at once, leaves fewer wavefronts: append and read back 109 us, so 102.)
template <typename T, bool WIDE, int G>
__global__ __launch_bounds__(256) void cache_append_fp4_kernel(AppendFp4Args a, int blocks_per_head) {
  const int groups = G ? G : fp4_groups(a.d), S = G ? G : fp4_scale_bytes(a.d), units = 4 * groups, at_once = 256 / units;
  const unsigned uhead = blockIdx.x / blocks_per_head, umb = uhead / a.kv;
  const int g = (int)(uhead - umb * a.kv), b = (int)(umb % a.B);
  const long mb = umb, m = umb / a.B, head = uhead;
  const int cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n, L = clamp_len(a.len[mb], a.C);
  const int end = min(cnt, a.C - L);                       // entries past the capacity are not written
  const int r = (int)threadIdx.x / units, u = (int)threadIdx.x - r * units, i = (int)(blockIdx.x - uhead * blocks_per_head) * at_once + r;
  if (r >= at_once || i >= end) return;                    // whole groups of lanes
  const int row = a.index ? a.index[mb * a.n + i] : i, first = a.start ? a.start[mb] : L;
  if (row < 0 || row >= a.T) return;
  const long at = m * a.stride_m + ((long)b * a.T + row) * a.stride_row + (long)g * a.d, slot = head * a.C + L + i;
  Eight<T, WIDE> k, v;
  k.load((const T*)a.K + at, 8 * u, a.d);
  v.load((const T*)a.V + at, 8 * u, a.d);
  uint32_t ks, vs;
  const uint32_t kc = k.codes(ks), vc = v.codes(vs);
  ((uint32_t*)a.Kc)[slot * units + u] = kc;
  ((uint32_t*)a.Vc)[slot * units + u] = vc;
  if constexpr (G == 4 || G == 2) {
    using Scales = std::conditional_t<G == 4, uint32_t, uint16_t>;
    const uint32_t ksum = gather_scales<G>(ks), vsum = gather_scales<G>(vs);
    if (u == 0) {
      ((Scales*)a.Ks)[slot] = (Scales)ksum;
      ((Scales*)a.Vs)[slot] = (Scales)vsum;
    }
  } else {
    if (u % 4 == 0) {
      a.Ks[slot * S + u / 4] = (uint8_t)ks;
      a.Vs[slot * S + u / 4] = (uint8_t)vs;
    }
    if (u == 0 && S > groups) {
      a.Ks[slot * S + groups] = 0;
      a.Vs[slot * S + groups] = 0;
    }
  }
  if (u == 0) {
    if (a.pos) a.pos[slot] = first + i;
    if (a.weight) a.weight[slot] = 0.f;
  }
}

struct ReadFp4Args {
  const uint8_t* Kc; const uint8_t* Ks; const uint8_t* Vc; const uint8_t* Vs; const int* first; const int* count;
  void* K; void* V;
  int M, B, n, C, kv, d;
};

// A workgroup takes entries of one head; a lane gives 16 bytes of an entry, of its key and of its value (two of codes for four features of float32, four for eight of bfloat16).  (Four
// entries to a lane: 231 us of the 16 caches above, so 206; keys and values in workgroups of their own 288.)  PAST: results that the second caches do not hold go past
// them (us, through them / past them: 1.07 GB 215 / 206, 268 MB 59 / 49, 134 MB 32 / 26, 50 MB 11.2 / 9.9, 17 MB 5.8 / 5.0, which whoever reads them next would pay for).
// Above 32 MB it depends on the reader (read back and read, us, through / past: one token over keys and values of bfloat16, 67 MB 39 / 40, 134 MB 54 / 57, 268 MB 105 / 99, 537 MB 207 / 202; keys
// alone and their weighing, 67 MB 33 / 29, 100 MB 44 / 42, 134 MB 54 / 53).
template <typename T, bool WIDE, bool PAST>
__global__ __launch_bounds__(256) void cache_read_fp4_kernel(ReadFp4Args a, int blocks_per_head) {
  constexpr int F = 16 / (int)sizeof(T);                   // features of a lane
  using Codes = std::conditional_t<F == 8, uint32_t, uint16_t>;
  const int S = fp4_scale_bytes(a.d), row = fp4_code_bytes(a.d) / (int)sizeof(Codes), units = (a.d + F - 1) / F, at_once = 256 / units;
  const unsigned uhead = blockIdx.x / blocks_per_head;
  const long head = uhead, mb = uhead / a.kv;
  const int r = (int)threadIdx.x / units, u = (int)threadIdx.x - r * units, i = (int)(blockIdx.x - uhead * blocks_per_head) * at_once + r;
  if (r >= at_once || i >= a.n) return;
  const int first = a.first ? a.first[mb] : 0, cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n;
  const long long slot = (long long)first + i;
  const bool there = i < cnt && slot >= 0 && slot < a.C;
  const long at = head * a.C + (there ? slot : 0), to = (head * a.n + i) * a.d + F * u;          // an entry that is not there: some entry's bytes, not used
  uint32_t code[2] = {}, scale[2] = {};
#pragma unroll
  for (int t = 0; t < 2; ++t)
    if (t == 0 || a.V) {
      code[t] = ((const Codes*)(t ? a.Vc : a.Kc))[at * row + u];
      scale[t] = (t ? a.Vs : a.Ks)[at * S + u * F / kFp4Group];
    }
#pragma unroll
  for (int t = 0; t < 2; ++t) {
    if (t == 1 && !a.V) break;
    T* out = (T*)(t ? a.V : a.K) + to;
    const uint32_t c = there ? code[t] : 0u;
    const float s = fp4_scale_value(there ? scale[t] : 127u);
    uint4 w;
    if constexpr (F == 8) {
      w = fp4_values_bf16(c, s);
    } else {
      const f32x2_t lo = fp4_pair_f32<0>(c, s), hi = fp4_pair_f32<1>(c, s);
      w = make_uint4(__float_as_uint(lo.x), __float_as_uint(lo.y), __float_as_uint(hi.x), __float_as_uint(hi.y));
    }
    if constexpr (WIDE && PAST) {
      __builtin_nontemporal_store(nf_u32x4_t{w.x, w.y, w.z, w.w}, (nf_u32x4_t*)out);
    } else if constexpr (WIDE) {
      *reinterpret_cast<uint4*>(out) = w;
    } else {
      T v[F];
      __builtin_memcpy(v, &w, 16);
#pragma unroll
      for (int e = 0; e < F; ++e)
        if (F * u + e < a.d) out[e] = v[e];
    }
  }
}

}  // namespace nf
