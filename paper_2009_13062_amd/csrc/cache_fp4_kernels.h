// A cache held in 4 bits: rows quantised as they are appended, entries read back.
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

// Eight features of a row from feature f on, those past d as 0.  WIDE: d, strides and pointers in 16-byte pieces.
template <typename T, bool WIDE> __device__ __forceinline__ void fp4_load8(const T* row, int f, int d, float (&x)[8]) {
  if constexpr (WIDE) {
#pragma unroll
    for (int h = 0; h < 8; h += 4) {
      const float4 v = f + h < d ? *reinterpret_cast<const float4*>(row + f + h) : make_float4(0.f, 0.f, 0.f, 0.f);
      x[h] = v.x; x[h + 1] = v.y; x[h + 2] = v.z; x[h + 3] = v.w;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = f + e < d ? load_f32(row + f + e) : 0.f;
  }
}

// The largest magnitude over the four lanes of a group: each has eight of its features.
__device__ __forceinline__ uint32_t group_top(uint32_t top) {
  top = max(top, (uint32_t)dpp<kQuadXor1>((int)top));
  return max(top, (uint32_t)dpp<kQuadXor2>((int)top));
}

// Eight features of a lane to their codes; the scale of the lane's group comes along.  Every lane of a quad has to come here.
template <typename T, bool WIDE> __device__ __forceinline__ uint32_t fp4_quantise8(const T* row, int f, int d, uint32_t& scale) {
  if constexpr (WIDE && sizeof(T) == 2) {
    const uint4 w = f < d ? *reinterpret_cast<const uint4*>(row + f) : make_uint4(0, 0, 0, 0);
    uint32_t top = 0;
    const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) top = max(top, max(ws[e] << 16 & 0x7fffffffu, ws[e] & 0x7fff0000u));
    scale = fp4_scale(group_top(top));
    return fp4_codes(w, scale);
  } else {
    float x[8];
    fp4_load8<T, WIDE>(row, f, d, x);
    uint32_t top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, __float_as_uint(x[e]) & 0x7fffffffu);
    scale = fp4_scale(group_top(top));
    return fp4_codes(x, scale);
  }
}

// A lane takes eight features of a key and its value, four lanes a group, so a head's row is read and written in one run.  A workgroup takes `rows` new rows of one sequence.
template <typename T, bool WIDE>
__global__ __launch_bounds__(256) void cache_append_fp4_kernel(AppendFp4Args a, int rows, int blocks_per_seq) {
  const unsigned umb = blockIdx.x / blocks_per_seq;
  const long mb = umb, m = umb / a.B;
  const int i0 = (int)(blockIdx.x % blocks_per_seq) * rows, b = (int)(umb % a.B);
  const int cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n, L = clamp_len(a.len[mb], a.C);
  const int end = min(min(i0 + rows, cnt), a.C - L);       // entries past the capacity are not written
  const int G = fp4_groups(a.d), S = fp4_scale_bytes(a.d), units = 4 * G, per_row = a.kv * units;
  for (int i = i0 + (int)threadIdx.x / per_row, c = (int)threadIdx.x % per_row; i < end;) {      // the lanes of a quad stay together: per_row is a multiple of 4
    const int row = a.index ? a.index[mb * a.n + i] : i;
    if (row >= 0 && row < a.T) {
      const int g = c / units, u = c % units;
      const long from = m * a.stride_m + ((long)b * a.T + row) * a.stride_row + (long)g * a.d, slot = (mb * a.kv + g) * a.C + L + i;
      uint32_t ks, vs;
      const uint32_t kc = fp4_quantise8<T, WIDE>((const T*)a.K + from, 8 * u, a.d, ks), vc = fp4_quantise8<T, WIDE>((const T*)a.V + from, 8 * u, a.d, vs);
      ((uint32_t*)a.Kc)[slot * units + u] = kc;
      ((uint32_t*)a.Vc)[slot * units + u] = vc;
      if (u % 4 == 0) {
        a.Ks[slot * S + u / 4] = (uint8_t)ks;
        a.Vs[slot * S + u / 4] = (uint8_t)vs;
      }
      if (u == 0) {
        if (S > G) a.Ks[slot * S + G] = 0, a.Vs[slot * S + G] = 0;
        if (a.pos) a.pos[slot] = (a.start ? a.start[mb] : L) + i;
        if (a.weight) a.weight[slot] = 0.f;
      }
    }
    c += 256;
    i += c / per_row;
    c %= per_row;
  }
}

struct ReadFp4Args {
  const uint8_t* Kc; const uint8_t* Ks; const uint8_t* Vc; const uint8_t* Vs; const int* first; const int* count;
  void* K; void* V;
  int M, B, n, C, kv, d;
};

// A lane gives eight features of an entry, of its key and of its value; UNROLL of them are on their way at a time.  A workgroup takes `rows` entries of one head.
template <typename T, bool WIDE, int UNROLL>
__global__ __launch_bounds__(256) void cache_read_fp4_kernel(ReadFp4Args a, int rows, int blocks_per_head) {
  const unsigned uhead = blockIdx.x / blocks_per_head;
  const long head = uhead, mb = uhead / a.kv;
  const int i0 = (int)(blockIdx.x % blocks_per_head) * rows, stop = min(rows, a.n - i0);
  const int first = a.first ? a.first[mb] : 0, cnt = a.count ? clamp_len(a.count[mb], a.n) : a.n;
  const int S = fp4_scale_bytes(a.d), words = fp4_code_bytes(a.d) / 4;
  const unsigned units = (unsigned)(a.d + 7) / 8, total = (unsigned)stop * units;
  for (unsigned k0 = threadIdx.x; k0 < total; k0 += 256 * UNROLL) {
    uint32_t code[2][UNROLL], scale[2][UNROLL];
#pragma unroll
    for (int x = 0; x < UNROLL; ++x) {
      const unsigned k = min(k0 + 256u * x, total - 1), i = k / units, u = k - i * units;
      const long long slot = (long long)first + i0 + i;
      const bool there = i0 + (int)i < cnt && slot >= 0 && slot < a.C;
      const long at = head * a.C + (there ? slot : 0);     // an entry that is not there: some entry's bytes, not used
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        code[t][x] = scale[t][x] = 0;
        if (t == 0 || a.V) {
          const uint32_t c = ((const uint32_t*)(t ? a.Vc : a.Kc))[at * words + u], s = (t ? a.Vs : a.Ks)[at * S + u / 4];
          code[t][x] = there ? c : 0u;
          scale[t][x] = there ? s : 127u;
        }
      }
    }
#pragma unroll
    for (int x = 0; x < UNROLL; ++x) {
      const unsigned k = k0 + 256u * x, i = k / units, u = k - i * units;
      if (k >= total) break;
      const long at = (head * a.n + i0 + i) * a.d + 8 * u;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        if (t == 1 && !a.V) break;
        T* out = (T*)(t ? a.V : a.K) + at;
        const float s = fp4_scale_value(scale[t][x]);
        if constexpr (sizeof(T) == 2 && WIDE) {
          *reinterpret_cast<uint4*>(out) = fp4_values_bf16(code[t][x], s);
        } else {
          float v[8];
          fp4_values_f32(code[t][x], s, v);
          if constexpr (WIDE) {
#pragma unroll
            for (int h = 0; h < 8; h += 4)
              if ((int)(8 * u) + h < a.d) *reinterpret_cast<float4*>(out + h) = make_float4(v[h], v[h + 1], v[h + 2], v[h + 3]);
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e)
              if ((int)(8 * u) + e < a.d) store_f32(out + e, v[e]);
          }
        }
      }
    }
  }
}

}  // namespace nf
